// Learned relative position bias by buckets, and the gradient of its rows.
//
//   bias[n,h,i,j] = rows[bucket(j - (start_n + i)), h]          grad_rows[b,h] = sum of grad[n,h,i,j] over bucket b
//
// A bucket is an interval of distances and a distance is one diagonal j - i of a head's matrix, so a matrix holds Q + K - 1
// different values and its gradient is wanted by diagonals first.  Both kernels work on diagonals: the forward reads a
// window of the diagonals' values per row, the backward keeps a diagonal's sum in a register while it walks down it.
#include "robe_internal.h"
#include "robe_rowops.cuh"

namespace robe {

namespace {

// ---- forward

constexpr int kBiasThreads = 256;
constexpr int kBiasRows = 64;     // rows of a tile
constexpr int kBiasPieces = 128;  // 16-byte pieces of a row of a tile

struct BiasArgs {
    BiasBuckets bk;
    const float* rows;
    int64_t rows_ld;
    uint32_t heads;
    int64_t q_len, k_len, q_start;
    const int64_t* q_starts;
    int causal;
    void* out;
    int64_t out_ld;
    uint32_t q_tiles, k_tiles;
    int lanes_log2;  // lanes that share a row
};

// Bucket of a distance r = key position - query position.
__device__ __forceinline__ uint32_t bucket_of(int64_t r, const int32_t* edges, uint32_t side, int two_sided) {
    const int64_t n = two_sided ? (r < 0 ? -r : r) : (r < 0 ? -r : 0);
    uint32_t lo = 0;
    if (n >= edges[side - 1]) {
        lo = side - 1;
    } else {  // the last edge that n reaches
        uint32_t hi = side - 1;
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (n >= edges[mid]) lo = mid;
            else hi = mid;
        }
    }
    return lo + (two_sided && r > 0 ? side : 0);
}

__device__ __forceinline__ int64_t start_of(int64_t q_start, const int64_t* q_starts, uint32_t n) {
    int64_t s = q_starts != nullptr ? __ldca((const long long*)q_starts + n) : q_start;
    // distances are below 2^32 within a call: a start further out changes nothing
    const int64_t far = 1ll << 34;
    return s > far ? far : s < -far ? -far : s;
}

// A tile of a head's matrix: the values of its diagonals go to shared memory once, then every 16-byte piece of every row is
// a window of them.  The window of a row starts anywhere, so the values are kept kPiece times, copy s from diagonal s on:
// whatever the start, one copy has the window on a 16-byte boundary.
template <class T>
__global__ void __launch_bounds__(kBiasThreads) bias_forward_kernel(BiasArgs a) {
    constexpr int V = kPiece<T>;
    constexpr int U = kBiasPieces + kBiasRows / V + 2;  // pieces of a copy
    __shared__ __align__(16) T lut[V][U * V];
    __shared__ int32_t edges[kBiasMaxSide];
    follow();
    for (uint32_t k = threadIdx.x; k < a.bk.side; k += kBiasThreads) edges[k] = a.bk.edges[k];
    uint32_t b = blockIdx.x;
    const uint32_t kt = b % a.k_tiles;
    b /= a.k_tiles;
    const uint32_t qt = b % a.q_tiles;
    b /= a.q_tiles;
    const uint32_t h = b % a.heads, n = b / a.heads;
    const int64_t i0 = (int64_t)qt * kBiasRows;
    const int64_t g0 = (int64_t)kt * kBiasPieces;
    const int rows = a.q_len - i0 < kBiasRows ? (int)(a.q_len - i0) : kBiasRows;
    // the first diagonal a window can start on: the last row, a piece that begins up to V - 1 columns early
    const int64_t t0 = g0 * V - (V - 1) - (i0 + rows - 1);
    const int64_t start = start_of(a.q_start, a.q_starts, n);
    const int count = kBiasPieces * V + rows - 1 + (V - 1);
    __syncthreads();
    for (int t = threadIdx.x; t < count; t += kBiasThreads) {
        const int64_t r = t0 + t - start;
        float v = -INFINITY;
        if (!a.causal || r <= 0) v = __ldca(a.rows + bucket_of(r, edges, a.bk.side, a.bk.two_sided) * a.rows_ld + h);
        const T e = narrow<T>(v);
#pragma unroll
        for (int s = 0; s < V; ++s)
            if (t >= s && ROBE_CHK(t - s < U * V, ROBE_DBG_SHARED)) lut[s][t - s] = e;
    }
    __syncthreads();
    const int lane = threadIdx.x & ((1 << a.lanes_log2) - 1);
    T* matrix = (T*)a.out + ((int64_t)n * a.heads + h) * a.q_len * a.out_ld;
    for (int i = threadIdx.x >> a.lanes_log2; i < rows; i += kBiasThreads >> a.lanes_log2) {
        T* row = matrix + (i0 + i) * a.out_ld;
        const int lead = (int)(((uintptr_t)row / sizeof(T)) & (V - 1));  // row begins inside a 16-byte piece
        const int x = (V - 1) - lead + (rows - 1 - i);                   // diagonal of the tile's first piece, from t0
        const T* window = lut[x & (V - 1)] + (x & ~(V - 1));
        for (int g = lane; g < kBiasPieces; g += 1 << a.lanes_log2) {
            const int64_t j = (g0 + g) * V - lead;
            if (j >= a.k_len) break;
            if (!ROBE_CHK((x & ~(V - 1)) + g * V + V <= U * V, ROBE_DBG_SHARED)) break;
            const Pack<T, V> e = *(const Pack<T, V>*)(window + g * V);
            if (j >= 0 && j + V <= a.k_len) {
                store_pack<true, T, V>(row + j, e);
            } else {
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (j + k >= 0 && j + k < a.k_len) row[j + k] = e.v[k];
            }
        }
    }
}

// ---- backward

constexpr int kGradBlocks = 8;       // blocks of kPiece rows that one CTA walks through
constexpr int kGradMaxThreads = 512;

struct BiasGradArgs {
    BiasBuckets bk;
    const void* grad;
    int64_t grad_ld;
    uint32_t heads, batch;
    int64_t q_len, k_len, q_start;
    const int64_t* q_starts;
    int causal;
    double* partial;  // [heads][buckets][parts], parts = batch * segments * chunks
    uint32_t segments, chunks, lanes;
    float* grad_rows;
    int64_t grad_rows_ld;
};

// Distances of bucket b: [lo, hi).
__device__ __forceinline__ void bucket_interval(uint32_t b, const BiasBuckets& bk, const int32_t* edges, int causal, int64_t& lo,
                                                int64_t& hi) {
    const int64_t far = 1ll << 40;
    const uint32_t k = b < bk.side ? b : b - bk.side;
    const int64_t e0 = edges[k], e1 = k + 1 < bk.side ? edges[k + 1] : far;
    if (b < bk.side) {
        lo = 1 - e1;
        hi = 1 - e0;
        if (k == 0 && !bk.two_sided) hi = far;
    } else {
        lo = e0 < 1 ? 1 : e0;
        hi = e1;
    }
    if (causal && hi > 1) hi = 1;
}

// Sums of a band of diagonals over a segment of rows.  A lane takes V x V squares (V = kPiece: one 16-byte load per row of
// a square) and moves from each to the next one down and to the right: the 2 V - 1 diagonals that cross its squares are the
// same all the way, their sums stay in registers, and every load is of a whole piece.
template <class T, bool ALIGNED>
__global__ void __launch_bounds__(kGradMaxThreads) bias_grad_kernel(BiasGradArgs a) {
    constexpr int V = kPiece<T>;
    extern __shared__ float sums[];  // upper[lanes * V], lower[lanes * V]
    __shared__ int32_t edges[kBiasMaxSide];
    follow();
    for (uint32_t k = threadIdx.x; k < a.bk.side; k += blockDim.x) edges[k] = a.bk.edges[k];
    uint32_t b = blockIdx.x;
    const uint32_t chunk = b % a.chunks;
    b /= a.chunks;
    const uint32_t seg = b % a.segments;
    b /= a.segments;
    const uint32_t h = b % a.heads, n = b / a.heads;
    const uint32_t part = (n * a.segments + seg) * a.chunks + chunk;
    const uint32_t parts = a.batch * a.segments * a.chunks;
    const int64_t start = start_of(a.q_start, a.q_starts, n);
    const int64_t row_blocks = (a.q_len + V - 1) / V, col_groups = (a.k_len + V - 1) / V;
    const int64_t rb0 = (int64_t)seg * kGradBlocks;
    const int64_t rb1 = rb0 + kGradBlocks < row_blocks ? rb0 + kGradBlocks : row_blocks;
    const int64_t first = (int64_t)chunk * a.lanes - (rb1 - 1);  // column group minus row block of lane 0
    const int64_t delta = first + threadIdx.x;
    float acc[2 * V - 1];
#pragma unroll
    for (int k = 0; k < 2 * V - 1; ++k) acc[k] = 0.0f;
    // the lane's lowest diagonal is V delta - (V - 1): beyond it nothing is seen under a causal mask
    if (!a.causal || V * delta - (V - 1) - start <= 0) {
        const int64_t lo = rb0 > -delta ? rb0 : -delta;
        const int64_t hi = rb1 < col_groups - delta ? rb1 : col_groups - delta;
        const T* matrix = (const T*)a.grad + ((int64_t)n * a.heads + h) * a.q_len * a.grad_ld;
        for (int64_t rb = lo; rb < hi; ++rb) {
            const int64_t i = rb * V, j = (rb + delta) * V;
            const T* p = matrix + i * a.grad_ld + j;
            if (ALIGNED && i + V <= a.q_len && j + V <= a.k_len) {
                Pack<T, V> e[V];
#pragma unroll
                for (int s = 0; s < V; ++s) e[s] = load_pack<true, T, V>(p + s * a.grad_ld);
#pragma unroll
                for (int s = 0; s < V; ++s)
#pragma unroll
                    for (int c = 0; c < V; ++c) acc[c - s + V - 1] += widen(e[s].v[c]);
            } else {
#pragma unroll
                for (int s = 0; s < V; ++s)
#pragma unroll
                    for (int c = 0; c < V; ++c)
                        if (i + s < a.q_len && j + c < a.k_len) acc[c - s + V - 1] += widen(p[s * a.grad_ld + c]);
            }
        }
    }
    // diagonal V delta + k: the lane's own upper half and the next lane's lower one
    float* upper = sums;
    float* lower = sums + (size_t)a.lanes * V;
    const int at = threadIdx.x * V;
#pragma unroll
    for (int k = 0; k < V; ++k) upper[at + k] = acc[V - 1 + k];
    lower[at] = 0.0f;
#pragma unroll
    for (int k = 1; k < V; ++k) lower[at + k] = acc[k - 1];  // diagonals V (delta - 1) + k
    __syncthreads();
    // lower[V l + k] belongs to upper[V (l - 1) + k]: in terms of diagonals from V (first - 1) on, upper starts at V
    const int64_t base = V * (first - 1);
    const int span = (int)a.lanes * V;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    for (uint32_t q = warp; q < a.bk.buckets; q += warps) {
        int64_t lo, hi;
        bucket_interval(q, a.bk, edges, a.causal, lo, hi);
        lo = lo + start - base;
        hi = hi + start - base;
        if (lo < 0) lo = 0;
        if (hi > span + V) hi = span + V;
        double sum = 0.0;
        for (int64_t d = lo + lane; d < hi; d += 32) {
            float v = 0.0f;
            if (d < span) v = lower[d];
            if (d >= V) v += upper[d - V];
            sum += (double)v;
        }
#pragma unroll
        for (int s = 16; s > 0; s >>= 1) sum += __shfl_down_sync(0xFFFFFFFFu, sum, s);
        if (lane == 0) a.partial[((uint64_t)h * a.bk.buckets + q) * parts + part] = sum;
    }
}

// One warp per (head, bucket): the parts' sums, in a fixed order.
__global__ void __launch_bounds__(32) bias_grad_join_kernel(BiasGradArgs a) {
    follow();
    const uint32_t h = blockIdx.x / a.bk.buckets, q = blockIdx.x % a.bk.buckets;
    const uint64_t parts = (uint64_t)a.batch * a.segments * a.chunks;
    const double* p = a.partial + (uint64_t)blockIdx.x * parts;
    double sum = 0.0;
    for (uint64_t k = threadIdx.x; k < parts; k += 32) sum += __ldcs(p + k);
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) sum += __shfl_down_sync(0xFFFFFFFFu, sum, s);
    if (threadIdx.x == 0) a.grad_rows[q * a.grad_rows_ld + h] = (float)sum;
}

struct GradShape {
    uint32_t segments, chunks, lanes;
    uint64_t parts;
};
// The split of a call over CTAs; from the sizes and the element type alone, so that the workspace can be sized by it.
GradShape grad_shape(int64_t batch, int64_t q_len, int64_t k_len, int V) {
    GradShape g = {0, 0, 0, 0};
    if (batch == 0 || q_len == 0 || k_len == 0) return g;
    const int64_t row_blocks = (q_len + V - 1) / V, col_groups = (k_len + V - 1) / V;
    const int64_t deltas = col_groups + (row_blocks < kGradBlocks ? row_blocks : kGradBlocks) - 1;
    g.segments = (uint32_t)((row_blocks + kGradBlocks - 1) / kGradBlocks);
    g.chunks = (uint32_t)((deltas + kGradMaxThreads - 1) / kGradMaxThreads);
    const int64_t per = (deltas + g.chunks - 1) / g.chunks;
    g.lanes = (uint32_t)((per + 31) / 32 * 32);
    g.parts = (uint64_t)batch * g.segments * g.chunks;
    return g;
}

}  // namespace

cudaError_t launch_bias_forward(const BiasProblem& pb, void* out, int64_t out_ld, int dtype, cudaStream_t st) {
    BiasArgs a;
    a.bk = pb.bk;
    a.rows = pb.rows;
    a.rows_ld = pb.rows_ld;
    a.heads = pb.heads;
    a.q_len = pb.q_len;
    a.k_len = pb.k_len;
    a.q_start = pb.q_start;
    a.q_starts = pb.q_starts;
    a.causal = pb.causal;
    a.out = out;
    a.out_ld = out_ld;
    const int V = dtype == 0 ? kPiece<float> : kPiece<__nv_bfloat16>;
    const int64_t pieces = (pb.k_len + V - 1 + V - 1) / V;  // (one more where a row begins inside a piece)
    a.k_tiles = (uint32_t)((pieces + kBiasPieces - 1) / kBiasPieces);
    a.q_tiles = (uint32_t)((pb.q_len + kBiasRows - 1) / kBiasRows);
    a.lanes_log2 = 0;
    while (a.lanes_log2 < 5 && (1 << a.lanes_log2) < pieces) ++a.lanes_log2;
    const unsigned __int128 grid = (unsigned __int128)pb.batch * pb.heads * a.q_tiles * a.k_tiles;
    if (grid >= (1u << 31)) return cudaErrorInvalidValue;
    if (dtype == 0) launch_next(bias_forward_kernel<float>, (unsigned)grid, kBiasThreads, 0, st, a);
    else launch_next(bias_forward_kernel<__nv_bfloat16>, (unsigned)grid, kBiasThreads, 0, st, a);
    return cudaGetLastError();
}

size_t bias_grad_workspace_bytes(uint32_t buckets, uint32_t heads, int64_t batch, int64_t q_len, int64_t k_len) {
    // for either element type: fp32 rows are cut into more segments, bf16 into no more chunks
    uint64_t parts = 0;
    for (int V : {kPiece<float>, kPiece<__nv_bfloat16>}) {
        const GradShape g = grad_shape(batch, q_len, k_len, V);
        if (g.parts > parts) parts = g.parts;
    }
    const unsigned __int128 bytes = (unsigned __int128)parts * buckets * heads * sizeof(double);
    if (bytes >= ((unsigned __int128)1 << 62)) return (size_t)1 << 62;
    return ((size_t)bytes + 255) / 256 * 256;
}

cudaError_t launch_bias_backward(const BiasProblem& pb, const void* grad, int64_t grad_ld, int dtype, float* grad_rows,
                                 int64_t grad_rows_ld, void* workspace, cudaStream_t st) {
    const int V = dtype == 0 ? kPiece<float> : kPiece<__nv_bfloat16>;
    const GradShape g = grad_shape(pb.batch, pb.q_len, pb.k_len, V);
    BiasGradArgs a;
    a.bk = pb.bk;
    a.grad = grad;
    a.grad_ld = grad_ld;
    a.heads = pb.heads;
    a.batch = (uint32_t)pb.batch;
    a.q_len = pb.q_len;
    a.k_len = pb.k_len;
    a.q_start = pb.q_start;
    a.q_starts = pb.q_starts;
    a.causal = pb.causal;
    a.partial = (double*)workspace;
    a.segments = g.segments;
    a.chunks = g.chunks;
    a.lanes = g.lanes;
    a.grad_rows = grad_rows;
    a.grad_rows_ld = grad_rows_ld;
    const unsigned __int128 grid = (unsigned __int128)g.parts * pb.heads;
    if (grid >= (1u << 31)) return cudaErrorInvalidValue;
    const int64_t size = dtype == 0 ? 4 : 2;
    const bool aligned = ((uintptr_t)grad & 15u) == 0 && grad_ld * size % 16 == 0;
    const size_t smem = (size_t)g.lanes * V * 2 * sizeof(float);
    if (g.parts > 0) {
        if (dtype == 0)
            launch_next(aligned ? bias_grad_kernel<float, true> : bias_grad_kernel<float, false>, (unsigned)grid, g.lanes, smem, st, a);
        else
            launch_next(aligned ? bias_grad_kernel<__nv_bfloat16, true> : bias_grad_kernel<__nv_bfloat16, false>, (unsigned)grid,
                        g.lanes, smem, st, a);
    }
    launch_next(bias_grad_join_kernel, (unsigned)(pb.heads * pb.bk.buckets), 32, 0, st, a);
    return cudaGetLastError();
}

}  // namespace robe
