// Learned relative position bias by buckets, and the gradient of its rows.
//
//   bias[n,h,i,j] = rows[bucket(j - (start_n + i)), h]          grad_rows[b,h] = sum of grad[n,h,i,j] over bucket b
//
// A bucket is an interval of distances and a distance is one diagonal j - i of a head's matrix, so a matrix holds Q + K - 1
// different values and its gradient is wanted by diagonals first.  Both kernels work on diagonals: the forward reads a
// window of the diagonals' values per row, the backward keeps a diagonal's sum in a register while it walks down it.
#include <type_traits>

#include "robe_internal.h"
#include "robe_rowops.cuh"

namespace robe {

namespace {

// ---- forward

constexpr int kBiasThreads = 256;
constexpr int kBiasRows = 64;     // rows of a tile
constexpr int kBiasPieces = 128;  // 16-byte pieces of a row of a tile
constexpr int kBiasFew = 4;       // up to so many queries, every piece finds its buckets itself

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
    int lanes_log2;  // lanes that share a row of a tile
    uint32_t top;    // largest power of two below side
    int32_t low, high;  // distances up to and from which there is one number each
};

__device__ __forceinline__ int64_t start_of(int64_t q_start, const int64_t* q_starts, uint32_t n) {
    int64_t s = q_starts != nullptr ? __ldca((const long long*)q_starts + n) : q_start;
    // distances are below 2^32 within a call: a start further out changes nothing
    const int64_t far = 1ll << 34;
    return s > far ? far : s < -far ? -far : s;
}

// A distance in 32 bits: those beyond 2^30 are past the last border, and stay so when they are cut.  (Calls are of less than
// 2^31 queries and keys; what is added to it later is below 2^20.)
__device__ __forceinline__ int32_t near_distance(int64_t r) {
    const int64_t far = (1ll << 31) - (1 << 21);
    return (int32_t)(r > far ? far : r < -far ? -far : r);
}

// The numbers of one head, by bucket, in shared memory: what a distance r = key position - query position is worth.  Up to
// `low` and from `high` on it is one number each.
struct HeadValues {
    float value[2 * kBiasMaxSide];
    int32_t edges[kBiasMaxSide];
    __device__ __forceinline__ void load(const BiasArgs& a, uint32_t h) {
        for (uint32_t k = threadIdx.x; k < a.bk.buckets; k += blockDim.x) value[k] = __ldca(a.rows + k * a.rows_ld + h);
        for (uint32_t k = threadIdx.x; k < kBiasMaxSide; k += blockDim.x) edges[k] = k < a.bk.side ? a.bk.edges[k] : 0x7FFFFFFF;
        __syncthreads();
    }
    __device__ __forceinline__ float at_low(const BiasArgs& a) const { return value[a.bk.side - 1]; }
    __device__ __forceinline__ float at_high(const BiasArgs& a) const {
        return a.causal ? -INFINITY : value[a.bk.two_sided ? a.bk.buckets - 1 : 0];
    }
    __device__ __forceinline__ float at(int32_t r, const BiasArgs& a) const {
        if (r <= a.low) return at_low(a);
        if (r >= a.high) return at_high(a);
        const int32_t n = r < 0 ? -r : r;
        uint32_t k = 0;  // the last border that n reaches, by halves
        for (uint32_t half = a.top; half > 0; half >>= 1)
            if (n >= edges[k + half]) k += half;
        return value[r > 0 ? k + a.bk.side : k];  // (r > 0 is below `high` only where buckets are two-sided)
    }
};

// Few queries: bound by the latency of a CTA's first loads and by issue, not by the 16.8 MB of 64 x 16 rows of 8191 bf16 (9.1 us;
// 33 with a tile's diagonals per row).  A CTA has kBiasThreads kBiasRowPieces pieces of one row.  Most are of one value, beyond the last border.
constexpr int kBiasRowPieces = 4;
template <class T>
__global__ void __launch_bounds__(kBiasThreads) bias_few_kernel(BiasArgs a) {
    constexpr int V = kPiece<T>;
    __shared__ HeadValues values;
    follow();
    const uint32_t line = a.k_tiles == 1 ? blockIdx.x : blockIdx.x / a.k_tiles;  // (n, h, i)
    const uint32_t kt = blockIdx.x - line * a.k_tiles;
    const uint32_t nh = a.q_len == 1 ? line : line / (uint32_t)a.q_len;
    const uint32_t i = line - nh * (uint32_t)a.q_len;
    const uint32_t n = nh / a.heads, h = nh - n * a.heads;
    const int64_t start = start_of(a.q_start, a.q_starts, n);
    values.load(a, h);
    T* row = (T*)a.out + (int64_t)line * a.out_ld;
    const int lead = (int)(((uintptr_t)row / sizeof(T)) & (V - 1));  // row begins inside a 16-byte piece
    const int64_t j0 = (int64_t)kt * (kBiasRowPieces * kBiasThreads * V) - lead;
    row += j0;
    const int32_t r0 = near_distance(j0 - start - i);
    const int begin = kt == 0 ? lead : 0;
    const int end = a.k_len - j0 < kBiasRowPieces * kBiasThreads * V ? (int)(a.k_len - j0) : kBiasRowPieces * kBiasThreads * V;
#pragma unroll
    for (int q = 0; q < kBiasRowPieces; ++q) {
        const int j = (q * kBiasThreads + threadIdx.x) * V;
        if (j >= end) break;
        const int32_t r = r0 + j;
        Pack<T, V> e;
        if (r + V - 1 <= a.low || r >= a.high) {
            const T same = narrow<T>(r >= a.high ? values.at_high(a) : values.at_low(a));
#pragma unroll
            for (int k = 0; k < V; ++k) e.v[k] = same;
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k) e.v[k] = narrow<T>(values.at(r + k, a));
        }
        if (j >= begin && j + V <= end) {
            if (!ROBE_CHK(j0 + j >= 0 && j0 + j + V <= a.k_len, ROBE_DBG_ROW_POS)) break;
            store_pack<true, T, V>(row + j, e);
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (j + k >= begin && j + k < end) row[j + k] = e.v[k];
        }
    }
}

// A tile of a head's matrix: the values of its diagonals go to shared memory once, then every 16-byte piece of every row is
// a window of them.  The window of a row starts anywhere, so the values are kept kPiece times, copy s from diagonal s on:
// whatever the start, one copy has the window on a 16-byte boundary.  A tile beyond the borders needs none of that.  16 matrices
// of 2048 x 2048 bf16 (134 MB written) 24.1 us, 5.6 TB/s; with the borders searched in 64 bits 30.
template <class T>
__global__ void __launch_bounds__(kBiasThreads, 8) bias_forward_kernel(BiasArgs a) {
    constexpr int V = kPiece<T>;
    constexpr int U = kBiasPieces + kBiasRows / V + 3;  // pieces of a copy, one in front that no window reads
    __shared__ __align__(16) T lut[V][U * V];
    __shared__ HeadValues values;
    follow();
    uint32_t b = blockIdx.x;
    const uint32_t kt = b % a.k_tiles;
    b /= a.k_tiles;
    const uint32_t qt = b % a.q_tiles;
    b /= a.q_tiles;
    const uint32_t h = b % a.heads, n = b / a.heads;
    const int64_t i0 = (int64_t)qt * kBiasRows;
    const int64_t j0 = (int64_t)kt * kBiasPieces * V;
    const int rows = a.q_len - i0 < kBiasRows ? (int)(a.q_len - i0) : kBiasRows;
    // the first diagonal a window can start on: the last row, a piece that begins up to V - 1 columns early
    const int64_t t0 = j0 - (V - 1) - (i0 + rows - 1);
    const int64_t start = start_of(a.q_start, a.q_starts, n);
    const int columns = a.k_len - j0 < kBiasPieces * V ? (int)(a.k_len - j0) : kBiasPieces * V;
    const int count = columns + rows - 1 + 2 * (V - 1);
    values.load(a, h);
    const int32_t r0 = near_distance(t0 - start);
    const bool high = r0 >= a.high, mixed = !high && r0 + count - 1 > a.low;
    if (mixed) {
        for (int t = threadIdx.x; t < count; t += kBiasThreads) {
            const T e = narrow<T>(values.at(r0 + t, a));
#pragma unroll
            for (int s = 0; s < V; ++s)
                if (ROBE_CHK(t + V - s < U * V, ROBE_DBG_SHARED)) lut[s][t + V - s] = e;
        }
        __syncthreads();
    }
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    T* tile = (T*)a.out + (((int64_t)n * a.heads + h) * a.q_len + i0) * a.out_ld + j0;
    Pack<T, V> e;
#pragma unroll
    for (int k = 0; k < V; ++k) e.v[k] = narrow<T>(high ? values.at_high(a) : values.at_low(a));
    for (int i = threadIdx.x >> a.lanes_log2; i < rows; i += kBiasThreads >> a.lanes_log2) {
        T* row = tile + i * a.out_ld;
        const int lead = (int)(((uintptr_t)row / sizeof(T)) & (V - 1));  // row begins inside a 16-byte piece
        const int x = (V - 1) - lead + (rows - 1 - i);                   // diagonal of the tile's first piece, from t0
        const T* window = lut[x & (V - 1)] + (x & ~(V - 1)) + V;
        row -= lead;
        // (in front of a tile's first whole piece is the last of the tile before it, which stores it)
        int from = lane, to = (columns + lead) / V;
        if (lead != 0) {
            if (lane == 0) {
                const Pack<T, V> w = *(const Pack<T, V>*)window;
#pragma unroll
                for (int k = 1; k < V; ++k)
                    if (k >= lead && k < columns + lead) row[k] = mixed ? w.v[k] : e.v[k];
                from += lanes;
            }
        }
        for (int g = from; g < to; g += lanes) {
            if (!ROBE_CHK(V + (x & ~(V - 1)) + g * V + V <= U * V, ROBE_DBG_SHARED)) break;
            if (mixed) e = *(const Pack<T, V>*)(window + g * V);
            if (!ROBE_CHK(g * V >= lead && j0 + g * V - lead + V <= a.k_len, ROBE_DBG_ROW_POS)) break;
            store_pack<true, T, V>(row + g * V, e);
        }
        if (lane == lanes - 1 && to * V < columns + lead && (to > 0 || lead == 0)) {  // the last elements, of no whole piece
            const Pack<T, V> w = *(const Pack<T, V>*)(window + to * V);
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (to * V + k < columns + lead) row[to * V + k] = mixed ? w.v[k] : e.v[k];
        }
    }
}

// ---- backward

constexpr int kGradBlocks = 8;  // blocks of kPiece rows that one CTA walks through, at least
constexpr int kGradMostBlocks = 32;
constexpr int kGradMaxThreads = 320;
constexpr int kGradStages = 2;

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
    int blocks;
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

// kPiece elements that begin `at` bytes into the 16 bytes at p (and go on in the next 16).
template <class T, bool ALIGNED>
__device__ __forceinline__ void take_piece(float (&v)[kPiece<T>], const uint4* p, uint32_t at) {
    uint32_t w[8];
    *(uint4*)w = p[0];
    if (!ALIGNED) {
        *(uint4*)(w + 4) = p[1];
        if (at & 8)
#pragma unroll
            for (int k = 0; k < 6; ++k) w[k] = w[k + 2];
        if (at & 4)
#pragma unroll
            for (int k = 0; k < 5; ++k) w[k] = w[k + 1];
        if (sizeof(T) == 2)
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], (at & 2) * 8);
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = widen_low(w[k]);
            v[2 * k + 1] = widen_high(w[k]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(w[k]);
    }
}

// Sums of a band of diagonals over a segment of rows.  A lane takes V x V squares (V = kPiece: a 16-byte piece per row of a
// square) and moves from each to the next one down and to the right: the 2 V - 1 diagonals that cross its squares are the
// same all the way, and their sums stay in registers.  A warp's squares, side by side, are copied to shared memory one
// ahead, in the aligned pieces that they lie in; rows that begin inside a piece are shifted into place when they are read.  16 x 16 matrices of 2048 x 2048
// bf16 (2.1 GB read): 341 us, 6.3 TB/s, which is what a copy reaches; loads into registers 437 (too few under way), three
// squares ahead 348 (fewer CTAs).  4 x 12 of 777 x 1001, masked: 23 us, of which the walk's 8 steps and the sums by buckets
// are latency.
template <class T, bool ALIGNED>
__global__ void __launch_bounds__(kGradMaxThreads, 3) bias_grad_kernel(BiasGradArgs a) {
    constexpr int V = kPiece<T>;
    constexpr int kRow = ALIGNED ? 32 : 33;  // pieces of a row of a warp's squares
    extern __shared__ __align__(16) uint4 pieces[];  // [warp][stage][V][kRow]; afterwards the sums
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
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const int64_t start = start_of(a.q_start, a.q_starts, n);
    const int row_blocks = (int)((a.q_len + V - 1) / V), col_groups = (int)((a.k_len + V - 1) / V);
    const int rb0 = (int)seg * a.blocks;
    const int rb1 = rb0 + a.blocks < row_blocks ? rb0 + a.blocks : row_blocks;
    const int first = (int)(chunk * a.lanes) - (rb1 - 1);  // column group minus row block of lane 0
    const int delta0 = first + warp * 32, delta = delta0 + lane;
    float acc[2 * V - 1], sum[2 * V - 1];
#pragma unroll
    for (int k = 0; k < 2 * V - 1; ++k) acc[k] = sum[k] = 0.0f;
    if (threadIdx.x < a.lanes) {  // (warps beyond only help with the buckets)
        // a lane's lowest diagonal is V delta - (V - 1): beyond it nothing is seen under a causal mask.  What a lane copies
        // the lane before it may read.
        const bool seen = !a.causal || (int64_t)V * delta - (V - 1) - start <= 0;
        const bool copied = !a.causal || (int64_t)V * (delta - 1) - (V - 1) - start <= 0;
        int lo = rb0 > -(delta0 + 31) ? rb0 : -(delta0 + 31);  // squares of the warp's lanes
        int hi = rb1 < col_groups - delta0 ? rb1 : col_groups - delta0;
        if (a.causal && (int64_t)V * delta0 - (V - 1) - start > 0) hi = lo;
        const char* begin = (const char*)a.grad;
        const char* end = begin + (((int64_t)a.batch * a.heads * a.q_len - 1) * a.grad_ld + a.k_len) * (int64_t)sizeof(T);
        const char* matrix = begin + ((int64_t)n * a.heads + h) * a.q_len * a.grad_ld * (int64_t)sizeof(T);
        const int64_t step = a.grad_ld * (int64_t)sizeof(T);
        // [lo_in, hi_in): squares of whole rows whose pieces all lie within the tensor.  Not those of its first row, where pieces
        // are not the rows' own: one may begin before it.  (A square's rows are 16 bytes at least: the next squares' pieces
        // do not.)  And none whose last row's last piece ends behind it: rows of few bytes reach that far from other
        // squares than the last, and from other matrices.
        const int lo_in = !ALIGNED && n == 0 && h == 0 && lo < 1 ? 1 : lo;
        int hi_in = (int)(a.q_len / V);
        if (hi_in > hi) hi_in = hi;
        auto last_end = [&] {  // of the square above hi_in
            const uintptr_t last = (uintptr_t)(matrix + ((int64_t)hi_in * V - 1) * step + (ALIGNED ? col_groups - 1 : col_groups) * 16ll);
            return (last & ~(uintptr_t)15) + 16;
        };
        while (hi_in > lo_in && last_end() > (uintptr_t)end) --hi_in;
        uint4* mine = pieces + (size_t)warp * kGradStages * (V * kRow);
        auto copy = [&](uint4* to, const char* from, const char* row) {  // the aligned piece at `from`, if the row has part of it
            if (from + 16 <= row || from >= row + a.k_len * (int64_t)sizeof(T)) return;
            if (from >= begin && from + 16 <= end) {
                copy_async<16>(to, from);
            } else {  // at the ends of the tensor
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (from + k * sizeof(T) >= begin && from + k * sizeof(T) < end) ((T*)to)[k] = ((const T*)from)[k];
            }
        };
        auto fetch = [&](int rb, int stage) {
            uint4* to = mine + stage * (V * kRow) + lane;
            const char* row = matrix + (int64_t)rb * V * step;
            if (rb >= lo_in && rb < hi_in) {
                const int g = rb + delta;
                if (copied && g >= 0 && g < (ALIGNED ? col_groups : col_groups + 1)) {
                    const char* from = row + (int64_t)g * 16;
#pragma unroll
                    for (int s = 0; s < V; ++s) {
                        if (!ROBE_CHK(((uintptr_t)from & ~(uintptr_t)15) >= (uintptr_t)begin && ((uintptr_t)from & ~(uintptr_t)15) + 16 <= (uintptr_t)end, ROBE_DBG_GRAD_POS)) break;
                        copy_async<16>(to + s * kRow, ALIGNED ? from : (const char*)((uintptr_t)from & ~(uintptr_t)15));
                        from += step;
                    }
                }
                const int last = rb + delta0 + 32;
                if (!ALIGNED && lane < V && last > 0 && last <= col_groups) {  // the piece behind the last lane's, a row a lane
                    const char* from = row + lane * step + (int64_t)last * 16;
                    if (ROBE_CHK(((uintptr_t)from & ~(uintptr_t)15) >= (uintptr_t)begin && ((uintptr_t)from & ~(uintptr_t)15) + 16 <= (uintptr_t)end, ROBE_DBG_GRAD_POS))
                        copy_async<16>(to - lane + lane * kRow + 32, (const char*)((uintptr_t)from & ~(uintptr_t)15));
                }
            } else if (rb < hi && copied) {
                const int rows = a.q_len - (int64_t)rb * V < V ? (int)(a.q_len - (int64_t)rb * V) : V;
                const int64_t at = ((int64_t)rb + delta) * 16;
                for (int s = 0; s < rows; ++s) {
                    const char* from = ALIGNED ? row + at : (const char*)((uintptr_t)(row + at) & ~(uintptr_t)15);
                    copy(to + s * kRow, from, row);
                    if (!ALIGNED && lane == 31) copy(to + s * kRow + 1, from + 16, row);
                    row += step;
                }
            }
            copies_close();
        };
        for (int s = 0; s + 1 < kGradStages; ++s) fetch(lo + s, s);
        int stage = 0;
        for (int rb = lo; rb < hi; ++rb) {
            fetch(rb + kGradStages - 1, stage == 0 ? kGradStages - 1 : stage - 1);
            copies_wait(kGradStages - 1);
            __syncwarp();
            const uint4* from = mine + stage * (V * kRow) + lane;
            uint32_t at = (uint32_t)(uintptr_t)(matrix + (int64_t)rb * V * step);  // (columns are whole pieces)
            const int64_t columns = a.k_len - ((int64_t)rb + delta) * V;
            const bool here = seen && rb + delta >= 0 && columns > 0;
            if (rb >= lo_in && rb < hi_in && columns >= V) {
                if (here) {
#pragma unroll
                    for (int s = 0; s < V; ++s) {
                        float v[V];
                        take_piece<T, ALIGNED>(v, from + s * kRow, at);
                        at += (uint32_t)step;
#pragma unroll
                        for (int c = 0; c < V; ++c) acc[c - s + V - 1] += v[c];
                    }
                }
            } else if (here) {
                const int rows = a.q_len - (int64_t)rb * V < V ? (int)(a.q_len - (int64_t)rb * V) : V;
#pragma unroll
                for (int s = 0; s < V; ++s) {
                    if (s >= rows) break;
                    float v[V];
                    take_piece<T, ALIGNED>(v, from + s * kRow, at);
                    at += (uint32_t)step;
#pragma unroll
                    for (int c = 0; c < V; ++c) acc[c - s + V - 1] += c < columns ? v[c] : 0.0f;
                }
            }
            __syncwarp();
            stage = stage + 1 == kGradStages ? 0 : stage + 1;
            if ((rb - lo) % kGradBlocks == kGradBlocks - 1 || rb + 1 == hi)  // short sums, then sums of those
#pragma unroll
                for (int k = 0; k < 2 * V - 1; ++k) {
                    sum[k] += acc[k];
                    acc[k] = 0.0f;
                }
        }
        copies_wait(0);
    }
    __syncthreads();
    // diagonal V delta + k: the lane's own upper half and the next lane's lower one
    float* upper = (float*)pieces;
    float* lower = upper + a.lanes * V;
    if (threadIdx.x < a.lanes) {
        const int at = threadIdx.x * V;
        static_assert(2 * V * sizeof(float) <= kGradStages * V * sizeof(uint4), "the sums fit the pieces' memory");
#pragma unroll
        for (int k = 0; k < V; ++k) upper[at + k] = sum[V - 1 + k];
        lower[at] = 0.0f;
#pragma unroll
        for (int k = 1; k < V; ++k) lower[at + k] = sum[k - 1];  // diagonals V (delta - 1) + k
    }
    __syncthreads();
    // lower[V l + k] belongs to upper[V (l - 1) + k]: in terms of diagonals from V (first - 1) on, upper starts at V
    const int64_t base = (int64_t)V * (first - 1);
    const int span = (int)a.lanes * V;
    // a bucket is a run of diagonals: so many lanes a bucket that the longest runs are no longer than the many short ones
    auto join = [&](auto lanes_of_a_bucket) {
        constexpr uint32_t kShare = decltype(lanes_of_a_bucket)::value, kEach = 32 / kShare;
        for (uint32_t q0 = warp * kEach; q0 < a.bk.buckets; q0 += warps * kEach) {
            const uint32_t q = q0 + lane / kShare;
            int64_t from = 0, to = 0;
            if (q < a.bk.buckets) bucket_interval(q, a.bk, edges, a.causal, from, to);
            from = from + start - base;
            to = to + start - base;
            const int d0 = from < 0 ? 0 : from > span + V ? span + V : (int)from;
            const int d1 = q >= a.bk.buckets || to < 0 ? 0 : to > span + V ? span + V : (int)to;
            double total = 0.0;
            if (kShare < 32 || d0 < d1) {
                for (int d = d0 + lane % kShare; d < d1; d += kShare) {
                    float v = 0.0f;
                    if (d < span) v = lower[d];
                    if (d >= V) v += upper[d - V];
                    total += (double)v;
                }
#pragma unroll
                for (int s = kShare / 2; s > 0; s >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, s);
            }
            if (lane % kShare == 0 && q < a.bk.buckets && ROBE_CHK(part < parts && h < a.heads, ROBE_DBG_ROW_POS)) a.partial[((uint64_t)h * a.bk.buckets + q) * parts + part] = total;
        }
    };
    if (span > 1024) join(std::integral_constant<uint32_t, 32>());
    else join(std::integral_constant<uint32_t, 8>());
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
    int blocks;  // of kPiece rows in a segment
    uint64_t parts;
};
// The split of a call over CTAs; from the sizes and the element type alone, so that the workspace can be sized by it.
GradShape grad_shape(uint32_t heads, int64_t batch, int64_t q_len, int64_t k_len, int V) {
    GradShape g = {0, 0, 0, 0, 0};
    if (batch == 0 || q_len == 0 || k_len == 0) return g;
    const int64_t row_blocks = (q_len + V - 1) / V, col_groups = (k_len + V - 1) / V;
    for (g.blocks = kGradBlocks;; g.blocks *= 2) {
        const int64_t deltas = col_groups + (row_blocks < g.blocks ? row_blocks : g.blocks) - 1;
        g.segments = (uint32_t)((row_blocks + g.blocks - 1) / g.blocks);
        g.chunks = (uint32_t)((deltas + kGradMaxThreads - 1) / kGradMaxThreads);
        const int64_t per = (deltas + g.chunks - 1) / g.chunks;
        g.lanes = (uint32_t)((per + 31) / 32 * 32);
        g.parts = (uint64_t)batch * g.segments * g.chunks;
        // longer walks while they leave many CTAs: fewer sums by buckets
        if (g.blocks * 2 > kGradMostBlocks || row_blocks < g.blocks * 2 || (unsigned __int128)g.parts * heads < 148 * 32) return g;
    }
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
    a.top = 1;
    while (a.top * 2 < pb.bk.side) a.top *= 2;
    a.low = -pb.bk.edges[pb.bk.side - 1];
    a.high = pb.causal ? 1 : pb.bk.two_sided ? pb.bk.edges[pb.bk.side - 1] : 0;
    const int V = dtype == 0 ? kPiece<float> : kPiece<__nv_bfloat16>;
    if (pb.q_len <= kBiasFew) {
        constexpr int kRow = kBiasThreads * kBiasRowPieces;
        a.k_tiles = (uint32_t)(((pb.k_len + V - 1 + V - 1) / V + kRow - 1) / kRow);  // (rows may begin inside a piece)
        const unsigned __int128 grid = (unsigned __int128)pb.batch * pb.heads * pb.q_len * a.k_tiles;
        if (grid >= (1u << 31)) return kGridTooSmall;
        if (dtype == 0) launch_next(bias_few_kernel<float>, (unsigned)grid, kBiasThreads, 0, st, a);
        else launch_next(bias_few_kernel<__nv_bfloat16>, (unsigned)grid, kBiasThreads, 0, st, a);
        return cudaGetLastError();
    }
    const int64_t pieces = (pb.k_len + V - 1) / V;
    a.k_tiles = (uint32_t)((pieces + kBiasPieces - 1) / kBiasPieces);
    a.q_tiles = (uint32_t)((pb.q_len + kBiasRows - 1) / kBiasRows);
    a.lanes_log2 = 0;
    while (a.lanes_log2 < 5 && (1 << a.lanes_log2) < pieces) ++a.lanes_log2;
    const unsigned __int128 grid = (unsigned __int128)pb.batch * pb.heads * a.q_tiles * a.k_tiles;
    if (grid >= (1u << 31)) return kGridTooSmall;
    if (dtype == 0) launch_next(bias_forward_kernel<float>, (unsigned)grid, kBiasThreads, 0, st, a);
    else launch_next(bias_forward_kernel<__nv_bfloat16>, (unsigned)grid, kBiasThreads, 0, st, a);
    return cudaGetLastError();
}

size_t bias_grad_workspace_bytes(uint32_t buckets, uint32_t heads, int64_t batch, int64_t q_len, int64_t k_len) {
    // for either element type: fp32 rows are cut into more segments, bf16 into no more chunks
    uint64_t parts = 0;
    for (int V : {kPiece<float>, kPiece<__nv_bfloat16>}) {
        const GradShape g = grad_shape(heads, batch, q_len, k_len, V);
        if (g.parts > parts) parts = g.parts;
    }
    const unsigned __int128 bytes = (unsigned __int128)parts * buckets * heads * sizeof(double);
    if (bytes >= ((unsigned __int128)1 << 62)) return (size_t)1 << 62;
    return ((size_t)bytes + 255) / 256 * 256;
}

cudaError_t launch_bias_backward(const BiasProblem& pb, const void* grad, int64_t grad_ld, int dtype, float* grad_rows,
                                 int64_t grad_rows_ld, void* workspace, cudaStream_t st) {
    const int V = dtype == 0 ? kPiece<float> : kPiece<__nv_bfloat16>;
    const GradShape g = grad_shape(pb.heads, pb.batch, pb.q_len, pb.k_len, V);
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
    a.blocks = g.blocks;
    a.grad_rows = grad_rows;
    a.grad_rows_ld = grad_rows_ld;
    const unsigned __int128 grid = (unsigned __int128)g.parts * pb.heads;
    if (grid >= (1u << 31)) return kGridTooSmall;
    const int64_t size = dtype == 0 ? 4 : 2;
    const bool aligned = ((uintptr_t)grad & 15u) == 0 && grad_ld * size % 16 == 0;
    const size_t smem = (size_t)kGradStages * g.lanes / 32 * V * (aligned ? 32 : 33) * 16;
    if (g.parts > 0) {
        void (*kernel)(BiasGradArgs) = dtype == 0 ? (aligned ? bias_grad_kernel<float, true> : bias_grad_kernel<float, false>)
                                       : aligned  ? bias_grad_kernel<__nv_bfloat16, true>
                                                  : bias_grad_kernel<__nv_bfloat16, false>;
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        launch_next(kernel, (unsigned)grid, g.lanes < 128 ? 128 : g.lanes, smem, st, a);
    }
    launch_next(bias_grad_join_kernel, (unsigned)(pb.heads * pb.bk.buckets), 32, 0, st, a);
    return cudaGetLastError();
}

}  // namespace robe
