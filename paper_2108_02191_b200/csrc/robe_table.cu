// Rows of a plain table: lookup with scaling, and the table's gradient by sorted ids.
//
// The lookup moves each row once: out[r] = scale * table[ids[r]], bound by memory.  The gradient
// S_v = sum of the gradient rows whose id is v needs them by id: ids and positions are sorted (stable radix sort, so the
// order of a sum is the order of the rows in the call), the sorted positions are cut into chunks of equal length however
// the ids repeat, a chunk sums its runs of equal ids in registers, and runs that cross a border between chunks are
// joined afterwards from one partial row per chunk.  No atomics on floating-point data, no waits between CTAs:
// the result is bit-reproducible.
#include "robe_internal.h"
#include "robe_rowops.cuh"

namespace robe {

namespace {

constexpr int kTableThreads = 256;

// V consecutive elements by accesses of at most 16 bytes
template <class T, int V>
constexpr int kAccess = V * (int)sizeof(T) > 16 ? kPiece<T> : V;
template <class T, int V>
struct Elements {
    Pack<T, kAccess<T, V>> p[V / kAccess<T, V>];
    __device__ __forceinline__ float get(int k) const { return widen(p[k / kAccess<T, V>].v[k % kAccess<T, V>]); }
    __device__ __forceinline__ void set(int k, float v) { p[k / kAccess<T, V>].v[k % kAccess<T, V>] = narrow<T>(v); }
    template <bool STREAM>
    __device__ __forceinline__ void load(const T* from) {
#pragma unroll
        for (int q = 0; q < V / kAccess<T, V>; ++q) p[q] = load_pack<STREAM, T, kAccess<T, V>>(from + q * kAccess<T, V>);
    }
    template <bool STREAM>
    __device__ __forceinline__ void store(T* to) const {
#pragma unroll
        for (int q = 0; q < V / kAccess<T, V>; ++q) store_pack<STREAM, T, kAccess<T, V>>(to + q * kAccess<T, V>, p[q]);
    }
};

// ---------------------------------------------------------------- lookup

struct LookupArgs {
    const void* table;
    int64_t table_ld, vocab;
    IdList ids;
    int64_t first;  // of ids
    void* out;      // row `first`
    int64_t out_ld;
    uint32_t items;   // rows x pieces of a row
    uint32_t pieces;  // of a row
    uint64_t magic;   // of pieces
    float scale;
};

// A thread takes ITEMS pieces of V elements, a CTA's width apart, all of their loads under way together.
template <class TT, class TO, int V, int ITEMS>
__global__ void __launch_bounds__(kTableThreads) lookup_kernel(LookupArgs a) {
    follow();
    const uint32_t t0 = blockIdx.x * (uint32_t)(kTableThreads * ITEMS) + threadIdx.x;
    Elements<TT, V> e[ITEMS];
    uint32_t row[ITEMS], piece[ITEMS];
    bool in[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t t = t0 + i * kTableThreads;
        row[i] = divide(t, a.pieces, a.magic);
        piece[i] = t - row[i] * a.pieces;
        in[i] = false;
        if (t < a.items) {
            const int64_t id = a.ids.load(a.first + row[i]);
            in[i] = id >= 0 && id < a.vocab;
            if (in[i]) e[i].template load<false>((const TT*)a.table + id * a.table_ld + (uint64_t)piece[i] * V);
        }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if (t0 + i * kTableThreads >= a.items) return;
        if (!ROBE_CHK(piece[i] < a.pieces && (uint64_t)row[i] * a.pieces + piece[i] < a.items, ROBE_DBG_ROW_POS)) return;
        Elements<TO, V> o;
#pragma unroll
        for (int k = 0; k < V; ++k) o.set(k, in[i] ? e[i].get(k) * a.scale : 0.0f);
        o.template store<false>((TO*)a.out + row[i] * a.out_ld + (uint64_t)piece[i] * V);
    }
}

// most elements of a piece: what both sides' addresses are aligned to and rows are made of
int piece_of(int most, int64_t d, const void* p, int64_t p_ld, int64_t p_size, const void* q, int64_t q_ld, int64_t q_size, int64_t rows) {
    for (int v = most; v > 1; v /= 2) {
        const int64_t pb = v * p_size > 16 ? 16 : v * p_size, qb = v * q_size > 16 ? 16 : v * q_size;
        if (d % v != 0 || (uintptr_t)p % pb != 0 || (uintptr_t)q % qb != 0) continue;
        if (rows > 1 && (p_ld * p_size % pb != 0 || q_ld * q_size % qb != 0)) continue;
        return v;
    }
    return 1;
}

template <class TT, class TO, int V>
void launch_lookup(const LookupArgs& a, cudaStream_t st) {
    // few pieces: one a thread, spread over more SMs
    constexpr int kItems = 4;
    const bool few = a.items < 148u * 4 * kTableThreads * kItems;
    const uint32_t per = kTableThreads * (few ? 1 : kItems);
    launch_next(few ? lookup_kernel<TT, TO, V, 1> : lookup_kernel<TT, TO, V, kItems>, (a.items + per - 1) / per, kTableThreads, 0, st, a);
}

template <class TT, class TO>
void launch_lookup(const LookupArgs& a, int piece, cudaStream_t st) {
    constexpr int kMost = sizeof(TT) == 4 && sizeof(TO) == 4 ? 4 : 8;
    if (kMost == 8 && piece == 8) launch_lookup<TT, TO, kMost>(a, st);
    else if (piece == 4) launch_lookup<TT, TO, 4>(a, st);
    else if (piece == 2) launch_lookup<TT, TO, 2>(a, st);
    else launch_lookup<TT, TO, 1>(a, st);
}

// ---------------------------------------------------------------- gradient

// Rows of a chunk of sorted positions.  Enough chunks for two waves of threads with eight columns each; at most 256 rows, so that
// no fp32 sum has more terms than that.
uint32_t chunk_rows(int64_t rows, int64_t d) {
    const unsigned __int128 threads = (unsigned __int128)rows * (uint64_t)((d + 7) / 8);
    uint32_t c = 16;
    while (c < 256 && threads / (2 * c) >= 2u * 148u * 2048u) c *= 2;
    return c;
}

struct GradLayout {
    size_t keys[2], places[2], counts, totals, flags, parts, total;
    uint32_t chunk;
    uint64_t chunks;
    int64_t parts_ld;
};
GradLayout grad_layout(int64_t rows, int64_t vocab, int64_t d) {
    GradLayout L;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) & ~(size_t)255;
        return here;
    };
    for (int k = 0; k < 2; ++k) {
        L.keys[k] = take((size_t)rows * 4);
        L.places[k] = take((size_t)rows * 4);
    }
    L.counts = take(sort_counts_bytes());
    L.totals = take(sort_totals_bytes());
    L.flags = take((size_t)vocab);
    L.chunk = chunk_rows(rows, d);
    L.chunks = ((uint64_t)rows + L.chunk - 1) / L.chunk;
    L.parts_ld = (d + 3) / 4 * 4;
    L.parts = take((size_t)L.chunks * 2 * L.parts_ld * 4);
    L.total = at;
    return L;
}

struct GradArgs {
    const void* grad;
    int64_t grad_ld;
    IdList ids;
    int64_t rows, vocab, d, skip;
    float* table;
    int64_t table_ld;
    float scale;
    int accumulate;
    uint32_t *keys, *places;  // sorted from grad_sums_kernel on
    uint8_t* flags;           // [vocab] row has a gradient; not looked at when accumulating
    float* parts;             // [chunks][2]: what a chunk has of the run it begins in, and of the run it ends in
    int64_t parts_ld;
    uint32_t chunk;
    uint64_t chunks;
    uint32_t slices;       // of columns: CTAs per row (sums), warps per row (join)
    uint32_t join_blocks;  // grad_join_kernel: CTAs that join; the others fill
    uint32_t pieces;       // fill: of a row
    uint64_t magic;        // of pieces
    int aligned;           // rows of `table` in pieces of four columns
};

// Sort keys: ids; what gets no gradient sorts behind them.
__global__ void __launch_bounds__(kTableThreads) grad_keys_kernel(GradArgs a) {
    follow<true>();
    const uint64_t t = (uint64_t)blockIdx.x * kTableThreads + threadIdx.x;
    if (t < (uint64_t)a.rows) {
        const int64_t id = a.ids.load((int64_t)t);
        a.keys[t] = id >= 0 && id < a.vocab && id != a.skip ? (uint32_t)id : (uint32_t)a.vocab;
        a.places[t] = (uint32_t)t;
    }
    if (a.accumulate) return;
    const uint64_t words = ((uint64_t)a.vocab + 15) / 16;  // (the workspace is in whole 256 bytes)
    for (uint64_t k = t; k < words; k += (uint64_t)gridDim.x * kTableThreads) ((uint4*)a.flags)[k] = make_uint4(0, 0, 0, 0);
}

// Sums of a chunk's runs, V columns a thread, `lanes` threads a row.
template <class T, int V>
__global__ void __launch_bounds__(kTableThreads) grad_sums_kernel(GradArgs a, uint32_t lanes) {
    constexpr int kAhead = V * sizeof(T) > 16 ? 4 : 8;  // rows under way
    extern __shared__ uint32_t staged[];  // keys, then places, of the CTA's chunks
    follow<true>();
    const uint32_t groups = kTableThreads / lanes;
    const uint64_t block = blockIdx.x / a.slices;
    const uint32_t slice = blockIdx.x - (uint32_t)block * a.slices;
    const uint64_t from = block * groups * a.chunk;
    const uint32_t staged_rows = groups * a.chunk;
    for (uint32_t k = threadIdx.x; k < staged_rows; k += kTableThreads)
        if (from + k < (uint64_t)a.rows) {
            staged[k] = a.keys[from + k];
            staged[staged_rows + k] = a.places[from + k];
        }
    __syncthreads();
    const uint32_t group = threadIdx.x / lanes;
    const uint64_t c = block * groups + group;
    const int64_t col = ((int64_t)slice * lanes + threadIdx.x % lanes) * V;
    if (c >= a.chunks || col >= a.d) return;
    const uint64_t begin = c * a.chunk;
    uint32_t count = (uint32_t)((uint64_t)a.rows - begin < a.chunk ? (uint64_t)a.rows - begin : a.chunk);
    const uint32_t* keys = staged + group * a.chunk;
    const uint32_t* places = keys + staged_rows;
    uint32_t key = keys[0];
    if (key >= (uint32_t)a.vocab) return;
    bool open = begin > 0 && a.keys[begin - 1] == key;  // the run began in an earlier chunk
    float sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] = 0.0f;
    auto close = [&](bool goes_on) {
        if (!open && !a.accumulate && col == 0) a.flags[key] = 1;
        if (open || goes_on) {
            float* to = a.parts + (c * 2 + (open ? 0 : 1)) * a.parts_ld + col;
#pragma unroll
            for (int v = 0; v < V; ++v) to[v] = sum[v];
            return;
        }
        float* to = a.table + (int64_t)key * a.table_ld + col;
        if (!ROBE_CHK(key < (uint32_t)a.vocab && col + V <= a.d, ROBE_DBG_ROW_POS)) return;
        Elements<float, V> o;
        if (a.accumulate) o.template load<true>(to);
#pragma unroll
        for (int v = 0; v < V; ++v) o.set(v, a.accumulate ? fmaf(a.scale, sum[v], o.get(v)) : a.scale * sum[v]);
        o.template store<true>(to);
    };
    for (uint32_t i = 0; i < count; i += kAhead) {
        Elements<T, V> e[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < count && ROBE_CHK(places[i + u] < (uint64_t)a.rows, ROBE_DBG_ROW_POS))
                e[u].template load<true>((const T*)a.grad + (int64_t)places[i + u] * a.grad_ld + col);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u >= count) break;
            const uint32_t k = keys[i + u];
            if (k != key) {
                close(false);
                if (k >= (uint32_t)a.vocab) return;  // (these are the last)
                key = k;
                open = false;
#pragma unroll
                for (int v = 0; v < V; ++v) sum[v] = 0.0f;
            }
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += e[u].get(v);
        }
    }
    close(begin + count < (uint64_t)a.rows && a.keys[begin + count] == key);
}

// Runs that end in a later chunk than they begin in: the chunks' parts in order, in 64 bits.  A warp takes a chunk's last run and
// 128 columns; runs over many chunks are shared by the CTA's warps.  The CTAs behind those write +0 where no id was.
constexpr int kJoinWarps = kTableThreads / 32;
constexpr uint32_t kJoinAlone = 16;  // parts that a warp adds by itself
__global__ void __launch_bounds__(kTableThreads) grad_join_kernel(GradArgs a) {
    follow();
    if (blockIdx.x >= a.join_blocks) {
        const uint64_t items = (uint64_t)a.vocab * a.pieces;
        constexpr uint32_t kItems = 8;
        const uint64_t first = (uint64_t)(blockIdx.x - a.join_blocks) * (kTableThreads * kItems);
        const uint64_t row0 = first / a.pieces;
        const uint32_t piece0 = (uint32_t)(first - row0 * a.pieces);
#pragma unroll
        for (uint32_t i = 0; i < kItems; ++i) {
            const uint32_t k = i * kTableThreads + threadIdx.x;
            if (first + k >= items) return;
            const uint32_t r = divide(piece0 + k, a.pieces, a.magic), piece = piece0 + k - r * a.pieces;
            const uint64_t row = row0 + r;
            if (!ROBE_CHK(row < (uint64_t)a.vocab, ROBE_DBG_ROW_POS)) return;
            if (__ldca(a.flags + row) != 0) continue;
            if (a.aligned) __stcs((float4*)(a.table + row * a.table_ld) + piece, make_float4(0.0f, 0.0f, 0.0f, 0.0f));
            else a.table[row * a.table_ld + piece] = 0.0f;
        }
        return;
    }
    __shared__ uint32_t shared_runs[kJoinWarps];  // parts of the runs that the warps share; 0: none
    __shared__ double sums[kJoinWarps][4][32];
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t blocks = blockIdx.x / a.slices;  // of kJoinWarps chunks
    const uint32_t slice = blockIdx.x - blocks * a.slices;
    const int64_t col = (int64_t)slice * 128 + lane * 4;
    auto parts_of = [&](uint64_t c) -> uint32_t {  // of the last run of chunk c, 0 where it ends there
        const uint64_t end = (c + 1) * a.chunk;
        if (c >= a.chunks || end >= (uint64_t)a.rows) return 0;
        const uint32_t key = a.keys[end - 1];
        if (key >= (uint32_t)a.vocab || a.keys[end] != key) return 0;
        if (c > 0 && a.keys[end - a.chunk - 1] == key) return 0;  // it began earlier
        // it reaches the end of chunk c + k: true up to some k; 32 places at a time, first powers of two, then between
        auto reaches = [&](uint64_t k) {
            const uint64_t e = (c + k + 1) * a.chunk;
            return a.keys[(e < (uint64_t)a.rows ? e : (uint64_t)a.rows) - 1] == key;
        };
        uint64_t yes = 0, no;  // it reaches the end of chunk c + yes and not of c + no
        {
            const uint64_t k = 1ull << lane;
            const uint32_t hit = __ballot_sync(0xFFFFFFFFu, c + k < a.chunks && reaches(k));
            const int hits = __popc(hit);
            if (hits > 0) yes = 1ull << (hits - 1);
            no = 1ull << hits;
            if (no > a.chunks - c) no = a.chunks - c;
        }
        while (no - yes > 1) {
            const uint64_t step = (no - yes + 31) / 32, k = yes + step * (lane + 1);
            const uint32_t hits = __popc(__ballot_sync(0xFFFFFFFFu, k < no && reaches(k)));
            const uint64_t up = yes + step * (hits + 1);
            yes += step * hits;
            if (up < no) no = up;
        }
        // chunks c .. c + yes end in it; it goes on into the next one if there is one and it begins with it
        const uint64_t next = (c + yes + 1) * a.chunk;
        return (uint32_t)(yes + 1 + (next < (uint64_t)a.rows && a.keys[next] == key ? 1 : 0));
    };
    auto add = [&](double (&s)[4], uint64_t c, uint32_t begin, uint32_t end) {  // parts begin .. end - 1 of the run of chunk c
        if (col >= a.d) return;
        for (uint32_t k = begin; k < end; k += 8) {
            float4 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (k + u < end) v[u] = __ldca((const float4*)(a.parts + ((c + k + u) * 2 + (k + u == 0 ? 1 : 0)) * a.parts_ld + col));
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (k + u < end) {
                    s[0] += v[u].x;
                    s[1] += v[u].y;
                    s[2] += v[u].z;
                    s[3] += v[u].w;
                }
        }
    };
    auto finish = [&](const double (&s)[4], uint64_t c) {
        const uint32_t key = a.keys[(c + 1) * a.chunk - 1];
        float* to = a.table + (int64_t)key * a.table_ld + col;
        if (col >= a.d || !ROBE_CHK(key < (uint32_t)a.vocab, ROBE_DBG_ROW_POS)) return;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (col + q < a.d) to[q] = a.accumulate ? fmaf(a.scale, (float)s[q], to[q]) : a.scale * (float)s[q];
    };
    const uint64_t mine = (uint64_t)blocks * kJoinWarps + warp;
    const uint32_t parts = parts_of(mine);
    if (lane == 0) shared_runs[warp] = parts > kJoinAlone ? parts : 0;
    if (parts > 0 && parts <= kJoinAlone) {
        double s[4] = {0.0, 0.0, 0.0, 0.0};
        add(s, mine, 0, parts);
        finish(s, mine);
    }
    __syncthreads();
    for (uint32_t w = 0; w < kJoinWarps; ++w) {
        const uint32_t n = shared_runs[w];
        if (n == 0) continue;
        const uint64_t c = (uint64_t)blocks * kJoinWarps + w;
        const uint32_t per = (n + kJoinWarps - 1) / kJoinWarps;
        const uint32_t begin = warp * per < n ? warp * per : n, end = begin + per < n ? begin + per : n;
        double s[4] = {0.0, 0.0, 0.0, 0.0};
        add(s, c, begin, end);
#pragma unroll
        for (int q = 0; q < 4; ++q) sums[warp][q][lane] = s[q];
        __syncthreads();
        if (warp == 0) {
            for (int k = 1; k < kJoinWarps; ++k)
#pragma unroll
                for (int q = 0; q < 4; ++q) s[q] += sums[k][q][lane];
            finish(s, c);
        }
        __syncthreads();
    }
}

template <class T, int V>
cudaError_t launch_sums(GradArgs& a, cudaStream_t st) {
    uint32_t lanes = 4;
    while (lanes < kTableThreads && (int64_t)lanes * V < a.d) lanes *= 2;
    // (the keys and places of a CTA's chunks are staged in shared memory: at most 32 KB)
    while (kTableThreads / lanes * a.chunk > 4096) lanes *= 2;
    a.slices = (uint32_t)((a.d + (int64_t)lanes * V - 1) / ((int64_t)lanes * V));
    const uint64_t groups = kTableThreads / lanes;
    const uint64_t grid = (a.chunks + groups - 1) / groups * a.slices;
    if (grid >= (1ull << 31)) return kGridTooSmall;
    launch_next(grad_sums_kernel<T, V>, (unsigned)grid, kTableThreads, groups * a.chunk * 8, st, a, lanes);
    return cudaSuccess;
}
template <class T>
cudaError_t launch_sums(GradArgs& a, int piece, cudaStream_t st) {
    constexpr int kMost = kPiece<T>;
    if (kMost == 8 && piece == 8) return launch_sums<T, kMost>(a, st);
    if (piece == 4) return launch_sums<T, 4>(a, st);
    if (piece == 2) return launch_sums<T, 2>(a, st);
    return launch_sums<T, 1>(a, st);
}

}  // namespace

cudaError_t launch_table_forward(const TableProblem& pb, void* out, int64_t out_ld, int out_dtype, cudaStream_t st) {
    const int64_t ts = pb.dtype == 0 ? 4 : 2, os = out_dtype == 0 ? 4 : 2;
    LookupArgs a;
    a.table = pb.table;
    a.table_ld = pb.table_ld;
    a.vocab = pb.vocab;
    a.ids = pb.ids;
    a.out_ld = out_ld;
    a.scale = pb.scale;
    const int piece = piece_of(ts + os == 8 ? 4 : 8, pb.d, pb.table, pb.table_ld, ts, out, out_ld, os, pb.rows > 1 || pb.vocab > 1 ? 2 : 1);
    a.pieces = (uint32_t)(pb.d / piece);
    a.magic = magic_of(a.pieces);
    // pieces are numbered in 32 bits: as many rows a launch as that allows
    const int64_t most = ((1ll << 31) - 1) / a.pieces;
    for (int64_t r = 0; r < pb.rows; r += most) {
        a.first = r;
        a.out = (char*)out + r * out_ld * os;
        a.items = (uint32_t)((pb.rows - r < most ? pb.rows - r : most) * a.pieces);
        if (pb.dtype == 0 && out_dtype == 0) launch_lookup<float, float>(a, piece, st);
        else if (pb.dtype == 0) launch_lookup<float, __nv_bfloat16>(a, piece, st);
        else if (out_dtype == 0) launch_lookup<__nv_bfloat16, float>(a, piece, st);
        else launch_lookup<__nv_bfloat16, __nv_bfloat16>(a, piece, st);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

size_t table_grad_workspace_bytes(int64_t rows, int64_t vocab, int64_t d) { return grad_layout(rows, vocab, d).total; }

cudaError_t launch_table_backward(const TableProblem& pb, const void* grad, int64_t grad_ld, int64_t skip, int accumulate, float* grad_table,
                                  int64_t grad_table_ld, void* workspace, cudaStream_t st) {
    if (accumulate && pb.rows == 0) return cudaSuccess;
    const GradLayout L = grad_layout(pb.rows, pb.vocab, pb.d);
    char* ws = (char*)workspace;
    GradArgs a;
    a.grad = grad;
    a.grad_ld = grad_ld;
    a.ids = pb.ids;
    a.rows = pb.rows;
    a.vocab = pb.vocab;
    a.d = pb.d;
    a.skip = skip;
    a.table = grad_table;
    a.table_ld = grad_table_ld;
    a.scale = pb.scale;
    a.accumulate = accumulate;
    a.flags = (uint8_t*)(ws + L.flags);
    a.parts = (float*)(ws + L.parts);
    a.parts_ld = L.parts_ld;
    a.chunk = L.chunk;
    a.chunks = L.chunks;
    a.aligned = piece_of(4, pb.d, grad_table, grad_table_ld, 4, grad_table, grad_table_ld, 4, 2) == 4;
    a.pieces = (uint32_t)(a.aligned ? pb.d / 4 : pb.d);
    a.magic = magic_of(a.pieces);
    const int64_t size = pb.dtype == 0 ? 4 : 2;
    // everything that is launched, before anything is
    a.slices = (uint32_t)((pb.d + 127) / 128);
    const uint64_t join = (L.chunks + kJoinWarps - 1) / kJoinWarps * a.slices;
    const unsigned __int128 fill = accumulate ? 0 : ((unsigned __int128)pb.vocab * a.pieces + kTableThreads * 8 - 1) / (kTableThreads * 8);
    if (join + fill >= (1ull << 31)) return kGridTooSmall;
    const int piece = piece_of(size == 4 ? 4 : 8, pb.d, grad, grad_ld, size, grad_table, grad_table_ld, 4, pb.rows > 1 || pb.vocab > 1 ? 2 : 1);
    if (L.chunks * (uint64_t)((pb.d + (int64_t)kTableThreads * piece - 1) / ((int64_t)kTableThreads * piece)) >= (1ull << 31)) return kGridTooSmall;

    uint32_t *keys[2] = {(uint32_t*)(ws + L.keys[0]), (uint32_t*)(ws + L.keys[1])},
             *places[2] = {(uint32_t*)(ws + L.places[0]), (uint32_t*)(ws + L.places[1])};
    a.keys = keys[0];
    a.places = places[0];
    const uint64_t threads = (uint64_t)pb.rows > (uint64_t)kTableThreads * 148 ? (uint64_t)pb.rows : (uint64_t)kTableThreads * 148;
    launch_next(grad_keys_kernel, (unsigned)((threads + kTableThreads - 1) / kTableThreads), kTableThreads, 0, st, a);
    if (pb.rows > 0) {
        uint32_t bits = 1;
        while (((uint64_t)pb.vocab >> bits) != 0) ++bits;  // (vocab itself is a key)
        const int in = launch_sort_pairs(keys, places, (uint64_t)pb.rows, bits, (uint32_t*)(ws + L.counts), (uint32_t*)(ws + L.totals), st);
        a.keys = keys[in];
        a.places = places[in];
        const cudaError_t e = pb.dtype == 0 ? launch_sums<float>(a, piece, st) : launch_sums<__nv_bfloat16>(a, piece, st);
        if (e != cudaSuccess) return e;
    }
    a.slices = (uint32_t)((pb.d + 127) / 128);
    a.join_blocks = (uint32_t)join;
    launch_next(grad_join_kernel, (unsigned)(join + (uint64_t)fill), kTableThreads, 0, st, a);
    return cudaGetLastError();
}

}  // namespace robe
