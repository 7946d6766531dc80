// Rows of a plain table: lookup with scaling, and the table's gradient by sorted ids.
//
// The lookup moves each row once: out[r] = scale * table[ids[r]], bound by memory.  The gradient
// S_v = sum of the gradient rows whose id is v needs them by id: ids and positions are sorted (stable radix sort, so the
// order of a sum is the order of the rows in the call), the sorted positions are cut into chunks of equal length however
// the ids repeat, a chunk sums its runs of equal ids in registers, and runs that cross a border between chunks are
// joined afterwards from one partial row per chunk.  No atomics on floating-point data, and CTAs wait for one another only
// within the cluster that sorts up to 65536 ids: the result is bit-reproducible.
#include "robe_internal.h"
#include "robe_rowops.cuh"

namespace robe {

namespace {

constexpr int kTableThreads = 256;

// V consecutive elements by accesses of at most 16 bytes.  Held as words: bf16 elements kept apart would take a register each.
template <class T, int V>
struct Elements {
    static constexpr int kBytes = V * (int)sizeof(T), kAccess = kBytes > 16 ? 16 : kBytes;
    using W = typename Word<kAccess>::type;
    union {
        W access[kBytes / kAccess];
        uint32_t word[(kBytes + 3) / 4];
    } e;
    __device__ __forceinline__ float get(int k) const {
        if (sizeof(T) == 4) return __uint_as_float(e.word[k]);
        if (V == 1) return widen_low((uint32_t) * (const unsigned short*)&e);
        return k % 2 ? widen_high(e.word[k / 2]) : widen_low(e.word[k / 2]);
    }
    __device__ __forceinline__ void set(const float (&v)[V]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int k = 0; k < V; ++k) e.word[k] = __float_as_uint(v[k]);
        } else if constexpr (V == 1) {
            e.word[0] = narrow2(v[0], 0.0f);
        } else {
#pragma unroll
            for (int k = 0; k < V; k += 2) e.word[k / 2] = narrow2(v[k], v[k + 1]);
        }
    }
    template <bool STREAM>
    __device__ __forceinline__ void load(const T* from) {
#pragma unroll
        for (int q = 0; q < kBytes / kAccess; ++q) e.access[q] = STREAM ? __ldcs((const W*)from + q) : __ldca((const W*)from + q);
    }
    template <bool STREAM>
    __device__ __forceinline__ void store(T* to) const {
#pragma unroll
        for (int q = 0; q < kBytes / kAccess; ++q) {
            if (STREAM) __stcs((W*)to + q, e.access[q]);
            else ((W*)to)[q] = e.access[q];
        }
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

// A thread takes a piece of V elements: few pieces, spread over the SMs.
template <class TT, class TO, int V>
__global__ void __launch_bounds__(kTableThreads) lookup_few_kernel(LookupArgs a) {
    follow();
    const uint32_t t = blockIdx.x * (uint32_t)kTableThreads + threadIdx.x;
    if (t >= a.items) return;
    const uint32_t row = divide(t, a.pieces, a.magic), piece = t - row * a.pieces;
    const int64_t id = a.ids.load(a.first + row);
    const bool in = id >= 0 && id < a.vocab;
    Elements<TT, V> e;
    if (in) e.template load<false>((const TT*)a.table + id * a.table_ld + (uint64_t)piece * V);
    float v[V];
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = in ? e.get(k) * a.scale : 0.0f;
    Elements<TO, V> o;
    o.set(v);
    o.template store<false>((TO*)a.out + row * a.out_ld + (uint64_t)piece * V);
}

// Many pieces: a CTA takes the ids of its rows to shared memory first, so that the latency of an id is paid once for kTiles rounds of
// loads (852 K rows of 128, fp32 to bf16: ids by each thread for itself 79 us, four pieces a thread under way 62, two
// 60).
constexpr int kTiles = 8;
constexpr int kLookupItems = 2;
constexpr uint32_t kLookupPieces = kTableThreads * kTiles * kLookupItems;
template <class TT, class TO, int V>
__global__ void __launch_bounds__(kTableThreads) lookup_kernel(LookupArgs a) {
    __shared__ uint32_t ids[kLookupPieces + 1];
    follow();
    const uint32_t t0 = blockIdx.x * kLookupPieces, end = a.items - t0 < kLookupPieces ? a.items : t0 + kLookupPieces;
    const uint32_t row0 = divide(t0, a.pieces, a.magic), rows = divide(end - 1, a.pieces, a.magic) - row0 + 1;
    for (uint32_t k = threadIdx.x; k < rows; k += kTableThreads) {
        const int64_t id = a.ids.load(a.first + row0 + k);
        if (ROBE_CHK(k < kLookupPieces + 1, ROBE_DBG_SHARED)) ids[k] = id >= 0 && id < a.vocab ? (uint32_t)id : 0xFFFFFFFFu;
    }
    __syncthreads();
    for (uint32_t base = t0 + threadIdx.x; base < end; base += kTableThreads * kLookupItems) {
        Elements<TT, V> e[kLookupItems];
        uint32_t row[kLookupItems], piece[kLookupItems], id[kLookupItems];
#pragma unroll
        for (int i = 0; i < kLookupItems; ++i) {
            const uint32_t t = base + i * kTableThreads;
            row[i] = divide(t, a.pieces, a.magic);
            piece[i] = t - row[i] * a.pieces;
            id[i] = t < end ? ids[row[i] - row0] : 0xFFFFFFFFu;
            if (id[i] != 0xFFFFFFFFu) e[i].template load<false>((const TT*)a.table + id[i] * a.table_ld + (uint64_t)piece[i] * V);
        }
#pragma unroll
        for (int i = 0; i < kLookupItems; ++i) {
            if (base + i * kTableThreads >= end) break;
            if (!ROBE_CHK(piece[i] < a.pieces && (uint64_t)row[i] * a.pieces + piece[i] < a.items, ROBE_DBG_ROW_POS)) return;
            float v[V];
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = id[i] != 0xFFFFFFFFu ? e[i].get(k) * a.scale : 0.0f;
            Elements<TO, V> o;
            o.set(v);
            o.template store<false>((TO*)a.out + row[i] * a.out_ld + (uint64_t)piece[i] * V);
        }
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
    if (a.items < 148u * kLookupPieces)
        launch_next(lookup_few_kernel<TT, TO, V>, (a.items + kTableThreads - 1) / kTableThreads, kTableThreads, 0, st, a);
    else launch_next(lookup_kernel<TT, TO, V>, (a.items + kLookupPieces - 1) / kLookupPieces, kTableThreads, 0, st, a);
}

template <class TT, class TO>
void launch_lookup(const LookupArgs& a, int piece, cudaStream_t st) {
    constexpr int kMost = sizeof(TO) == 4 ? 4 : 8;
    if (kMost == 8 && piece == 8) launch_lookup<TT, TO, kMost>(a, st);
    else if (piece == 4) launch_lookup<TT, TO, 4>(a, st);
    else if (piece == 2) launch_lookup<TT, TO, 2>(a, st);
    else launch_lookup<TT, TO, 1>(a, st);
}

// ---------------------------------------------------------------- gradient

// Rows of a chunk of sorted positions: as many as make one full wave of CTAs (four an SM, four columns a thread); at least 16, and at
// most 256, so that no fp32 sum has more terms than that.  A border costs a row of sums for the run that crosses it, and CTAs
// beyond a wave leave SMs empty (16384 x 4096 bf16, Zipf ids, accumulating: two waves 77 us, one
// and a half 79, one 72, three quarters of one 80; 852 K x 64 fp32 147, 153, 144, 146; with uniform ids, and 5000 x 1000 bf16, all alike).
constexpr uint32_t kChunkLeast = 16, kChunkMost = 256;
constexpr uint64_t kWave = 4 * 148 * kTableThreads;  // threads
uint32_t chunk_rows(int64_t rows, int64_t d) {
    const unsigned __int128 threads = (unsigned __int128)rows * (uint64_t)((d + 3) / 4);
    const unsigned __int128 c = (threads + kWave - 1) / kWave;
    return c < kChunkLeast ? kChunkLeast : c > kChunkMost ? kChunkMost : (uint32_t)c;
}
// Chunks x columns by fours, at least: what the largest of all calls with at most so many rows of at most so many columns has, so that a
// workspace for the largest call serves every smaller one.  (Chunks get longer with a call, so there may be fewer of them: but of c rows, c
// between the limits, there are at most ceil(kWave / fours), for c fours of such a row make up a wave at most.)
uint64_t most_parts(int64_t rows, int64_t d) {
    const uint64_t n = (uint64_t)rows, fours = (uint64_t)((d + 3) / 4), most = (n + kChunkMost - 1) / kChunkMost * fours;
    if (chunk_rows(rows, d) == kChunkLeast) return (n + kChunkLeast - 1) / kChunkLeast * fours;
    return most > kWave + fours ? most : kWave + fours;
}
// Where there are many chunks, the parts of a run that covers kFold of them are added up before the join.
constexpr uint32_t kFold = 32;
constexpr uint64_t kFoldFrom = 4096;

constexpr int64_t kClusterRows = 65536;  // up to so many ids one cluster sorts in its shared memory
constexpr int64_t kAloneRows = 512;      // up to so many every CTA that needs them sorts them for itself
struct GradLayout {
    size_t keys[2], places[2], counts, totals, parts, folds, total;
    uint32_t chunk;
    uint64_t chunks;
    int64_t parts_ld;
};
GradLayout grad_layout(int64_t rows, int64_t d) {
    GradLayout L;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) & ~(size_t)255;
        return here;
    };
    for (int k = 0; k < 2; ++k) {
        const bool used = k == 0 || rows > kClusterRows;
        L.keys[k] = take(used ? (size_t)rows * 4 : 0);
        L.places[k] = take(used ? (size_t)rows * 4 : 0);
    }
    L.counts = take(rows > kClusterRows ? sort_counts_bytes() : 0);
    L.totals = take(rows > kClusterRows ? sort_totals_bytes() : 0);
    L.chunk = chunk_rows(rows, d);
    L.chunks = ((uint64_t)rows + L.chunk - 1) / L.chunk;
    L.parts_ld = (d + 3) / 4 * 4;
    const size_t most = most_parts(rows, d);
    L.parts = take(most * 2 * 4 * sizeof(float));
    L.folds = take(most * 4 * sizeof(double) / kFold);
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
    uint32_t *keys, *places;  // sorted from grad_sums_kernel on, for few ids from the join on
    float* parts;             // [chunks][2]: what a chunk has of the run it begins in, and of the run it ends in
    int64_t parts_ld;
    double* folds;            // [chunks / kFold]: the first parts of kFold chunks that lie in one run as a whole; nullptr: none
    uint32_t chunk;
    uint64_t chunks;
    uint32_t slices;       // of columns: CTAs per row (sums), warps per row (join)
    uint32_t lanes;        // join: that take a part's columns of a slice, four each
    int flat;              // the table is one run of elements from a 16-byte boundary on
    int aligned;           // rows of `table` in pieces of four columns
};

// ---- ids and positions in the order of the ids, equal ids in the order of the call (least digit first, stable)

// The sort key of a position: the id; what gets no gradient sorts behind all of them.
__device__ __forceinline__ uint32_t key_of(const GradArgs& a, int64_t p) {
    const int64_t id = a.ids.load(p);
    return id >= 0 && id < a.vocab && id != a.skip ? (uint32_t)id : (uint32_t)a.vocab;
}
// +0 in every row of the table.  The sums write theirs over it: the order of kernels makes that safe, and knowing the rows without
// an id would take a pass over flags for each (the rows written twice are as many as the ids have values).
__device__ __forceinline__ void clear_table(const GradArgs& a, uint64_t thread, uint64_t threads) {
    if (a.flat) {
        const uint64_t elements = (uint64_t)a.vocab * (uint64_t)a.d;
        for (uint64_t k = thread; k < elements / 4; k += threads) __stcs((float4*)a.table + k, make_float4(0.0f, 0.0f, 0.0f, 0.0f));
        if (thread < elements % 4) a.table[elements / 4 * 4 + thread] = 0.0f;
    } else {
        for (uint64_t row = thread / 32; row < (uint64_t)a.vocab; row += threads / 32)
            for (int64_t col = thread % 32; col < a.d; col += 32) a.table[row * (uint64_t)a.table_ld + col] = 0.0f;
    }
}
// Keys and positions of many ids.
__global__ void __launch_bounds__(kTableThreads) grad_keys_kernel(GradArgs a) {
    follow<true>();
    const uint64_t t = (uint64_t)blockIdx.x * kTableThreads + threadIdx.x, threads = (uint64_t)gridDim.x * kTableThreads;
    for (uint64_t p = t; p < (uint64_t)a.rows; p += threads) {
        a.keys[p] = key_of(a, (int64_t)p);
        a.places[p] = (uint32_t)p;
    }
    if (!a.accumulate) clear_table(a, t, threads);
}

constexpr uint32_t kClusterMost = 8;  // CTAs
constexpr int kClusterBits = 9;       // of a digit, at most
// Ranks of a warp's ITEMS x 32 keys among its own by digit, in the order item, lane; counts[digit] is how many of each digit came before and
// is counted up.  The lanes of a digit come of one ballot a bit.
template <int ITEMS>
__device__ __forceinline__ void rank_in_warp(const uint32_t (&key)[ITEMS], uint32_t shift, uint32_t bits, uint16_t* counts, uint32_t (&rank)[ITEMS]) {
    const uint32_t lane = threadIdx.x & 31, mask = (1u << bits) - 1u;
#pragma unroll
    for (int r = 0; r < ITEMS; ++r) {
        const uint32_t digit = (key[r] >> shift) & mask;
        uint32_t peers = 0xFFFFFFFFu;
#pragma unroll
        for (uint32_t b = 0; b < kClusterBits; ++b) {
            if (b >= bits) break;
            const bool bit = (digit >> b) & 1u;
            const uint32_t with = __ballot_sync(0xFFFFFFFFu, bit);
            peers &= bit ? with : ~with;
        }
        const uint32_t below = peers & ((1u << lane) - 1u), before = counts[digit];
        __syncwarp();
        if (below == 0) counts[digit] = (uint16_t)(before + __popc(peers));
        __syncwarp();
        rank[r] = before + __popc(below);
    }
}
// Exclusive scan of a value per thread of a CTA of kRankThreads; contains barriers.
constexpr int kRankThreads = 1024, kRankWarps = kRankThreads / 32;
__device__ __forceinline__ uint32_t scan_in_cta(uint32_t v, uint32_t* warp_sums) {
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    uint32_t upto = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t b = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= (uint32_t)o) upto += b;
    }
    if (lane == 31) warp_sums[warp] = upto;
    __syncthreads();
    if (warp == 0) {
        uint32_t w = warp_sums[lane], sum = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t b = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= (uint32_t)o) sum += b;
        }
        warp_sums[lane] = sum - w;
    }
    __syncthreads();
    const uint32_t before = warp_sums[warp] + upto - v;
    __syncthreads();
    return before;
}

// Up to 65536 ids: a cluster of up to eight CTAs sorts them in its shared memory, in one launch.  The other clusters clear the table.
// (16384 ids of 17 bits: 11 us; keys, and three passes of three kernels each, 26.)
template <int ITEMS>
struct ClusterSmem {
    uint2 pair[2][kRankThreads * ITEMS];
    uint16_t warp_digit[kRankWarps][1 << kClusterBits];
    uint32_t total[1 << kClusterBits], start[1 << kClusterBits], base[1 << kClusterBits];
    uint32_t warp_sums[kRankWarps];
};
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t address_in(const void* p, uint32_t rank) {  // the same place in another CTA of the cluster
    uint32_t at;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return at;
}
template <int ITEMS>
__global__ void __launch_bounds__(kRankThreads) grad_cluster_sort_kernel(GradArgs a, uint32_t ctas, uint32_t passes, uint32_t bits) {
    extern __shared__ __align__(16) uint8_t sort_memory[];
    ClusterSmem<ITEMS>& sm = *(ClusterSmem<ITEMS>*)sort_memory;
    constexpr uint32_t kTile = kRankThreads * ITEMS;
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid / 32, rank_of_cta = blockIdx.x % ctas;
    follow<true>();
    if (blockIdx.x >= ctas) {
        clear_table(a, (uint64_t)(blockIdx.x - ctas) * kRankThreads + tid, (uint64_t)(gridDim.x - ctas) * kRankThreads);
        return;
    }
    const uint32_t local = warp * (32 * ITEMS) + lane, first = rank_of_cta * kTile;
    uint32_t key[ITEMS], place[ITEMS];
#pragma unroll
    for (int r = 0; r < ITEMS; ++r) {
        place[r] = first + local + r * 32;
        key[r] = place[r] < (uint64_t)a.rows ? key_of(a, place[r]) : 0xFFFFFFFFu;  // (behind all others, being the last)
    }
    for (uint32_t pass = 0; pass < passes; ++pass) {
        const uint32_t shift = pass * bits, bins = 1u << bits;
        if (pass > 0) {
#pragma unroll
            for (int r = 0; r < ITEMS; ++r) {
                const uint2 p = sm.pair[pass & 1][local + r * 32];
                key[r] = p.x;
                place[r] = p.y;
            }
        }
        for (uint32_t k = lane; k < bins / 2; k += 32) ((uint32_t*)sm.warp_digit[warp])[k] = 0;
        __syncwarp();
        uint32_t rank[ITEMS];
        rank_in_warp(key, shift, bits, sm.warp_digit[warp], rank);
        __syncthreads();
        if (tid < bins / 2) {  // two digits in a word (a CTA has fewer pairs than 16 bits hold)
            uint32_t sum = 0;
#pragma unroll 16
            for (int w = 0; w < kRankWarps; ++w) {
                uint32_t* both = (uint32_t*)sm.warp_digit[w] + tid;
                const uint32_t n = *both;
                *both = sum;
                sum += n;
            }
            sm.total[2 * tid] = sum & 0xFFFFu;
            sm.total[2 * tid + 1] = sum >> 16;
        }
        cluster_barrier();
        uint32_t all = 0, before = 0, own = 0;
        if (tid < bins) {
            uint32_t n[kClusterMost];
#pragma unroll
            for (uint32_t c = 0; c < kClusterMost; ++c) {
                n[c] = 0;
                if (c < ctas) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(n[c]) : "r"(address_in(&sm.total[tid], c)));
            }
            own = sm.total[tid];
#pragma unroll
            for (uint32_t c = 0; c < kClusterMost; ++c) {
                if (c < rank_of_cta) before += n[c];
                all += n[c];
            }
        }
        // where a digit starts among all pairs (at most 2^16) and among this CTA's, in one scan
        const uint32_t start = scan_in_cta(all | own << 17, sm.warp_sums);
        if (tid < bins) {
            sm.start[tid] = start >> 17;
            sm.base[tid] = (start & 0x1FFFFu) + before - (start >> 17);  // a pair at place k of this CTA goes to base + k
        }
        __syncthreads();
        // laid out by digit in this CTA first: pairs that go to neighbouring places are then written by neighbouring lanes
        uint2* const mine = sm.pair[pass & 1];
#pragma unroll
        for (int r = 0; r < ITEMS; ++r) {
            const uint32_t digit = (key[r] >> shift) & (bins - 1u);
            const uint32_t to = sm.start[digit] + sm.warp_digit[warp][digit] + rank[r];
            if (ROBE_CHK(to < kTile, ROBE_DBG_SHARED)) mine[to] = make_uint2(key[r], place[r]);
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ITEMS; ++r) {
            const uint32_t k = tid + r * kRankThreads;
            const uint2 p = mine[k];
            const uint32_t to = sm.base[(p.x >> shift) & (bins - 1u)] + k;
            if (!ROBE_CHK(to < ctas * kTile, ROBE_DBG_SHARED)) continue;
            const uint32_t at = address_in(&sm.pair[(pass + 1) & 1][to % kTile], to / kTile);
            asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(at), "r"(p.x), "r"(p.y) : "memory");
        }
        cluster_barrier();
    }
    for (uint32_t k = tid; k < kTile && first + k < (uint64_t)a.rows; k += kRankThreads) {
        const uint2 p = sm.pair[passes & 1][k];
        a.keys[first + k] = p.x;
        a.places[first + k] = p.y;
    }
}

// The table alone.
__global__ void __launch_bounds__(kTableThreads) grad_clear_kernel(GradArgs a) {
    follow<true>();
    clear_table(a, (uint64_t)blockIdx.x * kTableThreads + threadIdx.x, (uint64_t)gridDim.x * kTableThreads);
}

// Sums of a chunk's runs, V columns a thread, `lanes` threads a row.  ADD: to what is there, which is asked for together with the
// rows of the run's end.  HOW: kMany CTAs, a wave of them and more, kSome, so that a thread has more rows under way; kAlone: at most
// kAloneRows ids, which each CTA sorts by counting for each how many come before it.
enum SumsHow { kMany, kSome, kAlone };
template <class T, int V, bool ADD, SumsHow HOW>
__global__ void __launch_bounds__(kTableThreads, HOW == kMany ? 4 : 2) grad_sums_kernel(GradArgs a, uint32_t lanes) {
    // rows under way: few where four CTAs are resident (16384 x 4096 bf16, Zipf ids, accumulating, four columns: two rows 82 us, four 70, eight
    // 122; 852 K x 64 fp32: four 144, eight 148, bf16 149, 147; 5000 x 1000 bf16 36.9, 35.5; single elements gain nothing of more)
    constexpr int kMany4 = ADD ? 4 : sizeof(T) == 2 ? 8 : 4;
    constexpr int kAhead = HOW == kMany ? (V == 4 ? kMany4 : ADD ? 2 : 4) : (ADD ? 4 : 8);
    extern __shared__ uint32_t staged[];  // keys, then places, of the CTA's chunks (kAlone: of all)
    follow();
    const uint32_t groups = kTableThreads / lanes;
    const uint64_t block = blockIdx.x / a.slices;
    const uint32_t slice = blockIdx.x - (uint32_t)block * a.slices;
    const uint64_t from = HOW == kAlone ? 0 : block * groups * a.chunk;
    const uint32_t staged_rows = HOW == kAlone ? (uint32_t)kAloneRows : groups * a.chunk;
    if (HOW == kAlone) {
        __shared__ __align__(16) uint32_t ids[kAloneRows];
        constexpr int kIds = (int)kAloneRows / kTableThreads;
        uint32_t mine[kIds], before[kIds];
#pragma unroll
        for (int r = 0; r < kIds; ++r) {
            const uint32_t p = threadIdx.x + r * kTableThreads;
            mine[r] = p < (uint64_t)a.rows ? key_of(a, p) : 0xFFFFFFFFu;  // (behind all others, being the last)
            before[r] = 0;
            ids[p] = mine[r];
        }
        __syncthreads();
        for (uint32_t k = 0; k < (uint32_t)a.rows; k += 4) {
            const uint4 q = *(const uint4*)(ids + k);
#pragma unroll
            for (int r = 0; r < kIds; ++r) {
                const uint32_t p = threadIdx.x + r * kTableThreads, m = mine[r];
                before[r] += (q.x < m || (q.x == m && k < p)) + (q.y < m || (q.y == m && k + 1 < p)) + (q.z < m || (q.z == m && k + 2 < p)) +
                             (q.w < m || (q.w == m && k + 3 < p));
            }
        }
#pragma unroll
        for (int r = 0; r < kIds; ++r) {
            const uint32_t p = threadIdx.x + r * kTableThreads;
            if (p >= (uint64_t)a.rows || !ROBE_CHK(before[r] < (uint64_t)a.rows, ROBE_DBG_SHARED)) continue;
            staged[before[r]] = mine[r];
            staged[staged_rows + before[r]] = p;
            if (blockIdx.x == 0) a.keys[before[r]] = mine[r];  // for the join
        }
    } else {
        for (uint32_t k = threadIdx.x; k < staged_rows; k += kTableThreads)
            if (from + k < (uint64_t)a.rows) {
                staged[k] = a.keys[from + k];
                staged[staged_rows + k] = a.places[from + k];
            }
    }
    __syncthreads();
    const uint32_t group = threadIdx.x / lanes;
    const uint64_t c = block * groups + group;
    const int64_t col = ((int64_t)slice * lanes + threadIdx.x % lanes) * V;
    if (c >= a.chunks || col >= a.d) return;
    const uint64_t begin = c * a.chunk;
    const uint32_t count = (uint32_t)((uint64_t)a.rows - begin < a.chunk ? (uint64_t)a.rows - begin : a.chunk);
    const uint32_t vocab = (uint32_t)a.vocab;
    const uint32_t* keys = staged + (begin - from);
    const uint32_t* places = keys + staged_rows;
    if (keys[0] >= vocab) return;
    const uint32_t* const all = HOW == kAlone ? staged : a.keys;
    bool open = begin > 0 && all[begin - 1] == keys[0];  // the run began in an earlier chunk
    const uint32_t after = begin + count < (uint64_t)a.rows ? all[begin + count] : 0xFFFFFFFFu;
    float sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] = 0.0f;
    // two groups of rows under way: while one is added up, the other is on its way
    constexpr int G = kAhead / 2;
    Elements<T, V> e[2][G];
    Elements<float, V> old[2][ADD ? G : 1];
    uint32_t key[2][G];
    bool ends[2][G];  // its run ends with it
    auto fetch = [&](int half, uint32_t i) {
#pragma unroll
        for (int u = 0; u < G; ++u) {
            key[half][u] = 0xFFFFFFFFu;
            ends[half][u] = false;
            if (i + u >= count || keys[i + u] >= vocab || !ROBE_CHK(places[i + u] < (uint64_t)a.rows && col + V <= a.d, ROBE_DBG_ROW_POS)) continue;
            key[half][u] = keys[i + u];
            e[half][u].template load<true>((const T*)a.grad + (int64_t)places[i + u] * a.grad_ld + col);
            ends[half][u] = (i + u + 1 < count ? keys[i + u + 1] : after) != key[half][u];
            if (ADD && ends[half][u]) old[half][ADD ? u : 0].template load<true>(a.table + (int64_t)key[half][u] * a.table_ld + col);
        }
    };
    fetch(0, 0);
    for (uint32_t i = 0; i < count; i += kAhead) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            fetch(half ^ 1, i + (half + 1) * G);
#pragma unroll
            for (int u = 0; u < G; ++u) {
                const uint32_t k = key[half][u];
                if (k >= vocab) return;  // behind the chunk's end, or without a gradient as all that follow
#pragma unroll
                for (int v = 0; v < V; ++v) sum[v] += e[half][u].get(v);
                if (!ends[half][u] && i + half * G + u + 1 < count) continue;
                if (open || !ends[half][u]) {
                    float* to = a.parts + (c * 2 + (open ? 0 : 1)) * a.parts_ld + col;
#pragma unroll
                    for (int v = 0; v < V; ++v) to[v] = sum[v];
                } else {
                    float w[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) w[v] = ADD ? fmaf(a.scale, sum[v], old[half][ADD ? u : 0].get(v)) : a.scale * sum[v];
                    Elements<float, V> o;
                    o.set(w);
                    o.template store<true>(a.table + (int64_t)k * a.table_ld + col);
                }
                open = false;
#pragma unroll
                for (int v = 0; v < V; ++v) sum[v] = 0.0f;
            }
        }
    }
}

constexpr int kJoinWarps = kTableThreads / 32;
constexpr uint32_t kJoinAlone = 16;       // parts that a warp adds by itself

// Whether the chunks [g kFold, (g + 1) kFold) lie in the run of `key` as a whole, one that began before them.
__device__ __forceinline__ bool folds_in(const GradArgs& a, uint64_t g, uint32_t key) {
    const uint64_t end = (g + 1) * kFold * a.chunk;
    return (g + 1) * kFold <= a.chunks && a.keys[(end < (uint64_t)a.rows ? end : (uint64_t)a.rows) - 1] == key;
}
// Sums of kFold first parts each, a CTA per group.
__global__ void __launch_bounds__(kTableThreads) grad_fold_kernel(GradArgs a) {
    follow();
    const uint64_t g = blockIdx.x;
    if (g == 0) return;
    const uint64_t begin = g * kFold * a.chunk;
    const uint32_t key = a.keys[begin];
    if (key >= (uint32_t)a.vocab || a.keys[begin - 1] != key || !folds_in(a, g, key)) return;
    for (int64_t col = threadIdx.x; col < a.d; col += kTableThreads) {
        double s = 0.0;
#pragma unroll 8
        for (uint32_t k = 0; k < kFold; ++k) s += a.parts[(g * kFold + k) * 2 * a.parts_ld + col];
        a.folds[g * a.parts_ld + col] = s;
    }
}

// Runs that end in a later chunk than they begin in: the chunks' parts in order, in 64 bits.  A warp takes a chunk's last run and
// a slice of columns, as many parts side by side as its lanes hold; runs over many chunks are shared by the CTA's warps.
__global__ void __launch_bounds__(kTableThreads, 4) grad_join_kernel(GradArgs a) {
    __shared__ uint32_t shared_runs[kJoinWarps];  // parts of the runs that the warps share; 0: none
    __shared__ double sums[kJoinWarps][4][32];
    follow();
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t blocks = blockIdx.x / a.slices;  // of kJoinWarps chunks
    const uint32_t slice = blockIdx.x - blocks * a.slices;
    const uint32_t side = 32 / a.lanes, sub = lane / a.lanes;  // parts side by side, the lane's among them
    const int64_t col = (int64_t)slice * (a.lanes * 4) + lane % a.lanes * 4;
    auto key_before = [&](uint64_t e) { return a.keys[(e < (uint64_t)a.rows ? e : (uint64_t)a.rows) - 1]; };
    auto parts_of = [&](uint64_t c) -> uint32_t {  // of the last run of chunk c, 0 where it ends there
        const uint64_t end = (c + 1) * a.chunk;
        if (c >= a.chunks || end >= (uint64_t)a.rows) return 0;
        // it reaches the end of chunk c + k: true up to some k; 32 places at a time, first powers of two, then between
        const uint64_t far = c + (1ull << lane);
        const uint32_t key = a.keys[end - 1], next_key = a.keys[end], old_key = c > 0 ? a.keys[end - a.chunk - 1] : 0xFFFFFFFFu;
        const uint32_t far_key = far < a.chunks ? key_before((far + 1) * a.chunk) : 0xFFFFFFFFu;
        if (key >= (uint32_t)a.vocab || next_key != key || old_key == key) return 0;  // (it began earlier)
        const int first_hits = __popc(__ballot_sync(0xFFFFFFFFu, far_key == key));
        if (first_hits == 0) return 2;  // (it ends in the next chunk)
        uint64_t yes = 1ull << (first_hits - 1), no = 1ull << first_hits;  // it reaches the end of chunk c + yes and not of c + no
        if (no > a.chunks - c) no = a.chunks - c;
        while (no - yes > 1) {
            const uint64_t apart = (no - yes + 31) / 32, k = yes + apart * (lane + 1);
            const uint32_t hits = __popc(__ballot_sync(0xFFFFFFFFu, k < no && key_before((c + k + 1) * a.chunk) == key));
            const uint64_t up = yes + apart * (hits + 1);
            yes += apart * hits;
            if (up < no) no = up;
        }
        // chunks c .. c + yes end in it; it goes on into the next one if there is one and it begins with it
        const uint64_t next = (c + yes + 1) * a.chunk;
        return (uint32_t)(yes + 1 + (next < (uint64_t)a.rows && a.keys[next] == key ? 1 : 0));
    };
    // parts begin, begin + apart, .. before end of the run that begins in chunk c (part 0: its own last one)
    auto add = [&](double (&s)[4], uint64_t c, uint32_t begin, uint32_t end, uint32_t apart) {
        if (col >= a.d) return;
        for (uint32_t k = begin; k < end; k += 4 * apart) {
            float4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (k + u * apart < end) v[u] = __ldca((const float4*)(a.parts + ((c + k + u * apart) * 2 + (k + u * apart == 0 ? 1 : 0)) * a.parts_ld + col));
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (k + u * apart < end) {
                    s[0] += v[u].x;
                    s[1] += v[u].y;
                    s[2] += v[u].z;
                    s[3] += v[u].w;
                }
        }
    };
    auto over_sides = [&](double (&s)[4]) {
        for (uint32_t o = a.lanes; o < 32; o *= 2)
#pragma unroll
            for (int q = 0; q < 4; ++q) s[q] += __shfl_xor_sync(0xFFFFFFFFu, s[q], o);
    };
    auto finish = [&](const double (&s)[4], uint64_t c) {
        if (sub != 0 || col >= a.d) return;
        const uint32_t key = a.keys[(c + 1) * a.chunk - 1];
        if (!ROBE_CHK(key < (uint32_t)a.vocab, ROBE_DBG_ROW_POS)) return;
        float* to = a.table + (int64_t)key * a.table_ld + col;
        if (a.aligned) {
            float4 o = a.accumulate ? *(const float4*)to : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            o.x = a.accumulate ? fmaf(a.scale, (float)s[0], o.x) : a.scale * (float)s[0];
            o.y = a.accumulate ? fmaf(a.scale, (float)s[1], o.y) : a.scale * (float)s[1];
            o.z = a.accumulate ? fmaf(a.scale, (float)s[2], o.z) : a.scale * (float)s[2];
            o.w = a.accumulate ? fmaf(a.scale, (float)s[3], o.w) : a.scale * (float)s[3];
            *(float4*)to = o;
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (col + q < a.d) to[q] = a.accumulate ? fmaf(a.scale, (float)s[q], to[q]) : a.scale * (float)s[q];
        }
    };
    const uint64_t mine = (uint64_t)blocks * kJoinWarps + warp;
    const uint32_t parts = parts_of(mine);
    if (lane == 0) shared_runs[warp] = parts > kJoinAlone ? parts : 0;
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    if (parts > 0 && parts <= kJoinAlone) {
        add(s, mine, sub, parts, side);
        over_sides(s);
        finish(s, mine);
    }
    __syncthreads();
    for (uint32_t w = 0; w < kJoinWarps; ++w) {
        const uint32_t n = shared_runs[w];
        if (n == 0) continue;
        const uint64_t c = (uint64_t)blocks * kJoinWarps + w;
        const uint32_t who = warp * side + sub, all = kJoinWarps * side;
#pragma unroll
        for (int q = 0; q < 4; ++q) s[q] = 0.0;
        uint32_t plain = n;  // parts from the beginning on that are added one by one; then folds, then the rest
        if (a.folds != nullptr) {
            const uint64_t g0 = (c + kFold) / kFold, end = (c + n) / kFold;  // groups behind chunk c, and up to the run's last whole one
            const uint32_t key = a.keys[(c + 1) * a.chunk - 1];
            if (g0 < end) {
                plain = (uint32_t)(g0 * kFold - c);
                // (the last group's last chunk may end with another run; the one behind it cannot be whole)
                const uint64_t g1 = folds_in(a, end - 1, key) ? end : end - 1;
                for (uint64_t g = g0 + who; g < g1; g += all)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (col + q < a.d) s[q] += a.folds[g * a.parts_ld + col + q];
                add(s, c, (uint32_t)(g1 * kFold - c) + who, n, all);
            }
        }
        add(s, c, who, plain, all);
        over_sides(s);
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

template <int ITEMS>
cudaError_t launch_cluster_sort(const GradArgs& a, uint32_t bits, cudaStream_t st) {
    const uint32_t passes = (bits + kClusterBits - 1) / kClusterBits, per = (bits + passes - 1) / passes;
    const uint32_t ctas = a.rows <= kRankThreads ? 1 : kClusterMost;
    const size_t bytes = sizeof(ClusterSmem<ITEMS>);
    const cudaError_t e = with_shared<grad_cluster_sort_kernel<ITEMS>>(bytes);
    if (e != cudaSuccess) return e;
    // the table: as many others as the SMs hold beside the sort
    const unsigned __int128 pieces = (unsigned __int128)a.vocab * (uint64_t)a.d / (kRankThreads * 16) + 1;
    uint64_t others = a.accumulate ? 0 : pieces < 2 * 148 - kClusterMost ? (uint64_t)pieces : 2 * 148 - kClusterMost;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas + (unsigned)((others + ctas - 1) / ctas * ctas));
    cfg.blockDim = dim3(kRankThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, grad_cluster_sort_kernel<ITEMS>, a, ctas, passes, per);
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
    auto launch = [&](auto kernel, uint64_t rows) { launch_next(kernel, (unsigned)grid, kTableThreads, rows * 8, st, a, lanes); };
    const bool add = a.accumulate != 0;
    if (a.rows <= kAloneRows) add ? launch(grad_sums_kernel<T, V, true, kAlone>, kAloneRows) : launch(grad_sums_kernel<T, V, false, kAlone>, kAloneRows);
    else if (grid <= 148 * 2) add ? launch(grad_sums_kernel<T, V, true, kSome>, groups * a.chunk) : launch(grad_sums_kernel<T, V, false, kSome>, groups * a.chunk);
    else add ? launch(grad_sums_kernel<T, V, true, kMany>, groups * a.chunk) : launch(grad_sums_kernel<T, V, false, kMany>, groups * a.chunk);
    return cudaSuccess;
}
// (at most four columns a thread, whose sums are stored in 16 bytes: 16384 x 4096 bf16, uniform ids, accumulating 132 us with eight, 122
// with four, 5000 x 1000 43, 36)
template <class T>
cudaError_t launch_sums(GradArgs& a, int piece, cudaStream_t st) {
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
    // (what is written in 16 bytes a thread: 852 K rows of 64 from bf16 to fp32 in pieces of eight 74 us, of four 58; from fp32 to bf16 in
    // pieces of four 64 us for the 59 of eight, ids by Zipf)
    const int piece = piece_of(os == 4 ? 4 : 8, pb.d, pb.table, pb.table_ld, ts, out, out_ld, os, pb.rows > 1 || pb.vocab > 1 ? 2 : 1);
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

size_t table_grad_workspace_bytes(int64_t rows, int64_t d) { return grad_layout(rows, d).total; }

cudaError_t launch_table_backward(const TableProblem& pb, const void* grad, int64_t grad_ld, int64_t skip, int accumulate, float* grad_table,
                                  int64_t grad_table_ld, void* workspace, cudaStream_t st) {
    if (accumulate && pb.rows == 0) return cudaSuccess;
    const GradLayout L = grad_layout(pb.rows, pb.d);
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
    a.parts = (float*)(ws + L.parts);
    a.parts_ld = L.parts_ld;
    a.chunk = L.chunk;
    a.chunks = L.chunks;
    a.folds = L.chunks >= kFoldFrom ? (double*)(ws + L.folds) : nullptr;
    a.aligned = piece_of(4, pb.d, grad_table, grad_table_ld, 4, grad_table, grad_table_ld, 4, 2) == 4;
    a.flat = (uintptr_t)grad_table % 16 == 0 && (grad_table_ld == pb.d || pb.vocab == 1);
    const int64_t size = pb.dtype == 0 ? 4 : 2;
    // everything that is launched, before anything is
    a.lanes = 1;
    while (a.lanes < 32 && (int64_t)a.lanes * 4 < pb.d) a.lanes *= 2;
    const uint32_t join_slices = (uint32_t)((pb.d + a.lanes * 4 - 1) / (a.lanes * 4));
    const uint64_t join = (L.chunks + kJoinWarps - 1) / kJoinWarps * join_slices;
    if (join >= (1ull << 31)) return kGridTooSmall;
    const int piece = piece_of(4, pb.d, grad, grad_ld, size, grad_table, grad_table_ld, 4, pb.rows > 1 || pb.vocab > 1 ? 2 : 1);
    if (L.chunks * (uint64_t)((pb.d + (int64_t)kTableThreads * piece - 1) / ((int64_t)kTableThreads * piece)) >= (1ull << 31)) return kGridTooSmall;

    uint32_t *keys[2] = {(uint32_t*)(ws + L.keys[0]), (uint32_t*)(ws + L.keys[1])},
             *places[2] = {(uint32_t*)(ws + L.places[0]), (uint32_t*)(ws + L.places[1])};
    a.keys = keys[0];
    a.places = places[0];
    uint32_t bits = 1;
    while (((uint64_t)pb.vocab >> bits) != 0) ++bits;  // (vocab itself is a key)
    if (pb.rows <= kAloneRows) {
        if (!accumulate) launch_next(grad_clear_kernel, 148 * 8, kTableThreads, 0, st, a);
    } else if (pb.rows <= kClusterRows) {
        const cudaError_t e = pb.rows <= kClusterRows / 8   ? launch_cluster_sort<1>(a, bits, st)
                              : pb.rows <= kClusterRows / 4 ? launch_cluster_sort<2>(a, bits, st)
                              : pb.rows <= kClusterRows / 2 ? launch_cluster_sort<4>(a, bits, st)
                                                            : launch_cluster_sort<8>(a, bits, st);
        if (e != cudaSuccess) return e;
    } else {
        launch_next(grad_keys_kernel, 148 * 8, kTableThreads, 0, st, a);
        const int in = launch_sort_pairs(keys, places, (uint64_t)pb.rows, bits, (uint32_t*)(ws + L.counts), (uint32_t*)(ws + L.totals), st);
        a.keys = keys[in];
        a.places = places[in];
    }
    if (pb.rows > 0) {
        const cudaError_t e = pb.dtype == 0 ? launch_sums<float>(a, piece, st) : launch_sums<__nv_bfloat16>(a, piece, st);
        if (e != cudaSuccess) return e;
    }
    if (a.folds != nullptr) launch_next(grad_fold_kernel, (unsigned)(L.chunks / kFold), kTableThreads, 0, st, a);
    a.slices = join_slices;
    if (L.chunks > 1) launch_next(grad_join_kernel, (unsigned)join, kTableThreads, 0, st, a);
    return cudaGetLastError();
}

}  // namespace robe
