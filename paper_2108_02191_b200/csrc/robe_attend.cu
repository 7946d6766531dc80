// Attention of one new token of each sequence over a paged cache of keys and values in 8 bits, with the learned position
// bias by buckets.  With s_j = scale q.K_j + bias[bucket(j - pos), h] for the keys j = 0 .. pos of the sequence,
//     out = sum_j exp(s_j) V_j / sum_j exp(s_j).
//
// Bound by memory: 2 (dim + 4) bytes per key and head of the cache, each read once, for 4 dim operations per query head.  A warp
// works on 32 keys at a time (16 where heads have 256 columns) with m16n8k16 instructions (fp16, fp32 sums): a single token seldom has more query heads to a head
// of the cache than such an instruction has rows, so the tensor cores' larger tiles would stay empty.  (More are taken in blocks of 16, each
// of which copies and widens the keys and values anew: 64 sequences of up to 8191 keys, one head of 128, 16 / 32 / 64 query heads 34 / 54 / 82
// us.)  Codes of 8 bits are exact in
// fp16.  Since the order of a sum's terms is free, a thread reads 16 consecutive bytes of a key and calls them what the instruction
// wants of it, and the transposed values come of one byte permutation per pair of keys, which the widening needs anyway.
// Keys and values are copied ahead to shared memory, each warp for itself, in pieces of 16 bytes that are shuffled so that both
// ways of reading them meet no bank twice.  Keys' scales multiply the scores; values' scales go into the weights:
//     w_j = exp2(x_j - m) sv_j with m the running maximum of x_j + log2(sv_j)  (x_j = s_j log2(e)),
// so that weights are at most 1 and are rounded to fp16 relative to the largest CONTRIBUTION (half a step is at most 2^-11 of a
// weight down to 2^-14 of the largest, 2^-25 of the largest below, where a weight of half a step and less is 0: the result is
// bf16), while the divisor sum exp2(x_j - m) stays in fp32.
// The new tokens' queries are taken to fp16 after an exact division by a power of two (of the row's largest element):
// bf16 has fewer fraction bits than fp16, so elements down to 2^-16 of the largest stay exact.
//
// Work is split over the cache's length by what is really there: the sequences, whose lengths only the device knows, are cut
// into spans of equal length (by every CTA for itself, or by a kernel of its own where they are many), a CTA takes a span and a
// head of the cache in turn, and another kernel joins the spans of a sequence.
#include <initializer_list>

#include "robe_codes.cuh"
#include "robe_internal.h"

namespace robe {

namespace {

constexpr int kAttendWarps = 4;
constexpr int kAttendThreads = 32 * kAttendWarps;
template <int DIM>
constexpr int kTile = DIM > 128 ? 16 : 32;             // keys of a warp's step
constexpr uint32_t kSpanStep = 128;                    // spans are multiples of this, a step of four warps
constexpr uint32_t kSpanLeast = 2 * kSpanStep;
// From kSpanMany keys a CTA on, several spans of about kSpanLong are made for each, so that CTAs end together (64 sequences of up to 8191
// keys, 8 heads of 128: spans of about 512 147 us, 1024 139, 2048 139).
constexpr uint32_t kSpanMany = 1536, kSpanLong = 1024;
constexpr int kHeads = 16;                             // query heads of a CTA
constexpr int kPlanThreads = 1024;
constexpr uint32_t kPlanWarp = 256;                    // sequences of a call that a warp of each CTA plans for itself
constexpr uint32_t kSpansPerCta = 8;                   // most spans that are made for a CTA

// What the first kernel leaves: the spans' length, and spans before sequence n in first[n].
struct AttendPlan {
    uint32_t span;
    uint32_t pad[63];
};
struct AttendArgs {
    AttendProblem p;
    uint32_t blocks;       // heads of the cache x blocks of kHeads of their query heads
    uint32_t head_blocks;  // blocks per head of the cache
    uint32_t group;        // query heads per head of the cache
    uint32_t rows;         // query heads of the largest block
    uint32_t ctas;         // that spans are made for, at most most_ctas
    float share;           // of a CTA in a key of all: blocks / ctas, and a little more
    uint32_t page_magic, page_shift;  // key / page_rows = (key * magic >> 32) >> shift, for pages of more than one row
    uint32_t positions;    // that the page table has room for
    uint32_t code_page, code_ld;    // pieces of 16 bytes
    uint32_t scale_page, scale_ld;  // elements
    AttendPlan* plan;  // nullptr: few sequences, every CTA plans for itself
    uint32_t* first;   // [batch + 1]
    float* parts;     // [spans x blocks][rows][dim + 4]
};

// The spans' length and 2^7 over it, for counting them.  (Divisions by what only the device knows are what a plan would spend its time
// on, so each is one product and a step of correction.)
struct SpanLength {
    uint32_t span;
    float per_step;
};
__device__ __forceinline__ SpanLength span_length(uint32_t span) { return SpanLength{span, __frcp_rn((float)(span / kSpanStep))}; }
// spans of a sequence: one for a sequence without keys, too, whose results are +0
__device__ __forceinline__ uint32_t spans_of(uint32_t length, const SpanLength& s) {
    if (length <= s.span) return 1;
    const uint32_t steps = (length - 1) / kSpanStep, each = s.span / kSpanStep;  // (below 2^24: exact as fp32)
    uint32_t full = (uint32_t)((float)steps * s.per_step);
    const int left = (int)(steps - full * each);
    full = left < 0 ? full - 1 : left >= (int)each ? full + 1 : full;
    return full + 1;
}
// keys of a sequence whose new token stands at pos
__device__ __forceinline__ uint32_t length_at(const AttendArgs& a, int64_t pos) {
    return pos < 0 ? 0 : pos >= (int64_t)a.positions ? a.positions : (uint32_t)pos + 1;
}
__device__ __forceinline__ uint32_t length_of(const AttendArgs& a, int64_t n) {
    return length_at(a, __ldca(a.p.at.starts + n));
}

// Length of the spans for that many keys in all: no less than a CTA's share, or what a share is cut into, which fp32 takes up by 2^-20 of it.
__device__ __forceinline__ uint32_t span_of(const AttendArgs& a, unsigned long long keys) {
    const float share = (float)keys * a.share + 1.0f;
    const float many = share < (float)kSpanMany ? 1.0f : fminf(floorf(share * (1.0f / kSpanLong)), (float)kSpansPerCta);
    const float span = share * __frcp_ru(many) + 1.0f;
    const uint32_t length = span < 2147483648.0f ? (uint32_t)span : 1u << 31;  // (longer than any sequence)
    return length < kSpanLeast ? kSpanLeast : (length + kSpanStep - 1) / kSpanStep * kSpanStep;
}
// The plan of a call of at most kPlanWarp sequences, by the CTA's first warp: first[0 .. batch] and behind them the spans' length; where the
// new tokens stand.  Lane l has the sequences l, l + 32 and so on.
__device__ __forceinline__ void plan_in_cta(const AttendArgs& a, uint32_t* first, int64_t* stands) {
    constexpr uint32_t kEach = kPlanWarp / 32;
    const uint32_t batch = (uint32_t)a.p.at.batch, lane = threadIdx.x;
    uint32_t length[kEach], low = 0, high = 0;
#pragma unroll
    for (uint32_t k = 0; k < kEach; ++k) {
        length[k] = 0;
        if (k * 32 + lane < batch) {
            const int64_t pos = __ldca(a.p.at.starts + k * 32 + lane);
            stands[k * 32 + lane] = pos;
            length[k] = length_at(a, pos);
        }
    }
#pragma unroll
    for (uint32_t k = 0; k < kEach; ++k) {
        low += length[k] & 0xFFFFu;
        high += length[k] >> 16;
    }
    const unsigned long long keys = __reduce_add_sync(0xFFFFFFFFu, low) + ((unsigned long long)__reduce_add_sync(0xFFFFFFFFu, high) << 16);
    const SpanLength s = span_length(span_of(a, keys));
    uint32_t before = 0;
#pragma unroll
    for (uint32_t k = 0; k < kEach; ++k) {
        if (k * 32 >= batch) break;
        const uint32_t spans = k * 32 + lane < batch ? spans_of(length[k], s) : 0;
        uint32_t sum = spans;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t b = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= (uint32_t)o) sum += b;
        }
        if (k * 32 + lane < batch) first[k * 32 + lane + 1] = before + sum;
        before += __shfl_sync(0xFFFFFFFFu, sum, 31);
    }
    if (lane == 0) {
        first[0] = 0;
        first[kPlanWarp + 1] = s.span;
    }
}

__global__ void __launch_bounds__(kPlanThreads) attend_plan_kernel(AttendArgs a) {
    __shared__ unsigned long long keys;
    __shared__ uint32_t warp_sums[kPlanThreads / 32];
    __shared__ uint32_t carry;
    follow();
    if (threadIdx.x == 0) {
        keys = 0;
        carry = 0;
    }
    __syncthreads();
    unsigned long long mine = 0;
    for (int64_t n = threadIdx.x; n < a.p.at.batch; n += kPlanThreads) mine += length_of(a, n);
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xFFFFFFFFu, mine, o);
    if (threadIdx.x % 32 == 0) atomicAdd(&keys, mine);  // (whole numbers: the order does not matter)
    __syncthreads();
    const SpanLength s = span_length(span_of(a, keys));
    if (threadIdx.x == 0) a.plan->span = s.span;
    for (int64_t base = 0; base < a.p.at.batch; base += kPlanThreads) {
        const int64_t n = base + threadIdx.x;
        const uint32_t v = n < a.p.at.batch ? spans_of(length_of(a, n), s) : 0;
        uint32_t sum = v;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t b = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if ((threadIdx.x & 31) >= (uint32_t)o) sum += b;
        }
        if ((threadIdx.x & 31) == 31) warp_sums[threadIdx.x / 32] = sum;
        __syncthreads();
        uint32_t before = carry;
        for (uint32_t w = 0; w < threadIdx.x / 32; ++w) before += warp_sums[w];
        __syncthreads();
        if (n < a.p.at.batch) a.first[n] = before + sum - v;
        if (threadIdx.x == kPlanThreads - 1) carry = before + sum;
        __syncthreads();
    }
    if (threadIdx.x == 0) a.first[a.p.at.batch] = carry;
}

__device__ __forceinline__ uint32_t half2_of(float low, float high) {
    uint32_t w;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(high), "f"(low));
    return w;
}
__device__ __forceinline__ void multiply(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two codes as two fp16 numbers.  Whole numbers: with the sign bit turned over, the byte under fp16's 1024 is 1024 + 128 + v.
template <bool I8>
__device__ __forceinline__ uint32_t widen_pair(uint32_t w) {  // bytes 0 and 1; I8: bytes 0 and 2, sign bits turned over
    uint32_t h;
    if (I8) asm("{\n.reg .b32 t;\nlop3.b32 t, %1, 0x00FF00FF, 0x64006400, 0xEA;\nsub.rn.f16x2 %0, t, %2;\n}" : "=r"(h) : "r"(w), "r"(0x64806480u));
    else asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)w));
    return h;
}
template <bool I8>
__device__ __forceinline__ uint32_t signs_turned(uint32_t w) { return I8 ? w ^ 0x80808080u : w; }
// codes 2 half, 2 half + 1 of a word (signs turned)
template <bool I8>
__device__ __forceinline__ uint32_t pair_in_word(uint32_t w, int half) {
    if (I8) return widen_pair<true>(__byte_perm(w, 0, half ? 0x4342 : 0x4140));
    return widen_pair<false>(half ? w >> 16 : w);
}
// code `k` of each of two words
template <bool I8>
__device__ __forceinline__ uint32_t pair_of_words(uint32_t a, uint32_t b, int k) {
    return widen_pair<I8>(__byte_perm(a, b, I8 ? (k | (4 + k) << 8) | 0 : k | (4 + k) << 4));
}

__device__ __forceinline__ float exp2_of(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float log2_of(float v) {
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float most_nan(float a, float b) {  // NaN where either is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// copies to shared memory; bytes 0: zeros are written and nothing is read
__device__ __forceinline__ void copy_piece(uint32_t to, const void* from, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_word(uint32_t to, const void* from, uint32_t bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}

// Where byte `at` of key `row` of a step lies.  Rows of 64, 128 and 256 bytes: pieces of 16 bytes change places within 128 so
// that eight lanes of either way of reading (two keys x four pieces; four keys, two apart, x two pieces) meet all banks.
template <int DIM>
__device__ __forceinline__ uint32_t place_of(uint32_t row, uint32_t at) {
    constexpr uint32_t kPieces = DIM / 16;
    const uint32_t piece = row * kPieces + at / 16;
    uint32_t turn = 0;
    if (kPieces == 8 || kPieces == 16) turn = (row >> 1 & 3) << 1 ^ (row & 1) << 2;
    else if (kPieces == 4) turn = (row >> 1 & 3) << 1;
    return (piece ^ turn) * 16 + at % 16;
}
// reads of shared memory by its own addresses
__device__ __forceinline__ void read_words(uint32_t* w, uint32_t at, int words) {
    if (words == 4) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
    else if (words == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
    else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at));
}
// The columns of a key that thread t of four has: 16 of every 64, then a quarter of what is left; word w of them starts at
template <int DIM>
__device__ __forceinline__ constexpr int key_column(int t, int w) {
    return w < DIM / 64 * 4 ? w / 4 * 64 + t * 16 + w % 4 * 4 : DIM / 64 * 64 + t * (DIM % 64 / 4) + (w - DIM / 64 * 4) * 4;
}
// .. of a value that thread g of eight has: 16 of every 128, then an eighth of what is left; column k of them is
template <int DIM>
__device__ __forceinline__ constexpr int value_column(int g, int k) {
    return k < DIM / 128 * 16 ? k / 16 * 128 + g * 16 + k % 16 : DIM / 128 * 128 + g * (DIM % 128 / 8) + (k - DIM / 128 * 16);
}
// Reads of a row, and the words that come in one.
template <int DIM>
__device__ __forceinline__ constexpr int key_words(int read) { return read < DIM / 64 ? 4 : 2; }
template <int DIM>
__device__ __forceinline__ constexpr int value_words(int read) { return read < DIM / 128 ? 4 : DIM % 128 == 64 ? 2 : 1; }
template <int DIM>
constexpr int kKeyReads = DIM / 64 + (DIM % 64 ? 1 : 0);
template <int DIM>
constexpr int kValueReads = DIM / 128 + (DIM % 128 == 64 ? 1 : DIM % 128 / 32);

// A warp's steps ahead in shared memory: keys, values, and their scales.
constexpr int kStages = 2;
template <int DIM>
struct AttendStage {
    uint8_t keys[kTile<DIM> * DIM], values[kTile<DIM> * DIM];
    float key_scales[kTile<DIM>], value_scales[kTile<DIM>];
};
template <int DIM>
struct AttendSmem {
    union {
        AttendStage<DIM> stages[kAttendWarps][kStages];
        // after the last step: what a warp has, [kHeads][DIM + 4] in the place of its stages
        float parts[kAttendWarps][kStages * sizeof(AttendStage<DIM>) / 4];
    };
    static_assert(kStages * sizeof(AttendStage<DIM>) >= kHeads * (DIM + 4) * 4, "a warp's part has room in its stages");
    float warp_most[kAttendWarps][kHeads], warp_sum[kAttendWarps][kHeads];
    int32_t edges[kBiasMaxSide];
    int64_t stands[kPlanWarp];
    uint32_t first[kPlanWarp + 2];
    float bias[][kHeads + 1];  // as many rows as a side has buckets
};

// Most CTAs of a call: as many as the SMs' 228 KB of shared memory hold, at most eight an SM.
template <int DIM>
constexpr uint32_t kAttendCtas = 148 * (228 * 1024 / (sizeof(AttendSmem<DIM>) + 1024) < 8 ? 228 * 1024 / (sizeof(AttendSmem<DIM>) + 1024) : 8);
uint32_t most_ctas(int64_t dim) {
    return dim == 32 ? kAttendCtas<32> : dim == 64 ? kAttendCtas<64> : dim == 96 ? kAttendCtas<96> : dim == 128 ? kAttendCtas<128> : kAttendCtas<256>;
}

// WIDE: more than eight query heads to a CTA.
// 64 sequences of up to 8191 keys, 8 heads of 128, e4m3, four query heads each (631 MB): 130 us with the join's 9, 74 % of what a copy
// reaches; DRAM at 80 % while it runs, 11 warps an SM (shared memory, 167 registers) with 750 instructions for a warp's 32 keys. One of
// 65521 keys, 4 heads: 21 us. A call of one key: 4.2 us.  The next item's first keys asked for before this one's sum is joined: no
// faster (three CTAs an SM cover for one another).
template <int DIM, bool I8, bool WIDE>
__global__ void __launch_bounds__(kAttendThreads) attend_kernel(AttendArgs a) {
    constexpr int N = WIDE ? 2 : 1;  // blocks of eight query heads
    constexpr int T = kTile<DIM>, S = kStages;
    constexpr uint32_t kStep = T * kAttendWarps;
    constexpr float kLog2e = 1.4426950408889634f;
    constexpr float kMostFinite = 3.4028234663852886e38f;
    constexpr float kLeastScale = 7.8886090522101181e-31f;  // 2^-100: keys whose values have no scale count in the divisor too
    extern __shared__ __align__(128) uint8_t memory[];
    AttendSmem<DIM>& sm = *(AttendSmem<DIM>*)memory;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, g = lane / 4, t = lane % 4;
    follow();
    const uint32_t batch = (uint32_t)a.p.at.batch, side = a.p.biased ? a.p.bk.side : 0;
    for (uint32_t k = threadIdx.x; k < side; k += kAttendThreads) sm.edges[k] = a.p.bk.edges[k];
    if (a.plan == nullptr) {
        if (warp == 0) plan_in_cta(a, sm.first, sm.stands);
        __syncthreads();
    }
    const uint32_t* const firsts = a.plan == nullptr ? sm.first : a.first;
    const uint32_t span = a.plan == nullptr ? sm.first[kPlanWarp + 1] : a.plan->span;
    const uint32_t items = firsts[batch] * a.blocks;
    if (a.plan == nullptr && blockIdx.x == 0)
        for (uint32_t k = threadIdx.x; k <= batch; k += kAttendThreads) a.first[k] = sm.first[k];  // for the join
    // where a lane copies to and reads from, in a stage
    constexpr bool kPlain = 32 % (DIM / 16) == 0;  // (a lane's pieces are the same piece of different rows)
    const uint32_t stages = (uint32_t)__cvta_generic_to_shared(sm.stages[warp]);
    const uint8_t* const key_codes = (const uint8_t*)a.p.key_codes.p + (kPlain ? lane % (DIM / 16) * 16 : 0);
    const uint8_t* const value_codes = (const uint8_t*)a.p.value_codes.p + (kPlain ? lane % (DIM / 16) * 16 : 0);
    uint32_t copy_at[T * DIM / 512], key_at[kKeyReads<DIM>], value_at[2][kValueReads<DIM>];
#pragma unroll
    for (int i = 0; i < T * DIM / 512; ++i) copy_at[i] = place_of<DIM>((lane + 32 * i) / (DIM / 16), (lane + 32 * i) % (DIM / 16) * 16);
    // (rows eight apart are turned alike: their distance is 8 DIM)
#pragma unroll
    for (int i = 0; i < kKeyReads<DIM>; ++i) key_at[i] = place_of<DIM>(g, key_column<DIM>(t, 4 * i));
#pragma unroll
    for (int i = 0; i < kValueReads<DIM>; ++i) {
        const int column = i <= DIM / 128 ? value_column<DIM>(g, 16 * i) : value_column<DIM>(g, DIM / 128 * 16 + (i - DIM / 128) * 4);
        value_at[0][i] = T * DIM + place_of<DIM>(2 * t, column);
        value_at[1][i] = T * DIM + place_of<DIM>(2 * t + 1, column);
    }
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t piece = item / a.blocks, block = item - piece * a.blocks;
        uint32_t n = 0;
        for (uint32_t hi = batch; hi - n > 1;) {  // first[n] <= piece < first[n + 1]
            const uint32_t mid = (n + hi) / 2;
            if (firsts[mid] <= piece) n = mid;
            else hi = mid;
        }
        const uint32_t pieces = firsts[n + 1] - firsts[n];
        const uint32_t split = piece - firsts[n];
        const int64_t pos = a.plan == nullptr ? sm.stands[n] : __ldca(a.p.at.starts + n);
        const uint32_t length = length_at(a, pos);
        const uint32_t begin = split * span, end = length - begin < span ? length : begin + span;
        const uint32_t head = block / a.head_blocks;  // of the cache
        const uint32_t q0 = (block - head * a.head_blocks) * kHeads;  // first of its query heads
        const uint32_t in_block = a.group - q0 < (uint32_t)kHeads ? a.group - q0 : (uint32_t)kHeads;
        const uint32_t q_head = head * a.group + q0;

        // a step's copies: lane l knows where key l lies (of 16: l + 16 too)
        const int32_t* pages = a.p.at.pages + (int64_t)n * a.p.at.pages_ld;
        uint32_t next_row = 0;  // of its page: the key whose page was asked for last
        auto page_of = [&](uint32_t first_key) -> int32_t {
            const uint32_t j = first_key + lane % T;
            const uint32_t k = a.p.at.page_rows == 1 ? j : __umulhi(j, a.page_magic) >> a.page_shift;
            next_row = j - k * a.p.at.page_rows;
            return j < end ? __ldca(pages + k) : -1;
        };
        const uint32_t head_code = head * (DIM / 16);
        auto copy_step = [&](int32_t page, uint32_t stage) -> unsigned {  // keys that have a place
            const bool there = page >= 0 && page < a.p.at.num_pages;
            const unsigned mask = __ballot_sync(0xFFFFFFFFu, there);
            const uint32_t at = there ? page * a.code_page + (next_row * a.code_ld + head_code) : 0;
            const uint32_t scale_at = there ? page * a.scale_page + (next_row * a.scale_ld + head) : 0;
            const uint32_t to = stages + stage * (uint32_t)sizeof(AttendStage<DIM>);
#pragma unroll
            for (int i = 0; i < T * DIM / 512; ++i) {
                const uint32_t r = (lane + 32 * i) / (DIM / 16);
                const uint32_t from = __shfl_sync(0xFFFFFFFFu, at, r) + (kPlain ? 0 : (lane + 32 * i) % (DIM / 16));
                const uint32_t bytes = (mask >> r & 1) * 16;
                copy_piece(to + copy_at[i], key_codes + (uint64_t)from * 16, bytes);
                copy_piece(to + copy_at[i] + T * DIM, value_codes + (uint64_t)from * 16, bytes);
            }
            const uint32_t scales = to + 2 * T * DIM + lane * 4, bytes = there ? 4 : 0;
            copy_word(scales, (const float*)(T == 32 || lane < 16 ? a.p.key_scales.p : a.p.value_scales.p) + scale_at, bytes);
            if (T == 32) copy_word(scales + 128, (const float*)a.p.value_scales.p + scale_at, bytes);
            return mask;
        };
        uint32_t key0 = begin + warp * T;
        unsigned there[S - 1];
        int32_t next_page = page_of(key0);
#pragma unroll
        for (int k = 0; k < S - 1; ++k) {
            there[k] = copy_step(next_page, k);
            copies_close();
            next_page = page_of(key0 + (k + 1) * kStep);
        }

        for (uint32_t k = threadIdx.x; k < side * kHeads; k += kAttendThreads) {
            const uint32_t b = k / kHeads, h = k % kHeads;
            const float v = h < in_block ? __ldca(a.p.bias + b * a.p.bias_ld + head * a.group + q0 + h) : 0.0f;
            // (what is finite stays finite: where all keys have the type's lowest value they count alike, where all have -inf none does)
            sm.bias[b][h] = fabsf(v) < INFINITY ? fminf(fmaxf(v * kLog2e, -kMostFinite), kMostFinite) : v;
        }
        // queries: rows g and g + 8 of the instruction's first operand
        const bool q_pieces = ((uintptr_t)a.p.q.p | (uint64_t)a.p.q.ld * 2 | (uint64_t)a.p.q.page_ld * 2) % 8 == 0;
        uint32_t q[N][DIM / 16][2];
        float q_factor[N];
#pragma unroll
        for (int b = 0; b < N; ++b) {
            const uint32_t h = b * 8 + g;
            const bool on = h < in_block;
            const __nv_bfloat16* from = (const __nv_bfloat16*)a.p.q.p + n * a.p.q.page_ld + (q_head + h) * a.p.q.ld;
            uint32_t most = 0;
#pragma unroll
            for (int w = 0; w < DIM / 16; ++w) {
                const __nv_bfloat16* four = from + key_column<DIM>(t, w);
                uint2 v = make_uint2(0, 0);
                if (on && q_pieces) {
                    v = __ldca((const uint2*)four);
                } else if (on) {
                    const unsigned short* one = (const unsigned short*)four;
                    v = make_uint2(__ldca(one) | (uint32_t)__ldca(one + 1) << 16, __ldca(one + 2) | (uint32_t)__ldca(one + 3) << 16);
                }
                q[b][w][0] = v.x;  // (bf16 as it was)
                q[b][w][1] = v.y;
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    most = max(most, max(magnitude(widen_low(q[b][w][k])), magnitude(widen_high(q[b][w][k]))));
            }
            most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
            most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
            uint32_t e = most >> 23;  // (biased exponent of the largest)
            e = e < 1 ? 1 : e > 253 ? 253 : e;
            const float down = __uint_as_float((254 - e) << 23);
            q_factor[b] = __uint_as_float(e << 23) * a.p.scale * kLog2e;
#pragma unroll
            for (int w = 0; w < DIM / 16; ++w)
#pragma unroll
                for (int k = 0; k < 2; ++k) q[b][w][k] = half2_of(widen_low(q[b][w][k]) * down, widen_high(q[b][w][k]) * down);
        }
        __syncthreads();
        const float far_bias[2] = {side > 0 ? sm.bias[side - 1][g] : 0.0f, side > 0 && WIDE ? sm.bias[side - 1][8 + g] : 0.0f};
        // steps that begin before this key lie in the last bucket as a whole
        const int64_t far_end = side == 0 ? (int64_t)end : pos - (T - 1) - sm.edges[side > 0 ? side - 1 : 0] + 1;
        const uint32_t far_until = far_end < 0 ? 0 : far_end < (int64_t)end ? (uint32_t)far_end : end;

        float sum[N], most[N], out[N][DIM / 16][4];
#pragma unroll
        for (int b = 0; b < N; ++b) {
            sum[b] = 0.0f;
            most[b] = -INFINITY;
#pragma unroll
            for (int m = 0; m < DIM / 16; ++m)
#pragma unroll
                for (int k = 0; k < 4; ++k) out[b][m][k] = 0.0f;
        }
        uint32_t stage = 0, free_stage = S - 1;
        for (; key0 < end; key0 += kStep) {
            copies_wait(S - 2);
            __syncwarp();  // every lane's copies of this step are there, every lane has read the step before
            const unsigned here = there[0];
#pragma unroll
            for (int k = 0; k + 1 < S - 1; ++k) there[k] = there[k + 1];
            there[S - 2] = copy_step(next_page, free_stage);
            copies_close();
            next_page = page_of(key0 + S * kStep);
            const uint32_t from = stages + stage * (uint32_t)sizeof(AttendStage<DIM>);
            free_stage = stage;
            stage = stage + 1 < S ? stage + 1 : 0;
            // scores of query heads g (and g + 8) with keys 2 t, 2 t + 1 of each eight
            float s[T / 8][4];
#pragma unroll
            for (int u = 0; u < T / 8; ++u) {
                uint32_t key[DIM / 16];
#pragma unroll
                for (int i = 0; i < kKeyReads<DIM>; ++i) read_words(key + 4 * i, from + key_at[i] + u * 8 * DIM, key_words<DIM>(i));
#pragma unroll
                for (int k = 0; k < 4; ++k) s[u][k] = 0.0f;
#pragma unroll
                for (int w = 0; w < DIM / 16; ++w) {
                    const uint32_t c = signs_turned<I8>(key[w]);
                    multiply(s[u], q[0][w][0], WIDE ? q[N - 1][w][0] : 0u, q[0][w][1], WIDE ? q[N - 1][w][1] : 0u, pair_in_word<I8>(c, 0),
                             pair_in_word<I8>(c, 1));
                }
            }
            // the last bucket's bias, or none yet (a bias may be infinite: what is added cannot be taken away again)
            const bool far = key0 < far_until;
            float first_bias[N];
#pragma unroll
            for (int b = 0; b < N; ++b) first_bias[b] = far ? far_bias[b] : 0.0f;
            float value_scale[T / 8][2], value_log[T / 8][2];
#pragma unroll
            for (int u = 0; u < T / 8; ++u) {
                uint32_t k2[2], v2[2];
                read_words(k2, from + 2 * T * DIM + (8 * u + 2 * t) * 4, 2);
                read_words(v2, from + 2 * T * DIM + T * 4 + (8 * u + 2 * t) * 4, 2);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const bool in = here >> (8 * u + 2 * t + k) & 1;
                    value_scale[u][k] = __uint_as_float(v2[k]);
                    // (a scale that is no number has to come through: the comparison leaves it alone)
                    value_log[u][k] = in ? log2_of(value_scale[u][k] < kLeastScale ? kLeastScale : value_scale[u][k]) : -INFINITY;
#pragma unroll
                    for (int b = 0; b < N; ++b) {
                        float& x = s[u][2 * b + k];
                        x = in ? x * __uint_as_float(k2[k]) * q_factor[b] + first_bias[b] : -INFINITY;
                    }
                }
            }
            if (!far) {
                const int64_t d = pos - (int64_t)(key0 + lane % T);
                uint32_t bucket = 0;
                for (uint32_t hi = side; hi - bucket > 1;) {
                    const uint32_t mid = (bucket + hi) / 2;
                    if (sm.edges[mid] <= d) bucket = mid;
                    else hi = mid;
                }
#pragma unroll
                for (int u = 0; u < T / 8; ++u)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t of = __shfl_sync(0xFFFFFFFFu, bucket, 8 * u + 2 * t + k);
                        if (!(here >> (8 * u + 2 * t + k) & 1)) continue;
#pragma unroll
                        for (int b = 0; b < N; ++b) s[u][2 * b + k] += sm.bias[of][b * 8 + g];
                    }
            }
            uint32_t weights[N][T / 8];
            float shift[N];
            bool moved = false;
#pragma unroll
            for (int b = 0; b < N; ++b) {
                float top = -INFINITY;
#pragma unroll
                for (int u = 0; u < T / 8; ++u)
#pragma unroll
                    for (int k = 0; k < 2; ++k) top = most_nan(top, s[u][2 * b + k] + value_log[u][k]);
                top = most_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = most_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                const float old = most[b];
                most[b] = most_nan(old, top);
                moved = moved || most[b] != old;
                const float base = most[b] == -INFINITY ? 0.0f : most[b];
                shift[b] = exp2_of(old - base);
                float added = 0.0f;
#pragma unroll
                for (int u = 0; u < T / 8; ++u) {
                    const float e0 = exp2_of(s[u][2 * b] - base), e1 = exp2_of(s[u][2 * b + 1] - base);
                    added += e0 + e1;
                    weights[b][u] = half2_of(e0 * value_scale[u][0], e1 * value_scale[u][1]);
                }
                sum[b] = sum[b] * shift[b] + added;
            }
            if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
                for (int b = 0; b < N; ++b) {
                    const float f0 = __shfl_sync(0xFFFFFFFFu, shift[b], 8 * t), f1 = __shfl_sync(0xFFFFFFFFu, shift[b], 8 * t + 4);
#pragma unroll
                    for (int m = 0; m < DIM / 16; ++m) {
                        out[b][m][0] *= f0;
                        out[b][m][1] *= f1;
                        out[b][m][2] *= f0;
                        out[b][m][3] *= f1;
                    }
                }
            }
#pragma unroll
            for (int half = 0; half < T / 16; ++half) {
                uint32_t value[4][DIM / 32];  // of keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int i = 0; i < kValueReads<DIM>; ++i)
                        read_words(value[u] + (i <= DIM / 128 ? 4 * i : DIM / 128 * 4 + i - DIM / 128),
                                   from + value_at[u & 1][i] + (half * 16 + (u & 2) * 4) * DIM, value_words<DIM>(i));
#pragma unroll
                for (int w = 0; w < DIM / 32; ++w) {
                    uint32_t c[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) c[u] = signs_turned<I8>(value[u][w]);
#pragma unroll
                    for (int k = 0; k < 4; k += 2) {
                        const uint32_t a0 = pair_of_words<I8>(c[0], c[1], k), a1 = pair_of_words<I8>(c[0], c[1], k + 1),
                                       a2 = pair_of_words<I8>(c[2], c[3], k), a3 = pair_of_words<I8>(c[2], c[3], k + 1);
#pragma unroll
                        for (int b = 0; b < N; ++b)
                            multiply(out[b][w * 2 + k / 2], a0, a1, a2, a3, weights[b][2 * half], weights[b][2 * half + 1]);
                    }
                }
            }
        }
        copies_wait(0);
        // the four warps' parts
#pragma unroll
        for (int b = 0; b < N; ++b) {
            sum[b] += __shfl_xor_sync(0xFFFFFFFFu, sum[b], 1);
            sum[b] += __shfl_xor_sync(0xFFFFFFFFu, sum[b], 2);
            if (t == 0) {
                sm.warp_most[warp][b * 8 + g] = most[b];
                sm.warp_sum[warp][b * 8 + g] = sum[b];
            }
        }
        __syncthreads();
        auto most_of = [&](int h) {
            float m = sm.warp_most[0][h];
            for (int w = 1; w < kAttendWarps; ++w) m = most_nan(m, sm.warp_most[w][h]);
            return m;
        };
        auto factor_of = [&](int w, int h, float m) { return sm.warp_most[w][h] == -INFINITY ? 0.0f : exp2_of(sm.warp_most[w][h] - m); };
        // (this warp's own stages: nobody else reads or writes them)
#pragma unroll
        for (int b = 0; b < N; ++b) {
            const int h = b * 8 + 2 * t;
            const float f0 = factor_of(warp, h, most_of(h)), f1 = factor_of(warp, h + 1, most_of(h + 1));
#pragma unroll
            for (int m = 0; m < DIM / 16; ++m)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    sm.parts[warp][(h + (k & 1)) * (DIM + 4) + value_column<DIM>(g, 2 * m + k / 2)] = out[b][m][k] * (k & 1 ? f1 : f0);
        }
        __syncthreads();
        for (uint32_t k = threadIdx.x; k < in_block * (DIM / 4); k += kAttendThreads) {
            const uint32_t h = k / (DIM / 4), col = k % (DIM / 4) * 4;
            const float m = most_of(h);
            float total = 0.0f;
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < kAttendWarps; ++w) {
                total += sm.warp_sum[w][h] * factor_of(w, h, m);
                const float4 p = *(const float4*)&sm.parts[w][h * (DIM + 4) + col];
                v.x += p.x;
                v.y += p.y;
                v.z += p.z;
                v.w += p.w;
            }
            if (!ROBE_CHK(n < batch && head * a.group + q0 + h < (uint64_t)a.p.q_heads, ROBE_DBG_ROW_POS)) continue;
            if (pieces == 1) {
                const float by = total == 0.0f ? 0.0f : 1.0f / total;
                __nv_bfloat16* to = (__nv_bfloat16*)a.p.out.p + n * a.p.out.page_ld + (q_head + h) * a.p.out.ld + col;
                to[0] = narrow<__nv_bfloat16>(v.x * by);
                to[1] = narrow<__nv_bfloat16>(v.y * by);
                to[2] = narrow<__nv_bfloat16>(v.z * by);
                to[3] = narrow<__nv_bfloat16>(v.w * by);
            } else {
                float* to = a.parts + ((uint64_t)item * a.rows + h) * (DIM + 4);
                *(float4*)(to + col) = v;
                if (col == 0) {
                    to[DIM] = m;
                    to[DIM + 1] = total;
                }
            }
        }
        __syncthreads();  // (the next item's bias, sums and stages take their place)
    }
}

// The spans of a sequence: the warps of a query head take them in turn, eight under way at a time; a CTA has `each` query heads.
// Sequences of one span are done already.
constexpr int kSpanThreads = 256;
constexpr uint32_t kSpanWarps = kSpanThreads / 32;
template <int DIM>
__global__ void __launch_bounds__(kSpanThreads) attend_join_kernel(AttendArgs a, uint32_t each) {
    constexpr int E = DIM / 32, kAhead = DIM > 128 ? 4 : 8;
    __shared__ float sums[kSpanWarps][DIM], totals[kSpanWarps], mosts[kSpanWarps];
    const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, q_heads = (uint32_t)a.p.q_heads;
    const uint32_t per = kSpanWarps / each, sub = warp % per;  // warps of a query head
    const uint32_t ctas = (q_heads + each - 1) / each, n = blockIdx.x / ctas, h = (blockIdx.x - n * ctas) * each + warp / per;
    follow();
    const uint32_t first = __ldca(a.first + n), pieces = __ldca(a.first + n + 1) - first;
    if (pieces == 1) return;
    float sum[E], total = 0.0f, most = -INFINITY;
#pragma unroll
    for (int k = 0; k < E; ++k) sum[k] = 0.0f;
    if (h < q_heads) {
        const uint32_t head = h / a.group, in_group = h - head * a.group;
        const uint32_t block = head * a.head_blocks + in_group / kHeads;
        const float* parts = a.parts + (((uint64_t)first * a.blocks + block) * a.rows + in_group % kHeads) * (DIM + 4);
        const uint64_t step = (uint64_t)a.blocks * a.rows * (DIM + 4);
        for (uint32_t p = sub; p < pieces; p += per * kAhead) {
            float m[kAhead], l[kAhead], v[kAhead][E], top = most;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                m[u] = -INFINITY;
                if (p + u * per < pieces) {
                    const float* from = parts + (p + u * per) * step;
                    m[u] = __ldca(from + DIM);
                    l[u] = __ldca(from + DIM + 1);
#pragma unroll
                    for (int k = 0; k < E; ++k) v[u][k] = __ldca(from + k * 32 + lane);
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) top = most_nan(top, m[u]);
            const float base = top == -INFINITY ? 0.0f : top, f = exp2_of(most - base);
            total *= f;
#pragma unroll
            for (int k = 0; k < E; ++k) sum[k] *= f;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (p + u * per >= pieces) break;
                const float e = exp2_of(m[u] - base);
                total = fmaf(l[u], e, total);
#pragma unroll
                for (int k = 0; k < E; ++k) sum[k] = fmaf(v[u][k], e, sum[k]);
            }
            most = top;
        }
    }
#pragma unroll
    for (int k = 0; k < E; ++k) sums[warp][k * 32 + lane] = sum[k];
    if (lane == 0) {
        totals[warp] = total;
        mosts[warp] = most;
    }
    __syncthreads();
    for (uint32_t k = threadIdx.x; k < each * DIM; k += kSpanThreads) {
        const uint32_t of = k / DIM, col = k % DIM, w0 = of * per, head = (blockIdx.x - n * ctas) * each + of;
        if (head >= q_heads) break;
        float m = mosts[w0], v = 0.0f, l = 0.0f;
        for (uint32_t w = 1; w < per; ++w) m = most_nan(m, mosts[w0 + w]);
        const float base = m == -INFINITY ? 0.0f : m;
        for (uint32_t w = 0; w < per; ++w) {
            const float f = exp2_of(mosts[w0 + w] - base);
            v = fmaf(sums[w0 + w][col], f, v);
            l = fmaf(totals[w0 + w], f, l);
        }
        ((__nv_bfloat16*)a.p.out.p)[n * a.p.out.page_ld + head * a.p.out.ld + col] = narrow<__nv_bfloat16>(l == 0.0f ? 0.0f : v / l);
    }
}

uint32_t head_blocks_of(int64_t heads, int64_t q_heads) { return (uint32_t)((q_heads / heads + kHeads - 1) / kHeads); }

template <auto KERNEL>
struct Kernel {
    static constexpr auto value = KERNEL;
};
template <int DIM>
cudaError_t launch_attend_dim(AttendArgs& a, cudaStream_t st) {
    const size_t bytes = sizeof(AttendSmem<DIM>) + (a.p.biased ? a.p.bk.side : 0) * (kHeads + 1) * sizeof(float);
    constexpr size_t kMostBytes = sizeof(AttendSmem<DIM>) + kBiasMaxSide * (kHeads + 1) * sizeof(float);
    cudaError_t e = cudaSuccess;
    auto launch = [&](auto of) {
        constexpr auto kernel = decltype(of)::value;
        unsigned resident = 1;
        e = with_shared<kernel>(kMostBytes);
        if (e == cudaSuccess) e = resident_ctas<kernel>(kAttendThreads, bytes, resident);
        if (e != cudaSuccess) return;
        a.ctas = 148u * resident < kAttendCtas<DIM> ? 148u * resident : kAttendCtas<DIM>;
        a.share = (float)((double)a.blocks / a.ctas * (1.0 + 1.0 / (1 << 20)));
        if (a.plan != nullptr) launch_next(attend_plan_kernel, 1, kPlanThreads, 0, st, a);
        launch_next(kernel, a.ctas, kAttendThreads, bytes, st, a);
    };
    if (a.group > 8) a.p.i8 ? launch(Kernel<attend_kernel<DIM, true, true>>{}) : launch(Kernel<attend_kernel<DIM, false, true>>{});
    else a.p.i8 ? launch(Kernel<attend_kernel<DIM, true, false>>{}) : launch(Kernel<attend_kernel<DIM, false, false>>{});
    if (e != cudaSuccess) return e;
    if (a.positions > kSpanLeast) {  // (a sequence within one span is done)
        // few query heads: a CTA each, so that its warps share the spans; many: a warp each
        const uint32_t q_heads = (uint32_t)a.p.q_heads, each = (uint64_t)a.p.at.batch * q_heads < 148 * 4 ? 1 : kSpanWarps;
        launch_next(attend_join_kernel<DIM>, (unsigned)(a.p.at.batch * ((q_heads + each - 1) / each)), kSpanThreads, 0, st, a, each);
    }
    return cudaGetLastError();
}

// a sequence has at most one span more than its share of those that are made for the CTAs, and no span is shorter than kSpanLeast
uint64_t most_items(int64_t batch, uint32_t blocks, int64_t positions, int64_t dim) {
    const unsigned __int128 by_length = (unsigned __int128)batch * (positions > 0 ? (positions + kSpanLeast - 1) / kSpanLeast : 1) * blocks;
    const unsigned __int128 by_share = (unsigned __int128)most_ctas(dim) * kSpansPerCta + (unsigned __int128)batch * blocks;
    return (uint64_t)(by_length < by_share ? by_length : by_share);
}
uint32_t rows_of(int64_t heads, int64_t q_heads) { return q_heads / heads < kHeads ? (uint32_t)(q_heads / heads) : (uint32_t)kHeads; }
size_t plan_bytes(int64_t batch) { return sizeof(AttendPlan) + (((size_t)batch + 1) * 4 + 255) / 256 * 256; }

}  // namespace

size_t attend_workspace_bytes(int64_t batch, int64_t heads, int64_t q_heads, int64_t dim, int64_t positions) {
    return plan_bytes(batch) +
           most_items(batch, (uint32_t)heads * head_blocks_of(heads, q_heads), positions, dim) * rows_of(heads, q_heads) * (dim + 4) * 4;
}

cudaError_t launch_attend(const AttendProblem& pb, void* workspace, cudaStream_t st) {
    AttendArgs a;
    a.p = pb;
    if (pb.at.num_pages == 0)  // (copies of nothing name a place all the same)
        for (CacheRef* c : {&a.p.key_codes, &a.p.key_scales, &a.p.value_codes, &a.p.value_scales}) c->p = workspace;
    a.group = (uint32_t)(pb.q_heads / pb.heads);
    a.head_blocks = head_blocks_of(pb.heads, pb.q_heads);
    a.blocks = (uint32_t)pb.heads * a.head_blocks;
    a.rows = rows_of(pb.heads, pb.q_heads);
    // positions below 2^31: the quotient is exact with magic = floor(2^(31 + l) / page_rows) + 1, l = ceil(log2(page_rows))
    uint32_t l = 0;
    while ((1ull << l) < pb.at.page_rows) ++l;
    a.page_magic = pb.at.page_rows > 1 ? (uint32_t)((1ull << (31 + l)) / pb.at.page_rows + 1) : 0;
    a.page_shift = l > 0 ? l - 1 : 0;
    a.positions = (uint32_t)(pb.at.max_pages * pb.at.page_rows);
    // places are numbered in 32 bits: pieces of 16 bytes, scales
    const uint64_t pages = (uint64_t)(pb.at.num_pages > 0 ? pb.at.num_pages - 1 : 0), rows = pb.at.page_rows - 1;
    const unsigned __int128 last = (unsigned __int128)pages * pb.key_codes.page_ld + rows * (uint64_t)pb.key_codes.ld + pb.heads * pb.dim;
    const unsigned __int128 last_scale = (unsigned __int128)pages * pb.key_scales.page_ld + rows * (uint64_t)pb.key_scales.ld + pb.heads;
    if (last / 16 >= (1ull << 32) - 1 || last_scale >= (1ull << 32)) return kGridTooSmall;
    a.code_page = (uint32_t)(pb.key_codes.page_ld / 16);
    a.code_ld = (uint32_t)(pb.key_codes.ld / 16);
    a.scale_page = (uint32_t)pb.key_scales.page_ld;
    a.scale_ld = (uint32_t)pb.key_scales.ld;
    a.plan = pb.at.batch > kPlanWarp ? (AttendPlan*)workspace : nullptr;
    a.first = (uint32_t*)((char*)workspace + sizeof(AttendPlan));
    a.parts = (float*)((char*)workspace + plan_bytes(pb.at.batch));
    if (most_items(pb.at.batch, a.blocks, a.positions, pb.dim) >= (1ull << 32) - most_ctas(pb.dim)) return kGridTooSmall;
    switch (pb.dim) {
        case 32: return launch_attend_dim<32>(a, st);
        case 64: return launch_attend_dim<64>(a, st);
        case 96: return launch_attend_dim<96>(a, st);
        case 128: return launch_attend_dim<128>(a, st);
        default: return launch_attend_dim<256>(a, st);
    }
}

}  // namespace robe
