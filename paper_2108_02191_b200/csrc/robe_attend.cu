// Attention of one new token of each sequence over a paged cache of keys and values in 8 bits, with the learned position
// bias by buckets.  With s_j = scale q.K_j + bias[bucket(j - pos), h] for the keys j = 0 .. pos of the sequence,
//     out = sum_j exp(s_j) V_j / sum_j exp(s_j).
//
// Bound by memory: 2 (dim + 4) bytes per key and head of the cache, each read once, for 4 dim operations per query head.  A warp
// takes 16 keys at a time, straight from the cache into the registers of the matrix instructions (m16n8k16, fp16 with fp32
// sums): codes of 8 bits are exact in fp16, and since the order of a sum's terms is free, a thread loads 16 consecutive bytes
// of a key and calls them what the instruction wants of it; the transposed values come of one byte permutation per pair of
// keys, which the widening needs anyway.  Keys' scales multiply the scores; values' scales go into the weights:
//     w_j = exp2(x_j - m) sv_j with m the running maximum of x_j + log2(sv_j)  (x_j = s_j log2(e)),
// so that weights are at most 1 and are rounded to fp16 relative to the largest CONTRIBUTION (half a step is 2^-12 of a
// weight down to 2^-14 of the largest, 2^-25 of the largest below: the result is bf16), while the divisor
// sum exp2(x_j - m) stays in fp32.
// The new tokens' queries are taken to fp16 after an exact division by a power of two (of the row's largest element):
// bf16 has fewer fraction bits than fp16, so elements down to 2^-16 of the largest stay exact.
//
// Work is split over the cache's length by what is really there: a first kernel cuts the sequences, whose lengths it reads,
// into spans of equal length (at least kSpanLeast keys, as many spans as CTAs are resident), a second one takes a
// span and a head of the cache per CTA, and a third one joins the spans of a sequence.
#include "robe_codes.cuh"
#include "robe_internal.h"

namespace robe {

namespace {

constexpr int kAttendWarps = 4;
constexpr int kAttendThreads = 32 * kAttendWarps;
constexpr int kTile = 16;                              // keys of a warp's step
constexpr uint32_t kSpanStep = kTile * kAttendWarps;   // spans are multiples of this
constexpr uint32_t kSpanLeast = 4 * kSpanStep;
constexpr int kHeads = 16;                             // query heads of a CTA
constexpr int kPlanThreads = 1024;
constexpr uint32_t kAttendCtas = 148 * 4;              // most CTAs

// What the first kernel leaves: spans before sequence n in first[n], and their length.
struct AttendPlan {
    uint32_t span;
    uint32_t pad[63];
};
struct AttendArgs {
    AttendProblem p;
    uint32_t blocks;       // heads of the cache x blocks of kHeads of their query heads
    uint32_t head_blocks;  // blocks per head of the cache
    uint32_t group;        // query heads per head of the cache
    uint32_t ctas;         // that spans are made for, at most kAttendCtas
    uint64_t page_magic;
    uint32_t positions;    // that the page table has room for
    AttendPlan* plan;
    uint32_t* first;  // [batch + 1]
    float* parts;     // [spans x blocks][kHeads][dim + 2]
};

__device__ __forceinline__ uint32_t length_of(const AttendArgs& a, int64_t n) {
    const int64_t pos = __ldca(a.p.at.starts + n);
    return pos < 0 ? 0 : pos >= (int64_t)a.positions ? a.positions : (uint32_t)pos + 1;
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
    const unsigned long long each = (keys * a.blocks + a.ctas - 1) / a.ctas;
    unsigned long long span = (each + kSpanStep - 1) / kSpanStep * kSpanStep;
    span = span < kSpanLeast ? kSpanLeast : span;
    if (threadIdx.x == 0) a.plan->span = (uint32_t)span;
    for (int64_t base = 0; base < a.p.at.batch; base += kPlanThreads) {
        const int64_t n = base + threadIdx.x;
        const uint32_t v = n < a.p.at.batch ? (uint32_t)((length_of(a, n) + span - 1) / span) : 0;
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

// Bytes of a key that thread t of four loads: 16 of every 64, then a quarter of what is left; word w of them starts at
template <int DIM>
__device__ __forceinline__ constexpr int key_column(int t, int w) {
    return w < DIM / 64 * 4 ? w / 4 * 64 + t * 16 + w % 4 * 4 : DIM / 64 * 64 + t * (DIM % 64 / 4) + (w - DIM / 64 * 4) * 4;
}
template <int DIM>
__device__ __forceinline__ void load_key(uint32_t (&w)[DIM / 16], const uint8_t* p, int t) {
#pragma unroll
    for (int i = 0; i < DIM / 64; ++i) {
        const uint4 q = __ldcs((const uint4*)(p + i * 64 + t * 16));
        w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
    }
#pragma unroll
    for (int k = DIM / 64 * 4; k < DIM / 16; ++k) w[k] = __ldcs((const uint32_t*)(p + key_column<DIM>(t, k)));
}
// .. of a value that thread g of eight loads: 16 of every 128, then an eighth of what is left; column k of them is
template <int DIM>
__device__ __forceinline__ constexpr int value_column(int g, int k) {
    return k < DIM / 128 * 16 ? k / 16 * 128 + g * 16 + k % 16 : DIM / 128 * 128 + g * (DIM % 128 / 8) + (k - DIM / 128 * 16);
}
template <int DIM>
__device__ __forceinline__ void load_value(uint32_t (&w)[DIM / 32], const uint8_t* p, int g) {
#pragma unroll
    for (int i = 0; i < DIM / 128; ++i) {
        const uint4 q = __ldcs((const uint4*)(p + i * 128 + g * 16));
        w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
    }
    if (DIM % 128 == 64) {
        const uint2 q = __ldcs((const uint2*)(p + DIM / 128 * 128 + g * 8));
        w[DIM / 128 * 4] = q.x; w[DIM / 128 * 4 + 1] = q.y;
    } else {
#pragma unroll
        for (int k = DIM / 128 * 4; k < DIM / 32; ++k) w[k] = __ldcs((const uint32_t*)(p + value_column<DIM>(g, k * 4)));
    }
}

// WIDE: more than eight query heads to a CTA.
template <int DIM, bool I8, bool WIDE>
__global__ void __launch_bounds__(kAttendThreads) attend_kernel(AttendArgs a) {
    constexpr int N = WIDE ? 2 : 1;  // blocks of eight query heads
    constexpr float kLog2e = 1.4426950408889634f;
    constexpr float kLeastScale = 7.8886090522101181e-31f;  // 2^-100: keys whose values have no scale count in the divisor too
    __shared__ float joined[kHeads][DIM + 4];
    __shared__ float warp_most[kAttendWarps][kHeads], warp_sum[kAttendWarps][kHeads];
    __shared__ float bias[kBiasMaxSide][kHeads + 1];
    __shared__ int32_t edges[kBiasMaxSide];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, g = lane / 4, t = lane % 4;
    follow();
    const uint32_t span = a.plan->span;
    const uint32_t batch = (uint32_t)a.p.at.batch;
    const uint32_t items = __ldca(a.first + batch) * a.blocks;
    const uint32_t side = a.p.biased ? a.p.bk.side : 0;
    for (uint32_t k = threadIdx.x; k < side; k += kAttendThreads) edges[k] = a.p.bk.edges[k];
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t piece = item / a.blocks, block = item - piece * a.blocks;
        uint32_t n = 0;
        for (uint32_t hi = batch; hi - n > 1;) {  // first[n] <= piece < first[n + 1] (sequences without keys have no piece)
            const uint32_t mid = (n + hi) / 2;
            if (__ldca(a.first + mid) <= piece) n = mid;
            else hi = mid;
        }
        const uint32_t pieces = __ldca(a.first + n + 1) - __ldca(a.first + n);
        const uint32_t split = piece - __ldca(a.first + n);
        const uint32_t length = length_of(a, n);
        const int64_t pos = __ldca(a.p.at.starts + n);
        const uint32_t begin = split * span, end = length - begin < span ? length : begin + span;
        const uint32_t head = block / a.head_blocks;  // of the cache
        const uint32_t q0 = (block - head * a.head_blocks) * kHeads;  // first of its query heads
        const uint32_t in_block = a.group - q0 < (uint32_t)kHeads ? a.group - q0 : (uint32_t)kHeads;
        const int64_t q_row = (int64_t)n * a.p.q_heads + head * a.group + q0;
        for (uint32_t k = threadIdx.x; k < side * kHeads; k += kAttendThreads) {
            const uint32_t b = k / kHeads, h = k % kHeads;
            bias[b][h] = h < in_block ? __ldca(a.p.bias + b * a.p.bias_ld + head * a.group + q0 + h) * kLog2e : 0.0f;
        }
        // queries: rows g and g + 8 of the instruction's first operand
        uint32_t q[N][DIM / 16][2];
        float q_factor[N];
#pragma unroll
        for (int b = 0; b < N; ++b) {
            const uint32_t h = b * 8 + g;
            const bool on = h < in_block;
            const __nv_bfloat16* from = (const __nv_bfloat16*)a.p.q.p + (q_row + h) * a.p.q.ld;
            uint32_t most = 0;
#pragma unroll
            for (int w = 0; w < DIM / 16; ++w)
#pragma unroll
                for (int k = 0; k < 4; ++k) most = max(most, on ? magnitude(widen(from[key_column<DIM>(t, w) + k])) : 0u);
            most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
            most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
            uint32_t e = most >> 23;  // (biased exponent of the largest)
            e = e < 1 ? 1 : e > 253 ? 253 : e;
            const float down = __uint_as_float((254 - e) << 23);
            q_factor[b] = __uint_as_float(e << 23) * a.p.scale * kLog2e;
#pragma unroll
            for (int w = 0; w < DIM / 16; ++w) {
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = on ? widen(from[key_column<DIM>(t, w) + k]) * down : 0.0f;
                q[b][w][0] = half2_of(v[0], v[1]);
                q[b][w][1] = half2_of(v[2], v[3]);
            }
        }
        __syncthreads();
        const float far_bias[2] = {side > 0 ? bias[side - 1][g] : 0.0f, side > 0 && WIDE ? bias[side - 1][8 + g] : 0.0f};

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

        // a step's keys: lanes l and l + 16 know where key l lies
        const int32_t* pages = a.p.at.pages + (int64_t)n * a.p.at.pages_ld;
        auto page_of = [&](uint32_t first_key) -> int32_t {
            const uint32_t j = first_key + (lane & 15);
            if (first_key >= end || j >= end) return -1;
            const uint32_t k = divide(j, a.p.at.page_rows, a.page_magic);
            const int32_t page = __ldca(pages + k);
            return page >= 0 && page < a.p.at.num_pages ? page : -1;
        };
        uint32_t keys[2][DIM / 16], values[4][DIM / 32];
        float scale = 0.0f;
        int64_t at = -1;
        auto locate = [&](int32_t page, uint32_t first_key) {
            const uint32_t j = first_key + (lane & 15);
            const uint32_t k = divide(j, a.p.at.page_rows, a.page_magic);
            const uint32_t row = j - k * a.p.at.page_rows;
            at = page < 0 ? -1 : page * a.p.key_codes.page_ld + (int64_t)row * a.p.key_codes.ld + (int64_t)head * DIM;
            return page < 0 ? -1 : page * a.p.key_scales.page_ld + (int64_t)row * a.p.key_scales.ld + (int64_t)head;
        };
        auto load_keys = [&](int64_t scale_at) {
            scale = scale_at < 0 ? 0.0f : __ldca((const float*)(lane < 16 ? a.p.key_scales.p : a.p.value_scales.p) + scale_at);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int64_t from = __shfl_sync(0xFFFFFFFFu, at, u * 8 + g);
#pragma unroll
                for (int w = 0; w < DIM / 16; ++w) keys[u][w] = 0;
                if (from >= 0) load_key<DIM>(keys[u], (const uint8_t*)a.p.key_codes.p + from, t);
            }
        };
        auto load_values = [&]() {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t from = __shfl_sync(0xFFFFFFFFu, at, 2 * t + (u & 1) + (u & 2) * 4);
#pragma unroll
                for (int w = 0; w < DIM / 32; ++w) values[u][w] = 0;
                if (from >= 0) load_value<DIM>(values[u], (const uint8_t*)a.p.value_codes.p + from, g);
            }
        };
        uint32_t key0 = begin + warp * kTile;
        load_keys(locate(page_of(key0), key0));
        load_values();
        int32_t next_page = page_of(key0 + kSpanStep);
        for (; key0 < end; key0 += kSpanStep) {
            // what this step goes on with, before the next one's takes its place
            const unsigned there = __ballot_sync(0xFFFFFFFFu, at >= 0);
            const float log_scale = log2f(scale < kLeastScale ? kLeastScale : scale);  // (looked at for the values' only)
            float key_scale[4], value_scale[4], value_log[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int key = 2 * t + (u & 1) + (u & 2) * 4;
                key_scale[u] = __shfl_sync(0xFFFFFFFFu, scale, key);
                value_scale[u] = __shfl_sync(0xFFFFFFFFu, scale, key + 16);
                value_log[u] = __shfl_sync(0xFFFFFFFFu, log_scale, key + 16);
            }
            // scores of query heads g (and g + 8) with keys 2 t, 2 t + 1 of either eight
            float s[2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int k = 0; k < 4; ++k) s[u][k] = 0.0f;
#pragma unroll
                for (int w = 0; w < DIM / 16; ++w) {
                    const uint32_t c = signs_turned<I8>(keys[u][w]);
                    multiply(s[u], q[0][w][0], WIDE ? q[N - 1][w][0] : 0u, q[0][w][1], WIDE ? q[N - 1][w][1] : 0u, pair_in_word<I8>(c, 0),
                             pair_in_word<I8>(c, 1));
                }
            }
            const uint32_t next = key0 + kSpanStep;
            const int64_t next_scale = locate(next_page, next);
            load_keys(next_scale);
            next_page = page_of(next + kSpanStep);
            uint32_t weights[N][2];
            float bias_of[N][4];
            const int64_t nearest = pos - (int64_t)(key0 + kTile - 1);  // distance of the step's last key
            const bool far = side == 0 || nearest >= edges[side - 1];
            if (!far) {
                const int64_t d = pos - (int64_t)(key0 + (lane & 15));
                uint32_t b = 0;
                for (uint32_t hi = side; hi - b > 1;) {
                    const uint32_t mid = (b + hi) / 2;
                    if (edges[mid] <= d) b = mid;
                    else hi = mid;
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t bucket = __shfl_sync(0xFFFFFFFFu, b, 2 * t + (u & 1) + (u & 2) * 4);
#pragma unroll
                    for (int x = 0; x < N; ++x) bias_of[x][u] = bias[bucket][x * 8 + g];
                }
            } else {
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int x = 0; x < N; ++x) bias_of[x][u] = far_bias[x];
            }
            bool moved = false;
            float shift[N];
#pragma unroll
            for (int b = 0; b < N; ++b) {
                float x[4], top = -INFINITY;
                bool nan = false;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int key = 2 * t + (u & 1) + (u & 2) * 4;
                    x[u] = there >> key & 1 ? fmaf(s[u / 2][b * 2 + u % 2] * key_scale[u], q_factor[b], bias_of[b][u]) : -INFINITY;
                    const float with = there >> key & 1 ? x[u] + value_log[u] : -INFINITY;
                    nan = nan || with != with;
                    top = fmaxf(top, with);
                }
                if (nan) top = NAN;
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) {
                    const float other = __shfl_xor_sync(0xFFFFFFFFu, top, o);
                    top = top != top || other != other ? NAN : fmaxf(top, other);
                }
                const float old = most[b];
                most[b] = old != old || top != top ? NAN : fmaxf(old, top);
                const float base = most[b] == -INFINITY ? 0.0f : most[b];
                shift[b] = old == -INFINITY ? 0.0f : exp2f(old - base);  // (nothing summed so far: whatever the factor)
                moved = moved || most[b] != old;
                float e[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) e[u] = exp2f(x[u] - base);
                sum[b] = sum[b] * shift[b] + ((e[0] + e[1]) + (e[2] + e[3]));
                weights[b][0] = half2_of(e[0] * value_scale[0], e[1] * value_scale[1]);
                weights[b][1] = half2_of(e[2] * value_scale[2], e[3] * value_scale[3]);
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
            for (int w = 0; w < DIM / 32; ++w) {
                uint32_t c[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) c[u] = signs_turned<I8>(values[u][w]);
#pragma unroll
                for (int k = 0; k < 4; k += 2) {
                    const uint32_t a0 = pair_of_words<I8>(c[0], c[1], k), a1 = pair_of_words<I8>(c[0], c[1], k + 1),
                                   a2 = pair_of_words<I8>(c[2], c[3], k), a3 = pair_of_words<I8>(c[2], c[3], k + 1);
#pragma unroll
                    for (int b = 0; b < N; ++b) multiply(out[b][w * 2 + k / 2], a0, a1, a2, a3, weights[b][0], weights[b][1]);
                }
            }
            load_values();
        }
        // the four warps' parts
#pragma unroll
        for (int b = 0; b < N; ++b) {
            sum[b] += __shfl_xor_sync(0xFFFFFFFFu, sum[b], 1);
            sum[b] += __shfl_xor_sync(0xFFFFFFFFu, sum[b], 2);
            if (t == 0) {
                warp_most[warp][b * 8 + g] = most[b];
                warp_sum[warp][b * 8 + g] = sum[b];
            }
        }
        __syncthreads();
        auto most_of = [&](int h) {
            float m = -INFINITY;
            bool nan = false;
            for (int w = 0; w < kAttendWarps; ++w) {
                nan = nan || warp_most[w][h] != warp_most[w][h];
                m = fmaxf(m, warp_most[w][h]);
            }
            return nan ? NAN : m;
        };
        auto factor_of = [&](int w, int h, float m) { return warp_most[w][h] == -INFINITY ? 0.0f : exp2f(warp_most[w][h] - m); };
        for (int w = 0; w < kAttendWarps; ++w) {
            if (warp == w) {
#pragma unroll
                for (int b = 0; b < N; ++b) {
                    const int h = b * 8 + 2 * t;
                    const float f0 = factor_of(w, h, most_of(h)), f1 = factor_of(w, h + 1, most_of(h + 1));
#pragma unroll
                    for (int m = 0; m < DIM / 16; ++m)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            float* to = &joined[h + (k & 1)][value_column<DIM>(g, 2 * m + k / 2)];
                            const float v = out[b][m][k] * (k & 1 ? f1 : f0);
                            *to = w == 0 ? v : *to + v;
                        }
                }
            }
            __syncthreads();
        }
        for (uint32_t k = threadIdx.x; k < in_block * (DIM / 4); k += kAttendThreads) {
            const uint32_t h = k / (DIM / 4), col = k % (DIM / 4) * 4;
            const float m = most_of(h);
            float total = 0.0f;
            for (int w = 0; w < kAttendWarps; ++w) total += warp_sum[w][h] * factor_of(w, h, m);
            const float4 v = *(const float4*)&joined[h][col];
            if (!ROBE_CHK(n < batch && head * a.group + q0 + h < (uint64_t)a.p.q_heads, ROBE_DBG_ROW_POS)) continue;
            if (pieces == 1) {
                const float by = total == 0.0f ? 0.0f : 1.0f / total;
                __nv_bfloat16* to = (__nv_bfloat16*)a.p.out.p + (q_row + h) * a.p.out.ld + col;
                to[0] = narrow<__nv_bfloat16>(v.x * by);
                to[1] = narrow<__nv_bfloat16>(v.y * by);
                to[2] = narrow<__nv_bfloat16>(v.z * by);
                to[3] = narrow<__nv_bfloat16>(v.w * by);
            } else {
                float* to = a.parts + ((uint64_t)item * kHeads + h) * (DIM + 4);
                *(float4*)(to + col) = v;
                if (col == 0) {
                    to[DIM] = m;
                    to[DIM + 1] = total;
                }
            }
        }
        __syncthreads();  // (the next item's bias and sums take their place)
    }
}

// The spans of a sequence: a CTA per query head, warps taking spans in turn.  Sequences of one span are done already;
// those without keys get +0.
constexpr int kJoinThreads = 256;
template <int DIM>
__global__ void __launch_bounds__(kJoinThreads) attend_join_kernel(AttendArgs a) {
    constexpr int kWarps = kJoinThreads / 32, E = DIM / 32;
    __shared__ float sums[kWarps][DIM], totals[kWarps], mosts[kWarps];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    follow();
    const uint32_t n = blockIdx.x / (uint32_t)a.p.q_heads, h = blockIdx.x - n * (uint32_t)a.p.q_heads;
    const uint32_t first = __ldca(a.first + n), pieces = __ldca(a.first + n + 1) - first;
    __nv_bfloat16* to = (__nv_bfloat16*)a.p.out.p + ((int64_t)n * a.p.q_heads + h) * a.p.out.ld;
    if (pieces == 1) return;
    if (pieces == 0) {
        for (int k = threadIdx.x; k < DIM; k += kJoinThreads) to[k] = narrow<__nv_bfloat16>(0.0f);
        return;
    }
    const uint32_t head = h / a.group, in_group = h - head * a.group;
    const uint32_t block = head * a.head_blocks + in_group / kHeads;
    const float* parts = a.parts + (((uint64_t)first * a.blocks + block) * kHeads + in_group % kHeads) * (DIM + 4);
    const uint64_t step = (uint64_t)a.blocks * kHeads * (DIM + 4);
    float sum[E], total = 0.0f, most = -INFINITY;
#pragma unroll
    for (int k = 0; k < E; ++k) sum[k] = 0.0f;
    bool nan = false;
    for (uint32_t p = warp; p < pieces; p += kWarps) {
        const float* from = parts + p * step;
        const float m = __ldca(from + DIM), l = __ldca(from + DIM + 1);
        float v[E];
#pragma unroll
        for (int k = 0; k < E; ++k) v[k] = __ldca(from + k * 32 + lane);
        nan = nan || m != m;
        if (m == -INFINITY) continue;
        const float up = fmaxf(most, m), f = most == -INFINITY ? 0.0f : exp2f(most - up), e = exp2f(m - up);
#pragma unroll
        for (int k = 0; k < E; ++k) sum[k] = sum[k] * f + v[k] * e;
        total = total * f + l * e;
        most = up;
    }
    if (nan) most = NAN;
#pragma unroll
    for (int k = 0; k < E; ++k) sums[warp][k * 32 + lane] = sum[k];
    if (lane == 0) {
        totals[warp] = total;
        mosts[warp] = most;
    }
    __syncthreads();
    float m = -INFINITY;
    for (int w = 0; w < kWarps; ++w) m = m != m || mosts[w] != mosts[w] ? NAN : fmaxf(m, mosts[w]);
    for (int k = threadIdx.x; k < DIM; k += kJoinThreads) {
        float v = 0.0f, l = 0.0f;
        for (int w = 0; w < kWarps; ++w) {
            const float f = mosts[w] == -INFINITY ? 0.0f : exp2f(mosts[w] - m);
            v += sums[w][k] * f;
            l += totals[w] * f;
        }
        to[k] = narrow<__nv_bfloat16>(l == 0.0f ? 0.0f : v / l);
    }
}

uint32_t head_blocks_of(int64_t heads, int64_t q_heads) { return (uint32_t)((q_heads / heads + kHeads - 1) / kHeads); }

template <int DIM>
cudaError_t launch_attend_dim(AttendArgs& a, cudaStream_t st) {
    auto launch = [&](auto kernel) {
        int resident = 1;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, kernel, kAttendThreads, 0) != cudaSuccess || resident < 1) resident = 1;
        a.ctas = 148u * (unsigned)resident < kAttendCtas ? 148u * (unsigned)resident : kAttendCtas;
        launch_next(attend_plan_kernel, 1, kPlanThreads, 0, st, a);
        launch_next(kernel, a.ctas, kAttendThreads, 0, st, a);
    };
    if (a.group > 8) a.p.i8 ? launch(attend_kernel<DIM, true, true>) : launch(attend_kernel<DIM, false, true>);
    else a.p.i8 ? launch(attend_kernel<DIM, true, false>) : launch(attend_kernel<DIM, false, false>);
    launch_next(attend_join_kernel<DIM>, (unsigned)(a.p.at.batch * a.p.q_heads), kJoinThreads, 0, st, a);
    return cudaGetLastError();
}

// spans are made for at most kAttendCtas items; every sequence may have one more than its share, and no span is shorter than kSpanLeast
uint64_t most_items(int64_t batch, uint32_t blocks, int64_t positions) {
    const unsigned __int128 by_length = (unsigned __int128)batch * ((positions + kSpanLeast - 1) / kSpanLeast) * blocks;
    const unsigned __int128 by_share = (unsigned __int128)kAttendCtas + (unsigned __int128)batch * blocks;
    return (uint64_t)(by_length < by_share ? by_length : by_share);
}

}  // namespace

size_t attend_workspace_bytes(int64_t batch, int64_t heads, int64_t q_heads, int64_t dim, int64_t positions) {
    const size_t first = sizeof(AttendPlan) + (((size_t)batch + 1) * 4 + 255) / 256 * 256;
    return first + most_items(batch, (uint32_t)heads * head_blocks_of(heads, q_heads), positions) * kHeads * (dim + 4) * 4;
}

cudaError_t launch_attend(const AttendProblem& pb, void* workspace, cudaStream_t st) {
    AttendArgs a;
    a.p = pb;
    a.group = (uint32_t)(pb.q_heads / pb.heads);
    a.head_blocks = head_blocks_of(pb.heads, pb.q_heads);
    a.blocks = (uint32_t)pb.heads * a.head_blocks;
    a.page_magic = magic_of(pb.at.page_rows);
    a.positions = (uint32_t)(pb.at.max_pages * pb.at.page_rows);
    a.plan = (AttendPlan*)workspace;
    a.first = (uint32_t*)((char*)workspace + sizeof(AttendPlan));
    a.parts = (float*)((char*)workspace + sizeof(AttendPlan) + (((size_t)pb.at.batch + 1) * 4 + 255) / 256 * 256);
    if ((uint64_t)pb.at.batch * pb.q_heads >= (1ull << 31)) return kGridTooSmall;
    if (most_items(pb.at.batch, a.blocks, a.positions) >= (1ull << 32) - 148 * 16) return kGridTooSmall;
    switch (pb.dim) {
        case 32: return launch_attend_dim<32>(a, st);
        case 64: return launch_attend_dim<64>(a, st);
        case 96: return launch_attend_dim<96>(a, st);
        case 128: return launch_attend_dim<128>(a, st);
        default: return launch_attend_dim<256>(a, st);
    }
}

}  // namespace robe
