// Rows in 8 bits: the residual join whose norm leaves as codes with scales, and a paged cache of such rows, written and
// read back.  Formulas of codes and scales: robe_codes.cuh.  All of it moves data once and is bound by memory; the sums and
// largest magnitudes that it takes stay in registers and shuffles.
#include <initializer_list>
#include <type_traits>

#include "robe_codes.cuh"
#include "robe_internal.h"

namespace robe {

namespace {

constexpr int kCodeThreads = 256;
constexpr int kJoinMost = 512;       // threads a row
constexpr int64_t kGroupMost = 256;  // columns of a group that lanes of one warp hold; beyond: one scale a row

// Eight columns of a row, loaded and stored by pieces of P elements; where fewer than eight are left, one by one.
// (as words: kept apart, bf16 elements would take a register each)
template <class T>
struct Eight {
    uint32_t w[2 * sizeof(T)];
    __device__ __forceinline__ float get(int k) const {
        if (sizeof(T) == 4) return __uint_as_float(w[k]);
        return k % 2 ? widen_high(w[k / 2]) : widen_low(w[k / 2]);
    }
};
template <class T, int P>
constexpr int kStep = P * (int)sizeof(T) > 16 ? kPiece<T> : P;
template <class T, int P>
__device__ __forceinline__ void load_eight(Eight<T>& r, const T* p, int count) {
    constexpr int S = kStep<T, P>, B = S * (int)sizeof(T);
    if (count == 8 && B >= 4) {
        using W = typename Word<B >= 4 ? B : 4>::type;
#pragma unroll
        for (int q = 0; q < 8 / S; ++q) {
            union {
                W w;
                uint32_t u[B >= 4 ? B / 4 : 1];
            } e;
            e.w = __ldcs((const W*)(p + q * S));
#pragma unroll
            for (int k = 0; k < B / 4; ++k) r.w[q * (B / 4) + k] = e.u[k];
        }
    } else if (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < 8; ++k) r.w[k] = k < count ? __ldcs((const uint32_t*)p + k) : 0u;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            r.w[k] = 2 * k < count ? __ldcs((const unsigned short*)p + 2 * k) : 0u;
            if (2 * k + 1 < count) r.w[k] |= (uint32_t)__ldcs((const unsigned short*)p + 2 * k + 1) << 16;
        }
    }
}
template <class T, int P>
__device__ __forceinline__ void store_eight(const float (&v)[8], T* p, int count) {
    constexpr int S = kStep<T, P>;
    if (count == 8) {
#pragma unroll
        for (int q = 0; q < 8 / S; ++q) {
            Pack<T, S> e;
#pragma unroll
            for (int k = 0; k < S; ++k) e.v[k] = narrow<T>(v[q * S + k]);
            store_pack<true, T, S>(p + q * S, e);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < count) p[k] = narrow<T>(v[k]);
    }
}
// Eight elements of E bytes to an address that is no multiple of a piece: pieces are of what two lanes have, each lane stores the one that
// ends among its own, and single elements are left at the ends of rows and warps.  The whole warp calls it.  count: of the lane,
// chained: this lane and the one before have eight each that follow one another; given: this lane and the next.
template <int E>
__device__ __forceinline__ void store_chain(uint8_t* p, const uint32_t (&w)[2 * E], int count, bool chained, bool given) {
    constexpr int N = 2 * E, PB = N >= 4 ? 16 : 8, PW = PB / 4;
    const uint32_t off = (uint32_t)(uintptr_t)p & (PB - 1u);
    uint32_t c[PW + N + 1];  // the last piece of the lane before, the lane's own
#pragma unroll
    for (int k = 0; k < PW; ++k) c[k] = __shfl_up_sync(0xFFFFFFFFu, w[N - PW + k], 1);
#pragma unroll
    for (int k = 0; k < N; ++k) c[PW + k] = w[k];
    c[PW + N] = 0;
    // from `PB - off` bytes on; off = 0: the lane's own
    const uint32_t skip = PB - off;
    uint32_t o[PW + N];
    if (PW == 4) {
#pragma unroll
        for (int k = 0; k + 4 < PW + N + 1; ++k) c[k] = skip & 16 ? c[k + 4] : c[k];
#pragma unroll
        for (int k = 0; k + 2 < PW + N + 1; ++k) c[k] = skip & 8 ? c[k + 2] : c[k];
    } else {
#pragma unroll
        for (int k = 0; k + 2 < PW + N + 1; ++k) c[k] = skip & 8 ? c[k + 2] : c[k];
    }
#pragma unroll
    for (int k = 0; k + 1 < PW + N + 1; ++k) c[k] = skip & 4 ? c[k + 1] : c[k];
#pragma unroll
    for (int k = 0; k < N; ++k) o[k] = E == 4 ? c[k] : __funnelshift_r(c[k], c[k + 1], (skip & 3) * 8);
    const bool own = off == 0;
    if (count == 8) {
#pragma unroll
        for (int q = 0; q < N / PW; ++q) {
            if (q == 0 && !own && !chained) continue;
            if (PW == 4) *(uint4*)(p - off + q * 16) = make_uint4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
            else *(uint2*)(p - off) = make_uint2(o[0], o[1]);
        }
    }
    // elements before the first piece of the lane's own, behind its last, or all of a few
    const uint32_t head = own || chained ? 0 : skip, tail = own || given ? 8 * E : 8 * E - off;
    if (count > 0 && (count < 8 ? true : head > 0 || tail < 8 * E)) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < count && (count < 8 || k * E < (int)head || k * E >= (int)tail)) {
                if (E == 4) *(uint32_t*)(p + 4 * k) = w[k];
                else if (E == 2) *(uint16_t*)(p + 2 * k) = (uint16_t)(w[k / 2] >> (16 * (k % 2)));
                else p[k] = (uint8_t)(w[k / 4] >> (8 * (k % 4)));
            }
    }
}
template <class T>
__device__ __forceinline__ void store_chain(const float (&v)[8], T* p, int count, bool chained, bool given) {
    uint32_t w[2 * sizeof(T)];
#pragma unroll
    for (int k = 0; k < 2 * (int)sizeof(T); ++k) {
        if constexpr (sizeof(T) == 4) {
            w[k] = __float_as_uint(v[k]);
        } else {
            Pack<T, 2> e;
            e.v[0] = narrow<T>(v[2 * k]);
            e.v[1] = narrow<T>(v[2 * k + 1]);
            w[k] = *(const uint32_t*)&e;
        }
    }
    store_chain<(int)sizeof(T)>((uint8_t*)p, w, count, chained, given);
}
// eight codes, by pieces of `piece` bytes
__device__ __forceinline__ void store_codes(uint8_t* p, uint32_t low, uint32_t high, int count, int piece) {
    if (count == 8 && piece == 8) {
        *(uint2*)p = make_uint2(low, high);
    } else if (count == 8 && piece == 4) {
        ((uint32_t*)p)[0] = low;
        ((uint32_t*)p)[1] = high;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < count) p[k] = (uint8_t)((k < 4 ? low : high) >> (8 * (k % 4)));
    }
}
template <bool I8>
__device__ __forceinline__ void store_codes(uint8_t* p, const float (&v)[8], float factor, int count, int piece) {
    store_codes(p, codes_of<I8>(v, factor), codes_of<I8>(v + 4, factor), count, piece);
}
__device__ __forceinline__ uint32_t largest_of(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) m = max(m, magnitude(v[k]));
    return m;
}

// ---- where columns lie: a unit is eight columns of one group; `lanes` units (a power of two) hold a group, those behind its end
// nothing.  With one scale a row the units follow one another and the whole row is the group.
struct Columns {
    uint32_t d, group, shift, units;  // shift: of lanes; units: of a row
    int whole;                        // one scale a row
};
// FULL: rows and groups are of whole eights of columns: a unit has eight or none
template <bool FULL = false>
__device__ __forceinline__ uint32_t columns_of(const Columns& c, uint32_t unit, int& count) {
    const uint32_t begin = (unit >> c.shift) * c.group, in = (unit & ((1u << c.shift) - 1u)) * 8, col = begin + in;
    const uint32_t end = begin + c.group < c.d ? begin + c.group : c.d;
    if (FULL) count = in < c.group && col < c.d ? 8 : 0;
    else count = col >= end ? 0 : end - col >= 8 ? 8 : (int)(end - col);
    return col;  // (units behind the row's begin behind its end)
}
Columns columns(int64_t d, int64_t group) {
    Columns c;
    c.d = (uint32_t)d;
    c.whole = group > kGroupMost;
    if (c.whole) group = 8;
    c.group = (uint32_t)group;
    c.shift = 0;
    while ((8ll << c.shift) < group) ++c.shift;
    c.units = (uint32_t)((d + group - 1) / group) << c.shift;
    return c;
}

// rows and groups of whole eights of columns, whose codes are written in one piece
bool full_units(const Columns& c, int code_piece) { return c.d % 8 == 0 && c.group % 8 == 0 && code_piece == 8; }

// ---------------------------------------------------------------- the join

struct QuantizeArgs {
    int64_t rows;
    Columns c;
    int layer;
    float eps, scale, per_column;  // per_column: 1 / d
    const float* w;
    RowsRef x, residual, out, codes, scales;
    int code_piece, w_pieces;
    int chain;  // units follow one another in rows of many (store_chain)
    int i8;
    uint32_t threads;  // of a row
    // a cache takes the codes: rows of the call lie where `at` says
    int cached;
    CachePlaces at;
    int64_t codes_page, scales_page;
};

// where row r's codes and scales go; false: nowhere
__device__ __forceinline__ bool codes_row(const QuantizeArgs& a, int64_t r, uint8_t*& codes, float*& scales) {
    int64_t code = r * a.codes.ld, scale = r * a.scales.ld;
    if (a.cached) {
        const CacheRow at = cache_row(a.at, r);
        if (at.page < 0) return false;
        code = at.page * a.codes_page + at.row * a.codes.ld;
        scale = at.page * a.scales_page + at.row * a.scales.ld;
    }
    codes = (uint8_t*)a.codes.p + code;
    scales = (float*)a.scales.p + scale;
    return true;
}
// eight weights
__device__ __forceinline__ void load_weights(float (&w)[8], const QuantizeArgs& a, int64_t col, int count) {
    if (a.w_pieces && count == 8) {
        const float4 p = __ldca((const float4*)(a.w + col)), q = __ldca((const float4*)(a.w + col) + 1);
        w[0] = p.x; w[1] = p.y; w[2] = p.z; w[3] = p.w;
        w[4] = q.x; w[5] = q.y; w[6] = q.z; w[7] = q.w;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = k < count ? __ldca(a.w + col + k) : 0.0f;
    }
}

__device__ __forceinline__ float add_over(float v, uint32_t lanes) {
#pragma unroll
    for (uint32_t o = 1; o < 32; o <<= 1)
        if (o < lanes) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ __forceinline__ uint32_t most_over(uint32_t v, uint32_t lanes) {
#pragma unroll
    for (uint32_t o = 1; o < 32; o <<= 1)
        if (o < lanes) v = max(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}
// over the threads of a row: lanes of a warp, or whole warps that meet in shared memory (one word a warp)
__device__ __forceinline__ float add_over_row(float v, uint32_t threads, float* words) {
    if (threads <= 32) return add_over(v, threads);
    v = add_over(v, 32);
    const uint32_t warp = threadIdx.x / 32, per = threads / 32, first = warp / per * per;
    if (threadIdx.x % 32 == 0) words[warp] = v;
    __syncthreads();
    v = 0.0f;
    for (uint32_t k = 0; k < per; ++k) v += words[first + k];
    return v;
}
__device__ __forceinline__ uint32_t most_over_row(uint32_t v, uint32_t threads, uint32_t* words) {
    if (threads <= 32) return most_over(v, threads);
    v = most_over(v, 32);
    const uint32_t warp = threadIdx.x / 32, per = threads / 32, first = warp / per * per;
    if (threadIdx.x % 32 == 0) words[warp] = v;
    __syncthreads();
    v = 0;
    for (uint32_t k = 0; k < per; ++k) v = max(v, words[first + k]);
    return v;
}

// A row in the registers of its threads, K units each; two operations in one instruction.  What hides the loads' latency is CTAs, not
// rows asked for ahead.  (16384 x 4096 bf16, groups of 128, 472 MB: 87 us, 91 with the two units in different groups; elements one by one 117, bound by instructions; 252
// with two CTAs an SM that asked for the next row.)
// FULL: as columns_of has it, in 16-byte pieces and codes in eights, RESIDUAL and I8 known; otherwise these are asked for.
template <class T, int P, int K, int THREADS, bool FULL, bool RESIDUAL, bool I8>
__global__ void __launch_bounds__(THREADS, K == 4 ? 1 : THREADS == 256 ? 5 : 2) quantize_rows_kernel(QuantizeArgs a) {
    const bool joined = FULL ? RESIDUAL : a.residual.p != nullptr, i8 = FULL ? I8 : a.i8 != 0;
    __shared__ float sums[2][THREADS / 32];
    __shared__ uint32_t most[THREADS / 32];
    follow();
    uint32_t t = threadIdx.x;
    int64_t r = blockIdx.x;
    if (a.threads != blockDim.x) {  // several rows a CTA
        t = threadIdx.x % a.threads;
        r = (int64_t)blockIdx.x * (blockDim.x / a.threads) + threadIdx.x / a.threads;
    }
    const bool on_row = r < a.rows;
    // two units of a thread are one in each half of a group where it has two: they share its scale
    const bool paired = FULL && K == 2 && a.c.shift > 0;
    const uint32_t half = paired ? 1u << (a.c.shift - 1) : 0;
    Eight<T> x[K], y[K];
    uint32_t col[K];
    int count[K];
    const T* from = (const T*)a.x.p + r * a.x.ld;
    const T* beside = (const T*)a.residual.p + r * a.residual.ld;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        col[j] = columns_of<FULL>(a.c, paired ? t + (t & ~(half - 1u)) + j * half : t + j * a.threads, count[j]);
        if (!on_row || !ROBE_CHK(count[j] == 0 || col[j] + (uint32_t)count[j] <= (uint64_t)a.c.d, ROBE_DBG_ROW_POS)) count[j] = 0;
        if (count[j] > 0) load_eight<T, P>(x[j], from + col[j], FULL ? 8 : count[j]);
        if (joined && count[j] > 0) load_eight<T, P>(y[j], beside + col[j], FULL ? 8 : count[j]);
    }
    bool chained[K], given[K];  // (store_chain)
    if (P == 1) {
        const uint32_t lane = threadIdx.x & 31;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const uint32_t before = __shfl_up_sync(0xFFFFFFFFu, count[j] == 8 ? col[j] + 8 : 0u, 1);
            chained[j] = lane > 0 && t > 0 && count[j] == 8 && before == col[j];
            given[j] = __shfl_down_sync(0xFFFFFFFFu, chained[j], 1) && lane < 31;
        }
    }
    float2 v[K][4];  // (zeros behind the unit's columns)
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[j][k] = both(0.0f);
            if (count[j] > 0) {
                const float2 p = make_float2(x[j].get(2 * k), x[j].get(2 * k + 1));
                v[j][k] = joined ? fma2(both(a.scale), p, make_float2(y[j].get(2 * k), y[j].get(2 * k + 1))) : mul2(both(a.scale), p);
            }
        }
    if (a.out.p != nullptr) {
        T* to = (T*)a.out.p + r * a.out.ld;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            if (P == 1 && a.chain) store_chain<T>((const float(&)[8])v[j], to + col[j], count[j], chained[j], given[j]);
            else if (count[j] > 0) store_eight<T, P>((const float(&)[8])v[j], to + col[j], FULL ? 8 : count[j]);
        }
    }
    if (a.w != nullptr) {
        float2 sum = both(0.0f);
        if (a.layer) {
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) sum = add2(sum, v[j][k]);
            const float mean = add_over_row(sum.x + sum.y, a.threads, sums[0]) * a.per_column;
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    v[j][k].x = (FULL ? 0 : 2 * k) < count[j] ? v[j][k].x - mean : 0.0f;
                    v[j][k].y = (FULL ? 0 : 2 * k + 1) < count[j] ? v[j][k].y - mean : 0.0f;
                }
            sum = both(0.0f);
        }
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum = fma2(v[j][k], v[j][k], sum);
        const float2 factor = both(norm_factor(fmaf(add_over_row(sum.x + sum.y, a.threads, sums[1]), a.per_column, a.eps)));
#pragma unroll
        for (int j = 0; j < K; ++j) {
            if (count[j] == 0) continue;
            float w[8];
            load_weights(w, a, col[j], FULL ? 8 : count[j]);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[j][k] = mul2(mul2(v[j][k], factor), make_float2(w[2 * k], w[2 * k + 1]));
        }
    }
    uint8_t* const codes = (uint8_t*)a.codes.p + r * a.codes.ld;
    float* const scales = (float*)a.scales.p + r * a.scales.ld;
    const float q = i8 ? kLargestI8 : kLargestE4m3;
    auto largest = [&](int j) {
        float m = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) m = most_magnitude(m, v[j][k].x, v[j][k].y);
        return __float_as_uint(m);
    };
    GroupScale whole{};
    if (a.c.whole) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < K; ++j) m = max(m, largest(j));
        whole = group_scale(most_over_row(m, a.threads, most), q);
        if (on_row && t == 0) scales[0] = whole.scale;
    } else if (paired) {
        whole = group_scale(most_over(max(largest(0), largest(K - 1)), half), q);
        if (count[0] > 0 && (t & (half - 1u)) == 0) scales[t >> (a.c.shift - 1)] = whole.scale;
    }
#pragma unroll
    for (int j = 0; j < K; ++j) {
        GroupScale g = whole;
        if (!a.c.whole && !paired) {
            g = group_scale(most_over(largest(j), 1u << a.c.shift), q);
            const uint32_t unit = t + j * a.threads;
            if (count[j] > 0 && (unit & ((1u << a.c.shift) - 1u)) == 0) scales[unit >> a.c.shift] = g.scale;
        }
        if (P > 1 && count[j] == 0) continue;
        float c[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 p = mul2(v[j][k], both(g.factor));
            c[2 * k] = p.x;
            c[2 * k + 1] = p.y;
        }
        uint32_t low, high;
        if (i8) {
            low = codes_i8(c[0], c[1], c[2], c[3]);
            high = codes_i8(c[4], c[5], c[6], c[7]);
        } else {
            low = codes_e4m3(c[0], c[1], c[2], c[3]);
            high = codes_e4m3(c[4], c[5], c[6], c[7]);
        }
        if (FULL) __stcs((uint2*)(codes + col[j]), make_uint2(low, high));
        else if (P > 1 || !a.chain || a.code_piece >= 4) {
            if (count[j] > 0) store_codes(codes + col[j], low, high, count[j], a.code_piece);
        } else {
            const uint32_t words[2] = {low, high};
            store_chain<1>(codes + col[j], words, count[j], chained[j], given[j]);
        }
    }
}

// Rows of any length, a CTA each, read again for every step: statistics, the largest magnitude of a whole row, codes.
template <class T, int P>
__global__ void __launch_bounds__(kJoinMost) quantize_long_kernel(QuantizeArgs a) {
    __shared__ float sums[2][kJoinMost / 32];
    __shared__ uint32_t most[kJoinMost / 32];
    follow();
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        uint8_t* codes = nullptr;
        float* scales = nullptr;
        const bool to = codes_row(a, r, codes, scales);
        if (!to && a.out.p == nullptr) continue;  // (the same for the whole CTA)
        auto joined = [&](float (&v)[8], uint32_t unit, int64_t& col) {
            int count;
            col = columns_of(a.c, unit, count);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 0.0f;
            if (count == 0 || !ROBE_CHK(col + count <= a.c.d, ROBE_DBG_ROW_POS)) return 0;
            Eight<T> x, y;
            load_eight<T, P>(x, (const T*)a.x.p + r * a.x.ld + col, count);
            if (a.residual.p != nullptr) load_eight<T, P>(y, (const T*)a.residual.p + r * a.residual.ld + col, count);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (k < count) v[k] = a.residual.p != nullptr ? fmaf(a.scale, x.get(k), y.get(k)) : a.scale * x.get(k);
            }
            return count;
        };
        float mean = 0.0f, factor = 1.0f;
        if (a.w != nullptr) {
            if (a.layer) {
                float sum = 0.0f, v[8];
                int64_t col;
                for (uint32_t u = threadIdx.x; u < a.c.units; u += kJoinMost) {
                    joined(v, u, col);
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum += v[k];
                }
                mean = add_over_row(sum, kJoinMost, sums[0]) * a.per_column;
            }
            float sum = 0.0f, v[8];
            int64_t col;
            for (uint32_t u = threadIdx.x; u < a.c.units; u += kJoinMost) {
                const int count = joined(v, u, col);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < count) sum = fmaf(v[k] - mean, v[k] - mean, sum);
            }
            factor = norm_factor(fmaf(add_over_row(sum, kJoinMost, sums[1]), a.per_column, a.eps));
        }
        auto normed = [&](float (&n)[8], const float (&v)[8], int64_t col, int count) {
#pragma unroll
            for (int k = 0; k < 8; ++k) n[k] = v[k];
            if (a.w == nullptr || count == 0) return;
            float w[8];
            load_weights(w, a, col, count);
#pragma unroll
            for (int k = 0; k < 8; ++k) n[k] = k < count ? (v[k] - mean) * factor * w[k] : 0.0f;
        };
        GroupScale whole{};
        if (a.c.whole) {
            uint32_t m = 0;
            for (uint32_t u = threadIdx.x; u < a.c.units; u += kJoinMost) {
                float v[8], n[8];
                int64_t col;
                const int count = joined(v, u, col);
                normed(n, v, col, count);
                m = max(m, largest_of(n));
            }
            whole = group_scale(most_over_row(m, kJoinMost, most), a.i8 ? kLargestI8 : kLargestE4m3);
            if (to && threadIdx.x == 0) scales[0] = whole.scale;
        }
        // (out may be the residual itself: every element is read for the last time by the thread that then writes it)
        for (uint32_t u0 = 0; u0 < a.c.units; u0 += kJoinMost) {
            const uint32_t u = u0 + threadIdx.x;
            float v[8], n[8];
            int64_t col;
            const int count = joined(v, u, col);
            normed(n, v, col, count);
            if (a.out.p != nullptr && count > 0) store_eight<T, P>(v, (T*)a.out.p + r * a.out.ld + col, count);
            GroupScale g = whole;
            if (!a.c.whole) {
                g = group_scale(most_over(largest_of(n), 1u << a.c.shift), a.i8 ? kLargestI8 : kLargestE4m3);
                if (to && count > 0 && (u & ((1u << a.c.shift) - 1u)) == 0) scales[u >> a.c.shift] = g.scale;
            }
            if (to && count > 0) {
                if (a.i8) store_codes<true>(codes + col, n, g.factor, count, a.code_piece);
                else store_codes<false>(codes + col, n, g.factor, count, a.code_piece);
            }
        }
        __syncthreads();  // the words of the sums are read until here
    }
}

// elements of a piece that rows, groups and addresses allow
int piece_for(const Columns& c, int most, int64_t size, std::initializer_list<const RowsRef*> all, int64_t rows) {
    for (int v = most; v > 1; v /= 2) {
        bool ok = c.group % v == 0;
        for (const RowsRef* m : all)
            if (m->p != nullptr) ok = ok && (uintptr_t)m->p % (v * size) == 0 && (rows <= 1 || m->ld * size % (v * size) == 0);
        if (ok) return v;
    }
    return 1;
}

template <class T, int P>
cudaError_t launch_quantize(QuantizeArgs& a, bool in_registers, cudaStream_t st) {
    const uint32_t units = a.c.units;
    const int K = units <= 64 ? 1 : units <= 2 * kJoinMost ? 2 : 4;
    uint32_t threads = (units + K - 1) / K;
    if (threads <= 32) {
        uint32_t p = 1;
        while (p < threads) p *= 2;
        threads = p < (1u << a.c.shift) ? 1u << a.c.shift : p;
    } else {
        threads = (threads + 31) / 32 * 32;
    }
    a.threads = threads;
    const uint32_t block = threads >= 128 ? threads : 128 / threads * threads;
    const int64_t per = block / threads;
    const int64_t ctas = (a.rows + per - 1) / per;
    if (!in_registers || units > 4 * kJoinMost || ctas >= (1ll << 31)) {
        const int64_t grid = a.rows < 148 * 8 ? a.rows : 148 * 8;
        launch_next(quantize_long_kernel<T, P>, (unsigned)grid, kJoinMost, 0, st, a);
        return cudaGetLastError();
    }
    auto launch = [&](auto kernel) { launch_next(kernel, (unsigned)ctas, block, 0, st, a); };
    auto sized = [&](auto full, auto residual, auto eight) {
        constexpr bool F = decltype(full)::value, R = decltype(residual)::value, E = decltype(eight)::value;
        if (K == 1) launch(quantize_rows_kernel<T, P, 1, 256, F, R, E>);
        else if (K == 2 && block <= 256) launch(quantize_rows_kernel<T, P, 2, 256, F, R, E>);
        else if (K == 2) launch(quantize_rows_kernel<T, P, 2, 512, F, R, E>);
        else launch(quantize_rows_kernel<T, P, 4, 512, F, R, E>);
    };
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    if constexpr (P == kPiece<T>) {
        if (full_units(a.c, a.code_piece) && (a.w == nullptr || a.w_pieces)) {
            if (a.residual.p != nullptr) a.i8 ? sized(yes, yes, yes) : sized(yes, yes, no);
            else a.i8 ? sized(yes, no, yes) : sized(yes, no, no);
            return cudaGetLastError();
        }
    }
    sized(no, no, no);
    return cudaGetLastError();
}
template <class T>
cudaError_t launch_quantize(QuantizeArgs& a, bool in_registers, cudaStream_t st) {
    constexpr int kMost = kPiece<T>;
    const int piece = piece_for(a.c, kMost, sizeof(T), {&a.x, &a.residual, &a.out}, a.rows);
    if (piece == kMost) return launch_quantize<T, kMost>(a, in_registers, st);
    if (kMost == 8 && piece == 4) return launch_quantize<T, 4>(a, in_registers, st);
    if (piece == 2) return launch_quantize<T, 2>(a, in_registers, st);
    return launch_quantize<T, 1>(a, in_registers, st);
}

// ---------------------------------------------------------------- the cache

struct CacheArgs {
    CacheProblem c;
    Columns cols;
    RowsRef rows;
    int64_t n;
    uint32_t per_cta;  // rows
    uint32_t units;    // of a row: eight columns (write), W columns (read)
    uint64_t magic;    // of units
    uint64_t group_magic;
    int code_piece;
};
struct Place {
    int64_t code, scale;  // of the row's first; code -1: none, -2: of no sequence
};
constexpr int kCacheRows = 256;  // most rows of a CTA

// the places of the CTA's rows: one warp finds the first row's sequence, from which the others are near
__device__ __forceinline__ void find_places(const CacheArgs& a, Place* places, int64_t first, uint32_t rows) {
    if (threadIdx.x < 32) {
        int64_t near = 0;
        if (a.c.at.offsets != nullptr) near = sequence_of_warp(a.c.at, first);
        for (uint32_t k = threadIdx.x; k < rows; k += 32) {
            const CacheRow at = cache_row(a.c.at, first + k, near);
            Place p{at.page, 0};
            if (at.page >= 0) {
                p.code = at.page * a.c.codes.page_ld + at.row * a.c.codes.ld;
                p.scale = at.page * a.c.scales.page_ld + at.row * a.c.scales.ld;
            }
            places[k] = p;
        }
    }
    __syncthreads();
}

// FULL: rows and groups of whole eights of columns, 16-byte pieces, codes in eights: a unit has eight columns or none.
template <class T, int P, bool I8, int ITEMS, bool FULL>
__global__ void __launch_bounds__(kCodeThreads) cache_write_kernel(CacheArgs a) {
    __shared__ Place places[kCacheRows];
    follow();
    const int64_t first = (int64_t)blockIdx.x * a.per_cta;
    const uint32_t rows = a.n - first < a.per_cta ? (uint32_t)(a.n - first) : a.per_cta;
    const uint32_t items = rows * a.units, lanes = 1u << a.cols.shift;
    const T* from = (const T*)a.rows.p + first * a.rows.ld;
    for (uint32_t base = 0; base < items; base += kCodeThreads * ITEMS) {
        Eight<T> e[ITEMS];
        int count[ITEMS];
        uint32_t row[ITEMS], unit[ITEMS], col[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const uint32_t t = base + i * kCodeThreads + threadIdx.x;
            row[i] = divide(t, a.units, a.magic);
            unit[i] = t - row[i] * a.units;
            count[i] = 0;
            if (t < items) col[i] = columns_of<FULL>(a.cols, unit[i], count[i]);
            if (count[i] > 0) load_eight<T, P>(e[i], from + row[i] * a.rows.ld + col[i], FULL ? 8 : count[i]);
        }
        if (base == 0) find_places(a, places, first, rows);  // (while the rows are on their way)
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = count[i] > 0 ? e[i].get(k) : 0.0f;
            float m = 0.0f;
#pragma unroll
            for (int k = 0; k < 4; ++k) m = most_magnitude(m, v[2 * k], v[2 * k + 1]);
            const GroupScale g = group_scale(most_over(__float_as_uint(m), lanes), I8 ? kLargestI8 : kLargestE4m3);
            if (count[i] == 0) continue;
            const Place at = places[row[i]];
            if (at.code < 0) continue;
            if (!ROBE_CHK(col[i] + (uint32_t)count[i] <= (uint64_t)a.cols.d, ROBE_DBG_ROW_POS)) continue;
            if ((unit[i] & (lanes - 1u)) == 0) ((float*)a.c.scales.p)[at.scale + (unit[i] >> a.cols.shift)] = g.scale;
            uint8_t* to = (uint8_t*)a.c.codes.p + at.code + col[i];
            if (FULL) __stcs((uint2*)to, make_uint2(codes_of<I8>(v, g.factor), codes_of<I8>(v + 4, g.factor)));
            else store_codes<I8>(to, v, g.factor, count[i], a.code_piece);
        }
    }
}

// The same where groups have two units and more: a thread has one in each half of its group, so that places, shuffles and the scale are had
// once for sixteen columns.  (33 K rows of 1024 bf16, groups of 128: 27.5 us a unit at a time, 21.8 so, with one or two pairs under way, 25.7 with
// three; 100 K bf16 79 -> 61, fp32 92 -> 79)
template <class T, bool I8, int ITEMS>
__global__ void __launch_bounds__(kCodeThreads) cache_write_pairs_kernel(CacheArgs a) {
    constexpr int P = kPiece<T>;
    __shared__ Place places[kCacheRows];
    follow();
    const int64_t first = (int64_t)blockIdx.x * a.per_cta;
    const uint32_t rows = a.n - first < a.per_cta ? (uint32_t)(a.n - first) : a.per_cta;
    const uint32_t items = rows * a.units, shift = a.cols.shift - 1, lanes = 1u << shift;
    const T* from = (const T*)a.rows.p + first * a.rows.ld;
    for (uint32_t base = 0; base < items; base += kCodeThreads * ITEMS) {
        Eight<T> e[ITEMS][2];
        bool on[ITEMS][2];
        uint32_t row[ITEMS], group[ITEMS], col[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const uint32_t t = base + i * kCodeThreads + threadIdx.x;
            row[i] = divide(t, a.units, a.magic);
            const uint32_t unit = t - row[i] * a.units, in = (unit & (lanes - 1u)) * 8;
            group[i] = unit >> shift;
            col[i] = group[i] * a.cols.group + in;
            const T* const p = from + row[i] * a.rows.ld + col[i];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                on[i][h] = t < items && in + h * lanes * 8 < a.cols.group && col[i] + h * lanes * 8 < a.cols.d;
                if (on[i][h]) load_eight<T, P>(e[i][h], p + h * lanes * 8, 8);
            }
        }
        if (base == 0) find_places(a, places, first, rows);  // (while the rows are on their way)
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            float v[2][8], m = 0.0f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[h][k] = on[i][h] ? e[i][h].get(k) : 0.0f;
#pragma unroll
                for (int k = 0; k < 4; ++k) m = most_magnitude(m, v[h][2 * k], v[h][2 * k + 1]);
            }
            const GroupScale g = group_scale(most_over(__float_as_uint(m), lanes), I8 ? kLargestI8 : kLargestE4m3);
            if (!on[i][0]) continue;  // (its second half is none either)
            const Place at = places[row[i]];
            if (at.code < 0) continue;
            if (!ROBE_CHK(col[i] + 8 + (on[i][1] ? lanes * 8 : 0) <= (uint64_t)a.cols.d, ROBE_DBG_ROW_POS)) continue;
            if ((threadIdx.x & (lanes - 1u)) == 0) ((float*)a.c.scales.p)[at.scale + group[i]] = g.scale;
            uint8_t* const to = (uint8_t*)a.c.codes.p + at.code + col[i];
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (on[i][h]) __stcs((uint2*)(to + h * lanes * 8), make_uint2(codes_of<I8>(v[h], g.factor), codes_of<I8>(v[h] + 4, g.factor)));
        }
    }
}

// W columns a thread: one access of W bytes, W a power of two that divides the group
template <int W>
struct CodeWords {
    uint32_t w[W < 4 ? 1 : W / 4];
    __device__ __forceinline__ void load(const uint8_t* p) {
        if constexpr (W == 8) {
            const uint2 q = __ldcs((const uint2*)p);
            w[0] = q.x; w[1] = q.y;
        } else if constexpr (W == 4) {
            w[0] = __ldcs((const uint32_t*)p);
        } else {
            w[0] = __ldcs(p);
        }
    }
};
template <class T, int W, bool I8, int ITEMS>
__global__ void __launch_bounds__(kCodeThreads) cache_read_kernel(CacheArgs a) {
    __shared__ Place places[kCacheRows];
    follow();
    const int64_t first = (int64_t)blockIdx.x * a.per_cta;
    const uint32_t rows = a.n - first < a.per_cta ? (uint32_t)(a.n - first) : a.per_cta;
    find_places(a, places, first, rows);
    const uint32_t items = rows * a.units;
    for (uint32_t base = 0; base < items; base += kCodeThreads * ITEMS) {
        CodeWords<W> e[ITEMS];
        float scale[ITEMS];
        uint32_t row[ITEMS], col[ITEMS];
        int64_t code[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const uint32_t t = base + i * kCodeThreads + threadIdx.x;
            row[i] = divide(t, a.units, a.magic);
            col[i] = (t - row[i] * a.units) * W;
            code[i] = -2;
            if (t < items) {
                const Place at = places[row[i]];
                code[i] = at.code;
                if (at.code >= 0 && ROBE_CHK(col[i] + W <= (uint64_t)a.c.d, ROBE_DBG_ROW_POS)) {
                    e[i].load((const uint8_t*)a.c.codes.p + at.code + col[i]);
                    scale[i] = __ldca((const float*)a.c.scales.p + at.scale + divide(col[i], (uint32_t)a.c.group, a.group_magic));
                }
            }
        }
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (code[i] == -2) continue;
            float v[W < 4 ? 4 : W];
#pragma unroll
            for (int q = 0; q < (W < 4 ? 1 : W / 4); ++q) values_of<I8>(e[i].w[q], v + 4 * q);
            T* to = (T*)a.rows.p + (first + row[i]) * a.rows.ld + col[i];
            Pack<T, W> o;
#pragma unroll
            for (int k = 0; k < W; ++k) o.v[k] = narrow<T>(code[i] >= 0 ? v[k] * scale[i] : 0.0f);
            store_pack<true, T, W>(to, o);
        }
    }
}

// rows of a CTA: about `items` units a thread, so that finding the rows' places is shared by many, spread over the SMs where there are few (rows of
// 1024 bf16, written four units a thread 27.4 us, eight 26.5, sixteen 26.8; read eight 77, sixteen 75, thirty-two 77)
uint32_t rows_per_cta(int64_t n, uint32_t units, int items) {
    int64_t rows = (int64_t)kCodeThreads * items / units;
    if (rows > n / (148 * 2)) rows = n / (148 * 2);
    return (uint32_t)(rows < 1 ? 1 : rows > kCacheRows ? kCacheRows : rows);
}

template <class T, bool I8>
cudaError_t launch_write(CacheArgs& a, cudaStream_t st) {
    constexpr int kMost = kPiece<T>;
    const int piece = piece_for(a.cols, kMost, sizeof(T), {&a.rows}, a.n);
    const int64_t grid = (a.n + a.per_cta - 1) / a.per_cta;
    if (grid >= (1ll << 31)) return kGridTooSmall;
    auto launch = [&](auto kernel) { launch_next(kernel, (unsigned)grid, kCodeThreads, 0, st, a); };
    const bool full = piece == kMost && full_units(a.cols, a.code_piece);
    const bool few = a.n * a.units < 148ll * 2 * kCodeThreads * 4;
    if (full && few) launch(cache_write_kernel<T, kMost, I8, 1, true>);
    else if (full && a.cols.shift > 0) {
        a.units /= 2;
        a.magic = magic_of(a.units);
        launch(cache_write_pairs_kernel<T, I8, 2>);
    } else if (full) launch(cache_write_kernel<T, kMost, I8, 4, true>);
    else if (piece == kMost) launch(cache_write_kernel<T, kMost, I8, 2, false>);
    else if (kMost == 8 && piece == 4) launch(cache_write_kernel<T, 4, I8, 2, false>);
    else if (piece == 2) launch(cache_write_kernel<T, 2, I8, 2, false>);
    else launch(cache_write_kernel<T, 1, I8, 2, false>);
    return cudaGetLastError();
}

template <class T, bool I8>
cudaError_t launch_read(CacheArgs& a, int width, cudaStream_t st) {
    const int64_t grid = (a.n + a.per_cta - 1) / a.per_cta;
    if (grid >= (1ll << 31)) return kGridTooSmall;
    auto launch = [&](auto kernel) { launch_next(kernel, (unsigned)grid, kCodeThreads, 0, st, a); };
    if constexpr (sizeof(T) == 2) {
        if (width == 8) {
            launch(cache_read_kernel<T, 8, I8, 4>);
            return cudaGetLastError();
        }
    }
    if (width == 4) launch(cache_read_kernel<T, 4, I8, 4>);
    else launch(cache_read_kernel<T, 1, I8, 4>);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_residual_quantize(const QuantizeProblem& pb, int dtype, cudaStream_t st) {
    QuantizeArgs a{};
    a.rows = pb.rows;
    a.c = columns(pb.d, pb.group);
    a.per_column = 1.0f / (float)pb.d;
    a.layer = pb.layer;
    a.eps = pb.eps;
    a.scale = pb.scale;
    a.w = pb.w;
    a.x = pb.x;
    a.residual = pb.residual;
    a.out = pb.out;
    a.codes = pb.codes;
    a.scales = pb.scales;
    a.code_piece = piece_for(a.c, 8, 1, {&a.codes}, pb.rows);
    // (20 M elements bf16 in rows of 257 / 401 / 505 / 961 / 4099, element by element -> chained: 91 -> 106, 75 -> 75, 71 -> 61, 75 -> 61, 91 ->
    // 65 us; fp32 505 / 4099 43 -> 35, 103 -> 73)
    a.chain = a.c.units >= 64 && (a.c.group % 8 == 0 || pb.group == pb.d);
    a.w_pieces = (uintptr_t)pb.w % 16 == 0 && a.c.group % 4 == 0;
    a.i8 = pb.i8;
    return dtype == 0 ? launch_quantize<float>(a, true, st) : launch_quantize<__nv_bfloat16>(a, true, st);
}

cudaError_t launch_cache_write(const CacheProblem& pb, const void* rows, int64_t rows_ld, int64_t n, int dtype, cudaStream_t st) {
    const Columns cols = columns(pb.d, pb.group);
    const RowsRef codes{pb.codes.p, pb.codes.ld}, codes_pages{pb.codes.p, pb.codes.page_ld};
    const int code_piece = piece_for(cols, 8, 1, {&codes, &codes_pages}, 2);
    if (cols.whole) {  // one scale a row, over more columns than a warp holds: as the join does it
        QuantizeArgs a{};
        a.rows = n;
        a.c = cols;
        a.scale = 1.0f;
        a.x = RowsRef{(void*)rows, rows_ld};
        a.codes = codes;
        a.scales = RowsRef{pb.scales.p, pb.scales.ld};
        a.codes_page = pb.codes.page_ld;
        a.scales_page = pb.scales.page_ld;
        a.code_piece = code_piece;
        a.cached = 1;
        a.i8 = pb.i8;
        a.at = pb.at;
        return dtype == 0 ? launch_quantize<float>(a, false, st) : launch_quantize<__nv_bfloat16>(a, false, st);
    }
    CacheArgs a{};
    a.c = pb;
    a.cols = cols;
    a.rows = RowsRef{(void*)rows, rows_ld};
    a.n = n;
    a.units = cols.units;
    a.magic = magic_of(a.units);
    a.code_piece = code_piece;
    a.per_cta = rows_per_cta(n, a.units, 8);
    if (dtype == 0) return pb.i8 ? launch_write<float, true>(a, st) : launch_write<float, false>(a, st);
    return pb.i8 ? launch_write<__nv_bfloat16, true>(a, st) : launch_write<__nv_bfloat16, false>(a, st);
}

cudaError_t launch_cache_read(const CacheProblem& pb, void* rows, int64_t rows_ld, int64_t n, int dtype, cudaStream_t st) {
    const int64_t size = dtype == 0 ? 4 : 2;
    // (what is written in 16 bytes a thread: 133 K rows of 1024 to bf16 by sixteen codes a thread 91 us, eight 75; 100 K to fp32 by
    // eight 108, four 86)
    int width = dtype == 0 ? 4 : 8;
    for (; width > 1; width = width == 4 ? 1 : 4) {
        const int64_t bytes = width * size;
        if (pb.d % width == 0 && pb.group % width == 0 && (uintptr_t)pb.codes.p % width == 0 && pb.codes.ld % width == 0 &&
            pb.codes.page_ld % width == 0 && (uintptr_t)rows % bytes == 0 && (n <= 1 || rows_ld * size % bytes == 0))
            break;
    }
    CacheArgs a{};
    a.c = pb;
    a.rows = RowsRef{rows, rows_ld};
    a.n = n;
    a.units = (uint32_t)(pb.d / width);
    a.magic = magic_of(a.units);
    a.group_magic = magic_of((uint32_t)pb.group);
    a.per_cta = rows_per_cta(n, a.units, 16);
    if (dtype == 0) return pb.i8 ? launch_read<float, true>(a, width, st) : launch_read<float, false>(a, width, st);
    return pb.i8 ? launch_read<__nv_bfloat16, true>(a, width, st) : launch_read<__nv_bfloat16, false>(a, width, st);
}

}  // namespace robe
