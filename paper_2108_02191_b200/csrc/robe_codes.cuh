// Rows in 8 bits: codes with a scale for every group of columns, and where the rows of a paged cache lie.
//
// With m the largest magnitude of a group, Q = 448 (e4m3: sign, four bits of exponent, three of fraction) or 127 (whole
// numbers):  scale = max(m, 2^-90) / Q,  code = round(v * (1 / scale)) to the nearest even.  Each of the three operations is a
// rounded fp32 one, so codes and scales follow from the values bit for bit.  2^-90 keeps the reciprocal finite: a group of
// zeros has codes of zero.  A group with a NaN or an infinity reads back as NaN: its scale is NaN or infinite, and what the
// reciprocal leaves of the others is zero, or NaN.
#pragma once
#include "robe_internal.h"
#include "robe_rowops.cuh"

namespace robe {

struct GroupScale {
    float scale, factor;  // factor: what values are multiplied by
};
// largest: bits of the largest magnitude (as whole numbers magnitudes compare as they do as floats, NaN above all)
__device__ __forceinline__ GroupScale group_scale(uint32_t largest, float q) {
    constexpr uint32_t kSmallest = (127u - 90u) << 23;
    GroupScale g;
    g.scale = __fdiv_rn(__uint_as_float(largest > kSmallest ? largest : kSmallest), q);
    g.factor = __frcp_rn(g.scale);
    return g;
}
// the largest magnitude of three; NaN where one is
__device__ __forceinline__ float most_magnitude(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

constexpr float kLargestE4m3 = 448.0f, kLargestI8 = 127.0f;

// four codes, low byte first (values beyond the largest by a rounding become the largest; NaN: e4m3's NaN, 0 as a whole number)
__device__ __forceinline__ uint32_t codes_e4m3(float a, float b, float c, float d) {
    uint16_t low, high;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(low) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(high) : "f"(d), "f"(c));
    return (uint32_t)low | (uint32_t)high << 16;
}
__device__ __forceinline__ uint32_t codes_i8(float a, float b, float c, float d) {
    int32_t w[4];
    const float v[4] = {a, b, c, d};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        asm("cvt.rni.s32.f32 %0, %1;" : "=r"(w[k]) : "f"(v[k]));
        w[k] &= 0xFF;
    }
    return (uint32_t)(w[0] | w[1] << 8 | w[2] << 16 | w[3] << 24);
}
template <bool I8>
__device__ __forceinline__ uint32_t codes_of(const float* v, float factor) {
    const float a = v[0] * factor, b = v[1] * factor, c = v[2] * factor, d = v[3] * factor;
    return I8 ? codes_i8(a, b, c, d) : codes_e4m3(a, b, c, d);
}

// what four codes stand for, without their scale
template <bool I8>
__device__ __forceinline__ void values_of(uint32_t w, float* v) {
    if (I8) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (float)(int8_t)(w >> (8 * k));
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t h;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(w >> (16 * k))));
            asm("{\n.reg .f16 a, b;\nmov.b32 {a, b}, %2;\ncvt.f32.f16 %0, a;\ncvt.f32.f16 %1, b;\n}" : "=f"(v[2 * k]), "=f"(v[2 * k + 1]) : "r"(h));
        }
    }
}

// ---- a paged cache: where a row lies
struct CachePlaces {
    const int32_t* pages;  // [batch, max_pages], pages_ld apart
    int64_t pages_ld, batch, max_pages;
    int64_t num_pages;
    uint32_t page_rows;
    const int64_t* offsets;  // device [batch + 1] or nullptr: every sequence has `per` rows
    int64_t per;
    const int64_t* starts;  // device [batch] or nullptr (0)
};
struct CacheRow {
    int64_t page;  // -1: the row has no place; -2: it is of no sequence
    uint32_t row;
};
// the row at position `pos` of sequence s
__device__ __forceinline__ CacheRow cache_row_at(const CachePlaces& p, int64_t s, int64_t pos) {
    CacheRow at{-1, 0};
    if (pos < 0) return at;
    const uint64_t k = (uint64_t)pos / p.page_rows;
    if (k >= (uint64_t)p.max_pages) return at;
    const int32_t page = __ldca(p.pages + s * p.pages_ld + k);
    if (page < 0 || page >= p.num_pages) return at;
    at.page = page;
    at.row = (uint32_t)((uint64_t)pos - k * p.page_rows);
    return at;
}
// Sequence of row r of the call (offsets given): the last whose first row is at or before it, 0 where none is.  A warp looks at 32 places
// at a time.
__device__ __forceinline__ int64_t sequence_of_warp(const CachePlaces& p, int64_t r) {
    const int64_t lane = threadIdx.x & 31;
    int64_t lo = 0, hi = p.batch;  // offsets[lo] <= r, or lo is 0; offsets[hi] > r, or hi is batch
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + 31) / 32, at = lo + (lane + 1) * step;
        const int hits = __popc(__ballot_sync(0xFFFFFFFFu, at < hi && __ldca(p.offsets + at) <= r));
        const int64_t up = lo + (hits + 1) * step;
        lo += hits * step;
        if (up < hi) hi = up;
    }
    return lo;
}
// row r of the call; near: a sequence at or before its own (offsets given).  What it most likely needs is asked for together.
__device__ __forceinline__ CacheRow cache_row(const CachePlaces& p, int64_t r, int64_t near = 0) {
    int64_t s, t, start;
    if (p.offsets == nullptr) {
        s = r / p.per;
        t = r - s * p.per;
        start = p.starts != nullptr ? __ldca(p.starts + s) : 0;
    } else {
        if (p.batch == 0) return CacheRow{-2, 0};
        const int64_t first = __ldca(p.offsets), last = __ldca(p.offsets + p.batch), next = __ldca(p.offsets + near + 1);
        int64_t begin = __ldca(p.offsets + near);
        start = p.starts != nullptr ? __ldca(p.starts + near) : 0;
        if (r < first || r >= last) return CacheRow{-2, 0};
        s = near;
        if (next <= r) {
            int64_t lo = near + 1 < p.batch ? near + 1 : near, hi = p.batch;
            for (int64_t step = 1; lo + step < p.batch; step *= 2) {
                if (__ldca(p.offsets + lo + step) > r) {
                    hi = lo + step;
                    break;
                }
                lo += step;
            }
            while (hi - lo > 1) {  // offsets[lo] <= r < offsets[hi]
                const int64_t mid = (lo + hi) / 2;
                if (__ldca(p.offsets + mid) <= r) lo = mid;
                else hi = mid;
            }
            s = lo;
            begin = __ldca(p.offsets + s);
            start = p.starts != nullptr ? __ldca(p.starts + s) : 0;
        }
        t = (int64_t)((uint64_t)r - (uint64_t)begin);
    }
    return cache_row_at(p, s, (int64_t)((uint64_t)start + (uint64_t)t));  // (negative: no place)
}

struct CacheRef {  // codes or scales: rows ld elements apart, pages page_ld; queries: heads and sequences
    void* p;
    int64_t ld, page_ld;
};
struct CacheProblem {
    CachePlaces at;
    CacheRef codes, scales;
    int i8;
    int64_t d, group;  // group <= d
};

// ---- the join whose norm leaves as codes
struct QuantizeProblem {
    int64_t rows, d, group;
    int layer;
    float eps, scale;
    const float* w;  // or nullptr: no norm
    RowsRef x, residual, out, codes, scales;  // residual.p, out.p may be nullptr
    int i8;
};

// ---- attention of one new token over a cache of keys and one of values
struct AttendProblem {
    CachePlaces at;  // starts: where the new tokens stand
    CacheRef key_codes, key_scales, value_codes, value_scales;
    int i8;
    int64_t heads, q_heads, dim;  // heads of the cache, of the queries
    CacheRef q, out;              // bf16
    float scale;
    int biased;
    BiasBuckets bk;
    const float* bias;  // [buckets, q_heads]
    int64_t bias_ld;
};

}  // namespace robe
