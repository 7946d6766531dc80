// Dropout of rows from a counter-based generator: out[r,c] = keep(r,c) ? in[r,c] * scale : 0, the decision a function of
// (seed, offset, r, c) alone (robe_rowops.cuh), so that no mask is stored and the gradient is the same call on the
// output's gradient.
#include "robe_internal.h"
#include "robe_rowops.cuh"

namespace robe {

namespace {

constexpr int kDropThreads = 256;

struct DropArgs {
    const void* in;
    void* out;
    int64_t in_ld, out_ld;
    uint32_t in_step, out_step;  // bytes between rows, where a call's rows are taken by pieces
    uint32_t row0;    // number of the first row
    uint32_t items;   // rows * groups, below 2^31
    uint32_t groups;  // groups of 8 columns in a row
    uint32_t tail;    // columns of the last group
    uint64_t magic;   // floor((2^64 - 1) / groups) + 1
    DropParams drop;
};

// Eight elements by the words of their group.  Products are taken in fp32 and the decision made on them, so that what is
// dropped is +0 whatever it was.
__device__ __forceinline__ void drop_eight(uint4 (&e)[1], const uint4& w, const DropParams& d) {  // bf16
    uint32_t* v = (uint32_t*)e;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float low = widen_low(v[k]) * d.scale, high = widen_high(v[k]) * d.scale;
        v[k] = narrow2(drop_keeps(w, 2 * k, d) ? low : 0.0f, drop_keeps(w, 2 * k + 1, d) ? high : 0.0f);
    }
}
__device__ __forceinline__ void drop_eight(uint4 (&e)[2], const uint4& w, const DropParams& d) {  // fp32
    float* v = (float*)e;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = drop_keeps(w, k, d) ? v[k] * d.scale : 0.0f;
}

// A thread takes groups of eight columns, each decided by one evaluation of the generator (about 57 of the 110 instructions
// of a group): ITEMS of them a CTA's width apart, all loaded before the first is worked on.  With one group a thread too few
// bytes are under way: 852 K rows of 128 bf16 86 us, two 82, four 79 (5.5 TB/s, the read and the write of 436 MB; the plain copy
// of as much takes 67), eight 81.  The rest is the ALU, 58 % busy.
// PIECES: rows are 16-byte aligned and hold whole groups.
template <class T, bool PIECES, int ITEMS>
__global__ void __launch_bounds__(kDropThreads, 6) dropout_kernel(DropArgs a) {
    constexpr int kWords = 8 * sizeof(T) / 16;
    follow();
    const uint64_t offset = drop_offset(a.drop);
    const uint32_t t0 = blockIdx.x * (kDropThreads * ITEMS) + threadIdx.x;
    uint4 e[ITEMS][kWords];
    uint32_t row[ITEMS], group[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t t = t0 + i * kDropThreads;
        // t / groups: the upper half of a product (t < 2^32)
        row[i] = a.groups == 1 ? t : (uint32_t)(((a.magic >> 32) * t + (((a.magic & 0xFFFFFFFFu) * t) >> 32)) >> 32);
        group[i] = t - row[i] * a.groups;
        if (PIECES && t < a.items) {
            const uint4* in = (const uint4*)((const char*)a.in + (uint64_t)row[i] * a.in_step) + group[i] * kWords;
#pragma unroll
            for (int q = 0; q < kWords; ++q) e[i][q] = __ldcs(in + q);
        }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if (t0 + i * kDropThreads >= a.items) return;
        if (!ROBE_CHK(group[i] < a.groups && (uint64_t)row[i] * a.groups + group[i] < a.items, ROBE_DBG_ROW_POS)) return;
        const uint4 w = drop_words(a.row0 + row[i], group[i], offset, a.drop);
        if (PIECES) {
            drop_eight(e[i], w, a.drop);
#pragma unroll
            for (int q = 0; q < kWords; ++q)
                __stcs((uint4*)((char*)a.out + (uint64_t)row[i] * a.out_step) + group[i] * kWords + q, e[i][q]);
        } else {
            const T* in = (const T*)a.in + row[i] * a.in_ld + group[i] * 8ll;
            T* out = (T*)a.out + row[i] * a.out_ld + group[i] * 8ll;
            const int left = group[i] + 1 < a.groups ? 8 : (int)a.tail;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < left) out[k] = narrow<T>(a.drop.none || drop_keeps(w, k, a.drop) ? widen(in[k]) * a.drop.scale : 0.0f);
        }
    }
}

template <class T, bool PIECES>
void launch(const DropArgs& a, cudaStream_t st) {
    constexpr int kItems = PIECES ? (sizeof(T) == 2 ? 4 : 2) : 1;
    // few groups: one a thread, spread over more SMs
    const bool few = a.items < 148u * 4 * kDropThreads * kItems;
    const uint32_t per = kDropThreads * (few ? 1 : kItems);
    launch_next(few ? dropout_kernel<T, PIECES, 1> : dropout_kernel<T, PIECES, kItems>, (a.items + per - 1) / per, kDropThreads, 0,
                st, a);
}

// Rows laid end to end that are no whole pieces: the elements go by in 16-byte pieces all the same.  A CTA first evaluates the
// generator for the groups that its elements are of, once each, and leaves the decisions as a string of bits in the order
// of the elements; a piece then reads its own.  (901 K rows of 105 bf16: 258 us by elements, 131 by pieces.)
constexpr int kFlatItems = 4;
template <class T>
__global__ void __launch_bounds__(kDropThreads) dropout_flat_kernel(DropArgs a, uint64_t elements, uint64_t cols) {
    constexpr int V = kPiece<T>;
    constexpr int kTile = kDropThreads * kFlatItems * V;
    __shared__ uint32_t bits[kTile / 32 + 1];  // (a group may end behind the tile)
    __shared__ uint64_t place[2];
    follow();
    const uint64_t offset = drop_offset(a.drop);
    const uint64_t base = (uint64_t)blockIdx.x * kTile;
    const int count = elements - base < kTile ? (int)(elements - base) : kTile;
    const T* in = (const T*)a.in + base;
    T* out = (T*)a.out + base;
    uint4 e[kFlatItems];
#pragma unroll
    for (int i = 0; i < kFlatItems; ++i) {
        const int at = (i * kDropThreads + threadIdx.x) * V;
        if (at + V <= count) e[i] = __ldcs((const uint4*)(in + at));
    }
    for (int k = threadIdx.x; k < kTile / 32 + 1; k += kDropThreads) bits[k] = 0;
    if (threadIdx.x == 0) {
        place[0] = base / cols;
        place[1] = base - place[0] * cols;
    }
    __syncthreads();
    const uint32_t row0 = (uint32_t)place[0], col0 = (uint32_t)place[1];
    const uint32_t group0 = col0 / 8;
    // groups from (row0, group0) on, until one begins behind the tile
    for (uint32_t t = threadIdx.x;; t += kDropThreads) {
        const uint32_t k = t + group0;
        const uint32_t r = a.groups == 1 ? k : (uint32_t)(((a.magic >> 32) * k + (((a.magic & 0xFFFFFFFFu) * k) >> 32)) >> 32);
        const uint32_t g = k - r * a.groups;
        const int64_t at = (int64_t)((uint64_t)r * cols + g * 8ull) - col0;  // where the group begins in the tile, or before it
        if (at >= count) break;
        const uint4 w = drop_words(row0 + r, g, offset, a.drop);
        uint32_t keep = 0;
#pragma unroll
        for (int c = 0; c < 8; ++c) keep |= drop_keeps(w, c, a.drop) ? 1u << c : 0u;
        if (g + 1 == a.groups) keep &= (1u << a.tail) - 1;
        const uint32_t first = at < 0 ? keep >> -at : keep << (at & 31);
        const int word = at < 0 ? 0 : (int)(at >> 5);
        if (!ROBE_CHK(at > -8 && g < a.groups && word + 1 < kTile / 32 + 1, ROBE_DBG_SHARED)) break;
        if (first != 0) atomicOr(&bits[word], first);
        if (at > 0 && (at & 31) > 24) atomicOr(&bits[word + 1], keep >> (32 - (at & 31)));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kFlatItems; ++i) {
        const int at = (i * kDropThreads + threadIdx.x) * V;
        if (at >= count) return;
        const uint32_t keep = bits[at / 32] >> (at & 31);
        if (at + V <= count) {
            uint32_t* v = (uint32_t*)&e[i];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (sizeof(T) == 2) {
                    const float low = widen_low(v[k]) * a.drop.scale, high = widen_high(v[k]) * a.drop.scale;
                    v[k] = narrow2(keep >> (2 * k) & 1 ? low : 0.0f, keep >> (2 * k + 1) & 1 ? high : 0.0f);
                } else {
                    v[k] = __float_as_uint(keep >> k & 1 ? __uint_as_float(v[k]) * a.drop.scale : 0.0f);
                }
            }
            __stcs((uint4*)(out + at), e[i]);
        } else {
            for (int k = 0; at + k < count; ++k) out[at + k] = narrow<T>(keep >> k & 1 ? widen(in[at + k]) * a.drop.scale : 0.0f);
        }
    }
}

}  // namespace

cudaError_t launch_dropout(const void* in, int64_t in_ld, void* out, int64_t out_ld, int64_t rows, int64_t cols, int dtype,
                           const DropParams& drop, cudaStream_t st) {
    const int64_t size = dtype == 0 ? 4 : 2;
    DropArgs a;
    a.in_ld = in_ld;
    a.out_ld = out_ld;
    a.in_step = (uint32_t)(in_ld * size);
    a.out_step = (uint32_t)(out_ld * size);
    a.groups = (uint32_t)((cols + 7) / 8);
    a.tail = (uint32_t)(cols - (a.groups - 1) * 8ll);
    a.magic = ~0ull / a.groups + 1;
    a.drop = drop;
    const bool pieces = !drop.none && cols % 8 == 0 && (((uintptr_t)in | (uintptr_t)out) & 15u) == 0 &&
                        (rows == 1 || (in_ld * size % 16 == 0 && out_ld * size % 16 == 0 && in_ld < (1ll << 30) && out_ld < (1ll << 30)));
    const bool flat = !pieces && !drop.none && (rows == 1 || (in_ld == cols && out_ld == cols)) && (((uintptr_t)in | (uintptr_t)out) & 15u) == 0;
    if (flat) {
        a.in = in;
        a.out = out;
        const uint64_t elements = (uint64_t)rows * cols;
        const uint64_t tile = (uint64_t)kDropThreads * kFlatItems * (16 / size);
        const uint64_t grid = (elements + tile - 1) / tile;
        if (grid >= (1ull << 31)) return kGridTooSmall;
        if (dtype == 0) launch_next(dropout_flat_kernel<float>, (unsigned)grid, kDropThreads, 0, st, a, elements, (uint64_t)cols);
        else launch_next(dropout_flat_kernel<__nv_bfloat16>, (unsigned)grid, kDropThreads, 0, st, a, elements, (uint64_t)cols);
        return cudaGetLastError();
    }
    // items are numbered in 32 bits: as many rows a launch as that allows
    const int64_t most = ((1ll << 31) - 1) / a.groups;
    for (int64_t r = 0; r < rows; r += most) {
        a.row0 = (uint32_t)r;
        a.items = (uint32_t)((rows - r < most ? rows - r : most) * a.groups);
        a.in = (const char*)in + r * in_ld * size;
        a.out = (char*)out + r * out_ld * size;
        if (dtype == 0) pieces ? launch<float, true>(a, st) : launch<float, false>(a, st);
        else pieces ? launch<__nv_bfloat16, true>(a, st) : launch<__nv_bfloat16, false>(a, st);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace robe
