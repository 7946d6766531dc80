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
    int64_t in_ld, out_ld, cols;
    uint64_t items;   // rows * groups
    uint64_t groups;  // groups of 8 columns in a row
    uint64_t magic;   // floor((2^64 - 1) / groups) + 1
    DropParams drop;
};

// One thread per group of eight columns: one evaluation of the generator decides all of them.
template <class T, bool ALIGNED>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(DropArgs a) {
    follow();
    const uint64_t offset = drop_offset(a.drop);
    const uint64_t t = (uint64_t)blockIdx.x * kDropThreads + threadIdx.x;
    if (t >= a.items) return;
    const uint64_t r = a.groups == 1 ? t : (t >> 32) == 0 ? __umul64hi(a.magic, t) : t / a.groups;
    const uint64_t g = t - r * a.groups;
    const T* in = (const T*)a.in + r * a.in_ld + g * 8;
    T* out = (T*)a.out + r * a.out_ld + g * 8;
    const int64_t left = a.cols - (int64_t)g * 8;
    const uint4 w = drop_words((uint32_t)r, (uint32_t)g, offset, a.drop.seed);
    if (ALIGNED && left >= 8) {
        constexpr int V = kPiece<T>;
#pragma unroll
        for (int q = 0; q < 8 / V; ++q) {
            Pack<T, V> e = load_pack<true, T, V>(in + q * V);
#pragma unroll
            for (int k = 0; k < V; ++k)
                e.v[k] = drop_keeps(w, q * V + k, a.drop.threshold) ? narrow<T>(widen(e.v[k]) * a.drop.scale) : narrow<T>(0.0f);
            store_pack<true, T, V>(out + q * V, e);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < left)
                out[k] = drop_keeps(w, k, a.drop.threshold) ? narrow<T>(widen(in[k]) * a.drop.scale) : narrow<T>(0.0f);
    }
}

}  // namespace

cudaError_t launch_dropout(const void* in, int64_t in_ld, void* out, int64_t out_ld, int64_t rows, int64_t cols, int dtype,
                           const DropParams& drop, cudaStream_t st) {
    DropArgs a;
    a.in = in;
    a.out = out;
    a.in_ld = in_ld;
    a.out_ld = out_ld;
    a.cols = cols;
    a.groups = ((uint64_t)cols + 7) / 8;
    a.items = (uint64_t)rows * a.groups;
    a.magic = ~0ull / a.groups + 1;
    a.drop = drop;
    const int64_t size = dtype == 0 ? 4 : 2;
    const bool aligned = (((uintptr_t)in | (uintptr_t)out) & 15u) == 0 &&
                         (rows == 1 || (in_ld * size % 16 == 0 && out_ld * size % 16 == 0));
    const uint64_t grid = (a.items + kDropThreads - 1) / kDropThreads;
    if (grid >= (1ull << 31)) return cudaErrorInvalidValue;
    if (dtype == 0)
        launch_next(aligned ? dropout_kernel<float, true> : dropout_kernel<float, false>, (unsigned)grid, kDropThreads, 0, st, a);
    else
        launch_next(aligned ? dropout_kernel<__nv_bfloat16, true> : dropout_kernel<__nv_bfloat16, false>, (unsigned)grid,
                    kDropThreads, 0, st, a);
    return cudaGetLastError();
}

}  // namespace robe
