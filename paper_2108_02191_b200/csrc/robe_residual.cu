// The join at which a block's output enters the rows again, in one pass over its tensors:
//
//   y = norm(x) w_post  (or x);   out = residual + scale * gate * dropout(y);   normed = norm(out) w_pre
//
// and its backward, from x and out as they stand in memory: the norms' statistics are had again from the rows, nothing is
// kept between the passes.  With n = norm(v) and rstd its factor, the gradient through a norm is
//   d(v) = rstd (g - [mean g] - n mean(g n)),     g = (gradient of the normed row) * weight,   [..]: layer norm only.
#include <initializer_list>

#include "robe_internal.h"
#include "robe_rowops.cuh"

namespace robe {

namespace {

// Sum over the CTA's threads, in every thread.
__device__ __forceinline__ float block_sum(float v, float* scratch) {
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, s);
    __syncthreads();  // (the scratch may still be read from the call before)
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    float sum = 0.0f;
    for (unsigned w = 0; w < (blockDim.x >> 5); ++w) sum += scratch[w];
    return sum;
}

// ---- rows of any length, one CTA each, read again in every pass over the row: for rows too long for the kernels below.  A
// thread takes eight columns at a time (one evaluation of the dropout's generator), in 16-byte pieces where PIECES.  Bound by
// issue: every pass joins the row anew.  4000 rows of 8200 fp32, dropout: backward 670 us (788 MB, 1.2 TB/s).

constexpr int kAnyThreads = 512;

// Eight elements of a row from column c on, zeros beyond its end.
template <class T, bool PIECES>
__device__ __forceinline__ void load_eight(float (&v)[8], const T* row, int64_t c, int64_t d) {
    constexpr int V = kPiece<T>;
    if (PIECES) {  // (d is a multiple of V)
#pragma unroll
        for (int q = 0; q < 8 / V; ++q) {
            Pack<T, V> e;
            if (c + q * V < d) e = load_pack<false, T, V>(row + c + q * V);
#pragma unroll
            for (int k = 0; k < V; ++k) v[q * V + k] = c + q * V < d ? widen(e.v[k]) : 0.0f;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = c + k < d ? widen(row[c + k]) : 0.0f;
    }
}
template <class T, bool PIECES>
__device__ __forceinline__ void store_eight(T* row, const float (&v)[8], int64_t c, int64_t d) {
    constexpr int V = kPiece<T>;
    if (PIECES) {
#pragma unroll
        for (int q = 0; q < 8 / V; ++q) {
            Pack<T, V> e;
#pragma unroll
            for (int k = 0; k < V; ++k) e.v[k] = narrow<T>(v[q * V + k]);
            if (c + q * V < d) store_pack<true, T, V>(row + c + q * V, e);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (c + k < d) row[c + k] = narrow<T>(v[k]);
    }
}
__device__ __forceinline__ void weights_eight(float (&w)[8], const float* p, int64_t c, int64_t d) {
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = c + k < d ? __ldca(p + c + k) : 0.0f;
}

// Mean (0 without `layer`) and factor of the norm of a row whose eight elements from column c on `value` gives.
template <class F>
__device__ __forceinline__ void row_stats(F&& value, int64_t d, int layer, float eps, float* scratch, float& mean, float& rstd) {
    mean = 0.0f;
    float v[8];
    if (layer) {
        float s = 0.0f;
        for (int64_t c = threadIdx.x * 8; c < d; c += blockDim.x * 8) {
            value(v, c);
#pragma unroll
            for (int k = 0; k < 8; ++k) s += v[k];
        }
        mean = block_sum(s, scratch) / (float)d;
    }
    float q = 0.0f;
    for (int64_t c = threadIdx.x * 8; c < d; c += blockDim.x * 8) {
        value(v, c);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float x = v[k] - mean;
            q += c + k < d ? x * x : 0.0f;
        }
    }
    rstd = 1.0f / sqrtf(block_sum(q, scratch) / (float)d + eps);
}

// v, as dropout leaves it
__device__ __forceinline__ void drop_eight_of(float (&v)[8], const ResidualProblem& a, const uint4& w) {
    if (a.drop.none) return;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = drop_keeps(w, k, a.drop) ? v[k] * a.drop.scale : 0.0f;
}
__device__ __forceinline__ uint4 words_eight(const ResidualProblem& a, uint64_t offset, int64_t r, int64_t c) {
    return a.drop.none ? make_uint4(0, 0, 0, 0) : drop_words((uint32_t)r, (uint32_t)(c >> 3), offset, a.drop);
}
template <class T, bool PIECES>
__device__ __forceinline__ void gate_eight(float (&g)[8], const ResidualProblem& a, int64_t r, int64_t c) {
    if (a.gate_kind == 2) {
        load_eight<T, PIECES>(g, (const T*)a.gate.p + r / a.gate_rows * a.gate.ld, c, a.d);
    } else {
        const float v = a.gate_kind == 1 ? widen(((const T*)a.gate.p)[r * a.gate.ld]) : 1.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] = v;
    }
}

template <class T, bool PIECES>
__global__ void __launch_bounds__(kAnyThreads, 2) residual_any_kernel(ResidualProblem a) {
    __shared__ float scratch[kAnyThreads / 32];
    follow();
    const uint64_t offset = drop_offset(a.drop);
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = (const T*)a.x.p + r * a.x.ld;
        const T* residual = a.residual.p != nullptr ? (const T*)a.residual.p + r * a.residual.ld : nullptr;
        float mean1 = 0.0f, rstd1 = 1.0f, mean2 = 0.0f, rstd2 = 1.0f;
        if (a.w_post != nullptr)
            row_stats([&](float (&v)[8], int64_t c) { load_eight<T, PIECES>(v, x, c, a.d); }, a.d, a.layer, a.eps, scratch, mean1, rstd1);
        auto joined = [&](float (&y)[8], int64_t c) {  // (0 beyond the row's end, as the weights are)
            float w[8], g[8], e[8];
            load_eight<T, PIECES>(y, x, c, a.d);
            if (a.w_post != nullptr) {
                weights_eight(w, a.w_post, c, a.d);
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = (y[k] - mean1) * rstd1 * w[k];
            }
            drop_eight_of(y, a, words_eight(a, offset, r, c));
            gate_eight<T, PIECES>(g, a, r, c);
            if (residual != nullptr) load_eight<T, PIECES>(e, residual, c, a.d);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                y[k] = y[k] * a.scale * g[k];
                if (residual != nullptr) y[k] += e[k];
            }
        };
        if (a.w_pre != nullptr) row_stats(joined, a.d, a.layer, a.eps, scratch, mean2, rstd2);
        for (int64_t c = threadIdx.x * 8; c < a.d; c += kAnyThreads * 8) {
            float v[8], w[8];
            joined(v, c);
            store_eight<T, PIECES>((T*)a.out.p + r * a.out.ld, v, c, a.d);
            if (a.w_pre == nullptr) continue;
            weights_eight(w, a.w_pre, c, a.d);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = (v[k] - mean2) * rstd2 * w[k];
            store_eight<T, PIECES>((T*)a.normed.p + r * a.normed.ld, v, c, a.d);
        }
    }
}

// ---- rows kept close: `lanes` threads share a row, E elements each, which they copy to shared memory a row ahead and read
// from there; a thread reads what it copied itself, so nothing but the sums over a row is waited for together.  Up to 512
// elements (256 backward) a row is a part of a warp's, longer ones a CTA's, up to kMaxLanes E; beyond that the kernels for any
// length.  E is 16 (8 backward for parts of a warp, and for small pieces, whose code is longer), 32 for long rows of 16-byte
// pieces: the bf16 backward then spills, 4000 rows of 12288 390 us, 1218 by the kernel for any length.
//
// Measured (16384 rows of 4096 bf16, dropout): forward with a gate per element 130 us (671 MB, 5.2 TB/s; 1156 by the kernel for any
// length), backward with a gate vector per 1024 rows 207 (805 MB, 3.9 TB/s; 1833).  213 K rows of 128 fp32, layer norm, gate per
// row: forward 80 us (5.5 TB/s); of 100, backward 108 (4.7 TB/s).  The forward waits for memory; the backward is bound by
// issue and by its chains of dependent operations (128 registers a thread, so 16 warps an SM, which issue in half of the
// cycles): 32 elements a thread 241 us, 8 (twice the warps, twice the work per row) 284, the first two sums over a row joined into
// one 213, scalar for paired operations 327 against 310 at that time, no test of a row's end 219.

constexpr int kMaxLanes = 512;
constexpr int kWarpRowThreads = 256;
constexpr int kRowElems = 16, kGradWarpElems = 8;  // elements of a thread

// Sums of N values over the threads of a row, in each of them.  CTA: by turns in two halves of `scratch` (zero where there
// is no warp), so that one barrier a sum is enough.
constexpr int kSums = 3;
struct Scratch {
    float4 part[2][kSums][kMaxLanes / 128];
};
template <bool CTA, int N>
__device__ __forceinline__ void row_sums(float (&v)[kSums], int lanes, Scratch& scratch, int& turn) {
    if (CTA) {
#pragma unroll
        for (int s = 16; s > 0; s >>= 1)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], s);
        if (blockDim.x == 32) return;
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) ((float*)scratch.part[turn][k])[threadIdx.x >> 5] = v[k];
        __syncthreads();
        const int fours = (blockDim.x + 127) >> 7;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float4 p = scratch.part[turn][k][0];
            for (int w = 1; w < fours; ++w) {
                const float4 q = scratch.part[turn][k][w];
                p.x += q.x;
                p.y += q.y;
                p.z += q.z;
                p.w += q.w;
            }
            v[k] = (p.x + p.y) + (p.z + p.w);
        }
        turn ^= 1;
    } else {
        for (int s = lanes >> 1; s > 0; s >>= 1)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], s);
    }
}
template <bool CTA>
__device__ __forceinline__ void row_sums(float (&v)[kSums], int n, int lanes, Scratch& scratch, int& turn) {
    if (n == 1) row_sums<CTA, 1>(v, lanes, scratch, turn);
    else if (n == 2) row_sums<CTA, 2>(v, lanes, scratch, turn);
    else row_sums<CTA, 3>(v, lanes, scratch, turn);
}

// A thread's elements of a row: E of them as E / 2 pairs.  They are taken in units of pairs: a piece of V elements, or, where
// V is 1, two pieces.  Shared memory is [stage][tensor][piece][thread]; THREADS of a CTA, 0: asked at run time.
template <class T, int V, int E, int TENSORS, int THREADS>
struct Ring {
    static constexpr int P = V > 1 ? V / 2 : 1;  // pairs of a unit
    static constexpr int NP = E / V;             // pieces
    static constexpr int U = V > 1 ? NP : NP / 2;  // units
    static constexpr int kPieces = V > 1 ? 1 : 2;  // of a unit
    static constexpr int kSlot = V * (int)sizeof(T);
    static constexpr int kThread = TENSORS * E * (int)sizeof(T);  // bytes of a thread in a stage
    char* first;  // the thread's first piece of stage 0
    int lanes, lane, d;

    __device__ __forceinline__ Ring(unsigned char* bytes, int lanes_, int lane_, int64_t d_)
        : first((char*)bytes + threadIdx.x * kSlot), lanes(lanes_), lane(lane_), d((int)d_) {}
    static __device__ __forceinline__ int threads() { return THREADS > 0 ? THREADS : (int)blockDim.x; }
    __device__ __forceinline__ char* stage(int s) const { return first + s * threads() * kThread; }
    static __device__ __forceinline__ T* at(char* stage, int tensor, int k) {
        return (T*)(stage + (tensor * NP + k) * (threads() * kSlot));
    }
    __device__ __forceinline__ int col(int k) const { return (k * lanes + lane) * V; }
    __device__ __forceinline__ bool has(int k) const { return col(k) < d; }
    __device__ __forceinline__ int col_or_0(int k) const { return has(k) ? col(k) : 0; }
    // beyond a row's end there are zeros, once and for all
    __device__ __forceinline__ void clear(int stages) const {
        for (int s = 0; s < stages; ++s)
#pragma unroll
            for (int t = 0; t < TENSORS; ++t)
#pragma unroll
                for (int k = 0; k < NP; ++k)
                    if (!has(k))
#pragma unroll
                        for (int c = 0; c < V; ++c) at(stage(s), t, k)[c] = narrow<T>(0.0f);
    }
    __device__ __forceinline__ void fetch(char* stage, int tensor, const char* row) const {
        if constexpr (kSlot == 2) {  // (no asynchronous copy is as small: at least all loads of a row before the first store)
            unsigned short v[NP];
#pragma unroll
            for (int k = 0; k < NP; ++k)
                v[k] = has(k) && ROBE_CHK(col(k) + V <= d, ROBE_DBG_ROW_POS) ? __ldcs((const unsigned short*)row + col(k)) : 0;
#pragma unroll
            for (int k = 0; k < NP; ++k) *(unsigned short*)at(stage, tensor, k) = v[k];
        } else {
#pragma unroll
            for (int k = 0; k < NP; ++k)
                if (has(k) && ROBE_CHK(col(k) + V <= d, ROBE_DBG_ROW_POS))
                    copy_async<kSlot>(at(stage, tensor, k), row + (uint32_t)col(k) * (uint32_t)sizeof(T));
        }
    }
    static __device__ __forceinline__ void zero(char* stage, int tensor) {
#pragma unroll
        for (int k = 0; k < NP; ++k)
#pragma unroll
            for (int c = 0; c < V; ++c) at(stage, tensor, k)[c] = narrow<T>(0.0f);
    }
    static __device__ __forceinline__ void read(float2 (&v)[P], char* stage, int tensor, int u) {
        if constexpr (V == 1) {
            v[0] = make_float2(widen(*at(stage, tensor, 2 * u)), widen(*at(stage, tensor, 2 * u + 1)));
        } else {
            using W = typename Word<V * sizeof(T)>::type;
            union {
                W w;
                uint32_t bits[V * sizeof(T) / 4];
            } p;
            p.w = *(const W*)at(stage, tensor, u);
#pragma unroll
            for (int q = 0; q < P; ++q) {
                if constexpr (sizeof(T) == 2) v[q] = make_float2(widen_low(p.bits[q]), widen_high(p.bits[q]));
                else v[q] = make_float2(__uint_as_float(p.bits[2 * q]), __uint_as_float(p.bits[2 * q + 1]));
            }
        }
    }
    // .. straight from memory
    __device__ __forceinline__ void load(float2 (&v)[P], const char* row, int u) const {
#pragma unroll
        for (int q = 0; q < P; ++q) {
            const int k = kPieces * u, c = V > 1 ? col(k) + 2 * q : col(k);
            v[q].x = has(k) ? widen(((const T*)row)[c]) : 0.0f;
            v[q].y = has(k + kPieces - 1) ? widen(((const T*)row)[V > 1 ? c + 1 : col(k + 1)]) : 0.0f;
        }
    }
    __device__ __forceinline__ void store(char* row, const float2 (&v)[P], int u) const {
        if constexpr (V == 1) {
            if (has(2 * u)) ((T*)row)[col(2 * u)] = narrow<T>(v[0].x);
            if (has(2 * u + 1)) ((T*)row)[col(2 * u + 1)] = narrow<T>(v[0].y);
        } else if (has(u) && ROBE_CHK(col(u) + V <= d, ROBE_DBG_ROW_POS)) {
            using W = typename Word<V * sizeof(T)>::type;
            union {
                W w;
                uint32_t bits[V * sizeof(T) / 4];
            } p;
#pragma unroll
            for (int q = 0; q < P; ++q) {
                if constexpr (sizeof(T) == 2) {
                    p.bits[q] = narrow2(v[q].x, v[q].y);
                } else {
                    p.bits[2 * q] = __float_as_uint(v[q].x);
                    p.bits[2 * q + 1] = __float_as_uint(v[q].y);
                }
            }
            __stcs((W*)(row + (uint32_t)col(u) * (uint32_t)sizeof(T)), p.w);
        }
    }
    // fp32 weights (16-byte aligned from V = 4 on: the weights are, and columns are multiples of V); beyond the row's end
    // some others, which multiply zeros
    __device__ __forceinline__ void weights(float2 (&w)[P], const float* p, int u) const {
        if constexpr (V == 1) {
            w[0] = make_float2(__ldca(p + col_or_0(2 * u)), __ldca(p + col_or_0(2 * u + 1)));
        } else if constexpr (V >= 4) {
            const float4* at = (const float4*)(p + col_or_0(u));
#pragma unroll
            for (int q = 0; q < P; q += 2) {
                const float4 x = __ldca(at + q / 2);
                w[q] = make_float2(x.x, x.y);
                w[q + 1] = make_float2(x.z, x.w);
            }
        } else {
            const float* at = p + col_or_0(u);
            w[0] = make_float2(__ldca(at), __ldca(at + 1));
        }
    }
    // What dropout decides a row's elements by.  The 8 / V lanes whose pieces make up a group of eight columns evaluate the
    // generator for every 8 / V-th piece each, and hand each other the words.  (A row has that many lanes at least.)
    static constexpr int kShare = 8 / V;
    struct Draws {
        uint4 w[NP / kShare];
    };
    __device__ __forceinline__ void draw(Draws& w, const DropParams& drop, uint64_t offset, uint32_t r) const {
#pragma unroll
        for (int e = 0; e < NP / kShare; ++e)
            w.w[e] = drop_words(r, (uint32_t)col(e * kShare + lane % kShare) >> 3, offset, drop);
    }
    // .. of unit u: an element is kept when its number is above the limit.  (All lanes of a warp.)
    __device__ __forceinline__ void draws(uint32_t (&h)[2 * P], const Draws& w, int u) const {
#pragma unroll
        for (int c = 0; c < kPieces; ++c) {
            const int k = kPieces * u + c;
            const int at = col(k) & 7;
            uint4 v;
            if (kShare == 1) {
                v = w.w[k];
            } else {
                const uint4 mine = w.w[k / kShare];
                const int from = (threadIdx.x & 31) - lane % kShare + k % kShare;
                v.x = __shfl_sync(0xFFFFFFFFu, mine.x, from);
                v.y = __shfl_sync(0xFFFFFFFFu, mine.y, from);
                v.z = __shfl_sync(0xFFFFFFFFu, mine.z, from);
                v.w = __shfl_sync(0xFFFFFFFFu, mine.w, from);
            }
            if constexpr (V == 8) {
                const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    h[2 * q] = word[q] << 16;
                    h[2 * q + 1] = word[q];
                }
            } else {
                const uint32_t low = (at & 4) ? v.z : v.x, high = (at & 4) ? v.w : v.y;
                if constexpr (V == 4) {
                    h[0] = low << 16;
                    h[1] = low;
                    h[2] = high << 16;
                    h[3] = high;
                } else {
                    const uint32_t word = (at & 2) ? high : low;
                    if constexpr (V == 2) {
                        h[0] = word << 16;
                        h[1] = word;
                    } else {
                        h[c] = (at & 1) ? word : word << 16;
                    }
                }
            }
        }
    }
};
__device__ __forceinline__ float2 kept_of(float2 v, const uint32_t* h, uint32_t limit) {
    return make_float2(h[0] > limit ? v.x : 0.0f, h[1] > limit ? v.y : 0.0f);
}

// Rows of a tensor by bytes (a row is less than 2^32 bytes from the next where these kernels are used).
__device__ __forceinline__ char* row_of(const RowsRef& t, uint32_t r, uint32_t size) {
    return (char*)t.p + (uint64_t)r * ((uint32_t)t.ld * size);
}
// A row number that goes up by equal steps, with its gate vector's.
struct GateRow {
    uint32_t gate, step_gate;
    uint64_t in_gate, step_in, gate_rows;
    __device__ __forceinline__ GateRow(uint32_t r, uint32_t step, uint32_t rows_) : gate_rows(rows_) {
        gate = r / rows_;
        in_gate = r - (uint64_t)gate * rows_;
        step_gate = step / rows_;
        step_in = step - (uint64_t)step_gate * rows_;
    }
    __device__ __forceinline__ void next() {
        gate += step_gate;
        in_gate += step_in;
        if (in_gate >= gate_rows) {
            in_gate -= gate_rows;
            ++gate;
        }
    }
};

// Adds v to a unit's elements, not to the zeros beyond the row's end.
template <class R, int P>
__device__ __forceinline__ void center(const R& ring, float2 (&x)[P], float v, int u) {
#pragma unroll
    for (int q = 0; q < P; ++q) {
        x[q] = add2(x[q], both(v));
        if (!ring.has(R::kPieces * u)) x[q].x = 0.0f;
        if (!ring.has(R::kPieces * u + R::kPieces - 1)) x[q].y = 0.0f;
    }
}

// USUAL: both norms, something added to, and LAYER, DROP and VECTOR say the rest; otherwise that is asked in the row loop.
template <class T, int V, int E, bool CTA, bool USUAL, int LAYER, int DROP, int VECTOR>
__global__ void __launch_bounds__(CTA ? kMaxLanes : kWarpRowThreads)
residual_rows_kernel(ResidualProblem a, int lanes, int stages) {
    using R = Ring<T, V, E, 2 + VECTOR, CTA ? 0 : kWarpRowThreads>;
    constexpr int P = R::P, U = R::U;
    extern __shared__ __align__(16) unsigned char ring_bytes[];
    __shared__ Scratch scratch;
    follow();
    const uint64_t offset = drop_offset(a.drop);
    const bool post = USUAL || a.w_post != nullptr, pre = USUAL || a.w_pre != nullptr, added = USUAL || a.residual.p != nullptr;
    const bool layer = USUAL ? LAYER : a.layer, dropping = USUAL ? DROP : !a.drop.none, vector = USUAL ? VECTOR : a.gate_kind == 2;
    const R ring(ring_bytes, lanes, CTA ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1), a.d);
    const uint32_t groups = CTA ? 1 : kWarpRowThreads / lanes, group = CTA ? 0 : threadIdx.x / lanes;
    const uint32_t step = gridDim.x * groups, rows = (uint32_t)a.rows;
    const float over_d = 1.0f / (float)a.d;
    int turn = 0;
    ring.clear(stages);
    if (CTA) {
        for (unsigned k = threadIdx.x; k < sizeof(Scratch) / 4; k += blockDim.x) ((float*)&scratch)[k] = 0.0f;
        __syncthreads();
    }
    // (a warp's groups go through as many rows as its first one: sums over lanes need them all)
    uint64_t leader = (uint64_t)blockIdx.x * groups + (CTA ? 0 : (threadIdx.x & ~31u) / lanes);
    const uint32_t ahead = CTA ? 0 : group - (threadIdx.x & ~31u) / lanes;
    uint64_t next = leader + ahead;
    GateRow gate(next < rows ? (uint32_t)next : 0, step, vector ? (uint32_t)a.gate_rows : 1);
    auto fetch = [&](char* stage) {
        if (next < rows) {
            const uint32_t r = (uint32_t)next;
            if (!ROBE_CHK(!vector || gate.gate == r / a.gate_rows, ROBE_DBG_ROW_POS)) return;
            ring.fetch(stage, 0, row_of(a.x, r, sizeof(T)));
            if (added) ring.fetch(stage, 1, row_of(a.residual, r, sizeof(T)));
            if (vector) {
                ring.fetch(stage, 2, row_of(a.gate, gate.gate, sizeof(T)));
                gate.next();
            }
        }
        next += step;
        copies_close();
    };
    for (int s = 0; s + 1 < stages; ++s) fetch(ring.stage(s));
    int turn_of = 0;
    for (; leader < rows; leader += step) {
        const bool here = leader + ahead < rows;
        const uint32_t r = (uint32_t)leader + ahead;
        fetch(ring.stage(turn_of == 0 ? stages - 1 : turn_of - 1));
        char* stage = ring.stage(turn_of);
        copies_wait(stages - 1);
        float2 v[U][P];
#pragma unroll
        for (int u = 0; u < U; ++u) R::read(v[u], stage, 0, u);
        // norm of the row that v holds (0 beyond d): mean and factor
        auto stats = [&](float& mean, float& rstd) {
            float s[kSums];
            mean = 0.0f;
            if (layer) {
                float2 t = both(0.0f);
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int q = 0; q < P; ++q) t = add2(t, v[u][q]);
                s[0] = t.x + t.y;
                row_sums<CTA, 1>(s, lanes, scratch, turn);
                mean = s[0] * over_d;
            }
            float2 t = both(0.0f);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float2 c[P];
#pragma unroll
                for (int q = 0; q < P; ++q) c[q] = v[u][q];
                if (layer) center(ring, c, -mean, u);
#pragma unroll
                for (int q = 0; q < P; ++q) t = fma2(c[q], c[q], t);
            }
            s[0] = t.x + t.y;
            row_sums<CTA, 1>(s, lanes, scratch, turn);
            rstd = norm_factor(s[0] * over_d + a.eps);
        };
        float mean = 0.0f, rstd = 1.0f;
        if (post) stats(mean, rstd);
        float row_gate = a.scale;
        if (a.gate_kind == 1 && here) row_gate *= widen(*(const T*)row_of(a.gate, r, sizeof(T)));
        if (dropping) row_gate *= a.drop.scale;
        char* out = row_of(a.out, r, sizeof(T));
        typename R::Draws words;
        if (dropping) ring.draw(words, a.drop, offset, r);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (post) {
                float2 w[P];
                ring.weights(w, a.w_post, u);
                if (layer) center(ring, v[u], -mean, u);
#pragma unroll
                for (int q = 0; q < P; ++q) v[u][q] = mul2(mul2(v[u][q], both(rstd)), w[q]);
            }
            if (dropping) {
                uint32_t draws[2 * P];
                ring.draws(draws, words, u);
#pragma unroll
                for (int q = 0; q < P; ++q) v[u][q] = kept_of(v[u][q], draws + 2 * q, a.drop.limit);
            }
            if (vector) {
                float2 g[P];
                R::read(g, stage, 2, u);
#pragma unroll
                for (int q = 0; q < P; ++q) v[u][q] = mul2(v[u][q], g[q]);
            }
            if (added) {
                float2 e[P];
                R::read(e, stage, 1, u);
#pragma unroll
                for (int q = 0; q < P; ++q) v[u][q] = fma2(v[u][q], both(row_gate), e[q]);
            } else {
#pragma unroll
                for (int q = 0; q < P; ++q) v[u][q] = mul2(v[u][q], both(row_gate));
            }
            if (here) ring.store(out, v[u], u);
        }
        if (pre) {
            stats(mean, rstd);
            char* normed = row_of(a.normed, r, sizeof(T));
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float2 w[P];
                ring.weights(w, a.w_pre, u);
#pragma unroll
                for (int q = 0; q < P; ++q) w[q] = mul2(mul2(add2(v[u][q], both(-mean)), both(rstd)), w[q]);
                if (here) ring.store(normed, w, u);
            }
        }
        turn_of = turn_of + 1 == stages ? 0 : turn_of + 1;
    }
    copies_wait(0);
}

// Rows [row0(chunk), row1(chunk)): chunks never cross the border of a gate vector, or hold whole ones.
struct Chunks {
    int64_t rows, gate_rows;  // of all, that share a gate vector (rows where none does)
    int64_t per_gate;         // chunks of a gate vector's rows; 0: a chunk holds `gates` vectors' rows
    int64_t gates;
    int64_t length;           // rows of a chunk (the last of a gate vector's, or of all, may be shorter)
    int64_t count;
    __host__ __device__ int64_t row0(int64_t k) const {
        return per_gate > 0 ? k / per_gate * gate_rows + k % per_gate * length : k * length;
    }
    __host__ __device__ int64_t row1(int64_t k) const {
        const int64_t end = per_gate > 0 ? (k / per_gate + 1) * gate_rows : rows;
        return row0(k) + length < end ? row0(k) + length : end;
    }
};

struct JoinGradArgs {
    ResidualProblem p;
    Chunks chunks;
    float *part_post, *part_pre, *part_gate;  // [chunks][d]
};

// Columns' sums of the chunk in shared memory where they fit (IN_SHARED), else in the workspace: a column is always the same
// thread's.
template <class T, bool PIECES, bool IN_SHARED>
__global__ void __launch_bounds__(kAnyThreads, 1) residual_grad_any_kernel(JoinGradArgs args) {
    extern __shared__ float shared_sums[];
    __shared__ float scratch[kAnyThreads / 32];
    follow();
    const ResidualProblem& a = args.p;
    const uint64_t offset = drop_offset(a.drop);
    const float over_d = 1.0f / (float)a.d;
    const int64_t r0 = args.chunks.row0(blockIdx.x), r1 = args.chunks.row1(blockIdx.x);
    float* part_post = args.part_post + blockIdx.x * a.d;
    float* part_pre = args.part_pre + blockIdx.x * a.d;
    float* part_gate = args.part_gate + blockIdx.x * a.d;
    float* sum_post = IN_SHARED ? shared_sums : part_post;
    float* sum_pre = IN_SHARED ? shared_sums + a.d : part_pre;
    float* sum_gate = IN_SHARED ? shared_sums + 2 * a.d : part_gate;
    const bool gate_sums = a.gate_kind == 2 && a.grad_gate.p != nullptr;
    const bool whole_gates = a.gate_rows == 1 || args.chunks.per_gate == 0;
    for (int64_t r = r0; r < r1; ++r) {
        const T* x = (const T*)a.x.p + r * a.x.ld;
        const T* out = (const T*)a.out.p + r * a.out.ld;
        const T* go = a.grad_out.p != nullptr ? (const T*)a.grad_out.p + r * a.grad_out.ld : nullptr;
        const T* gn = (const T*)a.grad_normed.p + r * a.grad_normed.ld;
        float mean1 = 0.0f, rstd1 = 1.0f, mean2 = 0.0f, rstd2 = 1.0f, dot2 = 0.0f, sum2 = 0.0f;
        if (a.w_pre != nullptr) {
            row_stats([&](float (&v)[8], int64_t c) { load_eight<T, PIECES>(v, out, c, a.d); }, a.d, a.layer, a.eps, scratch, mean2, rstd2);
            float dot = 0.0f, sum = 0.0f;
            for (int64_t c = threadIdx.x * 8; c < a.d; c += kAnyThreads * 8) {
                float g[8], w[8], n[8];
                load_eight<T, PIECES>(g, gn, c, a.d);
                load_eight<T, PIECES>(n, out, c, a.d);
                weights_eight(w, a.w_pre, c, a.d);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    dot += g[k] * w[k] * ((n[k] - mean2) * rstd2);
                    sum += g[k] * w[k];
                }
            }
            dot2 = block_sum(dot, scratch) * over_d;
            if (a.layer) sum2 = block_sum(sum, scratch) * over_d;
        }
        // gradient of `out` from both sides, and the norm of out and its gradient
        auto total = [&](float (&t)[8], float (&n)[8], float (&g)[8], int64_t c) {
#pragma unroll
            for (int k = 0; k < 8; ++k) t[k] = n[k] = g[k] = 0.0f;
            if (go != nullptr) load_eight<T, PIECES>(t, go, c, a.d);
            if (a.w_pre == nullptr) return;
            float w[8];
            load_eight<T, PIECES>(n, out, c, a.d);
            load_eight<T, PIECES>(g, gn, c, a.d);
            weights_eight(w, a.w_pre, c, a.d);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                n[k] = (n[k] - mean2) * rstd2;
                t[k] += rstd2 * (g[k] * w[k] - sum2 - n[k] * dot2);
            }
        };
        if (a.w_post != nullptr)
            row_stats([&](float (&v)[8], int64_t c) { load_eight<T, PIECES>(v, x, c, a.d); }, a.d, a.layer, a.eps, scratch, mean1, rstd1);
        // of eight columns: norm of x, dropped gradient of the norm's row (u), weights, gradient of the gate
        auto back = [&](const float (&t)[8], float (&n)[8], float (&u)[8], float (&w)[8], float (&gg)[8], int64_t c) {
            float g[8], y[8];
            load_eight<T, PIECES>(n, x, c, a.d);
            if (a.w_post != nullptr) weights_eight(w, a.w_post, c, a.d);
            gate_eight<T, PIECES>(g, a, r, c);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                n[k] = (n[k] - mean1) * rstd1;
                if (a.w_post == nullptr) w[k] = 1.0f;
                y[k] = n[k] * w[k];
                u[k] = t[k] * a.scale * g[k];
            }
            const uint4 words = words_eight(a, offset, r, c);
            drop_eight_of(y, a, words);
            drop_eight_of(u, a, words);
#pragma unroll
            for (int k = 0; k < 8; ++k)  // (of what is dropped +0, whatever t is there)
                gg[k] = a.drop.none || drop_keeps(words, k, a.drop) ? y[k] * (a.scale * t[k]) : 0.0f;
        };
        float dot = 0.0f, sum = 0.0f, gate_sum = 0.0f;
        if (a.w_post != nullptr || a.gate_kind == 1)
            for (int64_t c = threadIdx.x * 8; c < a.d; c += kAnyThreads * 8) {
                float t[8], n2[8], g2[8], n[8], u[8], w[8], gg[8];
                total(t, n2, g2, c);
                back(t, n, u, w, gg, c);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (c + k >= a.d) break;
                    dot += u[k] * w[k] * n[k];
                    sum += u[k] * w[k];
                    gate_sum += gg[k];
                }
            }
        float dot1 = 0.0f, sum1 = 0.0f;
        if (a.w_post != nullptr) {
            dot1 = block_sum(dot, scratch) * over_d;
            if (a.layer) sum1 = block_sum(sum, scratch) * over_d;
        }
        if (a.gate_kind == 1 && a.grad_gate.p != nullptr) {
            gate_sum = block_sum(gate_sum, scratch);
            if (threadIdx.x == 0) ((T*)a.grad_gate.p)[r * a.grad_gate.ld] = narrow<T>(gate_sum);
        }
        const int64_t in_gate = r % a.gate_rows;
        for (int64_t c = threadIdx.x * 8; c < a.d; c += kAnyThreads * 8) {
            float t[8], n2[8], g2[8], n[8], u[8], w[8], gg[8];
            total(t, n2, g2, c);
            back(t, n, u, w, gg, c);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (c + k >= a.d) break;
                if (a.w_pre != nullptr) sum_pre[c + k] = (r == r0 ? 0.0f : sum_pre[c + k]) + g2[k] * n2[k];
                if (gate_sums) {
                    if (r != r0 && in_gate != 0) gg[k] += sum_gate[c + k];
                    sum_gate[c + k] = gg[k];
                }
                if (a.w_post != nullptr) {
                    sum_post[c + k] = (r == r0 ? 0.0f : sum_post[c + k]) + u[k] * n[k];
                    u[k] = rstd1 * (u[k] * w[k] - sum1 - n[k] * dot1);
                }
            }
            if (gate_sums && whole_gates && in_gate == a.gate_rows - 1)
                store_eight<T, PIECES>((T*)a.grad_gate.p + r / a.gate_rows * a.grad_gate.ld, gg, c, a.d);
            if (a.grad_residual.p != nullptr) store_eight<T, PIECES>((T*)a.grad_residual.p + r * a.grad_residual.ld, t, c, a.d);
            store_eight<T, PIECES>((T*)a.grad_x.p + r * a.grad_x.ld, u, c, a.d);
        }
    }
    if constexpr (IN_SHARED)
        for (int64_t c = threadIdx.x * 8; c < a.d; c += kAnyThreads * 8)
            for (int64_t k = c; k < c + 8 && k < a.d; ++k) {
                if (a.w_post != nullptr) part_post[k] = sum_post[k];
                if (a.w_pre != nullptr) part_pre[k] = sum_pre[k];
                if (gate_sums && !whole_gates) part_gate[k] = sum_gate[k];
            }
}

// One CTA per chunk.  The weights' gradients of a thread's columns are summed in registers over its rows, over the groups of
// a CTA in shared memory, over the chunks by the kernel below; a gate vector's likewise, or stored when its rows are done.
template <class T, int V, int E, bool CTA, bool USUAL, int LAYER, int DROP, int VECTOR>
__global__ void __launch_bounds__(CTA ? kMaxLanes : kWarpRowThreads, CTA ? 1 : VECTOR ? 2 : 3)
residual_grad_rows_kernel(JoinGradArgs args, int lanes, int stages) {
    using R = Ring<T, V, E, 4 + VECTOR, CTA ? 0 : kWarpRowThreads>;
    constexpr int P = R::P, U = R::U;
    extern __shared__ __align__(16) unsigned char ring_bytes[];
    __shared__ Scratch scratch;
    follow();
    const ResidualProblem& a = args.p;
    const uint64_t offset = drop_offset(a.drop);
    const bool post = USUAL || a.w_post != nullptr, pre = USUAL || a.w_pre != nullptr, skip = USUAL || a.grad_out.p != nullptr;
    const bool stream = USUAL || a.grad_residual.p != nullptr, vector = USUAL ? VECTOR : a.gate_kind == 2;
    const bool layer = USUAL ? LAYER : a.layer, dropping = USUAL ? DROP : !a.drop.none;
    const bool shared_gate = vector && a.gate_rows > 1;  // a gate vector of several rows
    const bool whole_gates = args.chunks.per_gate == 0;            // .. all in this chunk
    constexpr int kX = 0, kSkip = 1, kOut = 2, kNormed = 3, kGate = 4;
    const R ring(ring_bytes, lanes, CTA ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1), a.d);
    const uint32_t groups = CTA ? 1 : kWarpRowThreads / lanes, group = CTA ? 0 : threadIdx.x / lanes;
    const float over_d = 1.0f / (float)a.d;
    int turn = 0;
    ring.clear(stages);
    if (CTA) {
        for (unsigned k = threadIdx.x; k < sizeof(Scratch) / 4; k += blockDim.x) ((float*)&scratch)[k] = 0.0f;
        __syncthreads();
    }
    // the rows of a group: every groups-th of the chunk, or whole gate vectors in turn
    const uint32_t c0 = (uint32_t)args.chunks.row0(blockIdx.x), c1 = (uint32_t)args.chunks.row1(blockIdx.x);
    const uint32_t block = shared_gate && whole_gates ? (uint32_t)a.gate_rows : 1;
    // (as many rounds for all groups: sums over lanes need whole warps)
    const uint32_t rounds = ((c1 - c0 + block - 1) / block + groups - 1) / groups * block;
    // k-th row of this group and its gate vector; none from c1 on
    struct Place {
        uint32_t r, in_block, gate;
    };
    auto advance = [&](Place& p) {
        if (block == 1) {
            p.r += groups;
        } else {
            ++p.r;
            if (++p.in_block == block) {
                p.in_block = 0;
                p.r += (groups - 1) * block;
                p.gate += groups;
            }
        }
    };
    Place now{c0 + group * block, 0, 0};
    if (shared_gate) now.gate = c0 / (uint32_t)a.gate_rows + (whole_gates ? group : 0);
    Place next = now;
    float2 sum_post[U][P], sum_pre[U][P], sum_gate[U][P];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < P; ++q) sum_post[u][q] = sum_pre[u][q] = sum_gate[u][q] = both(0.0f);
    // the sum that a gate vector's rows share, as the weight's gradient and the gate's
    auto close_gate = [&](int u, const float2 (&g)[P]) {
        if (!post) return;
        float2 w[P];
        ring.weights(w, a.w_post, u);
#pragma unroll
        for (int q = 0; q < P; ++q) {
            sum_post[u][q] = fma2(sum_gate[u][q], g[q], sum_post[u][q]);
            sum_gate[u][q] = mul2(sum_gate[u][q], w[q]);
        }
    };
    auto fetch = [&](char* stage) {
        if (next.r < c1) {
            const uint32_t r = next.r;
            if (!ROBE_CHK(r >= c0 && r < a.rows && (!shared_gate || next.gate == r / a.gate_rows), ROBE_DBG_ROW_POS)) return;
            ring.fetch(stage, kX, row_of(a.x, r, sizeof(T)));
            if (skip) ring.fetch(stage, kSkip, row_of(a.grad_out, r, sizeof(T)));
            if (pre) {
                ring.fetch(stage, kOut, row_of(a.out, r, sizeof(T)));
                ring.fetch(stage, kNormed, row_of(a.grad_normed, r, sizeof(T)));
            }
            if (vector) ring.fetch(stage, kGate, row_of(a.gate, shared_gate ? next.gate : r, sizeof(T)));
        } else {  // no such row: zeros add nothing to the sums
#pragma unroll
            for (int k = 0; k < 4 + VECTOR; ++k) R::zero(stage, k);
        }
        advance(next);
        copies_close();
    };
    for (int s = 0; s + 1 < stages; ++s) fetch(ring.stage(s));
    int turn_of = 0;
    for (uint32_t round = 0; round < rounds; ++round) {
        const uint32_t r = now.r;
        const bool here = now.r < c1;
        fetch(ring.stage(turn_of == 0 ? stages - 1 : turn_of - 1));
        char* stage = ring.stage(turn_of);
        copies_wait(stages - 1);
        float2 t[U][P];  // out, its norm, then the gradient of out
        float s[kSums];
        float mean1 = 0.0f, mean2 = 0.0f;
        {
            float2 x[U][P];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                R::read(x[u], stage, kX, u);
                if (pre) R::read(t[u], stage, kOut, u);
                else
#pragma unroll
                    for (int q = 0; q < P; ++q) t[u][q] = both(0.0f);
            }
            float2 s1 = both(0.0f), s2 = both(0.0f);
            if (layer) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int q = 0; q < P; ++q) {
                        s1 = add2(s1, x[u][q]);
                        s2 = add2(s2, t[u][q]);
                    }
                s[0] = s1.x + s1.y;
                s[1] = s2.x + s2.y;
                row_sums<CTA, 2>(s, lanes, scratch, turn);
                mean1 = post ? s[0] * over_d : 0.0f;
                mean2 = s[1] * over_d;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    center(ring, x[u], -mean1, u);
                    center(ring, t[u], -mean2, u);
                }
                s1 = s2 = both(0.0f);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int q = 0; q < P; ++q) {
                    s1 = fma2(x[u][q], x[u][q], s1);
                    s2 = fma2(t[u][q], t[u][q], s2);
                }
            s[0] = s1.x + s1.y;
            s[1] = s2.x + s2.y;
        }
        if (post || pre) row_sums<CTA, 2>(s, lanes, scratch, turn);
        // (0 for no row: with eps = 0 its factor would be infinite)
        const float rstd1 = !here ? 0.0f : post ? norm_factor(s[0] * over_d + a.eps) : 1.0f;
        const float rstd2 = !here ? 0.0f : pre ? norm_factor(s[1] * over_d + a.eps) : 1.0f;
        if (pre) {
            // with g the normed row's gradient times the weight: t = (grad_out + rstd g) - rstd (mean(g n) n + [mean g])
            float2 both_sides[U][P];
            float2 s1 = both(0.0f), s2 = both(0.0f);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float2 g[P], w[P], e[P];
                R::read(g, stage, kNormed, u);
                ring.weights(w, a.w_pre, u);
                if (skip) R::read(e, stage, kSkip, u);
#pragma unroll
                for (int q = 0; q < P; ++q) {
                    t[u][q] = mul2(t[u][q], both(rstd2));
                    sum_pre[u][q] = fma2(g[q], t[u][q], sum_pre[u][q]);
                    w[q] = mul2(g[q], w[q]);
                    s1 = fma2(w[q], t[u][q], s1);
                    if (layer) s2 = add2(s2, w[q]);
                    both_sides[u][q] = skip ? fma2(w[q], both(rstd2), e[q]) : mul2(w[q], both(rstd2));
                }
            }
            s[0] = s1.x + s1.y;
            s[1] = s2.x + s2.y;
            row_sums<CTA>(s, layer ? 2 : 1, lanes, scratch, turn);
            const float dot = -s[0] * over_d * rstd2;
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int q = 0; q < P; ++q) t[u][q] = fma2(t[u][q], both(dot), both_sides[u][q]);
                if (layer) center(ring, t[u], -s[1] * over_d * rstd2, u);
            }
        } else if (skip) {
#pragma unroll
            for (int u = 0; u < U; ++u) R::read(t[u], stage, kSkip, u);
        }
        float2 x[U][P];  // norm of x
        float row_gate = 1.0f;
        if (a.gate_kind == 1 && here) row_gate = widen(*(const T*)row_of(a.gate, r, sizeof(T)));
        const float2 scale = both(dropping ? a.scale * a.drop.scale : a.scale);
        char* grad_residual = row_of(a.grad_residual, r, sizeof(T));
        float2 s0 = both(0.0f), s1 = both(0.0f);
        typename R::Draws words;
        if (dropping) ring.draw(words, a.drop, offset, r);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            R::read(x[u], stage, kX, u);
            if (layer) center(ring, x[u], -mean1, u);
            if (stream && here) ring.store(grad_residual, t[u], u);
            float2 w[P];
            if (post) ring.weights(w, a.w_post, u);
            uint32_t draws[2 * P];
            if (dropping) ring.draws(draws, words, u);
            // t: what comes back through dropout and scale; a gate that is one number of the row follows after the sums
#pragma unroll
            for (int q = 0; q < P; ++q) {
                x[u][q] = mul2(x[u][q], both(rstd1));
                t[u][q] = mul2(t[u][q], scale);
                if (dropping) {
                    t[u][q] = kept_of(t[u][q], draws + 2 * q, a.drop.limit);
                    if (!post) x[u][q] = kept_of(x[u][q], draws + 2 * q, a.drop.limit);
                }
            }
            if (vector) {
                float2 g[P];
                R::read(g, stage, kGate, u);
                if (shared_gate) {  // one sum for two gradients: times the weight it is the gate's, times the gate the weight's
#pragma unroll
                    for (int q = 0; q < P; ++q) sum_gate[u][q] = fma2(t[u][q], x[u][q], sum_gate[u][q]);
                } else if (a.grad_gate.p != nullptr && here) {
                    float2 gg[P];
#pragma unroll
                    for (int q = 0; q < P; ++q) gg[q] = mul2(post ? mul2(x[u][q], w[q]) : x[u][q], t[u][q]);
                    ring.store(row_of(a.grad_gate, r, sizeof(T)), gg, u);
                }
#pragma unroll
                for (int q = 0; q < P; ++q) t[u][q] = mul2(t[u][q], g[q]);
                if (post && !shared_gate)
#pragma unroll
                    for (int q = 0; q < P; ++q) sum_post[u][q] = fma2(t[u][q], x[u][q], sum_post[u][q]);
            } else if (post) {
#pragma unroll
                for (int q = 0; q < P; ++q) sum_post[u][q] = fma2(mul2(t[u][q], both(row_gate)), x[u][q], sum_post[u][q]);
            }
            if (post)
#pragma unroll
                for (int q = 0; q < P; ++q) t[u][q] = mul2(t[u][q], w[q]);
#pragma unroll
            for (int q = 0; q < P; ++q) {
                s0 = fma2(t[u][q], x[u][q], s0);
                if (layer) s1 = add2(s1, t[u][q]);
            }
        }
        s[0] = s0.x + s0.y;
        s[1] = s1.x + s1.y;
        if (post || a.gate_kind == 1) row_sums<CTA>(s, layer && post ? 2 : 1, lanes, scratch, turn);
        if (a.gate_kind == 1 && a.grad_gate.p != nullptr && here && ring.lane == 0)
            *(T*)row_of(a.grad_gate, r, sizeof(T)) = narrow<T>(s[0]);
        const float2 dot = both(-s[0] * over_d), mean = both(layer ? -s[1] * over_d : 0.0f);
        const float2 factor = both(post ? rstd1 * row_gate : row_gate);
        char* grad_x = row_of(a.grad_x, r, sizeof(T));
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int q = 0; q < P; ++q) t[u][q] = mul2(post ? fma2(x[u][q], dot, add2(t[u][q], mean)) : t[u][q], factor);
            if (here) ring.store(grad_x, t[u], u);
        }
        if (shared_gate && whole_gates && now.in_block == block - 1) {  // a gate vector's rows are done
            char* grad_gate = row_of(a.grad_gate, now.gate, sizeof(T));
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float2 g[P];
                R::read(g, stage, kGate, u);
                close_gate(u, g);
                if (a.grad_gate.p != nullptr && here) ring.store(grad_gate, sum_gate[u], u);
#pragma unroll
                for (int q = 0; q < P; ++q) sum_gate[u][q] = both(0.0f);
            }
        }
        advance(now);
        turn_of = turn_of + 1 == stages ? 0 : turn_of + 1;
    }
    copies_wait(0);
    if (shared_gate && !whole_gates) {
        const char* row = row_of(a.gate, c0 / (uint32_t)a.gate_rows, sizeof(T));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float2 g[P];
            ring.load(g, row, u);
            close_gate(u, g);
        }
    }
    // the chunk's sums
    auto store_sums = [&](const float2 (&v)[U][P], float* part) {
        if (!ROBE_CHK(blockIdx.x < args.chunks.count, ROBE_DBG_ROW_POS)) return;
        part += blockIdx.x * a.d;
        float* to = part;
        if (!CTA) {
            __syncthreads();
            to = (float*)ring_bytes + group * a.d;  // [groups][d]
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int q = 0; q < P; ++q) {
                const int k = V > 1 ? u : 2 * u, c = ring.col(k) + 2 * q;
                if (ring.has(k)) to[V > 1 ? c : ring.col(k)] = v[u][q].x;
                if (ring.has(V > 1 ? k : k + 1)) to[V > 1 ? c + 1 : ring.col(k + 1)] = v[u][q].y;
            }
        if (CTA) return;
        __syncthreads();
        for (int c = threadIdx.x; c < (int)a.d; c += kWarpRowThreads) {
            float s = 0.0f;
            for (uint32_t g = 0; g < groups; ++g) s += ((float*)ring_bytes)[g * a.d + c];
            part[c] = s;
        }
    };
    if (post) store_sums(sum_post, args.part_post);
    if (pre) store_sums(sum_pre, args.part_pre);
    if (shared_gate && !whole_gates && a.grad_gate.p != nullptr) store_sums(sum_gate, args.part_gate);
}

// Columns of [parts][d] summed: first the weights after the block, those before the next, then the gate vectors.  A CTA
// has kColumnThreads / share columns of one of them, `share` threads a column: 16, or 2 for gate vectors of few parts.
constexpr int kColumnThreads = 512, kColumnBatch = 8;

struct ColumnArgs {
    JoinGradArgs j;
    uint32_t weights, weight_tiles;  // sums of weights, CTAs of each
    int gate_share;
    uint32_t gate_tiles;
};

template <class T>
__global__ void __launch_bounds__(kColumnThreads) residual_columns_kernel(ColumnArgs args) {
    __shared__ double sums[kColumnThreads];
    follow();
    const ResidualProblem& a = args.j.p;
    const uint32_t ahead = args.weights * args.weight_tiles;
    const bool gate = blockIdx.x >= ahead;
    const uint32_t block = gate ? blockIdx.x - ahead : blockIdx.x, tiles = gate ? args.gate_tiles : args.weight_tiles;
    const int share = gate ? args.gate_share : 16, columns = kColumnThreads / share;
    const uint32_t what = block / tiles;
    const int lane = threadIdx.x & (columns - 1), row = threadIdx.x / columns;
    const int64_t c = (int64_t)(block - what * tiles) * columns + lane;
    const bool post = what == 0 && a.w_post != nullptr;
    const int64_t first = gate ? what * args.j.chunks.per_gate : 0;
    const int count = (int)(gate ? args.j.chunks.per_gate : args.j.chunks.count);
    const float* part = (gate ? args.j.part_gate : post ? args.j.part_post : args.j.part_pre) + first * a.d + c;
    double s = 0.0;
    if (c < a.d)
        for (int k = row; k < count; k += share * kColumnBatch) {
            float v[kColumnBatch];
#pragma unroll
            for (int q = 0; q < kColumnBatch; ++q) {
                const int at = k + q * share;
                v[q] = at < count ? __ldcs(part + at * a.d) : 0.0f;
            }
#pragma unroll
            for (int q = 0; q < kColumnBatch; ++q) s += (double)v[q];
        }
    sums[threadIdx.x] = s;
    __syncthreads();
    if (row != 0 || c >= a.d) return;
    s = 0.0;
    for (int k = 0; k < share; ++k) s += sums[k * columns + lane];
    if (gate) ((T*)a.grad_gate.p)[(int64_t)what * a.grad_gate.ld + c] = narrow<T>((float)s);
    else (post ? a.grad_w_post : a.grad_w_pre)[c] = (float)s;
}

// As many chunks as CTAs are resident at once by their registers, so that all end together: rows of a warp's part in CTAs of 256
// threads, others in CTAs of a row's threads (128 registers a thread: 512 of them an SM).  That is how many are resident in
// the usual bf16 calls.  Shared memory is not looked at: where a CTA's stages take more of it (fp32 rows of a CTA: 64 KB a stage
// at 256 threads), the chunks go by in more than one wave.
int64_t resident_chunks(int64_t d, bool gates) {
    if (d <= 32 * kGradWarpElems) return 148 * (gates ? 2 : 3);
    const int64_t threads = ((d + kRowElems - 1) / kRowElems + 31) / 32 * 32;
    return 148 * (threads >= 512 ? 1 : 512 / threads);
}

// Rows of a CTA at a time.
int64_t groups_of(int64_t d) {
    if (d > 32 * kGradWarpElems) return 1;
    int64_t lanes = 1;
    while (lanes * kGradWarpElems < d) lanes *= 2;
    return kWarpRowThreads / lanes;
}

// Rows that a thread sums in fp32 at most, whatever the call's: a sum of n like terms is off by up to n / 2 of its last places, and
// from 2^24 on takes nothing in.  The chunks' sums are joined in 64 bits.
constexpr int64_t kChainRows = 256;

// gates: gate vectors of more than one row that the rows share, or 0; vector: there is a gate of d columns at all; again: for the
// kernel that reads rows again.  The workspace is sized by the same call.
Chunks chunks_of(int64_t rows, int64_t d, int64_t gates, bool vector, bool again) {
    int64_t most = resident_chunks(d, vector);
    // .. but four rows of each beyond two a SM: fewer chunks' sums to join (1578 rows of 312 fp32 36 -> 26 us, 2000 of 1024 bf16
    // 34 -> 27)
    if (most > 296 && most > rows / 4) most = rows / 4 > 296 ? rows / 4 : 296;
    Chunks k;
    k.rows = rows;
    k.gate_rows = gates > 0 ? rows / gates : rows;
    k.per_gate = k.gates = k.length = k.count = 0;
    if (rows == 0) return k;
    // groups that are sure to share a chunk's rows (at least 8 lanes a row where pieces are of one element)
    const int64_t sharing = again ? 1 : groups_of(d) < kWarpRowThreads / 8 ? groups_of(d) : kWarpRowThreads / 8;
    // whole gate vectors, each by one of a CTA's groups, where there are enough for half of the groups; else a CTA's groups
    // share one vector's rows (608 vectors of 660 rows of 136: 947 us the first way)
    if (gates == 0 || 2 * gates < most * groups_of(d) || k.gate_rows > kChainRows) {
        k.per_gate = gates == 0 ? most : gates < most ? most / gates : 1;
        k.length = (k.gate_rows + k.per_gate - 1) / k.per_gate;
        if (k.length < groups_of(d)) k.length = groups_of(d);  // (a row for each of a CTA's groups)
        // longer than a chain: so many times the chunks, all alike
        const int64_t times = (k.length + kChainRows * sharing - 1) / (kChainRows * sharing);
        k.length = (k.length + times - 1) / times;
        k.per_gate = (k.gate_rows + k.length - 1) / k.length;
        k.count = (gates > 0 ? gates : 1) * k.per_gate;
    } else {
        k.gates = (gates + most - 1) / most;
        const int64_t chain = kChainRows / k.gate_rows * sharing, times = (k.gates + chain - 1) / chain;
        k.gates = (k.gates + times - 1) / times;
        k.length = k.gates * k.gate_rows;
        k.count = (rows + k.length - 1) / k.length;
    }
    return k;
}

}  // namespace

namespace {

// How a call's rows are cut: accesses of 16, 8 or 4 bytes, as every row and length allows, or of one element.
struct RowPlan {
    int vec;    // elements of a piece
    bool cta;   // a row is a CTA's
    int elems;  // of a thread
    int lanes;  // threads of a row; 0: too long or too far apart, the kernels that read rows again
};
RowPlan row_plan(const ResidualProblem& pb, std::initializer_list<RowsRef> tensors, int size, int warp_elems, bool longer) {
    uintptr_t bits = (uintptr_t)(pb.d * size);
    bool wide = pb.rows >= (1ll << 30);  // (row numbers are 32 bits, and go past the end)
    for (const RowsRef& t : {pb.gate, pb.grad_gate}) wide = wide || (t.p != nullptr && t.ld * size >= (1ll << 32));
    for (const RowsRef& t : tensors) {
        bits |= (uintptr_t)t.p;
        if (t.p == nullptr || pb.rows <= 1) continue;
        bits |= (uintptr_t)(t.ld * size);
        wide = wide || t.ld * size >= (1ll << 32);
    }
    uintptr_t weights = 0;
    for (const float* w : {pb.w_post, pb.w_pre}) weights |= (uintptr_t)w;
    RowPlan p;
    const bool w16 = (weights & 15) == 0;
    p.vec = (bits & 15) == 0 && w16 ? 16 / size : (bits & 7) == 0 && (size == 4 || w16) ? 8 / size : (bits & 3) == 0 ? 4 / size : 1;
    // smaller pieces make longer code of as many elements: half of them where that is enough threads
    const bool few = p.vec * size < 16 && pb.d <= 8 * kMaxLanes;
    if (few) warp_elems = 8;
    p.cta = pb.d > 32 * warp_elems;
    p.elems = p.cta ? (few ? 8 : kRowElems) : warp_elems;
    if (longer && p.vec * size == 16 && pb.d > p.elems * kMaxLanes) p.elems = 2 * kRowElems;
    if (pb.d > p.elems * kMaxLanes || wide) {
        p.lanes = 0;
    } else if (p.cta) {
        p.lanes = (int)((pb.d + p.elems - 1) / p.elems + 31) / 32 * 32;
    } else {
        p.lanes = p.vec < 8 ? 8 / p.vec : 1;  // (what shares an evaluation of the dropout's generator)
        while (p.lanes * p.elems < pb.d) p.lanes *= 2;
    }
    return p;
}

int stages_for(size_t stage_bytes) { return 2 * stage_bytes <= (200u << 10) ? 2 : 1; }

template <class K>
cudaError_t allow_shared(K kernel, size_t smem) {
    if (smem <= (40u << 10)) return cudaSuccess;  // (48 KB with the static part)
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
}

// One of the kernels of the usual calls, by layer norm, dropout, gate vectors.
#define ROBE_USUAL(name, T, V, E, CTA, pb)                                                                           \
    ((pb).layer ? ((pb).drop.none ? ((pb).gate_kind == 2 ? name<T, V, E, CTA, true, 1, 0, 1> : name<T, V, E, CTA, true, 1, 0, 0>)   \
                                  : ((pb).gate_kind == 2 ? name<T, V, E, CTA, true, 1, 1, 1> : name<T, V, E, CTA, true, 1, 1, 0>))  \
                : ((pb).drop.none ? ((pb).gate_kind == 2 ? name<T, V, E, CTA, true, 0, 0, 1> : name<T, V, E, CTA, true, 0, 0, 0>)   \
                                  : ((pb).gate_kind == 2 ? name<T, V, E, CTA, true, 0, 1, 1> : name<T, V, E, CTA, true, 0, 1, 0>)))

template <class T, int V, int E, bool CTA>
cudaError_t launch_forward_rows(const ResidualProblem& pb, const RowPlan& p, cudaStream_t st) {
    const bool usual = V * sizeof(T) == 16 && pb.w_post != nullptr && pb.w_pre != nullptr && pb.residual.p != nullptr;
    const int threads = CTA ? p.lanes : kWarpRowThreads;
    void (*kernel)(ResidualProblem, int, int) = residual_rows_kernel<T, V, E, CTA, false, 0, 0, 1>;
    int slots = 3 * E * (int)sizeof(T);
    if constexpr (V * sizeof(T) == 16 && E <= kRowElems) {
        if (usual) {
            kernel = ROBE_USUAL(residual_rows_kernel, T, V, E, CTA, pb);
            if (pb.gate_kind != 2) slots = 2 * E * (int)sizeof(T);
        }
    }
    const size_t stage = (size_t)slots * threads;
    const int stages = stages_for(stage);
    cudaError_t e = allow_shared(kernel, stage * stages);
    if (e != cudaSuccess) return e;
    const int64_t groups = CTA ? 1 : kWarpRowThreads / p.lanes;
    int64_t grid = (pb.rows + groups - 1) / groups;
    if (grid > 148) {  // CTAs that stay: no more than are resident at once
        int per_sm = 1;
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, stage * stages);
        if (e != cudaSuccess) return e;
        if (grid > 148ll * per_sm) grid = 148ll * per_sm;
    }
    launch_next(kernel, (unsigned)grid, threads, stage * stages, st, pb, p.lanes, stages);
    return cudaGetLastError();
}
template <class T, int V>
cudaError_t launch_forward_rows(const ResidualProblem& pb, const RowPlan& p, cudaStream_t st) {
    constexpr int kSmall = V * sizeof(T) < 16 ? 8 : kRowElems;
    if (!p.cta) return launch_forward_rows<T, V, kSmall, false>(pb, p, st);  // (rows this short: small pieces always take 8)
    if constexpr (V * sizeof(T) == 16)
        if (p.elems == 2 * kRowElems) return launch_forward_rows<T, V, 2 * kRowElems, true>(pb, p, st);
    return p.elems == 8 ? launch_forward_rows<T, V, kSmall, true>(pb, p, st) : launch_forward_rows<T, V, kRowElems, true>(pb, p, st);
}

}  // namespace

cudaError_t launch_residual_forward(const ResidualProblem& pb, int dtype, cudaStream_t st) {
    const RowPlan p = row_plan(pb, {pb.x, pb.residual, pb.gate_kind == 2 ? pb.gate : RowsRef{}, pb.out, pb.normed},
                               dtype == 0 ? 4 : 2, kRowElems, true);
    if (p.lanes > 0) {
        if (dtype == 0)
            return p.vec == 4   ? launch_forward_rows<float, 4>(pb, p, st)
                   : p.vec == 2 ? launch_forward_rows<float, 2>(pb, p, st)
                                : launch_forward_rows<float, 1>(pb, p, st);
        return p.vec == 8   ? launch_forward_rows<__nv_bfloat16, 8>(pb, p, st)
               : p.vec == 4 ? launch_forward_rows<__nv_bfloat16, 4>(pb, p, st)
               : p.vec == 2 ? launch_forward_rows<__nv_bfloat16, 2>(pb, p, st)
                            : launch_forward_rows<__nv_bfloat16, 1>(pb, p, st);
    }
    const unsigned grid = (unsigned)(pb.rows < 148 * 4 ? pb.rows : 148 * 4);
    const bool pieces = p.vec * (dtype == 0 ? 4 : 2) == 16;
    void (*kernel)(ResidualProblem) = dtype == 0 ? (pieces ? residual_any_kernel<float, true> : residual_any_kernel<float, false>)
                                      : pieces   ? residual_any_kernel<__nv_bfloat16, true>
                                                 : residual_any_kernel<__nv_bfloat16, false>;
    launch_next(kernel, grid, kAnyThreads, 0, st, pb);
    return cudaGetLastError();
}

size_t residual_workspace_bytes(int64_t rows, int64_t d, int64_t gates) {
    if (rows <= 0 || d <= 0) return 0;
    int64_t count = 0;  // (enough for a gate per row, per element, or none alike, and for either kernel)
    for (const bool vector : {false, true})
        for (const bool again : {false, true}) {
            const int64_t n = chunks_of(rows, d, gates < rows ? gates : 0, vector, again).count;
            if (n > count) count = n;
        }
    const unsigned __int128 bytes = (unsigned __int128)count * d * sizeof(float) * 3;
    if (bytes >= ((unsigned __int128)1 << 62)) return (size_t)1 << 62;
    return ((size_t)bytes + 255) / 256 * 256;
}

namespace {

template <class T, bool PIECES>
cudaError_t launch_backward_any(const JoinGradArgs& a, cudaStream_t st) {
    const size_t sums = (size_t)a.p.d * 3 * sizeof(float);
    if (sums > (200u << 10)) {
        launch_next(residual_grad_any_kernel<T, PIECES, false>, (unsigned)a.chunks.count, kAnyThreads, 0, st, a);
        return cudaGetLastError();
    }
    const cudaError_t e = allow_shared(residual_grad_any_kernel<T, PIECES, true>, sums);
    if (e != cudaSuccess) return e;
    launch_next(residual_grad_any_kernel<T, PIECES, true>, (unsigned)a.chunks.count, kAnyThreads, sums, st, a);
    return cudaGetLastError();
}

template <class T, int V, int E, bool CTA>
cudaError_t launch_backward_rows(const JoinGradArgs& a, const RowPlan& p, cudaStream_t st) {
    const ResidualProblem& pb = a.p;
    // the call of a training step, 16-byte pieces: both norms, both gradients, nothing left to ask in the row loop
    const bool usual = V * sizeof(T) == 16 && pb.w_post != nullptr && pb.w_pre != nullptr && pb.grad_out.p != nullptr &&
                       pb.grad_residual.p != nullptr;
    const int threads = CTA ? p.lanes : kWarpRowThreads;
    void (*kernel)(JoinGradArgs, int, int) = residual_grad_rows_kernel<T, V, E, CTA, false, 0, 0, 1>;
    int slots = 5 * E * (int)sizeof(T);
    if constexpr (V * sizeof(T) == 16 && E <= kRowElems) {
        if (usual) {
            kernel = ROBE_USUAL(residual_grad_rows_kernel, T, V, E, CTA, pb);
            if (pb.gate_kind != 2) slots = 4 * E * (int)sizeof(T);
        }
    }
    const size_t stage = (size_t)slots * threads;
    const int stages = stages_for(stage);
    size_t smem = stage * stages;
    if (!CTA) {  // (the groups' sums go through the same memory)
        const size_t sums = (size_t)kWarpRowThreads / p.lanes * pb.d * sizeof(float);
        if (smem < sums) smem = sums;
    }
    const cudaError_t e = allow_shared(kernel, smem);
    if (e != cudaSuccess) return e;
    launch_next(kernel, (unsigned)a.chunks.count, threads, smem, st, a, p.lanes, stages);
    return cudaGetLastError();
}
template <class T, int V>
cudaError_t launch_backward_rows(const JoinGradArgs& a, const RowPlan& p, cudaStream_t st) {
    constexpr int kSmall = V * sizeof(T) < 16 ? 8 : kRowElems;
    if (!p.cta) return launch_backward_rows<T, V, kGradWarpElems, false>(a, p, st);
    if constexpr (V * sizeof(T) == 16 && sizeof(T) == 2)
        if (p.elems == 2 * kRowElems) return launch_backward_rows<T, V, 2 * kRowElems, true>(a, p, st);
    return p.elems == 8 ? launch_backward_rows<T, V, kSmall, true>(a, p, st) : launch_backward_rows<T, V, kRowElems, true>(a, p, st);
}

}  // namespace

cudaError_t launch_residual_backward(const ResidualProblem& pb, int dtype, void* workspace, cudaStream_t st) {
    JoinGradArgs a;
    a.p = pb;
    const RowPlan p = row_plan(pb, {pb.x, pb.grad_out, pb.out, pb.grad_normed, pb.gate_kind == 2 ? pb.gate : RowsRef{}, pb.grad_x,
                                    pb.grad_residual, pb.gate_kind == 2 ? pb.grad_gate : RowsRef{}},
                               dtype == 0 ? 4 : 2, kGradWarpElems, dtype == 1);
    a.chunks = chunks_of(pb.rows, pb.d, pb.gate_kind == 2 && pb.gate_rows > 1 ? pb.rows / pb.gate_rows : 0, pb.gate_kind == 2,
                         p.lanes == 0);
    a.part_post = (float*)workspace;
    a.part_pre = a.part_post + a.chunks.count * pb.d;
    a.part_gate = a.part_pre + a.chunks.count * pb.d;
    ColumnArgs c;
    c.j = a;
    c.weights = (pb.w_post != nullptr) + (pb.w_pre != nullptr);
    c.weight_tiles = (uint32_t)((pb.d + kColumnThreads / 16 - 1) / (kColumnThreads / 16));
    c.gate_share = a.chunks.per_gate > 64 ? 16 : 2;
    c.gate_tiles = (uint32_t)((pb.d + kColumnThreads / c.gate_share - 1) / (kColumnThreads / c.gate_share));
    int64_t grid = (int64_t)c.weights * c.weight_tiles;
    if (pb.gate_kind == 2 && pb.gate_rows > 1 && pb.grad_gate.p != nullptr && a.chunks.per_gate > 0)
        grid += pb.rows / pb.gate_rows * c.gate_tiles;
    if (grid >= (1ll << 31)) return kGridTooSmall;
    cudaError_t e = cudaSuccess;
    if (a.chunks.count == 0) {
    } else if (p.lanes > 0) {
        if (dtype == 0)
            e = p.vec == 4   ? launch_backward_rows<float, 4>(a, p, st)
                : p.vec == 2 ? launch_backward_rows<float, 2>(a, p, st)
                             : launch_backward_rows<float, 1>(a, p, st);
        else
            e = p.vec == 8   ? launch_backward_rows<__nv_bfloat16, 8>(a, p, st)
                : p.vec == 4 ? launch_backward_rows<__nv_bfloat16, 4>(a, p, st)
                : p.vec == 2 ? launch_backward_rows<__nv_bfloat16, 2>(a, p, st)
                             : launch_backward_rows<__nv_bfloat16, 1>(a, p, st);
    } else {
        const bool pieces = p.vec * (dtype == 0 ? 4 : 2) == 16;
        e = dtype == 0 ? (pieces ? launch_backward_any<float, true>(a, st) : launch_backward_any<float, false>(a, st))
            : pieces   ? launch_backward_any<__nv_bfloat16, true>(a, st)
                       : launch_backward_any<__nv_bfloat16, false>(a, st);
    }
    if (e != cudaSuccess) return e;
    if (grid > 0) {
        if (dtype == 0) launch_next(residual_columns_kernel<float>, (unsigned)grid, kColumnThreads, 0, st, c);
        else launch_next(residual_columns_kernel<__nv_bfloat16>, (unsigned)grid, kColumnThreads, 0, st, c);
    }
    return cudaGetLastError();
}

}  // namespace robe
