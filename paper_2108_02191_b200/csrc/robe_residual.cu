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

constexpr int kJoinThreads = 256;

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

// ---- rows of any length, one CTA each, read again in every pass over the row: for rows too long for the kernels below

// Mean (0 without `layer`) and factor of the norm of a row whose elements `value` gives.
template <class F>
__device__ __forceinline__ void row_stats(F&& value, int64_t d, int layer, float eps, float* scratch, float& mean, float& rstd) {
    mean = 0.0f;
    if (layer) {
        float s = 0.0f;
        for (int64_t c = threadIdx.x; c < d; c += kJoinThreads) s += value(c);
        mean = block_sum(s, scratch) / (float)d;
    }
    float q = 0.0f;
    for (int64_t c = threadIdx.x; c < d; c += kJoinThreads) {
        const float v = value(c) - mean;
        q += v * v;
    }
    rstd = 1.0f / sqrtf(block_sum(q, scratch) / (float)d + eps);
}

__device__ __forceinline__ float drop_factor(const DropParams& drop, uint64_t offset, int64_t r, int64_t c) {
    if (drop.none) return 1.0f;
    const uint4 w = drop_words((uint32_t)r, (uint32_t)(c >> 3), offset, drop);
    return drop_keeps(w, (int)(c & 7), drop) ? drop.scale : 0.0f;
}
__device__ __forceinline__ float dropped(float v, float factor) { return factor == 0.0f ? 0.0f : v * factor; }

template <class T>
__device__ __forceinline__ float gate_of(const ResidualProblem& a, int64_t r, int64_t c) {
    if (a.gate_kind == 0) return 1.0f;
    const T* g = (const T*)a.gate.p + r / a.gate_rows * a.gate.ld;
    return widen(g[a.gate_kind == 1 ? 0 : c]);
}

template <class T>
__global__ void __launch_bounds__(kJoinThreads) residual_any_kernel(ResidualProblem a) {
    __shared__ float scratch[kJoinThreads / 32];
    follow();
    const uint64_t offset = drop_offset(a.drop);
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = (const T*)a.x.p + r * a.x.ld;
        const T* residual = a.residual.p != nullptr ? (const T*)a.residual.p + r * a.residual.ld : nullptr;
        float mean1 = 0.0f, rstd1 = 1.0f, mean2 = 0.0f, rstd2 = 1.0f;
        if (a.w_post != nullptr)
            row_stats([&](int64_t c) { return widen(x[c]); }, a.d, a.layer, a.eps, scratch, mean1, rstd1);
        auto joined = [&](int64_t c) {
            float y = widen(x[c]);
            if (a.w_post != nullptr) y = (y - mean1) * rstd1 * a.w_post[c];
            y = dropped(y, drop_factor(a.drop, offset, r, c)) * a.scale * gate_of<T>(a, r, c);
            return residual != nullptr ? widen(residual[c]) + y : y;
        };
        if (a.w_pre != nullptr) row_stats(joined, a.d, a.layer, a.eps, scratch, mean2, rstd2);
        for (int64_t c = threadIdx.x; c < a.d; c += kJoinThreads) {
            const float v = joined(c);
            ((T*)a.out.p)[r * a.out.ld + c] = narrow<T>(v);
            if (a.w_pre != nullptr) ((T*)a.normed.p)[r * a.normed.ld + c] = narrow<T>((v - mean2) * rstd2 * a.w_pre[c]);
        }
    }
}

// ---- rows kept close: `lanes` threads share a row, E elements each, which they copy to shared memory rows ahead and read
// from there; a thread reads what it copied itself, so nothing but the sums over a row is waited for together.  Up to 512
// elements (256 backward) a row is a part of a warp's, longer ones a CTA's, up to kMaxLanes E; beyond that the kernels for any length.

constexpr int kMaxLanes = 512;
constexpr int kWarpRowThreads = 256;

// Sums of N values over the threads of a row, in each of them.  CTA: by turns in two halves of `scratch`, so that one
// barrier a sum is enough.
template <bool CTA, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], int lanes, float (*scratch)[N][kMaxLanes / 32], int& turn) {
    if (CTA) {
#pragma unroll
        for (int s = 16; s > 0; s >>= 1)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], s);
        if (blockDim.x == 32) return;
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) scratch[turn][k][threadIdx.x >> 5] = v[k];
        __syncthreads();
        const int warps = blockDim.x >> 5;
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = 0.0f;
        for (int w = 0; w < warps; ++w)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += scratch[turn][k][w];
        turn ^= 1;
    } else {
        for (int s = lanes >> 1; s > 0; s >>= 1)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], s);
    }
}

// The rows' shared memory: [stage][tensor][piece][thread], V elements each.
template <class T, int V, int NP>
struct Ring {
    T* base;
    int tensors, lanes, lane;
    int64_t d;
    __device__ __forceinline__ T* at(int stage, int tensor, int k) const {
        return base + ((((size_t)stage * tensors + tensor) * NP + k) * blockDim.x + threadIdx.x) * V;
    }
    __device__ __forceinline__ int64_t col(int k) const { return (int64_t)(k * lanes + lane) * V; }
    __device__ __forceinline__ bool has(int k) const { return col(k) < d; }
    __device__ __forceinline__ void fetch(int stage, int tensor, const T* row) const {
#pragma unroll
        for (int k = 0; k < NP; ++k)
            if (has(k)) copy_async<V * sizeof(T)>(at(stage, tensor, k), row + col(k));
    }
    __device__ __forceinline__ Pack<T, V> read(int stage, int tensor, int k) const {
        return *(const Pack<T, V>*)at(stage, tensor, k);
    }
};

// What dropout multiplies the elements of a piece by.
template <int V>
__device__ __forceinline__ void drop_factors(float (&f)[V], const DropParams& drop, uint64_t offset, int64_t r, int64_t c) {
    const uint4 w = drop_words((uint32_t)r, (uint32_t)(c >> 3), offset, drop);
    const int first = (int)(c & 7);
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = drop_keeps(w, first + e, drop) ? drop.scale : 0.0f;
}
// fp32 weights of a piece (16-byte aligned from V = 4 on: the weights are, and columns are multiples of V)
template <int V>
__device__ __forceinline__ void weights_of(float (&w)[V], const float* p) {
    if constexpr (V >= 4) {
#pragma unroll
        for (int q = 0; q < V; q += 4) {
            const float4 x = __ldca((const float4*)(p + q));
            w[q] = x.x;
            w[q + 1] = x.y;
            w[q + 2] = x.z;
            w[q + 3] = x.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) w[e] = __ldca(p + e);
    }
}

template <class T, int V, int NP, bool CTA>
__global__ void __launch_bounds__(CTA ? kMaxLanes : kWarpRowThreads)
residual_rows_kernel(ResidualProblem a, int lanes, int stages) {
    extern __shared__ __align__(16) unsigned char ring_bytes[];
    __shared__ float scratch[2][1][kMaxLanes / 32];
    follow();
    const uint64_t offset = drop_offset(a.drop);
    const bool post = a.w_post != nullptr, pre = a.w_pre != nullptr, added = a.residual.p != nullptr;
    const int gate_at = added ? 2 : 1, tensors = gate_at + (a.gate_kind == 2);
    const Ring<T, V, NP> ring{(T*)ring_bytes, tensors, lanes, CTA ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1), a.d};
    const int groups = CTA ? 1 : kWarpRowThreads / lanes;
    const int64_t step = (int64_t)gridDim.x * groups;
    const int64_t first = (int64_t)blockIdx.x * groups + (CTA ? 0 : threadIdx.x / lanes);
    const float over_d = 1.0f / (float)a.d;
    int turn = 0;
    auto fetch = [&](int64_t r, int stage) {
        if (r < a.rows) {
            ring.fetch(stage, 0, (const T*)a.x.p + r * a.x.ld);
            if (added) ring.fetch(stage, 1, (const T*)a.residual.p + r * a.residual.ld);
            if (a.gate_kind == 2) ring.fetch(stage, gate_at, (const T*)a.gate.p + r / a.gate_rows * a.gate.ld);
        }
        copies_close();
    };
    for (int s = 0; s + 1 < stages; ++s) fetch(first + s * step, s);
    int stage = 0;
    // (a warp's groups go through as many rows as its first one: sums over lanes need them all)
    const int64_t leader = CTA ? first : (int64_t)blockIdx.x * groups + (threadIdx.x & ~31) / lanes;
    for (int64_t r0 = leader; r0 < a.rows; r0 += step) {
        const int64_t r = r0 + (first - leader);
        const bool here = r < a.rows;
        fetch(r + (int64_t)(stages - 1) * step, stage == 0 ? stages - 1 : stage - 1);
        copies_wait(stages - 1);
        float v[NP][V];
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            const Pack<T, V> e = ring.read(stage, 0, k);
#pragma unroll
            for (int c = 0; c < V; ++c) v[k][c] = here && ring.has(k) ? widen(e.v[c]) : 0.0f;
        }
        // norm of the row that v holds (0 beyond d): mean and factor
        auto stats = [&](float& mean, float& rstd) {
            float s[1];
            mean = 0.0f;
            if (a.layer) {
                s[0] = 0.0f;
#pragma unroll
                for (int k = 0; k < NP; ++k)
#pragma unroll
                    for (int c = 0; c < V; ++c) s[0] += v[k][c];
                row_sums<CTA, 1>(s, lanes, scratch, turn);
                mean = s[0] * over_d;
            }
            s[0] = 0.0f;
#pragma unroll
            for (int k = 0; k < NP; ++k)
#pragma unroll
                for (int c = 0; c < V; ++c) {
                    const float x = v[k][c] - mean;
                    s[0] += ring.has(k) ? x * x : 0.0f;
                }
            row_sums<CTA, 1>(s, lanes, scratch, turn);
            rstd = 1.0f / sqrtf(s[0] * over_d + a.eps);
        };
        float mean = 0.0f, rstd = 1.0f;
        if (post) stats(mean, rstd);
        float row_gate = a.scale;
        if (a.gate_kind == 1 && here) row_gate *= widen(((const T*)a.gate.p)[r * a.gate.ld]);
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            if (!ring.has(k) || !here) continue;
            const int64_t col = ring.col(k);
            if (post) {
                float w[V];
                weights_of<V>(w, a.w_post + col);
#pragma unroll
                for (int c = 0; c < V; ++c) v[k][c] = (v[k][c] - mean) * rstd * w[c];
            }
            if (!a.drop.none) {
                float f[V];
                drop_factors<V>(f, a.drop, offset, r, col);
#pragma unroll
                for (int c = 0; c < V; ++c) v[k][c] = dropped(v[k][c], f[c]);
            }
#pragma unroll
            for (int c = 0; c < V; ++c) v[k][c] *= row_gate;
            if (a.gate_kind == 2) {
                const Pack<T, V> g = ring.read(stage, gate_at, k);
#pragma unroll
                for (int c = 0; c < V; ++c) v[k][c] *= widen(g.v[c]);
            }
            if (added) {
                const Pack<T, V> e = ring.read(stage, 1, k);
#pragma unroll
                for (int c = 0; c < V; ++c) v[k][c] += widen(e.v[c]);
            }
            Pack<T, V> e;
#pragma unroll
            for (int c = 0; c < V; ++c) e.v[c] = narrow<T>(v[k][c]);
            store_pack<true, T, V>((T*)a.out.p + r * a.out.ld + col, e);
        }
        if (pre) {
            stats(mean, rstd);
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                if (!ring.has(k) || !here) continue;
                const int64_t col = ring.col(k);
                float w[V];
                weights_of<V>(w, a.w_pre + col);
                Pack<T, V> e;
#pragma unroll
                for (int c = 0; c < V; ++c) e.v[c] = narrow<T>((v[k][c] - mean) * rstd * w[c]);
                store_pack<true, T, V>((T*)a.normed.p + r * a.normed.ld + col, e);
            }
        }
        stage = stage + 1 == stages ? 0 : stage + 1;
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

template <class T>
__global__ void __launch_bounds__(kJoinThreads) residual_grad_any_kernel(JoinGradArgs args) {
    __shared__ float scratch[kJoinThreads / 32];
    follow();
    const ResidualProblem& a = args.p;
    const uint64_t offset = drop_offset(a.drop);
    const float over_d = 1.0f / (float)a.d;
    const int64_t r0 = args.chunks.row0(blockIdx.x), r1 = args.chunks.row1(blockIdx.x);
    float* part_post = args.part_post + blockIdx.x * a.d;
    float* part_pre = args.part_pre + blockIdx.x * a.d;
    float* part_gate = args.part_gate + blockIdx.x * a.d;
    for (int64_t r = r0; r < r1; ++r) {
        const T* x = (const T*)a.x.p + r * a.x.ld;
        const T* out = (const T*)a.out.p + r * a.out.ld;
        const T* go = a.grad_out.p != nullptr ? (const T*)a.grad_out.p + r * a.grad_out.ld : nullptr;
        const T* gn = (const T*)a.grad_normed.p + r * a.grad_normed.ld;
        float mean1 = 0.0f, rstd1 = 1.0f, mean2 = 0.0f, rstd2 = 1.0f, dot2 = 0.0f, sum2 = 0.0f;
        if (a.w_pre != nullptr) {
            row_stats([&](int64_t c) { return widen(out[c]); }, a.d, a.layer, a.eps, scratch, mean2, rstd2);
            float dot = 0.0f, sum = 0.0f;
            for (int64_t c = threadIdx.x; c < a.d; c += kJoinThreads) {
                const float g = widen(gn[c]) * a.w_pre[c];
                dot += g * ((widen(out[c]) - mean2) * rstd2);
                sum += g;
            }
            dot2 = block_sum(dot, scratch) * over_d;
            if (a.layer) sum2 = block_sum(sum, scratch) * over_d;
        }
        auto total = [&](int64_t c) {  // gradient of `out` from both sides
            float t = go != nullptr ? widen(go[c]) : 0.0f;
            if (a.w_pre != nullptr) {
                const float n = (widen(out[c]) - mean2) * rstd2;
                t += rstd2 * (widen(gn[c]) * a.w_pre[c] - sum2 - n * dot2);
            }
            return t;
        };
        if (a.w_post != nullptr)
            row_stats([&](int64_t c) { return widen(x[c]); }, a.d, a.layer, a.eps, scratch, mean1, rstd1);
        float dot = 0.0f, sum = 0.0f, gate_sum = 0.0f;
        for (int64_t c = threadIdx.x; c < a.d; c += kJoinThreads) {
            const float t = total(c), f = drop_factor(a.drop, offset, r, c);
            const float n = (widen(x[c]) - mean1) * rstd1;
            const float w = a.w_post != nullptr ? a.w_post[c] : 1.0f;
            const float g = dropped(t * a.scale * gate_of<T>(a, r, c), f) * w;
            dot += g * n;
            sum += g;
            gate_sum += dropped(n * w, f) * (a.scale * t);
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
        const int64_t in_gate = r % args.chunks.gate_rows;
        for (int64_t c = threadIdx.x; c < a.d; c += kJoinThreads) {
            const float t = total(c), f = drop_factor(a.drop, offset, r, c);
            const float n = (widen(x[c]) - mean1) * rstd1;
            const float w = a.w_post != nullptr ? a.w_post[c] : 1.0f;
            const float u = dropped(t * a.scale * gate_of<T>(a, r, c), f);
            if (a.w_pre != nullptr) {
                const float v = widen(gn[c]) * ((widen(out[c]) - mean2) * rstd2);
                part_pre[c] = (r == r0 ? 0.0f : part_pre[c]) + v;
            }
            if (a.gate_kind == 2 && a.grad_gate.p != nullptr) {
                float v = dropped(n * w, f) * (a.scale * t);
                if (r != r0 && in_gate != 0) v += part_gate[c];
                part_gate[c] = v;
                if (args.chunks.per_gate == 0 && in_gate == args.chunks.gate_rows - 1)
                    ((T*)a.grad_gate.p)[r / args.chunks.gate_rows * a.grad_gate.ld + c] = narrow<T>(v);
            }
            float gx = u;
            if (a.w_post != nullptr) {
                part_post[c] = (r == r0 ? 0.0f : part_post[c]) + u * n;
                gx = rstd1 * (u * w - sum1 - n * dot1);
            }
            if (a.grad_residual.p != nullptr) ((T*)a.grad_residual.p)[r * a.grad_residual.ld + c] = narrow<T>(t);
            ((T*)a.grad_x.p)[r * a.grad_x.ld + c] = narrow<T>(gx);
        }
    }
}

// One CTA per chunk.  The weights' gradients of a thread's columns are summed in registers over its rows, over the groups of
// a CTA in shared memory, over the chunks by the kernel below; a gate vector's likewise, or stored when its rows are done.
template <class T, int V, int NP, bool CTA>
__global__ void __launch_bounds__(CTA ? kMaxLanes : kWarpRowThreads)
residual_grad_rows_kernel(JoinGradArgs args, int lanes, int stages) {
    extern __shared__ __align__(16) unsigned char ring_bytes[];
    __shared__ float scratch[2][3][kMaxLanes / 32];
    follow();
    const ResidualProblem& a = args.p;
    const uint64_t offset = drop_offset(a.drop);
    const bool post = a.w_post != nullptr, pre = a.w_pre != nullptr, skip = a.grad_out.p != nullptr;
    const bool gate_sums = a.gate_kind == 2 && a.grad_gate.p != nullptr && args.chunks.gate_rows > 1;
    const bool whole_gates = args.chunks.per_gate == 0;
    const int skip_at = 1, out_at = skip_at + skip, normed_at = out_at + pre, gate_at = normed_at + pre;
    const int tensors = gate_at + (a.gate_kind == 2);
    const Ring<T, V, NP> ring{(T*)ring_bytes, tensors, lanes, CTA ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1), a.d};
    const int groups = CTA ? 1 : kWarpRowThreads / lanes;
    const int group = CTA ? 0 : threadIdx.x / lanes;
    const float over_d = 1.0f / (float)a.d;
    // the rows of a group: every groups-th of the chunk, or whole gate vectors in turn
    const int64_t c0 = args.chunks.row0(blockIdx.x), c1 = args.chunks.row1(blockIdx.x);
    const int64_t block = gate_sums && whole_gates ? args.chunks.gate_rows : 1;
    auto row_of = [&](int64_t k) {  // k-th row of this group, c1 or more beyond the last
        return block == 1 ? c0 + k * groups + group : c0 + ((k / block) * groups + group) * block + k % block;
    };
    // (as many rounds for all groups: sums over lanes need whole warps)
    const int64_t rounds = ((c1 - c0 + block - 1) / block + groups - 1) / groups * block;
    int turn = 0;
    float sum_post[NP][V], sum_pre[NP][V], sum_gate[NP][V];
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
        for (int c = 0; c < V; ++c) sum_post[k][c] = sum_pre[k][c] = sum_gate[k][c] = 0.0f;
    auto fetch = [&](int64_t k, int stage) {
        const int64_t r = row_of(k);
        if (k < rounds && r < c1) {
            ring.fetch(stage, 0, (const T*)a.x.p + r * a.x.ld);
            if (skip) ring.fetch(stage, skip_at, (const T*)a.grad_out.p + r * a.grad_out.ld);
            if (pre) {
                ring.fetch(stage, out_at, (const T*)a.out.p + r * a.out.ld);
                ring.fetch(stage, normed_at, (const T*)a.grad_normed.p + r * a.grad_normed.ld);
            }
            if (a.gate_kind == 2) ring.fetch(stage, gate_at, (const T*)a.gate.p + r / a.gate_rows * a.gate.ld);
        }
        copies_close();
    };
    for (int s = 0; s + 1 < stages; ++s) fetch(s, s);
    int stage = 0;
    for (int64_t q = 0; q < rounds; ++q) {
        const int64_t r = row_of(q);
        const bool here = r < c1;
        fetch(q + stages - 1, stage == 0 ? stages - 1 : stage - 1);
        copies_wait(stages - 1);
        float x[NP][V], t[NP][V];  // x, then its norm; out, its norm, then the gradient of out
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            const bool in = here && ring.has(k);
            const Pack<T, V> e = ring.read(stage, 0, k);
#pragma unroll
            for (int c = 0; c < V; ++c) x[k][c] = in ? widen(e.v[c]) : 0.0f;
            if (pre) {
                const Pack<T, V> o = ring.read(stage, out_at, k);
#pragma unroll
                for (int c = 0; c < V; ++c) t[k][c] = in ? widen(o.v[c]) : 0.0f;
            } else {
#pragma unroll
                for (int c = 0; c < V; ++c) t[k][c] = 0.0f;
            }
        }
        float s[3] = {0.0f, 0.0f, 0.0f};
        float mean1 = 0.0f, mean2 = 0.0f;
        if (a.layer) {
#pragma unroll
            for (int k = 0; k < NP; ++k)
#pragma unroll
                for (int c = 0; c < V; ++c) {
                    s[0] += x[k][c];
                    s[1] += t[k][c];
                }
            row_sums<CTA, 3>(s, lanes, scratch, turn);
            if (post) mean1 = s[0] * over_d;
            mean2 = s[1] * over_d;
        }
        s[0] = s[1] = s[2] = 0.0f;
#pragma unroll
        for (int k = 0; k < NP; ++k)
#pragma unroll
            for (int c = 0; c < V; ++c) {
                x[k][c] = ring.has(k) ? x[k][c] - mean1 : 0.0f;
                t[k][c] = ring.has(k) ? t[k][c] - mean2 : 0.0f;
                s[0] += x[k][c] * x[k][c];
                s[1] += t[k][c] * t[k][c];
            }
        row_sums<CTA, 3>(s, lanes, scratch, turn);
        const float rstd1 = post ? 1.0f / sqrtf(s[0] * over_d + a.eps) : 1.0f;
        const float rstd2 = pre ? 1.0f / sqrtf(s[1] * over_d + a.eps) : 1.0f;
        if (pre) {
            s[0] = s[1] = s[2] = 0.0f;
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                if (!ring.has(k) || !here) continue;
                const Pack<T, V> g = ring.read(stage, normed_at, k);
                float w[V];
                weights_of<V>(w, a.w_pre + ring.col(k));
#pragma unroll
                for (int c = 0; c < V; ++c) {
                    t[k][c] *= rstd2;
                    const float gn = widen(g.v[c]);
                    sum_pre[k][c] += gn * t[k][c];
                    s[0] += gn * w[c] * t[k][c];
                    s[1] += gn * w[c];
                }
            }
            row_sums<CTA, 3>(s, lanes, scratch, turn);
            const float dot = s[0] * over_d, sum = a.layer ? s[1] * over_d : 0.0f;
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                if (!ring.has(k) || !here) continue;
                const Pack<T, V> g = ring.read(stage, normed_at, k);
                float w[V];
                weights_of<V>(w, a.w_pre + ring.col(k));
#pragma unroll
                for (int c = 0; c < V; ++c) t[k][c] = rstd2 * (widen(g.v[c]) * w[c] - sum - t[k][c] * dot);
            }
        }
        float row_gate = 1.0f;
        if (a.gate_kind == 1 && here) row_gate = widen(((const T*)a.gate.p)[r * a.gate.ld]);
        s[0] = s[1] = s[2] = 0.0f;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            if (!ring.has(k) || !here) continue;
            const int64_t col = ring.col(k);
            if (skip) {
                const Pack<T, V> e = ring.read(stage, skip_at, k);
#pragma unroll
                for (int c = 0; c < V; ++c) t[k][c] += widen(e.v[c]);
            }
            if (a.grad_residual.p != nullptr) {
                Pack<T, V> e;
#pragma unroll
                for (int c = 0; c < V; ++c) e.v[c] = narrow<T>(t[k][c]);
                store_pack<true, T, V>((T*)a.grad_residual.p + r * a.grad_residual.ld + col, e);
            }
            float w[V], f[V];
#pragma unroll
            for (int c = 0; c < V; ++c) w[c] = f[c] = 1.0f;
            if (post) weights_of<V>(w, a.w_post + col);
            if (!a.drop.none) drop_factors<V>(f, a.drop, offset, r, col);
            if (a.gate_kind == 2) {
                const Pack<T, V> g = ring.read(stage, gate_at, k);
                Pack<T, V> e;
#pragma unroll
                for (int c = 0; c < V; ++c) {
                    x[k][c] *= rstd1;
                    const float st = a.scale * t[k][c];
                    const float gg = dropped(x[k][c] * w[c], f[c]) * st;
                    sum_gate[k][c] += gg;
                    e.v[c] = narrow<T>(gg);
                    t[k][c] = dropped(st * widen(g.v[c]), f[c]);
                }
                if (a.grad_gate.p != nullptr && args.chunks.gate_rows == 1)
                    store_pack<true, T, V>((T*)a.grad_gate.p + r * a.grad_gate.ld + col, e);
            } else {
#pragma unroll
                for (int c = 0; c < V; ++c) {
                    x[k][c] *= rstd1;
                    const float st = a.scale * t[k][c];
                    s[2] += dropped(x[k][c] * w[c], f[c]) * st;
                    t[k][c] = dropped(st * row_gate, f[c]);
                }
            }
            if (post) {
#pragma unroll
                for (int c = 0; c < V; ++c) {
                    sum_post[k][c] += t[k][c] * x[k][c];
                    t[k][c] *= w[c];
                    s[0] += t[k][c] * x[k][c];
                    s[1] += t[k][c];
                }
            }
        }
        if (post || a.gate_kind == 1) row_sums<CTA, 3>(s, lanes, scratch, turn);
        if (a.gate_kind == 1 && a.grad_gate.p != nullptr && here && ring.lane == 0)
            ((T*)a.grad_gate.p)[r * a.grad_gate.ld] = narrow<T>(s[2]);
        const float dot = post ? s[0] * over_d : 0.0f, sum = post && a.layer ? s[1] * over_d : 0.0f;
        const bool gate_done = gate_sums && whole_gates && q % block == block - 1 && here;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            if (!ring.has(k) || !here) continue;
            Pack<T, V> e;
#pragma unroll
            for (int c = 0; c < V; ++c) e.v[c] = narrow<T>(post ? rstd1 * (t[k][c] - sum - x[k][c] * dot) : t[k][c]);
            store_pack<true, T, V>((T*)a.grad_x.p + r * a.grad_x.ld + ring.col(k), e);
            if (gate_done) {
#pragma unroll
                for (int c = 0; c < V; ++c) {
                    e.v[c] = narrow<T>(sum_gate[k][c]);
                    sum_gate[k][c] = 0.0f;
                }
                store_pack<true, T, V>((T*)a.grad_gate.p + r / args.chunks.gate_rows * a.grad_gate.ld + ring.col(k), e);
            }
        }
        stage = stage + 1 == stages ? 0 : stage + 1;
    }
    copies_wait(0);
    // the chunk's sums
    auto store_sums = [&](const float (&v)[NP][V], float* part) {
        part += blockIdx.x * a.d;
        if (CTA) {
#pragma unroll
            for (int k = 0; k < NP; ++k)
                if (ring.has(k))
#pragma unroll
                    for (int c = 0; c < V; ++c) part[ring.col(k) + c] = v[k][c];
            return;
        }
        float* sums = (float*)ring_bytes;  // [groups][d]
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NP; ++k)
            if (ring.has(k))
#pragma unroll
                for (int c = 0; c < V; ++c) sums[group * a.d + ring.col(k) + c] = v[k][c];
        __syncthreads();
        for (int64_t c = threadIdx.x; c < a.d; c += kWarpRowThreads) {
            float s = 0.0f;
            for (int g = 0; g < groups; ++g) s += sums[g * a.d + c];
            part[c] = s;
        }
    };
    if (post) store_sums(sum_post, args.part_post);
    if (pre) store_sums(sum_pre, args.part_pre);
    if (gate_sums && !whole_gates) store_sums(sum_gate, args.part_gate);
}

// Columns of [parts][d] summed: blockIdx.y = 0 the weights after the block, 1 those before the next, 2.. gate vectors.
constexpr int kColumnLanes = 32, kColumnRows = 16;

template <class T>
__global__ void __launch_bounds__(kColumnLanes* kColumnRows) residual_columns_kernel(JoinGradArgs args) {
    __shared__ double sums[kColumnRows][kColumnLanes];
    follow();
    const ResidualProblem& a = args.p;
    const int lane = threadIdx.x % kColumnLanes, row = threadIdx.x / kColumnLanes;
    const uint32_t tiles = (uint32_t)((a.d + kColumnLanes - 1) / kColumnLanes);
    const uint32_t what = blockIdx.x / tiles;
    const int64_t c = (int64_t)(blockIdx.x % tiles) * kColumnLanes + lane;
    const int weights = (a.w_post != nullptr) + (a.w_pre != nullptr);
    const bool post = what == 0 && a.w_post != nullptr;
    const bool gate = (int)what >= weights;
    const int64_t first = gate ? (what - weights) * args.chunks.per_gate : 0;
    const int64_t count = gate ? args.chunks.per_gate : args.chunks.count;
    const float* part = (gate ? args.part_gate : post ? args.part_post : args.part_pre) + first * a.d;
    double s = 0.0;
    if (c < a.d)
        for (int64_t k = row; k < count; k += kColumnRows) s += (double)__ldcs(part + k * a.d + c);
    sums[row][lane] = s;
    __syncthreads();
    if (row != 0 || c >= a.d) return;
    s = 0.0;
    for (int k = 0; k < kColumnRows; ++k) s += sums[k][lane];
    if (gate) ((T*)a.grad_gate.p)[(what - weights) * a.grad_gate.ld + c] = narrow<T>((float)s);
    else (post ? a.grad_w_post : a.grad_w_pre)[c] = (float)s;
}

constexpr int64_t kMaxChunks = 592;  // four CTAs for each of 148 SMs

Chunks chunks_of(int64_t rows, int64_t gates) {
    Chunks k;
    k.rows = rows;
    k.gate_rows = gates > 0 ? rows / gates : rows;
    k.per_gate = k.gates = k.length = k.count = 0;
    if (rows == 0) return k;
    int64_t length = (rows + kMaxChunks - 1) / kMaxChunks;
    if (gates == 0 || k.gate_rows > length) {
        k.gates = 0;
        k.per_gate = (k.gate_rows + length - 1) / length;
        k.length = (k.gate_rows + k.per_gate - 1) / k.per_gate;
        k.count = (gates > 0 ? gates : 1) * k.per_gate;
    } else {
        k.per_gate = 0;
        k.gates = (length + k.gate_rows - 1) / k.gate_rows;
        k.length = k.gates * k.gate_rows;
        k.count = (rows + k.length - 1) / k.length;
    }
    return k;
}

}  // namespace

namespace {

// How a call's rows are cut: V elements an access (16 bytes where every row and length allows, else 4, else one element).
struct RowPlan {
    int vec;    // elements of a piece
    bool cta;   // a row is a CTA's
    int lanes;  // threads of a row; 0: too long, the kernels that read rows again
};
RowPlan row_plan(const ResidualProblem& pb, std::initializer_list<RowsRef> tensors, int size, int warp_elems, int cta_elems) {
    uintptr_t bits = (uintptr_t)(pb.d * size);
    for (const RowsRef& t : tensors) {
        bits |= (uintptr_t)t.p;
        if (t.p != nullptr && pb.rows > 1) bits |= (uintptr_t)(t.ld * size);
    }
    uintptr_t weights = 0;
    for (const float* w : {pb.w_post, pb.w_pre}) weights |= (uintptr_t)w;
    RowPlan p;
    p.vec = (bits & 15) == 0 && (weights & 15) == 0 ? 16 / size : (bits & 3) == 0 ? 4 / size : 1;
    p.cta = pb.d > 32 * warp_elems;
    const int64_t per = p.cta ? cta_elems : warp_elems;
    if (pb.d > per * kMaxLanes) {
        p.lanes = 0;
    } else if (p.cta) {
        p.lanes = (int)((pb.d + per - 1) / per + 31) / 32 * 32;
    } else {
        p.lanes = 1;
        while (p.lanes < 32 && p.lanes * per < pb.d) p.lanes *= 2;
    }
    return p;
}

constexpr size_t kRingBytes = 96 << 10;  // of a CTA: two fit an SM
int stages_for(size_t stage_bytes) {
    const size_t n = kRingBytes / stage_bytes;
    return n >= 3 ? 3 : n == 2 ? 2 : 2 * stage_bytes <= (200u << 10) ? 2 : 1;
}

template <class K, class A>
cudaError_t launch_ring(K* kernel, unsigned grid, int threads, size_t smem, cudaStream_t st, const A& a, int lanes, int stages) {
    if (smem > (40u << 10)) {  // (48 KB with the static part)
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    launch_next(kernel, grid, threads, smem, st, a, lanes, stages);
    return cudaGetLastError();
}

template <class T, int V>
cudaError_t launch_forward_rows(const ResidualProblem& pb, const RowPlan& p, cudaStream_t st) {
    constexpr int E = 16;
    const int threads = p.cta ? p.lanes : kWarpRowThreads;
    const int tensors = 1 + (pb.residual.p != nullptr) + (pb.gate_kind == 2);
    const size_t stage = (size_t)tensors * E * sizeof(T) * threads;
    const int stages = stages_for(stage);
    const int64_t groups = p.cta ? 1 : kWarpRowThreads / p.lanes;
    const int64_t want = (pb.rows + groups - 1) / groups;
    int64_t per_sm = (int64_t)((220u << 10) / (stage * stages + 1024));
    if (per_sm > 2048 / threads) per_sm = 2048 / threads;
    if (per_sm < 1) per_sm = 1;
    const unsigned grid = (unsigned)(want < 148 * per_sm ? want : 148 * per_sm);
    if (p.cta) return launch_ring(residual_rows_kernel<T, V, E / V, true>, grid, threads, stage * stages, st, pb, p.lanes, stages);
    return launch_ring(residual_rows_kernel<T, V, E / V, false>, grid, threads, stage * stages, st, pb, p.lanes, stages);
}

}  // namespace

cudaError_t launch_residual_forward(const ResidualProblem& pb, int dtype, cudaStream_t st) {
    const RowPlan p = row_plan(pb, {pb.x, pb.residual, pb.gate_kind == 2 ? pb.gate : RowsRef{}, pb.out, pb.normed},
                               dtype == 0 ? 4 : 2, 16, 16);
    if (p.lanes > 0) {
        if (dtype == 0) return p.vec == 4 ? launch_forward_rows<float, 4>(pb, p, st) : launch_forward_rows<float, 1>(pb, p, st);
        return p.vec == 8   ? launch_forward_rows<__nv_bfloat16, 8>(pb, p, st)
               : p.vec == 2 ? launch_forward_rows<__nv_bfloat16, 2>(pb, p, st)
                            : launch_forward_rows<__nv_bfloat16, 1>(pb, p, st);
    }
    const unsigned grid = (unsigned)(pb.rows < 148 * 8 ? pb.rows : 148 * 8);
    if (dtype == 0) launch_next(residual_any_kernel<float>, grid, kJoinThreads, 0, st, pb);
    else launch_next(residual_any_kernel<__nv_bfloat16>, grid, kJoinThreads, 0, st, pb);
    return cudaGetLastError();
}

size_t residual_workspace_bytes(int64_t rows, int64_t d, int64_t gates) {
    if (rows <= 0 || d <= 0) return 0;
    const unsigned __int128 bytes = (unsigned __int128)chunks_of(rows, gates).count * d * sizeof(float) * 3;
    if (bytes >= ((unsigned __int128)1 << 62)) return (size_t)1 << 62;
    return ((size_t)bytes + 255) / 256 * 256;
}

namespace {

template <class T, int V>
cudaError_t launch_backward_rows(const JoinGradArgs& a, const RowPlan& p, cudaStream_t st) {
    const ResidualProblem& pb = a.p;
    const int E = p.cta ? 16 : 8;
    const int threads = p.cta ? p.lanes : kWarpRowThreads;
    const int tensors = 1 + (pb.grad_out.p != nullptr) + 2 * (pb.w_pre != nullptr) + (pb.gate_kind == 2);
    const size_t stage = (size_t)tensors * E * sizeof(T) * threads;
    const int stages = stages_for(stage);
    size_t smem = stage * stages;
    if (!p.cta) {  // (the groups' sums go through the same memory)
        const size_t sums = (size_t)kWarpRowThreads / p.lanes * pb.d * sizeof(float);
        if (smem < sums) smem = sums;
    }
    const unsigned grid = (unsigned)a.chunks.count;
    if (p.cta) return launch_ring(residual_grad_rows_kernel<T, V, 16 / V, true>, grid, threads, smem, st, a, p.lanes, stages);
    return launch_ring(residual_grad_rows_kernel<T, V, 8 / V, false>, grid, threads, smem, st, a, p.lanes, stages);
}

}  // namespace

cudaError_t launch_residual_backward(const ResidualProblem& pb, int dtype, void* workspace, cudaStream_t st) {
    JoinGradArgs a;
    a.p = pb;
    a.chunks = chunks_of(pb.rows, pb.gate_kind == 2 ? pb.rows / pb.gate_rows : 0);
    a.part_post = (float*)workspace;
    a.part_pre = a.part_post + a.chunks.count * pb.d;
    a.part_gate = a.part_pre + a.chunks.count * pb.d;
    cudaError_t e = cudaSuccess;
    const RowPlan p = row_plan(pb, {pb.x, pb.grad_out, pb.out, pb.grad_normed, pb.gate_kind == 2 ? pb.gate : RowsRef{}, pb.grad_x,
                                    pb.grad_residual, pb.gate_kind == 2 ? pb.grad_gate : RowsRef{}},
                               dtype == 0 ? 4 : 2, 8, 16);
    if (a.chunks.count == 0) {
    } else if (p.lanes > 0) {
        if (dtype == 0)
            e = p.vec == 4 ? launch_backward_rows<float, 4>(a, p, st) : launch_backward_rows<float, 1>(a, p, st);
        else
            e = p.vec == 8   ? launch_backward_rows<__nv_bfloat16, 8>(a, p, st)
                : p.vec == 2 ? launch_backward_rows<__nv_bfloat16, 2>(a, p, st)
                             : launch_backward_rows<__nv_bfloat16, 1>(a, p, st);
    } else if (dtype == 0) {
        launch_next(residual_grad_any_kernel<float>, (unsigned)a.chunks.count, kJoinThreads, 0, st, a);
    } else {
        launch_next(residual_grad_any_kernel<__nv_bfloat16>, (unsigned)a.chunks.count, kJoinThreads, 0, st, a);
    }
    if (e != cudaSuccess) return e;
    const int64_t tiles = (pb.d + kColumnLanes - 1) / kColumnLanes;
    int64_t sums = (pb.w_post != nullptr) + (pb.w_pre != nullptr);
    if (pb.gate_kind == 2 && pb.grad_gate.p != nullptr && a.chunks.per_gate > 0) sums += pb.rows / pb.gate_rows;
    if (sums > 0) {
        if (dtype == 0) launch_next(residual_columns_kernel<float>, (unsigned)(tiles * sums), kColumnLanes * kColumnRows, 0, st, a);
        else launch_next(residual_columns_kernel<__nv_bfloat16>, (unsigned)(tiles * sums), kColumnLanes * kColumnRows, 0, st, a);
    }
    return cudaGetLastError();
}

}  // namespace robe
