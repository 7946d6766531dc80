// The join at which a block's output enters the rows again, in one pass over its tensors:
//
//   y = norm(x) w_post  (or x);   out = residual + scale * gate * dropout(y);   normed = norm(out) w_pre
//
// and its backward, from x and out as they stand in memory: the norms' statistics are had again from the rows, nothing is
// kept between the passes.  With n = norm(v) and rstd its factor, the gradient through a norm is
//   d(v) = rstd (g - [mean g] - n mean(g n)),     g = (gradient of the normed row) * weight,   [..]: layer norm only.
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

// ---- rows of any length, one CTA each, read again in every pass over the row

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
    if (drop.threshold == 0) return 1.0f;
    const uint4 w = drop_words((uint32_t)r, (uint32_t)(c >> 3), offset, drop.seed);
    return drop_keeps(w, (int)(c & 7), drop.threshold) ? drop.scale : 0.0f;
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

cudaError_t launch_residual_forward(const ResidualProblem& pb, int dtype, cudaStream_t st) {
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

cudaError_t launch_residual_backward(const ResidualProblem& pb, int dtype, void* workspace, cudaStream_t st) {
    JoinGradArgs a;
    a.p = pb;
    a.chunks = chunks_of(pb.rows, pb.gate_kind == 2 ? pb.rows / pb.gate_rows : 0);
    a.part_post = (float*)workspace;
    a.part_pre = a.part_post + a.chunks.count * pb.d;
    a.part_gate = a.part_pre + a.chunks.count * pb.d;
    if (a.chunks.count == 0) {
    } else if (dtype == 0)
        launch_next(residual_grad_any_kernel<float>, (unsigned)a.chunks.count, kJoinThreads, 0, st, a);
    else
        launch_next(residual_grad_any_kernel<__nv_bfloat16>, (unsigned)a.chunks.count, kJoinThreads, 0, st, a);
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
