// What the row operators (dropout, position bias, residual join) share: element types, 16-byte pieces of a row,
// and the counter-based generator of the dropout.
#pragma once
#include <cuda_bf16.h>

#include "robe_device.cuh"

namespace robe {

// ---- elements.  Everything is computed in fp32; bf16 is widened exactly and rounded once, to nearest even, where
// a result is stored.
template <class T>
constexpr int kPiece = 16 / (int)sizeof(T);  // elements of a 16-byte piece

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// two bf16 in a word, low one first
__device__ __forceinline__ uint32_t narrow2(float low, float high) {
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(high), "f"(low));
    return w;
}
__device__ __forceinline__ float widen_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float widen_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Two fp32 operations in one instruction.
#define ROBE_F2(name, op)                                                                                              \
    __device__ __forceinline__ float2 name(float2 a, float2 b) {                                                       \
        float2 d;                                                                                                      \
        asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\n" op " d, a, b;\nmov.b64 {%0, %1}, d;\n}" \
            : "=f"(d.x), "=f"(d.y)                                                                                     \
            : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));                                                                 \
        return d;                                                                                                      \
    }
ROBE_F2(add2, "add.rn.f32x2")
ROBE_F2(mul2, "mul.rn.f32x2")
#undef ROBE_F2
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\n"
        "fma.rn.f32x2 d, a, b, c;\nmov.b64 {%0, %1}, d;\n}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// V consecutive elements as one access of V * sizeof(T) bytes (aligned to that), V a power of two, at most 16 bytes
template <class T, int V>
struct alignas(V * sizeof(T)) Pack {
    T v[V];
};
template <int BYTES>
struct Word;
template <>
struct Word<16> { using type = uint4; };
template <>
struct Word<8> { using type = uint2; };
template <>
struct Word<4> { using type = unsigned; };
template <>
struct Word<2> { using type = unsigned short; };

// STREAM: the value is read (written) once and nothing else soon wants its line
template <bool STREAM, class T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T* p) {
    using W = typename Word<V * sizeof(T)>::type;
    union {
        W w;
        Pack<T, V> e;
    } u;
    u.w = STREAM ? __ldcs((const W*)p) : __ldca((const W*)p);
    return u.e;
}
template <bool STREAM, class T, int V>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, V>& e) {
    using W = typename Word<V * sizeof(T)>::type;
    union U {
        W w;
        Pack<T, V> e;
        __device__ U() {}
    } u;
    u.e = e;
    if (STREAM) __stcs((W*)p, u.w);
    else *(W*)p = u.w;
}

// Copies to shared memory that go on by themselves (BYTES 4, 8 or 16, both sides aligned to it; 2: a plain load and
// store); what a thread has copied it may read after copies_wait(n), which leaves its n latest groups in flight.
template <int BYTES>
__device__ __forceinline__ void copy_async(void* to, const void* from) {
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else if constexpr (BYTES >= 4)
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(BYTES) : "memory");
    else
        *(unsigned short*)to = __ldcs((const unsigned short*)from);
}
__device__ __forceinline__ void copies_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait(int left) {
    switch (left) {
        case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
        case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
        case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
        default: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
    }
}

// ---- generator: Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2,
// 3", 2011): a block cipher of the counter under the key, so any element's number is had from its position alone.
constexpr int kRounds = 10;
struct DropParams {
    uint32_t none;              // 1: nothing is dropped (t = 0), the generator is not asked
    uint32_t limit;             // (t << 16) - 1: an element is kept when its 16 bits, moved up by 16, are above
    float scale;                // 65536 / (65536 - t), what kept elements are multiplied by
    uint32_t keys[kRounds][2];  // the key of every round (made by the host: constants to the kernels)
    uint64_t offset;            // upper half of the counter
    const uint64_t* step;       // device, added to offset, or nullptr
};
inline void drop_keys(DropParams& d, uint64_t seed) {
    for (int k = 0; k < kRounds; ++k) {
        d.keys[k][0] = (uint32_t)seed + (uint32_t)k * 0x9E3779B9u;
        d.keys[k][1] = (uint32_t)(seed >> 32) + (uint32_t)k * 0xBB67AE85u;
    }
}

// The words that columns 8 g .. 8 g + 7 of row r are kept or dropped by: column 8 g + k by half k & 1 (low first) of
// word k / 2.
__device__ __forceinline__ uint4 drop_words(uint32_t r, uint32_t g, uint64_t offset, const DropParams& d) {
    uint32_t c0 = g, c1 = r, c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ d.keys[k][0];
        c1 = (uint32_t)p1;
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ d.keys[k][1];
        c3 = (uint32_t)p0;
    }
    return make_uint4(c0, c1, c2, c3);
}
__device__ __forceinline__ uint64_t drop_offset(const DropParams& d) {
    return d.offset + (d.step != nullptr ? __ldca((const unsigned long long*)d.step) : 0ull);
}
__device__ __forceinline__ bool drop_keeps(const uint4& w, int k, const DropParams& d) {
    const uint32_t word = k < 2 ? w.x : k < 4 ? w.y : k < 6 ? w.z : w.w;
    return ((k & 1) ? word : word << 16) > d.limit;
}

// 1 / sqrt(v), to about a rounding: the function's result (within two) and one step of Newton's method.  (A division and a
// square root, rounded each, took 4 to 10 % of a pass.)
__device__ __forceinline__ float norm_factor(float v) {
    const float y = rsqrtf(v), off = fmaf(-v * y, y, 1.0f);
    return off == off ? fmaf(0.5f * y, off, y) : y;  // (of 0 and of infinity there is nothing to mend)
}

// k / by for any 32-bit k, by a product
__device__ __forceinline__ uint32_t divide(uint32_t k, uint32_t by, uint64_t magic) {
    return by == 1 ? k : (uint32_t)__umul64hi(magic, k);
}
inline uint64_t magic_of(uint32_t by) { return by > 1 ? ~0ull / by + 1 : 0; }

// ---- the residual join: what one call is given
struct RowsRef {  // rows of a matrix, ld elements apart
    void* p;
    int64_t ld;
};
struct ResidualProblem {
    int64_t rows, d;
    int layer;        // 0: root mean square norm, 1: layer norm
    float eps, scale;
    int gate_kind;    // 0 none, 1 a number per row, 2 a vector of d per gate_rows rows
    int64_t gate_rows;
    DropParams drop;  // none: no dropout
    const float *w_post, *w_pre;  // or nullptr: no norm there
    RowsRef x, residual, gate, out, normed;  // forward; residual.p may be nullptr (nothing added to)
    // backward (x, gate and out as above)
    RowsRef grad_out, grad_normed, grad_x, grad_residual, grad_gate;  // grad_out.p, grad_residual.p, grad_gate.p may be nullptr
    float *grad_w_post, *grad_w_pre;
};

}  // namespace robe
