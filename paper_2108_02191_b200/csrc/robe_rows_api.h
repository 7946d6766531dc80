// What the C ABI of the row operators shares: where the bytes of an argument lie, and which of them may overlap.
#pragma once
#include "../../include/robe.h"
#include "robe_internal.h"
#include "robe_rowops.cuh"

struct robe_bias_ctx {
    uint64_t tag;  // kBiasTag: any other handle is refused
    uint32_t max_distance;
    robe::BiasBuckets bk;
};

namespace robe_rows_api_detail {  // (named: the debug build compiles all sources as one translation unit)
using namespace robe;

constexpr uint64_t kBiasTag = 0x7365676465736162ull;

// ---- matrices: where their bytes are
struct Span {
    const void* p;
    int64_t ld, rows, cols;
    int64_t size;
    bool empty() const { return p == nullptr || rows <= 0 || cols <= 0; }
    bool ok() const {  // pointer and leading dimension usable
        if (rows <= 0 || cols <= 0) return true;
        if (p == nullptr || (uintptr_t)p % (uintptr_t)size != 0) return false;
        if (rows == 1) return true;
        if (ld < cols) return false;
        const unsigned __int128 bytes = ((unsigned __int128)(rows - 1) * (uint64_t)ld + (uint64_t)cols) * (uint64_t)size;
        return bytes < ((unsigned __int128)1 << 60);
    }
    uintptr_t begin() const { return (uintptr_t)p; }
    uintptr_t end() const { return begin() + (uintptr_t)(((rows == 1 ? 0 : (rows - 1) * ld) + cols) * size); }
    bool same(const Span& o) const { return p == o.p && (rows == 1 || ld == o.ld); }
};
inline bool overlap(const Span& a, const Span& b) {
    if (a.empty() || b.empty() || a.end() <= b.begin() || b.end() <= a.begin()) return false;
    if (a.rows > 1 && b.rows > 1 && a.ld * a.size == b.ld * b.size) {  // columns of one matrix
        const uintptr_t step = (uintptr_t)(a.ld * a.size);
        const Span& low = a.begin() <= b.begin() ? a : b;
        const Span& high = a.begin() <= b.begin() ? b : a;
        const uintptr_t at = (high.begin() - low.begin()) % step;
        if (at >= (uintptr_t)(low.cols * low.size) && at + (uintptr_t)(high.cols * high.size) <= step) return false;
    }
    return true;
}
// outputs may overlap nothing but, exactly, what `twin` names for them
struct Checked {
    const Span* in[8];
    const Span* out[8];
    int ins = 0, outs = 0;
    void reads(const Span& s) { in[ins++] = &s; }
    void writes(const Span& s) { out[outs++] = &s; }
    bool ok(const Span* may = nullptr, const Span* be = nullptr) const {
        for (int k = 0; k < ins; ++k)
            if (!in[k]->ok()) return false;
        for (int k = 0; k < outs; ++k) {
            if (!out[k]->ok()) return false;
            for (int j = 0; j < ins; ++j)
                if (!(out[k] == may && in[j] == be && may->same(*be)) && overlap(*out[k], *in[j])) return false;
            for (int j = 0; j < k; ++j)
                if (overlap(*out[k], *out[j])) return false;
        }
        return true;
    }
};

inline int64_t size_of(int dtype) { return dtype == ROBE_F32 ? 4 : 2; }
inline bool type_ok(int dtype) { return dtype == ROBE_F32 || dtype == ROBE_BF16; }

inline int rows_status(cudaError_t e) {
    if (e == cudaSuccess) return ROBE_OK;
    if (e == kGridTooSmall) return ROBE_ERR_UNSUPPORTED;
    (void)cudaGetLastError();  // (a call that only asked or set something leaves its error there: the next launch would find it)
    return ROBE_ERR_CUDA;
}

inline RowsRef ref(const Span& s) { return RowsRef{(void*)s.p, s.ld}; }

}  // namespace robe_rows_api_detail
