// C ABI of the row operators: argument checks and dispatch.  Documented in include/robe.h.
#include <cmath>
#include <new>

#include "../../include/robe.h"
#include "robe_internal.h"
#include "robe_rowops.cuh"

using namespace robe;

struct robe_bias_ctx {
    uint64_t tag;  // kBiasTag: any other handle is refused
    uint32_t max_distance;
    BiasBuckets bk;
};

namespace robe_rows_api_detail {  // (named: the debug build compiles all sources as one translation unit)

constexpr uint64_t kBiasTag = 0x7365676465736162ull;

// ---- whole numbers of up to 128 * 31 bits, least significant word first: products of the bucket borders
struct Wide {
    static constexpr int kWords = 126;
    uint32_t w[kWords] = {1};
    int n = 1;
    void times(uint32_t f) {
        uint64_t carry = 0;
        for (int k = 0; k < n; ++k) {
            carry += (uint64_t)w[k] * f;
            w[k] = (uint32_t)carry;
            carry >>= 32;
        }
        if (carry != 0) w[n++] = (uint32_t)carry;
    }
    void times_power(uint32_t f, uint32_t times_) {
        for (uint32_t k = 0; k < times_; ++k) times(f);
    }
    bool at_least(const Wide& o) const {
        if (n != o.n) return n > o.n;
        for (int k = n; k-- > 0;)
            if (w[k] != o.w[k]) return w[k] > o.w[k];
        return true;
    }
};

// Smallest n with n^L >= E^(L-k) far^k: the root in floating point, put right in whole numbers.
uint32_t bucket_edge(uint32_t E, uint32_t L, uint32_t far, uint32_t k) {
    Wide reach;
    reach.times_power(E, L - k);
    reach.times_power(far, k);
    auto reached = [&](uint32_t n) {
        Wide p;
        p.times_power(n, L);
        return p.at_least(reach);
    };
    // (the powers' exponents are small and far < 2^30: the root is right to about 1e-14 of itself)
    uint32_t n = (uint32_t)(E * std::pow((double)far / E, (double)k / L));
    if (n < 1) n = 1;
    while (n > 1 && reached(n - 1)) --n;
    while (!reached(n)) ++n;
    return n;
}

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
bool overlap(const Span& a, const Span& b) {
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

int64_t size_of(int dtype) { return dtype == ROBE_F32 ? 4 : 2; }
bool type_ok(int dtype) { return dtype == ROBE_F32 || dtype == ROBE_BF16; }

bool drop_params(float p, uint64_t seed, uint64_t offset, const uint64_t* step, DropParams& d) {
    if (!(p >= 0.0f && p <= 1.0f) || (uintptr_t)step % 8 != 0) return false;
    const uint64_t t = (uint64_t)std::floor((double)p * 65536.0 + 0.5);
    d.none = t == 0;
    d.limit = (uint32_t)((t << 16) - 1);
    d.scale = t < 65536 ? (float)(65536.0 / (double)(65536 - t)) : 0.0f;
    drop_keys(d, seed);
    d.offset = offset;
    d.step = step;
    return true;
}

int rows_status(cudaError_t e) {
    if (e == cudaSuccess) return ROBE_OK;
    if (e == kGridTooSmall) return ROBE_ERR_UNSUPPORTED;
    (void)cudaGetLastError();  // (a call that only asked or set something leaves its error there: the next launch would find it)
    return ROBE_ERR_CUDA;
}

bool bias_sizes(robe_bias_t b, uint32_t heads, int64_t batch, int64_t q_len, int64_t k_len) {
    if (b == nullptr || b->tag != kBiasTag) return false;
    if (heads == 0 || heads >= (1u << 22) || batch < 0 || batch >= (1ll << 31)) return false;
    return q_len >= 0 && k_len >= 0 && q_len < (1ll << 31) && k_len < (1ll << 31) && q_len + k_len < (1ll << 31);
}

bool bias_matrix(Span& m, const void* p, int64_t ld, uint32_t heads, int64_t batch, int64_t q_len, int64_t k_len, int dtype) {
    // (batch, heads, q_len below 2^31, 2^22, 2^31)
    const unsigned __int128 rows = (unsigned __int128)batch * heads * q_len;
    if (rows >= ((unsigned __int128)1 << 62)) return false;
    m = Span{p, ld, (int64_t)rows, k_len, size_of(dtype)};
    return true;
}

BiasProblem bias_problem(robe_bias_t b, uint32_t heads, int64_t batch, int64_t q_len, int64_t k_len, int64_t q_start,
                         const int64_t* q_starts, int causal) {
    BiasProblem pb;
    pb.bk = b->bk;
    pb.rows = nullptr;
    pb.rows_ld = 0;
    pb.heads = heads;
    pb.batch = batch;
    pb.q_len = q_len;
    pb.k_len = k_len;
    pb.q_start = q_start;
    pb.q_starts = q_starts;
    pb.causal = causal;
    return pb;
}

// the parts of a residual call that both directions share
bool residual_problem(const robe_residual_t* c, ResidualProblem& pb, int64_t& gates, int64_t& gate_cols) {
    if (c == nullptr || !type_ok(c->dtype)) return false;
    if (c->rows < 0 || c->rows > (1ll << 32) || c->d < 1 || c->d > (1 << 20)) return false;
    if (c->norm != ROBE_NORM_RMS && c->norm != ROBE_NORM_LAYER) return false;
    if (!(c->eps >= 0.0f) || std::isinf(c->eps)) return false;
    pb.rows = c->rows;
    pb.d = c->d;
    pb.layer = c->norm;
    pb.eps = c->eps;
    pb.scale = c->scale;
    pb.gate_kind = c->gate;
    gates = gate_cols = 0;
    pb.gate_rows = 1;
    if (c->gate == ROBE_GATE_ROW) {
        gates = c->rows;
        gate_cols = 1;
    } else if (c->gate == ROBE_GATE_VECTOR) {
        if (c->gate_rows < 1 || c->rows % c->gate_rows != 0) return false;
        pb.gate_rows = c->gate_rows;
        gates = c->rows / c->gate_rows;
        gate_cols = c->d;
    } else if (c->gate != ROBE_GATE_NONE) {
        return false;
    }
    return drop_params(c->p, c->seed, c->offset, c->step, pb.drop);
}

// the counter that dropout's decisions go by: read by every CTA when it starts
Span counter(const uint64_t* step) { return Span{step, 1, step != nullptr, 1, 8}; }

RowsRef ref(const Span& s) { return RowsRef{(void*)s.p, s.ld}; }

}  // namespace robe_rows_api_detail
using namespace robe_rows_api_detail;

extern "C" {

int robe_dropout(const void* in, int64_t in_ld, void* out, int64_t out_ld, int64_t rows, int64_t cols,
                 int dtype, float p, uint64_t seed, uint64_t offset, const uint64_t* step, void* stream) {
    if (!type_ok(dtype) || rows < 0 || cols < 0 || rows > (1ll << 32) || cols > (1ll << 31)) return ROBE_ERR_INVALID_ARG;
    const Span from{in, in_ld, rows, cols, size_of(dtype)}, to{out, out_ld, rows, cols, size_of(dtype)}, at = counter(step);
    Checked c;
    c.reads(from);
    c.reads(at);
    c.writes(to);
    DropParams drop;
    if (!c.ok(&to, &from) || !drop_params(p, seed, offset, step, drop)) return ROBE_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return ROBE_OK;
    return rows_status(launch_dropout(in, in_ld, out, out_ld, rows, cols, dtype, drop, (cudaStream_t)stream));
}

int robe_bias_create(robe_bias_t* out, uint32_t num_buckets, uint32_t max_distance, int two_sided) {
    if (out == nullptr) return ROBE_ERR_INVALID_ARG;
    *out = nullptr;
    if (two_sided != 0 && two_sided != 1) return ROBE_ERR_INVALID_ARG;
    if (two_sided && num_buckets % 2 != 0) return ROBE_ERR_INVALID_ARG;
    const uint32_t side = two_sided ? num_buckets / 2 : num_buckets;
    if (side < 2 || side > kBiasMaxSide) return ROBE_ERR_INVALID_ARG;
    const uint32_t E = side / 2, L = side - E;
    if (max_distance <= E || max_distance >= (1u << 30)) return ROBE_ERR_INVALID_ARG;
    robe_bias_ctx* b = new (std::nothrow) robe_bias_ctx();
    if (b == nullptr) return ROBE_ERR_INVALID_ARG;
    b->tag = kBiasTag;
    b->max_distance = max_distance;
    b->bk.buckets = num_buckets;
    b->bk.side = side;
    b->bk.two_sided = two_sided;
    for (uint32_t k = 0; k < kBiasMaxSide; ++k)
        b->bk.edges[k] = k < E ? (int32_t)k : k < side ? (int32_t)bucket_edge(E, L, max_distance, k - E) : 0;
    *out = b;
    return ROBE_OK;
}

int robe_bias_destroy(robe_bias_t b) {
    if (b == nullptr || b->tag != kBiasTag) return ROBE_ERR_INVALID_ARG;
    b->tag = 0;
    delete b;
    return ROBE_OK;
}

int robe_bias_num_buckets(robe_bias_t b) {
    return b == nullptr || b->tag != kBiasTag ? ROBE_ERR_INVALID_ARG : (int)b->bk.buckets;
}

int robe_bias_get_edges(robe_bias_t b, int64_t* edges) {
    if (b == nullptr || b->tag != kBiasTag || edges == nullptr) return ROBE_ERR_INVALID_ARG;
    for (uint32_t k = 0; k < b->bk.buckets; ++k) {
        edges[k] = b->bk.edges[k % b->bk.side];
        if (k >= b->bk.side && edges[k] == 0) edges[k] = 1;
    }
    return ROBE_OK;
}

int robe_bias_forward(robe_bias_t b, const float* rows, int64_t rows_ld, uint32_t heads, int64_t batch,
                      int64_t q_len, int64_t k_len, int64_t q_start, const int64_t* q_starts, int causal,
                      void* out, int64_t out_ld, int dtype, void* stream) {
    if (!bias_sizes(b, heads, batch, q_len, k_len) || !type_ok(dtype)) return ROBE_ERR_INVALID_ARG;
    if ((causal != 0 && causal != 1) || (uintptr_t)q_starts % 8 != 0) return ROBE_ERR_INVALID_ARG;
    const Span table{rows, rows_ld, b->bk.buckets, heads, 4};
    const Span starts{q_starts, 1, q_starts != nullptr ? batch : 0, 1, 8};
    Span to;
    if (!bias_matrix(to, out, out_ld, heads, batch, q_len, k_len, dtype)) return ROBE_ERR_INVALID_ARG;
    Checked c;
    c.reads(table);
    c.reads(starts);
    c.writes(to);
    if (!c.ok()) return ROBE_ERR_INVALID_ARG;
    if (to.empty()) return ROBE_OK;
    BiasProblem pb = bias_problem(b, heads, batch, q_len, k_len, q_start, q_starts, causal);
    pb.rows = rows;
    pb.rows_ld = rows_ld;
    return rows_status(launch_bias_forward(pb, out, out_ld, dtype, (cudaStream_t)stream));
}

size_t robe_bias_backward_workspace_bytes(robe_bias_t b, uint32_t heads, int64_t batch, int64_t q_len, int64_t k_len) {
    if (!bias_sizes(b, heads, batch, q_len, k_len)) return 0;
    return bias_grad_workspace_bytes(b->bk.buckets, heads, batch, q_len, k_len);
}

int robe_bias_backward(robe_bias_t b, const void* grad, int64_t grad_ld, uint32_t heads, int64_t batch,
                       int64_t q_len, int64_t k_len, int64_t q_start, const int64_t* q_starts, int causal,
                       int dtype, float* grad_rows, int64_t grad_rows_ld, void* workspace,
                       size_t workspace_bytes, void* stream) {
    if (!bias_sizes(b, heads, batch, q_len, k_len) || !type_ok(dtype)) return ROBE_ERR_INVALID_ARG;
    if ((causal != 0 && causal != 1) || (uintptr_t)q_starts % 8 != 0) return ROBE_ERR_INVALID_ARG;
    const Span to{grad_rows, grad_rows_ld, b->bk.buckets, heads, 4};
    const Span starts{q_starts, 1, q_starts != nullptr ? batch : 0, 1, 8};
    Span from;
    if (!bias_matrix(from, grad, grad_ld, heads, batch, q_len, k_len, dtype)) return ROBE_ERR_INVALID_ARG;
    const size_t need = bias_grad_workspace_bytes(b->bk.buckets, heads, batch, q_len, k_len);
    const Span scratch{workspace, 1, 1, need < ((size_t)1 << 60) ? (int64_t)need : 0, 1};
    if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return ROBE_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 255u) != 0) return ROBE_ERR_WORKSPACE;
    Checked c;
    c.reads(from);
    c.reads(starts);
    c.writes(to);
    c.writes(scratch);
    if (!c.ok()) return ROBE_ERR_INVALID_ARG;
    const BiasProblem pb = bias_problem(b, heads, batch, q_len, k_len, q_start, q_starts, causal);
    return rows_status(launch_bias_backward(pb, grad, grad_ld, dtype, grad_rows, grad_rows_ld, workspace, (cudaStream_t)stream));
}

int robe_residual_forward(const robe_residual_t* c, const void* x, int64_t x_ld, const void* residual,
                          int64_t residual_ld, const void* gate, int64_t gate_ld, const float* w_post,
                          const float* w_pre, void* out, int64_t out_ld, void* normed, int64_t normed_ld,
                          void* stream) {
    ResidualProblem pb{};
    int64_t gates = 0, gate_cols = 0;
    if (!residual_problem(c, pb, gates, gate_cols)) return ROBE_ERR_INVALID_ARG;
    if ((w_pre != nullptr) != (normed != nullptr) && c->rows > 0) return ROBE_ERR_INVALID_ARG;
    if ((gate != nullptr) != (c->gate != ROBE_GATE_NONE) && c->rows > 0) return ROBE_ERR_INVALID_ARG;
    const int64_t n = c->rows, d = c->d, e = size_of(c->dtype);
    const Span sx{x, x_ld, n, d, e}, sr{residual, residual_ld, residual != nullptr ? n : 0, d, e},
        sg{gate, gate_ld, gates, gate_cols, e}, s1{w_post, d, w_post != nullptr, d, 4}, s2{w_pre, d, w_pre != nullptr, d, 4},
        so{out, out_ld, n, d, e}, sn{normed, normed_ld, w_pre != nullptr ? n : 0, d, e}, at = counter(c->step);
    Checked k;
    for (const Span* s : {&sx, &sr, &sg, &s1, &s2, &at}) k.reads(*s);
    for (const Span* s : {&so, &sn}) k.writes(*s);
    if (!k.ok(&so, &sr)) return ROBE_ERR_INVALID_ARG;
    if (n == 0) return ROBE_OK;
    pb.w_post = w_post;
    pb.w_pre = w_pre;
    pb.x = ref(sx);
    pb.residual = ref(sr);
    pb.gate = ref(sg);
    pb.out = ref(so);
    pb.normed = ref(sn);
    return rows_status(launch_residual_forward(pb, c->dtype, (cudaStream_t)stream));
}

size_t robe_residual_backward_workspace_bytes(int64_t rows, int64_t d, int64_t gates) {
    if (rows < 0 || rows > (1ll << 32) || d < 1 || d > (1 << 20) || gates < 0 || (gates > 0 && rows % gates != 0)) return 0;
    return residual_workspace_bytes(rows, d, gates);
}

int robe_residual_backward(const robe_residual_t* c, const void* grad_out, int64_t grad_out_ld,
                           const void* grad_normed, int64_t grad_normed_ld, const void* x, int64_t x_ld,
                           const void* out, int64_t out_ld, const void* gate, int64_t gate_ld,
                           const float* w_post, const float* w_pre, void* grad_x, int64_t grad_x_ld,
                           void* grad_residual, int64_t grad_residual_ld, void* grad_gate,
                           int64_t grad_gate_ld, float* grad_w_post, float* grad_w_pre, void* workspace,
                           size_t workspace_bytes, void* stream) {
    ResidualProblem pb{};
    int64_t gates = 0, gate_cols = 0;
    if (!residual_problem(c, pb, gates, gate_cols)) return ROBE_ERR_INVALID_ARG;
    const int64_t n = c->rows, d = c->d, e = size_of(c->dtype);
    if ((w_pre != nullptr) != (grad_w_pre != nullptr) || (w_post != nullptr) != (grad_w_post != nullptr)) return ROBE_ERR_INVALID_ARG;
    if (n > 0 && ((w_pre != nullptr) != (grad_normed != nullptr) || (gate != nullptr) != (c->gate != ROBE_GATE_NONE)))
        return ROBE_ERR_INVALID_ARG;
    if (grad_gate != nullptr && c->gate == ROBE_GATE_NONE) return ROBE_ERR_INVALID_ARG;
    const int64_t pre = w_pre != nullptr ? n : 0;
    const Span sgo{grad_out, grad_out_ld, grad_out != nullptr ? n : 0, d, e}, sgn{grad_normed, grad_normed_ld, pre, d, e},
        sx{x, x_ld, n, d, e}, so{out, out_ld, pre, d, e}, sg{gate, gate_ld, gates, gate_cols, e},
        s1{w_post, d, w_post != nullptr, d, 4}, s2{w_pre, d, w_pre != nullptr, d, 4},
        gx{grad_x, grad_x_ld, n, d, e}, gr{grad_residual, grad_residual_ld, grad_residual != nullptr ? n : 0, d, e},
        gg{grad_gate, grad_gate_ld, grad_gate != nullptr ? gates : 0, gate_cols, e},
        g1{grad_w_post, d, grad_w_post != nullptr, d, 4}, g2{grad_w_pre, d, grad_w_pre != nullptr, d, 4}, at = counter(c->step);
    const size_t need = residual_workspace_bytes(n, d, c->gate == ROBE_GATE_VECTOR ? gates : 0);
    if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return ROBE_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 255u) != 0) return ROBE_ERR_WORKSPACE;
    const Span scratch{workspace, 1, 1, need < ((size_t)1 << 60) ? (int64_t)need : 0, 1};
    Checked k;
    for (const Span* s : {&sgo, &sgn, &sx, &so, &sg, &s1, &s2, &at}) k.reads(*s);
    for (const Span* s : {&gx, &gr, &gg, &g1, &g2, &scratch}) k.writes(*s);
    if (!k.ok(&gr, &sgo)) return ROBE_ERR_INVALID_ARG;
    pb.w_post = w_post;
    pb.w_pre = w_pre;
    pb.x = ref(sx);
    pb.out = ref(so);
    pb.gate = ref(sg);
    pb.grad_out = ref(sgo);
    pb.grad_normed = ref(sgn);
    pb.grad_x = ref(gx);
    pb.grad_residual = ref(gr);
    pb.grad_gate = ref(gg);
    pb.grad_w_post = grad_w_post;
    pb.grad_w_pre = grad_w_pre;
    return rows_status(launch_residual_backward(pb, c->dtype, workspace, (cudaStream_t)stream));
}

}  // extern "C"
