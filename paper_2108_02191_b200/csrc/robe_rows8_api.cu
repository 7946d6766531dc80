// C ABI of plain tables and of rows in 8 bits: argument checks and dispatch.  Documented in include/robe.h.
#include <cmath>
#include <initializer_list>

#include "robe_rows_api.h"
#include "robe_codes.cuh"

using namespace robe;

namespace robe_rows8_api_detail {  // (named: the debug build compiles all sources as one translation unit)
using namespace robe_rows_api_detail;

// ids of a lookup
bool ids_span(Span& s, IdList& list, const void* ids, int index_type, int64_t rows) {
    if (index_type != ROBE_I64 && index_type != ROBE_I32) return false;
    s = Span{ids, 1, rows, 1, index_type == ROBE_I32 ? 4 : 8};
    list = IdList{ids, index_type == ROBE_I32 ? 1 : 0};
    return true;
}

// columns that share a scale: at most a warp's, or the whole row
bool group_ok(int64_t d, int64_t& group) {
    if (group == 0 || (group > d && group <= 256)) group = d;
    return group >= 1 && group <= d && (group <= 256 || group == d);
}

// the parts of a cache that a call reads or writes
struct CacheSpans {
    Span codes, scales, pages, offsets, starts;
};
// [pages, page_rows, cols] (of queries: sequences, heads, columns): equally far apart rows as a matrix, pages without gaps as its rows, others as the block of memory they lie in
bool paged(Span& s, const void* p, int64_t ld, int64_t page, int64_t pages, int64_t page_rows, int64_t cols, int64_t size) {
    s = Span{p, cols, 0, cols, size};
    if (pages == 0) return true;
    if (p == nullptr || (uintptr_t)p % (uintptr_t)size != 0 || (page_rows > 1 && ld < cols) || ld < 0 || page < 0) return false;
    const int64_t step = page_rows > 1 ? ld : 0;
    if (step >= (1ll << 60) || page >= (1ll << 60)) return false;
    const unsigned __int128 in_page = (unsigned __int128)(page_rows - 1) * step + cols;
    if (pages > 1 && (unsigned __int128)page < in_page) return false;
    const unsigned __int128 all = (unsigned __int128)(pages - 1) * page + in_page;
    if (all * size >= ((unsigned __int128)1 << 60)) return false;
    if (page_rows > 1 && (pages == 1 || (unsigned __int128)page == (unsigned __int128)ld * page_rows)) s = Span{p, ld, pages * page_rows, cols, size};
    else if (page_rows == 1 || ld == cols) s = Span{p, page, pages, cols * page_rows, size};
    else s = Span{p, (int64_t)all, 1, (int64_t)all, size};
    return true;
}
bool cache_problem(const robe_cache_t* c, CacheProblem& pb, CacheSpans& s) {
    if (c == nullptr || (c->code_type != ROBE_E4M3 && c->code_type != ROBE_I8)) return false;
    if (c->num_pages < 0 || c->num_pages >= (1ll << 31) || c->page_rows < 1 || c->page_rows >= (1ll << 31)) return false;
    if (c->d < 1 || c->d > (1 << 20) || c->batch < 0 || c->batch >= (1ll << 31) || c->max_pages < 0 || c->max_pages >= (1ll << 31)) return false;
    pb.d = c->d;
    pb.group = c->group;
    if (!group_ok(pb.d, pb.group)) return false;
    pb.i8 = c->code_type == ROBE_I8;
    const int64_t groups = (pb.d + pb.group - 1) / pb.group;
    if (!paged(s.codes, c->codes, c->codes_ld, c->codes_page, c->num_pages, c->page_rows, c->d, 1) ||
        !paged(s.scales, c->scales, c->scales_ld, c->scales_page, c->num_pages, c->page_rows, groups, 4))
        return false;
    s.pages = Span{c->pages, c->pages_ld, c->batch, c->max_pages, 4};
    s.offsets = Span{c->offsets, 1, c->offsets != nullptr ? c->batch + 1 : 0, 1, 8};
    s.starts = Span{c->starts, 1, c->starts != nullptr ? c->batch : 0, 1, 8};
    pb.codes = CacheRef{c->codes, c->codes_ld, c->codes_page};
    pb.scales = CacheRef{c->scales, c->scales_ld, c->scales_page};
    pb.at.pages = c->pages;
    pb.at.pages_ld = c->pages_ld;
    pb.at.batch = c->batch;
    pb.at.max_pages = c->max_pages;
    pb.at.num_pages = c->num_pages;
    pb.at.page_rows = (uint32_t)c->page_rows;
    pb.at.offsets = c->offsets;
    pb.at.per = 1;
    pb.at.starts = c->starts;
    return true;
}
// the rows of a cache call
bool cache_rows(const robe_cache_t* c, CacheProblem& pb, int64_t n, int dtype) {
    if (!type_ok(dtype) || n < 0 || n > (1ll << 32)) return false;
    if (c->offsets != nullptr || n == 0) return true;
    if (c->batch == 0 || n % c->batch != 0) return false;
    pb.at.per = n / c->batch;
    return true;
}

bool attend_sizes(int64_t batch, int64_t heads, int64_t q_heads, int64_t dim, int64_t positions) {
    if (batch < 0 || heads < 1 || q_heads < heads || q_heads % heads != 0 || q_heads >= (1ll << 20)) return false;
    if (batch >= (1ll << 31) || batch * q_heads >= (1ll << 31) || positions < 0 || positions >= (1ll << 31) - (1 << 16)) return false;
    return dim == 32 || dim == 64 || dim == 96 || dim == 128 || dim == 256;
}

bool table_grad_sizes(int64_t rows, int64_t vocab, int64_t d) {
    return rows >= 0 && rows < (1ll << 31) && vocab >= 0 && vocab < (1ll << 31) && d >= 1 && d <= (1 << 20);
}

}  // namespace robe_rows8_api_detail
using namespace robe_rows8_api_detail;

extern "C" {

int robe_table_forward(const void* table, int64_t table_ld, int64_t vocab, int64_t d, int table_dtype, const void* ids,
                       int index_type, int64_t rows, float scale, void* out, int64_t out_ld, int out_dtype, void* stream) {
    if (!type_ok(table_dtype) || !type_ok(out_dtype) || rows < 0 || rows >= (1ll << 62)) return ROBE_ERR_INVALID_ARG;
    if (vocab < 0 || vocab >= (1ll << 31) || d < 1 || d > (1 << 20)) return ROBE_ERR_INVALID_ARG;
    const Span from{table, table_ld, vocab, d, size_of(table_dtype)}, to{out, out_ld, rows, d, size_of(out_dtype)};
    Span list;
    TableProblem pb;
    if (!ids_span(list, pb.ids, ids, index_type, rows)) return ROBE_ERR_INVALID_ARG;
    Checked k;
    k.reads(from);
    k.reads(list);
    k.writes(to);
    if (!k.ok()) return ROBE_ERR_INVALID_ARG;
    if (rows == 0) return ROBE_OK;
    pb.table = table;
    pb.table_ld = table_ld;
    pb.vocab = vocab;
    pb.d = d;
    pb.dtype = table_dtype;
    pb.rows = rows;
    pb.scale = scale;
    return rows_status(launch_table_forward(pb, out, out_ld, out_dtype, (cudaStream_t)stream));
}

size_t robe_table_backward_workspace_bytes(int64_t rows, int64_t vocab, int64_t d) {
    return table_grad_sizes(rows, vocab, d) ? table_grad_workspace_bytes(rows, d) : 0;
}

int robe_table_backward(const void* grad, int64_t grad_ld, int dtype, const void* ids, int index_type, int64_t rows,
                        float scale, int64_t skip, int accumulate, float* grad_table, int64_t grad_table_ld, int64_t vocab,
                        int64_t d, void* workspace, size_t workspace_bytes, void* stream) {
    if (!type_ok(dtype) || !table_grad_sizes(rows, vocab, d) || (accumulate != 0 && accumulate != 1)) return ROBE_ERR_INVALID_ARG;
    const Span from{grad, grad_ld, rows, d, size_of(dtype)}, to{grad_table, grad_table_ld, vocab, d, 4};
    Span list;
    TableProblem pb;
    if (!ids_span(list, pb.ids, ids, index_type, rows)) return ROBE_ERR_INVALID_ARG;
    const size_t need = table_grad_workspace_bytes(rows, d);
    if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return ROBE_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 255u) != 0) return ROBE_ERR_WORKSPACE;
    const Span scratch{workspace, 1, 1, (int64_t)need, 1};
    Checked k;
    k.reads(from);
    k.reads(list);
    k.writes(to);
    k.writes(scratch);
    if (!k.ok()) return ROBE_ERR_INVALID_ARG;
    if (vocab == 0) return ROBE_OK;
    pb.table = nullptr;
    pb.table_ld = 0;
    pb.vocab = vocab;
    pb.d = d;
    pb.dtype = dtype;
    pb.rows = rows;
    pb.scale = scale;
    return rows_status(launch_table_backward(pb, grad, grad_ld, skip, accumulate, grad_table, grad_table_ld, workspace, (cudaStream_t)stream));
}

int robe_residual_quantize(int64_t rows, int64_t d, int dtype, int norm, float eps, float scale, const void* x, int64_t x_ld,
                           const void* residual, int64_t residual_ld, const float* w_pre, void* out, int64_t out_ld, void* codes,
                           int64_t codes_ld, int code_type, int64_t group, float* scales, int64_t scales_ld, void* stream) {
    if (!type_ok(dtype) || rows < 0 || rows > (1ll << 32) || d < 1 || d > (1 << 20)) return ROBE_ERR_INVALID_ARG;
    if ((norm != ROBE_NORM_RMS && norm != ROBE_NORM_LAYER) || !(eps >= 0.0f) || std::isinf(eps)) return ROBE_ERR_INVALID_ARG;
    if ((code_type != ROBE_E4M3 && code_type != ROBE_I8) || !group_ok(d, group)) return ROBE_ERR_INVALID_ARG;
    const int64_t e = size_of(dtype), groups = (d + group - 1) / group;
    const Span sx{x, x_ld, rows, d, e}, sr{residual, residual_ld, residual != nullptr ? rows : 0, d, e}, sw{w_pre, d, w_pre != nullptr, d, 4},
        so{out, out_ld, out != nullptr ? rows : 0, d, e}, sc{codes, codes_ld, rows, d, 1}, ss{scales, scales_ld, rows, groups, 4};
    Checked k;
    for (const Span* s : {&sx, &sr, &sw}) k.reads(*s);
    for (const Span* s : {&so, &sc, &ss}) k.writes(*s);
    if (!k.ok(&so, &sr)) return ROBE_ERR_INVALID_ARG;
    if (rows == 0) return ROBE_OK;
    QuantizeProblem pb;
    pb.rows = rows;
    pb.d = d;
    pb.group = group;
    pb.layer = norm == ROBE_NORM_LAYER;
    pb.eps = eps;
    pb.scale = scale;
    pb.w = w_pre;
    pb.x = ref(sx);
    pb.residual = ref(sr);
    pb.out = ref(so);
    pb.codes = ref(sc);
    pb.scales = ref(ss);
    pb.i8 = code_type == ROBE_I8;
    return rows_status(launch_residual_quantize(pb, dtype, (cudaStream_t)stream));
}

int robe_cache_write(const robe_cache_t* c, const void* rows, int64_t rows_ld, int64_t n, int dtype, void* stream) {
    CacheProblem pb;
    CacheSpans s;
    if (!cache_problem(c, pb, s) || !cache_rows(c, pb, n, dtype)) return ROBE_ERR_INVALID_ARG;
    const Span from{rows, rows_ld, n, c->d, size_of(dtype)};
    Checked k;
    for (const Span* r : std::initializer_list<const Span*>{&from, &s.pages, &s.offsets, &s.starts}) k.reads(*r);
    k.writes(s.codes);
    k.writes(s.scales);
    if (!k.ok()) return ROBE_ERR_INVALID_ARG;
    if (n == 0 || c->num_pages == 0) return ROBE_OK;
    return rows_status(launch_cache_write(pb, rows, rows_ld, n, dtype, (cudaStream_t)stream));
}

int robe_cache_read(const robe_cache_t* c, void* out, int64_t out_ld, int64_t n, int dtype, void* stream) {
    CacheProblem pb;
    CacheSpans s;
    if (!cache_problem(c, pb, s) || !cache_rows(c, pb, n, dtype)) return ROBE_ERR_INVALID_ARG;
    const Span to{out, out_ld, n, c->d, size_of(dtype)};
    Checked k;
    for (const Span* r : {&s.codes, &s.scales, &s.pages, &s.offsets, &s.starts}) k.reads(*r);
    k.writes(to);
    if (!k.ok()) return ROBE_ERR_INVALID_ARG;
    if (n == 0) return ROBE_OK;
    return rows_status(launch_cache_read(pb, out, out_ld, n, dtype, (cudaStream_t)stream));
}

size_t robe_cache_attention_workspace_bytes(int64_t batch, int64_t heads, int64_t q_heads, int64_t dim, int64_t positions) {
    return attend_sizes(batch, heads, q_heads, dim, positions) ? attend_workspace_bytes(batch, heads, q_heads, dim, positions) : 0;
}

int robe_cache_attention(const robe_cache_t* keys, const robe_cache_t* values, const void* q, int64_t q_ld, int64_t q_seq, int64_t q_heads,
                         float scale, robe_bias_t bias, const float* bias_rows, int64_t bias_ld, void* out, int64_t out_ld,
                         int64_t out_seq, void* workspace, size_t workspace_bytes, void* stream) {
    CacheProblem pk, pv;
    CacheSpans sk, sv;
    if (!cache_problem(keys, pk, sk) || !cache_problem(values, pv, sv)) return ROBE_ERR_INVALID_ARG;
    if (keys->code_type != values->code_type || keys->num_pages != values->num_pages || keys->page_rows != values->page_rows ||
        keys->d != values->d || pk.group != pv.group || keys->pages != values->pages || keys->pages_ld != values->pages_ld ||
        keys->batch != values->batch || keys->max_pages != values->max_pages || keys->starts != values->starts ||
        keys->offsets != nullptr || values->offsets != nullptr || keys->codes_ld != values->codes_ld ||
        keys->codes_page != values->codes_page || keys->scales_ld != values->scales_ld || keys->scales_page != values->scales_page)
        return ROBE_ERR_INVALID_ARG;
    const int64_t dim = pk.group, heads = pk.d / pk.group, batch = keys->batch;
    const unsigned __int128 room = (unsigned __int128)keys->max_pages * (uint64_t)keys->page_rows;
    if (pk.d % dim != 0 || room >= ((unsigned __int128)1 << 31) || !attend_sizes(batch, heads, q_heads, dim, (int64_t)room)) return ROBE_ERR_INVALID_ARG;
    if (bias != nullptr && bias->tag != kBiasTag) return ROBE_ERR_INVALID_ARG;
    if (batch > 0 && keys->starts == nullptr) return ROBE_ERR_INVALID_ARG;
    for (const robe_cache_t* c : {keys, values})
        if (c->num_pages > 0 && (((uintptr_t)c->codes | (uint64_t)c->codes_ld | (uint64_t)c->codes_page) & 15u) != 0) return ROBE_ERR_INVALID_ARG;
    Span sq, so;
    if (!paged(sq, q, q_ld, q_seq, batch, q_heads, dim, 2) || !paged(so, out, out_ld, out_seq, batch, q_heads, dim, 2)) return ROBE_ERR_INVALID_ARG;
    const Span sb{bias_rows, bias_ld, bias != nullptr ? (int64_t)bias->bk.buckets : 0, q_heads, 4};
    const size_t need = attend_workspace_bytes(batch, heads, q_heads, dim, (int64_t)room);
    if (workspace == nullptr || workspace_bytes < need || ((uintptr_t)workspace & 255u) != 0) return ROBE_ERR_WORKSPACE;
    const Span scratch{workspace, 1, 1, (int64_t)need, 1};
    Checked k;
    for (const Span* r : std::initializer_list<const Span*>{&sk.codes, &sk.scales, &sv.codes, &sv.scales, &sk.pages, &sk.starts, &sq, &sb})
        k.reads(*r);
    k.writes(so);
    k.writes(scratch);
    if (!k.ok()) return ROBE_ERR_INVALID_ARG;
    if (batch == 0) return ROBE_OK;
    AttendProblem pb{};
    pb.at = pk.at;
    pb.key_codes = pk.codes;
    pb.key_scales = pk.scales;
    pb.value_codes = pv.codes;
    pb.value_scales = pv.scales;
    pb.i8 = pk.i8;
    pb.heads = heads;
    pb.q_heads = q_heads;
    pb.dim = dim;
    pb.q = CacheRef{(void*)q, q_ld, q_seq};
    pb.out = CacheRef{out, out_ld, out_seq};
    pb.scale = scale;
    pb.biased = bias != nullptr;
    if (bias != nullptr) pb.bk = bias->bk;
    pb.bias = bias_rows;
    pb.bias_ld = bias_ld;
    return rows_status(launch_attend(pb, workspace, (cudaStream_t)stream));
}

}  // extern "C"
