// swr_hybrid_api.cpp -- C ABI of the hybrid model's operators: argument
// validation (done entirely before any HIP runtime call) and dispatch to their
// gfx950 kernels.
#include <stdint.h>

#include <cmath>
#include <initializer_list>

#include "../../include/swr_hybrid.h"
#include "swr_hybrid_launch.h"

namespace {

constexpr int64_t kMaxExtent = (int64_t)1 << 60;
constexpr int64_t kMaxRows = 0x7fffffffLL;
constexpr int64_t kMaxWidth = (int64_t)1 << 30;
constexpr int64_t kMaxPage = 65536;

struct Dim {
    int64_t size, stride;
};

// Largest offset of a strided tensor of these dimensions (all sizes at least
// 1), or -1 for a negative stride or one whose offsets are out of range.
int64_t max_offset(std::initializer_list<Dim> dims) {
    int64_t off = 0;
    for (const Dim& d : dims) {
        if (d.stride < 0) return -1;
        if (d.size <= 1 || d.stride == 0) continue;
        if (d.size - 1 > kMaxExtent / d.stride) return -1;
        off += (d.size - 1) * d.stride;
        if (off > kMaxExtent) return -1;
    }
    return off;
}

// Dimensions (up to four) of more than one element, of the least stride first.
struct Sorted {
    Dim d[4];
    int n = 0;
    explicit Sorted(std::initializer_list<Dim> dims) {
        for (const Dim& x : dims)
            if (x.size > 1) d[n++] = x;
        for (int i = 1; i < n; ++i)
            for (int j = i; j > 0 && d[j].stride < d[j - 1].stride; --j) {
                const Dim t = d[j];
                d[j] = d[j - 1];
                d[j - 1] = t;
            }
    }
};

// Whether different indices never name the same element.
bool apart(std::initializer_list<Dim> dims) {
    const Sorted s(dims);
    int64_t need = 1;
    for (int i = 0; i < s.n; ++i) {
        if (s.d[i].stride < need) return false;
        if (s.d[i].size > kMaxExtent / s.d[i].stride) return false;
        need = s.d[i].stride * s.d[i].size;
    }
    return true;
}

// Whether two tensors of these dimensions, apart, share an element when they begin
// `distance` elements from each other.  The lesser dimensions reach less far than a
// dimension's stride, so only its two differences of indices next to the distance count.
bool meet_at(const Sorted& s, int dims, int64_t distance) {
    if (dims == 0) return distance == 0;
    const Dim& d = s.d[dims - 1];
    const int64_t below = distance / d.stride - (distance % d.stride < 0);
    for (int64_t i = below; i <= below + 1; ++i)
        if (i > -d.size && i < d.size && meet_at(s, dims - 1, distance - i * d.stride)) return true;
    return false;
}

struct Span {
    uintptr_t lo, hi;
};
Span span(const void* p, int64_t bytes) { return {(uintptr_t)p, (uintptr_t)p + (uintptr_t)(p ? bytes : 0)}; }
bool overlap(const Span& a, const Span& b) { return a.lo < b.hi && b.lo < a.hi; }
bool overlaps(const Span& out, std::initializer_list<Span> others) {
    for (const Span& s : others)
        if (overlap(out, s)) return true;
    return false;
}

bool aligned(const void* p, int64_t bytes) { return (uintptr_t)p % (uintptr_t)bytes == 0; }
int size_of(int dtype) { return dtype == SWR_DTYPE_F32 ? 4 : dtype == SWR_DTYPE_BF16 ? 2 : 1; }
// Whether these strides are whole numbers of 16 bytes.
bool vectors(std::initializer_list<Dim> dims, int es) {
    for (const Dim& d : dims)
        if (d.size > 1 && d.stride % (16 / es) != 0) return false;
    return true;
}
bool plain(int dtype) { return dtype == SWR_DTYPE_F32 || dtype == SWR_DTYPE_BF16; }
int status(hipError_t e) { return e == hipSuccess ? SWR_OK : SWR_ERR_HIP; }

// ---------------------------------------------------------------------------
// Norm
// ---------------------------------------------------------------------------

// A tensor of rows as a call has it (p NULL: not there).
struct RowTensor {
    const void* p;
    int64_t so, si;
    int64_t bytes;   // that it spans
    int es;
};

struct Rows {
    bool empty;
    int es;
    int64_t rows, x, r, h, y;   // rows, and bytes that each tensor spans
};

// Whether two tensors of the norm's rows share an element.  Those of the same
// strides and type, as parts of one larger tensor are, may lie between each
// other's rows; others are taken to meet where their spans do.
bool meet(const swr_norm_t* n, const RowTensor& a, const RowTensor& b) {
    const Span sa = span(a.p, a.bytes), sb = span(b.p, b.bytes);
    if (!overlap(sa, sb)) return false;
    const int64_t distance = (int64_t)(sb.lo - sa.lo);
    const std::initializer_list<Dim> dims = {{n->outer, a.so}, {n->inner, a.si}, {n->width, 1}};
    if (a.so != b.so || a.si != b.si || a.es != b.es || distance % a.es != 0 || !apart(dims)) return true;
    const Sorted s(dims);
    return meet_at(s, s.n, distance / a.es);
}

// (Strides of tensors that a call does not have are not looked at: r is the residual, or dh.)
int resolve(const swr_norm_t* n, bool backward, bool has_r, bool has_h, Rows* out) {
    if (!n) return SWR_ERR_NULL;
    if (n->abi_version != SWR_ABI_VERSION) return SWR_ERR_VERSION;
    if (!plain(n->dtype) || (n->weight_dtype != n->dtype && n->weight_dtype != SWR_DTYPE_F32)) return SWR_ERR_DTYPE;
    if (n->out_dtype != n->dtype && (backward || n->out_dtype != SWR_DTYPE_FP8)) return SWR_ERR_DTYPE;
    if (n->reserved != 0 || !(n->eps >= 0.0f) || std::isinf(n->eps)) return SWR_ERR_UNSUPPORTED;
    if (n->outer < 0 || n->inner < 0 || n->width < 1) return SWR_ERR_SHAPE;
    out->es = size_of(n->dtype);
    out->empty = n->outer == 0 || n->inner == 0;
    if (n->width > kMaxWidth || n->outer > kMaxRows || n->inner > kMaxRows) return SWR_ERR_UNSUPPORTED;
    out->rows = n->outer * n->inner;
    if (out->rows > kMaxRows) return SWR_ERR_UNSUPPORTED;
    if (out->empty) return SWR_OK;
    const auto bytes = [&](int64_t so, int64_t si, int es, bool output, int64_t* b) {
        const int64_t off = max_offset({{n->outer, so}, {n->inner, si}, {n->width, 1}});
        if (off < 0 || (output && !apart({{n->outer, so}, {n->inner, si}, {n->width, 1}}))) return false;
        *b = (off + 1) * es;
        return off < kMaxExtent / 8;
    };
    const bool ok = bytes(n->sx_o, n->sx_i, out->es, false, &out->x) &&
                    (!has_r || bytes(n->sr_o, n->sr_i, out->es, false, &out->r)) &&
                    (!has_h || bytes(n->sh_o, n->sh_i, out->es, true, &out->h)) &&
                    bytes(n->sy_o, n->sy_i, size_of(n->out_dtype), !backward, &out->y);
    return ok ? SWR_OK : SWR_ERR_SHAPE;
}

swr::NormParams norm_params(const swr_norm_t* n, const Rows& r) {
    swr::NormParams p = {};
    p.rows = r.rows;
    p.inner = (uint32_t)n->inner;
    p.width = (int32_t)n->width;
    p.eps = n->eps;
    p.sx_o = n->sx_o; p.sx_i = n->sx_i;
    p.sr_o = n->sr_o; p.sr_i = n->sr_i;
    p.sh_o = n->sh_o; p.sh_i = n->sh_i;
    p.sy_o = n->sy_o; p.sy_i = n->sy_i;
    return p;
}

// Whether an output may not lie where `in` does: they share elements and are not
// one and the same tensor, which the kernels update in place.
bool clash(const swr_norm_t* n, const RowTensor& out, const RowTensor& in) {
    const bool same = out.p == in.p && out.so == in.so && out.si == in.si;
    return !same && meet(n, out, in);
}

int64_t norm_stats_bytes(const swr::NormPlan& plan, int64_t rows) {
    return plan.vpt == 0 ? (rows * 8 + 15) / 16 * 16 : 0;
}

}  // namespace

extern "C" {

int swr_rms_norm(const swr_norm_t* n, const void* x, const void* residual, const void* weight, void* y, float* scale,
                 void* h, void* stream) {
    Rows r = {};
    const int rc = resolve(n, false, residual != nullptr, h != nullptr, &r);
    if (rc != SWR_OK) return rc;
    if (r.empty) return SWR_OK;
    const bool fp8 = n->out_dtype == SWR_DTYPE_FP8;
    if (!x || !weight || !y || (fp8 && !scale)) return SWR_ERR_NULL;
    if (!aligned(x, r.es) || !aligned(residual, r.es) || !aligned(h, r.es) || !aligned(y, size_of(n->out_dtype)) ||
        !aligned(weight, size_of(n->weight_dtype)) || (fp8 && !aligned(scale, 4)))
        return SWR_ERR_ALIGN;
    const RowTensor tx{x, n->sx_o, n->sx_i, r.x, r.es}, tr{residual, n->sr_o, n->sr_i, r.r, r.es};
    const RowTensor th{h, n->sh_o, n->sh_i, r.h, r.es}, ty{y, n->sy_o, n->sy_i, r.y, size_of(n->out_dtype)};
    const Span sw = span(weight, n->width * size_of(n->weight_dtype)), ss = span(fp8 ? scale : nullptr, r.rows * 4);
    if (meet(n, ty, tx) || meet(n, ty, tr) || meet(n, ty, th) || clash(n, th, tx) || clash(n, th, tr) ||
        overlaps(span(y, r.y), {sw, ss}) || overlaps(span(h, r.h), {sw, ss}) ||
        overlaps(ss, {span(x, r.x), span(residual, r.r), sw}))
        return SWR_ERR_ALIAS;
    swr::NormParams p = norm_params(n, r);
    p.x = x; p.r = residual; p.w = weight; p.y = y; p.scale = scale; p.h = h;
    return status(swr::launch_norm(*n, swr::plan_norm(n->dtype, r.rows, n->width, false), p, stream));
}

int64_t swr_rms_norm_workspace_bytes(const swr_norm_t* n) {
    Rows r = {};
    const int rc = resolve(n, true, false, true, &r);
    if (rc != SWR_OK) return rc;
    if (r.empty) return 0;
    const swr::NormPlan plan = swr::plan_norm(n->dtype, r.rows, n->width, true);
    return norm_stats_bytes(plan, r.rows) + (int64_t)plan.blocks * n->width * 4;
}

int swr_rms_norm_backward(const swr_norm_t* n, const void* h, const void* weight, const void* dy, const void* dh,
                          void* dx, float* dweight, void* workspace, void* stream) {
    Rows r = {};
    const int rc = resolve(n, true, dh != nullptr, true, &r);
    if (rc != SWR_OK) return rc;
    if (!dweight) return SWR_ERR_NULL;
    if (!aligned(dweight, 4)) return SWR_ERR_ALIGN;
    swr::NormParams p = norm_params(n, r);
    p.dw = dweight;
    if (r.empty)   // no row: dweight is a sum of nothing
        return status(swr::launch_norm_backward(*n, swr::NormPlan{false, 0, 0, 0}, p, stream));
    if (!h || !weight || !dy || !dx || !workspace) return SWR_ERR_NULL;
    if (!aligned(h, r.es) || !aligned(dy, r.es) || !aligned(dh, r.es) || !aligned(dx, r.es) ||
        !aligned(weight, size_of(n->weight_dtype)) || !aligned(workspace, 16))
        return SWR_ERR_ALIGN;
    const swr::NormPlan plan = swr::plan_norm(n->dtype, r.rows, n->width, true);
    const int64_t stats = norm_stats_bytes(plan, r.rows);
    const RowTensor th{h, n->sx_o, n->sx_i, r.x, r.es}, td{dh, n->sr_o, n->sr_i, r.r, r.es};
    const RowTensor tx{dx, n->sh_o, n->sh_i, r.h, r.es}, ty{dy, n->sy_o, n->sy_i, r.y, r.es};
    const Span sw = span(weight, n->width * size_of(n->weight_dtype)), sg = span(dweight, n->width * 4);
    const Span ws = span(workspace, stats + (int64_t)plan.blocks * n->width * 4);
    const Span sh = span(h, r.x), sd = span(dh, r.r), sx = span(dx, r.h), sy = span(dy, r.y);
    if (meet(n, tx, th) || clash(n, tx, ty) || clash(n, tx, td) || overlaps(sx, {sw, sg, ws}) ||
        overlaps(sg, {sh, sd, sy, sw, ws}) || overlaps(ws, {sh, sd, sy, sw}))
        return SWR_ERR_ALIAS;
    p.x = h; p.r = dh; p.w = weight; p.y = const_cast<void*>(dy); p.h = dx;
    p.stats = (float2*)workspace;
    p.partial = (float*)((char*)workspace + stats);
    return status(swr::launch_norm_backward(*n, plan, p, stream));
}

// ---------------------------------------------------------------------------
// 4-bit weights
// ---------------------------------------------------------------------------

static int resolve_fp4(const swr_fp4_t* p, bool pack) {
    if (!p) return SWR_ERR_NULL;
    if (p->abi_version != SWR_ABI_VERSION) return SWR_ERR_VERSION;
    if (!plain(p->dtype) && (pack || p->dtype != SWR_DTYPE_FP8)) return SWR_ERR_DTYPE;
    if (!pack && !plain(p->out_dtype)) return SWR_ERR_DTYPE;
    if (p->reserved != 0) return SWR_ERR_UNSUPPORTED;
    if ((!pack && p->M < 0) || p->N < 0 || p->K < 1) return SWR_ERR_SHAPE;
    if ((!pack && p->M > kMaxWidth) || p->N > kMaxWidth || p->K > kMaxWidth) return SWR_ERR_UNSUPPORTED;
    const int64_t groups = (p->K + 31) / 32, rows = pack ? p->N : p->M;
    if (max_offset({{rows, p->sx}, {p->K, 1}}) < 0 || max_offset({{p->N, p->sc}, {groups * 16, 1}}) < 0 ||
        max_offset({{p->N, p->sp}, {groups, 1}}) < 0)
        return SWR_ERR_SHAPE;
    if (p->N > 1 && pack && (p->sc < groups * 16 || p->sp < groups)) return SWR_ERR_SHAPE;
    if (!pack && (max_offset({{p->M, p->sy}, {p->N, 1}}) < 0 || (p->M > 1 && p->sy < p->N))) return SWR_ERR_SHAPE;
    return SWR_OK;
}

struct Fp4Spans {
    Span x, codes, powers;
};
static Fp4Spans fp4_spans(const swr_fp4_t* p, int64_t rows, const void* x, const void* codes, const void* powers) {
    const int64_t groups = (p->K + 31) / 32;
    return {span(x, (max_offset({{rows, p->sx}, {p->K, 1}}) + 1) * size_of(p->dtype)),
            span(codes, max_offset({{p->N, p->sc}, {groups * 16, 1}}) + 1),
            span(powers, max_offset({{p->N, p->sp}, {groups, 1}}) + 1)};
}

int swr_fp4_linear(const swr_fp4_t* p, const void* x, const float* scale, const void* codes, const void* powers,
                   void* y, void* stream) {
    const int rc = resolve_fp4(p, false);
    if (rc != SWR_OK) return rc;
    if (p->M == 0 || p->N == 0) return SWR_OK;
    if (!x || !codes || !powers || !y) return SWR_ERR_NULL;
    if (!aligned(x, size_of(p->dtype)) || !aligned(y, size_of(p->out_dtype)) || !aligned(scale, 4) ||
        !aligned(codes, 16) || (p->N > 1 && p->sc % 16 != 0))
        return SWR_ERR_ALIGN;
    const Fp4Spans s = fp4_spans(p, p->M, x, codes, powers);
    const Span sy = span(y, (max_offset({{p->M, p->sy}, {p->N, 1}}) + 1) * size_of(p->out_dtype));
    if (overlaps(sy, {s.x, s.codes, s.powers, span(scale, p->M * 4)})) return SWR_ERR_ALIAS;
    const swr::Fp4Params q{x, scale, (const uint8_t*)codes, (const uint8_t*)powers, y, (int32_t)p->M, (int32_t)p->N,
                           (int32_t)p->K, p->sx, p->sy, p->sc, p->sp, 0};
    return status(swr::launch_fp4(p->dtype, p->out_dtype, q, stream));
}

int swr_fp4_pack(const swr_fp4_t* p, const void* w, void* codes, void* powers, void* stream) {
    const int rc = resolve_fp4(p, true);
    if (rc != SWR_OK) return rc;
    if (p->N == 0) return SWR_OK;
    if (!w || !codes || !powers) return SWR_ERR_NULL;
    if (!aligned(w, size_of(p->dtype)) || !aligned(codes, 16) || (p->N > 1 && p->sc % 16 != 0)) return SWR_ERR_ALIGN;
    const Fp4Spans s = fp4_spans(p, p->N, w, codes, powers);
    if (overlaps(s.codes, {s.x, s.powers}) || overlap(s.powers, s.x)) return SWR_ERR_ALIAS;
    return status(swr::launch_fp4_pack(p->dtype, w, p->N, p->K, p->sx, (uint8_t*)codes, (uint8_t*)powers, p->sc, p->sp,
                                       stream));
}

// ---------------------------------------------------------------------------
// Paged cache
// ---------------------------------------------------------------------------

int swr_block_tables(const swr_tables_t* p, const int32_t* lengths, const int32_t* new_tokens,
                     const int32_t* free_stack, const int32_t* free_count, int32_t* table, int64_t* slots,
                     int32_t* starts, int32_t* new_lengths, int32_t* new_free_count, void* stream) {
    if (!p) return SWR_ERR_NULL;
    if (p->abi_version != SWR_ABI_VERSION) return SWR_ERR_VERSION;
    if (p->reserved != 0) return SWR_ERR_UNSUPPORTED;
    if (p->batch < 0 || p->max_pages < 0 || p->tokens < 0 || p->free_pages < 0) return SWR_ERR_SHAPE;
    if (p->page_size < 1 || p->page_size > kMaxPage) return SWR_ERR_BLOCK;
    if (p->batch > kMaxWidth || p->max_pages > kMaxWidth || p->free_pages > kMaxWidth || p->tokens > kMaxRows)
        return SWR_ERR_UNSUPPORTED;
    const int64_t cells = max_offset({{p->batch, p->st}, {p->max_pages, 1}});
    if (cells < 0 || (p->batch > 1 && p->st < p->max_pages)) return SWR_ERR_SHAPE;
    const bool held = p->batch > 0 && p->max_pages > 0;
    if (!free_count || !starts || !new_free_count || (p->batch > 0 && (!lengths || !new_tokens || !new_lengths)) ||
        (held && !table) || (p->free_pages > 0 && !free_stack) || (p->tokens > 0 && !slots))
        return SWR_ERR_NULL;
    for (const void* q : std::initializer_list<const void*>{lengths, new_tokens, free_stack, free_count, table, starts,
                                                            new_lengths, new_free_count})
        if (!aligned(q, 4)) return SWR_ERR_ALIGN;
    if (!aligned(slots, 8)) return SWR_ERR_ALIGN;
    const Span in[4] = {span(lengths, p->batch * 4), span(new_tokens, p->batch * 4),
                        span(free_stack, p->free_pages * 4), span(free_count, 4)};
    const Span out[5] = {span(held ? table : nullptr, (cells + 1) * 4), span(slots, p->tokens * 8),
                         span(starts, (p->batch + 1) * 4), span(new_lengths, p->batch * 4), span(new_free_count, 4)};
    for (int i = 0; i < 5; ++i) {
        for (const Span& s : in)
            if (overlap(out[i], s)) return SWR_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return SWR_ERR_ALIAS;
    }
    swr::TableParams q = {};
    q.lengths = lengths; q.news = new_tokens; q.stack = free_stack; q.count = free_count;
    q.table = table; q.slots = slots; q.starts = starts; q.new_lengths = new_lengths; q.new_count = new_free_count;
    q.batch = (int32_t)p->batch; q.max_pages = (int32_t)p->max_pages; q.page_size = (int32_t)p->page_size;
    q.free_pages = (int32_t)p->free_pages;
    q.st = p->st; q.tokens = p->tokens; q.page = swr::Divisor(p->page_size);
    return status(swr::launch_tables(q, stream));
}

// The cache's checks; *bytes: what it spans.
static int resolve_cache(const swr_cache_t* c, int64_t* bytes) {
    if (c->abi_version != SWR_ABI_VERSION) return SWR_ERR_VERSION;
    if (!plain(c->dtype)) return SWR_ERR_DTYPE;
    if (c->pages < 0 || c->heads < 1 || c->D < 1) return SWR_ERR_SHAPE;
    if (c->page_size < 1 || c->page_size > kMaxPage) return SWR_ERR_BLOCK;
    if (c->D % 16 != 0 || c->D > 256 || c->pages > kMaxRows || c->heads > 65536) return SWR_ERR_UNSUPPORTED;
    const int es = size_of(c->dtype);
    const std::initializer_list<Dim> dims = {{c->pages, c->s_page}, {c->page_size, c->s_token}, {c->heads, c->s_head},
                                             {c->D, 1}};
    const int64_t off = max_offset(dims);
    if (off < 0 || !apart(dims)) return SWR_ERR_SHAPE;
    if (!vectors({{c->pages, c->s_page}, {c->page_size, c->s_token}, {c->heads, c->s_head}}, es)) return SWR_ERR_ALIGN;
    if (off >= ((int64_t)1 << 36) / es) return SWR_ERR_UNSUPPORTED;
    *bytes = c->pages ? (off + 1) * es : 0;
    return SWR_OK;
}

int swr_cache_append(const swr_cache_t* c, int64_t tokens, const int64_t* sk, const int64_t* sv, const void* k,
                     const void* v, const int64_t* slots, void* k_cache, void* v_cache, void* stream) {
    if (!c || !sk || !sv) return SWR_ERR_NULL;
    int64_t bytes;
    const int rc = resolve_cache(c, &bytes);
    if (rc != SWR_OK) return rc;
    if (tokens < 0) return SWR_ERR_SHAPE;
    if (tokens > kMaxRows) return SWR_ERR_UNSUPPORTED;
    const int es = size_of(c->dtype);
    const int64_t ok = max_offset({{tokens, sk[0]}, {c->heads, sk[1]}, {c->D, 1}});
    const int64_t ov = max_offset({{tokens, sv[0]}, {c->heads, sv[1]}, {c->D, 1}});
    if (ok < 0 || ov < 0) return SWR_ERR_SHAPE;
    if (!vectors({{tokens, sk[0]}, {tokens, sv[0]}, {c->heads, sk[1]}, {c->heads, sv[1]}}, es)) return SWR_ERR_ALIGN;
    if (tokens == 0 || c->pages == 0) return SWR_OK;
    if (!k || !v || !slots || !k_cache || !v_cache) return SWR_ERR_NULL;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(slots, 8))
        return SWR_ERR_ALIGN;
    const Span in[3] = {span(k, (ok + 1) * es), span(v, (ov + 1) * es), span(slots, tokens * 8)};
    const Span out[2] = {span(k_cache, bytes), span(v_cache, bytes)};
    // The two caches may be parts of one allocation, between each other's elements.
    const Sorted dims({{c->pages, c->s_page}, {c->page_size, c->s_token}, {c->heads, c->s_head}, {c->D, 1}});
    if (overlap(out[0], out[1]) && meet_at(dims, dims.n, (int64_t)(out[1].lo - out[0].lo) / es)) return SWR_ERR_ALIAS;
    for (const Span& s : in)
        if (overlaps(s, {out[0], out[1]})) return SWR_ERR_ALIAS;
    const int64_t unit = 16 / es;
    swr::AppendParams p = {};
    p.k = k; p.v = v; p.k_cache = k_cache; p.v_cache = v_cache; p.slots = slots;
    p.tokens = tokens;
    p.rows = c->pages * c->page_size;
    p.page_size = (uint32_t)c->page_size;
    p.per_head = (uint32_t)(c->D / unit);
    p.per_token = (uint32_t)(c->heads * (c->D / unit));
    p.sk_t = sk[0] / unit; p.sk_h = sk[1] / unit; p.sv_t = sv[0] / unit; p.sv_h = sv[1] / unit;
    p.s_page = c->s_page / unit; p.s_token = c->s_token / unit; p.s_head = c->s_head / unit;
    return status(swr::launch_append(p, stream));
}

// Scores are taken times log2 e, in float32.
static float log2_scale(const swr_paged_t* p) { return p->scale * 1.44269504088896340736f; }

static int resolve_paged(const swr_paged_t* p, int64_t* cache, int64_t* q, int64_t* y) {
    if (!p) return SWR_ERR_NULL;
    const int rc = resolve_cache(&p->cache, cache);
    if (rc != SWR_OK) return rc;
    if (p->batch < 0 || p->q_heads < 1 || p->q_heads % p->cache.heads != 0 || p->max_pages < 0 || p->window < 0)
        return SWR_ERR_SHAPE;
    if (p->reserved != 0 || !std::isfinite(log2_scale(p)) || p->q_heads > 65536 || p->batch > kMaxRows / 65536 ||
        p->max_pages > kMaxWidth)
        return SWR_ERR_UNSUPPORTED;
    const int es = size_of(p->cache.dtype);
    const int64_t cells = max_offset({{p->batch, p->st}, {p->max_pages, 1}});
    const int64_t oq = max_offset({{p->batch, p->sq_b}, {p->q_heads, p->sq_h}, {p->cache.D, 1}});
    const int64_t oy = max_offset({{p->batch, p->sy_b}, {p->q_heads, p->sy_h}, {p->cache.D, 1}});
    if (cells < 0 || oq < 0 || oy < 0 || !apart({{p->batch, p->sy_b}, {p->q_heads, p->sy_h}, {p->cache.D, 1}}))
        return SWR_ERR_SHAPE;
    if (!vectors({{p->batch, p->sq_b}, {p->batch, p->sy_b}, {p->q_heads, p->sq_h}, {p->q_heads, p->sy_h}}, es))
        return SWR_ERR_ALIGN;
    *q = (oq + 1) * es;
    *y = (oy + 1) * es;
    return SWR_OK;
}

int64_t swr_paged_workspace_bytes(const swr_paged_t* p) {
    int64_t cache, q, y;
    const int rc = resolve_paged(p, &cache, &q, &y);
    if (rc != SWR_OK) return rc;
    if (p->batch == 0) return 0;
    return swr::paged_work_floats(*p) * 4;
}

int swr_paged_attention(const swr_paged_t* p, const void* q, const void* k_cache, const void* v_cache,
                        const int32_t* table, const int32_t* lengths, void* y, float* lse, void* workspace,
                        void* stream) {
    int64_t bc, bq, by;
    const int rc = resolve_paged(p, &bc, &bq, &by);
    if (rc != SWR_OK) return rc;
    if (p->batch == 0) return SWR_OK;
    const bool cached = p->cache.pages > 0 && p->max_pages > 0;
    const int64_t work = swr::paged_work_floats(*p) * 4;
    if (!q || !y || !lengths || (work > 0 && !workspace)) return SWR_ERR_NULL;
    if (cached && (!k_cache || !v_cache || !table)) return SWR_ERR_NULL;
    if (!aligned(q, 16) || !aligned(y, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(table, 4) ||
        !aligned(lengths, 4) || !aligned(lse, 4) || !aligned(workspace, 16))
        return SWR_ERR_ALIGN;
    const int64_t cells = (max_offset({{p->batch, p->st}, {p->max_pages, 1}}) + 1) * 4;
    const Span in[5] = {span(q, bq), span(k_cache, bc), span(v_cache, bc), span(cached ? table : nullptr, cells),
                        span(lengths, p->batch * 4)};
    const Span out[3] = {span(y, by), span(lse, p->batch * p->q_heads * 4), span(workspace, work)};
    for (int i = 0; i < 3; ++i) {
        for (const Span& s : in)
            if (overlap(out[i], s)) return SWR_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return SWR_ERR_ALIAS;
    }
    const int64_t unit = 16 / size_of(p->cache.dtype);
    swr::PagedParams a = {};
    a.q = q; a.k = k_cache; a.v = v_cache; a.table = table; a.lengths = lengths; a.y = y; a.lse = lse;
    a.batch = (int32_t)p->batch;
    a.kv_heads = (int32_t)p->cache.heads;
    a.group = (int32_t)(p->q_heads / p->cache.heads);
    a.head_tiles = (a.group + 15) / 16;
    a.D = (int32_t)p->cache.D;
    a.max_pages = p->cache.pages > 0 ? (int32_t)p->max_pages : 0;   // (no page: no position)
    a.page = swr::Divisor(p->cache.page_size);
    a.pages = (int32_t)p->cache.pages;
    a.workgroups = swr::paged_workgroups(*p);
    a.cuts = (int32_t*)workspace;
    a.part = (float*)workspace + 4 * (int64_t)a.workgroups;
    a.st = p->st;
    a.window = p->window;
    a.sq_b = p->sq_b; a.sq_h = p->sq_h; a.sy_b = p->sy_b; a.sy_h = p->sy_h;
    a.s_page = (uint32_t)(p->cache.s_page / unit);
    a.s_token = (uint32_t)(p->cache.s_token / unit);
    a.s_head = (uint32_t)(p->cache.s_head / unit);
    a.scale_log2 = log2_scale(p);
    return status(swr::launch_paged(p->cache.dtype, a, stream));
}

}  // extern "C"
