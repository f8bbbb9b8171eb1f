// swr_lm_api.cpp -- C ABI of a recurrent language model's operators: argument
// validation (done entirely before any HIP runtime call) and dispatch to their
// gfx950 kernels.
#include <stdint.h>

#include <cmath>
#include <initializer_list>

#include "../../include/swr_lm.h"
#include "swr_checks.h"
#include "swr_lm_launch.h"

namespace {

constexpr int64_t kMostBatch = (int64_t)1 << 30;

bool all_aligned(std::initializer_list<const void*> ps, int64_t bytes) {
    for (const void* p : ps)
        if (!aligned(p, bytes)) return false;
    return true;
}
// Whether some output overlaps an input, or another output.
bool clashes(std::initializer_list<Span> out, std::initializer_list<Span> in) {
    for (const Span* o = out.begin(); o != out.end(); ++o) {
        if (overlaps(*o, in)) return true;
        for (const Span* q = out.begin(); q != o; ++q)
            if (overlap(*o, *q)) return true;
    }
    return false;
}
// A tensor of rows, [B, T] of them, as a call has it (p NULL: not there); sizes and strides in bytes.
struct RowTensor {
    const void* p;
    int64_t sb, st, width;
    Span span;
};
RowTensor rows_of(const void* p, int64_t sb, int64_t st, int64_t width, int es, int64_t bytes) {
    // (unsigned: a dimension of one has any stride)
    return {p, (int64_t)((uint64_t)sb * es), (int64_t)((uint64_t)st * es), width * es, span(p, bytes)};
}
// Whether a and b share a byte.  Parts of one larger tensor have its rows' strides, and lie between each other's
// elements: theirs are compared row by row; others are taken to meet where their spans do.
bool meet(int64_t B, int64_t T, const RowTensor& a, const RowTensor& b) {
    if (!overlap(a.span, b.span)) return false;
    if ((B > 1 && a.sb != b.sb) || (T > 1 && a.st != b.st)) return true;
    const int64_t width = a.width > b.width ? a.width : b.width;
    if (!apart({{B, a.sb}, {T, a.st}, {width, 1}})) return true;
    // Some rows are (i sb + j st) apart, |i| < B and |j| < T: they meet where that is within their widths of the
    // tensors' distance.  The lesser dimensions reach less far than a dimension's stride, so only its two multiples
    // next to what is left count.
    const Sorted s({{B, a.sb}, {T, a.st}});
    const auto rows = [&](const auto& self, int dims, int64_t distance) -> bool {
        if (dims == 0) return distance < a.width && -distance < b.width;
        const Dim& d = s.d[dims - 1];
        const int64_t below = distance / d.stride - (distance % d.stride < 0);
        for (int64_t i = below; i <= below + 1; ++i)
            if (i > -d.size && i < d.size && self(self, dims - 1, distance - i * d.stride)) return true;
        return false;
    };
    return rows(rows, s.n, (int64_t)(b.span.lo - a.span.lo));
}
bool meets(int64_t B, int64_t T, const RowTensor& out, std::initializer_list<RowTensor> in) {
    for (const RowTensor& t : in)
        if (meet(B, T, out, t)) return true;
    return false;
}
// Bytes that a tensor spans, or -1: its offsets are out of range.
int64_t extent(std::initializer_list<Dim> dims, int es) {
    for (const Dim& d : dims)
        if (d.size == 0) return 0;
    const int64_t off = max_offset(dims);
    return off < 0 || off >= kMaxExtent / 8 ? -1 : (off + 1) * es;
}
// a b, or -1 past the largest extent.
int64_t times(int64_t a, int64_t b) { return b != 0 && a > kMaxExtent / b ? -1 : a * b; }

// ---------------------------------------------------------------------------
// Embedding
// ---------------------------------------------------------------------------

struct EmbedSizes {
    int64_t tokens, table, rows;   // bytes
};
int resolve(const swr_embed_t* e, bool backward, EmbedSizes* s) {
    if (!e) return SWR_ERR_NULL;
    if (e->abi_version != SWR_ABI_VERSION) return SWR_ERR_VERSION;
    if (!plain(e->dtype) || (e->out_dtype != e->dtype && !(backward && e->out_dtype == SWR_DTYPE_F32)))
        return SWR_ERR_DTYPE;
    if (e->token_bytes != 4 && e->token_bytes != 8) return SWR_ERR_DTYPE;
    if (e->reserved != 0 || !std::isfinite(e->scale)) return SWR_ERR_UNSUPPORTED;
    if (e->tokens < 0 || e->vocab < 1 || e->width < 1) return SWR_ERR_SHAPE;
    if (e->tokens > kMaxRows || e->vocab > kMaxWidth || e->width > kMaxWidth) return SWR_ERR_UNSUPPORTED;
    const std::initializer_list<Dim> table = {{e->vocab, e->st}, {e->width, 1}}, rows = {{e->tokens, e->sy}, {e->width, 1}};
    s->tokens = e->tokens * e->token_bytes;
    s->table = extent(table, size_of(backward ? e->out_dtype : e->dtype));
    s->rows = extent(rows, size_of(e->dtype));
    if (s->table < 0 || s->rows < 0) return SWR_ERR_SHAPE;
    if (!apart({{e->vocab, e->st}, {e->width, 1}}) && backward) return SWR_ERR_SHAPE;
    if (!backward && e->tokens > 0 && !apart(rows)) return SWR_ERR_SHAPE;
    return SWR_OK;
}

swr::EmbedParams embed_params(const swr_embed_t* e, const void* tokens, const void* in, void* out) {
    swr::EmbedParams p = {};
    p.tokens = tokens;
    p.wide_tokens = e->token_bytes == 8;
    p.in = in;
    p.out = out;
    p.rows = e->tokens; p.vocab = e->vocab; p.width = e->width;
    p.scale = e->scale;
    return p;
}

// ---------------------------------------------------------------------------
// Convolution
// ---------------------------------------------------------------------------

struct ConvSizes {
    int64_t x, y, dx, w, bias, state, lengths;   // bytes
    bool empty;
};
int resolve(const swr_conv_t* p, bool backward, ConvSizes* s) {
    if (!p) return SWR_ERR_NULL;
    if (p->abi_version != SWR_ABI_VERSION) return SWR_ERR_VERSION;
    if (!plain(p->dtype)) return SWR_ERR_DTYPE;
    if (p->flags & ~SWR_CONV_SILU) return SWR_ERR_UNSUPPORTED;
    if (p->B < 0 || p->T < 0 || p->C < 1 || p->taps < 1) return SWR_ERR_SHAPE;
    if (p->taps > 8 || p->B > kMostBatch || p->T > kMostBatch || p->C > kMaxWidth) return SWR_ERR_UNSUPPORTED;
    const int64_t tokens = times(p->B, p->T);
    if (tokens < 0 || times(tokens, p->C) < 0 || times(p->B * 8, p->C) < 0) return SWR_ERR_UNSUPPORTED;
    if (tokens > ((int64_t)1 << 40)) return SWR_ERR_UNSUPPORTED;
    const int es = size_of(p->dtype);
    s->x = extent({{p->B, p->sx_b}, {p->T, p->sx_t}, {p->C, 1}}, es);
    s->y = extent({{p->B, p->sy_b}, {p->T, p->sy_t}, {p->C, 1}}, es);
    s->dx = backward ? extent({{p->B, p->sd_b}, {p->T, p->sd_t}, {p->C, 1}}, es) : 0;
    if (s->x < 0 || s->y < 0 || s->dx < 0) return SWR_ERR_SHAPE;
    s->empty = tokens == 0;
    if (!s->empty && !backward && !apart({{p->B, p->sy_b}, {p->T, p->sy_t}, {p->C, 1}})) return SWR_ERR_SHAPE;
    if (!s->empty && backward && !apart({{p->B, p->sd_b}, {p->T, p->sd_t}, {p->C, 1}})) return SWR_ERR_SHAPE;
    s->w = p->C * p->taps * es;
    s->bias = p->C * es;
    s->state = p->B * (p->taps - 1) * p->C * es;
    s->lengths = p->B * 4;
    return SWR_OK;
}

swr::ConvParams conv_params(const swr_conv_t* p, const void* x, const void* w, const void* bias, const int32_t* lengths) {
    swr::ConvParams q = {};
    q.x = x; q.w = w; q.bias = bias; q.lengths = lengths;
    q.B = p->B; q.T = p->T; q.C = p->C;
    q.sx_b = p->sx_b; q.sx_t = p->sx_t; q.sy_b = p->sy_b; q.sy_t = p->sy_t; q.sd_b = p->sd_b; q.sd_t = p->sd_t;
    q.silu = p->flags & SWR_CONV_SILU;
    return q;
}

// ---------------------------------------------------------------------------
// Scan
// ---------------------------------------------------------------------------

struct ScanSizes {
    int64_t x, dt, z, y, B, C, A, channel, state, lengths, dense, shared, carriers;   // bytes
    int es;
};
int resolve(const swr_scan_t* p, bool has_z, bool backward, ScanSizes* s) {
    if (!p) return SWR_ERR_NULL;
    if (p->abi_version != SWR_ABI_VERSION) return SWR_ERR_VERSION;
    if (!plain(p->dtype)) return SWR_ERR_DTYPE;
    if (p->flags & ~SWR_SCAN_SOFTPLUS) return SWR_ERR_UNSUPPORTED;
    if (p->B < 0 || p->T < 0 || p->D < 1 || p->G < 1 || p->D % p->G != 0 || p->N < 1) return SWR_ERR_SHAPE;
    if (p->N > 64 || p->B > kMostBatch || p->T > kMostBatch || p->D > kMostBatch / 4) return SWR_ERR_UNSUPPORTED;
    // (the largest tensors: states of every block of tokens, shares of the gradients)
    const int64_t tokens = times(p->B, p->T + SWR_SCAN_BLOCK);
    if (tokens < 0 || tokens > ((int64_t)1 << 40) || times(tokens, p->D * 256) < 0) return SWR_ERR_UNSUPPORTED;
    const int es = s->es = size_of(p->dtype);
    s->x = extent({{p->B, p->sx_b}, {p->T, p->sx_t}, {p->D, 1}}, es);
    s->dt = extent({{p->B, p->sdt_b}, {p->T, p->sdt_t}, {p->D, 1}}, es);
    s->z = has_z ? extent({{p->B, p->sz_b}, {p->T, p->sz_t}, {p->D, 1}}, es) : 0;
    s->y = extent({{p->B, p->sy_b}, {p->T, p->sy_t}, {p->D, 1}}, es);
    s->B = extent({{p->B, p->sB_b}, {p->T, p->sB_t}, {p->G, p->sB_g}, {p->N, 1}}, es);
    s->C = extent({{p->B, p->sC_b}, {p->T, p->sC_t}, {p->G, p->sC_g}, {p->N, 1}}, es);
    if (s->x < 0 || s->dt < 0 || s->z < 0 || s->y < 0 || s->B < 0 || s->C < 0) return SWR_ERR_SHAPE;
    if (!backward && p->B > 0 && p->T > 0 && !apart({{p->B, p->sy_b}, {p->T, p->sy_t}, {p->D, 1}})) return SWR_ERR_SHAPE;
    s->A = p->D * p->N * 4;
    s->channel = p->D * 4;
    s->state = p->B * p->D * p->N * 4;
    s->lengths = p->B * 4;
    s->dense = p->B * p->T * p->D * es;
    s->shared = p->B * p->T * p->G * p->N * es;
    s->carriers = p->B * ((p->T + SWR_SCAN_BLOCK - 1) / SWR_SCAN_BLOCK) * p->D * p->N * 4;
    return SWR_OK;
}

swr::ScanParams scan_params(const swr_scan_t* p, const swr_scan_inputs_t* in, const swr::ScanPlan& plan) {
    swr::ScanParams q = {};
    q.in = *in;
    q.B = p->B; q.T = p->T; q.D = p->D; q.G = p->G; q.Dg = p->D / p->G;
    q.N = p->N;
    q.softplus = p->flags & SWR_SCAN_SOFTPLUS;
    q.sx_b = p->sx_b; q.sx_t = p->sx_t; q.sdt_b = p->sdt_b; q.sdt_t = p->sdt_t; q.sz_b = p->sz_b; q.sz_t = p->sz_t;
    q.sy_b = p->sy_b; q.sy_t = p->sy_t;
    q.sB_b = p->sB_b; q.sB_t = p->sB_t; q.sB_g = p->sB_g; q.sC_b = p->sC_b; q.sC_t = p->sC_t; q.sC_g = p->sC_g;
    q.chunk = plan.chunk; q.chunks = plan.chunks; q.tiles = plan.tiles; q.work = plan.blocks(p->B, p->G);
    return q;
}

// ---------------------------------------------------------------------------
// Log probabilities
// ---------------------------------------------------------------------------

int resolve(const swr_logprob_t* p, bool backward, int64_t* logits, int64_t* gradient) {
    if (!p) return SWR_ERR_NULL;
    if (p->abi_version != SWR_ABI_VERSION) return SWR_ERR_VERSION;
    if (!plain(p->dtype) || (p->token_bytes != 4 && p->token_bytes != 8)) return SWR_ERR_DTYPE;
    if (p->reserved != 0 || !(p->scale > 0.0f) || !std::isfinite(p->scale * 1.44269504088896340736f))
        return SWR_ERR_UNSUPPORTED;
    if (p->rows < 0 || p->vocab < 1 || p->top < 0 || p->top > p->vocab) return SWR_ERR_SHAPE;
    if (p->rows > kMaxRows || p->vocab > kMaxWidth || p->top > SWR_TOP_MOST) return SWR_ERR_UNSUPPORTED;
    const int es = size_of(p->dtype);
    *logits = extent({{p->rows, p->sl}, {p->vocab, 1}}, es);
    *gradient = backward ? extent({{p->rows, p->sd}, {p->vocab, 1}}, es) : 0;
    if (*logits < 0 || *gradient < 0) return SWR_ERR_SHAPE;
    if (backward && p->rows > 0 && !apart({{p->rows, p->sd}, {p->vocab, 1}})) return SWR_ERR_SHAPE;
    return SWR_OK;
}

swr::LogProbParams logprob_params(const swr_logprob_t* p, const void* logits, const void* tokens) {
    swr::LogProbParams q = {};
    q.logits = logits; q.tokens = tokens;
    q.wide_tokens = p->token_bytes == 8;
    q.rows = p->rows; q.vocab = p->vocab; q.sl = p->sl; q.sd = p->sd;
    q.top = p->top;
    q.scale = p->scale;
    return q;
}

}  // namespace

extern "C" {

int swr_embedding(const swr_embed_t* e, const void* tokens, const void* table, void* y, void* stream) {
    EmbedSizes s;
    const int rc = resolve(e, false, &s);
    if (rc != SWR_OK) return rc;
    if (e->tokens == 0) return SWR_OK;
    if (!tokens || !table || !y) return SWR_ERR_NULL;
    const int es = size_of(e->dtype);
    if (!aligned(tokens, e->token_bytes) || !all_aligned({table, y}, es)) return SWR_ERR_ALIGN;
    if (clashes({span(y, s.rows)}, {span(tokens, s.tokens), span(table, s.table)})) return SWR_ERR_ALIAS;
    swr::EmbedParams p = embed_params(e, tokens, table, y);
    p.s_in = e->st; p.s_out = e->sy;
    return status(swr::launch_embed(e->dtype, p, stream));
}

int64_t swr_embedding_workspace_bytes(const swr_embed_t* e) {
    EmbedSizes s;
    const int rc = resolve(e, true, &s);
    return rc != SWR_OK ? rc : swr::embed_work_bytes(e->tokens, e->vocab, e->width);
}

int swr_embedding_backward(const swr_embed_t* e, const void* tokens, const void* dy, void* dtable, void* workspace,
                           void* stream) {
    EmbedSizes s;
    const int rc = resolve(e, true, &s);
    if (rc != SWR_OK) return rc;
    if (!dtable || (e->tokens > 0 && (!tokens || !dy || !workspace))) return SWR_ERR_NULL;
    if (!aligned(tokens, e->token_bytes) || !aligned(dy, size_of(e->dtype)) || !aligned(dtable, size_of(e->out_dtype)) ||
        !aligned(workspace, 16))
        return SWR_ERR_ALIGN;
    const int64_t work = swr::embed_work_bytes(e->tokens, e->vocab, e->width);
    if (clashes({span(dtable, s.table), span(workspace, work)}, {span(tokens, s.tokens), span(dy, s.rows)}))
        return SWR_ERR_ALIAS;
    swr::EmbedParams p = embed_params(e, tokens, dy, dtable);
    p.s_in = e->sy; p.s_out = e->st;
    return status(swr::launch_embed_backward(e->dtype, e->out_dtype, p, workspace, stream));
}

int swr_causal_conv(const swr_conv_t* p, const void* x, const void* w, const void* bias, const void* state,
                    const int32_t* lengths, void* y, void* state_out, void* stream) {
    ConvSizes s;
    const int rc = resolve(p, false, &s);
    if (rc != SWR_OK) return rc;
    const bool keeps = state_out && s.state > 0;
    if (p->B == 0 || (s.empty && !keeps)) return SWR_OK;
    if (!w || (!s.empty && (!x || !y))) return SWR_ERR_NULL;
    if (!all_aligned({x, w, bias, state, y, state_out}, size_of(p->dtype)) || !aligned(lengths, 4)) return SWR_ERR_ALIGN;
    const Span so = span(keeps ? state_out : nullptr, s.state), ss = span(state, s.state);
    const Span sx = span(x, s.x), sw = span(w, s.w), sb = span(bias, s.bias), sl = span(lengths, s.lengths);
    const int es = size_of(p->dtype);
    if (clashes({span(y, s.y), so}, {sw, sb, sl}) || overlap(so, sx) || overlap(span(y, s.y), ss) ||
        (state_out != state && overlap(so, ss)) ||
        meet(p->B, p->T, rows_of(y, p->sy_b, p->sy_t, p->C, es, s.y), rows_of(x, p->sx_b, p->sx_t, p->C, es, s.x)))
        return SWR_ERR_ALIAS;
    swr::ConvParams q = conv_params(p, x, w, bias, lengths);
    q.state = s.state > 0 ? state : nullptr;
    q.state_out = keeps ? state_out : nullptr;
    q.y = y;
    return status(swr::launch_conv(p->dtype, p->taps, q, stream));
}

int64_t swr_causal_conv_workspace_bytes(const swr_conv_t* p) {
    ConvSizes s;
    const int rc = resolve(p, true, &s);
    return rc != SWR_OK ? rc : swr::conv_work_bytes(p->B, p->T, p->C, p->taps);
}

int swr_causal_conv_backward(const swr_conv_t* p, const void* x, const void* w, const void* bias, const void* dy,
                             const int32_t* lengths, void* dx, float* dw, float* dbias, void* workspace,
                             void* stream) {
    ConvSizes s;
    const int rc = resolve(p, true, &s);
    if (rc != SWR_OK) return rc;
    if (!w || !dw || !workspace || (!s.empty && (!x || !dy || !dx))) return SWR_ERR_NULL;
    if (!all_aligned({x, w, bias, dy, dx}, size_of(p->dtype)) || !all_aligned({lengths, dw, dbias}, 4) ||
        !aligned(workspace, 16))
        return SWR_ERR_ALIGN;
    const int64_t work = swr::conv_work_bytes(p->B, p->T, p->C, p->taps);
    const int es = size_of(p->dtype);
    const Span sx = span(x, s.x), sy = span(dy, s.y);
    if (clashes({span(dx, s.dx), span(dw, p->C * p->taps * 4), span(dbias, p->C * 4), span(workspace, work)},
                {span(w, s.w), span(bias, s.bias), span(lengths, s.lengths)}) ||
        clashes({span(dw, p->C * p->taps * 4), span(dbias, p->C * 4), span(workspace, work)}, {sx, sy}) ||
        meets(p->B, p->T, rows_of(dx, p->sd_b, p->sd_t, p->C, es, s.dx),
              {rows_of(x, p->sx_b, p->sx_t, p->C, es, s.x), rows_of(dy, p->sy_b, p->sy_t, p->C, es, s.y)}))
        return SWR_ERR_ALIAS;
    swr::ConvParams q = conv_params(p, x, w, bias, lengths);
    q.dy = dy; q.dx = dx; q.dw = dw; q.db = dbias; q.partial = (float*)workspace;
    return status(swr::launch_conv_backward(p->dtype, p->taps, q, stream));
}

int64_t swr_selective_scan_workspace_bytes(const swr_scan_t* p) {
    ScanSizes s;
    const int rc = resolve(p, false, true, &s);
    if (rc != SWR_OK) return rc;
    return p->B == 0 ? 0 : swr::scan_work_floats(*p, swr::plan_scan(*p, false)) * 4;
}

int swr_selective_scan(const swr_scan_t* p, const swr_scan_inputs_t* in, void* y, float* carriers, float* h_last,
                       void* workspace, void* stream) {
    if (!in) return SWR_ERR_NULL;
    ScanSizes s;
    const int rc = resolve(p, in->z != nullptr, false, &s);
    if (rc != SWR_OK) return rc;
    if (p->B == 0 || (p->T == 0 && !h_last)) return SWR_OK;
    const swr::ScanPlan plan = swr::plan_scan(*p, false);
    const int64_t work = swr::scan_work_floats(*p, plan) * 4;
    if (!in->A || (p->T > 0 && (!in->x || !in->dt || !in->B || !in->C || !y)) || (work > 0 && !workspace))
        return SWR_ERR_NULL;
    if (!all_aligned({in->x, in->dt, in->B, in->C, in->z, y}, s.es) ||
        !all_aligned({in->A, in->bias, in->skip, in->h0, in->lengths, carriers, h_last}, 4) || !aligned(workspace, 16))
        return SWR_ERR_ALIGN;
    const Span sh = span(in->h0, s.state), so = span(h_last, s.state), sy = span(y, s.y), sc = span(carriers, s.carriers);
    const Span sw = span(workspace, work);
    // (B's and C's rows of a token, G of N elements, count as one from the first to the last)
    const int64_t wb = (p->G - 1) * p->sB_g + p->N, wc = (p->G - 1) * p->sC_g + p->N;
    if (clashes({sy, sc, so, sw}, {span(in->A, s.A), span(in->bias, s.channel), span(in->skip, s.channel),
                                   span(in->lengths, s.lengths)}) ||
        clashes({sc, so, sw}, {span(in->x, s.x), span(in->dt, s.dt), span(in->B, s.B), span(in->C, s.C), span(in->z, s.z)}) ||
        overlaps(sh, {sy, sc, sw}) || (h_last != in->h0 && overlap(sh, so)) ||
        meets(p->B, p->T, rows_of(y, p->sy_b, p->sy_t, p->D, s.es, s.y),
              {rows_of(in->x, p->sx_b, p->sx_t, p->D, s.es, s.x), rows_of(in->dt, p->sdt_b, p->sdt_t, p->D, s.es, s.dt),
               rows_of(in->z, p->sz_b, p->sz_t, p->D, s.es, s.z), rows_of(in->B, p->sB_b, p->sB_t, wb, s.es, s.B),
               rows_of(in->C, p->sC_b, p->sC_t, wc, s.es, s.C)}))
        return SWR_ERR_ALIAS;
    swr::ScanParams q = scan_params(p, in, plan);
    q.y = y; q.carriers = carriers; q.h_last = h_last;
    q.states = (float*)workspace;
    q.steps = q.states + p->B * plan.chunks * p->D * p->N;
    return status(swr::launch_scan(p->dtype, plan, q, stream));
}

int64_t swr_selective_scan_backward_workspace_bytes(const swr_scan_t* p) {
    ScanSizes s;
    const int rc = resolve(p, false, true, &s);
    if (rc != SWR_OK) return rc;
    return swr::scan_backward_work_floats(*p, swr::plan_scan(*p, true)) * 4;
}

int swr_selective_scan_backward(const swr_scan_t* p, const swr_scan_inputs_t* in, const void* dy,
                                const float* carriers, const float* dh_last, const swr_scan_gradients_t* out,
                                void* workspace, void* stream) {
    if (!in || !out) return SWR_ERR_NULL;
    ScanSizes s;
    const int rc = resolve(p, in->z != nullptr, true, &s);
    if (rc != SWR_OK) return rc;
    const swr::ScanPlan plan = swr::plan_scan(*p, true);
    const int64_t work = swr::scan_backward_work_floats(*p, plan) * 4;
    const bool tokens = p->B > 0 && p->T > 0;
    if (!in->A || !out->dA || (work > 0 && !workspace)) return SWR_ERR_NULL;
    if (tokens && (!in->x || !in->dt || !in->B || !in->C || !dy || !carriers || !out->dx || !out->ddt || !out->dB ||
                   !out->dC))
        return SWR_ERR_NULL;
    // Gradients of what there is, and of nothing else.
    if ((tokens && !in->z != !out->dz) || !in->bias != !out->dbias || !in->skip != !out->dskip) return SWR_ERR_NULL;
    if (!all_aligned({in->x, in->dt, in->B, in->C, in->z, dy, out->dx, out->ddt, out->dB, out->dC, out->dz}, s.es) ||
        !all_aligned({in->A, in->bias, in->skip, in->h0, in->lengths, carriers, dh_last, out->dA, out->dbias, out->dskip,
                      out->dh0}, 4) ||
        !aligned(workspace, 16))
        return SWR_ERR_ALIGN;
    if (clashes({span(out->dx, s.dense), span(out->ddt, s.dense), span(out->dA, s.A), span(out->dB, s.shared),
                 span(out->dC, s.shared), span(out->dbias, s.channel), span(out->dskip, s.channel), span(out->dz, s.dense),
                 span(out->dh0, s.state), span(workspace, work)},
                {span(in->x, s.x), span(in->dt, s.dt), span(in->A, s.A), span(in->B, s.B), span(in->C, s.C),
                 span(in->bias, s.channel), span(in->skip, s.channel), span(in->z, s.z), span(in->h0, s.state),
                 span(in->lengths, s.lengths), span(dy, s.y), span(carriers, s.carriers), span(dh_last, s.state)}))
        return SWR_ERR_ALIAS;
    swr::ScanParams q = scan_params(p, in, plan);
    q.dy = dy; q.carriers_in = carriers; q.dh_last = dh_last;
    q.out = *out;
    const int64_t runs = p->B * plan.chunks;
    q.states = (float*)workspace;
    q.steps = q.states + runs * p->D * p->N;
    q.shares = (float*)workspace + swr::scan_work_floats(*p, plan);
    q.sums = q.shares + p->B * p->T * p->G * plan.tiles * 2 * p->N;
    return status(swr::launch_scan_backward(p->dtype, plan, q, stream));
}

int64_t swr_log_probs_workspace_bytes(const swr_logprob_t* p) {
    int64_t logits, gradient;
    const int rc = resolve(p, false, &logits, &gradient);
    return rc != SWR_OK ? rc : swr::logprob_work_bytes(p->rows, p->vocab, p->top);
}

int swr_log_probs(const swr_logprob_t* p, const void* logits, const void* tokens, float* logp, float* lse,
                  float* entropy, float* top_logp, int64_t* top_tokens, void* workspace, void* stream) {
    int64_t bytes, gradient;
    const int rc = resolve(p, false, &bytes, &gradient);
    if (rc != SWR_OK) return rc;
    if (p->rows == 0) return SWR_OK;
    const int64_t work = swr::logprob_work_bytes(p->rows, p->vocab, p->top);
    if (!logits || !tokens || !logp || !lse || !entropy || (p->top > 0 && (!top_logp || !top_tokens)) ||
        (work > 0 && !workspace))
        return SWR_ERR_NULL;
    if (!aligned(logits, size_of(p->dtype)) || !aligned(tokens, p->token_bytes) || !all_aligned({logp, lse, entropy}, 4) ||
        (p->top > 0 && (!aligned(top_logp, 4) || !aligned(top_tokens, 8))) || !aligned(workspace, 16))
        return SWR_ERR_ALIGN;
    const int64_t top = p->rows * p->top;
    if (clashes({span(logp, p->rows * 4), span(lse, p->rows * 4), span(entropy, p->rows * 4),
                 span(top ? top_logp : nullptr, top * 4), span(top ? top_tokens : nullptr, top * 8), span(workspace, work)},
                {span(logits, bytes), span(tokens, p->rows * p->token_bytes)}))
        return SWR_ERR_ALIAS;
    swr::LogProbParams q = logprob_params(p, logits, tokens);
    q.logp = logp; q.lse = lse; q.entropy = entropy; q.top_logp = top_logp; q.top_tokens = top_tokens;
    q.work = workspace;
    q.parts = swr::logprob_parts(p->rows, p->vocab);
    return status(swr::launch_logprob(p->dtype, q, stream));
}

int swr_log_probs_backward(const swr_logprob_t* p, const void* logits, const void* tokens, const float* lse,
                           const float* entropy, const float* dlogp, const float* dlse, const float* dentropy,
                           void* dlogits, void* stream) {
    int64_t bytes, gradient;
    const int rc = resolve(p, true, &bytes, &gradient);
    if (rc != SWR_OK) return rc;
    if (p->rows == 0) return SWR_OK;
    if (!logits || !tokens || !lse || !entropy || !dlogits) return SWR_ERR_NULL;
    if (!all_aligned({logits, dlogits}, size_of(p->dtype)) || !aligned(tokens, p->token_bytes) ||
        !all_aligned({lse, entropy, dlogp, dlse, dentropy}, 4))
        return SWR_ERR_ALIGN;
    const Span out = span(dlogits, gradient);
    const bool same = dlogits == logits && (p->sd == p->sl || p->rows == 1);
    const int es = size_of(p->dtype);
    if ((!same && meet(1, p->rows, rows_of(dlogits, 0, p->sd, p->vocab, es, gradient),
                       rows_of(logits, 0, p->sl, p->vocab, es, bytes))) ||
        overlaps(out, {span(tokens, p->rows * p->token_bytes), span(lse, p->rows * 4), span(entropy, p->rows * 4),
                       span(dlogp, p->rows * 4), span(dlse, p->rows * 4), span(dentropy, p->rows * 4)}))
        return SWR_ERR_ALIAS;
    swr::LogProbParams q = logprob_params(p, logits, tokens);
    q.lse_in = lse; q.entropy_in = entropy; q.dlogp = dlogp; q.dlse = dlse; q.dentropy = dentropy; q.dlogits = dlogits;
    return status(swr::launch_logprob_backward(p->dtype, q, stream));
}

}  // extern "C"
