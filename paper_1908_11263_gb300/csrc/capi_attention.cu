// C ABI of the attention operators (declared in include/qnn.h): argument validation and dispatch.  Every check happens
// before anything is enqueued; a call that returns an error has launched nothing.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "attention.h"

namespace qnn {
namespace {

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
qnn_status from_cuda(cudaError_t e) { return e == cudaSuccess ? QNN_OK : QNN_ECUDA; }
bool flag_ok(int32_t v) { return v == 0 || v == 1; }

// Whether the elements of an array of these sizes and strides lie apart (rows of `inner` contiguous elements): with the
// dimensions in rising order of their strides, each has to step over all that the ones before it reach.
struct Dim {
    int64_t size, stride;
};
bool apart(std::initializer_list<Dim> dims, int64_t inner)
{
    Dim d[4];
    int n = 0;
    for (const Dim &x : dims) {
        if (x.size <= 0) return true;
        if (x.size > 1) d[n++] = x;
    }
    std::sort(d, d + n, [](const Dim &x, const Dim &y) { return x.stride < y.stride; });
    int64_t reach = inner;  // elements up to here are in use
    for (int i = 0; i < n; ++i) {
        if (d[i].stride < reach || d[i].stride > INT64_MAX / 4 / d[i].size) return false;
        reach += (d[i].size - 1) * d[i].stride;
    }
    return true;
}

constexpr int64_t kMaxRows = 0x7fffffff;  // tokens times heads
constexpr int64_t kMaxKeys = 1 << 30;     // of a sequence
constexpr int64_t kMaxStride = INT64_C(1) << 40;

bool stride_ok(int64_t s) { return s >= 0 && s <= kMaxStride; }

qnn_status check_cache(const qnn_cache_desc *c)
{
    if (!c || c->struct_size != sizeof(qnn_cache_desc)) return QNN_EINVAL;
    if (c->dtype != QNN_F16 && c->dtype != QNN_BF16 && c->dtype != QNN_F32) return QNN_EINVAL;
    if (c->kv_heads <= 0 || c->head_dim <= 0 || c->page_size <= 0 || c->pages < 0) return QNN_EINVAL;
    for (const int64_t s : {c->k_page, c->k_head, c->k_row, c->v_page, c->v_head, c->v_row})
        if (!stride_ok(s)) return QNN_EINVAL;
    if (c->dtype == QNN_F32 || c->head_dim % 8 || c->head_dim > 256) return QNN_EUNSUPPORTED;
    if (c->kv_heads > 1024 || c->page_size > kMaxKeys || c->pages > kMaxRows) return QNN_EUNSUPPORTED;
    for (const int64_t s : {c->k_page, c->k_head, c->k_row, c->v_page, c->v_head, c->v_row})
        if (s % 8) return QNN_EALIGN;
    return QNN_OK;
}

qnn_status check_batch(const qnn_batch_desc *b, int64_t page_size)
{
    if (!b || b->struct_size != sizeof(qnn_batch_desc)) return QNN_EINVAL;
    if (b->seqs < 0 || b->width < 0 || b->t < 0 || !flag_ok(b->ragged) || !stride_ok(b->ldt)) return QNN_EINVAL;
    if (!b->ragged && (b->seqs ? b->t % b->seqs : b->t)) return QNN_EINVAL;
    if (b->t > kMaxRows || b->width * page_size > kMaxKeys) return QNN_EUNSUPPORTED;
    return QNN_OK;
}

qnn_status check_rope(int32_t dim, int32_t d, int32_t interleaved, int32_t wide, float amplitude)
{
    if (dim < 0 || dim % 2 || dim > d || !flag_ok(interleaved) || !flag_ok(wide) || !std::isfinite(amplitude)) return QNN_EINVAL;
    return QNN_OK;
}

qnn_status check_attention(const qnn_cache_desc *c, const qnn_batch_desc *b, const qnn_attention_desc *a)
{
    qnn_status st = check_cache(c);
    if (st != QNN_OK && st != QNN_EALIGN) return st;
    const qnn_status sb = check_batch(b, c->page_size);
    if (sb == QNN_EINVAL) return sb;
    if (!a || a->struct_size != sizeof(qnn_attention_desc)) return QNN_EINVAL;
    if (a->heads <= 0 || a->heads % c->kv_heads || !flag_ok(a->causal) || a->window < 0) return QNN_EINVAL;
    // times log2(e) it has to be a normal number
    if (!(a->scale >= FLT_MIN) || !(a->scale <= FLT_MAX / 2)) return QNN_EINVAL;
    for (const int64_t s : {a->q_seq, a->ldq, a->hq, a->o_seq, a->ldo, a->ho})
        if (!stride_ok(s)) return QNN_EINVAL;
    if (sb != QNN_OK) return sb;
    if (b->t * a->heads > kMaxRows) return QNN_EUNSUPPORTED;
    const int64_t each = b->ragged || b->seqs == 0 ? b->t : b->t / b->seqs;
    if (!apart({{b->ragged ? 1 : b->seqs, a->o_seq}, {each, a->ldo}, {a->heads, a->ho}}, c->head_dim)) return QNN_EINVAL;
    return st;
}

// Rows (queries times the heads that share a key head) of a sequence up to which the streaming kernel takes it, and which
// kernels a call may need.  Without offsets all sequences have as many rows, and small calls, which latency bounds, stay with
// the streaming kernel: those of at most kFewUnits pieces of 16 rows and 64 keys an SM.  Measured on both sides (us, streaming /
// tensor cores, 8 key heads of 128): 64 sequences of 2048 keys with 16 rows 124 / 128, with 24 rows 199 / 130; 64 of 256 keys
// with 24 or 32 rows (two tiles of 16, 27 pieces an SM) 50 / 46-49; 8 of 1024 with 32 rows (13 pieces) 31 / 33, with 64 rows
// (27) 46 / 33; one of 8192 with 32 rows (13) 29 / 38, with 64 rows (27) 38 / 38.  The thresholds are those of heads of 128;
// heads of 64: 64 of 2048 with 16 rows 85 / 100, with 24 rows 132 / 106; 64 of 256 with 24 rows (27) 38 / 44, the slower side;
// 8 of 1024 with 64 rows 39 / 26.  Pieces are counted over the table's width, which the host knows; lengths and windows that
// leave most of it out make a call look larger (a window of 256 and 32 rows in a table of 128 K tokens 20 / 23).
// With offsets the host knows the call's rows only.  The tensor cores' kernel takes all sequences where those are more than
// kFewRows for each on average (a single token among chunks costs it a few units; a second pair of launches took 24 us of 150
// for 12 sequences with up to 600 new tokens over 8000), else the kernels share the sequences, and both are queued where one
// could have more than kFewRows: 64 single tokens, group 4, over 256 or 4096 keys take 45 or 200 us with offsets, 31 or 187
// without.  Rows in no sequence count as rows: the same tokens over 8192 keys in a call of 1024 rows take 391 us (tensor
// cores) against 358 in one of 64 (heads of 128), 289 against 237 (heads of 64).
constexpr int kFewRows = 16, kFewUnits = 24;
struct Kernels {
    bool rows, tc;
    int few;
    size_t rows_bytes, tc_bytes;  // workspaces
};
Kernels kernels_of(const qnn_cache_desc &c, const qnn_batch_desc &b, const qnn_attention_desc &d)
{
    Kernels k = {true, false, 0x7fffffff, 0, 0};
    if (b.t == 0 || b.seqs == 0) return k;
    const int64_t most = (b.ragged ? b.t : b.t / b.seqs) * (d.heads / c.kv_heads);
    if (c.head_dim <= 128) {
        const bool many = b.t * (d.heads / c.kv_heads) > static_cast<int64_t>(kFewRows) * b.seqs;  // on average
        k.few = b.ragged && many ? 0 : kFewRows;
        k.tc = most > kFewRows;
        if (!b.ragged) {
            const int64_t room = static_cast<int64_t>(b.width) * c.page_size;
            const double units = static_cast<double>(b.seqs) * c.kv_heads * ((most + 15) / 16) * ((room + 63) / 64);
            if (units <= static_cast<double>(kFewUnits) * device_sm_count()) k.tc = false;
        }
        if (!k.tc) k.few = 0x7fffffff;
        k.rows = !k.tc || (b.ragged && !many);
    }
    const int64_t room = static_cast<int64_t>(b.width) * c.page_size;
    if (k.rows && room > 64) k.rows_bytes = (attention_rows_workspace(c.head_dim) + 255) / 256 * 256;
    if (k.tc && room > 128) k.tc_bytes = attention_tc_workspace(c.head_dim);
    return k;
}

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" {

qnn_status qnn_rope_turns(const qnn_rope_scaling *s, uint64_t *turns)
{
    if (!s || s->struct_size != sizeof(qnn_rope_scaling) || !turns) return QNN_EINVAL;
    if (s->dim <= 0 || s->dim % 2) return QNN_EINVAL;
    if (s->scaling < QNN_ROPE_NONE || s->scaling > QNN_ROPE_RAMP) return QNN_EINVAL;
    if (!(s->base > 1.0) || std::isinf(s->base)) return QNN_EINVAL;
    if (s->scaling != QNN_ROPE_NONE && (!(s->factor >= 1.0) || std::isinf(s->factor))) return QNN_EINVAL;
    if (s->scaling == QNN_ROPE_RAMP && (s->context <= 0 || !(s->low < s->high) || std::isinf(s->low) || std::isinf(s->high)))
        return QNN_EINVAL;
    if (s->scaling == QNN_ROPE_BASE && s->dim == 2) return QNN_EINVAL;
    const double two_pi = 6.283185307179586476925;
    const double base = s->scaling == QNN_ROPE_BASE ? s->base * std::pow(s->factor, s->dim / (s->dim - 2.0)) : s->base;
    for (int i = 0; i < s->dim / 2; ++i) {
        double f = std::pow(base, -2.0 * i / s->dim);
        if (s->scaling == QNN_ROPE_LINEAR) f /= s->factor;
        if (s->scaling == QNN_ROPE_RAMP) {
            const double rotations = s->context * f / two_pi;
            const double keep = std::min(1.0, std::max(0.0, (rotations - s->low) / (s->high - s->low)));
            f *= keep + (1.0 - keep) / s->factor;
        }
        turns[i] = static_cast<uint64_t>(std::ldexp(f / two_pi, 64));  // below 2^62: f is at most 1
    }
    return QNN_OK;
}

qnn_status qnn_rope(const qnn_rope_desc *d, const uint64_t *turns, const void *positions, const void *x, void *y, void *stream)
{
    if (!d || d->struct_size != sizeof(qnn_rope_desc)) return QNN_EINVAL;
    if (d->dtype != QNN_F16 && d->dtype != QNN_BF16 && d->dtype != QNN_F32) return QNN_EINVAL;
    if (d->t < 0 || d->heads <= 0 || d->head_dim <= 0) return QNN_EINVAL;
    const qnn_status st = check_rope(d->dim, d->head_dim, d->interleaved, d->wide, d->amplitude);
    if (st != QNN_OK) return st;
    for (const int64_t s : {d->ldx, d->hx, d->ldy, d->hy})
        if (!stride_ok(s)) return QNN_EINVAL;
    if (!apart({{d->t, d->ldy}, {d->heads, d->hy}}, d->head_dim)) return QNN_EINVAL;
    if (d->t > 0 && (!x || !y || !positions || (d->dim && !turns))) return QNN_EINVAL;
    if (d->head_dim > 1024 || d->heads > kMaxRows || d->t * d->heads > kMaxRows) return QNN_EUNSUPPORTED;
    const uintptr_t size = d->dtype == QNN_F32 ? 4 : 2;
    if (!aligned(x, size) || !aligned(y, size) || !aligned(turns, 8) || !aligned(positions, d->wide ? 8 : 4)) return QNN_EALIGN;
    RotateArgs a = {};
    a.t = d->t; a.d = d->head_dim; a.half = d->dim / 2; a.interleaved = d->interleaved; a.wide = d->wide;
    a.amplitude = d->amplitude; a.turns = turns; a.positions = positions;
    a.heads = d->heads; a.x = x; a.y = y; a.ldx = d->ldx; a.hx = d->hx; a.ldy = d->ldy; a.hy = d->hy;
    a.seqs = -1;
    return from_cuda(launch_rotate(a, d->dtype, static_cast<cudaStream_t>(stream)));
}

qnn_status qnn_cache_append(const qnn_cache_desc *c, const qnn_batch_desc *b, const qnn_append_desc *d, const int32_t *table,
                            const int32_t *lengths, const int32_t *offsets, const uint64_t *turns, const void *positions,
                            const void *k, const void *v, const void *q, void *k_pages, void *v_pages, void *q_out,
                            void *stream)
{
    const qnn_status sc = check_cache(c);
    if (sc != QNN_OK && sc != QNN_EALIGN) return sc;
    const qnn_status sb = check_batch(b, c->page_size);
    if (sb == QNN_EINVAL) return sb;
    if (!d || d->struct_size != sizeof(qnn_append_desc) || d->heads < 0) return QNN_EINVAL;
    const qnn_status st = check_rope(d->dim, c->head_dim, d->interleaved, d->wide, d->amplitude);
    if (st != QNN_OK) return st;
    for (const int64_t s : {d->ldk, d->hk, d->ldv, d->hv, d->ldq, d->hq, d->ldo, d->ho})
        if (!stride_ok(s)) return QNN_EINVAL;
    const int64_t hd = c->head_dim;
    if (!apart({{c->pages, c->k_page}, {c->kv_heads, c->k_head}, {c->page_size, c->k_row}}, hd) ||
        !apart({{c->pages, c->v_page}, {c->kv_heads, c->v_head}, {c->page_size, c->v_row}}, hd) ||
        (d->heads && !apart({{b->t, d->ldo}, {d->heads, d->ho}}, hd)))
        return QNN_EINVAL;
    if (b->t > 0) {
        if (!k || !v || !lengths || (b->width > 0 && !table) || (b->ragged != 0) != (offsets != nullptr)) return QNN_EINVAL;
        if ((c->pages > 0 && (!k_pages || !v_pages)) || (d->heads > 0 && (!q || !q_out)) || (d->dim && !turns)) return QNN_EINVAL;
    }
    if (sb != QNN_OK) return sb;
    if (d->heads > kMaxRows || b->t * (static_cast<int64_t>(d->heads) + c->kv_heads) > kMaxRows) return QNN_EUNSUPPORTED;
    if (sc != QNN_OK || !aligned(k_pages, 16) || !aligned(v_pages, 16)) return QNN_EALIGN;
    for (const void *p : {k, v, q, static_cast<const void *>(q_out)})
        if (!aligned(p, 2)) return QNN_EALIGN;
    for (const void *p : {table, lengths, offsets})
        if (!aligned(p, 4)) return QNN_EALIGN;
    if (!aligned(turns, 8) || !aligned(positions, d->wide ? 8 : 4)) return QNN_EALIGN;
    RotateArgs a = {};
    a.t = b->t; a.d = c->head_dim; a.half = d->dim / 2; a.interleaved = d->interleaved; a.wide = d->wide;
    a.amplitude = d->amplitude; a.turns = turns; a.positions = positions;
    a.heads = d->heads; a.x = q; a.y = q_out; a.ldx = d->ldq; a.hx = d->hq; a.ldy = d->ldo; a.hy = d->ho;
    a.kv_heads = c->kv_heads; a.k = k; a.v = v; a.k_pages = k_pages; a.v_pages = v_pages;
    a.ldk = d->ldk; a.hk = d->hk; a.ldv = d->ldv; a.hv = d->hv;
    a.k_page = c->k_page; a.k_head = c->k_head; a.k_row = c->k_row;
    a.v_page = c->v_page; a.v_head = c->v_head; a.v_row = c->v_row;
    a.pages = c->pages; a.ldt = b->ldt; a.seqs = b->seqs; a.width = b->width; a.page_size = c->page_size;
    a.each = b->ragged || b->seqs == 0 ? 0 : b->t / b->seqs;
    a.table = table; a.lengths = lengths; a.offsets = b->ragged ? offsets : nullptr;
    return from_cuda(launch_rotate(a, c->dtype, static_cast<cudaStream_t>(stream)));
}

qnn_status qnn_attention_workspace_size(const qnn_cache_desc *c, const qnn_batch_desc *b, const qnn_attention_desc *d,
                                        size_t *bytes)
{
    if (!bytes) return QNN_EINVAL;
    const qnn_status st = check_attention(c, b, d);
    if (st != QNN_OK) return st;
    const Kernels k = kernels_of(*c, *b, *d);
    *bytes = k.rows_bytes + k.tc_bytes;
    return QNN_OK;
}

qnn_status qnn_attention(const qnn_cache_desc *c, const qnn_batch_desc *b, const qnn_attention_desc *d, const int32_t *table,
                         const int32_t *lengths, const int32_t *offsets, const void *q, const void *k_pages,
                         const void *v_pages, void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    const qnn_status st = check_attention(c, b, d);
    if (st != QNN_OK && st != QNN_EALIGN) return st;
    if (!table && b->width > 1) return QNN_EINVAL;
    if (b->t > 0) {
        if (!q || !out || (b->ragged != 0) != (offsets != nullptr)) return QNN_EINVAL;
        if (c->pages > 0 && b->width > 0 && (!k_pages || !v_pages)) return QNN_EINVAL;
    }
    if (st != QNN_OK || !aligned(k_pages, 16) || !aligned(v_pages, 16)) return QNN_EALIGN;
    if (!aligned(q, 2) || !aligned(out, 2) || !aligned(lse, 4)) return QNN_EALIGN;
    for (const void *p : {table, lengths, offsets})
        if (!aligned(p, 4)) return QNN_EALIGN;
    const Kernels use = kernels_of(*c, *b, *d);
    const size_t need = use.rows_bytes + use.tc_bytes;
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return QNN_EWORKSPACE;
    AttnArgs a = {};
    a.q = q; a.k = k_pages; a.v = v_pages; a.out = out; a.lse = lse;
    a.table = table; a.lengths = lengths; a.offsets = b->ragged ? offsets : nullptr;
    a.q_seq = d->q_seq; a.ldq = d->ldq; a.hq = d->hq; a.o_seq = d->o_seq; a.ldo = d->ldo; a.ho = d->ho;
    a.k_page = c->k_page; a.k_head = c->k_head; a.k_row = c->k_row;
    a.v_page = c->v_page; a.v_head = c->v_head; a.v_row = c->v_row;
    a.pages = c->pages; a.ldt = b->ldt; a.t = b->t;
    a.seqs = b->seqs; a.width = b->width; a.page_size = c->page_size;
    a.each = b->ragged || b->seqs == 0 ? 0 : static_cast<int>(b->t / b->seqs);
    a.heads = d->heads; a.kv_heads = c->kv_heads; a.group = d->heads / c->kv_heads; a.d = c->head_dim;
    a.causal = d->causal; a.window = d->window;
    a.q_vec = aligned(q, 16) && d->q_seq % 8 == 0 && d->ldq % 8 == 0 && d->hq % 8 == 0;
    a.out_vec = aligned(out, 4) && d->o_seq % 2 == 0 && d->ldo % 2 == 0 && d->ho % 2 == 0;
    a.out_vec8 = aligned(out, 16) && d->o_seq % 8 == 0 && d->ldo % 8 == 0 && d->ho % 8 == 0;
    a.few = use.few;
    a.scale = d->scale * 1.4426950408889634f;
    if (use.rows_bytes) a.part = static_cast<float *>(workspace);
    if (use.tc_bytes) a.tc_part = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + use.rows_bytes);
    const cudaStream_t st_ = static_cast<cudaStream_t>(stream);
    cudaError_t e = use.tc ? launch_attention_tc(a, c->dtype, st_) : cudaSuccess;
    if (e == cudaSuccess && use.rows) e = launch_attention_rows(a, c->dtype, st_);
    return from_cuda(e);
}

}  // extern "C"
