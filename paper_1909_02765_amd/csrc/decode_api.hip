// Entry points of the decoder-step operators: argument checks, workspace,
// device check and launch.  Declarations and contracts are in include/ilpm.h.
#include <algorithm>
#include <climits>
#include <cmath>
#include <exception>

#include "decode.h"

namespace ilpm {
namespace {

// A launch holds at most 2^32 - 1 threads along a dimension, here in
// workgroups of up to 256.
constexpr int64_t kMaxGroups = (1 << 24) - 1;
// Strides, in elements, are at most this (no device memory is larger).
constexpr int64_t kMaxStride = (int64_t)1 << 40;

bool type_ok(int dtype) { return dtype == ILPM_F32 || dtype == ILPM_F16 || dtype == ILPM_BF16; }

bool aligned(const void *p, int dtype) { return (uintptr_t)p % (unsigned)element_bytes(dtype) == 0; }

bool stride_ok(int64_t s) { return s >= 0 && s <= kMaxStride; }

// A strided set of runs: n0 x n1 x n2 runs of `run` bytes, s0 to s2 bytes apart.
struct Span {
    uintptr_t at;
    int64_t n[3], s[3], run;
    // (Sizes and strides within their limits do not overflow 128 bits.)
    __int128 bytes() const { return (__int128)(n[0] - 1) * s[0] + inner(); }
    __int128 inner() const { return (__int128)(n[1] - 1) * s[1] + (__int128)(n[2] - 1) * s[2] + run; }
};

// Whether two sets may touch each other.  Where both repeat with the same
// period (the rows of one packed tensor, or two pools in one allocation) and
// each fits in it, their places within the period decide; else all that lies
// between their first and last bytes counts as theirs.
bool touch(const Span &a, const Span &b)
{
    if ((__int128)a.at + a.bytes() <= b.at || (__int128)b.at + b.bytes() <= a.at) return false;
    const int64_t period = a.s[0];
    if (period > 0 && period == b.s[0]) {
        const __int128 ea = a.inner(), eb = b.inner();
        if (ea <= period && eb <= period) {
            const int64_t d = a.at <= b.at ? (int64_t)((b.at - a.at) % (uint64_t)period)
                                           : (period - (int64_t)((a.at - b.at) % (uint64_t)period)) % period;
            return d < ea || d + eb > period;
        }
    }
    return true;
}

// Whether a set that is written names no byte twice: from the smallest stride
// up, each passes over all that lies below it.
bool writes_once(const Span &a)
{
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int i, int j) { return a.s[i] < a.s[j]; });
    __int128 extent = a.run;
    for (int i : order) {
        if (a.n[i] <= 1) continue;
        if (a.s[i] < extent) return false;
        extent += (__int128)(a.n[i] - 1) * a.s[i];
    }
    return true;
}

Span span_of(const ilpm_heads &h, int64_t rows, int dim)
{
    const int64_t e = element_bytes(h.dtype);
    return {(uintptr_t)h.data, {rows, h.heads, 1}, {h.row_stride * e, h.head_stride * e, 0}, dim * e};
}

Span pool_span(const ilpm_kv_cache &c, bool v)
{
    const int64_t e = element_bytes(c.dtype);
    if (v) return {(uintptr_t)c.v, {c.n_pages, c.page_size, c.kv_heads}, {c.v_page_stride * e, c.v_slot_stride * e, c.v_head_stride * e}, c.head_dim * e};
    return {(uintptr_t)c.k, {c.n_pages, c.page_size, c.kv_heads}, {c.k_page_stride * e, c.k_slot_stride * e, c.k_head_stride * e}, c.head_dim * e};
}

Span flat_span(const void *p, int64_t bytes) { return {(uintptr_t)p, {1, 1, 1}, {0, 0, 0}, bytes}; }

Span rows_span(const void *p, int64_t rows, int64_t stride, int64_t run)
{
    return {(uintptr_t)p, {rows, 1, 1}, {stride, 0, 0}, run};
}

int check_heads(const ilpm_heads &h)
{
    if (!type_ok(h.dtype)) return ILPM_ERR_UNSUPPORTED;
    if (!h.data || h.heads <= 0 || !stride_ok(h.row_stride) || !stride_ok(h.head_stride) || !aligned(h.data, h.dtype))
        return ILPM_ERR_INVALID_ARG;
    return ILPM_OK;
}

// The sizes that planning goes by, and then the pools and the table.
int check_cache_sizes(const ilpm_kv_cache *c)
{
    if (!c || c->n_pages < 0 || c->page_size <= 0 || c->kv_heads <= 0 || c->head_dim <= 0 || c->n_seqs < 0 ||
        c->max_pages < 0)
        return ILPM_ERR_INVALID_ARG;
    return type_ok(c->dtype) ? ILPM_OK : ILPM_ERR_UNSUPPORTED;
}

int check_cache(const ilpm_kv_cache *c)
{
    const int rc = check_cache_sizes(c);
    if (rc != ILPM_OK) return rc;
    for (int64_t s : {c->k_page_stride, c->k_slot_stride, c->k_head_stride, c->v_page_stride, c->v_slot_stride,
                      c->v_head_stride, c->table_stride})
        if (!stride_ok(s)) return ILPM_ERR_INVALID_ARG;
    if (c->n_pages > 0 && (!c->k || !c->v)) return ILPM_ERR_INVALID_ARG;
    if (c->n_seqs > 0 && c->max_pages > 0 && !c->page_table) return ILPM_ERR_INVALID_ARG;
    if (!aligned(c->k, c->dtype) || !aligned(c->v, c->dtype) || (uintptr_t)c->page_table % 4) return ILPM_ERR_INVALID_ARG;
    return ILPM_OK;
}

Span table_span(const ilpm_kv_cache &c)
{
    return rows_span(c.page_table, std::max(c.n_seqs, 1), c.table_stride * 4, (int64_t)c.max_pages * 4);
}

// Keys that a row of the page table can name, as far as an int counts them.
int capacity_of(const ilpm_kv_cache &c)
{
    if (c.n_pages == 0) return 0;
    return (int)std::min<int64_t>((int64_t)c.max_pages * c.page_size, INT_MAX - 4096);
}

int attn_sizes(const ilpm_kv_cache *c, int q_heads, bool q32, int window, int max_len, AttnArgs *a, size_t *bytes)
{
    if (q_heads <= 0 || q_heads % c->kv_heads != 0 || window < 0 || max_len < 0) return ILPM_ERR_INVALID_ARG;
    if (c->head_dim > 256) return ILPM_ERR_UNSUPPORTED;
    if ((int64_t)c->n_seqs * q_heads > kMaxGroups) return ILPM_ERR_UNSUPPORTED;
    a->n_seqs = c->n_seqs;
    a->q_heads = q_heads;
    a->kv_heads = c->kv_heads;
    a->group = q_heads / c->kv_heads;
    a->dim = c->head_dim;
    a->window = window;
    a->capacity = capacity_of(*c);
    *bytes = attn_plan(a, c->dtype, q32, max_len > 0 ? std::min(max_len, a->capacity) : a->capacity);
    return ILPM_OK;
}

int kv_append(const ilpm_kv_cache *cache, const ilpm_heads *k, const ilpm_heads *v, const ilpm_heads *q,
              const ilpm_heads *q_out, const int32_t *seq_ids, const int32_t *positions, int n_tokens, const float *cos,
              const float *sin, int n_positions, int rot_dim, int pairs, hipStream_t stream)
{
    int rc = check_cache(cache);
    if (rc != ILPM_OK) return rc;
    const ilpm_kv_cache &c = *cache;
    if (!k || !v || n_tokens < 0 || n_positions < 0 || rot_dim < 0 || rot_dim % 2 || rot_dim > c.head_dim ||
        (pairs != 0 && pairs != 1) || !q != !q_out)
        return ILPM_ERR_INVALID_ARG;
    if (n_tokens == 0) return ILPM_OK;
    for (const ilpm_heads *h : {k, v, q, q_out})
        if (h && (rc = check_heads(*h)) != ILPM_OK) return rc;
    if (k->heads != c.kv_heads || v->heads != c.kv_heads || (q && q->heads != q_out->heads)) return ILPM_ERR_INVALID_ARG;
    if (k->dtype != v->dtype || (q && (q->dtype != k->dtype || q_out->dtype != k->dtype)) ||
        (k->dtype != c.dtype && k->dtype != ILPM_F32))
        return ILPM_ERR_UNSUPPORTED;
    if (!seq_ids || !positions || ((uintptr_t)seq_ids | (uintptr_t)positions) % 4) return ILPM_ERR_INVALID_ARG;
    if (rot_dim > 0 && n_positions > 0 && (!cos || !sin || ((uintptr_t)cos | (uintptr_t)sin) % 4)) return ILPM_ERR_INVALID_ARG;
    if (n_tokens > kMaxGroups || (int64_t)(q ? q->heads : 1) * c.head_dim > INT_MAX || (int64_t)c.kv_heads * c.head_dim > INT_MAX)
        return ILPM_ERR_UNSUPPORTED;

    // What is written: the pools and q_out.
    const int64_t angles = rot_dim > 0 ? (int64_t)n_positions * (rot_dim / 2) * 4 : 0;
    const Span read[] = {span_of(*k, n_tokens, c.head_dim), span_of(*v, n_tokens, c.head_dim),
                         flat_span(seq_ids, (int64_t)n_tokens * 4), flat_span(positions, (int64_t)n_tokens * 4),
                         flat_span(cos, angles), flat_span(sin, angles), table_span(c)};
    if (c.n_pages > 0) {
        const Span pk = pool_span(c, false), pv = pool_span(c, true);
        if (!writes_once(pk) || !writes_once(pv) || touch(pk, pv)) return ILPM_ERR_INVALID_ARG;
        for (const Span &s : read)
            if (s.at && s.bytes() > 0 && (touch(s, pk) || touch(s, pv))) return ILPM_ERR_INVALID_ARG;
        if (q) {
            const Span sq = span_of(*q, n_tokens, c.head_dim), so = span_of(*q_out, n_tokens, c.head_dim);
            if (touch(sq, pk) || touch(sq, pv) || touch(so, pk) || touch(so, pv)) return ILPM_ERR_INVALID_ARG;
        }
    }
    if (q) {
        const Span sq = span_of(*q, n_tokens, c.head_dim), so = span_of(*q_out, n_tokens, c.head_dim);
        const bool in_place = q->data == q_out->data && q->row_stride == q_out->row_stride && q->head_stride == q_out->head_stride;
        if (!writes_once(so) || (!in_place && touch(sq, so))) return ILPM_ERR_INVALID_ARG;
        for (const Span &s : read)
            if (s.at && s.bytes() > 0 && touch(s, so)) return ILPM_ERR_INVALID_ARG;
    }

    int dev = 0;
    if ((rc = api_device_check(&dev)) != ILPM_OK) return rc;
    AppendArgs a = {};
    a.k = k->data;
    a.k_row = k->row_stride;
    a.k_head = k->head_stride;
    a.v = v->data;
    a.v_row = v->row_stride;
    a.v_head = v->head_stride;
    if (q) {
        a.q = q->data;
        a.q_row = q->row_stride;
        a.q_head = q->head_stride;
        a.q_out = q_out->data;
        a.qo_row = q_out->row_stride;
        a.qo_head = q_out->head_stride;
        a.q_heads = q->heads;
    }
    a.n_tokens = n_tokens;
    a.kv_heads = c.kv_heads;
    a.dim = c.head_dim;
    a.kc = c.k;
    a.vc = c.v;
    a.kc_page = c.k_page_stride;
    a.kc_slot = c.k_slot_stride;
    a.kc_head = c.k_head_stride;
    a.vc_page = c.v_page_stride;
    a.vc_slot = c.v_slot_stride;
    a.vc_head = c.v_head_stride;
    a.table = c.page_table;
    a.table_stride = c.table_stride;
    a.n_seqs = c.n_seqs;
    a.max_pages = c.max_pages;
    a.n_pages = c.n_pages;
    a.page_size = c.page_size;
    a.seq_ids = seq_ids;
    a.positions = positions;
    a.cos = cos;
    a.sin = sin;
    a.n_positions = n_positions;
    a.rot_dim = rot_dim;
    a.pairs = pairs;
    (void)hipGetLastError();
    const hipError_t e = append_launch(a, k->dtype, c.dtype, stream);
    return e == hipSuccess ? ILPM_OK : api_hip_fail(e);
}

int attn_decode(const ilpm_kv_cache *cache, const ilpm_heads *q, const int32_t *lengths, const ilpm_attn_options *opt,
                const ilpm_heads *out, float *lse, void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    int rc = check_cache(cache);
    if (rc != ILPM_OK) return rc;
    const ilpm_kv_cache &c = *cache;
    if (!q || !out || !opt || q->heads <= 0 || out->heads != q->heads) return ILPM_ERR_INVALID_ARG;
    AttnArgs a = {};
    size_t need = 0;
    if ((rc = attn_sizes(cache, q->heads, q->dtype == ILPM_F32, opt->window, opt->max_len, &a, &need)) != ILPM_OK) return rc;
    // (Scores are formed times log2 e, or over softcap.)
    if (!std::isfinite(opt->scale * 1.5f) || !(opt->softcap >= 0.f) || !std::isfinite(opt->softcap * 1.5f) ||
        (opt->softcap > 0.f && !std::isfinite(opt->scale / opt->softcap)))
        return ILPM_ERR_INVALID_ARG;
    if (opt->mask && (opt->mask_len < 0 || !stride_ok(opt->mask_stride))) return ILPM_ERR_INVALID_ARG;
    if (c.n_seqs == 0) return ILPM_OK;
    if ((rc = check_heads(*q)) != ILPM_OK || (rc = check_heads(*out)) != ILPM_OK) return rc;
    if (q->dtype != out->dtype || (q->dtype != c.dtype && q->dtype != ILPM_F32)) return ILPM_ERR_UNSUPPORTED;
    if (!lengths || ((uintptr_t)lengths | (uintptr_t)lse) % 4 || (uintptr_t)workspace % 256) return ILPM_ERR_INVALID_ARG;

    // What is written: out, lse and the workspace.
    const Span sq = span_of(*q, c.n_seqs, c.head_dim), so = span_of(*out, c.n_seqs, c.head_dim);
    const bool in_place = q->data == out->data && q->row_stride == out->row_stride && q->head_stride == out->head_stride;
    if (!writes_once(so) || (!in_place && touch(sq, so))) return ILPM_ERR_INVALID_ARG;
    const Span sl = flat_span(lse, (int64_t)c.n_seqs * q->heads * 4);
    const Span sw = flat_span(workspace, (int64_t)std::min<size_t>(need, (size_t)1 << 60));
    const bool has_ws = workspace && need > 0;
    if (lse && (touch(sl, so) || touch(sl, sq))) return ILPM_ERR_INVALID_ARG;
    if (has_ws && (touch(sw, so) || touch(sw, sq) || (lse && touch(sw, sl)))) return ILPM_ERR_INVALID_ARG;
    Span read[5];
    int n = 0;
    read[n++] = flat_span(lengths, (int64_t)c.n_seqs * 4);
    if (a.capacity > 0) {
        read[n++] = pool_span(c, false);
        read[n++] = pool_span(c, true);
        read[n++] = table_span(c);
    }
    if (opt->mask && opt->mask_len > 0) read[n++] = rows_span(opt->mask, c.n_seqs, opt->mask_stride, opt->mask_len);
    for (int i = 0; i < n; ++i)
        if (touch(read[i], so) || (lse && touch(read[i], sl)) || (has_ws && touch(read[i], sw))) return ILPM_ERR_INVALID_ARG;

    int dev = 0;
    if ((rc = api_device_check(&dev)) != ILPM_OK) return rc;
    void *ws = workspace;
    if (need > 0) {
        if (!ws) rc = api_workspace(dev, need, stream, &ws);
        else if (workspace_bytes < need) rc = ILPM_ERR_WORKSPACE;
        if (rc != ILPM_OK) return rc;
    }
    a.q = q->data;
    a.q_row = q->row_stride;
    a.q_head = q->head_stride;
    a.out = out->data;
    a.o_row = out->row_stride;
    a.o_head = out->head_stride;
    a.lse = lse;
    a.q_dtype = q->dtype;
    a.k = c.k;
    a.v = c.v;
    a.k_page = c.k_page_stride;
    a.k_slot = c.k_slot_stride;
    a.k_head = c.k_head_stride;
    a.v_page = c.v_page_stride;
    a.v_slot = c.v_slot_stride;
    a.v_head = c.v_head_stride;
    a.table = c.page_table;
    a.table_stride = c.table_stride;
    a.n_pages = c.n_pages;
    a.page_size = c.page_size;
    a.lengths = lengths;
    a.mask = opt->mask;
    a.mask_stride = opt->mask_stride;
    a.mask_len = opt->mask_len;
    a.scale = opt->scale;
    a.softcap = opt->softcap;
    if (a.split) attn_workspace(&a, ws);
    (void)hipGetLastError();
    const hipError_t e = attn_launch(a, c.dtype, stream);
    return e == hipSuccess ? ILPM_OK : api_hip_fail(e);
}

int residual_norm(const ilpm_residual_norm_args *args, hipStream_t stream)
{
    if (!args) return ILPM_ERR_INVALID_ARG;
    const ilpm_residual_norm_args &g = *args;
    for (int kind : {g.post, g.pre})
        if (kind != ILPM_NORM_NONE && kind != ILPM_NORM_RMS && kind != ILPM_NORM_LAYER) return ILPM_ERR_INVALID_ARG;
    if (g.rows < 0 || g.width <= 0 || !(g.eps >= 0.f) || !std::isfinite(g.eps) || !std::isfinite(g.scale))
        return ILPM_ERR_INVALID_ARG;
    for (int64_t s : {g.x_stride, g.y_stride, g.r_stride, g.z_stride, g.gate_stride})
        if (!stride_ok(s)) return ILPM_ERR_INVALID_ARG;
    if (!type_ok(g.x_dtype) || !type_ok(g.y_dtype) || !type_ok(g.param_dtype)) return ILPM_ERR_UNSUPPORTED;
    if ((g.x_dtype != g.y_dtype && g.x_dtype != ILPM_F32) || (g.param_dtype != g.y_dtype && g.param_dtype != ILPM_F32))
        return ILPM_ERR_UNSUPPORTED;
    if (g.rows == 0) return ILPM_OK;
    if (g.rows > kMaxGroups) return ILPM_ERR_UNSUPPORTED;
    if (!g.x || (!g.r && !g.z) || !g.z != (g.pre == ILPM_NORM_NONE)) return ILPM_ERR_INVALID_ARG;
    if (!g.y && (g.gate || g.post != ILPM_NORM_NONE)) return ILPM_ERR_INVALID_ARG;
    if ((g.post == ILPM_NORM_NONE && (g.post_w || g.post_b)) || (g.pre == ILPM_NORM_NONE && (g.pre_w || g.pre_b)))
        return ILPM_ERR_INVALID_ARG;
    if (!aligned(g.x, g.x_dtype) || !aligned(g.r, g.x_dtype) || !aligned(g.y, g.y_dtype) || !aligned(g.z, g.y_dtype))
        return ILPM_ERR_INVALID_ARG;
    const void *params[] = {g.post_w, g.post_b, g.pre_w, g.pre_b, g.gate};
    for (const void *p : params)
        if (!aligned(p, g.param_dtype)) return ILPM_ERR_INVALID_ARG;

    const int64_t ex = element_bytes(g.x_dtype), ey = element_bytes(g.y_dtype), ep = element_bytes(g.param_dtype);
    const Span x = rows_span(g.x, g.rows, g.x_stride * ex, g.width * ex);
    const Span y = rows_span(g.y, g.rows, g.y_stride * ey, g.width * ey);
    const Span r = rows_span(g.r, g.rows, g.r_stride * ex, g.width * ex);
    const Span z = rows_span(g.z, g.rows, g.z_stride * ey, g.width * ey);
    const bool r_is_x = g.r == g.x && g.r_stride == g.x_stride, z_is_y = g.z == g.y && g.z_stride == g.y_stride;
    if (g.r && (!writes_once(r) || (!r_is_x && touch(r, x)) || (g.y && touch(r, y)))) return ILPM_ERR_INVALID_ARG;
    if (g.z && (!writes_once(z) || touch(z, x) || (g.y && !z_is_y && touch(z, y)))) return ILPM_ERR_INVALID_ARG;
    if (g.r && g.z && touch(r, z)) return ILPM_ERR_INVALID_ARG;
    for (const void *p : params) {
        if (!p) continue;
        const Span s = p == g.gate && g.gate_stride > 0 ? rows_span(p, g.rows, g.gate_stride * ep, g.width * ep)
                                                        : flat_span(p, g.width * ep);
        if ((g.r && touch(s, r)) || (g.z && touch(s, z))) return ILPM_ERR_INVALID_ARG;
    }

    int dev = 0;
    const int rc = api_device_check(&dev);
    if (rc != ILPM_OK) return rc;
    NormArgs a = {};
    a.x = g.x;
    a.y = g.y;
    a.r = g.r;
    a.z = g.z;
    a.x_row = g.x_stride;
    a.y_row = g.y_stride;
    a.r_row = g.r_stride;
    a.z_row = g.z_stride;
    a.post_w = g.post_w;
    a.post_b = g.post_b;
    a.pre_w = g.pre_w;
    a.pre_b = g.pre_b;
    a.gate = g.gate;
    a.gate_row = g.gate_stride;
    a.rows = g.rows;
    a.width = g.width;
    a.post = g.post;
    a.pre = g.pre;
    a.scale = g.scale;
    a.eps = g.eps;
    (void)hipGetLastError();
    const hipError_t e = norm_launch(a, g.x_dtype, g.y_dtype, g.param_dtype, stream);
    return e == hipSuccess ? ILPM_OK : api_hip_fail(e);
}

// No exception passes the C boundary (a mutex or an allocation of the
// workspace's bookkeeping may throw).
template <typename F> int guarded(F &&f)
{
    try {
        return f();
    } catch (const std::exception &) {
        return api_hip_fail(hipErrorUnknown);
    }
}

}  // namespace
}  // namespace ilpm

using namespace ilpm;

extern "C" {

int ilpm_kv_append(const ilpm_kv_cache *cache, const ilpm_heads *k, const ilpm_heads *v, const ilpm_heads *q,
                   const ilpm_heads *q_out, const int32_t *seq_ids, const int32_t *positions, int n_tokens,
                   const float *cos, const float *sin, int n_positions, int rot_dim, int pairs, hipStream_t stream)
{
    return guarded([&] {
        return kv_append(cache, k, v, q, q_out, seq_ids, positions, n_tokens, cos, sin, n_positions, rot_dim, pairs, stream);
    });
}

int ilpm_attn_decode(const ilpm_kv_cache *cache, const ilpm_heads *q, const int32_t *lengths,
                     const ilpm_attn_options *options, const ilpm_heads *out, float *lse, void *workspace,
                     size_t workspace_bytes, hipStream_t stream)
{
    return guarded([&] { return attn_decode(cache, q, lengths, options, out, lse, workspace, workspace_bytes, stream); });
}

int ilpm_attn_decode_workspace_size(const ilpm_kv_cache *cache, int q_heads, int window, int max_len, size_t *bytes)
{
    if (!bytes) return ILPM_ERR_INVALID_ARG;
    int rc = check_cache_sizes(cache);
    if (rc != ILPM_OK) return rc;
    AttnArgs a = {};
    // Of either type of queries, the larger.
    size_t other = 0;
    if ((rc = attn_sizes(cache, q_heads, true, window, max_len, &a, &other)) != ILPM_OK) return rc;
    rc = attn_sizes(cache, q_heads, false, window, max_len, &a, bytes);
    *bytes = std::max(*bytes, other);
    return rc;
}

int ilpm_residual_norm(const ilpm_residual_norm_args *args, hipStream_t stream)
{
    return guarded([&] { return residual_norm(args, stream); });
}

}  // extern "C"
