// Entry points of the operators of a drafted decoder step: argument checks,
// workspace, device check and launch.  Declarations and contracts are in
// include/ilpm.h.
#include <cmath>

#include "decode_checks.h"
#include "draft.h"

namespace ilpm {
namespace {

constexpr int kMostVocab = 1 << 30;
// Sequences are a dimension of a grid that holds at most this.
constexpr int kMostRows = 65535;

bool same_place(const ilpm_heads &a, const ilpm_heads &b)
{
    return a.data == b.data && a.row_stride == b.row_stride && a.head_stride == b.head_stride;
}

int kv_append_norm(const ilpm_kv_cache *cache, const ilpm_heads *k, const ilpm_heads *v, const ilpm_heads *q,
                   const ilpm_heads *q_out, const ilpm_append_options *opt, int n_tokens, hipStream_t stream)
{
    int rc = check_cache(cache);
    if (rc != ILPM_OK) return rc;
    const ilpm_kv_cache &c = *cache;
    if (!k || !v || !opt || n_tokens < 0 || !q != !q_out) return ILPM_ERR_INVALID_ARG;
    const ilpm_append_options &o = *opt;
    if (o.n_positions < 0 || o.rot_dim < 0 || o.rot_dim % 2 || o.rot_dim > c.head_dim || (o.pairs != 0 && o.pairs != 1))
        return ILPM_ERR_INVALID_ARG;
    if (o.norm != ILPM_NORM_NONE && o.norm != ILPM_NORM_RMS && o.norm != ILPM_NORM_LAYER) return ILPM_ERR_INVALID_ARG;
    if (!(o.eps >= 0.f) || !std::isfinite(o.eps)) return ILPM_ERR_INVALID_ARG;
    if ((o.norm == ILPM_NORM_NONE && (o.q_w || o.k_w)) || (!q && o.q_w)) return ILPM_ERR_INVALID_ARG;
    if (c.head_dim > 1024) return ILPM_ERR_UNSUPPORTED;
    if (n_tokens == 0) return ILPM_OK;
    for (const ilpm_heads *h : {k, v, q, q_out})
        if (h && (rc = check_heads(*h)) != ILPM_OK) return rc;
    if (k->heads != c.kv_heads || v->heads != c.kv_heads || (q && q->heads != q_out->heads)) return ILPM_ERR_INVALID_ARG;
    if (k->dtype != v->dtype || (q && (q->dtype != k->dtype || q_out->dtype != k->dtype)) ||
        (k->dtype != c.dtype && k->dtype != ILPM_F32))
        return ILPM_ERR_UNSUPPORTED;
    if ((o.q_w || o.k_w) && o.param_dtype != k->dtype && o.param_dtype != ILPM_F32) return ILPM_ERR_UNSUPPORTED;
    const int param = o.q_w || o.k_w ? o.param_dtype : k->dtype;
    if (!aligned(o.q_w, param) || !aligned(o.k_w, param)) return ILPM_ERR_INVALID_ARG;
    const int32_t *slots = o.slots ? o.slots : o.positions;
    if (!o.seq_ids || !o.positions || ((uintptr_t)o.seq_ids | (uintptr_t)o.positions | (uintptr_t)slots) % 4) return ILPM_ERR_INVALID_ARG;
    if (o.rot_dim > 0 && o.n_positions > 0 && (!o.cos || !o.sin || ((uintptr_t)o.cos | (uintptr_t)o.sin) % 4)) return ILPM_ERR_INVALID_ARG;
    const int64_t heads = (int64_t)(q ? q->heads : 0) + 2 * (int64_t)c.kv_heads;
    if (n_tokens > kMaxGroups || heads > kMaxGroups || heads * n_tokens > kMaxGroups * 4) return ILPM_ERR_UNSUPPORTED;

    // What is written: the pools and q_out.
    const int64_t angles = o.rot_dim > 0 ? (int64_t)o.n_positions * (o.rot_dim / 2) * 4 : 0;
    const int64_t ints = (int64_t)n_tokens * 4, weights = (int64_t)c.head_dim * element_bytes(param);
    const Span read[] = {span_of(*k, n_tokens, c.head_dim), span_of(*v, n_tokens, c.head_dim), flat_span(o.seq_ids, ints),
                         flat_span(o.positions, ints), flat_span(slots, ints), flat_span(o.cos, angles), flat_span(o.sin, angles),
                         flat_span(o.q_w, weights), flat_span(o.k_w, weights), table_span(c)};
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
        if (!writes_once(so) || (!same_place(*q, *q_out) && touch(sq, so))) return ILPM_ERR_INVALID_ARG;
        for (const Span &s : read)
            if (s.at && s.bytes() > 0 && touch(s, so)) return ILPM_ERR_INVALID_ARG;
    }

    int dev = 0;
    if ((rc = api_device_check(&dev)) != ILPM_OK) return rc;
    AppendNormArgs n = {};
    AppendArgs &a = n.a;
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
    a.seq_ids = o.seq_ids;
    a.positions = o.positions;
    a.cos = o.cos;
    a.sin = o.sin;
    a.n_positions = o.n_positions;
    a.rot_dim = o.rot_dim;
    a.pairs = o.pairs;
    n.slots = slots;
    n.q_w = o.q_w;
    n.k_w = o.k_w;
    n.norm = o.norm;
    n.eps = o.eps;
    (void)hipGetLastError();
    const hipError_t e = append_norm_launch(n, k->dtype, c.dtype, param, stream);
    return e == hipSuccess ? ILPM_OK : api_hip_fail(e);
}

int tree_sizes(const ilpm_kv_cache *c, int q_heads, int n_nodes, bool q32, int window, int sinks, int max_len, TreeArgs *t, size_t *bytes)
{
    if (q_heads <= 0 || q_heads % c->kv_heads != 0 || n_nodes < 0 || window < 0 || sinks < 0 || max_len < 0) return ILPM_ERR_INVALID_ARG;
    if (c->head_dim > 256 || n_nodes > ILPM_MAX_NODES) return ILPM_ERR_UNSUPPORTED;
    if ((int64_t)c->n_seqs * n_nodes * q_heads > kMaxGroups) return ILPM_ERR_UNSUPPORTED;
    AttnArgs &a = t->a;
    a.n_seqs = c->n_seqs;
    a.q_heads = q_heads;
    a.kv_heads = c->kv_heads;
    a.group = q_heads / c->kv_heads;
    a.dim = c->head_dim;
    a.window = window;
    a.capacity = capacity_of(*c);
    t->n_nodes = n_nodes;
    t->sinks = sinks;
    *bytes = tree_plan(t, c->dtype, q32, max_len > 0 ? std::min(max_len, a.capacity) : a.capacity);
    return ILPM_OK;
}

int attn_tree(const ilpm_kv_cache *cache, const ilpm_heads *q, const int32_t *lengths, const int32_t *parents, int n_nodes,
              const ilpm_tree_options *opt, const ilpm_heads *out, float *lse, void *workspace, size_t workspace_bytes,
              hipStream_t stream)
{
    int rc = check_cache(cache);
    if (rc != ILPM_OK) return rc;
    const ilpm_kv_cache &c = *cache;
    if (!q || !out || !opt || q->heads <= 0 || out->heads != q->heads) return ILPM_ERR_INVALID_ARG;
    TreeArgs t = {};
    size_t need = 0;
    if ((rc = tree_sizes(cache, q->heads, n_nodes, q->dtype == ILPM_F32, opt->window, opt->sinks, opt->max_len, &t, &need)) != ILPM_OK) return rc;
    // (Scores are formed times log2 e, or over softcap.)
    if (!std::isfinite(opt->scale * 1.5f) || !(opt->softcap >= 0.f) || !std::isfinite(opt->softcap * 1.5f) ||
        (opt->softcap > 0.f && !std::isfinite(opt->scale / opt->softcap)))
        return ILPM_ERR_INVALID_ARG;
    if (opt->mask && (opt->mask_len < 0 || !stride_ok(opt->mask_stride))) return ILPM_ERR_INVALID_ARG;
    if (c.n_seqs == 0 || n_nodes == 0) return ILPM_OK;
    if ((rc = check_heads(*q)) != ILPM_OK || (rc = check_heads(*out)) != ILPM_OK) return rc;
    if (q->dtype != out->dtype || (q->dtype != c.dtype && q->dtype != ILPM_F32)) return ILPM_ERR_UNSUPPORTED;
    if (!lengths || !parents || ((uintptr_t)lengths | (uintptr_t)parents | (uintptr_t)lse) % 4 || (uintptr_t)workspace % 256)
        return ILPM_ERR_INVALID_ARG;

    // What is written: out, lse and the workspace.
    const int64_t rows = (int64_t)c.n_seqs * n_nodes;
    const Span sq = span_of(*q, rows, c.head_dim), so = span_of(*out, rows, c.head_dim);
    if (!writes_once(so) || (!same_place(*q, *out) && touch(sq, so))) return ILPM_ERR_INVALID_ARG;
    const Span sl = flat_span(lse, rows * q->heads * 4);
    const Span sw = flat_span(workspace, (int64_t)std::min<size_t>(need, (size_t)1 << 60));
    const bool has_ws = workspace && need > 0;
    if (lse && (touch(sl, so) || touch(sl, sq))) return ILPM_ERR_INVALID_ARG;
    if (has_ws && (touch(sw, so) || touch(sw, sq) || (lse && touch(sw, sl)))) return ILPM_ERR_INVALID_ARG;
    Span read[6];
    int n = 0;
    read[n++] = flat_span(lengths, (int64_t)c.n_seqs * 4);
    read[n++] = flat_span(parents, rows * 4);
    if (t.a.capacity > 0) {
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
    AttnArgs &a = t.a;
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
    t.parents = parents;
    if (need > 0) tree_workspace(&t, ws);
    (void)hipGetLastError();
    const hipError_t e = tree_launch(t, c.dtype, stream);
    return e == hipSuccess ? ILPM_OK : api_hip_fail(e);
}

int verify_sizes(int n_seqs, int n_nodes, int vocab, VerifyArgs *a, size_t *bytes)
{
    if (n_seqs < 0 || n_nodes <= 0 || vocab <= 0) return ILPM_ERR_INVALID_ARG;
    if (n_nodes > ILPM_MAX_NODES || vocab > kMostVocab || n_seqs > kMostRows) return ILPM_ERR_UNSUPPORTED;
    a->v.n_seqs = n_seqs;
    a->v.n_nodes = n_nodes;
    a->v.vocab = vocab;
    *bytes = n_seqs > 0 ? verify_plan(a) : 0;
    return ILPM_OK;
}

int verify_drafts(const ilpm_verify_args *args, void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    if (!args) return ILPM_ERR_INVALID_ARG;
    VerifyArgs a = {};
    a.v = *args;
    const ilpm_verify_args &v = a.v;
    size_t need = 0;
    int rc = verify_sizes(v.n_seqs, v.n_nodes, v.vocab, &a, &need);
    if (rc != ILPM_OK) return rc;
    if (!type_ok(v.dtype)) return ILPM_ERR_UNSUPPORTED;
    for (int64_t s : {v.target_seq_stride, v.target_node_stride, v.draft_seq_stride, v.draft_node_stride})
        if (!stride_ok(s)) return ILPM_ERR_INVALID_ARG;
    if (v.n_seqs == 0) return ILPM_OK;
    if (!v.tokens || !v.parents || !v.target || !v.uniforms || !v.path || !v.counts || !v.next_tokens) return ILPM_ERR_INVALID_ARG;
    if (!aligned(v.target, v.dtype) || !aligned(v.draft, v.dtype) || (uintptr_t)workspace % 256) return ILPM_ERR_INVALID_ARG;
    for (const void *p : {(const void *)v.tokens, (const void *)v.parents, (const void *)v.uniforms, (const void *)v.path,
                          (const void *)v.counts, (const void *)v.next_tokens})
        if ((uintptr_t)p % 4) return ILPM_ERR_INVALID_ARG;

    const int64_t e = element_bytes(v.dtype), nodes = (int64_t)v.n_seqs * v.n_nodes * 4, seqs = (int64_t)v.n_seqs * 4;
    const bool has_ws = workspace && need > 0;
    const Span write[] = {flat_span(v.path, nodes), flat_span(v.counts, seqs), flat_span(v.next_tokens, seqs),
                          flat_span(workspace, (int64_t)need)};
    const int writes = has_ws ? 4 : 3;
    const Span read[] = {flat_span(v.tokens, nodes), flat_span(v.parents, nodes), flat_span(v.uniforms, nodes),
                         {(uintptr_t)v.target, {v.n_seqs, v.n_nodes, 1}, {v.target_seq_stride * e, v.target_node_stride * e, 0}, v.vocab * e},
                         {(uintptr_t)v.draft, {v.n_seqs, v.n_nodes, 1}, {v.draft_seq_stride * e, v.draft_node_stride * e, 0}, v.vocab * e}};
    for (int i = 0; i < writes; ++i) {
        for (int j = i + 1; j < writes; ++j)
            if (touch(write[i], write[j])) return ILPM_ERR_INVALID_ARG;
        for (const Span &r : read)
            if (r.at && touch(r, write[i])) return ILPM_ERR_INVALID_ARG;
    }

    int dev = 0;
    if ((rc = api_device_check(&dev)) != ILPM_OK) return rc;
    void *ws = workspace;
    if (need > 0) {
        if (!ws) rc = api_workspace(dev, need, stream, &ws);
        else if (workspace_bytes < need) rc = ILPM_ERR_WORKSPACE;
        if (rc != ILPM_OK) return rc;
        verify_workspace(&a, ws);
    }
    (void)hipGetLastError();
    const hipError_t err = verify_launch(a, stream);
    return err == hipSuccess ? ILPM_OK : api_hip_fail(err);
}

int kv_copy(const ilpm_kv_cache *cache, const int32_t *dst_table, int64_t dst_table_stride, int dst_max_pages,
            const int32_t *src_start, const int32_t *dst_start, const int32_t *counts, const int32_t *path,
            int64_t path_stride, int max_count, hipStream_t stream)
{
    int rc = check_cache(cache);
    if (rc != ILPM_OK) return rc;
    const ilpm_kv_cache &c = *cache;
    if (dst_max_pages < 0 || max_count < 0 || !stride_ok(dst_table_stride) || !stride_ok(path_stride)) return ILPM_ERR_INVALID_ARG;
    if (path && max_count > ILPM_MAX_NODES) return ILPM_ERR_UNSUPPORTED;
    if (c.n_seqs == 0 || max_count == 0) return ILPM_OK;
    if (!src_start || !dst_start || !counts) return ILPM_ERR_INVALID_ARG;
    for (const int32_t *p : {dst_table, src_start, dst_start, counts, path})
        if ((uintptr_t)p % 4) return ILPM_ERR_INVALID_ARG;
    if (dst_max_pages > 0 && !dst_table) return ILPM_ERR_INVALID_ARG;
    if (c.n_pages == 0 || c.max_pages == 0 || dst_max_pages == 0) return ILPM_OK;  // (no token has a place)
    const int64_t e = element_bytes(c.dtype);
    // (What a grid's dimensions hold, and a token's pieces an int.)
    if (c.n_seqs > kMostRows || (int64_t)c.kv_heads * c.head_dim > 1 << 26) return ILPM_ERR_UNSUPPORTED;

    // What is written: the pools.
    const Span pk = pool_span(c, false), pv = pool_span(c, true);
    if (!writes_once(pk) || !writes_once(pv) || touch(pk, pv)) return ILPM_ERR_INVALID_ARG;
    const int64_t ints = (int64_t)c.n_seqs * 4;
    const Span read[] = {table_span(c), rows_span(dst_table, c.n_seqs, dst_table_stride * 4, (int64_t)dst_max_pages * 4),
                         flat_span(src_start, ints), flat_span(dst_start, ints), flat_span(counts, ints),
                         rows_span(path, c.n_seqs, path_stride * 4, (int64_t)max_count * 4)};
    for (const Span &s : read)
        if (s.at && (touch(s, pk) || touch(s, pv))) return ILPM_ERR_INVALID_ARG;

    int dev = 0;
    if ((rc = api_device_check(&dev)) != ILPM_OK) return rc;
    CopyArgs a = {};
    a.k = c.k;
    a.v = c.v;
    a.k_page = c.k_page_stride * e;
    a.k_slot = c.k_slot_stride * e;
    a.k_head = c.k_head_stride * e;
    a.v_page = c.v_page_stride * e;
    a.v_slot = c.v_slot_stride * e;
    a.v_head = c.v_head_stride * e;
    a.row_bytes = (int)(c.head_dim * e);
    a.kv_heads = c.kv_heads;
    a.n_pages = c.n_pages;
    a.page_size = c.page_size;
    a.src_table = c.page_table;
    a.dst_table = dst_table;
    a.src_table_stride = c.table_stride;
    a.dst_table_stride = dst_table_stride;
    a.src_max_pages = c.max_pages;
    a.dst_max_pages = dst_max_pages;
    a.n_seqs = c.n_seqs;
    a.src_start = src_start;
    a.dst_start = dst_start;
    a.counts = counts;
    a.path = path;
    a.path_stride = path_stride;
    a.max_count = max_count;
    (void)hipGetLastError();
    const hipError_t err = copy_launch(a, stream);
    return err == hipSuccess ? ILPM_OK : api_hip_fail(err);
}

}  // namespace
}  // namespace ilpm

using namespace ilpm;

extern "C" {

int ilpm_kv_append_norm(const ilpm_kv_cache *cache, const ilpm_heads *k, const ilpm_heads *v, const ilpm_heads *q,
                        const ilpm_heads *q_out, const ilpm_append_options *options, int n_tokens, hipStream_t stream)
{
    return guarded([&] { return kv_append_norm(cache, k, v, q, q_out, options, n_tokens, stream); });
}

int ilpm_attn_tree(const ilpm_kv_cache *cache, const ilpm_heads *q, const int32_t *lengths, const int32_t *parents,
                   int n_nodes, const ilpm_tree_options *options, const ilpm_heads *out, float *lse, void *workspace,
                   size_t workspace_bytes, hipStream_t stream)
{
    return guarded([&] { return attn_tree(cache, q, lengths, parents, n_nodes, options, out, lse, workspace, workspace_bytes, stream); });
}

int ilpm_attn_tree_workspace_size(const ilpm_kv_cache *cache, int q_heads, int n_nodes, int window, int sinks,
                                  int max_len, size_t *bytes)
{
    if (!bytes) return ILPM_ERR_INVALID_ARG;
    int rc = check_cache_sizes(cache);
    if (rc != ILPM_OK) return rc;
    TreeArgs t = {};
    // Of either type of queries, the larger.
    size_t other = 0;
    if ((rc = tree_sizes(cache, q_heads, n_nodes, true, window, sinks, max_len, &t, &other)) != ILPM_OK) return rc;
    rc = tree_sizes(cache, q_heads, n_nodes, false, window, sinks, max_len, &t, bytes);
    *bytes = std::max(*bytes, other);
    return rc;
}

int ilpm_verify_drafts(const ilpm_verify_args *args, void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    return guarded([&] { return verify_drafts(args, workspace, workspace_bytes, stream); });
}

int ilpm_verify_drafts_workspace_size(int n_seqs, int n_nodes, int vocab, size_t *bytes)
{
    if (!bytes) return ILPM_ERR_INVALID_ARG;
    VerifyArgs a = {};
    return verify_sizes(n_seqs, n_nodes, vocab, &a, bytes);
}

int ilpm_kv_copy(const ilpm_kv_cache *cache, const int32_t *dst_table, int64_t dst_table_stride, int dst_max_pages,
                 const int32_t *src_start, const int32_t *dst_start, const int32_t *counts, const int32_t *path,
                 int64_t path_stride, int max_count, hipStream_t stream)
{
    return guarded([&] {
        return kv_copy(cache, dst_table, dst_table_stride, dst_max_pages, src_start, dst_start, counts, path, path_stride, max_count, stream);
    });
}

}  // extern "C"
