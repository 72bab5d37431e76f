// What the entry points of the decoder-step operators check arguments with:
// types, strides, the spans of strided tensors and whether two of them touch.
#pragma once

#include <algorithm>
#include <climits>
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
