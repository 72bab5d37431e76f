// The decoder-step operators as Python calls them: tensors checked, described
// in the C ABI's structures and handed to it, and outputs allocated on the
// current stream, without the interpreter's part in each of these (a small call
// takes 4.9 to 5.7 us in place of 12, of which its launch is 3.3).  Nothing is
// computed here.  The functions take
// all arguments by position, from the wrappers in __init__.py, and return what
// those return, or the negative status of the C call.
#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <ATen/hip/impl/HIPCachingAllocatorMasqueradingAsCUDA.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <climits>
#include <cmath>
#include <string>

#include "ilpm.h"

namespace {

[[noreturn]] void fail(PyObject *type, const std::string &what)
{
    PyErr_SetString(type, what.c_str());
    throw python_error();
}
[[noreturn]] void type_error(const std::string &what) { fail(PyExc_TypeError, what); }
[[noreturn]] void value_error(const std::string &what) { fail(PyExc_ValueError, what); }

std::string sizes(std::initializer_list<int64_t> v)
{
    std::string s = "[";
    for (int64_t n : v) s += (s.size() > 1 ? ", " : "") + (n < 0 ? std::string("...") : std::to_string(n));
    return s + "]";
}

// A CUDA tensor on the current device.
const at::Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) type_error(std::string(name) + " must be a CUDA tensor");
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda()) type_error(std::string(name) + " must be a CUDA tensor");
    if (t.get_device() != c10::hip::current_device()) value_error(std::string(name) + " is not on the current device");
    return t;
}

bool given(PyObject *o) { return o != Py_None; }

int int_arg(PyObject *o, const char *name)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    if (v < INT_MIN || v > INT_MAX) value_error(std::string(name) + " is out of range");
    return (int)v;
}

float float_arg(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return (float)v;
}

bool bool_arg(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v != 0;
}

int size_arg(int64_t n, const char *name)
{
    if (n > INT_MAX) value_error(std::string(name) + " is too large");
    return (int)n;
}

int dtype_of(const at::Tensor &t, const char *name)
{
    switch (t.scalar_type()) {
    case at::kFloat: return ILPM_F32;
    case at::kHalf: return ILPM_F16;
    case at::kBFloat16: return ILPM_BF16;
    default: type_error(std::string(name) + " must be a float32, float16 or bfloat16 tensor");
    }
}

bool last_contiguous(const at::Tensor &t) { return t.size(-1) <= 1 || t.stride(-1) == 1; }

ilpm_heads heads_of(const at::Tensor &t, const char *name, int64_t rows, int64_t dim)
{
    if (t.dim() != 3 || t.size(0) != rows || t.size(2) != dim || !last_contiguous(t))
        value_error(std::string(name) + " must be " + sizes({rows, -1, dim}) + ", [rows, heads, head_dim], with its last dimension contiguous");
    return {t.data_ptr(), t.stride(0), t.stride(1), dtype_of(t, name), size_arg(t.size(1), name)};
}

const int32_t *ints_of(const at::Tensor &t, const char *name, int dims)
{
    if (t.scalar_type() != at::kInt || t.dim() != dims) type_error(std::string(name) + " must be a " + std::to_string(dims) + "-dimensional int32 CUDA tensor");
    if (!last_contiguous(t)) value_error(std::string(name) + "'s last dimension must be contiguous");
    return (const int32_t *)t.data_ptr();
}

const float *floats_of(const at::Tensor &t, const char *name)
{
    if (t.scalar_type() != at::kFloat || !t.is_contiguous()) type_error(std::string(name) + " must be a contiguous float32 CUDA tensor");
    return (const float *)t.data_ptr();
}

ilpm_kv_cache cache_of(PyObject *k_pages, PyObject *v_pages, PyObject *page_table)
{
    const at::Tensor &k = tensor(k_pages, "k_pages"), &v = tensor(v_pages, "v_pages"), &table = tensor(page_table, "page_table");
    if (k.dim() != 4 || v.sizes() != k.sizes() || v.scalar_type() != k.scalar_type())
        value_error("k_pages and v_pages must be [n_pages, page_size, kv_heads, head_dim] of one type");
    if (!last_contiguous(k) || !last_contiguous(v)) value_error("the last dimension of k_pages and v_pages must be contiguous");
    ilpm_kv_cache c = {};
    c.k = k.data_ptr();
    c.v = v.data_ptr();
    c.k_page_stride = k.stride(0);
    c.k_slot_stride = k.stride(1);
    c.k_head_stride = k.stride(2);
    c.v_page_stride = v.stride(0);
    c.v_slot_stride = v.stride(1);
    c.v_head_stride = v.stride(2);
    c.page_table = ints_of(table, "page_table", 2);
    c.table_stride = table.stride(0);
    c.dtype = dtype_of(k, "k_pages");
    c.n_pages = size_arg(k.size(0), "n_pages");
    c.page_size = size_arg(k.size(1), "page_size");
    c.kv_heads = size_arg(k.size(2), "kv_heads");
    c.head_dim = size_arg(k.size(3), "head_dim");
    c.n_seqs = size_arg(table.size(0), "n_seqs");
    c.max_pages = size_arg(table.size(1), "max_pages");
    return c;
}

// On the current device.  (Straight from torch's allocator: by way of at::empty's
// dispatch a tensor costs 0.4 us more.)
at::Tensor empty(at::IntArrayRef shape, at::ScalarType type)
{
    return at::Tensor(at::detail::empty_generic(shape, c10::hip::HIPCachingAllocatorMasqueradingAsCUDA::get(),
                                                c10::DispatchKeySet(c10::DispatchKey::CUDA), type, std::nullopt));
}

hipStream_t current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

void count(Py_ssize_t got, Py_ssize_t want)
{
    if (got != want) type_error("takes " + std::to_string(want) + " arguments");
}

PyObject *none() { Py_RETURN_NONE; }

// (k, v, k_pages, v_pages, page_table, seq_ids, positions, q, cos, sin, pairs, q_out) -> q_out or None
PyObject *kv_append(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    count(n_args, 12);
    const at::Tensor &k = tensor(args[0], "k"), &v = tensor(args[1], "v");
    const ilpm_kv_cache c = cache_of(args[2], args[3], args[4]);
    const at::Tensor &seq = tensor(args[5], "seq_ids"), &pos = tensor(args[6], "positions");
    const int32_t *seq_p = ints_of(seq, "seq_ids", 1), *pos_p = ints_of(pos, "positions", 1);
    const int64_t n = pos.size(0);
    if (seq.size(0) != n) value_error("seq_ids and positions must be of one length");
    const ilpm_heads hk = heads_of(k, "k", n, c.head_dim), hv = heads_of(v, "v", n, c.head_dim);
    const float *cos = nullptr, *sin = nullptr;
    int n_positions = 0, half = 0;
    if (given(args[8]) || given(args[9])) {
        if (!given(args[8]) || !given(args[9])) value_error("cos and sin must both be given");
        const at::Tensor &tc = tensor(args[8], "cos"), &ts = tensor(args[9], "sin");
        if (tc.dim() != 2 || ts.sizes() != tc.sizes()) value_error("cos and sin must both be [n_positions, rot_dim / 2]");
        cos = floats_of(tc, "cos");
        sin = floats_of(ts, "sin");
        n_positions = size_arg(tc.size(0), "n_positions");
        half = size_arg(std::min<int64_t>(tc.size(1), INT_MAX / 2), "rot_dim");
    }
    ilpm_heads hq = {}, ho = {};
    at::Tensor out;
    if (given(args[7])) {
        const at::Tensor &q = tensor(args[7], "q");
        hq = heads_of(q, "q", n, c.head_dim);
        out = given(args[11]) ? tensor(args[11], "q_out") : empty(q.sizes(), q.scalar_type());
        ho = heads_of(out, "q_out", n, c.head_dim);
    } else if (given(args[11])) {
        value_error("q_out is given without q");
    }
    const bool has_q = out.defined();
    const int rc = ilpm_kv_append(&c, &hk, &hv, has_q ? &hq : nullptr, has_q ? &ho : nullptr, seq_p, pos_p, size_arg(n, "tokens"), cos,
                                  sin, n_positions, 2 * half, bool_arg(args[10]) ? 1 : 0, current_stream());
    if (rc != ILPM_OK) return PyLong_FromLong(rc);
    return has_q ? THPVariable_Wrap(out) : none();
    END_HANDLE_TH_ERRORS
}

// (q, k_pages, v_pages, page_table, lengths, scale, window, softcap, mask, max_len, out, lse, return_lse, workspace)
//  -> out or (out, lse)
PyObject *attn_decode(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    count(n_args, 14);
    const at::Tensor &q = tensor(args[0], "q");
    const ilpm_kv_cache c = cache_of(args[1], args[2], args[3]);
    const at::Tensor &lengths = tensor(args[4], "lengths");
    const int32_t *lengths_p = ints_of(lengths, "lengths", 1);
    if (lengths.size(0) != c.n_seqs) value_error("lengths must be " + sizes({c.n_seqs}));
    const ilpm_heads hq = heads_of(q, "q", c.n_seqs, c.head_dim);
    const at::Tensor out = given(args[10]) ? tensor(args[10], "out") : empty(q.sizes(), q.scalar_type());
    const ilpm_heads ho = heads_of(out, "out", c.n_seqs, c.head_dim);
    at::Tensor lse;
    if (given(args[11])) lse = tensor(args[11], "lse");
    else if (bool_arg(args[12])) lse = empty({c.n_seqs, hq.heads}, at::kFloat);
    if (lse.defined() && (lse.dim() != 2 || lse.size(0) != c.n_seqs || lse.size(1) != hq.heads)) value_error("lse must be " + sizes({c.n_seqs, hq.heads}));
    ilpm_attn_options o = {};
    o.scale = given(args[5]) ? float_arg(args[5]) : (float)(1.0 / std::sqrt((double)c.head_dim));
    o.window = int_arg(args[6], "window");
    o.softcap = float_arg(args[7]);
    o.max_len = int_arg(args[9], "max_len");
    if (given(args[8])) {
        const at::Tensor &mask = tensor(args[8], "mask");
        if (mask.scalar_type() != at::kBool && mask.scalar_type() != at::kByte) type_error("mask must be a bool or uint8 CUDA tensor");
        if (mask.dim() != 2 || mask.size(0) != c.n_seqs || !last_contiguous(mask))
            value_error("mask must be " + sizes({c.n_seqs, -1}) + ", [n_seqs, keys], with its last dimension contiguous");
        // (A mask of no columns has no memory, and still hides every key: it is never read then.)
        o.mask = (const uint8_t *)(mask.data_ptr() ? mask.data_ptr() : lengths.data_ptr());
        o.mask_stride = mask.stride(0);
        o.mask_len = size_arg(mask.size(1), "mask");
    }
    size_t need = 0;
    int rc = ilpm_attn_decode_workspace_size(&c, hq.heads, o.window, o.max_len, &need);
    if (rc != ILPM_OK) return PyLong_FromLong(rc);
    at::Tensor ws;
    if (given(args[13])) {
        ws = tensor(args[13], "workspace");
        // (Of a view the bytes between its elements are not the caller's to give, nor are there nbytes() behind an expanded one.)
        if (!ws.is_contiguous()) value_error("workspace must be contiguous");
    } else if (need > 0) ws = empty({(int64_t)need}, at::kByte);
    rc = ilpm_attn_decode(&c, &hq, lengths_p, &o, &ho, lse.defined() ? (float *)floats_of(lse, "lse") : nullptr,
                          ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? ws.nbytes() : 0, current_stream());
    if (rc != ILPM_OK) return PyLong_FromLong(rc);
    if (!lse.defined()) return THPVariable_Wrap(out);
    THPObjectPtr a(THPVariable_Wrap(out)), b(THPVariable_Wrap(lse));
    return a && b ? PyTuple_Pack(2, a.get(), b.get()) : nullptr;
    END_HANDLE_TH_ERRORS
}

// (k_pages, v_pages, page_table, q_heads, window, max_len) -> bytes, or a negative status
PyObject *attn_decode_workspace_size(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    count(n_args,  6);
    const ilpm_kv_cache c = cache_of(args[0], args[1], args[2]);
    size_t need = 0;
    const int rc = ilpm_attn_decode_workspace_size(&c, int_arg(args[3], "q_heads"), int_arg(args[4], "window"), int_arg(args[5], "max_len"), &need);
    return rc == ILPM_OK ? PyLong_FromSize_t(need) : PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

int64_t row_stride(const at::Tensor &t, const char *name, int64_t rows, int64_t width)
{
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != width || !last_contiguous(t))
        value_error(std::string(name) + " must be " + sizes({rows, width}) + " with its last dimension contiguous");
    return t.stride(0);
}

// (x, y, post, post_w, post_b, gate, scale, pre, pre_w, pre_b, eps, r, z) -> (r or x, z or None); post and pre
// are ILPM_NORM_*
PyObject *residual_norm(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    count(n_args, 13);
    const at::Tensor &x = tensor(args[0], "x");
    if (x.dim() != 2) value_error("x must be [rows, width]");
    const int64_t rows = x.size(0), width = x.size(1);
    ilpm_residual_norm_args g = {};
    g.rows = size_arg(rows, "rows");
    g.width = size_arg(width, "width");
    g.post = int_arg(args[2], "post");
    g.pre = int_arg(args[7], "pre");
    g.scale = float_arg(args[6]);
    g.eps = float_arg(args[10]);
    g.x = x.data_ptr();
    g.x_stride = row_stride(x, "x", rows, width);
    g.x_dtype = dtype_of(x, "x");
    at::Tensor y, r, z;
    if (given(args[1])) y = tensor(args[1], "y");
    if (given(args[11])) r = tensor(args[11], "r");
    else if (y.defined()) r = empty(x.sizes(), x.scalar_type());
    if (given(args[12])) z = tensor(args[12], "z");
    const at::Tensor &kind = y.defined() ? y : z.defined() ? z : x;  // of whose type blocks are
    if (!z.defined() && g.pre != ILPM_NORM_NONE) z = empty(x.sizes(), kind.scalar_type());
    g.y_dtype = dtype_of(kind, y.defined() ? "y" : "z");
    if (y.defined()) {
        g.y = y.data_ptr();
        g.y_stride = row_stride(y, "y", rows, width);
    }
    if (r.defined()) {
        if (r.scalar_type() != x.scalar_type()) type_error("r must be of x's type");
        g.r = r.data_ptr();
        g.r_stride = row_stride(r, "r", rows, width);
    }
    if (z.defined()) {
        if (z.scalar_type() != kind.scalar_type()) type_error("z must be of y's type");
        g.z = z.data_ptr();
        g.z_stride = row_stride(z, "z", rows, width);
    }
    at::ScalarType params = at::ScalarType::Undefined;
    auto same_type = [&](const at::Tensor &t) {
        if (params != at::ScalarType::Undefined && t.scalar_type() != params) type_error("weights, biases and gate must be of one type");
        params = t.scalar_type();
    };
    auto vector = [&](PyObject *o, const char *name) -> const void * {
        if (!given(o)) return nullptr;
        const at::Tensor &t = tensor(o, name);
        if (t.dim() != 1 || t.size(0) != width || !last_contiguous(t)) value_error(std::string(name) + " must be a contiguous CUDA tensor " + sizes({width}));
        same_type(t);
        return t.data_ptr();
    };
    g.post_w = vector(args[3], "post_w");
    g.post_b = vector(args[4], "post_b");
    g.pre_w = vector(args[8], "pre_w");
    g.pre_b = vector(args[9], "pre_b");
    if (given(args[5])) {
        const at::Tensor &gate = tensor(args[5], "gate");
        if (gate.dim() == 1) {
            g.gate = vector(args[5], "gate");
        } else {
            g.gate_stride = row_stride(gate, "gate", rows, width);
            g.gate = gate.data_ptr();
            same_type(gate);
        }
    }
    switch (params) {
    case at::ScalarType::Undefined: g.param_dtype = g.y_dtype; break;
    case at::kFloat: g.param_dtype = ILPM_F32; break;
    case at::kHalf: g.param_dtype = ILPM_F16; break;
    case at::kBFloat16: g.param_dtype = ILPM_BF16; break;
    default: type_error("weights, biases and gate must be float32, float16 or bfloat16 tensors");
    }
    const int rc = ilpm_residual_norm(&g, current_stream());
    if (rc != ILPM_OK) return PyLong_FromLong(rc);
    THPObjectPtr a(r.defined() ? THPVariable_Wrap(r) : THPVariable_Wrap(x)), b(z.defined() ? THPVariable_Wrap(z) : none());
    return a && b ? PyTuple_Pack(2, a.get(), b.get()) : nullptr;
    END_HANDLE_TH_ERRORS
}

// (k, v, k_pages, v_pages, page_table, seq_ids, positions, slots, q, norm, q_w, k_w, eps, cos, sin, pairs, q_out)
//  -> q_out or None; norm is ILPM_NORM_*
PyObject *kv_append_norm(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    count(n_args, 17);
    const at::Tensor &k = tensor(args[0], "k"), &v = tensor(args[1], "v");
    const ilpm_kv_cache c = cache_of(args[2], args[3], args[4]);
    ilpm_append_options o = {};
    const at::Tensor &seq = tensor(args[5], "seq_ids"), &pos = tensor(args[6], "positions");
    o.seq_ids = ints_of(seq, "seq_ids", 1);
    o.positions = ints_of(pos, "positions", 1);
    const int64_t n = pos.size(0);
    if (seq.size(0) != n) value_error("seq_ids and positions must be of one length");
    if (given(args[7])) {
        const at::Tensor &slots = tensor(args[7], "slots");
        o.slots = ints_of(slots, "slots", 1);
        if (slots.size(0) != n) value_error("slots and positions must be of one length");
    }
    const ilpm_heads hk = heads_of(k, "k", n, c.head_dim), hv = heads_of(v, "v", n, c.head_dim);
    o.norm = int_arg(args[9], "norm");
    o.eps = float_arg(args[12]);
    o.pairs = bool_arg(args[15]) ? 1 : 0;
    o.param_dtype = hk.dtype;
    auto weight = [&](PyObject *w, const char *name) -> const void * {
        if (!given(w)) return nullptr;
        const at::Tensor &t = tensor(w, name);
        if (t.dim() != 1 || t.size(0) != c.head_dim || !last_contiguous(t)) value_error(std::string(name) + " must be a contiguous CUDA tensor " + sizes({c.head_dim}));
        o.param_dtype = dtype_of(t, name);
        return t.data_ptr();
    };
    o.q_w = weight(args[10], "q_w");
    const int q_w_dtype = o.param_dtype;
    o.k_w = weight(args[11], "k_w");
    if (o.q_w && o.k_w && o.param_dtype != q_w_dtype) type_error("q_w and k_w must be of one type");
    if (given(args[13]) || given(args[14])) {
        if (!given(args[13]) || !given(args[14])) value_error("cos and sin must both be given");
        const at::Tensor &tc = tensor(args[13], "cos"), &ts = tensor(args[14], "sin");
        if (tc.dim() != 2 || ts.sizes() != tc.sizes()) value_error("cos and sin must both be [n_positions, rot_dim / 2]");
        o.cos = floats_of(tc, "cos");
        o.sin = floats_of(ts, "sin");
        o.n_positions = size_arg(tc.size(0), "n_positions");
        o.rot_dim = 2 * size_arg(std::min<int64_t>(tc.size(1), INT_MAX / 2), "rot_dim");
    }
    ilpm_heads hq = {}, ho = {};
    at::Tensor out;
    if (given(args[8])) {
        const at::Tensor &q = tensor(args[8], "q");
        hq = heads_of(q, "q", n, c.head_dim);
        out = given(args[16]) ? tensor(args[16], "q_out") : empty(q.sizes(), q.scalar_type());
        ho = heads_of(out, "q_out", n, c.head_dim);
    } else if (given(args[16]) || given(args[10])) {
        value_error("q_out or q_w is given without q");
    }
    const bool has_q = out.defined();
    const int rc = ilpm_kv_append_norm(&c, &hk, &hv, has_q ? &hq : nullptr, has_q ? &ho : nullptr, &o, size_arg(n, "tokens"), current_stream());
    if (rc != ILPM_OK) return PyLong_FromLong(rc);
    return has_q ? THPVariable_Wrap(out) : none();
    END_HANDLE_TH_ERRORS
}

// The workspace given, or one of `need` bytes.
at::Tensor workspace_of(PyObject *o, size_t need)
{
    if (!given(o)) return need > 0 ? empty({(int64_t)need}, at::kByte) : at::Tensor();
    const at::Tensor &ws = tensor(o, "workspace");
    if (!ws.is_contiguous()) value_error("workspace must be contiguous");  // (as of attn_decode)
    return ws;
}

// (q, k_pages, v_pages, page_table, lengths, parents, scale, window, sinks, softcap, mask, max_len, out, lse, return_lse,
//  workspace) -> out or (out, lse)
PyObject *attn_tree(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    count(n_args, 16);
    const at::Tensor &q = tensor(args[0], "q");
    const ilpm_kv_cache c = cache_of(args[1], args[2], args[3]);
    const at::Tensor &lengths = tensor(args[4], "lengths"), &parents = tensor(args[5], "parents");
    const int32_t *lengths_p = ints_of(lengths, "lengths", 1), *parents_p = ints_of(parents, "parents", 2);
    if (lengths.size(0) != c.n_seqs) value_error("lengths must be " + sizes({c.n_seqs}));
    if (parents.size(0) != c.n_seqs || !parents.is_contiguous()) value_error("parents must be contiguous, " + sizes({c.n_seqs, -1}));
    const int nodes = size_arg(parents.size(1), "nodes");
    const int64_t rows = (int64_t)c.n_seqs * nodes;
    const ilpm_heads hq = heads_of(q, "q", rows, c.head_dim);
    const at::Tensor out = given(args[12]) ? tensor(args[12], "out") : empty(q.sizes(), q.scalar_type());
    const ilpm_heads ho = heads_of(out, "out", rows, c.head_dim);
    at::Tensor lse;
    if (given(args[13])) lse = tensor(args[13], "lse");
    else if (bool_arg(args[14])) lse = empty({rows, hq.heads}, at::kFloat);
    if (lse.defined() && (lse.dim() != 2 || lse.size(0) != rows || lse.size(1) != hq.heads)) value_error("lse must be " + sizes({rows, hq.heads}));
    ilpm_tree_options o = {};
    o.scale = given(args[6]) ? float_arg(args[6]) : (float)(1.0 / std::sqrt((double)c.head_dim));
    o.window = int_arg(args[7], "window");
    o.sinks = int_arg(args[8], "sinks");
    o.softcap = float_arg(args[9]);
    o.max_len = int_arg(args[11], "max_len");
    if (given(args[10])) {
        const at::Tensor &mask = tensor(args[10], "mask");
        if (mask.scalar_type() != at::kBool && mask.scalar_type() != at::kByte) type_error("mask must be a bool or uint8 CUDA tensor");
        if (mask.dim() != 2 || mask.size(0) != c.n_seqs || !last_contiguous(mask))
            value_error("mask must be " + sizes({c.n_seqs, -1}) + ", [n_seqs, keys], with its last dimension contiguous");
        // (A mask of no columns has no memory, and still hides every key: it is never read then.)
        o.mask = (const uint8_t *)(mask.data_ptr() ? mask.data_ptr() : lengths.data_ptr());
        o.mask_stride = mask.stride(0);
        o.mask_len = size_arg(mask.size(1), "mask");
    }
    size_t need = 0;
    int rc = ilpm_attn_tree_workspace_size(&c, hq.heads, nodes, o.window, o.sinks, o.max_len, &need);
    if (rc != ILPM_OK) return PyLong_FromLong(rc);
    const at::Tensor ws = workspace_of(args[15], need);
    rc = ilpm_attn_tree(&c, &hq, lengths_p, parents_p, nodes, &o, &ho, lse.defined() ? (float *)floats_of(lse, "lse") : nullptr,
                        ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? ws.nbytes() : 0, current_stream());
    if (rc != ILPM_OK) return PyLong_FromLong(rc);
    if (!lse.defined()) return THPVariable_Wrap(out);
    THPObjectPtr a(THPVariable_Wrap(out)), b(THPVariable_Wrap(lse));
    return a && b ? PyTuple_Pack(2, a.get(), b.get()) : nullptr;
    END_HANDLE_TH_ERRORS
}

// (k_pages, v_pages, page_table, q_heads, nodes, window, sinks, max_len) -> bytes, or a negative status
PyObject *attn_tree_workspace_size(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    count(n_args, 8);
    const ilpm_kv_cache c = cache_of(args[0], args[1], args[2]);
    size_t need = 0;
    const int rc = ilpm_attn_tree_workspace_size(&c, int_arg(args[3], "q_heads"), int_arg(args[4], "nodes"), int_arg(args[5], "window"),
                                                 int_arg(args[6], "sinks"), int_arg(args[7], "max_len"), &need);
    return rc == ILPM_OK ? PyLong_FromSize_t(need) : PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// (tokens, parents, target, uniforms, draft, path, counts, next_tokens, workspace) -> (path, counts, next_tokens)
PyObject *verify_drafts(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    count(n_args, 9);
    const at::Tensor &tokens = tensor(args[0], "tokens"), &parents = tensor(args[1], "parents"), &target = tensor(args[2], "target");
    const at::Tensor &uniforms = tensor(args[3], "uniforms");
    ilpm_verify_args v = {};
    v.tokens = ints_of(tokens, "tokens", 2);
    v.parents = ints_of(parents, "parents", 2);
    const int64_t n = tokens.size(0), t = tokens.size(1);
    if (parents.sizes() != tokens.sizes() || !parents.is_contiguous() || !tokens.is_contiguous())
        value_error("tokens and parents must both be contiguous, [n_seqs, n_nodes]");
    if (uniforms.sizes() != tokens.sizes()) value_error("uniforms must be " + sizes({n, t}));
    v.uniforms = floats_of(uniforms, "uniforms");
    auto rows = [&](const at::Tensor &p, const char *name) {
        if (p.dim() != 3 || p.size(0) != n || p.size(1) != t || !last_contiguous(p))
            value_error(std::string(name) + " must be " + sizes({n, t, -1}) + ", [n_seqs, n_nodes, vocab], with its last dimension contiguous");
    };
    rows(target, "target");
    v.target = target.data_ptr();
    v.target_seq_stride = target.stride(0);
    v.target_node_stride = target.stride(1);
    v.dtype = dtype_of(target, "target");
    v.n_seqs = size_arg(n, "n_seqs");
    v.n_nodes = size_arg(t, "n_nodes");
    v.vocab = size_arg(target.size(2), "vocab");
    if (given(args[4])) {
        const at::Tensor &draft = tensor(args[4], "draft");
        rows(draft, "draft");
        if (draft.size(2) != target.size(2) || draft.scalar_type() != target.scalar_type()) value_error("draft must be of target's sizes and type");
        v.draft = draft.data_ptr();
        v.draft_seq_stride = draft.stride(0);
        v.draft_node_stride = draft.stride(1);
    }
    auto output = [&](PyObject *o, const char *name, at::IntArrayRef shape) {
        if (!given(o)) return empty(shape, at::kInt);
        const at::Tensor &p = tensor(o, name);
        if (p.scalar_type() != at::kInt || p.sizes() != shape || !p.is_contiguous()) type_error(std::string(name) + " must be a contiguous int32 CUDA tensor of its shape");
        return p;
    };
    const at::Tensor path = output(args[5], "path", {n, t}), counts = output(args[6], "counts", {n}), next = output(args[7], "next_tokens", {n});
    v.path = (int32_t *)path.data_ptr();
    v.counts = (int32_t *)counts.data_ptr();
    v.next_tokens = (int32_t *)next.data_ptr();
    size_t need = 0;
    int rc = ilpm_verify_drafts_workspace_size(v.n_seqs, v.n_nodes, v.vocab, &need);
    if (rc != ILPM_OK) return PyLong_FromLong(rc);
    const at::Tensor ws = workspace_of(args[8], need);
    rc = ilpm_verify_drafts(&v, ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? ws.nbytes() : 0, current_stream());
    if (rc != ILPM_OK) return PyLong_FromLong(rc);
    THPObjectPtr a(THPVariable_Wrap(path)), b(THPVariable_Wrap(counts)), d(THPVariable_Wrap(next));
    return a && b && d ? PyTuple_Pack(3, a.get(), b.get(), d.get()) : nullptr;
    END_HANDLE_TH_ERRORS
}

// (n_seqs, n_nodes, vocab) -> bytes, or a negative status
PyObject *verify_drafts_workspace_size(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    count(n_args, 3);
    size_t need = 0;
    const int rc = ilpm_verify_drafts_workspace_size(int_arg(args[0], "n_seqs"), int_arg(args[1], "n_nodes"), int_arg(args[2], "vocab"), &need);
    return rc == ILPM_OK ? PyLong_FromSize_t(need) : PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// (k_pages, v_pages, src_table, dst_table, src_start, dst_start, counts, path, max_count) -> None; max_count None: as many
// as the path has, or any number
PyObject *kv_copy(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    count(n_args, 9);
    const ilpm_kv_cache c = cache_of(args[0], args[1], args[2]);
    const at::Tensor &table = tensor(args[3], "dst_table");
    const int32_t *table_p = ints_of(table, "dst_table", 2);
    if (table.size(0) != c.n_seqs) value_error("dst_table must be " + sizes({c.n_seqs, -1}));
    const int wide = size_arg(table.size(1), "dst_table");
    auto row = [&](PyObject *o, const char *name) {
        const at::Tensor &t = tensor(o, name);
        const int32_t *p = ints_of(t, name, 1);
        if (t.size(0) != c.n_seqs) value_error(std::string(name) + " must be " + sizes({c.n_seqs}));
        return p;
    };
    const int32_t *src = row(args[4], "src_start"), *dst = row(args[5], "dst_start"), *counts = row(args[6], "counts"), *path = nullptr;
    int64_t path_stride = 0, max_count = INT_MAX;
    if (given(args[7])) {
        const at::Tensor &t = tensor(args[7], "path");
        path = ints_of(t, "path", 2);
        if (t.size(0) != c.n_seqs) value_error("path must be " + sizes({c.n_seqs, -1}));
        path_stride = t.stride(0);
        max_count = t.size(1);
        if (max_count == 0) return none();
    }
    if (given(args[8])) {
        const int n = int_arg(args[8], "max_count");
        if (path && n > max_count) value_error("max_count is more than the path has");
        max_count = std::min<int64_t>(n, max_count);
    }
    const int rc = ilpm_kv_copy(&c, table_p, table.stride(0), wide, src, dst, counts, path, path_stride, (int)std::min<int64_t>(max_count, INT_MAX), current_stream());
    return rc == ILPM_OK ? none() : PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"kv_append", (PyCFunction)(void (*)())kv_append, METH_FASTCALL, nullptr},
    {"attn_decode", (PyCFunction)(void (*)())attn_decode, METH_FASTCALL, nullptr},
    {"attn_decode_workspace_size", (PyCFunction)(void (*)())attn_decode_workspace_size, METH_FASTCALL, nullptr},
    {"residual_norm", (PyCFunction)(void (*)())residual_norm, METH_FASTCALL, nullptr},
    {"kv_append_norm", (PyCFunction)(void (*)())kv_append_norm, METH_FASTCALL, nullptr},
    {"attn_tree", (PyCFunction)(void (*)())attn_tree, METH_FASTCALL, nullptr},
    {"attn_tree_workspace_size", (PyCFunction)(void (*)())attn_tree_workspace_size, METH_FASTCALL, nullptr},
    {"verify_drafts", (PyCFunction)(void (*)())verify_drafts, METH_FASTCALL, nullptr},
    {"verify_drafts_workspace_size", (PyCFunction)(void (*)())verify_drafts_workspace_size, METH_FASTCALL, nullptr},
    {"kv_copy", (PyCFunction)(void (*)())kv_copy, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }
