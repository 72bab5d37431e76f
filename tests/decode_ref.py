"""The decoder-step operators by their definitions, in 64 bits on the CPU, with
bounds of what 32-bit arithmetic and one rounding may add.  Test
infrastructure: it shares no code with the library.

Rounding to a type with p bits of significand moves a value by at most 2^-p of
it (U), and by half its smallest step near 0 (TINY).  A 32-bit sum of n terms,
in any order, is off by at most n * 2^-24 of the sum of their magnitudes."""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}
E32 = 2.0 ** -24


def rotate(x, positions, cos, sin, pairs):
    """(rotated x, bound of its 32-bit error); x [tokens, heads, dim] double."""
    out, err = x.clone(), torch.zeros_like(x)
    if cos is None:
        return out, err
    half = cos.shape[1]
    for t, p in enumerate(positions):
        if not 0 <= p < cos.shape[0]:
            continue
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
            c, s = float(cos[p, i]), float(sin[p, i])
            u, v = x[t, :, a], x[t, :, b]
            out[t, :, a], out[t, :, b] = u * c - v * s, v * c + u * s
            # Two products and a sum, each rounded.
            err[t, :, a] = err[t, :, b] = 2 * E32 * (u.abs() + v.abs())
    return out, err


def append(k, v, k_pages, v_pages, table, seq_ids, positions, cos, sin, pairs):
    """(keys, their bound, values) of the pools after the call, in double; the
    pools given are not changed."""
    keys, values = k_pages.double().clone(), v_pages.double().clone()
    err = torch.zeros_like(keys)
    rot, rot_err = rotate(k.double(), positions, cos, sin, pairs)
    n_pages, size = k_pages.shape[:2]
    for t, (s, p) in enumerate(zip(seq_ids, positions)):
        if not 0 <= s < table.shape[0] or p < 0 or p // size >= table.shape[1]:
            continue
        page = int(table[s, p // size])
        if not 0 <= page < n_pages or (cos is not None and p >= cos.shape[0]):
            continue
        keys[page, p % size], err[page, p % size] = rot[t], rot_err[t]
        values[page, p % size] = v[t].double()
    return keys, err, values


def seen_keys(n_pages, size, table, length, s, window, mask):
    """The tokens that a new token of sequence s sees: [(token, page, slot)]."""
    got = []
    for j in range(max(0, min(length, table.shape[1] * size))):
        page = int(table[s, j // size])
        if window and j < length - window:
            continue
        if mask is not None and (j >= mask.shape[1] or not mask[s, j]):
            continue
        if 0 <= page < n_pages:
            got.append((j, page, j % size))
    return got


def attention(q, k_pages, v_pages, table, lengths, scale, window=0, softcap=0.0, mask=None):
    """(out, lse, bound of out, bound of lse) in double, for outputs of q's type."""
    b, hq, d = q.shape
    hk = k_pages.shape[2]
    group = hq // hk
    out = torch.zeros((b, hq, d), dtype=torch.float64)
    lse = torch.full((b, hq), -math.inf, dtype=torch.float64)
    e_out, e_lse = torch.zeros_like(out), torch.zeros_like(lse)
    # Probabilities of 16-bit queries may be held in two 16-bit parts (2^-16 of each).
    held = 0.0 if q.dtype == torch.float32 else 2.0 ** -16
    for s in range(b):
        at = seen_keys(k_pages.shape[0], k_pages.shape[1], table, int(lengths[s]), s, window, mask)
        if not at:
            continue
        pages, slots = torch.tensor([p for _, p, _ in at]), torch.tensor([i for _, _, i in at])
        for h in range(hq):
            k = k_pages[pages, slots, h // group].double()
            v = v_pages[pages, slots, h // group].double()
            qs = q[s, h].double()
            x = (k @ qs) * scale
            # A dot product of d terms, the scale and the logarithm's base.
            dx = (d + 6) * E32 * (k.abs() @ qs.abs()) * abs(scale)
            if softcap:
                x = softcap * torch.tanh(x / softcap)
                dx = dx + 8 * E32 * softcap
            m = x.max()
            p = torch.exp(x - m)
            total = p.sum()
            out[s, h] = (p @ v) / total
            lse[s, h] = m + torch.log(total)
            # A probability is off by what its score and the maximum's are, by
            # the subtraction from it, and by the exponential's own rounding.
            rel = 2 * dx.max() + 4 * E32 * ((x - m).abs().max() + m.abs()) + 8 * E32
            sums = (len(at) + 300) * E32
            e_out[s, h] = 2 * (rel + sums + held) * (p @ v.abs()) / total
            e_lse[s, h] = rel + sums + 4 * E32 * lse[s, h].abs()
    e_out = e_out + U[q.dtype] * (out.abs() + e_out) + TINY[q.dtype]
    return out, lse, e_out, e_lse


def _norm(v, ev, kind, w, b, eps):
    """(norm of the rows v, bound), where v itself is off by up to ev."""
    n = v.shape[1]
    sums = (n + 8) * E32
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    e_mean = sums * v.abs().mean(1, keepdim=True) + ev.mean(1, keepdim=True) if kind == "layer" else mean
    dev = v - mean
    e_dev = ev + e_mean + E32 * (v.abs() + mean.abs())
    var = (dev * dev).mean(1, keepdim=True) + eps
    e_var = (2 * dev.abs() * e_dev + e_dev * e_dev).mean(1, keepdim=True) + (sums + 4 * E32) * var
    out = dev / var.sqrt()
    # 1/sqrt moves by at most half the variance's relative error, over what is left of the variance.
    share = e_var / (var - e_var).clamp_min(1e-300)
    err = e_dev / var.sqrt() * (1 + share) + out.abs() * (0.5 * share + 6 * E32)
    if w is not None:
        out, err = out * w, err * w.abs() + 2 * E32 * (out * w).abs()
    if b is not None:
        out, err = out + b, err + 2 * E32 * (out.abs() + b.abs())
    return out, err


def residual_norm(x, y, post, post_w, post_b, gate, scale, pre, pre_w, pre_b, eps, x_dtype, y_dtype):
    """(r, z, bound of r, bound of z) in double, for outputs of these types."""
    dbl = [None if t is None else t.double() for t in (x, y, post_w, post_b, gate, pre_w, pre_b)]
    x, y, post_w, post_b, gate, pre_w, pre_b = dbl
    r, er = x, torch.zeros_like(x)
    if y is not None:
        n, en = y, torch.zeros_like(y)
        if post in ("rms", "layer"):
            n, en = _norm(y, en, post, post_w, post_b, eps)
        if gate is not None:
            n, en = n * gate, en * gate.abs() + E32 * (n * gate).abs()
        n, en = n * scale, en * abs(scale) + 2 * E32 * (n * scale).abs()
        r, er = x + n, en + 2 * E32 * (x.abs() + n.abs() + en)
    z = ez = None
    if pre in ("rms", "layer"):
        z, ez = _norm(r, er, pre, pre_w, pre_b, eps)
        ez = ez + U[y_dtype] * (z.abs() + ez) + TINY[y_dtype]
    er = er + U[x_dtype] * (r.abs() + er) + TINY[x_dtype]
    return r, z, er, ez
