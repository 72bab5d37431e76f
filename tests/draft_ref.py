"""The operators of a drafted decoder step by their definitions, in 64 bits on
the CPU, with bounds of what 32-bit arithmetic and one rounding may add (see
decode_ref.py for those).  Test infrastructure: it shares no code with the
library."""
import math

import torch

import decode_ref
from decode_ref import E32, TINY, U


def above(parents):
    """For each node of a row of parents the nodes that it sees, itself the last; None where there is no node."""
    got = []
    for i, p in enumerate(parents):
        if p == -1:
            got.append([i])
        elif 0 <= p < i and got[p] is not None:
            got.append(got[p] + [i])
        else:
            got.append(None)
    return got


def norm_rotate(x, positions, norm, w, eps, cos, sin, pairs):
    """(x normed and rotated, bound of its 32-bit error); x [tokens, heads, dim]."""
    x = x.double()
    t, h, d = x.shape
    err = torch.zeros_like(x)
    if norm != "none":
        out, e = decode_ref._norm(x.reshape(t * h, d), torch.zeros((t * h, d), dtype=torch.float64), norm,
                                  None if w is None else w.double(), None, eps)
        x, err = out.view(t, h, d), e.view(t, h, d)
    turned, e = decode_ref.rotate(x, positions, cos, sin, pairs)
    if cos is not None:
        half = cos.shape[1]
        for n, p in enumerate(positions):
            if not 0 <= p < cos.shape[0]:
                continue
            for i in range(half):
                a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
                c, s = abs(float(cos[p, i])), abs(float(sin[p, i]))
                # What came in is off by err, and so its products' roundings by as much of it.
                u, v = err[n, :, a].clone(), err[n, :, b].clone()
                e[n, :, a] += (c * u + s * v) * (1 + 4 * E32)
                e[n, :, b] += (c * v + s * u) * (1 + 4 * E32)
        keep = torch.ones(x.shape, dtype=torch.bool)
        for n, p in enumerate(positions):
            if 0 <= p < cos.shape[0]:
                keep[n, :, :2 * half] = False
        e = torch.where(keep, err, e)
    else:
        e = err
    return turned, e


def append(k, v, k_pages, v_pages, table, seq_ids, positions, slots, norm, k_w, eps, cos, sin, pairs):
    """(keys, their bound, values, which slots are written) of the pools after the call, in double."""
    keys, values = k_pages.double().clone(), v_pages.double().clone()
    err = torch.zeros_like(keys)
    new, e = norm_rotate(k, positions, norm, k_w, eps, cos, sin, pairs)
    n_pages, size = k_pages.shape[:2]
    written = torch.zeros(k_pages.shape[:2], dtype=torch.bool)
    for t, (s, p, at) in enumerate(zip(seq_ids, positions, slots)):
        if not 0 <= s < table.shape[0] or at < 0 or at // size >= table.shape[1]:
            continue
        page = int(table[s, at // size])
        if not 0 <= page < n_pages or (cos is not None and not 0 <= p < cos.shape[0]):
            continue
        keys[page, at % size], err[page, at % size] = new[t], e[t]
        values[page, at % size] = v[t].double()
        written[page, at % size] = True
    return keys, err, values, written


def seen_keys(n_pages, size, table, length, s, tree, node, nodes, window, sinks, mask):
    """The (page, slot) that a node of sequence s sees."""
    length = max(length, 0)
    if tree[node] is None:
        return []
    place = length + len(tree[node]) - 1
    keys = [(j, j) for j in range(length)] if length < 1 << 20 else []
    keys += [(length + a, length + len(tree[a]) - 1) for a in tree[node]]
    got = []
    for j, at in keys:
        if j >= table.shape[1] * size:
            continue
        if window and at <= place - window and at >= sinks:
            continue
        if mask is not None and (j >= mask.shape[1] or not mask[s, j]):
            continue
        page = int(table[s, j // size])
        if 0 <= page < n_pages:
            got.append((page, j % size))
    return got


def attention(q, k_pages, v_pages, table, lengths, parents, scale, window=0, sinks=0, softcap=0.0, mask=None):
    """(out, lse, bound of out, bound of lse) in double, for outputs of q's type; q [n_seqs * nodes, heads, dim]."""
    b, t = parents.shape
    rows, hq, d = q.shape
    hk = k_pages.shape[2]
    group = hq // hk
    out = torch.zeros((rows, hq, d), dtype=torch.float64)
    lse = torch.full((rows, hq), -math.inf, dtype=torch.float64)
    e_out, e_lse = torch.zeros_like(out), torch.zeros_like(lse)
    # Probabilities are held in parts: to 2^-17 of each under 16-bit queries, else to 2^-23 (the bounds are doubled below).
    held = 2.0 ** -23 if q.dtype == torch.float32 else 2.0 ** -17
    for s in range(b):
        tree = above([int(p) for p in parents[s]])
        for i in range(t):
            at = seen_keys(k_pages.shape[0], k_pages.shape[1], table, int(lengths[s]), s, tree, i, t, window, sinks, mask)
            if not at:
                continue
            pages, slots = torch.tensor([p for p, _ in at]), torch.tensor([j for _, j in at])
            k = k_pages[pages, slots].double().transpose(0, 1).repeat_interleave(group, 0)  # [heads, keys, dim]
            v = v_pages[pages, slots].double().transpose(0, 1).repeat_interleave(group, 0)
            qs = q[s * t + i].double()[:, :, None]
            x = (k @ qs)[..., 0] * scale
            # A dot product of d terms, the scale and the logarithm's base.
            dx = (d + 6) * E32 * (k.abs() @ qs.abs())[..., 0] * abs(scale)
            if softcap:
                x = softcap * torch.tanh(x / softcap)
                dx = dx + 8 * E32 * softcap
            m = x.amax(1, keepdim=True)
            p = torch.exp(x - m)
            total = p.sum(1, keepdim=True)
            r = s * t + i
            out[r] = (p[:, None] @ v)[:, 0] / total
            lse[r] = (m + torch.log(total))[:, 0]
            # A probability is off by what its score and the maximum's are, by the subtraction from it, and by the
            # exponential's own rounding.
            rel = 2 * dx.amax(1, keepdim=True) + 4 * E32 * ((x - m).abs().amax(1, keepdim=True) + m.abs()) + 8 * E32
            sums = (len(at) + 300) * E32
            e_out[r] = 2 * (rel + sums + held) * (p[:, None] @ v.abs())[:, 0] / total
            e_lse[r] = (rel + sums)[:, 0] + 4 * E32 * lse[r].abs()
    e_out = e_out + U[q.dtype] * (out.abs() + e_out) + TINY[q.dtype]
    return out, lse, e_out, e_lse


def verify(tokens, parents, target, uniforms, draft=None):
    """(path, counts, next tokens) as lists, by the walk's definition, a row at a time."""
    n, t = tokens.shape
    vocab = target.shape[2]

    def row(p):
        p = p.double()
        return torch.where(p > 0, p, 0.0).clamp(max=torch.finfo(torch.float32).max)

    paths, counts, last = [], [], []
    for s in range(n):
        tree = [int(p) for p in parents[s]]
        if tree[0] != -1:
            paths.append([-1] * t)
            counts.append(0)
            last.append(-1)
            continue
        way, cur = [0], 0
        while True:
            p = row(target[s, cur])
            q = None if draft is None else row(draft[s, cur])
            w, z, kept = p.clone(), 1.0, None
            for c in range(cur + 1, t):
                x = int(tokens[s, c])
                if tree[c] != cur or not 0 <= x < vocab or not z > 0:
                    continue
                u = float(uniforms[s, c])
                if (u * z if q is None else u * float(q[x]) * z) < float(w[x]):
                    kept = c
                    break
                if q is None:
                    z -= float(w[x])
                    w[x] = 0.0
                else:
                    w = (w / z - q).clamp(min=0)
                    z = float(w.sum())
            if kept is None:
                break
            way.append(kept)
            cur = kept
        if not float(w.sum()) > 0:
            w = p
        sums = w.cumsum(0)
        passed = (sums > float(uniforms[s, 0]) * sums[-1]) & (w > 0)
        if passed.any():
            last.append(int(passed.nonzero()[0]))
        else:
            last.append(int((w > 0).nonzero()[-1]) if (w > 0).any() else -1)
        paths.append(way + [-1] * (t - len(way)))
        counts.append(len(way))
    return paths, counts, last


def copy(pool, src_table, dst_table, src_start, dst_start, counts, path, max_count):
    """The pool after the call; the one given is not changed."""
    n_pages, size = pool.shape[:2]
    new = pool.clone()

    def place(table, s, token):
        if token < 0 or token // size >= table.shape[1] or not 0 <= int(table[s, token // size]) < n_pages:
            return None
        return int(table[s, token // size]), token % size

    for s in range(src_table.shape[0]):
        for i in range(min(int(counts[s]), max_count)):
            step = i if path is None else int(path[s, i])
            if step < 0:
                continue
            a, b = place(src_table, s, int(src_start[s]) + step), place(dst_table, s, int(dst_start[s]) + i)
            if a is not None and b is not None:
                new[b] = pool[a]
    return new
