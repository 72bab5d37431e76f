"""The operators of a single-token decoder step whose speed this repository answers for.

Between the projections of a decoder layer (1x1 convolutions of a 1x1 map, for one token) lie three operators:

  "append"  kv_append: the new tokens' keys and values go into a paged cache, keys and queries rotated by their
            positions on the way;
  "attn"    attn_decode: attention of one new token a sequence over that cache;
  "norm"    residual_norm: the norm after a block, its gate and residual scale, the residual sum, and the norm before
            the next block.

The plain forms are their formulas in elementary torch operations, in 32 bits, rounded once at the end.  `own` makes
run() call the package's kernels instead, on the same inputs.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6
GOLDEN = 0.6180339887498949


# ---- cases ------------------------------------------------------------------------------------------------------

def _append(name, tokens, seqs, q_heads, kv_heads, dim, rot, pairs, x, cache, page, start, packed):
    case = {"op": "append", "tokens": tokens, "seqs": seqs, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "rot": rot, "pairs": pairs, "x": x, "cache": cache, "page": page, "start": start, "packed": packed}
    return dict(case, name=name) if name else case


def _attn(name, seqs, length, ragged, q_heads, kv_heads, dim, x, cache, page, window=0, softcap=0.0, mask=False):
    case = {"op": "attn", "seqs": seqs, "length": length, "ragged": ragged, "q_heads": q_heads, "kv_heads": kv_heads,
            "dim": dim, "x": x, "cache": cache, "page": page, "window": window, "softcap": softcap, "mask": mask}
    return dict(case, name=name) if name else case


def _norm(name, rows, width, x, y, params, post, pre, gate, bias, scale):
    case = {"op": "norm", "rows": rows, "width": width, "x": x, "y": y, "params": params, "post": post, "pre": pre,
            "gate": gate, "bias": bias, "scale": scale}
    return dict(case, name=name) if name else case


def listed():
    return [
        # One token of a small model whose activations are this library's f32: the call itself is the cost.
        _append("append_one", 1, 1, 8, 2, 64, 64, False, "f32", "bf16", 16, 100, False),
        # One token for each of 64 sequences, straight from a packed projection.
        _append("append_batch", 64, 64, 32, 8, 128, 128, False, "bf16", "bf16", 16, 4000, True),
        # Several prompts of odd lengths at once, an odd head size, rotated in pairs and only in part.
        _append("append_prompts", 4093, 7, 12, 12, 80, 32, True, "f16", "f16", 32, 900, False),
        # A long prompt of a larger model.
        _append("append_long", 16381, 2, 40, 8, 128, 128, False, "bf16", "bf16", 16, 0, True),
        # A single short sequence in f32: latency.
        _attn("attn_short", 1, 77, False, 8, 2, 64, "f32", "f32", 16),
        # One user with a very long cache: work has to be split over its length.
        _attn("attn_one_long", 1, 131071, False, 32, 8, 128, "bf16", "bf16", 16),
        # A serving batch of mixed lengths, empty and one-token slots among them.
        _attn("attn_batch", 64, 8191, True, 32, 8, 128, "bf16", "bf16", 16),
        # A sliding window over an odd head size with a mask, capped scores, every head its own keys.
        _attn("attn_window", 24, 4097, True, 12, 12, 80, "f16", "f16", 32, window=1000, softcap=30.0, mask=True),
        # f32 queries of this library's projections over a 16-bit cache that all heads share.
        _attn("attn_shared", 8, 2049, True, 16, 1, 256, "f32", "bf16", 64),
        # One token's row between two blocks.
        _norm("norm_one", 1, 512, "f32", "f32", "f32", "rms", "rms", "none", False, 1.0),
        # One token for each of 64 sequences: a learned gate for each channel.
        _norm("norm_batch", 64, 4096, "bf16", "bf16", "bf16", "rms", "rms", "vec", False, 0.5),
        # A prompt's rows: f32 residual stream beside 16-bit blocks, a gate for each row, norms with biases.
        _norm("norm_prompt", 16381, 4096, "f32", "bf16", "f32", "layer", "layer", "rows", True, 0.7071),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _draw_once(rng):
    op = rng.choice(("append", "attn", "norm"))
    if op == "norm":
        y = rng.choice(("f32", "f16", "bf16"))
        return _norm(None, _log(rng, 1, 16384), _log(rng, 64, 8192), rng.choice(("f32", y)), y, rng.choice(("f32", y)),
                     rng.choice(("none", "rms", "layer")), rng.choice(("rms", "layer")),
                     rng.choice(("none", "vec", "rows")), rng.random() < 0.3, rng.choice((1.0, 0.5, 0.7071)))
    cache = rng.choice(("f32", "f16", "bf16"))
    x = rng.choice(("f32", cache))
    dim = rng.choice((64, 72, 80, 96, 128, 128, 192, 256))
    kv_heads, group = _log(rng, 1, 16), _log(rng, 1, 16)
    page = rng.choice((1, 16, 16, 17, 32, 64, 128, 256))
    if op == "append":
        tokens = _log(rng, 1, 16384)
        seqs = tokens if tokens <= 256 and rng.random() < 0.5 else min(tokens, _log(rng, 1, 64))
        return _append(None, tokens, seqs, kv_heads * group, kv_heads, dim, rng.choice((dim, dim, dim // 2, 0)),
                       rng.random() < 0.4, x, cache, page, rng.choice((0, _log(rng, 1, 4096))), rng.random() < 0.5)
    return _attn(None, _log(rng, 1, 128), _log(rng, 1, 131072), rng.random() < 0.7, kv_heads * group, kv_heads, dim, x,
                 cache, page, window=rng.choice((0, 0, _log(rng, 1, 8192))), softcap=rng.choice((0.0, 0.0, 30.0)),
                 mask=rng.random() < 0.3)


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0), work(c)["bytes"])
    while True:
        c = _draw_once(rng)
        if 3072 in c.values() or work(c)["bytes"] > most[c["op"]]:
            continue
        # The plain form works on caches padded to the longest, in 32 bits.
        if c["op"] == "attn" and c["seqs"] * c["length"] * c["kv_heads"] * c["dim"] > 1 << 29:
            continue
        if c["op"] == "attn" and c["seqs"] * c["length"] * c["q_heads"] > 1 << 27:
            continue
        return c


def _lengths(case):
    """Tokens of each sequence in the cache: all as long, or spread with an empty and a one-token slot among them."""
    n, top = case["seqs"], case["length"]
    if not case["ragged"]:
        return [top] * n
    got = [top] + [int((top + 1) * ((0.5 + i * GOLDEN) % 1.0)) for i in range(1, n)]
    if n > 4:
        got[2], got[3] = 1, 0
    return got


def _chunks(case):
    """How many new tokens each sequence gets, and where they begin."""
    n, t = case["seqs"], case["tokens"]
    if n == t:
        counts = [1] * n
    else:
        share = [0.1 + (i + 1) * GOLDEN % 1.0 for i in range(n)]
        counts = [1 + int((t - n) * s / sum(share)) for s in share]
        counts[0] += t - sum(counts)
    return counts, [int(case["start"] * ((i + 3) * GOLDEN % 1.0)) for i in range(n)]


# ---- inputs -----------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype)


def _table(lengths, page, seed):
    """A page table whose pages lie in the pool in no order, and the pool's size."""
    need = [-(-n // page) for n in lengths]
    g = torch.Generator()
    g.manual_seed(int(seed))
    order = torch.randperm(sum(need) + 3, generator=g, dtype=torch.int32)
    wide = max(1, max(need))
    table = torch.zeros((len(need), wide), dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return table.cuda(), len(order)


def _prepare_append(case, seed):
    g = _generator(seed)
    t, d, hq, hk = case["tokens"], case["dim"], case["q_heads"], case["kv_heads"]
    x, cache = TYPES[case["x"]], TYPES[case["cache"]]
    counts, start = _chunks(case)
    total = [a + b for a, b in zip(counts, start)]
    table, pages = _table(total, case["page"], seed)
    if case["packed"]:
        qkv = _normal(g, (t, hq + 2 * hk, d), x)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    else:
        q, k, v = _normal(g, (t, hq, d), x), _normal(g, (t, hk, d), x), _normal(g, (t, hk, d), x)
    n, first = torch.tensor(counts), torch.tensor(start)
    seq = torch.repeat_interleave(torch.arange(len(counts)), n)
    begin = torch.cumsum(n, 0) - n
    pos = torch.arange(t) - begin[seq] + first[seq]
    s = {"op": "append", "q": q, "k": k, "v": v, "pairs": case["pairs"], "page_table": table,
         "k_pages": torch.zeros((pages, case["page"], hk, d), device="cuda", dtype=cache),
         "v_pages": torch.zeros((pages, case["page"], hk, d), device="cuda", dtype=cache),
         "seq_ids": seq.to(torch.int32).cuda(), "positions": pos.to(torch.int32).cuda(), "cos": None, "sin": None}
    if case["rot"]:
        half = case["rot"] // 2
        rate = 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
        angle = torch.arange(max(total), dtype=torch.float64)[:, None] * rate
        s["cos"], s["sin"] = angle.cos().float().cuda(), angle.sin().float().cuda()
    return s


def _prepare_attn(case, seed):
    g = _generator(seed)
    lengths = _lengths(case)
    table, pages = _table(lengths, case["page"], seed)
    d, hk, cache = case["dim"], case["kv_heads"], TYPES[case["cache"]]
    s = {"op": "attn", "q": _normal(g, (case["seqs"], case["q_heads"], d), TYPES[case["x"]], 2.0),
         "k_pages": _normal(g, (pages, case["page"], hk, d), cache),
         "v_pages": _normal(g, (pages, case["page"], hk, d), cache),
         "page_table": table, "lengths": torch.tensor(lengths, dtype=torch.int32).cuda(),
         "scale": 1.0 / math.sqrt(d), "window": case["window"], "softcap": case["softcap"], "mask": None}
    if case["mask"]:
        # One key in ten left out; the second sequence's all.
        s["mask"] = torch.rand((case["seqs"], table.shape[1] * case["page"]), generator=g, device="cuda") < 0.9
        if case["seqs"] > 1:
            s["mask"][1] = False
    return s


def _prepare_norm(case, seed):
    g = _generator(seed)
    rows, c, p = case["rows"], case["width"], TYPES[case["params"]]
    s = {"op": "norm", "x": _normal(g, (rows, c), TYPES[case["x"]], 3.0), "y": _normal(g, (rows, c), TYPES[case["y"]]),
         "post": case["post"], "pre": case["pre"], "scale": case["scale"], "gate": None, "post_b": None, "pre_b": None,
         "post_w": _normal(g, (c,), p, 0.1) + 1 if case["post"] != "none" else None, "pre_w": _normal(g, (c,), p, 0.1) + 1}
    if case["gate"] != "none":
        s["gate"] = _normal(g, (c,) if case["gate"] == "vec" else (rows, c), p, 0.5)
    if case["bias"]:
        s["post_b"] = _normal(g, (c,), p, 0.1) if case["post"] != "none" else None
        s["pre_b"] = _normal(g, (c,), p, 0.1)
    return s


def prepare(case, seed):
    return {"append": _prepare_append, "attn": _prepare_attn, "norm": _prepare_norm}[case["op"]](case, seed)


# ---- the plain forms, in 32 bits --------------------------------------------------------------------------------

def _rotated(x, cos, sin, pairs):
    """x [tokens, heads, dim] in 32 bits, its first 2 * cos.shape[-1] values rotated."""
    x = x.float()
    if cos is None:
        return x
    half = cos.shape[-1]
    cos, sin = cos[:, None], sin[:, None]
    if pairs:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, x[..., 2 * half:]), -1)


def _plain_append(s):
    pos = s["positions"].long()
    size = s["k_pages"].shape[1]
    page, slot = s["page_table"][s["seq_ids"].long(), pos // size].long(), pos % size
    cos, sin = (None, None) if s["cos"] is None else (s["cos"][pos], s["sin"][pos])
    s["k_pages"][page, slot] = _rotated(s["k"], cos, sin, s["pairs"]).to(s["k_pages"].dtype)
    s["v_pages"][page, slot] = s["v"].to(s["v_pages"].dtype)
    return {"q": _rotated(s["q"], cos, sin, s["pairs"]).to(s["q"].dtype), "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_attn(s):
    q, table, n = s["q"], s["page_table"].long(), s["lengths"][:, None]
    b, hq, d = q.shape
    size, hk = s["k_pages"].shape[1:3]
    k = s["k_pages"][table].reshape(b, -1, hk, d).float()
    v = s["v_pages"][table].reshape(b, -1, hk, d).float()
    at = torch.arange(table.shape[1] * size, device=q.device)[None]
    seen = at < n
    if s["window"]:
        seen = seen & (at >= n - s["window"])
    if s["mask"] is not None:
        seen = seen & s["mask"]
    score = torch.matmul(q.float().reshape(b, hk, hq // hk, d), k.permute(0, 2, 3, 1)) * s["scale"]
    if s["softcap"]:
        score = s["softcap"] * torch.tanh(score / s["softcap"])
    score = torch.where(seen[:, None, None], score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    v = torch.where(seen[:, :, None, None], v, 0.0)
    out = torch.matmul(p, v.transpose(1, 2)) / torch.where(total == 0, 1.0, total)
    return {"out": out.reshape(b, hq, d).to(q.dtype), "lse": (top + torch.log(total)).reshape(b, hq)}


def _plain_norm_of(v, kind, w, b):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)
    v = v if w is None else v * w.float()
    return v if b is None else v + b.float()


def _plain_norm(s):
    n = s["y"].float()
    if s["post"] != "none":
        n = _plain_norm_of(n, s["post"], s["post_w"], s["post_b"])
    if s["gate"] is not None:
        n = n * s["gate"].float()
    r = s["x"].float() + s["scale"] * n
    return {"r": r.to(s["x"].dtype), "z": _plain_norm_of(r, s["pre"], s["pre_w"], s["pre_b"]).to(s["y"].dtype)}


# ---- one pass ---------------------------------------------------------------------------------------------------

def _own(s):
    import paper_1909_02765_amd as ilpm
    if s["op"] == "append":
        q = ilpm.kv_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["page_table"], s["seq_ids"], s["positions"],
                           q=s["q"], cos=s["cos"], sin=s["sin"], pairs=s["pairs"])
        return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if s["op"] == "attn":
        out, lse = ilpm.attn_decode(s["q"], s["k_pages"], s["v_pages"], s["page_table"], s["lengths"], scale=s["scale"],
                                    window=s["window"], softcap=s["softcap"], mask=s["mask"], return_lse=True)
        return {"out": out, "lse": lse}
    r, z = ilpm.residual_norm(s["x"], s["y"], post=s["post"], post_w=s["post_w"], post_b=s["post_b"], gate=s["gate"],
                              scale=s["scale"], pre=s["pre"], pre_w=s["pre_w"], pre_b=s["pre_b"], eps=EPS)
    return {"r": r, "z": z}


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "attn": _plain_attn, "norm": _plain_norm}[state["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    if case["op"] == "append":
        t, d, hq, hk = case["tokens"], case["dim"], case["q_heads"], case["kv_heads"]
        x, cache = BYTES[case["x"]], BYTES[case["cache"]]
        counts, start = _chunks(case)
        angles = min(t, max(a + b for a, b in zip(counts, start))) * case["rot"] * 4
        return {"bytes": t * d * (hq * 2 * x + hk * 2 * (x + cache)) + angles + 8 * t,
                "flops": 3 * t * (hq + hk) * case["rot"]}
    if case["op"] == "attn":
        d, hq, hk = case["dim"], case["q_heads"], case["kv_heads"]
        seen = [min(n, case["window"]) if case["window"] else n for n in _lengths(case)]
        masks = sum(seen) if case["mask"] else 0
        if case["mask"] and len(seen) > 1:
            seen[1] = 0
        keys = sum(seen)
        pages = sum(-(-n // case["page"]) for n in seen)
        return {"bytes": keys * hk * d * 2 * BYTES[case["cache"]] + case["seqs"] * hq * (2 * d * BYTES[case["x"]] + 4)
                + 4 * pages + 4 * case["seqs"] + masks,
                "flops": 4 * keys * hq * d}
    rows, c = case["rows"], case["width"]
    p = BYTES[case["params"]]
    vectors = (case["post"] != "none") + 1 + (case["gate"] == "vec") + case["bias"] * ((case["post"] != "none") + 1)
    return {"bytes": rows * c * 2 * (BYTES[case["x"]] + BYTES[case["y"]]) + vectors * c * p
            + (rows * c * p if case["gate"] == "rows" else 0),
            "flops": rows * c * 12}


# ---- the definitions in 64 bits, one sequence, token or row at a time -------------------------------------------

def _exact_append(s):
    keys, values = s["k_pages"].double(), s["v_pages"].double()
    size = keys.shape[1]
    place = torch.div(s["positions"], size, rounding_mode="floor").long()
    flat = s["page_table"].reshape(-1).long()[s["seq_ids"].long() * s["page_table"].shape[1] + place] * size
    flat = flat + s["positions"].long() % size

    def turn(x):
        x = x.double().clone()
        if s["cos"] is None:
            return x
        half = s["cos"].shape[1]
        angle = torch.complex(s["cos"].double(), s["sin"].double())[s["positions"].long()].unsqueeze(1)
        first, second = ((slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if s["pairs"]
                         else (slice(0, half), slice(half, 2 * half)))
        z = torch.complex(x[:, :, first], x[:, :, second]) * angle
        x[:, :, first], x[:, :, second] = z.real, z.imag
        return x

    keys.view(-1, *keys.shape[2:]).index_copy_(0, flat, turn(s["k"]))
    values.view(-1, *values.shape[2:]).index_copy_(0, flat, s["v"].double())
    return {"q": turn(s["q"]), "k_pages": keys, "v_pages": values}


def _exact_attn(s):
    b, hq, d = s["q"].shape
    size, hk = s["k_pages"].shape[1:3]
    out = torch.zeros((b, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((b, hq), -math.inf, dtype=torch.float64, device="cuda")
    for i, n in enumerate(s["lengths"].tolist()):
        first = max(0, n - s["window"]) if s["window"] else 0
        at = torch.arange(first, n, device="cuda")
        if s["mask"] is not None:
            at = at[s["mask"][i, first:n]]
        if not len(at):
            continue
        rows = s["page_table"][i].long()[at // size] * size + at % size
        for h in range(hk):
            k = s["k_pages"].view(-1, hk, d)[rows, h].double()
            v = s["v_pages"].view(-1, hk, d)[rows, h].double()
            heads = slice(h * (hq // hk), (h + 1) * (hq // hk))
            score = s["q"][i, heads].double() @ k.T * s["scale"]
            if s["softcap"]:
                score = torch.tanh(score / s["softcap"]) * s["softcap"]
            lse[i, heads] = torch.logsumexp(score, 1)
            out[i, heads] = torch.exp(score - lse[i, heads, None]) @ v
    return {"out": out, "lse": lse}


def _exact_norm(s):
    def norm(v, kind, w, b):
        mean = v.sum(1, keepdim=True) / v.shape[1] if kind == "layer" else 0.0
        v = (v - mean) * ((v - mean).pow(2).sum(1, keepdim=True) / v.shape[1] + EPS).rsqrt()
        v = v * (1.0 if w is None else w.double())
        return v + (0.0 if b is None else b.double())

    n = s["y"].double() if s["post"] == "none" else norm(s["y"].double(), s["post"], s["post_w"], s["post_b"])
    r = s["x"].double() + s["scale"] * n * (1.0 if s["gate"] is None else s["gate"].double())
    return {"r": r, "z": norm(r, s["pre"], s["pre_w"], s["pre_b"])}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attn, "norm": _exact_norm}[case["op"]](s)
