"""GPU: the operators of a drafted decoder step (kv_append_norm, attn_tree,
verify_drafts, kv_copy) against their 64-bit definitions in draft_ref.py, within
the bounds derived there: types, head layouts, trees, lengths from zero on, odd
sizes, strides, masks that leave rows empty, and cache contents that must not
matter."""
import math

import pytest
import torch

import draft_ref as ref
from decode_ref import TINY, U
from gpu_common import note, torch_cuda

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
PAIRS = [(F32, F32), (F16, F16), (BF16, BF16), (F32, F16), (F32, BF16)]


def lib():
    torch_cuda()
    import paper_1909_02765_amd as ilpm
    return ilpm


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g) * std).to(dtype)


def ints(v):
    return torch.tensor(v, dtype=torch.int32)


def near(got, want, err, what):
    got = got.double().cpu()
    off = (got - want).abs()
    bad = ~(off <= err) & ~(got == want)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} outside, the worst {off[bad].max()} "
                           f"where {err[bad][off[bad].argmax()]} is allowed")


# ---- kv_append_norm ----

def append_case(g, tokens, seqs, hq, hk, d, rot, x, cache, page, max_pages, norm, params=None):
    n_pages = seqs * max_pages + 2
    table = torch.randperm(n_pages, generator=g)[:seqs * max_pages].view(seqs, max_pages).to(torch.int32)
    spots = torch.randperm(seqs * max_pages * page, generator=g)[:tokens]
    seq, slots = spots // (max_pages * page), spots % (max_pages * page)
    most = max_pages * page + 5
    pos = torch.randint(0, most, (tokens,), generator=g)
    angle = torch.rand((most, rot // 2), generator=g) * 6.3
    w = None if norm == "none" else randn(g, (2, d), params or x, 0.2) + 1
    return dict(q=randn(g, (tokens, hq, d), x, 2.0), k=randn(g, (tokens, hk, d), x, 2.0), v=randn(g, (tokens, hk, d), x),
                kp=randn(g, (n_pages, page, hk, d), cache), vp=randn(g, (n_pages, page, hk, d), cache), table=table,
                seq=seq.to(torch.int32), pos=pos.to(torch.int32), slots=slots.to(torch.int32),
                cos=angle.cos() if rot else None, sin=angle.sin() if rot else None,
                q_w=None if w is None else w[0].contiguous(), k_w=None if w is None else w[1].contiguous())


def check_append(c, norm, pairs, what, cuda=None, q_out=None, eps=1e-5, stream=None):
    """Runs the call on `cuda` (the case's tensors there, or others of the same values) and checks all that it wrote."""
    ilpm = lib()
    note(f"[append] {what}")
    t = {k: (v.cuda() if v is not None else None) for k, v in c.items()}
    t.update(cuda or {})
    got = ilpm.kv_append_norm(t["k"], t["v"], t["kp"], t["vp"], t["table"], t["seq"], t["pos"], slots=t["slots"], q=t["q"],
                              norm=norm, q_w=t["q_w"] if t["q"] is not None else None, k_w=t["k_w"], eps=eps, cos=t["cos"],
                              sin=t["sin"], pairs=pairs, q_out=q_out, stream=stream)
    torch.cuda.synchronize()
    pos = c["pos"].tolist()
    keys, err, values, written = ref.append(c["k"], c["v"], c["kp"], c["vp"], c["table"], c["seq"].tolist(), pos,
                                            (c["pos"] if c["slots"] is None else c["slots"]).tolist(), norm, c["k_w"], eps,
                                            c["cos"], c["sin"], pairs)
    written = written[:, :, None, None]
    u, tiny = U[c["kp"].dtype], TINY[c["kp"].dtype]
    near(t["kp"], keys, torch.where(written, err + u * (keys.abs() + err) + tiny, 0.0), what + " keys")
    near(t["vp"], values, torch.where(written, u * values.abs() + tiny, 0.0), what + " values")
    if c["q"] is not None:
        want, err = ref.norm_rotate(c["q"], pos, norm, c["q_w"], eps, c["cos"], c["sin"], pairs)
        u, tiny = U[c["q"].dtype], TINY[c["q"].dtype]
        near(got, want, torch.where(err > 0, err + u * (want.abs() + err) + tiny, 0.0), what + " queries")


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("tokens,seqs,hq,hk,d,rot,page", [
    (1, 1, 1, 1, 2, 2, 1), (1, 1, 8, 2, 64, 64, 16), (5, 3, 6, 3, 80, 32, 17), (33, 4, 5, 5, 7, 6, 3),
    (64, 64, 32, 8, 128, 128, 16), (50, 2, 7, 1, 256, 128, 32), (9, 2, 4, 4, 72, 0, 16), (17, 3, 3, 2, 96, 96, 64)])
@pytest.mark.parametrize("norm,pairs", [("rms", False), ("layer", True), ("none", False), ("rms", True)])
def test_append(x, cache, tokens, seqs, hq, hk, d, rot, page, norm, pairs):
    c = append_case(gen(tokens * 1000 + d), tokens, seqs, hq, hk, d, rot, x, cache, page, -(-2 * tokens // (seqs * page)) + 1, norm)
    check_append(c, norm, pairs, f"{x}->{cache} {tokens}x({hq},{hk})x{d} rot {rot} page {page} {norm} pairs {pairs}")


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("pairs", [False, True])
def test_append_heads_that_do_not_divide(x, cache, pairs):
    """Heads of every remainder to a multiple of eight, what turns of them and what does not: copied and in place."""
    g = gen(17)
    for d, rot in [(d, rot) for d in (1, 3, 8, 9, 15, 21, 36, 75) for rot in range(0, d + 1, 2)]:
        c = append_case(g, 5, 2, 3, 1, d, rot, x, cache, 16, 2, "layer")
        check_append(c, "layer", pairs, f"d {d} rot {rot}")
        if rot and rot % 6 == 0:
            q = c["q"].cuda()
            check_append(c, "layer", pairs, f"d {d} rot {rot} in place", cuda=dict(q=q), q_out=q)


@pytest.mark.parametrize("d,rot", [(300, 100), (512, 512), (1000, 1000), (1024, 64), (1023, 0), (255, 2), (257, 256)])
@pytest.mark.parametrize("x,cache", [(F32, F32), (BF16, BF16), (F32, F16)], ids=str)
def test_append_large_heads(x, cache, d, rot):
    c = append_case(gen(d), 7, 2, 3, 2, d, rot, x, cache, 4, 3, "rms")
    check_append(c, "rms", False, f"d {d} rot {rot}")
    c = append_case(gen(d), 7, 2, 3, 2, d, rot, x, cache, 4, 3, "layer")
    q = c["q"].cuda()
    check_append(c, "layer", True, f"d {d} rot {rot} in place", cuda=dict(q=q), q_out=q)


@pytest.mark.parametrize("x", [F16, BF16], ids=str)
def test_append_weights_of_32_bits_or_none(x):
    c = append_case(gen(3), 9, 2, 4, 2, 64, 64, x, x, 16, 2, "rms", params=F32)
    check_append(c, "rms", False, "weights of 32 bits")
    c["q_w"] = None
    check_append(c, "rms", False, "a weight of keys only")
    c["k_w"] = None
    check_append(c, "layer", False, "no weights")


def test_append_without_queries_and_many_tokens():
    for d, rot in ((128, 128), (64, 32)):
        c = append_case(gen(d), 4000, 3, 2, 2, d, rot, BF16, BF16, 16, 100, "rms")
        c["q"] = None
        check_append(c, "rms", False, f"no queries, d {d}")


def test_append_by_positions():
    """Without slots tokens lie at their positions, and unnormed the call is kv_append."""
    ilpm = lib()
    c = append_case(gen(8), 40, 2, 6, 2, 128, 128, BF16, BF16, 16, 3, "none")
    c["pos"], c["slots"] = c["slots"], None
    check_append(c, "none", False, "by positions")
    t = {k: v.cuda() if v is not None else None for k, v in c.items()}
    kp, vp = t["kp"].clone(), t["vp"].clone()
    a = ilpm.kv_append(t["k"], t["v"], kp, vp, t["table"], t["seq"], t["pos"], q=t["q"], cos=t["cos"], sin=t["sin"])
    b = ilpm.kv_append_norm(t["k"], t["v"], t["kp"], t["vp"], t["table"], t["seq"], t["pos"], q=t["q"], norm=None, cos=t["cos"], sin=t["sin"])
    assert torch.equal(a, b) and torch.equal(kp, t["kp"]) and torch.equal(vp, t["vp"])


@pytest.mark.parametrize("pairs", [False, True])
def test_append_strided(pairs):
    """Slices of one packed projection, queries in place in it, pools with the heads outside the slots and keys and values
    in one allocation, and everything one element off its alignment."""
    g = gen(11)
    for d, shift in ((128, 0), (64, 1), (36, 0), (80, 3)):
        c = append_case(g, 37, 2, 6, 2, d, d // 2 * 2, BF16, BF16, 16, 3, "rms")
        packed = torch.empty(37 * 10 * d + shift, dtype=BF16)[shift:].view(37, 10, d)
        packed[:, :6], packed[:, 6:8], packed[:, 8:] = c["q"], c["k"], c["v"]
        gpu = torch.empty(37 * 10 * d + shift, dtype=BF16, device="cuda")[shift:].view(37, 10, d)
        gpu.copy_(packed)
        n = c["kp"].shape[0]
        pools = torch.empty((n, 2, 2, 16, d), dtype=BF16, device="cuda")   # [page][k or v][head][slot][d]
        kp, vp = pools[:, 0].transpose(1, 2), pools[:, 1].transpose(1, 2)
        kp.copy_(c["kp"])
        vp.copy_(c["vp"])
        w = torch.empty(2 * d + shift, dtype=BF16, device="cuda")[shift:]
        w[:d], w[d:] = c["q_w"].cuda(), c["k_w"].cuda()
        cuda = dict(q=gpu[:, :6], k=gpu[:, 6:8], v=gpu[:, 8:], kp=kp, vp=vp, q_w=w[:d], k_w=w[d:])
        check_append(c, "rms", pairs, f"strided d {d} shift {shift}", cuda, q_out=gpu[:, :6])
        assert torch.equal(gpu[:, 6:].cpu(), packed[:, 6:])


def test_append_leaves_out_what_names_no_place():
    c = append_case(gen(5), 14, 3, 4, 2, 64, 64, F32, BF16, 16, 2, "rms")
    c["seq"][:4] = ints([-1, 3, -2 ** 31, 2 ** 31 - 1])
    c["slots"][4:9] = ints([-1, 32, 2 ** 31 - 1, -2 ** 31, 33])
    c["table"][int(c["seq"][9]), int(c["slots"][9]) // 16] = -1
    c["table"][int(c["seq"][10]), int(c["slots"][10]) // 16] = c["kp"].shape[0]
    c["pos"][11:] = ints([-1, 2 ** 31 - 1, -2 ** 31])   # no angle: queries are normed only
    check_append(c, "rms", False, "no place")
    c["cos"], c["sin"] = c["cos"][:5], c["sin"][:5]     # positions beyond the table of angles
    check_append(c, "rms", False, "no angle")


def test_append_nothing():
    ilpm = lib()
    c = append_case(gen(1), 2, 1, 1, 1, 64, 64, F32, F32, 16, 1, "rms")
    t = {k: v.cuda() for k, v in c.items()}
    before = t["kp"].clone()
    q = ilpm.kv_append_norm(t["k"][:0], t["v"][:0], t["kp"], t["vp"], t["table"], t["seq"][:0], t["pos"][:0], q=t["q"][:0])
    assert q.shape == (0, 1, 64) and torch.equal(t["kp"], before)
    assert ilpm.kv_append_norm(t["k"], t["v"], t["kp"][:0], t["vp"][:0], t["table"], t["seq"], t["pos"]) is None


def test_append_is_not_the_norm_of_what_is_not_finite():
    """NaN and infinity stay in their own head."""
    ilpm = lib()
    c = append_case(gen(2), 6, 2, 4, 2, 64, 64, F32, F32, 16, 2, "rms")
    c["q"][1, 2, 5], c["k"][3, 0, 7], c["v"][2, 1, 3] = math.nan, math.inf, math.inf
    t = {k: v.cuda() for k, v in c.items()}
    q = ilpm.kv_append_norm(t["k"], t["v"], t["kp"], t["vp"], t["table"], t["seq"], t["pos"], slots=t["slots"], q=t["q"],
                            q_w=t["q_w"], k_w=t["k_w"], cos=t["cos"], sin=t["sin"]).cpu()
    odd = ~torch.isfinite(q).all(-1)
    assert odd[1, 2] and int(odd.sum()) == 1
    assert int((~torch.isfinite(t["kp"]).all(-1)).sum()) == 1 and int(torch.isinf(t["vp"]).sum()) == 1


# ---- attn_tree ----

def chain(n):
    return list(range(-1, n - 1))


def some_tree(g, n):
    """Any tree or trees, with what is no node among them and after them."""
    got = []
    for i in range(n):
        r = float(torch.rand((), generator=g))
        got.append(-1 if i == 0 or r < 0.08 else -2 if r < 0.12 else i + 1 if r < 0.15 else int(torch.randint(max(0, i - 6), i, (), generator=g)))
    return got


def attn_case(g, lengths, parents, hq, hk, d, x, cache, page, extra=0):
    nodes = len(parents[0])
    need = [-(-(max(n, 0) + nodes) // page) for n in lengths]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.full((len(lengths), max(1, max(need)) + extra), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return dict(q=randn(g, (len(lengths) * nodes, hq, d), x, 2.0), kp=randn(g, (n_pages, page, hk, d), cache),
                vp=randn(g, (n_pages, page, hk, d), cache), table=table, lengths=ints(lengths), parents=ints(parents))


def hide_unseen(c, **kw):
    """NaN in all that no node may see: slots of no key, other pages."""
    seen = torch.zeros(c["kp"].shape[:2], dtype=torch.bool)
    for s, row in enumerate(c["parents"].tolist()):
        tree = ref.above(row)
        for i in range(len(row)):
            for p, j in ref.seen_keys(c["kp"].shape[0], c["kp"].shape[1], c["table"], int(c["lengths"][s]), s, tree, i, len(row),
                                      kw.get("window", 0), kw.get("sinks", 0), kw.get("mask")):
                seen[p, j] = True
    # (What only some nodes see is finite: its weight is 0 for the others.)
    c["kp"][~seen] = math.nan
    c["vp"][~seen] = math.nan


def check_attn(c, what, cuda=None, stream=None, **kw):
    ilpm = lib()
    note(f"[attn_tree] {what}")
    t = {k: v.cuda() for k, v in c.items()}
    t.update(cuda or {})
    call = dict(kw)
    if call.get("mask") is not None:
        call["mask"] = call["mask"].cuda()
    scale = kw.get("scale", c["q"].shape[2] ** -0.5)
    got, lse = ilpm.attn_tree(t["q"], t["kp"], t["vp"], t["table"], t["lengths"], t["parents"], return_lse=True, stream=stream, **call)
    torch.cuda.synchronize()
    want, want_lse, err, err_lse = ref.attention(c["q"], c["kp"], c["vp"], c["table"], c["lengths"], c["parents"], scale,
                                                 kw.get("window", 0), kw.get("sinks", 0), kw.get("softcap", 0.0), kw.get("mask"))
    near(got, want, err, what + " out")
    near(lse, want_lse, err_lse, what + " lse")
    return got, lse


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("lengths,nodes,hq,hk,d,page", [
    ([0], 1, 1, 1, 2, 1), ([77], 6, 8, 2, 64, 16), ([0, 1, 15, 16, 17], 5, 6, 3, 80, 17), ([40, 0, 333], 16, 4, 4, 72, 3),
    ([200, 31], 64, 16, 1, 128, 16), ([130], 25, 12, 4, 128, 32), ([65, 3], 7, 16, 1, 256, 64), ([47], 33, 3, 3, 96, 16),
    ([300], 9, 10, 2, 192, 16), ([19], 11, 5, 1, 33, 7)])
def test_attention(x, cache, lengths, nodes, hq, hk, d, page):
    g = gen(nodes * 100 + d)
    trees = [chain(nodes)] + [some_tree(g, nodes) for _ in lengths[1:]] if len(lengths) > 1 else [some_tree(g, nodes)]
    c = attn_case(g, lengths, trees, hq, hk, d, x, cache, page)
    hide_unseen(c)
    check_attn(c, f"{x} over {cache}, {lengths} + {nodes}, ({hq},{hk})x{d} page {page}")


@pytest.mark.parametrize("nodes", [1, 2, 3, 8, 16, 17, 31, 32, 33, 48, 63, 64])
@pytest.mark.parametrize("group", [1, 3, 5])
def test_attention_rows(nodes, group):
    """Every number of nodes' rows against the kernels' blocks of them."""
    g = gen(nodes + group)
    for x, cache in ((BF16, BF16), (F32, F16), (F32, F32)):
        c = attn_case(g, [70, 5], [some_tree(g, nodes), chain(nodes)], 2 * group, 2, 64, x, cache, 16)
        hide_unseen(c)
        check_attn(c, f"{nodes} nodes of {group} heads, {x} over {cache}")


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 3), (10, 0), (16, 4), (40, 100), (100, 1), (1000, 5), (7, 33)])
def test_attention_window_and_sinks(x, cache, window, sinks):
    g = gen(window * 7 + sinks)
    c = attn_case(g, [0, 3, 64, 150, 299], [chain(12)] + [some_tree(g, 12) for _ in range(4)], 6, 2, 64, x, cache, 16)
    hide_unseen(c, window=window, sinks=sinks)
    check_attn(c, f"window {window}, {sinks} sinks, {x} over {cache}", window=window, sinks=sinks)


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
def test_attention_mask_softcap_and_scale(x, cache):
    g = gen(9)
    c = attn_case(g, [100, 30, 260, 5], [some_tree(g, 20) for _ in range(4)], 8, 2, 128, x, cache, 16)
    mask = torch.rand((4, 300), generator=g) < 0.7
    mask[1] = False          # a sequence that sees nothing
    mask[3, :5] = False      # one that sees only nodes
    hide_unseen(c, mask=mask)
    check_attn(c, "mask", mask=mask)
    check_attn(c, "mask of bytes, cap", mask=mask.to(torch.uint8) * 4, softcap=5.0, window=50, sinks=2)
    check_attn(c, "short mask", mask=mask[:, :50].contiguous(), scale=0.3)
    check_attn(c, "no mask columns", mask=mask[:, :0].contiguous())
    c = attn_case(g, [100, 30], [some_tree(g, 20) for _ in range(2)], 8, 2, 128, x, cache, 16)
    check_attn(c, "cap", softcap=20.0, scale=-0.5)
    check_attn(c, "no scale", scale=0.0)


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
def test_attention_large_scores(x, cache):
    """Scores whose exponentials reach over all of 32 bits."""
    g = gen(4)
    c = attn_case(g, [90], [some_tree(g, 14)], 4, 1, 64, x, cache, 16)
    check_attn(c, "large scores", scale=20.0)


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("softcap", [0.0, 10.0])
@pytest.mark.parametrize("hq,nodes", [(4, 14), (10, 14)])
def test_attention_scales_at_the_ends_of_a_float(x, cache, softcap, hq, nodes):
    """Queries and scales so small that their product is none, and so large, over keys of 0, that it is infinite: scores of 0."""
    g = gen(14)
    c = attn_case(g, [20], [some_tree(g, nodes)], hq, 1, 64, x, cache, 16)
    c["q"] = randn(g, c["q"].shape, F32, 2.0 ** -119).to(x)
    hide_unseen(c)
    check_attn(c, "small queries and scale", scale=2.0 ** -30, softcap=softcap)
    c["q"] = randn(g, c["q"].shape, F32, 2.0 ** 120).clamp(-65504.0, 65504.0).to(x) if x == F16 else randn(g, c["q"].shape, F32, 2.0 ** 120).to(x)
    c["kp"] = torch.where(torch.isnan(c["kp"]), c["kp"], torch.zeros((), dtype=cache))
    check_attn(c, "large queries and scale over keys of 0", scale=2.0 ** 30, softcap=softcap)


def test_attention_pages_that_are_none():
    g = gen(6)
    c = attn_case(g, [100, 50, 64], [some_tree(g, 10) for _ in range(3)], 4, 2, 64, BF16, BF16, 16)
    c["table"][0, 2], c["table"][1, 3], c["table"][2] = -1, c["kp"].shape[0], -5   # nodes' pages among them; a sequence without any
    hide_unseen(c)
    check_attn(c, "pages that are none")
    c["lengths"] = ints([2 ** 31 - 1, -3, 200])     # longer than the table, shorter than nothing, nodes beyond the table
    hide_all = dict(c, kp=c["kp"].clone(), vp=c["vp"].clone())
    hide_all["kp"].nan_to_num_(0.5)
    hide_all["vp"].nan_to_num_(0.25)
    hide_all["lengths"] = ints([150, -3, 200])
    check_attn(hide_all, "longer than the table")
    hide_all["lengths"] = ints([2 ** 31 - 1, 2 ** 31 - 5, 0])
    t = {k: v.cuda() for k, v in hide_all.items()}
    got = lib().attn_tree(t["q"], t["kp"], t["vp"], t["table"], t["lengths"], t["parents"], window=100)
    torch.cuda.synchronize()
    assert (got[:20] == 0).all()    # the window's places lie beyond the table


def test_attention_strided_and_unaligned():
    g = gen(12)
    for d, shift in ((128, 0), (64, 1), (72, 0), (80, 3), (33, 1)):
        for x, cache in ((BF16, BF16), (F32, BF16), (F32, F32)):
            c = attn_case(g, [60, 20], [some_tree(g, 9) for _ in range(2)], 6, 2, d, x, cache, 16)
            n = c["kp"].shape[0]
            pools = torch.empty(n * 2 * 2 * 16 * d + shift, dtype=cache, device="cuda")[shift:].view(n, 2, 2, 16, d)
            kp, vp = pools[:, 0].transpose(1, 2), pools[:, 1].transpose(1, 2)
            kp.copy_(c["kp"])
            vp.copy_(c["vp"])
            q = torch.empty(18 * 9 * d + shift, dtype=x, device="cuda")[shift:].view(18, 9, d)[:, 2:8]
            q.copy_(c["q"])
            out = torch.full((18, 8, d + 3), math.nan, dtype=x, device="cuda")
            check_attn(c, f"strided d {d} shift {shift}", dict(q=q, kp=kp, vp=vp), out=out[:, 1:7, :d])
            assert torch.isnan(out[:, 0]).all() and torch.isnan(out[:, 7]).all() and torch.isnan(out[:, :, d:]).all()
            check_attn(c, f"in place d {d} shift {shift}", dict(q=q, kp=kp, vp=vp), out=q)


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
def test_attention_long(x, cache):
    """Sequences that are split over workgroups, ragged, with given bounds and workspaces: the same within the bounds."""
    ilpm = lib()
    g = gen(21)
    c = attn_case(g, [3000, 1, 0, 700, 1500, 2999], [some_tree(g, 6) for _ in range(6)], 8, 2, 64, x, cache, 32, extra=200)
    hide_unseen(c)
    check_attn(c, "long")
    check_attn(c, "long, bound", max_len=3000)
    check_attn(c, "long, wrong bound", max_len=10)
    t = {k: v.cuda() for k, v in c.items()}
    need = ilpm.attn_tree_workspace_size(t["kp"], t["vp"], t["table"], 8, 6, max_len=3000)
    ws = torch.full((max(need, 1),), 0xff, dtype=torch.uint8, device="cuda")
    check_attn(c, "long, own workspace", max_len=3000, workspace=ws)
    check_attn(c, "long, window", window=900, sinks=20)


def test_attention_many_sequences():
    g = gen(22)
    for n in (70, 300):
        lengths = torch.randint(0, 40, (n,), generator=g).tolist()
        c = attn_case(g, lengths, [some_tree(g, 3) for _ in lengths], 2, 1, 64, F32, BF16, 16)
        hide_unseen(c)
        check_attn(c, f"{n} sequences")
        check_attn(c, f"{n} sequences, tables of unknown use", dict(table=torch.cat((c["table"], torch.full((n, 90), -1, dtype=torch.int32)), 1).cuda()))


def test_attention_rows_of_large_trees():
    """More rows than a workgroup takes, over a length that is split."""
    g = gen(23)
    for x, cache, d in ((BF16, BF16, 128), (F32, BF16, 256), (F16, F16, 80), (F32, F32, 64)):
        c = attn_case(g, [400], [some_tree(g, 61)], 10, 1, d, x, cache, 16, extra=100)
        hide_unseen(c)
        check_attn(c, f"610 rows of {d}, {x} over {cache}")


def test_attention_of_a_single_node_is_attn_decode():
    ilpm = lib()
    g = gen(24)
    c = attn_case(g, [100, 0, 33], [[-1]] * 3, 8, 2, 128, BF16, BF16, 16)
    t = {k: v.cuda() for k, v in c.items()}
    for kw in (dict(), dict(window=20), dict(softcap=10.0)):
        a, la = ilpm.attn_tree(t["q"], t["kp"], t["vp"], t["table"], t["lengths"], t["parents"], return_lse=True, **kw)
        b, lb = ilpm.attn_decode(t["q"], t["kp"], t["vp"], t["table"], t["lengths"] + 1, return_lse=True, **kw)
        assert (a.float() - b.float()).abs().max() <= 2 * U[BF16] * b.float().abs().max() and (la - lb).abs().max() < 1e-5


def test_attention_of_nothing():
    ilpm = lib()
    c = attn_case(gen(1), [5, 6], [chain(4)] * 2, 4, 2, 64, F32, F32, 16)
    t = {k: v.cuda() for k, v in c.items()}
    got = ilpm.attn_tree(t["q"][:0], t["kp"], t["vp"], t["table"][:0], t["lengths"][:0], t["parents"][:0])
    assert got.shape == (0, 4, 64)
    got = ilpm.attn_tree(t["q"][:0], t["kp"], t["vp"], t["table"], t["lengths"], t["parents"][:, :0].contiguous())
    assert got.shape == (0, 4, 64)
    got, lse = ilpm.attn_tree(t["q"], t["kp"][:0], t["vp"][:0], t["table"], t["lengths"], t["parents"], return_lse=True)
    assert (got == 0).all() and (lse == -math.inf).all()
    got, lse = ilpm.attn_tree(t["q"], t["kp"], t["vp"], t["table"], t["lengths"], torch.full_like(t["parents"], -2), return_lse=True)
    assert (got == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
def test_attention_of_what_is_not_finite(x, cache):
    """An infinite or NaN value that a node sees is in its output and in no other node's."""
    ilpm = lib()
    g = gen(25)
    c = attn_case(g, [40], [[-1, 0, 0, 1, 2]], 4, 2, 64, x, cache, 16)
    page, slot = int(c["table"][0, 41 // 16]), 41 % 16   # node 1: above node 3
    c["vp"][page, slot, 0, 9] = math.nan
    t = {k: v.cuda() for k, v in c.items()}
    got = ilpm.attn_tree(t["q"], t["kp"], t["vp"], t["table"], t["lengths"], t["parents"]).cpu()
    odd = torch.isnan(got)
    want = torch.zeros_like(odd)
    want[1, :2, 9] = want[3, :2, 9] = True
    assert torch.equal(odd, want)
    c["vp"][page, slot, 0, 9] = 1.0
    c["kp"][page, slot, 1, 3] = math.nan
    t = {k: v.cuda() for k, v in c.items()}
    got = ilpm.attn_tree(t["q"], t["kp"], t["vp"], t["table"], t["lengths"], t["parents"]).cpu()
    assert torch.isfinite(got[[0, 2, 4]]).all() and torch.isfinite(got[:, :2]).all() and not torch.isfinite(got[[1, 3], 2:]).any()


# ---- verify_drafts ----

def verify_case(g, n, t, vocab, dtype, draft, std=3.0, branch=None):
    logits = torch.randn((n, t, vocab), generator=g) * std
    target = torch.softmax(logits, -1).to(dtype)
    q = torch.softmax(logits + torch.randn((n, t, vocab), generator=g), -1).to(dtype)
    parents = ints([[-1] + [(i - 1) // branch if branch else int(torch.randint(max(0, i - 4), i, (), generator=g)) for i in range(1, t)] for _ in range(n)])
    tokens = torch.zeros((n, t), dtype=torch.int32)
    for s in range(n):
        for i in range(1, t):
            tokens[s, i] = int(torch.multinomial(q[s, int(parents[s, i])].float(), 1, generator=g))
    return dict(tokens=tokens, parents=parents, target=target, draft=q if draft else None, uniforms=torch.rand((n, t), generator=g))


def check_verify(c, what, cuda=None, **kw):
    ilpm = lib()
    note(f"[verify] {what}")
    t = {k: v.cuda() if v is not None else None for k, v in c.items()}
    t.update(cuda or {})
    path, counts, last = ilpm.verify_drafts(t["tokens"], t["parents"], t["target"], t["uniforms"], draft=t["draft"], **kw)
    torch.cuda.synchronize()
    want = ref.verify(c["tokens"], c["parents"], c["target"], c["uniforms"], c["draft"])
    assert counts.tolist() == want[1], what
    assert path.tolist() == want[0], what
    assert last.tolist() == want[2], what
    return counts.tolist()


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("draft", [False, True])
@pytest.mark.parametrize("n,t,vocab", [(1, 1, 1), (1, 8, 50), (5, 16, 333), (3, 64, 4096), (2, 9, 4097), (7, 6, 20000), (1, 5, 70001)])
def test_verify(dtype, draft, n, t, vocab):
    c = verify_case(gen(n * t + vocab), n, t, vocab, dtype, draft)
    check_verify(c, f"{n}x{t}x{vocab} {dtype} draft {draft}")


@pytest.mark.parametrize("draft", [False, True])
@pytest.mark.parametrize("branch", [1, 3, 8, 63])
def test_verify_trees_and_chains(draft, branch):
    g, kept = gen(branch), []
    for _ in range(3):
        c = verify_case(g, 20, 24, 40, F32, draft, std=1.5, branch=branch)
        kept += check_verify(c, f"branch {branch} draft {draft}")
    assert min(kept) == 1 and max(kept) >= 2


@pytest.mark.parametrize("draft", [False, True])
def test_verify_exact_fractions(draft):
    """Probabilities and numbers that are fractions of 64, so that borders are met exactly."""
    g = gen(5)
    n, t, vocab = 200, 6, 7
    cuts = torch.sort(torch.randint(0, 65, (2, n, t, vocab - 1), generator=g), -1).values
    rows = torch.diff(torch.cat((torch.zeros((2, n, t, 1)), cuts, torch.full((2, n, t, 1), 64.0)), -1)) / 64
    tokens = torch.randint(0, vocab, (n, t), generator=g).to(torch.int32)
    parents = ints([[-1] + [int(torch.randint(0, i, (), generator=g)) for i in range(1, t)] for _ in range(n)])
    u = torch.randint(0, 64, (n, t), generator=g).float() / 64
    for dtype in (F32, BF16):
        check_verify(dict(tokens=tokens, parents=parents, target=rows[0].to(dtype), draft=rows[1].to(dtype) if draft else None, uniforms=u), "fractions")


def test_verify_what_is_no_tree_and_no_token():
    c = verify_case(gen(7), 8, 10, 100, F32, False)
    c["parents"][1], c["parents"][2, 0], c["parents"][3, 0], c["parents"][4, 3:] = -2, 0, 5, -2
    c["parents"][5, 4], c["parents"][6, 2] = 7, -9
    c["tokens"][0, 1:4], c["tokens"][7, 1:] = ints([-1, 100, 2 ** 31 - 1]), -2 ** 31
    check_verify(c, "no tree")
    c["draft"] = verify_case(gen(8), 8, 10, 100, F32, True)["draft"]
    check_verify(c, "no tree, draft rows")


def test_verify_odd_probabilities():
    """Rows that are 0, NaN, negative or infinite in places, tokens twice among siblings, numbers that are none."""
    for draft in (False, True):
        c = verify_case(gen(9), 12, 8, 5000, F32, draft, branch=3)
        p = c["target"]
        p[0] = 0.0
        p[1, 0, :2500] = math.nan
        p[2, 0] = -1.0
        p[2, 0, 4321] = 0.5
        p[3, 0, 17] = math.inf
        p[4] = math.nan
        c["tokens"][5, 1:4] = int(c["tokens"][5, 1])
        c["uniforms"][6] = 1.0
        c["uniforms"][7] = math.nan
        c["uniforms"][8] = 0.0
        c["uniforms"][9] = -1.0
        if draft:
            c["draft"][10] = p[10]      # nothing is left after a refusal
            c["uniforms"][10, 1:] = 1.0
            c["draft"][11, 0, :100] = math.nan
            c["draft"][11, 1, 7] = math.inf
        check_verify(c, f"odd probabilities, draft {draft}")


@pytest.mark.parametrize("dtype,vocab,zeros", [(F32, 32768, 20000), (BF16, 65536, 40000), (F32, 300000, 270000), (F16, 300000, 262145)], ids=str)
@pytest.mark.parametrize("draft", [False, True])
def test_verify_numbers_below_zero_over_rows_that_begin_with_zeros(dtype, vocab, zeros, draft):
    """The next token of a number below 0 is the first that has a probability, however far from the row's beginning."""
    c = verify_case(gen(11), 4, 2, vocab, dtype, draft, std=1.0)
    c["target"][:, :, :zeros] = 0.0
    c["target"][:, :, zeros + 7] = 0.5   # (in every row above 0)
    c["uniforms"][:, 0] = torch.tensor([-1.0, -math.inf, -1e-30, 0.0])
    c["uniforms"][:, 1] = 2.0            # (the child is refused, except where that passes)
    check_verify(c, f"numbers below 0, {vocab} {dtype} draft {draft}")


def test_verify_strided_and_given_outputs():
    ilpm = lib()
    g = gen(10)
    c = verify_case(g, 4, 9, 777, BF16, True)
    both = torch.empty(4 * 9 * 2 * 800 + 1, dtype=BF16, device="cuda")[1:].view(4, 9, 2, 800)
    both[:, :, 0, :777], both[:, :, 1, :777] = c["target"].cuda(), c["draft"].cuda()
    cuda = dict(target=both[:, :, 0, :777], draft=both[:, :, 1, :777])
    check_verify(c, "strided", cuda)
    need = ilpm.verify_drafts_workspace_size(4, 9, 777)
    out = [torch.full(s, 7, dtype=torch.int32, device="cuda") for s in ((4, 9), (4,), (4,))]
    check_verify(c, "outputs given", cuda, path=out[0], counts=out[1], next_tokens=out[2],
                 workspace=torch.full((need,), 0xff, dtype=torch.uint8, device="cuda"))
    check_verify(dict(c, target=c["target"][:, :1].expand(4, 9, 777), draft=None), "one row for all nodes",
                 dict(target=c["target"].cuda()[:, :1].expand(4, 9, 777), draft=None))
    got = ilpm.verify_drafts(*(c[k][:0].cuda() for k in ("tokens", "parents", "target", "uniforms")))
    assert got[0].shape == (0, 9) and got[1].shape == got[2].shape == (0,)


# ---- kv_copy ----

def copy_case(g, n, pages_each, page, hk, d, cache):
    n_pages = 2 * n * pages_each + 2
    order = torch.randperm(n_pages, generator=g)[:2 * n * pages_each].view(2, n, pages_each).to(torch.int32)
    return dict(kp=randn(g, (n_pages, page, hk, d), cache), vp=randn(g, (n_pages, page, hk, d), cache), src=order[0].contiguous(), dst=order[1].contiguous())


def check_copy(c, src_start, dst_start, counts, path, what, cuda=None, same=False, **kw):
    ilpm = lib()
    note(f"[copy] {what}")
    t = {k: v.cuda() for k, v in c.items()}
    t.update(cuda or {})
    dst, dst_gpu = (c["src"], t["src"]) if same else (c["dst"], t["dst"])
    gpu = [ints(v).cuda() for v in (src_start, dst_start, counts)]
    ilpm.kv_copy(t["kp"], t["vp"], t["src"], dst_gpu, *gpu, path=None if path is None else path.cuda(), **kw)
    torch.cuda.synchronize()
    most = kw.get("max_count") or (path.shape[1] if path is not None else 1 << 20)
    for name in ("kp", "vp"):
        want = ref.copy(c[name], c["src"], dst, src_start, dst_start, counts, path, most)
        assert torch.equal(t[name].cpu(), want), f"{what} {name}"


@pytest.mark.parametrize("cache", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("hk,d,page", [(1, 1, 1), (2, 7, 3), (8, 128, 16), (3, 80, 17), (1, 36, 16), (5, 66, 64), (2, 256, 32)])
def test_copy_kept_nodes(cache, hk, d, page):
    """Any paths in their own place: ascending ones as a walk leaves them, others, and the same node several times."""
    g = gen(hk * d)
    for nodes in (1, 5, 8, 9, 16, 30, 33, 64):
        n = 5
        c = copy_case(g, n, -(-(70 + nodes) // page), page, hk, d, cache)
        path = torch.randint(-1, nodes, (n, nodes), generator=g).to(torch.int32)
        path[0] = torch.sort(path[0]).values
        path[1] = torch.arange(nodes - 1, -1, -1)
        counts = [nodes, nodes, nodes // 2, 0, nodes + 9]
        check_copy(c, [0, 3, 50, 60, 17], [0, 3, 50, 60, 17], counts, path, f"{nodes} nodes of ({hk},{d}) page {page}", same=True)
        check_copy(c, [0, 3, 50, 60, 17], [4, 0, 50, 1, 20], counts, path, f"{nodes} nodes elsewhere")


@pytest.mark.parametrize("cache", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("hk,d,page", [(1, 1, 1), (2, 7, 3), (8, 128, 16), (3, 80, 17), (1, 36, 16), (2, 256, 32)])
def test_copy_forks(cache, hk, d, page):
    g = gen(hk + d)
    for tokens in (1, 2, 15, 16, 17, 100, 333):
        c = copy_case(g, 4, -(-(tokens + 20) // page), page, hk, d, cache)
        check_copy(c, [0, 5, 20, 1], [0, 9, 3, 1], [tokens, tokens // 2, 0, -7], None, f"{tokens} tokens of ({hk},{d}) page {page}")
        check_copy(c, [0, 5, 20, 1], [0, 9, 3, 1], [tokens] * 4, None, f"{tokens} tokens, bounded", max_count=7)


def test_copy_leaves_out_what_names_no_place():
    g = gen(3)
    c = copy_case(g, 6, 4, 16, 2, 64, BF16)
    c["src"][0, 1], c["dst"][1, 2] = -1, c["kp"].shape[0]
    starts = [0, 0, -5, 2 ** 31 - 1, 10, 60]
    check_copy(c, starts, [0, 0, 0, 0, 2 ** 31 - 1, 40], [64, 64, 64, 64, 64, 64], None, "no place")
    path = torch.randint(-3, 64, (6, 10), generator=g).to(torch.int32)
    path[2, 4], path[5, 0] = 2 ** 31 - 1, -2 ** 31
    check_copy(c, starts, [0, 0, 0, 0, 2 ** 31 - 1, 60], [10] * 6, path, "no place on a path")


def test_copy_from_before_the_beginning():
    """Starts below 0: what lies before the beginning is left out, and all tokens that have places are copied, however many
    do not."""
    g = gen(5)
    c = copy_case(g, 6, 4, 16, 2, 64, BF16)
    src = [-10, -10, -100, -1, -2 ** 31, 3]
    dst = [-10, -3, -70, -64, -2 ** 31, -5]
    check_copy(c, src, dst, [80, 200, 2 ** 31 - 1, 128, 2 ** 31 - 1, 70], None, "before the beginning")
    check_copy(c, src, dst, [80, 200, 100, 128, 0, 70], None, "before the beginning, bounded", max_count=75)
    path = torch.randint(0, 64, (6, 40), generator=g).to(torch.int32)
    check_copy(c, src, dst, [40] * 6, path, "before the beginning on a path")


def test_copy_a_beam_from_one_row():
    """Rows that share their source, and tables of different widths."""
    g = gen(4)
    c = copy_case(g, 3, 5, 16, 2, 64, F16)
    c["src"] = c["src"][:1].expand(3, 5).contiguous()
    c["dst"] = c["dst"][:, :3].contiguous()
    check_copy(c, [3, 10, 16], [0, 1, 2], [20, 30, 47], None, "from one row")
    t = {k: v.cuda() for k, v in c.items()}
    check_copy(c, [3, 10, 16], [0, 1, 2], [20, 30, 47], None, "from an expanded row", dict(src=t["src"][:1].expand(3, 5)))


def test_copy_strided():
    g = gen(6)
    for d, shift in ((64, 0), (64, 1), (36, 3)):
        c = copy_case(g, 3, 4, 16, 2, d, BF16)
        n = c["kp"].shape[0]
        pools = torch.empty(n * 2 * 2 * 16 * d + shift, dtype=BF16, device="cuda")[shift:].view(n, 2, 2, 16, d)
        kp, vp = pools[:, 0].transpose(1, 2), pools[:, 1].transpose(1, 2)
        kp.copy_(c["kp"])
        vp.copy_(c["vp"])
        wide = torch.randint(0, 12, (3, 20), generator=g).to(torch.int32)
        check_copy(c, [0, 4, 30], [0, 4, 30], [9, 3, 7], wide[:, 3:12], f"strided d {d} shift {shift}", dict(kp=kp, vp=vp), same=True)


def test_copy_nothing():
    ilpm = lib()
    c = copy_case(gen(1), 2, 2, 16, 1, 64, F32)
    t = {k: v.cuda() for k, v in c.items()}
    z = torch.zeros(2, dtype=torch.int32, device="cuda")
    before = t["kp"].clone()
    ilpm.kv_copy(t["kp"], t["vp"], t["src"], t["dst"], z, z, z + 1, max_count=0)
    ilpm.kv_copy(t["kp"], t["vp"], t["src"], t["dst"], z, z, z + 1, path=torch.zeros((2, 0), dtype=torch.int32, device="cuda"))
    ilpm.kv_copy(t["kp"], t["vp"], t["src"][:0], t["dst"][:0], z[:0], z[:0], z[:0])
    ilpm.kv_copy(t["kp"][:0], t["vp"][:0], t["src"], t["dst"], z, z, z + 1)
    assert torch.equal(t["kp"], before)


# ---- streams, graphs and workspaces ----

def step_case(seed):
    """A batch's cache and one drafted step's inputs, and the calls of the step on them."""
    g = gen(seed)
    n, t, hq, hk, d, vocab = 4, 9, 8, 2, 64, 6000
    c = attn_case(g, [700, 20, 0, 333], [[-1] + [int(torch.randint(0, i, (), generator=g)) for i in range(1, t)] for _ in range(n)], hq, hk, d, BF16, BF16, 16)
    v = verify_case(g, n, t, vocab, F32, False, std=4.0)
    v["parents"] = c["parents"]
    angle = torch.rand((800, d // 2), generator=g) * 6.3
    depth = ints([[len(a) - 1 for a in ref.above(row)] for row in c["parents"].tolist()])
    s = {k: x.cuda() for k, x in dict(c, k=randn(g, (n * t, hk, d), BF16), v=randn(g, (n * t, hk, d), BF16), cos=angle.cos(), sin=angle.sin(),
                                      seq=ints([[i] * t for i in range(n)]).view(-1), pos=(c["lengths"][:, None] + depth).view(-1),
                                      slots=(c["lengths"][:, None] + torch.arange(t)).view(-1).to(torch.int32), tokens=v["tokens"],
                                      target=v["target"], uniforms=v["uniforms"]).items()}
    return s


def step(s, stream=None):
    ilpm = lib()
    q = ilpm.kv_append_norm(s["k"], s["v"], s["kp"], s["vp"], s["table"], s["seq"], s["pos"], slots=s["slots"], q=s["q"], cos=s["cos"],
                            sin=s["sin"], stream=stream)
    a, lse = ilpm.attn_tree(q, s["kp"], s["vp"], s["table"], s["lengths"], s["parents"], return_lse=True, stream=stream)
    path, counts, last = ilpm.verify_drafts(s["tokens"], s["parents"], s["target"], s["uniforms"], stream=stream)
    ilpm.kv_copy(s["kp"], s["vp"], s["table"], s["table"], s["lengths"], s["lengths"], counts, path=path, stream=stream)
    return [q, a, lse, path, counts, last, s["kp"], s["vp"]]


def same(a, b):
    return all(torch.equal(torch.nan_to_num(x.float(), 7.0), torch.nan_to_num(y.float(), 7.0)) for x, y in zip(a, b))


def fresh(s):
    return {k: v.clone() for k, v in s.items()}


def test_a_step_is_the_same_every_time_and_on_other_streams():
    s = step_case(31)
    note("[step] twice")
    want = step(fresh(s))
    again = step(fresh(s))
    torch.cuda.synchronize()
    assert same(want, again)
    streams = [torch.cuda.Stream() for _ in range(3)]
    cases = [fresh(s) for _ in streams]
    torch.cuda.synchronize()
    note("[step] three streams at once")
    got = [step(c, stream=st) for c, st in zip(cases, streams)]
    torch.cuda.synchronize()
    for x in got:
        assert same(want, x)
    note("[step] current stream")
    c = fresh(s)
    torch.cuda.synchronize()
    with torch.cuda.stream(streams[0]):
        x = step(c)
    torch.cuda.synchronize()
    assert same(want, x)


def test_two_steps_captured_and_replayed():
    """Two graphs of different inputs, each with its own memory, replayed in turn with eager work between."""
    a, b = step_case(32), step_case(33)
    wants = [step(fresh(a)), step(fresh(b))]
    torch.cuda.synchronize()
    graphs, outs, cases = [], [], []
    for s in (a, b):
        c = fresh(s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(c))
        graphs.append(g)
        cases.append(c)
    for turn in range(4):
        note(f"[step] replay {turn}")
        for g, s, c, out, want in zip(graphs, (a, b), cases, outs, wants):
            for k in ("kp", "vp"):
                c[k].copy_(s[k])
            g.replay()
            torch.cuda.synchronize()
            assert same(want, out), turn
        assert same(wants[0], step(fresh(a)))   # eager work between
        torch.cuda.synchronize()
    # Other inputs in the same memory: what was found in the replays before must not matter.
    c, out = cases[0], outs[0]
    for k in c:
        c[k].copy_(b[k])
    graphs[0].replay()
    torch.cuda.synchronize()
    assert same(wants[1], out)


def test_workspaces_of_the_caller():
    ilpm = lib()
    s = step_case(34)
    need = ilpm.attn_tree_workspace_size(s["kp"], s["vp"], s["table"], 8, 9)
    assert need > 0
    out = lambda **kw: ilpm.attn_tree(s["q"], s["kp"], s["vp"], s["table"], s["lengths"], s["parents"], **kw)  # noqa: E731
    want = out()
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    assert torch.equal(want, out(workspace=ws)) and torch.equal(want, out(workspace=ws))
    with pytest.raises(ilpm.IlpmError, match="workspace too small"):
        out(workspace=ws[:need - 1])
    with pytest.raises(ValueError, match="contiguous"):
        out(workspace=torch.empty((2, need), dtype=torch.uint8, device="cuda")[:, ::2])
    v = verify_case(gen(35), 2, 4, 100000, F32, False)
    need = ilpm.verify_drafts_workspace_size(2, 4, 100000)
    with pytest.raises(ilpm.IlpmError, match="workspace too small"):
        ilpm.verify_drafts(*(v[k].cuda() for k in ("tokens", "parents", "target", "uniforms")), workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))


def test_refusals_of_the_binding():
    ilpm = lib()
    s = step_case(36)

    def caller(f, names):
        return lambda **kw: f(*[kw.get(k, s[k]) for k in names], **{k: v for k, v in kw.items() if k not in names})

    append = caller(ilpm.kv_append_norm, ("k", "v", "kp", "vp", "table", "seq", "pos"))
    attn = caller(ilpm.attn_tree, ("q", "kp", "vp", "table", "lengths", "parents"))
    check = caller(ilpm.verify_drafts, ("tokens", "parents", "target", "uniforms"))
    with pytest.raises(ValueError, match="norm must be"):
        append(norm="l2")
    with pytest.raises(ValueError, match="slots"):
        append(slots=s["slots"][:3])
    with pytest.raises(ValueError, match="without q"):
        append(q_w=torch.ones(64, device="cuda"))
    with pytest.raises(ValueError, match="k_w must be"):
        append(k_w=torch.ones(65, device="cuda"))
    with pytest.raises(TypeError, match="of one type"):
        append(q=s["q"], q_w=torch.ones(64, device="cuda"), k_w=torch.ones(64, device="cuda", dtype=BF16))
    with pytest.raises(ilpm.IlpmError):
        append(norm=None, k_w=torch.ones(64, device="cuda"))
    with pytest.raises(TypeError, match="int32"):
        append(slots=s["slots"].long())
    with pytest.raises(ValueError, match="parents must be"):
        attn(parents=s["parents"][:2])
    with pytest.raises(ValueError, match="parents must be"):
        attn(parents=torch.zeros((4, 12), dtype=torch.int32, device="cuda")[:, :9])   # rows that are not together
    with pytest.raises(ValueError, match="q must be"):
        attn(q=s["q"][:-1])
    with pytest.raises(ilpm.IlpmError, match="unsupported"):
        attn(q=torch.zeros((4 * 65, 8, 64), dtype=BF16, device="cuda"), parents=torch.zeros((4, 65), dtype=torch.int32, device="cuda"))
    with pytest.raises(ilpm.IlpmError):
        attn(window=-1)
    with pytest.raises(ilpm.IlpmError):
        attn(sinks=-1)
    with pytest.raises(TypeError, match="mask"):
        attn(mask=torch.zeros((4, 9), device="cuda"))
    with pytest.raises(TypeError, match="CUDA"):
        attn(lengths=s["lengths"].cpu())
    with pytest.raises(ValueError, match="target must be"):
        check(target=s["target"][:, :5])
    with pytest.raises(ValueError, match="draft must be"):
        check(draft=s["target"].to(BF16))
    with pytest.raises(ValueError, match="uniforms"):
        check(uniforms=s["uniforms"][:, :3].contiguous())
    with pytest.raises(TypeError, match="float32"):
        check(uniforms=s["uniforms"].double())
    with pytest.raises(TypeError, match="path must be"):
        check(path=torch.zeros((4, 9), dtype=torch.int64, device="cuda"))
    with pytest.raises(ilpm.IlpmError):
        check(target=torch.zeros((4, 9, 0), device="cuda"))
    z = torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="dst_table"):
        ilpm.kv_copy(s["kp"], s["vp"], s["table"], s["table"][:2], z, z, z)
    with pytest.raises(ValueError, match="counts"):
        ilpm.kv_copy(s["kp"], s["vp"], s["table"], s["table"], z, z, z[:2])
    with pytest.raises(ValueError, match="path"):
        ilpm.kv_copy(s["kp"], s["vp"], s["table"], s["table"], z, z, z, path=torch.zeros((3, 4), dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="more than the path"):
        ilpm.kv_copy(s["kp"], s["vp"], s["table"], s["table"], z, z, z, path=torch.zeros((4, 4), dtype=torch.int32, device="cuda"), max_count=5)
    with pytest.raises(ilpm.IlpmError, match="unsupported"):
        ilpm.kv_copy(s["kp"], s["vp"], s["table"], s["table"], z, z, z, path=torch.zeros((4, 65), dtype=torch.int32, device="cuda"))
    with pytest.raises(ilpm.IlpmError):
        ilpm.kv_copy(s["kp"], s["vp"], s["table"], s["table"], z, z, z, max_count=-1)


# ---- places beyond 2^31 elements and 2^32 bytes ----

def test_places_beyond_32_bits():
    """Pools of 4.4 GB each, with the pages that are used at both ends; a row of probabilities behind 2^31 others."""
    ilpm = lib()
    g = gen(41)
    n_pages, page, hk, d = 67200, 16, 8, 256
    kp, vp = (torch.empty((n_pages, page, hk, d), dtype=BF16, device="cuda") for _ in range(2))
    used = [0, 1, n_pages - 3, n_pages - 2, n_pages - 1, 65537]
    small = attn_case(g, [40], [[-1, 0, 0, 1]], 16, hk, d, BF16, BF16, page)
    # The small case's pages, at these places.
    small["kp"], small["vp"] = (randn(g, (len(used), page, hk, d), BF16) for _ in range(2))
    order = torch.tensor([[4, 2, 3]])
    small["table"] = order.to(torch.int32)
    big = torch.tensor(used)[order].to(torch.int32).cuda()
    for i, p in enumerate(used):
        kp[p], vp[p] = small["kp"][i].cuda(), small["vp"][i].cuda()
    note("[far] attn_tree")
    check_attn(small, "far pages", dict(kp=kp, vp=vp, table=big))
    check_attn(small, "far pages, split", dict(kp=kp, vp=vp, table=torch.cat((big, torch.full((1, 500), -1, dtype=torch.int32, device="cuda")), 1)))
    note("[far] kv_append_norm")
    c = append_case(g, 4, 1, 16, hk, d, 128, BF16, BF16, page, 3, "rms")
    t = {k: v.cuda() for k, v in c.items()}
    c["table"], c["kp"], c["vp"] = small["table"], small["kp"], small["vp"]
    c["slots"] = ints([0, 15, 16, 47])
    ilpm.kv_append_norm(t["k"], t["v"], kp, vp, big, t["seq"], t["pos"], slots=c["slots"].cuda(), q=t["q"], norm="rms", q_w=t["q_w"], k_w=t["k_w"],
                        eps=1e-5, cos=t["cos"], sin=t["sin"])
    torch.cuda.synchronize()
    keys, err, values, written = ref.append(c["k"], c["v"], c["kp"], c["vp"], c["table"], c["seq"].tolist(), c["pos"].tolist(), c["slots"].tolist(),
                                            "rms", c["k_w"], 1e-5, c["cos"], c["sin"], False)
    err = torch.where(written[:, :, None, None], err + U[BF16] * (keys.abs() + err) + TINY[BF16], 0.0)
    for i, p in enumerate(used):
        near(kp[p], keys[i], err[i], f"page {p} keys")
        assert torch.equal(vp[p].cpu().double(), values[i])
    note("[far] kv_copy")
    now = [torch.stack([x[p] for p in used]).cpu() for x in (kp, vp)]
    src, dst = torch.tensor([[4, 2, 3]]), torch.tensor([[1, 5, 0]])
    path = ints([[20, 3, 40, 41, 0]])
    for p in (None, path):
        z, n = ints([0]).cuda(), ints([5 if p is not None else 45]).cuda()
        ilpm.kv_copy(kp, vp, torch.tensor(used)[src].to(torch.int32).cuda(), torch.tensor(used)[dst].to(torch.int32).cuda(), z, z, n,
                     path=None if p is None else p.cuda())
        torch.cuda.synchronize()
        now = [ref.copy(x, src, dst, [0], [0], n.tolist(), p, 48) for x in now]
        for x, want in zip((kp, vp), now):
            for i, at in enumerate(used):
                assert torch.equal(x[at].cpu(), want[i]), at
    del kp, vp
    note("[far] verify_drafts")
    for draft in (False, True):
        v = verify_case(g, 2, 3, 40000, BF16, draft)
        far = torch.empty((1 << 31) + 3 * 80000, dtype=BF16, device="cuda").as_strided((2, 3, 40000), ((1 << 31) + 7, 80000, 1))
        far.copy_(v["target"])
        cuda = dict(target=far)
        if draft:
            cuda["draft"] = torch.empty(3 * 80000 + (1 << 31), dtype=BF16, device="cuda").as_strided((2, 3, 40000), ((1 << 31) + 7, 80000, 1))
            cuda["draft"].copy_(v["draft"])
        check_verify(v, f"far rows, draft {draft}", cuda)


def test_attention_of_very_many_rows_of_a_head():
    """More rows of one key head than a dimension of a grid holds."""
    ilpm = lib()
    g = gen(42)
    c = attn_case(g, [600], [chain(64)], 1100, 1, 64, BF16, BF16, 16, extra=50)
    t = {k: v.cuda() for k, v in c.items()}
    got, lse = ilpm.attn_tree(t["q"], t["kp"], t["vp"], t["table"], t["lengths"], t["parents"], return_lse=True)
    torch.cuda.synchronize()
    few = [0, 1, 515, 1098, 1099]
    want, want_lse, err, err_lse = ref.attention(c["q"][:, few], c["kp"], c["vp"], c["table"], c["lengths"], c["parents"], 64 ** -0.5)
    near(got[:, few], want, err, "some heads of 1100")
    near(lse[:, few], want_lse, err_lse, "some heads of 1100, lse")
