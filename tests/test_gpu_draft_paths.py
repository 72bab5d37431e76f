"""GPU: the drafted step's kernels on the paths that a call's sizes choose: attention whose waves take rows, marks of values
that are not finite in every block and layout, verification of long rows for several sequences."""
import math

import pytest
import torch

import draft_ref as ref
import test_gpu_draft as base
from gpu_common import note
from test_gpu_draft import BF16, F16, F32, PAIRS, attn_case, chain, check_attn, check_verify, gen, hide_unseen, ints, lib, near, some_tree, verify_case

pytestmark = pytest.mark.gpu


# ---- attention whose waves take rows: more than 32 rows a key head and up to 4 tiles, or 16 where there are 32 workgroups ----

def trees(g, nodes, n):
    """A chain, a whole tree, one of two nodes, none, and any others."""
    got = [chain(nodes), some_tree(g, nodes), [-1, 0] + [-2] * (nodes - 2), [-2] * nodes]
    return (got + [some_tree(g, nodes) for _ in range(n)])[:n]


def by_rows_case(g, lengths, nodes, hq, hk, d, x, cache, page=16):
    return attn_case(g, lengths, trees(g, nodes, len(lengths)), hq, hk, d, x, cache, page)


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("d", [64, 72, 80, 96, 128, 160, 192, 256])
def test_rows_of_short_sequences(x, cache, d):
    ilpm = lib()
    g = gen(d)
    for lengths, nodes, hq, hk in (([20, 0, 9, 20], 12, 4, 1), ([3, 31, 16], 25, 8, 2), ([1], 33, 1, 1), ([15, 17], 64, 3, 1)):
        c = by_rows_case(g, lengths, nodes, hq, hk, d, x, cache)
        t = {k: c[k].cuda() for k in ("kp", "vp", "table")}
        assert ilpm.attn_tree_workspace_size(t["kp"], t["vp"], t["table"], hq, nodes) == 0
        hide_unseen(c)
        check_attn(c, f"{lengths} + {nodes}, ({hq},{hk})x{d} {x} over {cache}")


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("d", [64, 80, 96, 128, 192, 256])
def test_rows_of_many_units_over_up_to_16_tiles(x, cache, d):
    g = gen(d + 1)
    c = by_rows_case(g, [150, 64, 199, 30, 0, 1, 100, 177], 9, 16, 4, d, x, cache)
    hide_unseen(c)
    check_attn(c, f"32 units of up to 14 tiles, heads of {d}, {x} over {cache}")


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("d", [64, 96, 128, 192, 256])
def test_rows_of_sequences_longer_than_was_said(x, cache, d):
    """A bound that is too small: the waves go over many groups of four tiles."""
    g = gen(d + 2)
    c = by_rows_case(g, [300, 0, 129, 64], 10, 4, 1, d, x, cache)
    hide_unseen(c)
    check_attn(c, f"longer than was said, heads of {d}, {x} over {cache}", max_len=16)


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
def test_rows_with_windows_masks_and_caps(x, cache):
    g = gen(50)
    for d in (72, 128, 192):
        c = by_rows_case(g, [140, 20, 61], 12, 8, 2, d, x, cache)
        mask = torch.rand((3, 200), generator=g) < 0.7
        hide_unseen(c)
        check_attn(c, "mask", mask=mask, max_len=20)
        check_attn(c, "window, sinks, cap", window=9, sinks=3, softcap=7.0, max_len=20)
        check_attn(c, "in pages of 3", scale=-0.2, max_len=20)
    c = by_rows_case(g, [140, 20, 61], 12, 8, 2, 64, x, cache, page=7)
    hide_unseen(c, window=33)
    check_attn(c, "pages of 7, window", window=33, max_len=20)


# ---- values that are not finite, seen by some rows only ----

def check_marks(c, what, **kw):
    """Outputs are not finite exactly where they are by definition, and else within the bounds."""
    ilpm = lib()
    note(f"[marks] {what}")
    t = {k: v.cuda() for k, v in c.items()}
    got, lse = ilpm.attn_tree(t["q"], t["kp"], t["vp"], t["table"], t["lengths"], t["parents"], return_lse=True, **kw)
    torch.cuda.synchronize()
    want, want_lse, err, err_lse = ref.attention(c["q"], c["kp"], c["vp"], c["table"], c["lengths"], c["parents"], c["q"].shape[2] ** -0.5,
                                                 kw.get("window", 0), kw.get("sinks", 0))
    odd = ~torch.isfinite(want)
    assert odd.any() and not odd.all()
    assert torch.equal(~torch.isfinite(got.cpu()), odd), what
    near(torch.where(odd, 0.0, got.double().cpu()), torch.where(odd, 0.0, want), torch.where(odd, 0.0, err), what)
    near(lse, want_lse, err_lse, what + " lse")


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("d", [64, 80, 128, 192, 256])
@pytest.mark.parametrize("nodes,hq,hk", [(5, 4, 2), (7, 4, 1), (12, 4, 1), (25, 8, 2)])
def test_values_that_are_not_finite(x, cache, d, nodes, hq, hk):
    g = gen(nodes * 1000 + d)
    parents = [-1] + [(i - 1) // 2 for i in range(1, nodes)]
    # One short sequence (rows to the waves from 33 on), keys split among the waves, split over workgroups, windows.
    for what, length, extra, kw in (("short", 9, 0, {}), ("keys", 120, 0, {}), ("split", 1500, 40, {}), ("window", 120, 0, {"window": 30, "sinks": 2}),
                                    ("window, rows", 120, 0, {"window": 30, "sinks": 2, "max_len": 16})):
        c = attn_case(g, [length, length // 2], [parents, parents], hq, hk, d, x, cache, 16, extra=extra)
        bad = [length + 1, length + nodes - 1] + ([length - 29] if kw else [])   # two nodes; a key that the root alone sees
        for n, j in enumerate(bad):
            page, slot = int(c["table"][0, j // 16]), j % 16
            for i, e in enumerate((0, 3, d // 2 + n, d - 8, d - 1)):
                c["vp"][page, slot, n % hk, e] = (math.nan, math.inf, -math.inf)[(i + n) % 3]
        check_marks(c, f"{what}: {nodes} nodes of ({hq},{hk})x{d}, {x} over {cache}", **kw)


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("nodes,hq,hk", [(5, 4, 2), (25, 8, 2)])
@pytest.mark.parametrize("d", [64, 80, 256])
def test_rows_of_no_node_beside_values_that_are_not_finite(x, cache, nodes, hq, hk, d):
    """What is no node gives 0 and -infinity, whatever lies in the keys of the sequence and in those before its window."""
    ilpm = lib()
    g = gen(nodes + d)
    parents = [[-1, 0, -2] + [-2 if i % 2 else 1 for i in range(3, nodes)], [-2] * nodes, [2] + [0] * (nodes - 1)]
    none = torch.tensor([[a is None for a in ref.above(row)] for row in parents]).view(-1)
    for length in (9, 120):
        for window in (0, 1, 4):
            for extra in (0, 100):
                c = attn_case(g, [length, length - 3, length // 2], parents, hq, hk, d, x, cache, 16, extra=extra)
                c["vp"][:, :, :, d - 1], c["vp"][:, :, :, 1] = math.nan, math.inf
                t = {k: v.cuda() for k, v in c.items()}
                note(f"[no nodes] {length} + {nodes}, window {window}, extra {extra}")
                got, lse = ilpm.attn_tree(t["q"], t["kp"], t["vp"], t["table"], t["lengths"], t["parents"], window=window, return_lse=True)
                torch.cuda.synchronize()
                assert (got.cpu()[none] == 0).all() and (lse.cpu()[none] == -math.inf).all()
                assert torch.isnan(got.cpu()[~none][:, :, d - 1]).all() and torch.isfinite(lse.cpu()[~none]).all()
                assert torch.isfinite(got.cpu()[~none][:, :, 2:d - 1]).all()


# ---- splits ----

@pytest.mark.parametrize("x,cache", [(BF16, BF16), (F32, BF16), (F16, F16)], ids=str)
def test_a_long_sequence_is_the_same_every_time(x, cache):
    ilpm = lib()
    g = gen(60)
    c = attn_case(g, [40000, 3], [some_tree(g, 16), chain(16)], 8, 2, 128, x, cache, 16)
    t = {k: v.cuda() for k, v in c.items()}
    call = lambda: ilpm.attn_tree(t["q"], t["kp"], t["vp"], t["table"], t["lengths"], t["parents"], return_lse=True)  # noqa: E731
    want = call()
    for _ in range(10):
        got = call()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ---- verification of long rows (above 128 KB), several sequences ----

LONG = [(F32, 70001), (F16, 70001), (BF16, 131072)]


@pytest.mark.parametrize("dtype,vocab", LONG, ids=str)
@pytest.mark.parametrize("draft", [False, True])
def test_verify_long_rows(dtype, vocab, draft):
    for n, t, branch in ((6, 5, None), (3, 9, 3), (70, 2, 1)):
        check_verify(verify_case(gen(vocab + n), n, t, vocab, dtype, draft, branch=branch), f"long {n}x{t}x{vocab} {dtype} draft {draft}")


@pytest.mark.parametrize("dtype,vocab", LONG, ids=str)
@pytest.mark.parametrize("draft", [False, True])
def test_verify_long_exact_fractions(dtype, vocab, draft):
    """Fractions of 64 at places over all of a row, also the last of a chunk and the first of the next."""
    g = gen(6)
    n, t, some = 40, 6, 7
    cuts = torch.sort(torch.randint(0, 65, (2, n, t, some - 1), generator=g), -1).values
    few = torch.diff(torch.cat((torch.zeros((2, n, t, 1)), cuts, torch.full((2, n, t, 1), 64.0)), -1)) / 64
    places = torch.tensor([0, 1, 4095, 4096, 40000, 69632, vocab - 1])
    rows = torch.zeros((2, n, t, vocab))
    rows[..., places] = few
    tokens = places[torch.randint(0, some, (n, t), generator=g)].to(torch.int32)
    # (With draft rows a chain: behind a second refusal borders are no fractions of 64 any more.)
    parents = ints([chain(t) if draft else [-1] + [int(torch.randint(0, i, (), generator=g)) for i in range(1, t)] for _ in range(n)])
    u = torch.randint(0, 64, (n, t), generator=g).float() / 64
    check_verify(dict(tokens=tokens, parents=parents, target=rows[0].to(dtype), draft=rows[1].to(dtype) if draft else None, uniforms=u), "long fractions")


@pytest.mark.parametrize("vocab", [70001, 300000])
@pytest.mark.parametrize("draft", [False, True])
def test_verify_long_odd_probabilities(vocab, draft):
    """Sequences without a tree, tokens that are none, rows of nothing, of one value, of NaN; nothing left after a refusal."""
    c = verify_case(gen(12), 14, 5, vocab, F32, draft, branch=2)
    p = c["target"]
    p[0] = 0.0
    p[1, 0, :vocab // 2] = math.nan
    p[2, 0] = -1.0
    p[2, 0, vocab - 3] = 0.5
    p[3, 0, 17] = math.inf
    p[4] = math.nan
    c["tokens"][5, 1:3] = int(c["tokens"][5, 1])
    c["uniforms"][6] = 1.0
    c["uniforms"][7] = math.nan
    c["uniforms"][8] = 0.0
    c["parents"][9], c["parents"][10, 0] = -2, 3
    c["tokens"][11, 1:] = ints([-1, vocab, 2 ** 31 - 1, -2 ** 31])
    p[12] = 0.0                 # one token is all: refused, nothing is left
    p[12, 0, int(c["tokens"][12, 1])] = 1.0
    c["tokens"][12, 2:] = int(c["tokens"][12, 1])
    c["uniforms"][12, 1:] = 1.0
    if draft:
        c["draft"][13] = p[13]
        c["uniforms"][13, 1:] = 1.0
        c["draft"][12] = p[12]
    check_verify(c, f"long odd probabilities, draft {draft}")


@pytest.mark.parametrize("draft", [False, True])
def test_verify_long_workspaces(draft):
    """A workspace of the caller with anything in it, for one call after the other."""
    ilpm = lib()
    need = ilpm.verify_drafts_workspace_size(5, 6, 70001)
    assert need > 0
    ws = torch.full((need + 256,), 0xff, dtype=torch.uint8, device="cuda")
    for seed in (1, 2):
        check_verify(verify_case(gen(seed), 5, 6, 70001, F32, draft, branch=2), f"own workspace, draft {draft}", workspace=ws[:need])
        assert (ws[need:] == 0xff).all()
    ws.fill_(0xff)
    check_verify(dict(verify_case(gen(3), 5, 6, 70001, F32, draft), parents=torch.full((5, 6), -2, dtype=torch.int32)), "no tree", workspace=ws[:need])


# ---- a step with a large vocabulary: streams and graphs ----

def long_step_case(seed, draft):
    s = base.step_case(seed)
    v = verify_case(gen(seed), 4, 9, 70001, F32, draft, std=4.0)
    s.update(tokens=v["tokens"].cuda(), target=v["target"].cuda(), uniforms=v["uniforms"].cuda(), parents=v["parents"].cuda())
    depth = ints([[len(a) - 1 for a in ref.above(row)] for row in v["parents"].tolist()])
    s["pos"] = (s["lengths"][:, None] + depth.cuda()).view(-1)
    if draft:
        s["draft"] = v["draft"].cuda()
    return s


def long_step(s, stream=None):
    ilpm = lib()
    q = ilpm.kv_append_norm(s["k"], s["v"], s["kp"], s["vp"], s["table"], s["seq"], s["pos"], slots=s["slots"], q=s["q"], cos=s["cos"],
                            sin=s["sin"], stream=stream)
    a, lse = ilpm.attn_tree(q, s["kp"], s["vp"], s["table"], s["lengths"], s["parents"], return_lse=True, stream=stream)
    path, counts, last = ilpm.verify_drafts(s["tokens"], s["parents"], s["target"], s["uniforms"], draft=s.get("draft"), stream=stream)
    ilpm.kv_copy(s["kp"], s["vp"], s["table"], s["table"], s["lengths"], s["lengths"], counts, path=path, stream=stream)
    return [q, a, lse, path, counts, last, s["kp"], s["vp"]]


@pytest.mark.parametrize("draft", [False, True])
def test_long_steps_on_streams_and_in_graphs(draft):
    a, b = long_step_case(70, draft), long_step_case(71, draft)
    wants = [long_step(base.fresh(s)) for s in (a, b)]
    torch.cuda.synchronize()
    v = {k: (a[k].cpu() if k in a else None) for k in ("tokens", "parents", "target", "draft", "uniforms")}
    assert [x.tolist() for x in wants[0][3:6]] == list(ref.verify(*(v[k] for k in ("tokens", "parents", "target", "uniforms", "draft"))))
    streams, cases = [torch.cuda.Stream() for _ in range(3)], [base.fresh(s) for s in (a, b, a)]
    torch.cuda.synchronize()
    note("[long step] three streams at once")
    got = [long_step(c, stream=st) for c, st in zip(cases, streams)]
    torch.cuda.synchronize()
    for x, want in zip(got, (wants[0], wants[1], wants[0])):
        assert base.same(want, x)
    graphs, outs, cases = [], [], []
    for s in (a, b):
        c = base.fresh(s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(long_step(c))
        graphs.append(graph)
        cases.append(c)
    for turn in range(3):
        note(f"[long step] replay {turn}")
        for graph, s, c, out, want in zip(graphs, (a, b), cases, outs, wants):
            for k in ("kp", "vp"):
                c[k].copy_(s[k])
            graph.replay()
            torch.cuda.synchronize()
            assert base.same(want, out), turn
        assert base.same(wants[0], long_step(base.fresh(a)))
        torch.cuda.synchronize()
