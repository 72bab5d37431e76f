"""GPU: the decoder-step operators (kv_append, attn_decode, residual_norm)
against their 64-bit definitions in decode_ref.py, within the bounds derived
there: types, head layouts, lengths from zero on, odd sizes, strides, masks
that leave rows empty, and cache contents that must not matter."""
import math

import pytest
import torch

import decode_abi
import decode_ref as ref
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


def guarded(shape, dtype):
    """A CUDA tensor in the middle of a larger one of NaNs, and the check that these stayed."""
    n, pad = math.prod(shape), 64
    buf = torch.full((n + 2 * pad,), math.nan, dtype=dtype, device="cuda")
    return buf[pad:pad + n].view(shape), lambda: torch.isnan(buf[:pad]).all() and torch.isnan(buf[pad + n:]).all()


def near(got, want, err, what):
    got, bad = got.double().cpu(), None
    off = (got - want).abs()
    bad = ~(off <= err) & ~(got == want)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} outside, the worst {off[bad].max()} "
                           f"where {err[bad][off[bad].argmax()]} is allowed")


# ---- kv_append ----

def append_case(g, tokens, seqs, hq, hk, d, rot, x, cache, page, max_pages):
    n_pages = seqs * max_pages + 2
    table = torch.randperm(n_pages, generator=g)[:seqs * max_pages].view(seqs, max_pages).to(torch.int32)
    spots = torch.randperm(seqs * max_pages * page, generator=g)[:tokens]
    seq, pos = spots // (max_pages * page), spots % (max_pages * page)
    angle = torch.rand((max_pages * page, rot // 2), generator=g) * 6.3
    return dict(q=randn(g, (tokens, hq, d), x), k=randn(g, (tokens, hk, d), x), v=randn(g, (tokens, hk, d), x),
                kp=randn(g, (n_pages, page, hk, d), cache), vp=randn(g, (n_pages, page, hk, d), cache), table=table,
                seq=seq.to(torch.int32), pos=pos.to(torch.int32), cos=angle.cos() if rot else None,
                sin=angle.sin() if rot else None)


def check_append(c, pairs, what, cuda=None, q_out=None):
    """Runs the call on `cuda` (the case's tensors there, or others of the same values) and checks all that it wrote."""
    ilpm = lib()
    note(f"[append] {what}")
    t = {k: (v.cuda() if v is not None else None) for k, v in c.items()}
    t.update(cuda or {})
    got = ilpm.kv_append(t["k"], t["v"], t["kp"], t["vp"], t["table"], t["seq"], t["pos"], q=t["q"], cos=t["cos"],
                         sin=t["sin"], pairs=pairs, q_out=q_out)
    torch.cuda.synchronize()
    pos = c["pos"].tolist()
    keys, err, values = ref.append(c["k"], c["v"], c["kp"], c["vp"], c["table"], c["seq"].tolist(), pos, c["cos"],
                                   c["sin"], pairs)
    written = (keys != c["kp"].double()) | (values != c["vp"].double())
    u, tiny = ref.U[c["kp"].dtype], ref.TINY[c["kp"].dtype]
    near(t["kp"], keys, torch.where(written | (err > 0), err + u * (keys.abs() + err) + tiny, 0.0), what + " keys")
    near(t["vp"], values, torch.where(written, u * values.abs() + tiny, 0.0), what + " values")
    if c["q"] is not None:
        want, err = ref.rotate(c["q"].double(), pos, c["cos"], c["sin"], pairs)
        u, tiny = ref.U[c["q"].dtype], ref.TINY[c["q"].dtype]
        near(got, want, torch.where(err > 0, err + u * (want.abs() + err) + tiny, 0.0), what + " queries")


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("tokens,seqs,hq,hk,d,rot,page", [
    (1, 1, 1, 1, 2, 2, 1), (1, 1, 8, 2, 64, 64, 16), (5, 3, 6, 3, 80, 32, 17), (33, 4, 5, 5, 7, 6, 3),
    (64, 64, 32, 8, 128, 128, 16), (130, 2, 7, 1, 256, 128, 32), (9, 2, 4, 4, 72, 0, 16), (17, 3, 3, 2, 96, 96, 64)])
@pytest.mark.parametrize("pairs", [False, True])
def test_append(x, cache, tokens, seqs, hq, hk, d, rot, page, pairs):
    c = append_case(gen(tokens * 1000 + d), tokens, seqs, hq, hk, d, rot, x, cache, page, -(-2 * tokens // (seqs * page)) + 1)
    check_append(c, pairs, f"{x}->{cache} {tokens}x({hq},{hk})x{d} rot {rot} page {page} pairs {pairs}")


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("pairs", [False, True])
def test_append_heads_that_do_not_divide(x, cache, pairs):
    """What turns, what does not and whole heads of every remainder to a multiple of eight: copied and in place."""
    g = gen(17)
    for d, rot in [(d, rot) for d in (8, 9, 15, 21, 36, 75) for rot in range(0, d + 1, 2)]:
        c = append_case(g, 5, 2, 3, 1, d, rot, x, cache, 16, 2)
        check_append(c, pairs, f"d {d} rot {rot}")
        if rot and rot % 6 == 0:
            q = c["q"].cuda()
            check_append(c, pairs, f"d {d} rot {rot} in place", cuda=dict(q=q), q_out=q)


def test_append_without_queries_and_many_tokens():
    for d, rot in ((128, 128), (64, 32)):
        c = append_case(gen(d), 4000, 3, 2, 2, d, rot, BF16, BF16, 16, 100)
        c["q"] = None
        check_append(c, False, f"no queries, d {d}")


@pytest.mark.parametrize("pairs", [False, True])
def test_append_strided(pairs):
    """Slices of one packed projection, queries rotated in place in it, pools with the heads outside the slots and
    keys and values in one allocation, and everything one element off its alignment."""
    g = gen(11)
    for d, shift in ((128, 0), (64, 1), (36, 0)):
        c = append_case(g, 37, 2, 6, 2, d, d // 2 * 2, BF16, BF16, 16, 3)
        packed = torch.empty(37 * 10 * d + shift, dtype=BF16)[shift:].view(37, 10, d)
        packed[:, :6], packed[:, 6:8], packed[:, 8:] = c["q"], c["k"], c["v"]
        gpu = torch.empty(37 * 10 * d + shift, dtype=BF16, device="cuda")[shift:].view(37, 10, d)
        gpu.copy_(packed)
        n = c["kp"].shape[0]
        pools = torch.empty((n, 2, 2, 16, d), dtype=BF16, device="cuda")   # [page][k or v][head][slot][d]
        kp, vp = pools[:, 0].transpose(1, 2), pools[:, 1].transpose(1, 2)
        kp.copy_(c["kp"])
        vp.copy_(c["vp"])
        cuda = dict(q=gpu[:, :6], k=gpu[:, 6:8], v=gpu[:, 8:], kp=kp, vp=vp)
        check_append(c, pairs, f"strided d {d} shift {shift}", cuda, q_out=gpu[:, :6])
        assert torch.equal(gpu[:, 6:].cpu(), packed[:, 6:])


def test_append_leaves_out_what_names_no_place():
    c = append_case(gen(5), 12, 3, 4, 2, 64, 64, F32, BF16, 16, 2)
    c["seq"][:4] = torch.tensor([-1, 3, -2 ** 31, 2 ** 31 - 1])
    c["pos"][4:9] = torch.tensor([-1, 32, 2 ** 31 - 1, -2 ** 31, 33])
    c["table"][int(c["seq"][9]), int(c["pos"][9]) // 16] = -1
    c["table"][int(c["seq"][10]), int(c["pos"][10]) // 16] = c["kp"].shape[0]
    check_append(c, False, "no place")
    c["cos"], c["sin"] = c["cos"][:5], c["sin"][:5]     # positions beyond the table of angles
    check_append(c, False, "no angle")


def test_append_nothing():
    ilpm = lib()
    c = append_case(gen(1), 2, 1, 1, 1, 64, 64, F32, F32, 16, 1)
    t = {k: v.cuda() for k, v in c.items()}
    q = ilpm.kv_append(t["k"][:0], t["v"][:0], t["kp"], t["vp"], t["table"], t["seq"][:0], t["pos"][:0], q=t["q"][:0],
                       cos=t["cos"], sin=t["sin"])
    torch.cuda.synchronize()
    assert q.shape == (0, 1, 64) and torch.equal(t["kp"].cpu(), c["kp"])


# ---- attn_decode ----

def attn_case(g, lengths, hq, hk, d, x, cache, page, q_std=1.0, poison=math.nan):
    """Sequences of these lengths on scattered pages; every slot that holds no token holds `poison`."""
    seqs, wide = len(lengths), max(1, max(-(-max(n, 0) // page) for n in lengths))
    n_pages = seqs * wide + 3
    table = torch.randperm(n_pages, generator=g)[:seqs * wide].view(seqs, wide).to(torch.int32)
    kp, vp = (torch.full((n_pages, page, hk, d), poison, dtype=cache) for _ in range(2))
    for s, n in enumerate(lengths):
        for j in range(n):
            kp[table[s, j // page], j % page] = randn(g, (hk, d), cache)
            vp[table[s, j // page], j % page] = randn(g, (hk, d), cache)
    return dict(q=randn(g, (seqs, hq, d), x, q_std), kp=kp, vp=vp, table=table, lengths=torch.tensor(lengths, dtype=torch.int32))


def check_attn(c, what, cuda=None, mask=None, gpu_mask=None, scale=None, **options):
    ilpm = lib()
    note(f"[attn] {what}")
    t = {k: v.cuda() for k, v in c.items()}
    t.update(cuda or {})
    scale = c["q"].shape[-1] ** -0.5 if scale is None else scale
    window, softcap = options.get("window", 0), options.get("softcap", 0.0)
    out, untouched = guarded(c["q"].shape, c["q"].dtype)
    lse, untouched_lse = guarded(c["q"].shape[:2], F32)
    if gpu_mask is None and mask is not None:
        gpu_mask = mask.cuda()
    ilpm.attn_decode(t["q"], t["kp"], t["vp"], t["table"], t["lengths"], scale=scale, mask=gpu_mask, out=out, lse=lse,
                     **options)
    torch.cuda.synchronize()
    want, want_lse, err, err_lse = ref.attention(c["q"], c["kp"], c["vp"], c["table"], c["lengths"], scale, window,
                                                 softcap, mask)
    assert untouched() and untouched_lse(), what + ": a write outside"
    empty = want_lse == -math.inf
    assert (out.cpu()[empty] == 0).all() and (lse.cpu()[empty] == -math.inf).all(), what + ": empty rows"
    near(out, want, err, what + " out")
    near(lse, want_lse, err_lse, what + " lse")
    return out, lse


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("d", [1, 7, 64, 72, 80, 96, 120, 128, 192, 200, 256])
def test_attention_types_and_sizes(x, cache, d):
    c = attn_case(gen(d), [0, 1, 2, 15, 16, 17, 33, 64, 65, 150], 6, 2, d, x, cache, 16)
    check_attn(c, f"{x} over {cache}, d {d}")


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("hq,hk", [(1, 1), (3, 3), (8, 2), (16, 1), (17, 1), (40, 1), (48, 2)])
def test_attention_head_layouts(x, cache, hq, hk):
    c = attn_case(gen(hq), [5, 130, 0, 31], hq, hk, 64, x, cache, 16)
    check_attn(c, f"{x} over {cache}, heads {hq}/{hk}")


@pytest.mark.parametrize("page", [1, 3, 16, 17, 64, 256])
def test_attention_page_sizes(page):
    for d, (x, cache) in ((64, (F32, F32)), (128, (BF16, BF16))):
        check_attn(attn_case(gen(page), [300, 17, page, page + 1], 4, 2, d, x, cache, page), f"page {page} d {d}")


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("hq,hk,d", [(4, 1, 128), (8, 4, 80), (2, 2, 256), (20, 1, 64)])
def test_attention_split_over_the_length(x, cache, hq, hk, d):
    """Lengths that several splits share, beside short ones in the same call."""
    c = attn_case(gen(d), [2100, 700, 1, 0, 129], hq, hk, d, x, cache, 16, q_std=2.0)
    check_attn(c, f"split {x} over {cache} ({hq},{hk})x{d}")
    check_attn(c, f"split {x} over {cache} ({hq},{hk})x{d}, max_len too small", max_len=200)
    check_attn(c, f"split {x} over {cache} ({hq},{hk})x{d}, max_len known", max_len=2100)


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("window", [1, 5, 16, 100, 1000, 5000])
def test_attention_window(x, cache, window):
    check_attn(attn_case(gen(window), [1300, 99, 100, 101, 1, 0], 4, 2, 64, x, cache, 16), f"window {window}", window=window)


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
def test_attention_softcap_and_large_scores(x, cache):
    c = attn_case(gen(8), [300, 40], 4, 2, 64, x, cache, 16, q_std=30.0)
    check_attn(c, "large scores")
    check_attn(c, "softcap", softcap=30.0)
    check_attn(c, "softcap and scale", softcap=5.0, scale=0.7)
    check_attn(c, "negative scale", scale=-0.2)
    check_attn(c, "scale 0", scale=0.0)


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_attention_masked_places_have_no_part(x, cache, bad):
    """Masked keys, keys beyond the length, keys in no page and keys out of the window hold NaN or infinities; some
    rows are left empty."""
    g = gen(21)
    c = attn_case(g, [700, 100, 33, 16, 650], 6, 3, 72, x, cache, 16, poison=bad)
    mask = torch.rand((5, 44 * 16), generator=g) < 0.7
    mask[1] = False
    mask[2, :32], mask[2, 32] = False, True
    mask[3, :15] = False
    for s in range(5):
        for j in range(int(c["lengths"][s])):
            if not mask[s, j]:
                c["kp"][c["table"][s, j // 16], j % 16] = bad
                c["vp"][c["table"][s, j // 16], j % 16] = bad
    for s, at, page in ((0, 3, -1), (0, 20, c["kp"].shape[0]), (4, 0, -2 ** 31), (4, 1, 2 ** 31 - 1)):
        c["kp"][c["table"][s, at]], c["vp"][c["table"][s, at]] = bad, bad
        c["table"][s, at] = page
    check_attn(c, f"mask, {bad}", mask=mask)
    check_attn(c, f"mask as bytes, {bad}", mask=mask, gpu_mask=(mask.to(torch.uint8) * 128).cuda())
    check_attn(c, f"mask and window, {bad}", mask=mask, window=40)
    check_attn(c, f"short mask, {bad}", mask=mask[:, :50])
    wide = torch.zeros((5, 1000), dtype=torch.bool, device="cuda")
    wide[:, 7:7 + mask.shape[1]] = mask.cuda()
    check_attn(c, f"strided mask, {bad}", mask=mask, gpu_mask=wide[:, 7:7 + mask.shape[1]])


def test_attention_without_a_key_anywhere():
    c = attn_case(gen(2), [40, 1, 0], 4, 2, 64, BF16, BF16, 16)
    c["table"][:] = -1
    check_attn(c, "no pages")
    c["lengths"] = torch.tensor([-5, 0, -2 ** 31], dtype=torch.int32)
    check_attn(c, "no lengths")
    c = attn_case(gen(2), [40], 4, 2, 64, F32, F32, 16)
    check_attn(c, "all masked", mask=torch.zeros((1, 48), dtype=torch.bool))
    check_attn(c, "mask of no keys", mask=torch.zeros((1, 0), dtype=torch.bool))
    ilpm = lib()
    t = {k: v.cuda() for k, v in c.items()}
    out, lse = ilpm.attn_decode(t["q"][:0], t["kp"], t["vp"], t["table"][:0], t["lengths"][:0], return_lse=True)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    out, lse = ilpm.attn_decode(t["q"], t["kp"][:0], t["vp"][:0], t["table"], t["lengths"], return_lse=True)
    torch.cuda.synchronize()
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("seqs,hq,hk,d", [(600, 4, 2, 64), (70, 17, 1, 72), (90, 5, 5, 33), (1300, 1, 1, 64)])
def test_attention_of_many_sequences(seqs, hq, hk, d):
    """More units than workgroups and fewer, some of which begin in one workgroup and end in another."""
    g = gen(seqs)
    lengths = torch.randint(0, 300, (seqs,), generator=g).tolist()
    lengths[seqs // 2], lengths[-1] = 3001, 1777
    c = attn_case(g, lengths, hq, hk, d, F32, BF16, 64)
    check_attn(c, f"{seqs} sequences")
    check_attn(c, f"{seqs} sequences, window", window=290)


def test_attention_length_beyond_the_table():
    c = attn_case(gen(4), [48, 48], 4, 2, 64, BF16, BF16, 16)
    c["lengths"] = torch.tensor([1000, 2 ** 31 - 1], dtype=torch.int32)
    check_attn(c, "beyond the table")
    check_attn(c, "beyond the table, window", window=970)


@pytest.mark.parametrize("x,cache", PAIRS, ids=str)
def test_attention_keys_that_are_not_finite(x, cache):
    """What is seen counts: NaN and infinities in it reach the rows that see them, and no others."""
    ilpm = lib()
    c = attn_case(gen(6), [200, 200, 200, 200], 4, 2, 64, x, cache, 16)
    c["kp"][c["table"][0, 3], 5, 0, 7] = math.nan       # heads 0 and 1 of sequence 0
    c["vp"][c["table"][1, 3], 5, 1, 7] = math.inf       # element 7 of heads 2 and 3 of sequence 1
    c["q"][2, 1] = 0.0
    c["q"][2, 1, 0], c["kp"][c["table"][2, 0], 3, 0, 0] = 1.0, math.inf   # a score of +inf
    c["kp"][c["table"][3, 0], 3, 0] = 0.0
    c["kp"][c["table"][3, 0], 3, 0, 0], c["q"][3, 0, 0], c["q"][3, 1, 0] = -math.inf, 1.0, 2.0   # scores of -inf
    note(f"[attn] not finite, {x} over {cache}")
    t = {k: v.cuda() for k, v in c.items()}
    out, lse = (o.double().cpu() for o in ilpm.attn_decode(*t.values(), return_lse=True))
    want, want_lse, err, err_lse = ref.attention(c["q"], c["kp"], c["vp"], c["table"], c["lengths"], 0.125)
    assert torch.isnan(out[0, :2]).all() and torch.isnan(lse[0, :2]).all()
    assert out[1, 2, 7] == out[1, 3, 7] == math.inf
    assert torch.isnan(out[2, 1]).all()
    assert torch.isfinite(out[0, 2:]).all() and torch.isfinite(out[1, :2]).all() and torch.isfinite(out[3]).all()
    fine = torch.isfinite(want)
    near(out[fine], want[fine], err[fine], "finite outputs")


def test_attention_strided():
    """Queries out of a packed projection, outputs into a wider buffer and over the queries themselves, pools with the
    heads outside the slots, keys and values in one allocation, a shared table, and everything off its alignment."""
    g = gen(31)
    for d, shift, (x, cache) in ((128, 0, (BF16, BF16)), (64, 1, (BF16, BF16)), (80, 0, (F32, F16)), (64, 3, (F32, F32)),
                                 (256, 4, (F16, F16))):
        c = attn_case(g, [150, 40, 65], 6, 2, d, x, cache, 16)
        packed = torch.zeros((3, 10, d), dtype=x, device="cuda")
        packed[:, 2:8] = c["q"].cuda()
        n = c["kp"].shape[0]
        pools = torch.empty(n * 2 * 2 * 16 * d + shift, dtype=cache, device="cuda")[shift:].view(n, 2, 2, 16, d)
        kp, vp = pools[:, 0].transpose(1, 2), pools[:, 1].transpose(1, 2)
        kp.copy_(c["kp"])
        vp.copy_(c["vp"])
        out, _ = check_attn(c, f"strided d {d} shift {shift}", dict(q=packed[:, 2:8], kp=kp, vp=vp))
        lib().attn_decode(packed[:, 2:8], kp, vp, c["table"].cuda(), c["lengths"].cuda(), out=packed[:, 2:8])
        torch.cuda.synchronize()
        assert torch.equal(packed[:, 2:8], out) and (packed[:, :2] == 0).all() and (packed[:, 8:] == 0).all()
    c = attn_case(g, [100], 4, 2, 64, BF16, BF16, 16)
    q, lengths = randn(g, (100, 4, 64), BF16), torch.arange(1, 101, dtype=torch.int32)
    one = dict(c, q=q, table=c["table"].expand(100, -1), lengths=lengths)   # a prompt's rows over its own keys
    check_attn(one, "shared table", dict(table=c["table"].cuda().expand(100, -1)))


def test_attention_workspaces():
    ilpm = lib()
    c = attn_case(gen(9), [1500, 900], 8, 2, 128, BF16, BF16, 16)
    t = {k: v.cuda() for k, v in c.items()}
    need = ilpm.attn_decode_workspace_size(t["kp"], t["vp"], t["table"], 8)
    assert need > 0
    want = ilpm.attn_decode(*t.values())
    ws = torch.full((need + 512,), 255, dtype=torch.uint8, device="cuda")   # NaN bytes
    got = ilpm.attn_decode(*t.values(), workspace=ws[:need])
    torch.cuda.synchronize()
    assert torch.equal(got, want) and (ws[need:] == 255).all()
    with pytest.raises(ilpm.IlpmError) as e:
        ilpm.attn_decode(*t.values(), workspace=ws[:need - 1])
    assert e.value.status == ilpm.ERR_WORKSPACE
    with pytest.raises(ilpm.IlpmError) as e:
        ilpm.attn_decode(*t.values(), workspace=ws[16:])
    assert e.value.status == ilpm.ERR_INVALID_ARG
    # Without one the C call takes the workspace of the split plans.
    out = torch.empty_like(want)
    call = (decode_abi.cache(t["kp"], t["vp"], t["table"], ilpm.BF16), decode_abi.heads(t["q"], ilpm.BF16),
            t["lengths"].data_ptr(), decode_abi.OPTIONS.pack(0, 0, 128 ** -0.5, 0.0, 0, 0, 0),
            decode_abi.heads(out, ilpm.BF16), None, None, 0, ilpm._stream_handle())
    try:
        ilpm.set_workspace(ws[:256])
        assert ilpm.lib.ilpm_attn_decode(*call) == ilpm.ERR_WORKSPACE
        ilpm.set_workspace(ws)
        assert ilpm.lib.ilpm_attn_decode(*call) == ilpm.OK
    finally:
        ilpm.set_workspace(None)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_attention_repeats_bit_for_bit_on_any_stream():
    ilpm = lib()
    c = attn_case(gen(10), [3000, 10, 1200], 8, 2, 64, F16, F16, 16)
    t = {k: v.cuda() for k, v in c.items()}
    want = ilpm.attn_decode(*t.values(), return_lse=True)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(3)], []
    for i in range(9):
        if i < 6:
            with torch.cuda.stream(streams[i % 3]):
                got.append(ilpm.attn_decode(*t.values(), return_lse=True))
        else:
            got.append(ilpm.attn_decode(*t.values(), return_lse=True, stream=streams[i % 3]))
    torch.cuda.synchronize()
    for o, l in got:
        assert torch.equal(o, want[0]) and torch.equal(l, want[1])


def test_attention_offsets_beyond_32_bits():
    """A pool of more than 2^32 elements, a sequence on its first and last pages."""
    ilpm = lib()
    d, page, hk = 128, 16, 8
    n_pages = 2 ** 32 // (d * page * hk) + 3
    kp, vp = (torch.zeros((n_pages, page, hk, d), dtype=BF16, device="cuda") for _ in range(2))
    c = attn_case(gen(12), [40], 16, hk, d, BF16, BF16, page)
    pages = torch.tensor([n_pages - 1, 0, n_pages - 2])
    kp[pages.cuda()], vp[pages.cuda()] = c["kp"][c["table"][0].long()].cuda(), c["vp"][c["table"][0].long()].cuda()
    check_attn(c, "offsets beyond 32 bits", dict(kp=kp, vp=vp, table=pages.to(torch.int32).view(1, 3).cuda()))
    k, v = randn(gen(1), (2, hk, d), BF16), randn(gen(2), (2, hk, d), BF16)
    note("[append] offsets beyond 32 bits")
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    ilpm.kv_append(k.cuda(), v.cuda(), kp, vp, table, torch.zeros(2, dtype=torch.int32, device="cuda"),
                   torch.tensor([15, 16], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    for pool, x in ((kp, k), (vp, v)):
        assert torch.equal(pool[n_pages - 1, 15].cpu(), x[0]) and torch.equal(pool[n_pages - 2, 0].cpu(), x[1])


# ---- residual_norm ----

NORM_TYPES = [(F32, F32, F32), (F16, F16, F16), (BF16, BF16, BF16), (F32, F16, F32), (F32, BF16, BF16), (BF16, BF16, F32),
              (F32, F16, F16), (F16, F16, F32), (F32, BF16, F32)]


def norm_case(g, rows, width, x, y, p, post, pre, gate, weights, bias):
    c = dict(x=randn(g, (rows, width), x, 3.0), y=randn(g, (rows, width), y) if y is not None else None, post=post, pre=pre,
             post_w=None, post_b=None, pre_w=None, pre_b=None, gate=None)
    for name, kind in (("post", post), ("pre", pre)):
        if kind is not None:
            c[name + "_w"] = (randn(g, (width,), F32, 0.2) + 1).to(p) if weights else None
            c[name + "_b"] = randn(g, (width,), p, 0.3) if bias else None
    if gate:
        c["gate"] = randn(g, (width,) if gate == "vec" else (rows, width), p)
    return c


def check_norm(c, what, scale=0.5, eps=1e-6, cuda=None, y_dtype=None):
    ilpm = lib()
    note(f"[norm] {what}")
    t = {k: (v.cuda() if isinstance(v, torch.Tensor) else v) for k, v in c.items()}
    t.update(cuda or {})
    rows, width = c["x"].shape
    y_dtype = c["y"].dtype if c["y"] is not None else y_dtype or c["x"].dtype
    outs, checks = {}, []
    if "r" not in t:
        outs["r"], ok = guarded((rows, width), c["x"].dtype)
        checks.append(ok)
    if "z" not in t and c["pre"] is not None:
        outs["z"], ok = guarded((rows, width), y_dtype)
        checks.append(ok)
    r, z = ilpm.residual_norm(**dict(t, **outs), scale=scale, eps=eps)
    torch.cuda.synchronize()
    want_r, want_z, er, ez = ref.residual_norm(c["x"], c["y"], c["post"], c["post_w"], c["post_b"], c["gate"], scale, c["pre"],
                                               c["pre_w"], c["pre_b"], eps, c["x"].dtype, y_dtype)
    assert all(ok() for ok in checks), what + ": a write outside"
    near(r, want_r, er, what + " r")
    if z is None:
        assert c["pre"] is None
    else:
        near(z, want_z, ez, what + " z")


@pytest.mark.parametrize("types", NORM_TYPES, ids=str)
@pytest.mark.parametrize("rows,width", [(1, 1), (1, 64), (3, 7), (5, 512), (2, 1000), (7, 1023), (3, 2048), (4, 4096), (2, 5120), (2, 8191)])
def test_norm_types_and_sizes(types, rows, width):
    for post, pre, gate, bias in (("rms", "rms", None, False), ("layer", "layer", "rows", True), (None, "rms", "vec", True)):
        c = norm_case(gen(width), rows, width, *types, post, pre, gate, True, bias)
        check_norm(c, f"{types} {rows}x{width} {post} {pre} gate {gate}")


@pytest.mark.parametrize("post", [None, "rms", "layer"])
@pytest.mark.parametrize("pre", [None, "rms", "layer"])
@pytest.mark.parametrize("gate", [None, "vec", "rows"])
def test_norm_kinds(post, pre, gate):
    for weights, bias, width in ((False, False, 640), (True, True, 96), (False, True, 1001)):
        check_norm(norm_case(gen(3), 4, width, F32, BF16, F32, post, pre, gate, weights, bias),
                   f"{post} {pre} {gate} weights {weights} bias {bias}", scale=-1.5)


@pytest.mark.parametrize("rows,width", [(1, 20000), (2, 16384), (2, 32768), (300, 64), (1000, 1)])
def test_norm_wide_and_many_rows(rows, width):
    for types in ((F32, F32, F32), (BF16, BF16, BF16)):
        check_norm(norm_case(gen(4), rows, width, *types, "rms", "layer", "vec", True, False), f"{types} {rows}x{width}")


def test_norm_alone_and_in_place():
    g = gen(13)
    for width in (512, 777):
        c = norm_case(g, 5, width, F32, None, F32, None, "rms", None, True, False)
        check_norm(c, "norm alone", cuda=dict(r=None))
        z = torch.empty((5, width), dtype=BF16, device="cuda")
        c["pre_w"] = None
        check_norm(c, "norm alone into bf16", cuda=dict(r=None, z=z), y_dtype=BF16)
        c = norm_case(g, 5, width, BF16, BF16, BF16, "layer", "rms", "rows", True, True)
        x, y = c["x"].cuda(), c["y"].cuda()
        check_norm(c, "in place", cuda=dict(x=x, r=x, y=y, z=y))


@pytest.mark.parametrize("rows,width", [(33000, 20), (5001, 130), (2100, 515), (1030, 2001), (600, 4090), (300, 7001), (300, 9000)])
def test_norm_in_place_over_many_rows(rows, width):
    """More rows than run at once: a row is read while the one before it is written, over itself."""
    for types in ((F32, BF16, F32), (F16, F16, F16)):
        c = norm_case(gen(width), rows, width, *types, "rms", "layer", "rows", True, True)
        x, y = c["x"].cuda(), c["y"].cuda()
        check_norm(c, f"{types} {rows}x{width}", cuda=dict(x=x, r=x, y=y, z=y))


def test_norm_of_rows_that_come_from_memory():
    """So many bytes that workgroups are launched by another rule: the rows are those of calls of a few of them."""
    ilpm = lib()
    g = torch.Generator(device="cuda").manual_seed(8)
    x, y = (torch.randn((11000, 4088), generator=g, device="cuda").to(BF16) for _ in range(2))
    w = torch.randn(4088, generator=g, device="cuda").to(BF16)
    r, z = ilpm.residual_norm(x, y, post="rms", pre="layer", post_w=w, pre_b=w)
    for i in (0, 511, 5300, 10990):
        some_r, some_z = ilpm.residual_norm(x[i:i + 10], y[i:i + 10], post="rms", pre="layer", post_w=w, pre_b=w)
        assert torch.equal(r[i:i + 10], some_r) and torch.equal(z[i:i + 10], some_z)
    assert torch.isfinite(r).all() and torch.isfinite(z).all()


def test_norm_strided():
    g = gen(14)
    for width, shift in ((512, 0), (512, 8), (512, 1), (1000, 0), (77, 3)):
        c = norm_case(g, 6, width, BF16, BF16, F32, "rms", "layer", "rows", True, True)
        cuda = {}
        for name in ("x", "y", "gate"):
            wide = torch.full((6, 2 * width + 16), math.nan, dtype=c[name].dtype, device="cuda")
            cuda[name] = wide[:, shift:shift + width]
            cuda[name].copy_(c[name])
        out = torch.full((6, 2 * width + 20), math.nan, dtype=BF16, device="cuda")
        cuda["r"], cuda["z"] = out[:, shift:shift + width], out[:, shift + width + 2:shift + 2 * width + 2]
        for name in ("post_w", "pre_b"):
            cuda[name] = torch.empty(width + shift, dtype=F32, device="cuda")[shift:]
            cuda[name].copy_(c[name])
        check_norm(c, f"strided {width} shift {shift}", cuda=cuda)
        rest = torch.ones_like(out, dtype=torch.bool)
        rest[:, shift:shift + width] = rest[:, shift + width + 2:shift + 2 * width + 2] = False
        assert torch.isnan(out[rest]).all(), "a write outside"


def test_norm_of_rows_that_are_far_from_zero_or_all_alike():
    """The variance is taken from the deviations: a mean a thousand times the spread costs only what the bounds give it."""
    g = gen(15)
    c = norm_case(g, 3, 1024, F32, F32, F32, "layer", "layer", None, True, False)
    c["y"] += 1000.0
    c["x"] -= 3000.0
    check_norm(c, "far from zero")
    c["x"][:], c["y"][:] = 2.5, -7.0
    check_norm(c, "all alike")
    c["x"][:], c["y"][:] = 0.0, 0.0
    check_norm(c, "zeros")
    c["pre"] = c["post"] = "rms"
    check_norm(c, "zeros, rms")


def test_norm_of_rows_that_are_not_finite():
    ilpm = lib()
    for width in (512, 1001):
        x, y = torch.randn(4, width, device="cuda"), torch.randn(4, width, device="cuda")
        x[1, 3], y[2, 5] = math.nan, math.inf
        r, z = ilpm.residual_norm(x, y, post="rms", pre="layer")
        torch.cuda.synchronize()
        assert torch.isnan(z[1]).all() and torch.isnan(r[1, 3]) and torch.isfinite(r[1, :3]).all()
        assert torch.isnan(z[2]).all() and torch.isnan(r[2, 5])
        assert torch.isfinite(z[0]).all() and torch.isfinite(z[3]).all()


def test_outputs_are_ordinary_tensors():
    ilpm = lib()
    x = torch.randn((4, 64), device="cuda")
    for mode in (torch.enable_grad, torch.no_grad, torch.inference_mode):
        with mode():
            r, z = ilpm.residual_norm(x, x.half(), post="rms")
            for t, dtype in ((r, F32), (z, F16)):
                assert t.device == x.device and t.dtype == dtype and t.is_contiguous() and not t.requires_grad
                assert t.untyped_storage().device == x.device and t.is_inference() == (mode is torch.inference_mode)
                assert torch.equal(t.clone(), t) and torch.isfinite(t * 2).all()
    w = torch.ones(64, device="cuda", requires_grad=True)
    (ilpm.residual_norm(x, x)[0] * w).sum().backward()
    assert torch.isfinite(w.grad).all()
    del r, z, t
    held = torch.cuda.memory_allocated()
    r, z = ilpm.residual_norm(x, x)
    assert torch.cuda.memory_allocated() == held + 2 * 4 * 64 * 4
    del r, z
    assert torch.cuda.memory_allocated() == held


def test_norm_nothing():
    r, z = lib().residual_norm(torch.empty((0, 64), device="cuda"), torch.empty((0, 64), device="cuda"))
    assert r.shape == z.shape == (0, 64)


# ---- together ----

def test_a_captured_step_replays_with_new_inputs():
    """Append, attention and norm in one graph: each replay, with other inputs and lengths in the same buffers and
    eager work between, gives the eager call's bits."""
    ilpm = lib()
    g = gen(17)
    c = attn_case(g, [700, 260], 8, 2, 64, BF16, BF16, 16)
    t = {k: v.cuda() for k, v in c.items()}
    k, v = torch.empty((2, 2, 64), dtype=BF16, device="cuda"), torch.empty((2, 2, 64), dtype=BF16, device="cuda")
    q, x = torch.empty((2, 8, 64), dtype=BF16, device="cuda"), torch.empty((2, 512), dtype=F32, device="cuda")
    seq, pos = torch.arange(2, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    angle = torch.rand((704, 32), generator=g) * 6.3
    cos, sin = angle.cos().cuda(), angle.sin().cuda()

    def step():
        qr = ilpm.kv_append(k, v, t["kp"], t["vp"], t["table"], seq, pos, q=q, cos=cos, sin=sin)
        out = ilpm.attn_decode(qr, t["kp"], t["vp"], t["table"], t["lengths"])
        return ilpm.residual_norm(x, out.view(2, 512), post="rms", pre="layer")

    def fill(i):
        for b, std in ((k, 1.0), (v, 1.0), (q, 1.0), (x, 3.0)):
            b.copy_(randn(gen(100 + i), b.shape, b.dtype, std))
        pos.copy_(torch.tensor([(690, 3, 402)[i % 3], (0, 258, 100)[i % 3]]))
        t["lengths"].copy_(pos + 1)

    fill(0)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        r, z = step()
    for i in range(6):
        note(f"[step] replay {i}")
        fill(i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = r.clone(), z.clone()
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
