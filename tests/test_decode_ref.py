"""Pins of the decoder-step operators' 64-bit definitions (tests/decode_ref.py)
on cases worked out by hand, and against other ways to write them."""
import math

import numpy as np
import torch

import decode_ref as ref

D = torch.float64


def test_rotation_by_hand():
    x = torch.tensor([[[1.0, 2.0, 3.0, 4.0, 9.0]]], dtype=D)
    cos, sin = torch.tensor([[1.0, 1.0], [0.0, 0.6]], dtype=D), torch.tensor([[0.0, 0.0], [1.0, 0.8]], dtype=D)
    halves, _ = ref.rotate(x, [1], cos, sin, False)   # (1, 3) by 90 degrees, (2, 4) by acos 0.6
    torch.testing.assert_close(halves, torch.tensor([[[-3.0, 2 * .6 - 4 * .8, 1.0, 4 * .6 + 2 * .8, 9.0]]], dtype=D))
    pairs, _ = ref.rotate(x, [1], cos, sin, True)     # (1, 2) by 90 degrees, (3, 4) by acos 0.6
    torch.testing.assert_close(pairs, torch.tensor([[[-2.0, 1.0, 3 * .6 - 4 * .8, 4 * .6 + 3 * .8, 9.0]]], dtype=D))
    assert torch.equal(ref.rotate(x, [0], cos, sin, False)[0], x)
    assert torch.equal(ref.rotate(x, [2], cos, sin, False)[0], x)  # beyond the table: as it is


def test_rotated_scores_depend_on_the_distance_alone():
    half = 8
    angle = torch.arange(40, dtype=D)[:, None] * 10000.0 ** (-torch.arange(half, dtype=D) / half)
    q, k = torch.randn(1, 1, 2 * half, dtype=D), torch.randn(1, 1, 2 * half, dtype=D)
    for pairs in (False, True):
        turn = lambda x, p: ref.rotate(x, [p], angle.cos(), angle.sin(), pairs)[0].flatten()  # noqa: E731
        a, b = turn(q, 7) @ turn(k, 3), turn(q, 39) @ turn(k, 35)
        assert abs(a - b) < 1e-10


def test_append_places_tokens_by_the_table():
    pools = torch.zeros(3, 2, 1, 1), torch.zeros(3, 2, 1, 1)
    table = torch.tensor([[2, 0], [1, 7]])
    k = torch.tensor([1.0, 2.0, 3.0, 4.0, 5.0]).view(5, 1, 1)
    keys, _, values = ref.append(k, k + 10, *pools, table, [0, 0, 1, 1, -1], [1, 2, 0, 3, 0], None, None, False)
    want = torch.zeros(3, 2)
    want[2, 1], want[0, 0], want[1, 0] = 1, 2, 3   # token 3's page is none, token 4 is padding
    assert torch.equal(keys.view(3, 2).float(), want)
    assert torch.equal(values.view(3, 2).float(), torch.where(want > 0, want + 10, want))


def test_attention_by_hand():
    k, v = torch.zeros(2, 2, 1, 2), torch.zeros(2, 2, 1, 2)
    # Tokens 0..2 lie in pages 1 and 0; scores ln 1, ln 2, ln 5.
    for (page, slot), score, val in (((1, 0), 1.0, 8.0), ((1, 1), 2.0, 16.0), ((0, 0), 5.0, 24.0)):
        k[page, slot, 0] = torch.tensor([math.log(score), 77.0])
        v[page, slot, 0] = torch.tensor([val, -val])
    q, table = torch.tensor([[[2.0, 0.0]]]), torch.tensor([[1, 0]])
    out, lse, _, _ = ref.attention(q, k, v, table, [3], 0.5)
    np.testing.assert_allclose(out.flatten(), [(8 + 32 + 120) / 8, -(8 + 32 + 120) / 8], rtol=1e-6)
    np.testing.assert_allclose(lse, [[math.log(8)]], rtol=1e-6)
    out, lse, _, _ = ref.attention(q, k, v, table, [3], 0.5, window=2)
    np.testing.assert_allclose(out.flatten()[0], (32 + 120) / 7, rtol=1e-6)
    out, lse, _, _ = ref.attention(q, k, v, table, [3], 0.5, mask=torch.tensor([[True, True, False]]))
    np.testing.assert_allclose(out.flatten()[0], 40 / 3, rtol=1e-6)
    out, lse, _, _ = ref.attention(q, k, v, table, [0], 0.5)
    assert torch.equal(out, torch.zeros_like(out)) and lse.item() == -math.inf
    out, _, _, _ = ref.attention(q, k, v, table, [3], 0.5, softcap=1e-9)  # all scores alike
    np.testing.assert_allclose(out.flatten()[0], 16.0, rtol=1e-6)


def test_attention_agrees_with_a_dense_softmax():
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(s, generator=g, dtype=D) for s in ((2, 6, 5), (4, 3, 2, 5), (4, 3, 2, 5)))
    table = torch.tensor([[3, 0], [1, 2]])
    out, lse, _, _ = ref.attention(q.float(), k, v, table, [6, 5], 0.3)
    for s, n in ((0, 6), (1, 5)):
        ks, vs = (t[table[s]].reshape(6, 2, 5)[:n].repeat_interleave(3, 1) for t in (k, v))
        x = torch.einsum("hd,nhd->hn", q[s].float().double(), ks) * 0.3
        torch.testing.assert_close(out[s], torch.einsum("hn,nhd->hd", torch.softmax(x, 1), vs))
        torch.testing.assert_close(lse[s], torch.logsumexp(x, 1))


def test_norms_by_hand():
    x = torch.tensor([[1.0, -1.0, 3.0, 5.0]], dtype=D)
    y = torch.tensor([[2.0, 2.0, 4.0, 4.0]], dtype=D)
    f = torch.float32
    r, z, _, _ = ref.residual_norm(x, y, "layer", None, None, None, 2.0, "rms", None, None, 0.0, f, f)
    torch.testing.assert_close(r, torch.tensor([[-1.0, -3.0, 5.0, 7.0]], dtype=D))
    torch.testing.assert_close(z, r / math.sqrt(21.0))
    w, b, gate = torch.tensor([1.0, 2.0, 3.0, 4.0], dtype=D), torch.ones(4, dtype=D), torch.tensor([0.0, 1.0, 1.0, 2.0], dtype=D)
    r, z, _, _ = ref.residual_norm(x, y, "layer", w, b, gate, 1.0, None, None, None, 0.0, f, f)
    torch.testing.assert_close(r, torch.tensor([[1.0, -2.0, 7.0, 15.0]], dtype=D))
    assert z is None
    r, z, _, _ = ref.residual_norm(x, None, None, None, None, None, 1.0, "layer", None, None, 0.0, f, f)
    torch.testing.assert_close(r, x)
    torch.testing.assert_close(z, torch.tensor([[-1.0, -3.0, 1.0, 3.0]], dtype=D) / math.sqrt(5.0))


def test_bounds_hold_for_32_bit_arithmetic():
    """The definitions in 32 bits stay within the bounds, and most of the way inside."""
    g = torch.Generator().manual_seed(5)
    x, y = torch.randn(3, 257, generator=g), torch.randn(3, 257, generator=g)
    for kind in ("rms", "layer"):
        r, z, er, ez = ref.residual_norm(x, y, kind, None, None, None, 0.5, kind, None, None, 1e-6, torch.float32, torch.float32)

        def norm(v):
            v = v - v.mean(1, keepdim=True) if kind == "layer" else v
            return v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6)
        r32 = x + 0.5 * norm(y)
        assert ((r32.double() - r).abs() <= er).all() and ((norm(r32).double() - z).abs() <= ez).all()
