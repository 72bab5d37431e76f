"""The bounds of tests/decode_exact.py hold for 32-bit arithmetic, and do not for a kernel that drops a part of a query
or of a probability, or that forms probabilities at a larger exponent (emulated here in 32 bits on the CPU)."""
import math

import pytest
import torch

import decode_exact as exact

LOG2E, LN2 = torch.tensor(math.log2(math.e), dtype=torch.float32), torch.tensor(math.log(2), dtype=torch.float32)


def in_parts(v, dtype, parts):
    """v in 32 bits as the sum of its first 16-bit parts, each what the ones before it leave, rounded."""
    total, left = torch.zeros_like(v, dtype=torch.float64), v.clone()
    for _ in range(parts):
        part = left.to(dtype).float()
        total, left = total + part.double(), left - part
    return total.float()


def score_errors(q):
    """lse of one key, by the way of base 2 in 32 bits, against the query's element: errors in units of the bound."""
    def of(kept):
        return ((kept * LOG2E * LN2).double() - q.double()).abs() / (exact.SCORE * q.double().abs())
    return of


def test_scores():
    q = exact.full_mantissas(torch.Generator().manual_seed(1), (4096,), 0.5, 2.0)
    of = score_errors(q)
    assert of(q).max() <= 1
    for dtype in (torch.bfloat16, torch.float16):
        assert torch.equal(in_parts(q, dtype, 3), q)
    assert of(in_parts(q, torch.bfloat16, 2)).max() > 10 and (of(in_parts(q, torch.bfloat16, 2)) > 1).float().mean() > 0.5
    assert (of(in_parts(q, torch.float16, 1)) > 1).float().mean() > 0.9
    # Of f16 the third part holds a last bit alone, which the bound leaves room for and equal bits do not.
    assert ((in_parts(q, torch.float16, 2) * LOG2E * LN2) != q * LOG2E * LN2).float().mean() > 0.1


def of_two(x, probability, kept, shift=0):
    """(errors of out, of lse) in units of their bounds: p = probability(score in base 2) in 32 bits, held as kept(p)."""
    s = -x.float() * LOG2E
    p = probability(s)
    one, p_held, one_held = probability(torch.zeros_like(s)), kept(p), kept(probability(torch.zeros_like(s)))
    total = one + p
    out = (one_held - p_held) / total
    lse = (torch.log2(total.double()).float() - shift) * LN2
    want, want_lse = exact.expected_of_two(x.float().double())
    return (out.double() - want).abs() / exact.OUT, (lse.double() - want_lse).abs() / exact.LSE


def exp2(s):
    return torch.exp2(s.double()).float()


def test_probabilities():
    x = exact.full_mantissas(torch.Generator().manual_seed(2), (4096,), 1 / 64, 1 / 32).abs().double()

    def scaled(dtype, parts):
        return lambda p: in_parts(p * 2.0 ** 15, dtype, parts) * 2.0 ** -15

    # 32 bits, three bf16 parts, and two f16 parts of which the second's last bit is a unit of 32 bits.
    for kept in (lambda p: p, lambda p: in_parts(p, torch.bfloat16, 3), scaled(torch.float16, 2), scaled(torch.float16, 3)):
        out, lse = of_two(x, exp2, kept)
        assert out.max() <= 1 and lse.max() <= 1
    out, _ = of_two(x, exp2, lambda p: in_parts(p, torch.bfloat16, 2))
    assert out.max() > 4 and (out > 1).float().mean() > 0.5
    out, _ = of_two(x, exp2, scaled(torch.float16, 1))
    assert (out > 1).float().mean() > 0.9
    # 2^(score + 15): the sum is rounded at a magnitude of 15.
    out, lse = of_two(x, lambda s: exp2(s + 15.0), lambda p: p, shift=15.0)
    assert out.max() > 1.2 and lse.max() > 1.2


@pytest.mark.parametrize("dtype,held", [(torch.bfloat16, 2.0 ** -17), (torch.float16, 2.0 ** -23)], ids=str)
def test_two_parts_hold_what_the_header_says(dtype, held):
    p = exact.full_mantissas(torch.Generator().manual_seed(3), (1 << 16,), 0.25, 1.0).abs()
    off = (in_parts(p * 2.0 ** 15, dtype, 2).double() * 2.0 ** -15 - p.double()).abs() / p.double()
    assert held / 2 < off.max() <= held


@pytest.mark.parametrize("x", [1 / 64, 1 / 32])
def test_two_keys_by_hand(x):
    out, lse = exact.expected_of_two(torch.tensor(x, dtype=torch.float64))
    p = math.exp(-x)
    assert abs(out - (1 - p) / (1 + p)) < 1e-15 and abs(lse - math.log(1 + p)) < 1e-15
