"""GPU: how many bits of scores and of probabilities attention keeps under 32-bit queries (tests/decode_exact.py derives
the bounds, tests/test_decode_exact.py shows what they tell apart), for every element of a query, every head size's
kernel, tiles of one wave and of several, one workgroup a unit and several."""
import pytest
import torch

import decode_exact as exact
from gpu_common import note, torch_cuda

pytestmark = pytest.mark.gpu
CACHES = [torch.float32, torch.float16, torch.bfloat16]
SIZES = [5, 64, 72, 80, 96, 128, 192, 256]
PAGE = 16


def call(q, keys, values, seen, factor=1.0):
    """attn_decode of sequences that share one paged cache [keys][kv_heads][d], sequence s seeing the keys seen[s]."""
    torch_cuda()
    import paper_1909_02765_amd as ilpm
    n, pages = q.shape[0], -(-keys.shape[0] // PAGE)
    mask = torch.zeros((n, pages * PAGE), dtype=torch.bool)
    mask.scatter_(1, seen, True)
    kp, vp = (torch.zeros((pages * PAGE, *t.shape[1:]), dtype=t.dtype) for t in (keys, values))
    kp[:keys.shape[0]], vp[:keys.shape[0]] = keys, values
    kp, vp = (t.view(pages, PAGE, *t.shape[1:]).cuda() for t in (kp, vp))
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1).expand(n, -1)
    lengths = torch.full((n,), keys.shape[0], dtype=torch.int32, device="cuda")
    out, lse = ilpm.attn_decode(q.cuda(), kp, vp, table, lengths, scale=factor, mask=mask.cuda(), return_lse=True)
    torch.cuda.synchronize()
    return out.double().cpu(), lse.double().cpu()


@pytest.mark.parametrize("cache", CACHES, ids=str)
@pytest.mark.parametrize("d", SIZES)
@pytest.mark.parametrize("keys,kv_heads", [(0, 1), (600, 2)])  # (0: as many keys as elements)
def test_scores_keep_32_bits(cache, d, keys, kv_heads):
    g = torch.Generator().manual_seed(d)
    # Key j is 1 at element j % d; sequence s sees one key of its own.
    n = d if keys == 0 else 30
    count = max(keys, d)
    own = torch.arange(d) if keys == 0 else torch.randperm(keys, generator=g)[:n]
    k = exact.one_hot(torch.arange(count) % d, d).unsqueeze(1).expand(-1, kv_heads, -1).to(cache)
    v = torch.ones((count, kv_heads, d), dtype=cache)
    q = exact.full_mantissas(g, (n, 16 * kv_heads, d), 0.5, 2.0)
    note(f"[attn] scores, {cache}, d {d}, {count} keys")
    out, lse = call(q, k, v, own.unsqueeze(1))
    want = q.double()[torch.arange(n), :, own % d]
    off = (lse - want).abs() / (exact.SCORE * want.abs())
    assert off.max() <= 1, off.max()
    assert (out == 1).all()


@pytest.mark.parametrize("d", SIZES)
def test_scores_are_the_same_bits_over_every_cache(d):
    """One-hot keys are exact in each type, and three parts hold all of a query: what follows is the same arithmetic.
    (The last bit of 32 is in the third part of f16 as of bf16.)"""
    q = exact.full_mantissas(torch.Generator().manual_seed(d), (d, 16, d), 0.5, 2.0)
    note(f"[attn] the same scores over every cache, d {d}")
    got = [call(q, exact.one_hot(torch.arange(d), d).unsqueeze(1).to(cache), torch.ones((d, 1, d), dtype=cache),
                torch.arange(d).unsqueeze(1))[1] for cache in CACHES]
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


@pytest.mark.parametrize("cache", CACHES, ids=str)
@pytest.mark.parametrize("d", SIZES)
# The second key: of the same tile, of another wave's, of another tile of the wave; few keys and many.
@pytest.mark.parametrize("keys,apart", [(16, 5), (40, 17), (200, 70), (700, 3), (700, 300)])
def test_probabilities_keep_32_bits(cache, d, keys, apart):
    g = torch.Generator().manual_seed(keys + d)
    n = 12
    first = torch.randint(0, keys - apart, (n,), generator=g)
    # A sequence's first key scores 0 by its query, the second -x: of keys that are one-hot at an element of their own.
    at = torch.stack((torch.randint(0, d - 1, (n,), generator=g), torch.full((n,), d - 1)), 1)
    q = torch.zeros((n, 16, d))
    x = exact.full_mantissas(g, (n, 16), 1 / 64, 1 / 32).abs()
    q[torch.arange(n), :, at[:, 0]] = -x
    note(f"[attn] probabilities, {cache}, d {d}, {keys} keys, {apart} apart")
    outs, lses = [], []
    for s in range(n):  # a cache of its own for each
        k, v = torch.zeros((keys, 1, d), dtype=cache), torch.zeros((keys, 1, d), dtype=cache)
        seen = torch.tensor([[int(first[s]), int(first[s]) + apart]])
        k[seen[0], 0, at[s].flip(0)] = 1.0
        v[seen[0, 0]], v[seen[0, 1]] = 1.0, -1.0
        out, lse = call(q[s:s + 1], k, v, seen)
        outs.append(out)
        lses.append(lse)
    out, lse = torch.cat(outs), torch.cat(lses)
    want, want_lse = exact.expected_of_two(x.double())
    off, off_lse = (out - want.unsqueeze(-1)).abs() / exact.OUT, (lse - want_lse).abs() / exact.LSE
    assert off.max() <= 1, off.max()
    assert off_lse.max() <= 1, off_lse.max()


@pytest.mark.parametrize("x", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("keys,apart", [(16, 5), (700, 300)])
def test_lse_keeps_32_bits_under_16_bit_queries(x, keys, apart):
    g = torch.Generator().manual_seed(keys)
    q = torch.zeros((1, 64, 128), dtype=x)
    q[:, :, 0] = -exact.full_mantissas(g, (1, 64), 1 / 64, 1 / 32).abs().to(x)
    k, v = torch.zeros((keys, 4, 128), dtype=x), torch.ones((keys, 4, 128), dtype=x)
    k[apart, :, 0] = 1.0
    note(f"[attn] lse, {x}, {keys} keys")
    out, lse = call(q, k, v, torch.tensor([[0, apart]]))
    _, want = exact.expected_of_two(-q[:, :, 0].double())
    assert ((lse - want).abs() <= exact.LSE).all() and (out == 1).all()


@pytest.mark.parametrize("cache", CACHES, ids=str)
@pytest.mark.parametrize("keys", [2, 600])
def test_queries_up_to_the_largest_value(cache, keys):
    """Finite queries beyond the range of 16-bit types, under a scale that leaves scores of magnitude 256: no part of
    them is infinite, and a key that is 0 there scores 0."""
    top = torch.finfo(torch.float32).max
    rows = torch.tensor([top, -top, 3.3962e38, 3.3961e38, 3.3895314e38, 3.39e38, -3.4e38, 1e38])
    q = torch.zeros((len(rows), 16, 64))
    q[:, :, 37] = rows.unsqueeze(1)
    q[:, :, 11] = 1.0
    k, v = torch.zeros((keys, 1, 64), dtype=cache), torch.ones((keys, 1, 64), dtype=cache)
    k[1, 0, 37] = 1.0   # key 1 scores by the large element, key 0 by none
    note(f"[attn] largest queries, {cache}, {keys} keys")
    out, lse = call(q, k, v, torch.tensor([[0, 1]]).expand(len(rows), -1), factor=2.0 ** -120)
    x = rows.double() * 2.0 ** -120
    want = torch.logsumexp(torch.stack((torch.zeros_like(x), x)), 0).unsqueeze(1)
    assert ((lse - want).abs() <= exact.SCORE * want.abs().clamp_min(1)).all() and (out == 1).all()
