"""The 64-bit definitions that the operators of a drafted decoder step are held
to, against cases worked by hand and against each other's special cases."""
import math

import torch

import decode_ref
import draft_ref as ref

D = torch.float64


def test_nodes_above():
    assert ref.above([-1, 0, 0, 1, -1, 4, -2, 6, 9, 5]) == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [4, 5], None, None, None, [4, 5, 9]]
    assert ref.above([0, -1]) == [None, [1]]


def test_a_head_normed_and_turned():
    x = torch.tensor([[[3.0, 4.0]]], dtype=D)     # rms: 3 and 4 over sqrt(12.5)
    cos, sin = torch.tensor([[0.0]]), torch.tensor([[1.0]])
    got, err = ref.norm_rotate(x, [0], "rms", torch.tensor([2.0, 1.0]), 0.0, cos, sin, False)
    r = math.sqrt(12.5)
    assert torch.allclose(got[0, 0], torch.tensor([-4 / r, 6 / r], dtype=D), atol=1e-12) and (err > 0).all() and (err < 1e-5).all()
    got, _ = ref.norm_rotate(x, [0], "layer", None, 0.0, None, None, False)
    assert torch.allclose(got[0, 0], torch.tensor([-1.0, 1.0], dtype=D), atol=1e-12)


def test_a_single_node_is_a_decoded_token():
    g = torch.Generator().manual_seed(1)
    kp, vp = torch.randn((9, 4, 2, 8), generator=g), torch.randn((9, 4, 2, 8), generator=g)
    table = torch.tensor([[3, 1, 7], [0, 5, 2]], dtype=torch.int32)
    q = torch.randn((2, 4, 8), generator=g)
    for window in (0, 1, 3):
        one = ref.attention(q, kp, vp, table, [7, 0], torch.tensor([[-1], [-1]]), 0.3, window=window)
        two = decode_ref.attention(q, kp, vp, table, [8, 1], 0.3, window=window)
        assert torch.allclose(one[0], two[0], atol=1e-12) and torch.allclose(one[1], two[1], atol=1e-12)


def test_windows_go_by_places_and_keep_sinks():
    tree = ref.above([-1, 0, 0, 2])    # depths 0 1 1 2
    table = torch.arange(8).view(1, 8)
    def seen(node, window, sinks):
        return [p for p, _ in ref.seen_keys(8, 1, table, 4, 0, tree, node, 4, window, sinks, None)]
    assert seen(3, 0, 0) == [0, 1, 2, 3, 4, 6, 7]
    assert seen(3, 3, 0) == [4, 6, 7]          # places 4, 5, 6
    assert seen(3, 2, 1) == [0, 6, 7]
    assert seen(1, 1, 2) == [0, 1, 5]
    assert seen(1, 3, 5) == [0, 1, 2, 3, 4, 5]


def test_the_walk():
    p = torch.tensor([[[0.5, 0.25, 0.25], [0.0, 1.0, 0.0], [0.25, 0.0, 0.75], [1.0, 0.0, 0.0]]])
    tokens, tree = torch.tensor([[9, 0, 1, 2]]), torch.tensor([[-1, 0, 0, 2]])
    # Node 1 is kept below 0.5; else node 2 below 0.25 of the half that is left.
    assert ref.verify(tokens, tree, p, torch.tensor([[0.0, 0.49, 0.0, 0.0]])) == ([[0, 1, -1, -1]], [2], [1])
    assert ref.verify(tokens, tree, p, torch.tensor([[0.9, 0.5, 0.49, 0.9]])) == ([[0, 2, -1, -1]], [2], [0])
    assert ref.verify(tokens, tree, p, torch.tensor([[0.9, 0.5, 0.49, 0.7]])) == ([[0, 2, 3, -1]], [3], [0])
    assert ref.verify(tokens, tree, p, torch.tensor([[0.0, 0.5, 0.5, 0.0]])) == ([[0, -1, -1, -1]], [1], [2])


def test_the_walk_with_draft_rows():
    p = torch.tensor([[[0.5, 0.25, 0.25], [0.2, 0.3, 0.5], [1.0, 0.0, 0.0]]])
    q = torch.tensor([[[0.25, 0.75, 0.0], [0.2, 0.3, 0.5], [1.0, 0.0, 0.0]]])
    tokens, tree = torch.tensor([[9, 1, 2]]), torch.tensor([[-1, 0, 0]])
    # Token 1 is kept below 1/3; what is left of the row then is 0.25, 0, 0.25.
    assert ref.verify(tokens, tree, p, torch.tensor([[0.55, 0.33, 0.0]]), q) == ([[0, 1, -1]], [2], [2])
    # Token 2, which the draft never gives, is kept from any number.
    assert ref.verify(tokens, tree, p, torch.tensor([[0.0, 0.34, 0.99]]), q) == ([[0, 2, -1]], [2], [0])
    tokens = torch.tensor([[9, 1, 1]])
    # Refused twice: max(2 * (0.25, 0, 0.25) - q, 0) = 0.25, 0, 0.5.
    assert ref.verify(tokens, tree, p, torch.tensor([[0.34, 0.34, 0.0]]), q) == ([[0, -1, -1]], [1], [2])
    assert ref.verify(tokens, tree, p, torch.tensor([[0.33, 0.34, 0.0]]), q) == ([[0, -1, -1]], [1], [0])


def test_the_walk_keeps_the_targets_distribution():
    """Over all outcomes of two drafted children and the random numbers on a grid, the first token after the root comes
    out as often as its probability says."""
    p, q = torch.tensor([0.5, 0.3125, 0.1875]), torch.tensor([0.25, 0.25, 0.5])
    grid = (torch.arange(16) + 0.5) / 16
    for draft in (False, True):
        share = torch.zeros(3, dtype=D)
        kids = [(a, b, float(q[a] * q[b])) for a in range(3) for b in range(3)] if draft else [(2, 0, 1.0)]
        for a, b, odds in kids:
            u = torch.cartesian_prod(grid, grid, grid)
            n = len(u)
            tokens, tree = torch.tensor([[9, a, b]]).expand(n, 3), torch.tensor([[-1, 0, 0]]).expand(n, 3)
            rows = [t.expand(n, 3, 3) for t in (p, q)]
            path, count, last = ref.verify(tokens, tree, rows[0], u, rows[1] if draft else None)
            for w, c, x in zip(path, count, last):
                share[(a, b)[w[1] - 1] if c > 1 else x] += odds / n
        assert (share - p).abs().max() < 0.03, share   # (a threshold between two places of the grid moves a share by up to 1/32)


def test_copies_read_before_they_write():
    pool = torch.arange(6).view(6, 1)
    table = torch.arange(6).view(1, 6)
    assert ref.copy(pool, table, table, [1], [1], [3], torch.tensor([[2, 0, 0]]), 3).flatten().tolist() == [0, 3, 1, 1, 4, 5]
    assert ref.copy(pool, table, table, [4], [0], [9], None, 9).flatten().tolist() == [4, 5, 2, 3, 4, 5]
