"""The sizes up to which the entry points of a drafted decoder step go, as include/ilpm.h states them: on the host, where one
more is refused and the last is not.  Pointers are compared, never dereferenced, and no kernel is launched (what passes the
sizes is refused for a pointer)."""
import ctypes

import pytest

import paper_1909_02765_amd as ilpm
from test_decode_abi import GB, cache, heads
from test_draft_abi import append, attn, copy, verify

BAD, LIMIT = ilpm.ERR_INVALID_ARG, ilpm.ERR_UNSUPPORTED


def wide(n, **kw):
    """A cache of heads of n values."""
    return cache(dim=n, kh=n, vh=n, ks=8 * n, vs=8 * n, kp=128 * n, vp=128 * n, **kw)


@pytest.mark.parametrize("n,q_heads,got", [(1 << 24, 0, LIMIT), ((1 << 22) - 1, 0, BAD), (1 << 22, 0, LIMIT), ((1 << 20) - 1, 48, BAD), (1 << 20, 48, LIMIT)])
def test_append_of_many_tokens(n, q_heads, got):
    """With 16 heads of keys and values: 2^26 - 4 heads in all.  (Positions that lie in the pool are refused later.)"""
    q = dict(q=heads(200 * GB, q_heads), q_out=heads(400 * GB, q_heads)) if q_heads else dict(q=None, q_out=None, q_w=None)
    assert append(n=n, k=heads(600 * GB), v=heads(800 * GB), pos=GB, slots=None, **q) == got


def test_append_of_large_heads():
    one = dict(k=heads(4 * GB, row=9000, head=1100), v=heads(5 * GB, row=9000, head=1100), q=None, q_out=None, q_w=None, pos=GB, slots=None)
    assert append(c=wide(1024), **one) == BAD
    assert append(c=wide(1025), **one) == LIMIT


@pytest.mark.parametrize("seqs,nodes,heads_,got", [((1 << 19) - 1, 1, 32, ilpm.OK), (1 << 19, 1, 32, LIMIT), (8191, 64, 32, ilpm.OK), (8192, 64, 32, LIMIT)])
def test_attention_of_many_rows(seqs, nodes, heads_, got):
    need = ctypes.c_size_t(0)
    assert ilpm.lib.ilpm_attn_tree_workspace_size(cache(seqs=seqs), heads_, nodes, 0, 0, 0, ctypes.byref(need)) == got


def test_attention_of_large_heads():
    assert attn(c=wide(256), lengths=None) == BAD
    assert attn(c=wide(257), lengths=None) == LIMIT


def test_verification_of_many_sequences_and_tokens():
    assert verify(n=65535, tokens=None) == BAD and verify(n=65536, tokens=None) == LIMIT
    assert verify(vocab=1 << 30, tokens=None) == BAD and verify(vocab=(1 << 30) + 1, tokens=None) == LIMIT


def test_copies_of_many_rows_and_heads():
    """(Starts that lie in the pool are refused later.)"""
    assert copy(c=cache(seqs=65535), src_start=GB) == BAD and copy(c=cache(seqs=65536), src_start=GB) == LIMIT
    def big(n):
        return cache(heads=1 << 13, dim=n, kh=n, vh=n, ks=n << 13, vs=n << 13, kp=n << 17, vp=n << 17)
    assert copy(c=big(1 << 13), src_start=GB) == BAD and copy(c=big((1 << 13) + 1), src_start=GB) == LIMIT
