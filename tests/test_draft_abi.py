"""The entry points of a drafted decoder step on the host: structure layouts,
workspace sizes, and every refusal that include/ilpm.h states.  Pointers are
compared, never dereferenced, and no kernel is launched."""
import ctypes
import math
import os
import re
import shutil
import subprocess

import pytest

import draft_abi
import paper_1909_02765_amd as ilpm
from test_decode_abi import GB, ROOT, cache, heads

F32, F16, BF16 = ilpm.F32, ilpm.F16, ilpm.BF16


def test_structures_have_the_c_compilers_sizes(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "ilpm.h"\nint main(void) { printf("%zu %zu %zu\\n", sizeof(ilpm_append_options), '
                   'sizeof(ilpm_tree_options), sizeof(ilpm_verify_args)); return 0; }\n')
    subprocess.run([shutil.which("gcc"), "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include",
                    str(src), "-o", str(tmp_path / "sizes")], check=True)
    got = subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(v) for v in got] == [draft_abi.APPEND.size, draft_abi.TREE.size, draft_abi.VERIFY.size]


def test_constants_agree_with_the_header():
    text = open(os.path.join(ROOT, "include", "ilpm.h")).read()
    assert int(re.search(r"#define ILPM_MAX_NODES (\d+)", text).group(1)) == ilpm.MAX_NODES


# ---- kv_append_norm ----

def append_options(seq=8 * GB, pos=9 * GB, slots=12 * GB, cos=10 * GB, sin=11 * GB, q_w=13 * GB, k_w=14 * GB, n_pos=320, rot=128,
                   pairs=0, norm=1, param=BF16, eps=1e-6):
    return draft_abi.APPEND.pack(seq or 0, pos or 0, slots or 0, cos or 0, sin or 0, q_w or 0, k_w or 0, n_pos, rot, pairs, norm, param, eps)


def append(c=None, k=heads(4 * GB), v=heads(5 * GB), q=heads(6 * GB, 32), q_out=heads(7 * GB, 32), n=10, opt=True, **kw):
    return ilpm.lib.ilpm_kv_append_norm(cache() if c is None else c, k, v, q, q_out, append_options(**kw) if opt else None, n, None)


@pytest.mark.parametrize("kw", [
    dict(c=cache(k=0)), dict(c=cache(v=0)), dict(c=cache(table=0)), dict(c=cache(k=GB + 1)), dict(c=cache(table=3 * GB + 2)),
    dict(c=cache(size=0)), dict(c=cache(heads=0)), dict(c=cache(dim=0)), dict(c=cache(pages=-1)), dict(c=cache(seqs=-1)),
    dict(c=cache(kp=-1)), dict(c=cache(ks=1 << 41)), dict(c=cache(kp=0)), dict(c=cache(ks=128)), dict(c=cache(v=GB)),
    dict(k=None), dict(v=None), dict(k=heads(0)), dict(k=heads(4 * GB + 1)), dict(k=heads(4 * GB, 4)), dict(v=heads(5 * GB, 9)),
    dict(k=heads(4 * GB, row=-1)), dict(q=None), dict(q_out=None), dict(q_out=heads(7 * GB, 31)), dict(q_out=heads(7 * GB, 32, row=0)),
    dict(q_out=heads(6 * GB + 256, 32)), dict(q_out=heads(4 * GB, 32)), dict(q_out=heads(GB, 32)), dict(q_out=heads(8 * GB, 32)),
    dict(q_out=heads(12 * GB, 32)), dict(q_out=heads(13 * GB, 32)), dict(q_out=heads(14 * GB, 32)), dict(q_out=heads(3 * GB, 32)),
    dict(q=heads(2 * GB, 32)), dict(k=heads(GB + 4096)), dict(v=heads(GB)),
    dict(opt=False), dict(seq=None), dict(pos=None), dict(seq=8 * GB + 2), dict(pos=GB), dict(slots=2 * GB + 64), dict(slots=12 * GB + 1),
    dict(cos=None), dict(sin=None), dict(cos=10 * GB + 2), dict(cos=GB), dict(q_w=GB), dict(k_w=2 * GB), dict(q_w=13 * GB + 1),
    dict(k_w=14 * GB + 2, param=F32), dict(norm=0), dict(norm=0, q_w=None), dict(norm=0, k_w=None), dict(norm=3), dict(norm=-1),
    dict(q=None, q_out=None), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf),
    dict(n=-1), dict(n_pos=-1), dict(rot=-2), dict(rot=63), dict(rot=130), dict(pairs=2)])
def test_append_refuses(kw):
    assert append(**kw) == ilpm.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(c=cache(dtype=3)), dict(k=heads(4 * GB, dtype=7)), dict(k=heads(4 * GB, dtype=F16), v=heads(5 * GB, dtype=F16)),
    dict(k=heads(4 * GB, dtype=F32)), dict(q=heads(6 * GB, 32, dtype=F32)), dict(q_out=heads(7 * GB, 32, dtype=F32)),
    dict(param=F16), dict(param=9), dict(c=cache(dim=1025, kh=1025, vh=1025, ks=8 * 1025, vs=8 * 1025, kp=128 * 1025, vp=128 * 1025)),
    dict(n=1 << 24, k=heads(20 * GB), v=heads(60 * GB), q=None, q_out=None, q_w=None)])
def test_append_does_not_support(kw):
    assert append(**kw) == ilpm.ERR_UNSUPPORTED


def test_append_of_nothing_is_fine():
    assert append(n=0) == ilpm.OK
    assert append(n=0, k=heads(0), v=heads(0), q=None, q_out=None, q_w=None, seq=None, pos=None, slots=None) == ilpm.OK


# ---- attn_tree ----

def options(mask=0, mstride=0, scale=0.1, cap=0.0, mlen=0, window=0, sinks=0, max_len=0):
    return draft_abi.TREE.pack(mask, mstride, scale, cap, mlen, window, sinks, max_len)


def attn(c=None, q=heads(4 * GB, 32), lengths=5 * GB, parents=10 * GB, nodes=7, opt=None, out=heads(6 * GB, 32), lse=7 * GB,
         ws=8 * GB, ws_bytes=GB):
    return ilpm.lib.ilpm_attn_tree(cache() if c is None else c, q, lengths, parents, nodes, options() if opt is None else opt, out,
                                   lse, ws, ws_bytes, None)


@pytest.mark.parametrize("kw", [
    dict(c=cache(k=0)), dict(c=cache(v=0)), dict(c=cache(table=0)), dict(c=cache(size=0)), dict(c=cache(kp=-1)),
    dict(c=cache(v=2 * GB + 1)), dict(q=None), dict(out=None), dict(lengths=None), dict(parents=None), dict(q=heads(0, 32)),
    dict(out=heads(0, 32)), dict(q=heads(4 * GB, 30), out=heads(6 * GB, 30)), dict(q=heads(4 * GB, 0), out=heads(6 * GB, 0)),
    dict(q=heads(4 * GB, 30)), dict(q=heads(4 * GB + 1, 32)), dict(lengths=5 * GB + 1), dict(parents=10 * GB + 2), dict(lse=7 * GB + 2),
    dict(ws=8 * GB + 128), dict(nodes=-1),
    dict(opt=options(window=-1)), dict(opt=options(sinks=-1)), dict(opt=options(max_len=-1)), dict(opt=options(scale=math.nan)),
    dict(opt=options(scale=math.inf)), dict(opt=options(cap=-1.0)), dict(opt=options(cap=math.nan)), dict(opt=options(cap=math.inf)),
    dict(opt=options(scale=3e38)), dict(opt=options(cap=3e38)), dict(opt=options(cap=1e-40)),
    dict(opt=options(mask=9 * GB, mlen=-1)), dict(opt=options(mask=9 * GB, mlen=320, mstride=-320)),
    dict(out=heads(6 * GB, 32, row=0)), dict(out=heads(6 * GB, 32, head=64)),   # outputs that name a place twice
    dict(out=heads(4 * GB + 256, 32)), dict(out=heads(GB, 32)), dict(out=heads(2 * GB, 32)), dict(out=heads(3 * GB, 32)),
    dict(out=heads(5 * GB, 32)), dict(out=heads(10 * GB, 32)), dict(lse=4 * GB), dict(lse=6 * GB), dict(lse=GB), dict(lse=3 * GB),
    dict(lse=5 * GB), dict(lse=10 * GB), dict(opt=options(mask=6 * GB, mlen=320, mstride=320)),
    dict(opt=options(mask=7 * GB, mlen=320, mstride=320))])
def test_attention_refuses(kw):
    assert attn(**kw) == ilpm.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(c=cache(dtype=5)), dict(q=heads(4 * GB, 32, dtype=F16)), dict(out=heads(6 * GB, 32, dtype=F32)),
    dict(q=heads(4 * GB, 32, dtype=F16), out=heads(6 * GB, 32, dtype=F16)), dict(nodes=65),
    dict(c=cache(dim=257, kh=257, vh=257, ks=8 * 257, vs=8 * 257, kp=128 * 257, vp=128 * 257)),
    dict(c=cache(seqs=1 << 20), nodes=16, q=heads(400 * GB, 32), out=heads(600 * GB, 32))])
def test_attention_does_not_support(kw):
    assert attn(**kw) == ilpm.ERR_UNSUPPORTED


def test_attention_of_nothing_is_fine():
    assert attn(c=cache(seqs=0)) == ilpm.OK
    assert attn(nodes=0, parents=None) == ilpm.OK


def test_attention_workspace_sizes():
    need = ctypes.c_size_t(7)
    size = ilpm.lib.ilpm_attn_tree_workspace_size
    assert size(cache(), 32, 7, 0, 0, 0, None) == ilpm.ERR_INVALID_ARG
    assert size(cache(), 31, 7, 0, 0, 0, ctypes.byref(need)) == ilpm.ERR_INVALID_ARG
    assert size(cache(), 32, 65, 0, 0, 0, ctypes.byref(need)) == ilpm.ERR_UNSUPPORTED
    assert size(cache(), 32, -1, 0, 0, 0, ctypes.byref(need)) == ilpm.ERR_INVALID_ARG
    assert size(cache(k=0, v=0, table=0), 32, 7, 0, 0, 0, ctypes.byref(need)) == ilpm.OK
    assert size(cache(seqs=0), 32, 7, 0, 0, 0, ctypes.byref(need)) == ilpm.OK and need.value == 0


# ---- verify_drafts ----

def verify(tokens=GB, parents=2 * GB, target=10 * GB, draft=20 * GB, strides=(7 * 1000, 1000, 7 * 1000, 1000), uniforms=3 * GB, path=4 * GB,
           counts=5 * GB, last=6 * GB, n=4, nodes=7, vocab=1000, dtype=F32, ws=7 * GB, ws_bytes=GB):
    args = draft_abi.VERIFY.pack(tokens or 0, parents or 0, target or 0, draft or 0, *strides, uniforms or 0, path or 0, counts or 0,
                                 last or 0, n, nodes, vocab, dtype)
    return ilpm.lib.ilpm_verify_drafts(args, ws, ws_bytes, None)


@pytest.mark.parametrize("kw", [
    dict(tokens=None), dict(parents=None), dict(target=None), dict(uniforms=None), dict(path=None), dict(counts=None), dict(last=None),
    dict(tokens=GB + 1), dict(parents=2 * GB + 2), dict(target=10 * GB + 2), dict(draft=20 * GB + 1), dict(uniforms=3 * GB + 3),
    dict(path=4 * GB + 1), dict(counts=5 * GB + 2), dict(last=6 * GB + 1), dict(ws=7 * GB + 128), dict(n=-1), dict(nodes=0), dict(nodes=-1),
    dict(vocab=0), dict(vocab=-5), dict(strides=(-1, 1000, 7000, 1000)), dict(strides=(7000, -1, 7000, 1000)),
    dict(strides=(7000, 1000, -1, 1000)), dict(strides=(7000, 1000, 7000, 1 << 41)),
    dict(path=GB), dict(path=2 * GB), dict(path=10 * GB + 4000), dict(counts=3 * GB), dict(counts=4 * GB), dict(last=5 * GB),
    dict(last=20 * GB)] + [dict(ws=n * GB, target=30 * GB, draft=40 * GB, vocab=1000000, strides=(7000000, 1000000) * 2) for n in (30, 40, 1, 2, 3, 4, 5, 6)])
def test_verification_refuses(kw):
    assert verify(**kw) == ilpm.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(nodes=65), dict(vocab=(1 << 30) + 1), dict(n=65536), dict(dtype=3), dict(dtype=-1)])
def test_verification_does_not_support(kw):
    assert verify(**kw) == ilpm.ERR_UNSUPPORTED


def test_verification_of_nothing_and_its_workspace():
    assert verify(n=0, tokens=None, path=None, ws=None) == ilpm.OK
    assert ilpm.lib.ilpm_verify_drafts(None, None, 0, None) == ilpm.ERR_INVALID_ARG
    need = ctypes.c_size_t(0)
    size = ilpm.lib.ilpm_verify_drafts_workspace_size
    assert size(4, 7, 1000000, ctypes.byref(need)) == ilpm.OK and need.value > 0
    assert size(4, 7, 1000, ctypes.byref(need)) == ilpm.OK
    assert size(0, 7, 1000, ctypes.byref(need)) == ilpm.OK and need.value == 0
    assert size(4, 7, 1000, None) == ilpm.ERR_INVALID_ARG
    assert size(4, 0, 1000, ctypes.byref(need)) == ilpm.ERR_INVALID_ARG


# ---- kv_copy ----

def copy(c=None, dst=4 * GB, dst_stride=30, dst_wide=30, src_start=5 * GB, dst_start=6 * GB, counts=7 * GB, path=8 * GB, path_stride=16, most=16):
    return ilpm.lib.ilpm_kv_copy(cache() if c is None else c, dst, dst_stride, dst_wide, src_start, dst_start, counts, path,
                                 path_stride, most, None)


@pytest.mark.parametrize("kw", [
    dict(c=cache(k=0)), dict(c=cache(v=0)), dict(c=cache(table=0)), dict(c=cache(size=0)), dict(c=cache(kp=-1)), dict(c=cache(kp=0)),
    dict(c=cache(ks=128)), dict(c=cache(v=GB)), dict(dst=None), dict(dst=4 * GB + 2), dict(dst=GB), dict(dst=2 * GB + 4),
    dict(dst_stride=-1), dict(dst_wide=-1), dict(src_start=None), dict(dst_start=None), dict(counts=None), dict(src_start=5 * GB + 1),
    dict(dst_start=GB), dict(counts=2 * GB), dict(counts=7 * GB + 2), dict(path=GB), dict(path=8 * GB + 3), dict(path_stride=-1), dict(most=-1)])
def test_copies_refuse(kw):
    assert copy(**kw) == ilpm.ERR_INVALID_ARG


def test_copies_that_are_not_supported():
    assert copy(most=65) == ilpm.ERR_UNSUPPORTED
    assert copy(c=cache(dtype=4)) == ilpm.ERR_UNSUPPORTED
    assert copy(c=cache(seqs=65536)) == ilpm.ERR_UNSUPPORTED


def test_copies_of_nothing_are_fine():
    assert copy(most=0) == ilpm.OK and copy(c=cache(seqs=0)) == ilpm.OK and copy(c=cache(pages=0, k=0, v=0)) == ilpm.OK
    assert copy(dst=None, dst_wide=0) == ilpm.OK and copy(most=0, src_start=None) == ilpm.OK
