"""The decoder-step entry points on the host: structure layouts, workspace
sizes, and every refusal that include/ilpm.h states.  Pointers are compared,
never dereferenced, and no kernel is launched."""
import ctypes
import math
import os
import re
import shutil
import subprocess

import pytest

import decode_abi
import paper_1909_02765_amd as ilpm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GB = 1 << 30
F32, F16, BF16 = ilpm.F32, ilpm.F16, ilpm.BF16


def test_structures_have_the_c_compilers_sizes(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "ilpm.h"\nint main(void) { printf("%zu %zu %zu %zu\\n", sizeof(ilpm_heads), '
                   'sizeof(ilpm_kv_cache), sizeof(ilpm_attn_options), sizeof(ilpm_residual_norm_args)); return 0; }\n')
    cc = shutil.which("gcc")
    subprocess.run([cc, "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include", str(src),
                    "-o", str(tmp_path / "sizes")], check=True)
    got = subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(v) for v in got] == [decode_abi.HEADS.size, decode_abi.CACHE.size, decode_abi.OPTIONS.size, decode_abi.NORM.size]


def test_constants_agree_with_the_header():
    text = open(os.path.join(ROOT, "include", "ilpm.h")).read()
    for name, value in re.findall(r"ILPM_(F32|F16|BF16) = (\d)", text):
        assert getattr(ilpm, name) == int(value)
    for name, value in re.findall(r"ILPM_NORM_(NONE|RMS|LAYER) = (\d)", text):
        assert ilpm.NORMS[name.lower()] == int(value)


def cache(**kw):
    """A cache of 100 bf16 pages of 16 slots, 8 heads of 128, for 4 sequences of up to 20 pages."""
    c = dict(k=GB, v=2 * GB, kp=16 * 8 * 128, ks=8 * 128, kh=128, vp=16 * 8 * 128, vs=8 * 128, vh=128, table=3 * GB, tstride=20,
             dtype=BF16, pages=100, size=16, heads=8, dim=128, seqs=4, wide=20)
    c.update(kw)
    return decode_abi.CACHE.pack(*c.values())


def heads(at, n=8, dtype=BF16, row=None, head=128):
    return decode_abi.HEADS.pack(at, n * 128 if row is None else row, head, dtype, n)


def append(c=None, k=heads(4 * GB), v=heads(5 * GB), q=heads(6 * GB, 32), q_out=heads(7 * GB, 32), seq=8 * GB, pos=9 * GB,
           n=10, cos=10 * GB, sin=11 * GB, n_pos=320, rot=128, pairs=0):
    return ilpm.lib.ilpm_kv_append(cache() if c is None else c, k, v, q, q_out, seq, pos, n, cos, sin, n_pos, rot, pairs, None)


@pytest.mark.parametrize("kw", [
    dict(c=cache(k=0)), dict(c=cache(v=0)), dict(c=cache(table=0)), dict(c=cache(k=GB + 1)), dict(c=cache(table=3 * GB + 2)),
    dict(c=cache(size=0)), dict(c=cache(heads=0)), dict(c=cache(dim=0)), dict(c=cache(pages=-1)), dict(c=cache(seqs=-1)),
    dict(c=cache(wide=-1)), dict(c=cache(kp=-1)), dict(c=cache(vh=-128)), dict(c=cache(tstride=-1)), dict(c=cache(ks=1 << 41)),
    dict(c=cache(kp=0)), dict(c=cache(ks=128)), dict(c=cache(vh=64)),     # pools that name a place twice
    dict(c=cache(v=GB)), dict(c=cache(v=GB + 2 * 128)),                   # values over keys
    dict(k=None), dict(v=None), dict(k=heads(0)), dict(k=heads(4 * GB + 1)), dict(k=heads(4 * GB, 4)), dict(v=heads(5 * GB, 9)),
    dict(k=heads(4 * GB, row=-1)), dict(k=heads(4 * GB, head=-128)),
    dict(q=None), dict(q_out=None), dict(q_out=heads(7 * GB, 31)), dict(q_out=heads(7 * GB, 32, row=0)),
    dict(q_out=heads(7 * GB, 32, head=64)), dict(q_out=heads(6 * GB + 256, 32)), dict(q_out=heads(4 * GB, 32)),
    dict(q_out=heads(5 * GB, 32)), dict(q_out=heads(GB, 32)), dict(q_out=heads(8 * GB, 32)), dict(q_out=heads(10 * GB, 32)),
    dict(q_out=heads(3 * GB, 32)), dict(q=heads(2 * GB, 32)), dict(k=heads(GB + 4096)), dict(v=heads(GB)), dict(k=heads(2 * GB)),
    dict(seq=None), dict(pos=None), dict(seq=8 * GB + 2), dict(pos=GB), dict(seq=2 * GB + 64),
    dict(cos=None), dict(sin=None), dict(cos=10 * GB + 2), dict(cos=GB), dict(sin=2 * GB),
    dict(n=-1), dict(n_pos=-1), dict(rot=-2), dict(rot=63), dict(rot=130), dict(pairs=2)])
def test_append_refuses(kw):
    assert append(**kw) == ilpm.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(c=cache(dtype=3)), dict(k=heads(4 * GB, dtype=7)), dict(k=heads(4 * GB, dtype=F16), v=heads(5 * GB, dtype=F16)),
    dict(k=heads(4 * GB, dtype=F32)), dict(q=heads(6 * GB, 32, dtype=F32)), dict(q_out=heads(7 * GB, 32, dtype=F32)),
    dict(c=cache(dtype=F32)), dict(n=1 << 24, k=heads(20 * GB), v=heads(60 * GB), q=None, q_out=None)])
def test_append_does_not_support(kw):
    assert append(**kw) == ilpm.ERR_UNSUPPORTED


def test_append_of_nothing_is_fine():
    assert append(n=0) == ilpm.OK
    assert append(n=0, k=heads(0), v=heads(0), q=None, q_out=None, seq=None, pos=None) == ilpm.OK
    assert ilpm.lib.ilpm_kv_append(None, heads(4 * GB), heads(5 * GB), None, None, 8 * GB, 9 * GB, 0, None, None, 0, 0, 0,
                                   None) == ilpm.ERR_INVALID_ARG


def options(mask=0, mstride=0, scale=0.1, cap=0.0, mlen=0, window=0, max_len=0):
    return decode_abi.OPTIONS.pack(mask, mstride, scale, cap, mlen, window, max_len)


def attn(c=None, q=heads(4 * GB, 32), lengths=5 * GB, opt=None, out=heads(6 * GB, 32), lse=7 * GB, ws=8 * GB, ws_bytes=GB):
    return ilpm.lib.ilpm_attn_decode(cache() if c is None else c, q, lengths, options() if opt is None else opt, out, lse, ws,
                                     ws_bytes, None)


@pytest.mark.parametrize("kw", [
    dict(c=cache(k=0)), dict(c=cache(v=0)), dict(c=cache(table=0)), dict(c=cache(size=0)), dict(c=cache(kp=-1)),
    dict(c=cache(v=2 * GB + 1)), dict(q=None), dict(out=None), dict(lengths=None), dict(q=heads(0, 32)), dict(out=heads(0, 32)),
    dict(q=heads(4 * GB, 30)), dict(q=heads(4 * GB, 30), out=heads(6 * GB, 30)), dict(q=heads(4 * GB, 0), out=heads(6 * GB, 0)),
    dict(q=heads(4 * GB + 1, 32)), dict(lengths=5 * GB + 1), dict(lse=7 * GB + 2), dict(ws=8 * GB + 128),
    dict(opt=options(window=-1)), dict(opt=options(max_len=-1)), dict(opt=options(scale=math.nan)), dict(opt=options(scale=math.inf)),
    dict(opt=options(cap=-1.0)), dict(opt=options(cap=math.nan)), dict(opt=options(cap=math.inf)),
    dict(opt=options(scale=3e38)), dict(opt=options(cap=3e38)), dict(opt=options(cap=1e-40)),
    dict(opt=options(mask=9 * GB, mlen=-1)), dict(opt=options(mask=9 * GB, mlen=320, mstride=-320)),
    dict(out=heads(6 * GB, 32, row=0)), dict(out=heads(6 * GB, 32, head=64)),   # outputs that name a place twice
    dict(out=heads(4 * GB + 256, 32)), dict(out=heads(GB, 32)), dict(out=heads(2 * GB, 32)), dict(out=heads(3 * GB, 32)),
    dict(out=heads(5 * GB, 32)), dict(lse=4 * GB), dict(lse=6 * GB), dict(lse=GB), dict(lse=3 * GB), dict(lse=5 * GB),
    dict(ws=4 * GB), dict(ws=6 * GB), dict(ws=GB), dict(ws=2 * GB), dict(ws=3 * GB), dict(ws=5 * GB), dict(ws=7 * GB),
    dict(opt=options(mask=6 * GB, mlen=320, mstride=320)), dict(opt=options(mask=7 * GB, mlen=320, mstride=320)),
    dict(opt=options(mask=8 * GB, mlen=320, mstride=320))])
def test_attention_refuses(kw):
    assert attn(**kw) == ilpm.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(c=cache(dtype=5)), dict(q=heads(4 * GB, 32, dtype=F16)), dict(out=heads(6 * GB, 32, dtype=F32)),
    dict(q=heads(4 * GB, 32, dtype=F16), out=heads(6 * GB, 32, dtype=F16)), dict(c=cache(dim=257)),
    dict(c=cache(seqs=1 << 20))])
def test_attention_does_not_support(kw):
    assert attn(**kw) == ilpm.ERR_UNSUPPORTED


def test_attention_of_nothing_is_fine():
    assert attn(c=cache(seqs=0, table=0), q=heads(0, 32), out=heads(0, 32), lengths=None, lse=None, ws=None) == ilpm.OK


def size(q_heads=32, window=0, max_len=0, **kw):
    n = ctypes.c_size_t()
    assert ilpm.lib.ilpm_attn_decode_workspace_size(cache(**kw), q_heads, window, max_len, ctypes.byref(n)) == ilpm.OK
    return n.value


def test_workspace_sizes():
    assert size(wide=1) == size(window=16) == size(max_len=16) == size(pages=0) == size(seqs=0) == 0
    # At most 1024 workgroups, each with 16 bytes of its own and two parts of up to 16 heads.
    most = 1024 * (16 + 2 * 16 * 130 * 4)
    long = size(seqs=1, wide=1 << 16)
    assert 0 < long <= most
    assert 0 < size(seqs=1, wide=1 << 16, max_len=2048) < long
    assert size(seqs=100000, q_heads=8) <= most
    assert size(seqs=1, wide=1 << 30) <= most     # more keys than an int counts
    assert size(seqs=1 << 19, q_heads=8, wide=1 << 30) == 0   # more tiles than an int counts: no split
    n = ctypes.c_size_t()
    f = ilpm.lib.ilpm_attn_decode_workspace_size
    for args, want in (((None, 32, 0, 0), ilpm.ERR_INVALID_ARG), ((cache(), 30, 0, 0), ilpm.ERR_INVALID_ARG),
                       ((cache(), 0, 0, 0), ilpm.ERR_INVALID_ARG), ((cache(), 32, -1, 0), ilpm.ERR_INVALID_ARG),
                       ((cache(), 32, 0, -1), ilpm.ERR_INVALID_ARG), ((cache(size=0), 32, 0, 0), ilpm.ERR_INVALID_ARG),
                       ((cache(dim=300), 32, 0, 0), ilpm.ERR_UNSUPPORTED), ((cache(dtype=9), 32, 0, 0), ilpm.ERR_UNSUPPORTED)):
        assert f(*args, ctypes.byref(n)) == want
    assert f(cache(), 32, 0, 0, None) == ilpm.ERR_INVALID_ARG


def norm(**kw):
    a = dict(x=GB, y=2 * GB, r=3 * GB, z=4 * GB, post_w=5 * GB, post_b=6 * GB, pre_w=7 * GB, pre_b=8 * GB, gate=9 * GB, xs=512, ys=512,
             rs=512, zs=512, gs=512, rows=10, width=512, xd=F32, yd=BF16, pd=F32, post=1, pre=2, scale=1.0, eps=1e-6)
    a.update(kw)
    return ilpm.lib.ilpm_residual_norm(decode_abi.NORM.pack(*a.values()), None)


@pytest.mark.parametrize("kw", [
    dict(x=0), dict(r=0, z=0), dict(z=0), dict(pre=0, pre_w=0, pre_b=0), dict(y=0), dict(y=0, gate=0), dict(post=0), dict(post=0, post_w=0),
    dict(pre=0, z=0), dict(pre=0, z=0, pre_w=0), dict(post=3), dict(pre=-1), dict(rows=-1), dict(width=0), dict(width=-3),
    dict(eps=-1e-6), dict(eps=math.nan), dict(eps=math.inf), dict(scale=math.nan), dict(scale=math.inf),
    dict(xs=-1), dict(ys=-512), dict(gs=-1), dict(zs=1 << 41), dict(rs=511), dict(zs=0),
    dict(x=GB + 2), dict(y=2 * GB + 1), dict(r=3 * GB + 2), dict(z=4 * GB + 1), dict(pre_w=7 * GB + 2), dict(gate=9 * GB + 1),
    dict(r=GB + 4), dict(r=GB, rs=600), dict(r=2 * GB), dict(z=GB), dict(z=2 * GB + 2), dict(z=3 * GB), dict(z=2 * GB, zs=600),
    dict(r=5 * GB), dict(r=6 * GB), dict(r=7 * GB), dict(z=8 * GB), dict(r=9 * GB), dict(z=9 * GB + 512)])
def test_norm_refuses(kw):
    assert norm(**kw) == ilpm.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(xd=4), dict(yd=-1), dict(pd=3), dict(xd=F16), dict(pd=F16), dict(yd=F32, xd=BF16),
                                dict(rows=1 << 24)])
def test_norm_does_not_support(kw):
    assert norm(**kw) == ilpm.ERR_UNSUPPORTED


def test_norm_of_nothing_is_fine():
    assert norm(rows=0) == ilpm.OK
    assert norm(rows=0, x=0, y=0, r=0, z=0) == ilpm.OK
    assert ilpm.lib.ilpm_residual_norm(None, None) == ilpm.ERR_INVALID_ARG


def test_binding_refuses_what_is_not_on_the_gpu():
    import torch
    x = torch.zeros(2, 4, 64)
    pages, table, ints = torch.zeros(3, 16, 4, 64), torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        ilpm.kv_append(x, x, pages, pages, table, ints, ints)
    with pytest.raises(TypeError):
        ilpm.attn_decode(x, pages, pages, table, ints)
    with pytest.raises(TypeError):
        ilpm.residual_norm(torch.zeros(2, 64), torch.zeros(2, 64))
    with pytest.raises(ValueError):
        ilpm.residual_norm(torch.zeros(2, 64), torch.zeros(2, 64), post="batch")
