"""GPU: residual_norm over so many bytes that its workgroups are launched by another rule, for each width at the ends of
that rule and each kind of types: rows against their 64-bit definition, and against calls of a few of them bit for bit."""
import pytest
import torch

import decode_ref as ref
from gpu_common import note, torch_cuda

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
BYTES = {F32: 4, F16: 2, BF16: 2}


@pytest.mark.parametrize("x,y,p,gates", [(F32, BF16, F32, True), (F32, F16, F16, False), (BF16, BF16, F32, True), (F32, F32, F32, False)],
                         ids=str)
@pytest.mark.parametrize("width", [3576, 3584, 4096, 4104])
def test_norm_of_rows_that_come_from_memory(x, y, p, gates, width):
    torch_cuda()
    import paper_1909_02765_amd as ilpm
    rows = 350_000_000 // (width * (2 * BYTES[x] + 2 * BYTES[y] + BYTES[p] * gates))
    g = torch.Generator(device="cuda").manual_seed(width)

    def randn(*shape, dtype, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)

    t = dict(x=randn(rows, width, dtype=x, std=3.0), y=randn(rows, width, dtype=y), gate=randn(rows, width, dtype=p) if gates else None,
             post_w=randn(width, dtype=p), post_b=randn(width, dtype=p), pre_w=randn(width, dtype=p), pre_b=randn(width, dtype=p))
    note(f"[norm] {rows} rows of {width}, {x} {y} {p}")
    r, z = ilpm.residual_norm(**t, post="rms", pre="layer", scale=0.5)
    torch.cuda.synchronize()
    of_rows = ("x", "y", "gate")
    for i in (0, rows // 2, rows - 7):
        some = {k: v if v is None or k not in of_rows else v[i:i + 7] for k, v in t.items()}
        some_r, some_z = ilpm.residual_norm(**some, post="rms", pre="layer", scale=0.5)
        assert torch.equal(r[i:i + 7], some_r) and torch.equal(z[i:i + 7], some_z)
        c = {k: None if v is None else v.cpu() for k, v in some.items()}
        want_r, want_z, er, ez = ref.residual_norm(c["x"], c["y"], "rms", c["post_w"], c["post_b"], c["gate"], 0.5, "layer", c["pre_w"],
                                                   c["pre_b"], 1e-6, x, y)
        assert ((some_r.double().cpu() - want_r).abs() <= er).all() and ((some_z.double().cpu() - want_z).abs() <= ez).all()
    assert torch.isfinite(r).all() and torch.isfinite(z).all()
