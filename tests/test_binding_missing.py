"""The convolutions' binding works without the decoder-step operators' module, and those say that it is missing."""
import os
import subprocess
import sys

import pytest

import paper_1909_02765_amd as ilpm

CODE = """
import torch
import paper_1909_02765_amd as ilpm
assert ilpm.PKG == {pkg!r}
print(ilpm.plan(64, 56, 56, 64, 3, 1, 1).as_dict()["grid"])
x = torch.zeros(1, 2, 64)
for call in (lambda: ilpm.kv_append(x, x, x, x, x, x, x), lambda: ilpm.attn_decode(x, x, x, x, x),
             lambda: ilpm.attn_decode_workspace_size(x, x, x, 8), lambda: ilpm.residual_norm(x[0], x[0])):
    try:
        call()
    except ImportError as e:
        assert "_binding.so is not built" in str(e) and "build.py" in str(e)
    else:
        raise SystemExit("no error")
"""


@pytest.mark.parametrize("module", [None, b"", b"not a library"], ids=["none", "empty", "broken"])
def test_without_the_decoder_steps_module(tmp_path, module):
    pkg = tmp_path / "paper_1909_02765_amd"
    pkg.mkdir()
    for name in ("__init__.py", "libilpm.so"):
        os.symlink(os.path.join(ilpm.PKG, name), pkg / name)
    if module is not None:
        (pkg / "_binding.so").write_bytes(module)
    # (A child of its own: this process holds the library already.)
    got = subprocess.run([sys.executable, "-c", CODE.format(pkg=str(pkg))], cwd=tmp_path, capture_output=True, text=True,
                         timeout=300, env=dict(os.environ, PYTHONPATH=str(tmp_path)))
    assert got.returncode == 0, got.stderr
    assert int(got.stdout) == ilpm.plan(64, 56, 56, 64, 3, 1, 1).grid
