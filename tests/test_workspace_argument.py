"""set_workspace takes device memory that lies together, and nothing else (no GPU needed: refused before the C call)."""
import pytest
import torch

import paper_1909_02765_amd as ilpm


@pytest.mark.parametrize("buf", [torch.zeros(4096, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8).expand(4096),
                                 torch.zeros((16, 512), dtype=torch.uint8)[:, :256], bytearray(4096)],
                         ids=["host", "expanded", "strided", "bytes"])
def test_set_workspace_refuses(buf):
    with pytest.raises(TypeError, match="contiguous CUDA tensor"):
        ilpm.set_workspace(buf)
