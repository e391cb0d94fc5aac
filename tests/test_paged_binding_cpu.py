"""What the paged cache's bindings refuse before anything reaches the library (no GPU)."""
import pytest
import torch

import paper_2508_02401_amd as ckv


def _pool(device="cpu"):
    return torch.zeros(5, 2, 16, 64, dtype=torch.bfloat16, device=device)


def test_pools_on_two_devices():
    for k, v in ((_pool(), _pool("meta")), (_pool("meta"), _pool())):
        with pytest.raises(ValueError, match="device"):
            ckv.paged_cache(k, v)
