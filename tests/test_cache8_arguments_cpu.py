"""Arguments of the 8-bit cache's and the rotation's calls that the binding or the library
settles before any launch; none of these needs a GPU."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2609_34606_amd as P

BF = torch.bfloat16


def test_a_workspace_on_another_device_is_refused():
    """(tensors without memory that say that they are on a GPU)"""
    cfg = P.config(1, 2, 64, 64, BF)
    cache = P.HsaCache8(1, 2, 64, 64, BF, "cpu", num_slots=2, max_pages=2).pool
    with FakeTensorMode():
        q, o = (torch.empty((1, 3, 2, 64), dtype=BF, device="cuda:0") for _ in range(2))
        for where in ("cpu", "cuda:1"):
            ws = torch.empty(256, dtype=torch.uint8, device=where)
            with pytest.raises(ValueError, match="ws is on"):
                P.hsa_cache8_attn(cfg, q, 3, cache, None, 0, None, 0, 2, o, ws=ws)
