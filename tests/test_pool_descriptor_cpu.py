"""The pool's descriptor is checked without the built library."""
import pytest
import torch

import paper_2609_34606_amd as P
from paper_2609_34606_amd import hsa


def test_checks_without_the_library(monkeypatch, tmp_path):
    monkeypatch.setattr(hsa, "_lib", None)
    monkeypatch.setattr(hsa, "_torch", None)
    monkeypatch.setattr(hsa, "LIB_PATH", str(tmp_path / "none.so"))
    cfg = P.config(2, 3, 64, 8, torch.bfloat16)
    k, v = torch.zeros((5, 3, 8, 64), dtype=torch.bfloat16), torch.zeros((5, 3, 64, 8), dtype=torch.bfloat16)
    pt = torch.zeros((2, 4), dtype=torch.int32)
    pool = P.kv_pool(k, v, pt, cfg)
    assert (pool.num_slots, pool.max_pages, pool.k) == (5, 4, k.data_ptr())
    for bad in ((k.float(), v, pt), (k, v[:4], pt), (k, v, pt.long()), (k, v, pt[:1]), (k, v, pt[0]), (v, v, pt)):
        with pytest.raises(ValueError):
            P.kv_pool(*bad, cfg)
    with pytest.raises(P.LibraryNotBuilt):
        P.lib()
