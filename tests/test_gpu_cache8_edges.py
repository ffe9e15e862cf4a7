"""The 8-bit cache's attention and appends at the edges of their ranges, against the fp64
oracle (bounds: test_gpu_cache8.py), and past 32-bit offsets."""
import pytest
import torch

import paper_2609_34606_amd as P
from test_gpu_cache8 import BF, F32, run_case
from test_gpu_tokens import host, i32, source

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("d", [64, 128])
def test_queries_before_the_first_token(d):
    """More queries than tokens, far more: the first ones see nothing, also where the list
    ends inside a tile."""
    run_case(d, 2, 2, 2, d, 72, 300, BF, 3, kv_len=[72, 216], q_len=[256, 300], causal=True)
    run_case(d + 1, 1, 2, 1, d, 72, 200, BF, 5, first=3, n=1, k_max=1, kv_len=[5 * 72], causal=True)
    run_case(d + 2, 1, 2, 1, d, 40, 150, F32, 2, kv_len=[33], causal=True)


def test_a_cache_on_another_device_is_refused():
    """(before any launch)"""
    c = P.HsaCache8(1, 2, 64, 64, BF, "cpu", num_slots=2, max_pages=2)
    layer = P.HsaLayer(1, 2, 64, 64, BF, "cpu", num_slots=2, max_pages=2)
    x = torch.zeros((1, 3, 2, 64), dtype=BF, device=DEV)
    for call in (lambda: c.write(x, x), lambda: c.attend(x, 2), lambda: layer.write_tokens(x, x)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        P.hsa_rope_apply(P.config(1, 2, 64, 64, BF), P.rope(64), x, 3, torch.empty(x.shape, dtype=BF))
