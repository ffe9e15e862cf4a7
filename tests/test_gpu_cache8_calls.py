"""Single calls of the 8-bit cache and the rotation that a program makes and the other tests do
not: a first append inside a block."""
import pytest
import torch

import paper_2609_34606_amd as P
from test_gpu_cache8 import BF, F32
from test_gpu_tokens import i32, source

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("P_", [16, 72, 200])
def test_first_append_inside_a_block(P_, dt):
    """A new cache's sequence that begins inside a block has the scale of its own tokens: the bits of
    one whose earlier tokens are zeros."""
    at, n = 5, 2 * P_ - 9
    k, v = source(P_, 2, n, 2, 64, dt, False)
    zero = torch.zeros((2, at, 2, 64), dtype=dt, device=DEV)
    held = []
    for before in (False, True):
        c = P.HsaCache8(2, 2, 64, P_, dt, DEV, num_slots=4, max_pages=2)
        c.page_table.copy_(torch.tensor([[3, 0], [1, 2]]))
        if before:
            c.write(zero, zero)
        c.write(k, v, i32([at, at]))
        held.append(c)
    new, old = held
    for b, pages in enumerate(([3, 0], [1, 2])):
        for i, s in enumerate(pages):
            first, last = at if i == 0 else 0, min(P_, at + n - i * P_)
            blocks = -(-last // 64)
            assert torch.equal(new.k[s, :, first:last], old.k[s, :, first:last])
            assert torch.equal(new.v[s, ..., first:last], old.v[s, ..., first:last])
            assert torch.equal(new.k_exp[s, :, :blocks], old.k_exp[s, :, :blocks])
            assert torch.equal(new.v_exp[s, :, :blocks], old.v_exp[s, :, :blocks])
