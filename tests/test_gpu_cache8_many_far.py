"""The many-rows kernel of the 8-bit cache's attention past 32-bit offsets: pages at the end of a
cache of more than 2^32 elements and in a small one give the same bits."""
import pytest
import torch

import paper_2609_34606_amd as P
from test_gpu_cache8 import BF
from test_gpu_tokens import i32, source

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HEADS = 8
# d, page, slots, pages of the sequence, queries (test_cache8_plan_cpu.py holds that these take the kernel)
FAR = [(128, 1560, 2800, 2, 600), (64, 1560, 5600, 2, 1400), (128, 56, 76000, 40, 600), (64, 56, 151000, 40, 1900),
       (128, 8, 530000, 200, 1000)]


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("d,P_,slots,pages,n_q", FAR)
def test_offsets_past_32_bits(d, P_, slots, pages, n_q, ragged):
    print(d, P_, slots, pages, n_q, flush=True)
    n = pages * P_
    far = [slots - 1 - 2 * i for i in range(pages)]
    assert min(far) * HEADS * P_ * d > 2 ** 32
    q = source(6, 1, n_q, HEADS, d, BF, False)[0]
    k, v = source(7, 1, n, HEADS, d, BF, True)
    got = []
    for num, at in ((slots, far), (pages, list(range(pages))[::-1])):
        c = P.HsaCache8(1, HEADS, d, P_, BF, DEV, num_slots=num, max_pages=pages)
        c.page_table.copy_(torch.tensor([at]))
        assert P.hsa_cache8_attn_plan(c.cfg, n_q, HEADS, 0, pages, ragged)[0]
        c.write(k, v)
        lse = torch.full((1, HEADS, n_q), 5.0, device=DEV)
        out = torch.full_like(q, 3.0)
        c.attend(q, pages, kv_len=i32([n - 3]) if ragged else None, q_len=i32([n_q - 9]) if ragged else None,
                 causal=ragged, out=out, lse=lse)
        got.append((out.clone(), lse.clone()))
        del c
        torch.cuda.empty_cache()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert got[0][0].float().abs().max() > 0.1 and torch.isfinite(got[0][0].float()).all()
