"""Attention over long lists of the 8-bit cache, cut into pieces (bounds:
test_gpu_cache8.py). The page table names a small cache's pages again and again, so that
the lists are long and the cache and the oracle's copy of it are not."""
import numpy as np
import pytest
import torch

import paper_2609_34606_amd as P
from oracle import hsa_cache8_oracle as O
from test_gpu_cache8 import BF, F32, check
from test_gpu_tokens import arrays, cache, i32, source

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def long_case(seed, B, H, kv, d, P_, n_q, dt, pages, times, kv_len=None, causal=False):
    c, pt = cache(seed, B, H, d, P_, dt, pages, kv=kv)
    w = P.HsaCache8(B, H, d, P_, torch.float32, DEV, kv_heads=kv, k=c.k, v=c.v, k_exp=c.k_exp, v_exp=c.v_exp,
                    page_table=c.page_table)
    w.write(*source(seed, B, pages * P_, kv, d, torch.float32, False, 0.3))
    pt = np.tile(pt, (1, times))
    c = P.HsaCache8(B, H, d, P_, dt, DEV, kv_heads=kv, k=c.k, v=c.v, k_exp=c.k_exp, v_exp=c.v_exp,
                    page_table=torch.from_numpy(pt).to(DEV))
    q = torch.randn((B, n_q, H, d), generator=torch.Generator().manual_seed(seed + 1)).to(dt).to(DEV)
    out = torch.full((B, n_q, H, d), 3.0, dtype=dt, device=DEV)
    lse = torch.full((B, H, n_q), 5.0, device=DEV)
    n = pages * times
    c.attend(q, n, kv_len=None if kv_len is None else i32(kv_len), causal=causal, out=out, lse=lse)
    k, v = O.dequantise(arrays(c))
    check(q, out, lse, k, v, pt, [[list(range(n))] * kv] * B, [n * P_] * B if kv_len is None else kv_len, [n_q] * B,
          causal, d ** -0.5)


@pytest.mark.parametrize("P_", [8, 24, 64, 200])
@pytest.mark.parametrize("H,kv,n_q,d,dt", [(4, 2, 1, 128, BF), (8, 2, 1, 64, BF), (2, 2, 1, 128, F32), (6, 2, 2, 128, BF),
                                           (4, 2, 10, 64, BF), (16, 2, 8, 64, BF), (16, 2, 3, 128, F32),
                                           (10, 2, 5, 64, F32)])
def test_equal_and_ragged_lengths(P_, H, kv, n_q, d, dt):
    """Every width of the four-wave workgroups: all tokens, and a length that ends in the first
    piece beside one that ends in the last."""
    pages = 520 // P_ + 1
    rows = (n_q * H // kv + 15) // 16
    times = 4096 // (4 * rows) * 64 // (pages * P_) + 2  # more than 4096 tiles of 16 rows in all
    cap = pages * P_ * times
    print(P_, H, n_q, d, dt, cap, flush=True)
    long_case(P_ + n_q, 2, H, kv, d, P_, n_q, dt, pages, times, kv_len=[cap - 11, 70], causal=True)
    if n_q <= 3:
        long_case(P_ + n_q, 2, H, kv, d, P_, n_q, dt, pages, times)
