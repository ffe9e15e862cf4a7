"""Kept tokens whose sources are no tokens of the table: what they would have gone to stays, in the
8-bit cache its numbers as well (a block of which none is kept keeps its scale, one of which some are the larger scale)."""
import numpy as np
import pytest
import torch

import paper_2609_34606_amd as P
from oracle import hsa_tree_oracle as O
from test_gpu_tokens import arrays, cache, i32, one_nan, source

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def filled(seed, B, H, d, P_, pages, spread=2.5):
    """An 8-bit cache of whole sequences, tokens of very different size."""
    c, pt = cache(seed, B, H, d, P_, BF, pages)
    k, v = source(seed, B, pages * P_, H, d, F32, False, spread)
    P.HsaCache8(B, H, d, P_, F32, DEV, kv_heads=H, k=c.k, v=c.v, k_exp=c.k_exp, v_exp=c.v_exp, page_table=c.page_table).write(k, v)
    return c, pt


def equal(c, want):
    got = arrays(c)
    for e in ("k_exp", "v_exp"):
        assert np.array_equal(got[e], want[e]), e
    for e in ("k", "v"):
        assert np.array_equal(one_nan(got[e]), one_nan(want[e])), e


@pytest.mark.parametrize("share", [0.1, 0.5, 0.97])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P_,first,count,n", [
    (8, [0, 13, 5], [16, 9, 3], 16), (64, [60, 0, 7], [40, 33, 1], 40), (72, [70, 1, 64], [8, 5, 8], 8),
    (392, [391, 300, 0], [256, 200, 77], 256)])
def test_sources_outside_the_table(P_, first, count, n, d, share):
    """Any share of the sources, single ones and runs of them."""
    print(P_, n, d, share, flush=True)
    B, H = 3, 2
    pages = (max(first) + 2 * n) // P_ + 2
    c, pt = filled(n, B, H, d, P_, pages)
    r = np.random.default_rng(n + d)
    for at_once in (1, 7):
        index = r.integers(0, 2 * n, (B, n))
        out = np.repeat(r.random((B, -(-n // at_once))) < share, at_once, 1)[:, :n]
        index[out] = r.choice([2 ** 31 - 1, pages * P_, -10 ** 6, -2 ** 31], out.sum())
        want = arrays(c)
        O.keep8(want, pt, first, index, count)
        c.keep_tokens(i32(first), i32(index.tolist()), count=i32(count))
        equal(c, want)


def test_no_source_at_all():
    """Nothing changes, scales of blocks that begin with such tokens among it."""
    c, pt = filled(3, 2, 2, 64, 64, 3)
    want = arrays(c)
    c.keep_tokens(i32([0, 64]), i32([[-1] * 70, [10 ** 6] * 70]))
    equal(c, want)
