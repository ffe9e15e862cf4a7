"""Kept tokens of an accepted path: moved as they are in the pool, appended anew in the 8-bit cache.
Both equal the oracle (nothing is computed but scales, exact powers of two, and codes rounded to nearest even)."""
import numpy as np
import pytest
import torch

import paper_2609_34606_amd as P
from oracle import hsa_cache8_oracle as C8
from oracle import hsa_tree_oracle as O
from test_gpu_tokens import arrays, cache, host, i32, one_nan, source, table

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def path(r, n, most):
    return np.sort(r.permutation(most)[:n])


SIZES = [  # P, first, count, n
    (8, [0, 13, 5], [1, 1, 0], 1), (8, [3, 30, 0], [16, 9, 3], 16), (64, [60, 0, 7], [40, 33, 1], 40),
    (72, [70, 1, 64], [8, 5, 8], 8), (200, [190, 63, 128], [64, 64, 64], 64), (392, [391, 300, 0], [256, 200, 77], 256)]


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P_,first,count,n", SIZES)
def test_pool(P_, first, count, n, d, dt):
    print(P_, n, d, dt, flush=True)
    B, H = 3, 3
    pages = (max(first) + 2 * n) // P_ + 2
    pt, slots = table(n, B, pages)
    c = P.HsaLayer(B, H, d, P_, dt, DEV, num_slots=slots, max_pages=pages)
    c.page_table.copy_(torch.from_numpy(pt))
    g = torch.Generator().manual_seed(n)
    for t in (c.k_pool, c.v_pool):
        t.copy_(torch.randn(t.shape, generator=g))
        t[0] = float("nan")
    r = np.random.default_rng(n)
    for index in (np.stack([path(r, n, 2 * n) for _ in range(B)]),       # a path
                  r.integers(0, 2 * n, (B, n)),                          # any, some twice
                  np.stack([np.arange(n)[::-1] for _ in range(B)])):     # turned round
        wk, wv = host(c.k_pool), host(c.v_pool)
        c.keep_tokens(i32(first), i32(index.tolist()), count=i32(count))
        O.keep(wk, wv, pt, first, index, count)
        assert np.array_equal(host(c.k_pool), wk, equal_nan=True) and np.array_equal(host(c.v_pool), wv, equal_nan=True)
    wk, wv = host(c.k_pool), host(c.v_pool)
    c.keep_tokens(None, i32(index.tolist()))  # from the first token, all of them
    O.keep(wk, wv, pt, [0] * B, index, [n] * B)
    assert np.array_equal(host(c.k_pool), wk, equal_nan=True) and np.array_equal(host(c.v_pool), wv, equal_nan=True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P_,first,count,n", SIZES)
def test_codes(P_, first, count, n, d):
    print(P_, n, d, flush=True)
    B, H = 3, 2
    pages = (max(first) + 2 * n) // P_ + 2
    c, pt = cache(n, B, H, d, P_, BF, pages)
    r = np.random.default_rng(n)
    # whole sequences, tokens of very different size; codes that become subnormal, NaN among them
    k, v = source(n, B, pages * P_, H, d, F32, False, 2.5)
    c32 = P.HsaCache8(B, H, d, P_, F32, DEV, kv_heads=H, k=c.k, v=c.v, k_exp=c.k_exp, v_exp=c.v_exp, page_table=c.page_table)
    c32.write(k, v)
    c.k[1, 0, 3] = 0x7f
    c.v[1, 0, 3] = 0xff
    for index in (np.stack([path(r, n, 2 * n) for _ in range(B)]), r.integers(0, 2 * n, (B, n))):
        want = arrays(c)
        c.keep_tokens(i32(first), i32(index.tolist()), count=i32(count))
        O.keep8(want, pt, first, index, count)
        got = arrays(c)
        for e in ("k_exp", "v_exp"):
            assert np.array_equal(got[e], want[e]), e
        for e in ("k", "v"):
            assert np.array_equal(one_nan(got[e]), one_nan(want[e])), e


@pytest.mark.parametrize("kind", ["pool", "codes"])
def test_tokens_outside_the_table(kind):
    """Neither read nor written, nor is what they would have gone to."""
    B, H, d, P_, pages, n = 2, 2, 64, 72, 2, 6
    first = [P_ * pages - 3, -2]
    index = np.array([[0, 1, 2, 0, 1, 2], [0, 3, 2, 5, 4, 9]])
    if kind == "pool":
        pt, slots = table(1, B, pages)
        c = P.HsaLayer(B, H, d, P_, BF, DEV, num_slots=slots, max_pages=pages)
        c.page_table.copy_(torch.from_numpy(pt))
        c.k_pool.normal_()
        c.v_pool.normal_()
        wk, wv = host(c.k_pool), host(c.v_pool)
        c.keep_tokens(i32(first), i32(index.tolist()))
        O.keep(wk, wv, pt, first, index, [n] * B)
        assert np.array_equal(host(c.k_pool), wk) and np.array_equal(host(c.v_pool), wv)
        index[0, :3] = [3, 0, 2 ** 31 - 1]
        c.keep_tokens(i32(first), i32(index.tolist()))
        O.keep(wk, wv, pt, first, index, [n] * B)
        assert np.array_equal(host(c.k_pool), wk) and np.array_equal(host(c.v_pool), wv)
    else:
        c, pt = cache(2, B, H, d, P_, BF, pages)
        before = arrays(c)
        c.keep_tokens(i32([P_ * pages, -n]), i32(index.tolist()))
        c.keep_tokens(i32([0, 0]), i32(index.tolist()), count=i32([0, 0]))
        for e, x in arrays(c).items():
            assert np.array_equal(x, before[e])


def test_captured_call_follows_its_inputs():
    B, H, d, P_, pages, n = 2, 2, 64, 40, 4, 8
    c, pt = cache(3, B, H, d, P_, BF, pages)
    k, v = source(3, B, pages * P_, H, d, F32, False, 1.0)
    c32 = P.HsaCache8(B, H, d, P_, F32, DEV, k=c.k, v=c.v, k_exp=c.k_exp, v_exp=c.v_exp, page_table=c.page_table)
    c32.write(k, v)
    first, index, count = i32([0, 0]), i32([[0] * n] * B), i32([0, 0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.keep_tokens(first, index, count=count)
    r = np.random.default_rng(1)
    for f, m in (([0, 40], [8, 3]), ([39, 70], [8, 8]), ([11, 5], [0, 1])):
        x = np.stack([path(r, n, 20) for _ in range(B)])
        for t, y in ((first, f), (index, x.tolist()), (count, m)):
            t.copy_(i32(y))
        want = arrays(c)
        O.keep8(want, pt, f, x, m)
        g.replay()
        torch.cuda.synchronize()
        got = arrays(c)
        for e in want:
            assert np.array_equal(one_nan(got[e]) if e in "kv" else got[e], one_nan(want[e]) if e in "kv" else want[e]), e
