"""Writes through a page table that has no slot for some pages (-1, as HsaSlots leaves those of ended sequences and
those that found no free slot; or an entry past the pool): tokens of such pages are dropped, and the
slots of other sequences, slot 0 above all, keep every byte."""
import numpy as np
import pytest
import torch

import paper_2609_34606_amd as P
from oracle import hsa_cache8_oracle as C8
from oracle import hsa_tree_oracle as O
from test_gpu_keep_staying import equal, filled
from test_gpu_tokens import arrays, host, i32, source

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
KINDS = pytest.mark.parametrize("kind,dt", [("pool", BF), ("pool", F32), ("codes", BF), ("codes", F32)],
                                ids=["pool-bf16", "pool-f32", "codes-bf16", "codes-f32"])


def holed(pt, num_slots):
    """The table with row 1 freed, and holes in row 2."""
    t = pt.copy()
    t[1] = -1
    t[2, 1::3] = -1
    t[2, 2] = num_slots
    return t


def made(kind, seed, B, H, d, P_, pages, dt):
    """A filled pool or cache, its table and number of slots."""
    c, pt = filled(seed, B, H, d, P_, pages)
    slots = c.k.shape[0]
    if kind == "codes":
        return P.HsaCache8(B, H, d, P_, dt, DEV, kv_heads=H, k=c.k, v=c.v, k_exp=c.k_exp, v_exp=c.v_exp,
                           page_table=c.page_table), pt, slots
    c = P.HsaLayer(B, H, d, P_, dt, DEV, num_slots=slots, max_pages=pages)
    g = torch.Generator().manual_seed(seed)
    for t in (c.k_pool, c.v_pool):
        t.copy_(torch.randn(t.shape, generator=g))
    return c, pt, slots


def with_spare(table, num_slots):
    """The table with a slot behind the pool for every entry that has none, and how many there are."""
    t, bad = table.copy(), (table < 0) | (table >= num_slots)
    t[bad] = num_slots + np.arange(bad.sum())
    return t, int(bad.sum())


def longer(x, n):
    return np.concatenate([x, np.zeros((n,) + x.shape[1:], x.dtype)])


@KINDS
@pytest.mark.parametrize("P_,n,first", [(8, 1, [9, 3, 8]), (8, 50, [3, 0, 5]), (64, 130, [61, 0, 0]), (72, 200, [5, 71, 30]),
                                        (392, 900, [3, 391, 100])])
def test_appends(P_, n, first, kind, dt):
    print(P_, n, kind, dt, flush=True)
    B, H, d = 3, 2, 64
    pages = (max(first) + n) // P_ + 4
    c, pt, slots = made(kind, n, B, H, d, P_, pages, dt)
    table = holed(pt, slots)
    c.page_table.copy_(torch.from_numpy(table))
    k, v = source(n, B, n, H, d, dt, False)
    t, spare = with_spare(table, slots)
    count = [n, n - 1, n]
    if kind == "pool":
        wk, wv = longer(host(c.k_pool), spare), longer(host(c.v_pool), spare)
        c.write_tokens(k, v, i32(first), count=i32(count))
        C8.write_tokens(wk, wv, t, host(k), host(v), first, count)
        assert np.array_equal(host(c.k_pool), wk[:slots]) and np.array_equal(host(c.v_pool), wv[:slots])
    else:
        want = {e: longer(x, spare) for e, x in arrays(c).items()}
        c.write(k, v, i32(first), count=i32(count))
        C8.write8(want, t, host(k), host(v), first, count)
        equal(c, {e: x[:slots] for e, x in want.items()})


@KINDS
@pytest.mark.parametrize("P_,first,count,n", [(8, [0, 13, 5], [16, 9, 3], 16), (64, [60, 0, 7], [40, 33, 1], 40),
                                              (72, [70, 1, 64], [8, 5, 8], 8), (200, [190, 63, 128], [64, 64, 64], 64)])
def test_kept_tokens(P_, first, count, n, kind, dt):
    """Of a page without a slot no token is read either."""
    print(P_, n, kind, dt, flush=True)
    B, H, d = 3, 2, 128
    pages = (max(first) + 2 * n) // P_ + 4
    c, pt, slots = made(kind, n, B, H, d, P_, pages, dt)
    table = holed(pt, slots)
    c.page_table.copy_(torch.from_numpy(table))
    r = np.random.default_rng(n)
    for index in (np.sort(np.stack([r.permutation(2 * n)[:n] for _ in range(B)])), r.integers(0, 2 * n, (B, n))):
        if kind == "pool":
            wk, wv = host(c.k_pool), host(c.v_pool)
            c.keep_tokens(i32(first), i32(index.tolist()), count=i32(count))
            O.keep(wk, wv, table, first, index, count)
            assert np.array_equal(host(c.k_pool), wk) and np.array_equal(host(c.v_pool), wv)
        else:
            want = arrays(c)
            c.keep_tokens(i32(first), i32(index.tolist()), count=i32(count))
            O.keep8(want, table, first, index, count)
            equal(c, want)


@pytest.mark.parametrize("kind", ["pool", "codes"])
def test_an_ended_and_an_unserved_row(kind):
    """A captured step (take, append, keep) of all rows: the first is full, the second has ended, the third finds no
    free slot for its second page. Slots 0 and 1 are the first one's."""
    B, H, d, P_ = 3, 2, 64, 8
    s = P.HsaSlots(B, P_, DEV, num_slots=3, max_pages=2)
    if kind == "pool":
        c = P.HsaLayer(B, H, d, P_, BF, DEV, num_slots=3, page_table=s.page_table,
                       k_pool=torch.randn((3, H, P_, d), device=DEV).to(BF), v_pool=torch.randn((3, H, d, P_), device=DEV).to(BF))
        write, state = c.write_tokens, (c.k_pool, c.v_pool)
    else:
        c = P.HsaCache8(B, H, d, P_, BF, DEV, num_slots=3, page_table=s.page_table)
        write, state = c.write, (c.k, c.v, c.k_exp, c.v_exp)
    k, v = source(1, B, 16, H, d, BF, False)
    s.take(None, i32([16, 0, 4]))
    write(k, v, count=i32([16, 0, 4]))
    assert s.page_table.tolist() == [[0, 1], [-1, -1], [2, -1]]
    was = [x.clone() for x in state]
    first, end, index = i32([16, 0, 4]), i32([16, 0, 12]), i32([[1, 3, 5, 7]] * B)
    k, v = source(2, B, 8, H, d, BF, False)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.take(first, end)
        write(k, v, first)
        c.keep_tokens(first, index)
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert s.page_table.tolist() == [[0, 1], [-1, -1], [2, -1]] and int(s.missing) == 1
        for x, y in zip(state, was):
            assert torch.equal(x[:2], y[:2])
        if kind == "pool":  # tokens 4 to 7 are the step's, then 4 takes 5 and 5 takes 7; 9 and 11 were never there
            want = torch.stack([k[2, i] for i in (1, 3, 2, 3)])
            assert torch.equal(c.k_pool[2, :, 4:].transpose(0, 1), want) and torch.equal(c.k_pool[2, :, :4], was[0][2, :, :4])


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("P_", [8, 72, 200])
def test_whole_pages(P_, dt):
    B, H, d, pages = 3, 2, 128, 6
    c, pt, slots = made("pool", P_, B, H, d, P_, pages, dt)
    table = holed(pt, slots)
    c.page_table.copy_(torch.from_numpy(table))
    k, v = source(P_, B, 4 * P_, H, d, dt, False)
    t, spare = with_spare(table, slots)
    wk, wv = longer(host(c.k_pool), spare), longer(host(c.v_pool), spare)
    P.hsa_page_write(c.cfg, c.pool, k, v, 1, 4)
    C8.write_tokens(wk, wv, t, host(k), host(v), [P_] * B, [4 * P_] * B)
    assert np.array_equal(host(c.k_pool), wk[:slots]) and np.array_equal(host(c.v_pool), wv[:slots])
