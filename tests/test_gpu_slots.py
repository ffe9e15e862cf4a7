"""Page tables on the device against the oracle: whole numbers, and copies, all equal."""
import numpy as np
import pytest
import torch

import paper_2609_34606_amd as P
from oracle import hsa_tree_oracle as O
from test_gpu_tokens import arrays, cache, host, i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def make(r, B, pages, slots, P_, used=0.6):
    """A table whose rows hold a part of the slots, each once."""
    s = P.HsaSlots(B, P_, DEV, num_slots=slots, max_pages=pages)
    held = r.integers(0, pages + 1, B)
    lists, at = r.permutation(slots)[:int(slots * used) + 1], 0
    t = np.full((B, pages), -1)
    for b in range(B):
        n = min(held[b], len(lists) - at)
        t[b, :n] = lists[at:at + n]
        at += n
    s.page_table.copy_(i32(t.tolist()))
    s.refs.copy_(i32(O.counts(t, slots).tolist()))
    return s, t


def same(s, table, refs):
    assert np.array_equal(s.page_table.cpu().numpy(), table)
    assert np.array_equal(s.refs.cpu().numpy(), refs)
    assert np.array_equal(O.counts(table, len(refs)), refs)


SIZES = [(1, 1, 1, 8), (1, 5, 4, 16), (3, 7, 12, 64), (8, 40, 200, 8), (64, 16, 1200, 256), (130, 33, 5000, 24), (2000, 3, 40000, 40),
         (5, 2100, 9000, 8), (4096, 1, 3000, 8), (1, 4097, 5000, 8), (9000, 2, 20000, 16)]


@pytest.mark.parametrize("B,pages,slots,P_", SIZES)
def test_a_programs_steps(B, pages, slots, P_):
    """Forks, takes, frees and compactions in turn; with few slots some find none."""
    print(B, pages, slots, P_, flush=True)
    r = np.random.default_rng(B * pages)
    s, t = make(r, B, pages, slots, P_)
    refs = O.counts(t, slots)
    cap = pages * P_
    for step in range(6):
        parent = r.integers(-1, B + 1, B)
        if step % 2:
            parent = np.where(r.random(B) < 0.5, -1, parent)
        s.fork(i32(parent.tolist()))
        t = O.fork(t, parent)
        refs = O.counts(t, slots)
        same(s, t, refs)
        first = r.integers(-3, cap + 1, B)
        end = np.minimum(first + r.integers(0, 3 * P_ + 2, B), cap + 5)
        if step == 3:
            first, end = np.zeros(B, int), np.full(B, cap)
        moves = s.take(i32(first.tolist()), i32(end.tolist()))
        t, refs, want, missing = O.take(t, refs, first, end, P_)
        same(s, t, refs)
        assert np.array_equal(moves.cpu().numpy(), want) and int(s.missing) == missing
        keep = np.where(r.random(B) < 0.3, -1, r.integers(0, cap + 1, B))
        s.free(i32(keep.tolist()))
        t = O.free(t, keep, P_)
        refs = O.counts(t, slots)
        same(s, t, refs)
        n_moves = [slots, max(1, slots // 7)][step % 2]
        moves = torch.full((n_moves, 3), -9, dtype=torch.int32, device=DEV)
        out = [torch.full_like(x, -7) for x in (s.page_table, s.refs)]
        s.compact(moves, table_out=out[0], refs_out=out[1])
        same(s, t, refs)
        t, refs, want = O.compact(t, refs, n_moves, P_)
        assert np.array_equal(out[0].cpu().numpy(), t) and np.array_equal(out[1].cpu().numpy(), refs)
        assert np.array_equal(moves.cpu().numpy(), want)
        s.compact(moves.fill_(-9))
        same(s, t, refs)
        assert np.array_equal(moves.cpu().numpy(), want)


def test_a_shared_slot_stays_with_the_last_holder_that_writes():
    s = P.HsaSlots(4, 8, DEV, num_slots=6, max_pages=2)
    s.take(None, i32([5, 0, 0, 0]))
    s.fork(i32([0, 0, 0, 0]))
    assert s.page_table[:, 0].tolist() == [0] * 4 and s.refs.tolist() == [4, 0, 0, 0, 0, 0]
    moves = s.take(i32([5, 5, 5, 5]), i32([6, 5, 9, 6]))  # row 1 writes nothing
    assert moves.tolist() == [[0, 1, 5], [-1, -1, -1], [0, 2, 5], [0, 4, 5]]
    assert s.page_table.tolist() == [[1, -1], [0, -1], [2, 3], [4, -1]] and s.refs.tolist() == [1, 1, 1, 1, 1, 0]
    assert int(s.missing) == 0
    s.take(i32([0] * 4), i32([16] * 4))
    assert int(s.missing) == 2 and s.page_table.tolist() == [[1, 5], [0, -1], [2, 3], [4, -1]]


def test_entries_past_the_pool_are_left_alone():
    s = P.HsaSlots(2, 8, DEV, num_slots=3, max_pages=2)
    s.page_table.copy_(i32([[99, -1], [1, 7]]))
    s.refs.copy_(i32([0, 1, 0]))
    s.take(None, i32([16, 16]))
    assert s.page_table.tolist() == [[99, 0], [1, 7]]
    s.fork(i32([1, 1]))
    s.free(i32([0, -1]))
    assert s.page_table.tolist() == [[-1, -1], [1, 7]] and s.refs.tolist() == [0, 1, 0]


def filled(kind, seed, dt, H, d, P_, slots):
    if kind == "codes":
        c = cache(seed, 1, H, d, P_, dt, slots - 2)[0]
        return c, arrays(c), lambda: arrays(c)
    c = P.HsaLayer(1, H, d, P_, dt, DEV, num_slots=slots, max_pages=1)
    g = torch.Generator().manual_seed(seed)
    for t in (c.k_pool, c.v_pool):
        t.copy_(torch.randn(t.shape, generator=g))
    now = lambda: dict(k=host(c.k_pool), v=host(c.v_pool))
    return c, now(), now


@pytest.mark.parametrize("kind,dt", [("pool", BF), ("pool", F32), ("codes", BF)])
@pytest.mark.parametrize("P_", [8, 24, 64, 200, 392])
@pytest.mark.parametrize("H,d", [(1, 64), (5, 128)])
def test_copies(H, d, P_, kind, dt):
    print(H, d, P_, kind, dt, flush=True)
    slots = 14
    c, want, now = filled(kind, P_, dt, H, d, P_, slots)
    big = 2 ** 31 - 1
    moves = [[0, 7, 1], [1, 8, P_ - 1], [2, 9, P_], [3, 10, big], [0, 11, 9], [4, 12, 0], [5, 13, -3], [-1, 6, P_],
             [5, -1, P_], [5, slots, P_], [slots, 6, P_], [big, big, big], [4, 4, P_]]
    c.copy_pages(i32(moves))
    O.page_copy(want, moves, P_)
    got = now()
    for e in want:
        assert np.array_equal(got[e], want[e]), e


def test_compressed_pages_move_too():
    c, _, _ = filled("pool", 1, BF, 2, 64, 64, 6)
    e = torch.randn((2, 32, 64), device=DEV).to(BF)
    c.set_projections(e, e)
    c.ck.normal_()
    c.cv.normal_()
    ck, cv = c.ck.clone(), c.cv.clone()
    c.copy_pages(i32([[1, 4, 64], [0, 5, 64], [-1, -1, -1]]))
    for now, was in ((c.ck, ck), (c.cv, cv)):
        was[4], was[5] = was[1], was[0]
        assert torch.equal(now, was)


def test_captured_steps_follow_their_inputs():
    """A beam step (fork, take, copy) and a compaction in one graph, replayed with eager work between."""
    B, pages, slots, P_, H, d = 6, 5, 50, 16, 2, 64
    r = np.random.default_rng(4)
    s = P.HsaSlots(B, P_, DEV, num_slots=slots, max_pages=pages)
    c = P.HsaLayer(B, H, d, P_, BF, DEV, num_slots=slots, page_table=s.page_table,
                   k_pool=torch.randn((slots, H, P_, d), device=DEV).to(BF), v_pool=torch.randn((slots, H, d, P_), device=DEV).to(BF))
    parent, first, end, keep = i32([0] * B), i32([0] * B), i32([0] * B), i32([0] * B)
    moves, packed = torch.zeros((B, 3), dtype=torch.int32, device=DEV), torch.zeros((slots, 3), dtype=torch.int32, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.fork(parent)
        s.take(first, end, moves=moves)
        c.copy_pages(moves)
        s.free(keep)
        s.compact(packed)
        c.copy_pages(packed)
    s.page_table.fill_(-1)
    s.refs.zero_()
    t, refs = np.full((B, pages), -1), np.zeros(slots, int)
    held = dict(k=host(c.k_pool), v=host(c.v_pool))
    length = np.zeros(B, int)
    for step in range(8):
        p = r.integers(0, B, B)
        grow = r.integers(1, 9, B)
        f = length[p]
        e = np.minimum(f + grow, pages * P_)
        kp = np.where(r.random(B) < 0.3, 0, e)
        for x, y in ((parent, p), (first, f), (end, e), (keep, kp)):
            x.copy_(i32(y.tolist()))
        t = O.fork(t, p)
        t, refs, m, missing = O.take(t, O.counts(t, slots), f, e, P_)
        O.page_copy(held, m, P_)
        t = O.free(t, kp, P_)
        t, refs, m2 = O.compact(t, O.counts(t, slots), slots, P_)
        O.page_copy(held, m2, P_)
        length = kp
        g.replay()
        torch.cuda.synchronize()
        assert missing == 0 and int(s.missing) == 0
        same(s, t, refs)
        assert np.array_equal(moves.cpu().numpy(), m) and np.array_equal(packed.cpu().numpy(), m2)
        assert np.array_equal(host(c.k_pool), held["k"]) and np.array_equal(host(c.v_pool), held["v"])
