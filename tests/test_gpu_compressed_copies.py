"""Copies of a page's first tokens, as HsaSlots.take asks for: the compressed page goes along whole."""
import pytest
import torch

import paper_2609_34606_amd as P
from test_gpu_tokens import i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def made(dt, rank, P_=136, H=2, d=64, slots=8):
    g = torch.Generator().manual_seed(rank)
    c = P.HsaLayer(1, H, d, P_, dt, DEV, num_slots=slots, max_pages=2)
    e = torch.randn((H, rank, P_), generator=g).to(DEV).to(dt)
    c.set_projections(e, e)
    for t in (c.k_pool, c.v_pool, c.ck, c.cv):
        t.copy_(torch.randn(t.shape, generator=g))
    return c


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rank", [32, 64, 128])
def test_parts_of_pages(rank, dt):
    print(rank, dt, flush=True)
    c = made(dt, rank)
    was = [t.clone() for t in (c.k_pool, c.v_pool, c.ck, c.cv)]
    moves = i32([[0, 3, 5], [1, 4, 130], [2, 5, 2 ** 31 - 1], [0, 6, 0], [1, 7, -2 ** 31], [-1, -1, -1]])
    given = moves.clone()
    c.copy_pages(moves)
    assert torch.equal(moves, given)
    for now, old in zip((c.ck, c.cv), was[2:]):
        old[3:6] = old[0:3]
        assert torch.equal(now, old)
    was[0][3, :, :8], was[0][4], was[0][5] = was[0][0, :, :8], was[0][1], was[0][2]  # (of 136 tokens, 130 are 136 rounded up)
    was[1][3, :, :, :8], was[1][4], was[1][5] = was[1][0, :, :, :8], was[1][1], was[1][2]
    assert torch.equal(c.k_pool, was[0]) and torch.equal(c.v_pool, was[1])


def test_side_stream_and_captured():
    c = made(torch.bfloat16, 64)
    was = c.ck.clone()
    side = torch.cuda.Stream()
    moves = i32([[0, 3, 5]])
    torch.cuda.synchronize()
    c.copy_pages(moves, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(c.ck[3], was[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.copy_pages(moves)
    for src, dst in ((1, 4), (2, 5), (1, 6)):
        moves.copy_(i32([[src, dst, 9]]))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.ck[dst], was[src])
