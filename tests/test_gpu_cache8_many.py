"""Attention over the 8-bit cache for calls of many query rows, which take a kernel of their own
(bounds: test_gpu_cache8.py). The launch is planned for n_q and the listed pages' room; the
lengths on the device keep the oracle's work small."""
import pytest
import torch

from test_gpu_cache8 import BF, run_case
from test_gpu_tokens import i32, source

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROOM = {64: 4200, 128: 2200}  # tokens that 1024 queries of 4 heads, 2 sequences, need for that


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P_", [8, 16, 24, 32, 40, 48, 56, 64, 72, 136, 200, 256, 392])
def test_page_sizes(P_, d):
    """Tiles that run from page to page, lengths that end anywhere, in one piece or several."""
    pages = ROOM[d] // P_ + 1
    cap = pages * P_
    print(P_, d, flush=True)
    run_case(P_, 2, 4, 2, d, P_, 1024, BF, pages, kv_len=[cap - 3, 70], q_len=[130, 69], causal=True)
    run_case(P_ + 1, 2, 4, 2, d, P_, 1024, BF, pages, kv_len=[P_ + 1, 0], q_len=[40, 1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P_", [8, 24, 72, 200])
def test_selected_pages(P_, d):
    """Selected pages before the run of pages: budgets per head, short rows, none."""
    pages = ROOM[d] // P_ + 3
    k = pages - 2
    print(P_, d, flush=True)
    run_case(P_, 1, 8, 4, d, P_, 1024, BF, pages, first=k, k_max=k, k_h=[k, 0, 3, k - 1], sel_valid=[k, 5, 1, k],
             kv_len=[pages * P_ - 5], q_len=[60], causal=True)
    run_case(P_ + 1, 2, 4, 2, d, P_, 1024, BF, pages, first=k, k_max=k, sel_valid=[7, 0, k], q_len=[33, 0])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P_", [16, 40, 72, 104])
def test_queries_before_the_first_token(P_, d):
    """More queries than tokens, by far: the first ones see nothing, also where the list ends
    inside a tile."""
    pages = ROOM[d] // P_ + 1
    run_case(P_, 2, 4, 2, d, P_, 1024, BF, pages, kv_len=[P_, 3 * P_], q_len=[256, 300], causal=True)


@pytest.mark.parametrize("P_,d,H,kv", [(16, 64, 4, 2), (200, 64, 6, 3), (40, 128, 8, 4), (256, 128, 3, 3)])
def test_all_rows(P_, d, H, kv):
    """Every query of a call, groups that straddle items, scores far apart."""
    pages = ROOM[d] * 2 // P_ + 1
    print(P_, d, H, kv, flush=True)
    run_case(P_, 1, H, kv, d, P_, 1111, BF, pages, kv_len=[1300], causal=True, spread=1.2)


@pytest.mark.parametrize("P_", [24, 200])
@pytest.mark.parametrize("d", [64, 128])
def test_same_bits_and_captured(P_, d):
    """The same call gives the same bits; captured calls follow their lengths, and two graphs
    share nothing."""
    pages = ROOM[d] // P_ + 1
    c, q, out, lse = run_case(3, 2, 4, 2, d, P_, 1024, BF, pages, kv_len=[1000, 777], q_len=[70, 50])
    for _ in range(3):
        o2, l2 = torch.full_like(out, 3.0), torch.full_like(lse, 5.0)
        c.attend(q, pages, kv_len=i32([1000, 777]), q_len=i32([70, 50]), out=o2, lse=l2)
        assert torch.equal(out, o2) and torch.equal(lse, l2)
    qs = [q, (q * 0.5).contiguous()]
    c.write(*source(4, 2, pages * P_, 2, d, BF, False))
    lens, qlen = i32([900, 100]), i32([900, 100])
    outs = [torch.zeros_like(q) for _ in range(2)]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for x, o, graph in zip(qs, outs, graphs):
        with torch.cuda.graph(graph):
            c.attend(x, pages, kv_len=lens, q_len=qlen, causal=True, out=o)
    for kl, ql in (([1500, 130], [1024, 130]), ([2160, 1024], [5, 1000]), ([700, 0], [700, 0])):
        lens.copy_(torch.tensor(kl))
        qlen.copy_(torch.tensor(ql))
        want = [torch.zeros_like(q) for _ in qs]
        for o in outs:
            o.zero_()
        graphs[0].replay()
        graphs[1].replay()
        for x, o in zip(qs, want):
            c.attend(x, pages, kv_len=lens, q_len=qlen, causal=True, out=o)
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)
