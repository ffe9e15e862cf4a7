"""Page tables of HsaSlots worked on from several streams: a call's workspace is memory of its own stream, and
the table's tensors are not given away while a stream's calls on them are on their way."""
import pytest
import torch

import paper_2609_34606_amd as P
from test_gpu_tokens import i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_a_calls_workspace_is_of_its_stream(monkeypatch):
    """The calls of each stream have a workspace allocated on it, a captured call one of its graph."""
    made = []
    real = torch.empty

    def empty(*a, **kw):
        t = real(*a, **kw)
        if t.is_cuda and t.dtype is torch.uint8:
            made.append((torch.cuda.current_stream().cuda_stream, t.data_ptr()))
        return t

    s = P.HsaSlots(2, 8, DEV, num_slots=9, max_pages=4)
    side = torch.cuda.Stream()
    end, parent = i32([17, 9]), i32([1, 1])
    moves = torch.zeros((3, 3), dtype=torch.int32, device=DEV)
    seen = []
    for name in ("hsa_slots_take", "hsa_slots_fork", "hsa_slots_compact"):
        def call(*a, fn=getattr(P.lib(), name)):
            seen.append(a[-3])  # ws
            return fn(*a)
        monkeypatch.setattr(P.lib(), name, call)
    torch.cuda.synchronize()
    monkeypatch.setattr(torch, "empty", empty)
    s.take(None, end, stream=side)
    s.fork(parent, stream=side.cuda_stream)
    with torch.cuda.stream(side):
        s.compact(moves)
    assert [x for x, _ in made] == [side.cuda_stream] and seen == [made[0][1]] * 3
    torch.cuda.synchronize()  # (calls on one table follow each other)
    s.fork(parent)
    here = torch.cuda.current_stream().cuda_stream
    assert [x for x, _ in made] == [side.cuda_stream, here] and seen[3] == made[1][1] != seen[0]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            s.fork(parent)
            s.take(None, end)
    torch.cuda.synchronize()
    assert len({x for x in seen[:4]} & set(seen[4:])) == 0 and len(seen) == 8
    monkeypatch.undo()
    for g in graphs + graphs:
        g.replay()
    s.compact(moves)
    torch.cuda.synchronize()
    held = s.page_table[s.page_table >= 0].tolist()
    assert int(s.missing) == 0 and s.refs.tolist() == [held.count(x) for x in range(9)]


@pytest.mark.parametrize("how", ["argument", "current"])
def test_tensors_outlive_a_side_streams_calls(how):
    """The tables of a released object are written to by what a side stream has yet to run: tensors made in their place
    stay what they are."""
    side = torch.cuda.Stream()
    wait = torch.cuda.Event()
    big = torch.randn((4096, 4096), device=DEV)
    big @ big
    for size in (9, 700):
        s = P.HsaSlots(4, 8, DEV, num_slots=size, max_pages=4)
        end = i32([32] * 4)
        torch.cuda.synchronize()
        at = {t.data_ptr() for t in (s.page_table, s.refs, s.missing)}
        with torch.cuda.stream(side):
            for _ in range(30):
                big @ big
            if how == "current":
                s.take(None, end)
        if how == "argument":
            s.take(None, end, stream=side)
        wait.record(side)
        shapes = [x.shape for x in (s.page_table, s.refs, s.missing)]
        del s
        new = [torch.full(x, 77, dtype=torch.int32, device=DEV) for x in shapes for _ in range(3)]
        busy = not wait.query()
        assert not (busy and at & {t.data_ptr() for t in new})
        torch.cuda.synchronize()
        assert all(bool((t == 77).all()) for t in new)
