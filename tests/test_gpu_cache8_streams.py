"""Calls of the 8-bit cache and the rotation on a stream of their own: the memory that they take for
themselves belongs to that stream, so nothing waits and nothing is shared."""
import pytest
import torch

import paper_2609_34606_amd as P
from test_gpu_cache8 import BF, run_case
from test_gpu_tokens import i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def split_case():
    """A call that is cut into pieces, so that it needs a workspace."""
    pages = 20
    c, q, _, _ = run_case(9, 1, 8, 2, 128, 128, 1, BF, pages)
    assert P.hsa_cache8_attn_workspace_size(c.cfg, 1, 2, 0, pages) > 0
    return c, q, pages


class Spy:
    """The library's attention call, its workspace and output addresses noted."""

    def __init__(self, monkeypatch):
        self.fn, self.seen = P.lib().hsa_cache8_attn, []
        monkeypatch.setattr(P.lib(), "hsa_cache8_attn", self)

    def __call__(self, *args):
        self.seen.append((args[14], args[12]))  # (ws, o)
        return self.fn(*args)


@pytest.mark.parametrize("as_handle", [False, True])
def test_a_side_stream_does_not_get_the_current_streams_memory(monkeypatch, as_handle):
    """Blocks that a call on the current stream let go may still be written by it: a call on another
    stream, right after, gets others, and the other way round."""
    c, q, pages = split_case()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    spy = Spy(monkeypatch)
    on = s.cuda_stream if as_handle else s
    for _ in range(3):
        c.attend(q, pages)
        c.attend(q, pages, stream=on)
    torch.cuda.synchronize()
    for column in (0, 1):
        here = {x[column] for x in spy.seen[0::2]}
        there = {x[column] for x in spy.seen[1::2]}
        assert not here & there


@pytest.mark.parametrize("as_handle", [False, True])
def test_current_and_side_stream_without_a_wait(as_handle):
    """Split calls issued on the current stream and on a side stream in turn, outputs and workspaces
    their own: the serial results."""
    c, q, pages = split_case()
    q2 = (q * 0.5).contiguous()
    c.rope = P.rope(128)
    first = i32([7])
    want, want2 = c.attend(q, pages), c.attend(q2, pages)
    turned = c.rotate(q2, first=first)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    on = s.cuda_stream if as_handle else s
    outs, outs2, turns = [], [], []
    for _ in range(20):
        outs.append(c.attend(q, pages))
        outs2.append(c.attend(q2, pages, stream=on))
        turns.append(c.rotate(q2, first=first, stream=on))
    torch.cuda.synchronize()
    for got, w in ((outs, want), (outs2, want2), (turns, turned)):
        for o in got:
            assert torch.equal(o, w)


def test_an_output_let_go_is_not_written_before_its_reader_is_done(monkeypatch):
    """An output made on a side stream and read on the current one (after a wait): letting it go does
    not give its memory to the side stream's next call while the reader is queued."""
    c, q, pages = split_case()
    q2 = (q * 0.5).contiguous()
    want = c.attend(q, pages).float()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = torch.randn((4096, 4096), device=DEV)
    out = c.attend(q, pages, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    for _ in range(20):
        busy = busy @ busy * 1e-3  # the reader is queued behind this
    read = out.float()
    del out
    for _ in range(5):
        c.attend(q2, pages, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(read, want)


def test_default_stream_handle():
    """Handle 0 is the default stream."""
    c, q, pages = split_case()
    assert torch.equal(c.attend(q, pages, stream=0), c.attend(q, pages))
