"""Which kernel a call of the 8-bit cache's attention is planned for. The GPU tests of the
many-rows kernel are sized by this: a rule that moves them to the other kernel fails here."""
import ctypes

import pytest

import paper_2609_34606_amd as P
import test_gpu_cache8_many as many
import test_gpu_cache8_many_far as far


def plan(B, H, kv, d, P_, n_q, k_max, n, ragged=False, dtype="bf16"):
    return P.hsa_cache8_attn_plan(P.config(B, H, d, P_, dtype), n_q, kv, k_max, n, ragged)


@pytest.mark.parametrize("d", [64, 128])
def test_the_many_rows_tests_reach_their_kernel(d):
    room = many.ROOM[d]
    rows = {64: 128, 128: 256}[d]
    for P_ in (8, 16, 24, 32, 40, 48, 56, 64, 72, 104, 136, 200, 256, 392):
        is_many, per, pieces = plan(2, 4, 2, d, P_, 1024, 0, room // P_ + 1, True)
        assert is_many and per == rows and pieces > 1, P_
        pages = room // P_ + 3
        for B, H in ((1, 8), (2, 4)):  # over selected pages
            assert plan(B, H, H // 2, d, P_, 1024, pages - 2, 2, True)[0], P_
    for P_, dd, H, kv in ((16, 64, 4, 2), (200, 64, 6, 3), (40, 128, 8, 4), (256, 128, 3, 3)):
        assert plan(1, H, kv, dd, P_, 1111, 0, many.ROOM[dd] * 2 // P_ + 1, True)[0]


def test_the_far_offset_tests_reach_their_kernel():
    for d, P_, _, pages, n_q in far.FAR:
        for ragged in (False, True):
            is_many, _, pieces = plan(1, far.HEADS, far.HEADS, d, P_, n_q, 0, pages, ragged)
            assert is_many and pieces > 1, (d, P_)


def test_kinds_of_calls():
    """Single tokens and small calls go to the few-rows kernel, fp32 always does."""
    assert plan(32, 32, 8, 128, 256, 1, 0, 64, True)[:2] == (False, 16)
    assert plan(1, 12, 12, 128, 1560, 1, 0, 120)[2] > 1
    assert plan(1, 12, 12, 128, 1560, 4680, 4, 3)[:2] == (True, 256)
    assert plan(3, 16, 4, 64, 200, 1001, 0, 8, True)[:2] == (True, 128)
    assert plan(2, 4, 2, 64, 256, 4680, 0, 40, dtype="f32")[:2] == (False, 32)
    assert plan(1, 8, 8, 128, 1560, 100, 0, 2)[0] is False


def test_plan_refusals():
    lib, by = P.lib(), ctypes.byref
    cfg = P.config(1, 4, 64, 256, "bf16")

    def status(n_q=2, kv=2, k_max=0, n=4, cfg=cfg):
        return lib.hsa_cache8_attn_plan(None if cfg is None else by(cfg), n_q, kv, k_max, n, 0, None, None, None)
    assert status() == 0
    assert status(cfg=None) == 1
    for kw in (dict(n_q=0), dict(kv=0), dict(kv=3), dict(k_max=-1), dict(n=-1), dict(n=0)):
        assert status(**kw) == 1, kw
    assert status(n_q=1 << 30) == 2
    assert status(cfg=P.config(70000, 4, 64, 256, "bf16")) == 2
    assert status(cfg=P.config(1, 4, 96, 256, "bf16")) == 2
