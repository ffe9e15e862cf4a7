"""Refusals of the calls of drafted trees, kept tokens and page tables: they return before any launch, so
none of these needs a GPU."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2609_34606_amd as P
from paper_2609_34606_amd import hsa as H

by = ctypes.byref
FAKE = 0x10000
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
POOL = lambda **kw: _with(H.HsaKvPool(FAKE, FAKE, FAKE, 4, 4), **kw)
CACHE = lambda **kw: _with(H.HsaCache8Pool(FAKE, FAKE, FAKE, FAKE, FAKE, 4, 4, 2), **kw)
SLOTS = lambda **kw: _with(H.HsaSlotTable(FAKE, FAKE, 4, 4), **kw)


def _with(c, **kw):
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_the_package_has_every_call():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hsa.h")).read(), flags=re.S)
    names = {n for n in re.findall(r"\b(hsa_[a-z0-9_]+)\s*\(", src) if re.match(r"hsa_(tree|slots|token_keep|page_copy|cache8)", n)}
    assert len(names) == 18
    for n in names:
        assert hasattr(P.lib(), n) and hasattr(P, n), n


def test_mask_refusals():
    cfg = P.config(1, 1, 64, 8, "bf16")

    def call(cfg=cfg, parent=FAKE, n=4, mask=FAKE):
        return P.lib().hsa_tree_mask(by(cfg), parent, n, None, None, mask, None, None)
    assert call(n=0, parent=None, mask=None) == 0
    assert call(parent=None) == 1 and call(mask=None) == 1 and call(n=-1) == 1
    assert call(n=257) == 2 and call(cfg=P.config(1, 1, 96, 8, "bf16")) == 2


def test_attention_refusals():
    cfg = P.config(1, 4, 64, 256, "bf16")
    kh = np.array([1, 3], np.int32)

    def pool(dst=POOL(), kv=2, q=FAKE, n_q=2, sel=None, k_max=0, k_h=None, first=0, n=4, o=FAKE, ws=None, nb=0, cfg=cfg):
        return P.lib().hsa_tree_attn(by(cfg), q, n_q, None if dst is None else by(dst), kv, sel, k_max, k_h, first, n, None,
                                     None, None, o, None, ws, nb, None)

    def codes(dst=CACHE(), q=FAKE, n_q=2, sel=None, k_max=0, k_h=None, first=0, n=4, o=FAKE, ws=None, nb=0, cfg=cfg):
        return P.lib().hsa_cache8_tree_attn(by(cfg), q, n_q, None if dst is None else by(dst), sel, k_max, k_h, first, n,
                                            None, None, None, o, None, ws, nb, None)
    for attn, make, size in ((pool, POOL, P.hsa_tree_attn_workspace_size),
                             (codes, CACHE, P.hsa_cache8_tree_attn_workspace_size)):
        assert attn(n_q=0) == 0
        assert attn(dst=None) == 1 and attn(q=None) == 1 and attn(o=None) == 1
        assert attn(n_q=-1) == 1 and attn(first=-1) == 1 and attn(n=-1) == 1 and attn(k_max=-1) == 1
        assert attn(n=0) == 1                                    # an empty list
        assert attn(k_max=2) == 1                                # no selection
        assert attn(sel=FAKE, k_max=2, k_h=kh.ctypes.data) == 1  # a budget above k_max
        assert attn(first=1) == 3                                # pages past the table
        assert attn(q=FAKE + 2) == 2 and attn(o=FAKE + 8) == 2
        assert attn(sel=FAKE, k_max=2000) == 2 and attn(n_q=257) == 2
        assert attn(dst=make(k=FAKE + 8)) == 2 and attn(dst=make(v=FAKE + 2)) == 2
        assert attn(dst=make(max_pages=1 << 23)) == 2            # 2^31 tokens
        assert attn(cfg=P.config(70000, 4, 64, 256, "bf16")) == 2
        # a list of 2^31 tokens, though the sequence has fewer
        big = P.config(1, 4, 64, 1 << 21, "bf16")
        assert attn(cfg=big, dst=make(max_pages=900), sel=FAKE, k_max=1000, n=100) == 2
        need = size(cfg, 2, 2, 0, 400)
        assert need > 0 and need % 256 == 0
        for ws, nb in ((None, 0), (FAKE, need - 1), (FAKE + 16, need)):
            assert attn(dst=make(max_pages=400), n=400, ws=ws, nb=nb) == 4
        for bad in ((0, 2, 0, 4), (2, 3, 0, 4), (2, 2, -1, 4), (2, 2, 0, 0), (2, 0, 0, 4), (257, 2, 0, 4)):
            assert size(cfg, *bad) == 0
    assert pool(kv=3) == 1 and pool(kv=0) == 1 and codes(dst=CACHE(kv_heads=3)) == 1


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_workspace_serves_every_shorter_list(dt, eight):
    size = P.hsa_cache8_tree_attn_workspace_size if eight else P.hsa_tree_attn_workspace_size
    for B, heads, kv, n_q, P_ in ((1, 12, 12, 1, 1560), (32, 32, 8, 16, 256), (2, 6, 2, 25, 40), (1, 16, 2, 256, 8)):
        cfg = P.config(B, heads, 128, P_, dt)
        sizes = [size(cfg, n_q, kv, 0, n) for n in range(1, 400)]
        assert sizes == sorted(sizes) and sizes[-1] > 0
        assert size(cfg, n_q, kv, 100, 299) == sizes[398]


def test_keep_refusals():
    cfg = P.config(1, 2, 64, 256, "f32")
    for name, make in (("hsa_token_keep", POOL), ("hsa_cache8_keep", CACHE)):
        def keep(dst=make(), index=FAKE, n=3, cfg=cfg):
            return getattr(P.lib(), name)(by(cfg), None if dst is None else by(dst), FAKE, index, n, None, None)
        assert keep(n=0, index=None) == 0
        assert keep(dst=None) == 1 and keep(index=None) == 1 and keep(n=-1) == 1
        assert keep(n=257) == 2 and keep(dst=make(k=FAKE + 8)) == 2 and keep(dst=make(max_pages=1 << 23)) == 2
        assert keep(cfg=P.config(70000, 2, 64, 256, "f32")) == 2 and keep(cfg=P.config(1, 2, 64, 12, "f32")) == 2


def test_page_copy_refusals():
    cfg = P.config(1, 2, 64, 256, "bf16")
    for name, make in (("hsa_page_copy", POOL), ("hsa_cache8_page_copy", CACHE)):
        def copy(dst=make(), moves=FAKE, n=3, cfg=cfg):
            return getattr(P.lib(), name)(by(cfg), None if dst is None else by(dst), moves, n, None)
        assert copy(n=0, moves=None) == 0
        assert copy(dst=None) == 1 and copy(moves=None) == 1 and copy(n=-1) == 1
        assert copy(dst=make(v=FAKE + 8)) == 2 and copy(n=1 << 30) == 2
        assert copy(cfg=P.config(1, 2, 64, (1 << 24) + 8, "bf16")) == 2


def test_slot_refusals():
    cfg = P.config(3, 1, 64, 16, "bf16")
    lib = P.lib()
    need = P.hsa_slots_workspace_size(cfg, 4, 4)
    assert need > 0 and need % 256 == 0

    def take(slots=SLOTS(), end=FAKE, ws=FAKE, nb=need, cfg=cfg):
        return lib.hsa_slots_take(by(cfg), None if slots is None else by(slots), None, end, None, None, ws, nb, None)

    def fork(slots=SLOTS(), parent=FAKE, ws=FAKE, nb=need, cfg=cfg):
        return lib.hsa_slots_fork(by(cfg), None if slots is None else by(slots), parent, ws, nb, None)

    def free(slots=SLOTS(), keep=FAKE, cfg=cfg):
        return lib.hsa_slots_free(by(cfg), None if slots is None else by(slots), keep, None)

    def compact(slots=SLOTS(), moves=FAKE, n=4, ws=FAKE, nb=need, cfg=cfg):
        return lib.hsa_slots_compact(by(cfg), None if slots is None else by(slots), moves, n, None, None, ws, nb, None)
    for call in (take, fork, free, compact):
        for bad in (None, SLOTS(page_table=None), SLOTS(refs=None), SLOTS(num_slots=0), SLOTS(max_pages=0)):
            assert call(slots=bad) == 1
        assert call(slots=SLOTS(max_pages=1 << 27)) == 2 and call(slots=SLOTS(num_slots=(1 << 30) + 1)) == 2
        assert call(cfg=P.config(70000, 1, 64, 16, "bf16")) == 2
        assert call(cfg=P.config(60000, 1, 64, 16, "bf16"), slots=SLOTS(max_pages=20000)) == 2
    for call in (take, fork, compact):
        assert call(nb=need - 1) == 4 and call(ws=None) == 4 and call(ws=FAKE + 16) == 4
    assert take(end=None) == 1 and fork(parent=None) == 1 and free(keep=None) == 1
    assert compact(moves=None) == 1 and compact(n=-1) == 1 and compact(n=(1 << 29) + 1) == 2
    for bad in ((0, 4), (4, 0), (4, 1 << 27)):
        assert P.hsa_slots_workspace_size(cfg, *bad) == 0


def test_binding_refuses_wrong_tensors():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    layer = P.HsaLayer(2, 2, 64, 72, torch.bfloat16, "cpu", num_slots=3, max_pages=2)
    cache = P.HsaCache8(2, 4, 64, 72, torch.bfloat16, "cpu", kv_heads=2, num_slots=3, max_pages=2)
    q = torch.zeros((2, 3, 4, 64), dtype=torch.bfloat16)
    for c in (layer, cache):
        for args, kw in (((q.float(),), {}), ((q,), dict(kv_len=i32(1))), ((q,), dict(mask=i32(2, 3, 2))),
                         ((q,), dict(mask=torch.zeros((2, 3, 1)))), ((q,), dict(sel=i32(2, 4, 1))),
                         ((q,), dict(lse=torch.zeros(5))), ((q,), dict(q_len=i32(3)))):
            with pytest.raises(ValueError):
                c.attend_tree(*args, 1, **kw)
        for args, kw in (((i32(1), i32(2, 3)), {}), ((i32(2), i32(3, 3)), {}), ((i32(2), i32(2, 3)), dict(count=i32(3))),
                         ((i32(2).float(), i32(2, 3)), {})):
            with pytest.raises(ValueError):
                c.keep_tokens(*args, **kw)
        for moves in (i32(3, 2), i32(3, 3).float()):
            with pytest.raises(ValueError):
                c.copy_pages(moves)
    s = P.HsaSlots(2, 8, "cpu", num_slots=5, max_pages=3)
    assert s.page_table.tolist() == [[-1] * 3] * 2 and s.refs.tolist() == [0] * 5
    for call in (lambda: s.take(i32(1), i32(2)), lambda: s.take(None, i32(3)), lambda: s.take(None, i32(2), moves=i32(1, 3)),
                 lambda: s.fork(i32(3)), lambda: s.free(i32(1)), lambda: s.compact(i32(4, 2)),
                 lambda: s.compact(i32(4, 3), table_out=i32(5)), lambda: s.compact(i32(4, 3), refs_out=i32(4))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        P.HsaSlots(2, 8, "cpu", page_table=i32(2, 3))
    with pytest.raises(ValueError):
        P.HsaSlots(2, 8, "cpu", page_table=i32(3, 3), refs=i32(4))
    with pytest.raises(ValueError):
        P.hsa_tree_mask(P.config(2, 1, 64, 8, "bf16"), i32(2, 3), 3, i32(2, 3, 2))
