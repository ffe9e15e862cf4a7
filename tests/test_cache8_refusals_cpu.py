"""Refusals of the rotary, append and 8-bit cache calls: they return before any
launch, so none of these needs a GPU."""
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


def test_every_declared_function_is_exported():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hsa.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(hsa_[a-z0-9_]+)\s*\(", src))
    assert {"hsa_rope_apply", "hsa_token_write", "hsa_cache8_write", "hsa_cache8_attn"} <= names
    for n in names:
        assert hasattr(P.lib(), n), n


def _rope_call(cfg, rope, x=FAKE, o=FAKE, n=4, heads=2, pos=None, xb=64, xt=64):
    return P.lib().hsa_rope_apply(by(cfg), None if rope is None else by(rope), x, xb, xt, n, heads, pos, None, 0, o,
                                  64, 64, None)


def test_rope_refusals():
    cfg = P.config(1, 2, 64, 64, "bf16")
    ok = P.rope(64)
    assert _rope_call(cfg, ok, n=0) == 0
    assert _rope_call(cfg, None) == 1
    assert _rope_call(cfg, ok, x=None) == 1 and _rope_call(cfg, ok, o=None) == 1
    assert _rope_call(cfg, ok, n=-1) == 1 and _rope_call(cfg, ok, heads=0) == 1
    assert _rope_call(cfg, ok, xb=-1) == 1 and _rope_call(cfg, ok, xt=-64) == 1
    assert _rope_call(cfg, ok, heads=65) == 2
    assert _rope_call(cfg, ok, n=1 << 30) == 2
    assert _rope_call(P.config(1, 2, 96, 64, "bf16"), ok) == 2

    def changed(**kw):
        r = P.rope(64)
        for k, v in kw.items():
            setattr(r, k, v)
        return r
    nan = float("nan")
    for bad in (dict(rot_dim=63), dict(rot_dim=66), dict(rot_dim=0), dict(layout=2), dict(axes=0), dict(axes=4),
                dict(axes=2), dict(theta=0.0), dict(theta=nan), dict(scaling=3), dict(scaling=1, factor=0.0),
                dict(scaling=2, factor=2.0, low=4.0, high=4.0, orig_len=10),
                dict(scaling=2, factor=2.0, low=1.0, high=4.0, orig_len=0), dict(amplitude=nan)):
        assert _rope_call(cfg, changed(**bad)) == 1, bad
    three = P.rope(64, axis_dims=[20, 22, 22])
    assert _rope_call(cfg, three) == 1                  # axes without positions
    assert _rope_call(cfg, three, pos=FAKE, n=0) == 0
    three.axis_dim[0] = 18
    assert _rope_call(cfg, three, pos=FAKE) == 1        # they no longer sum to rot_dim
    for kw in (dict(layout="both"), dict(scaling="more"), dict(axis_dims=[32, 16]), dict(axis_dims=[16] * 4)):
        with pytest.raises(ValueError):
            P.rope(64, **kw)


def _cache(**kw):
    c = H.HsaCache8Pool(FAKE, FAKE, FAKE, FAKE, FAKE, 4, 4, 2)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_write_refusals():
    lib = P.lib()
    cfg = P.config(1, 4, 64, 256, "f32")
    pool = H.HsaKvPool(FAKE, FAKE, FAKE, 4, 4)

    def write(name, dst, k=FAKE, v=FAKE, n=3, kt=256, rope=None, pos=None, cfg=cfg):
        return getattr(lib, name)(by(cfg), None if dst is None else by(dst), rope, k, 0, kt, v, 0, 256, n, pos, None,
                                  None, None)
    for name, dst in (("hsa_token_write", pool), ("hsa_cache8_write", _cache())):
        assert write(name, dst, n=0) == 0
        assert write(name, None) == 1
        assert write(name, dst, k=None) == 1 and write(name, dst, v=None) == 1
        assert write(name, dst, n=-1) == 1 and write(name, dst, kt=-1) == 1
        assert write(name, dst, rope=by(P.rope(66))) == 1
        assert write(name, dst, cfg=P.config(1, 4, 64, 12, "f32")) == 2
        assert write(name, dst, cfg=P.config(70000, 4, 64, 256, "f32")) == 2
    assert write("hsa_token_write", H.HsaKvPool(FAKE, FAKE, FAKE, 0, 4)) == 1
    assert write("hsa_token_write", H.HsaKvPool(FAKE, FAKE, FAKE, 4, 1 << 23)) == 2  # 2^31 tokens
    for bad in (dict(k=None), dict(v_exp=None), dict(page_table=None), dict(num_slots=0), dict(kv_heads=0),
                dict(kv_heads=3)):
        assert write("hsa_cache8_write", _cache(**bad)) == 1, bad
    assert write("hsa_cache8_write", _cache(k=FAKE + 8)) == 2


def test_attention_refusals():
    lib = P.lib()
    cfg = P.config(1, 4, 64, 256, "bf16")
    kh = np.array([1, 3], np.int32)

    def attn(cache=_cache(), q=FAKE, n_q=2, sel=None, k_max=0, k_h=None, first=0, n=4, o=FAKE, ws=None, nb=0, cfg=cfg):
        return lib.hsa_cache8_attn(by(cfg), q, n_q, None if cache is None else by(cache), sel, k_max, k_h, first, n,
                                   None, None, 0, o, None, ws, nb, None)
    assert attn(n_q=0) == 0
    assert attn(cache=None) == 1 and attn(q=None) == 1 and attn(o=None) == 1
    assert attn(n_q=-1) == 1 and attn(first=-1) == 1 and attn(n=-1) == 1 and attn(k_max=-1) == 1
    assert attn(n=0) == 1                                # an empty list
    assert attn(k_max=2) == 1                            # no selection
    assert attn(sel=FAKE, k_max=2, k_h=kh.ctypes.data) == 1  # a budget above k_max
    assert attn(first=1) == 3                            # pages past the table
    assert attn(q=FAKE + 2) == 2 and attn(o=FAKE + 8) == 2
    assert attn(sel=FAKE, k_max=2000) == 2
    assert attn(cache=_cache(kv_heads=3)) == 1
    assert attn(cache=_cache(max_pages=1 << 23)) == 2
    assert attn(cfg=P.config(70000, 4, 64, 256, "bf16")) == 2
    long = _cache(max_pages=400)
    size = P.hsa_cache8_attn_workspace_size(cfg, 2, 2, 0, 400)
    assert size > 0 and size % 256 == 0
    for ws, nb in ((None, 0), (FAKE, size - 1), (FAKE + 16, size)):
        assert attn(cache=long, n=400, ws=ws, nb=nb) == 4
    for bad in ((0, 2, 0, 4), (2, 3, 0, 4), (2, 2, -1, 4), (2, 2, 0, 0), (2, 0, 0, 4)):
        assert P.hsa_cache8_attn_workspace_size(cfg, *bad) == 0
    assert P.hsa_cache8_attn_workspace_size(P.config(1, 4, 96, 256, "bf16"), 2, 2, 0, 4) == 0


def test_binding_refuses_wrong_tensors():
    c = P.HsaCache8(2, 4, 64, 72, torch.bfloat16, "cpu", kv_heads=2, num_slots=3, max_pages=2, rope=P.rope(64))
    assert c.k.shape == (3, 2, 72, 64) and c.v.shape == (3, 2, 64, 72) and c.k_exp.shape == (3, 2, 2)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)
    good = bf(2, 5, 2, 64)
    for k, v, kw in ((bf(2, 5, 4, 64), good, {}), (good, bf(2, 4, 2, 64), {}), (good.float(), good, {}),
                     (bf(2, 5, 64, 2).transpose(2, 3), good, {}), (good, good, dict(first=i32(1))),
                     (good, good, dict(first=torch.zeros(2))), (good, good, dict(count=i32(1, 2, 3))),
                     (good, good, dict(pos=i32(1, 2)))):
        with pytest.raises(ValueError):
            c.write(k, v, **kw)
    q = bf(2, 3, 4, 64)
    for args, kw in (((bf(2, 3, 2, 64),), {}), ((q.float(),), {}), ((q,), dict(kv_len=i32(1))),
                     ((q,), dict(sel=torch.zeros((2, 4, 1), dtype=torch.int32))),
                     ((q,), dict(sel=torch.zeros((2, 2, 1), dtype=torch.int32), k_h=[1])),
                     ((q,), dict(lse=torch.zeros(5))), ((q,), dict(lse=torch.zeros(2, 4, 3, dtype=torch.float64)))):
        with pytest.raises(ValueError):
            c.attend(*args, 1, **kw)
    with pytest.raises(ValueError):
        c.rotate(q, pos=i32(1))
    with pytest.raises(ValueError):
        c.rotate(q, out=bf(2, 3, 4, 128))
    with pytest.raises(ValueError):
        P.cache8_pool(c.k, c.v, c.k_exp, c.v_exp[..., :1], c.page_table, c.cfg)
    with pytest.raises(ValueError):
        P.HsaCache8(2, 4, 64, 72, torch.bfloat16, "cpu", kv_heads=4, k=c.k, v=c.v, k_exp=c.k_exp, v_exp=c.v_exp,
                    page_table=c.page_table)


def test_empty_and_overlapping_calls():
    """No tokens need no memory; an output whose tokens share a place is refused."""
    cfg, rope = P.config(2, 2, 64, 64, "bf16"), P.rope(64)

    def apply(n, ob, ot, x=FAKE, o=FAKE):
        return P.lib().hsa_rope_apply(by(cfg), by(rope), x, 0, 0, n, 2, None, None, 0, o, ob, ot, None)
    assert apply(0, 0, 0, x=None, o=None) == 0
    for n, ob, ot in ((3, 384, 0), (3, 0, 128), (3, 300, 128), (3, 384, 100), (1, 100, 128), (3, 128, 200)):
        assert apply(n, ob, ot) == 1, (n, ob, ot)
    pool = H.HsaKvPool(FAKE, FAKE, FAKE, 4, 4)
    for name, dst in (("hsa_token_write", pool), ("hsa_cache8_write", _cache())):
        assert getattr(P.lib(), name)(by(cfg), by(dst), None, None, 0, 128, None, 0, 128, 0, None, None, None, None) == 0
    assert P.lib().hsa_cache8_attn(by(cfg), None, 0, by(_cache()), None, 0, None, 0, 4, None, None, 0, None, None,
                                   None, 0, None) == 0


def test_sizes_past_a_launch_are_refused():
    lib = P.lib()
    cfg, pool = P.config(1, 64, 64, 64, "bf16"), H.HsaKvPool(FAKE, FAKE, FAKE, 4, 4)
    assert lib.hsa_token_write(by(cfg), by(pool), None, FAKE, 0, 4096, FAKE, 0, 4096, 1 << 23, None, None, None,
                               None) == 2
    assert lib.hsa_cache8_attn(by(cfg), FAKE, 1 << 29, by(_cache()), None, 0, None, 0, 4, None, None, 0, FAKE, None,
                               None, 0, None) == 2
    assert lib.hsa_cache8_attn(by(P.config(1, 2, 64, (1 << 24) + 8, "bf16")), FAKE, 1, by(_cache()), None, 0, None,
                               0, 4, None, None, 0, FAKE, None, None, 0, None) == 2


def test_a_cache_without_rope_does_not_rotate():
    c = P.HsaCache8(1, 2, 64, 64, torch.bfloat16, "cpu", num_slots=2, max_pages=2)
    with pytest.raises(ValueError):
        c.rotate(torch.zeros((1, 3, 2, 64), dtype=torch.bfloat16))
