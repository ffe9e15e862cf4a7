"""Arguments of the 8-bit cache's and the rotation's calls that the binding or the library
settles before any launch; none of these needs a GPU."""
import ctypes
import math

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2609_34606_amd as P

BF = torch.bfloat16


def test_a_workspace_on_another_device_is_refused():
    """(tensors without memory that say that they are on a GPU)"""
    cfg = P.config(1, 2, 64, 64, BF)
    cache = P.HsaCache8(1, 2, 64, 64, BF, "cpu", num_slots=2, max_pages=2).pool
    with FakeTensorMode():
        q, o = (torch.empty((1, 3, 2, 64), dtype=BF, device="cuda:0") for _ in range(2))
        for where in ("cpu", "cuda:1"):
            ws = torch.empty(256, dtype=torch.uint8, device=where)
            with pytest.raises(ValueError, match="ws is on"):
                P.hsa_cache8_attn(cfg, q, 3, cache, None, 0, None, 0, 2, o, ws=ws)


def _apply(rope, pos=None, n=1):
    """Status of a call that reads no memory where it is refused (without a GPU the launch of a
    valid one fails: 5)."""
    cfg = P.config(1, 1, 64, 64, BF)
    return P.lib().hsa_rope_apply(ctypes.byref(cfg), ctypes.byref(rope), 0x10000, 64, 64, n, 1, pos, None, 0, 0x10000,
                                  64, 64, None)


def test_ropes_out_of_the_kernels_range_are_refused():
    """An amplitude beyond fp32, and frequencies whose angle at a far position no longer has its
    fraction of a quarter turn in fp64: 2^18 pi radians a position are 2^19 quarters."""
    most = 2.0 ** 18 * math.pi
    f32_max = float(torch.finfo(torch.float32).max)
    for kw in (dict(amplitude=1e39), dict(amplitude=-1e39), dict(amplitude=f32_max * (1 + 2.0 ** -24)),
               dict(scaling="linear", factor=1 / (most * 1.001)), dict(scaling="linear", factor=1e-300),
               dict(scaling="parts", factor=1e-9, low=10.0, high=11.0, orig_len=10), dict(theta=1e-12),
               dict(theta=1e-300)):
        assert _apply(P.rope(64, **kw), n=1) == 1, kw
        # 8-bit and pool appends take the same table
        cfg, pool = P.config(1, 2, 64, 64, BF), P.HsaKvPool(*[0x10000] * 3, 4, 4)
        assert P.lib().hsa_token_write(ctypes.byref(cfg), ctypes.byref(pool), ctypes.byref(P.rope(64, **kw)), 0x10000, 0,
                                       128, 0x10000, 0, 128, 0, None, None, None, None) == 1, kw
    for kw in (dict(amplitude=f32_max), dict(scaling="linear", factor=1.001 / most), dict(theta=1e-4),
               dict(theta=0.5), dict(amplitude=1e-60)):
        assert _apply(P.rope(64, **kw), n=0) == 0, kw


def test_a_new_cache_has_zero_exponents():
    """Whatever its memory held: a first append that begins inside a block keeps the larger of its own
    exponent and the byte there, and 255 would make every code 0."""
    held = torch.are_deterministic_algorithms_enabled(), torch.utils.deterministic.fill_uninitialized_memory
    torch.use_deterministic_algorithms(True)
    torch.utils.deterministic.fill_uninitialized_memory = True  # (new memory: 255 in every byte)
    try:
        assert (torch.empty(4, dtype=torch.uint8) == 255).all()
        c = P.HsaCache8(1, 2, 64, 72, BF, "cpu", num_slots=3, max_pages=2)
    finally:
        torch.use_deterministic_algorithms(held[0])
        torch.utils.deterministic.fill_uninitialized_memory = held[1]
    for e in (c.k_exp, c.v_exp):
        assert e.shape == (3, 2, 2) and (e == 0).all()


def test_rotate_keeps_the_gradient(monkeypatch):
    """The rotated queries of a tensor that needs a gradient have one: the opposite rotation's,
    twice differentiable. (The kernel is replaced by the same map, quarter turns here, on the CPU.)"""
    calls = []

    def turn(cfg, rope, x, n, o, pos=None, first=None, inverse=False, stream=None):
        half = rope.rot_dim // 2
        a, b = x[..., :half], x[..., half:]
        assert x.stride(3) == 1 and x.stride(2) == x.shape[3]
        o.copy_(torch.cat([b, -a] if inverse else [-b, a], -1) * first.view(-1, 1, 1, 1))
        calls.append((inverse, stream))
    monkeypatch.setattr(P.hsa, "hsa_rope_apply", turn)
    c = P.HsaCache8(2, 3, 64, 64, torch.float32, "cpu", num_slots=2, max_pages=2, rope=P.rope(64))
    g = torch.Generator().manual_seed(1)
    q = torch.randn((2, 4, 3, 64), generator=g, requires_grad=True)
    up = torch.randn((2, 4, 3, 64), generator=g)
    first = torch.tensor([2, 3], dtype=torch.int32)
    out = c.rotate(q, first=first)
    assert out.requires_grad
    out.backward(up)
    by = first.view(-1, 1, 1, 1)
    assert torch.equal(q.grad, torch.cat([up[..., 32:], -up[..., :32]], -1) * by)
    assert [x[0] for x in calls] == [False, True]
    # through a sum (an expanded gradient), and twice
    grad, = torch.autograd.grad((c.rotate(q, first=first) ** 2).sum(), q, create_graph=True)
    want = 2 * q * by ** 2  # (this product rounds once, the two by 3 of the other side once each: half a step, 2^-24)
    assert ((grad - want).abs() <= 3 * 2.0 ** -24 * want.abs()).all()
    twice, = torch.autograd.grad(grad.sum(), q)
    assert torch.equal(twice, (2 * by ** 2).expand_as(q))
    c.rotate(q, first=first).sum().backward()
    # no graph where none is asked for
    with torch.no_grad():
        assert not c.rotate(q, first=first, out=torch.empty_like(q)).requires_grad
    assert not c.rotate(q.detach(), first=first).requires_grad
    with pytest.raises(ValueError, match="gradient"):
        c.rotate(q, first=first, out=torch.empty_like(q))
    # positions changed before the backward pass are noticed
    out = c.rotate(q, first=first)
    first += 1
    with pytest.raises(RuntimeError, match="modified"):
        out.sum().backward()
