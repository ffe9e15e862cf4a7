"""Single calls of the 8-bit cache and the rotation that a program makes and the other tests do
not: a first append inside a block, the gradient of rotated queries, one
workspace for lists of many lengths, pages listed twice, infinities beside the largest numbers."""
import numpy as np
import pytest
import torch

import paper_2609_34606_amd as P
from oracle import hsa_cache8_oracle as O
from test_gpu_cache8 import BF, F32
from test_gpu_cache8 import check as attended
from test_gpu_rope import EPS, check
from test_gpu_tokens import arrays, cache, host, i32, one_nan, source

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("P_", [16, 72, 200])
def test_first_append_inside_a_block(P_, dt):
    """A new cache's sequence that begins inside a block has the scale of its own tokens: the bits of
    one whose earlier tokens are zeros."""
    at, n = 5, 2 * P_ - 9
    k, v = source(P_, 2, n, 2, 64, dt, False)
    zero = torch.zeros((2, at, 2, 64), dtype=dt, device=DEV)
    held = []
    for before in (False, True):
        c = P.HsaCache8(2, 2, 64, P_, dt, DEV, num_slots=4, max_pages=2)
        c.page_table.copy_(torch.tensor([[3, 0], [1, 2]]))
        if before:
            c.write(zero, zero)
        c.write(k, v, i32([at, at]))
        held.append(c)
    new, old = held
    for b, pages in enumerate(([3, 0], [1, 2])):
        for i, s in enumerate(pages):
            first, last = at if i == 0 else 0, min(P_, at + n - i * P_)
            blocks = -(-last // 64)
            assert torch.equal(new.k[s, :, first:last], old.k[s, :, first:last])
            assert torch.equal(new.v[s, ..., first:last], old.v[s, ..., first:last])
            assert torch.equal(new.k_exp[s, :, :blocks], old.k_exp[s, :, :blocks])
            assert torch.equal(new.v_exp[s, :, :blocks], old.v_exp[s, :, :blocks])


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_gradient_through_rotate(layout, dt):
    """The gradient of rotated queries against the oracle's opposite rotation (bound:
    test_gpu_rope.py), of a fused projection's part, with a stream of its own, captured and replayed."""
    kw = dict(rot=48, layout=layout, amplitude=1.5)
    c = P.HsaCache8(2, 3, 64, 64, dt, DEV, num_slots=2, max_pages=2, rope=P.rope(48, layout=layout, amplitude=1.5))
    first = i32([7, 9001])
    where = O.places(first.cpu().numpy(), 33)
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((2, 33, 3, 3, 64), generator=g).to(dt).to(DEV).requires_grad_()
    up = torch.randn((2, 33, 3, 64), generator=g).to(dt).to(DEV)
    s = torch.cuda.Stream()
    for stream in (None, s):
        qkv.grad = None
        out = c.rotate(qkv[:, :, 1], first=first, stream=stream)
        torch.cuda.current_stream().wait_stream(s)
        check(host(qkv[:, :, 1].detach()), host(out.detach()), where, kw, EPS[dt])
        out.backward(up)
        check(host(up), host(qkv.grad[:, :, 1]), where, dict(kw, inverse=True), EPS[dt])
        assert (qkv.grad[:, :, 0] == 0).all() and (qkv.grad[:, :, 2] == 0).all()
    # captured: the forward and the backward pass, replayed on other positions
    q = qkv.detach()[:, :, 1].contiguous().requires_grad_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # (a first pass outside, as captured training needs)
        torch.autograd.grad(c.rotate(q, first=first), q, up)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = c.rotate(q, first=first)
        grad, = torch.autograd.grad(out, q, up)
    out = out.detach()
    for at in ([7, 9001], [0, 70000], [123, 5]):
        first.copy_(torch.tensor(at))
        graph.replay()
        torch.cuda.synchronize()
        eager = c.rotate(q, first=first)
        assert torch.equal(out, eager)
        assert torch.equal(grad, torch.autograd.grad(eager, q, up)[0])
        del eager


def test_rotated_attention_trains():
    """Rotated queries and keys in a plain attention: the gradient of the projections against
    differences of the loss in fp64 of the oracle's rotation."""
    B, n, heads, d = 1, 5, 2, 64
    c = P.HsaCache8(B, heads, d, 64, F32, DEV, num_slots=1, max_pages=1, rope=P.rope(d))
    g = torch.Generator().manual_seed(4)
    q, k = (torch.randn((B, n, heads, d), generator=g) for _ in range(2))
    where = O.places([11], n)

    def loss64(a, b):
        x, y = (O.rope(t, where, d) for t in (a, b))
        s = np.einsum("bihd,bjhd->bhij", x, y) / d ** 0.5
        return np.log(np.exp(s).sum(-1)).sum()
    ql, kl = (t.to(DEV).requires_grad_() for t in (q, k))
    first = i32([11])
    x, y = c.rotate(ql, first=first), c.rotate(kl, first=first)
    s = (x[:, :, None] * y[:, None]).sum(-1) / d ** 0.5  # [B, i, j, heads]
    torch.logsumexp(s, 2).sum().backward()
    # Differences of fp64 with a step of 2^-13 are off by about 2^-26 of the third derivative, and
    # fp32 by some 100 roundings of numbers of the gradient's size (below 3): 2^-14 covers both.
    r = np.random.default_rng(5)
    a, b = q.double().numpy(), k.double().numpy()
    for _ in range(3):
        da, db = r.standard_normal(a.shape), r.standard_normal(b.shape)
        size = np.sqrt((da ** 2).sum() + (db ** 2).sum())
        da, db = da / size, db / size
        h = 2.0 ** -13
        num = (loss64(a + h * da, b + h * db) - loss64(a - h * da, b - h * db)) / (2 * h)
        got = (host(ql.grad) * da).sum() + (host(kl.grad) * db).sum()
        assert abs(num - got) < 2.0 ** -14 * max(1.0, np.sqrt((host(ql.grad) ** 2).sum() + (host(kl.grad) ** 2).sum()))


@pytest.mark.parametrize("B,H,kv,d,P_,n_q,pages", [(1, 12, 12, 128, 256, 1, 64), (2, 4, 2, 64, 40, 5, 150),
                                                   (1, 12, 12, 128, 200, 700, 40), (8, 8, 8, 128, 64, 128, 60)])
def test_one_workspace_for_every_list_up_to_the_longest(B, H, kv, d, P_, n_q, pages):
    """A program's own workspace, as large as its longest list asks for: the bits of calls that take
    their own."""
    c, _ = cache(5, B, H, d, P_, BF, pages, kv=kv)
    c.write(*source(5, B, pages * P_, kv, d, BF, False))
    q = source(6, B, n_q, H, d, BF, False)[0]
    ws = torch.empty(P.hsa_cache8_attn_workspace_size(c.cfg, n_q, kv, 0, pages), dtype=torch.uint8, device=DEV)
    assert ws.numel() > 0
    cut = 0
    for n in list(range(1, pages, 3)) + [pages]:
        for ragged in (False, True):
            lens = i32([n * P_ - 5 * b for b in range(B)]) if ragged else None
            cut += P.hsa_cache8_attn_plan(c.cfg, n_q, kv, 0, n, ragged)[2] > 1
            out = torch.full_like(q, 3.0)
            P.hsa_cache8_attn(c.cfg, q, n_q, c.pool, None, 0, None, 0, n, out, kv_len=lens, ws=ws)
            assert torch.equal(out, c.attend(q, n, kv_len=lens)), n
    assert cut > 4


@pytest.mark.parametrize("d,P_,n_q,dt", [(128, 200, 1, BF), (64, 40, 3, F32), (64, 72, 30, BF), (128, 136, 1024, BF),
                                         (64, 24, 1024, BF)])
def test_a_page_listed_twice_counts_twice(d, P_, n_q, dt):
    """Among the selected pages, and as a selected one and one of the run."""
    B, H, kv, times = 2, 4, 2, 1 if n_q < 1024 else -(-4400 // P_ // 4)
    c, pt = cache(8, B, H, d, P_, dt, 4, kv=kv)
    w = P.HsaCache8(B, H, d, P_, F32, DEV, kv_heads=kv, k=c.k, v=c.v, k_exp=c.k_exp, v_exp=c.v_exp, page_table=c.page_table)
    w.write(*source(8, B, 4 * P_, kv, d, F32, False, 0.3))
    rows = [[3, 3, 0, 2] * times, [1, 1, 1, 1] * times]
    sel = i32([rows] * B)
    if n_q == 1024:
        assert P.hsa_cache8_attn_plan(c.cfg, n_q, kv, 4 * times, 2, True)[0]
    q = source(9, B, n_q, H, d, dt, False)[0]
    out, lse = torch.full_like(q, 3.0), torch.full((B, H, n_q), 5.0, device=DEV)
    lens, q_len = [4 * P_ - 3, 3 * P_ + 1], [min(n_q, 20), min(n_q, 7)]
    c.attend(q, 2, first_page=2, sel=sel, kv_len=i32(lens), q_len=i32(q_len), causal=True, out=out, lse=lse)
    kd, vd = O.dequantise(arrays(c))
    attended(q, out, lse, kd, vd, pt, [[r + [2, 3] for r in rows]] * B, lens, q_len, True, d ** -0.5)


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("P_,at,n", [(16, 0, 5), (16, 3, 40), (200, 0, 200), (200, 70, 3), (72, 5, 100)])
@pytest.mark.parametrize("rot", [0, 2])
def test_infinities_beside_the_largest_numbers(rot, P_, at, n, dt):
    """A block whose scale is the largest, 2^120, of which 448 is no fp32 number: infinities still become
    the largest code and NaN a NaN code, in a block of their own and in one that holds older tokens."""
    H, d = 3, 64
    c, pt = cache(7, 1, H, d, P_, dt, (at + n) // P_ + 1, rope=P.rope(rot) if rot else None)
    top = torch.finfo(dt).max
    g = np.random.default_rng(n)
    some = np.array([top, -top, np.inf, -np.inf, np.nan, 1e38, -2.0 ** 120, 1.0, 0.0])
    where = []
    for first, count in ((0, at), (at, n)):
        if not count:
            continue
        x = torch.from_numpy(g.choice(some, (2, 1, count, H, d))).to(dt).to(DEV)
        x[:, 0, 0, :, 5] = top  # (each block's scale is 2^120 from its first token on)
        x[0, ..., :rot] = 0.0   # (so that the rotated keys are exact)
        want = arrays(c)
        c.write(x[0], x[1], i32([first]))
        O.write8(want, pt, host(x[0]), host(x[1]), [first], [count])
        got = arrays(c)
        # the sign of the rotated zeros is the angle's
        for name in ("k", "v"):
            a, b = got[name], want[name]
            if name == "k":
                a, b = a[..., rot:], b[..., rot:]
            assert np.array_equal(one_nan(a), one_nan(b)), name
            assert np.array_equal(got[name + "_exp"], want[name + "_exp"])
        where.append(int((got["v"] == 0x7e).sum() + (got["k"] == 0x7e).sum()))
    assert min(where) > 0
