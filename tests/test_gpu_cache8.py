"""Attention over the 8-bit cache against the fp64 oracle, and the operators used
together.

Bound of an output in bf16: the weights and the output are rounded to bf16 once each (half a
step, 2^-8 of the value): 2^-8 (mean |v| + |o|). A score is an fp32 sum of d exact products,
off by (d + 4) 2^-24 of sum |q k|, scaled and subtracted in fp32 (2^-23 of its size,
twice), and exp2 and the sums over n keys round fp32 numbers: a weight is off by less than
w = 2 (d + 8) 2^-24 S + 2^-20, S the largest scaled sum |q k| of the row (at least
the score's own size), and the sum of n weighted values by n 2^-24 mean |v|. fp32 has no bf16
rounding (three parts leave 2^-24): the same without the first term. Weights below 2^-126 of
the largest have no normal fp32 (or bf16) number and may become 0: n 2^-126 max |v| more
(a row whose one heavy key has a zero there has no other term). The log-sum-exp is off
by w + n 2^-24 and its own rounding, 2^-23 of it.
"""
import numpy as np
import pytest
import torch

import paper_2609_34606_amd as P
from oracle import hsa_cache8_oracle as O
from test_gpu_tokens import arrays, cache, host, i32, source

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def run_case(seed, B, H, kv, d, P_, n_q, dt, pages, first=0, n=None, k_h=None, k_max=0, kv_len=None, q_len=None,
             causal=False, spread=0.3, scale=0.0, sel_valid=None):
    """Fills a cache up to kv_len (garbage, NaN among it, elsewhere), attends, checks."""
    n = pages - first if n is None else n
    r = np.random.default_rng(seed)
    c, pt = cache(seed, B, H, d, P_, dt, pages, kv=kv)
    if scale:
        c.cfg.sm_scale = scale
    cap = pages * P_
    lens = [cap] * B if kv_len is None else kv_len
    ks, vs = source(seed, B, cap, kv, d, torch.float32, False, spread)
    w = P.HsaCache8(B, H, d, P_, torch.float32, DEV, kv_heads=kv, k=c.k, v=c.v, k_exp=c.k_exp, v_exp=c.v_exp,
                    page_table=c.page_table)
    w.write(ks, vs, count=i32(lens))
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn((B, n_q, H, d), generator=g).to(dt).to(DEV)
    sel = None
    listed = [[list(range(first, first + n)) for _ in range(kv)] for _ in range(B)]
    if k_max:
        sel = np.full((B, kv, k_max), -1, np.int32)
        for b in range(B):
            for h in range(kv):
                m = k_max if sel_valid is None else sel_valid[(b * kv + h) % len(sel_valid)]
                sel[b, h, :m] = r.permutation(max(first, m))[:m]
                most = k_max if k_h is None else k_h[h]
                listed[b][h] = sel[b, h, :min(m, most)].tolist() + listed[b][h]
        sel = torch.from_numpy(sel).to(DEV)
    out = torch.full((B, n_q, H, d), 3.0, dtype=dt, device=DEV)
    lse = torch.full((B, H, n_q), 5.0, device=DEV)
    c.attend(q, n, first_page=first, sel=sel, k_h=k_h, kv_len=None if kv_len is None else i32(kv_len),
             q_len=None if q_len is None else i32(q_len), causal=causal, out=out, lse=lse)
    ql = [n_q] * B if q_len is None else q_len
    ol = [(first + n) * P_ if causal and kv_len is None else x for x in lens]
    k, v = O.dequantise(arrays(c))
    check(q, out, lse, k, v, pt, listed, ol, ql, causal, scale or d ** -0.5)
    return c, q, out, lse


def check(q, out, lse, k, v, pt, listed, kv_len, q_len, causal, scale):
    d = q.shape[-1]
    o, l, va, S, vm = O.attend(host(q), k, v, pt, listed, kv_len, q_len, causal, scale)
    got, gl = host(out), host(lse)
    n = max(len(x) for y in listed for x in y) * k.shape[2]
    wt = (2 * (d + 8) * 2.0 ** -24 * S + 2.0 ** -20).transpose(0, 2, 1)[..., None]
    bf = 2.0 ** -8 if out.dtype == torch.bfloat16 else 0.0
    tol = (2 * wt + n * 2.0 ** -24 + bf) * va + (bf + 2.0 ** -23) * np.abs(o)
    tol = tol + n * 2.0 ** -126 * vm.transpose(0, 2, 1)[..., None]
    row = ~np.isnan(o)
    err = np.abs(got - o)
    if row.any():
        print(f"  worst error over its bound: {np.max(err[row] / np.maximum(tol[row], 1e-30)):.3f}", flush=True)
    assert (err[row] <= tol[row]).all()
    assert (got[~row] == 3.0).all()  # rows past q_len stay
    seen = np.isfinite(l)
    ltol = 2 * (d + 8) * 2.0 ** -24 * S[seen] + 2.0 ** -20 + n * 2.0 ** -24 + 2.0 ** -23 * np.abs(l[seen])
    assert (np.abs(gl[seen] - l[seen]) <= ltol).all()
    assert np.isneginf(gl[np.isneginf(l)]).all()
    assert (gl[np.isnan(l)] == 5.0).all()


BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P_,pages", [(8, 20), (16, 9), (24, 5), (32, 3), (40, 4), (56, 3), (64, 3), (72, 3), (120, 2),
                                      (200, 2), (256, 1), (392, 1)])
def test_page_sizes(P_, pages, d, dt):
    print(P_, pages, d, dt, flush=True)
    cap = P_ * pages
    run_case(P_ + d, 3, 4, 2, d, P_, 1, dt, pages, kv_len=[cap, 1, cap - 5])


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("H,kv,n_q", [(1, 1, 1), (12, 12, 1), (16, 1, 1), (8, 4, 7), (24, 2, 2), (40, 1, 1), (64, 1, 1),
                                      (6, 3, 33), (4, 4, 65), (2, 1, 130), (3, 3, 300)])
def test_heads_and_query_counts(H, kv, n_q, dt):
    print(H, kv, n_q, dt, flush=True)
    run_case(H * 7 + n_q, 2, H, kv, 128, 104, n_q, dt, 3, kv_len=[312, 290])
    run_case(H * 7 + n_q, 2, H, kv, 64, 48, n_q, dt, 8, kv_len=[max(384, n_q), max(n_q, 200)], causal=True)


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("P_", [16, 40, 64, 136])
def test_causal_ragged(P_, dt):
    """Lengths from none to all, sequences with more queries than tokens (the first see
    nothing), no queries, one."""
    pages = -(-400 // P_)
    print(P_, dt, flush=True)
    run_case(P_, 6, 4, 2, 64, P_, 90, dt, pages, kv_len=[400, 90, 60, 0, 1, 333], q_len=[90, 90, 90, 5, 1, 0], causal=True)
    run_case(P_ + 1, 2, 4, 2, 64, P_, 21, dt, pages, causal=True)
    run_case(P_ + 2, 3, 3, 3, 128, P_, 4, dt, pages, kv_len=[0, 399, 64], q_len=[4, 0, 2])


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("P_", [8, 40, 72, 256])
def test_selected_pages(P_, dt):
    """Selected pages before the run of pages: budgets per head, short rows, none, a length
    that ends inside them."""
    print(P_, dt, flush=True)
    run_case(P_, 2, 4, 2, 64, P_, 50, dt, 9, first=6, k_max=4, k_h=[4, 2])
    run_case(P_ + 1, 2, 4, 4, 128, P_, 3, dt, 9, first=7, k_max=5, sel_valid=[0, 3, 5])
    run_case(P_ + 2, 1, 2, 1, 64, P_, 1, dt, 9, first=8, n=0, k_max=3)
    run_case(P_ + 3, 2, 2, 2, 64, P_, 20, dt, 9, first=6, k_max=6, kv_len=[3 * P_ + 5, 8 * P_ + 1], q_len=[20, 11], causal=True)
    run_case(P_ + 4, 1, 2, 2, 64, P_, 5, dt, 9, first=9, n=0, k_max=2, sel_valid=[0, 2])


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
def test_long_splits_and_large_scores(dt):
    """Many pieces, and scores far apart (the running maximum moves often)."""
    run_case(1, 1, 2, 1, 128, 1560, 1, dt, 6, kv_len=[9000])
    run_case(2, 2, 2, 2, 64, 256, 40, dt, 8, spread=1.5)
    run_case(3, 1, 4, 1, 64, 64, 3, dt, 40, kv_len=[2500], scale=1.5)


@pytest.mark.parametrize("n_q", [1, 100])
def test_same_call_gives_the_same_bits(n_q):
    c, q, out, lse = run_case(7, 2, 4, 2, 128, 200, n_q, BF, 12, kv_len=[2400, 1777])
    for _ in range(3):
        o2, l2 = torch.full_like(out, 3.0), torch.full_like(lse, 5.0)
        c.attend(q, 12, kv_len=i32([2400, 1777]), out=o2, lse=l2)
        assert torch.equal(out, o2) and torch.equal(lse, l2)


@pytest.mark.parametrize("n_q", [1, 100])
def test_captured_call_follows_lengths_and_two_graphs_share_nothing(n_q):
    B, H, kv, d, P_, pages = 2, 4, 2, 64, 72, 30
    c, _, _, _ = run_case(8, B, H, kv, d, P_, n_q, BF, pages)
    g = torch.Generator().manual_seed(2)
    qs = [torch.randn((B, n_q, H, d), generator=g).bfloat16().to(DEV) for _ in range(2)]
    lens, qlen = i32([2000, 2100]), i32([n_q, n_q])
    outs = [torch.zeros_like(qs[0]) for _ in range(2)]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for q, o, graph in zip(qs, outs, graphs):
        with torch.cuda.graph(graph):
            c.attend(q, pages, kv_len=lens, q_len=qlen, causal=True, out=o)
    for step in ([1500, 130], [2160, n_q], [n_q, 700]):
        lens.copy_(torch.tensor(step))
        graphs[0].replay()
        graphs[1].replay()
        want = [c.attend(q, pages, kv_len=lens, q_len=qlen, causal=True) for q in qs]
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)


def test_two_streams_at_once():
    B, H, kv, d, P_, pages = 1, 8, 2, 128, 128, 20
    c, q, _, _ = run_case(9, B, H, kv, d, P_, 1, BF, pages)
    q2 = (q * 0.5).contiguous()
    want = c.attend(q, pages), c.attend(q2, pages)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(q) for _ in range(5)] for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(5):
        for s, x, o in zip(streams, (q, q2), outs):
            c.attend(x, pages, out=o[i], stream=s)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        for x in o:
            assert torch.equal(x, w)


def test_check_mode_reports_bad_pages(monkeypatch):
    monkeypatch.setenv("HSA_CHECK", "1")
    c, q, _, _ = run_case(10, 1, 2, 2, 64, 64, 1, BF, 4)
    c.page_table[0, 3] = -1
    c.attend(q, 4, kv_len=i32([192]))           # the bad page holds no token yet
    with pytest.raises(P.HsaError):
        c.attend(q, 4, kv_len=i32([193]))
    k, v = source(1, 1, 3, 2, 64, BF, False)
    c.write(k, v, i32([180]))
    for first in (190, 191, 250, -1, 255):
        with pytest.raises(P.HsaError):
            c.write(k, v, i32([first]))


# ---------------------------------------------------------------- together
def test_decoding_step_by_step():
    """A prompt, then tokens one at a time: rotate, append, attend, each step against the
    oracle on the cache as it stands."""
    B, H, kv, d, P_, pages, n = 2, 4, 2, 64, 40, 4, 70
    rope = P.rope(64, scaling="linear", factor=2.0)
    c, pt = cache(21, B, H, d, P_, BF, pages, rope=rope, kv=kv)
    lens = [n, 41]
    for step in range(25):
        m = n if step == 0 else 1
        g = torch.Generator().manual_seed(step)
        q = torch.randn((B, m, H, d), generator=g).bfloat16().to(DEV)
        k, v = source(50 + step, B, m, kv, d, BF, True)
        count = lens if step == 0 else [1, 1]
        first = [0, 0] if step == 0 else lens
        c.write(k, v, i32(first), count=i32(count))
        qr = c.rotate(q, first=i32(first))
        lens = [f + x for f, x in zip(first, count)]
        out, lse = torch.full_like(q, 3.0), torch.full((B, H, m), 5.0, device=DEV)
        c.attend(qr, pages, kv_len=i32(lens), q_len=i32(count), causal=True, out=out, lse=lse)
        kd, vd = O.dequantise(arrays(c))
        check(qr, out, lse, kd, vd, pt, [[list(range(pages))] * kv] * B, lens, count, True, d ** -0.5)
        # the rotated keys in the cache stand for the rotated inputs: e4m3's half step, 2^-4
        # of the largest of a block at most
        b = 0
        turned = O.rope(host(k), O.places(first, m), 64, scaling="linear", factor=2.0)[b, :count[b]]
        held = np.stack([kd[pt[b, t // P_], :, t % P_] for t in range(first[b], lens[b])])
        assert (np.abs(held - turned) <= 2.0 ** -4 * np.abs(turned) + 2.0 ** -9 * np.abs(kd[pt[b]][np.isfinite(kd[pt[b]])]).max() / 256).all()


def test_streamed_chunk_over_selected_8bit_history():
    """A video layer's chunk: rotated keys appended to a small pool of the chunk's pages and
    folded into the page index, history in 8 bits, pages selected by the index, attention over the selected
    and the chunk's own pages."""
    B, H, d, P_, cand, cur, n = 1, 4, 64, 120, 6, 2, 240
    total = cand + cur
    rope = P.rope(64, layout="interleaved", axis_dims=[24, 20, 20])
    c, pt = cache(31, B, H, d, P_, BF, total, rope=rope)
    pool = P.HsaLayer(B, H, d, P_, BF, DEV, num_slots=cur, max_pages=total)
    for chunk in range(total // cur):
        t = torch.arange(n, dtype=torch.int32)
        pos = torch.stack([chunk * cur + t // P_, t % P_ // 12, t % 12], -1)[None].contiguous().to(DEV)
        first = i32([chunk * n])
        k, v = source(60 + chunk, B, n, H, d, BF, True)
        pool.page_table[0, chunk * cur:(chunk + 1) * cur] = torch.arange(cur, dtype=torch.int32, device=DEV)
        pool.write_tokens(k, v, first, rope=rope, pos=pos)
        pool.fold(chunk * cur, cur)
        c.write(k, v, first, pos=pos)
    q, _ = source(70, B, n, H, d, BF, True)
    q = c.rotate(q, pos=pos)
    k_h, k_max = [3, 1, 2, 3], 3
    sel = torch.empty((B, H, k_max), dtype=torch.int32, device=DEV)
    P.hsa_page_select(pool.cfg, q, n, pool.page_kmean, total, cand, k_h, k_max, sel)
    out, lse = torch.full_like(q, 3.0), torch.full((B, H, n), 5.0, device=DEV)
    c.attend(q, cur, first_page=cand, sel=sel, k_h=k_h, out=out, lse=lse)
    kd, vd = O.dequantise(arrays(c))
    rows = sel.cpu().numpy()
    listed = [[[p for p in rows[0, h] if p >= 0] + [cand, cand + 1] for h in range(H)]]
    assert [len(x) for x in listed[0]] == [k + cur for k in k_h]
    check(q, out, lse, kd, vd, pt, listed, [total * P_], [n], False, d ** -0.5)
