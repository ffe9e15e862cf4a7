"""Trees of drafted tokens: their ancestor bits (whole numbers) and their attention over the pool and
the 8-bit cache, against the oracle.

Bound of an output: as for the attention over the 8-bit cache (test_gpu_cache8.py). The weights and the
output of a bf16 call are rounded to bf16 once each, 2^-8 (mean |v| + |o|); a score, a sum of d exact products (or,
fp32 over the pool, of products rounded by 2^-24), is off by (d + 4) 2^-24 of sum |q k|, and a weight by
less than w = 2 (d + 8) 2^-24 S + 2^-20 with S the largest scaled sum |q k| of the row; the sum of n
weighted values by n 2^-24 mean |v|, and n 2^-126 max |v| for weights without a normal number.
"""
import numpy as np
import pytest
import torch

import paper_2609_34606_amd as P
from oracle import hsa_cache8_oracle as C8
from oracle import hsa_tree_oracle as O
from test_gpu_tokens import arrays, cache, host, i32, source, table

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def words(bits):
    return torch.from_numpy(O.pack(bits).view(np.int32)).to(DEV)


def a_tree(r, B, n, back=6):
    return np.array([[max(-1, i - 1 - int(r.integers(0, back))) for i in range(n)] for _ in range(B)])


# ---------------------------------------------------------------- ancestors
@pytest.mark.parametrize("shape", ["chain", "star", "roots", "drawn", "wild"])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 64, 65, 200, 256])
def test_ancestor_bits(n, shape):
    print(n, shape, flush=True)
    r = np.random.default_rng(n)
    B = 4
    i = np.arange(n)
    parent = {"chain": np.tile(i - 1, (B, 1)), "star": np.tile(np.where(i > 0, 0, -1), (B, 1)),
              "roots": np.full((B, n), -1), "drawn": a_tree(r, B, n),
              "wild": r.integers(-2 ** 31, 2 ** 31, (B, n))}[shape]
    if shape == "wild":  # parents at and behind the node, and beyond any: roots
        parent[:, ::3] = i[::3] + r.integers(0, 3, (B, len(i[::3])))
    count, first = [n, max(0, n - 3), 0, 1], [0, 7, 100, 187199]
    mask = torch.full((B, n, -(-n // 32)), 77, dtype=torch.int32, device=DEV)
    pos = torch.full((B, n), -5, dtype=torch.int32, device=DEV)
    cfg = P.config(B, 1, 64, 8, BF)
    P.hsa_tree_mask(cfg, i32(parent.tolist()), n, mask, pos=pos, count=i32(count), first=i32(first))
    bits, at = O.tree_mask(parent, count, first)
    row = np.arange(n) < np.array(count)[:, None]
    want = np.where(row[..., None], O.pack(bits).view(np.int32), 77)
    assert np.array_equal(mask.cpu().numpy(), want)
    assert np.array_equal(pos.cpu().numpy(), np.where(row, at, -5))
    P.hsa_tree_mask(cfg, i32(parent.tolist()), n, mask)  # neither counts nor positions
    assert np.array_equal(mask.cpu().numpy(), O.pack(O.tree_mask(parent, [n] * B, [0] * B)[0]).view(np.int32))


# ---------------------------------------------------------------- attention
def make(kind, seed, B, H, kv, d, P_, dt, pages, lens, spread):
    """A pool or cache filled up to each length (garbage, NaN among it, elsewhere): (its object, page
    table, keys and values [slots, kv, P, d])."""
    cap = pages * P_
    ks, vs = source(seed, B, cap, kv, d, torch.float32, False, spread)
    if kind == "codes":
        c, pt = cache(seed, B, H, d, P_, dt, pages, kv=kv)
        w = P.HsaCache8(B, H, d, P_, torch.float32, DEV, kv_heads=kv, k=c.k, v=c.v, k_exp=c.k_exp, v_exp=c.v_exp,
                        page_table=c.page_table)
        w.write(ks, vs, count=i32(lens))
        return (c, pt) + C8.dequantise(arrays(c))
    pt, slots = table(seed, B, pages)
    c = P.HsaLayer(B, kv, d, P_, dt, DEV, num_slots=slots, max_pages=pages)
    c.page_table.copy_(torch.from_numpy(pt))
    for t in (c.k_pool, c.v_pool):
        t.fill_(float("nan"))
        t[::2] = float("inf")
    c.write_tokens(ks.to(dt), vs.to(dt), count=i32(lens))
    return c, pt, host(c.k_pool), host(c.v_pool).transpose(0, 1, 3, 2)


def run_case(kind, seed, B, H, kv, d, P_, n_q, dt, pages, first=0, n=None, k_h=None, k_max=0, kv_len=None,
             q_len=None, mask="tree", spread=0.3, scale=0.0, sel_valid=None, change=None, many=False):
    n = pages - first if n is None else n
    r = np.random.default_rng(seed)
    lens = [pages * P_] * B if kv_len is None else kv_len
    c, pt, k, v = make(kind, seed, B, H, kv, d, P_, dt, pages, lens, spread)
    if change:
        change(c, pt)
        if kind == "codes":
            k, v = C8.dequantise(arrays(c))
        else:
            k, v = host(c.k_pool), host(c.v_pool).transpose(0, 1, 3, 2)
    c.cfg.sm_scale = scale
    ql = [n_q] * B if q_len is None else q_len
    bits = None
    if mask == "tree":
        bits = O.tree_mask(a_tree(r, B, n_q), [n_q] * B, [0] * B)[0]
    elif mask == "any":  # bits of no tree, rows without any among them, and set past the nodes
        bits = r.random((B, n_q, n_q)) < 0.4
        bits[:, ::3] = False
    q = torch.randn((B, n_q, H, d), generator=torch.Generator().manual_seed(seed + 1)).to(dt).to(DEV)
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
    c.attend_tree(q, n, mask=None if bits is None else words(bits), first_page=first, sel=sel, k_h=k_h,
                  kv_len=None if kv_len is None else i32(kv_len), q_len=None if q_len is None else i32(q_len),
                  out=out, lse=lse)
    ol = [(first + n) * P_ if kv_len is None else x for x in lens]
    check(q, out, lse, k, v, pt, listed, ol, ql, bits, scale or d ** -0.5, many)
    return c, q, out, lse


def check(q, out, lse, k, v, pt, listed, kv_len, q_len, bits, scale, many=False):
    d = q.shape[-1]
    attend = (lambda *a: O.attend_many(*a, device=DEV)) if many else O.attend
    o, l, va, S, vm = attend(host(q), k, v, pt, listed, kv_len, q_len, bits, scale)
    got, gl = host(out), host(lse)
    past = np.isnan(va) & np.isnan(o) & (np.arange(o.shape[1])[None, :] >= np.array(q_len)[:, None])[..., None, None]
    assert (got[past] == 3.0).all()  # rows past q_len stay
    n = max(len(x) for y in listed for x in y) * k.shape[2]
    wt = (2 * (d + 8) * 2.0 ** -24 * S + 2.0 ** -20).transpose(0, 2, 1)[..., None]
    bf = 2.0 ** -8 if out.dtype == BF else 0.0
    with np.errstate(invalid="ignore"):
        tol = (2 * wt + n * 2.0 ** -24 + bf) * va + (bf + 2.0 ** -23) * np.abs(o)
        tol = tol + n * 2.0 ** -126 * vm.transpose(0, 2, 1)[..., None]
        fine, err = np.isfinite(o), np.abs(got - o)
    row = ~past
    assert np.array_equal(np.isfinite(got)[row], fine[row])
    use = row & fine
    if use.any():
        print(f"  worst error over its bound: {np.max(err[use] / np.maximum(tol[use], 1e-30)):.3f}", flush=True)
    assert (err[use] <= tol[use]).all()
    inf = row & np.isinf(o)
    assert np.array_equal(got[inf], o[inf]) and np.isnan(got[row & np.isnan(o)]).all()
    seen = np.isfinite(l)
    ltol = 2 * (d + 8) * 2.0 ** -24 * S[seen] + 2.0 ** -20 + n * 2.0 ** -24 + 2.0 ** -23 * np.abs(l[seen])
    assert (np.abs(gl[seen] - l[seen]) <= ltol).all()
    assert np.isneginf(gl[np.isneginf(l)]).all()
    for b, x in enumerate(q_len):
        assert (gl[b, :, x:] == 5.0).all()


KINDS = [("pool", BF), ("pool", F32), ("codes", BF), ("codes", F32)]
kinds = pytest.mark.parametrize("kind,dt", KINDS, ids=["pool-bf16", "pool-f32", "codes-bf16", "codes-f32"])


@kinds
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P_,pages", [(8, 20), (16, 9), (24, 5), (40, 4), (56, 3), (64, 3), (72, 3), (200, 2), (256, 1),
                                      (392, 1)])
def test_page_sizes(P_, pages, d, kind, dt):
    print(P_, pages, d, kind, dt, flush=True)
    cap = P_ * pages
    run_case(kind, P_ + d, 3, 4, 2, d, P_, 11, dt, pages, kv_len=[cap, 11, cap - 5])


@kinds
@pytest.mark.parametrize("H,kv,n_q", [(1, 1, 1), (12, 12, 1), (16, 1, 1), (8, 4, 7), (24, 2, 2), (64, 1, 1), (6, 3, 33),
                                      (4, 4, 65), (2, 1, 130), (3, 3, 256)])
def test_heads_and_node_counts(H, kv, n_q, kind, dt):
    print(H, kv, n_q, kind, dt, flush=True)
    run_case(kind, H * 7 + n_q, 2, H, kv, 128, 104, n_q, dt, 3, kv_len=[312, 290])
    run_case(kind, H * 7 + n_q, 2, H, kv, 64, 48, n_q, dt, 8, kv_len=[max(384, n_q), max(n_q, 200)], mask=None)


@kinds
@pytest.mark.parametrize("mask", ["tree", "any", None])
@pytest.mark.parametrize("P_", [16, 40, 64, 136])
def test_ragged(P_, mask, kind, dt):
    """Sequences that are nothing but their tree, trees longer than the sequence (nodes before the first
    token are no tokens), no nodes, one."""
    pages = -(-400 // P_)
    print(P_, mask, kind, dt, flush=True)
    run_case(kind, P_, 6, 4, 2, 64, P_, 90, dt, pages, kv_len=[400, 90, 60, 0, 1, 333], q_len=[90, 90, 90, 5, 1, 0], mask=mask)
    run_case(kind, P_ + 1, 2, 4, 2, 64, P_, 21, dt, pages, mask=mask)
    run_case(kind, P_ + 2, 3, 3, 3, 128, P_, 4, dt, pages, kv_len=[0, 399, 64], q_len=[4, 0, 2], mask=mask)


@kinds
@pytest.mark.parametrize("P_", [8, 40, 72, 256])
def test_selected_pages(P_, kind, dt):
    """Selected pages before the run of pages: budgets per head, short rows, none; a run that leaves out a part of the
    tree, nodes in selected pages."""
    print(P_, kind, dt, flush=True)
    run_case(kind, P_, 2, 4, 2, 64, P_, 50, dt, 9, first=6, k_max=4, k_h=[4, 2])
    run_case(kind, P_ + 1, 2, 4, 4, 128, P_, 3, dt, 9, first=7, k_max=5, sel_valid=[0, 3, 5])
    run_case(kind, P_ + 2, 1, 2, 1, 64, P_, 1, dt, 9, first=8, n=0, k_max=3, kv_len=[9 * P_])
    run_case(kind, P_ + 3, 2, 2, 2, 64, P_, 20, dt, 9, first=6, k_max=6, kv_len=[3 * P_ + 5, 8 * P_ + 1], q_len=[20, 11])
    run_case(kind, P_ + 4, 1, 2, 2, 64, P_, 5, dt, 9, first=9, n=0, k_max=2, sel_valid=[0, 2], kv_len=[2 * P_])


@kinds
@pytest.mark.parametrize("H,kv,n_q,d", [(4, 1, 1, 128), (8, 1, 4, 128), (8, 1, 8, 64), (12, 1, 3, 64), (2, 1, 40, 128)])
@pytest.mark.parametrize("P_", [8, 16, 64, 200, 1560])
def test_long_lists_in_pieces(P_, H, kv, n_q, d, kind, dt):
    """Lists long enough to be cut; a sequence that ends in the first piece, and one in the last."""
    pages = -(-6000 // P_)
    cap = pages * P_
    print(P_, H, n_q, d, kind, dt, flush=True)
    run_case(kind, P_ + n_q, 2, H, kv, d, P_, n_q, dt, pages, kv_len=[cap - 1, 50])
    run_case(kind, P_ + n_q, 1, H, kv, d, P_, n_q, dt, pages)


@kinds
def test_large_scores(kind, dt):
    """Scores far apart: the running maximum moves often."""
    run_case(kind, 2, 2, 2, 2, 64, 256, 40, dt, 8, spread=1.5)
    run_case(kind, 3, 1, 4, 1, 64, 64, 3, dt, 40, kv_len=[2500], scale=1.5)


@kinds
@pytest.mark.parametrize("d", [64, 128])
def test_what_a_node_does_not_see_does_not_reach_it(d, kind, dt):
    """NaN and infinities among the nodes' keys and values: only the nodes that see them have them."""
    nan, inf = float("nan"), float("inf")

    def change(c, pt):
        # tokens of entry 0, whose base is 100 (pages of 40): nodes 3, 7, 20
        for t, key, value in ((103, nan, 1.0), (107, 1.0, nan), (120, 1.0, inf)):
            s, o = int(pt[0, t // 40]), t % 40
            if kind == "codes":
                c.k[s, :, o] = 0x7f if key != key else 0x30
                c.v[s, :, :, o] = 0x7f if value != 1.0 else 0x30
            else:
                c.k_pool[s, :, o] = key
                c.v_pool[s, :, :, o] = value
    for n_q, H, kv in ((30, 2, 2), (30, 4, 1), (30, 2, 1)):
        _, _, out, _ = run_case(kind, n_q + H, 2, H, kv, d, 40, n_q, dt, 6, kv_len=[130, 225], q_len=[30, 25], change=change)
        fine = torch.isfinite(out[0]).all(-1).all(-1)
        assert fine.any() and not fine.all() and torch.isfinite(out[1, :25]).all()


# rows of a key head 16, 30, 64, 100 and 250: every kernel of calls that are not little work
MUCH = pytest.mark.parametrize("B,H,kv,n_q", [(33, 16, 8, 8), (18, 16, 8, 15), (9, 16, 8, 32), (20, 32, 16, 50), (10, 32, 16, 125)])


@kinds
@MUCH
@pytest.mark.parametrize("d", [64, 128])
def test_much_work(B, H, kv, n_q, d, kind, dt):
    """Ragged batches of many rows over pages of several sizes, selected pages, masks of any bits, rows
    that see nothing."""
    print(B, H, kv, n_q, d, kind, dt, flush=True)
    r = np.random.default_rng(n_q)
    for P_, mask in ((64, "tree"), (40, "any"), (136, None)):
        pages = -(-1152 // P_)
        kv_len = [1152, n_q, n_q + 1, 0] + r.integers(n_q, 1153, B - 4).tolist()
        q_len = [n_q, n_q, n_q, 0] + r.integers(0, n_q + 1, B - 4).tolist()
        run_case(kind, P_ + n_q, B, H, kv, d, P_, n_q, dt, pages, kv_len=kv_len, q_len=q_len, mask=mask, many=True)
    kv_len[1:3] = [1100, n_q - 1]
    run_case(kind, n_q, B, H, kv, d, 72, n_q, dt, 16, first=10, k_max=9, k_h=[9 - h % 9 for h in range(kv)], kv_len=kv_len, q_len=q_len, many=True)
    run_case(kind, n_q, B, H, kv, d, 8, n_q, dt, 144, mask="any", many=True)


@kinds
@pytest.mark.parametrize("B,H,kv,n_q", [(8, 16, 8, 8), (8, 16, 4, 8), (8, 16, 8, 32), (4, 8, 4, 125)])
@pytest.mark.parametrize("d", [64, 128])
def test_much_work_in_pieces(B, H, kv, n_q, d, kind, dt):
    """Long lists of many rows; captured calls follow lengths and masks."""
    print(B, H, kv, n_q, d, kind, dt, flush=True)
    P_, pages = 200, 42
    kv_len = [8301, n_q, 5000, 8400, 0, 1, 6000, 7777][:B]
    q_len = [n_q, n_q, n_q - 1, n_q, 0, 1, 3, n_q][:B]
    c, q, out, lse = run_case(kind, n_q, B, H, kv, d, P_, n_q, dt, pages, kv_len=kv_len, q_len=q_len, many=True)
    run_case(kind, n_q, B, H, kv, d, P_, n_q, dt, pages, mask="any", many=True)
    lens, nodes, words_ = i32(kv_len), i32(q_len), -(-n_q // 32)
    mask = torch.zeros((B, n_q, words_), dtype=torch.int32, device=DEV)
    got = torch.empty_like(out)
    call = lambda to: c.attend_tree(q, pages, mask=mask, kv_len=lens, q_len=nodes, out=to)
    call(got)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(got)
    r = np.random.default_rng(0)
    for i in range(3):
        lens.copy_(i32(r.permutation(kv_len).tolist()))
        nodes.copy_(i32(r.permutation(q_len).tolist()))
        mask.copy_(words(r.random((B, n_q, n_q)) < 0.5))
        out.fill_(2.0)
        got.fill_(2.0)
        call(out)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(bits_of(got), bits_of(out))


@kinds
@MUCH
@pytest.mark.parametrize("d", [64, 128])
def test_much_work_and_what_a_node_does_not_see(B, H, kv, n_q, d, kind, dt):
    """NaN and infinities among the nodes, as above, of every kernel of larger calls."""
    nan, inf = float("nan"), float("inf")
    print(B, H, kv, n_q, d, kind, dt, flush=True)

    def change(c, pt):
        for t, key, value in ((603, nan, 1.0), (605, 1.0, nan), (606, 1.0, inf)):  # nodes 3, 5, 6
            s, o = int(pt[1, t // 40]), t % 40
            if kind == "codes":
                c.k[s, :, o] = 0x7f if key != key else 0x30
                c.v[s, :, :, o] = 0x7f if value != 1.0 else 0x30
            else:
                c.k_pool[s, :, o] = key
                c.v_pool[s, :, :, o] = value
    kv_len = [1160 - b for b in range(B)]
    kv_len[1] = 600 + n_q
    _, _, out, _ = run_case(kind, n_q, B, H, kv, d, 40, n_q, dt, 29, kv_len=kv_len, change=change, many=True)
    fine = torch.isfinite(out[1]).all(-1).all(-1)
    assert fine.any() and not fine.all() and torch.isfinite(out[0]).all() and torch.isfinite(out[2:]).all()


def bits_of(t):
    return t.view(torch.int16 if t.dtype == BF else torch.int32)


@kinds
def test_same_bits_captured_and_shared_workspace(kind, dt):
    """The same call gives the same bits; captured calls follow lengths, masks and tables, and two graphs
    may share a workspace."""
    B, H, kv, d, P_, n_q, pages = 2, 4, 2, 64, 64, 20, 60
    c, q, out, lse = run_case(kind, 5, B, H, kv, d, P_, n_q, dt, pages, kv_len=[3840, 3000])
    r = np.random.default_rng(0)
    size = P.hsa_tree_attn_workspace_size if kind == "pool" else P.hsa_cache8_tree_attn_workspace_size
    cfg = P.config(B, H, d, P_, dt)
    nbytes = size(cfg, n_q, kv, 0, pages)
    assert nbytes > 0
    ws = torch.full((nbytes,), 255, dtype=torch.uint8, device=DEV)
    kv_len, q_len = i32([3840, 3000]), i32([20, 20])
    mask = torch.zeros((B, n_q, 1), dtype=torch.int32, device=DEV)
    outs = [torch.zeros_like(out) for _ in range(2)]

    def call(i):
        if kind == "pool":
            P.hsa_tree_attn(cfg, q, n_q, c.pool, kv, None, 0, None, 0, pages, outs[i], mask=mask, kv_len=kv_len, q_len=q_len, ws=ws)
        else:
            P.hsa_cache8_tree_attn(cfg, q, n_q, c.pool, None, 0, None, 0, pages, outs[i], mask=mask, kv_len=kv_len, q_len=q_len, ws=ws)
    call(0)
    call(1)
    assert torch.equal(outs[0], outs[1])
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g):
            call(i)
    for lens, nodes in (([3840, 3000], [20, 20]), ([17, 3839], [17, 3]), ([0, 1], [0, 1]), ([3840, 64], [1, 20])):
        kv_len.copy_(i32(lens))
        q_len.copy_(i32(nodes))
        mask.copy_(words(O.tree_mask(a_tree(r, B, n_q), [n_q] * B, [0] * B)[0]))
        outs[0].fill_(3.0)
        call(0)
        want = outs[0].clone()
        for i, g in enumerate(graphs):
            outs[i].fill_(3.0)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(bits_of(outs[i]), bits_of(want))  # (memory past the second entry's tokens: NaN)


def test_a_chain_is_the_causal_call():
    """Without a mask the nodes are a causal run: what hsa_cache8_attn computes, within both bounds."""
    B, H, kv, d, P_, n_q, pages = 2, 8, 2, 128, 72, 33, 9
    c, q, out, _ = run_case("codes", 8, B, H, kv, d, P_, n_q, BF, pages, kv_len=[648, 500], mask=None)
    want = c.attend(q, pages, kv_len=i32([648, 500]), causal=True)
    assert (out.float() - want.float()).abs().max() <= 2.0 ** -6
    i = np.arange(n_q)
    chain = words(np.broadcast_to(i[None, :] <= i[:, None], (B, n_q, n_q)).copy())
    assert torch.equal(c.attend_tree(q, pages, mask=chain, kv_len=i32([648, 500])), out)


def test_side_stream_takes_its_own_memory():
    c, q, out, _ = run_case("pool", 9, 1, 8, 8, 128, 128, 3, BF, 60, kv_len=[7600])
    want = c.attend_tree(q, 60, kv_len=i32([7600]))
    s = torch.cuda.Stream()
    n = i32([7600])
    torch.cuda.synchronize()
    outs = []
    for _ in range(10):
        outs += [c.attend_tree(q, 60, kv_len=n), c.attend_tree(q, 60, kv_len=n, stream=s)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("kind,dt", [("pool", BF), ("codes", BF), ("pool", F32)])
def test_offsets_past_32_bits(kind, dt):
    """Pages at the end of a cache of more than 2^32 elements and in a small one: the same bits."""
    H, d, P_, n_q = 8, 128, 1560, 9
    n, got = 2 * P_ - 92, []
    slots = 2800 if dt == BF else 2700
    for num, at in ((slots, [slots - 1, slots - 30]), (2, [1, 0])):
        c = P.HsaCache8(1, H, d, P_, dt, DEV, num_slots=num, max_pages=2) if kind == "codes" else \
            P.HsaLayer(1, H, d, P_, dt, DEV, num_slots=num, max_pages=2)
        c.page_table.copy_(torch.tensor([at]))
        k, v = source(4, 1, n, H, d, dt, True)
        (c.write if kind == "codes" else c.write_tokens)(k, v)
        index, moves = i32([[0, 3, 5]]), i32([[at[0], at[1], 8]])
        q = source(6, 1, n_q, H, d, dt, False)[0]
        outs = [c.attend_tree(q, 2, kv_len=i32([n]))]
        c.keep_tokens(i32([n - 9]), index)
        outs.append(c.attend_tree(q, 2, kv_len=i32([n - 6]), q_len=i32([n_q])))
        c.copy_pages(moves)
        outs.append(c.attend_tree(q, 2, kv_len=i32([n - 6])))
        got.append([t.clone() for t in outs])
        del c, k, v, outs
        torch.cuda.empty_cache()
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert not torch.equal(got[0][0], got[0][1]) and not torch.equal(got[0][1], got[0][2])
