"""Drafting with a tree, used together: beams share a prompt's pages, each step drafts a tree of tokens,
attends, keeps an accepted path and goes on. The cache then holds what a program without drafts would have
written, and a last token attends to the same."""
import numpy as np
import pytest
import torch

import paper_2609_34606_amd as P
from oracle import hsa_cache8_oracle as C8
from oracle import hsa_tree_oracle as O
from test_gpu_tokens import arrays, host, i32
from test_gpu_tree import check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


@pytest.mark.parametrize("kind", ["pool", "codes"])
def test_drafted_steps(kind):
    B, H, kv, d, P_, pages, slots, n = 3, 4, 2, 64, 40, 8, 40, 12
    r = np.random.default_rng(7)
    rope = P.rope(d)
    s = P.HsaSlots(B, P_, DEV, num_slots=slots, max_pages=pages)
    if kind == "codes":
        c = P.HsaCache8(B, H, d, P_, BF, DEV, kv_heads=kv, num_slots=slots, page_table=s.page_table, rope=rope)
        write = lambda k, v, first, pos, count: c.write(k, v, first, count=count, pos=pos)
    else:
        c = P.HsaLayer(B, kv, d, P_, BF, DEV, num_slots=slots, page_table=s.page_table)
        write = lambda k, v, first, pos, count: c.write_tokens(k, v, first, count=count, rope=rope, pos=pos)
    kvs = lambda n: [torch.randn((B, n, kv, d), device=DEV).to(BF) for _ in range(2)]
    # a prompt in row 0, shared by the others; each goes on alone
    start = 51
    k0, v0 = kvs(start)
    s.take(None, i32([start, 0, 0]))
    write(k0, v0, i32([0] * B), None, i32([start, 0, 0]))
    s.fork(i32([0] * B))
    kept = [[(0, k0, v0, i) for i in range(start)] for _ in range(B)]  # (row, keys, values, index) of each token
    length = np.full(B, start)
    all_k, all_v = [k0], [v0]
    for step in range(5):
        nodes = r.integers(1, n + 1, B)
        first, end = i32(length.tolist()), i32((length + nodes).tolist())
        c.copy_pages(s.take(first, end))
        assert int(s.missing) == 0
        parent = np.array([[i - 1 - r.integers(0, min(i, 3) + 1) for i in range(n)] for _ in range(B)])
        mask = torch.zeros((B, n, 1), dtype=torch.int32, device=DEV)
        pos = torch.zeros((B, n), dtype=torch.int32, device=DEV)
        P.hsa_tree_mask(s.cfg, i32(parent.tolist()), n, mask, pos=pos, count=i32(nodes.tolist()), first=first)
        k, v = kvs(n)
        all_k.append(k)
        all_v.append(v)
        write(k, v, first, pos, i32(nodes.tolist()))
        q = torch.randn((B, n, H, d), device=DEV).to(BF)
        out = torch.full_like(q, 3.0)
        c.attend_tree(q, pages, mask=mask, kv_len=end, q_len=i32(nodes.tolist()), out=out)
        assert torch.isfinite(out).all()
        # the path to some node is accepted
        bits, _ = O.tree_mask(parent, nodes, [0] * B)
        paths = [np.flatnonzero(bits[b, r.integers(0, nodes[b])]) for b in range(B)]
        index = np.zeros((B, n), int)
        for b, p in enumerate(paths):
            index[b, :len(p)] = p
            kept[b] += [(b, k, v, int(i)) for i in p]
        count = np.array([len(p) for p in paths])
        c.keep_tokens(first, i32(index.tolist()), count=i32(count.tolist()))
        length = length + count
        s.free(i32(length.tolist()))
    # the same tokens appended one after another, in a cache of its own
    most = int(length.max())
    k, v = [torch.zeros((B, most, kv, d), dtype=BF, device=DEV) for _ in range(2)]
    for b in range(B):
        for t, (row, ks, vs, i) in enumerate(kept[b]):
            k[b, t], v[b, t] = ks[row, i], vs[row, i]
    plain = torch.arange(B * pages, dtype=torch.int32, device=DEV).reshape(B, pages)
    if kind == "codes":
        w = P.HsaCache8(B, H, d, P_, BF, DEV, kv_heads=kv, num_slots=B * pages, page_table=plain, rope=rope)
        w.write(k, v, count=i32(length.tolist()))
    else:
        w = P.HsaLayer(B, kv, d, P_, BF, DEV, num_slots=B * pages, page_table=plain)
        w.write_tokens(k, v, count=i32(length.tolist()), rope=rope)
    # a last token attends to both alike
    q = torch.randn((B, 1, H, d), device=DEV).to(BF)
    outs = []
    for x, pt in ((c, s.page_table), (w, plain)):
        out, lse = torch.full_like(q, 3.0), torch.zeros((B, H, 1), device=DEV)
        x.attend_tree(q, pages, kv_len=i32(length.tolist()), out=out, lse=lse)
        outs.append(out)
        ks, vs = C8.dequantise(arrays(x)) if kind == "codes" else (host(x.k_pool), host(x.v_pool).transpose(0, 1, 3, 2))
        used = [list(range(-(-int(length.max()) // P_)))] * kv
        check(q, out, lse, ks, vs, pt.cpu().numpy(), [used] * B, length, [1] * B, None, d ** -0.5)
    numbers = []  # of both caches, token by token
    for x, pt in ((c, s.page_table.cpu().numpy()), (w, plain.cpu().numpy())):
        ks, vs = C8.dequantise(arrays(x)) if kind == "codes" else (host(x.k_pool), host(x.v_pool).transpose(0, 1, 3, 2))
        numbers.append([np.stack([y[pt[b, t // P_], :, t % P_] for b in range(B) for t in range(length[b])]) for y in (ks, vs)])
    if kind == "pool":  # the same numbers in other slots
        assert torch.equal(*outs)
        assert all(np.array_equal(x, y) for x, y in zip(*numbers))
    else:
        # A draft may have raised a block's scale 2^e, at most to what the largest drafted number x needs. A
        # number is rounded by 2^-4 of it once (a change of the scale is exact but for subnormal codes), and by half a
        # subnormal step, 2^-10 2^e, for each scale that its block had: below 2^-9 2^e in all, scales being
        # powers of two. The same on either side: 2 (2^-4 |x| + 2^-9 2^e).
        for x, y, most in zip(numbers[0], numbers[1], (max(float(t.float().abs().max()) for t in all_k) * 2 ** 0.5,
                                                       max(float(t.float().abs().max()) for t in all_v))):
            step = 2.0 ** C8.exponent(most)
            true = np.maximum(np.abs(x), np.abs(y)) / (1 - 2.0 ** -4) + 2.0 ** -9 * step
            assert (np.abs(x - y) <= 2 * (2.0 ** -4 * true + 2.0 ** -9 * step)).all()
    refs = O.counts(s.page_table.cpu().numpy(), slots)
    assert np.array_equal(s.refs.cpu().numpy(), refs)
