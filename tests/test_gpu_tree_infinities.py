"""Infinite values among the nodes of a tree: a node that sees one has it, whatever the weights are by
which the waves, the halves of a tile and the pieces of a list are joined (0 for those of which a node sees nothing, or
whose scores lie far below the others')."""
import numpy as np
import pytest
import torch

from oracle import hsa_cache8_oracle as C8
from test_gpu_tokens import arrays, host, i32
from test_gpu_tree import BF, DEV, F32, check, kinds, make, words

pytestmark = pytest.mark.gpu
INF = float("inf")


def with_infinities(kind, c, pt, P_, wild):
    """Values of tokens wild (of entry, token) become infinite; keys and values as the call has them. (A code stands
    for an infinity at the largest scale, 2^120: those of its block become 2^111, its own 2^128.)"""
    for b, t in wild:
        s, o = int(pt[b, t // P_]), t % P_
        if kind == "codes":
            blk = o // 64
            c.v_exp[s, :, blk] = 120 + 127
            c.v[s, :, :, 64 * blk:64 * blk + 64] = 0x01
    for b, t in wild:
        s, o = int(pt[b, t // P_]), t % P_
        if kind == "codes":
            c.v[s, :, :, o] = 0x78
        else:
            c.v_pool[s, :, :, o] = INF
    if kind == "codes":
        k, v = C8.dequantise(arrays(c))
        return k, np.where(np.abs(v) >= 2.0 ** 128, np.copysign(INF, v), v)
    return host(c.k_pool), host(c.v_pool).transpose(0, 1, 3, 2)


def attend(kind, seed, B, H, kv, d, P_, n_q, dt, pages, kv_len, q_len, bits, wild, scale=0.0, spread=0.3):
    c, pt, _, _ = make(kind, seed, B, H, kv, d, P_, dt, pages, kv_len, spread)
    k, v = with_infinities(kind, c, pt, P_, wild)
    c.cfg.sm_scale = scale
    q = torch.randn((B, n_q, H, d), generator=torch.Generator().manual_seed(seed + 1)).to(dt).to(DEV)
    out = torch.full((B, n_q, H, d), 3.0, dtype=dt, device=DEV)
    lse = torch.full((B, H, n_q), 5.0, device=DEV)
    c.attend_tree(q, pages, mask=words(bits), kv_len=i32(kv_len), q_len=i32(q_len), out=out, lse=lse)
    listed = [[list(range(pages))] * kv] * B
    check(q, out, lse, k, v, pt, listed, kv_len, q_len, bits, scale or d ** -0.5, many=True)
    return out


@kinds
@pytest.mark.parametrize("B,H,kv,n_q,d", [(1, 1, 1, 64, 128), (1, 2, 1, 200, 64), (3, 4, 4, 130, 128), (24, 16, 16, 100, 128),
                                          (24, 32, 8, 40, 64), (24, 16, 16, 64, 128), (24, 16, 16, 64, 64), (24, 32, 16, 128, 128)])
def test_of_roots_alone(B, H, kv, n_q, d, kind, dt):
    """A sequence that is nothing but nodes that see themselves alone (and one other each): most waves and halves of a
    tile have nothing for a row."""
    print(B, H, kv, n_q, d, kind, dt, flush=True)
    P_, pages = 64, 19
    r = np.random.default_rng(n_q)
    bits = np.tile(np.eye(n_q, dtype=bool), (B, 1, 1))
    bits[:, np.arange(n_q), r.integers(0, n_q, n_q)] = True
    kv_len = [n_q] + [1216 - b for b in range(1, B)]
    wild = [(0, t) for t in sorted({1, n_q // 3, 40 % n_q, n_q - 2})]
    out = attend(kind, n_q, B, H, kv, d, P_, n_q, dt, pages, kv_len, [n_q] * B, bits, wild)
    assert torch.isinf(out[0]).any() and torch.isfinite(out[1:]).all()


@kinds
@pytest.mark.parametrize("B,H,kv,n_q,d", [(1, 1, 1, 16, 64), (1, 2, 1, 100, 128), (1, 4, 2, 32, 128), (16, 16, 16, 64, 64),
                                          (16, 32, 16, 100, 128)])
def test_of_scores_far_below(B, H, kv, n_q, d, kind, dt):
    """Long lists in pieces, scores up to some hundred apart: weights of whole waves and pieces round to 0."""
    print(B, H, kv, n_q, d, kind, dt, flush=True)
    P_, pages = 200, 30
    bits = np.tile(np.tril(np.ones((n_q, n_q), bool)), (B, 1, 1))
    kv_len = [6000 - 7 * b for b in range(B)]
    t0 = kv_len[0] - n_q
    wild = [(0, t0 + n_q // 2)]
    out = attend(kind, n_q, B, H, kv, d, P_, n_q, dt, pages, kv_len, [n_q] * B, bits, wild, scale=20.0 * d ** -0.5)
    assert torch.isinf(out[0, n_q // 2:]).all() and torch.isfinite(out[0, :n_q // 2]).all() and torch.isfinite(out[1:]).all()
