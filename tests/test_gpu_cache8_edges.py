"""The 8-bit cache's attention and appends at the edges of their ranges, against the fp64
oracle (bounds: test_gpu_cache8.py), and past 32-bit offsets."""
import pytest
import torch

import paper_2609_34606_amd as P
from test_gpu_cache8 import BF, F32, run_case
from test_gpu_tokens import i32, source

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("d", [64, 128])
def test_queries_before_the_first_token(d):
    """More queries than tokens, far more: the first ones see nothing, also where the list
    ends inside a tile."""
    run_case(d, 2, 2, 2, d, 72, 300, BF, 3, kv_len=[72, 216], q_len=[256, 300], causal=True)
    run_case(d + 1, 1, 2, 1, d, 72, 200, BF, 5, first=3, n=1, k_max=1, kv_len=[5 * 72], causal=True)
    run_case(d + 2, 1, 2, 1, d, 40, 150, F32, 2, kv_len=[33], causal=True)


def test_a_cache_on_another_device_is_refused():
    """(before any launch)"""
    c = P.HsaCache8(1, 2, 64, 64, BF, "cpu", num_slots=2, max_pages=2)
    layer = P.HsaLayer(1, 2, 64, 64, BF, "cpu", num_slots=2, max_pages=2)
    x = torch.zeros((1, 3, 2, 64), dtype=BF, device=DEV)
    for call in (lambda: c.write(x, x), lambda: c.attend(x, 2), lambda: layer.write_tokens(x, x)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        P.hsa_rope_apply(P.config(1, 2, 64, 64, BF), P.rope(64), x, 3, torch.empty(x.shape, dtype=BF))


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
def test_pages_of_48(dt):
    """The last 16 tokens of a tile are past such a page, here in the last slot too."""
    run_case(1, 2, 4, 2, 64, 48, 1, dt, 5, kv_len=[240, 191])
    run_case(2, 1, 4, 2, 128, 48, 20, dt, 60, causal=True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P_", [72, 200, 256])
def test_many_rows_over_selected_pages_in_pieces(P_, d):
    """Tiles that run from page to page, through selected and chunk pages, cut into pieces."""
    pages = 2600 // P_
    run_case(P_, 1, 2, 1, d, P_, 90, BF, pages, first=pages - 2, k_max=pages - 4, k_h=[pages - 5])
    run_case(P_ + 1, 2, 6, 3, d, P_, 300, BF, 12, first=9, k_max=7, k_h=[7, 0, 3], sel_valid=[7, 5, 1],
             kv_len=[12 * P_ - 3, 9 * P_ + 1], q_len=[300, 211], causal=True)


@pytest.mark.parametrize("H,kv,n_q,d,dt", [(4, 1, 1, 128, BF), (8, 1, 4, 128, BF), (8, 1, 8, 64, BF), (12, 1, 3, 64, F32),
                                           (2, 1, 8, 64, F32), (2, 1, 40, 128, BF)])
@pytest.mark.parametrize("P_", [8, 16, 24, 64, 200])
def test_long_lists_in_pieces(P_, H, kv, n_q, d, dt):
    """Every width of the few-rows kernel over lists long enough to be cut, of small pages too; a
    sequence that ends in the first piece, and one in the last."""
    pages = 4000 // P_
    cap = pages * P_
    print(P_, H, n_q, d, dt, flush=True)
    run_case(P_ + n_q, 2, H, kv, d, P_, n_q, dt, pages, kv_len=[cap - 1, 50], causal=True)
    run_case(P_ + n_q, 1, H, kv, d, P_, n_q, dt, pages)


@pytest.mark.parametrize("n_q", [1, 100])
def test_offsets_past_32_bits(n_q):
    """Pages at the end of a cache of more than 2^32 elements and in a small one: the same
    bits, of the appends and of the attention."""
    H, d, P_, slots = 8, 128, 1560, 2800
    n = 2 * P_ - 92
    got = []
    for num, at in ((slots, [slots - 1, slots - 30]), (2, [1, 0])):
        c = P.HsaCache8(1, H, d, P_, BF, DEV, num_slots=num, max_pages=2, rope=P.rope(d))
        layer = P.HsaLayer(1, H, d, P_, BF, DEV, num_slots=num, max_pages=2)
        for t in (c, layer):
            t.page_table.copy_(torch.tensor([at]))
        for first, count, by in ((0, n - 1, 1.0), (n - 1, 1, 64.0)):  # (the last token grows its block's scale)
            k, v = source(first, 1, count, H, d, BF, True)
            c.write(k * by, v * by, i32([first]))
            layer.write_tokens(k, v, i32([first]), rope=c.rope)
        q = source(6, 1, n_q, H, d, BF, False)[0]
        lse = torch.empty((1, H, n_q), device=DEV)
        out = c.attend(q, 2, kv_len=i32([n]), causal=True, lse=lse)
        held = [out, lse]
        for e in (c.k_exp, c.v_exp):  # (what lies behind the last token was never written)
            held += [e[at[0]], e[at[1], :, :-(-(n - P_) // 64)]]
        for k, v in ((c.k, c.v), (layer.k_pool, layer.v_pool)):
            held += [k[at[0]], v[at[0]], k[at[1], :, :n - P_], v[at[1], :, :, :n - P_]]
        got.append([t.clone() for t in held])
        del c, layer, t, k, v, held
        torch.cuda.empty_cache()
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_rotation_strides_past_32_bits():
    big = torch.empty(2 ** 31 + 4096, dtype=BF, device=DEV)
    x = source(8, 2, 3, 2, 64, BF, False)[0]
    far = big.as_strided((2, 3, 2, 64), (2 ** 31, 256, 64, 1))
    far.copy_(x)
    cfg, rope = P.config(2, 2, 64, 64, BF), P.rope(64)
    want, apart = torch.empty_like(x), torch.empty_like(x)
    P.hsa_rope_apply(cfg, rope, x, 3, want, first=i32([5, 9]))
    P.hsa_rope_apply(cfg, rope, far, 3, apart, first=i32([5, 9]))
    P.hsa_rope_apply(cfg, rope, far, 3, far, first=i32([5, 9]))
    assert torch.equal(apart, want) and torch.equal(far, want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P_", [8, 16, 24, 40, 56])
def test_many_rows_over_small_pages(P_, d):
    """Tiles of two to eight pages: in pieces, over selected pages, with lengths that end
    inside a page, queries that see nothing, a head without pages."""
    pages = 2000 // P_
    print(P_, d, flush=True)
    run_case(P_, 1, 2, 1, d, P_, 90, BF, pages, first=pages - 2, k_max=pages - 4, k_h=[pages - 5])
    run_case(P_ + 1, 2, 6, 3, d, P_, 200, BF, 30, first=20, k_max=17, k_h=[17, 0, 3], sel_valid=[17, 5, 1],
             kv_len=[30 * P_ - 3, 20 * P_ + 1], q_len=[200, 111], causal=True)
    run_case(P_ + 2, 3, 2, 2, d, P_, 130, BF, pages, kv_len=[pages * P_ - 9, 70, 0], q_len=[130, 129, 3], causal=True)
