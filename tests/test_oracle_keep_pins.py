"""The oracle of kept tokens in the 8-bit cache against appends of their numbers, and tokens that stay."""
import numpy as np
import pytest

from oracle import hsa_cache8_oracle as C8
from oracle import hsa_tree_oracle as O


def cache(r, slots, H, P, d):
    nb = -(-P // C8.BLOCK)
    c = dict(k=r.integers(0, 256, (slots, H, P, d)).astype(np.uint8), v=r.integers(0, 256, (slots, H, d, P)).astype(np.uint8),
             k_exp=r.integers(120, 134, (slots, H, nb)).astype(np.uint8), v_exp=r.integers(120, 134, (slots, H, nb)).astype(np.uint8))
    for n in "kv":
        c[n][(c[n] & 127) == 127] = 0x30  # (a NaN's two codes are alike)
    return c


@pytest.mark.parametrize("P", [8, 24, 64, 72, 200])
def test_kept_tokens_are_appended(P):
    r = np.random.default_rng(P)
    B, pages, n = 2, 400 // P + 2, 30
    c = cache(r, B * pages, 2, P, 4)
    table = r.permutation(B * pages).reshape(B, pages)
    first, count, index = [5, 61], [30, 17], r.integers(0, 60, (B, n))
    want = {k: x.copy() for k, x in c.items()}
    num = C8.dequantise(c)
    new = [np.zeros((B, n, 2, 4)) for _ in num]
    for b in range(B):
        for i in range(n):
            t = first[b] + index[b, i]
            for x, y in zip(new, num):
                x[b, i] = y[table[b, t // P], :, t % P]
    C8.write8(want, table, *new, first, count)
    O.keep8(c, table, first, index, count)
    for k in c:
        assert np.array_equal(c[k], want[k]), k


def test_tokens_that_stay():
    """Pages of 8: of a run whose second source is no token, the second stays; of one without any source, all."""
    r = np.random.default_rng(0)
    c = cache(r, 3, 1, 8, 4)
    c["k_exp"][:], c["v_exp"][:] = 120, 133
    c["k_exp"][1, 0, 0] = 130  # where the kept keys come from
    was = {k: x.copy() for k, x in c.items()}
    before = C8.dequantise(c)
    O.keep8(c, np.array([[0, 1, 2]]), [0], np.array([[9, 99, 10] + [-1] * 13]), [16])
    after = C8.dequantise(c)
    for x, y in zip(before, after):
        assert np.array_equal(y[0, 0, 0], x[1, 0, 1]) and np.array_equal(y[0, 0, 2], x[1, 0, 2])
        assert (np.abs(y[0, 0, [1, 3, 4, 5, 6, 7]] - x[0, 0, [1, 3, 4, 5, 6, 7]]) <= 2.0 ** -10 * 2.0 ** 3).all()
    assert c["k_exp"][0, 0, 0] > 120 and c["v_exp"][0, 0, 0] == 133
    for k in c:
        assert np.array_equal(c[k][1:], was[k][1:]), k
