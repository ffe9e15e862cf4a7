"""The oracle of drafted trees, kept tokens and page tables on cases small enough to write down."""
import numpy as np

from oracle import hsa_cache8_oracle as C8
from oracle import hsa_tree_oracle as O


def test_ancestors_and_positions():
    #      0   1  2  3  4   5: two roots, 1 and 2 under 0, 3 under 1, 4 under 3, 5 under the second root
    parent = np.array([[-1, 0, 0, 1, 3, 9], [-1, -1, 1, 2, 2, 0]])
    bits, pos = O.tree_mask(parent, [6, 5], [10, 0])
    want = [[0], [0, 1], [0, 2], [0, 1, 3], [0, 1, 3, 4], [5]]
    assert [list(np.flatnonzero(r)) for r in bits[0]] == want
    assert pos[0].tolist() == [10, 11, 11, 12, 13, 10]
    assert [list(np.flatnonzero(r)) for r in bits[1]] == [[0], [1], [1, 2], [1, 2, 3], [1, 2, 4], []]
    assert O.pack(bits)[0, :, 0].tolist() == [1, 3, 5, 11, 27, 32]


def test_words_of_a_wide_tree():
    bits = np.zeros((1, 70, 70), bool)
    bits[0, 69, [0, 31, 32, 64, 69]] = True
    assert O.pack(bits)[0, 69].tolist() == [0x80000001, 1, 0x21]


def test_attention_sees_the_sequence_and_the_bits():
    """Scores of 0 average what is seen."""
    B, P, d = 1, 8, 4
    k, v = np.zeros((2, 1, P, d)), np.arange(2 * P, dtype=float).reshape(2, 1, P, 1).repeat(d, 3)
    bits = np.array([[[1, 0, 0], [1, 1, 0], [0, 0, 0]]], bool)
    o, lse, *_ = O.attend(np.zeros((B, 3, 1, d)), k, v, np.array([[0, 1]]), [[[0, 1]]], [10], [3], bits, 1.0)
    # base 7: tokens 0..6, then nodes 7, 8, 9
    assert np.allclose(o[0, :, 0, 0], [np.mean(range(8)), np.mean(range(9)), np.mean(range(7))])
    assert np.allclose(lse[0, 0], np.log([8, 9, 7]))
    o, lse, *_ = O.attend(np.zeros((B, 3, 1, d)), k, v, np.array([[0, 1]]), [[[0, 1]]], [3], [3], bits, 1.0)
    assert o[0, 2, 0, 0] == 0 and np.isneginf(lse[0, 0, 2])
    o, *_ = O.attend(np.zeros((B, 3, 1, d)), k, v, np.array([[0, 1]]), [[[1]]], [10], [3], None, 1.0)
    assert np.allclose(o[0, 1:, 0, 0], [8, 8.5]) and o[0, 0, 0, 0] == 0


def test_kept_tokens():
    k = np.arange(16.0).reshape(2, 1, 8, 1)
    v = k.transpose(0, 1, 3, 2).copy()
    table = np.array([[1, 0]])
    O.keep(k, v, table, [6], np.array([[0, 2, 5, 5]]), [3])
    # tokens 6, 7 are in slot 1, 8.. in slot 0: 7 takes 8, 8 takes 11
    assert k[1, 0, :, 0].tolist() == [8, 9, 10, 11, 12, 13, 14, 0] and k[0, 0, 0, 0] == 3
    assert (v == k.transpose(0, 1, 3, 2)).all()


def test_kept_tokens_in_eight_bits():
    cache = dict(k=np.zeros((1, 1, 8, 4), np.uint8), v=np.zeros((1, 1, 4, 8), np.uint8),
                 k_exp=np.full((1, 1, 1), 127, np.uint8), v_exp=np.full((1, 1, 1), 127, np.uint8))
    cache["k"][0, 0, :, 0] = C8.encode(np.array([1, 2, 3, 448, 5, 6, 7, 8.0]))
    O.keep8(cache, np.array([[0]]), [0], np.array([[0, 2, 4]]), [3])
    k, _ = C8.dequantise(cache)
    assert k[0, 0, :3, 0].tolist() == [1, 3, 5]  # and the block's scale is that of 5
    assert cache["k_exp"][0, 0, 0] == 127 + C8.exponent(5.0)


def test_page_tables():
    table = np.array([[4, 2, -1], [0, -1, -1], [1, 3, -1]])
    refs = O.counts(table, 7)
    assert refs.tolist() == [1, 1, 1, 1, 1, 0, 0]
    forked = O.fork(table, [1, -1, 1])
    assert forked.tolist() == [[0, -1, -1]] * 3
    refs = O.counts(forked, 7)
    # pages of 8 tokens, three tokens each: every row but the last copies
    t, r, moves, missing = O.take(forked, refs, [3, 3, 3], [4, 4, 4], 8)
    assert t.tolist() == [[1, -1, -1], [2, -1, -1], [0, -1, -1]] and missing == 0
    assert moves.tolist() == [[0, 1, 3], [0, 2, 3], [-1, -1, -1]]
    assert (r == O.counts(t, 7)).all()
    # a holder that takes no part keeps the slot
    t, r, moves, _ = O.take(forked, refs, [3, 3, 3], [4, 4, 0], 8)
    assert t[:, 0].tolist() == [1, 2, 0] and r[0] == 1
    # too few slots: the last entries go without
    t, r, moves, missing = O.take(forked, refs, [0, 8, 0], [24, 24, 0], 8)
    assert missing == 0 and t.tolist() == [[1, 2, 3], [0, 4, 5], [0, -1, -1]]
    t, r, moves, missing = O.take(forked, refs, [0, 8, 8], [24, 24, 24], 8)
    assert missing == 1 and t.tolist() == [[1, 2, 3], [0, 4, 5], [0, 6, -1]]
    assert O.free(t, [9, -1, 0], 8).tolist() == [[1, 2, -1], [0, 4, 5], [-1, -1, -1]]


def test_compaction():
    table = np.array([[5, 1, -1], [7, 5, 6]])
    refs = O.counts(table, 8)
    t, r, moves = O.compact(table, refs, 4, 16)
    # four slots are in use: 5, 6, 7 go to 0, 2, 3
    assert moves.tolist() == [[5, 0, 16], [6, 2, 16], [7, 3, 16], [-1, -1, -1]]
    assert t.tolist() == [[0, 1, -1], [3, 0, 2]] and r.tolist() == [2, 1, 1, 1, 0, 0, 0, 0]
    t, r, moves = O.compact(table, refs, 1, 16)
    assert t.tolist() == [[0, 1, -1], [7, 0, 6]] and r.tolist() == [2, 1, 0, 0, 0, 0, 1, 1]


def test_copied_pages():
    a = dict(k=np.arange(3.0 * 16).reshape(3, 1, 16, 1), v=np.arange(3.0 * 16).reshape(3, 1, 1, 16))
    O.page_copy(a, [[0, 2, 3], [-1, 1, 16], [0, 1, 0]], 16)
    assert a["k"][2, 0, :, 0].tolist() == list(range(8)) + list(range(40, 48))
    assert a["v"][1, 0, 0].tolist() == list(range(16, 32))


def test_both_forms_of_the_attention():
    r = np.random.default_rng(3)
    B, n_q, H, kv, d, P = 4, 9, 4, 2, 8, 8
    k, v = r.standard_normal((9, kv, P, d)), r.standard_normal((9, kv, P, d))
    q, table = r.standard_normal((B, n_q, H, d)), r.integers(0, 9, (B, 4))
    k[table[0, 2], 1, 3], v[table[0, 2], :, 5], v[table[0, 2], 0, 6, 2] = np.nan, np.nan, np.inf
    kv_len, q_len, bits = [25, 5, 0, 32], [9, 9, 3, 1], r.random((B, n_q, n_q)) < 0.4
    bits[:, ::4] = False
    pages = [[[2, 0, 1, 3], [3, 2]], [[0], [1]], [[0, 1], []], [[0, 1, 2, 3], [0, 1, 2, 3]]]
    for m in (bits, None):
        a = O.attend(q, k, v, table, pages, kv_len, q_len, m, 0.7)
        b = O.attend_many(q, k, v, table, pages, kv_len, q_len, m, 0.7)
        use = np.isfinite(a[0])
        assert np.array_equal(use, np.isfinite(b[0])) and np.array_equal(np.isinf(a[0]), np.isinf(b[0]))
        assert (~use).any() and use.any()
        rows = use.all(-1).transpose(0, 2, 1)
        for x, y in zip(a, b):
            w = use if x.ndim == 4 else rows
            assert np.allclose(x[w], y[w], rtol=1e-12, atol=1e-13)
