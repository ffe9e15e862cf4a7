"""Pins of the rotary, append and 8-bit attention oracle against independent
forms: torch's e4m3 type, complex rotation, finite differences, dense attention."""
import numpy as np
import torch

from oracle import hsa_cache8_oracle as O


def test_e4m3_table_and_rounding_match_torch():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.decode(codes), want, equal_nan=True)
    r = np.random.default_rng(1)
    x = np.concatenate([r.standard_normal(20000) * 2.0 ** r.integers(-14, 9, 20000), want[~np.isnan(want)],
                        # the ties between neighbouring numbers
                        (np.sort(want[np.isfinite(want)])[1:] + np.sort(want[np.isfinite(want)])[:-1]) / 2])
    x = x[np.abs(x) <= 448].astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(O.encode(x), want)
    assert O.encode(np.array([np.inf, -np.inf, np.nan, 1e30])).tolist() == [126, 254, 127, 126]


def test_scale_exponent_is_the_smallest_that_fits():
    for a in (448.0, 448.0001, 1.75, 1.7500001, 1.0, 3e38, 1e-3, 2.0 ** -126):
        e = O.exponent(a)
        assert a <= 448 * 2.0 ** e or e == O.E_MAX
        assert e == O.E_MIN or a > 448 * 2.0 ** (e - 1)
    assert O.exponent(0.0) == O.E_MIN


def test_rope_is_a_complex_turn_and_keeps_relative_positions():
    r = np.random.default_rng(2)
    x, y = r.standard_normal((2, 1, 7, 1, 16))
    pos = O.places([5], 7)
    for layout in ("half", "interleaved"):
        got = O.rope(x, pos, 12, layout)
        assert np.array_equal(got[..., 12:], x[..., 12:])
        pair = (lambda v: v[..., :6] + 1j * v[..., 6:12]) if layout == "half" else (lambda v: v[..., :12:2] + 1j * v[..., 1:12:2])
        f = 10000.0 ** (-np.arange(6) / 6)
        want = pair(x) * np.exp(1j * pos[..., None, :] * f)
        assert np.allclose(pair(got), want, atol=1e-13)
        # products depend on the distance alone
        a = (O.rope(x, pos, 12, layout) * O.rope(y, pos + 3, 12, layout)).sum(-1)
        b = (O.rope(x, pos + 90, 12, layout) * O.rope(y, pos + 93, 12, layout)).sum(-1)
        assert np.allclose(a, b, atol=1e-11)


def test_rope_inverse_is_the_gradient_by_differences():
    r = np.random.default_rng(3)
    x, g = r.standard_normal((2, 1, 3, 2, 8))
    kw = dict(rot=6, layout="half", amplitude=1.3, axis_dims=[2, 4], scaling="linear", factor=4.0)
    pos = r.integers(0, 1000, (1, 3, 2))
    grad = O.rope(g, pos, inverse=True, **kw)
    for at in [(0, 0, 0, 0), (0, 1, 1, 4), (0, 2, 0, 5), (0, 2, 1, 7)]:
        h = np.zeros_like(x)
        h[at] = 0.5
        diff = ((O.rope(x + h, pos, **kw) - O.rope(x - h, pos, **kw)) * g).sum()
        assert abs(diff - grad[at]) < 1e-12


def test_scaled_frequencies():
    base = [f for f, _ in O.frequencies(16)]
    lin = [f for f, _ in O.frequencies(16, scaling="linear", factor=4.0)]
    assert np.allclose(np.array(lin) * 4, base)
    part = np.array([f for f, _ in O.frequencies(16, scaling="parts", factor=4.0, low=1.0, high=32.0, orig_len=512)])
    turns = 512 * np.array(base) / (2 * np.pi)
    assert np.allclose(part[turns >= 32], np.array(base)[turns >= 32])
    assert np.allclose(part[turns <= 1] * 4, np.array(base)[turns <= 1])
    assert (np.diff(part) < 0).all()


def test_streamed_append_equals_bulk_but_for_subnormals():
    r = np.random.default_rng(4)
    H, P, d, n = 2, 72, 8, 100
    k, v = r.standard_normal((2, 1, n, H, d)) * 2.0 ** r.integers(-3, 4, (2, 1, n, 1, 1))
    pt = np.array([[1, 0]])
    def empty():
        nb = -(-P // 64)
        z = lambda *s: np.full(s, 127, np.uint8)
        return dict(k=z(2, H, P, d), v=z(2, H, d, P), k_exp=z(2, H, nb), v_exp=z(2, H, nb))
    bulk, step = empty(), empty()
    O.write8(bulk, pt, k, v, [0], [n])
    for i in range(n):
        O.write8(step, pt, k[:, i:i + 1], v[:, i:i + 1], [i], [1])
    assert np.array_equal(bulk["k_exp"], step["k_exp"]) and np.array_equal(bulk["v_exp"], step["v_exp"])
    for a, b in zip(O.dequantise(bulk), O.dequantise(step)):
        seen = ~np.isnan(a)
        assert np.array_equal(seen, ~np.isnan(b))
        # a code that became subnormal was rounded twice: within one subnormal step, 2^-9
        # times the largest scale
        top = 2.0 ** (max(bulk["k_exp"].max(), bulk["v_exp"].max()) - 127.0)
        assert np.abs(a - b)[seen].max() <= 2.0 ** -9 * top


def test_attention_is_dense_softmax():
    r = np.random.default_rng(5)
    q = r.standard_normal((1, 4, 4, 8))
    k, v = r.standard_normal((2, 3, 2, 8, 8))
    pt = np.array([[2, 0, 1]])
    o, lse, _, _, _ = O.attend(q, k, v, pt, [[[0, 1, 2]] * 2], [21], [3], True, 0.5)
    kk = k[[2, 0, 1]].transpose(1, 0, 2, 3).reshape(2, 24, 8)[:, :21]
    vv = v[[2, 0, 1]].transpose(1, 0, 2, 3).reshape(2, 24, 8)[:, :21]
    for h in range(4):
        s = torch.from_numpy(q[0, :3, h] @ kk[h // 2].T * 0.5)
        s = s.masked_fill(torch.arange(21)[None] > 18 + torch.arange(3)[:, None], float("-inf"))
        assert np.allclose(o[0, :3, h], (torch.softmax(s, 1) @ torch.from_numpy(vv[h // 2])).numpy())
        assert np.allclose(lse[0, h, :3], torch.logsumexp(s, 1).numpy())
    assert np.isnan(o[0, 3]).all()
