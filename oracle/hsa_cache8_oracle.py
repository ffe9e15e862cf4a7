"""fp64 oracle of the rotary positions, the token append and the attention over
the 8-bit cache (include/hsa.h: hsa_rope_apply, hsa_token_write, hsa_cache8_write,
hsa_cache8_attn). numpy, loops over tokens and heads, written from the definitions.
"""
from __future__ import annotations

import numpy as np

BLOCK = 64
E_MIN, E_MAX = -100, 120


# ---------------------------------------------------------------- e4m3
def _e4m3_table():
    """Number of each code: sign, 4 exponent bits (bias 7), 3 fraction bits; no
    infinities, the all-ones magnitude is NaN."""
    t = np.empty(256)
    for c in range(256):
        s, e, m = -1.0 if c & 128 else 1.0, c >> 3 & 15, c & 7
        if e == 15 and m == 7:
            t[c] = np.nan
        elif e == 0:
            t[c] = s * m * 2.0 ** -9
        else:
            t[c] = s * (8 + m) * 2.0 ** (e - 10)
    return t


E4M3 = _e4m3_table()


def decode(codes):
    return E4M3[np.asarray(codes, np.uint8)]


def encode(x):
    """Codes of x, to nearest even; beyond the largest number: that one; NaN: NaN."""
    x = np.asarray(x, np.float64)
    mag = np.minimum(np.abs(np.nan_to_num(x, nan=0.0, posinf=1e9, neginf=1e9)), 448.0)
    e = np.maximum(np.floor(np.log2(np.maximum(mag, 2.0 ** -60))), -6.0)
    e = np.where(2.0 ** (e + 1) <= mag, e + 1, e)  # (log2 rounds)
    e = np.where(2.0 ** np.maximum(e, -6) > np.maximum(mag, 2.0 ** -6), e - 1, e)
    e = np.maximum(e, -6.0)
    q = np.rint(mag / 2.0 ** (e - 3))  # in units of the last place, ties to even
    carry = q >= 16
    e, q = np.where(carry, e + 1, e), np.where(carry, 8, q)
    code = np.where(q < 8, q, (e + 7) * 8 + (q - 8)).astype(np.int64)
    code = np.where(np.isnan(x), 127, code)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def exponent(amax):
    """Smallest e in [E_MIN, E_MAX] with amax <= 448 * 2^e."""
    if not amax > 0:
        return E_MIN
    e = int(np.floor(np.log2(amax))) - 10
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return min(max(e, E_MIN), E_MAX)


def finite_max(x):
    x = np.abs(x)
    x = x[np.isfinite(x)]
    return float(x.max()) if x.size else 0.0


# ---------------------------------------------------------------- rotary positions
def frequencies(rot, axis_dims=None, theta=10000.0, scaling="none", factor=1.0, low=1.0, high=32.0, orig_len=0):
    """(frequency, axis) of each pair."""
    out = []
    for a, n in enumerate(axis_dims or [rot]):
        for j in range(n // 2):
            f = theta ** (-2.0 * j / n)
            if scaling == "linear":
                f /= factor
            elif scaling == "parts":
                w = min(1.0, max(0.0, (orig_len * f / (2 * np.pi) - low) / (high - low)))
                f = w * f + (1 - w) * f / factor
            out.append((f, a))
    return out


def rope(x, pos, rot, layout="half", amplitude=1.0, inverse=False, **kw):
    """x [B, n, H, d] float64, pos [B, n, axes]."""
    y = np.array(x, np.float64)
    for i, (f, a) in enumerate(frequencies(rot, **kw)):
        ang = pos[..., a].astype(np.float64) * (-f if inverse else f)
        c, s = amplitude * np.cos(ang)[..., None], amplitude * np.sin(ang)[..., None]
        j, k = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
        y[..., j] = x[..., j] * c - x[..., k] * s
        y[..., k] = x[..., k] * c + x[..., j] * s
    return y


def places(first, n, axes=1):
    """Default positions: token i of entry b at first[b] + i."""
    p = np.asarray(first, np.int64)[:, None] + np.arange(n)
    return np.repeat(p[..., None], axes, -1)


# ---------------------------------------------------------------- append
def write_tokens(k_pool, v_pool, page_table, k, v, first, count):
    """Pool [slots, H, P, d] / [slots, H, d, P] after the append, in the given type."""
    P = k_pool.shape[2]
    for b in range(k.shape[0]):
        for i in range(count[b]):
            t = first[b] + i
            if 0 <= t < page_table.shape[1] * P:
                s = page_table[b, t // P]
                k_pool[s, :, t % P] = k[b, i]
                v_pool[s, :, :, t % P] = v[b, i]


def write8(cache, page_table, k, v, first, count):
    """cache: dict of uint8 k, v, k_exp, v_exp, changed in place; k, v float64
    [B, n, H, d] (keys already turned). Returns the exact numbers, in units of the block's
    scale, that the written codes round: [slots, H, P, d] each, NaN elsewhere."""
    H, P, d = cache["k"].shape[1:]
    exact = {"k": np.full(cache["k"].shape, np.nan), "v": np.full(cache["k"].shape, np.nan)}
    for b in range(k.shape[0]):
        lo = max(first[b], 0)
        hi = min(first[b] + count[b], page_table.shape[1] * P)
        t = lo
        while t < hi:
            slot, o = page_table[b, t // P], t % P
            blk = o // BLOCK
            base, stop = blk * BLOCK, min((blk + 1) * BLOCK, P)
            n = min(stop - o, hi - t)
            for name, src in (("k", k), ("v", v)):
                codes = cache[name] if name == "k" else cache[name].transpose(0, 1, 3, 2)
                for h in range(H):
                    new = src[b, t - first[b]:t - first[b] + n, h]
                    e = exponent(finite_max(new))
                    if o > base:
                        old = int(cache[name + "_exp"][slot, h, blk]) - 127
                        e = max(e, old)
                        if e > old:
                            kept = decode(codes[slot, h, base:o]) * 2.0 ** (old - e)
                            codes[slot, h, base:o] = encode(kept)
                            exact[name][slot, h, base:o] = kept
                    cache[name + "_exp"][slot, h, blk] = e + 127
                    codes[slot, h, o:o + n] = encode(new * 2.0 ** -e)
                    exact[name][slot, h, o:o + n] = new * 2.0 ** -e
            t += n
    return exact


def dequantise(cache):
    """(k, v) as float64 [slots, H, P, d]."""
    P = cache["k"].shape[2]
    per = lambda e: (2.0 ** (e.astype(np.float64) - 127))[..., np.arange(P) // BLOCK][..., None]
    return decode(cache["k"]) * per(cache["k_exp"]), decode(cache["v"]).transpose(0, 1, 3, 2) * per(cache["v_exp"])


# ---------------------------------------------------------------- attention
def attend(q, k, v, page_table, pages, kv_len, q_len, causal, scale):
    """q [B, n_q, H, d]; k, v [slots, Hk, P, d]; pages[b][hk]: listed logical pages.
    Returns o and lse (rows past q_len are NaN), the softmax mean of |v|, the
    largest sum |q . k| and the largest |v| of each row (for error bounds)."""
    B, n_q, H, d = q.shape
    Hk, P = k.shape[1], k.shape[2]
    G = H // Hk
    o = np.full(q.shape, np.nan)
    va = np.full(q.shape, np.nan)
    lse, sa, vm = np.full((B, H, n_q), np.nan), np.zeros((B, H, n_q)), np.zeros((B, H, n_q))
    for b in range(B):
        for h in range(H):
            pg = [p for p in pages[b][h // G] if p * P < kv_len[b]]
            t = np.concatenate([np.arange(p * P, p * P + P) for p in pg] + [np.zeros(0, np.int64)])
            slots = page_table[b, np.asarray(pg, np.int64)]
            kk = k[slots, h // G].reshape(-1, d)[t < kv_len[b]]
            vv = v[slots, h // G].reshape(-1, d)[t < kv_len[b]]
            t = t[t < kv_len[b]]
            for i in range(q_len[b]):
                see = t <= kv_len[b] - q_len[b] + i if causal else np.ones(len(t), bool)
                if not see.any():
                    o[b, i, h], va[b, i, h], lse[b, h, i] = 0.0, 0.0, -np.inf
                    continue
                s = kk[see] @ q[b, i, h] * scale
                p = np.exp(s - s.max())
                o[b, i, h] = p @ vv[see] / p.sum()
                va[b, i, h] = p @ np.abs(vv[see]) / p.sum()
                lse[b, h, i] = s.max() + np.log(p.sum())
                sa[b, h, i] = (np.abs(kk[see]) @ np.abs(q[b, i, h])).max() * scale
                vm[b, h, i] = np.abs(vv[see]).max()
    return o, lse, va, sa, vm
