"""Oracle of drafted trees, kept tokens and page tables (include/hsa.h: hsa_tree_mask,
hsa_tree_attn, hsa_cache8_tree_attn, hsa_token_keep, hsa_cache8_keep, hsa_slots_*, hsa_page_copy). numpy,
loops over nodes, tokens and entries, written from the definitions; attention in fp64.
"""
from __future__ import annotations

import numpy as np
import torch

from . import hsa_cache8_oracle as C8


# ---------------------------------------------------------------- trees
def tree_mask(parent, count, first):
    """(bits bool [B, n, n], pos int [B, n]); rows at or past count are False and 0."""
    B, n = parent.shape
    bits, pos = np.zeros((B, n, n), bool), np.zeros((B, n), np.int64)
    for b in range(B):
        for i in range(count[b]):
            j, depth = i, -1
            while True:
                bits[b, i, j] = True
                depth += 1
                p = parent[b, j]
                if not 0 <= p < j:
                    break
                j = p
            pos[b, i] = first[b] + depth
    return bits, pos


def pack(bits):
    """Bits [B, n, n] as uint32 words [B, n, ceil(n / 32)]."""
    B, n, m = bits.shape
    out = np.zeros((B, n, -(-m // 32)), np.uint32)
    for j in range(m):
        out[:, :, j // 32] |= bits[:, :, j].astype(np.uint32) << np.uint32(j % 32)
    return out


def attend(q, k, v, page_table, pages, kv_len, q_len, bits, scale):
    """q [B, n_q, H, d]; k, v [slots, Hk, P, d]; pages[b][hk]: listed logical pages; bits [B, n_q,
    n_q]: which nodes a node sees, None: those up to itself. Returns o and lse (rows past q_len are NaN),
    the softmax mean of |v|, the largest sum |q . k| and the largest |v| of each row."""
    B, n_q, H, d = q.shape
    Hk, P = k.shape[1], k.shape[2]
    G = H // Hk
    o, va = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, sa, vm = np.full((B, H, n_q), np.nan), np.zeros((B, H, n_q)), np.zeros((B, H, n_q))
    for b in range(B):
        base = kv_len[b] - q_len[b]
        for hk in range(Hk):
            pg = [p for p in pages[b][hk] if p * P < kv_len[b]]
            t = np.concatenate([np.arange(p * P, p * P + P) for p in pg] + [np.zeros(0, np.int64)]).astype(np.int64)
            slots = page_table[b, np.asarray(pg, np.int64)]
            use = t < kv_len[b]
            kk, vv, t = k[slots, hk].reshape(-1, d)[use], v[slots, hk].reshape(-1, d)[use], t[use]
            for i in range(q_len[b]):
                see = t < base
                for x in np.flatnonzero(~see):
                    j = t[x] - base
                    see[x] = j <= i if bits is None else bits[b, i, j]
                for h in range(hk * G, hk * G + G):
                    if not see.any():
                        o[b, i, h], va[b, i, h], lse[b, h, i] = 0.0, 0.0, -np.inf
                        continue
                    with np.errstate(invalid="ignore", over="ignore"):
                        s = kk[see] @ q[b, i, h] * scale
                        p = np.exp(s - s.max())
                        o[b, i, h] = p @ vv[see] / p.sum()
                        va[b, i, h] = p @ np.abs(vv[see]) / p.sum()
                        lse[b, h, i] = s.max() + np.log(p.sum())
                        sa[b, h, i] = (np.abs(kk[see]) @ np.abs(q[b, i, h])).max() * scale
                        vm[b, h, i] = np.abs(vv[see]).max()
    return o, lse, va, sa, vm


def attend_many(q, k, v, page_table, pages, kv_len, q_len, bits, scale, device="cpu"):
    """attend for larger calls: the same numbers, a key head's rows at once in torch's fp64."""
    B, n_q, H, d = q.shape
    Hk, P = k.shape[1], k.shape[2]
    G = H // Hk
    o, va = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, sa, vm = np.full((B, H, n_q), np.nan), np.zeros((B, H, n_q)), np.zeros((B, H, n_q))
    put = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(device)
    for b in range(B):
        base, n = kv_len[b] - q_len[b], q_len[b]
        for hk in range(Hk if n else 0):
            pg = np.asarray([p for p in pages[b][hk] if p * P < kv_len[b]], np.int64)
            t = (pg[:, None] * P + np.arange(P)).ravel()
            slots, use = page_table[b, pg], t < kv_len[b]
            kk, vv, t = put(k[slots, hk].reshape(-1, d)[use]), put(v[slots, hk].reshape(-1, d)[use]), t[use]
            i, j = np.arange(n)[:, None], np.clip(t - base, 0, n_q - 1)
            see = put((t < base)[None] | (j <= i if bits is None else bits[b, :n][:, j]))
            good, any_ = torch.isfinite(vv), see.any(1)
            for h in range(hk * G, hk * G + G):
                qq = put(q[b, :n, h])
                s = torch.where(see, qq @ kk.T * scale, -torch.inf)
                top = torch.where(any_, s.max(1).values if len(t) else 0.0, 0.0)
                p = torch.where(see, torch.exp(s - top[:, None]), 0.0)
                l = p.sum(1)
                x, y = p @ torch.where(good, vv, 0.0), p @ torch.where(good, vv, 0.0).abs()
                for w in torch.nonzero(~good.all(1)).ravel().tolist():  # (values only their seers have)
                    bad, who = torch.where(good[w], 0.0, vv[w]), see[:, w]
                    x[who] += torch.where(good[w], 0.0, p[who, w, None] * bad)
                    y[who] += torch.where(good[w], 0.0, p[who, w, None] * bad.abs())
                none = ~any_[:, None]
                o[b, :n, h] = torch.where(none, 0.0, x / l[:, None]).cpu().numpy()
                va[b, :n, h] = torch.where(none, 0.0, y / l[:, None]).cpu().numpy()
                lse[b, h, :n] = torch.where(any_, top + torch.log(l), -torch.inf).cpu().numpy()
                if len(t):
                    sa[b, h, :n] = torch.where(see, qq.abs() @ kk.abs().T, 0.0).max(1).values.cpu().numpy() * scale
                    vm[b, h, :n] = torch.where(see, vv.abs().max(1).values, 0.0).max(1).values.cpu().numpy()
    return o, lse, va, sa, vm


# ---------------------------------------------------------------- kept tokens
def _place(page_table, b, t, P, slots):
    """(slot, token of the page) of a sequence's token, None outside the table and of a page without a slot."""
    if not 0 <= t < page_table.shape[1] * P or not 0 <= page_table[b, t // P] < slots:
        return None
    return int(page_table[b, t // P]), t % P


def _kept(page_table, P, slots, first, index, count):
    """(batch entry, place that is read, place that is written) of the tokens that are kept."""
    for b in range(page_table.shape[0]):
        for i in range(count[b]):
            src = _place(page_table, b, int(first[b]) + int(index[b, i]), P, slots)
            dst = _place(page_table, b, int(first[b]) + i, P, slots)
            if src and dst:
                yield b, src, dst


def keep(k_pool, v_pool, page_table, first, index, count):
    """The pool [slots, H, P, d] / [slots, H, d, P], changed in place."""
    old_k, old_v = k_pool.copy(), v_pool.copy()
    for _, (s, o), (w, x) in _kept(page_table, k_pool.shape[2], len(k_pool), first, index, count):
        k_pool[w, :, x] = old_k[s, :, o]
        v_pool[w, :, :, x] = old_v[s, :, :, o]


def keep8(cache, page_table, first, index, count):
    """cache: dict of uint8 k, v, k_exp, v_exp, changed in place, as by an append of the kept tokens' numbers.
    Tokens that stay before or among a block's kept ones keep its scale from shrinking, and their numbers."""
    slots, _, P, _ = cache["k"].shape
    numbers = dict(zip("kv", C8.dequantise(cache)))
    kept = list(_kept(page_table, P, slots, first, index, count))
    for b in range(page_table.shape[0]):
        to = {dst: src for c, src, dst in kept if c == b}
        last = {}  # of each block, the last token of the run that the call brings
        for t in range(int(first[b]), int(first[b]) + int(count[b])):
            at = _place(page_table, b, t, P, slots)
            if at:
                last[at[0], at[1] // C8.BLOCK] = at[1]
        for (slot, blk), o1 in last.items():
            run = range(blk * C8.BLOCK, o1 + 1)
            if not any((slot, o) in to for o in run):
                continue
            stay = [o for o in run if (slot, o) not in to]
            for name, x in numbers.items():
                codes = cache[name] if name == "k" else cache[name].transpose(0, 1, 3, 2)
                for h in range(codes.shape[1]):
                    new = {o: x[to[slot, o][0], h, to[slot, o][1]] for o in run if (slot, o) in to}
                    e = C8.exponent(C8.finite_max(np.stack(list(new.values()))))
                    old = int(cache[name + "_exp"][slot, h, blk]) - 127
                    if stay:
                        e = max(e, old)
                        if e > old:
                            codes[slot, h, stay] = C8.encode(C8.decode(codes[slot, h, stay]) * 2.0 ** (old - e))
                    cache[name + "_exp"][slot, h, blk] = e + 127
                    for o, y in new.items():
                        codes[slot, h, o] = C8.encode(y * 2.0 ** -e)


# ---------------------------------------------------------------- page tables
def counts(table, num_slots):
    refs = np.zeros(num_slots, np.int64)
    for s in table.ravel():
        if 0 <= s < num_slots:
            refs[s] += 1
    return refs


def fork(table, parent):
    B = table.shape[0]
    return np.stack([table[parent[b] if 0 <= parent[b] < B else b] for b in range(B)])


def free(table, keep, P):
    table = table.copy()
    for b in range(table.shape[0]):
        if keep[b] >= 0:
            table[b, -(-int(keep[b]) // P):] = -1
    return table


def take(table, refs, first, end, P):
    """(table, refs, moves, missing)."""
    table, refs = table.copy(), refs.copy()
    B, n_pages = table.shape
    moves = np.full((B, 3), -1, np.int64)
    spare = [s for s in range(len(refs)) if refs[s] == 0]
    wanted = []
    for b in range(B):
        f = max(int(first[b]), 0)
        if end[b] > f:
            wanted += [(b, p) for p in range(f // P, min(-(-int(end[b]) // P), n_pages))]
    # a shared slot stays with the last entry that wants it, if all that hold it do
    holders = {}
    for b, p in wanted:
        s = table[b, p]
        if 0 <= s < len(refs) and refs[s] > 1:
            holders.setdefault(s, []).append((b, p))
    stay = {h[-1] for s, h in holders.items() if len(h) == refs[s]}
    shared = {e for h in holders.values() for e in h}
    missing = 0
    for b, p in wanted:
        if not (table[b, p] < 0 or ((b, p) in shared and (b, p) not in stay)):
            continue
        if not spare:
            missing += 1
            continue
        was, now = table[b, p], spare.pop(0)
        table[b, p] = now
        refs[now] = 1
        if was >= 0:
            refs[was] -= 1
            f = max(int(first[b]), 0)
            if p == f // P and f % P:
                moves[b] = was, now, f % P
    return table, refs, moves, missing


def compact(table, refs, n_moves, P):
    """(table, refs, moves)."""
    n = int((refs > 0).sum())
    holes = [s for s in range(n) if refs[s] == 0]
    movers = [s for s in range(n, len(refs)) if refs[s] > 0]
    table_out, refs_out = table.copy(), refs.copy()
    moves = np.full((n_moves, 3), -1, np.int64)
    for i, (src, dst) in enumerate(zip(movers, holes)):
        if i == n_moves:
            break
        moves[i] = src, dst, P
        table_out[table == src] = dst
        refs_out[dst], refs_out[src] = refs[src], 0
    return table_out, refs_out, moves


def page_copy(arrays, moves, P):
    """arrays: dict of k [slots, H, P, d], v [slots, H, d, P] and maybe k_exp, v_exp, changed in place."""
    old = {n: a.copy() for n, a in arrays.items()}
    slots = arrays["k"].shape[0]
    for src, dst, tokens in np.asarray(moves).tolist():
        n = min(-(-min(tokens, P) // 8) * 8, P)
        if not (0 <= src < slots and 0 <= dst < slots) or n <= 0 or src == dst:
            continue
        arrays["k"][dst, :, :n] = old["k"][src, :, :n]
        arrays["v"][dst, :, :, :n] = old["v"][src, :, :, :n]
        for e in ("k_exp", "v_exp"):
            if e in arrays:
                m = -(-n // C8.BLOCK)
                arrays[e][dst, :, :m] = old[e][src, :, :m]
