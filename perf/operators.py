"""Measured cases of the rotary, append and 8-bit cache operators.

A serving program of a layer with rotated keys does three things per step:
it rotates the step's queries by their positions (``rope``), appends the
step's keys and values to the paged cache at any token, keys rotated on the
way, in the pool's type (``write``) or in 8 bits (``write8``), and attends
over the 8-bit cache (``attn8``): single tokens of many sequences, ragged
prompts with a causal mask, or a chunk of a streamed video over its selected
pages and its own. Training a layer with rotated queries needs the rotation's
gradient as well (``inverse``).

The 8-bit cache holds OCP e4m3 codes and, for each block of 64 tokens of a page
and key head, a power of two 2^e as the exponent byte e + 127. Both are returned as
the numbers they stand for (float8_e4m3fn and float8_e8m0fnu views of the
cache's own buffers), so that no pass dequantises what a user leaves in 8 bits.

Sizes are those of the repository's workloads (12 heads of 128, 4680 queries
in three pages of 1560 tokens, pages of 256 for the small ones) and ragged or
generic ones.
"""
import math
from types import SimpleNamespace

import torch

own = False

DEV = "cuda:0"
BLOCK = 64        # tokens of a page that share a scale
E_MIN = -100      # smallest exponent of a scale


def listed():
    rope = dict(kind="rope", batch=1, heads=12, d=128, rot=128, layout="half", axes="", scaling="none",
                dtype="bf16", inverse=False, fused=False, at=0)
    write = dict(rope, kind="write8", kv=12, page=256, pages=8, ragged=False)
    attn = dict(kind="attn8", batch=1, heads=12, kv=12, d=128, n_q=1, page=256, pages=1, cand=0, k="0",
                causal=False, ragged=False, dtype="bf16")
    return [
        # One decoded token's queries far into a long sequence: latency.
        dict(rope, name="rope_token", n=1, at=187199),
        # The queries of a streamed 480p chunk: three frames of 30 x 52 tokens,
        # the head's pairs divided over time, row and column, read out of a
        # fused projection.
        dict(rope, name="rope_chunk", n=4680, layout="interleaved", axes="44,42,42", fused=True),
        # The gradient in fp32 of a partly rotated head with positions scaled
        # for a longer context, odd lengths.
        dict(rope, name="rope_gradient_f32", batch=2, n=4097, heads=5, d=64, rot=48, scaling="parts",
             dtype="f32", inverse=True),
        # A ragged batch of prompts appended to the pool in its own type.
        dict(write, name="write_pool_ragged", kind="write", batch=3, n=777, heads=5, kv=5, d=64, rot=64, page=392,
             pages=4, at=300, ragged=True),
        # One token of each of 32 sequences, 8-bit cache: latency.
        dict(write, name="write8_tokens", batch=32, n=1, kv=8, scaling="linear", at=1500, ragged=True),
        # A streamed chunk's keys and values into the 8-bit cache.
        dict(write, name="write8_chunk", n=4680, page=1560, pages=9, layout="interleaved", axes="44,42,42",
             at=3 * 1560, fused=True),
        # One decoded token over a short sequence: latency.
        dict(attn, name="attn8_token", n_q=1, pages=4, ragged=True),
        # 32 sequences of up to 16384 tokens decode together, four query heads
        # to a key head.
        dict(attn, name="attn8_tokens_batch", batch=32, heads=32, kv=8, pages=64, ragged=True),
        # One token over the repository's long history (187,200 keys).
        dict(attn, name="attn8_token_long", page=1560, pages=120),
        # Ragged prompts with a causal mask, odd lengths, pages that end inside
        # a block.
        dict(attn, name="attn8_prompts_ragged", batch=3, heads=16, kv=4, d=64, n_q=1001, page=200, pages=8,
             causal=True, ragged=True),
        # A streamed chunk over four selected history pages and its own three.
        dict(attn, name="attn8_chunk", n_q=4680, page=1560, pages=3, cand=21, k="4"),
        # The small workload's chunk in fp32, as a numerical check of a layer
        # runs it.
        dict(attn, name="attn8_chunk_f32", batch=2, heads=4, kv=2, d=64, n_q=256, pages=1, cand=8, k="2,5",
             dtype="f32"),
    ]


def _log(rng, lo, hi, step=1):
    """A size of [lo, hi], spread over its logarithm, a multiple of step."""
    return max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))) // step * step)


def draw(rng):
    """Another case of the same ranges."""
    kind = rng.choice(["rope", "write", "write8", "write8", "attn8", "attn8", "attn8"])
    d = rng.choice([64, 128])
    if kind != "attn8":
        n = _log(rng, 1, 4680)
        c = dict(kind=kind, batch=max(1, min(rng.choice([1, 2, 3, 8, 32]), 4680 // n)), n=n, d=d,
                 heads=rng.randint(1, 16), rot=rng.choice([d, d, 2 * rng.randint(1, d // 2)]),
                 layout=rng.choice(["half", "interleaved"]), axes="", inverse=False,
                 scaling=rng.choice(["none", "none", "linear", "parts"]),
                 dtype=rng.choice(["bf16", "bf16", "f32"]), fused=rng.random() < 0.5,
                 at=_log(rng, 1, 200000) - 1)
        if rng.random() < 0.4 and c["rot"] >= 6:
            a = 2 * rng.randint(1, c["rot"] // 2 - 2)
            b = 2 * rng.randint(1, (c["rot"] - a) // 2 - 1)
            c["axes"] = "%d,%d,%d" % (a, b, c["rot"] - a - b)
        if kind == "rope":
            c["inverse"] = rng.random() < 0.5
        else:
            page = _log(rng, 8, 1560, 8)
            c.update(page=page, at=_log(rng, 1, 3000) - 1, ragged=rng.random() < 0.5, kv=c["heads"])
            c["pages"] = (c["at"] + n) // page + 2
        return c
    shape = rng.choice(["tokens", "tokens", "prompts", "chunk", "f32"])
    kv = rng.choice([1, 2, 4, 8, 12])
    c = dict(kind=kind, batch=1, kv=kv, heads=kv * rng.choice([1, 2, 4]), d=d, n_q=1, page=_log(rng, 16, 1560, 8),
             pages=1, cand=0, k="0", causal=False, ragged=rng.random() < 0.6, dtype="bf16")
    if shape == "tokens":     # up to 200,000 tokens of context over the batch
        c.update(batch=rng.choice([1, 1, 2, 7, 32]), n_q=rng.choice([1, 1, 1, 2, 5]), causal=rng.random() < 0.5)
        c["pages"] = max(1, _log(rng, 1, 200000 // c["batch"]) // c["page"])
    elif shape == "prompts":
        c.update(batch=rng.randint(1, 4), n_q=_log(rng, 2, 2000), causal=True)
        c["pages"] = -(-(c["n_q"] + rng.randint(0, 2000)) // c["page"])
    else:
        c.update(n_q=_log(rng, 16, 4680), page=_log(rng, 200, 1560, 8), pages=rng.randint(1, 3),
                 cand=rng.randint(1, 21), ragged=False)
        if shape == "f32":
            c.update(dtype="f32", batch=rng.randint(1, 2), n_q=min(c["n_q"], 300), page=min(c["page"], 256),
                     kv=min(kv, 4), heads=min(kv, 4) * rng.choice([1, 2]))
        elif c["heads"] > 16:
            c["heads"] = kv
        c["k"] = ",".join(str(min(c["cand"], rng.randint(0, 5))) for _ in range(rng.randint(1, 3)))
    return c


# ---------------------------------------------------------------- sizes that follow from a case
def _fractions(n):
    """n shares of a length, the first whole, the others spread."""
    return [1.0] + [(0.31 + 0.6180339887 * b) % 1.0 for b in range(1, n)]


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _counts(c):
    """First token written and number of tokens of each batch entry."""
    B, n, at = c["batch"], c["n"], c["at"]
    if not c["ragged"]:
        return [at] * B, [n] * B
    f = _fractions(B)
    if n == 1:  # one token each, at places of their own
        return [max(0, int(at * x)) for x in f], [1] * B
    return [max(0, int(at * f[B - 1 - b])) for b in range(B)], [max(1, int(n * f[b])) for b in range(B)]


def _lengths(c):
    """Cached tokens and queries of each batch entry."""
    B, n_q, full = c["batch"], c["n_q"], (c["cand"] + c["pages"]) * c["page"]
    if not c["ragged"]:
        return [full] * B, [n_q] * B
    f = _fractions(B)
    q = [max(1, int(n_q * x)) for x in f]
    kv = [max(q[b] if c["causal"] else 1, int((full - 3) * f[B - 1 - b])) for b in range(B)]
    return [min(full, x) for x in kv], q


def _budgets(c):
    k = [int(x) for x in c["k"].split(",")]
    return [k[h % len(k)] for h in range(c["kv"])]


def _axes(c):
    return [int(x) for x in c["axes"].split(",")] if c["axes"] else [c["rot"]]


THETA, FACTOR, LOW, HIGH, ORIG = 10000.0, 8.0, 1.0, 32.0, 4096
AMPLITUDE = {"none": 1.0, "linear": 1.0, "parts": 0.1 * math.log(FACTOR) + 1.0}


# ---------------------------------------------------------------- inputs
def _pow2(e):
    """2^e as fp32 numbers, exactly (powers below the smallest normal one become that)."""
    return ((e.clamp(-126, 127).int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """Codes (uint8 e4m3) and exponent bytes of x [..., tokens, d], a scale for each 64 tokens."""
    n, lead = x.shape[-2], x.shape[:-2]
    nb = -(-n // BLOCK)
    amax = torch.nn.functional.pad(x.abs().amax(-1), (0, nb * BLOCK - n)).reshape(*lead, nb, BLOCK).amax(-1)
    m, k = torch.frexp(amax)
    e = torch.where(m <= 0.875, k - 9, k - 8).clamp(E_MIN, 120)
    e = torch.where(amax > 0, e, torch.full_like(e, E_MIN))
    per = e.repeat_interleave(BLOCK, -1)[..., :n, None]
    codes = (x * _pow2(-per)).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, (e + 127).to(torch.uint8)


def _cache(c, g, slots):
    """An 8-bit cache whose every slot holds tokens: normal keys and values, some
    tokens and heads larger than others."""
    H, P, d = c["kv"], c["page"], c["d"]
    nb = -(-P // BLOCK)
    u8 = dict(dtype=torch.uint8, device=DEV)
    k, v = torch.empty((slots, H, P, d), **u8), torch.empty((slots, H, d, P), **u8)
    k_exp, v_exp = torch.empty((slots, H, nb), **u8), torch.empty((slots, H, nb), **u8)
    step = max(1, (1 << 26) // (H * P * d))
    for s in range(0, slots, step):
        n = min(step, slots - s)
        for codes, exps, turn in ((k, k_exp, False), (v, v_exp, True)):
            x = torch.randn((n, H, P, d), generator=g, device=DEV)
            x *= torch.exp(0.3 * torch.randn((n, H, P, 1), generator=g, device=DEV))
            q, e = _quantise(x)
            codes[s:s + n] = q.transpose(-1, -2) if turn else q
            exps[s:s + n] = e
    return SimpleNamespace(k=k, v=v, k_exp=k_exp, v_exp=v_exp)


def _inputs(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 29)
    x = SimpleNamespace()
    B, d, dt = c["batch"], c["d"], _dtype(c)
    i32 = dict(dtype=torch.int32, device=DEV)

    def randn(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    if c["kind"] == "attn8":
        n_pages = c["cand"] + c["pages"]
        x.page_table = torch.randperm(B * n_pages, generator=g, device=DEV).reshape(B, n_pages).to(torch.int32)
        x.cache = _cache(c, g, B * n_pages)
        x.q = randn(B, c["n_q"], c["heads"], d).to(dt)
        kv, ql = _lengths(c)
        x.kv_len = torch.tensor(kv, **i32) if c["ragged"] else None
        x.q_len = torch.tensor(ql, **i32) if c["ragged"] else None
        x.k_h = _budgets(c)
        x.sel = None
        if max(x.k_h):
            order = torch.rand((B, c["kv"], c["cand"]), generator=g, device=DEV).argsort(-1)
            pad = torch.arange(max(x.k_h), device=DEV) >= torch.tensor(x.k_h, device=DEV)[:, None]
            x.sel = order[..., :max(x.k_h)].masked_fill(pad, -1).to(torch.int32).contiguous()
        x.o = torch.zeros((B, c["n_q"], c["heads"], d), dtype=dt, device=DEV)
        x.lse = torch.zeros((B, c["heads"], c["n_q"]), device=DEV)
        return x
    n, H = c["n"], c["kv"] if c["kind"] != "rope" else c["heads"]
    # queries, keys and values of the step, out of one projection or apart
    if c["fused"]:
        x.src = randn(B, n, 3, H, d).to(dt)
        x.k, x.v = x.src[:, :, 1], x.src[:, :, 2]
    else:
        x.k, x.v = randn(B, n, H, d).to(dt), randn(B, n, H, d).to(dt)
    first, count = _counts(c) if c["kind"] != "rope" else ([c["at"]] * B, [n] * B)
    x.first = torch.tensor(first, **i32)
    x.count = torch.tensor(count, **i32) if c["kind"] != "rope" and c["ragged"] else None
    x.pos = None
    if c["axes"]:  # frame, row and column of each token
        t = torch.arange(n, device=DEV)
        x.pos = torch.stack([c["at"] // 1560 + t // 1560, t % 1560 // 52, t % 52], -1).to(torch.int32)
        x.pos = x.pos.expand(B, n, 3).contiguous()
    if c["kind"] == "rope":
        x.out = torch.empty((B, n, H, d), dtype=dt, device=DEV)
        return x
    n_pages = c["pages"]
    x.page_table = torch.randperm(B * n_pages, generator=g, device=DEV).reshape(B, n_pages).to(torch.int32)
    if c["kind"] == "write8":
        x.cache = _cache(c, g, B * n_pages)
    else:
        x.k_pool = randn(B * n_pages, H, c["page"], d).to(dt)
        x.v_pool = randn(B * n_pages, H, d, c["page"]).to(dt)
    return x


def prepare(case, seed):
    st = SimpleNamespace(case=case, x=_inputs(case, seed))
    if own:
        _handles(st)
    return st


# ---------------------------------------------------------------- the framework's calls
def _handles(st):
    """The descriptors a program keeps beside its tensors."""
    import paper_2609_34606_amd as hsa
    c, x = st.case, st.x
    st.hsa = hsa
    st.rope = None
    if c["kind"] != "attn8":
        scaled = dict(scaling=c["scaling"], factor=FACTOR, low=LOW, high=HIGH, orig_len=ORIG) \
            if c["scaling"] != "none" else {}
        st.rope = hsa.rope(c["rot"], layout=c["layout"], theta=THETA, axis_dims=_axes(c) if c["axes"] else None,
                           amplitude=AMPLITUDE[c["scaling"]], **scaled)
    if c["kind"] in ("write8", "attn8"):
        heads = c["heads"] if c["kind"] == "attn8" else c["kv"]  # an append has no query heads
        st.cache = hsa.HsaCache8(c["batch"], heads, c["d"], c["page"], _dtype(c), DEV, kv_heads=c["kv"],
                                 k=x.cache.k, v=x.cache.v, k_exp=x.cache.k_exp, v_exp=x.cache.v_exp,
                                 page_table=x.page_table, rope=st.rope)
    elif c["kind"] == "write":
        st.layer = hsa.HsaLayer(c["batch"], c["kv"], c["d"], c["page"], _dtype(c), DEV, k_pool=x.k_pool,
                                v_pool=x.v_pool, page_table=x.page_table)
    else:
        st.cfg = hsa.config(c["batch"], c["heads"], c["d"], 64, _dtype(c))


def _own(st):
    c, x = st.case, st.x
    if c["kind"] == "rope":
        st.hsa.hsa_rope_apply(st.cfg, st.rope, x.k, c["n"], x.out, pos=x.pos, first=x.first,
                              inverse=c["inverse"])
        return x.out
    if c["kind"] == "write":
        st.layer.write_tokens(x.k, x.v, x.first, count=x.count, rope=st.rope, pos=x.pos)
        return dict(k=x.k_pool, v=x.v_pool)
    if c["kind"] == "write8":
        st.cache.write(x.k, x.v, x.first, count=x.count, pos=x.pos)
        return _numbers(x.cache)
    st.cache.attend(x.q, c["pages"], first_page=c["cand"], sel=x.sel, k_h=x.k_h if x.sel is not None else None,
                    kv_len=x.kv_len, q_len=x.q_len, causal=c["causal"], out=x.o, lse=x.lse)
    return dict(o=x.o, lse=x.lse)


def _numbers(cache):
    return dict(k=cache.k.view(torch.float8_e4m3fn), v=cache.v.view(torch.float8_e4m3fn),
                k_scale=cache.k_exp.view(torch.float8_e8m0fnu), v_scale=cache.v_exp.view(torch.float8_e8m0fnu))


# ---------------------------------------------------------------- plain forms
def _frequencies(c):
    """Angle per position of each pair, in 64 bits, and the axis of each pair."""
    dims = _axes(c)
    i = torch.cat([torch.arange(n // 2, device=DEV, dtype=torch.float64) / n for n in dims])
    axis = torch.cat([torch.full((n // 2,), a, device=DEV, dtype=torch.int64) for a, n in enumerate(dims)])
    f = THETA ** (-2.0 * i)
    if c["scaling"] == "linear":
        f = f / FACTOR
    elif c["scaling"] == "parts":
        w = ((ORIG * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        f = w * f + (1 - w) * f / FACTOR
    return f, axis


def _positions(c, x):
    if x.pos is not None:
        return x.pos
    return (x.first[:, None] + torch.arange(c["n"], device=DEV, dtype=torch.int32))[..., None]


def _rotate(c, x, src):
    """The heads of src [B, n, H, d] rotated, in 32 bits; angles in 64."""
    rot = c["rot"]
    f, axis = _frequencies(c)
    angle = (_positions(c, x).double()[..., axis] * f)[:, :, None]
    cos = (angle.cos() * AMPLITUDE[c["scaling"]]).float()
    sin = (angle.sin() * AMPLITUDE[c["scaling"]]).float()
    if c.get("inverse"):
        sin = -sin
    y = src.float()
    part = y[..., :rot]
    if c["layout"] == "half":
        a, b = part[..., :rot // 2], part[..., rot // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], -1)


def _plain_write(c, x):
    """Tokens past a sequence's count repeat its last one, so that they write the
    same values to the same place."""
    B, n, P = c["batch"], c["n"], c["page"]
    count = x.count[:, None] if x.count is not None else torch.full((B, 1), n, device=DEV)
    i = torch.minimum(torch.arange(n, device=DEV)[None], count - 1)
    rows = torch.arange(B, device=DEV)[:, None]
    tok = x.first[:, None] + i
    slot = torch.gather(x.page_table.long(), 1, (tok // P).long())
    x.k_pool[slot, :, tok % P] = _rotate(c, x, x.k).to(x.k_pool.dtype)[rows, i]
    x.v_pool[slot, :, :, tok % P] = x.v[rows, i]
    return dict(k=x.k_pool, v=x.v_pool)


def _plain_write8(c, x):
    """The touched blocks are gathered whole, quantised and put back. Units past
    a sequence's last block repeat its first one, and tokens past a page's end its
    last one: they write the same values to the same place."""
    B, n, P = c["batch"], c["n"], c["page"]
    nb = -(-P // BLOCK)
    first = x.first[:, None].long()
    count = x.count[:, None].long() if x.count is not None else torch.full((B, 1), n, device=DEV)

    def block_of(tok):
        return tok // P * nb + tok % P // BLOCK

    units = 2 + n // BLOCK + (n // P + 2 if P % BLOCK else 0)
    u = block_of(first) + torch.arange(units, device=DEV)
    u = torch.where(u <= block_of(first + count - 1), u, block_of(first))            # [B, units]
    slot, blk = torch.gather(x.page_table.long(), 1, u // nb), u % nb
    off = (blk * BLOCK)[..., None] + torch.arange(BLOCK, device=DEV)
    off = off.clamp(max=P - 1)                                                       # [B, units, 64]
    i = (u // nb * P)[..., None] + off - first[..., None]                            # token of the step
    new = (i >= 0) & (i < count[..., None])
    older = i < 0
    fresh = ~older.any(-1)
    i = i.clamp(0, n - 1)
    rows = torch.arange(B, device=DEV)[:, None, None]
    for src, codes, exps, turn in ((_rotate(c, x, x.k), x.cache.k, x.cache.k_exp, False),
                                   (x.v.float(), x.cache.v, x.cache.v_exp, True)):
        held = codes.transpose(-1, -2) if turn else codes                            # [slots, H, P, d]
        val = torch.where(new[..., None, None], src[rows, i], 0.0)                   # [B, units, 64, H, d]
        amax = val.abs().amax((2, 4))                                                # [B, units, H]
        m, k = torch.frexp(amax)
        e = torch.where(m <= 0.875, k - 9, k - 8).clamp(E_MIN, 120)
        e = torch.where(amax > 0, e, torch.full_like(e, E_MIN))
        e_old = exps[slot, :, blk].int() - 127
        e = torch.where(fresh[..., None], e, torch.maximum(e, e_old))
        was = held[slot[..., None], :, off]                                          # [B, units, 64, H, d]
        shift = (e_old - e)[:, :, None, :, None]
        kept = was.view(torch.float8_e4m3fn).float() * _pow2(shift)
        now = torch.where(new[..., None, None], val * _pow2(-e)[:, :, None, :, None], kept)
        now = now.to(torch.float8_e4m3fn).view(torch.uint8)
        now = torch.where((new | older)[..., None, None], now, was)                  # what follows stays
        held[slot[..., None], :, off] = now
        exps[slot, :, blk] = (e + 127).to(torch.uint8)
    return _numbers(x.cache)


def _dequantised(codes, exps, turn):
    """Codes [..., P, d] (or d-major) and block exponents as numbers [..., P, d]."""
    P = codes.shape[-1 if turn else -2]
    scale = _pow2(exps.int() - 127).repeat_interleave(BLOCK, -1)[..., :P]
    y = codes.view(torch.float8_e4m3fn).float()
    return (y * scale[..., None, :]).transpose(-1, -2) if turn else y * scale[..., None]


def _plain_attn8(c, x):
    B, n_q, H, kv, d, P = (c[k] for k in ("batch", "n_q", "heads", "kv", "d", "page"))
    G = H // kv
    cur = torch.arange(c["cand"], c["cand"] + c["pages"], device=DEV).expand(B, kv, -1)
    pages = cur if x.sel is None else torch.cat([x.sel.long(), cur], -1)             # [B, kv, L]
    slot = torch.gather(x.page_table.long()[:, None].expand(B, kv, -1), 2, pages.clamp(min=0))
    head = torch.arange(kv, device=DEV)[None, :, None]
    keys = _dequantised(x.cache.k[slot, head], x.cache.k_exp[slot, head], False).reshape(B, kv, -1, d)
    vals = _dequantised(x.cache.v[slot, head], x.cache.v_exp[slot, head], True).reshape(B, kv, -1, d)
    tok = (pages[..., None] * P + torch.arange(P, device=DEV)).flatten(2)            # [B, kv, T]
    seen = (pages >= 0).repeat_interleave(P, -1)
    full = torch.full((B,), (c["cand"] + c["pages"]) * P, device=DEV, dtype=torch.int32)
    kv_len, q_len = (full if x.kv_len is None else x.kv_len), (full * 0 + n_q if x.q_len is None else x.q_len)
    seen = (seen & (tok < kv_len[:, None, None]))[:, :, None]                        # [B, kv, 1, T]
    i = torch.arange(n_q, device=DEV)
    if c["causal"]:
        last = (kv_len - q_len)[:, None] + i                                         # [B, n_q]
        last = last.repeat_interleave(G, 1)[:, None, :, None]
        seen = seen & (tok[:, :, None] <= last)
    q = x.q.float().reshape(B, n_q, kv, G, d).permute(0, 2, 1, 3, 4).reshape(B, kv, n_q * G, d)
    s = torch.matmul(q, keys.transpose(-1, -2)).mul_(1 / math.sqrt(d)).masked_fill_(~seen, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = s.sub_(top).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, vals) / torch.where(l > 0, l, 1.0)
    lse = (top + l.log())[..., 0]
    o = o.reshape(B, kv, n_q, G, d).permute(0, 2, 1, 3, 4).reshape(B, n_q, H, d)
    lse = lse.reshape(B, kv, n_q, G).permute(0, 1, 3, 2).reshape(B, H, n_q)
    row = i < q_len[:, None]
    return dict(o=torch.where(row[..., None, None], o.to(x.o.dtype), x.o),
                lse=torch.where(row[:, None], lse, x.lse))


def run(state):
    if own:
        return _own(state)
    c, x = state.case, state.x
    if c["kind"] == "rope":
        return _rotate(c, x, x.k).to(x.k.dtype)
    return {"write": _plain_write, "write8": _plain_write8, "attn8": _plain_attn8}[c["kind"]](c, x)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    B, d = c["batch"], c["d"]
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "rope":
        x = B * c["n"] * c["heads"] * d
        return dict(bytes=2 * x * e, flops=3 * x)
    if c["kind"] in ("write", "write8"):
        x = sum(_counts(c)[1]) * c["kv"] * d
        held = e if c["kind"] == "write" else 1
        return dict(bytes=2 * x * (e + held), flops=6 * x)
    rows = keys = pairs = 0
    for n, q in zip(*_lengths(c)):
        for k in _budgets(c):
            cur = max(0, n - c["cand"] * c["page"])
            listed_keys = k * c["page"] + cur
            rows, keys = rows + q, keys + listed_keys
            # causal: query i sees all but the last q - 1 - i tokens
            pairs += q * listed_keys - (q * (q - 1) // 2 if c["causal"] else 0)
    G = c["heads"] // c["kv"]
    return dict(bytes=2 * keys * d + 2 * rows * G * d * e, flops=4 * pairs * G * d)


# ---------------------------------------------------------------- 64-bit references
def _turn64(c, x, src):
    """Rotation by complex numbers, in 64 bits."""
    rot, out = c["rot"], src.double().clone()
    half = c["layout"] == "half"
    a = out[..., :rot // 2] if half else out[..., :rot:2]
    b = out[..., rot // 2:rot] if half else out[..., 1:rot:2]
    at = x.pos.double() if x.pos is not None else (x.first.double()[:, None] + torch.arange(c["n"], device=DEV))[..., None]
    steps, col = [], 0
    for axis, n in enumerate(_axes(c)):
        for i in range(n // 2):
            f = math.pow(THETA, -2 * i / n)
            if c["scaling"] == "linear":
                f /= FACTOR
            if c["scaling"] == "parts":
                w = min(1.0, max(0.0, (f * ORIG / (2 * math.pi) - LOW) / (HIGH - LOW)))
                f *= w + (1 - w) / FACTOR
            steps.append(at[..., axis] * (-f if c.get("inverse") else f))
            col += 1
    z = torch.complex(a, b) * torch.polar(torch.full_like(steps[0], AMPLITUDE[c["scaling"]])[..., None],
                                          torch.stack(steps, -1))[:, :, None]
    if half:
        out[..., :rot // 2], out[..., rot // 2:rot] = z.real, z.imag
    else:
        out[..., :rot:2], out[..., 1:rot:2] = z.real, z.imag
    return out


def _exact_write(c, x):
    """What the cache holds before its last rounding: keys and values in units of
    their block's scale (1 in the pool's own type)."""
    P, eight = c["page"], c["kind"] == "write8"
    k, v = _turn64(c, x, x.k), x.v.double()
    held = [x.cache.k.view(torch.float8_e4m3fn).double(), x.cache.v.view(torch.float8_e4m3fn).double().transpose(2, 3)] \
        if eight else [x.k_pool.double(), x.v_pool.double().transpose(2, 3)]
    scale = [2.0 ** (t.double() - 127) for t in (x.cache.k_exp, x.cache.v_exp)] if eight else [None, None]
    for b, (first, count) in enumerate(zip(*_counts(c))):
        t = first
        while t < first + count:
            slot, o = int(x.page_table[b, t // P]), t % P
            stop = min((o // BLOCK + 1) * BLOCK, P) if eight else P
            n = min(stop - o, first + count - t)
            for src, h, s in zip((k, v), held, scale):
                part = src[b, t - first:t - first + n].transpose(0, 1)               # [H, n, d]
                if eight:
                    blk, base = o // BLOCK, o // BLOCK * BLOCK
                    amax = part.abs().amax((1, 2))
                    need = torch.exp2(torch.ceil(torch.log2(amax / 448)).clamp(E_MIN, 120))
                    to = need if o == base else torch.maximum(need, s[slot, :, blk])
                    h[slot, :, base:o] *= (s[slot, :, blk] / to)[:, None, None]
                    s[slot, :, blk] = to
                    part = part / to[:, None, None]
                h[slot, :, o:o + n] = part
            t += n
    out = dict(k=held[0], v=held[1].transpose(2, 3).contiguous())
    return dict(out, k_scale=scale[0], v_scale=scale[1]) if eight else out


def exact(case, seed):
    c, x = case, _inputs(case, seed)
    if c["kind"] == "rope":
        return _turn64(c, x, x.k)
    if c["kind"] != "attn8":
        return _exact_write(c, x)
    P, d, G = c["page"], c["d"], c["heads"] // c["kv"]
    o, lse = x.o.double(), x.lse.double()
    kv_len, q_len = _lengths(c)
    block = torch.arange(P, device=DEV) // BLOCK
    for b in range(c["batch"]):
        for h in range(c["kv"]):
            pages = list(range(c["cand"], c["cand"] + c["pages"]))
            if x.sel is not None:
                pages = [p for p in x.sel[b, h].tolist() if p >= 0] + pages
            slots = x.page_table[b, pages].long()
            ks = 2.0 ** (x.cache.k_exp[slots, h].double() - 127)[:, block]
            vs = 2.0 ** (x.cache.v_exp[slots, h].double() - 127)[:, block]
            k = (x.cache.k[slots, h].view(torch.float8_e4m3fn).double() * ks[:, :, None]).reshape(-1, d)
            v = (x.cache.v[slots, h].view(torch.float8_e4m3fn).double() * vs[:, None]).transpose(1, 2).reshape(-1, d)
            at = (torch.tensor(pages, device=DEV)[:, None] * P + torch.arange(P, device=DEV)).reshape(-1)
            for hq in range(h * G, (h + 1) * G):
                s = x.q[b, :q_len[b], hq].double() @ k.t() / math.sqrt(d)
                s[:, at >= kv_len[b]] = -math.inf
                if c["causal"]:
                    i = torch.arange(q_len[b], device=DEV)[:, None]
                    s.masked_fill_(at > kv_len[b] - q_len[b] + i, -math.inf)
                lse[b, hq, :q_len[b]] = torch.logsumexp(s, 1)
                o[b, :q_len[b], hq] = torch.softmax(s, 1).nan_to_num_(0.0) @ v
    return dict(o=o, lse=lse)
