"""Device buffers of one HSA attention layer, driven through the C ABI."""
from __future__ import annotations

import functools
from typing import Optional, Sequence

from . import hsa as _h


class HsaLayer:
    """Paged KV pool, page table, linear state and page index of one layer.

    Shapes follow include/hsa.h: k_pool [slots,H,P,d], v_pool [slots,H,d,P],
    page_table [B,max_pages], kv_state [B,H,d,d], k_state [B,H,d],
    page_kmean [B,H,max_pages,d]; gate logits [B,n_q,H], or [B,n_q,H,d] with
    gate_dims = d.
    """

    def __init__(self, batch: int, heads: int, head_dim: int, page_size: int,
                 dtype, device, k_pool=None, v_pool=None, page_table=None,
                 num_slots: int = 0, max_pages: int = 0, sm_scale: float = 0.0,
                 gate_dims: int = 0):
        import torch
        self.torch = torch
        self.device = torch.device(device)
        self.dtype = dtype
        self.cfg = _h.config(batch, heads, head_dim, page_size, dtype, sm_scale, gate_dims)
        if k_pool is None:
            k_pool = torch.empty((num_slots, heads, page_size, head_dim), dtype=dtype, device=device)
            v_pool = torch.empty((num_slots, heads, head_dim, page_size), dtype=dtype, device=device)
        if page_table is None:
            page_table = torch.full((batch, max_pages), -1, dtype=torch.int32, device=device)
        self.k_pool, self.v_pool, self.page_table = k_pool, v_pool, page_table
        self.max_pages = int(page_table.shape[-1])
        self.kv_state = torch.zeros((batch, heads, head_dim, head_dim), dtype=torch.float32, device=device)
        self.k_state = torch.zeros((batch, heads, head_dim), dtype=torch.float32, device=device)
        self.page_kmean = torch.zeros((batch, heads, self.max_pages, head_dim), dtype=torch.float64,
                                      device=device)
        self._ws = {}

    @property
    def pool(self) -> _h.HsaKvPool:
        return _h.kv_pool(self.k_pool, self.v_pool, self.page_table, self.cfg)

    def workspace(self, key, nbytes: int):
        if nbytes == 0:
            return None
        w = self._ws.get(key)
        if w is None or w.numel() < nbytes:
            w = self.torch.empty(nbytes, dtype=self.torch.uint8, device=self.device)
            self._ws[key] = w
        return w

    def set_projections(self, e_k, e_v):
        """Linformer projections ([H, rank, P] each, e[h][j][t] = E^(h)[t][j])
        and a compressed pool for every slot of the layer's pool."""
        torch = self.torch
        H, rank = e_k.shape[0], e_k.shape[1]
        self.e_k, self.e_v, self.rank = e_k, e_v, rank
        slots = self.k_pool.shape[0]
        d = self.k_pool.shape[-1]
        self.ck = torch.empty((slots, H, rank, d), dtype=self.k_pool.dtype, device=self.device)
        self.cv = torch.empty((slots, H, d, rank), dtype=self.k_pool.dtype, device=self.device)

    def compress(self, first_page: int, n_pages: int, stream=None):
        """Compress logical pages [first, first+n) with the Linformer projections."""
        ws = self.workspace("compress", _h.hsa_linformer_compress_workspace_size(
            self.cfg, self.rank, n_pages))
        _h.hsa_linformer_compress(self.cfg, self.pool, self.e_k, self.e_v, self.rank, first_page,
                                  n_pages, self.ck, self.cv, ws=ws, stream=stream)

    def reset_state(self):
        self.kv_state.zero_()
        self.k_state.zero_()

    def fold(self, first_page: int, n_pages: int, stream=None):
        """Fold logical pages [first, first+n) into the state and page index."""
        ws = self.workspace("state", _h.hsa_state_update_workspace_size(self.cfg, n_pages))
        _h.hsa_state_update(self.cfg, self.pool, first_page, n_pages, self.kv_state,
                            self.k_state, self.page_kmean, ws=ws, stream=stream)

    def write_tokens(self, k, v, first=None, count=None, rope=None, pos=None, stream=None):
        """Append tokens: k, v [B, n, H, d] become tokens first[b] + i, i < count[b],
        of each sequence (int32 [B]; default 0 and n), keys turned by rope."""
        _same_device(k, self.k_pool)
        _h.hsa_token_write(self.cfg, self.pool, k, v, k.shape[1], first=first, count=count, rope=rope, pos=pos,
                           stream=stream)

    def forward(self, q, n_cand: int, n_cur: int, k_h: Sequence[int], k_max: Optional[int] = None,
                g_lin=None, g_sp=None, out=None, sel_out=None, stream=None):
        B, n_q = q.shape[0], q.shape[1]
        k_max = max(1, max(k_h)) if k_max is None else k_max
        if out is None:
            out = self.torch.empty_like(q)
        ws = self.workspace("fwd", _h.hsa_forward_workspace_size(self.cfg, n_q, k_max, n_cur))
        _h.hsa_forward(self.cfg, q, n_q, self.pool, n_cand, n_cur, k_h, k_max, self.kv_state,
                       self.k_state, self.page_kmean, g_lin, g_sp, out, sel_out=sel_out, ws=ws,
                       stream=stream)
        return out

    def forward_selected(self, q, sel, n_cand: int, n_cur: int, k_h: Sequence[int],
                         k_max: Optional[int] = None, g_lin=None, g_sp=None, out=None, stream=None):
        """The forward pass for a selection already in `sel` ([B,H,k_max] int32)."""
        B, n_q = q.shape[0], q.shape[1]
        k_max = int(sel.shape[-1]) if k_max is None else k_max
        if out is None:
            out = self.torch.empty_like(q)
        ws = self.workspace("fwd", _h.hsa_forward_workspace_size(self.cfg, n_q, k_max, n_cur))
        _h.hsa_forward_selected(self.cfg, q, n_q, self.pool, sel, k_max, k_h, n_cand, n_cur,
                                self.kv_state, self.k_state, g_lin, g_sp, out, ws=ws, stream=stream)
        return out

    def forward_adaptive(self, q, n_cand: int, n_cur: int, k_h: Sequence[int],
                         k_max: Optional[int] = None, tau_min: float = _h.TAU_MIN,
                         tau_max: float = _h.TAU_MAX, g_lin=None, g_sp=None, out=None,
                         sel_out=None, stream=None):
        """The forward pass with the head-adaptive block-sparse sparse branch."""
        B, n_q = q.shape[0], q.shape[1]
        k_max = max(1, max(k_h)) if k_max is None else k_max
        if out is None:
            out = self.torch.empty_like(q)
        ws = self.workspace("fwd_adaptive", _h.hsa_adaptive_workspace_size(self.cfg, n_q, k_max, n_cur))
        _h.hsa_forward_adaptive(self.cfg, q, n_q, self.pool, n_cand, n_cur, k_h, k_max,
                                self.kv_state, self.k_state, self.page_kmean, g_lin, g_sp, out,
                                tau_min=tau_min, tau_max=tau_max, sel_out=sel_out, ws=ws,
                                stream=stream)
        return out

    def forward_linformer(self, q, n_cand: int, n_cur: int, k_h: Sequence[int],
                          k_max: Optional[int] = None, tau_min: float = _h.TAU_MIN,
                          tau_max: float = _h.TAU_MAX, g_lin=None, g_sp=None, out=None,
                          sel_out=None, stream=None):
        """The forward pass with the Linformer linear branch over the compressed
        pages and the head-adaptive block-sparse sparse branch."""
        B, n_q = q.shape[0], q.shape[1]
        k_max = max(1, max(k_h)) if k_max is None else k_max
        if out is None:
            out = self.torch.empty_like(q)
        ws = self.workspace("fwd_linformer", _h.hsa_linformer_workspace_size(self.cfg, n_q, k_max, n_cur))
        _h.hsa_forward_linformer(self.cfg, q, n_q, self.pool, self.ck, self.cv, self.rank, n_cand,
                                 n_cur, k_h, k_max, self.page_kmean, g_lin, g_sp, out,
                                 tau_min=tau_min, tau_max=tau_max, sel_out=sel_out, ws=ws,
                                 stream=stream)
        return out


def _same_device(t, pool):
    """A call runs where its tokens are, and the cache has to be there too."""
    if t.get_device() != pool.get_device():
        raise ValueError(f"the tensors are on {t.device}, the cache on {pool.device}")


@functools.lru_cache(None)
def _rotation():
    """The rotation as a node of an autograd graph: its gradient is the opposite rotation (with the
    same amplitude), which has a gradient of its own."""
    import torch

    class Rotation(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, cfg, rope, pos, first, inverse, stream):
            ctx.call = cfg, rope, inverse
            ctx.save_for_backward(pos, first)
            out = _h.out_like(q, stream)
            _h.hsa_rope_apply(cfg, rope, q, q.shape[1], out, pos=pos, first=first, inverse=inverse, stream=stream)
            return out

        @staticmethod
        def backward(ctx, g):
            # on the stream that was current in the forward pass, where autograd keeps the gradient
            cfg, rope, inverse = ctx.call
            pos, first = ctx.saved_tensors
            if g.stride(3) != 1 or g.stride(2) != g.shape[3]:  # (of a sum: expanded)
                g = g.contiguous()
            return Rotation.apply(g, cfg, rope, pos, first, not inverse, None), None, None, None, None, None, None

    return Rotation


class HsaCache8:
    """Paged 8-bit KV cache of one layer: e4m3 codes k [slots, Hk, P, d] and v
    [slots, Hk, d, P], exponent bytes of the scales of 64-token blocks k_exp, v_exp [slots,
    Hk, ceil(P / 64)], page_table [B, max_pages]; tensors not given are allocated (exponent
    bytes as 0, for appends that begin inside a block that nothing was written to). The tensors stay
    the same over the cache's life (fill the page table in place). ``heads`` are the query heads,
    kv_heads (default: as many) the cached ones. rope turns the keys that are
    written and the queries given to ``rotate``.
    """

    def __init__(self, batch: int, heads: int, head_dim: int, page_size: int, dtype, device,
                 kv_heads: Optional[int] = None, k=None, v=None, k_exp=None, v_exp=None, page_table=None,
                 num_slots: int = 0, max_pages: int = 0, sm_scale: float = 0.0, rope=None):
        import torch
        self.torch = torch
        self.device = torch.device(device)
        self.cfg = _h.config(batch, heads, head_dim, page_size, dtype, sm_scale)
        kv = heads if kv_heads is None else kv_heads
        nb = -(-page_size // _h.CACHE8_BLOCK)
        u8 = dict(dtype=torch.uint8, device=device)
        if k is None:
            k = torch.empty((num_slots, kv, page_size, head_dim), **u8)
            v = torch.empty((num_slots, kv, head_dim, page_size), **u8)
            # (an append that begins inside a block keeps a larger exponent than its own)
            k_exp, v_exp = torch.zeros((num_slots, kv, nb), **u8), torch.zeros((num_slots, kv, nb), **u8)
        if page_table is None:
            page_table = torch.full((batch, max_pages), -1, dtype=torch.int32, device=device)
        if int(k.shape[1]) != kv:
            raise ValueError(f"k must hold {kv} heads, got {tuple(k.shape)}")
        if len({t.device for t in (k, v, k_exp, v_exp, page_table)}) > 1:
            raise ValueError("the cache's tensors must be on one device")
        self.k, self.v, self.k_exp, self.v_exp, self.page_table = k, v, k_exp, v_exp, page_table
        self.rope = rope
        self.pool = _h.cache8_pool(k, v, k_exp, v_exp, page_table, self.cfg)

    def rotate(self, q, pos=None, first=None, out=None, inverse: bool = False, stream=None):
        """q [B, n, heads, d] turned by its tokens' positions, with its gradient if q needs one."""
        if self.rope is None:
            raise ValueError("the cache has no rope")
        if q.requires_grad and self.torch.is_grad_enabled():
            if out is not None:
                raise ValueError("an out of the caller's does not keep the gradient that q needs")
            return _rotation().apply(q, self.cfg, self.rope, pos, first, inverse, stream)
        if out is None:
            out = _h.out_like(q, stream)
        _h.hsa_rope_apply(self.cfg, self.rope, q, q.shape[1], out, pos=pos, first=first, inverse=inverse,
                          stream=stream)
        return out

    def write(self, k, v, first=None, count=None, pos=None, stream=None):
        """Append tokens: k, v [B, n, kv_heads, d] become tokens first[b] + i, i <
        count[b], of each sequence (int32 [B]; default 0 and n)."""
        _same_device(k, self.k)
        _h.hsa_cache8_write(self.cfg, self.pool, k, v, k.shape[1], first=first, count=count, rope=self.rope, pos=pos,
                            stream=stream)

    def attend(self, q, n_pages: int, first_page: int = 0, sel=None, k_h: Optional[Sequence[int]] = None, kv_len=None,
               q_len=None, causal: bool = False, out=None, lse=None, stream=None):
        """Attention of q [B, n_q, heads, d] over the selected pages (sel int32 [B,
        kv_heads, k_max], at most k_h of each head) and pages [first_page, + n_pages)."""
        _same_device(q, self.k)
        if out is None:
            out = _h.out_like(q, stream)
        _h.hsa_cache8_attn(self.cfg, q, q.shape[1], self.pool, sel, 0 if sel is None else int(sel.shape[-1]), k_h,
                           first_page, n_pages, out, lse=lse, kv_len=kv_len, q_len=q_len, causal=causal,
                           stream=stream)
        return out
