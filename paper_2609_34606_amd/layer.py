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

    def attend_tree(self, q, n_pages: int, mask=None, first_page: int = 0, sel=None,
                    k_h: Optional[Sequence[int]] = None, kv_len=None, q_len=None, out=None, lse=None, stream=None):
        """Attention of a step's nodes q [B, n_q, heads, d] (heads: the layer's, or a multiple) over the
        selected pages (sel int32 [B, H, k_max], at most k_h of each head) and pages [first_page, + n_pages):
        tokens before kv_len[b] - q_len[b], and those of the node's mask bits after (hsa_tree_mask; None: up
        to the node itself, as for a single token)."""
        _same_device(q, self.k_pool)
        heads = self.cfg.num_heads
        cfg = self.cfg if q.shape[2] == heads else _h.HsaConfig(self.cfg.batch, q.shape[2], self.cfg.head_dim,
                                                                self.cfg.page_size, self.cfg.dtype,
                                                                self.cfg.sm_scale, 0)
        if out is None:
            out = _h.out_like(q, stream)
        _h.hsa_tree_attn(cfg, q, q.shape[1], self.pool, heads, sel, 0 if sel is None else int(sel.shape[-1]), k_h,
                         first_page, n_pages, out, lse=lse, mask=mask, kv_len=kv_len, q_len=q_len, stream=stream)
        return out

    def keep_tokens(self, first, index, count=None, stream=None):
        """Token first[b] + i takes what token first[b] + index[b][i] holds, i < count[b] (index int32
        [B, n]): the accepted path of a tree becomes the sequence's next tokens."""
        _same_device(index, self.k_pool)
        _h.hsa_token_keep(self.cfg, self.pool, first, index, index.shape[1], count=count, stream=stream)

    def copy_pages(self, moves, stream=None):
        """Copies pages between slots (moves int32 [n, 3] of HsaSlots). Compressed pages go along whole, whatever part of
        a page is copied: their rows are projections of all its tokens."""
        _same_device(moves, self.k_pool)
        _h.hsa_page_copy(self.cfg, self.pool, moves, moves.shape[0], stream=stream)
        if getattr(self, "ck", None) is not None:
            c = self.cfg
            cfg = _h.HsaConfig(c.batch, c.num_heads, c.head_dim, self.rank, c.dtype, c.sm_scale, 0)
            whole = _h.whole_pages(moves, self.rank, stream)
            _h.hsa_page_copy(cfg, _h.kv_pool(self.ck, self.cv, self.page_table), whole, whole.shape[0], stream=stream)

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

    def attend_tree(self, q, n_pages: int, mask=None, first_page: int = 0, sel=None,
                    k_h: Optional[Sequence[int]] = None, kv_len=None, q_len=None, out=None, lse=None, stream=None):
        """Attention of a step's nodes q [B, n_q, heads, d] over the selected pages and pages [first_page, +
        n_pages): tokens before kv_len[b] - q_len[b], and those of the node's mask bits after
        (hsa_tree_mask; None: up to the node itself)."""
        _same_device(q, self.k)
        if out is None:
            out = _h.out_like(q, stream)
        _h.hsa_cache8_tree_attn(self.cfg, q, q.shape[1], self.pool, sel, 0 if sel is None else int(sel.shape[-1]), k_h,
                                first_page, n_pages, out, lse=lse, mask=mask, kv_len=kv_len, q_len=q_len,
                                stream=stream)
        return out

    def keep_tokens(self, first, index, count=None, stream=None):
        """Token first[b] + i takes what token first[b] + index[b][i] holds, i < count[b] (index int32
        [B, n]), as ``write`` appends its numbers."""
        _same_device(index, self.k)
        _h.hsa_cache8_keep(self.cfg, self.pool, first, index, index.shape[1], count=count, stream=stream)

    def copy_pages(self, moves, stream=None):
        """Copies pages between slots (moves int32 [n, 3] of HsaSlots)."""
        _same_device(moves, self.k)
        _h.hsa_cache8_page_copy(self.cfg, self.pool, moves, moves.shape[0], stream=stream)


class HsaSlots:
    """A page table [B, max_pages] whose rows may share slots, and the count of its entries that hold each
    slot, refs [num_slots], on the device (tensors not given are made, with no page and every slot
    free). Layers and caches that are given its page_table follow it; their ``copy_pages`` carries out the
    moves. missing int32 [1]: the entries that found no free slot in the last ``take``.
    """

    def __init__(self, batch: int, page_size: int, device, num_slots: int = 0, max_pages: int = 0, page_table=None,
                 refs=None, missing=None):
        import torch
        self.torch = torch
        i32 = dict(dtype=torch.int32, device=device)
        if (page_table is None) != (refs is None):
            raise ValueError("a page table and its slots' counts are given together")
        if page_table is None:
            page_table, refs = torch.full((batch, max_pages), -1, **i32), torch.zeros(num_slots, **i32)
        self.page_table, self.refs = page_table, refs
        self.missing = torch.zeros(1, **i32) if missing is None else missing
        if len({t.device for t in (self.page_table, self.refs, self.missing)}) > 1:
            raise ValueError("the table's tensors must be on one device")
        self.cfg = _h.config(batch, 1, 64, page_size, _h.HSA_DTYPE_BF16)
        self.table = _h.slot_table(page_table, refs, self.cfg)
        # Calls on one table follow each other, so those of a stream share a workspace, which is that stream's memory.
        self._ws, self._ws_bytes = {}, _h.hsa_slots_workspace_size(self.cfg, self.table.num_slots, self.table.max_pages)

    def _workspace(self, t, stream):
        """The workspace of a call with t on stream."""
        dev = self.refs.get_device()
        if t.get_device() != dev or dev < 0:
            return _same_device(t, self.refs)
        ws = self._ws.get(_h.raw_stream(dev, stream))
        return self._first_call(_h.raw_stream(dev, stream), stream) if ws is None else ws

    def _first_call(self, at, stream):
        _h.used_on(stream, self.page_table, self.refs, self.missing)
        ws, captured = _h.empty_of(self._ws_bytes, self.refs.device, stream)
        if not captured:  # (memory of a graph stays the graph's)
            self._ws[at] = ws
        return ws

    def take(self, first, end, moves=None, stream=None):
        """Makes the pages that hold tokens [first[b], end[b]) of each row (int32 [B]) its own before they are
        written; returns the moves (int32 [B, 3]) that carry over what a shared first page holds."""
        ws = self._workspace(end, stream)
        if moves is None:
            moves = _h.empty_on((self.cfg.batch, 3), self.torch.int32, end.device, stream)
        _h.hsa_slots_take(self.cfg, self.table, first, end, moves=moves, missing=self.missing, ws=ws, stream=stream)
        return moves

    def fork(self, parent, stream=None):
        """Row b becomes what row parent[b] (int32 [B]; outside [0, B): itself) was, sharing its slots."""
        _h.hsa_slots_fork(self.cfg, self.table, parent, ws=self._workspace(parent, stream), stream=stream)

    def free(self, keep, stream=None):
        """Row b lets go of its pages behind its first keep[b] tokens (int32 [B]; 0: all, below 0: none)."""
        self._workspace(keep, stream)
        _h.hsa_slots_free(self.cfg, self.table, keep, stream=stream)

    def compact(self, moves, table_out=None, refs_out=None, stream=None):
        """Moves the slots in use to the front of the pool, at most as many as moves (int32 [n, 3]) has rows; the
        new table and counts go to table_out and refs_out, or in place."""
        _h.hsa_slots_compact(self.cfg, self.table, moves, moves.shape[0], table_out=table_out, refs_out=refs_out,
                             ws=self._workspace(moves, stream), stream=stream)
        return moves
