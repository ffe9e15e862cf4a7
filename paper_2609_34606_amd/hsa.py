"""ctypes binding of libhsa.so (include/hsa.h).

Argument marshalling only: tensors are passed as raw device pointers, the
per-head budgets as a host int32 array, and the stream as the current torch
stream. Every step of the computation runs in the library's HIP kernels.
There is no fallback: if the library is not built, loading it raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib", "libhsa.so")

HSA_DTYPE_BF16 = 0
HSA_DTYPE_F32 = 1
STATUS = {0: "HSA_OK", 1: "HSA_ERR_INVALID_ARG", 2: "HSA_ERR_UNSUPPORTED",
          3: "HSA_ERR_OUT_OF_RANGE", 4: "HSA_ERR_WORKSPACE", 5: "HSA_ERR_DEVICE",
          6: "HSA_ERR_IO"}

c_i32, c_vp, c_sz = ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t


class HsaConfig(ctypes.Structure):
    _fields_ = [("batch", c_i32), ("num_heads", c_i32), ("head_dim", c_i32),
                ("page_size", c_i32), ("dtype", c_i32), ("sm_scale", ctypes.c_float),
                ("gate_dims", c_i32)]


class HsaTierStats(ctypes.Structure):
    _fields_ = [("evictions", ctypes.c_int64), ("fetches", ctypes.c_int64),
                ("spills", ctypes.c_int64), ("reloads", ctypes.c_int64),
                ("prefetched", ctypes.c_int64), ("backups", ctypes.c_int64)]


class HsaKvPool(ctypes.Structure):
    _fields_ = [("k", c_vp), ("v", c_vp), ("page_table", c_vp),
                ("num_slots", c_i32), ("max_pages", c_i32)]


class HsaRope(ctypes.Structure):
    _fields_ = [("rot_dim", c_i32), ("layout", c_i32), ("axes", c_i32), ("axis_dim", c_i32 * 3),
                ("scaling", c_i32), ("orig_len", c_i32), ("theta", ctypes.c_double),
                ("factor", ctypes.c_double), ("low", ctypes.c_double), ("high", ctypes.c_double),
                ("amplitude", ctypes.c_double)]


class HsaCache8Pool(ctypes.Structure):
    _fields_ = [("k", c_vp), ("v", c_vp), ("k_exp", c_vp), ("v_exp", c_vp), ("page_table", c_vp),
                ("num_slots", c_i32), ("max_pages", c_i32), ("kv_heads", c_i32)]


class HsaSlotTable(ctypes.Structure):
    _fields_ = [("page_table", c_vp), ("refs", c_vp), ("num_slots", c_i32), ("max_pages", c_i32)]


class HsaError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} failed: {STATUS.get(status, status)}")
        self.status = status


class LibraryNotBuilt(RuntimeError):
    pass


_lib = None
_torch = None  # torch, once the library is loaded


def lib():
    """The loaded libhsa.so; raises if it has not been built."""
    global _lib, _torch
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise LibraryNotBuilt(f"{LIB_PATH} missing: build it with `python -m paper_2609_34606_amd.build`")
    # torch's HIP runtime first: the library's libamdhip64.so.7 then binds to
    # that copy (same soname). Loaded the other way round, torch loads its own
    # copy beside the system one, and memory and streams of one runtime are
    # not valid in the other (the library's launches then fail).
    import torch
    _torch = torch
    L = ctypes.CDLL(LIB_PATH)
    P = ctypes.POINTER
    L.hsa_status_string.restype = ctypes.c_char_p
    L.hsa_status_string.argtypes = [ctypes.c_int]
    for n, extra in (("hsa_state_update_workspace_size", [c_i32]),
                     ("hsa_page_select_workspace_size", [c_i32]),
                     ("hsa_sparse_attn_workspace_size", [c_i32, c_i32, c_i32]),
                     ("hsa_forward_workspace_size", [c_i32, c_i32, c_i32]),
                     ("hsa_adaptive_workspace_size", [c_i32, c_i32, c_i32])):
        f = getattr(L, n)
        f.restype = c_sz
        f.argtypes = [P(HsaConfig)] + extra
    for n, extra in (("hsa_linformer_compress_workspace_size", [c_i32, c_i32]),
                     ("hsa_linformer_workspace_size", [c_i32, c_i32, c_i32])):
        f = getattr(L, n)
        f.restype = c_sz
        f.argtypes = [P(HsaConfig)] + extra
    L.hsa_linformer_compress.restype = ctypes.c_int
    L.hsa_linformer_compress.argtypes = [P(HsaConfig), P(HsaKvPool), c_vp, c_vp, c_i32, c_i32,
                                         c_i32, c_vp, c_vp, c_vp, c_sz, c_vp]
    L.hsa_forward_linformer.restype = ctypes.c_int
    L.hsa_forward_linformer.argtypes = [P(HsaConfig), c_vp, c_i32, P(HsaKvPool), c_vp, c_vp, c_i32,
                                        c_i32, c_i32, c_vp, c_i32, ctypes.c_double,
                                        ctypes.c_double, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_sz,
                                        c_vp]
    L.hsa_retrieval_workspace_size.restype = c_sz
    L.hsa_retrieval_workspace_size.argtypes = [P(HsaConfig), c_i32, c_i32, c_i32]
    L.hsa_chunk_select.restype = ctypes.c_int
    L.hsa_chunk_select.argtypes = [P(HsaConfig), c_vp, c_vp, c_i32, c_i32, c_vp, c_i32, c_vp, c_vp,
                                   c_vp, c_vp]
    L.hsa_forward_retrieval.restype = ctypes.c_int
    L.hsa_forward_retrieval.argtypes = [P(HsaConfig), c_vp, c_i32, P(HsaKvPool), c_vp, c_vp, c_i32,
                                        c_i32, c_vp, c_i32, c_i32, c_vp, c_i32, c_vp, c_vp, c_vp,
                                        c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_sz, c_vp]
    L.hsa_tier_create.restype = ctypes.c_int
    L.hsa_tier_create.argtypes = [P(HsaConfig), P(HsaKvPool), c_vp, c_vp, c_i32, ctypes.c_char_p,
                                  c_i32, c_i32, P(c_vp)]
    L.hsa_tier_destroy.restype = None
    L.hsa_tier_destroy.argtypes = [c_vp]
    L.hsa_tier_place.restype = ctypes.c_int
    L.hsa_tier_place.argtypes = [c_vp, c_i32, c_i32, P(c_i32), c_vp]
    L.hsa_tier_fetch.restype = ctypes.c_int
    L.hsa_tier_fetch.argtypes = [c_vp, c_vp, c_i32, c_vp]
    L.hsa_tier_prefetch.restype = ctypes.c_int
    L.hsa_tier_prefetch.argtypes = [c_vp, c_vp, c_i32, c_vp]
    L.hsa_tier_commit.restype = ctypes.c_int
    L.hsa_tier_commit.argtypes = [c_vp, c_vp]
    L.hsa_tier_drop.restype = ctypes.c_int
    L.hsa_tier_drop.argtypes = [c_vp, c_vp]
    L.hsa_tier_locate.restype = c_i32
    L.hsa_tier_locate.argtypes = [c_vp, c_i32, c_i32]
    L.hsa_tier_stats.restype = None
    L.hsa_tier_stats.argtypes = [c_vp, P(HsaTierStats)]
    L.hsa_forward_noalloc_bytes.restype = c_sz
    L.hsa_forward_noalloc_bytes.argtypes = [P(HsaConfig), c_i32, c_i32, c_i32, c_vp, c_i32]
    L.hsa_forward_noalloc.restype = ctypes.c_int
    L.hsa_forward_noalloc.argtypes = [P(HsaConfig), c_vp, c_i32, P(HsaKvPool), c_i32, c_i32, c_vp,
                                      c_i32, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp]
    L.hsa_page_write.restype = ctypes.c_int
    L.hsa_page_write.argtypes = [P(HsaConfig), P(HsaKvPool), c_vp, c_vp, c_i32, c_i32, c_vp, c_vp]
    L.hsa_cube_order.restype = c_i32
    L.hsa_cube_order.argtypes = [c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, c_vp]
    L.hsa_attention_plan.restype = ctypes.c_int
    L.hsa_attention_plan.argtypes = [P(HsaConfig), c_i32, c_vp, c_i32, c_vp, c_vp, c_vp]
    L.hsa_block_count.restype = c_i32
    L.hsa_block_count.argtypes = [P(HsaConfig), c_i32, c_i32]
    c_f64 = ctypes.c_double
    L.hsa_block_select.restype = ctypes.c_int
    L.hsa_block_select.argtypes = [P(HsaConfig), c_vp, c_i32, P(HsaKvPool), c_vp, c_i32, c_i32,
                                   c_i32, c_f64, c_f64, c_vp, c_vp, c_vp, c_vp, c_vp, c_i32, c_vp,
                                   c_sz, c_vp]
    L.hsa_sparse_attn_adaptive.restype = ctypes.c_int
    L.hsa_sparse_attn_adaptive.argtypes = [P(HsaConfig), c_vp, c_i32, P(HsaKvPool), c_vp, c_i32,
                                           c_vp, c_i32, c_i32, c_f64, c_f64, c_vp, c_vp, c_vp,
                                           c_sz, c_vp]
    L.hsa_forward_adaptive.restype = ctypes.c_int
    L.hsa_forward_adaptive.argtypes = [P(HsaConfig), c_vp, c_i32, P(HsaKvPool), c_i32, c_i32, c_vp,
                                       c_i32, c_f64, c_f64, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp,
                                       c_vp, c_vp, c_sz, c_vp]
    L.hsa_state_update.restype = ctypes.c_int
    L.hsa_state_update.argtypes = [P(HsaConfig), P(HsaKvPool), c_i32, c_i32, c_vp, c_vp, c_vp,
                                   c_vp, c_sz, c_vp]
    L.hsa_page_select.restype = ctypes.c_int
    L.hsa_page_select.argtypes = [P(HsaConfig), c_vp, c_i32, c_vp, c_i32, c_i32, c_vp, c_i32,
                                  c_vp, c_vp, c_vp, c_sz, c_vp]
    L.hsa_sparse_attn.restype = ctypes.c_int
    L.hsa_sparse_attn.argtypes = [P(HsaConfig), c_vp, c_i32, P(HsaKvPool), c_vp, c_i32, c_vp,
                                  c_i32, c_i32, c_vp, c_vp, c_vp, c_sz, c_vp]
    L.hsa_forward.restype = ctypes.c_int
    L.hsa_forward.argtypes = [P(HsaConfig), c_vp, c_i32, P(HsaKvPool), c_i32, c_i32, c_vp,
                              c_i32, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_sz, c_vp]
    L.hsa_forward_selected.restype = ctypes.c_int
    L.hsa_forward_selected.argtypes = [P(HsaConfig), c_vp, c_i32, P(HsaKvPool), c_vp, c_i32, c_vp,
                                       c_i32, c_i32, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_sz, c_vp]
    c_i64 = ctypes.c_int64
    L.hsa_rope_apply.restype = ctypes.c_int
    L.hsa_rope_apply.argtypes = [P(HsaConfig), P(HsaRope), c_vp, c_i64, c_i64, c_i32, c_i32, c_vp, c_vp,
                                 c_i32, c_vp, c_i64, c_i64, c_vp]
    for n, pool in (("hsa_token_write", HsaKvPool), ("hsa_cache8_write", HsaCache8Pool)):
        f = getattr(L, n)
        f.restype = ctypes.c_int
        f.argtypes = [P(HsaConfig), P(pool), P(HsaRope), c_vp, c_i64, c_i64, c_vp, c_i64, c_i64, c_i32,
                      c_vp, c_vp, c_vp, c_vp]
    L.hsa_cache8_attn_workspace_size.restype = c_sz
    L.hsa_cache8_attn_workspace_size.argtypes = [P(HsaConfig), c_i32, c_i32, c_i32, c_i32]
    L.hsa_cache8_attn_plan.restype = ctypes.c_int
    L.hsa_cache8_attn_plan.argtypes = [P(HsaConfig), c_i32, c_i32, c_i32, c_i32, c_i32, c_vp, c_vp, c_vp]
    L.hsa_cache8_attn.restype = ctypes.c_int
    L.hsa_cache8_attn.argtypes = [P(HsaConfig), c_vp, c_i32, P(HsaCache8Pool), c_vp, c_i32, c_vp, c_i32,
                                  c_i32, c_vp, c_vp, c_i32, c_vp, c_vp, c_vp, c_sz, c_vp]
    i = ctypes.c_int
    cfg, tree = P(HsaConfig), [c_vp, c_i32, c_vp, c_i32, c_i32, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_sz, c_vp]
    for n, res, args in (
            ("hsa_tree_mask", i, [c_vp, c_i32, c_vp, c_vp, c_vp, c_vp, c_vp]),
            ("hsa_tree_attn_workspace_size", c_sz, [c_i32, c_i32, c_i32, c_i32]),
            ("hsa_cache8_tree_attn_workspace_size", c_sz, [c_i32, c_i32, c_i32, c_i32]),
            ("hsa_tree_attn", i, [c_vp, c_i32, P(HsaKvPool), c_i32] + tree),
            ("hsa_cache8_tree_attn", i, [c_vp, c_i32, P(HsaCache8Pool)] + tree),
            ("hsa_token_keep", i, [P(HsaKvPool), c_vp, c_vp, c_i32, c_vp, c_vp]),
            ("hsa_cache8_keep", i, [P(HsaCache8Pool), c_vp, c_vp, c_i32, c_vp, c_vp]),
            ("hsa_page_copy", i, [P(HsaKvPool), c_vp, c_i32, c_vp]),
            ("hsa_cache8_page_copy", i, [P(HsaCache8Pool), c_vp, c_i32, c_vp]),
            ("hsa_slots_workspace_size", c_sz, [c_i32, c_i32]),
            ("hsa_slots_take", i, [P(HsaSlotTable), c_vp, c_vp, c_vp, c_vp, c_vp, c_sz, c_vp]),
            ("hsa_slots_fork", i, [P(HsaSlotTable), c_vp, c_vp, c_sz, c_vp]),
            ("hsa_slots_free", i, [P(HsaSlotTable), c_vp, c_vp]),
            ("hsa_slots_compact", i, [P(HsaSlotTable), c_vp, c_i32, c_vp, c_vp, c_vp, c_sz, c_vp])):
        f = getattr(L, n)
        f.restype, f.argtypes = res, [cfg] + args
    _lib = L
    return L


# ------------------------------------------------------------------ helpers
def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if hasattr(t, "data_ptr"):
        if not t.is_contiguous():
            raise ValueError("tensor arguments must be contiguous")
        return t.data_ptr()
    return int(t)


def _out(t, n: int, dtype: str, what: str) -> Optional[int]:
    """Pointer of an optional output of at least n elements of dtype
    ('int32', 'float32' or 'float64'), or None."""
    if t is None:
        return None
    if hasattr(t, "dtype") and str(t.dtype) != f"torch.{dtype}":
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    if hasattr(t, "numel") and t.numel() < n:
        raise ValueError(f"{what}: {t.numel()} elements, need {n}")
    return _ptr(t)


def _gate(cfg, g, n_q: int) -> Optional[int]:
    """Pointer of a gate-logit tensor after checking that it holds what the
    kernels read: fp32, [B, n_q, H] or, with cfg.gate_dims = d, [B, n_q, H, d]."""
    if g is None:
        return None
    per = cfg.head_dim if cfg.gate_dims > 1 else 1
    want = cfg.batch * n_q * cfg.num_heads * per
    if hasattr(g, "numel"):
        if g.numel() != want or str(g.dtype) != "torch.float32":
            raise ValueError(f"gate logits must be {want} fp32 values ([B, n_q, H"
                             f"{', d' if per > 1 else ''}]), got {tuple(g.shape)} {g.dtype}")
    return _ptr(g)


def _elem_dtype(cfg) -> str:
    return "torch.bfloat16" if cfg.dtype == HSA_DTYPE_BF16 else "torch.float32"


def _rows(cfg, t, n_q: int, what: str, fp32: bool = False) -> Optional[int]:
    """Pointer of a [B, n_q, H, d] tensor (queries or outputs) after checking
    its size and element type against the config (the kernels index it with
    these sizes and read or write elements of the config's dtype; fp32 = True
    for the fp32 sparse-branch output)."""
    if t is not None and hasattr(t, "numel"):
        want = cfg.batch * n_q * cfg.num_heads * cfg.head_dim
        if t.numel() != want:
            raise ValueError(f"{what} must hold [B, n_q, H, d] = {want} values, "
                             f"got {tuple(t.shape)}")
        dt = "torch.float32" if fp32 else _elem_dtype(cfg)
        if str(t.dtype) != dt:
            raise ValueError(f"{what} must be {dt}, got {t.dtype}")
    return _ptr(t)


def _stream(stream) -> Optional[int]:
    """A HIP stream handle: an int, a torch stream, or None for torch's
    current stream."""
    if stream is not None:
        return int(getattr(stream, "cuda_stream", stream))
    import torch
    return torch.cuda.current_stream().cuda_stream


def _budgets(k_h: Optional[Sequence[int]]):
    if k_h is None:
        return None, None
    arr = np.ascontiguousarray(np.asarray(k_h, dtype=np.int32))
    return arr, arr.ctypes.data_as(c_vp)


def _check(fn: str, status: int):
    if status != 0:
        raise HsaError(fn, status)


def _workspace(nbytes: int, device):
    import torch
    if nbytes == 0:
        return None
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def config(batch: int, num_heads: int, head_dim: int, page_size: int, dtype,
           sm_scale: float = 0.0, gate_dims: int = 0) -> HsaConfig:
    """gate_dims: 0 for gate logits per (query, head), head_dim for logits per
    (query, head, dim)."""
    if not isinstance(dtype, int):
        dtype = HSA_DTYPE_BF16 if str(dtype).endswith("bfloat16") or dtype == "bf16" else HSA_DTYPE_F32
    return HsaConfig(batch, num_heads, head_dim, page_size, dtype, sm_scale, gate_dims)


def kv_pool(k_pool, v_pool, page_table, cfg: Optional[HsaConfig] = None) -> HsaKvPool:
    """The pool descriptor. With cfg, the tensors are checked against it
    first: k_pool [slots, H, P, d] and v_pool [slots, H, d, P] of the config's
    dtype, page_table [B, max_pages] int32."""
    ks, ps = k_pool.shape, page_table.shape
    if cfg is not None:
        torch = _torch
        if torch is None:  # (the library need not be there)
            import torch
        dt = torch.bfloat16 if cfg.dtype == HSA_DTYPE_BF16 else torch.float32
        H, P, d, slots = cfg.num_heads, cfg.page_size, cfg.head_dim, ks[0]
        for name, t, got, shape in (("k_pool", k_pool, ks, (slots, H, P, d)),
                                    ("v_pool", v_pool, v_pool.shape, (slots, H, d, P))):
            if t.dtype is not dt or got != shape:
                raise ValueError(f"{name} must be {dt} {shape}, got {t.dtype} {tuple(got)}")
        if page_table.dtype is not torch.int32 or len(ps) != 2 or ps[0] != cfg.batch:
            raise ValueError(f"page_table must be int32 [B={cfg.batch}, max_pages], got "
                             f"{page_table.dtype} {tuple(ps)}")
    return HsaKvPool(_ptr(k_pool), _ptr(v_pool), _ptr(page_table), ks[0], ps[-1])


# ------------------------------------------------------------------ C ABI calls
def hsa_state_update_workspace_size(cfg: HsaConfig, n_pages: int) -> int:
    return lib().hsa_state_update_workspace_size(ctypes.byref(cfg), n_pages)


def hsa_page_select_workspace_size(cfg: HsaConfig, n_q: int) -> int:
    return lib().hsa_page_select_workspace_size(ctypes.byref(cfg), n_q)


def hsa_sparse_attn_workspace_size(cfg: HsaConfig, n_q: int, k_max: int, n_cur_pages: int) -> int:
    return lib().hsa_sparse_attn_workspace_size(ctypes.byref(cfg), n_q, k_max, n_cur_pages)


def hsa_forward_workspace_size(cfg: HsaConfig, n_q: int, k_max: int, n_cur_pages: int) -> int:
    return lib().hsa_forward_workspace_size(ctypes.byref(cfg), n_q, k_max, n_cur_pages)


def hsa_adaptive_workspace_size(cfg: HsaConfig, n_q: int, k_max: int, n_cur_pages: int) -> int:
    return lib().hsa_adaptive_workspace_size(ctypes.byref(cfg), n_q, k_max, n_cur_pages)


def hsa_block_count(cfg: HsaConfig, n_hist_pages: int, n_cur_pages: int) -> int:
    return lib().hsa_block_count(ctypes.byref(cfg), n_hist_pages, n_cur_pages)


def hsa_status_string(status: int) -> str:
    return lib().hsa_status_string(status).decode()


def hsa_state_update(cfg, pool, first_page, n_pages, kv_state, k_state, page_kmean,
                     ws=None, stream=None, check=True) -> int:
    if ws is None:
        ws = _workspace(hsa_state_update_workspace_size(cfg, n_pages), kv_state.device)
    st = lib().hsa_state_update(ctypes.byref(cfg), ctypes.byref(pool), first_page, n_pages,
                                _ptr(kv_state), _ptr(k_state), _ptr(page_kmean), _ptr(ws),
                                0 if ws is None else ws.numel(), _stream(stream))
    if check:
        _check("hsa_state_update", st)
    return st


def hsa_page_write(cfg, pool, k_src, v_src, first_page, n_pages, src_of=None, stream=None,
                   check=True) -> int:
    """Append pages: k_src / v_src [B, n_pages * P, H, d] (raster order) into
    the pool slots of logical pages [first_page, first_page + n_pages),
    optionally permuted by src_of (device int32 [P], e.g. from
    hsa_cube_order)."""
    want = cfg.batch * n_pages * cfg.page_size * cfg.num_heads * cfg.head_dim
    for name, t in (("k_src", k_src), ("v_src", v_src)):
        if hasattr(t, "numel") and (t.numel() != want or str(t.dtype) != _elem_dtype(cfg)):
            raise ValueError(f"{name} must hold {want} values of {_elem_dtype(cfg)} "
                             f"([B, n_pages * P, H, d]), got {tuple(t.shape)} {t.dtype}")
    if src_of is not None and hasattr(src_of, "numel"):
        if src_of.numel() != cfg.page_size or str(src_of.dtype) != "torch.int32":
            raise ValueError("src_of must be int32 [P]")
    st = lib().hsa_page_write(ctypes.byref(cfg), ctypes.byref(pool), _ptr(k_src), _ptr(v_src),
                              first_page, n_pages, _ptr(src_of), _stream(stream))
    if check:
        _check("hsa_page_write", st)
    return st


def hsa_cube_order(frames: int, height: int, width: int, cube=(4, 8, 4)):
    """(src_of, whole): src_of[i] = raster index of the token stored at
    position i of a page in cube order (int32 numpy array), and the number of
    positions covered by whole cubes."""
    n = frames * height * width
    out = np.empty(n, np.int32)
    whole = lib().hsa_cube_order(frames, height, width, int(cube[0]), int(cube[1]), int(cube[2]),
                                 out.ctypes.data_as(c_vp))
    if whole < 0:
        raise ValueError("invalid cube order sizes")
    return out, whole


def hsa_page_select(cfg, q, n_q, page_kmean, max_pages, n_cand, k_h, k_max, sel,
                    sel_score=None, ws=None, stream=None, check=True) -> int:
    if ws is None:
        ws = _workspace(hsa_page_select_workspace_size(cfg, n_q), q.device)
    _keep, kp = _budgets(k_h)
    st = lib().hsa_page_select(ctypes.byref(cfg), _rows(cfg, q, n_q, "q"), n_q, _ptr(page_kmean), max_pages,
                               n_cand, kp, k_max, _ptr(sel), _ptr(sel_score), _ptr(ws),
                               0 if ws is None else ws.numel(), _stream(stream))
    if check:
        _check("hsa_page_select", st)
    return st


def hsa_sparse_attn(cfg, q, n_q, pool, sel, k_max, k_h, cur_first_page, n_cur_pages, o_sp,
                    lse=None, ws=None, stream=None, check=True) -> int:
    if ws is None:
        ws = _workspace(hsa_sparse_attn_workspace_size(cfg, n_q, k_max, n_cur_pages), q.device)
    _keep, kp = _budgets(k_h)
    qp, op = _rows(cfg, q, n_q, "q"), _rows(cfg, o_sp, n_q, "o_sp", fp32=True)
    st = lib().hsa_sparse_attn(ctypes.byref(cfg), qp, n_q, ctypes.byref(pool), _ptr(sel),
                               k_max, kp, cur_first_page, n_cur_pages, op, _ptr(lse),
                               _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream))
    if check:
        _check("hsa_sparse_attn", st)
    return st


def hsa_forward(cfg, q, n_q, pool, n_cand, n_cur_pages, k_h, k_max, kv_state, k_state,
                page_kmean, g_lin, g_sp, o, sel_out=None, ws=None, stream=None,
                check=True) -> int:
    if ws is None:
        ws = _workspace(hsa_forward_workspace_size(cfg, n_q, k_max, n_cur_pages), q.device)
    _keep, kp = _budgets(k_h)
    qp, op = _rows(cfg, q, n_q, "q"), _rows(cfg, o, n_q, "o")
    glp, gsp = _gate(cfg, g_lin, n_q), _gate(cfg, g_sp, n_q)
    st = lib().hsa_forward(ctypes.byref(cfg), qp, n_q, ctypes.byref(pool), n_cand,
                           n_cur_pages, kp, k_max, _ptr(kv_state), _ptr(k_state),
                           _ptr(page_kmean), glp, gsp, op, _ptr(sel_out),
                           _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream))
    if check:
        _check("hsa_forward", st)
    return st


def hsa_forward_selected(cfg, q, n_q, pool, sel, k_max, k_h, n_cand, n_cur_pages, kv_state,
                         k_state, g_lin, g_sp, o, ws=None, stream=None, check=True) -> int:
    if ws is None:
        ws = _workspace(hsa_forward_workspace_size(cfg, n_q, k_max, n_cur_pages), q.device)
    _keep, kp = _budgets(k_h)
    qp, op = _rows(cfg, q, n_q, "q"), _rows(cfg, o, n_q, "o")
    glp, gsp = _gate(cfg, g_lin, n_q), _gate(cfg, g_sp, n_q)
    st = lib().hsa_forward_selected(ctypes.byref(cfg), qp, n_q, ctypes.byref(pool), _ptr(sel),
                                    k_max, kp, n_cand, n_cur_pages, _ptr(kv_state), _ptr(k_state),
                                    glp, gsp, op, _ptr(ws),
                                    0 if ws is None else ws.numel(), _stream(stream))
    if check:
        _check("hsa_forward_selected", st)
    return st


def hsa_forward_noalloc_bytes(cfg, n_q, n_cand, n_cur_pages, k_h, k_max) -> int:
    _keep, kp = _budgets(k_h)
    return lib().hsa_forward_noalloc_bytes(ctypes.byref(cfg), n_q, n_cand, n_cur_pages, kp, k_max)


def hsa_forward_noalloc(cfg, q, n_q, pool, n_cand, n_cur_pages, k_h, k_max, kv_state, k_state,
                        page_kmean, g_lin, g_sp, o, sel_out=None, stream=None, check=True) -> int:
    """hsa_forward with the library's static per-GPU workspace (no device
    allocation by the library or by this binding)."""
    _keep, kp = _budgets(k_h)
    qp, op = _rows(cfg, q, n_q, "q"), _rows(cfg, o, n_q, "o")
    glp, gsp = _gate(cfg, g_lin, n_q), _gate(cfg, g_sp, n_q)
    st = lib().hsa_forward_noalloc(ctypes.byref(cfg), qp, n_q, ctypes.byref(pool), n_cand,
                                   n_cur_pages, kp, k_max, _ptr(kv_state), _ptr(k_state),
                                   _ptr(page_kmean), glp, gsp, op, _ptr(sel_out), _stream(stream))
    if check:
        _check("hsa_forward_noalloc", st)
    return st


# Paper's setting of the coverage thresholds (tau_max, tau_min) = (1.00, 0.35).
TAU_MIN, TAU_MAX = 0.35, 1.00
BLOCK_Q = 64  # queries per query block (HSA_BLOCK_Q)


def hsa_block_select(cfg, q, n_q, pool, sel, k_max, cur_first_page, n_cur_pages,
                     tau_min=TAU_MIN, tau_max=TAU_MAX, gini=None, tau=None, n_kept=None,
                     kept=None, pooled=None, kept_len=0, ws=None, stream=None,
                     check=True) -> int:
    if ws is None:
        ws = _workspace(hsa_adaptive_workspace_size(cfg, n_q, k_max, n_cur_pages), q.device)
    bh = cfg.batch * cfg.num_heads
    n_qb = -(-n_q // BLOCK_Q)
    st = lib().hsa_block_select(ctypes.byref(cfg), _rows(cfg, q, n_q, "q"), n_q, ctypes.byref(pool), _ptr(sel),
                                k_max, cur_first_page, n_cur_pages, float(tau_min),
                                float(tau_max), _out(gini, bh, "float64", "gini"),
                                _out(tau, bh, "float64", "tau"),
                                _out(n_kept, bh * n_qb, "int32", "n_kept"),
                                _out(kept, bh * n_qb * kept_len, "int32", "kept"),
                                _out(pooled, bh * n_qb * kept_len, "float64", "pooled"), kept_len,
                                _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream))
    if check:
        _check("hsa_block_select", st)
    return st


def hsa_sparse_attn_adaptive(cfg, q, n_q, pool, sel, k_max, k_h, cur_first_page, n_cur_pages,
                             o_sp, lse=None, tau_min=TAU_MIN, tau_max=TAU_MAX, ws=None,
                             stream=None, check=True) -> int:
    if ws is None:
        ws = _workspace(hsa_adaptive_workspace_size(cfg, n_q, k_max, n_cur_pages), q.device)
    _keep, kp = _budgets(k_h)
    st = lib().hsa_sparse_attn_adaptive(ctypes.byref(cfg), _rows(cfg, q, n_q, "q"), n_q,
                                        ctypes.byref(pool), _ptr(sel), k_max, kp, cur_first_page,
                                        n_cur_pages, float(tau_min), float(tau_max),
                                        _rows(cfg, o_sp, n_q, "o_sp", fp32=True), _ptr(lse),
                                        _ptr(ws), 0 if ws is None else ws.numel(),
                                        _stream(stream))
    if check:
        _check("hsa_sparse_attn_adaptive", st)
    return st


def hsa_forward_adaptive(cfg, q, n_q, pool, n_cand, n_cur_pages, k_h, k_max, kv_state, k_state,
                         page_kmean, g_lin, g_sp, o, tau_min=TAU_MIN, tau_max=TAU_MAX,
                         sel_out=None, ws=None, stream=None, check=True) -> int:
    if ws is None:
        ws = _workspace(hsa_adaptive_workspace_size(cfg, n_q, k_max, n_cur_pages), q.device)
    _keep, kp = _budgets(k_h)
    qp, op = _rows(cfg, q, n_q, "q"), _rows(cfg, o, n_q, "o")
    glp, gsp = _gate(cfg, g_lin, n_q), _gate(cfg, g_sp, n_q)
    st = lib().hsa_forward_adaptive(ctypes.byref(cfg), qp, n_q, ctypes.byref(pool), n_cand,
                                    n_cur_pages, kp, k_max, float(tau_min), float(tau_max),
                                    _ptr(kv_state), _ptr(k_state), _ptr(page_kmean), glp,
                                    gsp, op, _ptr(sel_out), _ptr(ws),
                                    0 if ws is None else ws.numel(), _stream(stream))
    if check:
        _check("hsa_forward_adaptive", st)
    return st


def hsa_linformer_compress_workspace_size(cfg: HsaConfig, rank: int, n_pages: int) -> int:
    return lib().hsa_linformer_compress_workspace_size(ctypes.byref(cfg), rank, n_pages)


def hsa_linformer_workspace_size(cfg: HsaConfig, n_q: int, k_max: int, n_cur_pages: int) -> int:
    return lib().hsa_linformer_workspace_size(ctypes.byref(cfg), n_q, k_max, n_cur_pages)


def hsa_linformer_compress(cfg, pool, e_k, e_v, rank, first_page, n_pages, ck, cv, ws=None,
                           stream=None, check=True) -> int:
    if ws is None:
        ws = _workspace(hsa_linformer_compress_workspace_size(cfg, rank, n_pages), ck.device)
    st = lib().hsa_linformer_compress(ctypes.byref(cfg), ctypes.byref(pool), _ptr(e_k), _ptr(e_v),
                                      rank, first_page, n_pages, _ptr(ck), _ptr(cv), _ptr(ws),
                                      0 if ws is None else ws.numel(), _stream(stream))
    if check:
        _check("hsa_linformer_compress", st)
    return st


def hsa_forward_linformer(cfg, q, n_q, pool, ck, cv, rank, n_cand, n_cur_pages, k_h, k_max,
                          page_kmean, g_lin, g_sp, o, tau_min=TAU_MIN, tau_max=TAU_MAX,
                          sel_out=None, ws=None, stream=None, check=True) -> int:
    if ws is None:
        ws = _workspace(hsa_linformer_workspace_size(cfg, n_q, k_max, n_cur_pages), q.device)
    _keep, kp = _budgets(k_h)
    qp, op = _rows(cfg, q, n_q, "q"), _rows(cfg, o, n_q, "o")
    glp, gsp = _gate(cfg, g_lin, n_q), _gate(cfg, g_sp, n_q)
    st = lib().hsa_forward_linformer(ctypes.byref(cfg), qp, n_q, ctypes.byref(pool), _ptr(ck),
                                     _ptr(cv), rank, n_cand, n_cur_pages, kp, k_max,
                                     float(tau_min), float(tau_max), _ptr(page_kmean), glp,
                                     gsp, op, _ptr(sel_out), _ptr(ws),
                                     0 if ws is None else ws.numel(), _stream(stream))
    if check:
        _check("hsa_forward_linformer", st)
    return st


def hsa_retrieval_workspace_size(cfg: HsaConfig, n_q: int, k_max: int, n_cur_pages: int) -> int:
    return lib().hsa_retrieval_workspace_size(ctypes.byref(cfg), n_q, k_max, n_cur_pages)


def hsa_chunk_select(cfg, prompt_emb, chunk_emb, emb_dim, n_chunks, chunk_first, n_cand,
                     cand_range, chunk_out=None, chunk_score=None, stream=None,
                     check=True) -> int:
    st = lib().hsa_chunk_select(ctypes.byref(cfg), _ptr(prompt_emb), _ptr(chunk_emb), emb_dim,
                                n_chunks, _ptr(chunk_first), n_cand, _ptr(chunk_out),
                                _ptr(chunk_score), _ptr(cand_range), _stream(stream))
    if check:
        _check("hsa_chunk_select", st)
    return st


def hsa_forward_retrieval(cfg, q, n_q, pool, prompt_emb, chunk_emb, emb_dim, n_chunks,
                          chunk_first, n_cand, n_cur_pages, k_h, k_max, kv_state, k_state,
                          page_kmean, g_lin, g_sp, o, chunk_out=None, sel_out=None, ws=None,
                          stream=None, check=True) -> int:
    if ws is None:
        ws = _workspace(hsa_retrieval_workspace_size(cfg, n_q, k_max, n_cur_pages), q.device)
    _keep, kp = _budgets(k_h)
    qp, op = _rows(cfg, q, n_q, "q"), _rows(cfg, o, n_q, "o")
    glp, gsp = _gate(cfg, g_lin, n_q), _gate(cfg, g_sp, n_q)
    st = lib().hsa_forward_retrieval(ctypes.byref(cfg), qp, n_q, ctypes.byref(pool),
                                     _ptr(prompt_emb), _ptr(chunk_emb), emb_dim, n_chunks,
                                     _ptr(chunk_first), n_cand, n_cur_pages, kp, k_max,
                                     _ptr(kv_state), _ptr(k_state), _ptr(page_kmean), glp,
                                     gsp, op, _ptr(chunk_out), _ptr(sel_out), _ptr(ws),
                                     0 if ws is None else ws.numel(), _stream(stream))
    if check:
        _check("hsa_forward_retrieval", st)
    return st


# ------------------------------------------------------------------ rotary positions, tokens, 8-bit cache
CACHE8_BLOCK = 64  # tokens of a page that share a scale (HSA_CACHE8_BLOCK)
_LAYOUTS = {"half": 0, "interleaved": 1}
_SCALINGS = {"none": 0, "linear": 1, "parts": 2}


def rope(rot_dim: int, layout: str = "half", theta: float = 10000.0, axis_dims: Optional[Sequence[int]] = None,
         scaling: str = "none", factor: float = 1.0, low: float = 1.0, high: float = 32.0, orig_len: int = 0,
         amplitude: float = 1.0) -> HsaRope:
    """Rotary positions (hsa_rope_t of include/hsa.h): the first rot_dim dims of
    a head in pairs (i, i + rot_dim/2) ("half") or (2i, 2i+1) ("interleaved").
    axis_dims: dims of each of 2 or 3 position axes. scaling: "none", "linear"
    (every frequency / factor) or "parts" (only those that turn fewer than `high`
    times over orig_len, wholly below `low`). amplitude multiplies the result."""
    if layout not in _LAYOUTS or scaling not in _SCALINGS:
        raise ValueError(f"unknown layout {layout!r} or scaling {scaling!r}")
    dims = [int(x) for x in axis_dims] if axis_dims is not None else [int(rot_dim)]
    if not 1 <= len(dims) <= 3 or sum(dims) != rot_dim:
        raise ValueError(f"axis_dims {dims} must be 1 to 3 numbers that sum to rot_dim = {rot_dim}")
    return HsaRope(rot_dim, _LAYOUTS[layout], len(dims), (c_i32 * 3)(*(dims + [0, 0])[:3]), _SCALINGS[scaling],
                   orig_len, theta, factor, low, high, amplitude)


def cache8_pool(k, v, k_exp, v_exp, page_table, cfg: HsaConfig) -> HsaCache8Pool:
    """The 8-bit cache's descriptor after checking its tensors: k [slots, Hk, P, d],
    v [slots, Hk, d, P], k_exp and v_exp [slots, Hk, ceil(P / 64)] uint8,
    page_table [B, max_pages] int32."""
    slots, kv = int(k.shape[0]), int(k.shape[1])
    P, d = cfg.page_size, cfg.head_dim
    nb = -(-P // CACHE8_BLOCK)
    for name, t, shape in (("k", k, (slots, kv, P, d)), ("v", v, (slots, kv, d, P)),
                           ("k_exp", k_exp, (slots, kv, nb)), ("v_exp", v_exp, (slots, kv, nb))):
        if tuple(t.shape) != shape or str(t.dtype) != "torch.uint8":
            raise ValueError(f"{name} must be torch.uint8 {shape}, got {t.dtype} {tuple(t.shape)}")
    if page_table.dim() != 2 or page_table.shape[0] != cfg.batch or str(page_table.dtype) != "torch.int32":
        raise ValueError(f"page_table must be int32 [B={cfg.batch}, max_pages], got "
                         f"{page_table.dtype} {tuple(page_table.shape)}")
    return HsaCache8Pool(_ptr(k), _ptr(v), _ptr(k_exp), _ptr(v_exp), _ptr(page_table), slots,
                         int(page_table.shape[-1]), kv)


# The calls below may serve a single token, where the host's time counts: their checks
# compare types, shapes and devices without building strings or objects. Each takes the
# library first (lib()), which sets _torch.
def _i32s(t, n: int, dev: int, what: str) -> Optional[int]:
    """Address of a contiguous int32 tensor of n elements on device dev, or None."""
    if t is None:
        return None
    if t.dtype is not _torch.int32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what} must hold {n} contiguous int32 values, got {tuple(t.shape)} {t.dtype}")
    if t.get_device() != dev:
        raise ValueError(f"{what} is on {t.device}, not on the call's device")
    return t.data_ptr()


def _strided(shape, dtype, t, what: str):
    """(batch stride, token stride, device) of a [B, n, heads, d] tensor whose heads
    are contiguous within a token."""
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{what} must be {dtype} {shape}, got {t.dtype} {tuple(t.shape)}")
    sb, st, sh, sd = t.stride()
    if (sd != 1 or sh != shape[3]) and (sd != 1 or shape[2] > 1) and t.numel():
        raise ValueError(f"{what}: the heads of a token must be contiguous, got strides {t.stride()}")
    return sb, st, t.get_device()


def _elem(cfg):
    return _torch.bfloat16 if cfg.dtype == HSA_DTYPE_BF16 else _torch.float32


def _apart(what: str, t):
    return ValueError(f"{what} is on {t.device}, not on the call's device")


def _call(fn, dev: int, stream, *args) -> int:
    """fn(*args, stream) with the tensors' device current (kernels launch there)."""
    if dev < 0:
        raise ValueError("the tensors must be on a GPU")
    if dev != _torch.cuda.current_device():
        with _torch.cuda.device(dev):
            return fn(*args, raw_stream(dev, stream))
    return fn(*args, raw_stream(dev, stream))


def raw_stream(dev: int, stream) -> int:
    """The handle of stream (None: the current one of device dev)."""
    if stream is not None:
        return int(getattr(stream, "cuda_stream", stream))
    return _torch._C._cuda_getCurrentRawStream(dev)


def _empty(shape, dtype, device, stream):
    """An uninitialised tensor that a launch on stream (None: the current one) may write at
    once. It comes from that stream's memory: a block of the current stream's may still be in use by
    what is queued there, and the launch does not wait for that."""
    if stream is None:
        return _torch.empty(shape, dtype=dtype, device=device)
    with _torch.cuda.stream(_torch_stream(stream, device)):
        return _torch.empty(shape, dtype=dtype, device=device)


def _torch_stream(stream, device):
    if isinstance(stream, _torch.cuda.Stream):
        return stream
    return _torch.cuda.ExternalStream(int(getattr(stream, "cuda_stream", stream)), device=device)


def used_on(stream, *tensors):
    """Tensors of a GPU that calls on stream (None: the current one) read or write and that may be let go before those
    have run: their memory then waits for the stream."""
    device = tensors[0].device
    on = _torch.cuda.current_stream(device) if stream is None else _torch_stream(stream, device)
    for t in tensors:
        t.record_stream(on)


def empty_of(nbytes, device, stream):
    """Memory of stream (None: the current one), and whether the stream is being captured."""
    with _torch.cuda.stream(None if stream is None else _torch_stream(stream, device)), _torch.cuda.device(device):
        return _torch.empty(nbytes, dtype=_torch.uint8, device=device), _torch.cuda.is_current_stream_capturing()


def empty_on(shape, dtype, device, stream=None):
    """An uninitialised tensor that a call on stream writes, to be read on the current stream (once that waits
    for the call)."""
    lib()
    if stream is None or _torch.device(device).type != "cuda":
        return _torch.empty(shape, dtype=dtype, device=device)
    t = _empty(shape, dtype, device, stream)
    t.record_stream(_torch.cuda.current_stream(device))  # not written anew before its reader is done
    return t


def out_like(t, stream=None):
    """A contiguous output of t's shape, type and device for a call on stream, to be read on the
    current stream (once that waits for the call)."""
    return empty_on(t.shape, t.dtype, t.device, stream)


def hsa_rope_apply(cfg, rope, x, n, o, pos=None, first=None, inverse=False, stream=None,
                   check=True) -> int:
    """Turns x [B, n, heads, d] by its tokens' positions (pos int32 [B, n, axes], or
    first int32 [B] + the token's index) into o (x itself, or apart from it).
    inverse: by the opposite angles, the gradient's map. No autograd graph is
    recorded (HsaCache8.rotate records one)."""
    fn = lib().hsa_rope_apply
    B = cfg.batch
    heads = x.shape[2] if x.dim() == 4 else 0
    shape, dtype = (B, n, heads, cfg.head_dim), _elem(cfg)
    xb, xt, dev = _strided(shape, dtype, x, "x")
    ob, ot, at = _strided(shape, dtype, o, "o")
    if at != dev:
        raise _apart("o", o)
    st = _call(fn, dev, stream, ctypes.byref(cfg), ctypes.byref(rope), x.data_ptr(), xb, xt, n, heads,
               None if pos is None else _i32s(pos, B * n * rope.axes, dev, "pos"),
               None if first is None else _i32s(first, B, dev, "first"), 1 if inverse else 0, o.data_ptr(), ob, ot)
    if check and st:
        _check("hsa_rope_apply", st)
    return st


def _token_write(name, fn, cfg, pool, heads, k_src, v_src, n, rope, pos, first, count, stream, check) -> int:
    B = cfg.batch
    shape, dtype = (B, n, heads, cfg.head_dim), _elem(cfg)
    kb, kt, dev = _strided(shape, dtype, k_src, "k_src")
    vb, vt, at = _strided(shape, dtype, v_src, "v_src")
    if at != dev:
        raise _apart("v_src", v_src)
    st = _call(fn, dev, stream, ctypes.byref(cfg), ctypes.byref(pool),
               None if rope is None else ctypes.byref(rope), k_src.data_ptr(), kb, kt, v_src.data_ptr(), vb, vt, n,
               None if rope is None or pos is None else _i32s(pos, B * n * rope.axes, dev, "pos"),
               None if first is None else _i32s(first, B, dev, "first"),
               None if count is None else _i32s(count, B, dev, "count"))
    if check and st:
        _check(name, st)
    return st


def hsa_token_write(cfg, pool, k_src, v_src, n, first=None, count=None, rope=None, pos=None, stream=None,
                    check=True) -> int:
    """Append tokens: k_src / v_src [B, n, H, d] become tokens first[b] + i, i <
    count[b], of each sequence in the pool, keys turned by rope on the way."""
    return _token_write("hsa_token_write", lib().hsa_token_write, cfg, pool, cfg.num_heads, k_src, v_src, n, rope,
                        pos, first, count, stream, check)


def hsa_cache8_write(cfg, cache, k_src, v_src, n, first=None, count=None, rope=None, pos=None, stream=None,
                     check=True) -> int:
    """hsa_token_write into the 8-bit cache: k_src / v_src [B, n, kv_heads, d]."""
    return _token_write("hsa_cache8_write", lib().hsa_cache8_write, cfg, cache, cache.kv_heads, k_src, v_src, n,
                        rope, pos, first, count, stream, check)


def hsa_cache8_attn_workspace_size(cfg: HsaConfig, n_q: int, kv_heads: int, k_max: int, n_cur_pages: int) -> int:
    return lib().hsa_cache8_attn_workspace_size(ctypes.byref(cfg), n_q, kv_heads, k_max, n_cur_pages)


def hsa_cache8_attn_plan(cfg: HsaConfig, n_q: int, kv_heads: int, k_max: int, n_cur_pages: int, ragged: bool = False):
    """(many_rows, rows_per_item, n_pieces) of such a call's launch, without making it; ragged: it has kv_len."""
    out = (c_i32 * 3)()
    at = ctypes.addressof(out)
    _check("hsa_cache8_attn_plan", lib().hsa_cache8_attn_plan(ctypes.byref(cfg), n_q, kv_heads, k_max, n_cur_pages,
                                                              1 if ragged else 0, at, at + 4, at + 8))
    return bool(out[0]), out[1], out[2]


def _paged_attn(name, fn, size, cfg, q, n_q, pages, kv_heads, sel, k_max, k_h, cur_first_page, n_cur_pages, o, lse,
                kv_len, q_len, how, how_name, ws, stream, check, lead=()) -> int:
    """What the attention calls over paged tokens share; how: the last argument before the outputs, a
    flag or (how_name) an int32 tensor or None."""
    B, H, dtype = cfg.batch, cfg.num_heads, _elem(cfg)
    shape = (B, n_q, H, cfg.head_dim)
    for t, what in ((q, "q"), (o, "o")):
        if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{what} must be contiguous {dtype} {shape}, got {t.dtype} {tuple(t.shape)}")
    dev = q.get_device()
    if o.get_device() != dev:
        raise _apart("o", o)
    lp = kp = keep = None
    if lse is not None:
        if lse.dtype is not _torch.float32 or lse.shape != (B, H, n_q) or not lse.is_contiguous():
            raise ValueError(f"lse must be contiguous float32 {(B, H, n_q)}, got {lse.dtype} {tuple(lse.shape)}")
        if lse.get_device() != dev:
            raise _apart("lse", lse)
        lp = lse.data_ptr()
    if k_h is not None:
        if len(k_h) != kv_heads:
            raise ValueError(f"k_h must hold {kv_heads} budgets, got {len(k_h)}")
        keep = (c_i32 * len(k_h))(*[int(k) for k in k_h])
        kp = ctypes.addressof(keep)
    sp = None if sel is None else _i32s(sel, B * kv_heads * k_max, dev, "sel")
    kvp = None if kv_len is None else _i32s(kv_len, B, dev, "kv_len")
    qlp = None if q_len is None else _i32s(q_len, B, dev, "q_len")
    if how_name is not None and how is not None:
        how = _i32s(how, B * n_q * -(-n_q // 32), dev, how_name)
    cp, hp = ctypes.byref(cfg), ctypes.byref(pages)
    if ws is None:
        wp, nbytes = None, size(cp, n_q, kv_heads, k_max, n_cur_pages)
        if nbytes:
            ws = _empty(nbytes, _torch.uint8, q.device, stream if dev >= 0 else None)
            wp = ws.data_ptr()
    else:
        if ws.get_device() != dev:
            raise _apart("ws", ws)
        wp, nbytes = _ptr(ws), ws.numel() * ws.element_size()
    st = _call(fn, dev, stream, cp, q.data_ptr(), n_q, hp, *lead, sp, k_max, kp, cur_first_page, n_cur_pages, kvp, qlp,
               how, o.data_ptr(), lp, wp, nbytes)
    del keep
    if check and st:
        _check(name, st)
    return st


def hsa_cache8_attn(cfg, q, n_q, cache, sel, k_max, k_h, cur_first_page, n_cur_pages, o, lse=None, kv_len=None,
                    q_len=None, causal=False, ws=None, stream=None, check=True) -> int:
    """Attention of q [B, n_q, H, d] over the 8-bit cache's listed pages: sel int32 [B,
    kv_heads, k_max], then [cur_first_page, + n_cur_pages); tokens below kv_len[b]."""
    L = lib()
    return _paged_attn("hsa_cache8_attn", L.hsa_cache8_attn, L.hsa_cache8_attn_workspace_size, cfg, q, n_q, cache,
                       cache.kv_heads, sel, k_max, k_h, cur_first_page, n_cur_pages, o, lse, kv_len, q_len,
                       1 if causal else 0, None, ws, stream, check)


# ------------------------------------------------------------------ drafted trees
def hsa_tree_mask(cfg, parent, n, mask, pos=None, count=None, first=None, stream=None, check=True) -> int:
    """The ancestors of every node as bits, mask int32 [B, n, ceil(n / 32)], from parent int32 [B, n] (a
    smaller node, or -1 for a root), and pos int32 [B, n] = first[b] + depth; nodes at or past
    count[b] are left out."""
    L = lib()
    B, dev = cfg.batch, parent.get_device()
    st = _call(L.hsa_tree_mask, dev, stream, ctypes.byref(cfg), _i32s(parent, B * n, dev, "parent"), n,
               _i32s(count, B, dev, "count"), _i32s(first, B, dev, "first"),
               _i32s(mask, B * n * -(-n // 32), dev, "mask"), _i32s(pos, B * n, dev, "pos"))
    if check and st:
        _check("hsa_tree_mask", st)
    return st


def hsa_tree_attn_workspace_size(cfg: HsaConfig, n_q: int, kv_heads: int, k_max: int, n_cur_pages: int) -> int:
    return lib().hsa_tree_attn_workspace_size(ctypes.byref(cfg), n_q, kv_heads, k_max, n_cur_pages)


def hsa_cache8_tree_attn_workspace_size(cfg: HsaConfig, n_q: int, kv_heads: int, k_max: int, n_cur_pages: int) -> int:
    return lib().hsa_cache8_tree_attn_workspace_size(ctypes.byref(cfg), n_q, kv_heads, k_max, n_cur_pages)


def hsa_tree_attn(cfg, q, n_q, pool, kv_heads, sel, k_max, k_h, cur_first_page, n_cur_pages, o, lse=None, mask=None,
                  kv_len=None, q_len=None, ws=None, stream=None, check=True) -> int:
    """Attention of a step's nodes q [B, n_q, H, d] over the pool's listed pages (kv_heads heads): tokens
    before kv_len[b] - q_len[b], and of the q_len[b] after them those of the node's mask bits (mask
    None: those up to the node itself)."""
    L = lib()
    return _paged_attn("hsa_tree_attn", L.hsa_tree_attn, L.hsa_tree_attn_workspace_size, cfg, q, n_q, pool, kv_heads,
                       sel, k_max, k_h, cur_first_page, n_cur_pages, o, lse, kv_len, q_len, mask, "mask", ws, stream,
                       check, (kv_heads,))


def hsa_cache8_tree_attn(cfg, q, n_q, cache, sel, k_max, k_h, cur_first_page, n_cur_pages, o, lse=None, mask=None,
                         kv_len=None, q_len=None, ws=None, stream=None, check=True) -> int:
    """hsa_tree_attn over the 8-bit cache."""
    L = lib()
    return _paged_attn("hsa_cache8_tree_attn", L.hsa_cache8_tree_attn, L.hsa_cache8_tree_attn_workspace_size, cfg, q,
                       n_q, cache, cache.kv_heads, sel, k_max, k_h, cur_first_page, n_cur_pages, o, lse, kv_len,
                       q_len, mask, "mask", ws, stream, check)


def _pages_call(name, fn, cfg, pages, stream, check, *args) -> int:
    st = _call(fn, args[0].get_device(), stream, ctypes.byref(cfg), ctypes.byref(pages), *args[1:])
    if check and st:
        _check(name, st)
    return st


def _keep(name, fn, cfg, pages, first, index, n, count, stream, check) -> int:
    B, dev = cfg.batch, index.get_device()
    return _pages_call(name, fn, cfg, pages, stream, check, index, _i32s(first, B, dev, "first"),
                       _i32s(index, B * n, dev, "index"), n, _i32s(count, B, dev, "count"))


def hsa_token_keep(cfg, pool, first, index, n, count=None, stream=None, check=True) -> int:
    """Token first[b] + i of the pool takes what token first[b] + index[b][i] holds, i < count[b], all
    read before any is written (index int32 [B, n])."""
    return _keep("hsa_token_keep", lib().hsa_token_keep, cfg, pool, first, index, n, count, stream, check)


def hsa_cache8_keep(cfg, cache, first, index, n, count=None, stream=None, check=True) -> int:
    """hsa_token_keep in the 8-bit cache."""
    return _keep("hsa_cache8_keep", lib().hsa_cache8_keep, cfg, cache, first, index, n, count, stream, check)


# ------------------------------------------------------------------ pages
def hsa_page_copy(cfg, pool, moves, n, stream=None, check=True) -> int:
    """Copies pages between the pool's slots: moves int32 [n, 3], rows {from, to, tokens}."""
    L = lib()
    return _pages_call("hsa_page_copy", L.hsa_page_copy, cfg, pool, stream, check, moves,
                       _i32s(moves, 3 * n, moves.get_device(), "moves"), n)


def hsa_cache8_page_copy(cfg, cache, moves, n, stream=None, check=True) -> int:
    """hsa_page_copy in the 8-bit cache."""
    L = lib()
    return _pages_call("hsa_cache8_page_copy", L.hsa_cache8_page_copy, cfg, cache, stream, check, moves,
                       _i32s(moves, 3 * n, moves.get_device(), "moves"), n)


def whole_pages(moves, page_size: int, stream=None):
    """The moves with whole pages of page_size rows for those that copy any token."""
    with _torch.cuda.stream(None if stream is None else _torch_stream(stream, moves.device)):
        whole = moves.clone()
        whole[:, 2].clamp_(0, 1).mul_(page_size)
        return whole


def slot_table(page_table, refs, cfg: HsaConfig) -> HsaSlotTable:
    """The descriptor of a page table (int32 [B, max_pages]) and its slots' counts (int32 [num_slots])."""
    if page_table.dim() != 2 or page_table.shape[0] != cfg.batch or str(page_table.dtype) != "torch.int32":
        raise ValueError(f"page_table must be int32 [B={cfg.batch}, max_pages], got "
                         f"{page_table.dtype} {tuple(page_table.shape)}")
    if refs.dim() != 1 or str(refs.dtype) != "torch.int32":
        raise ValueError(f"refs must be int32 [num_slots], got {refs.dtype} {tuple(refs.shape)}")
    return HsaSlotTable(_ptr(page_table), _ptr(refs), int(refs.shape[0]), int(page_table.shape[1]))


def hsa_slots_workspace_size(cfg: HsaConfig, num_slots: int, max_pages: int) -> int:
    return lib().hsa_slots_workspace_size(ctypes.byref(cfg), num_slots, max_pages)


def _slots_ws(cfg, slots, ws, like, stream):
    """Address and size of the workspace of a slot call (one of its own where ws is None), and its tensor."""
    if ws is None:
        n = hsa_slots_workspace_size(cfg, slots.num_slots, slots.max_pages)
        ws = _empty(n, _torch.uint8, like.device, stream if like.is_cuda else None)
    elif ws.get_device() != like.get_device():
        raise _apart("ws", ws)
    return _ptr(ws), ws.numel() * ws.element_size(), ws


def hsa_slots_take(cfg, slots, first, end, moves=None, missing=None, ws=None, stream=None, check=True) -> int:
    """Makes the pages of tokens [first[b], end[b]) the rows' own; moves int32 [B, 3] for hsa_page_copy,
    missing int32 [1]: entries that found no free slot."""
    L = lib()
    B, dev = cfg.batch, end.get_device()
    f, e = _i32s(first, B, dev, "first"), _i32s(end, B, dev, "end")
    m, x = _i32s(moves, 3 * B, dev, "moves"), _i32s(missing, 1, dev, "missing")
    wp, nbytes, ws = _slots_ws(cfg, slots, ws, end, stream)
    return _pages_call("hsa_slots_take", L.hsa_slots_take, cfg, slots, stream, check, end, f, e, m, x, wp, nbytes)


def hsa_slots_fork(cfg, slots, parent, ws=None, stream=None, check=True) -> int:
    """Row b of the page table becomes what row parent[b] was, sharing its slots."""
    L = lib()
    at = _i32s(parent, cfg.batch, parent.get_device(), "parent")
    wp, nbytes, ws = _slots_ws(cfg, slots, ws, parent, stream)
    return _pages_call("hsa_slots_fork", L.hsa_slots_fork, cfg, slots, stream, check, parent, at, wp, nbytes)


def hsa_slots_free(cfg, slots, keep, stream=None, check=True) -> int:
    """Row b lets go of its pages behind its first keep[b] tokens."""
    return _pages_call("hsa_slots_free", lib().hsa_slots_free, cfg, slots, stream, check, keep,
                       _i32s(keep, cfg.batch, keep.get_device(), "keep"))


def hsa_slots_compact(cfg, slots, moves, n_moves, table_out=None, refs_out=None, ws=None, stream=None,
                      check=True) -> int:
    """Moves the slots in use to the front of the pool (moves int32 [n_moves, 3] for hsa_page_copy)."""
    L = lib()
    dev = moves.get_device()
    m = _i32s(moves, 3 * n_moves, dev, "moves")
    t = _i32s(table_out, cfg.batch * slots.max_pages, dev, "table_out")
    r = _i32s(refs_out, slots.num_slots, dev, "refs_out")
    wp, nbytes, ws = _slots_ws(cfg, slots, ws, moves, stream)
    return _pages_call("hsa_slots_compact", L.hsa_slots_compact, cfg, slots, stream, check, moves, m, n_moves, t, r, wp, nbytes)


class HsaTier:
    """Host-managed tiers of a layer's KV pool (include/hsa.h, hsa_tier_*):
    logical pages live in the pool's slots (L1), in pinned host slots (L2) or
    in slots of an unnamed file under ``l3_dir`` (L3). ``pool`` None makes a
    plan-only tier (bookkeeping without copies). ``backup`` keeps a copy of
    every page in the file (``commit`` writes new pages, ``drop`` releases
    the pool and host copies)."""

    def __init__(self, cfg: HsaConfig, pool: Optional[HsaKvPool], l2_slots: int, host_k=None,
                 host_v=None, num_slots: int = 0, max_pages: int = 0, l3_dir: Optional[str] = None,
                 l3_slots: int = 0, backup: bool = False):
        if pool is None:
            pool = HsaKvPool(None, None, None, num_slots, max_pages)
        self._keep = (cfg, pool, host_k, host_v)
        h = c_vp()
        _check("hsa_tier_create", lib().hsa_tier_create(
            ctypes.byref(cfg), ctypes.byref(pool), _ptr(host_k), _ptr(host_v), l2_slots,
            None if l3_dir is None else str(l3_dir).encode(), l3_slots, int(bool(backup)),
            ctypes.byref(h)))
        self._h = h

    def close(self):
        if self._h:
            lib().hsa_tier_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _stream(self, stream):
        return None if self._keep[1].k is None else _stream(stream)

    def place(self, b: int, page: int, stream=None, check=True):
        slot = c_i32(-1)
        st = lib().hsa_tier_place(self._h, b, page, ctypes.byref(slot), self._stream(stream))
        if check:
            _check("hsa_tier_place", st)
            return slot.value
        return st, slot.value

    def _move(self, fn, pages, stream, check):
        arr = np.ascontiguousarray(np.asarray(pages, dtype=np.int32))
        n = arr.shape[-1] if arr.ndim else 0
        st = getattr(lib(), fn)(self._h, arr.ctypes.data_as(c_vp), n, self._stream(stream))
        if check:
            _check(fn, st)
        return st

    def fetch(self, pages, stream=None, check=True) -> int:
        return self._move("hsa_tier_fetch", pages, stream, check)

    def prefetch(self, pages, stream=None, check=True) -> int:
        return self._move("hsa_tier_prefetch", pages, stream, check)

    def commit(self, stream=None, check=True) -> int:
        st = lib().hsa_tier_commit(self._h, self._stream(stream))
        if check:
            _check("hsa_tier_commit", st)
        return st

    def drop(self, stream=None, check=True) -> int:
        st = lib().hsa_tier_drop(self._h, self._stream(stream))
        if check:
            _check("hsa_tier_drop", st)
        return st

    def locate(self, b: int, page: int) -> int:
        return lib().hsa_tier_locate(self._h, b, page)

    def stats(self) -> dict:
        s = HsaTierStats()
        lib().hsa_tier_stats(self._h, ctypes.byref(s))
        return {k: getattr(s, k) for k, _ in HsaTierStats._fields_}

    def counters(self):
        """(pages moved out of the pool, pages brought into it)."""
        s = self.stats()
        return s["evictions"], s["fetches"]
