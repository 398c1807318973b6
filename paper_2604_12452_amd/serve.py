"""Binding of the serving operators (include/lca_serve.h): ragged batches over a paged 8-bit cache, and packed prompts.  As in ``lca``:
argument marshalling only (in native code, binding/bind.cpp, for plain descriptors and tensors, here for the others), torch provides device memory and
streams, every step runs in the library's HIP kernels.
"""
from __future__ import annotations

import ctypes
import warnings
from dataclasses import dataclass
from functools import lru_cache
from operator import index

from . import lca

EXPORTS = ("lca_serve_workspace_size", "lca_page_tables", "lca_page_release", "lca_page_store_q8", "lca_page_attn_q8", "lca_packed_attn")

_INTS = ("B", "T", "H", "S", "d_pool", "d_sel", "dtype", "page", "n_blocks", "max_blocks", "max_q", "max_kv", "window")
_ROWS = ("q_row", "sel_row", "pool_row")


class _CDesc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in _INTS] + [("scale", ctypes.c_float), ("softcap", ctypes.c_float)] + [(n, ctypes.c_int64) for n in _ROWS])


@dataclass
class Desc:
    """Mirror of ``lca_serve_desc``; the fields a call does not read may keep their defaults."""
    B: int
    T: int
    H: int
    S: int
    d_pool: int
    d_sel: int
    dtype: int = lca.BF16
    page: int = 16
    n_blocks: int = 0
    max_blocks: int = 0
    max_q: int = 0
    max_kv: int = 0
    window: int = 0
    scale: float = 1.0
    softcap: float = 0.0
    q_row: int = 0
    sel_row: int = 0
    pool_row: int = 0

    def _key(self):
        return tuple(index(getattr(self, n)) for n in _INTS) + (float(self.scale), float(self.softcap)) + tuple(index(getattr(self, n)) for n in _ROWS)


@lru_cache(maxsize=256, typed=True)
def _c_desc(*key):
    """The C structure of a descriptor's field values: shared by later calls with equal values and only ever read."""
    return _CDesc(*key)


_lib = None
_bind = None            # the native marshalling, as in lca.py


def load() -> ctypes.CDLL:
    """The library, with these entry points' argument types declared."""
    global _lib, _bind
    if _lib is None:
        lib = lca.load()
        p, n = ctypes.c_void_p, ctypes.c_size_t
        for name, args in {"lca_serve_workspace_size": [p, p], "lca_page_tables": [p] * 12 + [p, n, p], "lca_page_release": [p] * 7,
                           "lca_page_store_q8": [p] * 8, "lca_page_attn_q8": [p] * 12 + [p, n, p], "lca_packed_attn": [p] * 9 + [p, n, p]}.items():
            f = getattr(lib, name)
            f.restype, f.argtypes = ctypes.c_int, args
        _lib = lib
        if lca._bind is not None:
            _load_bind(lib, lca._bind)
    return _lib


def _load_bind(lib, bind) -> None:
    """The native marshalling of these calls, where lca has it; everything works without it."""
    global _bind
    try:
        import torch
        bind.setup_serve(Desc, {name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in EXPORTS},
                         getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device))
        _bind = bind
    except Exception as e:
        warnings.warn(f"{lca.BIND_PATH} is not used by serve, its calls are marshalled in Python: {e}", RuntimeWarning)


def workspace_size(desc: Desc) -> int:
    n = ctypes.c_size_t(0)
    lca._check(load().lca_serve_workspace_size(ctypes.byref(_c_desc(*desc._key())), ctypes.byref(n)))
    return int(n.value)


def alloc_workspace(desc: Desc, device="cuda"):
    import torch
    return torch.empty(max(workspace_size(desc), 256), dtype=torch.uint8, device=device)


def alloc_cache(desc: Desc, device="cuda"):
    """A pool's buffers: (sel_q8, pool_q8, scales), of zeros."""
    import torch
    u8 = dict(dtype=torch.uint8, device=device)
    return (torch.zeros((desc.n_blocks, desc.S, desc.page, desc.d_sel), **u8), torch.zeros((desc.n_blocks, desc.S, desc.page // 16, desc.d_pool, 16), **u8),
            torch.zeros((desc.n_blocks, desc.S, 2), dtype=torch.float32, device=device))


def _same_device(**tensors):
    """Every tensor on the current device: the library launches there, whatever the tensors say."""
    here = None
    for name, t in tensors.items():
        if t is None or isinstance(t, int) or not t.is_cuda:          # (_ptr refuses what is on no device)
            continue
        if here is None:
            import torch
            here = torch.cuda.current_device()
        if t.device.index != here:
            raise ValueError(f"{name} is on {t.device}, the current device is cuda:{here}")


def _fit(desc, kind, *tensors):
    """``lca._fit`` over (tensor, name, elements, optional) entries."""
    for t, name, elems, *optional in tensors:
        lca._fit(desc, t, name, elems, kind, bool(optional and optional[0]))


def _fit_rows(desc, t, name, heads, d, row):
    """A [T, heads, d] tensor whose tokens lie `row` elements apart (0: next to each other); a view of a larger tensor passes."""
    row = row or heads * d
    if t is None or isinstance(t, int) or t.is_contiguous() or desc.T == 0:
        return lca._fit(desc, t, name, (desc.T - 1) * row + heads * d if desc.T else 0)
    lca._fit(desc, t, name, desc.T * heads * d)
    if tuple(t.shape) != (desc.T, heads, d) or t.stride(2) != 1 or (heads > 1 and t.stride(1) != d) or (desc.T > 1 and t.stride(0) != row):
        raise ValueError(f"{name} has shape {tuple(t.shape)} and strides {tuple(t.stride())}, the descriptor needs [{desc.T}, {heads}, {d}] with tokens {row} elements apart")


def _row_ptr(t):
    """``lca._ptr`` of a tensor that _fit_rows has seen: its tokens may lie apart."""
    if t is None or isinstance(t, int) or t.is_contiguous():
        return lca._ptr(t)
    if not t.is_cuda:
        raise ValueError(f"a tensor of shape {tuple(t.shape)} is not a device tensor: liblca takes device pointers")
    return t.data_ptr()


def _call(name, desc, *args):
    lca._check(getattr(load(), name)(ctypes.byref(_c_desc(*desc._key())), *args))


def page_tables(desc: Desc, cached_len, new_len, free_list, free_count, free_left, block_table, q_start, seq_len, slot, position, request, workspace, stream=None):
    if _bind is not None and lca._done(_bind.page_tables(desc, cached_len, new_len, free_list, free_count, free_left, block_table, q_start, seq_len, slot, position, request, workspace, stream)):
        return
    B, T = desc.B, desc.T
    _fit(desc, "i32", (cached_len, "cached_len", B), (new_len, "new_len", B), (free_list, "free_list", desc.n_blocks), (free_count, "free_count", 1),
         (free_left, "free_left", 1), (block_table, "block_table", B * desc.max_blocks), (q_start, "q_start", B + 1), (seq_len, "seq_len", B), (slot, "slot", T),
         (position, "position", T), (request, "request", T))
    _same_device(cached_len=cached_len, new_len=new_len, free_list=free_list, free_count=free_count, free_left=free_left, block_table=block_table, q_start=q_start,
                 seq_len=seq_len, slot=slot, position=position, request=request, workspace=workspace)
    _call("lca_page_tables", desc, *map(lca._ptr, (cached_len, new_len, free_list, free_count, free_left, block_table, q_start, seq_len, slot, position, request,
                                                   workspace)), lca._nbytes(workspace), lca._stream(stream))


def page_release(desc: Desc, finished, cached_len, block_table, free_list, free_count, stream=None):
    if _bind is not None and lca._done(_bind.page_release(desc, finished, cached_len, block_table, free_list, free_count, stream)):
        return
    _fit(desc, "i32", (finished, "finished", desc.B), (cached_len, "cached_len", desc.B), (block_table, "block_table", desc.B * desc.max_blocks),
         (free_list, "free_list", desc.n_blocks), (free_count, "free_count", 1))
    _same_device(finished=finished, cached_len=cached_len, block_table=block_table, free_list=free_list, free_count=free_count)
    _call("lca_page_release", desc, *map(lca._ptr, (finished, cached_len, block_table, free_list, free_count)), lca._stream(stream))


def _fit_cache(desc, sel_q8, pool_q8, scales):
    tokens = desc.n_blocks * desc.page * desc.S
    _fit(desc, "u8", (sel_q8, "sel_q8", tokens * desc.d_sel), (pool_q8, "pool_q8", tokens * desc.d_pool))
    _fit(desc, "f32", (scales, "scales", desc.n_blocks * desc.S * 2))


def page_store_q8(desc: Desc, SEL, POOL, slot, sel_q8, pool_q8, scales, stream=None):
    if _bind is not None and lca._done(_bind.page_store_q8(desc, SEL, POOL, slot, sel_q8, pool_q8, scales, stream)):
        return
    _fit_rows(desc, SEL, "SEL", desc.S, desc.d_sel, desc.sel_row)
    _fit_rows(desc, POOL, "POOL", desc.S, desc.d_pool, desc.pool_row)
    _fit(desc, "i32", (slot, "slot", desc.T))
    _fit_cache(desc, sel_q8, pool_q8, scales)
    _same_device(SEL=SEL, POOL=POOL, slot=slot, sel_q8=sel_q8, pool_q8=pool_q8, scales=scales)
    _call("lca_page_store_q8", desc, _row_ptr(SEL), _row_ptr(POOL), *map(lca._ptr, (slot, sel_q8, pool_q8, scales)), lca._stream(stream))


def _fit_rule(desc, prefix_len, slopes, O, lse):
    _fit(desc, "i32", (prefix_len, "prefix_len", desc.B, True))
    _fit(desc, "f32", (slopes, "slopes", desc.H, True), (lse, "lse", desc.T * desc.H, True))
    _fit(desc, "elt", (O, "O", desc.T * desc.H * desc.d_pool))


def page_attn_q8(desc: Desc, q, q_start, seq_len, prefix_len, slopes, block_table, sel_q8, pool_q8, scales, O, lse, workspace, stream=None):
    if _bind is not None and lca._done(_bind.page_attn_q8(desc, q, q_start, seq_len, prefix_len, slopes, block_table, sel_q8, pool_q8, scales, O, lse, workspace, stream)):
        return
    _fit_rows(desc, q, "q", desc.H, desc.d_sel, desc.q_row)
    _fit(desc, "i32", (q_start, "q_start", desc.B + 1), (seq_len, "seq_len", desc.B), (block_table, "block_table", desc.B * desc.max_blocks))
    _fit_rule(desc, prefix_len, slopes, O, lse)
    _fit_cache(desc, sel_q8, pool_q8, scales)
    _same_device(q=q, q_start=q_start, seq_len=seq_len, prefix_len=prefix_len, slopes=slopes, block_table=block_table, sel_q8=sel_q8, pool_q8=pool_q8, scales=scales,
                 O=O, lse=lse, workspace=workspace)
    _call("lca_page_attn_q8", desc, _row_ptr(q), *map(lca._ptr, (q_start, seq_len, prefix_len, slopes, block_table, sel_q8, pool_q8, scales, O, lse, workspace)),
          lca._nbytes(workspace), lca._stream(stream))


def packed_attn(desc: Desc, Q, SEL, POOL, doc_start, prefix_len, slopes, O, lse, workspace, stream=None):
    if _bind is not None and lca._done(_bind.packed_attn(desc, Q, SEL, POOL, doc_start, prefix_len, slopes, O, lse, workspace, stream)):
        return
    _fit_rows(desc, Q, "Q", desc.H, desc.d_sel, desc.q_row)
    _fit_rows(desc, SEL, "SEL", desc.S, desc.d_sel, desc.sel_row)
    _fit_rows(desc, POOL, "POOL", desc.S, desc.d_pool, desc.pool_row)
    _fit(desc, "i32", (doc_start, "doc_start", desc.B + 1))
    _fit_rule(desc, prefix_len, slopes, O, lse)
    _same_device(Q=Q, SEL=SEL, POOL=POOL, doc_start=doc_start, prefix_len=prefix_len, slopes=slopes, O=O, lse=lse, workspace=workspace)
    _call("lca_packed_attn", desc, _row_ptr(Q), _row_ptr(SEL), _row_ptr(POOL), *map(lca._ptr, (doc_start, prefix_len, slopes, O, lse, workspace)), lca._nbytes(workspace),
          lca._stream(stream))
