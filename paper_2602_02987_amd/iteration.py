"""The operators of one batch iteration: what a simulated server stands for, on the GPU (include/gnr_iter.h).

Argument marshalling only, like `binding`: the work runs in the library's HIP kernels, on torch's current stream of the
tensors' device. PyTorch provides the tensors, among them outputs and workspaces that are not given. Nothing waits for the GPU
but `check`.

A cache is two tensors of [pages, kv_heads, page_size, head_dim] in any memory order with the last dimension dense: torch.bfloat16,
torch.float16, or torch.float8_e4m3fn with exponent bytes [pages, kv_heads, page_size] beside each (`new_cache` makes them). A batch is
`q_start` (requests + 1 bounds of the requests' tokens), `kv_len` (tokens in each request's cache, the new ones included) and
`page_table` ([requests, width] page numbers), all int32 on the device.

`status`, an int32 tensor of one word (`new_status`), collects what only the kernels can see: `check` raises if a batch had bounds, page
or adapter numbers out of range, which the kernels treat as absent.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from .binding import SimError, lib

SIM_EINVAL = -1
BAD_BATCH, BAD_PAGE, BAD_ADAPTER = 1, 2, 4
_TYPE = {torch.bfloat16: 0, torch.float16: 1, torch.float8_e4m3fn: 2}


class PlaneC(C.Structure):
    _fields_ = [("data", C.c_void_p), ("exp", C.c_void_p), ("page_stride", C.c_int64), ("head_stride", C.c_int64),
                ("place_stride", C.c_int64), ("exp_page_stride", C.c_int64), ("exp_head_stride", C.c_int64),
                ("exp_place_stride", C.c_int64)]


class CacheC(C.Structure):
    _fields_ = [("type", C.c_int), ("kv_heads", C.c_int), ("head_dim", C.c_int), ("page", C.c_int), ("pages", C.c_int64),
                ("k", PlaneC), ("v", PlaneC)]


class RowsC(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class BatchC(C.Structure):
    _fields_ = [("requests", C.c_int), ("tokens", C.c_int64), ("max_q", C.c_int64), ("q_start", C.c_void_p),
                ("kv_len", C.c_void_p), ("page_table", C.c_void_p), ("table_stride", C.c_int64), ("table_width", C.c_int64)]


class AdapterSetC(C.Structure):
    _fields_ = [("adapters", C.c_int), ("rank", C.c_int), ("width_in", C.c_int64), ("width_out", C.c_int64),
                ("down", C.c_void_p), ("up", C.c_void_p), ("scale", C.c_void_p)]


_ready = None


def _lib():
    global _ready
    if _ready is None:
        L = lib()
        cache, rows, p = C.POINTER(CacheC), C.POINTER(RowsC), C.c_void_p
        L.iter_kv_write.argtypes = [cache, C.c_int, rows, rows, p, C.c_int64, p]
        L.iter_kv_read.argtypes = [cache, C.c_int, rows, rows, p, C.c_int64, p]
        L.iter_attention_bytes.argtypes = [cache, C.POINTER(BatchC), C.c_int, C.POINTER(C.c_size_t)]
        L.iter_attention.argtypes = [cache, C.POINTER(BatchC), C.c_int, C.c_int, rows, rows, C.c_double, C.c_int64, p, C.c_size_t, p, p]
        L.iter_adapters_bytes.argtypes = [C.POINTER(AdapterSetC), C.c_int64, C.POINTER(C.c_size_t)]
        L.iter_adapters.argtypes = [C.POINTER(AdapterSetC), C.c_int, C.c_int, C.c_int64, p, p, p, C.c_int64, p, C.c_int64, p, C.c_int64,
                                    p, C.c_size_t, p, p]
        L.iter_abi_sizes.argtypes = [p]
        _ready = L
    return _ready


def _check(rc, where):
    if rc != 0:
        raise SimError(rc, where)


def _want(ok, what):
    if not ok:
        raise ValueError(what)


class _On:
    """The device of the call is current while the library is in it (torch's own guard costs more than the launch)."""

    def __init__(self, device):
        self.index = device.index

    def __enter__(self):
        self.before = torch.cuda.current_device()
        if self.before != self.index:
            torch.cuda.set_device(self.index)
        return torch.cuda.current_stream(self.index).cuda_stream

    def __exit__(self, *_):
        if self.before != self.index:
            torch.cuda.set_device(self.before)


def _on_gpu(device, **tensors):
    _want(device.type == "cuda", "the operators need a GPU: tensors have to be on a HIP device")
    for name, t in tensors.items():
        _want(t is None or t.device == device, f"{name} is on another device")


def new_cache(pages, kv_heads, page_size, head_dim, dtype=torch.bfloat16, device="cuda"):
    """(k, v, k_exp, v_exp) of an empty cache, laid out by heads within a page; the exponents are None unless dtype is 8-bit."""
    _want(dtype in _TYPE, "a cache is torch.bfloat16, torch.float16 or torch.float8_e4m3fn")
    shape = (pages, kv_heads, page_size, head_dim)
    k, v = (torch.zeros(shape, dtype=dtype, device=device) for _ in range(2))
    if dtype != torch.float8_e4m3fn:
        return k, v, None, None
    return k, v, *(torch.full(shape[:3], 127, dtype=torch.uint8, device=device) for _ in range(2))


def new_status(device="cuda"):
    return torch.zeros(1, dtype=torch.int32, device=device)


def check(status):
    """Waits for the work before it and raises SimError if a kernel found bounds, page or adapter numbers out of range."""
    word = int(status.item())
    if word:
        found = [n for b, n in ((BAD_BATCH, "batch bounds"), (BAD_PAGE, "page numbers"), (BAD_ADAPTER, "adapter numbers")) if word & b]
        raise SimError(SIM_EINVAL, " and ".join(found) + " out of range")


def _strides(t, n):
    """The first n strides; a dimension of one element has none that matter."""
    st, sh = t.stride(), t.shape
    return [st[i] if sh[i] > 1 else 0 for i in range(n)]


def _plane(t, exp, name):
    _want(t.stride(3) == 1, f"the last dimension of {name} has to be dense")
    if exp is None:
        return PlaneC(t.data_ptr(), None, *_strides(t, 3), 0, 0, 0)
    _want(exp.dtype == torch.uint8 and exp.shape == t.shape[:3], f"{name}_exp has to be uint8 [pages, kv_heads, page_size]")
    return PlaneC(t.data_ptr(), exp.data_ptr(), *_strides(t, 3), *_strides(exp, 3))


def _cache(k, v, k_exp, v_exp):
    _want(k.dim() == 4 and k.shape == v.shape and k.dtype == v.dtype and k.dtype in _TYPE,
          "a cache is two tensors [pages, kv_heads, page_size, head_dim] of bfloat16, float16 or float8_e4m3fn")
    fp8 = k.dtype == torch.float8_e4m3fn
    _want((k_exp is not None) == fp8 and (v_exp is not None) == fp8, "an 8-bit cache, and no other, has exponents beside it")
    _on_gpu(k.device, v_cache=v, k_exp=k_exp, v_exp=v_exp)
    pages, heads, page, dim = k.shape
    return CacheC(_TYPE[k.dtype], heads, dim, page, pages, _plane(k, k_exp, "k"), _plane(v, v_exp, "v"))


def _rows(t, heads, dim, dtype, name):
    _want(t.dim() == 3 and t.shape[1] == heads and t.shape[2] == dim and t.dtype == dtype,
          f"{name} has to be [tokens, {heads}, {dim}] of {dtype}")
    _want(t.stride(2) == 1, f"the last dimension of {name} has to be dense")
    return RowsC(t.data_ptr(), *_strides(t, 2))


def _ints(t, name, shape, dtype=torch.int32):
    _want(t.dtype == dtype and t.shape == shape and t.is_contiguous(), f"{name} has to be {dtype} {tuple(shape)} without gaps")
    return t.data_ptr()


def _status_ptr(status):
    if status is None:
        return None
    _want(status.dtype == torch.int32 and status.numel() == 1, "status is one int32 word")
    return status.data_ptr()


def kv_write(k, v, k_cache, v_cache, slots, k_exp=None, v_exp=None):
    """Writes k and v ([tokens, kv_heads, head_dim], bfloat16 or float16) into the slots (int64, page * page_size + place, distinct; one
    outside the cache is no place). An 8-bit cache takes each row in units of the least power of two that brings it within 448."""
    c = _cache(k_cache, v_cache, k_exp, v_exp)
    _want(k.dtype in (torch.bfloat16, torch.float16) and (c.type == 2 or k.dtype == k_cache.dtype),
          "k and v have to be of the cache's type, or bfloat16 or float16 for an 8-bit cache")
    _on_gpu(k_cache.device, k=k, v=v, slots=slots)
    kr, vr = _rows(k, c.kv_heads, c.head_dim, k.dtype, "k"), _rows(v, c.kv_heads, c.head_dim, k.dtype, "v")
    _want(k.shape[0] == v.shape[0], "k and v have to have as many tokens")
    at = _ints(slots, "slots", k.shape[:1], torch.int64)
    with _On(k.device) as stream:
        _check(_lib().iter_kv_write(C.byref(c), _TYPE[k.dtype], C.byref(kr), C.byref(vr), at, k.shape[0], stream), "iter_kv_write")


def kv_read(k_cache, v_cache, slots, k_exp=None, v_exp=None, dtype=None, k=None, v=None):
    """(k, v) of the slots (int64; one outside the cache reads as zeros), [tokens, kv_heads, head_dim] of `dtype` (bfloat16 or float16; the
    cache's own unless that has 8 bits), into the tensors given or new ones."""
    c = _cache(k_cache, v_cache, k_exp, v_exp)
    dtype = dtype or (torch.bfloat16 if c.type == 2 else k_cache.dtype)
    _want(dtype in (torch.bfloat16, torch.float16) and (c.type == 2 or dtype == k_cache.dtype),
          "dtype has to be the cache's, or bfloat16 or float16 for an 8-bit cache")
    shape = (slots.numel(), c.kv_heads, c.head_dim)
    k = torch.empty(shape, dtype=dtype, device=k_cache.device) if k is None else k
    v = torch.empty(shape, dtype=dtype, device=k_cache.device) if v is None else v
    _on_gpu(k_cache.device, k=k, v=v, slots=slots)
    kr, vr = _rows(k, c.kv_heads, c.head_dim, dtype, "k"), _rows(v, c.kv_heads, c.head_dim, dtype, "v")
    _want(k.shape[0] == shape[0] and v.shape[0] == shape[0], "k and v have to have a row for every slot")
    at = _ints(slots, "slots", k.shape[:1], torch.int64)
    with _On(k.device) as stream:
        _check(_lib().iter_kv_read(C.byref(c), _TYPE[dtype], C.byref(kr), C.byref(vr), at, shape[0], stream), "iter_kv_read")
    return k, v


def attention(q, k_cache, v_cache, page_table, q_start, kv_len, k_exp=None, v_exp=None, max_q=None, scale=None, window=0, out=None,
              workspace=None, status=None):
    """Attention of a batch's tokens q ([tokens, heads, head_dim]) over their requests' caches: the token at position p of its request sees
    the positions max(0, p - window + 1) .. p (window 0: all up to p). `scale` is 1 / sqrt(head_dim) unless given, `max_q` the longest chunk
    the host expects (it selects kernels only). Returns [tokens, heads, head_dim], in `out` if given."""
    c = _cache(k_cache, v_cache, k_exp, v_exp)
    _want(q.dim() == 3, "q has to be [tokens, heads, head_dim]")
    tokens, heads, dim = q.shape
    _want(q.dtype in (torch.bfloat16, torch.float16) and (c.type == 2 or q.dtype == k_cache.dtype),
          "q has to be of the cache's type, or bfloat16 or float16 over an 8-bit cache")
    out = torch.empty((tokens, heads, dim), dtype=q.dtype, device=q.device) if out is None else out
    _on_gpu(q.device, k_cache=k_cache, page_table=page_table, q_start=q_start, kv_len=kv_len, out=out, workspace=workspace, status=status)
    qr, outr = _rows(q, heads, c.head_dim, q.dtype, "q"), _rows(out, heads, c.head_dim, q.dtype, "out")
    _want(out.shape[0] == tokens, "out has to have q's tokens")
    _want(kv_len.dim() == 1, "kv_len has to be [requests]")
    n = kv_len.shape[0]
    _want(page_table.dim() == 2 and page_table.shape[0] == n and page_table.dtype == torch.int32 and
          (page_table.stride(1) == 1 or page_table.shape[1] <= 1), "page_table has to be int32 [requests, width] with dense rows")
    b = BatchC(n, tokens, tokens if max_q is None else max_q, _ints(q_start, "q_start", (n + 1,)), _ints(kv_len, "kv_len", (n,)),
               page_table.data_ptr(), _strides(page_table, 1)[0], page_table.shape[1])
    L = _lib()
    need = C.c_size_t(0)
    _check(L.iter_attention_bytes(C.byref(c), C.byref(b), heads, C.byref(need)), "iter_attention_bytes")
    work, size = _workspace(workspace, need.value, q.device)
    with _On(q.device) as stream:
        _check(L.iter_attention(C.byref(c), C.byref(b), _TYPE[q.dtype], heads, C.byref(qr), C.byref(outr),
                                1.0 / math.sqrt(dim) if scale is None else scale, window, work.data_ptr() if size else None, size,
                                _status_ptr(status), stream), "iter_attention")
    return out


def _workspace(given, need, device):
    if given is not None:
        _want(given.is_contiguous(), "the workspace has to be without gaps")
        return given, given.numel() * given.element_size()
    return (torch.empty(need, dtype=torch.uint8, device=device) if need else None), need


def adapters(x, base, down, up, scale, q_start, adapter, out=None, workspace=None, status=None):
    """base + scale[a] * up[a] (down[a] x) for the tokens of every request, a = adapter[request] (-1: base as it is). x [tokens, width_in],
    base [tokens, width_out], down [adapters, rank, width_in], up [adapters, width_out, rank], all bfloat16 or all float16; scale float32
    [adapters], q_start and adapter int32. `out` may be `base`."""
    _want(x.dim() == 2 and base.dim() == 2 and down.dim() == 3 and up.dim() == 3, "x and base have two dimensions, down and up three")
    tokens, wi = x.shape
    n, rank, wo = down.shape[0], down.shape[1], up.shape[1]
    out = torch.empty((tokens, wo), dtype=x.dtype, device=x.device) if out is None else out
    _want(x.dtype in (torch.bfloat16, torch.float16) and all(t.dtype == x.dtype for t in (base, down, up, out)),
          "x, base, down, up and out have to be all bfloat16 or all float16")
    _want(base.shape == (tokens, wo) and out.shape == (tokens, wo), f"base and out have to be [{tokens}, {wo}]")
    _want(down.shape == (n, rank, wi) and up.shape == (n, wo, rank) and down.is_contiguous() and up.is_contiguous(),
          "down has to be [adapters, rank, width_in] and up [adapters, width_out, rank], without gaps")
    for t, name in ((x, "x"), (base, "base"), (out, "out")):
        _want(t.stride(1) == 1, f"the last dimension of {name} has to be dense")
    _on_gpu(x.device, base=base, down=down, up=up, scale=scale, q_start=q_start, adapter=adapter, out=out, workspace=workspace, status=status)
    _want(adapter.dim() == 1, "adapter has to be [requests]")
    r = adapter.shape[0]
    s = AdapterSetC(n, rank, wi, wo, down.data_ptr(), up.data_ptr(), _ints(scale, "scale", (n,), torch.float32))
    qs, ad = _ints(q_start, "q_start", (r + 1,)), _ints(adapter, "adapter", (r,))
    L = _lib()
    need = C.c_size_t(0)
    _check(L.iter_adapters_bytes(C.byref(s), tokens, C.byref(need)), "iter_adapters_bytes")
    work, size = _workspace(workspace, need.value, x.device)
    with _On(x.device) as stream:
        _check(L.iter_adapters(C.byref(s), _TYPE[x.dtype], r, tokens, qs, ad, x.data_ptr(), _strides(x, 1)[0], base.data_ptr(), _strides(base, 1)[0],
                               out.data_ptr(), _strides(out, 1)[0], work.data_ptr() if size else None, size, _status_ptr(status), stream),
               "iter_adapters")
    return out
