"""The operators of one batch iteration: what a simulated server stands for, on the GPU (include/gnr_iter.h).

Argument marshalling only, like `binding`: the work runs in the library's HIP kernels, on torch's current stream of the
tensors' device, and has no derivatives (tensors that require gradients are refused outside `torch.no_grad()`, those with a forward-mode tangent always). PyTorch provides the tensors, among them outputs and workspaces that are not given. Nothing waits for the GPU
but `check`. The marshalling itself is compiled (csrc_iter/gnr_iter_python.cpp); ValueError is its word for arguments that do not fit
each other, SimError the library's.

A cache is two tensors of [pages, kv_heads, page_size, head_dim] in any memory order with the last dimension dense: torch.bfloat16,
torch.float16, torch.float8_e4m3fn with exponent bytes [pages, kv_heads, page_size] beside each, or torch.float4_e2m1fn_x2, whose last dimension is head_dim / 2, with
exponent bytes [pages, kv_heads, page_size, head_dim / 32] (`new_cache` makes them). A batch is
`q_start` (requests + 1 bounds of the requests' tokens), `kv_len` (tokens in each request's cache, the new ones included) and
`page_table` ([requests, width] page numbers), all int32 on the device.

Positions are turns: `turns` (int64 on the device, `rotary_turns` makes them from frequencies, `rotary_frequencies` those) says what part of a full turn a position is worth for each of
dims / 2 pairs of elements.

`status`, an int32 tensor of one word (`new_status`), collects what only the kernels can see: `check` raises if a batch had bounds, page
or adapter numbers out of range, which the kernels treat as absent.
"""
from __future__ import annotations

import ctypes as C
import math
from fractions import Fraction

import torch

from .binding import SimError, lib

lib()                          # (torch first, then the library, then what links against both)
try:
    from . import _iteration   # noqa: E402
except ImportError as e:
    raise ImportError("the compiled binding is missing or does not fit this torch: run `python -m paper_2602_02987_amd.build`") from e

SIM_EINVAL = -1
BAD_BATCH, BAD_PAGE, BAD_ADAPTER = 1, 2, 4
_TYPE = {torch.bfloat16: 0, torch.float16: 1, torch.float8_e4m3fn: 2, torch.float4_e2m1fn_x2: 3}


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


class TurnsC(C.Structure):
    _fields_ = [("dims", C.c_int), ("interleaved", C.c_int), ("inverse", C.c_int), ("magnitude", C.c_float), ("turns", C.c_void_p)]


_ready = None


def _lib():
    """The C ABI itself, with its argument types (what the compiled binding calls)."""
    global _ready
    if _ready is None:
        L = lib()
        p = C.c_void_p
        L.iter_kv_write.argtypes = [p, C.c_int, p, p, p, C.c_int64, p]
        L.iter_kv_read.argtypes = [p, C.c_int, p, p, p, C.c_int64, p]
        L.iter_attention_bytes.argtypes = [p, p, C.c_int, p]
        L.iter_attention.argtypes = [p, p, C.c_int, C.c_int, p, p, C.c_double, C.c_int64, p, C.c_size_t, p, p]
        L.iter_adapters_bytes.argtypes = [p, C.c_int64, p]
        L.iter_adapters.argtypes = [p, C.c_int, C.c_int, C.c_int64, p, p, p, C.c_int64, p, C.c_int64, p, C.c_int64, p, C.c_size_t, p, p]
        L.iter_rotary.argtypes = [C.c_int, C.c_int, C.c_int, p, p, C.c_int64, p, p, p]
        L.iter_rotary_write.argtypes = [p, C.c_int, C.c_int, p, p, p, p, p, p, p, C.c_int64, p]
        L.iter_copy_pages.argtypes = [p, C.c_int, p, p, p, C.c_int64, p]
        L.iter_turns_size.argtypes = [p]
        L.iter_abi_sizes.argtypes = [p]
        _ready = L
    return _ready


def new_cache(pages, kv_heads, page_size, head_dim, dtype=torch.bfloat16, device="cuda"):
    """(k, v, k_exp, v_exp) of an empty cache, laid out by heads within a page; the exponents are None unless dtype has 8 or 4 bits."""
    if dtype not in _TYPE:
        raise ValueError("a cache is torch.bfloat16, torch.float16, torch.float8_e4m3fn or torch.float4_e2m1fn_x2")
    shape = (pages, kv_heads, page_size, head_dim)
    if dtype == torch.float4_e2m1fn_x2:
        if head_dim % 32:
            raise ValueError("a cache of 4 bits has an exponent for every 32 elements")
        k, v = (torch.zeros((*shape[:3], head_dim // 2), dtype=torch.uint8, device=device).view(dtype) for _ in range(2))
        return k, v, *(torch.full((*shape[:3], head_dim // 32), 127, dtype=torch.uint8, device=device) for _ in range(2))
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


def kv_write(k, v, k_cache, v_cache, slots, k_exp=None, v_exp=None):
    """Writes k and v ([tokens, kv_heads, head_dim], bfloat16 or float16) into the slots (int64, page * page_size + place, distinct; one
    outside the cache is no place). An 8-bit cache takes each row in units of the least power of two that brings it within 448, a cache of 4 bits every 32 elements in units
    of the least one that brings them within 6."""
    rc = _iteration.kv_write(k, v, k_cache, v_cache, slots, k_exp, v_exp)
    if rc is not None:
        raise SimError(rc, "iter_kv_write")


def kv_read(k_cache, v_cache, slots, k_exp=None, v_exp=None, dtype=None, k=None, v=None):
    """(k, v) of the slots (int64; one outside the cache reads as zeros), [tokens, kv_heads, head_dim] of `dtype` (bfloat16 or float16; the
    cache's own, bfloat16 where that has 8 or 4 bits), into the tensors given or new ones."""
    wanted = -1 if dtype is None else _TYPE.get(dtype, 2)
    if wanted >= 2:
        raise ValueError("dtype has to be bfloat16 or float16")
    out = _iteration.kv_read(k_cache, v_cache, slots, k_exp, v_exp, wanted, k, v)
    if type(out) is int:
        raise SimError(out, "iter_kv_read")
    return out


def attention(q, k_cache, v_cache, page_table, q_start, kv_len, k_exp=None, v_exp=None, max_q=None, scale=None, window=0, out=None,
              workspace=None, status=None):
    """Attention of a batch's tokens q ([tokens, heads, head_dim]) over their requests' caches: the token at position p of its request sees
    the positions max(0, p - window + 1) .. p (window 0: all up to p). `scale` is 1 / sqrt(head_dim) unless given, `max_q` the longest chunk
    the host expects (it selects kernels only). Over a cache of 8 or 4 bits keys and values are what `kv_read` gives in the type of q. Returns
    [tokens, heads, head_dim], in `out` if given (which must not overlap q)."""
    if max_q is not None and max_q < 0:
        raise ValueError("max_q has to be 0 or more")
    o = _iteration.attention(q, k_cache, v_cache, page_table, q_start, kv_len, k_exp, v_exp, -1 if max_q is None else max_q, scale, window, out,
                             workspace, status)
    if type(o) is int:
        raise SimError(o, "iter_attention")
    return o


def adapters(x, base, down, up, scale, q_start, adapter, out=None, workspace=None, status=None):
    """base + scale[a] * up[a] (down[a] x) for the tokens of every request, a = adapter[request] (-1: base as it is). x [tokens, width_in],
    base [tokens, width_out], down [adapters, rank, width_in], up [adapters, width_out, rank], all bfloat16 or all float16; scale float32
    [adapters], q_start and adapter int32. `out` may be `base` (or is apart from it), and may overlap `x`."""
    o = _iteration.adapters(x, base, down, up, scale, q_start, adapter, out, workspace, status)
    if type(o) is int:
        raise SimError(o, "iter_adapters")
    return o


def rotary_frequencies(dims, base=10000.0, scaling=None, factor=1.0, original=8192, low=1.0, high=4.0):
    """Radians a position of dims / 2 pairs, base ** (-2 i / dims), scaled for contexts `factor` times as long as the `original` one:

    None: as they are (the factor has to be 1). "linear": all divided by the factor. "base": the base raised by factor ** (dims / (dims - 2)), which divides the slowest by the factor and leaves the fastest. "parts": those that make
    at least `high` turns in the original context stay, those with at most `low` are divided by the factor, and between them the two are mixed in proportion to the turns."""
    if dims < 2 or dims % 2 or base <= 0 or factor <= 0 or original <= 0:
        raise ValueError("dims has to be even, base, factor and original positive")
    if scaling not in (None, "linear", "base", "parts"):
        raise ValueError("scaling has to be None, 'linear', 'base' or 'parts'")
    if scaling is None and factor != 1.0:
        raise ValueError("a factor needs a scaling that uses it")
    if scaling == "base":
        if dims == 2:
            raise ValueError("a single pair has no slowest and fastest frequency")
        base = base * factor ** (dims / (dims - 2))
    f = [base ** (-2.0 * i / dims) for i in range(dims // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "parts":
        if not high > low:
            raise ValueError("high has to be above low")
        kept = [min(1.0, max(0.0, (original * x / (2.0 * math.pi) - low) / (high - low))) for x in f]
        f = [x * k + x / factor * (1.0 - k) for x, k in zip(f, kept)]
    return f


def rotary_turns(frequencies, device="cuda"):
    """`turns` for frequencies in radians a position: parts of a full turn in units of 2**-64 (whole turns are left out), so that the angle of any position is exact modulo a turn."""
    whole = 1 << 64
    t = [round(Fraction(float(f)) / Fraction(2.0 * math.pi) * whole) % whole for f in frequencies]
    return torch.tensor([x - whole if x >= whole >> 1 else x for x in t], dtype=torch.int64).to(device)


def rotary(x, positions, turns, interleaved=False, magnitude=1.0, inverse=False, out=None):
    """x ([tokens, heads, head_dim], bfloat16 or float16) with the first dims = 2 * len(turns) elements of every row turned by the angles of its token's position (int64 [tokens]), times
    `magnitude`: pairs are the elements i and i + dims / 2, or 2 i and 2 i + 1 if `interleaved`; other elements stay. `inverse` turns back. dims has to be a multiple of 16. Returns the rows, in `out` if
    given, which may be x."""
    o = _iteration.rotary(x, positions, turns, interleaved, magnitude, inverse, out)
    if type(o) is int:
        raise SimError(o, "iter_rotary")
    return o


def rotary_write(q, k, v, positions, turns, k_cache, v_cache, slots, k_exp=None, v_exp=None, interleaved=False, magnitude=1.0, out=None):
    """`rotary` of the queries q and the keys k, and `kv_write` of these keys and the values v, in one launch, with the same bits as one after the other. Returns the queries, in `out`
    if given, which may be q."""
    o = _iteration.rotary_write(q, k, v, positions, turns, k_cache, v_cache, slots, k_exp, v_exp, interleaved, magnitude, out)
    if type(o) is int:
        raise SimError(o, "iter_rotary_write")
    return o


def copy_pages(caches, source, target, places=None):
    """Copies pages source[i] to target[i], or their first places[i] places, in every cache of the list `caches` of (k, v, k_exp, v_exp), the layers of a model, which are alike
    (or `caches` is one such tuple, of tensors that have the layers as a first dimension). The numbers are on the host (lists, or int64 tensors on the CPU): what does not fit, a target that is named twice and one that is a source too are refused before anything is copied, and a graph copies the
    pages it was captured with."""
    rc = _iteration.copy_pages(caches, source, target, places)
    if rc is not None:
        raise SimError(rc, "iter_copy_pages")
