"""Plain 64-bit implementations of the iteration operators, on the CPU, and the bounds their results are held to."""
import math

import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp8": torch.float8_e4m3fn}
E4M3 = np.array([(-1.0) ** (c >> 7) * (math.nan if c & 127 == 127 else (c & 7) / 8 * 2.0 ** -6 if (c >> 3) & 15 == 0
                                       else (1 + (c & 7) / 8) * 2.0 ** (((c >> 3) & 15) - 7)) for c in range(256)])


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def quantise(x):
    """(code values, exponents e) of rows of float64: the least whole e >= -126 with max|x| <= 448 * 2^e, codes nearest even."""
    values, exps = np.zeros_like(x), np.zeros(x.shape[:-1], np.int64)
    # the codes 0..126 ascend from 0 to 448, so a tie goes to the even one of two neighbouring codes
    grid = E4M3[:127]
    for i in np.ndindex(x.shape[:-1]):
        row = x[i]
        if not np.isfinite(row).all():
            values[i] = math.nan
            continue
        most = np.abs(row).max()
        e = 0
        if most > 0:
            e = -126
            while most > 448.0 * 2.0 ** e:
                e += 1
        y = np.abs(row) / 2.0 ** e
        hi = np.minimum(np.searchsorted(grid, y), 126)
        lo = np.maximum(hi - 1, 0)
        below, above = y - grid[lo], grid[hi] - y
        code = np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))
        values[i] = np.copysign(grid[code], row)
        exps[i] = e
    return values, exps


def cache_values(t, exp):
    """float64 values of a cache tensor (any device) [pages, heads, places, dim]."""
    if exp is None:
        return t.cpu().double().numpy()
    codes = t.view(torch.uint8).cpu().numpy()
    return E4M3[codes] * 2.0 ** (exp.cpu().numpy().astype(np.float64) - 127.0)[..., None]


def attention(q, k, v, table, q_start, kv_len, scale=None, window=0):
    """(out, bound-ingredients) in float64: q [tokens, heads, dim], k / v [pages, kv_heads, places, dim] float64 arrays."""
    tokens, heads, dim = q.shape
    places, group = k.shape[2], heads // k.shape[1]
    scale = 1.0 / math.sqrt(dim) if scale is None else scale
    out, spread, most, total, reach = (np.zeros(q.shape) for _ in range(5))
    for r in range(len(kv_len)):
        n = int(kv_len[r])
        kr = np.concatenate([k[table[r][j]] for j in range(-(-n // places))], 1)[:, :n] if n > 0 else k[0][:, :0]
        vr = np.concatenate([v[table[r][j]] for j in range(-(-n // places))], 1)[:, :n] if n > 0 else v[0][:, :0]
        for t in range(int(q_start[r]), int(q_start[r + 1])):
            p = n - int(q_start[r + 1]) + t
            a, b = (max(0, p - window + 1) if window else 0), p + 1
            if b <= a:
                continue
            for h in range(heads):
                kk, vv = kr[h // group, a:b], vr[h // group, a:b]
                s = kk @ q[t, h] * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out[t, h] = w @ vv
                spread[t, h] = w @ np.abs(vv)
                most[t, h] = np.abs(vv).sum(0)
                total[t, h] = (np.abs(kk) @ np.abs(q[t, h])).max() * abs(scale)
                reach[t, h] = b - a
    return out, (spread, most, total, reach)


def attention_bound(out, parts, dtype, dim):
    """What rounding may cost: the weights to `dtype` (half a step of each, or of the smallest number for those far below the row's
    largest), the output to `dtype`, and 32-bit scores (dim products and sums), exponentials and sums over the keys."""
    spread, most, total, reach = parts
    u = half_step(dtype)
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2
    f = 2.0 ** -24 * (2 * (dim + 16) * total + reach + 64)
    return u * (spread + np.abs(out)) * (1 + u) + f * spread * (1 + u) + tiny * (most + 1)


def adapters(x, base, down, up, scale, q_start, adapter):
    """(out, size of what is summed, error of the inner product in 32 bits)"""
    out, inner, outer = base.copy(), np.zeros_like(base), np.zeros_like(base)
    for r, a in enumerate(adapter):
        s = slice(int(q_start[r]), int(q_start[r + 1]))
        if a < 0:
            continue
        h = x[s] @ down[a].T
        out[s] = base[s] + scale[a] * (h @ up[a].T)
        size = np.abs(x[s]) @ np.abs(down[a]).T
        inner[s] = abs(scale[a]) * (size @ np.abs(up[a]).T)
        outer[s] = abs(scale[a]) * (np.abs(h) @ np.abs(up[a]).T)
    return out, inner, outer


def adapters_bound(out, base, inner, outer, dtype, width_in, rank):
    """The output to `dtype`; the inner product summed in 32 bits over width_in, held to at least 16 bits of mantissa, and the
    outer one summed in 32 bits."""
    u = half_step(dtype)
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2
    rest = 2.0 ** -24 * ((width_in + 8) * inner + (rank + 8) * outer + np.abs(base)) + 2.0 ** -16 * outer
    return u * np.abs(out) + rest * (1 + u) + tiny
