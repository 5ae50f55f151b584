"""Timed cases of the operators that a served model's iteration has beside those of `operators.py`: positions, a cache in 4 bits, and pages
that requests share or that change places.

`rotary` turns pairs of elements of queries and keys by angles that grow with the token's position. `rotary_write` does that for a batch's
queries and keys and puts the keys, with the values, into the paged cache in the same launch. A cache in 4 bits holds rows as e2m1 codes, 32 to
a power of two: `kv_write` and `kv_read` take rows there and back, `attention` reads it. `copy_pages` copies pages of all layers' caches: the last,
unfinished page of a request that goes on in several ways, or the pages that are moved down when a cache is made smaller.

Sizes come from the repository's configurations: chunks of up to 8191 tokens, up to 127 decodes beside one, lognormal lengths of up to 32768
tokens, and for contexts that the 4 bits are meant for four times that. Head layouts are generic.
"""
from __future__ import annotations

import math
import random

import torch

own = False   # False: elementary torch operations; True: the framework's operators

_TYPE = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp8": torch.float8_e4m3fn, "fp4": torch.float4_e2m1fn_x2}
_MOST_LEN = 32768
_LEAST_WORDS = {"fp8": 1, "fp4": 0.5, "bf16": 2, "fp16": 2}


def _rotary(name, tokens, heads, dim, dims, interleaved, q, base, factor, far):
    """`far`: positions go up to this."""
    c = dict(op="rotary", tokens=tokens, heads=heads, dim=dim, dims=dims, interleaved=interleaved, q=q, base=base, factor=factor, far=far)
    return dict(c, name=name) if name else c


def _rotary_write(name, tokens, chunk, heads, kv_heads, dim, dims, page, interleaved, q, cache, far, token_major=False):
    """`chunk`: the tokens are one request's, else a decode each."""
    c = dict(op="rotary_write", tokens=tokens, chunk=chunk, heads=heads, kv_heads=kv_heads, dim=dim, dims=dims, page=page, interleaved=interleaved, q=q,
             cache=cache, base=500000.0, factor=1.0, far=far, token_major=token_major)
    return dict(c, name=name) if name else c


def _store(name, tokens, kv_heads, dim, page, q, token_major=False):
    c = dict(op="store", tokens=tokens, kv_heads=kv_heads, dim=dim, page=page, q=q, cache="fp4", token_major=token_major)
    return dict(c, name=name) if name else c


def _attention(name, requests, chunk, chunk_context, median, heads, kv_heads, dim, page, q, lengths, window=0, token_major=False):
    c = dict(op="attention", requests=requests, chunk=chunk, chunk_context=chunk_context, median=median, heads=heads, kv_heads=kv_heads, dim=dim,
             page=page, q=q, cache="fp4", lengths=lengths, window=window, token_major=token_major)
    return dict(c, name=name) if name else c


def _copy(name, layers, pages, moves, fork, kv_heads, dim, page, cache):
    """`fork`: this many places of one page go to all targets; 0: whole pages, each to a place of its own."""
    c = dict(op="copy", layers=layers, pages=pages, moves=moves, fork=fork, kv_heads=kv_heads, dim=dim, page=page, cache=cache)
    return dict(c, name=name) if name else c


def listed():
    return [
        # queries and keys of one decode's token: a launch
        _rotary("rotary_one_token", 1, 40, 128, 128, False, "bf16", 10000.0, 1.0, 1093),
        # the largest chunk, half of each head turned, positions far behind what the frequencies were made for
        _rotary("rotary_prompt", 8191, 40, 128, 64, True, "fp16", 10000.0, 8.0, 1000000),
        # the new tokens of a full decode batch, into a cache of 8 bits
        _rotary_write("rotary_write_decode_batch", 128, False, 32, 8, 128, 128, 64, False, "bf16", "fp8", 32768),
        # the largest chunk's queries, keys and values, after as many tokens before it
        _rotary_write("rotary_write_prompt", 8191, True, 32, 8, 128, 128, 64, False, "bf16", "bf16", 2 * 8191),
        # new rows of a decode batch, stored in 4 bits and read back
        _store("store_4_bits_decode_batch", 128, 8, 128, 64, "bf16"),
        # the longest request of the configurations is stored and taken out again for another server
        _store("store_4_bits_long", 32768 + 5, 8, 128, 16, "fp16"),
        # a single decode at a median prompt: latency
        _attention("attention_4_bits_one_decode", 1, 0, 0, 1093, 32, 8, 128, 64, "bf16", 1),
        # the full decode batch of the largest configuration
        _attention("attention_4_bits_decode_batch", 127, 0, 0, 2767, 32, 8, 128, 64, "bf16", 2),
        # few requests with contexts of four times the longest length, seven heads to a kv head: what a cache of 4 bits is for
        _attention("attention_4_bits_long_decodes", 3, 0, 0, 4 * _MOST_LEN - 7, 28, 4, 128, 16, "fp16", 3),
        # a long prompt's last chunk
        _attention("attention_4_bits_prompt_chunk", 0, 251, 32768 - 251, 0, 32, 8, 128, 64, "bf16", 4),
        # a prompt of which eight samples are drawn: the last page, 5 tokens of it, is copied for each in every layer
        _copy("copy_pages_fork", 32, 48, 8, 5, 8, 128, 64, "fp8"),
        # a cache made smaller: pages of all layers move to places further down
        _copy("copy_pages_compact", 16, 1024, 300, 0, 8, 128, 64, "bf16"),
    ]


_LAYOUTS = [(32, 8, 128), (16, 16, 64), (28, 4, 128), (64, 8, 128), (8, 1, 128), (40, 10, 64), (8, 8, 128), (24, 2, 64), (16, 4, 256)]


def draw(rng):
    """One more case of the listed ones' ranges."""
    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rotary", "rotary_write", "store", "attention", "attention", "attention", "copy"])
    q = rng.choice(["bf16", "fp16"])
    heads, kv_heads, dim = rng.choice(_LAYOUTS)
    if op == "rotary":
        return _rotary(None, log_uniform(1, 8191), rng.randint(1, 40), dim, rng.choice([dim, dim // 2, 16, 48]), rng.random() < 0.5, q,
                       rng.choice([10000.0, 500000.0]), rng.choice([1.0, 4.0, 8.0]), log_uniform(8192, 4000000))
    if op == "rotary_write":
        tokens = log_uniform(1, 8191)
        chunk = tokens > 128 or rng.random() < 0.3
        # (rows of an 8-bit cache are compared code by code: few of them, so that none is likely to lie next to a border)
        cache = rng.choice([q, "fp8"]) if tokens <= 1024 else q
        return _rotary_write(None, tokens, chunk, min(heads, 32), min(kv_heads, 8) if min(heads, 32) % min(kv_heads, 8) == 0 else 1, dim, rng.choice([dim, dim // 2, 16]),
                             rng.choice([16, 32, 64, 128]), rng.random() < 0.5, q, cache, log_uniform(16384, 1000000), rng.random() < 0.3)
    if op == "store":
        return _store(None, log_uniform(1, 32768), rng.choice([1, 4, 8]), dim, rng.choice([16, 32, 64, 128]), q, rng.random() < 0.3)
    if op == "copy":
        kind = rng.choice(["fork", "compact"])
        page = rng.choice([16, 32, 64, 128])
        moves = log_uniform(1, 16) if kind == "fork" else log_uniform(1, 300)
        return _copy(None, rng.randint(1, 32 if kind == "fork" else 16), 2 * moves + rng.randint(2, 40), moves, rng.randint(1, page) if kind == "fork" else 0,
                     rng.choice([1, 4, 8]), rng.choice([64, 128]), page, rng.choice(["bf16", "fp16", "fp8"]))
    kind = rng.choice(["decode", "decode", "mixed", "chunk"])
    requests = 0 if kind == "chunk" else log_uniform(1, 100)
    chunk = 0 if kind == "decode" else log_uniform(2, 2000) if kind == "chunk" else log_uniform(2, 512)
    context = 0 if kind == "decode" else rng.choice([0, log_uniform(1, 6000)])
    return _attention(None, requests, chunk, context, log_uniform(16, 2700 if requests > 4 else 60000) if requests else 0, heads, kv_heads, dim,
                      rng.choice([16, 32, 64, 128]), q, rng.randint(10, 1 << 30), rng.choice([0, 0, 0, log_uniform(16, 4096)]), rng.random() < 0.3)


def _lens(case):
    """(new tokens, cached tokens) of every request: the decodes, then the chunk's request."""
    r = random.Random(case["lengths"])
    n = case["requests"]
    if n <= 4:                                  # a few decodes: about the median each
        kv = [max(1, case["median"] - 3 * i) for i in range(n)]
    else:
        kv = [max(1, min(_MOST_LEN, round(case["median"] * math.exp(r.gauss(0.0, 0.8))))) for _ in range(n)]
    q = [1] * n
    if case["chunk"]:
        q, kv = q + [case["chunk"]], kv + [case["chunk"] + case["chunk_context"]]
    return q, kv


def _frequencies(case):
    """Radians a position, float64: the geometric series, divided by the factor where a turn takes longer than 1/8 of 8192 positions."""
    f = [case["base"] ** (-2.0 * i / case["dims"]) for i in range(case["dims"] // 2)]
    return [x / case["factor"] if 8192.0 * x / (2.0 * math.pi) < 8.0 else x for x in f]


def _turns(freqs):
    """The same as 64-bit fractions of a turn."""
    whole = 1 << 64
    t = [round(x / (2.0 * math.pi) * whole) % whole for x in freqs]
    return [x - whole if x >= whole // 2 else x for x in t]


def _codes(gen, shape, typ, dev):
    """A cache's contents: (values or codes, exponent bytes or None)."""
    if typ == "fp4":
        pages, heads, page, dim = shape
        codes = torch.randint(0, 256, (pages, heads, page, dim // 2), generator=gen, device=dev, dtype=torch.uint8)
        return codes.view(torch.float4_e2m1fn_x2), torch.randint(123, 127, (pages, heads, page, dim // 32), generator=gen, device=dev, dtype=torch.uint8)
    if typ == "fp8":
        x = (torch.randn(shape, generator=gen, device=dev, dtype=torch.bfloat16) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
        return x, torch.randint(118, 122, shape[:-1], generator=gen, device=dev, dtype=torch.uint8)
    return torch.randn(shape, generator=gen, device=dev, dtype=_TYPE[typ]), None


def _empty(shape, typ, dev):
    if typ == "fp4":
        return torch.zeros((*shape[:3], shape[3] // 2), device=dev, dtype=torch.uint8).view(_TYPE[typ]), torch.full((*shape[:3], shape[3] // 32), 127, device=dev, dtype=torch.uint8)
    return torch.zeros(shape, device=dev, dtype=_TYPE[typ]), torch.full(shape[:3], 127, device=dev, dtype=torch.uint8) if typ == "fp8" else None


def _laid_out(t, token_major):
    """The same [pages, kv heads, page, ...] tensor, in memory by head or by token."""
    if t is None or not token_major:
        return t
    bytes_ = t.view(torch.uint8) if t.element_size() == 1 else t
    return bytes_.transpose(1, 2).contiguous().transpose(1, 2).view(t.dtype)


def _projections(gen, tokens, heads, kv_heads, dim, typ, dev):
    """A projection's output: queries, keys with channels much larger than the others, and values beside each other."""
    wide = 1.0 + 7.0 * (torch.rand((kv_heads, dim), generator=gen, device=dev) < 0.03)
    x = torch.randn((tokens, heads + 2 * kv_heads, dim), generator=gen, device=dev)
    x[:, heads:heads + kv_heads] *= wide
    return x.to(typ).split((heads, kv_heads, kv_heads), dim=1)


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    op = case["op"]
    state = dict(op=op)
    if op in ("rotary", "rotary_write"):
        f = _frequencies(case)
        state.update(freqs=torch.tensor(f, dtype=torch.float64, device=dev), turns=torch.tensor(_turns(f), dtype=torch.int64, device=dev), interleaved=case["interleaved"],
                     magnitude=1.0 if case["factor"] == 1.0 else 0.1 * math.log(case["factor"]) + 1.0)
        T = case["tokens"]
        # a chunk's positions ascend, decodes have one each
        state["positions"] = case["far"] - T + torch.arange(T, device=dev) if case.get("chunk", T > 128) else torch.randint(0, case["far"], (T,), generator=gen, device=dev)
    if op == "rotary":
        state["x"] = torch.randn((T, case["heads"], case["dim"]), generator=gen, device=dev).to(_TYPE[case["q"]])
        return state
    h, d, page = case["kv_heads"], case["dim"], case["page"]
    tm = case.get("token_major", False)
    if op == "copy":
        shape = (case["layers"] * case["pages"], h, page, d)
        order = torch.randperm(case["pages"], generator=torch.Generator().manual_seed(seed))
        n = case["moves"]
        for name in ("k", "v"):
            x, e = _codes(gen, shape, case["cache"], dev)
            state[name], state[name + "_exp"] = x.unflatten(0, (case["layers"], -1)), None if e is None else e.unflatten(0, (case["layers"], -1))
        state.update(source=order[:1].expand(n).contiguous() if case["fork"] else order[:n].contiguous(), target=order[n:2 * n].contiguous(),
                     places=torch.full((n,), case["fork"]) if case["fork"] else None)
        return state
    if op in ("rotary_write", "store"):
        T = case["tokens"]
        pages = -(-T // page) + 3
        order = torch.randperm(pages, generator=gen, device=dev)
        at = torch.arange(T, device=dev)
        q, k, v = _projections(gen, T, case.get("heads", 0), h, d, _TYPE[case["q"]], dev)
        state.update(q=q, k_new=k, v_new=v, slots=order[at // page] * page + at % page, dtype=_TYPE[case["q"]])
        k, ke = _empty((pages, h, page, d), case["cache"], dev)
        v, ve = _empty((pages, h, page, d), case["cache"], dev)
    else:
        q_len, kv_len = _lens(case)
        need = [-(-n // page) for n in kv_len]
        pages = sum(need) + 1
        order = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
        table = torch.zeros((len(need), max(need)), dtype=torch.int32, device=dev)
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = order[at:at + n]
            at += n
        start = [0]
        for n in q_len:
            start.append(start[-1] + n)
        k, ke = _codes(gen, (pages, h, page, d), "fp4", dev)
        v, ve = _codes(gen, (pages, h, page, d), "fp4", dev)
        state.update(q=(2.0 * torch.randn((start[-1], case["heads"], d), generator=gen, device=dev)).to(_TYPE[case["q"]]), table=table,
                     q_start=torch.tensor(start, dtype=torch.int32, device=dev), kv_len=torch.tensor(kv_len, dtype=torch.int32, device=dev), q_lens=q_len,
                     kv_lens=kv_len, window=case["window"], page=page)
    state.update(k=_laid_out(k, tm), v=_laid_out(v, tm), k_exp=_laid_out(ke, tm), v_exp=_laid_out(ve, tm))
    return state


# ---- plain forms

def _plain_rotary(x, s):
    """Rows turned, fp32; the angles of far positions need 64 bits."""
    angle = s["positions"].double().unsqueeze(-1) * s["freqs"]
    cos, sin = (f(angle).float().unsqueeze(1) * s["magnitude"] for f in (torch.cos, torch.sin))
    n = s["freqs"].numel()
    x = x.float()
    part = x[..., :2 * n].unflatten(-1, (n, 2)).transpose(-1, -2) if s["interleaved"] else x[..., :2 * n].unflatten(-1, (2, n))
    a, b = part[..., 0, :], part[..., 1, :]
    turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1 if s["interleaved"] else -2).flatten(-2)
    return torch.cat((turned, x[..., 2 * n:]), -1)


def _plain_quantise8(x):
    """Codes (e4m3) and exponent bytes of rows: the least power of two that brings the row within 448."""
    x = x.float()
    most = x.abs().amax(-1, keepdim=True)
    fraction, e = torch.frexp(most)
    e = torch.where(fraction <= 0.875, e - 9, e - 8).clamp(-126, 127)
    e = torch.where(most == 0, torch.zeros_like(e), e)
    return torch.ldexp(x, -e).to(torch.float8_e4m3fn), (e + 127).squeeze(-1).to(torch.uint8)


def _plain_quantise4(x):
    """Codes (e2m1, two to a byte, the first in the lower half) and exponent bytes: 32 elements to the least power of two that brings them within 6."""
    x = x.float().unflatten(-1, (-1, 32))
    most = x.abs().amax(-1, keepdim=True)
    fraction, e = torch.frexp(most)
    e = torch.where(fraction <= 0.75, e - 3, e - 2).clamp(-126, 127)
    e = torch.where(most == 0, torch.zeros_like(e), e)
    y = torch.ldexp(x, -e)
    m = y.abs()
    # to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6; from the middle to the even code
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)).to(torch.uint8)
    code = (code + 8 * (y < 0).to(torch.uint8)).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], (e + 127).squeeze(-1).to(torch.uint8)


def _plain_values4(codes, exps):
    """fp32 values of e2m1 codes, two to a byte."""
    both = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()
    e, m = (both >> 1) & 3, both & 1
    size = torch.where(e == 0, 0.5 * m, torch.ldexp(1.0 + 0.5 * m, e - 1))
    return torch.ldexp((size * (1.0 - 2.0 * (both >> 3))).unflatten(-1, (-1, 32)), exps.int().unsqueeze(-1) - 127).flatten(-2)


def _plain_put(s, k, v):
    """Rows into the slots of the cache."""
    place = s["k"].shape[2]
    at, off = s["slots"] // place, s["slots"] % place
    for new, cache, exps in ((k, s["k"], s["k_exp"]), (v, s["v"], s["v_exp"])):
        if exps is None:
            cache[at, :, off] = new
        else:
            codes, e = (_plain_quantise4 if cache.dtype == torch.float4_e2m1fn_x2 else _plain_quantise8)(new)
            cache.view(torch.uint8)[at, :, off] = codes.view(torch.uint8)
            exps[at, :, off] = e


def _plain_rotary_write(s):
    # (keys are rounded to the activations' type before they are stored, as the queries are)
    q, k = (_plain_rotary(s[name], s).to(s["dtype"]) for name in ("q", "k_new"))
    _plain_put(s, k, s["v_new"])
    return _written(s, q)


def _written(s, q):
    """The queries and the cache; exponent bytes as the powers of two that they stand for."""
    out = dict(q=q, k=s["k"], v=s["v"])
    return out if s["k_exp"] is None else dict(out, k_exp=s["k_exp"].view(torch.float8_e8m0fnu), v_exp=s["v_exp"].view(torch.float8_e8m0fnu))


def _plain_store(s):
    _plain_put(s, s["k_new"], s["v_new"])
    place = s["k"].shape[2]
    at, off = s["slots"] // place, s["slots"] % place
    return tuple(_plain_values4(c.view(torch.uint8)[at, :, off], e[at, :, off]).to(s["dtype"]) for c, e in ((s["k"], s["k_exp"]), (s["v"], s["v_exp"])))


def _pages(cache, exps, pages):
    """Values of whole pages, fp32: [..., kv heads, tokens, dim] from page numbers [..., n]."""
    return _plain_values4(cache.view(torch.uint8)[pages.long()], exps[pages.long()]).movedim(-4, -3).flatten(-3, -2)


def _plain_softmax_product(score, value, keep):
    """softmax over the kept keys, times the values; zero where none is kept."""
    score = score.masked_fill(~keep, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    return torch.matmul(p, value) / p.sum(-1, keepdim=True).clamp_min(1e-30)


def _plain_attention(s):
    q, page, window = s["q"], s["page"], s["window"]
    heads, dim = q.shape[1:]
    kv_heads = s["k"].shape[1]
    group = heads // kv_heads
    n = sum(1 for v in s["q_lens"] if v == 1)   # the decodes come first
    out = torch.empty_like(q)
    scale = 1.0 / math.sqrt(dim)
    if n:
        used = -(-max(s["kv_lens"][:n]) // page)
        k = _pages(s["k"], s["k_exp"], s["table"][:n, :used])
        score = torch.matmul(q[:n].float().view(n, kv_heads, group, dim) * scale, k.transpose(-1, -2))
        del k
        pos = torch.arange(used * page, device=q.device)
        last = s["kv_len"][:n].view(n, 1, 1, 1) - 1
        keep = (pos <= last) & (pos > last - window) if window else pos <= last
        v = _pages(s["v"], s["v_exp"], s["table"][:n, :used])
        out[:n] = _plain_softmax_product(score, v, keep).view(n, heads, dim).to(q.dtype)
    if n < len(s["q_lens"]):                    # then one chunk
        rows, length = s["q_lens"][n], s["kv_lens"][n]
        used = -(-length // page)
        k = _pages(s["k"], s["k_exp"], s["table"][n, :used])[:, :length]
        v = _pages(s["v"], s["v_exp"], s["table"][n, :used])[:, :length]
        qc = q[n:].float().view(rows, kv_heads, group, dim).permute(1, 2, 0, 3).reshape(kv_heads, group * rows, dim) * scale
        score = torch.matmul(qc, k.transpose(-1, -2))
        pos = torch.arange(length, device=q.device)
        last = torch.arange(length - rows, length, device=q.device).view(rows, 1)
        keep = (pos <= last) & (pos > last - window) if window else pos <= last
        o = _plain_softmax_product(score.view(kv_heads, group, rows, length), v.unsqueeze(1), keep)
        out[n:] = o.permute(2, 0, 1, 3).reshape(rows, heads, dim).to(q.dtype)
    return out


def _plain_copy(s):
    source, target = (s[name].to(s["k"].device) for name in ("source", "target"))
    for c in (s["k"], s["v"], s["k_exp"], s["v_exp"]):
        if c is not None:
            c = c.view(torch.uint8) if c.element_size() == 1 else c
            if s["places"] is None:
                c[:, target] = c[:, source]
            else:
                n = int(s["places"][0])         # (a fork's are all the same)
                c[:, target, :, :n] = c[:, source, :, :n]
    return _layers(s)


def _layers(s):
    out = dict(k=s["k"], v=s["v"])
    return out if s["k_exp"] is None else dict(out, k_exp=s["k_exp"], v_exp=s["v_exp"])


def run(state):
    s = state
    if not own:
        if s["op"] == "rotary":
            return _plain_rotary(s["x"], s).to(s["x"].dtype)
        return {"rotary_write": _plain_rotary_write, "store": _plain_store, "attention": _plain_attention, "copy": _plain_copy}[s["op"]](s)
    from paper_2602_02987_amd import iteration
    if s["op"] == "rotary":
        return iteration.rotary(s["x"], s["positions"], s["turns"], interleaved=s["interleaved"], magnitude=s["magnitude"])
    if s["op"] == "rotary_write":
        q = iteration.rotary_write(s["q"], s["k_new"], s["v_new"], s["positions"], s["turns"], s["k"], s["v"], s["slots"], s["k_exp"], s["v_exp"],
                                   interleaved=s["interleaved"], magnitude=s["magnitude"])
        return _written(s, q)
    if s["op"] == "store":
        iteration.kv_write(s["k_new"], s["v_new"], s["k"], s["v"], s["slots"], s["k_exp"], s["v_exp"])
        return iteration.kv_read(s["k"], s["v"], s["slots"], s["k_exp"], s["v_exp"], dtype=s["dtype"])
    if s["op"] == "attention":
        return iteration.attention(s["q"], s["k"], s["v"], s["table"], s["q_start"], s["kv_len"], s["k_exp"], s["v_exp"], window=s["window"], max_q=max(s["q_lens"]))
    # a program has a cache for each layer
    exps = ([None] * len(s["k"]),) * 2 if s["k_exp"] is None else (s["k_exp"], s["v_exp"])
    iteration.copy_pages(list(zip(s["k"], s["v"], *exps)), s["source"], s["target"], s["places"])
    return _layers(s)


# ---- work and exact values

def _attended(q, kv, window):
    """(query, key) pairs of a request."""
    pairs = q * (kv - q + 1) + q * (q - 1) // 2
    return pairs - sum(max(0, kv - q + i + 1 - window) for i in range(q)) if window else pairs


def _row_bytes(case):
    d = case["dim"]
    return int(d * _LEAST_WORDS[case["cache"]]) + (1 if case["cache"] == "fp8" else d // 32 if case["cache"] == "fp4" else 0)


def work(case):
    op, d = case["op"], case["dim"]
    if op == "rotary":
        n = case["tokens"] * case["heads"]
        return {"bytes": 4 * n * d + 8 * case["tokens"], "flops": 3 * n * case["dims"]}
    if op == "copy":
        # a source is read once, however many targets it has
        places = case["fork"] or case["page"]
        each = 2 * case["layers"] * case["kv_heads"] * places * _row_bytes(case)
        return {"bytes": each * ((1 if case["fork"] else case["moves"]) + case["moves"]), "flops": 0}
    h = case["kv_heads"]
    if op == "rotary_write":
        T = case["tokens"]
        return {"bytes": T * (4 * case["heads"] * d + 2 * h * (2 * d + _row_bytes(case)) + 16), "flops": 3 * T * (case["heads"] + h) * case["dims"] + (3 * T * 2 * h * d if case["cache"] == "fp8" else 0)}
    if op == "store":                           # rows and codes are written and read
        n = 2 * case["tokens"] * h
        return {"bytes": n * (4 * d + 2 * _row_bytes(case)) + 16 * case["tokens"], "flops": 4 * n * d}
    q_len, kv_len = _lens(case)
    read = sum(min(kv, case["window"] + q - 1) if case["window"] else kv for q, kv in zip(q_len, kv_len))
    return {"bytes": 4 * sum(q_len) * case["heads"] * d + 2 * read * h * _row_bytes(case),
            "flops": 4 * d * case["heads"] * sum(_attended(q, kv, case["window"]) for q, kv in zip(q_len, kv_len))}


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_rotary(x, s, case):
    y = x.double()
    f = torch.tensor(_frequencies(case), dtype=torch.float64, device=x.device)
    n = f.numel()
    first = torch.arange(n, device=x.device) * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else n)
    z = torch.polar(torch.full_like(f, s["magnitude"]).expand(len(s["positions"]), n), s["positions"].double()[:, None] * f)[:, None]
    w = torch.complex(y[..., first], y[..., second]) * z
    y[..., first], y[..., second] = w.real, w.imag
    return y


def _exact_stored4(x):
    """What rows are after they were held in 4 bits."""
    x = x.double().unflatten(-1, (-1, 32))
    most = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(most, -126.0)
    for step in range(-126, 20):                # the least whole number with most <= 6 * 2^e
        e = torch.where(most > 6.0 * 2.0 ** step, torch.full_like(e, step + 1.0), e)
    unit = torch.pow(2.0, e)
    y = (x / unit).abs()
    best, far = torch.zeros_like(y), y.clone()
    for code in (1, 2, 3, 4, 5, 6, 7):          # (an even code takes a tie from the odd one before it, an odd one takes none)
        off = (y - _E2M1[code]).abs()
        closer = off <= far if code % 2 == 0 else off < far
        best, far = torch.where(closer, torch.full_like(y, _E2M1[code]), best), torch.minimum(off, far)
    return (torch.copysign(best, x) * unit).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    op, page = case["op"], case.get("page")
    if op == "rotary":
        return _exact_rotary(s["x"], s, case)
    if op == "rotary_write":
        out = dict(q=_exact_rotary(s["q"], s, case), k=None, v=None)
        if s["k_exp"] is not None:
            return dict(out, k_exp=None, v_exp=None)
        for name, rows in (("k", _exact_rotary(s["k_new"], s, case)), ("v", s["v_new"].double())):
            flat = s[name].double().transpose(1, 2).flatten(0, 1)
            flat[s["slots"]] = rows
            out[name] = flat.view(-1, page, *flat.shape[1:]).transpose(1, 2)
        return out
    if op == "store":
        return tuple(_exact_stored4(s[name]) for name in ("k_new", "v_new"))
    if op == "copy":                            # nothing is computed
        return None
    values = torch.tensor(_E2M1 + tuple(-x for x in _E2M1), dtype=torch.float64, device=s["q"].device)
    group = case["heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    t = 0
    for r, (n, length) in enumerate(zip(s["q_lens"], s["kv_lens"])):
        rows = s["table"][r, :-(-length // page)].long()
        for h in range(case["kv_heads"]):
            def gather(c, e):
                c = c.view(torch.uint8)[:, h][rows].flatten(0, 1)[:length].int()
                x = torch.empty((length, case["dim"]), dtype=torch.float64, device=c.device)
                x[:, 0::2], x[:, 1::2] = values[c % 16], values[c // 16]
                return x * torch.pow(2.0, e[:, h][rows].flatten(0, 1)[:length].double() - 127.0).repeat_interleave(32, -1)
            k, v = gather(s["k"], s["k_exp"]), gather(s["v"], s["v_exp"])
            j = torch.arange(length, device=k.device)
            pos = torch.arange(length - n, length, device=k.device)[:, None]
            hidden = j > pos
            if case["window"]:
                hidden |= j <= pos - case["window"]
            for g in range(h * group, (h + 1) * group):
                w = (s["q"][t:t + n, g].double() @ k.T / math.sqrt(case["dim"])).masked_fill(hidden, -math.inf).softmax(-1)
                out[t:t + n, g] = w @ v
        t += n
    return out
