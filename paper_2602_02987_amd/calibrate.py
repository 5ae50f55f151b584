"""Iteration-time coefficients of the simulator, measured: the attention block of a served model, run on the GPU with the iteration operators.

`python -m paper_2602_02987_amd.calibrate` times iterations of a prefill chunk and decodes and fits the simulator's law
c0 + c_pre * prefill_tokens + c_dec * n_decode to them; what it prints can be handed to `workloads.config(n, c0=..., c_pre=..., c_dec=...)`.

`Server` is the block itself: a paged cache (8-bit or as the activations), projections that all requests share (plain matrix products of the
library), an adapter for each class beside them, and attention of all tokens of an iteration over their requests' caches. A request can be
moved from the server of its prefill to the one of its decode. Weights are random: only sizes matter to the time. The law is that of a model's attention blocks on the
GPU: its feed-forward blocks and what the host does between launches are not in these times.
"""
from __future__ import annotations

import argparse
import json
import math
from dataclasses import dataclass
from typing import List, Sequence, Tuple

import numpy as np
import torch

from . import iteration


@dataclass
class Block:
    """Sizes of the block: `rank` and `classes` of the adapters, `page` tokens to a page of the cache."""
    heads: int = 32
    kv_heads: int = 8
    head_dim: int = 128
    rank: int = 16
    classes: int = 8
    page: int = 64
    dtype: torch.dtype = torch.bfloat16
    cache: torch.dtype = torch.float8_e4m3fn

    @property
    def width(self) -> int:
        return self.heads * self.head_dim


class Weights:
    """Random weights: query / key / value and output projection, and both projections' adapters, (down, up) each."""

    def __init__(self, block: Block, seed: int = 1, device="cuda"):
        gen = torch.Generator()
        gen.manual_seed(seed)
        b, dim = block, block.head_dim

        def of(*shape):
            return (torch.randn(shape, generator=gen) / math.sqrt(shape[-1])).to(b.dtype).to(device)
        into = (b.heads + 2 * b.kv_heads) * dim
        self.qkv, self.out = of(into, b.width), of(b.width, b.width)
        self.qkv_adapter = of(b.classes, b.rank, b.width), of(b.classes, into, b.rank)
        self.out_adapter = of(b.classes, b.rank, b.width), of(b.classes, b.width, b.rank)
        self.scale = torch.ones(b.classes, device=device)

    def copy(self) -> "Weights":
        """The same numbers in other memory."""
        w = Weights.__new__(Weights)
        for name, value in vars(self).items():
            setattr(w, name, tuple(t.clone() for t in value) if isinstance(value, tuple) else value.clone())
        return w

    def bytes(self) -> int:
        return sum(t.nbytes for value in vars(self).values() for t in (value if isinstance(value, tuple) else (value,)))


@dataclass
class Plan:
    """An iteration's batch on the device (`Server.plan`)."""
    q_start: torch.Tensor
    kv_len: torch.Tensor
    table: torch.Tensor
    slots: torch.Tensor
    adapter: torch.Tensor
    tokens: int
    longest: int


class Server:
    """The block with a cache of `pages` pages. Requests are numbers; each has a class (its adapter), pages and a length."""

    def __init__(self, block: Block, weights: Weights, pages: int, device="cuda"):
        self.block, self.weights, self.device = block, weights, torch.device(device)
        self.k, self.v, self.k_exp, self.v_exp = iteration.new_cache(pages, block.kv_heads, block.page, block.head_dim, block.cache, device)
        self.status = iteration.new_status(device)
        self._free = list(range(pages))[::-1]
        self._pages, self._length, self._class = {}, {}, {}
        self._next = 0

    def bytes(self) -> int:
        """Of the cache."""
        return sum(t.nbytes for t in (self.k, self.v, self.k_exp, self.v_exp) if t is not None)

    def copy_cache(self, other: "Server") -> None:
        """Contents of another server's cache of the same size."""
        for name in ("k", "v", "k_exp", "v_exp"):
            mine, its = getattr(self, name), getattr(other, name)
            if mine is not None and mine is not its:
                mine.copy_(its)

    def admit(self, which: int) -> int:
        """A request of class `which` (-1: without an adapter) that has no tokens yet."""
        r, self._next = self._next, self._next + 1
        self._pages[r], self._length[r], self._class[r] = [], 0, which
        return r

    def length(self, r: int) -> int:
        return self._length[r]

    def leave(self, r: int) -> None:
        self._free += self._pages.pop(r)
        del self._length[r], self._class[r]

    def _missing(self, r: int, n: int) -> int:
        """Pages that request r lacks for n tokens more."""
        return -(-(self._length[r] + n) // self.block.page) - len(self._pages[r])

    def _grow(self, r: int, n: int) -> range:
        """Room for n tokens more; their positions."""
        at, missing = self._length[r], self._missing(r, n)
        self._need(missing)
        self._pages[r] += [self._free.pop() for _ in range(missing)]
        self._length[r] = at + n
        return range(at, at + n)

    def _need(self, pages: int) -> None:
        if pages > len(self._free):
            raise MemoryError(f"the cache has {len(self._free)} pages left, {pages} are needed")

    def _slots(self, r: int, positions: Sequence[int]) -> List[int]:
        page, pages = self.block.page, self._pages[r]
        return [pages[j // page] * page + j % page for j in positions]

    def _whole(self, numbers, dtype) -> torch.Tensor:
        return torch.tensor(numbers, dtype=dtype).to(self.device)

    def plan(self, batch: Sequence[Tuple[int, int]]) -> Plan:
        """Makes room for an iteration that brings n tokens of request r for every (r, n): 1 for a decode, a chunk's for the prefill. A batch that does not
        fit raises MemoryError and leaves every request as it was: a longer one would have tokens that were never written."""
        if len({r for r, _ in batch}) < len(batch):
            raise ValueError("a batch has a request once at most: the positions of its tokens are the last ones of its cache")
        if any(n < 0 for _, n in batch):
            raise ValueError("a request cannot bring fewer than no tokens")
        self._need(sum(self._missing(r, n) for r, n in batch))
        slots, start = [], [0]
        for r, n in batch:
            slots += self._slots(r, self._grow(r, n))
            start.append(start[-1] + n)
        width = max([len(self._pages[r]) for r, _ in batch] + [1])
        i32 = torch.int32
        return Plan(self._whole(start, i32), self._whole([self._length[r] for r, _ in batch], i32),
                    self._whole([self._pages[r] + [0] * (width - len(self._pages[r])) for r, _ in batch], i32).view(len(batch), width),
                    self._whole(slots, torch.int64), self._whole([self._class[r] for r, _ in batch], i32), start[-1],
                    max([n for _, n in batch] + [0]))

    @torch.no_grad()
    def iterate(self, x: torch.Tensor, p: Plan) -> torch.Tensor:
        """The block's output for the activations x [tokens, width] of a plan's tokens; their keys and values go to the cache."""
        b, w = self.block, self.weights
        qkv = x @ w.qkv.T
        iteration.adapters(x, qkv, *w.qkv_adapter, w.scale, p.q_start, p.adapter, out=qkv, status=self.status)
        rows = qkv.view(p.tokens, b.heads + 2 * b.kv_heads, b.head_dim)
        q, k, v = rows.split((b.heads, b.kv_heads, b.kv_heads), dim=1)
        iteration.kv_write(k, v, self.k, self.v, p.slots, self.k_exp, self.v_exp)
        o = iteration.attention(q, self.k, self.v, p.table, p.q_start, p.kv_len, self.k_exp, self.v_exp, max_q=p.longest, status=self.status)
        o = o.view(p.tokens, b.width)
        y = o @ w.out.T
        return iteration.adapters(o, y, *w.out_adapter, w.scale, p.q_start, p.adapter, out=y, status=self.status)

    @torch.no_grad()
    def move(self, r: int, to: "Server") -> int:
        """Moves a request with its cache to another server; its number there. If that one has no room for it, or a cache that is not
        made for its rows, nothing changes on either."""
        n = self._length[r]
        to._need(-(-n // to.block.page))
        k, v = iteration.kv_read(self.k, self.v, self._whole(self._slots(r, range(n)), torch.int64), self.k_exp, self.v_exp, dtype=self.block.dtype)
        there = to.admit(self._class[r])
        slots = to._whole(to._slots(there, to._grow(there, n)), torch.int64)
        try:
            iteration.kv_write(k, v, to.k, to.v, slots, to.k_exp, to.v_exp)
        except Exception:
            to.leave(there)
            raise
        self.leave(r)
        return there


def fit(samples: Sequence[Tuple[int, int, float]]) -> dict:
    """Least squares of c0 + c_pre * prefill_tokens + c_dec * n_decode to (prefill_tokens, n_decode, seconds), none of the three below zero;
    `residual` is the largest deviation relative to the sample."""
    from scipy.optimize import nnls
    s = np.asarray(samples, dtype=np.float64)
    a = np.stack([np.ones(len(s)), s[:, 0], s[:, 1]], 1)
    size = np.abs(a).max(0).clip(min=1.0)                       # (columns of one magnitude)
    c = nnls(a / size, s[:, 2])[0] / size
    return dict(c0=float(c[0]), c_pre=float(c[1]), c_dec=float(c[2]), residual=float((np.abs(a @ c - s[:, 2]) / s[:, 2]).max()))


_LAST_LEVEL_CACHE = 256 << 20


def measure(block: Block, chunks: Sequence[int], decodes: Sequence[int], context: int, passes: int = 20, device="cuda", layers: int = 32) -> List[Tuple[int, int, float]]:
    """Seconds of an iteration of one block on the GPU for every (chunk, decodes) but (0, 0), every request with `context` tokens before it.

    A model goes through the weights and caches of all its layers before it comes back to one's, so the passes go through as many blocks as a model of `layers` layers
    has, or as few as are twice the chip's last-level cache. What the host takes to launch an iteration, which is longer than one of a few tokens runs, is not in the
    times: all passes are queued before the first begins."""
    most = max(decodes) + 1
    pages = most * -(-(context + max(chunks) + 1) // block.page)
    first = Weights(block, device=device)
    servers = [Server(block, first, pages, device)]
    each = first.bytes() + servers[0].bytes()
    fit_in = 1 + int(0.75 * torch.cuda.mem_get_info(device)[0]) // each     # (with the longest caches fewer have to do)
    servers += [Server(block, first.copy(), pages, device) for _ in range(min(layers, fit_in, -(-2 * _LAST_LEVEL_CACHE // first.bytes())) - 1)]
    gen = torch.Generator(device=device)
    gen.manual_seed(1)
    room = torch.zeros(1 << 28, device=device)                  # 1 GiB, to keep the GPU busy while passes are queued
    samples = []
    for chunk in chunks:
        for n in decodes:
            if chunk + n == 0:
                continue
            before = torch.randn((context, block.width), generator=gen, device=device).to(block.dtype)
            plans = []
            for s in servers:
                requests = [s.admit(i % block.classes) for i in range(n + (chunk > 0))]
                for r in requests:                              # what came before: the same pages on every server, written on one
                    p = s.plan([(r, context)])
                    if s is servers[0]:
                        s.iterate(before, p)
                s.copy_cache(servers[0])
                plans.append(s.plan([(r, 1) for r in requests[:n]] + [(r, chunk) for r in requests[n:]]))
            x = torch.randn((plans[0].tokens, block.width), generator=gen, device=device).to(block.dtype)

            def run(count):                                     # (the same tokens again: an iteration's time does not depend on that)
                for i in range(count):
                    servers[i % len(servers)].iterate(x, plans[i % len(servers)])
            run(3)
            samples.append((chunk, n, _seconds_ahead(lambda: run(passes), room) / passes))
            for s in servers:
                for r in list(s._length):
                    s.leave(r)
    for s in servers:
        iteration.check(s.status)
    return samples


def _seconds_ahead(run, room: torch.Tensor) -> float:
    """Seconds that the GPU takes for what run() launches, all of which the host has launched by the time the GPU begins with it."""
    for fills in (8, 32, 128, 512):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        for _ in range(fills):
            room.add_(1.0)
        begin.record()
        run()
        end.record()
        late = begin.query()
        end.synchronize()
        if not late:
            return begin.elapsed_time(end) / 1e3
    raise RuntimeError("the host does not get ahead of the GPU: measure fewer passes at a time")


def main() -> None:
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--chunks", type=int, nargs="+", default=[0, 64, 128, 256], help="prefill tokens of an iteration")
    a.add_argument("--decodes", type=int, nargs="+", default=[0, 16, 32, 64, 127], help="decodes of an iteration")
    a.add_argument("--context", type=int, default=1024, help="tokens each request has in its cache")
    a.add_argument("--layers", type=int, default=32, help="blocks of the model, by which the times are multiplied")
    a.add_argument("--cache", choices=["fp8", "bf16"], default="fp8")
    o = a.parse_args()
    block = Block(cache=torch.float8_e4m3fn if o.cache == "fp8" else torch.bfloat16)
    samples = [(c, n, t * o.layers) for c, n, t in measure(block, o.chunks, o.decodes, o.context, layers=o.layers)]
    print(json.dumps(dict(fit(samples), of="attention blocks", layers=o.layers, context=o.context, cache=o.cache, samples=[dict(chunk=c, decodes=n, seconds=t) for c, n, t in samples])))


if __name__ == "__main__":
    main()
