"""Attention where a workgroup has many blocks of keys, and where rows are computed again, against 64 bits on the GPU.

Few rows: pieces of more than 32 blocks of 128 keys (a wave looks up the pages of 32 at a time). Chunks: pieces of more than 17 blocks of 64 keys (pages of 16 at a
time, two buffers that take turns), and more tiles than workgroups. A batch has that many when its blocks of keys, over the kv heads, exceed as many times the workgroups
of a launch: 256 for each that a compute unit holds (256 elements a head: 1; 128: 2; 64: 3 for few rows, 2 for chunks)."""
import math

import pytest
import torch

import iteration_reference as R
from paper_2602_02987_amd import iteration as I
from test_gpu_iteration import DEV

pytestmark = pytest.mark.gpu


def _case(c, seed, rising=True):
    """Requests whose pages are the same ones in another order; keys grow along the first one, so that its running maximum keeps moving."""
    heads, kv_heads, dim, place, qt, kind, q_len, kv_len, _ = c
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    pages = max(-(-n // place) for n in kv_len) + 1
    shape = (pages, kv_heads, place, dim)
    grow = torch.linspace(0.2, 6.0 if rising else 0.2, pages, device=DEV).view(pages, 1, 1, 1)
    ke = ve = None
    if kind == "fp8":
        k, v = ((100 * torch.randn(shape, generator=gen, device=DEV)).clamp(-448, 448).to(torch.float8_e4m3fn) for _ in range(2))
        ke, ve = (torch.randint(117, 120, shape[:3], generator=gen, device=DEV) for _ in range(2))
        ke = (ke + (grow[..., 0] / 2).long()).to(torch.uint8)
        ve = ve.to(torch.uint8)
    else:
        k, v = ((torch.randn(shape, generator=gen, device=DEV) * g).to(R.TYPES[kind]) for g in (grow, 1.0))
    table = torch.stack([torch.arange(pages, device=DEV)] + [torch.randperm(pages, generator=gen, device=DEV) for _ in q_len[1:]]).to(torch.int32)
    start = torch.tensor([sum(q_len[:i]) for i in range(len(q_len) + 1)], dtype=torch.int32, device=DEV)
    q = (2 * torch.randn((sum(q_len), heads, dim), generator=gen, device=DEV)).to(R.TYPES[qt])
    return q, (k, v, ke, ve), table, start, torch.tensor(kv_len, dtype=torch.int32, device=DEV)


def _values(codes, exps):
    if exps is None:
        return codes.double()
    e4m3 = torch.from_numpy(R.E4M3).to(codes.device)
    return e4m3[codes.view(torch.uint8).long()] * torch.pow(2.0, exps.double() - 127.0).unsqueeze(-1)


def _reference(q, cache, table, start, length, window=0, scale=None, absent=None):
    """(out, bound) in 64 bits; absent[r]: numbers of request r's pages that count as not there."""
    k, v = _values(cache[0], cache[2]), _values(cache[1], cache[3])
    heads, dim = q.shape[1:]
    group, place = heads // k.shape[1], k.shape[2]
    scale = 1.0 / math.sqrt(dim) if scale is None else scale
    out, spread, most, total, reach = (torch.zeros(q.shape, dtype=torch.float64, device=DEV) for _ in range(5))
    for r, n in enumerate(length.tolist()):
        a, b = int(start[r]), int(start[r + 1])
        rows = table[r, :-(-n // place)].long().clamp(0, k.shape[0] - 1)
        pos, j = torch.arange(n - b + a, n, device=DEV)[:, None], torch.arange(n, device=DEV)
        seen = j <= pos
        if window:
            seen = seen & (j > pos - window)
        for page in (absent or {}).get(r, []):
            seen = seen & (j // place != page)
        for h in range(heads):
            kk, vv = (t[rows, h // group].flatten(0, 1)[:n] for t in (k, v))
            s = (torch.matmul(q[a:b, h].double(), kk.T) * scale).masked_fill(~seen, -math.inf)
            w = torch.exp(s - s.amax(-1, keepdim=True).clamp_min(-1e300))
            w = w / w.sum(-1, keepdim=True).clamp_min(1e-300)
            out[a:b, h], spread[a:b, h], most[a:b, h] = torch.matmul(w, vv), torch.matmul(w, vv.abs()), torch.matmul(seen.double(), vv.abs())
            total[a:b, h] = (torch.matmul(q[a:b, h].double().abs(), kk.abs().T) * seen).amax(-1, keepdim=True) * abs(scale)
            reach[a:b, h] = seen.sum(-1, keepdim=True).double()
    on_cpu = [t.cpu().numpy() for t in (out, spread, most, total, reach)]
    return out, torch.from_numpy(R.attention_bound(on_cpu[0], on_cpu[1:], q.dtype, dim)).to(DEV)


def _close(got, ref, bound, where=None):
    over = (got.double() - ref).abs() - bound
    over = over if where is None else over[where]
    assert bool((over <= 0).all()), float(over.max())            # (a NaN is not within it either)


def _attend(q, cache, table, start, length, **kw):
    k, v, ke, ve = cache
    return I.attention(q, k, v, table, start, length, ke, ve, **kw)


def _id(c):
    return f"{c[0]}x{c[1]}x{c[2]}-page{c[3]}-{c[4]}-{c[5]}-{len(c[6])}r{sum(c[6])}t{max(c[7])}k-w{c[8]}"


LONG = [33000 - 101 * i for i in range(14)]
# (heads, kv_heads, dim, page, q type, cache, new tokens, cached tokens, window)
MANY = [
    # few rows: 33 to 42 blocks a piece
    (16, 8, 64, 16, "fp16", "fp16", [1] * 14, LONG, 0), (16, 8, 64, 64, "bf16", "fp8", [1] * 14, LONG, 0),
    (32, 8, 128, 64, "bf16", "bf16", [1] * 10, LONG[:10], 0), (56, 8, 128, 16, "fp16", "fp8", [1, 2] * 5, LONG[:10], 0),
    (16, 8, 256, 16, "bf16", "fp8", [1, 2, 1, 1, 8], [35000, 36001, 34000, 35500, 30000], 0), (16, 8, 256, 128, "fp16", "fp16", [1] * 5, [35000, 36001, 34000, 35500, 30000], 0),
    (32, 8, 128, 8, "bf16", "bf16", [1] * 10, LONG[:10], 0), (32, 8, 128, 4, "bf16", "fp8", [1] * 10, LONG[:10], 0),
    (32, 8, 128, 16, "bf16", "bf16", [1, 3] * 6, LONG[:12], 25000),
    # chunks whose keys are cut into pieces of 20 blocks
    (32, 8, 64, 16, "bf16", "bf16", [250], [9900], 0), (32, 8, 64, 64, "fp16", "fp8", [250], [9900], 0),
    (32, 8, 128, 16, "fp16", "fp16", [250], [9900], 0), (32, 8, 128, 64, "bf16", "bf16", [250], [9900], 0),
    (32, 8, 128, 16, "bf16", "fp8", [250], [9900], 0), (32, 8, 128, 64, "fp16", "fp8", [250], [9900], 0),
    (32, 8, 256, 16, "bf16", "bf16", [250], [5000], 0), (32, 8, 256, 64, "fp16", "fp8", [250], [5000], 0),
    (32, 8, 128, 8, "bf16", "bf16", [250], [9900], 0), (32, 8, 128, 1, "fp16", "fp8", [250], [9900], 0),
    # more tiles than workgroups, none of them cut
    (32, 8, 64, 16, "fp16", "fp16", [2090], [2090], 0), (32, 8, 64, 16, "bf16", "fp8", [2090], [2090], 0),
    (32, 8, 128, 64, "bf16", "bf16", [2090], [2090], 0), (32, 8, 128, 64, "bf16", "fp8", [2090], [2100], 0), (32, 8, 128, 16, "fp16", "fp16", [2090], [2090], 700),
    (32, 8, 256, 32, "bf16", "bf16", [1100], [1100], 0), (32, 8, 256, 16, "bf16", "fp8", [1100], [1100], 0), (32, 8, 128, 4, "bf16", "bf16", [2090], [2090], 0),
    # both kernels
    (32, 8, 128, 64, "bf16", "bf16", [1] * 30 + [300, 700], [3000] * 30 + [12000, 900], 0), (28, 4, 128, 16, "fp16", "fp8", [1] * 40 + [600], [5000] * 40 + [9000], 4000),
]


@pytest.mark.parametrize("case", MANY, ids=_id)
def test_many_blocks_of_keys(case):
    data = _case(case, 41)
    status = I.new_status(DEV)
    got = _attend(*data, window=case[8], max_q=max(case[6]), status=status)
    I.check(status)
    _close(got, *_reference(*data, case[8]))


@pytest.mark.parametrize("case", [c for c in MANY if c[3] >= 16 and c[6] in ([250], [2090], [1100])], ids=_id)
def test_a_value_that_is_no_number_in_the_midst_of_many_blocks(case):
    """What the tokens before it do not see does not matter to them; the others get it in its place and nowhere else."""
    data = _case(case, 43, rising=False)
    q, cache, table, start, length = data
    ref, bound = _reference(*data, case[8])
    tokens, n = case[6][0], case[7][0]
    first, group = n - tokens, case[0] // case[1]
    at = first + tokens // 2 + 3                                   # a position within the chunk
    page, place = int(table[0, at // case[3]]), at % case[3]
    _, v, _, ve = cache
    if ve is None:
        v[page, 1, place, 9] = math.nan
    else:
        v.view(torch.uint8)[page, 1, place, 9] = 0x7F
    got = _attend(*data, window=case[8])
    pos = torch.arange(first, n, device=DEV)
    sees = torch.zeros(q.shape, dtype=torch.bool, device=DEV)
    sees[(pos >= at) & (pos < at + case[8] if case[8] else pos >= at), group:2 * group, 9] = True
    assert bool(got[sees].isnan().all())
    _close(got, ref, bound, ~sees)


# Rows that the join computes again: (heads, kv_heads, dim, page, q type, cache, new tokens, cached tokens, window); requests of two to four tokens, cut (more
# than 128 keys) and whole
AGAIN = [(4, 2, 64, 16, "bf16", "bf16", [1, 3, 2], [40, 700, 90], 0), (8, 2, 128, 16, "fp16", "fp8", [4, 1, 2], [500, 300, 33], 0), (4, 2, 256, 16, "bf16", "fp8", [2, 4, 1], [40, 1000, 20], 0),
         (6, 2, 64, 8, "fp16", "fp8", [3, 1, 4], [300, 40, 60], 0), (8, 2, 128, 64, "bf16", "bf16", [4, 2, 1], [1500, 70, 10], 0), (4, 2, 256, 16, "fp16", "fp16", [3, 2, 1], [70, 600, 300], 37),
         (12, 2, 128, 16, "bf16", "fp8", [2, 1, 2], [100, 300, 400], 50)]


@pytest.mark.parametrize("scale", [None, -0.13])
@pytest.mark.parametrize("case", AGAIN, ids=_id)
def test_few_tokens_of_which_some_see_a_value_that_is_no_number(case, scale):
    data = _case(case, 47, rising=False)
    q, (k, v, ke, ve), table, start, length = data
    table[1:] += k.shape[0]                                        # every request with pages of its own
    table[2:] += k.shape[0]
    cache = tuple(None if t is None else torch.cat([t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t] * 3).view(t.dtype) for t in (k, v, ke, ve))
    data = q, cache, table, start, length
    ref, bound = _reference(*data, case[8], scale)
    group, window = case[0] // case[1], case[8]
    sees = torch.zeros(q.shape, dtype=torch.bool, device=DEV)
    for r, (n, kv) in enumerate(zip(case[6], case[7])):
        # the last token's own place; with a window also the first one of the first token's, which the others do not see
        for at, d in [(kv - 1, 5)] + ([(kv - n - window + 1, 6)] if window else []):
            if at < 0:
                continue
            page, place = int(table[r, at // case[3]]), at % case[3]
            if ve is None:
                cache[1][page, 1, place, d] = math.inf
            else:
                cache[1].view(torch.uint8)[page, 1, place, d] = 0xFF
            token = int(start[r]) + (n - 1 if d == 5 else 0)
            sees[token, group:2 * group, d] = True
    got = _attend(*data, window=window, scale=scale)
    assert not bool(got[sees].isfinite().any())
    _close(got, ref, bound, ~sees)


@pytest.mark.parametrize("scale", [None, -0.13])
@pytest.mark.parametrize("bad", [-1, 2 ** 31 - 1])
@pytest.mark.parametrize("case", AGAIN + [(8, 2, 64, 16, "bf16", "bf16", [1, 1, 60], [100, 900, 200], 0), (4, 2, 256, 16, "bf16", "fp8", [1, 40, 1], [60, 200, 300], 0),
                                          (8, 2, 128, 4, "bf16", "fp8", [1, 1, 50], [30, 700, 90], 0)], ids=_id)
def test_pages_that_are_missing_count_as_absent(case, bad, scale):
    data = _case(case, 53, rising=False)
    q, cache, table, start, length = data
    absent = {}
    for r, (n, kv) in enumerate(zip(case[6], case[7])):
        # the last page, and one in the midst of what is seen
        seen = (max(0, kv - n - case[8] + 1) if case[8] else 0) // case[3], (kv - 1) // case[3]
        absent[r] = sorted({seen[1], (seen[0] + seen[1]) // 2} if r != 1 else {(seen[0] + seen[1]) // 2})
        for page in absent[r]:
            table[r, page] = bad
    status = I.new_status(DEV)
    got = _attend(*data, window=case[8], scale=scale, status=status)
    assert int(status.item()) == I.BAD_PAGE
    _close(got, *_reference(*data, case[8], scale, absent))


def test_as_many_requests_as_a_batch_can_have():
    """1024 requests of all kinds: what the kernels keep for each of them still fits beside their tiles, for every head size."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(59)
    for dim, kind in ((64, "bf16"), (128, "fp8"), (256, "bf16"), (256, "fp8")):
        q_len = [(1, 1, 2, 0, 1, 20)[i % 6] for i in range(1024)]
        case = (4, 1, dim, 16, "bf16", kind, q_len, [n + 7 * i % 90 for i, n in enumerate(q_len)], 0)
        data = _case(case, 61, rising=False)
        status = I.new_status(DEV)
        got = _attend(*data, status=status)
        I.check(status)
        _close(got, *_reference(*data))


@pytest.mark.parametrize("rank", [16, 64, 128])
@pytest.mark.parametrize("tokens", [1024, 3000])
def test_as_many_adapters_as_a_set_can_have(rank, tokens):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(rank)
    n, width, out = 2048, 64, 520
    which = torch.randint(-1, n, (1024,), generator=gen, device=DEV, dtype=torch.int32)
    start = (torch.arange(1025, device=DEV) * tokens // 1024).to(torch.int32)
    x, base, down, up = ((torch.randn(s, generator=gen, device=DEV) * by).bfloat16() for s, by in (((tokens, width), 1.0), ((tokens, out), 1.0), ((n, rank, width), width ** -0.5),
                                                                                                 ((n, out, rank), rank ** -0.5)))
    scale = 0.5 + torch.rand(n, generator=gen, device=DEV)
    status = I.new_status(DEV)
    got = I.adapters(x, base, down, up, scale, start, which, status=status)
    I.check(status)
    a = which[torch.searchsorted(start, torch.arange(tokens, device=DEV, dtype=torch.int32), right=True) - 1].long()
    ref, inner, outer = base.double().clone(), torch.zeros_like(base, dtype=torch.float64), torch.zeros_like(base, dtype=torch.float64)
    for t in range(tokens):
        if a[t] >= 0:
            d, u, s, row = down[a[t]].double(), up[a[t]].double(), scale[a[t]].double(), x[t].double()
            h = d @ row
            ref[t] += s * (u @ h)
            inner[t], outer[t] = s * (u.abs() @ (d.abs() @ row.abs())), s * (u.abs() @ h.abs())
    on_cpu = [t.cpu().double().numpy() for t in (ref, base, inner, outer)]
    bound = R.adapters_bound(*on_cpu, torch.bfloat16, width, rank)
    _close(got, ref, torch.from_numpy(bound).to(DEV))
