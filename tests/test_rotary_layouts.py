"""Rows that are turned in place beside others, whatever the order in memory: what counts as apart, and that nothing but the rows is written."""
import ctypes as C
import random

import pytest
import torch

from paper_2602_02987_amd import iteration as I

EINVAL, BASE, DIM = I.SIM_EINVAL, 1 << 40, 64
no_gpu = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="the addresses are numbers: calls that are not refused have to end for want of a device")


def _refused(a, b, heads, tokens):
    """Whether rows a (first element, token stride, head stride) may not be turned into rows b."""
    t = I.TurnsC(DIM, 0, 0, 1.0, BASE)
    x, out = (I.RowsC(BASE + 2 * at, token, head) for at, token, head in (a, b))
    return I._lib().iter_rotary(0, heads, DIM, C.byref(t), BASE, tokens, C.byref(x), C.byref(out), None) == EINVAL


def _store_refused(q, k, v, heads, kv_heads, tokens):
    plane = I.PlaneC(8 * BASE, None, 16 * DIM * kv_heads, 16 * DIM, DIM, 0, 0, 0)
    c, t = I.CacheC(0, kv_heads, DIM, 16, 4, plane, plane), I.TurnsC(DIM, 0, 0, 1.0, BASE)
    q, k, v = (C.byref(I.RowsC(BASE + 2 * at, token, head)) for at, token, head in (q, k, v))
    return I._lib().iter_rotary_write(C.byref(c), 0, heads, C.byref(t), BASE, q, q, k, v, BASE, tokens, None) == EINVAL


def _share(a, b, heads, tokens):
    pieces = [[at + t * token + h * head for t in range(tokens) for h in range(heads)] for at, token, head in (a, b)]
    return any(abs(x - y) < DIM for x in pieces[0] for y in pieces[1])


@no_gpu
@pytest.mark.parametrize("tokens", [1, 2, 7])
@pytest.mark.parametrize("heads", [1, 2, 16])
def test_queries_keys_and_values_in_every_order(heads, tokens):
    d, h, n = DIM, heads, tokens
    orders = {"[tokens, 3, heads, dim]": (3 * h * d, d, h * d), "[tokens, heads, 3, dim]": (3 * h * d, 3 * d, d), "[3, tokens, heads, dim]": (h * d, d, n * h * d),
              "[heads, tokens, 3, dim]": (3 * d, n * 3 * d, d), "[heads, 3, tokens, dim]": (d, 3 * n * d, n * d), "[3, heads, tokens, dim]": (d, n * d, n * h * d),
              "[tokens, heads, 3, dim] with a gap behind a token": (3 * h * d + 8, 3 * d, d), "[tokens, heads, 3 dim + gap]": (h * (3 * d + 24), 3 * d + 24, d)}
    for name, (token, head, step) in orders.items():
        q, k, v = ((i * step, token, head) for i in range(3))
        assert not _store_refused(q, k, v, h, h, n), name
        assert not _refused(k, q, h, n) and not _refused(q, k, h, n) and not _refused(q, v, h, n) and not _refused(v, k, h, n), name
        shifted = (k[0] - 8, token, head)                             # the keys' rows are the queries' last elements
        if step == d:
            assert _store_refused(q, shifted, v, h, h, n) and _refused(q, shifted, h, n), name
        assert not _refused(q, q, h, n) and _refused(q, (8, token, head), h, n), name


@no_gpu
def test_fewer_keys_than_queries_and_one_head():
    # [tokens, 2 heads of q, 1 of k, 1 of v] and one head of each in turn
    for tokens in (1, 5):
        assert not _store_refused((0, 4 * DIM, DIM), (2 * DIM, 4 * DIM, 0), (3 * DIM, 4 * DIM, 0), 2, 1, tokens)
        assert not _store_refused((0, 3 * DIM, 0), (DIM, 3 * DIM, 0), (2 * DIM, 3 * DIM, 0), 1, 1, tokens)
        assert _store_refused((0, 4 * DIM, DIM), (DIM, 4 * DIM, 0), (3 * DIM, 4 * DIM, 0), 2, 1, tokens)
        # a head of keys between every two of queries, which are twice as many
        assert not _store_refused((0, 8 * DIM, 2 * DIM), (DIM, 8 * DIM, 4 * DIM), (3 * DIM, 8 * DIM, 4 * DIM), 4, 2, tokens)


@no_gpu
def test_rows_that_share_elements_are_refused_whatever_their_strides():
    r = random.Random(11)
    taken = shared = 0
    for _ in range(20000):
        heads, tokens = r.randint(1, 4), r.randint(1, 4)
        strides = [8 * r.choice([r.randint(0, 60), 8 * r.randint(0, 12)]) for _ in range(4)]
        token, head = strides[:2]
        other = (token, head) if r.random() < 0.6 else tuple(strides[2:])
        a, b = (4000, token, head), (4000 + 8 * r.randint(-150, 150), *other)
        if a == b or a[0] == b[0]:
            continue
        share = _share(a, b, heads, tokens)
        refused = _refused(a, b, heads, tokens)
        assert refused or not share, (a, b, heads, tokens)
        taken += not refused
        shared += share
    assert taken > 1000 and shared > 5000


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [1, 2, 37, 700])
@pytest.mark.parametrize("order", ["heads", "gap", "tokens"])
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float8_e4m3fn, torch.float4_e2m1fn_x2])
def test_in_place_where_queries_keys_and_values_alternate(tokens, order, kind):
    heads, dim, dev = 6, 128, "cuda:0"
    gen = torch.Generator().manual_seed(tokens)
    wide = torch.randn((heads, tokens, 3, dim) if order == "tokens" else (tokens, heads * 3 * dim + (8 if order == "gap" else 0)), generator=gen).to(torch.bfloat16).to(dev)
    x = wide.permute(1, 0, 2, 3) if order == "tokens" else wide[:, :heads * 3 * dim].unflatten(1, (heads, 3, dim))
    q, k, v = x.unbind(2)
    turns, at, slots = I.rotary_turns(I.rotary_frequencies(dim), dev), torch.arange(tokens, device=dev) * 3, torch.randperm(tokens, generator=gen).to(dev)
    pages = -(-tokens // 16)
    one, two = (I.new_cache(pages, heads, 16, dim, kind, dev) for _ in range(2))
    want = I.rotary_write(q.contiguous(), k.contiguous(), v.contiguous(), at, turns, one[0], one[1], slots, one[2], one[3])
    before, rest = wide.clone(), wide.clone()
    (rest.permute(1, 0, 2, 3) if order == "tokens" else rest[:, :heads * 3 * dim].unflatten(1, (heads, 3, dim)))[:, :, 0] = want
    assert I.rotary_write(q, k, v, at, turns, two[0], two[1], slots, two[2], two[3], out=q) is q
    assert torch.equal(wide.view(torch.int16), rest.view(torch.int16))                        # the queries turned, everything else as it was
    assert all(a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(one, two))
    wide.copy_(before)
    keys = I.rotary(k.contiguous(), at, turns)
    I.rotary(k, at, turns, out=q)                                                             # beside the rows that are read
    assert torch.equal(q.contiguous().view(torch.int16), keys.view(torch.int16)) and torch.equal(k, (before.permute(1, 0, 2, 3) if order == "tokens" else before[:, :heads * 3 * dim].unflatten(1, (heads, 3, dim)))[:, :, 1])
