"""The iteration operators on the GPU where tensors overlap, pages or exponents that nobody looks at are out of range, and pieces of work are many."""
import numpy as np
import pytest
import torch

import iteration_reference as R
from paper_2602_02987_amd import iteration as I
from test_gpu_iteration import DEV, _adapter_case, _adapters_close, _attention_case, _close, _reference

pytestmark = pytest.mark.gpu


# (type, rank, width, tokens of each request): as small as one launch does both products, then as large as two
IN_PLACE = [("bf16", 16, 1024, [1] * 127 + [1]), ("fp16", 32, 1032, [1] * 30 + [99, 0, 3]), ("bf16", 64, 520, [700]), ("bf16", 8, 512, [40, 1]), ("fp16", 24, 2048, [33]),
            ("bf16", 16, 4096, [1] * 128), ("fp16", 128, 776, [50, 1]), ("bf16", 32, 640, [2100, 1])]


@pytest.mark.parametrize("case", IN_PLACE, ids=lambda c: f"{c[0]}-r{c[1]}-{c[2]}-{sum(c[3])}t")
def test_adapters_on_their_own_input(case):
    """x, base and out are one tensor, or out lies over parts of x: every column of out needs all of x as it was."""
    t, rank, width, q_len = case
    which = [i % 4 - 1 if i % 5 else 1 for i in range(len(q_len))]
    data = list(_adapter_case((t, rank, width, width, 3, q_len, which), rank))
    data[1] = data[0]
    dev = [u.to(DEV) for u in data]
    for _ in range(3):
        y = dev[0].clone()
        assert I.adapters(y, y, *dev[2:], out=y) is y
        _adapters_close(y, data)
    # x and out side by side in one buffer; out eight columns into x; out three tokens behind x
    T = sum(q_len)
    room = torch.zeros((T + 3, 2 * width + 8), dtype=R.TYPES[t], device=DEV)
    for x, out in ((room[:T, :width], room[:T, width:2 * width]), (room[:T, :width], room[:T, 8:width + 8]), (room[:T, 8:width + 8], room[3:, :width])):
        room.zero_()
        x.copy_(dev[0])
        I.adapters(x, dev[1], *dev[2:], out=out)
        _adapters_close(out, data)


def test_adapters_overlap_with_other_strides():
    case = ("bf16", 16, 1024, 776, 2, [60, 1], [0, 1])
    data = _adapter_case(case, 5)
    dev = [u.to(DEV) for u in data]
    room = torch.zeros(61 * 2048, dtype=torch.bfloat16, device=DEV)
    x, out = room.view(61, 2048)[:, :1024], room[:61 * 776].view(61, 776)
    x.copy_(dev[0])
    I.adapters(x, *dev[1:], out=out)
    _adapters_close(out, data)


# ---- attention

# (heads, kv_heads, dim, page, q type, cache, new tokens, cached tokens, window)
WINDOWS = [(8, 2, 128, 16, "bf16", "bf16", [1, 3, 70], [1000, 333, 700], 51), (4, 1, 64, 1, "fp16", "fp8", [1, 1, 40], [300, 90, 150], 21), (4, 2, 256, 8, "bf16", "fp8", [2, 1, 30], [130, 65, 190], 3),
           (8, 2, 128, 32, "fp16", "fp16", [1, 17, 200], [97, 127, 500], 1), (2, 2, 64, 16, "bf16", "bf16", [1, 16], [2000, 900], 700)]


@pytest.mark.parametrize("case", WINDOWS, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}-page{c[3]}-{c[4]}-{c[5]}-{sum(c[6])}t-w{c[8]}")
def test_pages_before_every_window_do_not_matter(case):
    """A server has given away the pages that no token sees any more: their entries of the table are no pages."""
    case = (*case, False)
    q, cache, table, start, length, window = _attention_case(case, 31)
    k, v, ke, ve = cache
    gone = table.clone()
    for r, (n, kv) in enumerate(zip(case[6], case[7])):
        gone[r, :max(0, kv - n - window + 1) // case[3]] = -1
        gone[r, -(-kv // case[3]):] = -1
    assert (gone < 0).any()
    status = I.new_status(DEV)
    got = [I.attention(q.to(DEV), k, v, t.to(DEV), start.to(DEV), length.to(DEV), ke, ve, window=window, status=status) for t in (table, gone)]
    I.check(status)
    assert torch.equal(*got)
    _close(got[0], *_reference(q, cache, table, start, length, window))


@pytest.mark.parametrize("byte", [255, 0])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_exponents_that_nobody_looks_at(dim, byte):
    """The bytes of places beyond a request's last token and before its window are whatever the memory held."""
    for window in (0, 19):
        case = (4, 2, dim, 16, "bf16", "fp8", [1, 1, 3, 40], [50, 300, 29, 75], window, False)
        q, cache, table, start, length, _ = _attention_case(case, 37)
        ref = _reference(q, cache, table, start, length, window)
        k, v, ke, ve = cache
        seen = torch.zeros((k.shape[0], 16), dtype=torch.bool)
        for r, (n, kv) in enumerate(zip(case[6], case[7])):
            for j in range(max(0, kv - n - window + 1) if window else 0, kv):
                seen[int(table[r, j // 16]), j % 16] = True
        pages, places = (~seen).nonzero(as_tuple=True)
        for t, e in ((k, ke), (v, ve)):
            t.view(torch.uint8)[pages.to(DEV), :, places.to(DEV)] = 0x7F if byte else 0x38
            e[pages.to(DEV), :, places.to(DEV)] = byte
        got = I.attention(q.to(DEV), k, v, table.to(DEV), start.to(DEV), length.to(DEV), ke, ve, window=window)
        _close(got, *ref)


# ---- what is refused before anything is launched

def test_results_whose_rows_share_memory_are_refused():
    k, v, ke, ve = I.new_cache(4, 2, 16, 64, torch.float8_e4m3fn, device=DEV)
    slots = torch.tensor([0, 5, 17], device=DEV)
    rows = torch.ones((3, 2, 64), dtype=torch.bfloat16, device=DEV)
    start, length, table = (torch.tensor(n, dtype=torch.int32, device=DEV) for n in ([0, 3], [3], [[0]]))
    y = torch.ones((3, 64), dtype=torch.bfloat16, device=DEV)
    down, up = (torch.ones(s, dtype=torch.bfloat16, device=DEV) for s in ((2, 8, 64), (2, 64, 8)))
    a = (y, y, down, up, torch.ones(2, device=DEV), start, length - 3)
    one, head = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device=DEV).expand(3, 2, 64), torch.zeros((3, 1, 64), dtype=torch.bfloat16, device=DEV).expand(3, 2, 64)
    for call in (lambda: I.attention(rows, k, v, table, start, length, ke, ve, out=one), lambda: I.attention(rows, k, v, table, start, length, ke, ve, out=head),
                 lambda: I.kv_read(k, v, slots, ke, ve, k=one), lambda: I.kv_read(k, v, slots, ke, ve, v=head), lambda: I.adapters(*a, out=y[:1].expand(3, 64)),
                 lambda: I.kv_write(rows, rows, k[:, :1].expand(4, 2, 16, 64), v, slots, ke, ve), lambda: I.kv_write(rows, rows, k, v, slots, ke[:1].expand(4, 2, 16), ve)):
        with pytest.raises(ValueError, match="share memory"):
            call()
    # inputs may be expanded
    I.kv_write(one, head, k, v, slots, ke, ve)
    assert I.attention(one, k[:, :1].expand(4, 2, 16, 64), v, table, start, length, ke, ve).shape == (3, 2, 64)
    assert torch.equal(I.adapters(y[:1].expand(3, 64), *a[1:]), I.adapters(*a))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("q_len,kv_len", [([1, 1], [200, 47]), ([2, 60], [90, 150])])
def test_cached_rows_are_taken_as_they_are_read_back(dim, q_len, kv_len):
    """float16 queries over 8-bit rows whose exponents reach far below (rounded to multiples of 2^-24) and above what float16 holds exactly."""
    case = (4, 2, dim, 16, "fp16", "fp8", q_len, kv_len, 0, False)
    q, cache, table, start, length, _ = _attention_case(case, 73)
    k, v, ke, ve = cache
    gen = torch.Generator()
    gen.manual_seed(dim)
    for e, low in ((ke, 103), (ve, 106)):                       # keys around 2^-18, values around 2^-15, down to float16's last bits
        e.copy_(torch.randint(low, low + 5, e.shape, generator=gen).to(torch.uint8))
    scale = 2.0 ** 13 / dim ** 0.5                              # scores as usual
    slots = torch.arange(k.shape[0] * 16, device=DEV)
    read = [t.cpu().double().numpy().reshape(k.shape[0], 16, 2, dim).transpose(0, 2, 1, 3) for t in I.kv_read(k, v, slots, ke, ve, dtype=torch.float16)]
    exact = [R.cache_values(t, e) for t, e in ((k, ke), (v, ve))]
    assert (read[1] != exact[1]).any() and np.abs(read[1] - exact[1]).max() <= 2.0 ** -25
    got = I.attention(q.to(DEV), k, v, table.to(DEV), start.to(DEV), length.to(DEV), ke, ve, scale=scale)
    ref, parts = R.attention(q.double().numpy(), *read, table.numpy(), start.numpy(), length.numpy(), scale)
    _close(got, ref, R.attention_bound(ref, parts, torch.float16, dim))
    # values of 40000 and more, whose average float16 holds
    ve.fill_(127 + 7)
    read = [t.cpu().double().numpy().reshape(k.shape[0], 16, 2, dim).transpose(0, 2, 1, 3) for t in I.kv_read(k, v, slots, ke, ve, dtype=torch.float16)]
    assert np.abs(read[1]).max() > 4e4
    got = I.attention(q.to(DEV), k, v, table.to(DEV), start.to(DEV), length.to(DEV), ke, ve, scale=scale)
    ref, parts = R.attention(q.double().numpy(), *read, table.numpy(), start.numpy(), length.numpy(), scale)
    _close(got, ref, R.attention_bound(ref, parts, torch.float16, dim))
