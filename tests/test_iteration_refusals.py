"""What the iteration operators refuse on the host, before anything reaches a GPU. The pointers are numbers: a call that
went through would fail for want of a device, not with SIM_EINVAL."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2602_02987_amd import iteration as I

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ENOMEM = -1, -2
P = 1 << 20   # an aligned address that nothing reads


def _cache(typ=0, **kw):
    d = 128
    f = dict(type=typ, kv_heads=2, head_dim=d, page=16, pages=4)
    exp = (P, 2 * 16, 16, 1) if typ == 2 else (None, 0, 0, 0)
    plane = I.PlaneC(P, exp[0], 2 * 16 * d, 16 * d, d, *exp[1:])
    c = I.CacheC(k=plane, v=plane, **f)
    for name, value in kw.items():
        setattr(c, name, value)
    return c


def _plane(c, **kw):
    for name, value in kw.items():
        setattr(c.k, name, value)
    return c


def _rows(data=P, token=256, head=128):
    return I.RowsC(data, token, head)


def _batch(**kw):
    b = I.BatchC(2, 5, 4, P, P, P, 4, 4)
    for name, value in kw.items():
        setattr(b, name, value)
    return b


def _write(cache, typ=0, k=None, v=None, slots=P, tokens=5):
    L = I._lib()
    return L.iter_kv_write(C.byref(cache) if cache else None, typ, C.byref(k or _rows()), C.byref(v or _rows()), slots, tokens, None)


def test_the_library_exports_the_header_and_agrees_on_the_structures():
    header = open(os.path.join(ROOT, "include", "gnr_iter.h")).read()
    names = set(re.findall(r"^int (iter_[a-z_]+)\(", header, flags=re.M))
    assert {"iter_kv_write", "iter_kv_read", "iter_attention", "iter_attention_bytes", "iter_adapters", "iter_adapters_bytes"} <= names
    L = I._lib()
    for n in names:
        assert hasattr(L, n), n
    sizes = (C.c_size_t * 5)()
    assert L.iter_abi_sizes(sizes) == 0
    assert list(sizes) == [C.sizeof(s) for s in (I.PlaneC, I.CacheC, I.RowsC, I.BatchC, I.AdapterSetC)]
    assert L.iter_abi_sizes(None) == EINVAL


BAD_CACHES = [dict(type=3), dict(type=-1), dict(kv_heads=0), dict(head_dim=96), dict(head_dim=0), dict(page=0), dict(page=24), dict(page=1 << 17),
              dict(pages=-1), dict(pages=1 << 31)]
BAD_PLANES = [dict(data=None), dict(data=P + 8), dict(page_stride=-8), dict(head_stride=4), dict(place_stride=129), dict(page_stride=1 << 41), dict(place_stride=1 << 25),
              dict(exp=P)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_caches_that_are_refused(bad):
    assert _write(_cache(**bad)) == EINVAL


@pytest.mark.parametrize("bad", BAD_PLANES)
def test_planes_that_are_refused(bad):
    assert _write(_plane(_cache(), **bad)) == EINVAL
    if "exp" not in bad:
        c = _cache()
        for name, value in bad.items():
            setattr(c.v, name, value)
        assert _write(c) == EINVAL


def test_exponents_go_with_8_bits():
    assert _write(_plane(_cache(2), exp=None)) == EINVAL
    assert _write(_plane(_cache(2), exp_place_stride=-1)) == EINVAL and _write(_plane(_cache(2), exp_place_stride=1 << 25)) == EINVAL
    assert _write(_plane(_cache(2), place_stride=136)) == EINVAL    # rows of 8 bits are aligned to 16 bytes as well


def test_cache_calls_that_are_refused():
    L = I._lib()
    assert _write(None) == EINVAL
    assert _write(_cache(), typ=1) == EINVAL and _write(_cache(), typ=2) == EINVAL and _write(_cache(2), typ=2) == EINVAL
    assert _write(_cache(), tokens=-1) == EINVAL and _write(_cache(), slots=None) == EINVAL
    assert _write(_cache(), k=_rows(None)) == EINVAL and _write(_cache(), v=_rows(P + 2)) == EINVAL
    assert _write(_cache(), k=_rows(token=4)) == EINVAL and _write(_cache(), k=_rows(head=-128)) == EINVAL
    assert L.iter_kv_read(C.byref(_cache()), 1, C.byref(_rows()), C.byref(_rows()), P, 5, None) == EINVAL
    assert L.iter_kv_read(C.byref(_cache()), 0, None, C.byref(_rows()), P, 5, None) == EINVAL
    assert _write(_cache(), tokens=0, slots=None) == 0               # nothing to do


def _attend(cache=None, batch=None, typ=0, heads=4, q=None, out=None, scale=1.0, window=0, work=P, size=1 << 40):
    c, b = cache or _cache(), batch or _batch()
    return I._lib().iter_attention(C.byref(c), C.byref(b), typ, heads, C.byref(q or _rows()), C.byref(out or _rows(2 * P)), scale, window, work, size,
                                   None, None)


def test_attention_calls_that_are_refused():
    for bad in BAD_CACHES:
        assert _attend(_cache(**bad)) == EINVAL
    for bad in BAD_PLANES:
        assert _attend(_plane(_cache(), **bad)) == EINVAL
    for bad in (dict(requests=-1), dict(requests=1025), dict(tokens=-1), dict(tokens=1 << 31), dict(max_q=-1), dict(q_start=None), dict(kv_len=None),
                dict(page_table=None), dict(table_stride=-1), dict(table_width=-1), dict(table_width=1 << 31)):
        assert _attend(batch=_batch(**bad)) == EINVAL, bad
    assert _attend(heads=3) == EINVAL and _attend(heads=0) == EINVAL and _attend(heads=8192) == EINVAL
    assert _attend(typ=1) == EINVAL and _attend(typ=2) == EINVAL
    assert _attend(q=_rows(None)) == EINVAL and _attend(out=_rows(P + 4)) == EINVAL and _attend(q=_rows(token=100)) == EINVAL
    assert _attend(scale=float("nan")) == EINVAL and _attend(scale=float("inf")) == EINVAL and _attend(window=-1) == EINVAL
    need = C.c_size_t(0)
    L = I._lib()
    assert L.iter_attention_bytes(C.byref(_cache()), C.byref(_batch()), 4, None) == EINVAL
    assert L.iter_attention_bytes(C.byref(_cache()), C.byref(_batch()), 4, C.byref(need)) == 0
    if need.value:
        assert _attend(work=None) == EINVAL and _attend(work=P + 4) == EINVAL and _attend(size=need.value - 1) == ENOMEM
    assert _attend(batch=_batch(tokens=0)) == 0 and _attend(batch=_batch(tokens=0, requests=0)) == 0   # nothing to do
    assert _attend(batch=_batch(requests=0)) == EINVAL                  # tokens of nobody
    assert _attend(out=_rows()) == EINVAL                               # over the queries
    limit = 1 << 21
    assert _attend(batch=_batch(tokens=limit + 1)) == EINVAL and _attend(_cache(kv_heads=1), _batch(tokens=limit), heads=17) == EINVAL


def _adapt(typ=0, requests=2, tokens=5, q_start=P, adapter=P, x=P, xs=64, base=P, bs=128, out=P, os_=128, work=P, size=1 << 40, **kw):
    s = I.AdapterSetC(3, 16, 64, 128, P, P, P)
    for name, value in kw.items():
        setattr(s, name, value)
    return I._lib().iter_adapters(C.byref(s), typ, requests, tokens, q_start, adapter, x, xs, base, bs, out, os_, work, size, None, None)


def test_adapter_calls_that_are_refused():
    for bad in (dict(adapters=-1), dict(adapters=2049), dict(rank=0), dict(rank=12), dict(rank=136), dict(width_in=60), dict(width_in=0),
                dict(width_out=4), dict(width_out=130), dict(down=None), dict(up=None), dict(up=P + 8), dict(scale=None), dict(typ=2), dict(typ=-1),
                dict(requests=-1), dict(requests=1025), dict(tokens=-1), dict(q_start=None), dict(adapter=None), dict(x=None), dict(x=P + 2),
                dict(base=None), dict(out=None), dict(xs=60), dict(bs=-128), dict(os_=132)):
        assert _adapt(**bad) == EINVAL, bad
    need = C.c_size_t(0)
    s = I.AdapterSetC(3, 16, 64, 128, P, P, P)
    assert I._lib().iter_adapters_bytes(C.byref(s), 5, C.byref(need)) == 0
    if need.value:
        assert _adapt(work=None) == EINVAL and _adapt(size=need.value - 1) == ENOMEM
    assert _adapt(tokens=0) == 0 and _adapt(tokens=0, requests=0) == 0
    assert _adapt(requests=0) == EINVAL and _adapt(tokens=(1 << 21) + 1) == EINVAL


def test_the_binding_refuses_what_does_not_fit():
    k, v, ke, ve = I.new_cache(4, 2, 16, 64, torch.float8_e4m3fn, device="cpu")
    x, slots = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: I.kv_write(x, x, k, v, slots),                                      # no exponents
                 lambda: I.kv_write(x, x, k, v, slots, ke, ve),                              # not on a GPU
                 lambda: I.kv_write(x, x, k, v[:2], slots, ke, ve),
                 lambda: I.kv_read(k, v, slots, ke[:, :1], ve),
                 lambda: I.new_cache(4, 2, 16, 64, torch.float32, device="cpu"),
                 lambda: I.kv_read(k.view(torch.uint8), v.view(torch.uint8), slots)):
        with pytest.raises(ValueError):
            call()
    k, v, _, _ = I.new_cache(4, 2, 16, 64, device="cpu")
    i = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: I.attention(x.float(), k, v, i.view(1, 2), i, i[:1]), lambda: I.attention(x.half(), k, v, i.view(1, 2), i, i[:1]),
                 lambda: I.attention(x, k, v, i.view(1, 2), i, i[:1]), lambda: I.attention(x[0], k, v, i.view(1, 2), i, i[:1])):
        with pytest.raises(ValueError):
            call()
    y = torch.zeros(3, 64, dtype=torch.bfloat16)
    d = torch.zeros(2, 8, 64, dtype=torch.bfloat16)
    u = torch.zeros(2, 64, 8, dtype=torch.bfloat16)
    for call in (lambda: I.adapters(y, y, d, u, torch.ones(2), i, i[:1]), lambda: I.adapters(y, y.half(), d, u, torch.ones(2), i, i[:1]),
                 lambda: I.adapters(y, y, d, u.transpose(1, 2), torch.ones(2), i, i[:1]), lambda: I.adapters(y, y[:2], d, u, torch.ones(2), i, i[:1])):
        with pytest.raises(ValueError):
            call()


def test_tensors_that_require_gradients_are_refused():
    k, v, _, _ = I.new_cache(4, 2, 16, 64, device="cpu")
    i, slots = torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16, requires_grad=True)
    y, up = torch.zeros(3, 64, dtype=torch.bfloat16), torch.zeros(2, 64, 8, dtype=torch.bfloat16)
    down = torch.zeros(2, 8, 64, dtype=torch.bfloat16, requires_grad=True)
    for call in (lambda: I.kv_write(x, x, k, v, slots), lambda: I.attention(x, k, v, i.view(1, 2), i, i[:1]),
                 lambda: I.adapters(y, y, down, up, torch.ones(2), i, i[:1])):
        with pytest.raises(ValueError, match="backward"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):   # (the next thing that is wrong)
            call()


def test_check_says_what_was_out_of_range():
    s = I.new_status("cpu")
    I.check(s)
    s[0] = I.BAD_BATCH | I.BAD_PAGE
    with pytest.raises(I.SimError, match="batch bounds and page numbers") as e:
        I.check(s)
    assert e.value.code == EINVAL
    s[0] = I.BAD_ADAPTER
    with pytest.raises(I.SimError, match="adapter numbers"):
        I.check(s)
