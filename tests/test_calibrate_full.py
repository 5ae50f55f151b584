"""Servers of the calibration whose cache is full: what does not fit changes nothing."""
import pytest
import torch

from paper_2602_02987_amd import calibrate as K
from paper_2602_02987_amd import iteration as I


def _state(s):
    return dict(s._length), {r: list(p) for r, p in s._pages.items()}, sorted(s._free), dict(s._class)


def _server(pages, **kw):
    return K.Server(K.Block(**dict(dict(heads=2, kv_heads=1, head_dim=64, rank=8, classes=1, page=16), **kw)), None, pages, device="cpu")


def test_a_batch_that_does_not_fit_leaves_every_request_as_it_was():
    s = _server(4)
    a, b, c = (s.admit(0) for _ in range(3))
    s.plan([(a, 20), (b, 10)])                                  # three pages of four
    before = _state(s)
    for batch in ([(a, 13), (b, 7), (c, 1)], [(b, 30), (a, 1)], [(b, 1), (c, 33)]):
        with pytest.raises(MemoryError):
            s.plan(batch)
        assert _state(s) == before
    assert s.plan([(a, 12), (b, 6), (c, 16)]).kv_len.tolist() == [32, 16, 16]   # what fits still does


def test_a_request_that_has_no_room_elsewhere_stays(monkeypatch):
    calls = []
    monkeypatch.setattr(I, "kv_read", lambda *a, **kw: calls.append("read") or (None, None))
    monkeypatch.setattr(I, "kv_write", lambda *a, **kw: calls.append("write"))
    one, two = _server(4), _server(2)
    r = one.admit(0)
    one.plan([(r, 33)])
    before = _state(one), _state(two)
    with pytest.raises(MemoryError):
        one.move(r, two)
    assert (_state(one), _state(two)) == before and calls == []
    wide = _server(4, page=32)
    there = one.move(r, wide)
    assert wide.length(there) == 33 and len(wide._pages[there]) == 2 and len(one._free) == 4 and calls == ["read", "write"]


def test_a_request_that_another_cache_refuses_stays(monkeypatch):
    def refuses(*a, **kw):
        raise ValueError("rows of another kind")
    monkeypatch.setattr(I, "kv_read", lambda *a, **kw: (None, None))
    monkeypatch.setattr(I, "kv_write", refuses)
    one, two = _server(4), _server(4, head_dim=128, cache=torch.bfloat16)
    r = one.admit(0)
    one.plan([(r, 33)])
    before = _state(one), _state(two)
    with pytest.raises(ValueError):
        one.move(r, two)
    assert (_state(one), _state(two)) == before


def test_batches_that_make_no_sense_are_refused():
    s = _server(4)
    a, b = s.admit(0), s.admit(0)
    s.plan([(a, 20), (b, 10)])
    before = _state(s)
    for batch in ([(a, 1), (b, 1), (a, 1)], [(a, -3)], [(b, 1), (a, -1)]):
        with pytest.raises(ValueError):
            s.plan(batch)
        assert _state(s) == before
    with pytest.raises(KeyError):
        s.plan([(a, 1), (99, 1)])
    assert _state(s) == before and s.plan([]).tokens == 0 and s.plan([(a, 0)]).kv_len.tolist() == [20]
