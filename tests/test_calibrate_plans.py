"""Plans of an iteration whose requests' pages change before it runs. The operators are stood in for: these are the host's books."""
from dataclasses import replace

import pytest
import torch

from paper_2602_02987_amd import calibrate as K
from paper_2602_02987_amd import iteration as I
from test_calibrate_pages import _cpu_copy

BLOCK = K.Block(heads=2, kv_heads=1, head_dim=64, rank=8, classes=1, page=16, cache=torch.bfloat16)


def _write(k, v, k_cache, v_cache, slots, k_exp=None, v_exp=None):
    places = k_cache.shape[2]
    for rows, cache in ((k, k_cache), (v, v_cache)):
        cache[slots // places, :, slots % places] = rows


@pytest.fixture
def server(monkeypatch):
    """A server whose keys are the first head's elements of the activations."""
    monkeypatch.setattr(I, "adapters", lambda x, base, *a, out=None, **kw: out)
    monkeypatch.setattr(I, "kv_write", _write)
    monkeypatch.setattr(I, "attention", lambda q, *a, **kw: torch.zeros(q.shape, dtype=q.dtype))
    _cpu_copy(monkeypatch)
    weights = K.Weights(BLOCK, device="cpu")
    weights.qkv.zero_()
    weights.qkv[2 * 64:3 * 64, :64] = torch.eye(64)
    return K.Server(BLOCK, weights, 12, device="cpu")


def _tokens(first, n):
    return torch.arange(first, first + n, dtype=torch.bfloat16).view(n, 1).expand(n, BLOCK.width).contiguous()


def _reads(s, r):
    return [int(s.k[s._pages[r][j // 16], 0, j % 16, 0]) for j in range(s.length(r))]


def _state(s):
    return s.k.clone(), s.v.clone(), list(s._free), list(s._held), {r: list(p) for r, p in s._pages.items()}


def _same(a, b):
    return torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and a[2:] == b[2:]


def test_a_plan_from_before_pages_were_moved_is_refused(server):
    first, second, third = (server.admit(0) for _ in range(3))
    for r, at, n in ((first, 10, 20), (second, 40, 20), (third, 70, 5)):
        server.iterate(_tokens(at, n), server.plan([(r, n)]))
    late, kept = server.plan([(second, 3), (third, 2)]), server.plan([(first, 1)])
    server.leave(third)
    third = server.admit(0)
    server.iterate(_tokens(80, 40), server.plan([(third, 40)]))
    server.iterate(_tokens(60, 3), server.plan([(second, 3)]))
    server.leave(first)
    assert server.compact() == 5 and _reads(server, third) == list(range(80, 120)) and _reads(server, second)[:20] == list(range(40, 60))
    before = _state(server)
    with pytest.raises(ValueError, match="no use any more"):
        server.iterate(_tokens(60, 5), late)
    with pytest.raises(ValueError, match="no use any more"):       # its request has left, and its pages are another's now
        server.iterate(_tokens(30, 1), kept)
    assert _same(before, _state(server))
    server.iterate(_tokens(63, 4), server.plan([(second, 4)]))    # one that was made after it is not
    assert _reads(server, second)[26:] == [63, 64, 65, 66] and _reads(server, third) == list(range(80, 120))


def test_a_plan_that_was_iterated_before_pages_are_moved(server):
    gone, r = server.admit(0), server.admit(0)
    server.iterate(_tokens(1, 33), server.plan([(gone, 33)]))
    p = server.plan([(r, 18)])
    server.iterate(_tokens(5, 18), p)
    server.leave(gone)
    assert server.compact() == 2 and _reads(server, r) == list(range(5, 23))
    with pytest.raises(ValueError, match="no use any more"):       # again: its slots are nobody's now
        server.iterate(_tokens(5, 18), p)


def test_plans_stay_where_no_page_of_theirs_moves(server):
    a, b, gone, c = (server.admit(0) for _ in range(4))
    server.iterate(_tokens(1, 8), server.plan([(a, 8)]))
    p, q = server.plan([(a, 2)]), server.plan([(b, 3), (c, 0)])
    assert server.compact() == 2                                  # nothing to move
    server.iterate(_tokens(9, 2), p)
    server.iterate(_tokens(30, 17), server.plan([(gone, 17)]))
    server.iterate(_tokens(50, 17), server.plan([(c, 17)]))
    server.leave(gone)
    assert server.compact() == 4                                  # c's pages alone; q brings no tokens of it
    server.iterate(_tokens(20, 3), q)
    assert [_reads(server, r) for r in (a, b, c)] == [list(range(1, 11)), [20, 21, 22], list(range(50, 67))]
    for r in (a, b, c):
        server.leave(r)
    assert not server._changed


def test_a_plan_from_before_its_request_went_on_in_several_ways_is_refused(server):
    r, other = server.admit(0), server.admit(0)
    server.iterate(_tokens(1, 18), server.plan([(r, 18)]))
    planned, apart = server.plan([(other, 1), (r, 2)]), server.plan([(other, 1)])
    forks = server.fork(r, 2)
    before = _state(server)
    with pytest.raises(ValueError, match="several ways"):          # the forks' pages were copied without these tokens
        server.iterate(_tokens(19, 3), planned)
    assert _same(before, _state(server))
    server.iterate(_tokens(70, 1), apart)                         # a plan of others
    assert _reads(server, other)[1] == 70
    server.leave(r)
    with pytest.raises(ValueError, match="left"):
        server.iterate(_tokens(19, 3), planned)
    assert [_reads(server, f)[:18] for f in forks] == [list(range(1, 19))] * 2


def test_a_plan_that_was_iterated_before_its_request_went_on(server):
    r = server.admit(0)
    p = server.plan([(r, 18)])
    server.iterate(_tokens(1, 18), p)
    assert server.fork(r, 0) == []
    server.iterate(_tokens(1, 18), p)                             # there are no forks
    (f,) = server.fork(r)
    with pytest.raises(ValueError, match="several ways"):          # again: the first page is the fork's as well
        server.iterate(_tokens(40, 18), p)
    for first, q in ((60, r), (80, f)):
        server.iterate(_tokens(first, 3), server.plan([(q, 3)]))
    assert _reads(server, r) == list(range(1, 19)) + [60, 61, 62] and _reads(server, f) == list(range(1, 19)) + [80, 81, 82]
    p = server.plan([(f, 2)])
    (g,) = server.fork(r)                                         # r's, not f's
    server.iterate(_tokens(83, 2), p)
    assert _reads(server, f)[18:] == [80, 81, 82, 83, 84] and _reads(server, g) == _reads(server, r)


def test_a_fork_without_room_leaves_plans_as_they_are(server):
    r = server.admit(0)
    p = server.plan([(r, 18)])
    with pytest.raises(MemoryError):
        server.fork(r, 11)
    server.iterate(_tokens(1, 18), p)
    assert _reads(server, r) == list(range(1, 19))


KINDS = [None, K.Positions(), K.Positions(base=500000.0), K.Positions(dims=32), K.Positions(interleaved=True), K.Positions(magnitude=1.1), K.Positions(scaling="linear", factor=2.0)]


@pytest.mark.parametrize("mine", range(len(KINDS)))
def test_a_request_stays_where_the_other_server_has_other_positions(mine, monkeypatch):
    moved = []
    monkeypatch.setattr(I, "kv_read", lambda k, v, slots, *a, **kw: (slots, slots))
    monkeypatch.setattr(I, "kv_write", lambda *a: moved.append(a))
    one, *others = (K.Server(replace(BLOCK, positions=p), None, 6, device="cpu") for p in [KINDS[mine]] + KINDS)
    r, empty = one.admit(0), one.admit(0)
    one.plan([(r, 20)])
    for i, two in enumerate(others):
        if i == mine:
            continue
        before = _state(one), _state(two), two._next
        with pytest.raises(ValueError, match="positions"):
            one.move(r, two)
        assert _same(before[0], _state(one)) and _same(before[1], _state(two)) and two._next == before[2] and one.length(r) == 20 and not moved
    assert others[(mine + 1) % len(others)].length(one.move(empty, others[(mine + 1) % len(others)])) == 0    # nothing was turned yet
    moved.clear()
    there = one.move(r, others[mine])
    assert others[mine].length(there) == 20 and len(moved) == 1 and len(one._free) == 6


def test_positions_that_are_written_in_other_words_are_the_same(monkeypatch):
    monkeypatch.setattr(I, "kv_read", lambda k, v, slots, *a, **kw: (slots, slots))
    monkeypatch.setattr(I, "kv_write", lambda *a: None)
    one, two = (K.Server(replace(BLOCK, positions=p), None, 6, device="cpu") for p in (K.Positions(), K.Positions(dims=64, scaling="linear", factor=1.0)))
    r = one.admit(0)
    one.plan([(r, 20)])
    assert two.length(one.move(r, two)) == 20
