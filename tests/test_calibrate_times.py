"""What the calibration times: the GPU's part of iterations that go through a model's layers."""
import time

import pytest
import torch

from paper_2602_02987_amd import calibrate as K
from paper_2602_02987_amd import iteration as I

SMALL = K.Block(heads=4, kv_heads=2, head_dim=64, rank=8, classes=2, page=16)


def test_copies_of_weights_are_the_same_numbers_in_other_memory():
    w = K.Weights(SMALL, 3, "cpu")
    c = w.copy()
    pairs = [(a, b) for name in vars(w) for a, b in (zip(*(getattr(t, name) for t in (w, c))) if isinstance(getattr(w, name), tuple) else [(getattr(w, name), getattr(c, name))])]
    assert len(pairs) == 7 and all(torch.equal(a, b) and a.data_ptr() != b.data_ptr() for a, b in pairs)
    assert w.bytes() == sum(a.nbytes for a, _ in pairs) == c.bytes()


@pytest.mark.gpu
def test_passes_go_through_the_layers(monkeypatch):
    used = []
    write = I.kv_write
    monkeypatch.setattr(I, "kv_write", lambda k, v, kc, *a, **kw: used.append(kc.data_ptr()) or write(k, v, kc, *a, **kw))
    K.measure(SMALL, [16], [2], 20, passes=12, layers=5)
    last = used[-12:]
    assert len(set(last)) == 5 and last[:5] == last[5:10] and last[:2] == last[10:]
    big = K.Block()
    assert K._LAST_LEVEL_CACHE < 7 * K.Weights(big, device="cuda:0").bytes()


@pytest.mark.gpu
def test_a_slow_host_is_not_in_the_times(monkeypatch):
    write = I.kv_write

    def slow(*a, **kw):
        time.sleep(0.004)
        return write(*a, **kw)
    monkeypatch.setattr(I, "kv_write", slow)
    samples = K.measure(SMALL, [0], [1, 3], 20, passes=3, layers=2)
    assert all(0 < t < 0.001 for _, _, t in samples), samples


@pytest.mark.gpu
def test_caches_of_the_layers_hold_the_same_and_fit(monkeypatch):
    servers = []
    make = K.Server.__init__
    monkeypatch.setattr(K.Server, "__init__", lambda self, *a, **kw: servers.append(self) or make(self, *a, **kw))
    fp8 = K.Block(heads=4, kv_heads=2, head_dim=64, rank=8, classes=2, page=16)
    K.measure(fp8, [0, 16], [0, 2], 50, passes=2, layers=3)
    assert len(servers) == 3 and bool((servers[0].k.view(torch.uint8) != 0).any())
    for s in servers[1:]:
        # everything but the places of the last passes' tokens, which are not on all of the servers
        same = [torch.equal(a.view(torch.uint8)[:, :, :2], b.view(torch.uint8)[:, :, :2]) for a, b in ((s.k, servers[0].k), (s.v, servers[0].v))]
        assert all(same) and s.k.data_ptr() != servers[0].k.data_ptr()
    servers.clear()
    monkeypatch.setattr(torch.cuda, "mem_get_info", lambda *a: (0, 1 << 38))
    K.measure(fp8, [0], [2], 20, passes=2, layers=3)
    assert len(servers) == 1
