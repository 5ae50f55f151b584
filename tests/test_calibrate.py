"""The block that the iteration operators make together, and the iteration-time coefficients that it is timed for."""
import numpy as np
import pytest
import torch

import iteration_reference as R
from paper_2602_02987_amd import calibrate as K
from paper_2602_02987_amd import iteration as I
from paper_2602_02987_amd import workloads as W

DEV = "cuda:0"


def test_fit_finds_the_law_it_was_given():
    law = dict(c0=0.01, c_pre=5e-5, c_dec=2e-4)
    samples = [(p, n, law["c0"] + law["c_pre"] * p + law["c_dec"] * n) for p in (0, 64, 256) for n in (0, 1, 32, 127)]
    got = K.fit(samples)
    for name, value in law.items():
        assert got[name] == pytest.approx(value, rel=1e-9)
    assert got["residual"] < 1e-9
    assert W.config(1, **{n: got[n] for n in law}).c_pre == pytest.approx(5e-5)


def test_fit_gives_no_coefficient_below_zero():
    got = K.fit([(0, 1, 0.02), (0, 100, 0.01), (64, 1, 0.03), (64, 100, 0.03)])
    assert min(got["c0"], got["c_pre"], got["c_dec"]) >= 0 and got["residual"] > 0


def test_a_server_says_when_its_cache_is_full():
    b = K.Block(heads=2, kv_heads=1, head_dim=64, rank=8, classes=1, page=16)
    s = K.Server(b, None, 3, device="cpu")
    r, other = s.admit(0), s.admit(-1)
    p = s.plan([(r, 17), (other, 1)])
    assert p.tokens == 18 and p.longest == 17 and p.q_start.tolist() == [0, 17, 18] and p.kv_len.tolist() == [17, 1] and p.adapter.tolist() == [0, -1]
    assert len(set(p.slots.tolist())) == 18 and [int(p.table[0, j // 16]) * 16 + j % 16 for j in range(17)] == p.slots.tolist()[:17]
    with pytest.raises(MemoryError):
        s.plan([(other, 16)])
    s.leave(r)
    assert s.plan([(other, 16)]).kv_len.tolist() == [17] and s.length(other) == 17


BLOCKS = [K.Block(heads=8, kv_heads=2, head_dim=64, rank=8, classes=3, page=16, cache=torch.bfloat16), K.Block(heads=6, kv_heads=2, head_dim=128, rank=24, classes=3, page=32),
          K.Block(heads=4, kv_heads=4, head_dim=64, rank=16, classes=3, page=16, dtype=torch.float16)]


@pytest.mark.gpu
@pytest.mark.parametrize("block", BLOCKS, ids=["bf16", "fp8-bf16", "fp8-fp16"])
def test_iterations_of_a_chunk_among_decodes(block, monkeypatch):
    """Every operator's part of three iterations against 64 bits, from what it was given: what it adds, what the cache holds then, what is attended."""
    weights = K.Weights(block, 3, DEV)
    server = K.Server(block, weights, 60, DEV)
    gen = torch.Generator()
    gen.manual_seed(5)
    seen = []

    def watched(name):
        f = getattr(I, name)

        def call(*a, **kw):
            before = [t.clone() if isinstance(t, torch.Tensor) else t for t in a]
            out = f(*a, **kw)
            seen.append((name, before, kw, out.clone() if isinstance(out, torch.Tensor) else out))
            return out
        return call
    for name in ("adapters", "kv_write", "attention"):
        monkeypatch.setattr(I, name, watched(name))
    a, b, c = (server.admit(i) for i in (0, 2, -1))
    for batch in ([(a, 40), (b, 7)], [(a, 1), (b, 1), (c, 50)], [(a, 1), (b, 1), (c, 3)]):
        p = server.plan(batch)
        x = torch.randn((p.tokens, block.width), generator=gen).to(block.dtype).to(DEV)
        seen.clear()
        y = server.iterate(x, p)
        I.check(server.status)
        assert y.shape == x.shape and [s[0] for s in seen] == ["adapters", "kv_write", "attention", "adapters"]
        for name, t, _, out in (seen[0], seen[3]):
            d = [u.cpu().double().numpy() for u in t[:5]]
            ref, inner, outer = R.adapters(*d, t[5].cpu().numpy(), t[6].cpu().numpy())
            bound = R.adapters_bound(ref, d[1], inner, outer, block.dtype, block.width, block.rank)
            assert (np.abs(out.cpu().double().numpy() - ref) <= bound).all()
        new = [u.cpu().double().numpy() for u in seen[1][1][:2]]
        at = p.slots.cpu().numpy()
        held = [R.cache_values(u, e) for u, e in ((server.k, server.k_exp), (server.v, server.v_exp))]
        for x64, values in zip(new, held):
            if block.cache == torch.float8_e4m3fn:
                code, exp = R.quantise(x64)
                x64 = code * 2.0 ** exp[..., None]
            assert np.array_equal(values[at // block.page, :, at % block.page], x64)
        q, out = seen[2][1][0], seen[2][3]
        ref, parts = R.attention(q.cpu().double().numpy(), *held, p.table.cpu().numpy(), p.q_start.cpu().numpy(), p.kv_len.cpu().numpy())
        assert (np.abs(out.cpu().double().numpy() - ref) <= R.attention_bound(ref, parts, block.dtype, block.head_dim)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("block", BLOCKS, ids=["bf16", "fp8-bf16", "fp8-fp16"])
def test_a_request_that_moves_takes_its_cache_along(block):
    """Prefill here, decode there: the same bits as if the request had stayed (values read back fit the 16-bit types, and quantising
    them again loses nothing)."""
    weights = K.Weights(block, 7, DEV)
    gen = torch.Generator()
    gen.manual_seed(9)
    x = torch.randn((90, block.width), generator=gen).to(block.dtype).to(DEV)
    one, two = K.Server(block, weights, 20, DEV), K.Server(block, weights, 30, DEV)
    other = two.admit(0)
    two.iterate(x[:33], two.plan([(other, 33)]))
    stays, moves = one.admit(1), one.admit(1)
    for r in (stays, moves):
        one.iterate(x[:50], one.plan([(r, 50)]))
        one.iterate(x[50:83], one.plan([(r, 33)]))
    free = len(one._free)
    there = one.move(moves, two)
    assert two.length(there) == 83 and len(one._free) == free + -(-83 // block.page)
    for t in range(83, 90):
        want = one.iterate(x[t:t + 1], one.plan([(stays, 1)]))
        assert torch.equal(two.iterate(x[t:t + 1], two.plan([(there, 1)])), want)
    I.check(one.status)
    I.check(two.status)


@pytest.mark.gpu
def test_measured_samples():
    block = K.Block(heads=4, kv_heads=2, head_dim=64, rank=8, classes=2, page=16)
    samples = K.measure(block, [0, 20], [0, 3], 40, passes=2)
    assert [s[:2] for s in samples] == [(0, 3), (20, 0), (20, 3)] and all(0 < s[2] < 1 for s in samples)
    got = K.fit(samples)
    assert got["c0"] >= 0 and got["c_pre"] >= 0 and got["c_dec"] >= 0
