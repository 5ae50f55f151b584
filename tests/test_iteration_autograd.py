"""What the binding of the iteration operators does about autograd: nothing has a derivative, and what is written counts as written."""
import pytest
import torch
import torch.autograd.forward_ad as fw

from paper_2602_02987_amd import iteration as I


def _calls(device, q=None, k=None, x=None, scale=None):
    """kv_write, kv_read, attention and adapters on small tensors; those given take the place of one of a call's."""
    kc, vc, _, _ = I.new_cache(4, 2, 16, 64, device=device)
    kc = kc if k is None else k
    rows = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device=device)
    slots = torch.zeros(3, dtype=torch.int64, device=device)
    start, length = (torch.tensor(n, dtype=torch.int32, device=device) for n in ([0, 3], [3]))
    table = torch.zeros((1, 1), dtype=torch.int32, device=device)
    y = torch.zeros(3, 64, dtype=torch.bfloat16, device=device)
    down, up = (torch.zeros(s, dtype=torch.bfloat16, device=device) for s in ((2, 8, 64), (2, 64, 8)))
    scale = torch.ones(2, device=device) if scale is None else scale
    return dict(kv_write=lambda **kw: I.kv_write(rows if q is None else q, rows, kc, vc, slots, **kw), kv_read=lambda **kw: I.kv_read(kc, vc, slots, **kw),
                attention=lambda **kw: I.attention(rows if q is None else q, kc, vc, table, start, length, **kw),
                adapters=lambda **kw: I.adapters(y if x is None else x, y, down, up, scale, start, length - 3, **kw))


def test_tangents_of_forward_mode_are_refused():
    def dual(*shape, dtype=torch.bfloat16):
        return fw.make_dual(torch.zeros(shape, dtype=dtype), torch.ones(shape, dtype=dtype))
    with fw.dual_level():
        for name, kw in (("kv_write", dict(q=dual(3, 2, 64))), ("kv_read", dict(k=dual(4, 2, 16, 64))), ("attention", dict(q=dual(3, 2, 64))), ("attention", dict(k=dual(4, 2, 16, 64))),
                         ("adapters", dict(x=dual(3, 64))), ("adapters", dict(scale=dual(2, dtype=torch.float32)))):
            call = _calls("cpu", **kw)[name]
            with pytest.raises(ValueError, match="forward-mode"):
                call()
            with torch.no_grad(), pytest.raises(ValueError, match="forward-mode"):   # (which does not stop tangents)
                call()
            with fw._set_fwd_grad_enabled(False), pytest.raises(ValueError, match="GPU"):   # (the next thing that is wrong)
                call()


def test_results_that_require_gradients_are_refused():
    rows, y = (torch.zeros(s, dtype=torch.bfloat16, requires_grad=True) for s in ((3, 2, 64), (3, 64)))
    calls = _calls("cpu")
    for name, kw in (("kv_read", dict(k=rows)), ("kv_read", dict(v=rows)), ("attention", dict(out=rows)), ("adapters", dict(out=y))):
        with pytest.raises(ValueError, match="backward"):
            calls[name](**kw)
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):   # (the next thing that is wrong)
            calls[name](**kw)


@pytest.mark.gpu
def test_what_is_written_counts_as_written():
    dev = "cuda:0"
    calls, status = _calls(dev), I.new_status(dev)
    rows, other = (torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=dev) for _ in range(2))
    y = torch.zeros((3, 64), dtype=torch.bfloat16, device=dev)
    work = torch.zeros(1 << 24, dtype=torch.uint8, device=dev)
    for name, kw in (("kv_read", dict(k=rows, v=other)), ("attention", dict(out=rows, status=status, workspace=work)), ("adapters", dict(out=y, status=status, workspace=work))):
        before = {n: t._version for n, t in kw.items()}
        calls[name](**kw)
        assert {n: t._version > before[n] for n, t in kw.items()} == {n: True for n in kw}, name
    k, v, ke, ve = I.new_cache(4, 2, 16, 64, torch.float8_e4m3fn, device=dev)
    slots = torch.zeros(3, dtype=torch.int64, device=dev)
    slots[1:] = torch.tensor([5, 17], device=dev)
    before = [t._version for t in (k, v, ke, ve)]
    I.kv_write(rows, other, k, v, slots, ke, ve)
    assert all(t._version > b for t, b in zip((k, v, ke, ve), before))
    I.kv_read(k, v, slots, ke, ve)
    assert [t._version for t in (k, v, ke, ve)] == [b + 1 for b in before]          # reading is not writing
    # a product that kept its factor for the backward pass
    w = torch.ones((3, 2, 64), dtype=torch.bfloat16, device=dev, requires_grad=True)
    z = (w * rows).sum()
    I.kv_read(k, v, slots, ke, ve, k=rows)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()
    with torch.inference_mode():
        kept = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=dev)
        I.kv_read(k, v, slots, ke, ve, k=kept)
    I.kv_read(k, v, slots, ke, ve, k=kept)                                          # an inference tensor, outside
    assert torch.equal(kept, rows)
