"""Attention of few rows: the weights are held as two numbers of the rows' type, so that the result's own rounding is all that shows."""
import numpy as np
import pytest
import torch

import iteration_reference as R
from paper_2602_02987_amd import iteration as I
from test_gpu_iteration import ATTENTION, DEV, _attention_case, _id

pytestmark = pytest.mark.gpu


def _bound(out, parts, dtype, dim):
    """As R.attention_bound, but for the weights: the upper number is cut off (a step, 2 u, and the factor before it, u / 2), the lower one, which holds what that leaves, is
    rounded (u of it)."""
    spread, most, total, reach = parts
    u = R.half_step(dtype)
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2
    f = 2.0 ** -24 * (2 * (dim + 16) * total + reach + 64)
    return u * np.abs(out) * (1 + u) + (2.5 * u * u + f) * spread * (1 + u) + tiny * (most + 1)


FEW = [c for c in ATTENTION if max(c[6]) * c[0] // c[1] <= 16] + [(8, 2, 128, 64, "bf16", "bf16", [1, 1], [3000, 1500], 0, False), (4, 1, 64, 16, "fp16", "fp8", [1, 3], [2500, 700], 0, True),
                                                                  (2, 1, 256, 16, "bf16", "fp8", [1, 2], [1700, 900], 333, False)]


@pytest.mark.parametrize("case", FEW, ids=_id)
def test_weights_of_few_rows(case):
    q, (k, v, ke, ve), table, start, length, window = _attention_case(case, 67)
    got = I.attention(q.to(DEV), k, v, table.to(DEV), start.to(DEV), length.to(DEV), ke, ve, max_q=max(case[6]), window=window).cpu().double().numpy()
    ref, parts = R.attention(q.double().numpy(), R.cache_values(k, ke), R.cache_values(v, ve), table.numpy(), start.numpy(), length.numpy(), None, window)
    over = np.abs(got - ref) - _bound(ref, parts, q.dtype, q.shape[2])
    assert over.max() <= 0, over.max()


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_an_infinite_value_comes_out_as_it_is(kind, dim, sign):
    """Whatever the weight's two numbers are: the first and the last key's, one of a key with a small weight, one of the only key."""
    case = (4, 2, dim, 16, kind, kind, [1, 1, 1], [300, 1, 47], 0, False)
    q, (k, v, _, _), table, start, length, _ = _attention_case(case, 71)
    k[int(table[0, 3]), :, 5] *= 3.0                             # (scores of twelve and more on either side of zero)
    for r, at, d in ((0, 0, 1), (0, 299, 2), (0, 3 * 16 + 5, 3), (1, 0, 4), (2, 20, 5)):
        v[int(table[r, at // 16]), 1, at % 16, d] = sign * float("inf")
    got = I.attention(q.to(DEV), k, v, table.to(DEV), start.to(DEV), length.to(DEV)).cpu().double()
    expect = torch.zeros(got.shape, dtype=torch.bool)
    for r, d in ((0, 1), (0, 2), (0, 3), (1, 4), (2, 5)):
        expect[r, 2:, d] = True
    assert (got[expect] == sign * float("inf")).all() and got[~expect].isfinite().all()
