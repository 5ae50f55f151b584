"""The iteration operators on the GPU where tensors overlap, pages or exponents that nobody looks at are out of range, and pieces of work are many."""
import numpy as np
import pytest
import torch

import iteration_reference as R
from paper_2602_02987_amd import iteration as I
from test_gpu_iteration import DEV, _adapter_case, _adapters_close

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
