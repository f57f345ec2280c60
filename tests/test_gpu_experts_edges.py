"""Routed-expert operators at the edges of their contracts.

Tolerances are those of test_gpu_experts.py, derived there; where a case adds to them it says so."""
import numpy as np
import pytest

from paper_2502_07021_b200 import binding as fs
from test_gpu_experts import ROUND, TYPES, dev, host, quantized, t_

pytestmark = pytest.mark.gpu


# ---- product --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("first,sizes,outs,cols", [(1, [1], 16, 64), (5, [4, 0, 21], 130, 96), (37, [20, 0, 3], 70, 544),
                                                   (300, [130, 64], 200, 256), (9, [0, 0], 33, 32)])
def test_product_of_a_slice_of_the_groups(first, sizes, outs, cols):
    """offsets + 2: the rows of the groups before the slice are in none of its groups, so their results are 0."""
    import torch
    rng = np.random.default_rng(first + outs)
    groups, rows = len(sizes), first + sum(sizes) + 4
    xq, xs, xv = quantized(rng.standard_normal((rows, cols)))
    wq, ws, wv = quantized(rng.standard_normal((groups * outs, cols)))
    off = np.concatenate([[0, first // 2, first], first + np.cumsum(sizes), [rows]]).astype(np.int32)
    mine = dev(off)[2:]
    off = off[2:]
    for dtype in TYPES:
        y = torch.full((rows, outs + 1), 7.0, dtype=t_(dtype), device="cuda")
        fs.fs_mx4_product(xq, xq.stride(0), xs, xs.stride(0), rows, wq, wq.stride(0), ws, ws.stride(0), groups, mine, outs, cols, y,
                          fs.fs_dtype(y), y.stride(0), None)
        got = host(y[:, :outs])
        want, size = np.zeros((rows, outs)), np.zeros((rows, outs))
        for g in range(groups):
            a, w = xv[off[g]:off[g + 1]], wv[g * outs:(g + 1) * outs]
            want[off[g]:off[g + 1]], size[off[g]:off[g + 1]] = a @ w.T, np.abs(a) @ np.abs(w).T
        assert np.all(got[:first] == 0) and np.all(got[off[groups]:] == 0)
        assert np.all(np.abs(got - want) <= (cols / 64 + 4) * 2.0 ** -22 * size + 1.01 * ROUND[dtype] * np.abs(want) + 2.0 ** -25 * (size > 0))
        assert torch.all(y[:, outs:] == 7.0)
