"""The dense rectification over an 8-bit cache where a block's key factor (its
scale times the softmax scale) underflows. Bounds as in test_gpu_q8_units.py."""
import numpy as np
import pytest
import torch

import paper_2506_04108_amd as R
from rows_ref import D, check, f64, i32, randn
from test_gpu_q8 import Pair, rows
from test_gpu_q8_units import reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("sm_scale", [2.0 ** -30, 2.0 ** -120])
def test_key_factors_that_underflow(fmt, sm_scale):
    """Keys of zeros (a scale of 2^-100 / Q) times a softmax scale that leaves
    nothing of it: all weights are the same, masked keys stay masked."""
    L, g = 70, 4
    k, v = rows(L, 1, 1210)
    k[20:] = 0
    p = Pair(1, 1, 80, 16, fmt, [L])
    q = randn((L, g, D), 1211).cuda()
    out, lse = R.dense_rectify_q8(p.dev, q, k, v, i32([0, L]), i32([L]), L, sm_scale=sm_scale)
    torch.cuda.synchronize()
    p.ref.store(f64(k), f64(v), [0, L], [L])
    x = p.ref.values("v", 0, 0, L)
    for h in range(g):  # scores are below 2^-20
        o, bound, l, lbound = reference(np.zeros((L, D)), x, x, np.arange(L), True)
        slack = np.cumsum(np.abs(x), 0) / np.arange(1, L + 1)[:, None] * 2.0 ** -18
        check(f64(out)[:, h], o, bound + slack, f"{fmt} {sm_scale} out")
        check(lse.cpu().numpy()[:, h], l, lbound + 2.0 ** -18, f"{fmt} {sm_scale} lse")
