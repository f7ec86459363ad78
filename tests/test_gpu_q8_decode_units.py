"""The sparse decode over an 8-bit cache whose values change size along a wave's
tokens. Bound, element by element and key by key: the weight's score and
exponential (half of rows_ref.score_error each for the weight and for the sum),
sums, terms and merges in fp32 or 22 bits (2^-20)."""
import numpy as np
import pytest
import torch

import paper_2506_04108_amd as R
from rows_ref import D, check, f64, i32, randn, score_error
from test_gpu_q8 import SCALE, Pair, rows

pytestmark = pytest.mark.gpu


def decode(p, q, L, splits):
    b, H = p.b, p.ref.kmin.shape[1]
    M = -(-L // b)
    idx = torch.arange(M, dtype=torch.int32, device="cuda").expand(1, H, M).contiguous()
    out, lse = R.sparse_decode_q8(p.dev, q, i32([L]), idx, torch.full((1, H), M, dtype=torch.int32, device="cuda"),
                                  num_splits=splits)
    torch.cuda.synchronize()
    return out.cpu().numpy()[0], lse.cpu().numpy()[0]


def verify(p, q, L, splits, what):
    got, gl = decode(p, q, L, splits)
    H, hq = p.ref.kmin.shape[1], q.shape[1]
    for h in range(hq):
        k, v = p.ref.values("k", 0, h // (hq // H), L), p.ref.values("v", 0, h // (hq // H), L)
        x = f64(q)[0, h]
        s, e = (k @ x) * SCALE, score_error((np.abs(k) @ np.abs(x)) * SCALE) / 2
        w = np.exp(s - s.max())
        total = w.sum()
        w, av, off = w / total, np.abs(v), (w / total * e).sum()
        o = w @ v
        check(got[h], o, (w * e) @ av + (w @ av) * 2.0 ** -20 + np.abs(o) * off + 1e-36, f"{what} out {h}")
        l = np.log(total) + s.max()
        check(gl[h:h + 1], np.array([l]), 2 * off + 2.0 ** -20 + abs(l) * 2.0 ** -22, f"{what} lse {h}")


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("ratio", [0, 10, 20, 30, 40, 80])
@pytest.mark.parametrize("fmt,b,g", [("int8", 16, 4), ("e4m3", 32, 8), ("int8", 64, 1)])
def test_large_values_then_higher_scores(fmt, b, g, ratio, splits):
    """Every wave meets values of 2^ratio first, later ones of 1 whose scores
    are higher, in steps, by 2^50 and more."""
    L = 512 * splits
    k, v = rows(L, 2, 1300)
    step = 128 * splits
    v[:step] *= 2.0 ** ratio
    v[step:2 * step] *= 2.0 ** (ratio // 2)
    for i in range(3):
        k[i * step:(i + 1) * step, :, 0] = -120.0 + 40 * i
    k[3 * step:, :, 0] = 0
    q = randn((1, 2 * g, D), 1301)
    q[:, :, 0] = 10.0
    p = Pair(1, 2, L, b, fmt, [L])
    p.store(k, v, [0, L], [L])
    verify(p, q.cuda(), L, splits, f"{fmt} b={b} 2^{ratio}")


@pytest.mark.parametrize("splits", [1, 2])
@pytest.mark.parametrize("small", [0.0, 2.0 ** -90])
@pytest.mark.parametrize("large", [2.0 ** 20, 2.0 ** 60, 2.0 ** 90])
@pytest.mark.parametrize("fmt,b", [("int8", 16), ("e4m3", 64)])
def test_values_of_zero_and_large_ones_without_weight(fmt, b, large, small, splits):
    """Zeros (a scale of 2^-100 / Q) hold all the weight; the large values that
    follow have a weight of zero, for one head exactly."""
    L = 384 * splits
    k, v = rows(L, 1, 1310)
    v[:128 * splits] *= small
    v[128 * splits:] *= large
    k[:, 0, 0] = 0
    k[128 * splits:, 0, 0] = -300.0
    q = randn((1, 2, D), 1311)
    q[0, 0, 0], q[0, 1, 0] = 40.0, 2.0
    p = Pair(1, 1, L, b, fmt, [L])
    p.store(k, v, [0, L], [L])
    verify(p, q.cuda(), L, splits, f"{fmt} b={b} {small} {large}")
