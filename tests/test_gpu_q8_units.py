"""Value scales far apart under the dense rectification over an 8-bit cache: a
row's precision follows the keys that it sees and weighs, not those of its
neighbours.

Bound, element by element, key by key. The exact weight w_j is off by its
score's and exponential's error e_j (half of rows_ref.score_error each for the
weight and for the sum) and by its rounding to fp16, 2^-11 of itself where it is
a normal number. Below that:
 scales within 2^6 of each other   2^-25 of a unit that is at most 2^7 scales,
                                   beside a reference not above the largest
                                   weight: 2^-18 |v_j|
 further apart                     2^-25 beside 2^14 for the largest weight of
                                   its 16 keys: 2^-39 of that
Sums and merges are fp32 (2^-20), the result is rounded to bf16 (2^-8)."""
import numpy as np
import pytest
import torch

import paper_2506_04108_amd as R
from rows_ref import D, check, cumulative, f64, i32, randn, score_error
from test_gpu_q8 import SCALE, Pair, rows

pytestmark = pytest.mark.gpu


def reference(q, k, v, last, shared):
    """Rows q [R, D] over keys [n, D], row r up to last[r]: out, its bound, lse and its bound."""
    n = k.shape[0]
    see = np.arange(n)[None, :] <= np.asarray(last)[:, None]
    s = np.where(see, (q @ k.T) * SCALE, -np.inf)
    m = s.max(1, keepdims=True)
    p = np.exp(s - m)
    total = p.sum(1, keepdims=True)
    w, av = p / total, np.abs(v)
    e = np.where(see, score_error((np.abs(q) @ np.abs(k).T) * SCALE) / 2, 0)
    out, off = w @ v, (w * e).sum(1, keepdims=True)
    most = np.maximum.reduceat(w, np.arange(0, n, 16), axis=1).repeat(16, 1)[:, :n] * see
    small = (see @ av) * 2.0 ** -18 if shared else (most @ av) * 2.0 ** -39
    bound = ((w * e) @ av + (w @ av) * (2.0 ** -11 + 2.0 ** -20) + small + np.abs(out) * off) * (1 + 2.0 ** -8)
    lse = (np.log(total) + m)[:, 0]
    return out, bound + np.abs(out) * 2.0 ** -8, lse, 2 * off[:, 0] + 2.0 ** -20 + np.abs(lse) * 2.0 ** -22


def check_rows(p, q, cu, lens, out, lse, shared, what, heads):
    g = q.shape[1] // p.ref.kmin.shape[1]
    got, gl, q64 = f64(out), lse.cpu().numpy(), f64(q)
    for s, L in enumerate(lens):
        n = cu[s + 1] - cu[s]
        for h in heads:
            k, v = p.ref.values("k", s, h // g, L), p.ref.values("v", s, h // g, L)
            o, bound, l, lbound = reference(q64[cu[s]:cu[s + 1], h], k, v, L - n + np.arange(n), shared)
            check(got[cu[s]:cu[s + 1], h], o, bound, f"{what} out {s},{h}")
            check(gl[cu[s]:cu[s + 1], h], l, lbound, f"{what} lse {s},{h}")


def rectify(p, k, v, q, n, lens):
    """All rows stored, the last n[s] of each sequence by the rectification."""
    cu, at = cumulative(n), cumulative(lens)
    new = np.concatenate([np.arange(at[s + 1] - n[s], at[s + 1]) for s in range(len(lens))])
    old = [L - x for L, x in zip(lens, n)]
    if sum(old):
        first = np.concatenate([np.arange(at[s], at[s + 1] - n[s]) for s in range(len(lens))])
        p.store(k[first], v[first], cumulative(old), old)
    kn, vn = k[new].contiguous(), v[new].contiguous()
    out, lse = R.dense_rectify_q8(p.dev, q, kn, vn, i32(cu), i32(lens), max(lens))
    torch.cuda.synchronize()
    p.ref.store(f64(kn), f64(vn), cu, lens)
    return cu, out, lse


@pytest.mark.parametrize("ratio", [-60, -20, 4, 12, 20, 40, 90])
@pytest.mark.parametrize("fmt,b", [("int8", 16), ("e4m3", 16), ("int8", 32), ("e4m3", 64)])
def test_rows_that_see_one_block_only(fmt, b, ratio):
    """A prompt whose second block is 2^ratio times the first: the first block's
    rows see nothing of it, in the same tile or the next one."""
    L, g = 2 * b + 5, 3
    k, v = rows(L, 1, 1100 + b)
    v[b:2 * b] *= 2.0 ** ratio
    p = Pair(1, 1, 3 * b, b, fmt, [L])
    q = randn((L, g, D), 1101).cuda()
    cu, out, lse = rectify(p, k, v, q, [L], [L])
    check_rows(p, q, cu, [L], out, lse, ratio == 4, f"{fmt} b={b} 2^{ratio}", range(g))


@pytest.mark.parametrize("where", [0, 300, 1150])
@pytest.mark.parametrize("n,g", [(16, 2), (32, 4), (300, 2)])
@pytest.mark.parametrize("fmt,paged", [("int8", False), ("e4m3", True)])
def test_heads_that_weigh_one_block_away(fmt, paged, n, g, where):
    """A block of values 2^60 times the others', seen by every row and weighed
    by the second head of each kv head alone."""
    L, H = 1200, 2
    k, v = rows(L, H, 1110)
    at = where // 16 * 16
    v[at:at + 16] *= 2.0 ** 60
    k[:, :, 0] = 0
    k[at:at + 16, :, 0] = -300.0
    q = randn((n, H * g, D), 1111)
    q[:, :, 0] = 40.0
    q[:, 1::g, 0] = -0.5
    q = q.cuda()
    p = Pair(1, H, 1200, 16, fmt, [L], paged)
    cu, out, lse = rectify(p, k, v, q, [n], [L])
    check_rows(p, q, cu, [L], out, lse, False, f"{fmt} n={n} at {at}", [0, 1, H * g - 1])


@pytest.mark.parametrize("spread,shared", [(1, True), (30, False)])
@pytest.mark.parametrize("n,g,b", [([17, 3, 32], 4, 16), ([150, 257, 60], 2, 16), ([40, 9, 100], 4, 64)])
def test_every_block_of_a_scale_of_its_own(n, g, b, spread, shared):
    """Splits of more than 64 blocks; every scale a power of two up to 2^spread
    (either way) away from the others."""
    lens, H = [9000, 6000, 777], 2
    at = cumulative(lens)
    k, v = rows(at[-1], H, 1120)
    rng = np.random.default_rng(b)
    for s, L in enumerate(lens):
        f = np.exp2(rng.integers(-spread, spread + 1, -(-L // b))).repeat(b)[:L]
        v[at[s]:at[s + 1]] *= torch.from_numpy(f).cuda().bfloat16()[:, None, None]
    p = Pair(3, H, 9024, b, "int8" if b == 16 else "e4m3", lens, paged=b == 64)
    q = randn((sum(n), H * g, D), 1121).cuda()
    cu, out, lse = rectify(p, k, v, q, n, lens)
    check_rows(p, q, cu, lens, out, lse, shared, f"2^{spread} n={n}", [0, H * g - 1])
    p.same(lens, "scales of their own")


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_blocks_of_zeros(fmt):
    """Blocks of zeros (a scale of 2^-100 / Q) and one of 2^-90, which the first head of each two attends to."""
    L, n = 640, 64
    k, v = rows(L, 1, 1130)
    v[32:64] = 0
    v[600:] = 0
    p = Pair(1, 1, L, 16, fmt, [L])
    q = randn((n, 4, D), 1131).cuda()
    cu, out, lse = rectify(p, k, v, q, [n], [L])
    check_rows(p, q, cu, [L], out, lse, True, f"zeros {fmt}", range(4))
    v[:16] *= 2.0 ** -90
    k[:, :, 0] = 0
    k[:16, :, 0] = 300.0
    q[:, ::2, 0] = 10.0
    p = Pair(1, 1, L, 16, fmt, [L])
    cu, out, lse = rectify(p, k, v, q, [n], [L])
    check_rows(p, q, cu, [L], out, lse, False, f"zeros and small {fmt}", range(4))
