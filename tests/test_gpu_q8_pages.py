"""The dense rectification over blocks whose table entry lies outside the pool:
rows that see nothing of such a block are as without it, rows that see it find
zeros. Bounds as in test_gpu_q8_units.py."""
import numpy as np
import pytest
import torch

import paper_2506_04108_amd as R
from rows_ref import D, check, cumulative, f64, i32, randn
from test_gpu_q8 import Pair, rows
from test_gpu_q8_units import reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [0.0, float("nan"), float("inf"), 2.0 ** 60])
@pytest.mark.parametrize("fmt,b,stray", [("int8", 16, -1), ("e4m3", 16, 10 ** 6), ("int8", 32, -7), ("e4m3", 64, -1)])
@pytest.mark.parametrize("n,g", [(None, 2), (20, 4), (150, 2)])
def test_pages_outside_the_pool(fmt, b, stray, scale, n, g):
    """Block 3 of the first of two sequences has no page; page 0, whose scales a
    careless read would take, holds anything."""
    lens, H = [5 * b - 3, 200], 2
    n = [lens[0] if n is None else min(n, lens[0]), 9]
    p = Pair(2, H, max(5 * b, 256), b, fmt, [5 * b, 256], paged=True)
    for s in range(2):  # page 0 to nobody: its owner, if it has one, moves to the spare pages
        at = np.argwhere(p.table[s] == 0)
        if len(at):
            free = max(set(range(p.dev.k.shape[0])) - set(p.table.flatten().tolist()))
            p.table[s, at[0, 0]] = free
    p.table[0, 3] = stray
    p.dev.block_table.copy_(torch.from_numpy(p.table))
    for t in (p.dev.k_scale, p.dev.v_scale):
        t[0] = scale
    at = cumulative(lens)
    k, v = rows(at[-1], H, 1200)
    old = [L - x for L, x in zip(lens, n)]
    keep = np.concatenate([np.arange(at[s], at[s] + old[s]) for s in range(2)])
    new = np.concatenate([np.arange(at[s] + old[s], at[s + 1]) for s in range(2)])
    R.store_rows_q8(p.dev, k[keep], v[keep], i32(cumulative(old)), i32(old))
    p.ref.store(f64(k[keep]), f64(v[keep]), cumulative(old), old)
    q, cu = randn((len(new), H * g, D), 1201).cuda(), cumulative(n)
    out, lse = R.dense_rectify_q8(p.dev, q, k[new], v[new], i32(cu), i32(lens), max(lens))
    torch.cuda.synchronize()
    p.ref.store(f64(k[new]), f64(v[new]), cu, lens)
    for name in "kv":
        p.ref.codes[name][0, :, 3] = 0
    got, gl, q64 = f64(out), lse.cpu().numpy(), f64(q)
    for s, L in enumerate(lens):
        for h in (0, H * g - 1):
            o, bound, l, lbound = reference(q64[cu[s]:cu[s + 1], h], p.ref.values("k", s, h // g, L),
                                            p.ref.values("v", s, h // g, L), L - n[s] + np.arange(n[s]), True)
            check(got[cu[s]:cu[s + 1], h], o, bound, f"{fmt} b={b} out {s},{h}")
            check(gl[cu[s]:cu[s + 1], h], l, lbound, f"{fmt} b={b} lse {s},{h}")
