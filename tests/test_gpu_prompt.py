"""Packed prompt attention against the plain 64-bit form.

Bound, element by element, with A = sum_j w_j |v_j| of the exact weights: a
weight is off by its score's and exponential's error (rows_ref.score_error) and
by its rounding to bf16, 2^-8 of itself (half of bf16's eps); the result is
rounded to bf16, 2^-8 of itself. lse is fp32: the score's error, and 2^-22 of
its size."""
import numpy as np
import pytest
import torch

import paper_2506_04108_amd as R
from rows_ref import D, attend, check, cumulative, f64, i32, randn, score_error

pytestmark = pytest.mark.gpu


def reference(q, k, v, lens, start, scale, heads=None):
    """out, lse and their bounds for the packed rows from `start` on."""
    hq, g = q.shape[1], q.shape[1] // k.shape[1]
    T = sum(lens)
    out, bound = np.zeros((T, hq, D)), np.ones((T, hq, D))
    lse, lbound = np.zeros((T, hq)), np.ones((T, hq))
    at = 0
    for n in lens:
        lo = start + at
        for h in heads or range(hq):
            o, l, A, reach = attend(q[lo:lo + n, h], k[lo:lo + n, h // g], v[lo:lo + n, h // g], scale, np.arange(n))
            e = score_error(reach)[:, None]
            out[at:at + n, h], lse[at:at + n, h] = o, l
            bound[at:at + n, h] = A * (e + 2.0 ** -8) * (1 + 2.0 ** -8) + np.abs(o) * 2.0 ** -8 + 1e-30
            lbound[at:at + n, h] = e[:, 0] + np.abs(l) * 2.0 ** -22
        at += n
    return out, lse, bound, lbound


def inputs(lens, hq, hkv, seed, fused=False, spread=1.0, pad=0):
    T = sum(lens) + pad
    x = randn((T, hq + 2 * hkv, D), seed, spread).cuda()
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    return (q, k, v) if fused else (q.contiguous(), k.contiguous(), v.contiguous())


def run(lens, hq, hkv, seed=1, fused=False, spread=1.0, scale=D ** -0.5, heads=None):
    q, k, v = inputs(lens, hq, hkv, seed, fused, spread)
    out, lse = R.prompt_attention(q, k, v, i32(cumulative(lens)), sm_scale=scale)
    torch.cuda.synchronize()
    assert out.dtype == torch.bfloat16 and out.shape == q.shape and lse.shape == q.shape[:2]
    ro, rl, bo, bl = reference(f64(q), f64(k), f64(v), lens, 0, scale, heads)
    sel = list(heads or range(hq))
    what = f"prompt lens={lens[:6]} heads={hq}/{hkv} seed={seed}"
    check(f64(out)[:, sel], ro[:, sel], bo[:, sel], what + " out")
    check(lse.cpu().numpy()[:, sel], rl[:, sel], bl[:, sel], what + " lse")


@pytest.mark.parametrize("hq,hkv", [(1, 1), (2, 1), (6, 2), (4, 1), (5, 1), (12, 2), (14, 2), (16, 2)])
def test_group_sizes(hq, hkv):
    run([1, 37, 130], hq, hkv, seed=hq)


@pytest.mark.parametrize("lens", [[1], [2], [31, 32, 33], [63, 64, 65], [127, 128, 129], [0, 1, 0, 0, 5, 0], [300],
                                  [255, 1, 256, 2, 257], [513]])
def test_lengths(lens):
    run(lens, 8, 2, seed=sum(lens))


@pytest.mark.parametrize("lens,hq,hkv,heads", [([4700, 33, 1501], 32, 8, [0, 13, 31]), ([3001] * 3, 28, 4, [6, 20]),
                                               ([6007], 32, 8, [5]), ([9001, 100], 16, 2, [9])])
def test_long(lens, hq, hkv, heads):
    """Enough query blocks for workgroups of 8 waves."""
    run(lens, hq, hkv, seed=3, heads=heads)


def test_many_sequences():
    """More sequences than a wave has lanes, some empty."""
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 40, 150)]
    lens[70], lens[149] = 333, 1
    run(lens, 8, 2, seed=5, heads=[1, 6])


def test_parts_of_a_projection():
    run([77, 1, 190], 8, 2, seed=6, fused=True)
    run([4096, 1801], 32, 8, seed=7, fused=True, heads=[3])


@pytest.mark.parametrize("scale", [0.0, -0.09, 1.5])
def test_scales(scale):
    run([65, 200], 8, 2, seed=8, scale=scale, spread=0.7)


def test_peaked_logits():
    """Scores of some hundreds: the softmax reference has to move."""
    run([700], 4, 1, seed=9, spread=4.0, scale=1.0)


def test_climbing_logits():
    lens = [900]
    q, k, v = inputs(lens, 4, 1, 10)
    q[..., 7] = 8.0
    k[:, 0, 7] = torch.linspace(0, 400, 900).bfloat16().cuda()
    out, lse = R.prompt_attention(q, k, v, i32([0, 900]))
    torch.cuda.synchronize()
    ro, rl, bo, bl = reference(f64(q), f64(k), f64(v), lens, 0, D ** -0.5)
    check(f64(out), ro, bo, "climbing out")
    check(lse.cpu().numpy(), rl, bl, "climbing lse")


@pytest.mark.parametrize("scale", [2.0 ** 96, 2.0 ** 60, 2.0 ** -90])
def test_range_of_values(scale):
    q, k, v = inputs([150], 4, 1, 11)
    v = (v.float().clamp(-1, 1) * scale).bfloat16()
    out, _ = R.prompt_attention(q, k, v, i32([0, 150]))
    torch.cuda.synchronize()
    ro, _, bo, _ = reference(f64(q), f64(k), f64(v), [150], 0, D ** -0.5)
    check(f64(out) / scale, ro / scale, bo / scale, f"V of {scale:.0e}")


@pytest.mark.parametrize("lens,hq,hkv", [([200], 4, 1), ([90, 150, 64], 14, 2), ([5000], 32, 8)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_values_that_are_not_finite_where_masked(lens, hq, hkv, bad):
    """A V value that is no number reaches the rows that see its key, in its
    dim, and no others; a K row that holds one spoils the rows that see it."""
    g = hq // hkv
    q, k, v = inputs(lens, hq, hkv, 12)
    clean = f64(v)
    cu = cumulative(lens)
    spots = [(cu[i] + n * 5 // 8, i, 5 + i) for i, n in enumerate(lens)]
    for row, _, dim in spots:
        v[row, 0, dim] = bad
    out, lse = R.prompt_attention(q, k, v, i32(cu))
    torch.cuda.synchronize()
    heads = list(range(hq)) if len(lens) > 1 or lens[0] < 1000 else [0, g - 1, g]
    ro, rl, bo, bl = reference(f64(q), f64(k), clean, lens, 0, D ** -0.5, heads)
    got = f64(out)
    for row, i, dim in spots:
        seen = got[row:cu[i + 1], :g, dim]
        assert (np.isnan(seen) if bad != bad else seen == bad).all(), (i, row)
        got[row:cu[i + 1], :g, dim] = ro[row:cu[i + 1], :g, dim]
    check(got[:, heads], ro[:, heads], bo[:, heads], f"masked {bad} out")
    check(lse.cpu().numpy()[:, heads], rl[:, heads], bl[:, heads], f"masked {bad} lse")
    # keys
    q, k, v = inputs(lens, hq, hkv, 12)
    for row, _, dim in spots:
        k[row, 0, dim] = bad
    out, lse = R.prompt_attention(q, k, v, i32(cu))
    torch.cuda.synchronize()
    got = f64(out)
    for row, i, _ in spots:
        if bad != bad:
            assert np.isnan(got[row:cu[i + 1], :g]).all()
        got[row:cu[i + 1], :g] = ro[row:cu[i + 1], :g]
    check(got[:, heads], ro[:, heads], bo[:, heads], f"masked key {bad}")


def test_rows_of_no_sequence():
    """Rows before, between (an interval that the offsets skip is not possible:
    they are shared) and behind the sequences: not read, not written."""
    lens, start, T = [40, 0, 70], 9, 150
    q, k, v = (x.clone() for x in inputs([T], 8, 2, 13))
    for x in (q, k, v):
        x[:start] = float("nan")
        x[start + sum(lens):] = float("nan")
    cu = [start + c for c in cumulative(lens)]
    out = torch.full((T, 8, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, 8), 7.0, device="cuda")
    R.prompt_attention(q, k, v, i32(cu), out=out, lse=lse)
    torch.cuda.synchronize()
    ro, rl, bo, bl = reference(f64(q), f64(k), f64(v), lens, start, D ** -0.5)
    got, gl = f64(out), lse.cpu().numpy()
    end = start + sum(lens)
    check(got[start:end], ro, bo, "inner rows")
    check(gl[start:end], rl, bl, "inner lse")
    assert (got[:start] == 7).all() and (got[end:] == 7).all() and (gl[:start] == 7).all() and (gl[end:] == 7).all()


def test_offsets_are_cut_to_the_rows():
    """Offsets past the rows, or falling, name no row outside the tensors."""
    q, k, v = inputs([60], 4, 1, 14)
    out, lse = R.prompt_attention(q, k, v, i32([-5, 20, 1000, 900]))
    torch.cuda.synchronize()
    ro, rl, bo, bl = reference(f64(q), f64(k), f64(v), [20, 40], 0, D ** -0.5)
    check(f64(out), ro, bo, "cut offsets")
    check(lse.cpu().numpy(), rl, bl, "cut offsets lse")


def test_no_rows_and_no_lse():
    q, k, v = inputs([0], 4, 1, 15)
    out, lse = R.prompt_attention(q, k, v, i32([0, 0]))
    assert out.shape == (0, 4, D) and lse.shape == (0, 4)
    q, k, v = inputs([33], 4, 1, 16)
    a, _ = R.prompt_attention(q, k, v, i32([0, 33]))
    b, none = R.prompt_attention(q, k, v, i32([0, 33]), with_lse=False)
    torch.cuda.synchronize()
    assert none is None and torch.equal(a, b)


def test_graph_and_streams():
    """Recorded once and replayed with other inputs and other lengths; on a
    stream of the caller's."""
    T = 400
    sets = [(inputs([T], 8, 2, 20 + i), cumulative(l)) for i, l in enumerate(([T], [1, 399], [200, 150, 50]))]
    q, k, v = (torch.zeros_like(x) for x in sets[0][0])
    cu = i32([0, 0, 0, 0])
    out, lse = torch.zeros_like(q), torch.zeros((T, 8), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    R.prompt_attention(q, k, v, cu, out=out, lse=lse, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        R.prompt_attention(q, k, v, cu, out=out, lse=lse)
    for _ in range(2):
        for (a, b, c), offsets in sets:
            q.copy_(a), k.copy_(b), v.copy_(c)
            cu.copy_(i32(offsets + [T] * (4 - len(offsets))))
            graph.replay()
            torch.cuda.synchronize()
            want, wl = R.prompt_attention(a, b, c, i32(offsets))
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(lse, wl)


def test_refusals():
    q, k, v = inputs([16], 4, 2, 17)
    cu = i32([0, 16])
    with pytest.raises(TypeError):
        R.prompt_attention(q.half(), k, v, cu)
    with pytest.raises(ValueError, match="shape"):
        R.prompt_attention(q, k, v[:8], cu)
    with pytest.raises(ValueError, match="within a row"):
        R.prompt_attention(q.transpose(1, 2).contiguous().transpose(1, 2), k, v, cu)
    with pytest.raises(R.ResaError, match="stride"):
        R.prompt_attention(q[:1].expand(16, 4, D), k, v, cu)
    with pytest.raises(ValueError, match="gradient"):
        R.prompt_attention(q.requires_grad_(), k, v, cu)
    with pytest.raises(R.ResaError, match="finite"):
        R.prompt_attention(q.detach(), k, v, cu, sm_scale=float("inf"))
    with pytest.raises(TypeError):
        R.prompt_attention(q.detach(), k, v, cu.long())
