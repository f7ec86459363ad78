"""Packed prompts and the 8-bit cache at their far ends: contexts over many
tables of block factors, long lists, many sequences, offsets past 32 bits, two
graphs on one workspace, a cache whose tensors change. Bounds as in
test_gpu_q8.py and test_gpu_prompt.py."""
import numpy as np
import pytest
import torch

import paper_2506_04108_amd as R
from rows_ref import D, DTYPE, cumulative, f64, i32, randn
from test_gpu_prompt import run
from test_gpu_q8 import decode_check, filled, rectify, rectify_check, rows, some_blocks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,b,paged", [("int8", 16, True), ("e4m3", 16, False), ("int8", 32, False),
                                         ("e4m3", 64, True)])
def test_rectify_long_splits(fmt, b, paged):
    """Splits of more than 64 blocks, with a scale for each block far from its
    neighbours', 4 waves (short windows) and 8 (long ones)."""
    lens, H = [9000, 8871, 6000, 8999], 8
    p = filled(4, H, b, fmt, lens, 900 + b, paged)
    for name in "kv":
        scale = getattr(p.dev, name + "_scale")
        f = torch.exp2(torch.randint(-3, 2, scale.shape, generator=torch.Generator().manual_seed(b)).float()).cuda()
        scale.mul_(f)
        for s, L in enumerate(lens):
            for m in range(-(-L // b)):
                fs = f[s, :, m] if not paged else f[int(p.table[s, m])]
                p.ref.scale[name][s, :, m] *= fs.cpu().numpy()
    for n, g in (([17, 3, 32, 1], 4), ([150, 60, 257, 200], 2)):
        q, cu, out, lse = rectify(p, lens, n, H * g, 901)
        rectify_check(p, q, cu, lens, out, lse, f"{fmt} b={b} paged={paged} n={n}", heads=[0, H * g - 1])


def test_rectify_many_sequences():
    """More sequences than a wave has lanes, some without rows."""
    B, H, g = 150, 1, 4
    lens = [(37 * s) % 211 for s in range(B)]
    n = [min(L, (5 * s) % 23) for s, L in enumerate(lens)]
    p = filled(B, H, 16, "int8", lens, 910)
    q, cu, out, lse = rectify(p, lens, n, H * g, 911)
    rectify_check(p, q, cu, lens, out, lse, "150 sequences", heads=[0, 3])
    p.same(lens, "150 sequences")


@pytest.mark.parametrize("b", [16, 64])
@pytest.mark.parametrize("splits", [1, 3])
def test_decode_long_lists(b, splits):
    """Lists of more blocks than a split holds at a time, every block of 20000 tokens."""
    lens, H, g = [20000, 12345], 1, 4
    p = filled(2, H, b, "int8", lens, 920)
    ids, nsel = some_blocks(lens, H, b, -(-20000 // b), 1)
    q = randn((2, H * g, D), 921).cuda()
    out, lse = R.sparse_decode_q8(p.dev, q, i32(lens), torch.from_numpy(ids).cuda(), torch.from_numpy(nsel).cuda(),
                                  num_splits=splits)
    torch.cuda.synchronize()
    decode_check(p, q, lens, ids, nsel, out, lse, f"b={b} splits={splits}")


def test_prompt_lengths_around_the_tiles():
    """Every length next to a tile and to a workgroup's rows, in one call and alone."""
    run([1, 17, 18, 19, 36, 37, 38, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257], 14, 2, seed=930)
    for n in (16, 17, 33, 65):
        run([n], 8, 1, seed=931)


def test_prompt_rows_far_apart():
    """Rows 32 MB apart: offsets past 2^32 bytes."""
    n, stride = 300, 1 << 24
    big = torch.empty(n * stride, dtype=torch.bfloat16, device="cuda").view(n, stride)
    x = big[:, :6 * D].view(n, 6, D)
    near = randn((n, 6, D), 940).cuda()
    x.copy_(near)
    q, k, v = x[:, :4], x[:, 4:5], x[:, 5:]
    assert q.stride(0) == stride
    cu = i32([0, 130, 300])
    out, lse = R.prompt_attention(q, k, v, cu)
    want, wl = R.prompt_attention(*(t.contiguous() for t in (near[:, :4], near[:, 4:5], near[:, 5:])), cu)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, wl)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_caches_of_2_gib(fmt):
    """The last sequence and kv head of a cache of 2^31 codes: the same bits as in a
    cache of its own."""
    B, H, cap, b, n = 8, 8, 1 << 18, 16, 40
    lens = [0] * (B - 1) + [cap - 3]
    big, one = R.KVCacheQ8.empty(B, H, cap, b, DTYPE[fmt]), R.KVCacheQ8.empty(1, H, cap, b, DTYPE[fmt])
    gen = torch.Generator(device="cuda").manual_seed(950)
    for name in ("k", "v"):
        t = torch.randint(0, 100, (H, cap, D), generator=gen, device="cuda", dtype=torch.int8)
        for c in (big, one):
            getattr(c, name)[-1] = t.view(DTYPE[fmt])
            getattr(c, name + "_scale")[-1] = 0.01
    k, v = rows(n, H, 951)
    q = randn((n, 4 * H, D), 952).cuda()
    cu = [0] * B + [n]
    ids = torch.arange(cap // b - 900, cap // b, dtype=torch.int32, device="cuda").expand(1, H, 900).contiguous()
    results = []
    for c, L, at in ((big, lens, cu), (one, lens[-1:], [0, n])):
        batch = len(L)
        nsel = torch.zeros((batch, H), dtype=torch.int32, device="cuda")
        nsel[-1] = 900
        idx = ids.expand(batch, H, 900).contiguous()
        R.store_rows_q8(c, k, v, i32(at), i32(L))
        back = R.load_rows_q8(c, i32(at), i32(L), n)
        qs = q[:1].expand(batch, 4 * H, D).contiguous()
        dec = R.sparse_decode_q8(c, qs, i32(L), idx, nsel, num_splits=16)
        rec = R.dense_rectify_q8(c, q, k, v, i32(at), i32(L), cap)
        torch.cuda.synchronize()
        results.append((*back, dec[0][-1], dec[1][-1], c.k[-1, :, -48:].view(torch.int8).clone(), c.k_scale[-1].clone(),
                        c.kmin[-1].clone()))
        results[-1] += (rec[0], rec[1])
    for i, (x, y) in enumerate(zip(*results)):
        if i < 7:
            assert torch.equal(x, y), i
    # The splits of the two calls differ: fp32 sums, then bf16 (2^-8 each).
    (xo, xl), (yo, yl) = results[0][-2:], results[1][-2:]
    assert ((xo.float() - yo.float()).abs() <= 2.0 ** -7 * yo.float().abs() + 2.0 ** -10 * yo.float().abs().max()).all()
    assert ((xl - yl).abs() <= 2.0 ** -18 * yl.abs()).all()


@pytest.mark.parametrize("kind", ["decode", "rectify"])
def test_two_graphs_on_one_workspace(kind):
    """Two calls of different sizes recorded apart, replayed in turn, with the
    program's own calls on the same workspace between them."""
    lens, H, b = [1500, 700], 2, 16
    p = filled(2, H, b, "int8", lens, 960)
    lt, calls = i32(lens), []
    for n in (60, 20):
        if kind == "decode":
            ids, nsel = (torch.from_numpy(x).cuda() for x in some_blocks(lens, H, b, n, 2))
            q = randn((2, 8, D), 961 + n).cuda()
            calls.append(lambda q=q, ids=ids, nsel=nsel, **kw: R.sparse_decode_q8(p.dev, q, lt, ids, nsel, **kw))
        else:
            k, v = rows(2 * n, H, 962)
            q, cu = randn((2 * n, 8, D), 963).cuda(), i32([0, n, 2 * n])
            calls.append(lambda q=q, k=k, v=v, cu=cu, **kw: R.dense_rectify_q8(p.dev, q, k, v, cu, lt, max(lens), **kw))
            calls[-1]()
    want = []
    for call in calls:
        call()
        want.append([x.clone() for x in call()])
    ws, outs, graphs = R.Workspace("cuda"), [], []
    for call in calls:
        outs.append(call(workspace=ws))
    torch.cuda.synchronize()
    for call, (out, lse) in zip(calls, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(out=out, lse=lse, workspace=ws)
    for turn in ((0, 1), (1, 0), (0, 0), (1, 1), (1, 0)):
        for i in turn:
            for x in outs[i]:
                x.fill_(float("nan"))
            graphs[i].replay()
            torch.cuda.synchronize()
            if kind == "decode":
                assert torch.equal(outs[i][0], want[i][0]) and torch.equal(outs[i][1], want[i][1]), (turn, i)
            else:  # the calls store into one cache: each is checked against its own, made now
                for x, w in zip(outs[i], calls[i](workspace=ws)):
                    assert torch.equal(x, w), (turn, i)


def test_cache_whose_tensors_change():
    """A tensor that is replaced, or moved by set_, is the one the next call reads."""
    lens, H, b = [50], 1, 16
    a, c = filled(1, H, b, "int8", lens, 970), filled(1, H, b, "int8", lens, 971)
    cu, lt = i32([0, 50]), i32(lens)

    def read(cache):
        k, v = R.load_rows_q8(cache, cu, lt, 50)
        torch.cuda.synchronize()
        return f64(k)

    first, second = read(a.dev), read(c.dev)
    assert not np.array_equal(first, second)
    a.dev.k, a.dev.k_scale = c.dev.k, c.dev.k_scale
    assert np.array_equal(read(a.dev), second)
    p = filled(1, H, b, "int8", lens, 972, paged=True)
    before = read(p.dev)
    turned = torch.full((1, p.dev.block_table.shape[1] + 64), -1, dtype=torch.int32, device="cuda")
    turned[0, :4] = p.dev.block_table[0, :4].flip(0)
    p.dev.block_table.set_(turned[:, :4].contiguous())
    assert np.array_equal(read(p.dev)[16:32], before[32:48])  # full blocks 1 and 2 have changed places
    assert not np.array_equal(read(p.dev), before)
    p.dev.block_table.set_(torch.full((1, 3), -1, dtype=torch.int32, device="cuda"))
    with pytest.raises((ValueError, R.ResaError)):
        R.load_rows_q8(p.dev, cu, lt, 50)


@pytest.mark.parametrize("lens,hq,hkv,heads", [([6000, 1, 64, 0, 9001], 32, 8, [3, 30]), ([2561, 2600, 2599], 28, 4, [0, 27]),
                                               ([8192], 8, 8, [7])])
def test_prompts_long_on_average(lens, hq, hkv, heads):
    run(lens, hq, hkv, seed=980, heads=heads)


@pytest.mark.parametrize("lens,n,g", [([12000, 100, 3000, 17, 700, 5], [20, 20, 0, 17, 9, 5], 4),
                                      ([200, 15000, 64, 1], [90, 60, 64, 1], 8),
                                      ([9000, 300], [700, 300], 3), ([33] * 80 + [7000, 2], [3] * 80 + [16, 2], 4)])
@pytest.mark.parametrize("paged", [False, True])
def test_rectify_lengths_far_apart(lens, n, g, paged):
    """The long sequences take more splits than the short ones."""
    H = 1 if len(lens) > 10 else 2
    p = filled(len(lens), H, 32, "int8" if paged else "e4m3", lens, 990, paged)
    ws = R.Workspace("cuda")
    for _ in range(2):
        q, cu, out, lse = rectify(p, lens, n, H * g, 991, ws=ws)
        rectify_check(p, q, cu, lens, out, lse, f"lens={lens[:6]} n={n[:6]} g={g} paged={paged}", heads=[0, H * g - 1])
    p.same(lens, "lengths far apart")
