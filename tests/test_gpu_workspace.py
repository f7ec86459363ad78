"""One Workspace over calls of other batches, kv heads and operations, in turn and
recorded in graphs: the results of workspaces of their own."""
import pytest
import torch

import paper_2506_04108_amd as R
from rows_ref import D, cumulative, i32, randn
from test_gpu_q8 import filled, rows, some_blocks

pytestmark = pytest.mark.gpu


def decode_call(B, H, L, seed, splits, g=4):
    lens = [L + 3 * s for s in range(B)]
    p = filled(B, H, 16, "int8", lens, seed)
    ids, nsel = (torch.from_numpy(x).cuda() for x in some_blocks(lens, H, 16, 40, seed))
    q, lt = randn((B, H * g, D), seed + 1).cuda(), i32(lens)
    return lambda **kw: R.sparse_decode_q8(p.dev, q, lt, ids, nsel, num_splits=splits, **kw)


def bf16_decode_call(B, H, L, seed, splits, g=4):
    c = R.KVCache.empty(B, H, -(-L // 16) * 16, 16)
    c.k.copy_(randn(c.k.shape, seed)), c.v.copy_(randn(c.v.shape, seed + 1))
    ids, nsel = (torch.from_numpy(x).cuda() for x in some_blocks([L] * B, H, 16, 40, seed))
    q, lt = randn((B, H * g, D), seed + 2).cuda(), i32([L] * B)
    return lambda **kw: R.sparse_decode(c, q, lt, ids, nsel, num_splits=splits, **kw)


def select_call(B, H, L, seed, g=4):
    lens = [L] * B
    p = filled(B, H, 16, "int8", lens, seed)
    q, lt = randn((B, H * g, D), seed + 1).cuda(), i32(lens)

    def call(out=None, lse=None, **kw):
        ids, n = R.select_blocks(p.dev, q, lt, L, 0.8, 4, 1, **kw)
        return ids, n
    return call


def rectify_call(B, H, L, n, seed, g=4):
    lens = [L] * B
    p = filled(B, H, 16, "int8", lens, seed)
    (k, v), q = rows(B * n, H, seed + 1), randn((B * n, H * g, D), seed + 2).cuda()
    cu, lt = i32(cumulative([n] * B)), i32(lens)
    first = R.dense_rectify_q8(p.dev, q, k, v, cu, lt, L)
    assert first[0].isfinite().all()
    return lambda **kw: R.dense_rectify_q8(p.dev, q, k, v, cu, lt, L, **kw)


def some_calls():
    return [decode_call(1, 2, 900, 1, 0), decode_call(4, 2, 700, 2, 20), bf16_decode_call(2, 4, 800, 3, 20),
            select_call(3, 2, 6000, 4), rectify_call(2, 2, 3000, 8, 5), decode_call(2, 3, 600, 6, 3),
            select_call(1, 2, 6000, 7), decode_call(4, 2, 700, 8, 20)]


def test_calls_in_turn():
    ws, calls = R.Workspace(), some_calls()
    want = [[x.clone() for x in call()] for call in calls]
    for order in (range(8), reversed(range(8)), (1, 0, 1, 3, 6, 3, 2, 4, 1, 4, 7, 5, 0)):
        for i in order:
            for x, y in zip(calls[i](workspace=ws), want[i]):
                assert torch.equal(x, y), i


def test_graphs_in_turn():
    ws, calls = R.Workspace(), some_calls()
    calls = [c for i, c in enumerate(calls) if i not in (3, 6)]
    want = [[x.clone() for x in call()] for call in calls]
    outs = [call(workspace=ws) for call in calls]
    torch.cuda.synchronize()
    graphs = []
    for call, (out, lse) in zip(calls, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(out=out, lse=lse, workspace=ws)
    for order in (range(6), reversed(range(6)), (1, 0, 1, 3, 2, 4, 1, 4, 5, 0)):
        for i in order:
            for x in outs[i]:
                x.fill_(float("nan"))
            graphs[i].replay()
            eager = calls[(i + 1) % 6](workspace=ws)
            torch.cuda.synchronize()
            for x, y in zip(outs[i], want[i]):
                assert torch.equal(x, y), i
            for x, y in zip(eager, want[(i + 1) % 6]):
                assert torch.equal(x, y), (i, "eager")


@pytest.mark.parametrize("kind", ["decode", "rectify"])
def test_graph_before_a_larger_call(kind):
    """A graph recorded on a small buffer, replayed after a larger call took a
    larger one and other tensors came and went."""
    ws = R.Workspace()
    small, large = ((decode_call(2, 2, 700, 21, 4), decode_call(2, 2, 900, 22, 200)) if kind == "decode" else
                    (rectify_call(1, 2, 1500, 2, 23), rectify_call(1, 2, 9000, 16, 24)))
    want, want_large = ([x.clone() for x in c()] for c in (small, large))
    out, lse = small(workspace=ws)
    torch.cuda.synchronize()
    graph, size = torch.cuda.CUDAGraph(), ws.buf.numel()
    with torch.cuda.graph(graph):
        small(out=out, lse=lse, workspace=ws)
    for turn in range(3):
        got = large(workspace=ws)
        assert ws.buf.numel() > size
        junk = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
        out.fill_(float("nan")), lse.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all((j == 255).all() for j in junk), turn
        for x, y in zip((out, lse, *got), (*want, *want_large)):
            assert torch.equal(x, y), turn
        del junk


@pytest.mark.parametrize("i", range(5))
def test_calls_on_a_stream_while_the_current_one_is_busy(i):
    """Nothing of a call on a side stream waits for the current stream, or
    overtakes what it needs there."""
    call = some_calls()[i]
    want = [x.clone() for x in call()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        junk = [torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        del junk
        torch.cuda._sleep(20_000_000)  # some 10 ms
        got = call(stream=side)
        side.synchronize()
        with torch.cuda.stream(side):
            same = [torch.equal(x, y) for x, y in zip(got, want)]
        assert all(same)
        torch.cuda.synchronize()
