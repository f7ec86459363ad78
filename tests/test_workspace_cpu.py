"""What a Workspace hands out, on the CPU."""
import gc
import weakref

import torch

import paper_2506_04108_amd as R


def test_each_layout_has_its_own_memory():
    """A call of another batch, head count or operation never finds what an
    earlier one keeps (tickets that do not start at zero)."""
    ws = R.Workspace("cpu")
    a = ws.get(1000, ("decode", 2, 8))
    a.fill_(7)
    b = ws.get(500, ("decode", 4, 8))
    assert b.data_ptr() != a.data_ptr() and not b.any() and ws.buf is b
    b.fill_(9)
    c = ws.get(500, ("select", 4, 8))
    assert not c.any() and len({x.data_ptr() for x in (a, b, c)}) == 3
    assert ws.get(900, ("decode", 2, 8)) is a and (a == 7).all() and ws.buf is a
    assert ws.get(500, ("decode", 4, 8)) is b and (b == 9).all()
    grown = ws.get(2000, ("decode", 4, 8))
    assert grown.numel() == 2000 and not grown.any()
    assert ws.turn_to(("decode", 2, 8)) is a and ws.turn_to(("decode", 4, 8)) is grown
    assert ws.turn_to(("step", 4, 8)) is None


def test_a_buffer_sized_beforehand():
    ws = R.Workspace("cpu")
    a = ws.get(4096)
    assert ws.get(100, ("step", 1, 2)) is a and ws.get(50) is a
    assert ws.get(100, ("step", 2, 2)) is not a


def test_a_recorded_buffer_stays(monkeypatch):
    """A larger buffer does not free the one whose address a graph holds."""
    class OnGpu(torch.Tensor):
        is_cuda = True

    zeros = torch.zeros
    monkeypatch.setattr(torch, "zeros", lambda *size, **kw: zeros(*size, **kw).as_subclass(OnGpu))
    ws, recording = R.Workspace("cpu"), [True]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: recording[0])
    first = weakref.ref(ws.get(1000, ("decode", 1, 1)))
    second = weakref.ref(ws.get(2000, ("decode", 1, 1)))
    recording[0] = False
    third = weakref.ref(ws.get(3000, ("decode", 1, 1)))
    ws.get(4000, ("decode", 1, 1))
    gc.collect()
    assert first() is not None and second() is not None and third() is None
    recording[0] = True
    for _ in range(3):
        ws.get(100)
    assert len(ws._recorded) == 3
