"""What a Workspace hands out, on CPU tensors that call themselves GPU tensors."""
import gc
import weakref

import pytest
import torch

import paper_2506_04108_amd as R

A, B, C = ("decode", 2, 8), ("decode", 4, 8), ("select", 4, 8)


class OnGpu(torch.Tensor):
    is_cuda = True


@pytest.fixture
def recording(monkeypatch):
    """A switch: whether a graph is being recorded."""
    on, zeros = [False], torch.zeros
    monkeypatch.setattr(torch, "zeros", lambda *size, **kw: zeros(*size, **kw).as_subclass(OnGpu))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: on[0])
    return on


def test_no_layout_finds_what_another_left(recording):
    """A call of another batch, head count or operation never finds what an
    earlier one keeps (tickets that do not start at zero)."""
    ws = R.Workspace("cpu")
    a = ws.get(1000, A)
    a.fill_(7)
    assert ws.get(900, A) is a and (a == 7).all()
    for size, layout in ((500, B), (500, C), (1000, A), (20, B)):
        b = ws.get(size, layout)
        assert b is a and ws.buf is b and not b.any()  # one buffer, cleared
        b.fill_(9)
    grown = ws.get(2000, B)
    assert grown.numel() == 2000 and not grown.any()
    grown.fill_(5)
    assert ws.turn_to(C) is grown and not grown.any()


def test_a_buffer_sized_beforehand(recording):
    ws = R.Workspace("cpu")
    a = ws.get(4096)
    a.fill_(1)  # not by a call: it is the caller's to keep at zero
    assert ws.get(100, ("step", 1, 2)) is a and ws.get(50) is a and (a == 1).all()


def test_a_recorded_buffer_belongs_to_its_layout(recording):
    """Graphs of two layouts and eager calls of a third: each on memory that no
    other touches, in any order."""
    ws = R.Workspace("cpu")
    a = ws.get(1000, A)
    recording[0] = True
    assert ws.get(1000, A) is a
    b = ws.get(1000, B)
    recording[0] = False
    a.fill_(1), b.fill_(2)
    c = ws.get(1000, C)
    assert c is not a and c is not b and not c.any()
    c.fill_(3)
    for layout, want, value in ((A, a, 1), (C, c, 0), (B, b, 2), (A, a, 1), (B, b, 2), (("step", 1, 1), c, 0), (C, c, 0)):
        got = ws.get(800, layout)
        assert got is want and (got == value).all(), layout
        c.fill_(4)
    recording[0] = True
    d = ws.get(100, ("step", 9, 9))
    assert all(d is not x for x in (a, b, c)) and (a == 1).all() and (b == 2).all()


def test_a_recorded_buffer_stays(recording):
    """A larger buffer does not free the one whose address a graph holds."""
    ws = R.Workspace("cpu")
    recording[0] = True
    first = weakref.ref(ws.get(1000, A))
    second = weakref.ref(ws.get(2000, A))
    recording[0] = False
    third = weakref.ref(ws.get(3000, A))
    ws.get(4000, A)
    gc.collect()
    assert first() is not None and second() is not None and third() is None
    recording[0] = True
    for _ in range(3):
        ws.get(100)
    assert len(ws._recorded) == 3
