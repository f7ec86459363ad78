"""Calls that are given a stream make their new tensors on it, on CPU tensors that
call themselves GPU tensors and with a library that does nothing."""
import contextlib

import pytest
import torch

import paper_2506_04108_amd as R

B, H, HQ, CAP, F = 2, 2, 4, 64, 16


class OnGpu(torch.Tensor):
    is_cuda = True


class Library:
    """Sizes are 512 bytes, calls succeed."""

    def __getattr__(self, name):
        return lambda *args: 512 if name.endswith("_size") else 0


@pytest.fixture
def made(monkeypatch):
    """The streams on which tensors were made."""
    current, made = [None], []

    @contextlib.contextmanager
    def on(stream):
        before, current[0] = current[0], stream
        yield
        current[0] = before

    def noted(make):
        def wrapper(*args, **kw):
            made.append(current[0])
            return make(*args, **{**kw, "device": "cpu"}).as_subclass(OnGpu)
        return wrapper

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(R, "lib", lambda: Library())
    monkeypatch.setattr(R, "_stream", lambda stream: 0)
    monkeypatch.setattr(R, "_devices", 1)
    for name in ("empty", "zeros"):
        monkeypatch.setattr(torch, name, noted(getattr(torch, name)))
    monkeypatch.setattr(OnGpu, "new_empty", noted(torch.Tensor.new_empty), raising=False)
    return made


def calls():
    bf = lambda *shape: torch.ones(shape, dtype=torch.bfloat16).as_subclass(OnGpu)  # noqa: E731
    ints = lambda *shape: torch.ones(shape, dtype=torch.int32).as_subclass(OnGpu)  # noqa: E731
    c = R.KVCache.empty(B, H, CAP, 16)
    q8 = R.KVCacheQ8.empty(B, H, CAP, 16)
    q, kv, lens, idx, n = bf(B, HQ, 128), bf(B, H, 128), ints(B), ints(B, H, 1), ints(B, H)
    select = dict(max_seq_len=40, sparsity=0.5, min_blocks=1)
    return {
        "select_blocks": lambda s: R.select_blocks(c, q, lens, stream=s, **select),
        "select_blocks over 8 bits": lambda s: R.select_blocks(q8, q, lens, stream=s, **select),
        "append_select": lambda s: R.append_select(c, kv, kv, q, lens, stream=s, **select),
        "sparse_decode": lambda s: R.sparse_decode(c, q, lens, idx, n, stream=s),
        "decode_step": lambda s: R.decode_step(c, kv, kv, q, lens, stream=s, **select),
        "dense_rectify": lambda s: R.dense_rectify(c, bf(B, HQ, F, 128), bf(B, H, F, 128), bf(B, H, F, 128), lens, 40,
                                                   stream=s),
        "prompt_attention": lambda s: R.prompt_attention(q, kv, kv, ints(B + 1), stream=s),
        "load_rows_q8": lambda s: R.load_rows_q8(q8, ints(B + 1), lens, 3, stream=s),
        "sparse_decode_q8": lambda s: R.sparse_decode_q8(q8, q, lens, idx, n, stream=s),
        "dense_rectify_q8": lambda s: R.dense_rectify_q8(q8, q, kv, kv, ints(B + 1), lens, 40, stream=s),
    }


@pytest.mark.parametrize("name", [
    "select_blocks", "select_blocks over 8 bits", "append_select", "sparse_decode", "decode_step", "dense_rectify",
    "prompt_attention", "load_rows_q8", "sparse_decode_q8", "dense_rectify_q8"])
def test_new_tensors_belong_to_the_stream(made, name):
    call = calls()[name]
    made.clear()
    call("side")
    assert made and set(made) == {"side"}, made
    made.clear()
    call(None)
    assert made and set(made) == {None}, made
