"""The description that an 8-bit cache hands to the library, on CPU tensors that
call themselves GPU tensors: no call here reaches the library's device code."""
import copy
import dataclasses
import pickle

import pytest
import torch

import paper_2506_04108_amd as R

B, H, CAP, BS, PAGES = 4, 2, 64, 16, 8


class OnGpu(torch.Tensor):
    is_cuda = True


def on_gpu(t):
    return t.as_subclass(OnGpu)


@pytest.fixture(params=[False, True], ids=["contiguous", "paged"])
def cache(request, monkeypatch):
    monkeypatch.setattr(R, "_devices", 1)
    c = (R.KVCacheQ8.empty_paged(B, H, CAP, BS, PAGES, device="cpu") if request.param
         else R.KVCacheQ8.empty(B, H, CAP, BS, device="cpu"))
    for name in ("k", "v", "k_scale", "v_scale", "kmin", "kmax", "block_table"):
        if getattr(c, name) is not None:
            setattr(c, name, on_gpu(getattr(c, name)))
    c.desc_q8()
    return c


def tensors(c):
    return {n: getattr(c, n) for n in ("k", "v", "k_scale", "v_scale", "kmin", "kmax", "block_table")
            if getattr(c, n) is not None}


def test_fewer_sequences_or_pages_at_the_same_address(cache):
    for name, t in tensors(cache).items():
        t.set_(t[:2])
    d = cache.desc_q8()
    assert d.base.batch == 2 and d.base.num_pages == (2 if cache.paged else 0)
    assert d.base.k == cache.k.data_ptr() and d.base.capacity == CAP


def test_pool_of_fewer_pages(cache):
    if not cache.paged:
        pytest.skip("a pool")
    for name in ("k", "v", "k_scale", "v_scale"):
        t = getattr(cache, name)
        t.set_(t[:4])
    assert cache.desc_q8().base.num_pages == 4


def test_codes_of_another_format_at_the_same_address(cache):
    assert cache.desc_q8().format == 0
    for t in (cache.k, cache.v):
        t.data = t.data.view(torch.float8_e4m3fn)
    assert cache.desc_q8().format == 1


@pytest.mark.parametrize("name", ["k", "v", "k_scale", "v_scale", "kmin", "kmax", "block_table"])
@pytest.mark.parametrize("change", ["rows", "strides", "type"])
def test_one_tensor_that_no_longer_fits(cache, name, change):
    t = getattr(cache, name)
    if t is None:
        pytest.skip("no table")
    if change == "rows":
        t.set_(t[:1])
    elif change == "strides":
        t.as_strided_(t.shape, (0,) * t.dim())
    else:
        t.data = t.data.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()]
                             if name != "block_table" else torch.float32)
    with pytest.raises((TypeError, ValueError)):
        cache.desc_q8()


@pytest.mark.parametrize("used", [False, True])
def test_copies(used, monkeypatch):
    """Copies and pickles of a cache, before its first call and after it."""
    monkeypatch.setattr(R, "_devices", 1)
    c = R.KVCacheQ8.empty_paged(B, H, CAP, BS, PAGES, device="cpu")
    c.k.fill_(3)
    if used:
        gpu = R.KVCacheQ8(*(on_gpu(t) for t in (c.k, c.v, c.k_scale, c.v_scale, c.kmin, c.kmax)), BS,
                          on_gpu(c.block_table))
        gpu.desc_q8()
        shallow = copy.copy(gpu)
        assert shallow.k is gpu.k and shallow.desc_q8().base.k == gpu.k.data_ptr()
        shallow.block_table = on_gpu(gpu.block_table.clone())
        assert shallow.desc_q8().base.block_table != gpu.desc_q8().base.block_table
        object.__setattr__(c, "_checked", gpu._checked)
    for d in (copy.deepcopy(c), pickle.loads(pickle.dumps(c)), dataclasses.replace(c)):
        assert isinstance(d, R.KVCacheQ8) and d.block_size == BS and d.capacity == CAP and d.paged
        for name, t in tensors(c).items():
            assert torch.equal(getattr(d, name).view(torch.int8), t.view(torch.int8)), name
        with pytest.raises(ValueError, match="on the GPU"):
            d.desc_q8()


def calls(c):
    """Each call that takes rows, as a function of one of its tensors, and that tensor."""
    x, cu, lens = on_gpu(torch.zeros((3, H, 128), dtype=torch.bfloat16)), on_gpu(torch.zeros(B + 1, dtype=torch.int32)), \
        on_gpu(torch.zeros(B, dtype=torch.int32))
    q = on_gpu(torch.zeros((B, H, 128), dtype=torch.bfloat16))
    idx, n = on_gpu(torch.zeros((B, H, 1), dtype=torch.int32)), on_gpu(torch.zeros((B, H), dtype=torch.int32))
    return {
        "prompt": (x, lambda t: R.prompt_attention(x, t, x, cu)),
        "store": (x, lambda t: R.store_rows_q8(c, x, t, cu, lens)),
        "decode": (q, lambda t: R.sparse_decode_q8(c, t, lens, idx, n)),
        "rectify": (x, lambda t: R.dense_rectify_q8(c, t, x, x, cu, lens, CAP)),
    }


@pytest.mark.parametrize("name", ["prompt", "store", "decode", "rectify"])
def test_gradients_are_refused(cache, name):
    t, call = calls(cache)[name]
    with pytest.raises(ValueError, match="requires a gradient"):
        call(on_gpu(t.clone()).requires_grad_())
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(ValueError, match="tangent"):
            call(torch.autograd.forward_ad.make_dual(t, on_gpu(torch.ones_like(t))))
