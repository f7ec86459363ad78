"""Host-side checks of the packed-row and 8-bit cache calls: bad arguments are
refused before the device is touched (no call here reaches a kernel), sizes of
workspaces, and the binding's own checks."""
import ctypes as C

import pytest
import torch

import paper_2506_04108_amd as R
from paper_2506_04108_amd import _lib as L

FAKE = 0x100000  # 16-byte aligned stand-in address: only used on rejected calls
SC = 0.088


def cache(**kw):
    own = {n: kw.pop(n) for n in ("k_scale", "v_scale", "format") if n in kw}
    d = dict(k=FAKE, v=FAKE, kmin=FAKE, kmax=FAKE, batch=2, num_kv_heads=2, head_dim=128, capacity=1024,
             block_size=16)
    d.update(kw)
    return L.KVCacheQ8Desc(L.KVCacheDesc(**d), own.get("k_scale", FAKE), own.get("v_scale", FAKE),
                           own.get("format", 0))


def expect(rc, code, text):
    assert rc == code, (rc, L.lib().resa_last_error())
    assert text in L.lib().resa_last_error().decode()


PROMPT = dict(q=FAKE, k=FAKE, v=FAKE, qs=1024, ks=256, vs=256, hq=8, hkv=2, d=128, cu=FAKE, B=2, T=64, sc=SC, out=FAKE,
              lse=FAKE)


@pytest.mark.parametrize("change,code,text", [
    (dict(q=None), 1, "q is NULL"), (dict(k=FAKE + 8), 1, "k is not 16-byte aligned"), (dict(v=None), 1, "v is NULL"),
    (dict(cu=FAKE + 2), 1, "cu_seqlens"), (dict(out=FAKE + 4), 1, "out"), (dict(lse=FAKE + 1), 1, "lse"),
    (dict(d=64), 2, "head_dim"), (dict(B=0), 1, "batch"), (dict(T=-1), 1, "num_rows"), (dict(hkv=0), 1, "num_kv_heads"),
    (dict(hq=7), 1, "multiple"), (dict(hq=18, qs=2304), 2, "group size"), (dict(qs=1020), 1, "q_stride"),
    (dict(ks=128), 1, "k_stride"), (dict(vs=1 << 26), 1, "v_stride"), (dict(vs=-256), 1, "v_stride"),
    (dict(sc=float("nan")), 1, "finite"), (dict(B=40000), 2, "65535"), (dict(T=2 ** 31 - 1), 2, "launch"),
])
def test_prompt_refusals(change, code, text):
    a = {**PROMPT, **change}
    rc = L.lib().resa_prompt_attention(a["q"], a["k"], a["v"], a["qs"], a["ks"], a["vs"], a["hq"], a["hkv"], a["d"],
                                       a["cu"], a["B"], a["T"], a["sc"], a["out"], a["lse"], None)
    expect(rc, code, text)


def test_no_rows_is_nothing_to_do():
    lib, c = L.lib(), cache()
    a = PROMPT
    assert lib.resa_prompt_attention(FAKE, FAKE, FAKE, 1024, 256, 256, 8, 2, 128, FAKE, 2, 0, SC, FAKE, None, None) == 0
    assert lib.resa_store_rows_q8(C.byref(c), FAKE, FAKE, 256, 256, FAKE, 0, FAKE, None) == 0
    assert lib.resa_load_rows_q8(C.byref(c), FAKE, 0, FAKE, FAKE, FAKE, None) == 0
    assert lib.resa_dense_rectify_q8(C.byref(c), FAKE, FAKE, FAKE, a["qs"], 256, 256, 8, FAKE, 0, FAKE, 100, SC, FAKE,
                                     None, None, 0, None) == 0


@pytest.mark.parametrize("kw,code,text", [
    (dict(k=None), 1, "k is NULL"), (dict(v=FAKE + 8), 1, "aligned"), (dict(k_scale=None), 1, "k_scale is NULL"),
    (dict(v_scale=FAKE + 2), 1, "v_scale"), (dict(format=2), 2, "format"), (dict(head_dim=64), 2, "head_dim"),
    (dict(block_size=8), 2, "block_size"), (dict(capacity=1000), 1, "capacity"), (dict(kmin=None), 1, "kmin"),
    (dict(block_table=FAKE, num_pages=0), 1, "num_pages"), (dict(block_table=FAKE, num_pages=1 << 26), 2, "2^31"),
    (dict(batch=0), 1, "batch"),
])
def test_every_call_checks_the_cache(kw, code, text):
    lib, c = L.lib(), cache(**kw)
    expect(lib.resa_store_rows_q8(C.byref(c), FAKE, FAKE, 256, 256, FAKE, 4, FAKE, None), code, text)
    expect(lib.resa_load_rows_q8(C.byref(c), FAKE, 4, FAKE, FAKE, FAKE, None), code, text)
    expect(lib.resa_sparse_decode_q8(C.byref(c), FAKE, 8, FAKE, FAKE, FAKE, 4, 1, SC, FAKE, None, FAKE, 1 << 30, None),
           code, text)
    expect(lib.resa_dense_rectify_q8(C.byref(c), FAKE, FAKE, FAKE, 1024, 256, 256, 8, FAKE, 4, FAKE, 100, SC, FAKE,
                                     None, FAKE, 1 << 30, None), code, text)


def test_store_and_load_refusals():
    lib, c = L.lib(), cache()
    run = lambda k=FAKE, v=FAKE, ks=256, vs=256, cu=FAKE, T=4, lens=FAKE: lib.resa_store_rows_q8(  # noqa: E731
        C.byref(c), k, v, ks, vs, cu, T, lens, None)
    expect(run(k=None), 1, "k_rows is NULL")
    expect(run(v=FAKE + 8), 1, "v_rows")
    expect(run(ks=255), 1, "k_stride")
    expect(run(vs=128), 1, "v_stride")
    expect(run(cu=None), 1, "cu_rows is NULL")
    expect(run(lens=FAKE + 1), 1, "seq_lens")
    expect(run(T=-4), 1, "num_rows")
    expect(lib.resa_load_rows_q8(C.byref(c), FAKE, 4, FAKE, None, FAKE, None), 1, "k_rows is NULL")
    expect(lib.resa_load_rows_q8(C.byref(c), FAKE, 4, FAKE, FAKE, FAKE + 4, None), 1, "v_rows")
    expect(lib.resa_store_rows_q8(None, FAKE, FAKE, 256, 256, FAKE, 4, FAKE, None), 1, "descriptor")


def test_decode_refusals():
    lib, c = L.lib(), cache()
    run = lambda q=FAKE, hq=8, lens=FAKE, idx=FAKE, n=FAKE, cap=4, s=1, sc=SC, out=FAKE, lse=None, ws=FAKE, nb=1 << 30: (  # noqa: E731
        lib.resa_sparse_decode_q8(C.byref(c), q, hq, lens, idx, n, cap, s, sc, out, lse, ws, nb, None))
    expect(run(q=FAKE + 8), 1, "q is not")
    expect(run(hq=9), 1, "multiple")
    expect(run(hq=18), 2, "group")
    expect(run(lens=None), 1, "seq_lens")
    expect(run(idx=None), 1, "block_idx")
    expect(run(n=None), 1, "num_sel")
    expect(run(cap=-1, s=0), 1, "n_cap")
    expect(run(s=257), 1, "num_splits")
    expect(run(s=-1), 1, "num_splits")
    expect(run(sc=float("inf")), 1, "finite")
    expect(run(out=None), 1, "out")
    expect(run(lse=FAKE + 2), 1, "lse")
    expect(run(ws=None), 3, "workspace")
    expect(run(nb=16), 3, "workspace")
    expect(run(ws=FAKE + 8), 1, "workspace")


def test_rectify_refusals():
    lib, c = L.lib(), cache()
    run = lambda q=FAKE, qs=1024, hq=8, T=4, mx=1024, sc=SC, out=FAKE, lse=None, ws=FAKE, nb=1 << 30: (  # noqa: E731
        lib.resa_dense_rectify_q8(C.byref(c), q, FAKE, FAKE, qs, 256, 256, hq, FAKE, T, FAKE, mx, sc, out, lse, ws, nb,
                                  None))
    expect(run(q=None), 1, "q_rows is NULL")
    expect(run(qs=1016), 1, "q_stride")
    expect(run(hq=5), 1, "multiple")
    expect(run(hq=32, qs=4096), 2, "group")
    expect(run(mx=0), 1, "max_seq_len")
    expect(run(mx=1025), 1, "max_seq_len")
    expect(run(sc=float("-inf")), 1, "finite")
    expect(run(out=FAKE + 8), 1, "out")
    expect(run(lse=FAKE + 2), 1, "lse")
    expect(run(ws=None), 3, "workspace")
    expect(run(nb=100), 3, "workspace")
    expect(run(ws=FAKE + 8), 1, "workspace")
    expect(run(T=2 ** 30), 2, "launch")


def test_workspace_sizes():
    """They grow with the length, and are 0 where the arguments are no sizes."""
    lib = L.lib()
    for T in (1, 8, 32, 256, 4096):
        last = 0
        for n in list(range(1, 5000, 37)) + [65535, 65536, 65537, 262144]:
            now = lib.resa_rectify_q8_workspace_size(8, 8, 32, T, n)
            assert now >= last
            last = now
    assert lib.resa_rectify_q8_workspace_size(0, 8, 32, 8, 100) == 0
    assert lib.resa_rectify_q8_workspace_size(8, 8, 4, 8, 100) == 0
    assert lib.resa_decode_q8_workspace_size(8, 8, 32, -1, 16, 0) == 0
    assert lib.resa_decode_q8_workspace_size(8, 8, 32, 100, 16, 0) > 0
    assert lib.resa_decode_q8_workspace_size(8, 8, 32, 100, 16, 8) > lib.resa_decode_q8_workspace_size(8, 8, 32, 100, 16, 1)


def test_binding_refuses_before_the_device():
    """Types and devices, on CPU tensors: no call gets further."""
    x = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    cu = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        R.prompt_attention(x.float(), x, x, cu)
    with pytest.raises(ValueError, match="on the GPU"):
        R.prompt_attention(x, x, x, cu)
    c = R.KVCacheQ8.empty(1, 2, 64, 16, device="cpu")
    with pytest.raises(ValueError, match="on the GPU"):
        R.store_rows_q8(c, x, x, cu, cu[:1])
    with pytest.raises(ValueError, match="on the GPU"):
        c.desc_q8()
    with pytest.raises(TypeError, match="8-bit"):
        c.desc()
    c.k = c.k.view(torch.uint8)
    with pytest.raises(TypeError, match="int8"):
        c.desc_q8()
    assert R.KVCacheQ8.empty_paged(2, 3, 64, 16, 9, torch.float8_e4m3fn, "cpu").capacity == 64
