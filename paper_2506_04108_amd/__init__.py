"""ReSA (Rectified Sparse Attention) decode path for AMD MI355X.

A thin binding over libresa.so: it marshals torch tensors into the C ABI of
include/resa.h (device pointers, sizes, the current HIP stream) and allocates
outputs and workspaces with torch when the caller does not pass them. Every
step of the path runs in the library's HIP kernels.

    cache = KVCache.empty(batch, kv_heads, capacity, block_size, device="cuda")
    block_summarize(cache, seq_lens)
    idx, nsel = select_blocks(cache, q, seq_lens, max_seq_len, sparsity=0.9,
                              min_blocks=128, n_local=1)
    out, lse = sparse_decode(cache, q, seq_lens, idx, nsel)
    dense_rectify(cache, q_f, k_f, v_f, seq_lens, max_seq_len)

Packed prompts and an 8-bit cache (a scale for each block and kv head); rows
of sequence s are rows [cu[s], cu[s + 1]) of the packed tensors, its last ones:

    out, lse = prompt_attention(q, k, v, cu_seqlens)
    cache = KVCacheQ8.empty(batch, kv_heads, capacity, block_size, torch.int8)
    store_rows_q8(cache, k, v, cu_seqlens, seq_lens)        # a prompt, or one token each
    idx, nsel = select_blocks(cache, q, seq_lens, max_seq_len, ...)
    out, lse = sparse_decode_q8(cache, q, seq_lens, idx, nsel)
    out, lse = dense_rectify_q8(cache, q_rows, k_rows, v_rows, cu_rows, seq_lens, max_seq_len)
"""
from __future__ import annotations

import contextlib
import ctypes as C
import dataclasses
import functools
import math

import torch
from torch.autograd import forward_ad

from ._lib import KVCacheDesc, KVCacheQ8Desc, ResaError, SelectParams, check, lib

__all__ = ["KVCache", "Workspace", "ResaError", "num_selected", "block_summarize", "append_kv",
           "select_blocks", "append_select", "sparse_decode", "decode_step", "dense_rectify",
           "decode_num_splits", "version", "KVCacheQ8", "prompt_attention", "store_rows_q8",
           "load_rows_q8", "sparse_decode_q8", "dense_rectify_q8"]

HEAD_DIM = 128
_SCALE = 1.0 / math.sqrt(HEAD_DIM)


def _ptr(t: torch.Tensor | None) -> int | None:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    # The current stream of the current device, without building a Stream
    # object for it (0.2 against 1.3 us).
    return _raw_stream(_current_device())


def _current_raw_stream(device: int) -> int:
    return torch.cuda.current_stream(device).cuda_stream


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _current_raw_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _on_its_stream(call):
    """A call given a stream makes its new tensors there too: a workspace is
    cleared in order with the kernels, and no memory goes back to another
    stream while they run."""
    @functools.wraps(call)
    def wrapper(*args, stream=None, **kw):
        if stream is None:
            return call(*args, **kw)
        with torch.cuda.stream(stream):
            return call(*args, **kw)
    return wrapper


def _need(t: torch.Tensor, name: str, dtype, shape=None):
    # One expression for the usual case; which check failed is found out only
    # where one did.
    try:
        if t.dtype is dtype and t.is_cuda and t.is_contiguous() and (shape is None or t.shape == shape) \
                and isinstance(t, torch.Tensor):
            return t
    except AttributeError:
        pass
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return t


def version() -> str:
    return lib().resa_version().decode()


@dataclasses.dataclass
class KVCache:
    """A layer's KV cache and block-key cache (caller-owned device tensors).

    Contiguous layout: k, v are ``[B, Hkv, capacity, 128]``. Paged layout
    (``block_table`` given): k, v are page pools ``[num_pages, Hkv,
    block_size, 128]`` and ``block_table`` (int32 ``[B, capacity /
    block_size]``) names the page of each logical block of each sequence.
    Summaries are per sequence in both layouts."""

    k: torch.Tensor      # bf16 [B, Hkv, capacity, 128] or [num_pages, Hkv, b, 128]
    v: torch.Tensor
    kmin: torch.Tensor   # bf16 [B, Hkv, capacity / block_size, 128]
    kmax: torch.Tensor
    block_size: int
    block_table: torch.Tensor | None = None  # int32 [B, capacity / block_size]

    @classmethod
    def empty(cls, batch, kv_heads, capacity, block_size, device="cuda"):
        shape = (batch, kv_heads, capacity, HEAD_DIM)
        mb = capacity // block_size
        mk = dict(dtype=torch.bfloat16, device=device)
        return cls(torch.zeros(shape, **mk), torch.zeros(shape, **mk),
                   torch.zeros((batch, kv_heads, mb, HEAD_DIM), **mk),
                   torch.zeros((batch, kv_heads, mb, HEAD_DIM), **mk), block_size)

    @classmethod
    def empty_paged(cls, batch, kv_heads, capacity, block_size, num_pages, device="cuda"):
        """Zeroed page pools of ``num_pages`` pages and an identity-free table
        (all entries -1: the caller assigns pages)."""
        mk = dict(dtype=torch.bfloat16, device=device)
        pool = (num_pages, kv_heads, block_size, HEAD_DIM)
        mb = capacity // block_size
        return cls(torch.zeros(pool, **mk), torch.zeros(pool, **mk),
                   torch.zeros((batch, kv_heads, mb, HEAD_DIM), **mk),
                   torch.zeros((batch, kv_heads, mb, HEAD_DIM), **mk), block_size,
                   torch.full((batch, mb), -1, dtype=torch.int32, device=device))

    @property
    def paged(self) -> bool:
        return self.block_table is not None

    @property
    def batch(self):
        return self.kmin.shape[0]

    @property
    def kv_heads(self):
        return self.k.shape[1]

    @property
    def capacity(self):
        return self.kmin.shape[2] * self.block_size

    def desc(self) -> KVCacheDesc:
        k, v, kmin, kmax, b, table = self.k, self.v, self.kmin, self.kmax, self.block_size, self.block_table
        bf16 = torch.bfloat16
        try:  # the usual case in one expression
            fine = (k.dtype is bf16 and v.dtype is bf16 and kmin.dtype is bf16 and kmax.dtype is bf16 and k.is_cuda
                    and v.is_cuda and kmin.is_cuda and kmax.is_cuda and k.is_contiguous() and v.is_contiguous()
                    and kmin.is_contiguous() and kmax.is_contiguous())
        except AttributeError:
            fine = False
        if not fine:
            for name in ("k", "v", "kmin", "kmax"):
                _need(getattr(self, name), name, bf16)
        B, H, mb = kmin.shape[:3]
        if table is None:
            shape, pages, tp = (B, H, mb * b, HEAD_DIM), 0, None
        else:
            pages = k.shape[0]
            shape = (pages, H, b, HEAD_DIM)
        if k.shape != shape or v.shape != shape:
            _need(k, "k", bf16, shape)
            _need(v, "v", bf16, shape)
        if table is not None:
            tp = _need(table, "block_table", torch.int32, (B, mb)).data_ptr()
        return KVCacheDesc(k.data_ptr(), v.data_ptr(), kmin.data_ptr(), kmax.data_ptr(), B, H, HEAD_DIM, mb * b,
                           b, tp, pages)


class Workspace:
    """A zero-initialised device scratch buffer that grows on demand.

    Use one per operation kind. The decode kernel keeps one merge counter per
    group at the start of its workspace and leaves it at zero after every
    call (and a count of merged calls that tags its ready flags), so the
    buffer is cleared only when it is (re)allocated, or when a call of another
    operation, batch or head count takes it over: where what is kept lies
    follows from these. A buffer that a call recorded in a graph uses is neither
    taken over nor freed; ``buf`` is the one used last. Calls that share a
    workspace must be ordered on one stream.
    """

    def __init__(self, device="cuda"):
        self.device = device
        self.buf = None
        self._layout = None  # what buf is used as: (operation, batch, kv heads)
        self._recorded = []  # buffers that recorded calls use
        self._others = {}    # those of them that are used as something else than buf
        self._spare = None   # a buffer that is not, while buf is one of them

    def _is_recorded(self) -> bool:
        return any(b is self.buf for b in self._recorded)

    def _capturing(self) -> bool:
        return self.buf.is_cuda and torch.cuda.is_current_stream_capturing()

    def turn_to(self, layout: tuple) -> torch.Tensor | None:
        """A buffer for calls of that layout, if there is one."""
        if layout != self._layout:
            unused = self._layout is None
            if not unused and self.buf is not None and self._is_recorded():
                self._others[self._layout], self.buf, self._spare = self.buf, self._spare, None
            self._layout = layout
            if layout in self._others:
                self._spare, self.buf = self.buf, self._others.pop(layout)
            elif not unused and self.buf is not None:
                if self._capturing():  # a graph is not to clear it each time
                    self.buf = None
                else:
                    self.buf.zero_()
        return self.buf

    def record(self) -> None:
        """Keeps the buffer at hand where the call that uses it is being recorded."""
        if self._capturing() and not self._is_recorded():
            self._recorded.append(self.buf)

    def get(self, nbytes: int, layout: tuple | None = None) -> torch.Tensor:
        if layout is not None:
            self.turn_to(layout)
        if self.buf is None or self.buf.numel() < nbytes:
            self.buf = torch.zeros(max(nbytes, 256), dtype=torch.uint8, device=self.device)
        self.record()
        return self.buf


def num_selected(num_blocks: int, sparsity: float, min_blocks: int, n_local: int) -> int:
    """Eq. 5 block count (host arithmetic of the library)."""
    n = lib().resa_num_selected(num_blocks, sparsity, min_blocks, n_local)
    if n < 0:
        raise ResaError(1, lib().resa_last_error().decode())
    return n


def decode_num_splits(batch, kv_heads, n_cap, block_size) -> int:
    return lib().resa_decode_num_splits(batch, kv_heads, n_cap, block_size)


def block_summarize(cache: KVCache, seq_lens: torch.Tensor, blk_begin: int = 0, blk_end: int = -1,
                    stream=None) -> None:
    """Eq. 3 summaries of blocks [blk_begin, blk_end) of every sequence."""
    _need(seq_lens, "seq_lens", torch.int32, (cache.batch,))
    d = cache.desc()
    check(lib().resa_block_summarize(C.byref(d), seq_lens.data_ptr(), blk_begin, blk_end,
                                     _stream(stream)))


def append_kv(cache: KVCache, k_new: torch.Tensor, v_new: torch.Tensor, seq_lens: torch.Tensor,
              max_seq_len: int, stream=None) -> None:
    """Alg. 1 append of one token per sequence; seq_lens is incremented in place."""
    shape = (cache.batch, cache.kv_heads, HEAD_DIM)
    _need(k_new, "k_new", torch.bfloat16, shape)
    _need(v_new, "v_new", torch.bfloat16, shape)
    _need(seq_lens, "seq_lens", torch.int32, (cache.batch,))
    d = cache.desc()
    check(lib().resa_append_kv(C.byref(d), k_new.data_ptr(), v_new.data_ptr(), seq_lens.data_ptr(),
                               max_seq_len, _stream(stream)))


@_on_its_stream
def select_blocks(cache: KVCache, q: torch.Tensor, seq_lens: torch.Tensor, max_seq_len: int,
                  sparsity: float, min_blocks: int, n_local: int = 1, n_cap: int | None = None,
                  block_idx: torch.Tensor | None = None, num_sel: torch.Tensor | None = None,
                  scores_out: torch.Tensor | None = None, workspace: Workspace | None = None,
                  stream=None):
    """Pooled-query Quest scores (Eq. 4) and the Eq. 5 top-n per group.

    Returns ``(block_idx [B, Hkv, n_cap] int32 ascending, -1 padded,
    num_sel [B, Hkv] int32)``. Reads only the summaries: ``cache`` may be a
    :class:`KVCacheQ8` too.
    """
    B, Hkv = cache.kmin.shape[0], cache.k.shape[1]
    hq = q.shape[1]
    _need(q, "q", torch.bfloat16, (B, hq, HEAD_DIM))
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    mseq = -(-max_seq_len // cache.block_size)
    if n_cap is None:
        n_cap = max(num_selected(mseq, sparsity, min_blocks, n_local), 1)
    if block_idx is None:
        block_idx = torch.empty((B, Hkv, n_cap), dtype=torch.int32, device=q.device)
    if num_sel is None:
        num_sel = torch.empty((B, Hkv), dtype=torch.int32, device=q.device)
    _need(block_idx, "block_idx", torch.int32, (B, Hkv, n_cap))
    _need(num_sel, "num_sel", torch.int32, (B, Hkv))
    if scores_out is not None:
        _need(scores_out, "scores_out", torch.float32, (B, Hkv, mseq))
    ws_bytes = lib().resa_select_workspace_size(B, Hkv, max_seq_len, cache.block_size)
    ws = (workspace or Workspace(q.device)).get(ws_bytes, ("select", B, Hkv))
    ws_ptr, ws_bytes = ws.data_ptr(), ws.numel()
    params = SelectParams(float(sparsity), int(min_blocks), int(n_local))
    d = cache.desc_q8().base if isinstance(cache, KVCacheQ8) else cache.desc()
    check(lib().resa_select_blocks(C.byref(d), q.data_ptr(), hq, seq_lens.data_ptr(), max_seq_len,
                                   C.byref(params), block_idx.data_ptr(), num_sel.data_ptr(), n_cap,
                                   _ptr(scores_out), ws_ptr, ws_bytes, _stream(stream)))
    return block_idx, num_sel


@_on_its_stream
def append_select(cache: KVCache, k_new: torch.Tensor, v_new: torch.Tensor, q: torch.Tensor,
                  seq_lens: torch.Tensor, max_seq_len: int, sparsity: float, min_blocks: int,
                  n_local: int = 1, n_cap: int | None = None, block_idx: torch.Tensor | None = None,
                  num_sel: torch.Tensor | None = None, scores_out: torch.Tensor | None = None,
                  workspace: Workspace | None = None, stream=None):
    """Alg. 1 append of one token per sequence fused with the Eq. 4-5
    selection over the grown sequences (one launch); seq_lens is incremented
    in place. ``max_seq_len`` bounds seq_lens before the call. Returns
    ``(block_idx, num_sel)`` as :func:`select_blocks`."""
    B, Hkv = cache.kmin.shape[0], cache.k.shape[1]
    hq = q.shape[1]
    shape = (B, Hkv, HEAD_DIM)
    _need(k_new, "k_new", torch.bfloat16, shape)
    _need(v_new, "v_new", torch.bfloat16, shape)
    _need(q, "q", torch.bfloat16, (B, hq, HEAD_DIM))
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    sel_len = max_seq_len + 1
    mseq = -(-sel_len // cache.block_size)
    if n_cap is None:
        n_cap = max(num_selected(mseq, sparsity, min_blocks, n_local), 1)
    if block_idx is None:
        block_idx = torch.empty((B, Hkv, n_cap), dtype=torch.int32, device=q.device)
    if num_sel is None:
        num_sel = torch.empty((B, Hkv), dtype=torch.int32, device=q.device)
    _need(block_idx, "block_idx", torch.int32, (B, Hkv, n_cap))
    _need(num_sel, "num_sel", torch.int32, (B, Hkv))
    if scores_out is not None:
        _need(scores_out, "scores_out", torch.float32, (B, Hkv, mseq))
    ws_bytes = lib().resa_select_workspace_size(B, Hkv, sel_len, cache.block_size)
    ws = (workspace or Workspace(q.device)).get(ws_bytes, ("select", B, Hkv))
    params = SelectParams(float(sparsity), int(min_blocks), int(n_local))
    d = cache.desc()
    check(lib().resa_append_select(C.byref(d), k_new.data_ptr(), v_new.data_ptr(), q.data_ptr(), hq,
                                   seq_lens.data_ptr(), max_seq_len, C.byref(params),
                                   block_idx.data_ptr(), num_sel.data_ptr(), n_cap, _ptr(scores_out),
                                   ws.data_ptr(), ws.numel(), _stream(stream)))
    return block_idx, num_sel


@_on_its_stream
def sparse_decode(cache: KVCache, q: torch.Tensor, seq_lens: torch.Tensor, block_idx: torch.Tensor,
                  num_sel: torch.Tensor, num_splits: int = 0, sm_scale: float | None = None,
                  out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                  with_lse: bool = True, workspace: Workspace | None = None, stream=None):
    """Eq. 2 / Alg. 2 block-sparse flash decoding. Returns ``(out fp32 [B, Hq, 128],
    lse fp32 [B, Hq] or None)``."""
    B, Hkv = cache.kmin.shape[0], cache.k.shape[1]
    hq = q.shape[1]
    _need(q, "q", torch.bfloat16, (B, hq, HEAD_DIM))
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    n_cap = block_idx.shape[-1]
    _need(block_idx, "block_idx", torch.int32, (B, Hkv, n_cap))
    _need(num_sel, "num_sel", torch.int32, (B, Hkv))
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(HEAD_DIM)
    if out is None:
        out = torch.empty((B, hq, HEAD_DIM), dtype=torch.float32, device=q.device)
    _need(out, "out", torch.float32, (B, hq, HEAD_DIM))
    if lse is None and with_lse:
        lse = torch.empty((B, hq), dtype=torch.float32, device=q.device)
    if lse is not None:
        _need(lse, "lse", torch.float32, (B, hq))
    ws_bytes = lib().resa_decode_workspace_size(B, Hkv, hq, n_cap, cache.block_size, num_splits)
    ws = (workspace or Workspace(q.device)).get(ws_bytes, ("decode", B, Hkv))
    d = cache.desc()
    check(lib().resa_sparse_decode(C.byref(d), q.data_ptr(), hq, seq_lens.data_ptr(),
                                   block_idx.data_ptr(), num_sel.data_ptr(), n_cap, num_splits,
                                   float(sm_scale), out.data_ptr(), _ptr(lse), ws.data_ptr(),
                                   ws.numel(), _stream(stream)))
    return out, lse


@_on_its_stream
def decode_step(cache: KVCache, k_new: torch.Tensor, v_new: torch.Tensor, q: torch.Tensor,
                seq_lens: torch.Tensor, max_seq_len: int, sparsity: float, min_blocks: int,
                n_local: int = 1, n_cap: int | None = None, num_splits: int = 0,
                sm_scale: float | None = None, block_idx: torch.Tensor | None = None,
                num_sel: torch.Tensor | None = None, out: torch.Tensor | None = None,
                lse: torch.Tensor | None = None, with_lse: bool = True,
                workspace: Workspace | None = None, stream=None):
    """One decode token (Alg. 1) in one call: append (seq_lens incremented
    in place), Eq. 4-5 selection and Eq. 2 / Alg. 2 sparse decoding.
    ``max_seq_len`` bounds seq_lens before the call. Returns
    ``(block_idx, num_sel, out, lse)`` as :func:`append_select` and
    :func:`sparse_decode`."""
    B, Hkv = cache.kmin.shape[0], cache.k.shape[1]
    hq = q.shape[1]
    shape = (B, Hkv, HEAD_DIM)
    _need(k_new, "k_new", torch.bfloat16, shape)
    _need(v_new, "v_new", torch.bfloat16, shape)
    _need(q, "q", torch.bfloat16, (B, hq, HEAD_DIM))
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    mseq = -(-(max_seq_len + 1) // cache.block_size)
    if n_cap is None:
        n_cap = max(num_selected(mseq, sparsity, min_blocks, n_local), 1)
    if block_idx is None:
        block_idx = torch.empty((B, Hkv, n_cap), dtype=torch.int32, device=q.device)
    if num_sel is None:
        num_sel = torch.empty((B, Hkv), dtype=torch.int32, device=q.device)
    _need(block_idx, "block_idx", torch.int32, (B, Hkv, n_cap))
    _need(num_sel, "num_sel", torch.int32, (B, Hkv))
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(HEAD_DIM)
    if out is None:
        out = torch.empty((B, hq, HEAD_DIM), dtype=torch.float32, device=q.device)
    _need(out, "out", torch.float32, (B, hq, HEAD_DIM))
    if lse is None and with_lse:
        lse = torch.empty((B, hq), dtype=torch.float32, device=q.device)
    if lse is not None:
        _need(lse, "lse", torch.float32, (B, hq))
    ws_bytes = lib().resa_step_workspace_size(B, Hkv, hq, max_seq_len, cache.block_size, n_cap,
                                              num_splits)
    ws = (workspace or Workspace(q.device)).get(ws_bytes, ("step", B, Hkv))
    params = SelectParams(float(sparsity), int(min_blocks), int(n_local))
    d = cache.desc()
    check(lib().resa_decode_step(C.byref(d), k_new.data_ptr(), v_new.data_ptr(), q.data_ptr(), hq,
                                 seq_lens.data_ptr(), max_seq_len, C.byref(params),
                                 block_idx.data_ptr(), num_sel.data_ptr(), n_cap, num_splits,
                                 float(sm_scale), out.data_ptr(), _ptr(lse), ws.data_ptr(), ws.numel(),
                                 _stream(stream)))
    return block_idx, num_sel, out, lse


@_on_its_stream
def dense_rectify(cache: KVCache, q_f: torch.Tensor, k_f: torch.Tensor, v_f: torch.Tensor,
                  seq_lens: torch.Tensor, max_seq_len: int, sm_scale: float | None = None,
                  out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                  with_lse: bool = True, refresh: bool = True, workspace: Workspace | None = None,
                  seq_mask: torch.Tensor | None = None, stream=None):
    """Sec. 2.2 rectification of the last f rows. Returns ``(out fp32 [B, Hq, f, 128], lse)``.
    ``seq_mask`` (int32 [B] on the device, or None for every sequence) selects the
    sequences rectified by this call; the others are left untouched."""
    B, Hkv = cache.kmin.shape[0], cache.k.shape[1]
    hq, f = q_f.shape[1], q_f.shape[2]
    _need(q_f, "q_f", torch.bfloat16, (B, hq, f, HEAD_DIM))
    _need(k_f, "k_f", torch.bfloat16, (B, Hkv, f, HEAD_DIM))
    _need(v_f, "v_f", torch.bfloat16, (B, Hkv, f, HEAD_DIM))
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    if seq_mask is not None:
        _need(seq_mask, "seq_mask", torch.int32, (B,))
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(HEAD_DIM)
    if out is None:
        out = torch.empty((B, hq, f, HEAD_DIM), dtype=torch.float32, device=q_f.device)
    _need(out, "out", torch.float32, (B, hq, f, HEAD_DIM))
    if lse is None and with_lse:
        lse = torch.empty((B, hq, f), dtype=torch.float32, device=q_f.device)
    if lse is not None:
        _need(lse, "lse", torch.float32, (B, hq, f))
    ws_bytes = lib().resa_rectify_workspace_size(B, Hkv, hq, f, max_seq_len)
    ws = (workspace or Workspace(q_f.device)).get(ws_bytes, ("rectify",))
    d = cache.desc()
    check(lib().resa_dense_rectify(C.byref(d), q_f.data_ptr(), k_f.data_ptr(), v_f.data_ptr(), hq, f,
                                   seq_lens.data_ptr(), _ptr(seq_mask), max_seq_len, float(sm_scale),
                                   out.data_ptr(), _ptr(lse), int(bool(refresh)), ws.data_ptr(),
                                   ws.numel(), _stream(stream)))
    return out, lse

# ------------------------------------------------- packed rows, 8-bit cache

_Q8_FORMATS = {torch.int8: 0, torch.float8_e4m3fn: 1}


@dataclasses.dataclass
class KVCacheQ8:
    """A layer's KV cache in 8 bits (caller-owned device tensors): a value is
    its code times the scale of its (block, kv head).

    ``k``, ``v`` hold codes (``torch.int8`` or ``torch.float8_e4m3fn``) in the
    layouts of :class:`KVCache`, contiguous or paged; ``k_scale``, ``v_scale``
    are fp32 ``[B, Hkv, capacity / block_size]``, with a block table
    ``[num_pages, Hkv]``; the summaries are a :class:`KVCache`'s."""

    k: torch.Tensor        # int8 / e4m3 [B, Hkv, capacity, 128] or [num_pages, Hkv, b, 128]
    v: torch.Tensor
    k_scale: torch.Tensor  # fp32 [B, Hkv, capacity / block_size] or [num_pages, Hkv]
    v_scale: torch.Tensor
    kmin: torch.Tensor     # bf16 [B, Hkv, capacity / block_size, 128]
    kmax: torch.Tensor
    block_size: int
    block_table: torch.Tensor | None = None  # int32 [B, capacity / block_size]

    @classmethod
    def empty(cls, batch, kv_heads, capacity, block_size, dtype=torch.int8, device="cuda"):
        mb = capacity // block_size
        codes = [torch.zeros((batch, kv_heads, capacity, HEAD_DIM), dtype=torch.int8, device=device).view(dtype)
                 for _ in "kv"]
        scales = [torch.zeros((batch, kv_heads, mb), dtype=torch.float32, device=device) for _ in "kv"]
        sums = [torch.zeros((batch, kv_heads, mb, HEAD_DIM), dtype=torch.bfloat16, device=device) for _ in "kv"]
        return cls(*codes, *scales, *sums, block_size)

    @classmethod
    def empty_paged(cls, batch, kv_heads, capacity, block_size, num_pages, dtype=torch.int8, device="cuda"):
        """Zeroed pools of ``num_pages`` pages and a table of -1 (the caller
        assigns pages)."""
        mb = capacity // block_size
        codes = [torch.zeros((num_pages, kv_heads, block_size, HEAD_DIM), dtype=torch.int8,
                             device=device).view(dtype) for _ in "kv"]
        scales = [torch.zeros((num_pages, kv_heads), dtype=torch.float32, device=device) for _ in "kv"]
        sums = [torch.zeros((batch, kv_heads, mb, HEAD_DIM), dtype=torch.bfloat16, device=device) for _ in "kv"]
        return cls(*codes, *scales, *sums, block_size,
                   torch.full((batch, mb), -1, dtype=torch.int32, device=device))

    @property
    def paged(self) -> bool:
        return self.block_table is not None

    @property
    def batch(self):
        return self.kmin.shape[0]

    @property
    def kv_heads(self):
        return self.k.shape[1]

    @property
    def capacity(self):
        return self.kmin.shape[2] * self.block_size

    def desc(self):
        raise TypeError("an 8-bit cache: use the calls that end in _q8 (and select_blocks)")

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        object.__setattr__(self, "_checked", None)

    def __getstate__(self):
        # A copy is checked by itself (and a description holds addresses).
        return {**self.__dict__, "_checked": None}

    def desc_q8(self) -> KVCacheQ8Desc:
        """The library's description of this cache."""
        return self._described()[1]

    def _described(self):
        """(what was checked, the cache's description, a reference to that, batch,
        kv heads). The tensors are checked once, and again after one was replaced
        or has another address, shape, type or order (checking them takes 8 us,
        seeing that nothing has changed 1.5)."""
        k, v, ks, vs, lo, hi, table = (self.k, self.v, self.k_scale, self.v_scale, self.kmin, self.kmax,
                                       self.block_table)
        seen = (k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), lo.data_ptr(), hi.data_ptr(), k.shape,
                v.shape, ks.shape, vs.shape, lo.shape, hi.shape, k.dtype, v.dtype, ks.dtype, vs.dtype, lo.dtype,
                hi.dtype, None if table is None else (table.data_ptr(), table.shape, table.dtype))
        checked = self._checked
        if checked is not None and checked[0] == seen and k.is_contiguous() and v.is_contiguous() \
                and ks.is_contiguous() and vs.is_contiguous() and lo.is_contiguous() and hi.is_contiguous() \
                and (table is None or table.is_contiguous()):
            return checked
        b = self.block_size
        fmt = _Q8_FORMATS.get(k.dtype)
        if fmt is None:
            raise TypeError(f"k must be torch.int8 or torch.float8_e4m3fn, got {k.dtype}")
        B, H, mb = lo.shape[:3]
        if table is None:
            shape, pages, tp, scales = (B, H, mb * b, HEAD_DIM), 0, None, (B, H, mb)
        else:
            pages = k.shape[0]
            shape, scales = (pages, H, b, HEAD_DIM), (pages, H)
            tp = _need(table, "block_table", torch.int32, (B, mb)).data_ptr()
        _need(k, "k", k.dtype, shape)
        _need(v, "v", k.dtype, shape)
        _need(ks, "k_scale", torch.float32, scales)
        _need(vs, "v_scale", torch.float32, scales)
        _need(lo, "kmin", torch.bfloat16, (B, H, mb, HEAD_DIM))
        _need(hi, "kmax", torch.bfloat16, (B, H, mb, HEAD_DIM))
        _one_device(k, v, ks, vs, lo, hi, table)
        d = KVCacheQ8Desc(KVCacheDesc(seen[0], seen[1], seen[4], seen[5], B, H, HEAD_DIM, mb * b, b, tp, pages),
                          seen[2], seen[3], fmt)
        checked = (seen, d, C.byref(d), B, H)
        object.__setattr__(self, "_checked", checked)
        return checked


def _no_gradient(t: torch.Tensor, name: str) -> None:
    """Refuses what a call would silently drop: a gradient asked for, or a tangent."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient: there is no backward pass")
    if forward_ad._current_level >= 0 and forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError(f"{name} has a tangent: there is no forward-mode derivative")


def _packed(t: torch.Tensor, name: str, rows: int, heads: int) -> int:
    """Checks packed rows ``[rows, heads, 128]`` (bf16, a row contiguous) and
    returns the elements from one row to the next."""
    try:  # the usual case in one expression
        row, head, dim = t.stride()
        if t.dtype is torch.bfloat16 and t.is_cuda and t.shape == (rows, heads, HEAD_DIM) and dim == 1 \
                and head == HEAD_DIM and not t.requires_grad and forward_ad._current_level < 0:
            return row if rows > 1 else heads * HEAD_DIM
    except (AttributeError, TypeError, ValueError):
        pass
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype is not torch.bfloat16:
        raise TypeError(f"{name} must be {torch.bfloat16}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    if t.shape != (rows, heads, HEAD_DIM):
        raise ValueError(f"{name} must have shape {(rows, heads, HEAD_DIM)}, got {tuple(t.shape)}")
    _no_gradient(t, name)
    row, head, dim = t.stride()
    if rows and (dim != 1 or (heads > 1 and head != HEAD_DIM)):
        raise ValueError(f"{name} must be contiguous within a row")
    return row if rows > 1 else heads * HEAD_DIM


_devices = None


def _one_device(first: torch.Tensor, *others) -> None:
    """Every tensor of a call lies on the current device, whose stream it runs on."""
    global _devices
    if _devices is None:
        _devices = torch.cuda.device_count()
    if _devices == 1:  # what is on a GPU is on this one
        return
    index = first.get_device()
    if index != _current_device():
        raise ValueError(f"tensors are on device {index}, the current device is {_current_device()}")
    for t in others:
        if t is not None and t.get_device() != index:
            raise ValueError(f"tensors are on devices {index} and {t.get_device()}")


def _new(stream, like: torch.Tensor, *wanted):
    """New tensors ((shape, dtype), ...) on like's device that belong to the
    stream a call runs on."""
    with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):
        return [like.new_empty(shape, dtype=dtype, requires_grad=False) for shape, dtype in wanted]


def _with_workspace(call, needs, workspace, layout, device):
    """call(pointer, bytes) on the workspace's buffer of that layout as it is; where
    the library finds it too small (before it enqueues anything), on one of
    needs() bytes."""
    ws = workspace.turn_to(layout) if workspace is not None else None
    if ws is not None:
        rc = call(ws.data_ptr(), ws.numel())
        if rc != _ERR_WORKSPACE:
            workspace.record()
            return check(rc)
    ws = (workspace or Workspace(device)).get(needs(), layout)
    check(call(ws.data_ptr(), ws.numel()))


_ERR_WORKSPACE = 3


def prompt_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_seqlens: torch.Tensor,
                     sm_scale: float | None = None, out: torch.Tensor | None = None,
                     lse: torch.Tensor | None = None, with_lse: bool = True, stream=None):
    """Causal attention of packed prompts: sequence s has rows ``[cu_seqlens[s],
    cu_seqlens[s + 1])`` (int32, on the device) of q ``[T, Hq, 128]`` and k, v
    ``[T, Hkv, 128]`` (bf16; from row to row any stride that is a multiple of
    8, so that they may be parts of one projection's output). Returns ``(out
    bf16 [T, Hq, 128], lse fp32 [T, Hq] or None)``; rows of no sequence are
    not written."""
    T, hq, hkv = q.shape[0], q.shape[1], k.shape[1]
    qs, ks, vs = _packed(q, "q", T, hq), _packed(k, "k", T, hkv), _packed(v, "v", T, hkv)
    B = cu_seqlens.shape[0] - 1
    _need(cu_seqlens, "cu_seqlens", torch.int32, (B + 1,))
    if sm_scale is None:
        sm_scale = _SCALE
    if out is None:
        out, = _new(stream, q, ((T, hq, HEAD_DIM), torch.bfloat16))
    if lse is None and with_lse:
        lse, = _new(stream, q, ((T, hq), torch.float32))
    _need(out, "out", torch.bfloat16, (T, hq, HEAD_DIM))
    if lse is not None:
        _need(lse, "lse", torch.float32, (T, hq))
    _one_device(q, k, v, cu_seqlens, out, lse)
    if T:  # an empty tensor has no address
        check(lib().resa_prompt_attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), qs, ks, vs, hq, hkv, HEAD_DIM,
                                          cu_seqlens.data_ptr(), B, T, float(sm_scale), out.data_ptr(), _ptr(lse),
                                          _stream(stream)))
    return out, lse


def store_rows_q8(cache: KVCacheQ8, k_rows: torch.Tensor, v_rows: torch.Tensor, cu_rows: torch.Tensor,
                  seq_lens: torch.Tensor, stream=None) -> None:
    """The last rows of each sequence into an 8-bit cache (a prompt, a chunk,
    one decoded token), with the summaries of the blocks they touch. Rows
    ``[cu_rows[s], cu_rows[s + 1])`` of k_rows, v_rows ``[T, Hkv, 128]`` (bf16)
    become the last positions of sequence s, whose ``seq_lens`` already counts
    them."""
    _, _, ref, B, H = cache._described()
    T = k_rows.shape[0]
    ks, vs = _packed(k_rows, "k_rows", T, H), _packed(v_rows, "v_rows", T, H)
    _need(cu_rows, "cu_rows", torch.int32, (B + 1,))
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    _one_device(cache.k, k_rows, v_rows, cu_rows, seq_lens)
    if T:
        check(lib().resa_store_rows_q8(ref, k_rows.data_ptr(), v_rows.data_ptr(), ks, vs, cu_rows.data_ptr(),
                                       T, seq_lens.data_ptr(), _stream(stream)))


def load_rows_q8(cache: KVCacheQ8, cu_rows: torch.Tensor, seq_lens: torch.Tensor, num_rows: int | None = None,
                 out: tuple | None = None, stream=None):
    """The last rows of each sequence as bf16, ``(k_rows, v_rows)`` of ``[T,
    Hkv, 128]``: ``out``, or new tensors of ``num_rows`` rows."""
    _, _, ref, B, H = cache._described()
    if out is None:
        if num_rows is None:
            raise ValueError("either num_rows or out must be given")
        out = tuple(_new(stream, cache.k, *[((num_rows, H, HEAD_DIM), torch.bfloat16)] * 2))
    k_rows, v_rows = out
    T = k_rows.shape[0]
    _need(k_rows, "k_rows", torch.bfloat16, (T, H, HEAD_DIM))
    _need(v_rows, "v_rows", torch.bfloat16, (T, H, HEAD_DIM))
    _need(cu_rows, "cu_rows", torch.int32, (B + 1,))
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    _one_device(cache.k, k_rows, v_rows, cu_rows, seq_lens)
    if T:
        check(lib().resa_load_rows_q8(ref, cu_rows.data_ptr(), T, seq_lens.data_ptr(), k_rows.data_ptr(),
                                      v_rows.data_ptr(), _stream(stream)))
    return k_rows, v_rows


@_on_its_stream
def sparse_decode_q8(cache: KVCacheQ8, q: torch.Tensor, seq_lens: torch.Tensor, block_idx: torch.Tensor,
                     num_sel: torch.Tensor, num_splits: int = 0, sm_scale: float | None = None,
                     out: torch.Tensor | None = None, lse: torch.Tensor | None = None, with_lse: bool = True,
                     workspace: Workspace | None = None, stream=None):
    """:func:`sparse_decode` over an 8-bit cache. Returns ``(out fp32 [B, Hq,
    128], lse fp32 [B, Hq] or None)``."""
    _, _, ref, B, H = cache._described()
    hq, n_cap = q.shape[1], block_idx.shape[-1]
    _need(q, "q", torch.bfloat16, (B, hq, HEAD_DIM))
    _no_gradient(q, "q")
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    _need(block_idx, "block_idx", torch.int32, (B, H, n_cap))
    _need(num_sel, "num_sel", torch.int32, (B, H))
    if out is None:
        out, = _new(stream, q, ((B, hq, HEAD_DIM), torch.float32))
    if lse is None and with_lse:
        lse, = _new(stream, q, ((B, hq), torch.float32))
    _need(out, "out", torch.float32, (B, hq, HEAD_DIM))
    if lse is not None:
        _need(lse, "lse", torch.float32, (B, hq))
    _one_device(cache.k, q, seq_lens, block_idx, num_sel, out, lse)
    scale = _SCALE if sm_scale is None else float(sm_scale)
    ptrs = (ref, q.data_ptr(), hq, seq_lens.data_ptr(), block_idx.data_ptr(), num_sel.data_ptr(), n_cap,
            num_splits, scale, out.data_ptr(), _ptr(lse))
    run, st = lib().resa_sparse_decode_q8, _stream(stream)
    _with_workspace(lambda ws, size: run(*ptrs, ws, size, st),
                    lambda: lib().resa_decode_q8_workspace_size(B, H, hq, n_cap, cache.block_size, num_splits),
                    workspace, ("decode", B, H), q.device)
    return out, lse


@_on_its_stream
def dense_rectify_q8(cache: KVCacheQ8, q_rows: torch.Tensor, k_rows: torch.Tensor, v_rows: torch.Tensor,
                     cu_rows: torch.Tensor, seq_lens: torch.Tensor, max_seq_len: int,
                     sm_scale: float | None = None, out: torch.Tensor | None = None,
                     lse: torch.Tensor | None = None, with_lse: bool = True,
                     workspace: Workspace | None = None, stream=None):
    """Rectification (Sec. 2.2) or a prompt chunk over an 8-bit cache:
    :func:`store_rows_q8` of the packed k_rows, v_rows, then dense causal
    attention of q_rows ``[T, Hq, 128]`` (bf16) over the whole cache.
    ``max_seq_len`` bounds seq_lens. Returns ``(out bf16 [T, Hq, 128], lse fp32
    [T, Hq] or None)``; rows of sequences without rows in the call are not
    written."""
    _, _, ref, B, H = cache._described()
    T, hq = q_rows.shape[0], q_rows.shape[1]
    qs = _packed(q_rows, "q_rows", T, hq)
    ks, vs = _packed(k_rows, "k_rows", T, H), _packed(v_rows, "v_rows", T, H)
    _need(cu_rows, "cu_rows", torch.int32, (B + 1,))
    _need(seq_lens, "seq_lens", torch.int32, (B,))
    if out is None:
        out, = _new(stream, q_rows, ((T, hq, HEAD_DIM), torch.bfloat16))
    if lse is None and with_lse:
        lse, = _new(stream, q_rows, ((T, hq), torch.float32))
    _need(out, "out", torch.bfloat16, (T, hq, HEAD_DIM))
    if lse is not None:
        _need(lse, "lse", torch.float32, (T, hq))
    _one_device(cache.k, q_rows, k_rows, v_rows, cu_rows, seq_lens, out, lse)
    if T:
        scale = _SCALE if sm_scale is None else float(sm_scale)
        ptrs = (ref, q_rows.data_ptr(), k_rows.data_ptr(), v_rows.data_ptr(), qs, ks, vs, hq,
                cu_rows.data_ptr(), T, seq_lens.data_ptr(), max_seq_len, scale, out.data_ptr(), _ptr(lse))
        run, st = lib().resa_dense_rectify_q8, _stream(stream)
        _with_workspace(lambda ws, size: run(*ptrs, ws, size, st),
                        lambda: lib().resa_rectify_q8_workspace_size(B, H, hq, T, max_seq_len),
                        workspace, ("rectify",), q_rows.device)
    return out, lse
