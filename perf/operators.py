"""Performance cases of the packed prompt attention and of the 8-bit cache: what
a serving program does with them in one attention layer on one GPU.

A case names a kind of call and its sizes:

* ``prompt``   ``prompt_attention``: causal attention of packed prompts of
               different lengths, grouped heads;
* ``store``    ``store_rows_q8`` of each sequence's last rows (a prompt, a chunk,
               one decoded token), then ``load_rows_q8`` of the rows of the
               blocks it touched: what the cache holds for them;
* ``decode``   ``sparse_decode_q8``: one token over the selected blocks;
* ``rectify``  ``dense_rectify_q8``: the last rows of each sequence written again
               and their queries attended densely over the whole cache.

Sequence i of a batch has ``len`` tokens less a share that grows with i where
``ragged`` is set; ``rows`` is the number of new rows of a sequence (0: all of
them). ``fused`` takes q, k and v as parts of one projection's output
[T, Hq + 2 Hkv, 128], so a token's rows are not next to the following one's.
Inputs are drawn on the GPU from the seed: N(0, 1) rounded to bf16, keys scaled
per (kv head, channel) by LogNormal(0, 0.5) as in caches with outlier channels.

The definition of a stored block: its scale is A / Q (Q 127 for int8, 448 for
e4m3) in fp32, A the largest magnitude of its rows (2^-100 at least); where
rows written earlier stay in the block, the larger of that and the block's
scale. A code is the value over the scale rounded to the nearest code, ties to
even, the quotient first to 19 significant bits (so that a tie of the exact
quotient is one, whatever the division's last bits); codes that stay are
rounded again when the scale grows.
"""
import math

import torch

own = False

D = 128
Q_MAX = {"int8": 127.0, "e4m3": 448.0}
LEAST = 2.0 ** -100


def listed():
    return [
        # The smallest prompt: one short question, where launches count most.
        dict(name="prompt_300", kind="prompt", batch=1, hq=32, hkv=8, len=300, ragged=False, fused=True),
        # A serving batch's new prompts, packed: odd lengths from 77 tokens to
        # 2000, a 7B-class layer of 28 query and 4 kv heads.
        dict(name="prompt_packed_g7", kind="prompt", batch=16, hq=28, hkv=4, len=2000, ragged=True, fused=False),
        # One long prompt.
        dict(name="prompt_16k", kind="prompt", batch=1, hq=32, hkv=8, len=16384, ragged=False, fused=True),
        # A decoded token of a batch of eight: the new row's block is rounded
        # again where the row raises its scale.
        dict(name="store_token_b8", kind="store", batch=8, hkv=8, len=8180, rows=1, block=16, fmt="int8",
             ragged=True, paged=False),
        # The prompts of a batch enter the cache.
        dict(name="store_prompts", kind="store", batch=8, hkv=8, len=8192, rows=0, block=16, fmt="int8",
             ragged=True, paged=False),
        # The smallest decode: one sequence of 4K (selection as in a 0.9
        # sparsity loop with a budget of 1024 tokens at least).
        dict(name="decode_4k", kind="decode", batch=1, hq=32, hkv=8, len=4096, block=16, sparsity=0.9,
             min_tokens=1024, fmt="int8", ragged=False, paged=False),
        # The benchmark's decode over an 8-bit cache: 8 sequences of 64K.
        dict(name="decode_64k_b8", kind="decode", batch=8, hq=32, hkv=8, len=65536, block=16, sparsity=0.9,
             min_tokens=2048, fmt="int8", ragged=False, paged=False),
        # One very long sequence.
        dict(name="decode_256k", kind="decode", batch=1, hq=32, hkv=8, len=262144, block=16, sparsity=0.95,
             min_tokens=4096, fmt="e4m3", ragged=False, paged=False),
        # A continuous batch: ragged odd lengths on a shuffled page pool,
        # 32-token blocks, 8 query heads to a kv head.
        dict(name="decode_paged", kind="decode", batch=6, hq=64, hkv=8, len=50001, block=32, sparsity=0.9,
             min_tokens=2048, fmt="e4m3", ragged=True, paged=True),
        # The rectification of a short sequence.
        dict(name="rectify_4k", kind="rectify", batch=1, hq=32, hkv=8, len=4096, rows=16, block=16, fmt="int8",
             ragged=False, paged=False),
        # The benchmark's rectification over an 8-bit cache.
        dict(name="rectify_64k_b8", kind="rectify", batch=8, hq=32, hkv=8, len=65536, rows=32, block=16,
             fmt="int8", ragged=False, paged=False),
        # Chunked prefill in a continuous batch: an odd chunk behind ragged
        # contexts, paged, 28 query and 4 kv heads.
        dict(name="rectify_chunk_paged", kind="rectify", batch=2, hq=28, hkv=4, len=33001, rows=2033, block=32,
             fmt="e4m3", ragged=True, paged=True),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 200)


def draw(rng):
    largest = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["prompt", "store", "decode", "rectify"])
        hkv = rng.choice([1, 2, 4, 8])
        c = dict(kind=kind, batch=rng.randint(1, 16), hkv=hkv, ragged=rng.random() < 0.6)
        if kind != "store":
            c["hq"] = hkv * rng.randint(1, 8)
        if kind == "prompt":
            c["fused"] = rng.random() < 0.5
            c["len"] = _spread(rng, 1, 16384)
            scores = c["batch"] * c["hq"] * c["len"] ** 2
        else:
            c["batch"] = min(c["batch"], 8)
            c["block"] = rng.choice([16, 16, 32, 64])
            c["fmt"] = rng.choice(["int8", "e4m3"])
            c["paged"] = rng.random() < 0.4
            c["len"] = _spread(rng, 40, 262144)
            scores = 0
        if kind == "decode":
            c["sparsity"] = rng.choice([0.0, 0.8, 0.9, 0.9, 0.95])
            c["min_tokens"] = rng.choice([1024, 2048, 4096])
        if kind == "store":
            c["rows"] = rng.choice([0, 1, 1, _spread(rng, 1, c["len"])])
        if kind == "rectify":
            c["rows"] = _spread(rng, 1, min(c["len"], 2048))
            scores = c["batch"] * c["hq"] * c["rows"] * c["len"]
        # The plain forms write every score and hold the stored rows in 64
        # bits; a cache has at most 2 Gi elements.
        stored = c["batch"] * hkv * D * ((c.get("rows") or c["len"]) if kind in ("store", "rectify") else 0)
        read = c["batch"] * hkv * c["len"] * D * 2 if kind in ("rectify", "decode") else 0
        if scores > 1 << 33 or stored > 1 << 26 or read > 1 << 31:
            continue
        if _cost(c) <= largest:
            return c


# ------------------------------------------------------------------- inputs

def _lens(case):
    """Length of each sequence, the new rows counted."""
    L, B = case["len"], case["batch"]
    if not case["ragged"]:
        return [L] * B
    return [max(1, L - i * L // B - (i * 7) % 5 * (L > 64)) for i in range(B)]


def _rows(case):
    """New rows of each sequence."""
    n = case.get("rows", 0)
    return [min(n or L, L) for L in _lens(case)]


def _capacity(case):
    b = case["block"]
    return -(-case["len"] // b) * b


def _read_rows(case):
    """Rows of each sequence that are read back: all of the blocks that were written to."""
    b = case["block"]
    return [L - (L - n) // b * b for L, n in zip(_lens(case), _rows(case))]


def _selected(case):
    """Selected blocks of each sequence (Eq. 5)."""
    b, keep = case["block"], round((1 - case["sparsity"]) * 1000000)
    least = max(1, -(-case["min_tokens"] // b))
    return [min(M, max(least, -(-M * keep // 1000000))) for M in (-(-L // b) for L in _lens(case))]


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cumulative(counts):
    total = [0]
    for n in counts:
        total.append(total[-1] + n)
    return _i32(total)


class _Cache:
    """The tensors of an 8-bit cache."""


def _fill(case, gen):
    """A cache with every sequence's rows in it, as a serving loop leaves it."""
    B, H, b, fmt = case["batch"], case["hkv"], case["block"], case["fmt"]
    cap = _capacity(case)
    mb = cap // b
    c = _Cache()
    c.block_size, c.fmt, c.block_table = b, fmt, None
    channel = torch.exp(0.5 * torch.randn((H, 1, D), generator=gen, device="cuda"))
    dtype = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
    parts = {"k": [], "v": []}
    c.kmin = torch.empty((B, H, mb, D), dtype=torch.bfloat16, device="cuda")
    c.kmax = torch.empty_like(c.kmin)
    for s in range(B):
        for name in "kv":
            x = torch.randn((H, cap, D), generator=gen, device="cuda")
            x = (x * channel if name == "k" else x).bfloat16().float().view(H, mb, b, D)
            if name == "k":
                c.kmin[s], c.kmax[s] = x.amin(2), x.amax(2)
            scale = x.abs().amax((2, 3)) / Q_MAX[fmt]
            x = (x / scale[..., None, None]).clamp(-Q_MAX[fmt], Q_MAX[fmt])
            parts[name].append(((x.round() if fmt == "int8" else x).to(dtype), scale))
    for name in "kv":
        codes = torch.stack([p[0].view(torch.int8) for p in parts[name]])  # [B, H, mb, b, D]
        scales = torch.stack([p[1] for p in parts[name]])                  # [B, H, mb]
        if case["paged"]:
            if c.block_table is None:
                pages = B * mb + 7
                order = torch.randperm(pages, generator=gen, device="cuda")[:B * mb]
                c.block_table = order.to(torch.int32).view(B, mb)
            pool = torch.zeros((pages, H, b, D), dtype=torch.int8, device="cuda")
            pool[order] = codes.permute(0, 2, 1, 3, 4).reshape(B * mb, H, b, D)
            scale_pool = torch.ones((pages, H), device="cuda")
            scale_pool[order] = scales.permute(0, 2, 1).reshape(B * mb, H)
            codes, scales = pool, scale_pool
        else:
            codes = codes.view(B, H, cap, D)
        setattr(c, name, codes.view(dtype))
        setattr(c, name + "_scale", scales.contiguous())
    return c, channel


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = {"case": case, "out": None}
    lens, rows = _lens(case), _rows(case)
    st["lens"], st["longest"] = _i32(lens), max(lens)
    H = case["hkv"]
    if case["kind"] == "prompt":
        T, hq = sum(lens), case["hq"]
        channel = torch.exp(0.5 * torch.randn((H, D), generator=gen, device="cuda"))
        x = torch.randn((T, hq + 2 * H, D), generator=gen, device="cuda")
        x[:, hq:hq + H] *= channel
        x = x.bfloat16()
        st["q"], st["k"], st["v"] = x[:, :hq], x[:, hq:hq + H], x[:, hq + H:]
        if not case["fused"]:
            st["q"], st["k"], st["v"] = st["q"].contiguous(), st["k"].contiguous(), st["v"].contiguous()
        st["cu"], st["counts"] = _cumulative(lens), lens
        st["result"] = (torch.empty((T, hq, D), dtype=torch.bfloat16, device="cuda"),
                        torch.empty((T, hq), device="cuda"))
        return st
    st["cache"], channel = _fill(case, gen)
    if case["kind"] == "decode":
        B, M, n = case["batch"], -(-max(lens) // case["block"]), _selected(case)
        rank = torch.rand((B, H, M), generator=gen, device="cuda")
        last = (st["lens"].long() - 1) // case["block"]
        blocks = torch.arange(M, device="cuda")
        rank = torch.where(blocks > last[:, None, None], -1.0, rank)
        rank = torch.where(blocks == last[:, None, None], 2.0, rank)
        idx = rank.topk(max(n), dim=2).indices
        keep = torch.arange(max(n), device="cuda") < _i32(n)[:, None, None]
        idx = torch.where(keep, idx, M).sort(2).values
        st["idx"] = torch.where(keep, idx, -1).to(torch.int32).contiguous()
        st["nsel"] = _i32(n)[:, None].expand(B, H).contiguous()
        st["q"] = torch.randn((B, case["hq"], D), generator=gen, device="cuda").bfloat16()
        st["result"] = (torch.empty((B, case["hq"], D), device="cuda"), torch.empty((B, case["hq"]), device="cuda"))
    else:
        T = sum(rows)
        st["k"] = (torch.randn((T, H, D), generator=gen, device="cuda") * channel[:, 0]).bfloat16()
        st["v"] = torch.randn((T, H, D), generator=gen, device="cuda").bfloat16()
        st["cu"], st["counts"] = _cumulative(rows), rows
        st["back"], st["back_counts"] = _cumulative(_read_rows(case)), _read_rows(case)
        if case["kind"] == "rectify":
            st["q"] = torch.randn((T, case["hq"], D), generator=gen, device="cuda").bfloat16()
            st["result"] = (torch.empty((T, case["hq"], D), dtype=torch.bfloat16, device="cuda"),
                            torch.empty((T, case["hq"]), device="cuda"))
        back = sum(st["back_counts"])
        st["values"] = tuple(torch.empty((back, H, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    if own:
        import paper_2506_04108_amd as R
        c = st["cache"]
        st["handle"] = R.KVCacheQ8(c.k, c.v, c.k_scale, c.v_scale, c.kmin, c.kmax, c.block_size, c.block_table)
        st["workspace"] = R.Workspace("cuda")
    return st


# -------------------------------------------------------------------- passes

def run(st):
    case = st["case"]
    if own:
        return _own(st, case)
    if case["kind"] == "prompt":
        return _plain_prompt(st, case)
    if case["kind"] == "decode":
        return _plain_decode(st, case)
    _plain_store(st, case)
    result = {}
    if case["kind"] == "rectify":
        result["out"], result["lse"] = _plain_rectify(st, case)
    return {**result, **_state(st["cache"]), **_plain_load(st, case)}


def _state(c):
    return {"k_scale": c.k_scale, "v_scale": c.v_scale, "kmin": c.kmin, "kmax": c.kmax}


def _own(st, case):
    import paper_2506_04108_amd as R
    if case["kind"] == "prompt":
        out, lse = R.prompt_attention(st["q"], st["k"], st["v"], st["cu"], out=st["result"][0], lse=st["result"][1])
        return {"out": out, "lse": lse}
    c = st["handle"]
    if case["kind"] == "decode":
        out, lse = R.sparse_decode_q8(c, st["q"], st["lens"], st["idx"], st["nsel"], out=st["result"][0],
                                      lse=st["result"][1], workspace=st["workspace"])
        return {"out": out, "lse": lse}
    result = {}
    if case["kind"] == "store":
        R.store_rows_q8(c, st["k"], st["v"], st["cu"], st["lens"])
    else:
        result["out"], result["lse"] = R.dense_rectify_q8(
            c, st["q"], st["k"], st["v"], st["cu"], st["lens"], st["longest"], out=st["result"][0],
            lse=st["result"][1], workspace=st["workspace"])
    k, v = R.load_rows_q8(c, st["back"], st["lens"], out=st["values"])
    return {**result, **_state(c), "k": k, "v": v}


def _places(counts, longest):
    """Of packed rows: (row of [B, longest] or 0 where there is none, whether there is one)."""
    n = torch.tensor(counts, device="cuda")
    i = torch.arange(longest, device="cuda")
    there = i < n[:, None]
    return torch.where(there, (n.cumsum(0) - n)[:, None] + i, 0), there


def _softmax_product(s, v):
    """softmax(s) v and the log of the sum, over the last axis of s; empty rows give 0 and -inf."""
    m = s.amax(-1, keepdim=True)
    p = (s - torch.where(m == -math.inf, 0.0, m)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    return out, (total.log() + m)[..., 0]


def _plain_prompt(st, case):
    H, G, n = case["hkv"], case["hq"] // case["hkv"], max(st["counts"])
    at, there = _places(st["counts"], n)                                          # [B, n]
    q = st["q"].float()[at].view(*at.shape, H, G, D).permute(0, 2, 3, 1, 4)       # [B, H, G, n, D]
    k = st["k"].float()[at].permute(0, 2, 3, 1)[:, :, None]                       # [B, H, 1, D, n]
    v = st["v"].float()[at].permute(0, 2, 1, 3)[:, :, None]
    i = torch.arange(n, device="cuda")
    s = torch.matmul(q.contiguous() * D ** -0.5, k.contiguous())
    s.masked_fill_((i > i[:, None]), -math.inf)
    out, lse = _softmax_product(s, v.contiguous())
    back = there.flatten().nonzero()[:, 0]
    out = out.permute(0, 3, 1, 2, 4).reshape(-1, H * G, D)[back]
    lse = lse.permute(0, 3, 1, 2).reshape(-1, H * G)[back]
    return {"out": out.bfloat16(), "lse": lse}


def _block_rows(c, blocks):
    """Page or (sequence, block) index of blocks [B, ...], for codes [.., H, b, D] and scales [.., H]."""
    B = blocks.shape[0]
    seq = torch.arange(B, device="cuda").view(B, *[1] * (blocks.dim() - 1)).expand(blocks.shape)
    if c.block_table is not None:
        return c.block_table[seq, blocks].long()
    return seq * (c.kmin.shape[2]) + blocks


def _by_block(c, name):
    """(codes [pages, H, b, D], scales [pages, H]) of a cache, one page a block, in an order of their own."""
    codes, scale = getattr(c, name), getattr(c, name + "_scale")
    if c.block_table is not None:
        return codes, scale
    B, H, mb = scale.shape
    return (codes.view(torch.int8).view(B, H, mb, c.block_size, D).transpose(1, 2).reshape(B * mb, H, c.block_size, D).view(codes.dtype),
            scale.transpose(1, 2).reshape(B * mb, H))


def _values(codes, scale):
    return codes.float() * scale[..., None, None]


def _plain_decode(st, case):
    c, b, H, G = st["cache"], case["block"], case["hkv"], case["hq"] // case["hkv"]
    B, n = case["batch"], st["idx"].shape[2]
    idx = st["idx"].long()
    token = idx[..., None] * b + torch.arange(b, device="cuda")
    used = (idx >= 0)[..., None] & (token < st["lens"].long().view(B, 1, 1, 1))
    head = torch.arange(H, device="cuda")[:, None]
    at = idx.clamp(min=0)

    def rows(name):
        codes, scale = getattr(c, name), getattr(c, name + "_scale")
        if c.block_table is not None:
            page = _block_rows(c, at)
            x, s = codes.view(torch.int8)[page, head], scale[page, head]
        else:
            seq = torch.arange(B, device="cuda")[:, None, None]
            x, s = codes.view(torch.int8).view(B, H, -1, b, D)[seq, head, at], scale[seq, head, at]
        return _values(x.view(codes.dtype), s).view(B, H, n * b, D)

    q = st["q"].float().view(B, H, G, D)
    s = torch.matmul(q * D ** -0.5, rows("k").transpose(2, 3).contiguous())
    s.masked_fill_(~used.view(B, H, 1, n * b), -math.inf)
    out, lse = _softmax_product(s, rows("v"))
    return {"out": out.reshape(B, H * G, D), "lse": lse.reshape(B, H * G)}


def _to_code(y, fmt):
    """y (64 bits) to 19 significant bits, then to the nearest code value, ties to even."""
    m, e = torch.frexp(y)
    y = torch.ldexp((m * 2.0 ** 19).round() / 2.0 ** 19, e)
    if fmt == "int8":
        return y.round().clamp(-127, 127)
    step = torch.ldexp(torch.ones_like(y), torch.frexp(y)[1].clamp(min=-5) - 4)
    return ((y / step).round() * step).clamp(-448, 448)


def _plain_store(st, case):
    """Every block that a sequence's new rows touch, at once."""
    c, b, H, B, fmt = st["cache"], case["block"], case["hkv"], case["batch"], case["fmt"]
    L = st["lens"].long()
    first = L - torch.tensor(st["counts"], device="cuda")
    per = max((x + b - 1) // b - (x - n) // b for x, n in zip(_lens(case), st["counts"]))
    block = (first // b)[:, None] + torch.arange(per, device="cuda")                # [B, per]
    touched = block * b < L[:, None]
    block = torch.where(touched, block, 0)[touched]                                 # [P]
    seq = torch.arange(B, device="cuda")[:, None].expand(B, per)[touched]
    token = block[:, None] * b + torch.arange(b, device="cuda")                     # [P, b]
    new = (token >= first[seq, None]) & (token < L[seq, None])
    kept = token < first[seq, None]
    source = torch.where(new, st["cu"].long()[seq, None] + token - first[seq, None], 0)
    some = kept.any(1)[:, None]                                                     # [P, 1]
    head = torch.arange(H, device="cuda")
    page = None if c.block_table is None else c.block_table[seq, block].long()
    for name in "kv":
        x = st[name][source].permute(0, 2, 1, 3)                                    # [P, H, b, D]
        x = torch.where(new[:, None, :, None], x, 0).double()
        codes, scale = getattr(c, name), getattr(c, name + "_scale")
        dtype = codes.dtype
        if page is None:
            codes = codes.view(torch.int8).view(B, H, -1, b, D)
            at = (seq[:, None], head, block[:, None])
        else:
            codes, at = codes.view(torch.int8), (page[:, None], head)
        old, old_scale = codes[at].view(dtype), scale[at].double()
        s = (x.abs().amax((2, 3)).clamp(min=LEAST) / Q_MAX[fmt]).float().double()
        s = torch.where(some, torch.maximum(s, old_scale), s)                       # [P, H]
        y = torch.where(kept[:, None, :, None], old.to(torch.float32).double() * old_scale[..., None, None], x)
        y = _to_code(y / s[..., None, None], fmt).to(torch.float32)
        y = torch.where(kept[:, None, :, None] & (s <= old_scale)[..., None, None], old.to(torch.float32), y)
        codes[at] = torch.where((kept | new)[:, None, :, None], y.to(dtype).view(torch.int8), old.view(torch.int8))
        scale[at] = s.float()
        if name == "k":
            lo = torch.where(new[:, None, :, None], x, math.inf).amin(2)
            hi = torch.where(new[:, None, :, None], x, -math.inf).amax(2)
            where = (seq[:, None], head, block[:, None])
            lo = torch.where(some[..., None], torch.minimum(lo, c.kmin[where].double()), lo)
            hi = torch.where(some[..., None], torch.maximum(hi, c.kmax[where].double()), hi)
            c.kmin[where], c.kmax[where] = lo.bfloat16(), hi.bfloat16()


def _plain_load(st, case):
    """The last rows of every sequence, as the values that their codes stand for."""
    c, b, n = st["cache"], case["block"], max(st["back_counts"])
    at, there = _places(st["back_counts"], n)
    i = torch.arange(n, device="cuda")
    token = (st["lens"].long() - torch.tensor(st["back_counts"], device="cuda"))[:, None] + i
    seq = torch.arange(case["batch"], device="cuda")[:, None].expand(token.shape)[there]
    token = token[there]
    head = torch.arange(case["hkv"], device="cuda")
    result = {}
    for name in "kv":
        codes, scale = getattr(c, name), getattr(c, name + "_scale")
        if c.block_table is None:
            x = codes.view(torch.int8)[seq[:, None], head, token[:, None]].view(codes.dtype)
            s = scale[seq[:, None], head, token[:, None] // b]
        else:
            page = c.block_table[seq, token // b].long()[:, None]
            x = codes.view(torch.int8)[page, head, token[:, None] % b].view(codes.dtype)
            s = scale[page, head]
        result[name] = (x.float() * s[..., None]).bfloat16()
    return result


def _plain_rectify(st, case):
    c, b, H, G, B = st["cache"], case["block"], case["hkv"], case["hq"] // case["hkv"], case["batch"]
    M, n = -(-st["longest"] // b), max(st["counts"])

    def rows(name):
        codes, scale = getattr(c, name), getattr(c, name + "_scale")
        if c.block_table is None:
            return _values(codes.view(B, H, -1, b, D), scale)[:, :, :M].reshape(B, H, 1, M * b, D)
        page = c.block_table.long()[:, :M]
        x = _values(codes.view(torch.int8)[page].view(codes.dtype), scale[page])    # [B, M, H, b, D]
        return x.transpose(1, 2).reshape(B, H, 1, M * b, D)

    at, there = _places(st["counts"], n)
    q = st["q"].float()[at].view(B, n, H, G, D).permute(0, 2, 3, 1, 4)              # [B, H, G, n, D]
    s = torch.matmul(q.contiguous() * D ** -0.5, rows("k").transpose(3, 4).contiguous())
    first = st["lens"].long() - torch.tensor(st["counts"], device="cuda")
    last = first[:, None] + torch.arange(n, device="cuda")                          # [B, n]
    token = torch.arange(M * b, device="cuda")
    s.masked_fill_((token > last[..., None])[:, None, None], -math.inf)
    out, lse = _softmax_product(s, rows("v"))
    back = there.flatten().nonzero()[:, 0]
    out = out.permute(0, 3, 1, 2, 4).reshape(-1, H * G, D)[back]
    return out.bfloat16(), lse.permute(0, 3, 1, 2).reshape(-1, H * G)[back]


# ---------------------------------------------------------------------- work

def work(case):
    lens, rows, H = _lens(case), _rows(case), case["hkv"]
    T = sum(rows)
    if case["kind"] == "prompt":
        pairs = sum(n * (n + 1) // 2 for n in lens)
        return {"bytes": T * D * 2 * (2 * case["hq"] + 2 * H) + 4 * T * case["hq"] + 4 * len(lens),
                "flops": 4 * D * case["hq"] * pairs}
    b, blocks = case["block"], lambda n: -(-n // case["block"])
    if case["kind"] == "decode":
        tokens = sum(min(n * b, L) for n, L in zip(_selected(case), lens))
        return {"bytes": H * (2 * D * tokens + 12 * sum(_selected(case))) + case["batch"] * case["hq"] * (6 * D + 4),
                "flops": 4 * D * case["hq"] * tokens}
    touched = sum(blocks(L) - (L - n) // b for L, n in zip(lens, rows))
    # The new rows in, their codes, scales and summaries out; rows read back.
    moved = H * (T * 2 * D * 3 + touched * (8 + 4 * D)) + H * sum(_read_rows(case)) * 2 * D * 3
    if case["kind"] == "store":
        return {"bytes": moved, "flops": 8 * H * D * T}
    pairs = sum(n * (L - n) + n * (n + 1) // 2 for L, n in zip(lens, rows))
    return {"bytes": moved + H * sum(2 * D * L + 8 * blocks(L) for L in lens) + T * case["hq"] * (4 * D + 4),
            "flops": 4 * D * case["hq"] * pairs}


# --------------------------------------------------------------------- exact

def _attend64(q, k, v, scale_k, scale_v, visible):
    """Rows of q [R, D] over keys k, v [n, D] with a factor a key; visible [R, n] or None."""
    s = (q.double() @ k.double().t()) * (scale_k * D ** -0.5)
    if visible is not None:
        s = torch.where(visible, s, -math.inf)
    lse = torch.logsumexp(s, 1)
    return torch.exp(s - lse[:, None]) @ (v.double() * scale_v[:, None]), lse


def _pieces(rows, keys):
    """Row ranges of a product of at most 2^27 scores each."""
    step = max(1, (1 << 27) // max(1, keys))
    return [(r, min(rows, r + step)) for r in range(0, rows, step)]


def _nearest(x, fmt):
    """Nearest code value of each x (64 bits), ties to the even code."""
    if fmt == "int8":
        return torch.round(x)
    code = torch.arange(127, dtype=torch.uint8, device="cuda")  # the codes of 0 .. 448, rising
    grid = code.view(torch.float8_e4m3fn).double()
    mid = (grid[1:] + grid[:-1]) / 2
    lo, hi = torch.searchsorted(mid, x.abs().contiguous()), torch.searchsorted(mid, x.abs().contiguous(), right=True)
    return grid[torch.where((lo % 2 == 0), lo, hi)] * x.sign()


def exact(case, seed):
    st = prepare(case, seed)
    lens, rows, H = _lens(case), _rows(case), case["hkv"]
    out, lse = [], []
    if case["kind"] == "prompt":
        G, start = case["hq"] // H, 0
        one = torch.ones((), dtype=torch.float64, device="cuda")
        for n in lens:
            o = torch.empty((n, case["hq"], D), dtype=torch.float64, device="cuda")
            m = torch.empty((n, case["hq"]), dtype=torch.float64, device="cuda")
            for h in range(case["hq"]):
                k, v = st["k"][start:start + n, h // G], st["v"][start:start + n, h // G]
                for lo, hi in _pieces(n, n):
                    see = torch.arange(hi, device="cuda") <= torch.arange(lo, hi, device="cuda")[:, None]
                    o[lo:hi, h], m[lo:hi, h] = _attend64(st["q"][start + lo:start + hi, h], k[:hi], v[:hi], one,
                                                         one.expand(hi), see)
            out.append(o)
            lse.append(m)
            start += n
        return {"out": torch.cat(out), "lse": torch.cat(lse)}
    c, b, fmt = st["cache"], case["block"], case["fmt"]
    Qm = Q_MAX[fmt]

    def place(name, s, m):
        """Codes [H, b, D] and scales [H] of block m of sequence s: views."""
        codes, scale = getattr(c, name), getattr(c, name + "_scale")
        if c.block_table is None:
            return codes[s, :, m * b:(m + 1) * b], scale[s, :, m]
        page = table[s][m]
        return codes[page], scale[page]

    table = None if c.block_table is None else c.block_table.tolist()

    def whole(name, s, n):
        """Codes [H, n, D] of a sequence's first n tokens in 32 bits, and a scale for each token [H, n]."""
        codes, scale = getattr(c, name), getattr(c, name + "_scale")
        if c.block_table is None:
            return codes[s, :, :n].float(), scale[s].double().repeat_interleave(b, 1)[:, :n]
        pages = c.block_table[s, :-(-n // b)].long()
        x = codes.view(torch.int8)[pages].view(codes.dtype).float().transpose(0, 1).reshape(H, -1, D)
        return x[:, :n], scale[pages].double().t().repeat_interleave(b, 1)[:, :n]

    if case["kind"] == "decode":
        G = case["hq"] // H
        for s, L in enumerate(lens):
            k, ks = whole("k", s, L)
            v, vs = whole("v", s, L)
            for h in range(H):
                ids = st["idx"][s, h, :int(st["nsel"][s, h])].long()
                t = (ids[:, None] * b + torch.arange(b, device="cuda")).flatten()
                t = t[t < L]
                o, m = _attend64(st["q"][s, h * G:(h + 1) * G], k[h, t], v[h, t], ks[h, t], vs[h, t], None)
                out.append(o)
                lse.append(m)
        return {"out": torch.cat(out).view(len(lens), -1, D), "lse": torch.cat(lse).view(len(lens), -1)}
    # The stored blocks: those with rows that stay one by one, the others of a sequence at once. The state's
    # own buffers take the new codes (they are values of the code's type); scales and summaries in 64 bits.
    scales = {name: getattr(c, name + "_scale").double() for name in "kv"}
    kmin, kmax = c.kmin.double(), c.kmax.double()
    values, start = {"k": [], "v": []}, 0
    for s, (L, n, back) in enumerate(zip(lens, rows, _read_rows(case))):
        first = L - n
        for name in "kv":
            x = st[name][start:start + n].double().transpose(0, 1)                  # [H, n, D]
            t, read = first, []
            while t < L:
                m, edge = t // b, t % b != 0
                # A block that keeps rows, or whole blocks up to the last.
                end = min(L, (m + 1) * b) if edge or L - t < b else t + (L - t) // b * b
                y = x[:, t - first:end - first]
                y = y.view(H, 1, -1, D) if edge or end - t < b else y.reshape(H, -1, b, D)
                A = y.abs().amax((2, 3)).clamp(min=LEAST)                           # [H, blocks]
                count = y.shape[1]
                if edge:
                    codes, old = place(name, s, m)
                    A_old = (old.double() * Qm).bfloat16().double()  # the magnitude that the scale was made of
                    grown = torch.maximum(A, A_old[:, None])
                    before = codes[:, :t % b].to(torch.float32).double()            # [H, kept, D]
                    again = _nearest(before * A_old[:, None, None] / grown[:, :, None], fmt)
                    again = torch.where((A > A_old[:, None])[:, :, None], again, before)
                    codes[:, :t % b] = again.float().to(codes.dtype)
                    A = grown
                    read.append(again * (A / Qm)[:, :, None])
                new = _nearest(y * Qm / A[..., None, None], fmt)
                read.append((new * (A / Qm)[..., None, None]).reshape(H, -1, D))
                for j in range(count):
                    codes, _ = place(name, s, m + j)
                    at = t % b
                    codes[:, at:at + new.shape[2]] = new[:, j].float().to(codes.dtype)
                    if c.block_table is None:
                        scales[name][s, :, m + j] = A[:, j] / Qm
                    else:
                        scales[name][table[s][m + j]] = A[:, j] / Qm
                if name == "k":
                    lo, hi = y.amin(2), y.amax(2)
                    if edge:
                        lo, hi = torch.minimum(lo, kmin[s, :, m:m + 1]), torch.maximum(hi, kmax[s, :, m:m + 1])
                    kmin[s, :, m:m + count], kmax[s, :, m:m + count] = lo, hi
                t = end
            values[name].append(torch.cat(read, 1).transpose(0, 1))
        start += n
    result = {"k_scale": scales["k"], "v_scale": scales["v"], "kmin": kmin, "kmax": kmax,
              "k": torch.cat(values["k"]), "v": torch.cat(values["v"])}
    if case["kind"] == "store":
        return result
    c.k_scale, c.v_scale = scales["k"], scales["v"]
    G, start = case["hq"] // H, 0
    for s, (L, n) in enumerate(zip(lens, rows)):
        k, ks = whole("k", s, L)
        v, vs = whole("v", s, L)
        o = torch.empty((n, case["hq"], D), dtype=torch.float64, device="cuda")
        m = torch.empty((n, case["hq"]), dtype=torch.float64, device="cuda")
        for h in range(case["hq"]):
            for lo, hi in _pieces(n, L):
                see = torch.arange(L, device="cuda") <= (L - n + torch.arange(lo, hi, device="cuda"))[:, None]
                o[lo:hi, h], m[lo:hi, h] = _attend64(st["q"][start + lo:start + hi, h], k[h // G], v[h // G],
                                                     ks[h // G], vs[h // G], see)
        out.append(o)
        lse.append(m)
        start += n
    return {"out": torch.cat(out), "lse": torch.cat(lse), **result}
