"""Plain 64-bit forms of the packed-row calls and of the 8-bit cache, on the
CPU (numpy), and helpers that build their inputs. Written from the definitions
in include/resa.h; nothing of the library is used."""
from __future__ import annotations

import math

import numpy as np
import torch

Q = {"int8": 127.0, "e4m3": 448.0}
DTYPE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
LEAST = 2.0 ** -100
D = 128


def f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().to(torch.float32).double().numpy()


def bf16(x: np.ndarray) -> np.ndarray:
    """Nearest bf16 of fp32 values, as float64."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).bfloat16().double().numpy()


_E4M3 = np.arange(127, dtype=np.uint8)
_GRID = torch.from_numpy(_E4M3.copy()).view(torch.float8_e4m3fn).double().numpy()  # 0 .. 448, rising


def nearest_code(y: np.ndarray, fmt: str) -> np.ndarray:
    """The quotient to 19 significant bits, then the nearest code value, ties to even."""
    m, e = np.frexp(y)
    y = np.ldexp(np.floor(np.abs(m) * 2.0 ** 19 + 0.5) * np.sign(m), e - 19)
    if fmt == "int8":
        return np.clip(np.rint(y), -127, 127)
    mag = np.minimum(np.abs(y), 448.0)
    mid = (_GRID[1:] + _GRID[:-1]) / 2
    lo, hi = np.searchsorted(mid, mag), np.searchsorted(mid, mag, side="right")
    return _GRID[np.where(lo % 2 == 0, lo, hi)] * np.sign(y)


class RefCache:
    """A cache as code values, scales and summaries, [B, H, blocks, ...], float64."""

    def __init__(self, B, H, cap, b, fmt):
        mb = cap // b
        self.b, self.fmt, self.cap = b, fmt, cap
        self.codes = {n: np.zeros((B, H, mb, b, D)) for n in "kv"}
        self.scale = {n: np.zeros((B, H, mb), np.float32) for n in "kv"}
        self.kmin, self.kmax = np.zeros((B, H, mb, D)), np.zeros((B, H, mb, D))

    def store(self, k, v, cu, lens):
        """k, v: float64 [T, H, D]; the last rows of each sequence."""
        T = k.shape[0]
        for s, L in enumerate(lens):
            lo, hi = min(max(cu[s], 0), T), min(max(cu[s + 1], 0), T)
            n = hi - lo
            if n <= 0 or n > L or L > self.cap:
                continue
            first = L - n
            for m in range(first // self.b, (L - 1) // self.b + 1):
                t0, t1 = max(first, m * self.b), min(L, (m + 1) * self.b)
                keep = t0 - m * self.b
                for name, x in (("k", k), ("v", v)):
                    new = x[lo + t0 - first:lo + t1 - first].transpose(1, 0, 2)     # [H, rows, D]
                    A = np.abs(new).max((1, 2))
                    bad = ~np.isfinite(new).all((1, 2))
                    with np.errstate(invalid="ignore"):
                        sc = (np.maximum(np.where(bad, 0, A), LEAST) / Q[self.fmt]).astype(np.float32)
                    old = self.scale[name][s, :, m].copy()
                    if keep:
                        bad = bad | np.isnan(old)
                        sc = np.maximum(sc, np.where(np.isnan(old), 0, old)).astype(np.float32)
                    sc = np.where(bad, np.float32(np.nan), sc)
                    codes = self.codes[name][s, :, m]
                    for h in range(len(sc)):
                        if bad[h]:
                            codes[h, :keep + t1 - t0] = 0
                            continue
                        if keep and old[h] != sc[h]:
                            codes[h, :keep] = nearest_code(codes[h, :keep] * np.float64(old[h]) / np.float64(sc[h]), self.fmt)
                        codes[h, keep:keep + t1 - t0] = nearest_code(new[h] / np.float64(sc[h]), self.fmt)
                    self.scale[name][s, :, m] = sc
                new = k[lo + t0 - first:lo + t1 - first].transpose(1, 0, 2)
                mn, mx = new.min(1), new.max(1)
                if keep:
                    mn, mx = np.minimum(mn, self.kmin[s, :, m]), np.maximum(mx, self.kmax[s, :, m])
                self.kmin[s, :, m], self.kmax[s, :, m] = mn, mx

    def values(self, name, s, h, L):
        """float64 [L, D]: code times scale."""
        x = self.codes[name][s, h] * self.scale[name][s, h][:, None, None].astype(np.float64)
        return x.reshape(-1, D)[:L]

    def loaded(self, cu, lens, T):
        """bf16(code * scale) of the last rows, and which packed rows there are."""
        H = self.codes["k"].shape[1]
        out, there = {n: np.zeros((T, H, D)) for n in "kv"}, np.zeros(T, bool)
        for s, L in enumerate(lens):
            n = cu[s + 1] - cu[s]
            if n <= 0 or n > L or L > self.cap:
                continue
            there[cu[s]:cu[s + 1]] = True
            for name in "kv":
                for h in range(H):
                    c = self.codes[name][s, h].reshape(-1, D)[L - n:L].astype(np.float32)
                    sc = np.repeat(self.scale[name][s, h], self.b)[L - n:L]
                    out[name][cu[s]:cu[s + 1], h] = bf16(c * sc[:, None])
        return out, there


def attend(q, k, v, scale, last=None):
    """Rows of q [R, D] over keys [n, D]; row r sees keys up to last[r] (all if None).
    Returns out, lse, and A = sum of weight * |v| (what a relative error of the
    weights multiplies), spread = the largest sum of |q_d k_d| * scale a row meets."""
    s = (q @ k.T) * scale
    reach = (np.abs(q) @ np.abs(k).T) * abs(scale)
    if last is not None:
        hide = np.arange(k.shape[0])[None, :] > np.asarray(last)[:, None]
        s = np.where(hide, -np.inf, s)
        reach = np.where(hide, 0.0, reach)
    if s.shape[1] == 0:
        z = np.zeros((q.shape[0], D))
        return z, np.full(q.shape[0], -np.inf), z, np.zeros(q.shape[0])
    m = s.max(1, keepdims=True)
    p = np.exp(s - np.where(np.isfinite(m), m, 0.0))
    l = p.sum(1, keepdims=True)
    w = p / np.where(l == 0, 1.0, l)
    with np.errstate(divide="ignore"):
        lse = (np.log(l) + np.where(np.isfinite(m), m, 0.0))[:, 0]
    return w @ v, lse, w @ np.abs(v), reach.max(1)


def score_error(reach):
    """Relative error of a weight from its score in fp32: 128 products summed (at
    most 128 roundings of partial sums no larger than reach), the products with
    the scales, and the exponential, for the weight and for the sum."""
    return 2 * (np.asarray(reach) * math.log2(math.e) * 132 * 2.0 ** -24 + 2.0 ** -21)


def check(got, want, bound, what):
    """Every element within its bound; prints the worst share of it."""
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == want.shape
    assert np.isfinite(got).all(), f"{what}: not finite"
    d = np.abs(got - want)
    share = float((d / np.maximum(bound, 1e-300)).max()) if d.size else 0.0
    print(f"{what}: worst {float(d.max()) if d.size else 0:.2e}, {share:.3f} of the bound", flush=True)
    assert share <= 1.0, f"{what}: {share} of the bound"


def cumulative(counts):
    return [0] + [int(x) for x in np.cumsum(counts)]


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def randn(shape, seed, spread=1.0):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g) * spread).bfloat16()
