"""64-bit CPU reference of the quantised cache and of attention over a shared
prefix, from their definitions in include/wavefilter.h."""
from __future__ import annotations

import math

import numpy as np
import torch

TOP = {"e4m3": 448.0, "e2m1": 6.0}
BITS = {"e4m3": 8, "e2m1": 4}


def numbers(fmt: str) -> np.ndarray:
    """The number of every code, from its sign, exponent and mantissa bits."""
    if fmt == "e4m3":
        eb, mb, bias = 4, 3, 7
    else:
        eb, mb, bias = 2, 1, 1
    c = np.arange(1 << (1 + eb + mb))
    sign, e, m = c >> (eb + mb), (c >> mb) & ((1 << eb) - 1), c & ((1 << mb) - 1)
    mag = np.where(e == 0, np.ldexp(m / 2.0 ** mb, 1 - bias),
                   np.ldexp(1 + m / 2.0 ** mb, e - bias))
    v = np.where(sign == 1, -mag, mag)
    if fmt == "e4m3":
        v[[0x7f, 0xff]] = np.nan
    return v


def quantise(x: torch.Tensor, fmt: str):
    """Codes (one per channel, uint8) and exponent bytes of rows x [..., d]."""
    x = x.double().numpy()
    y = x.reshape(*x.shape[:-1], -1, 32)
    with np.errstate(invalid="ignore"):
        bad = ~np.isfinite(y).all(-1)
    y = np.where(bad[..., None], 0.0, y)
    m, k = np.frexp(np.abs(y).max(-1) / TOP[fmt])
    e = np.maximum(np.where(m == 0.5, k - 1, k), -126)
    e[np.abs(y).max(-1) == 0] = -126
    y = np.ldexp(y, -e[..., None]).reshape(x.shape)
    # to the nearest number, ties to the even code
    half = (1 << (BITS[fmt] - 1)) - (1 if fmt == "e4m3" else 0)
    pos = numbers(fmt)[:half]
    a = np.abs(y)
    hi = np.clip(np.searchsorted(pos, a), 1, half - 1)
    lo = hi - 1
    dl, dh = a - pos[lo], pos[hi] - a
    code = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
    code = code | (np.signbit(y).astype(np.int64) << (BITS[fmt] - 1))
    byte = np.where(bad, 255, e + 127)
    code = np.where(np.repeat(bad, 32, -1), 0, code.reshape(x.shape))
    return torch.from_numpy(code.astype(np.uint8)), torch.from_numpy(byte.astype(np.uint8))


def pack(code: torch.Tensor, fmt: str) -> torch.Tensor:
    return code if fmt == "e4m3" else code[..., 0::2] | (code[..., 1::2] << 4)


def values(codes: torch.Tensor, byte: torch.Tensor, fmt: str) -> torch.Tensor:
    """float64 values of packed codes."""
    c = codes.numpy()
    if fmt == "e2m1":
        c = np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:-1], -1)
    b = byte.numpy().astype(np.int64)
    s = np.where(b == 0, 0.0, np.where(b == 255, np.inf, np.ldexp(1.0, b - 127)))
    with np.errstate(invalid="ignore"):
        v = numbers(fmt)[c].reshape(*b.shape, 32) * s[..., None]
    return torch.from_numpy(v.reshape(c.shape))


def prefix_attention(Q, K, V, *, prefixes, share, heads, group, scale, plen=None, tlen=None,
                     rows=None, row_idx=None, Kt=None, Vt=None, dtype=torch.bfloat16):
    """O, lse in float64 and how far the kernel may be off, elementwise.

    Q [n, heads group, B, d], K, V [prefixes, heads, cap, d], row_idx
    [prefixes, heads, rows].  A row's weights w sum to 1; with A = sum w |v|:
      scores: products are exact in fp32 (bf16) or off by 2^-24 each (fp32),
        summed in fp32: es = (2 d + 4) 2^-24 max_j scale sum_i |q_i k_ji|, and
        the exponent's argument and 2^x add a few fp32 steps of the score;
      a relative error es of every weight and of their sum: 2 es A;
      sums over n keys in fp32: (n + 8) 2^-24 of A and of the sum of weights;
      bf16: weights rounded to half a step 2^-8, the output to 2^-8 of it."""
    n_seq, hq, B, d = Q.shape
    Q, K, V = (None if x is None else x.double() for x in (Q, K, V))
    O = torch.zeros((n_seq, hq, B, d), dtype=torch.float64)
    lse = torch.full((n_seq, hq, B), -math.inf, dtype=torch.float64)
    tol, ltol = torch.zeros_like(O), torch.zeros_like(lse)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for n in range(n_seq):
        i = n // share
        for x in range(hq):
            h = x // group
            keys, vals = torch.zeros((0, d)).double(), torch.zeros((0, d)).double()
            if rows:
                L = rows if plen is None else min(max(int(plen[i]), 0), rows)
                at = torch.arange(L) if row_idx is None else row_idx[i, h, :L].long()
                keys, vals = K[i, h][at], V[i, h][at]
            if Kt is not None:
                T = Kt.shape[2]
                t = T if tlen is None else min(max(int(tlen[n]), 0), T)
                keys = torch.cat([keys, Kt[n, h, :t].double()])
                vals = torch.cat([vals, Vt[n, h, :t].double()])
            if len(keys) == 0:
                continue
            s = scale * Q[n, x] @ keys.T.contiguous()
            mag = (abs(scale) * Q[n, x].abs() @ keys.abs().T.contiguous()).amax(-1)
            w = torch.softmax(s, -1)
            O[n, x], lse[n, x] = w @ vals, torch.logsumexp(s, -1)
            A = w @ vals.abs()
            es = ((2 * d + 4) * mag + 4) * 2.0 ** -24
            sums = (len(keys) + 8) * 2.0 ** -24
            tol[n, x] = A * (2 * es + 2 * sums + (half if dtype == torch.bfloat16 else 0)
                             )[:, None] + half * 1.01 * O[n, x].abs()
            ltol[n, x] = es + sums + 2.0 ** -22 * (1 + lse[n, x].abs())
    return O, lse, tol, ltol
