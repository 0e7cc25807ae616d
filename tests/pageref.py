"""CPU reference of rotary positions and of a cache in pages, from their
definitions in include/wavefilter.h."""
from __future__ import annotations

import numpy as np
import torch

import cacheref


def frequencies(half: int, base: float = 10000.0) -> torch.Tensor:
    return (base ** (-torch.arange(half, dtype=torch.float64) / half)).float()


def turn(pos, freq, axis, factor=1.0):
    """Cosines and sines [..., pairs], 64-bit angles rounded once to fp32; pos
    [axes, ...], axis: that of each pair."""
    t = np.moveaxis(pos.numpy().astype(np.float64), 0, -1)[..., list(axis)]
    th = t * freq.numpy().astype(np.float64)
    f = float(np.float32(factor))
    return (np.cos(th) * f).astype(np.float32), (np.sin(th) * f).astype(np.float32)


def rotate(x, c, s, layout="halves", exact=False):
    """Rows x [..., d] with their first 2 len(pairs) channels rotated, as fp32
    numbers (each product and sum rounded by itself), or in 64 bits."""
    y = x.double().numpy() if exact else x.float().numpy()
    if exact:
        c, s = c.astype(np.float64), s.astype(np.float64)
    r = 2 * c.shape[-1]
    y = y.copy()
    a, b = ((y[..., 0:r:2], y[..., 1:r:2]) if layout == "pairs"
            else (y[..., :r // 2], y[..., r // 2:r]))
    u, v = a * c - b * s, b * c + a * s
    if layout == "pairs":
        y[..., 0:r:2], y[..., 1:r:2] = u, v
    else:
        y[..., :r // 2], y[..., r // 2:r] = u, v
    return torch.from_numpy(y)


def pool_like(wf, p, seed=7):
    """A pool of rows that were there before."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for t in wf.alloc_pages(p, "cpu"):
        if t is None:
            out.append(None)
        elif t.dtype == torch.uint8:
            out.append(torch.randint(0, 256, t.shape, generator=g, dtype=torch.uint8) & 0xf7)
        else:
            out.append(torch.randn(t.shape, generator=g).to(t.dtype))
    return out


def append(pool, fmt, dtype, K, V, slot, page_rows):
    """The pool with fp32 rows K, V [tokens, heads, d] written at their slots."""
    out = [None if t is None else t.clone() for t in pool]
    rows = pool[0].shape[0] * page_rows
    new = []
    for x in (K, V):
        if fmt is None:
            new += [x.to(dtype), None]
        else:
            code, byte = cacheref.quantise(x, fmt)
            new += [cacheref.pack(code, fmt), byte]
    for n, at in enumerate(slot.tolist()):
        if 0 <= at < rows:
            for o, x in zip(out, new):
                if o is not None:
                    o[at // page_rows, :, at % page_rows] = x[n]
    return out


def move(pool, table, first, source, page_rows):
    """The pool with rows moved: all are read before one is written."""
    out = [None if t is None else t.clone() for t in pool]
    pages, tp = pool[0].shape[0], table.shape[1]

    def place(b, t):
        if not 0 <= t < tp * page_rows:
            return None
        page = int(table[b, t // page_rows])
        return (page, t % page_rows) if 0 <= page < pages else None

    for b in range(table.shape[0]):
        for i, s in enumerate(source[b].tolist()):
            to, of = place(b, int(first[b]) + i), place(b, int(first[b]) + s)
            if s < 0 or to is None or of is None:
                continue
            for o, x in zip(out, pool):
                if o is not None:
                    o[to[0], :, to[1]] = x[of[0], :, of[1]]
    return out
