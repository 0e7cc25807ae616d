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


# ------------------------------------------------------------ attention

def cached_rows(pool, table, b, head, L, page_rows, fmt):
    """K and V rows 0 .. L - 1 of a sequence's head in float64."""
    pages = pool[0].shape[0]
    out = []
    if L == 0:
        return [torch.zeros((0, 1), dtype=torch.float64)] * 2
    for c, x in ((pool[0], pool[1]), (pool[2], pool[3])):
        at = table[b, :-(-L // page_rows)].long().clamp(0, pages - 1)
        rows = c[at, head].flatten(0, 1)[:L]
        if fmt is not None:
            rows = cacheref.values(rows, x[at, head].flatten(0, 1)[:L], fmt)
        out.append(rows.double())
    return out


def sees(i, n, L, mask=None, causal=False):
    """Which of L rows query row i of n sees; mask: its words."""
    t = torch.arange(L)
    j = t - (L - n)
    if mask is not None:
        word = mask.long()[(j.clamp(min=0) // 32).clamp(max=len(mask) - 1)] & 0xffffffff
        new = (word >> (j.clamp(min=0) % 32)) & 1 == 1
    else:
        new = j <= i if causal else torch.ones(L, dtype=torch.bool)
    return (j < 0) | new


def tree_attention(Q, pool, table, length, start, mask, *, page_rows, heads, group, max_rows,
                   max_len, scale, causal=False, fmt=None):
    """O, lse in float64 and how far the kernel may be off, elementwise (as in
    cacheref.prefix_attention, whose tolerances are derived there), for the
    tokens of a sequence; the others keep NaN.  A row's hidden keys take no
    part, whatever they hold.  One more term: a weight below 2^-126 of the
    largest one, or a product of it below 2^-126, may be taken as 0 (the fp32
    range; the largest weight is 1 at least), which moves an output by up to
    2^-126 (1 + max |v|) for each of n keys."""
    tokens, hq, d = Q.shape
    bf = Q.dtype == torch.bfloat16
    half = 2.0 ** -8 if bf else 2.0 ** -24
    O = torch.full((tokens, hq, d), float("nan"), dtype=torch.float64)
    lse = torch.full((tokens, hq), float("nan"), dtype=torch.float64)
    tol, ltol = torch.zeros_like(O), torch.zeros_like(lse)
    for b in range(len(length)):
        L = min(max(int(length[b]), 0), max_len)
        first = b * max_rows if start is None else int(start[b])
        n = max_rows if start is None else min(max(int(start[b + 1]) - first, 0), max_rows)
        for h in range(heads):
            K, V = cached_rows(pool, table, b, h, L, page_rows, fmt)
            for i in range(n):
                at = first + i
                if not 0 <= at < tokens:
                    continue
                s = sees(i, n, L, None if mask is None else mask[at], causal)
                k, v = K[s], V[s]
                x = slice(h * group, (h + 1) * group)
                if len(k) == 0:
                    O[at, x], lse[at, x] = 0.0, -np.inf
                    continue
                q = Q[at, x].double()
                sc = scale * q @ k.T.contiguous()
                mag = (abs(scale) * q.abs() @ k.abs().T.contiguous()).amax(-1)
                w = torch.softmax(sc, -1)
                O[at, x], lse[at, x] = w @ v, torch.logsumexp(sc, -1)
                A = w @ v.abs()
                es = ((2 * d + 4) * mag + 4) * 2.0 ** -24
                sums = (len(k) + 8) * 2.0 ** -24
                tol[at, x] = A * (2 * es + 2 * sums + (half if bf else 0))[:, None] \
                    + half * 1.01 * O[at, x].abs() \
                    + len(k) * 2.0 ** -126 * (1 + v.abs().amax(0))
                ltol[at, x] = es + sums + 2.0 ** -22 * (1 + lse[at, x].abs())
    return O, lse, tol, ltol


def ancestors(n, seed):
    """Masks [n, words] of a random tree: a row sees itself and its ancestors."""
    g = torch.Generator().manual_seed(seed)
    seen = torch.zeros((n, -(-n // 32) * 32), dtype=torch.bool)
    for i in range(n):
        if i:
            seen[i] = seen[int(torch.randint(0, i, (1,), generator=g))]
        seen[i, i] = True
    return words(seen)


def words(seen):
    w = (seen.unflatten(-1, (-1, 32)).long() << torch.arange(32)).sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).int()
