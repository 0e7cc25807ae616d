"""wf_tree_attn where a row's scores are far apart, or far from 0, as where keys hold
the type's lowest value: the far lower ones have no weight and the others keep their
differences, equal ones at any distance from 0 have equal weights."""
from __future__ import annotations

import math

import pytest
import torch

import cacheref
import pageref
from test_gpu_tree import FORMATS, Case, wf  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

LOWEST = float(torch.finfo(torch.bfloat16).min)
# the type's lowest value, and one that the formats keep as it is
VALUES = [LOWEST, -1.5 * 2.0 ** 127]
ROWS = [1, 12, 150]  # 16 and 32 query rows a workgroup, and the kernel of many


def case(wf, rows, dtype, fmt, d, scale=0.0):  # noqa: F811
    L = 2000 + rows
    return Case(wf, lens=[L, L], rows=rows, group=2, heads=1, d=d, dtype=dtype, fmt=fmt,
                mask="all", scale=scale)


def set_channel(c, at, value):
    """Channel 0 of the sequences' rows `at` is `value`, of all others 0; 1 in Q."""
    P = c.p.page_rows
    K = c.pool[0].float()
    if c.fmt:
        K = cacheref.values(c.pool[0], c.pool[1], c.fmt).float()
    K[..., 0] = 0.0
    for b in range(c.p.batch):
        K[c.table[b, at // P].long(), :, at % P, 0] = value
    if c.fmt:
        code, byte = cacheref.quantise(K, c.fmt)
        c.pool[0], c.pool[1] = cacheref.pack(code, c.fmt), byte
    else:
        c.pool[0] = K.to(c.Q.dtype)
    c.Q[..., 0] = 1.0


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("low", [LOWEST, -1e7])
def test_behind_far_lower_ones(wf, dtype, fmt, d, rows, low):  # noqa: F811
    """The low keys end inside a block of 32 keys or between two; the reference is of
    the keys behind them."""
    for cut in (304, 320):
        c = case(wf, rows, dtype, fmt, d)
        set_channel(c, torch.arange(cut), low)
        for ws in ("own", None):
            O, lse = c.run(wf, ws=ws)
            rO, rl, tol, ltol = pageref.tree_attention(
                c.Q, c.pool, c.table[:, cut // 16:].contiguous(), c.len - cut, None, None,
                page_rows=16, heads=1, group=2, max_rows=rows, max_len=c.p.max_len,
                scale=c.scale, fmt=fmt)
            assert ((O.double() - rO).abs() <= tol).all()
            assert ((lse.double() - rl).abs() <= ltol).all()


def alike(c, at, got):
    """Of the rows `at`, whose scores are equal and above all others, each has the same
    weight: sums of n values, none of whose weights is rounded, and an output rounded
    once."""
    O, lse = got
    P, d, n = c.p.page_rows, c.p.head_dim, len(at)
    K, V = c.pool[0].double(), c.pool[2].double()
    if c.fmt:
        K, V = (cacheref.values(c.pool[i], c.pool[i + 1], c.fmt).double() for i in (0, 2))
    key = float(K[int(c.table[0, int(at[0]) // P]), 0, int(at[0]) % P, 0])
    if abs(key) > torch.finfo(torch.float32).max:
        # codes whose value, 2^128, is infinite in fp32: no weight, or the rows NaN
        if c.scale * key < 0:
            assert not O.any() and (lse == -math.inf).all()
        else:
            assert O.isnan().all() and lse.isnan().all()
        return
    half = 2.0 ** -8 if O.dtype == torch.bfloat16 else 2.0 ** -24
    O, lse = (x.view(c.p.batch, c.p.max_rows, c.p.heads, c.p.group, -1).double() for x in (O, lse))
    for b in range(c.p.batch):
        v = V[c.table[b, at // P].long(), :, at % P]          # [n, heads, d]
        ref, A = v.mean(0)[None, :, None], v.abs().mean(0)[None, :, None]
        tol = 2 * (n + 8) * 2.0 ** -24 * A + 1.01 * half * ref.abs()
        assert ((O[b] - ref).abs() <= tol).all()
    want = c.scale * key  # (log n is nothing beside it)
    assert ((lse - want).abs() <= 2.0 ** -21 * abs(want)).all()


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("value,sign", [(VALUES[0], 1), (VALUES[1], 1), (VALUES[1], -1)])
def test_the_highest_scores(wf, dtype, fmt, rows, value, sign):  # noqa: F811
    """Rows with a largest value among ordinary ones; with a negative scale, a lowest."""
    c = case(wf, rows, dtype, fmt, 128, scale=0.125 * sign)
    at = torch.arange(100, 2000, 41)
    set_channel(c, at, -value * sign)
    alike(c, at, c.run(wf))


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("value", VALUES)
def test_rows_that_see_the_lowest_only(wf, dtype, fmt, rows, value):  # noqa: F811
    """All keys hold a lowest value (by a negative scale, a largest): their scores are
    equal."""
    for scale in (0.125, 0.17, -0.17):
        c = case(wf, rows, dtype, fmt, 64, scale=scale)
        at = torch.arange(2000 + rows)
        set_channel(c, at, value if scale > 0 else -value)
        alike(c, at, c.run(wf))
