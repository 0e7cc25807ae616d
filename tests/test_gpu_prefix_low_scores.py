"""wf_prefix_attn where a row's first scores are far below the others, as where
keys hold the type's lowest value: their weights are 0 and the other scores keep
their differences.  Against the 64-bit reference of the keys behind them."""
from __future__ import annotations

import math

import pytest
import torch

import cacheref
from test_gpu_prefix import ARGS, make, wf  # noqa: F401 (a fixture)
from test_gpu_prefix_forms import LONG, NAMES, expect, shape

pytestmark = pytest.mark.gpu

LOWEST = float(torch.finfo(torch.bfloat16).min)
# the type's lowest value, and one that the formats keep as it is
VALUES = [LOWEST, -1.5 * 2.0 ** 127]


def compare(wf, p, c, cut):  # noqa: F811
    """c's call against the reference without the first `cut` keys of the
    prefix, or of the own rows where there is no prefix."""
    O, lse = wf.prefix_attend(p, **{k: None if c[k] is None else c[k].cuda() for k in ARGS},
                              want_lse=True)
    K, V, Kt, Vt = c.get("Kv"), c.get("Vv"), c["Kt"], c["Vt"]
    if p.prefix_rows:
        K, V = K[:, :, cut:], V[:, :, cut:]
    else:
        Kt, Vt = Kt[:, :, cut:], Vt[:, :, cut:]
    ref, rl, tol, ltol = cacheref.prefix_attention(
        c["Q"], K, V, prefixes=p.prefixes, share=p.share, heads=p.heads, group=p.group,
        scale=p.head_dim ** -0.5, rows=max(p.prefix_rows - cut, 0), Kt=Kt, Vt=Vt,
        dtype=c["Q"].dtype)
    off = (O.cpu().double() - ref).abs() - tol
    assert bool((off <= 0).all()), f"{int((off > 0).sum())} of {off.numel()}"
    assert bool(((lse.cpu().double() - rl).abs() <= ltol).all())


@pytest.mark.parametrize("low", [LOWEST, -1e7])
@pytest.mark.parametrize("dtype,fmt,rows,waves,M,P", LONG, ids=NAMES)
def test_prefix(wf, dtype, fmt, rows, waves, M, P, low):  # noqa: F811
    """The low keys end inside a block of 32 keys or between two; what they leave
    of a range has many blocks."""
    for cut in (300, 320) if M == 150 else (300,):
        p, c = make(wf, **shape(M, dtype=dtype, fmt=fmt, d=64, prefixes=2, heads=24, P=P, T=3))
        expect(wf, p, rows, waves)
        K = c["Kv"].float().clone()
        K[..., 0] = 0.0
        K[:, :, :cut, 0] = low
        c["Q"][..., 0] = 1.0
        c["Kt"][..., 0] = 0.0
        if fmt:
            code, byte = cacheref.quantise(K, fmt)
            c["K"], c["Kx"] = cacheref.pack(code, fmt), byte
            c["Kv"] = cacheref.values(c["K"], byte, fmt)
        else:
            c["K"] = c["Kv"] = K.to(c["Q"].dtype)
        compare(wf, p, c, cut)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("low", [LOWEST, -1e7])
@pytest.mark.parametrize("d", [64, 128])
def test_own_rows(wf, dtype, low, d):  # noqa: F811
    p, c = make(wf, dtype=dtype, P=0, T=300, share=3, heads=2, B=20, d=d)
    c["Kt"][..., 0] = 0.0
    c["Kt"][:, :, :103, 0] = low
    c["Q"][..., 0] = 1.0
    compare(wf, p, c, 103)


def set_channel(c, fmt, at, value):
    """Channel 0 of the prefix's rows `at` is `value`, of the others 0."""
    K = c["Kv"].float().clone()
    K[..., 0] = 0.0
    K[:, :, at, 0] = value
    if fmt:
        code, byte = cacheref.quantise(K, fmt)
        c["K"], c["Kx"] = cacheref.pack(code, fmt), byte
        c["Kv"] = cacheref.values(c["K"], byte, fmt)
    else:
        c["K"] = c["Kv"] = K.to(c["Q"].dtype)
    c["Q"][..., 0] = 1.0
    c["Kt"][..., 0] = 0.0


def alike(wf, p, c, at):  # noqa: F811
    """Of the prefix's rows `at`, whose scores are equal and above all others,
    each has the same weight: sums of n values, none of whose weights is
    rounded, and an output rounded once."""
    O, lse = wf.prefix_attend(p, **{k: None if c[k] is None else c[k].cuda() for k in ARGS},
                              want_lse=True)
    scale = p.scale or p.head_dim ** -0.5
    key = float(c["Kv"][0, 0, at, 0][0])
    if abs(key) > torch.finfo(torch.float32).max:
        # codes whose value, 2^128, is infinite in fp32: no weight, or the rows NaN
        if scale * key < 0:
            assert not bool(O.any()) and bool((lse == -math.inf).all())
        else:
            assert bool(O.isnan().all()) and bool(lse.isnan().all())
        return
    V = c["Vv"].double()[:, :, at]
    n = V.shape[2]
    own = lambda x: x.mean(2).view(p.prefixes, 1, p.heads, 1, 1, p.head_dim).expand(  # noqa: E731
        p.prefixes, p.share, p.heads, p.group, p.q_len, p.head_dim).reshape(O.shape)
    ref, A = own(V), own(V.abs())
    half = 2.0 ** -8 if O.dtype == torch.bfloat16 else 2.0 ** -24
    tol = 2 * (n + 8) * 2.0 ** -24 * A + 1.01 * half * ref.abs()
    assert bool(((O.cpu().double() - ref).abs() <= tol).all())
    want = scale * key  # (log n is nothing beside it)
    assert bool(((lse.cpu().double() - want).abs() <= 2.0 ** -21 * abs(want)).all())


@pytest.mark.parametrize("value,sign", [(VALUES[0], 1), (VALUES[1], 1), (VALUES[1], -1)])
@pytest.mark.parametrize("dtype,fmt,rows,waves,M,P", LONG, ids=NAMES)
def test_the_highest_scores(wf, dtype, fmt, rows, waves, M, P, value, sign):  # noqa: F811
    """Rows of a prefix with a largest value, behind ordinary ones; with a
    negative scale, a lowest."""
    p, c = make(wf, **shape(M, dtype=dtype, fmt=fmt, d=64, prefixes=2, heads=24, P=P, T=3,
                            scale=0.125 * sign))
    expect(wf, p, rows, waves)
    at = torch.arange(100, P, 41)
    set_channel(c, fmt, at, -value * sign)
    alike(wf, p, c, at)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("scale", [0.125, 0.17])
@pytest.mark.parametrize("value", VALUES)
@pytest.mark.parametrize("dtype,fmt", [("bf16", None), ("bf16", "e2m1"), ("f32", "e4m3")])
def test_rows_that_see_the_lowest_only(wf, dtype, fmt, value, scale, sign):  # noqa: F811
    """All keys hold a lowest value (by a negative scale, a largest): their
    scores are equal."""
    p, c = make(wf, **shape(150, dtype=dtype, fmt=fmt, d=64, prefixes=2, heads=24, P=3000, T=3,
                            scale=scale * sign, tlen=[0] * 4))
    set_channel(c, fmt, torch.arange(3000), value * sign)
    alike(wf, p, c, torch.arange(3000))
