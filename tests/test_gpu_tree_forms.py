"""Each form of wf_tree_attn's kernel of many query rows, as its plan says: a far lower part
of the context, a few far higher keys, and old rows without numbers."""
from __future__ import annotations

import math

import pytest
import torch

import cacheref
import treeforms
from test_gpu_tree import Case, wf  # noqa: F401 (a fixture)
from test_gpu_tree_bad_blocks import stored_odd

pytestmark = pytest.mark.gpu

MANY = [a for a in treeforms.ALL if a[3] == "many"]
LOWEST = float(torch.finfo(torch.bfloat16).min)
HIGH = 1.5 * 2.0 ** 127  # (the formats keep it)


def case(wf, form):  # noqa: F811
    kw = treeforms.find(wf, *form)
    L, rows, b = kw["length"], kw["max_rows"], kw["batch"]
    n = -(-L // 16)
    c = Case(wf, lens=[0] * (b - 1) + [L], counts=[0] * (b - 1) + [rows], rows=rows,
             heads=kw["heads"], group=kw["group"], d=kw["head_dim"], P=16, dtype=kw["dtype"],
             fmt=kw["format"], max_len=kw["max_len"], pool_pages=n + 1, mask="causal")
    c.table[b - 1, :n] = torch.randperm(n + 1, generator=torch.Generator().manual_seed(2))[:n].int()
    assert treeforms.form_of(wf.tree_plan(c.p)) == form[3:]
    return c, L, rows


def rows_of(c, L):
    """K and V [heads, L, d] of the last sequence, in 64 bits."""
    at, out = c.table[-1, :-(-L // 16)].long(), []
    for code, byte in ((c.pool[0], c.pool[1]), (c.pool[2], c.pool[3])):
        x = code[at].double() if c.fmt is None else cacheref.values(code[at], byte[at], c.fmt)
        out.append(x.double().transpose(0, 1).flatten(1, 2)[:, :L].contiguous())
    return out


def set_channel(c, at, value):
    """Channel 0 of the last sequence's rows `at` is `value`, of all others 0; 1 in Q."""
    K = (c.pool[0] if c.fmt is None else cacheref.values(c.pool[0], c.pool[1], c.fmt)).float()
    K[..., 0] = 0.0
    K[c.table[-1, at // 16].long(), :, at % 16, 0] = value
    if c.fmt:
        code, byte = cacheref.quantise(K, c.fmt)
        c.pool[0], c.pool[1] = cacheref.pack(code, c.fmt), byte
    else:
        c.pool[0] = K.to(c.Q.dtype)
    c.Q[..., 0] = 1.0


def check(c, got, L, cut=0):
    """Against 64 bits, over the keys from cut on; tolerances as in pageref."""
    n, g, d = c.p.max_rows, c.p.group, c.p.head_dim
    bf = c.Q.dtype == torch.bfloat16
    half = 2.0 ** -8 if bf else 2.0 ** -24
    t, i = torch.arange(L)[None], torch.arange(n).repeat_interleave(g)[:, None]
    sees = (t >= cut) & (t - (L - n) <= i)
    K, V = rows_of(c, L)
    for h in range(c.p.heads):
        O, lse = (x[:, h * g:(h + 1) * g].double().flatten(0, 1) for x in got)
        q = c.Q[:, h * g:(h + 1) * g].double().flatten(0, 1)
        s = (c.scale * q @ K[h].T.contiguous()).masked_fill(~sees, -math.inf)
        mag = (abs(c.scale) * q.abs() @ K[h].abs().T.contiguous()).masked_fill(~sees, 0).amax(-1)
        w, keys = torch.softmax(s, -1), sees.sum(-1)
        odd = V[h].isnan()                # (no part of rows that do not see them)
        v = V[h].masked_fill(odd, 0)
        want, A = w @ v, w @ v.abs()
        es = ((2 * d + 4) * mag + 4) * 2.0 ** -24
        sums = (keys + 8) * 2.0 ** -24
        top = v[cut:].abs().amax(0)
        tol = A * (2 * es + 2 * sums + (half if bf else 0))[:, None] + half * 1.01 * want.abs() \
            + keys[:, None] * 2.0 ** -126 * (1 + top)
        none = sees.double() @ odd.double() > 0
        assert torch.equal(O.isnan(), none)
        assert ((O - want).abs() <= tol)[~none].all()
        wl = torch.logsumexp(s, -1)
        assert ((lse - wl).abs() <= es + sums + 2.0 ** -22 * (1 + wl.abs())).all()


def alike(c, got, L, at):
    """Every row sees the rows `at`, whose scores are equal and above all others: sums of
    values whose weights are not rounded, and an output rounded once."""
    V, g, n = rows_of(c, L)[1], c.p.group, len(at)
    half = 2.0 ** -8 if c.Q.dtype == torch.bfloat16 else 2.0 ** -24
    O = got[0].double().unflatten(1, (c.p.heads, g))
    ref, A = (x[:, at].mean(1)[None, :, None] for x in (V, V.abs()))
    assert ((O - ref).abs() <= 2 * (n + 8) * 2.0 ** -24 * A + 1.01 * half * ref.abs()).all()
    want = c.scale * HIGH  # (log n is nothing beside it)
    assert ((got[1].double() - want).abs() <= 2.0 ** -21 * want).all()


@pytest.mark.parametrize("form", MANY, ids=str)
def test_behind_far_lower_ones(wf, form):  # noqa: F811
    """The low keys end inside a block of 32 keys, or between two."""
    for cut, low in ((112, LOWEST), (192, -1e7)):
        c, L, rows = case(wf, form)
        set_channel(c, torch.arange(cut), low)
        check(c, c.run(wf), L, cut)


@pytest.mark.parametrize("form", MANY, ids=str)
def test_the_highest_scores(wf, form):  # noqa: F811
    c, L, rows = case(wf, form)
    at = torch.arange(5, L - rows, 41)
    set_channel(c, at, HIGH)
    alike(c, c.run(wf), L, at)


@pytest.mark.parametrize("form", [a for a in MANY if a[1]], ids=str)
def test_blocks_without_numbers(wf, form):  # noqa: F811
    """In the context, beside the first tile that hides keys from some rows, and among the
    new rows; other channels keep their values."""
    c, L, rows = case(wf, form)
    last, d = c.p.batch - 1, c.p.head_dim
    for t, channel in ((70, 3), (L - rows - 1, 3), (L - 1, d - 1)):
        stored_odd(c, last, t, channel)
    if form[1] == "e4m3":                 # a code of NaN
        c.pool[2][int(c.table[last, 6]), :, 3, 40] = 0x7f
    O, lse = c.run(wf)
    check(c, (O, lse), L)
    assert O[..., :32].isnan().all() and not O[:rows - 1, :, d - 1].isnan().any()
