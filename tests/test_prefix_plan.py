"""wf_prefix_plan: the split that a workspace of a size gives (host arithmetic,
no GPU needed)."""
import ctypes
import random

import pytest

import paper_2606_00724_amd as wf


def _p(**kw):
    return wf.make_prefix_params(**{**dict(share=8, heads=8, group=4, q_len=1, head_dim=128,
                                           prefix_cap=4096, tail_cap=64), **kw})


def _tuple(s):
    return tuple(getattr(s, n) for n, _ in s._fields_)


def test_refusals():
    lib, s = wf.library(), wf.WfPrefixSplit()
    assert lib.wf_prefix_plan(None, 0, ctypes.byref(s)) == 1
    assert lib.wf_prefix_plan(ctypes.byref(_p()), 0, None) == 1
    assert lib.wf_prefix_plan(ctypes.byref(_p(head_dim=80)), 0, ctypes.byref(s)) == 2
    with pytest.raises(wf.WfError):
        wf.prefix_plan(_p(share=0))
    assert _tuple(wf.prefix_plan(_p(prefix_rows=0))) == (0,) * 5


def test_splits_over_the_range():
    """The asked size gives the split of any larger one; with less the ranges
    fit it, one at least, and cover the prefix."""
    rng = random.Random(3)
    for _ in range(300):
        p = _p(share=rng.choice([1, 3, 32, 100]), heads=rng.choice([1, 3, 8, 32]),
               group=rng.choice([1, 4, 7]), q_len=rng.choice([1, 5, 32]),
               head_dim=rng.choice([64, 128]), prefix_cap=int(2 ** rng.uniform(0, 18)),
               tail_cap=rng.choice([0, 1, 100]), dtype=rng.choice(["bf16", "f32"]),
               format=rng.choice([None, "e4m3", "e2m1"]))
        rows = p.share * p.heads * p.group * p.q_len
        nb, one = wf.prefix_workspace_bytes(p), rows * (p.head_dim + 2) * 4
        s = wf.prefix_plan(p)
        assert _tuple(s) == _tuple(wf.prefix_plan(p, 1 << 60))
        assert nb == (0 if s.ranges == 1 and p.tail_cap == 0 else s.ranges * one)
        for k in (0, 1, 2, rng.randint(1, max(1, s.ranges))):
            s = wf.prefix_plan(p, k * one)
            assert 1 <= s.ranges <= max(k, 1)
            assert s.ranges * s.range_rows >= p.prefix_rows > (s.ranges - 1) * s.range_rows
            assert s.range_rows % 64 == 0 and s.wave_rows in (32, 64)
            assert s.group_rows * s.key_waves in (4 * s.wave_rows, 8 * s.wave_rows)
