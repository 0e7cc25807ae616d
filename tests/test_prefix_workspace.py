"""One workspace for wf_prefix_attn while prompts and batches change: the size
of a call is enough for every call with a shorter prefix or fewer query rows.
No GPU: a call that passes its argument and workspace checks then fails at its
first launch (WF_ERR_HIP), so the pointers are never followed."""
import ctypes
import random

import pytest
import torch

PTR = ctypes.c_void_p(1 << 20)  # aligned, never read
WORKSPACE, HIP = 3, 4


@pytest.fixture(scope="module")
def wf():
    if torch.cuda.is_available():
        pytest.skip("the calls would be launched")
    import paper_2606_00724_amd as m
    return m


def _call(wf, p, nbytes):
    f = PTR
    x = f if p.format else None
    t = f if p.tail_cap else None
    return wf.library().wf_prefix_attn(ctypes.byref(p), f, f, x, f, x, f, None, t, t, None, f,
                                       None, f if nbytes else None, nbytes, None)


def _p(wf, **kw):
    return wf.make_prefix_params(**{**dict(share=8, heads=8, group=4, q_len=1, head_dim=128,
                                           prefix_cap=4096, tail_cap=64), **kw})


@pytest.mark.parametrize("kept,now", [
    (dict(prefix_rows=2304), dict(prefix_rows=2048)),
    (dict(share=15), dict(share=14)),
    (dict(share=32, tail_cap=0), dict(share=3, tail_cap=0, prefix_rows=700)),
    (dict(share=400, q_len=4, tail_cap=0), dict(q_len=4, tail_cap=0)),  # one range: no bytes
])
def test_shorter_calls(wf, kept, now):
    assert _call(wf, _p(wf, **now), wf.prefix_workspace_bytes(_p(wf, **kept))) == HIP


def test_shorter_calls_over_the_range(wf):
    rng = random.Random(11)
    larger = 0
    for _ in range(400):
        kw = dict(share=rng.choice([1, 3, 32, 100]), heads=rng.choice([1, 3, 8, 32]),
                  group=rng.choice([1, 4, 7]), q_len=rng.choice([1, 5, 32]),
                  head_dim=rng.choice([64, 128]), prefixes=rng.choice([1, 2, 5]),
                  prefix_cap=1 << 18, prefix_rows=int(2 ** rng.uniform(1, 18)),
                  tail_cap=rng.choice([0, 1, 100]), dtype=rng.choice(["bf16", "f32"]),
                  format=rng.choice([None, "e4m3", "e2m1"]))
        have = wf.prefix_workspace_bytes(_p(wf, **kw))
        for name in ("share", "group", "q_len", "prefix_rows", "prefixes", "heads"):
            less = _p(wf, **{**kw, name: rng.randint(1, kw[name])})
            larger += wf.prefix_workspace_bytes(less) > have
            assert _call(wf, less, have) == HIP, (kw, name)
    assert larger > 0  # (or no call above took fewer ranges than it would)


def test_less_than_a_range_is_refused(wf):
    for dtype in ("bf16", "f32"):
        p = _p(wf, dtype=dtype)
        one = 8 * 8 * 4 * (128 + 2) * 4  # the partials of one range
        assert wf.prefix_workspace_bytes(p) > one
        assert _call(wf, p, one) == HIP
        assert _call(wf, p, one - 256) == WORKSPACE
        assert _call(wf, p, 0) == WORKSPACE
        # without own rows one range needs none
        assert _call(wf, _p(wf, dtype=dtype, tail_cap=0), 0) == HIP
