"""Every form of the prefix kernel (query rows of a wave, waves over the keys of
a tile) against the 64-bit reference with the tolerance that
cacheref.prefix_attention derives: long ranges, lists, maxima that come late,
one range without own rows, more row ids than the LDS holds at once.  Each test
asserts the form that its shape is there for, as the library splits it on 256
CUs."""
from __future__ import annotations

import pytest
import torch

import cacheref
from test_gpu_prefix import check, make, wf  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

# M query rows a K/V head: share, group, q_len
ROWS = {20: (2, 1, 10), 100: (2, 2, 25), 150: (2, 3, 25)}
# (dtype, format), (query rows of a wave, waves over the keys), M, rows of a
# prefix: 48 units with several ranges of eight tiles of 64 keys or more
LONG = ([("bf16", None, 32, 2, 20, 3000), ("bf16", None, 32, 1, 100, 3000),
         ("bf16", None, 64, 1, 150, 3000)]
        + [("bf16", f, 32, kw, M, 2100) for f in ("e4m3", "e2m1")
           for kw, M in ((4, 20), (2, 100), (1, 150))]
        + [("f32", f, 32, kw, M, 3000) for f in (None, "e4m3", "e2m1")
           for kw, M in ((2, 20), (1, 100))])
NAMES = [f"{t}-{f}-{r}x{k}" for t, f, r, k, _, _ in LONG]


def shape(M, **kw):
    share, group, B = ROWS[M]
    return dict(share=share, group=group, B=B, **kw)


def expect(wf, p, rows, waves, *, ranges=None, at_least=512, nbytes=None):  # noqa: F811
    """The split's form; its ranges hold at_least keys."""
    s = wf.prefix_plan(p, nbytes)
    assert (s.wave_rows, s.key_waves) == (rows, waves), (s.wave_rows, s.key_waves)
    assert s.range_rows >= at_least
    assert s.ranges == ranges if ranges else s.ranges > 1


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("listed", [False, True], ids=["dense", "list"])
@pytest.mark.parametrize("dtype,fmt,rows,waves,M,P", LONG, ids=NAMES)
def test_long_ranges_in_every_form(wf, dtype, fmt, rows, waves, M, P, listed, d):  # noqa: F811
    """One prefix ends inside a tile, one inside a range."""
    p, c = make(wf, **shape(M, dtype=dtype, fmt=fmt, d=d, prefixes=2, heads=24, P=P,
                            n=P - 7 if listed else 0, T=3, plen=[P - 10, P * 7 // 10]))
    expect(wf, p, rows, waves)
    check(wf, p, c)


@pytest.mark.parametrize("dtype,fmt,rows,waves,M,P", LONG, ids=NAMES)
def test_late_maxima_in_every_form(wf, dtype, fmt, rows, waves, M, P, d=128):  # noqa: F811
    """Scores that rise along the keys, so that the reference of the softmax is
    raised in many blocks, by more in the second half of a unit's query rows,
    and a first block far below the others."""
    p, c = make(wf, **shape(M, dtype=dtype, fmt=fmt, d=d, prefixes=2, heads=24, P=P, T=3,
                            gain=0.05))
    expect(wf, p, rows, waves)
    K = c["Kv"].clone()
    ramp = torch.linspace(-60, 60, P)
    ramp[:32] = -300
    K[..., 0] = ramp.to(K.dtype)
    if fmt:
        code, byte = cacheref.quantise(K, fmt)
        c["K"], c["Kx"] = cacheref.pack(code, fmt), byte
        K = cacheref.values(c["K"], byte, fmt)
    else:
        c["K"] = K
    c["Kv"] = K
    c["Q"][..., 0] = torch.linspace(2, 6, p.q_len).to(c["Q"].dtype)
    check(wf, p, c)


@pytest.mark.parametrize("dtype,fmt,rows,waves,M,d", [
    ("bf16", None, 32, 2, 20, 128), ("bf16", None, 64, 1, 150, 64), ("bf16", None, 64, 1, 150, 128),
    ("bf16", "e4m3", 32, 1, 150, 128), ("bf16", "e2m1", 32, 1, 150, 64),
    ("f32", None, 32, 1, 100, 128), ("f32", "e4m3", 32, 1, 100, 64)])
def test_one_range_without_own_rows(wf, dtype, fmt, rows, waves, M, d):  # noqa: F811
    """The prefix kernel writes the outputs itself."""
    p, c = make(wf, **shape(M, dtype=dtype, fmt=fmt, d=d, prefixes=2, heads=96, P=700,
                            plen=[700, 641]))
    expect(wf, p, rows, waves, ranges=1)
    assert wf.prefix_workspace_bytes(p) == 0
    check(wf, p, c)


class OneRange:
    """The library with a workspace for one range."""

    def __init__(self, wf, nbytes):  # noqa: F811
        self.wf, self.nbytes = wf, nbytes

    def prefix_attend(self, p, **kw):
        ws = torch.empty(self.nbytes, dtype=torch.uint8, device="cuda")
        return self.wf.prefix_attend(p, **kw, workspace=ws)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,fmt,rows,waves,M,heads,n", [
    ("bf16", None, 32, 2, 20, 1, 13000), ("bf16", None, 32, 1, 100, 96, 4500),
    ("bf16", None, 64, 1, 150, 96, 4500),
    ("bf16", "e4m3", 32, 4, 20, 1, 13000), ("bf16", "e2m1", 32, 4, 20, 1, 13000),
    ("bf16", "e4m3", 32, 2, 100, 96, 4500), ("bf16", "e2m1", 32, 1, 150, 96, 4500),
    ("f32", None, 32, 2, 20, 1, 13000), ("f32", "e2m1", 32, 2, 20, 1, 13000),
    ("f32", None, 32, 1, 100, 96, 4500), ("f32", "e4m3", 32, 1, 100, 96, 4500)])
def test_more_ids_than_the_lds_holds(wf, dtype, fmt, rows, waves, M, heads, n, d):  # noqa: F811
    """The LDS has 4096 ids of a range's list at once: the others replace them
    while the range's tiles are in use."""
    p, c = make(wf, **shape(M, dtype=dtype, fmt=fmt, d=d, prefixes=2, heads=heads, P=500, n=n, T=3,
                            plen=[n, n - 150]))
    nbytes = 2 * heads * M * (d + 2) * 4
    expect(wf, p, rows, waves, ranges=1, at_least=4097, nbytes=nbytes)
    check(OneRange(wf, nbytes), p, c)
