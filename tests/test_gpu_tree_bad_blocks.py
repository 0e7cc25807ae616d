"""wf_tree_attn over rows that were stored with a NaN or an infinity: their blocks of V
have the byte 255, which makes these 32 channels NaN for the query rows that see them,
wherever in the context they stand, and costs no more there than other blocks."""
from __future__ import annotations

import pytest
import torch

from test_gpu_tree import Case, wf  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

CODES = [(t, f) for t in ("bf16", "f32") for f in ("e4m3", "e2m1")]


def stored_odd(c, b, t, channel):
    """Row t of sequence b as it is stored with a NaN at this channel of V."""
    page, r, g = int(c.table[b, t // c.p.page_rows]), t % c.p.page_rows, channel // 32
    n = 32 if c.fmt == "e4m3" else 16
    c.pool[2][page, :, r, n * g:n * (g + 1)] = 0
    c.pool[3][page, :, r, g] = 255


@pytest.mark.parametrize("dtype,fmt", CODES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,group,mask", [(1, 4, "none"), (12, 2, "tree"), (16, 1, "causal"),
                                             (150, 1, "causal")])
def test_blocks_without_numbers(wf, dtype, fmt, d, rows, group, mask):  # noqa: F811
    """In the context, at either side of the first block that hides keys from some rows,
    among the new rows, and in several of these at once; other channels and sequences
    keep their values."""
    L = 900 + rows                        # (base 900: blocks of 32 hide keys from 896 on)
    for odd in ([(100, 5)], [(895, 40)], [(896, 5)], [(L - 1, 63)],
                [(0, 40), (511, 33), (L - 1, 3)]):
        c = Case(wf, lens=[L, L - 50, 70 + rows], rows=rows, heads=2, group=group, d=d,
                 dtype=dtype, fmt=fmt, mask=mask)
        for t, channel in odd:
            stored_odd(c, 0, t, channel)
        stored_odd(c, 1, 300, d - 1)
        if fmt == "e4m3":                 # codes of NaN beside them
            page = int(c.table[0, 300 // 16])
            c.pool[2][page, :, 300 % 16, d - 7] = 0x7f
        for ws in ("own", None):
            O, lse = c.run(wf, ws=ws)
            c.check((O, lse))
            assert lse.isfinite().all() and O.isnan().any() and not O.isnan().all()


def least_us(wf, c):  # noqa: F811
    dev = [t.cuda() for t in c.pool]
    up = [c.table.cuda(), c.len.cuda()]
    Q, O = c.Q.cuda(), torch.empty_like(c.Q, device="cuda")
    times = []
    for _ in range(8):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        wf.wf_tree_attn(c.p, Q, *dev, *up, None, None, O, None, None)
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 1e3)
    return min(times), O


@pytest.mark.parametrize("dtype,fmt", CODES)
def test_an_old_one_costs_nothing(wf, dtype, fmt):  # noqa: F811
    """One range of 32K keys: a search for the bad values key by key takes tens of times
    as long as the call (200 to 500 us): a chain of round trips to memory for each key."""
    c = Case(wf, lens=[32768], rows=1, heads=1, group=4, mask="none", P=64, dtype=dtype, fmt=fmt)
    assert wf.tree_plan(c.p, 0).group_rows == 16
    good, O = least_us(wf, c)
    assert O.isfinite().all()
    stored_odd(c, 0, 100, 40)
    bad, O = least_us(wf, c)
    assert O[..., 32:].isnan().all() and O[..., :32].isfinite().all()
    assert bad < 3 * good, f"{good:.0f} us, and {bad:.0f} with a bad block"
