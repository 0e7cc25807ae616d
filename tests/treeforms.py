"""Shapes that take each form of the attention over a cache in pages: its kernel of few
query rows (16 or 32 a workgroup), and that of many (64, 128 or 256 a workgroup), with one
range of the keys or several."""
from __future__ import annotations

import itertools

FORMATS = [(t, f) for t in ("bf16", "f32") for f in (None, "e4m3", "e2m1")]


def forms(dtype):
    """(kernel, query rows of a workgroup)"""
    few = [16, 32] if dtype == "bf16" else [16]
    return [("few", n) for n in few] + [("many", n)
                                        for n in ([64, 128, 256] if dtype == "bf16" else [64, 128])]


ALL = [(t, f, d, kernel, n, ranges) for t, f in FORMATS for d in (64, 128)
       for kernel, n in forms(t) for ranges in (False, True)]


def form_of(s):
    few = s.key_waves == 4 and s.group_rows == s.wave_rows
    return "few" if few else "many", s.group_rows, s.ranges > 1


def find(wf, dtype, fmt, d, kernel, block, ranges):
    """Parameters of the first shape of this form: room for one sequence of `rows` new rows
    behind 200 others at least (with several ranges, behind one of them), among `batch`."""
    want = (kernel, block, ranges)
    for most, b, h, g, rows in itertools.product((500, 1100, 2000, 8000, 16000, 60000),
                                                 (1, 4, 16, 64), (1, 2, 8), (1, 2, 3, 8),
                                                 (1, 17, 33, 64, 100, 200, 256)):
        if rows + 240 > most or b * h * g * rows > 400000:
            continue
        kw = dict(page_rows=16, heads=h, head_dim=d, batch=b, max_rows=rows, tokens=rows, group=g,
                  table_pages=-(-most // 16), max_len=most, dtype=dtype, format=fmt)
        s = wf.tree_plan(wf.make_tree_params(pages=1, **kw))
        length = min(most, rows + (s.range_rows + 37 if ranges else 470))
        if (form_of(s) == want and rows + 240 <= length <= 6000
                and (length > s.range_rows) == ranges):
            return dict(kw, length=length)
    raise AssertionError(f"no shape of the form {(dtype, fmt, d) + want}")
