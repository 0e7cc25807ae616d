"""wf_page_move with one to four 16-byte pieces of rows a thread (a kernel each), with and
without exponent bytes, rows in one column of workgroups and in several."""
from __future__ import annotations

import pytest
import torch

import pageref
from test_gpu_page import same, wf  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def split(d, fmt, moves):
    """(16-byte pieces of a row in a workgroup, pieces of a thread of 256)"""
    pieces = {None: 2 * d, "e4m3": d, "e2m1": d // 2}[fmt] // 16
    while pieces * moves > 1024:
        pieces //= 2
    return pieces, -(-pieces * moves // 256)


@pytest.mark.parametrize("fmt,d,moves,pieces", [
    (None, 128, 16, 1), (None, 128, 31, 2), (None, 64, 65, 3), (None, 128, 40, 3),
    (None, 64, 101, 4), (None, 64, 200, 4), ("e4m3", 128, 32, 1), ("e4m3", 128, 64, 2),
    ("e4m3", 128, 96, 3), ("e4m3", 128, 129, 3), ("e4m3", 64, 64, 1), ("e4m3", 64, 127, 2),
    ("e4m3", 64, 190, 3), ("e4m3", 64, 256, 4), ("e2m1", 128, 64, 1), ("e2m1", 128, 100, 2),
    ("e2m1", 128, 191, 3), ("e2m1", 128, 193, 4), ("e2m1", 64, 128, 1), ("e2m1", 64, 255, 2),
])
def test_move(wf, fmt, d, moves, pieces):  # noqa: F811
    assert split(d, fmt, moves)[1] == pieces
    b, h, P, tp = 3, 2, 16, 40
    pages = b * tp + 2
    p = wf.make_move_params(pages=pages, page_rows=P, heads=h, head_dim=d, batch=b,
                            table_pages=tp, moves=moves, format=fmt)
    pool = pageref.pool_like(wf, p)
    g = torch.Generator().manual_seed(moves)
    table = torch.randperm(pages, generator=g)[:b * tp].view(b, tp).int()
    first = torch.tensor([3, 100, tp * P - moves // 2]).int()   # (rows past the table's end)
    source = torch.randint(-1, 2 * moves, (b, moves), generator=g).int()
    source[0] = torch.arange(moves).flip(0).int()               # each row read and written
    source[1] = torch.randperm(moves, generator=g).int()
    want = pageref.move(pool, table, first, source, P)
    dev = [None if t is None else t.cuda() for t in pool]
    wf.wf_page_move(p, table.cuda(), first.cuda(), source.cuda(), *dev)
    for name, x, y in zip(("Kc", "Kx", "Vc", "Vx"), dev, want):
        if y is not None:
            same(name, x, y)
