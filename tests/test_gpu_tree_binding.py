"""tree_attend: what it allocates fits the parameters, whatever their strides."""
from __future__ import annotations

import pytest
import torch

from test_gpu_tree import Case, wf  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,counts,rows", [([100, 60], None, 5), ([40], None, 1),
                                              ([90, 80], [3, 5], 5)])
def test_outputs_of_a_row_stride(wf, dtype, lens, counts, rows):  # noqa: F811
    c = Case(wf, lens=lens, counts=counts, rows=rows, group=2, dtype=dtype, spare=2 if counts else 0)
    base = c.run(wf)
    up = [t if t is None else t.cuda() for t in (c.table, c.len, c.start, c.mask)]
    pool = [t if t is None else t.cuda() for t in c.pool]
    tok, hq, d = c.Q.shape
    for o_row in (0, hq * d, hq * d + 64):
        c.p.o_row = o_row
        O, lse = wf.tree_attend(c.p, c.Q.cuda(), pool, *up, want_lse=True)
        assert O.shape == c.Q.shape and O.dtype == c.Q.dtype
        assert tok == 1 or O.stride(0) == (o_row or hq * d)
        used = (base[1] != 7).all(-1)           # (tokens of no sequence: 0 and -inf)
        assert torch.equal(O.cpu()[used], base[0][used])
        assert torch.equal(lse.cpu()[used], base[1][used])
        assert not O.cpu()[~used].any() and (lse.cpu()[~used] == float("-inf")).all()
    c.p.o_row = hq * d - 64                     # (refused)
    with pytest.raises((ValueError, wf.WfError)):
        wf.tree_attend(c.p, c.Q.cuda(), pool, *up)
