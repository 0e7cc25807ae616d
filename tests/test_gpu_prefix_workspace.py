"""wf_prefix_attn with fewer bytes than it would take: fewer key ranges, down
to one, against the 64-bit reference with the tolerance that
cacheref.prefix_attention derives."""
from __future__ import annotations

import pytest
import torch

from test_gpu_prefix import ARGS, check, make, wf  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


class _With:
    """The library with a workspace of its own size given to every call."""

    def __init__(self, wf, nbytes):
        self.wf = wf
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None

    def prefix_attend(self, p, **kw):
        if self.ws is not None:
            self.ws.fill_(255)  # old contents do not matter
            return self.wf.prefix_attend(p, **kw, workspace=self.ws)
        O = torch.empty_like(kw["Q"])
        lse = torch.empty(O.shape[:-1], dtype=torch.float32, device=O.device)
        names = ("Q", "K", "Kx", "V", "Vx", "row_idx", "prefix_len", "Kt", "Vt", "tail_len")
        self.wf.wf_prefix_attn(p, *(kw[k] for k in names), O, lse, None)
        return O, lse


@pytest.mark.parametrize("dtype,fmt,n", [("bf16", None, 0), ("bf16", "e4m3", 0), ("f32", None, 0),
                                         ("bf16", "e2m1", 2900), ("f32", "e4m3", 2900)])
@pytest.mark.parametrize("T", [0, 37])
def test_fewer_ranges(wf, dtype, fmt, n, T):  # noqa: F811
    kw = dict(dtype=dtype, fmt=fmt, P=3000, n=n, T=T, share=2, heads=2, B=9, d=64, plen=[2777])
    p, c = make(wf, **kw)
    one = p.share * p.heads * p.q_len * (p.head_dim + 2) * 4
    ranges = wf.prefix_workspace_bytes(p) // one
    assert ranges > 4
    for k in (1 if T else 0, 2, 3, ranges - 1):
        check(_With(wf, k * one), p, c)
    # and more than it would take changes nothing
    dev = {k: None if c[k] is None else c[k].cuda() for k in ARGS}
    a = wf.prefix_attend(p, **dev)
    more = torch.empty((ranges + 3) * one, dtype=torch.uint8, device="cuda")
    assert torch.equal(a, wf.prefix_attend(p, **dev, workspace=more))
