"""Blocks that wf_page_append keeps in 8 or 4 bits and that are no ordinary ones, bit by bit:
NaN and infinities, zeros of both signs, subnormals, the largest finite numbers (whose
rotation may overflow), and these beside ordinary channels."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import pageref
from test_gpu_page import DT, append_case, same, wf  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

HEADS = 2


def rows_with(kind, x, dtype):
    """Rows x [tokens, heads, d] with what is odd in channels of each block of 32: one of
    them (another from row to row), some, or all."""
    info, (n, h, d) = torch.finfo(DT[dtype]), x.shape
    y = x.clone().unflatten(-1, (-1, 32))                     # [n, h, blocks, 32]
    i = torch.arange(n * h * (d // 32)).view(n, h, d // 32)
    one = torch.nn.functional.one_hot(i * 7 % 32, 32).bool() & (i % 3 != 2)[..., None]
    alternate = torch.where(i[..., None] % 2 == 0, 1.0, -1.0).to(y.dtype)
    if kind == "nan":
        y[one] = float("nan")
    elif kind == "inf":
        y = torch.where(one, alternate * float("inf"), y)
    elif kind == "zeros":
        y = torch.where(i[..., None] % 2 == 0, torch.zeros_like(y), torch.copysign(y * 0, y))
    elif kind == "small":       # multiples of the least subnormal, and its block's first normal
        least = info.smallest_normal * info.eps
        y = (torch.round(y.float() * 8) * least).to(y.dtype)
        y[one] = info.smallest_normal
    elif kind == "largest":
        y = torch.where(one, alternate * info.max, y)
    elif kind == "all largest":
        y = torch.copysign(torch.full_like(y, info.max), y)
    return y.flatten(-2)


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot,layout", [(64, 48, "halves"), (128, 48, "halves"), (128, 128, "halves"),
                                          (64, 32, "pairs"), (64, 0, "halves")])
@pytest.mark.parametrize("kind", ["nan", "inf", "zeros", "small", "largest", "all largest"])
def test_append(wf, fmt, dtype, d, rot, layout, kind):  # noqa: F811
    """With 48 channels in halves the eights of a block are those of several threads."""
    P, tokens = 16, 21
    p, (q, k, v), pos, freq, slot, pool, _, _ = append_case(
        wf, tokens=tokens, heads=HEADS, group=1, d=d, P=P, fmt=fmt, dtype=dtype, rot=rot,
        layout=layout)
    K, V = (rows_with(kind, x.cpu(), dtype) for x in (k, v))
    turned = K
    if rot:
        c, s = pageref.turn(pos, freq, [0] * (rot // 2))
        with np.errstate(all="ignore"):
            turned = pageref.rotate(K, c[:, None], s[:, None], layout)
    want = pageref.append(pool, fmt, DT[dtype], turned.float(), V.float(), slot, P)
    dev = [t.cuda() for t in pool]
    wf.wf_page_append(p, q, K.cuda(), V.cuda(), *((pos.cuda(), freq.cuda()) if rot else (None, None)),
                      slot.cuda(), *dev, torch.empty_like(q))
    for name, x, y in zip(("Kc", "Kx", "Vc", "Vx"), dev, want):
        same(name, x, y)
    kept = [at for at in slot.tolist() if 0 <= at < p.pages * P]
    vx = torch.stack([want[3][at // P, :, at % P] for at in kept])
    assert len(kept) > 10
    if kind in ("nan", "inf"):
        assert (vx == 255).any() and (vx != 255).any()
    elif kind in ("zeros", "small"):
        assert (vx == 1).all()
    else:
        # the least 2^e with 2^128 <= 448 2^e (e = 120), 2^128 <= 6 2^e (e = 126)
        top = 127 + (120 if fmt == "e4m3" else 126)
        assert (vx == top).any() and (vx <= top).all()
