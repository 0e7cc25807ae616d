"""wf_prefix_attn decodes a cache with instructions of its own: every code at
every exponent byte, by calls whose one key has weight 1, against wf_cache_load,
whose values are tested bit by bit.  Blocks that were not finite read NaN."""
from __future__ import annotations

import pytest
import torch

from test_gpu_prefix import wf  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def every_code(fmt, d, last):
    """Packed codes [n, 1, 1, ..] and exponent bytes: all finite codes of a format
    at the bytes 1 .. last, n rows of d channels."""
    codes = torch.arange(256 if fmt == "e4m3" else 16, dtype=torch.int64)
    codes = codes[(codes & 0x7f) != 0x7f] if fmt == "e4m3" else codes
    blocks = codes.repeat(-(-len(codes) // 32) * 32)[: -(-len(codes) // 32) * 32].view(-1, 32)
    byte = torch.arange(1, last + 1).repeat_interleave(len(blocks))
    blocks = blocks.repeat(last, 1)
    # rotated from block to block: every code at each place of a word
    at = (torch.arange(32) + byte.unsqueeze(1)) % 32
    blocks = blocks.gather(1, at)
    pad = -len(blocks) % (d // 32)
    blocks = torch.cat([blocks, blocks[:pad]]).view(-1, 1, 1, d)
    byte = torch.cat([byte, byte[:pad]]).view(-1, 1, 1, d // 32)
    if fmt == "e2m1":
        blocks = blocks[..., 0::2] | (blocks[..., 1::2] << 4)
    return blocks.to(torch.uint8).cuda(), byte.to(torch.uint8).cuda()


def params(wf, n, d, dtype, fmt, **kw):  # noqa: F811
    return (wf.make_prefix_params(prefixes=n, share=1, heads=1, head_dim=d, prefix_cap=1,
                                  dtype=dtype, format=fmt, **kw),
            wf.make_cache_params(batch=n, heads=1, capacity=1, head_dim=d, rows=1, dtype=dtype,
                                 format=fmt))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_values(wf, dtype, fmt, d):  # noqa: F811
    V, Vx = every_code(fmt, d, 254)
    n = len(V)
    p, pc = params(wf, n, d, dtype, fmt, q_len=3)
    K, Kx = torch.zeros_like(V), torch.ones_like(Vx)
    Q = torch.randn((n, 1, 3, d), device="cuda").to(DT[dtype])
    want = wf.cache_load(pc, (K, Kx, V, Vx))[1]
    O = wf.prefix_attend(p, Q, K, V, Kx=Kx, Vx=Vx)
    assert torch.equal(O, want.expand(n, 1, 3, d))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_keys(wf, dtype, fmt, d):  # noqa: F811
    """One key and d query rows, row c of which is 1 in channel c: the row's lse is
    the key's channel times the scale.  (The bytes above make some keys infinite.)"""
    K, Kx = every_code(fmt, d, 245 if fmt == "e4m3" else 252)
    n = len(K)
    p, pc = params(wf, n, d, dtype, fmt, q_len=d, scale=1 / 16)
    Q = torch.eye(d, device="cuda").to(DT[dtype]).expand(n, 1, d, d).contiguous()
    want = wf.cache_load(pc, (K, Kx, K, Kx))[0].double().view(n, 1, d) / 16
    _, lse = wf.prefix_attend(p, Q, K, torch.zeros_like(K), Kx=Kx, Vx=torch.ones_like(Kx),
                              want_lse=True)
    # log2(e) and ln 2, each product rounded; subnormals
    tol = 2.0 ** -21 * want.abs() + 2.0 ** -126
    assert bool(((lse.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_blocks_that_were_not_finite(wf, dtype, fmt, d):  # noqa: F811
    """A block of V with byte 255 makes its 32 channels NaN, one of K the rows."""
    g = torch.Generator().manual_seed(1)
    P, B = 200, 5
    pc = wf.make_cache_params(batch=1, heads=3, capacity=P, head_dim=d, rows=P, dtype=dtype,
                              format=fmt)
    K, V = (torch.randn((1, 3, P, d), generator=g).to(DT[dtype]) for _ in range(2))
    V[0, 1, 77, 40] = float("inf")
    K[0, 2, 150, 3] = float("nan")
    cache = wf.alloc_cache(pc, "cuda")
    wf.wf_cache_store(pc, K.cuda(), V.cuda(), None, *cache)
    p = wf.make_prefix_params(share=2, heads=3, q_len=B, head_dim=d, prefix_cap=P, dtype=dtype,
                              format=fmt)
    Q = torch.randn((2, 3, B, d), generator=g).to(DT[dtype]).cuda()
    O = wf.prefix_attend(p, Q, cache[0], cache[2], Kx=cache[1], Vx=cache[3])
    nan = torch.zeros((2, 3, B, d), dtype=torch.bool)
    nan[:, 1, :, 32:64] = True
    nan[:, 2] = True
    assert torch.equal(O.isnan().cpu(), nan)
