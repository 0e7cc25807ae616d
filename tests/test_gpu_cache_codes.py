"""wf_cache_load of caches that hold every code: negative E2M1 codes on even
channels, E4M3 codes with an odd exponent field, at every place of a row."""
from __future__ import annotations

import pytest
import torch

import cacheref
from test_gpu_prefix import wf  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def any_cache(wf, p, fmt, seed=9):  # noqa: F811
    """Random code bytes, but for E4M3's NaN, and every exponent byte but those of
    infinite values."""
    g = torch.Generator().manual_seed(seed)
    cache = [torch.randint(0, 256, t.shape, generator=g, dtype=torch.uint8)
             for t in wf.alloc_cache(p, "cpu")]
    for m in (0, 2):
        if fmt == "e4m3":
            cache[m][(cache[m] & 0x7f) == 0x7f] ^= 1
        cache[m].view(-1)[:256] = torch.arange(256, dtype=torch.uint8) & (
            0xff if fmt == "e2m1" else 0xfe)
    for m in (1, 3):
        cache[m] = 1 + cache[m] % 245
    return cache


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("listed", [False, True], ids=["range", "list"])
def test_load_reads_every_code(wf, fmt, dtype, d, listed):  # noqa: F811
    p = wf.make_cache_params(batch=2, heads=3, capacity=333, head_dim=d, rows=333, dtype=dtype,
                             format=fmt)
    cache = any_cache(wf, p, fmt)
    codes = torch.cat([cache[0].view(-1), cache[2].view(-1)]).unique()
    assert len(codes) == (256 if fmt == "e2m1" else 254)
    g = torch.Generator().manual_seed(2)
    idx = torch.stack([torch.randperm(333, generator=g) for _ in range(6)]).int().view(2, 3, 333)
    got = wf.cache_load(p, [t.cuda() for t in cache], idx.cuda() if listed else None)
    for m, x in ((0, got[0]), (2, got[1])):
        v = cacheref.values(cache[m], cache[m + 1], fmt)
        if listed:
            v = v.gather(2, idx.long().unsqueeze(-1).expand(-1, -1, -1, d))
        assert torch.equal(x.cpu(), v.float().to(DT[dtype]))
        if fmt == "e2m1":  # (what an oracle that drops a sign would not see)
            assert bool((x[..., 0::2] < 0).any()) and bool((x[..., 1::2] < 0).any())


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_store_overwrites_any_old_byte(wf, fmt):  # noqa: F811
    p = wf.make_cache_params(batch=2, heads=3, capacity=100, head_dim=128, rows=41, format=fmt)
    old = any_cache(wf, p, fmt)
    g = torch.Generator().manual_seed(4)
    K, V = (torch.randn((2, 3, 41, 128), generator=g).bfloat16() for _ in range(2))
    idx = torch.stack([torch.randperm(100, generator=g)[:41] for _ in range(2)]).int()
    cache = [t.cuda() for t in old]
    wf.wf_cache_store(p, K.cuda(), V.cuda(), idx.cuda(), *cache)
    for m, x in ((0, K), (2, V)):
        code, byte = cacheref.quantise(x, fmt)
        code = cacheref.pack(code, fmt)
        for b in range(2):
            old[m][b][:, idx[b].long()] = code[b]
            old[m + 1][b][:, idx[b].long()] = byte[b]
    for a, b in zip(cache, old):
        assert torch.equal(a.cpu(), b)
