"""Refusals of the quantised cache and the shared-prefix attention: on the
host, before anything is queued (no GPU needed)."""
import ctypes

import pytest

import paper_2606_00724_amd as wf

GOOD, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008)


def cache_params(**kw):
    return wf.make_cache_params(**{**dict(batch=1, heads=2, capacity=64, head_dim=64, rows=8),
                                   **kw})


def prefix_params(**kw):
    return wf.make_prefix_params(**{**dict(share=2, heads=2, q_len=4, head_dim=64, prefix_cap=64,
                                           tail_cap=8), **kw})


@pytest.mark.parametrize("change,code", [
    (dict(batch=0), 1), (dict(heads=0), 1), (dict(capacity=0), 1), (dict(head_dim=96), 2),
    (dict(rows=-1), 1), (dict(first=-1), 1), (dict(first=57), 1), (dict(rows=65), 1),
    (dict(first=2 ** 31 - 1), 1), (dict(dtype=7), 1), (dict(format=None), 1), (dict(format=9), 1),
    (dict(batch=1 << 20, heads=1 << 10), 2),
    (dict(batch=1 << 12, heads=1 << 12, rows=1 << 20, capacity=1 << 20), 2),
])
def test_cache_parameters(change, code):
    p = cache_params(**change)
    lib = wf.library()
    for fn in (lib.wf_cache_store, lib.wf_cache_load):
        assert fn(ctypes.byref(p), *[GOOD, GOOD, None, GOOD, GOOD, GOOD, GOOD]
                  if fn is lib.wf_cache_store else [GOOD, GOOD, GOOD, GOOD, None, GOOD, GOOD],
                  None) == code
        assert lib.wf_last_error().decode()


def test_cache_pointers():
    lib, p = wf.library(), cache_params()
    for fn, idx in ((lib.wf_cache_store, 2), (lib.wf_cache_load, 4)):
        for i in range(7):
            for bad in (None, ODD):
                args = [GOOD] * 7
                args[i] = bad
                if i == idx and bad is None:
                    continue
                assert fn(ctypes.byref(p), *args, None) == 1
    assert lib.wf_cache_store(None, *[GOOD] * 7, None) == 1
    # nothing to move: nothing is looked at
    p = cache_params(rows=0)
    assert lib.wf_cache_store(ctypes.byref(p), *[None] * 7, None) == 0
    assert lib.wf_cache_load(ctypes.byref(p), *[None] * 7, None) == 0


@pytest.mark.parametrize("change,code", [
    (dict(prefixes=0), 1), (dict(share=0), 1), (dict(heads=-1), 1), (dict(group=0), 1),
    (dict(q_len=0), 1), (dict(head_dim=80), 2), (dict(prefix_cap=-1), 1), (dict(tail_cap=-1), 1),
    (dict(prefix_rows=0, tail_cap=0), 1), (dict(prefix_cap=0, prefix_rows=5), 1),
    (dict(prefix_rows=65), 1),  # without a list
    (dict(prefix_cap=(1 << 30) + 1, prefix_rows=4), 2), (dict(dtype=3), 1), (dict(format=5), 1),
    (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
    (dict(prefixes=1 << 15, share=1 << 15, heads=2), 2),
    (dict(share=2 ** 31 - 1, heads=2 ** 31 - 1, group=2 ** 31 - 1, q_len=2 ** 31 - 1), 2),
])
def test_prefix_parameters(change, code):
    p = prefix_params(**change)
    lib = wf.library()
    args = [GOOD, GOOD, None, GOOD, None, None, None, GOOD, GOOD, None, GOOD, None, GOOD, 1 << 50]
    assert lib.wf_prefix_attn(ctypes.byref(p), *args, None) == code, lib.wf_last_error()
    assert lib.wf_last_error().decode()
    if change != dict(prefix_rows=65):
        assert wf.prefix_workspace_bytes(p) == 0


def test_prefix_pointers_and_workspace():
    lib, p = wf.library(), prefix_params(format="e4m3")
    need = wf.prefix_workspace_bytes(p)
    assert need > 0
    args = [GOOD] * 13 + [need]
    nullable = {5, 6, 9, 11}
    for i in range(12):
        for bad in (None, ODD):
            if i in nullable and bad is None:
                continue
            a = list(args)
            a[i] = bad
            assert lib.wf_prefix_attn(ctypes.byref(p), *a, None) == 1, i
    for ws, nb in ((None, need), (GOOD, need - 1), (ctypes.c_void_p(0x10010), need)):
        assert lib.wf_prefix_attn(ctypes.byref(p), *args[:12], ws, nb, None) == 3
    assert lib.wf_prefix_attn(None, *args, None) == 1
    # one key range and no own rows: nothing to merge, no workspace
    assert wf.prefix_workspace_bytes(prefix_params(prefix_cap=16, tail_cap=0)) == 0


def test_binding_refuses_what_the_parameters_do_not_describe():
    import torch
    p = cache_params()
    K = torch.zeros((1, 2, 8, 64), dtype=torch.bfloat16)
    cache = wf.alloc_cache(p, "cpu")
    assert cache[0].shape == (1, 2, 64, 64) and cache[1].shape == (1, 2, 64, 2)
    assert wf.alloc_cache(cache_params(format="e2m1"), "cpu")[0].shape == (1, 2, 64, 32)
    idx = torch.zeros((1, 8), dtype=torch.int32)
    for bad, err in ((dict(K=K.float()), TypeError), (dict(V=K[:, :, :7]), ValueError),
                     (dict(idx=idx.long()), TypeError), (dict(idx=idx[:, :7]), ValueError),
                     (dict(Kc=cache[0][:, :, :63]), ValueError),
                     (dict(Kx=cache[1].to(torch.int8)), TypeError), (dict(), ValueError)):
        a = {**dict(K=K, V=K, idx=idx, Kc=cache[0], Kx=cache[1]), **bad}
        with pytest.raises(err):  # (the last: tensors of the host)
            wf.wf_cache_store(p, a["K"], a["V"], a["idx"], a["Kc"], a["Kx"], *cache[2:])
    q = prefix_params()
    Q = torch.zeros((2, 2, 4, 64), dtype=torch.bfloat16)
    Kp = torch.zeros((1, 2, 64, 64), dtype=torch.bfloat16)
    Kt = torch.zeros((2, 2, 8, 64), dtype=torch.bfloat16)
    ok = dict(Q=Q, K=Kp, Kx=None, V=Kp, Vx=None, row_idx=None, prefix_len=None, Kt=Kt, Vt=Kt,
              tail_len=None, O=Q, lse=None)
    for bad, err in ((dict(Q=Q.float()), TypeError), (dict(K=Kp[:, :, :3]), ValueError),
                     (dict(Vt=None), ValueError), (dict(tail_len=torch.zeros(3).int()), ValueError),
                     (dict(lse=torch.zeros(16, dtype=torch.float64)), TypeError),
                     (dict(Kx=torch.zeros(4, dtype=torch.uint8)), ValueError),
                     (dict(K=None), ValueError), (dict(), ValueError)):
        with pytest.raises(err):
            wf.wf_prefix_attn(q, *{**ok, **bad}.values(), None)


def test_workspaces_over_the_range_hold_whole_partials():
    """A partial is (d + 2) floats per query row; a call has as many as ranges
    of its prefix, and none where one range and no own rows are all."""
    import random
    rng = random.Random(4)
    for _ in range(300):
        p = prefix_params(prefixes=rng.choice([1, 2, 5]), share=rng.choice([1, 3, 32, 300]),
                          heads=rng.choice([1, 3, 8, 32]), group=rng.choice([1, 4, 7]),
                          q_len=rng.choice([1, 5, 32, 256]), head_dim=rng.choice([64, 128]),
                          prefix_cap=int(2 ** rng.uniform(0, 18)),
                          tail_cap=rng.choice([0, 1, 100, 5000]), dtype=rng.choice(["bf16", "f32"]),
                          format=rng.choice([None, "e4m3", "e2m1"]))
        rows = p.prefixes * p.share * p.heads * p.group * p.q_len
        nb = wf.prefix_workspace_bytes(p)
        assert nb % (rows * (p.head_dim + 2) * 4) == 0
        slots = nb // (rows * (p.head_dim + 2) * 4)
        assert slots > (1 if p.tail_cap == 0 else 0) or (slots == 0 and p.tail_cap == 0)
        p.prefix_rows = 0
        assert wf.prefix_workspace_bytes(p) == 0


def test_launches_of_two_to_the_32_threads_are_refused():
    lib = wf.library()
    # 2^24 units, a workgroup of 256 threads each
    p = cache_params(batch=1 << 12, heads=1 << 12, rows=1, capacity=1)
    assert lib.wf_cache_store(ctypes.byref(p), GOOD, GOOD, None, *[GOOD] * 4, None) == 2
    assert lib.wf_cache_load(ctypes.byref(p), *[GOOD] * 4, None, GOOD, GOOD, None) == 2
    for change in (dict(prefix_cap=16, tail_cap=0), dict(prefix_cap=0, tail_cap=4)):
        q = prefix_params(prefixes=1 << 12, share=1, heads=1 << 12, q_len=1, **change)
        args = [GOOD, GOOD, None, GOOD, None, None, None, GOOD, GOOD, None, GOOD, None, GOOD,
                1 << 50]
        assert lib.wf_prefix_attn(ctypes.byref(q), *args, None) == 2, change
