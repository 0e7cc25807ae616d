"""Refusals of rotary positions and of the cache in pages: on the host, before
anything is queued (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2606_00724_amd as wf

GOOD, ODD, WORD = (ctypes.c_void_p(x) for x in (0x10000, 0x10008, 0x10004))


def rope_params(**kw):
    return wf.make_rope_params(**{**dict(batch=2, heads=3, rows=5, head_dim=64), **kw})


def append_params(**kw):
    return wf.make_append_params(**{**dict(pages=4, page_rows=16, heads=2, head_dim=64, tokens=5,
                                           group=2), **kw})


def move_params(**kw):
    return wf.make_move_params(**{**dict(pages=4, page_rows=16, heads=2, head_dim=64, batch=2,
                                         table_pages=2, moves=3), **kw})


ROTATION = [
    (dict(rot_dim=8), 2), (dict(rot_dim=24), 2), (dict(rot_dim=80), 2), (dict(layout=2), 1),
    (dict(factor=float("nan")), 1), (dict(factor=float("inf")), 1),
    (dict(sections=[30, 1, 0, 0, 1]), 1),
]


@pytest.mark.parametrize("change,code", ROTATION + [
    (dict(batch=0), 1), (dict(heads=0), 1), (dict(rows=-1), 1), (dict(head_dim=96), 2),
    (dict(dtype=5), 1), (dict(rot_dim=0), 2), (dict(heads=(1 << 20) + 1), 2),
    (dict(batch=1 << 16, rows=1 << 15), 2), (dict(x_strides=(960, 320, 63)), 1),
    (dict(y_strides=(960, 320, 0)), 1), (dict(y_strides=(960, 320, 60)), 1),
    (dict(x_strides=(960, -320, 64)), 1), (dict(x_strides=(1 << 41, 320, 64)), 1),
    (dict(x_strides=(964, 320, 64)), 1), (dict(batch=1 << 12, heads=1 << 16, rows=1 << 12), 2),
])
def test_rope_parameters(change, code):
    p = rope_params(**change)
    assert wf.library().wf_rope(ctypes.byref(p), GOOD, GOOD, GOOD, GOOD, None) == code
    assert wf.library().wf_last_error().decode()


def test_rope_axes_and_pointers():
    lib, p = wf.library(), rope_params(sections=[10, 12, 10])
    p.axes = 2
    assert lib.wf_rope(ctypes.byref(p), *[GOOD] * 4, None) == 1
    p = rope_params()
    for i, bads in enumerate(((None, ODD), (None, ctypes.c_void_p(0x10002)),
                              (None, ctypes.c_void_p(0x10001)), (None, ODD))):
        for bad in bads:
            a = [GOOD] * 4
            a[i] = bad
            assert lib.wf_rope(ctypes.byref(p), *a, None) == 1
    # in place, but to other rows
    q = rope_params(y_strides=(64, 640, 128))
    assert lib.wf_rope(ctypes.byref(q), *[GOOD] * 4, None) == 1
    assert lib.wf_rope(None, *[GOOD] * 4, None) == 1
    assert lib.wf_rope(ctypes.byref(rope_params(rows=0)), *[None] * 4, None) == 0
    for bad in (dict(sections=[30]), dict(axis=[0] * 33), dict(axis=[256] * 32),
                dict(axis=[-1] * 32), dict(rot_dim=256)):
        with pytest.raises(ValueError):
            rope_params(**bad)


POOL = [
    (dict(pages=0), 1), (dict(heads=0), 1), (dict(page_rows=8), 2), (dict(page_rows=24), 2),
    (dict(page_rows=2048), 2), (dict(head_dim=32), 2), (dict(dtype=9), 1), (dict(format=3), 1),
    (dict(pages=(1 << 26) + 1), 2), (dict(heads=(1 << 20) + 1), 2), (dict(page_rows=-16), 2),
]


@pytest.mark.parametrize("change,code", POOL + ROTATION + [
    (dict(tokens=-1), 1), (dict(group=-1), 1), (dict(group=1 << 20), 2), (dict(k_row=64), 1),
    (dict(q_row=128), 1), (dict(v_row=132), 1), (dict(qr_row=-256), 1),
    (dict(tokens=1 << 30, heads=64, group=14), 2),
])
def test_append_parameters(change, code):
    p = append_params(**change)
    args = [GOOD] * 6 + [GOOD, None, GOOD, None, GOOD]
    if "format" not in change:
        assert wf.library().wf_page_append(ctypes.byref(p), *args, None) == code
        assert wf.library().wf_last_error().decode()
    args = [GOOD] * 11
    assert wf.library().wf_page_append(ctypes.byref(p), *args, None) == code


def test_append_pointers():
    lib = wf.library()
    #       Q     K     V     pos   freq  slot  Kc    Kx    Vc    Vx    Qr
    words = {3, 4, 5}
    for fmt in (None, "e2m1"):
        p = append_params(format=fmt)
        for i in range(11):
            for bad in (None, ctypes.c_void_p(0x10002) if i in words else ODD):
                if bad is None and fmt is None and i in (7, 9):
                    continue
                a = [GOOD] * 11
                a[10] = ctypes.c_void_p(0x20000)
                a[i] = bad
                assert lib.wf_page_append(ctypes.byref(p), *a, None) == 1, (fmt, i)
    p = append_params(q_row=512)
    assert lib.wf_page_append(ctypes.byref(p), *[GOOD] * 11, None) == 1  # in place, other rows
    p = append_params(tokens=0)
    assert lib.wf_page_append(ctypes.byref(p), *[None] * 11, None) == 0
    assert lib.wf_page_append(None, *[GOOD] * 11, None) == 1


@pytest.mark.parametrize("change,code", POOL + [
    (dict(batch=0), 1), (dict(table_pages=0), 1), (dict(moves=-1), 1), (dict(moves=257), 2),
    (dict(batch=1 << 13, heads=1 << 12), 2), (dict(batch=1 << 12, heads=1 << 12), 2),
])
def test_move_parameters(change, code):
    p = move_params(**change)
    assert wf.library().wf_page_move(ctypes.byref(p), *[GOOD] * 7, None) == code
    assert wf.library().wf_last_error().decode()


def test_move_pointers():
    lib, p = wf.library(), move_params(format="e4m3")
    for i in range(7):
        for bad in (None, ctypes.c_void_p(0x10002) if i < 3 else ODD):
            a = [GOOD] * 7
            a[i] = bad
            assert lib.wf_page_move(ctypes.byref(p), *a, None) == 1
    assert lib.wf_page_move(ctypes.byref(move_params(moves=0)), *[None] * 7, None) == 0
    assert lib.wf_page_move(None, *[GOOD] * 7, None) == 1


def test_binding_refuses_what_the_parameters_do_not_describe():
    p = rope_params()
    X, pos, f = torch.zeros((2, 3, 5, 64)).bfloat16(), torch.zeros((1, 2, 5)).int(), torch.ones(32)
    for bad, err in ((dict(X=X.float()), TypeError), (dict(X=X[:, :, :4]), ValueError),
                     (dict(X=X.transpose(0, 1).contiguous().transpose(0, 1)), ValueError),
                     (dict(Y=X[:, :, :, ::2]), ValueError), (dict(Y=None), ValueError),
                     (dict(X=torch.zeros(1).bfloat16().expand(2, 3, 5, 64)), ValueError),
                     (dict(pos=pos.long()), TypeError), (dict(f=f[:31]), ValueError),
                     (dict(), ValueError)):  # (the last: tensors of the host)
        a = {**dict(X=X, pos=pos, f=f, Y=X), **bad}
        with pytest.raises(err):
            wf.wf_rope(p, a["X"], a["pos"], a["f"], a["Y"])
    p = append_params(format="e4m3")
    Kc, Kx, Vc, Vx = wf.alloc_pages(p, "cpu")
    assert Kc.shape == (4, 2, 16, 64) and Kx.shape == (4, 2, 16, 2) and Vc.dtype == torch.uint8
    plain = wf.alloc_pages(append_params(), "cpu")
    assert plain[0].shape == (4, 2, 16, 64) and plain[0].dtype == torch.bfloat16
    assert plain[1] is None
    assert wf.alloc_pages(append_params(format="e2m1"), "cpu")[2].shape == (4, 2, 16, 32)
    ok = dict(Q=torch.zeros((5, 4, 64)).bfloat16(), K=torch.zeros((5, 2, 64)).bfloat16(),
              V=torch.zeros((5, 2, 64)).bfloat16(), pos=torch.zeros((1, 5)).int(), f=f,
              slot=torch.zeros(5).int(), Kc=Kc, Kx=Kx, Vc=Vc, Vx=Vx,
              Qr=torch.zeros((5, 4, 64)).bfloat16())
    for bad, err in ((dict(Q=None), ValueError), (dict(K=ok["K"].float()), TypeError),
                     (dict(V=ok["Q"][:, :2]), ValueError), (dict(slot=None), ValueError),
                     (dict(Kx=None), ValueError), (dict(Kc=Kc[:3]), ValueError),
                     (dict(Vx=Kc), ValueError), (dict(Qr=ok["K"]), ValueError),
                     (dict(), ValueError)):
        with pytest.raises(err):
            wf.wf_page_append(p, *{**ok, **bad}.values())
    q = append_params(group=0)
    with pytest.raises(ValueError):
        wf.wf_page_append(q, *{**ok, "Kc": plain[0], "Kx": None}.values())
    m = move_params()
    i = torch.zeros(6).int()
    for bad in (dict(table=i), dict(first=i), dict(source=i[:5]), dict(Kc=None), dict()):
        a = {**dict(table=i[:4], first=i[:2], source=i, Kc=plain[0], Kx=None, Vc=plain[2],
                    Vx=None), **bad}
        with pytest.raises(ValueError):
            wf.wf_page_move(m, *a.values())


# ------------------------------------------------------------ attention

def tree_params(**kw):
    return wf.make_tree_params(**{**dict(pages=4, page_rows=16, heads=2, head_dim=64, batch=2,
                                         max_rows=3, table_pages=2, group=2), **kw})


@pytest.mark.parametrize("change,code", POOL + [
    (dict(group=0), 1), (dict(batch=0), 1), (dict(tokens=0), 1), (dict(table_pages=0), 1),
    (dict(max_rows=0), 1), (dict(max_rows=257), 2), (dict(max_len=-1), 1), (dict(max_len=33), 1),
    (dict(scale=float("nan")), 1), (dict(scale=float("-inf")), 1), (dict(scale=3e38), 1),
    (dict(group=1 << 20), 2), (dict(batch=1 << 22, max_rows=128), 2), (dict(q_row=192), 1),
    (dict(o_row=252), 1), (dict(o_row=260), 1),
    (dict(batch=1 << 20, heads=1 << 8, max_rows=1, group=1, head_dim=128), 2),
])
def test_tree_parameters(change, code):
    p = tree_params(**change)
    args = [GOOD] * 9 + [ctypes.c_void_p(0x20000), GOOD, GOOD, 1 << 50]
    lib = wf.library()
    assert lib.wf_tree_attn(ctypes.byref(p), *args, None) == code, lib.wf_last_error()
    assert lib.wf_last_error().decode()
    assert wf.tree_workspace_bytes(p) == 0
    with pytest.raises(wf.WfError):
        wf.tree_plan(p, 0)


def test_tree_pointers_and_workspace():
    #       Q  Kc Kx Vc Vx table len start mask O lse
    lib, nullable, words = wf.library(), {7, 8, 10}, {5, 6, 7, 8, 10}
    p = tree_params(format="e4m3", page_rows=1024, table_pages=8)
    need = wf.tree_workspace_bytes(p)
    assert need > 0
    args = [GOOD] * 9 + [ctypes.c_void_p(0x20000), GOOD, GOOD, need]
    for i in range(11):
        for bad in (None, ctypes.c_void_p(0x10002) if i in words else ODD):
            if bad is None and i in nullable:
                continue
            a = list(args)
            a[i] = bad
            assert lib.wf_tree_attn(ctypes.byref(p), *a, None) == 1, i
    assert lib.wf_tree_attn(ctypes.byref(p), *args[:9], GOOD, *args[10:], None) == 1  # O is Q
    assert lib.wf_tree_attn(ctypes.byref(p), *args[:11], ctypes.c_void_p(0x10010), need, None) == 3
    assert lib.wf_tree_attn(None, *args, None) == 1
    p.causal = 2
    assert lib.wf_tree_attn(ctypes.byref(p), *args, None) == 1
    p = tree_params(tokens=5)
    a = list(args)
    a[7] = None
    assert lib.wf_tree_attn(ctypes.byref(p), *a, None) == 1  # tokens need row_start
    assert lib.wf_tree_plan(ctypes.byref(tree_params()), 0, None) == 1


def test_tree_workspaces_hold_whole_partials():
    import random
    rng = random.Random(5)
    for _ in range(300):
        P = rng.choice([16, 64, 1024])
        p = tree_params(page_rows=P, table_pages=rng.choice([1, 7, 300, 2048]),
                        pages=1 << 16 if P < 1024 else 4096, heads=rng.choice([1, 3, 8, 32]),
                        group=rng.choice([1, 4, 7]), batch=rng.choice([1, 3, 64, 300]),
                        max_rows=rng.choice([1, 5, 32, 256]), head_dim=rng.choice([64, 128]),
                        dtype=rng.choice(["bf16", "f32"]),
                        format=rng.choice([None, "e4m3", "e2m1"]))
        nb, rows = wf.tree_workspace_bytes(p), p.tokens * p.heads * p.group
        s = wf.tree_plan(p)
        assert nb == (rows * s.ranges * (p.head_dim + 2) * 4 if s.ranges > 1 else 0)
        assert s.ranges * s.range_rows >= p.max_len > (s.ranges - 1) * s.range_rows
        assert s.range_rows % 64 == 0
        for have in (0, nb // 2, nb):
            t = wf.tree_plan(p, have)
            assert t.ranges == 1 or rows * t.ranges * (p.head_dim + 2) * 4 <= have
        # a cache without rows
        p.max_len = 0
        assert wf.tree_workspace_bytes(p) == 0 and wf.tree_plan(p).ranges == 1


def test_tree_binding_refuses_what_the_parameters_do_not_describe():
    p = tree_params()
    Kc, _, Vc, _ = wf.alloc_pages(p, "cpu")
    Q = torch.zeros((6, 4, 64)).bfloat16()
    i32 = torch.zeros(64).int()
    ok = dict(Q=Q, Kc=Kc, Kx=None, Vc=Vc, Vx=None, table=i32[:4], length=i32[:2], row_start=None,
              mask=None, O=Q.clone(), lse=None, workspace=None)
    for bad, err in ((dict(Q=Q.float()), TypeError), (dict(O=Q[:5]), ValueError),
                     (dict(Q=torch.zeros((6, 5, 64)).bfloat16()[:, 1:]), ValueError),
                     (dict(Kc=Kc[:3]), ValueError), (dict(Vc=Vc.float()), TypeError),
                     (dict(table=i32[:3]), ValueError), (dict(length=None), ValueError),
                     (dict(row_start=i32[:2]), ValueError), (dict(mask=i32[:12]), ValueError),
                     (dict(mask=i32[:6].long()), TypeError), (dict(lse=i32[:24]), TypeError),
                     (dict(), ValueError)):
        with pytest.raises(err):
            wf.wf_tree_attn(p, *{**ok, **bad}.values())
