"""wf_prefix_attn against the 64-bit reference, with the elementwise tolerance
that cacheref.prefix_attention derives."""
from __future__ import annotations

import math

import pytest
import torch

import cacheref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2606_00724_amd as wf
    return wf


DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(wf, seed=1, *, prefixes=1, share=1, heads=1, group=1, B=1, d=64, P=0, n=0, T=0,
         dtype="bf16", fmt=None, scale=0.0, plen=None, tlen=None, gain=1.0):
    """Inputs on the CPU, and the parameters.  n: length of a row list; gain:
    factor of the queries."""
    g = torch.Generator().manual_seed(seed)
    dt = DT[dtype]
    rnd = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    c = dict(Q=(gain * rnd(prefixes * share, heads * group, B, d)).to(dt), Kx=None, Vx=None,
             row_idx=None, Kt=None, Vt=None, K=None, V=None)
    for m in "KV":
        if P:
            x = rnd(prefixes, heads, P, d).to(dt)
            if fmt:
                code, byte = cacheref.quantise(x, fmt)
                c[m], c[m + "x"] = cacheref.pack(code, fmt), byte
                c[m + "v"] = cacheref.values(c[m], byte, fmt)
            else:
                c[m] = c[m + "v"] = x
        if T:
            c[m + "t"] = rnd(prefixes * share, heads, T, d).to(dt)
    if n:
        c["row_idx"] = torch.stack([torch.randperm(max(P, n), generator=g)[:n] % P
                                    for _ in range(prefixes * heads)]).int().view(
                                        prefixes, heads, n)
    for name, v in (("prefix_len", plen), ("tail_len", tlen)):
        c[name] = None if v is None else torch.tensor(v, dtype=torch.int32)
    p = wf.make_prefix_params(prefixes=prefixes, share=share, heads=heads, group=group, q_len=B,
                              head_dim=d, prefix_cap=P, prefix_rows=n or P, tail_cap=T,
                              dtype=dtype, format=fmt, scale=scale)
    return p, c


ARGS = ("Q", "K", "V", "Kx", "Vx", "row_idx", "prefix_len", "Kt", "Vt", "tail_len")


def call(wf, p, c, **kw):
    return wf.prefix_attend(p, **{k: None if c[k] is None else c[k].cuda() for k in ARGS},
                            want_lse=True, **kw)


def check(wf, p, c):
    O, lse = call(wf, p, c)
    O, lse = O.cpu().double(), lse.cpu().double()
    scale = p.scale or 1 / math.sqrt(p.head_dim)
    ref, rl, tol, ltol = cacheref.prefix_attention(
        c["Q"], c.get("Kv"), c.get("Vv"), prefixes=p.prefixes, share=p.share, heads=p.heads,
        group=p.group, scale=scale, plen=c["prefix_len"], tlen=c["tail_len"],
        rows=p.prefix_rows, row_idx=c["row_idx"], Kt=c["Kt"], Vt=c["Vt"], dtype=c["Q"].dtype)
    off = (O - ref).abs() - tol
    assert bool((off <= 0).all()), (f"off by {float((O - ref).abs().max())}, "
                                    f"{int((off > 0).sum())} of {off.numel()}")
    same = torch.where(torch.isinf(rl), lse == rl, (lse - rl).abs() <= ltol)
    assert bool(same.all()), f"lse off by {float((lse - rl).abs().max())}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", [None, "e4m3", "e2m1"])
@pytest.mark.parametrize("kw", [
    dict(P=1), dict(P=33, B=3), dict(P=128, B=32, d=128), dict(P=129, B=33, share=2),
    dict(P=300, B=17, share=3, heads=2, d=128, T=5),
    dict(P=257, B=5, share=5, heads=2, group=4, T=70, d=128),        # 100 rows a K/V head
    dict(P=640, B=64, share=4, heads=1, group=2, T=129),             # 512 rows
    dict(P=1500, B=1, share=2, heads=3, group=7, T=1, d=128, prefixes=2),
    dict(P=400, n=333, B=16, share=2, heads=2, T=40, prefixes=2),
    dict(P=400, n=900, B=40, share=2, d=128),                        # rows named more than once
], ids=lambda k: "-".join(f"{a}{b}" for a, b in k.items()))
def test_against_the_reference(wf, dtype, fmt, kw):
    check(wf, *make(wf, dtype=dtype, fmt=fmt, **kw))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_own_rows_only(wf, dtype):
    check(wf, *make(wf, dtype=dtype, P=0, T=77, share=3, heads=2, B=9))
    check(wf, *make(wf, dtype=dtype, P=0, T=1, share=2, heads=2, B=1, tlen=[0, 1]))


@pytest.mark.parametrize("dtype,fmt", [("bf16", None), ("bf16", "e4m3"), ("f32", None),
                                       ("f32", "e2m1")])
@pytest.mark.parametrize("plen,tlen", [
    ([0, 300], [0, 5, 70, 1]), ([1, 129], [70, 0, 0, 69]), ([-5, 9999], [-1, 200, 3, 64]),
    ([128, 256], [32, 33, 64, 65]),
])
def test_lengths(wf, dtype, fmt, plen, tlen):
    """Ragged lengths, out of range on both sides, rows that see no key; what
    is behind a length is NaN and infinite."""
    p, c = make(wf, dtype=dtype, fmt=fmt, prefixes=2, share=2, heads=2, group=2, B=7, d=128,
                P=300, T=70, plen=plen, tlen=tlen)
    for i, L in enumerate(plen):
        L = min(max(L, 0), 300)
        if fmt:
            for m in ("Kx", "Vx"):
                c[m][i, :, L:] = 255
            for m in ("K", "V"):
                c[m][i, :, L:] = 0
        else:
            c["K"][i, :, L:], c["V"][i, :, L:] = math.nan, math.inf
    for n, t in enumerate(tlen):
        t = min(max(t, 0), 70)
        c["Kt"][n, :, t:], c["Vt"][n, :, t:] = math.inf, math.nan
    check(wf, p, c)
    if plen[0] == 0:
        O, lse = call(wf, p, c)
        assert int(O[0].abs().max()) == 0 and bool((lse[0] == -math.inf).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.37, -0.2, 1e-3])
def test_scales(wf, dtype, scale):
    check(wf, *make(wf, dtype=dtype, P=200, T=33, share=2, B=20, d=64, scale=scale))


def test_large_scores_keep_their_differences(wf):
    """Scores of some thousands, whose maximum comes late in the row."""
    p, c = make(wf, dtype="f32", P=700, share=2, B=20, d=64, gain=300.0)
    order = (c["Q"][0, 0, 0] @ c["K"][0, 0].T).argsort()
    c["K"][0, 0] = c["K"][0, 0][order]
    c["Kv"] = c["K"]
    check(wf, p, c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_and_nan_keys(wf, dtype):
    """A key row that scores -inf for every query has weight 0 (its value is
    finite); one that scores +inf or NaN makes the rows NaN, as the formula
    does; blocks of -inf scores before the first finite one add nothing."""
    p, c = make(wf, dtype=dtype, P=200, T=10, share=2, B=3, d=64)
    c["Q"][..., 0] = 1.0
    c["Kt"][..., 0] = 0.0
    c["K"][0, 0, :70, 0] = -math.inf
    O, lse = call(wf, p, c)
    keep = {**c, "K": c["K"][:, :, 70:].contiguous(), "V": c["V"][:, :, 70:].contiguous()}
    keep |= {"Kv": keep["K"], "Vv": keep["V"]}
    p2 = wf.make_prefix_params(share=2, heads=1, q_len=3, head_dim=64, prefix_cap=130, tail_cap=10,
                               dtype=dtype)
    check(wf, p2, keep)
    O2, lse2 = call(wf, p2, keep)
    fine = 2.0 ** -6 if dtype == "bf16" else 2.0 ** -18
    assert float((O - O2).abs().max()) <= fine * float(O2.abs().max())
    for v in (math.inf, math.nan):
        c["K"][0, 0, 100, 0] = v
        O, lse = call(wf, p, c)
        assert bool(O.isnan().all()) and bool(lse.isnan().all())


def test_list_ids_outside_are_clamped(wf):
    p, c = make(wf, P=50, n=64, B=8, share=2, heads=2)
    c["row_idx"][0, 0, :3] = torch.tensor([-1, 50, 2 ** 31 - 1], dtype=torch.int32)
    a = call(wf, p, c)[0]
    c["row_idx"].clamp_(0, 49)
    assert torch.equal(a, call(wf, p, c)[0])
    check(wf, p, c)


def test_long_lists_take_their_ids_in_turn(wf):
    """More ids than the LDS holds at once, in one range of keys."""
    p, c = make(wf, P=9000, n=9000, B=64, share=8, heads=8, group=4, d=64)
    a = call(wf, p, c)[0]
    idx = c["row_idx"].long()
    for k in range(8):
        for m in "KV":
            c[m][0, k] = c[m][0, k][idx[0, k]]
    c["row_idx"] = None
    assert torch.equal(a, call(wf, p, c)[0])


@pytest.mark.parametrize("fmt", [None, "e4m3"])
def test_repeats_graphs_and_streams(wf, fmt):
    """Equal bits from run to run, from replays with new inputs (eager calls
    between them) and from a stream of its own; the workspace's old contents
    do not matter."""
    p, c = make(wf, fmt=fmt, P=3000, T=40, share=4, heads=2, group=2, B=8, d=128,
                tlen=[0, 40, 7, 33])
    dev = {k: None if c[k] is None else c[k].cuda() for k in ARGS}
    O, lse = wf.prefix_attend(p, **dev, want_lse=True)
    ws = wf.alloc_prefix_workspace(p, "cuda")
    ws.fill_(255)
    again = wf.prefix_attend(p, **dev, workspace=ws, want_lse=True)
    assert torch.equal(O, again[0]) and torch.equal(lse, again[1])
    Og, lg = torch.empty_like(O), torch.empty_like(lse)
    order = [dev[k] for k in ("Q", "K", "Kx", "V", "Vx", "row_idx", "prefix_len", "Kt", "Vt",
                              "tail_len")]
    wf.wf_init()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wf.wf_prefix_attn(p, *order, Og, lg, ws)
    for seed in range(4):
        dev["Q"].copy_(make(wf, seed=seed, fmt=fmt, P=1, T=40, share=4, heads=2, group=2, B=8,
                            d=128)[1]["Q"])
        dev["tail_len"].add_(1)
        graph.replay()
        torch.cuda.synchronize()
        e = wf.prefix_attend(p, **dev, want_lse=True)
        assert torch.equal(Og, e[0]) and torch.equal(lg, e[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    s = wf.prefix_attend(p, **dev, want_lse=True, stream=side)
    side.synchronize()
    assert torch.equal(Og, s[0]) and torch.equal(lg, s[1])


def test_filtered_step_on_a_quantised_shared_prompt(wf):
    """The operators together, as a server with one prompt and several
    sequences uses them: the prompt's keys and values are stored quantised;
    the coarse keys (wf_dwt_keys, of the values kept) pick the regions; their
    rows are read back and scanned for the tokens; every sequence then attends
    over those tokens in place and over its own rows.  The selection is
    checked against the same calls on an unquantised cache of the read-back
    values, the output against the 64-bit reference."""
    h, L, d, B, share, J, S, k = 2, 1024, 64, 16, 3, 4, 16, 100
    g = torch.Generator().manual_seed(5)
    K, V = (torch.randn((1, h, L, d), generator=g).to(torch.bfloat16) for _ in range(2))
    Q = torch.randn((share, h, B, d), generator=g).to(torch.bfloat16)
    Kt, Vt = (torch.randn((share, h, B, d), generator=g).to(torch.bfloat16) for _ in range(2))
    Kd, Vd = K.cuda(), V.cuda()
    pc = wf.make_cache_params(batch=1, heads=h, capacity=L, head_dim=d, rows=L)
    cache = wf.alloc_cache(pc, "cuda")
    wf.wf_cache_store(pc, Kd, Vd, None, *cache)
    Kr, Vr = wf.cache_load(pc, cache)
    # the sequences' query rows stacked: one selection per K/V head
    Qs = Q.transpose(0, 1).reshape(1, h, share * B, d).contiguous().cuda()
    p = wf.make_params(batch=1, heads=h, ctx_len=L, head_dim=d, q_len=share * B, levels=J,
                       segments=S, budget=k)
    approx = wf.dwt_approx(p, Kr)
    W = torch.empty((1, h, L >> J), dtype=torch.float32, device="cuda")
    seg = torch.empty((1, h, S), dtype=torch.int32, device="cuda")
    wf.wf_skim_score(p, Qs, approx, W, seg, wf.alloc_workspace(p, wf.OP_SKIM, "cuda"))
    pool = (seg.unsqueeze(-1) * (1 << J) + torch.arange(1 << J, device="cuda", dtype=torch.int32)
            ).flatten(2).contiguous()
    pl = wf.make_cache_params(batch=1, heads=h, capacity=L, head_dim=d, rows=S << J)
    Kp, _ = wf.cache_load(pl, cache, pool)
    # the pool is a prompt of its own, of which all regions are scanned
    pp = wf.make_params(batch=1, heads=h, ctx_len=S << J, head_dim=d, q_len=share * B, levels=J,
                        segments=S, budget=k)
    every = torch.arange(S, dtype=torch.int32, device="cuda").expand(1, h, S).contiguous()
    pos = torch.empty((1, h, k), dtype=torch.int32, device="cuda")
    wf.wf_scan_select(pp, Qs, Kp, every, None, pos, wf.alloc_workspace(pp, wf.OP_SCAN, "cuda"))
    tok = pool.gather(2, pos.long())
    ref_tok = torch.empty_like(tok)
    wf.wf_scan_select(p, Qs, Kr, seg, None, ref_tok, wf.alloc_workspace(p, wf.OP_SCAN, "cuda"))
    assert torch.equal(tok, ref_tok)
    pa = wf.make_prefix_params(share=share, heads=h, q_len=B, head_dim=d, prefix_cap=L,
                               prefix_rows=k, tail_cap=B, format="e4m3")
    O = wf.prefix_attend(pa, Q.cuda(), cache[0], cache[2], Kx=cache[1], Vx=cache[3], row_idx=tok,
                         Kt=Kt.cuda(), Vt=Vt.cuda())
    ref, _, tol, _ = cacheref.prefix_attention(
        Q, Kr.cpu(), Vr.cpu(), prefixes=1, share=share, heads=h, group=1, scale=d ** -0.5,
        rows=k, row_idx=tok.cpu(), Kt=Kt, Vt=Vt)
    assert bool(((O.cpu().double() - ref).abs() <= tol).all())


@pytest.mark.parametrize("dtype,fmt,d", [("bf16", None, 128), ("bf16", None, 64),
                                         ("bf16", "e4m3", 128), ("bf16", "e2m1", 64),
                                         ("f32", None, 128), ("f32", "e2m1", 128)])
@pytest.mark.parametrize("listed", [False, True], ids=["dense", "list"])
@pytest.mark.parametrize("share,group,B", [(1, 1, 7), (2, 2, 15), (2, 2, 25), (2, 2, 75)],
                         ids=["7", "60", "100", "300"])
def test_long_ranges(wf, dtype, fmt, d, listed, share, group, B):
    """Units enough that a range has many tiles, at every split of a
    workgroup's waves over query rows and keys; one prefix ends inside a tile,
    one inside a range."""
    check(wf, *make(wf, dtype=dtype, fmt=fmt, d=d, prefixes=2, share=share, heads=32, group=group,
                    B=B, P=1100, n=1090 if listed else 0, T=3, plen=[1090, 777]))


def test_late_maxima_in_long_ranges(wf):
    """Scores that rise along the keys, so that the reference of the softmax is
    raised in many blocks, and a first block far below the others."""
    for M in (60, 100, 300):
        p, c = make(wf, prefixes=2, share=1, heads=32, B=M, d=128, P=1100, gain=0.05)
        ramp = torch.linspace(-60, 60, 1100)
        ramp[:32] = -300
        c["K"][..., 0] = ramp.to(torch.bfloat16)
        c["Q"][..., 0] = 4.0
        check(wf, p, c)


def test_two_calls_at_once(wf):
    """Two streams with a workspace each."""
    calls = []
    for k, fmt in enumerate((None, "e4m3")):
        p, c = make(wf, seed=k, fmt=fmt, P=5000, T=20, share=4, heads=4, group=2, B=8, d=128)
        dev = {a: None if c[a] is None else c[a].cuda() for a in ARGS}
        calls.append((p, dev, wf.prefix_attend(p, **dev), wf.alloc_prefix_workspace(p, "cuda"),
                      torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = [[wf.prefix_attend(p, **dev, workspace=ws, stream=s) for p, dev, _, ws, s in calls]
            for _ in range(5)]
    torch.cuda.synchronize()
    for pair in outs:
        for O, (_, _, want, _, _) in zip(pair, calls):
            assert torch.equal(O, want)


@pytest.mark.parametrize("fmt", [None, "e2m1"])
def test_offsets_past_32_bits(wf, fmt):
    """Rows behind 2^32 bytes of K and V: the last ones of a long prefix, by a
    list and by their place, equal to the same rows in a short one."""
    d, n, B = 128, 200, 8
    cap = (1 << 24) + 4096 if fmt is None else (1 << 26) + 4096
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("less than 24 GB of device memory free")
    p, c = make(wf, fmt=fmt, P=n, B=B, share=2, d=d)
    want = call(wf, p, c)
    dev = {k: None if c[k] is None else c[k].cuda() for k in ARGS}
    for m in ("K", "V", "Kx", "Vx"):
        if dev[m] is not None:
            long = torch.zeros((1, 1, cap, dev[m].shape[-1]), dtype=dev[m].dtype, device="cuda")
            long[:, :, -n:] = dev[m]
            dev[m] = long
    dev["row_idx"] = torch.arange(cap - n, cap, dtype=torch.int32, device="cuda").view(1, 1, n)
    q = wf.make_prefix_params(share=2, heads=1, q_len=B, head_dim=d, prefix_cap=cap,
                              prefix_rows=n, format=fmt)
    got = wf.prefix_attend(q, **dev, want_lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # all rows: the cleared ones have score 0 and value 0
    dev["row_idx"] = None
    q = wf.make_prefix_params(share=2, heads=1, q_len=B, head_dim=d, prefix_cap=cap,
                              prefix_rows=cap, format=fmt)
    O, lse = wf.prefix_attend(q, **dev, want_lse=True)
    z = want[1].double().exp()
    ref = want[0].double() * (z / (z + cap - n))[..., None]
    # both outputs rounded to bf16 and their weights too (half a step 2^-8 each, the
    # weights' of sum w |v| <= max |v|); fp32 sums of at most cap / 256 terms each
    sums = cap / 256 * 2.0 ** -24
    share_ = (z / (z + cap - n))[..., None]
    tol = (2 * 2.0 ** -8 * 1.01 + sums) * ref.abs() + 2 * 2.0 ** -8 * float(c["Vv"].abs().max()) * share_
    assert bool(((O.double() - ref).abs() <= tol).all())
    assert bool(((lse.double() - (z + cap - n).log()).abs() <= 20 * 2.0 ** -20 + sums).all())


@pytest.mark.parametrize("dtype,fmt,d", [("bf16", None, 128), ("bf16", "e4m3", 64),
                                         ("f32", None, 128), ("f32", None, 64)])
@pytest.mark.parametrize("share,group,B,T", [(1, 1, 1, 1), (2, 1, 1, 300), (1, 5, 1, 20),
                                             (2, 1, 33, 20), (3, 4, 10, 300), (1, 1, 200, 64)])
def test_few_units_of_a_long_prefix(wf, dtype, fmt, d, share, group, B, T):
    """Many ranges of the keys for few query rows, whose partials are merged by
    several workgroups of a sequence and several threads of a row; the same
    without own keys."""
    check(wf, *make(wf, dtype=dtype, fmt=fmt, d=d, share=share, heads=1, group=group, B=B,
                    P=7001, T=T, tlen=[T - i for i in range(share)]))
    check(wf, *make(wf, dtype=dtype, fmt=fmt, d=d, share=share, heads=1, group=group, B=B, P=7001))
