"""Attention of new rows over a cache in pages against the 64-bit reference."""
from __future__ import annotations

import math
import os
import subprocess
import sys

import pytest
import torch

import cacheref
import pageref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def wf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2606_00724_amd as wf
    return wf


class Case:
    """A pool, its sequences and their query rows, on the CPU."""

    def __init__(self, wf, *, lens, counts=None, rows=1, heads=2, group=1, d=64, P=16, dtype="bf16",
                 fmt=None, mask="tree", spare=0, seed=1, max_len=None, scale=0.0, pool_pages=None):
        g = torch.Generator().manual_seed(seed)
        b = len(lens)
        self.fmt, self.dtype, self.scale = fmt, dtype, scale or 1 / math.sqrt(d)
        tp = max(1, -(-max(max(lens), max_len or 0) // P))
        pages = pool_pages or b * tp + 2
        tokens = (b * rows if counts is None else sum(counts)) + spare
        self.p = wf.make_tree_params(pages=pages, page_rows=P, heads=heads, head_dim=d, batch=b,
                                     tokens=tokens, max_rows=rows, table_pages=tp, group=group,
                                     max_len=max_len, dtype=dtype, format=fmt,
                                     causal=mask == "causal", scale=scale)
        if pool_pages:                      # (sequences share pages)
            self.table = torch.randint(0, pages, (b, tp), generator=g).int()
        else:
            self.table = torch.randperm(pages, generator=g)[:b * tp].view(b, tp).int()
        for i, L in enumerate(lens):        # behind the last page: anything
            self.table[i, max(0, -(-L // P)):] = [-1, 2 ** 31 - 1, -2 ** 31, pages][i % 4]
        shape = (pages, heads, P)
        rowsof = [torch.randn(shape + (d,), generator=g) for _ in range(2)]
        self.pool = []
        for x in rowsof:
            if fmt is None:
                self.pool += [x.to(DT[dtype]), None]
            else:
                code, byte = cacheref.quantise(x, fmt)
                self.pool += [cacheref.pack(code, fmt), byte]
        self.Q = torch.randn((tokens, heads * group, d), generator=g).to(DT[dtype])
        self.len = torch.tensor(lens).int()
        self.start = None
        if counts is not None:
            self.start = torch.tensor([0] + counts).cumsum(0).int()
        self.mask = None
        if mask == "tree":
            w = (rows + 31) // 32
            self.mask = torch.randint(-2 ** 31, 2 ** 31 - 1, (tokens, w), generator=g).int()
            at = 0
            for i in range(b):
                n = rows if counts is None else counts[i]
                if i != 1:                  # (one sequence's masks are random bits)
                    self.mask[at:at + n] = 0
                    m = pageref.ancestors(n, seed + i) if n else torch.zeros((0, 1)).int()
                    self.mask[at:at + n, :m.shape[1]] = m
                at += n

    def run(self, wf, ws="own", stream=None):
        dev = [None if t is None else t.cuda() for t in self.pool]
        tok, hq, d = self.Q.shape
        O = torch.full((tok, hq, d), 7.0, dtype=self.Q.dtype, device="cuda")
        lse = torch.full((tok, hq), 7.0, device="cuda")
        up = [None if t is None else t.cuda() for t in (self.table, self.len, self.start,
                                                        self.mask)]
        w = wf.alloc_tree_workspace(self.p, "cuda") if ws == "own" else ws
        if w is not None:
            w.fill_(255)  # NaN
        wf.wf_tree_attn(self.p, self.Q.cuda(), *dev, *up, O, lse, w, stream)
        torch.cuda.synchronize()
        return O.cpu(), lse.cpu()

    def want(self):
        p = self.p
        return pageref.tree_attention(
            self.Q, self.pool, self.table, self.len, self.start, self.mask, page_rows=p.page_rows,
            heads=p.heads, group=p.group, max_rows=p.max_rows, max_len=p.max_len,
            scale=self.scale, causal=bool(p.causal), fmt=self.fmt)

    def check(self, got):
        O, lse = got
        wO, wl, tol, ltol = self.want()
        none = wl.isnan()                   # tokens of no sequence: as they were
        assert (O[none] == 7).all() and (lse[none] == 7).all()
        O, wO, tol = O[~none].double(), wO[~none], tol[~none]
        lse, wl, ltol = lse[~none].double(), wl[~none], ltol[~none]
        empty = wl == -math.inf
        assert (lse[empty] == -math.inf).all() and (O[empty] == 0).all()
        off = (lse - wl).abs()[~empty]
        assert (off <= ltol[~empty]).all(), f"lse off by {off.max()}"
        fine = wO.isfinite()
        assert (O[wO == math.inf] == math.inf).all() and (O[wO == -math.inf] == -math.inf).all()
        assert O[wO.isnan()].isnan().all()
        off = (O - wO).abs()
        assert (off[fine] <= tol[fine]).all(), \
            f"O off by {off[fine].max()}, {(off[fine] / tol[fine].clamp(min=1e-30)).max()} of the bound"


FORMATS = [("bf16", None), ("bf16", "e4m3"), ("bf16", "e2m1"), ("f32", None), ("f32", "e4m3"),
           ("f32", "e2m1")]


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("kw", [
    # single tokens, lengths around tiles and pages, empty and one
    dict(lens=[1, 0, 64, 65, 127, 700, 16, 33], mask="none", group=4),
    dict(lens=[300, 129], mask="none", d=128, P=64, heads=3),
    # trees over short and long contexts, rows of a page and more, ragged
    dict(lens=[40, 200, 513, 70], rows=24, counts=[24, 13, 0, 17], group=3, spare=5),
    dict(lens=[33, 300], rows=33, P=32, d=128, group=2),
    dict(lens=[600, 257, 255, 400], rows=256, counts=[256, 200, 255, 1], heads=1, d=128),
    # more new rows than the cache holds
    dict(lens=[5, 3, 0], rows=17, group=2),
    # blocks
    dict(lens=[100, 64, 31], rows=32, mask="all", d=128, P=256, group=4),
    dict(lens=[190, 77, 45], rows=45, mask="causal", counts=[45, 30, 44], P=64, group=2),
])
def test_tree(wf, dtype, fmt, kw):
    c = Case(wf, dtype=dtype, fmt=fmt, **kw)
    c.check(c.run(wf))


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
def test_long_caches_split_and_not(wf, dtype, fmt, d):
    """Ranges over a long cache of pages of every size, and no workspace: one
    range; both within the tolerance, equal parameters give equal bits."""
    for P, rows, mask in ((16, 1, "none"), (1024, 40, "tree")):
        c = Case(wf, lens=[5000, 3001], rows=rows, dtype=dtype, fmt=fmt, d=d, P=P, heads=1,
                 mask=mask, group=2)
        assert wf.tree_plan(c.p).ranges > 1
        a = c.run(wf)
        c.check(a)
        b = c.run(wf)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        assert wf.tree_plan(c.p, 0).ranges == 1
        c.check(c.run(wf, ws=None))


def test_pages_of_more_keys_than_are_in_lds_at_once(wf):
    """One range of 70000 keys in pages of 16: their numbers are loaded three
    times."""
    for fmt in (None, "e4m3"):
        for rows, mask in ((1, "none"), (150, "causal")):
            c = Case(wf, lens=[70000], rows=rows, heads=1, P=16, mask=mask, d=64, fmt=fmt)
            c.check(c.run(wf, ws=None))


def poison(c, where, fmt, rows):
    """NaN and infinities in three new rows of each sequence (of `rows` at
    least), in rows behind the last one, and in the pages of no sequence."""
    m, P = 0 if where == "K" else 2, c.p.page_rows
    x = c.pool[m] if fmt is None else c.pool[m + 1]
    bad, used = 255 if fmt else math.nan, set()
    for b, L in enumerate(c.len.tolist()):
        used |= {int(c.table[b, t]) for t in range(-(-L // P))}
    for b, L in enumerate(c.len.tolist()):
        if L == 0:
            continue
        for t in range(L, -(-L // P) * P):
            x[int(c.table[b, t // P]), :, t % P] = bad
        for j, v in ((2, math.inf), (5, math.nan), (7, -math.inf)):
            t = L - rows + j
            row = x[int(c.table[b, t // P]), :, t % P]
            row[:, 1 if fmt else 40] = 255 if fmt else v
            if where == "V" and fmt is None:
                row[:, 41] = math.inf
            if where == "V" and fmt == "e4m3":      # a code of NaN, too
                c.pool[2][int(c.table[b, t // P]), :, t % P, 3] = 0x7f
    for page in range(c.p.pages):
        if page not in used:
            x[page] = bad


def check_poisoned(c, got, where):
    """As check; for keys: rows that see a NaN key are NaN, the others as ever."""
    if where == "V":
        return c.check(got)
    O, lse = got
    wO, wl, tol, ltol = c.want()
    clean = wl.isfinite() & ~wO.isnan().any(-1)
    assert 5 < int(clean.sum()) < clean.numel() - 5
    assert ((O.double() - wO).abs() <= tol)[clean].all()
    assert ((lse.double() - wl).abs() <= ltol)[clean].all()
    dirty = wl.isnan() & (O != 7).any(-1)
    assert lse[dirty].isnan().all()


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("where", ["K", "V"])
def test_hidden_rows_may_hold_anything(wf, dtype, fmt, where):
    for group in (1, 20):
        c = Case(wf, lens=[90, 70, 64], rows=9, dtype=dtype, fmt=fmt, d=128, group=group, P=16,
                 seed=3)
        poison(c, where, fmt, 9)
        check_poisoned(c, c.run(wf), where)


# sequences, K/V heads, most rows, group, most keys, channels -> query rows of a
# workgroup, with several ranges of the keys or one (the lengths are far below)
FORMS = [(16, 2, 17, 3, 16000, 128, 64, True), (32, 8, 21, 3, 8000, 64, 64, False),
         (16, 1, 33, 2, 16000, 64, 128, True), (64, 1, 100, 3, 300, 128, 128, False),
         (16, 2, 64, 3, 16000, 128, 256, True), (16, 8, 100, 3, 300, 64, 256, False)]


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("b,h,rows,g,most,d,block,ranges", FORMS)
@pytest.mark.parametrize("bad", [None, "K", "V"])
def test_every_form_of_the_kernel_of_many_rows(wf, dtype, fmt, b, h, rows, g, most, d, block,
                                               ranges, bad):
    lens, counts = [0] * b, [0] * b
    for i, (L, n) in enumerate(((290, rows), (130, 9), (300, 12))):
        lens[5 * i], counts[5 * i] = L, n
    c = Case(wf, lens=lens, counts=counts, rows=rows, heads=h, group=g, d=d, P=16, dtype=dtype,
             fmt=fmt, max_len=most, pool_pages=60, seed=4)
    s = wf.tree_plan(c.p)
    if dtype == "bf16":
        assert (s.group_rows, s.ranges > 1) == (block, ranges)
    if bad:
        c.table = (torch.randperm(57)[:57].repeat(b * 20)[:b * c.table.shape[1]]
                   .view(b, -1) % 57).int()
        for i in (0, 5, 10):                # their own pages, and three of nobody's
            c.table[i, :19] = torch.arange(19).int() + 19 * (i // 5)
        poison(c, bad, fmt, 9)
    got = c.run(wf)
    check_poisoned(c, got, bad) if bad else c.check(got)


def test_strides_of_fused_rows(wf):
    """Queries as slices of a fused projection, outputs into a wider row."""
    c = Case(wf, lens=[100, 60], rows=5, group=2)
    base = c.run(wf)
    tok, hq, d = c.Q.shape
    x = torch.zeros((tok, hq + 3, d), dtype=torch.bfloat16, device="cuda")
    x[:, 1:1 + hq] = c.Q.cuda()
    o = torch.full((tok, hq + 2, d), 7.0, dtype=torch.bfloat16, device="cuda")
    c.p.q_row, c.p.o_row = x.stride(0), o.stride(0)
    wf.wf_tree_attn(c.p, x[:, 1:1 + hq], *[t if t is None else t.cuda() for t in c.pool],
                    c.table.cuda(), c.len.cuda(), None, c.mask.cuda(), o[:, 2:], None,
                    wf.alloc_tree_workspace(c.p, "cuda"))
    assert torch.equal(o[:, 2:].cpu(), base[0]) and (o[:, :2] == 7).all()


def test_lengths_and_starts_outside_are_taken_as_the_nearest_inside(wf):
    c = Case(wf, lens=[100, 60, 80], rows=4, counts=[4, 3, 4], max_len=96)
    for lens, start in (([2 ** 31 - 1, -5, 50], [0, 4, 7, 11]), ([90, 60, 70], [-2, 2, 5, 40]),
                        ([90, 60, 70], [0, 4, 2, 2 ** 31 - 1]),
                        ([50, 60, 96], [-2 ** 31, 2 ** 31 - 1, 5, 6])):
        c.len, c.start = torch.tensor(lens).int(), torch.tensor(start).int()
        got = c.run(wf)
        owners = [0] * 11
        for b in range(3):
            n = min(max(start[b + 1] - start[b], 0), 4)
            for i in range(n):
                if 0 <= start[b] + i < 11:
                    owners[start[b] + i] += 1
        if max(owners) <= 1:                # (else two sequences write one row)
            c.check(got)


def test_scales_of_either_sign_and_far_scores(wf):
    for scale in (-0.125, 40.0, 1e-3):
        c = Case(wf, lens=[200, 90], rows=20, scale=scale, dtype="f32", d=64)
        c.check(c.run(wf))


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("scale", [-0.125, 40.0, 1e-39])
def test_scales_in_every_kernel(wf, dtype, fmt, scale):
    for rows, lens in ((1, [200, 90, 5]), (12, [200, 90, 5]), (150, [260, 170])):
        c = Case(wf, lens=lens, rows=rows, scale=scale, dtype=dtype, fmt=fmt, d=128, group=2,
                 heads=1)
        c.check(c.run(wf))


def test_a_pool_past_two_to_the_32_bytes(wf):
    """Pages whose rows lie behind 2^32 bytes of K (2^21 rows of 8 heads)."""
    heads, d, P = 8, 128, 64
    pages = (1 << 21) // P + 3
    K = torch.zeros((pages, heads, P, d), dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    c = Case(wf, lens=[100, 150], rows=3, heads=heads, d=d, P=P)
    far = torch.arange(c.p.pages) % 2 * 7 + pages - 2 * c.p.pages + torch.arange(c.p.pages)
    K[far.cuda()], V[far.cuda()] = c.pool[0].cuda(), c.pool[2].cuda()
    base = c.run(wf)
    c.check(base)
    table = torch.where((c.table >= 0) & (c.table < c.p.pages),
                        far[c.table.clamp(0, c.p.pages - 1).long()].int(), c.table)
    c.p.pages = pages
    O, lse = wf.tree_attend(c.p, c.Q.cuda(), (K, None, V, None), table.cuda(), c.len.cuda(), None,
                            c.mask.cuda(), want_lse=True)
    assert torch.equal(O.cpu(), base[0]) and torch.equal(lse.cpu(), base[1])


def test_decoding_steps_in_a_graph(wf):
    """A loop as a program runs it: drafted rows appended, attended, the
    accepted branch moved, captured once and replayed with new rows, lengths,
    pages and masks, against the reference step by step."""
    heads, group, d, P, b, n = 2, 3, 64, 16, 3, 8
    hq, tp = heads * group, 12
    pages, tok = b * tp + 1, b * n
    pa = wf.make_append_params(pages=pages, page_rows=P, heads=heads, head_dim=d, tokens=tok,
                               group=group, format="e4m3")
    pt = wf.make_tree_params(pages=pages, page_rows=P, heads=heads, head_dim=d, batch=b,
                             max_rows=n, table_pages=tp, group=group, format="e4m3")
    pm = wf.make_move_params(pages=pages, page_rows=P, heads=heads, head_dim=d, batch=b,
                             table_pages=tp, moves=4, format="e4m3")
    pool = pageref.pool_like(wf, pa, 5)
    pool[1], pool[3] = (x % 8 + 120 for x in (pool[1], pool[3]))
    freq = pageref.frequencies(d // 2)
    dev = [x.cuda() for x in pool]
    buf = dict(Q=torch.zeros((tok, hq, d)).bfloat16(), K=torch.zeros((tok, heads, d)).bfloat16(),
               V=torch.zeros((tok, heads, d)).bfloat16(), pos=torch.zeros((1, tok)).int(),
               slot=torch.full((tok,), -1).int(), table=torch.zeros((b, tp)).int(),
               len=torch.zeros(b).int(), mask=torch.zeros((tok, 1)).int(),
               first=torch.zeros(b).int(), source=torch.full((b, 4), -1).int())
    G = {k: v.cuda() for k, v in buf.items()}
    gf, O = freq.cuda(), torch.zeros((tok, hq, d), dtype=torch.bfloat16, device="cuda")
    Qr, lse = torch.zeros_like(O), torch.zeros((tok, hq), device="cuda")
    ws = wf.alloc_tree_workspace(pt, "cuda")

    def step():
        wf.wf_page_append(pa, G["Q"], G["K"], G["V"], G["pos"], gf, G["slot"], *dev, Qr)
        wf.wf_tree_attn(pt, Qr, *dev, G["table"], G["len"], None, G["mask"], O, lse, ws)
        wf.wf_page_move(pm, G["table"], G["first"], G["source"], *dev)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    for x, y in zip(dev, pool):
        x.copy_(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    g = torch.Generator().manual_seed(9)
    table = torch.randperm(pages, generator=g)[:b * tp].view(b, tp).int()
    ctx = [0, 77, 150]
    for it in range(5):
        new = {k: torch.randn(buf[k].shape, generator=g).bfloat16() for k in ("Q", "K", "V")}
        mask = torch.cat([pageref.ancestors(n, 10 * it + i) for i in range(b)])
        at = torch.tensor([[c + i for i in range(n)] for c in ctx])
        slot = torch.stack([table[i, at[i] // P] * P + at[i] % P for i in range(b)]).int()
        pos = at.int().view(1, tok)
        source = torch.tensor([[0, 2, 5, -1], [1, 3, 4, 7], [0, 1, -1, -1]]).roll(it, 0).int()
        now = dict(new, pos=pos, slot=slot.view(-1), table=table, mask=mask, source=source,
                   len=torch.tensor([c + n for c in ctx]).int(), first=torch.tensor(ctx).int())
        for k, v in now.items():
            G[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        c, sn = pageref.turn(pos, freq, [0] * (d // 2))
        K = pageref.rotate(new["K"], c[:, None], sn[:, None])
        q = pageref.rotate(new["Q"], c[:, None], sn[:, None]).to(torch.bfloat16)
        assert torch.equal(Qr.cpu(), q)
        pool = pageref.append(pool, "e4m3", torch.bfloat16, K, new["V"].float(), slot.view(-1), P)
        case = Case.__new__(Case)
        case.p, case.Q, case.pool, case.table, case.len = pt, q, pool, table, now["len"]
        case.start, case.mask, case.scale, case.fmt = None, mask, 1 / math.sqrt(d), "e4m3"
        case.check((O.cpu(), lse.cpu()))
        pool = pageref.move(pool, table, now["first"], source, P)
        for name, x, y in zip(("Kc", "Kx", "Vc", "Vx"), dev, pool):
            assert torch.equal(x.cpu(), y), name
        ctx = [c + int((source[i] >= 0).sum()) for i, c in enumerate(ctx)]
        (Qr.float() * 2).sum()  # eager work between the replays


def test_two_streams_at_once(wf):
    cases = [Case(wf, lens=[900, 1100], rows=rows, group=2, fmt=fmt, seed=seed)
             for rows, fmt, seed in ((1, None, 1), (30, "e4m3", 2))]
    alone = [c.run(wf) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    dev = []
    for c in cases:
        dev.append([[t if t is None else t.cuda() for t in c.pool], c.Q.cuda(), c.table.cuda(),
                    c.len.cuda(), c.mask.cuda()])
    torch.cuda.synchronize()
    outs = []
    for _ in range(4):
        for c, s, (pool, Q, table, length, mask) in zip(cases, streams, dev):
            outs.append((c, wf.tree_attend(c.p, Q, pool, table, length, None, mask, want_lse=True,
                                           stream=s)))
    torch.cuda.synchronize()
    for c, (O, lse) in outs:
        want = alone[cases.index(c)]
        assert torch.equal(O.cpu(), want[0]) and torch.equal(lse.cpu(), want[1])


@pytest.mark.parametrize("dtype,fmt", FORMATS)
def test_a_batch_of_many_sequences(wf, dtype, fmt):
    """Single tokens of 700 sequences that share pages, empty ones among them, with
    an odd group of heads."""
    g = torch.Generator().manual_seed(7)
    lens = torch.randint(-20, 90, (700,), generator=g).clamp(min=0).tolist()
    c = Case(wf, lens=lens, group=7, mask="none", d=128, dtype=dtype, fmt=fmt, pool_pages=31)
    c.check(c.run(wf))


@pytest.mark.parametrize("dtype,fmt", FORMATS)
def test_lengths_far_below_the_most(wf, dtype, fmt):
    """Ranges that no sequence reaches are empty."""
    for rows, mask in ((1, "none"), (60, "tree")):
        c = Case(wf, lens=[70, 0, 2500], rows=rows, mask=mask, P=64, max_len=400000, dtype=dtype,
                 fmt=fmt, pool_pages=50)
        assert wf.tree_plan(c.p).ranges > 8
        c.check(c.run(wf))


@pytest.mark.parametrize("dtype,fmt", FORMATS)
def test_many_heads_of_a_group(wf, dtype, fmt):
    c = Case(wf, lens=[300, 77], rows=256, counts=[256, 3], heads=1, group=32, dtype=dtype,
             fmt=fmt)
    c.check(c.run(wf))
    c = Case(wf, lens=[90, 5], rows=3, heads=2, group=71, dtype=dtype, fmt=fmt, d=128)
    c.check(c.run(wf))


def test_two_graphs_share_a_workspace(wf):
    """Calls of other shapes, captured each in a graph, leave their partials in one
    workspace and take no notice of what stands in it."""
    cases = [Case(wf, lens=[900, 1500], rows=rows, group=2, fmt=fmt, heads=1, seed=rows)
             for rows, fmt in ((1, None), (40, None), (20, "e2m1"))]
    want = [c.run(wf) for c in cases]
    assert all(wf.tree_plan(c.p).ranges > 1 for c in cases)
    ws = torch.empty(max(wf.tree_workspace_bytes(c.p) for c in cases), dtype=torch.uint8,
                     device="cuda")
    s = torch.cuda.Stream()
    graphs, outs, keep = [], [], []
    for c, (O, lse) in zip(cases, want):
        up = [t if t is None else t.cuda() for t in c.pool + [c.table, c.len, None, c.mask]]
        out = (torch.zeros_like(O, device="cuda"), torch.zeros_like(lse, device="cuda"))
        Q = c.Q.cuda()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            # (the whole workspace: the split is of the parameters, not of its size)
            wf.wf_tree_attn(c.p, Q, *up, *out, ws)
        graphs.append(graph)
        outs.append(out)
        keep.append((up, Q))
    for i in (0, 1, 2, 1, 0, 2, 2, 0):
        for x in outs[i]:
            x.fill_(7)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x.cpu(), y) for x, y in zip(outs[i], want[i]))
        ws.random_(0, 256)  # eager work between the replays


FRESH = """
import torch
import paper_2606_00724_amd as wf
wf.wf_init()
g = torch.Generator().manual_seed(1)
for rows in (1, 250):
    p = wf.make_tree_params(pages=40, page_rows=64, heads=2, head_dim=128, batch=1,
                            max_rows=rows, table_pages=40, group=16, causal=True)
    Q, K, V = (torch.randn(s, generator=g).bfloat16().cuda()
               for s in ((rows, 32, 128), (40, 2, 64, 128), (40, 2, 64, 128)))
    table = torch.arange(40, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
    length = torch.tensor([2500], dtype=torch.int32, device="cuda")
    assert wf.tree_plan(p).group_rows == (16 if rows == 1 else 128)
    ws, O = wf.alloc_tree_workspace(p, "cuda"), torch.zeros_like(Q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wf.wf_tree_attn(p, Q, K, None, V, None, table, length, None, None, O, None, ws)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(O, wf.tree_attend(p, Q, (K, None, V, None), table, length))
    assert O.abs().sum() > 0
print("done")
"""


def test_first_calls_of_a_process_may_be_captured(wf):
    """After wf_init nothing is left to load: each kernel's first launch is captured."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", FRESH], cwd=root, capture_output=True, text=True,
                         timeout=100)
    assert run.returncode == 0 and "done" in run.stdout, run.stderr
