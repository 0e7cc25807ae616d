"""Performance cases of a paged cache: rotary positions, rows appended, rows moved, and the
attention of newly drafted rows over it.

A case is one call that a decoder makes for one layer: queries or keys rotated by positions of one
or several axes (rope), the rows of new tokens rotated and written into the pages of a cache
(append), the accepted rows of a tree of drafted tokens brought together behind their context
(move), and the attention of such a tree, of a block of rows that see each other, or of single
tokens (tree).  Sizes follow the workloads of synth.WORKLOADS; keys are AR(1) sequences with planted
16-token needles towards which the queries lean, as there, drawn on the GPU.  With `own` the
library's entry points run, otherwise the same operators in elementary torch operations on 32-bit
values (angles in 64).

A cache is a pool of pages, [pages][heads][page_rows][d] each for K and V; a sequence's row t is in
page table[t // page_rows].  The formats of its rows: the call's type, or blocks of 32 consecutive
channels of a row that share a power of two 2^(byte - 127), the smallest one (byte >= 1) with which
the block's largest magnitude is at most 448 (e4m3) or 6 (e2m1); the codes are the channels divided
by it, rounded to the nearest, ties to even.
"""
from __future__ import annotations

import math

import torch

own = False

_NEEDLE = 16
_TOP = {"e4m3": 448.0, "e2m1": 6.0}     # largest code of a format
_BITS = {"e4m3": 8, "e2m1": 4, "none": 0}
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # the queries of one denoising step's block of 32 rows, far into a text; latency
        _rope("rope_block", batch=1, heads=32, rows=32, d=128),
        # the queries of four videos (frames of 16 x 32 patches), slices of the fused projection
        _rope("rope_video8k", batch=4, heads=32, rows=8192, d=128, axes=3, fused=True),
        # single tokens of 64 sequences appended, their queries rotated beside; latency
        _append("append_token64", tokens=64, heads=8, group=4, d=128, P=16),
        # fp32 rows of a small model, adjacent pairs of half the channels, padded, kept in 4 bits
        _append("append_f32_odd", tokens=517, heads=3, group=1, d=64, P=32, rot=32, pairs=True,
                padded=True, dtype="f32", fmt="e2m1"),
        # a 32K prompt of text, images and video appended at once, kept in 8 bits
        _append("append_prompt32k", tokens=32768, heads=8, group=4, d=128, P=64, axes=3,
                fused=True, fmt="e4m3"),
        # six accepted of 64 drafted rows of 32 sequences brought together; latency
        _move("move_draft", batch=32, heads=8, d=128, P=16, L=4096, rows=64, moves=6),
        # blocks of 256 rows of 128 sequences, 64 of them kept
        _move("move_block256", batch=128, heads=8, d=128, P=64, L=4096, rows=256, moves=64,
              fmt="e4m3"),
        # one sequence's 24 drafted rows over a 4K context; latency
        _tree("tree_draft4k", batch=1, heads=8, group=4, rows=24, d=128, P=16, L=4096, lse=True),
        # single tokens of 64 sequences of up to 8K rows, ragged
        _tree("tree_token8k", batch=64, heads=8, group=4, rows=1, d=128, P=16, L=8192,
              ragged=True),
        # single tokens of 32 sequences of up to 32K rows kept in 8 bits, ragged
        _tree("tree_token32k_e4m3", batch=32, heads=8, group=4, rows=1, d=128, P=64, L=32768,
              ragged=True, fmt="e4m3"),
        # 64 drafted rows of each of 16 sequences over 16K contexts
        _tree("tree_draft16k", batch=16, heads=8, group=4, rows=64, d=128, P=64, L=16384),
        # two sequences' blocks of 32 rows that see each other, over 128K rows kept in 4 bits
        _tree("tree_block128k_e2m1", batch=2, heads=8, group=4, rows=32, d=128, P=256, L=131072,
              mask="all", fmt="e2m1", lse=True),
    ]


def _named(c, name):
    if name is not None:
        c["name"] = name
    return c


def _rope(name, *, batch, heads, rows, d, rot=0, axes=1, pairs=False, fused=False, dtype="bf16"):
    """rot: channels rotated (0: all); pairs: adjacent channels are rotated together, not halves;
    fused: rows are slices [batch][rows][heads][d] of a projection that holds more heads."""
    return _named(dict(kind="rope", batch=batch, heads=heads, rows=rows, d=d, rot=rot or d,
                       axes=axes, pairs=pairs, fused=fused, dtype=dtype), name)


def _append(name, *, tokens, heads, group, d, P, rot=0, axes=1, pairs=False, fused=False,
            padded=False, dtype="bf16", fmt="none"):
    """group: query heads per K/V head, 0 for no queries; P: rows of a page; padded: the last
    tokens have no row."""
    return _named(dict(kind="append", tokens=tokens, heads=heads, group=group, d=d, P=P,
                       rot=rot or d, axes=axes, pairs=pairs, fused=fused, padded=padded,
                       dtype=dtype, fmt=fmt), name)


def _move(name, *, batch, heads, d, P, L, rows, moves, dtype="bf16", fmt="none"):
    """moves of the last `rows` rows of a sequence, of L rows at most, are kept."""
    return _named(dict(kind="move", batch=batch, heads=heads, d=d, P=P, L=L, rows=rows,
                       moves=moves, dtype=dtype, fmt=fmt), name)


def _tree(name, *, batch, heads, group, rows, d, P, L, mask="tree", ragged=False, lse=False,
          dtype="bf16", fmt="none", rho=0.98):
    """rows: new rows of a sequence, L: rows of its cache, these among them (ragged: at most);
    mask: which new rows a new row sees (its ancestors in a tree, those up to it, or all)."""
    return _named(dict(kind="tree", batch=batch, heads=heads, group=group, rows=rows, d=d, P=P,
                       L=L, mask=mask, ragged=ragged, lse=lse, dtype=dtype, fmt=fmt, rho=rho),
                  name)


def _log(rng, lo, hi):
    return int(round(2 ** rng.uniform(math.log2(lo), math.log2(hi))))


def draw(rng):
    kind = rng.choice(["rope", "append", "append", "move", "tree", "tree", "tree", "tree"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    d = rng.choice([64, 128, 128])
    P = rng.choice([16, 16, 32, 64, 128, 256])
    fmt = rng.choice(["none", "none", "e4m3", "e4m3", "e2m1"])
    turn = dict(rot=rng.choice([d, d, d, d // 2, 48]), axes=rng.choice([1, 1, 2, 3]),
                pairs=rng.random() < 0.3, fused=rng.random() < 0.5)
    if kind == "rope":
        batch, heads = rng.choice([1, 1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 8, 32, 40])
        most = (1 << 27) // (batch * heads * d) // (2 if dtype == "f32" else 1)
        return _rope(None, batch=batch, heads=heads, rows=_log(rng, 1, min(32768, most)), d=d,
                     dtype=dtype, **turn)
    if kind == "append":
        heads, group = rng.choice([(1, 8), (2, 1), (3, 1), (8, 1), (8, 4), (8, 0), (4, 7), (32, 1)])
        most = (1 << 27) // (heads * (group + 2) * d) // (2 if dtype == "f32" else 1)
        return _append(None, tokens=_log(rng, 1, min(32768, most)), heads=heads, group=group, d=d,
                       P=P, padded=rng.random() < 0.3, dtype=dtype, fmt=fmt, **turn)
    if kind == "move":
        rows = _log(rng, 2, 256)
        return _move(None, batch=_log(rng, 1, 128), heads=rng.choice([1, 3, 8, 8]), d=d, P=P,
                     L=_log(rng, max(300, rows), 4096), rows=rows,
                     moves=max(1, min(rows // 2, _log(rng, 1, 64))), dtype=dtype, fmt=fmt)
    heads, group = rng.choice([(2, 1), (3, 1), (8, 1), (8, 4), (8, 8), (4, 7), (1, 16), (32, 1)])
    rows = rng.choice([1, 1, 1, 4, 5, 8, 17, 24, 32, 45, 64, 100, 256])
    c = _tree(None, batch=_log(rng, 1, 64), heads=heads, group=group, rows=rows, d=d, P=P,
              L=_log(rng, 256, 131072), mask=rng.choice(["tree", "tree", "causal", "all"]),
              ragged=rng.random() < 0.6, lse=rng.random() < 0.4, dtype=dtype, fmt=fmt,
              rho=rng.choice([0.95, 0.98, 0.99]))
    # at most the largest listed cases' products (an eighth of them in fp32), elements and scores
    most = 2.7e11 / (8 if dtype == "f32" else 1)
    while (work(c)["flops"] > most
           or c["batch"] * heads * c["L"] * d > 1 << (28 if dtype == "f32" else 29)
           or c["batch"] * heads * group * rows * c["L"] > 1 << 29):
        if c["batch"] == 1 or c["L"] > 4096 and rng.random() < 0.5:
            c["L"] = max(256, c["L"] * 2 // 3)
        else:
            c["batch"] = c["batch"] * 2 // 3
    return c


# ------------------------------------------------------------ inputs

def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _gen(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * int(seed) + 31)
    return gen


def _rand(gen, shape, dtype):
    """Normal numbers of a large tensor, a part at a time in 32 bits."""
    x = torch.empty(shape, dtype=dtype, device="cuda")
    for part in x.view(-1).split(1 << 26):
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda"))
    return x


def _ints(gen, lo, hi, shape):
    """Whole numbers lo .. hi - 1."""
    return torch.randint(lo, hi, shape, generator=gen, device="cuda", dtype=torch.int32)


def _keys(gen, units, L, d, rho, u):
    """AR(1) sequences [units, L, d] with two needles each along u [units, 1, d]."""
    x = torch.randn((units, L, d), generator=gen, device="cuda")
    x[:, 1:] *= math.sqrt(1 - rho * rho)
    s = 1
    while s < L and rho ** s > 1e-6:  # by doubling
        x[:, s:] += rho ** s * x[:, :-s].clone()
        s *= 2
    x += 0.3 * torch.randn((units, L, d), generator=gen, device="cuda")
    for start in (L // 3, 2 * L // 3):
        x[:, start:start + _NEEDLE] += 3.0 * u
    return x


def _sections(c):
    """Pairs of each axis: a quarter in time and the rest in height and width, or equal parts."""
    n, a = c["rot"] // 2, c["axes"]
    if a == 1:
        return [n]
    if a == 3:
        return [n // 4, (n - n // 4) // 2, n - n // 4 - (n - n // 4) // 2]
    return [n // 2, n - n // 2]


def _turns(c, gen, seqs, rows):
    """Positions [axes][seqs][rows] and the pairs' frequencies."""
    t = torch.arange(rows, device="cuda", dtype=torch.int32) + _ints(gen, 0, 100000, (seqs, 1))
    pos = [t]
    if c["axes"] > 1:                       # patches of 16 x 32, frame after frame
        at = torch.arange(rows, device="cuda", dtype=torch.int32).expand(seqs, -1)
        pos = [t[:, :1] + at // 512, at // 32 % 16, at % 32]
        pos = pos[3 - c["axes"]:]
    n = c["rot"] // 2
    f = 10000.0 ** (-torch.arange(n, device="cuda", dtype=torch.float64) / n)
    return torch.stack(pos).contiguous(), f.float()


def _pool(c, gen, pages):
    """Pages in use: rows of earlier steps."""
    shape, st = (pages, c["heads"], c["P"]), {}
    for m in ("K", "V"):
        if c["fmt"] == "none":
            st[m + "c"], st[m + "x"] = _rand(gen, shape + (c["d"],), _dtype(c)), None
        else:  # (without the e4m3 code of NaN)
            st[m + "c"] = torch.randint(0, 256, shape + (c["d"] * _BITS[c["fmt"]] // 8,),
                                        generator=gen, device="cuda", dtype=torch.uint8) & 0xf7
            st[m + "x"] = torch.randint(116, 126, shape + (c["d"] // 32,), generator=gen,
                                        device="cuda", dtype=torch.uint8)
    return st


def _tables(c, gen, length):
    """A sequence's pages, anywhere in the pool; entries behind its last page are -1.  Returns the
    table and the pool's size (some pages belong to nobody)."""
    b, tp = c["batch"], -(-c["L"] // c["P"])
    pages = b * tp + 3
    table = torch.randperm(pages, generator=gen, device="cuda")[:b * tp].view(b, tp)
    used = torch.arange(tp, device="cuda") * c["P"] < length.unsqueeze(1)
    return torch.where(used, table, -1).to(torch.int32).contiguous(), pages


def _sees(c, gen, counts):
    """[batch][rows][rows] truth values: which new row a new row sees."""
    b, n = c["batch"], c["rows"]
    if c["mask"] == "all":
        return torch.ones((b, n, n), dtype=torch.bool, device="cuda")
    if c["mask"] == "causal":
        return torch.ones((n, n), dtype=torch.bool, device="cuda").tril().expand(b, n, n)
    parent = (torch.rand((b, n), generator=gen, device="cuda")
              * torch.arange(n, device="cuda")).long().cpu()
    seen = torch.zeros((b, n, n), dtype=torch.bool)
    at = torch.arange(b)
    for i in range(n):
        if i:
            seen[:, i] = seen[at, parent[:, i]]
        seen[:, i, i] = True
    return seen.cuda()


def _words(seen):
    """The truth values [..., n] as bits of 32-bit words."""
    n = seen.shape[-1]
    bits = torch.nn.functional.pad(seen, (0, -n % 32)).unflatten(-1, (-1, 32)).long()
    w = (bits << torch.arange(32, device=seen.device)).sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def prepare(case, seed):
    c = case
    gen = _gen(seed)
    dt, d = _dtype(c), c["d"]
    st = dict(case=c)
    if c["kind"] == "rope":
        b, h, n = c["batch"], c["heads"], c["rows"]
        if c["fused"]:
            st["X"] = _rand(gen, (b, n, h + 4, d), dt)[:, :, :h].transpose(1, 2)
            st["Y"] = torch.empty((b, n, h, d), dtype=dt, device="cuda").transpose(1, 2)
        else:
            st["X"] = _rand(gen, (b, h, n, d), dt)
            st["Y"] = torch.empty_like(st["X"])
        st["pos"], st["freq"] = _turns(c, gen, b, n)
    elif c["kind"] == "append":
        n, h, hq = c["tokens"], c["heads"], c["heads"] * c["group"]
        if c["fused"]:
            x = _rand(gen, (n, hq + 2 * h, d), dt)
            q, st["K"], st["V"] = x.split([hq, h, h], dim=1)
        else:
            q, st["K"], st["V"] = (_rand(gen, (n, k, d), dt) for k in (hq, h, h))
        st["Q"], st["Qr"] = (q, torch.empty((n, hq, d), dtype=dt, device="cuda")) if hq else (None,
                                                                                              None)
        pos, st["freq"] = _turns(c, gen, 1, n)
        st["pos"] = pos.view(c["axes"], n)
        pages = -(-n // c["P"]) * 5 // 4 + 2
        st |= _pool(c, gen, pages)
        # whole pages anywhere in the pool, from some row of the first one on
        page = torch.randperm(pages, generator=gen, device="cuda")
        t = torch.arange(n, device="cuda") + _ints(gen, 0, c["P"], (1,)).long()
        slot = page[t // c["P"]] * c["P"] + t % c["P"]
        if c["padded"]:
            slot[max(1, n - n // 8):] = -1
        st["slot"] = slot.to(torch.int32)
    elif c["kind"] == "move":
        b, n, k = c["batch"], c["rows"], c["moves"]
        length = _ints(gen, n, c["L"] + 1, (b,))
        st["table"], pages = _tables(c, gen, length)
        st |= _pool(c, gen, pages)
        st["first"] = length - n
        # the root stays, the others come from behind the rows that are written (a pass can be
        # repeated); some sequences keep fewer
        src = torch.rand((b, n - k), generator=gen, device="cuda").argsort(dim=1)[:, :k] + k
        src = src.sort(dim=1).values.to(torch.int32)
        src[:, 0] = 0
        kept = _ints(gen, k // 2 + 1, k + 1, (b, 1))
        st["src"] = torch.where(torch.arange(k, device="cuda") < kept, src, -1).contiguous()
    else:
        st |= _prepare_tree(c, gen)
    if own:  # what a serving loop keeps: the parameters and the workspace
        st |= _kept(c, st)
    return st


def _prepare_tree(c, gen):
    b, h, g, n, d, P, L = (c[k] for k in ("batch", "heads", "group", "rows", "d", "P", "L"))
    dt, st = _dtype(c), {}
    counts = torch.full((b,), n, dtype=torch.int32, device="cuda")
    length = torch.full((b,), L, dtype=torch.int32, device="cuda")
    if c["ragged"]:
        length = _ints(gen, max(1, L // 2), L + 1, (b,))
        counts = torch.minimum(_ints(gen, (n + 1) // 2, n + 1, (b,)), length)
    st["start"] = None
    tokens = b * n
    if c["ragged"] and n > 1:       # the sequences' rows after each other, a batch of fixed size
        st["start"] = torch.nn.functional.pad(counts.cumsum(0), (1, 0)).to(torch.int32)
    st["counts"], st["len"] = counts, length
    st["table"], pages = _tables(c, gen, length)
    st |= _pool(c, gen, pages)
    u = torch.randn((b, h, 1, d), generator=gen, device="cuda")
    u /= u.norm(dim=-1, keepdim=True)
    tp = st["table"].shape[1]
    for i in range(b):
        used = -(-int(length[i]) // P)
        at = st["table"][i, :used].long()
        K = _keys(gen, h, tp * P, d, c["rho"], u[i])[:, :used * P]
        V = torch.randn((h, used * P, d), generator=gen, device="cuda")
        for m, x in (("K", K), ("V", V)):
            if c["fmt"] == "none":
                st[m + "c"][at] = x.view(h, used, P, d).transpose(0, 1).to(dt)
            else:
                codes, byte = _quantise(x, c["fmt"])
                st[m + "c"][at] = codes.view(h, used, P, -1).transpose(0, 1)
                st[m + "x"][at] = byte.view(h, used, P, -1).transpose(0, 1)
    z = torch.randn((b, n, h, g, d), generator=gen, device="cuda")
    z = (z / math.sqrt(d) + 2.0 * u.view(b, 1, h, 1, d)).to(dt).view(b, n, h * g, d)
    seen = _sees(c, gen, counts)
    words = _words(seen) if c["mask"] == "tree" else None
    st["Q"] = torch.zeros((tokens, h * g, d), dtype=dt, device="cuda")
    st["mask"] = words
    live = torch.arange(n, device="cuda") < counts.unsqueeze(1)
    if st["start"] is None:
        st["Q"].copy_(z.view(tokens, h * g, d))
        if words is not None:
            st["mask"] = words.view(tokens, -1).contiguous()
    else:
        k = int(st["start"][-1])
        st["Q"][:k] = z[live]
        if words is not None:
            st["mask"] = torch.zeros((tokens, words.shape[-1]), dtype=torch.int32, device="cuda")
            st["mask"][:k] = words[live]
    st["seen"] = seen               # (for the plain form, which reads it in place of the bits)
    st["O"] = torch.zeros_like(st["Q"])
    st["lse"] = (torch.zeros((tokens, h * g), dtype=torch.float32, device="cuda")
                 if c["lse"] else None)
    return st


def _kept(c, st):
    import paper_2606_00724_amd as wf
    wf.wf_init()
    if c["kind"] == "rope":
        p = wf.make_rope_params(batch=c["batch"], heads=c["heads"], rows=c["rows"],
                                head_dim=c["d"], rot_dim=c["rot"], sections=_sections(c),
                                layout="pairs" if c["pairs"] else "halves", dtype=c["dtype"],
                                x_strides=st["X"].stride()[:3], y_strides=st["Y"].stride()[:3])
        return dict(wf=wf, p=p)
    pool = dict(pages=st["Kc"].shape[0], page_rows=c["P"], heads=c["heads"], head_dim=c["d"],
                dtype=c["dtype"], format=None if c["fmt"] == "none" else c["fmt"])
    if c["kind"] == "append":
        p = wf.make_append_params(**pool, tokens=c["tokens"], group=c["group"], rot_dim=c["rot"],
                                  sections=_sections(c),
                                  layout="pairs" if c["pairs"] else "halves",
                                  q_row=st["Q"].stride(0) if c["group"] else 0,
                                  k_row=st["K"].stride(0), v_row=st["V"].stride(0))
        return dict(wf=wf, p=p)
    if c["kind"] == "move":
        p = wf.make_move_params(**pool, batch=c["batch"], table_pages=st["table"].shape[1],
                                moves=c["moves"])
        return dict(wf=wf, p=p)
    p = wf.make_tree_params(**pool, group=c["group"], batch=c["batch"], tokens=st["Q"].shape[0],
                            max_rows=c["rows"], table_pages=st["table"].shape[1], max_len=c["L"],
                            causal=c["mask"] == "causal")
    return dict(wf=wf, p=p, ws=wf.alloc_tree_workspace(p, "cuda"))


# ------------------------------------------------------------ the calls

def run(state):
    st = state
    c = st["case"]
    if c["kind"] == "rope":
        if own:
            st["wf"].wf_rope(st["p"], st["X"], st["pos"], st["freq"], st["Y"])
        else:
            cos, sin = _angles(c, st["pos"], st["freq"])            # [batch, rows, pairs]
            st["Y"].copy_(_turned(c, st["X"].float(), cos.unsqueeze(1), sin.unsqueeze(1)))
        return [st["Y"]]
    pool = [st[k] for k in ("Kc", "Kx", "Vc", "Vx")]
    if c["kind"] == "tree":
        if own:
            st["wf"].wf_tree_attn(st["p"], st["Q"], *pool, st["table"], st["len"], st["start"],
                                  st["mask"], st["O"], st["lse"], st["ws"])
        else:
            _plain_tree(st)
        return [st["O"]] + ([st["lse"]] if c["lse"] else [])
    if c["kind"] == "append":
        if own:
            st["wf"].wf_page_append(st["p"], st["Q"], st["K"], st["V"], st["pos"], st["freq"],
                                    st["slot"], *pool, st["Qr"])
        else:
            _plain_append(st)
    elif own:
        st["wf"].wf_page_move(st["p"], st["table"], st["first"], st["src"], *pool)
    else:
        _plain_move(st)
    if c["fmt"] == "e4m3":
        pool[0], pool[2] = (x.view(torch.float8_e4m3fn) for x in (pool[0], pool[2]))
    return [x for x in pool + [st.get("Qr")] if x is not None]


# ------------------------------------------------------------ plain forms

def _angles(c, pos, freq):
    """Cosines and sines [..., pairs] at positions [axes][...]: angles in 64 bits."""
    axis = torch.repeat_interleave(torch.arange(c["axes"]), torch.tensor(_sections(c)))
    t = pos.double().movedim(0, -1)[..., axis.to(pos.device)] * freq.double()
    return t.cos().float(), t.sin().float()


def _turned(c, x, cos, sin):
    """Rows x [..., d] with their first channels rotated."""
    r = c["rot"]
    if c["pairs"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return y if r == c["d"] else torch.cat([y, x[..., r:]], -1)


def _quantise(x, fmt):
    """Codes and exponent bytes of fp32 rows x [..., d]."""
    y = x.unflatten(-1, (-1, 32))
    bits = y.abs().amax(-1).view(torch.int32)
    # one more where the mantissa is above 1.75 (448) or 1.5 (6)
    byte = ((bits + (0x1fffff if fmt == "e4m3" else 0x3fffff) >> 23)
            - (8 if fmt == "e4m3" else 2)).clamp(min=1)
    y = (y * (254 - byte << 23).view(torch.float32).unsqueeze(-1)).flatten(-2)
    if fmt == "e4m3":
        return y.to(torch.float8_e4m3fn).view(torch.uint8), byte.to(torch.uint8)
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5)
            + (a >= 3.5) + (a > 5)) | (torch.signbit(y).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4), byte.to(torch.uint8)


def _values(codes, byte, fmt):
    """The fp32 values of codes [..., d or d / 2] with exponent bytes [..., d / 32]."""
    if fmt == "e4m3":
        y = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=codes.device)
        y = table[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()]
    scale = (byte.int() << 23).view(torch.float32).unsqueeze(-1)
    return (y.unflatten(-1, (-1, 32)) * scale).flatten(-2)


def _plain_append(st):
    c = st["case"]
    cos, sin = (x.unsqueeze(1) for x in _angles(c, st["pos"], st["freq"]))
    if c["group"]:
        st["Qr"].copy_(_turned(c, st["Q"].float(), cos, sin))
    slot = st["slot"].long()
    # a token that is left out writes what the first kept one does
    keep = (slot >= 0) & (slot < st["Kc"].shape[0] * c["P"])
    n = torch.where(keep, torch.arange(len(slot), device=slot.device), keep.int().argmax())
    page, row = slot[n] // c["P"], slot[n] % c["P"]
    for m, x in (("K", _turned(c, st["K"].float(), cos, sin)), ("V", st["V"].float())):
        new = (x.to(_dtype(c)),) if c["fmt"] == "none" else _quantise(x, c["fmt"])
        for k, a in zip("cx", new):
            st[m + k].transpose(1, 2)[page, row] = a[n]


def _plain_move(st):
    c = st["case"]
    P, src = c["P"], st["src"].long()
    at = torch.arange(c["moves"], device=src.device)
    src = torch.where(src >= 0, src, at)        # (a row that stays is written as it is)
    to, of = (st["first"].long().unsqueeze(1) + t for t in (at, src))
    pt, po = (st["table"].long().gather(1, t // P) for t in (to, of))
    for k in ("Kc", "Kx", "Vc", "Vx"):
        if st[k] is not None:
            rows = st[k].transpose(1, 2)
            rows[pt, to % P] = rows[po, of % P]


def _plain_tree(st):
    c = st["case"]
    b, h, g, n, d, P, L = (c[k] for k in ("batch", "heads", "group", "rows", "d", "P", "L"))
    at = st["table"].clamp(min=0).long()                            # [b, pages]
    rows = {}
    for m in ("K", "V"):
        x = st[m + "c"][at].transpose(1, 2).flatten(2, 3)[:, :, :L]
        if c["fmt"] != "none":
            x = _values(x, st[m + "x"][at].transpose(1, 2).flatten(2, 3)[:, :, :L], c["fmt"])
        rows[m] = x.float()                                         # [b, h, L, d]
    count = st["counts"].long().unsqueeze(1)
    i = torch.arange(n, device=at.device)
    if st["start"] is None:
        q = st["Q"].view(b, n, h * g, d)
    else:
        tok = (st["start"][:-1].long().unsqueeze(1) + i).clamp(max=len(st["Q"]) - 1)
        q = st["Q"][tok]
    q = q.float().view(b, n, h, g, d).transpose(1, 2).reshape(b, h, n * g, d) / math.sqrt(d)
    S = q @ rows["K"].transpose(-1, -2).contiguous()                # [b, h, n g, L]
    t = torch.arange(L, device=at.device)
    length = st["len"].long().view(b, 1)
    j = t - (length - count)                                        # [b, L]
    sees = st["seen"].gather(2, j.clamp(0, n - 1).unsqueeze(1).expand(b, n, L))
    sees = ((j < 0).unsqueeze(1) | sees) & (t < length).unsqueeze(1)
    S = S.view(b, h, n, g, L).masked_fill_(~sees.view(b, 1, n, 1, L), -math.inf)
    M = S.amax(-1, keepdim=True)
    M = torch.where(M > -math.inf, M, 0.0)                          # rows without any key
    S = S.sub_(M).exp_()
    Z = S.sum(-1, keepdim=True)
    # what lies behind a sequence's rows takes no part
    rows["V"].masked_fill_((t >= length).view(b, 1, L, 1), 0.0)
    O = (S.view(b, h, n * g, L) @ rows["V"]).view(b, h, n, g, d) / torch.where(Z > 0, Z, 1.0)
    O = O.transpose(1, 2).reshape(b, n, h * g, d)
    lse = (torch.log(Z) + M).squeeze(-1).transpose(1, 2).reshape(b, n, h * g)
    if st["start"] is None:
        st["O"].copy_(O.view(b * n, h * g, d))
        if c["lse"]:
            st["lse"].copy_(lse.view(b * n, h * g))
        return
    # rows that are not there write what the first one of their sequence does
    k = torch.where(i < count, i, 0)
    tok, one = st["start"][:-1].long().unsqueeze(1) + k, torch.arange(b, device=at.device)[:, None]
    st["O"][tok] = O[one, k].to(_dtype(c))
    if c["lse"]:
        st["lse"][tok] = lse[one, k]


# ------------------------------------------------------------ work

def work(case):
    c = case
    es, d = (2 if c["dtype"] == "bf16" else 4), c["d"]
    if c["kind"] == "rope":
        n = c["batch"] * c["heads"] * c["rows"]
        return {"bytes": 2 * n * d * es + 4 * c["axes"] * c["batch"] * c["rows"],
                "flops": 3 * n * c["rot"]}
    bits = _BITS[c["fmt"]]
    kept = d * bits / 8 + d / 32 if bits else d * es    # bytes of a row of the cache
    if c["kind"] == "append":
        n, h, g = c["tokens"], c["heads"], c["group"]
        k = n - n // 8 if c["padded"] else n
        return {"bytes": 2 * n * h * g * d * es + 2 * k * h * (d * es + kept)
                + 4 * (c["axes"] + 1) * n,
                "flops": 3 * n * h * (g + 1) * c["rot"] + (4 * 2 * k * h * d if bits else 0)}
    if c["kind"] == "move":
        n = c["batch"] * c["heads"] * max(1, 3 * c["moves"] // 4)
        return {"bytes": 4 * n * kept, "flops": 0}
    L, n = c["L"], c["rows"]
    if c["ragged"]:
        L, n = 0.75 * L, 0.75 * n if n > 1 else 1
    q = c["batch"] * c["heads"] * c["group"] * n
    return {"bytes": c["batch"] * c["heads"] * L * 2 * kept + 2 * q * d * es
            + (4 * q if c["lse"] else 0),
            "flops": 4 * q * L * d}


# ------------------------------------------------------------ 64 bits

def _round64(y, least, mantissa):
    """y to `mantissa` bits behind the point of its power of two, at least 2^least; ties to even."""
    k = torch.frexp(y).exponent.double() - 1
    step = torch.exp2(k.clamp(min=least) - mantissa)
    return torch.round(y / step) * step


def _codes64(x, fmt):
    """The codes' values and the scales of rows x."""
    y = x.double().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    ratio = y.abs().max(-1).values / _TOP[fmt]
    m, k = torch.frexp(ratio)                                     # ratio = m 2^k, 0.5 <= m < 1
    e = torch.where(m == 0.5, k - 1, k).double().clamp(min=-126)
    y = y / torch.exp2(e).unsqueeze(-1)
    y = _round64(y, -6, 3) if fmt == "e4m3" else _round64(y, 0, 1)
    return y.reshape(x.shape), torch.exp2(e)


def _read64(codes, byte, fmt):
    """The values of a cache's rows."""
    k = codes.long()
    if fmt == "e2m1":
        k = torch.stack([k % 16, k // 16], -1).reshape(*k.shape[:-1], -1)
        sign, ex, man, bias, mb = k // 8, k // 2 % 4, k % 2, 1, 2
    else:
        sign, ex, man, bias, mb = k // 128, k // 8 % 16, k % 8, 7, 8
    low = ex == 0
    mag = torch.where(low, man / mb, 1 + man / mb).double() * torch.exp2(
        torch.where(low, 1, ex).double() - bias)
    v, s = mag * (1 - 2 * sign), torch.exp2(byte.double() - 127)
    return (v.reshape(*s.shape, 32) * s.unsqueeze(-1)).reshape(v.shape)


def _turn64(c, x, pos, freq):
    """Rows x [n][heads][d] at positions [axes][n]: pairs as complex numbers times e^(i angle)."""
    r, y = c["rot"], x.double()
    if r == 0:
        return y
    turn, i = torch.empty((len(x), r // 2), dtype=torch.float64, device=x.device), 0
    for axis, k in enumerate(_sections(c)):
        turn[:, i:i + k] = torch.outer(pos[axis].double(), freq[i:i + k].double())
        i += k
    turn = torch.polar(torch.ones_like(turn), turn).unsqueeze(1)
    y = y.clone()
    if c["pairs"]:
        z = torch.view_as_complex(y[..., :r].reshape(*y.shape[:-1], r // 2, 2)) * turn
        y[..., :r] = torch.view_as_real(z).reshape(*y.shape[:-1], r)
    else:
        z = torch.complex(y[..., :r // 2], y[..., r // 2:r]) * turn
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    return y


def exact(case, seed):
    c = case
    st = prepare(c, seed)
    if c["kind"] == "rope":
        Y = torch.empty(st["Y"].shape, dtype=torch.float64, device="cuda")
        for i in range(c["batch"]):
            Y[i] = _turn64(c, st["X"][i].transpose(0, 1), st["pos"][:, i], st["freq"]).transpose(0, 1)
        return [Y]
    if c["kind"] == "tree":
        return _exact_tree(c, st)
    out = []
    for m in ("K", "V"):
        codes = st[m + "c"]
        if c["fmt"] == "e2m1":      # two codes to a byte: no number
            out += [None, None]
            continue
        v = (codes if c["fmt"] == "none" else codes.view(torch.float8_e4m3fn)).double()
        if c["kind"] == "append":
            x = st[m] if m == "V" else _turn64(c, st["K"], st["pos"], st["freq"])
            new = x.double() if c["fmt"] == "none" else _codes64(x, c["fmt"])[0]
            for n, s in enumerate(st["slot"].tolist()):
                if 0 <= s < v.shape[0] * c["P"]:
                    v[s // c["P"], :, s % c["P"]] = new[n]
        else:
            old = v.clone()
            first, src, table = (st[k].tolist() for k in ("first", "src", "table"))
            for i in range(c["batch"]):
                for k, s in enumerate(src[i]):
                    if s >= 0:
                        to, of = first[i] + k, first[i] + s
                        v[table[i][to // c["P"]], :, to % c["P"]] = \
                            old[table[i][of // c["P"]], :, of % c["P"]]
        out += [v] + ([] if c["fmt"] == "none" else [None])
    if c["kind"] == "append" and c["group"]:
        out.append(_turn64(c, st["Q"], st["pos"], st["freq"]))
    return out


def _exact_tree(c, st):
    h, g, d, P, n = c["heads"], c["group"], c["d"], c["P"], c["rows"]
    O = torch.zeros(st["Q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(O.shape[:2], dtype=torch.float64, device="cuda")
    start = range(0, len(O), n) if st["start"] is None else st["start"].tolist()
    for i in range(c["batch"]):
        L, m, first = int(st["len"][i]), int(st["counts"][i]), start[i]
        pages = st["table"][i, :-(-L // P)].long()
        sees = torch.ones((m, L), dtype=torch.bool, device="cuda")
        sees[:, L - m:] = st["seen"][i, :m, :m]
        for k in range(h):
            kv = []
            for x in ("K", "V"):
                y = st[x + "c"][pages, k].reshape(len(pages) * P, -1)[:L]
                if c["fmt"] != "none":
                    y = _read64(y, st[x + "x"][pages, k].reshape(len(pages) * P, -1)[:L], c["fmt"])
                kv.append(y.double())
            q = st["Q"][first:first + m, k * g:(k + 1) * g].double().reshape(m * g, d)
            x = q @ kv[0].T.contiguous() / math.sqrt(d)
            x = x.view(m, g, L).masked_fill(~sees.unsqueeze(1), -math.inf)
            lse[first:first + m, k * g:(k + 1) * g] = torch.logsumexp(x, -1)
            w = torch.softmax(x, -1).view(m * g, L)
            O[first:first + m, k * g:(k + 1) * g] = (w @ kv[1]).view(m, g, d)
    return [O] + ([lse] if c["lse"] else [])
