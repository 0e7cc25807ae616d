"""Performance cases of the quantised cache (store, load) and of attention over a shared prefix.

A case is one call that a decoder makes for one layer: rows of keys and values written into a
quantised cache, rows of it read back, or the attention of a batch whose sequences share a prompt.
Sizes follow the workloads of synth.WORKLOADS; keys are AR(1) sequences with planted 16-token
needles towards which the queries lean, as there, drawn on the GPU.  With `own` the library's
entry points run, otherwise the same operators in elementary torch operations on 32-bit values.

The formats: blocks of 32 consecutive channels of a row share a power of two 2^(byte - 127), the
smallest one (byte >= 1) with which the block's largest magnitude is at most 448 (e4m3) or 6
(e2m1); the codes are the channels divided by it, rounded to the nearest, ties to even.
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
        # one denoising step's block of 32 rows written at its positions in a 4K cache
        _rows("store", "store_block", batch=1, heads=32, d=128, cap=4096, rows=32, at="list"),
        # a batch of four 32K prompts written once
        _rows("store", "store_prompt32k", batch=4, heads=32, d=128, cap=32768, rows=32768),
        # fp32 keys of an odd number of padded rows, written as 4 bits and read back at a list
        _rows("reload", "reload_f32_odd", batch=2, heads=3, d=64, cap=1999, rows=517, n=1001,
              at="padded", dtype="f32", fmt="e2m1"),
        # the pool of the selected regions of four 32K prompts, for the scan
        _rows("load", "load_pool32k", batch=4, heads=32, d=128, cap=32768, n=4096, at="list"),
        # a whole 128K prompt of an 8-head layer kept in 4 bits
        _rows("load", "load_prompt128k_e2m1", batch=1, heads=8, d=128, cap=131072, n=131072,
              fmt="e2m1"),
        # three fp32 sequences of a small model, ragged lengths
        _prefix("prefix_tiny_f32", share=3, heads=2, B=17, d=64, P=1021, T=45, ragged=True,
                lse=True, dtype="f32"),
        # single tokens of eight sequences with a 4K system prompt; latency
        _prefix("prefix_token4k", share=8, heads=8, group=4, B=1, P=4096, T=64),
        # single tokens of 32 sequences over a 32K prompt kept in 8 bits, ragged own rows
        _prefix("prefix_token32k_e4m3", share=32, heads=8, group=4, B=1, P=32768, T=256,
                ragged=True, fmt="e4m3"),
        # the 8B layer: four candidates of one prompt, a block of 32 rows each
        _prefix("prefix_block4k", share=4, heads=32, B=32, P=4096, T=32),
        # the tokens that the filter selected of a 32K prompt kept in 8 bits
        _prefix("prefix_selected32k_e4m3", share=4, heads=32, B=64, P=32768, n=2048, T=64,
                fmt="e4m3"),
        # sixteen sequences of a 32K prompt, grouped heads: 2048 query rows a KV head
        _prefix("prefix_block32k", share=16, heads=8, group=4, B=32, P=32768, T=256, lse=True),
        # two sequences of a 128K prompt kept in 4 bits
        _prefix("prefix_block128k_e2m1", share=2, heads=8, group=4, B=32, P=131072, T=32,
                fmt="e2m1"),
    ]


def _named(c, name):
    if name is not None:
        c["name"] = name
    return c


def _rows(kind, name, *, batch, heads, d, cap, rows=0, n=0, at="range", dtype="bf16",
          fmt="e4m3"):
    """rows written, n rows read back; at: a range from row 0, a list of rows, or a list padded
    with -1 (for reload: the rows written; it reads at a list)."""
    return _named(dict(kind=kind, batch=batch, heads=heads, d=d, cap=cap, rows=rows, n=n, at=at,
                       dtype=dtype, fmt=fmt), name)


def _prefix(name, *, share, heads, B, P, T, prefixes=1, group=1, d=128, n=0, ragged=False,
            lse=False, dtype="bf16", fmt="none", rho=0.98):
    """n: rows of a list (0: the first P rows of the prefix); T: own rows of a sequence."""
    return _named(dict(kind="prefix", prefixes=prefixes, share=share, heads=heads, group=group,
                       B=B, d=d, P=P, n=n, T=T, ragged=ragged, lse=lse, dtype=dtype, fmt=fmt,
                       rho=rho), name)


def _log(rng, lo, hi):
    return int(round(2 ** rng.uniform(math.log2(lo), math.log2(hi))))


def draw(rng):
    kind = rng.choice(["store", "load", "reload", "prefix", "prefix", "prefix", "prefix"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    d = rng.choice([64, 128, 128])
    if kind != "prefix":
        batch, heads = rng.choice([1, 1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 8, 8, 32])
        most = (1 << 29) // (batch * heads * d) // (2 if dtype == "f32" else 1)
        cap = _log(rng, 64, min(131072, most))
        fmt = "e4m3" if kind == "store" else rng.choice(["e4m3", "e2m1"])
        rows = 0 if kind == "load" else min(cap, _log(rng, 1, cap))
        n = 0 if kind == "store" else min(cap, _log(rng, 1, cap))
        at = rng.choice(["range", "list", "padded"] if kind != "load" else ["range", "list"])
        return _rows(kind, None, batch=batch, heads=heads, d=d, cap=cap, rows=rows, n=n, at=at,
                     dtype=dtype, fmt=fmt)
    prefixes = rng.choice([1, 1, 1, 2, 3])
    heads, group = rng.choice([(2, 1), (3, 1), (8, 1), (8, 4), (8, 8), (4, 7), (32, 1)])
    share = _log(rng, 1, 32)
    B = rng.choice([1, 1, 1, 5, 16, 17, 32, 32, 45, 64])
    P = _log(rng, 128, 131072)
    T = rng.choice([0, 1, B, 2 * B + 3, _log(rng, 16, 1024)])
    n = min(P, _log(rng, 32, 4096)) if rng.random() < 0.25 else 0
    fmt = rng.choice(["none", "none", "e4m3", "e4m3", "e2m1"])
    c = _prefix(None, share=share, heads=heads, B=B, P=P, T=T, prefixes=prefixes, group=group,
                d=d, n=n, ragged=rng.random() < 0.4, lse=rng.random() < 0.4, dtype=dtype, fmt=fmt,
                rho=rng.choice([0.95, 0.98, 0.99]))
    # at most the largest listed case's products, an eighth of them in fp32
    most = 2.7e11 / (8 if dtype == "f32" else 1)
    while work(c)["flops"] > most or c["prefixes"] * c["heads"] * c["P"] * d > 1 << 28:
        if c["P"] > 4096 and c["n"] == 0 or c["share"] == 1:
            c["P"] = c["P"] * 2 // 3
            c["n"] = min(c["n"], c["P"])
        else:
            c["share"] = max(1, c["share"] * 2 // 3)
    return c


# ------------------------------------------------------------ inputs

def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _gen(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * int(seed) + 29)
    return gen


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


def _distinct(gen, lists, n, below):
    """`lists` ascending lists of n distinct rows below `below`."""
    at = torch.rand((lists, below), generator=gen, device="cuda").argsort(dim=1)[:, :n]
    return at.sort(dim=1).values.to(torch.int32)


def _old_cache(c, gen):
    """A cache in use: rows of earlier steps."""
    shape = (c["batch"], c["heads"], c["cap"])
    nb = c["d"] * _BITS[c["fmt"]] // 8
    st = {}
    for m in ("K", "V"):  # (without the e4m3 code of NaN)
        st[m + "c"] = torch.randint(0, 256, shape + (nb,), generator=gen, device="cuda",
                                    dtype=torch.uint8) & 0xf7
        st[m + "x"] = torch.randint(116, 126, shape + (c["d"] // 32,), generator=gen,
                                    device="cuda", dtype=torch.uint8)
    return st


def prepare(case, seed):
    c = case
    gen = _gen(seed)
    dt, d = _dtype(c), c["d"]
    st = dict(case=c)
    if c["kind"] == "prefix":
        p, s, h, g, B, P, T, n = (c[k] for k in ("prefixes", "share", "heads", "group", "B", "P",
                                                 "T", "n"))
        u = torch.randn((p * h, 1, d), generator=gen, device="cuda")
        u /= u.norm(dim=-1, keepdim=True)
        K = torch.empty((p * h, P, d), dtype=dt, device="cuda")
        V = torch.empty_like(K)
        for i in range(0, p * h, 8):
            m = min(8, p * h - i)
            K[i:i + m] = _keys(gen, m, P, d, c["rho"], u[i:i + m])
            V[i:i + m] = torch.randn((m, P, d), generator=gen, device="cuda")
        K, V = K.view(p, h, P, d), V.view(p, h, P, d)
        z = torch.randn((p, s, h, g * B, d), generator=gen, device="cuda")
        st["Q"] = (z / math.sqrt(d) + 2.0 * u.view(p, 1, h, 1, d)).to(dt).view(p * s, h * g, B, d)
        st["Kt"] = st["Vt"] = None
        if T:
            st["Kt"], st["Vt"] = (torch.randn((p * s, h, T, d), generator=gen, device="cuda").to(dt)
                                  for _ in range(2))
        st["Kx"] = st["Vx"] = None
        if c["fmt"] == "none":
            st["K"], st["V"] = K, V
        else:
            st["K"], st["Kx"] = _quantise(K.float(), c["fmt"])
            st["V"], st["Vx"] = _quantise(V.float(), c["fmt"])
        st["list"] = _distinct(gen, p * h, n, P).view(p, h, n) if n else None
        rows = n or P
        st["plen"] = st["tlen"] = None
        if c["ragged"]:
            st["plen"] = torch.randint(rows // 2, rows + 1, (p,), generator=gen, device="cuda",
                                       dtype=torch.int32)
            if T:
                st["tlen"] = torch.randint(0, T + 1, (p * s,), generator=gen, device="cuda",
                                           dtype=torch.int32)
        st["O"] = torch.empty_like(st["Q"])
        st["lse"] = (torch.empty((p * s, h * g, B), dtype=torch.float32, device="cuda")
                     if c["lse"] else None)
    else:
        b, h, rows, n, cap = (c[k] for k in ("batch", "heads", "rows", "n", "cap"))
        st |= _old_cache(c, gen)
        st["rows"] = st["list"] = None
        if rows:
            u = torch.randn((b * h, 1, d), generator=gen, device="cuda")
            u /= u.norm(dim=-1, keepdim=True)
            st["K"] = torch.empty((b, h, rows, d), dtype=dt, device="cuda")
            st["V"] = torch.empty_like(st["K"])
            for i in range(b):
                st["K"][i] = _keys(gen, h, rows, d, 0.98, u[i * h:(i + 1) * h])
                st["V"][i] = torch.randn((h, rows, d), generator=gen, device="cuda")
            if c["at"] != "range":
                st["rows"] = _distinct(gen, b, rows, cap)
                if c["at"] == "padded":  # a batch padded to one length
                    st["rows"][:, max(1, rows - rows // 8):] = -1
        if n:
            if c["kind"] == "reload" or c["at"] != "range":
                st["list"] = _distinct(gen, b * h, n, cap).view(b, h, n)
            st["Ko"] = torch.empty((b, h, n, d), dtype=dt, device="cuda")
            st["Vo"] = torch.empty_like(st["Ko"])
    if own:  # what a serving loop keeps: the parameters and the workspace
        st |= _kept(c)
    return st


def _kept(c):
    import paper_2606_00724_amd as wf
    wf.wf_init()
    fmt = None if c["fmt"] == "none" else c["fmt"]
    if c["kind"] == "prefix":
        p = wf.make_prefix_params(prefixes=c["prefixes"], share=c["share"], heads=c["heads"],
                                  group=c["group"], q_len=c["B"], head_dim=c["d"],
                                  prefix_cap=c["P"], prefix_rows=c["n"] or c["P"],
                                  tail_cap=c["T"], dtype=c["dtype"], format=fmt)
        return dict(wf=wf, p=p, ws=wf.alloc_prefix_workspace(p, "cuda"))
    both = [wf.make_cache_params(batch=c["batch"], heads=c["heads"], capacity=c["cap"],
                                 head_dim=c["d"], rows=k, dtype=c["dtype"], format=fmt)
            for k in (c["rows"], c["n"])]
    return dict(wf=wf, pw=both[0], pr=both[1])


# ------------------------------------------------------------ the calls

def run(state):
    st = state
    c = st["case"]
    if c["kind"] == "prefix":
        if own:
            st["wf"].wf_prefix_attn(st["p"], st["Q"], st["K"], st["Kx"], st["V"], st["Vx"],
                                    st["list"], st["plen"], st["Kt"], st["Vt"], st["tlen"],
                                    st["O"], st["lse"], st["ws"])
        else:
            _plain_prefix(st)
        return [st["O"]] + ([st["lse"]] if c["lse"] else [])
    if c["rows"]:
        if own:
            st["wf"].wf_cache_store(st["pw"], st["K"], st["V"], st["rows"], st["Kc"], st["Kx"],
                                    st["Vc"], st["Vx"])
        else:
            _plain_store(st)
    if c["n"]:
        if own:
            st["wf"].wf_cache_load(st["pr"], st["Kc"], st["Kx"], st["Vc"], st["Vx"], st["list"],
                                   st["Ko"], st["Vo"])
        else:
            _plain_load(st)
        return [st["Ko"], st["Vo"]]
    f8 = torch.float8_e4m3fn
    return [st["Kc"].view(f8), st["Kx"], st["Vc"].view(f8), st["Vx"]]


# ------------------------------------------------------------ plain forms

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


def _plain_store(st):
    c = st["case"]
    b, rows, cap = c["batch"], c["rows"], c["cap"]
    new = {m: _quantise(st[m].float(), c["fmt"]) for m in ("K", "V")}
    if st["rows"] is None:
        for m in ("K", "V"):
            st[m + "c"][:, :, :rows] = new[m][0]
            st[m + "x"][:, :, :rows] = new[m][1]
        return
    at = st["rows"].long()
    keep = (at >= 0) & (at < cap)
    # a row that is left out writes what the first kept one does
    r = torch.where(keep, torch.arange(rows, device=at.device), keep.int().argmax(1, keepdim=True))
    at = at.gather(1, r)
    one = torch.arange(b, device=at.device).unsqueeze(1)
    for m in ("K", "V"):
        for k, a in zip("cx", new[m]):
            st[m + k].transpose(1, 2)[one, at] = a.transpose(1, 2)[one, r]


def _plain_load(st):
    c = st["case"]
    for m in ("K", "V"):
        codes, byte = st[m + "c"], st[m + "x"]
        if st["list"] is None:
            codes, byte = codes[:, :, :c["n"]], byte[:, :, :c["n"]]
        else:
            at = st["list"].long().unsqueeze(-1)
            codes = codes.gather(2, at.expand(-1, -1, -1, codes.shape[-1]))
            byte = byte.gather(2, at.expand(-1, -1, -1, byte.shape[-1]))
        st[m + "o"].copy_(_values(codes, byte, c["fmt"]))


def _plain_prefix(st):
    c = st["case"]
    p, s, h, g, B, d, T = (c[k] for k in ("prefixes", "share", "heads", "group", "B", "d", "T"))
    R = g * B
    rows = {}
    for m in ("K", "V"):
        x, e = st[m], st[m + "x"]
        if st["list"] is not None:
            at = st["list"].long().unsqueeze(-1)
            x = x.gather(2, at.expand(-1, -1, -1, x.shape[-1]))
            e = e if e is None else e.gather(2, at.expand(-1, -1, -1, e.shape[-1]))
        rows[m] = x.float() if e is None else _values(x, e, c["fmt"])
    Q = st["Q"].float().view(p, s, h, R, d) / math.sqrt(d)
    Qp = Q.transpose(1, 2).reshape(p, h, s * R, d)
    S = Qp @ rows["K"].transpose(-1, -2)                          # [p, h, s R, P]
    if st["plen"] is not None:
        off = torch.arange(S.shape[-1], device=S.device) >= st["plen"].view(p, 1, 1, 1)
        S = S.masked_fill(off, -math.inf)
    M = S.amax(-1)
    if T:
        St = Q.view(p * s, h, R, d) @ st["Kt"].float().transpose(-1, -2)   # [p s, h, R, T]
        if st["tlen"] is not None:
            off = torch.arange(T, device=S.device) >= st["tlen"].view(p * s, 1, 1, 1)
            St = St.masked_fill(off, -math.inf)
        Mt = St.amax(-1).view(p, s, h, R).transpose(1, 2).reshape(p, h, s * R)
        M = torch.maximum(M, Mt)
    ref = torch.where(M > -math.inf, M, 0.0)                      # rows without any key
    S = S.sub_(ref.unsqueeze(-1)).exp_()
    Z = S.sum(-1)
    O = S @ rows["V"]
    if T:
        rt = ref.view(p, h, s, R).transpose(1, 2).reshape(p * s, h, R, 1)
        St = (St - rt).exp()
        back = lambda x: x.view(p, s, h, R, -1).transpose(1, 2).reshape(p, h, s * R, -1)  # noqa: E731
        Z = Z + back(St.sum(-1, keepdim=True)).squeeze(-1)
        O = O + back(St @ st["Vt"].float())
    O = O / torch.where(Z > 0, Z, 1.0).unsqueeze(-1)
    st["O"].copy_(O.view(p, h, s, R, d).transpose(1, 2).reshape(p * s, h * g, B, d))
    if c["lse"]:
        lse = torch.log(Z) + ref
        st["lse"].copy_(lse.view(p, h, s, R).transpose(1, 2).reshape(p * s, h * g, B))


# ------------------------------------------------------------ work

def work(case):
    c = case
    es, bits, d = (2 if c["dtype"] == "bf16" else 4), _BITS[c["fmt"]], c["d"]
    kept = d * bits / 8 + d / 32            # bytes of a quantised row
    if c["kind"] != "prefix":
        rows = c["batch"] * c["heads"] * (c["rows"] + c["n"])
        return {"bytes": 2 * rows * (d * es + kept), "flops": 4 * 2 * rows * d}
    P, T = c["n"] or c["P"], c["T"]
    if c["ragged"]:
        P, T = 0.75 * P, 0.5 * T
    p, seqs, R = c["prefixes"], c["prefixes"] * c["share"], c["group"] * c["B"]
    q = seqs * c["heads"] * R
    return {"bytes": p * c["heads"] * P * 2 * (kept if bits else d * es)
            + seqs * c["heads"] * T * 2 * d * es + 2 * q * d * es + (4 * q if c["lse"] else 0),
            "flops": 4 * q * (P + T) * d}


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
    """The codes' values and the scales of a cache."""
    k = codes.long()
    if fmt == "e2m1":
        k = torch.stack([k % 16, k // 16], -1).reshape(*k.shape[:-1], -1)
        sign, ex, man, bias, mb = k // 8, k // 2 % 4, k % 2, 1, 2
    else:
        sign, ex, man, bias, mb = k // 128, k // 8 % 16, k % 8, 7, 8
    low = ex == 0
    mag = torch.where(low, man / mb, 1 + man / mb).double() * torch.exp2(
        torch.where(low, 1, ex).double() - bias)
    return mag * (1 - 2 * sign), torch.exp2(byte.double() - 127)


def _times(v, s):
    return (v.reshape(*s.shape, 32) * s.unsqueeze(-1)).reshape(v.shape)


def exact(case, seed):
    c = case
    st = prepare(c, seed)
    if c["kind"] == "prefix":
        return _exact_prefix(c, st)
    out = []
    for m in ("K", "V"):
        codes, scale = [], []
        for i in range(c["batch"]):
            v, s = _read64(st[m + "c"][i], st[m + "x"][i], c["fmt"])
            if c["rows"]:
                nv, ns = _codes64(st[m][i], c["fmt"])
                at = torch.arange(c["rows"], device=v.device)
                r = at
                if st["rows"] is not None:
                    ok = (st["rows"][i] >= 0) & (st["rows"][i] < c["cap"])
                    r = ok.nonzero().squeeze(1)
                    at = st["rows"][i][r].long()
                v[:, at], s[:, at] = nv[:, r], ns[:, r]
            if not c["n"]:
                codes.append(v.float())  # (codes are fp32 numbers)
                continue
            w = _times(v, s)
            if st["list"] is None:
                codes.append(w[:, :c["n"]])
            else:
                codes.append(torch.stack([w[k][st["list"][i, k].long()]
                                          for k in range(c["heads"])]))
        out += [torch.stack(codes).double()] + ([] if c["n"] else [None])
    return out


def _exact_prefix(c, st):
    h, g, s, d, B = c["heads"], c["group"], c["share"], c["d"], c["B"]
    O = torch.zeros(st["Q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(O.shape[:3], -math.inf, dtype=torch.float64, device="cuda")
    for i in range(c["prefixes"]):
        for k in range(h):
            kv = []
            for m in ("K", "V"):
                x = st[m][i, k]
                if st["list"] is not None:
                    x = x[st["list"][i, k].long()]
                if c["fmt"] == "none":
                    x = x.double()
                else:
                    e = st[m + "x"][i, k]
                    e = e if st["list"] is None else e[st["list"][i, k].long()]
                    x = _times(*_read64(x, e, c["fmt"]))
                kv.append(x if st["plen"] is None else x[:int(st["plen"][i])])
            for n in range(i * s, i * s + s):
                keys, vals = kv
                if c["T"]:
                    t = c["T"] if st["tlen"] is None else int(st["tlen"][n])
                    keys = torch.cat([keys, st["Kt"][n, k, :t].double()])
                    vals = torch.cat([vals, st["Vt"][n, k, :t].double()])
                if not len(keys):
                    continue
                q = st["Q"][n, k * g:(k + 1) * g].double().reshape(g * B, d)
                x = q @ keys.T.contiguous() / math.sqrt(d)
                lse[n, k * g:(k + 1) * g] = torch.logsumexp(x, -1).view(g, B)
                O[n, k * g:(k + 1) * g] = (torch.softmax(x, -1) @ vals).view(g, B, d)
    return [O] + ([lse] if c["lse"] else [])
