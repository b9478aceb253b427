"""The operators of the 4-bit prefix cache, as cases that can be prepared, run and compared.

A serving program that keeps its committed prefix in 4 bits writes a prompt's or a token's rows into it (`write`), commits the
accepted rows of a verified tree (`commit`), attends the draft tree against it (`attn`; a tree of one node is plain decoding)
and takes rows back out of it (`read`), for instance to move a sequence elsewhere.

The cache: groups of 32 consecutive channels of one row of one KV head.  A group has 32 e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6;
bit 3 is the sign), two to a byte with the even channel in the low half, and one byte s that scales them by 2^(s-127).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MARGIN = 2      # rows before and behind the written ones that a `write` or `commit` case reads back with them


def _case(name, kind, **kw):
    c = dict(name=name, kind=kind, B=1, layers=1, Hkv=8, d=128, dtype="bf16", block=16)
    c.update(kw)
    return c


def listed():
    return [
        # one user decoding without a draft: a single query token against a short chat, nothing but latency
        _case("attn_token_b1", "attn", T=1, n_lo=1, Hq=32, P=2048, P_lo=2048, block=0),
        # a full serving batch with a small tree: reading the cache is all there is
        _case("attn_b32_t8", "attn", B=32, T=8, n_lo=8, Hq=32, P=4096, P_lo=4096),
        # a small serving batch of ragged sequences with trees of the usual size, larger pages
        _case("attn_ragged_b8_t60", "attn", B=8, T=60, n_lo=45, Hq=32, P=8192, P_lo=512, block=64),
        # the full batch with the largest tree budget of the benchmark's sweep: bound by the products
        _case("attn_b32_t128", "attn", B=32, T=128, n_lo=128, Hq=32, P=4096, P_lo=4096),
        # fp32 throughout, for a teacher that is checked or run at full precision; odd sizes
        _case("attn_f32_b2", "attn", B=2, T=33, n_lo=29, Hq=16, Hkv=4, dtype="f32", P=1003, P_lo=771),
        # one long document, a model with heads of 64
        _case("attn_d64_long", "attn", T=48, n_lo=48, Hq=32, d=64, P=32768, P_lo=32768, block=0),
        # decoding: one new token of every sequence, all layers
        _case("write_token_b8", "write", B=8, S=1, n_lo=1, layers=32, P=2000, P_lo=1000),
        # prompts of different length, some layers of a model
        _case("write_prompt_b2", "write", B=2, S=4096, n_lo=3001, layers=8, P=100, P_lo=3, block=0),
        # the commit of one user's step: a path of a few rows, all layers
        _case("commit_b1", "commit", T=60, W=7, layers=32, P=2048, P_lo=2048),
        # the commit of a full batch with deep trees, fp32 tree rows
        _case("commit_f32_b32", "commit", B=32, T=128, W=11, layers=16, dtype="f32", P=700, P_lo=90),
        # a short odd-sized sequence for inspection, in fp32
        _case("read_f32_b1", "read", S=777, n_lo=777, Hkv=4, d=64, dtype="f32", P=1003, P_lo=1003, block=48),
        # sequences that leave the card or change their form: whole prefixes of some layers
        _case("read_b8", "read", B=8, S=4096, n_lo=2000, layers=4, P=4200, P_lo=4100),
    ]


# ---------------------------------------------------------------------------------------------------------------
def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / (1e15 if c["dtype"] == "bf16" else 1e14))


def draw(rng):
    most = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in ("attn", "write", "commit", "read")}
    kind = rng.choice(["attn", "attn", "attn", "write", "commit", "read"])
    while True:
        c = dict(kind=kind, B=_log(rng, 1, 32), layers=1, d=rng.choice([128, 128, 64]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]),
                 block=rng.choice([0, 0, 16, 16, 32, 48, 64, 256]))
        P = _log(rng, 16, 32768)
        c["P"], c["P_lo"] = P, rng.choice([P, rng.randint(max(MARGIN, P // 16), P)])
        if kind == "attn":
            Hq, c["Hkv"] = rng.choice([(32, 8), (32, 8), (32, 8), (8, 2), (8, 8), (16, 4), (32, 32), (28, 4), (8, 1)])
            T = _log(rng, 1, 256)
            c.update(Hq=Hq, T=T, n_lo=rng.randint(max(1, (3 * T) // 4), T))
        else:
            c.update(Hkv=rng.choice([1, 4, 8]), layers=rng.randint(1, 32))
            if kind == "commit":
                c.update(T=_log(rng, 2, 256), W=rng.randint(2, 12))
            else:
                S = _log(rng, 1, 8192)
                c.update(S=S, n_lo=rng.randint(max(1, S // 2), S))
                if kind == "read":
                    c["P"], c["P_lo"] = S + P, S + c["P_lo"]
        # the pool of a case stays below some GiB, and its cost below that of the largest listed one
        if _cost(c) <= most[kind] and c["layers"] * c["B"] * (c["P"] + c.get("S", 0)) * c["Hkv"] * c["d"] <= 1 << 32:
            return c


def _spread(lo, hi, n):
    """n whole numbers from hi down to lo, evenly."""
    return [hi] if n == 1 else [int(round(hi - (hi - lo) * i / (n - 1))) for i in range(n)]


def work(c):
    e = 4 if c["dtype"] == "f32" else 2
    q4 = c["d"] // 2 + c["d"] // 32                                  # bytes of one row of one head in the cache
    if c["kind"] == "attn":
        by = fl = 0
        # which length meets which tree is drawn by the seed: the mean of the products stands for it
        P, n = _spread(c["P_lo"], c["P"], c["B"]), _spread(c["n_lo"], c["T"], c["B"])
        for b in range(c["B"]):
            by += 2 * P[b] * c["Hkv"] * q4 + 2 * n[b] * c["Hkv"] * c["d"] * e + n[b] * c["Hq"] * (2 * c["d"] * e + 4)
            fl += 4 * c["Hq"] * c["d"] * n[b] * (sum(P) / c["B"] + n[b])
        return {"bytes": by, "flops": fl}
    heads = 2 * c["layers"] * c["Hkv"]                               # K and V
    if c["kind"] == "read":
        return {"bytes": heads * sum(_spread(c["n_lo"], c["S"], c["B"])) * (q4 + c["d"] * e), "flops": 0}
    rows = c["B"] * (c["W"] + 1) // 2 if c["kind"] == "commit" else sum(_spread(c["n_lo"], c["S"], c["B"]))
    # the rows are read, written in 4 bits, and what the cache then holds is read back, with some rows around them
    back = rows + 2 * MARGIN * c["B"]
    return {"bytes": heads * (rows * (c["d"] * e + q4) + back * (q4 + c["d"] * e)), "flops": 0}


# ---------------------------------------------------------------------------------------------------------------
# inputs
def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _i32(xs):
    return _dev(np.asarray(xs, dtype=np.int32))


def _table(c, rng, rows):
    """Pages for `rows` positions of every sequence, in any order: block table, pool size, capacity."""
    need = [-(-r // c["block"]) for r in rows]
    pool = sum(need) + 3
    ids = rng.permutation(pool).astype(np.int32)
    table, at = np.zeros((c["B"], max(need)), dtype=np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    return table, pool, [n * c["block"] for n in need]


def _tree(rng, n, depth):
    """Parents of a random tree of n nodes, no deeper than `depth` below the root."""
    parent, level = np.zeros(n, dtype=np.int64), np.zeros(n, dtype=np.int64)
    for k in range(1, n):
        p = int(rng.integers(max(0, k - 12), k))
        while level[p] >= depth:
            p = int(parent[p])
        parent[k], level[k] = p, level[p] + 1
    return parent


def _ancestors(parent, T):
    m = np.zeros((T, T), dtype=bool)
    for k, p in enumerate(parent):
        if k:
            m[k] = m[p]
        m[k, k] = True
    return m


def prepare(case, seed):
    c, rng, gen = case, np.random.default_rng(seed), torch.Generator(device=DEV).manual_seed(seed)
    B, dt, d = c["B"], DTYPES[c["dtype"]], c["d"]
    normal = lambda *shape: torch.empty(shape, dtype=dt, device=DEV).normal_(generator=gen)
    Ps = [int(x) for x in rng.permutation(_spread(c["P_lo"], c["P"], B))]
    s = {"case": c, "Ps": Ps, "P_max": max(Ps), "prefix_len": _i32(Ps), "block_table": None}
    extra = {"attn": 0, "write": c.get("S", 0) + MARGIN, "commit": c.get("W", 0) + MARGIN, "read": 0}[c["kind"]]
    s["rows"] = max(Ps) + extra
    if c["block"]:
        s["table"], pool, room = _table(c, rng, [P + extra for P in Ps])
        s["block_table"], s["capacity"], page = _dev(s["table"]), _i32(room), c["block"]
    else:
        pool, page, s["capacity"] = B, s["rows"], _i32([s["rows"]] * B)
    shape = (c["layers"], pool, c["Hkv"], page)
    if c["kind"] == "attn":
        ns = [int(x) for x in rng.permutation(_spread(c["n_lo"], c["T"], B))]
        # keys have a few strong channels, as a trained model's do; values do not
        strong = 1.0 + 3.0 * (torch.rand((c["Hkv"], 1, d), device=DEV, generator=gen) > 0.95)
        parts = [[], [], [], []]
        for _ in range(2):
            for lo in range(0, pool, 1024):
                x = torch.empty((min(1024, pool - lo), c["Hkv"], page, d), device=DEV).normal_(generator=gen)
                for part, piece in zip(parts[2 * _:], _quantise(x * strong if _ == 0 else x)):
                    part.append(piece)
        s["kc"], s["ks"], s["vc"], s["vs"] = (torch.cat(p)[None] for p in parts)
        s["q"] = normal(B, c["T"], c["Hq"], d)
        s["kt"], s["vt"] = normal(B, c["T"], c["Hkv"], d) * strong[:, 0].to(dt), normal(B, c["T"], c["Hkv"], d)
        vis = np.stack([_ancestors(_tree(rng, n, 10), c["T"]) for n in ns])
        words = (c["T"] + 63) // 64
        bits = np.zeros((B, c["T"], 64 * words), dtype=bool)
        bits[:, :, :c["T"]] = vis
        s["bitmask"] = _dev(np.packbits(bits, axis=2, bitorder="little").view(np.int64))
        s["vis"], s["ns"], s["n_nodes"] = _dev(vis), ns, _i32(ns)
    else:
        for name in ("kc", "vc"):
            s[name] = torch.randint(0, 256, shape + (d // 2,), dtype=torch.uint8, device=DEV, generator=gen)
        for name in ("ks", "vs"):
            s[name] = torch.randint(118, 130, shape + (d // 32,), dtype=torch.uint8, device=DEV, generator=gen)
    if c["kind"] == "commit":
        W, T = c["W"], c["T"]
        parents = [_tree(rng, T, W - 1) for _ in range(B)]
        acc, A = np.zeros((B, W), dtype=np.int32), []
        for b, par in enumerate(parents):
            path = [int(rng.integers(T))]
            while path[0]:
                path.insert(0, int(par[path[0]]))
            A.append(int(rng.integers(len(path))))
            acc[b, :A[b] + 1] = path[:A[b] + 1]
        s["acc"], s["A"] = acc, A
        s["acc_nodes"], s["accept_len"], s["n_nodes"] = _dev(acc), _i32(A), _i32([T] * B)
        s["k"], s["v"] = normal(c["layers"], B, T, c["Hkv"], d), normal(c["layers"], B, T, c["Hkv"], d)
        s["counts"], s["window"] = [a + 1 for a in A], W + 2 * MARGIN
    elif c["kind"] != "attn":
        s["counts"] = [int(x) for x in rng.permutation(_spread(c["n_lo"], c["S"], B))]
        s["n_rows"], s["window"] = _i32(s["counts"]), c["S"] + (2 * MARGIN if c["kind"] == "write" else 0)
        if c["kind"] == "write":
            s["k"], s["v"] = normal(c["layers"], B, c["S"], c["Hkv"], d), normal(c["layers"], B, c["S"], c["Hkv"], d)
    if c["kind"] == "read":
        s["lo"] = [int(rng.integers(0, P - n + 1)) for P, n in zip(Ps, s["counts"])]
        s["back"] = s["counts"]
    elif c["kind"] != "attn":
        s["lo"], s["back"] = [P - MARGIN for P in Ps], [n + 2 * MARGIN for n in s["counts"]]
    if c["kind"] != "attn":
        s["first"], s["back_rows"] = _i32(s["lo"]), _i32(s["back"])
    if own:
        from paper_2603_08088_amd import api
        s["cache"] = api.KVCacheQ4(s["kc"], s["ks"], s["vc"], s["vs"])
        if c["kind"] == "attn":
            # what a decoding loop keeps from step to step
            s["layer"] = s["cache"].layer(0)
            s["desc"] = api.attn_q4_desc(s["q"], s["layer"], s["kt"], s["block_table"], s["P_max"])
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty((B, c["Hq"], c["T"]), dtype=torch.float32, device=DEV)
            s["workspace"] = torch.empty((max(256, api.tree_verify_attention_q4_workspace_bytes(s["desc"])),), dtype=torch.uint8, device=DEV)
        else:
            shape = (c["layers"], B, s["window"], c["Hkv"], d)
            s["k_back"], s["v_back"] = torch.empty(shape, dtype=dt, device=DEV), torch.empty(shape, dtype=dt, device=DEV)
    return s


# ---------------------------------------------------------------------------------------------------------------
# the plain forms
def _quantise(x):
    """float [..., d] -> codes uint8 [..., d/2], scales uint8 [..., d/32]."""
    g = x.float().unflatten(-1, (-1, 32))
    a = g.abs().amax(-1)
    # the exponent of the largest magnitude, rounded to two significant bits: 7/8 of the next power of two counts as that power
    e = ((a.view(torch.int32) + 0x200000) >> 23) - 2
    s = e.clamp(2, 252)
    bad = ~torch.isfinite(g).all(-1)
    y = g.abs() * torch.exp2((127 - s).float())[..., None]
    code = ((y > 0.25).byte() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)).to(torch.uint8)
    code = (code | (torch.signbit(g).byte() << 3)).masked_fill_(bad[..., None], 0).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.where(bad, 255, s).to(torch.uint8)


def _values(codes, scales):
    """codes [..., d/2], scales [..., d/32] -> float32 [..., d]."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    nib = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    f = torch.where(scales == 255, math.nan, torch.exp2(scales.float() - 127))
    return (table[nib.int()].unflatten(-1, (-1, 32)) * f[..., None]).flatten(-2)


def _places(s, b, lo, n):
    """Where positions lo .. lo + n - 1 of sequence b lie: page, offset."""
    p = torch.arange(lo, lo + n, device=DEV)
    if s["block_table"] is None:
        return torch.full_like(p, b), p
    size = s["case"]["block"]
    return s["block_table"][b].long()[p // size], p % size


def _plain_attn(s):
    c, (q, kt, vt) = s["case"], (s["q"], s["kt"], s["vt"])
    B, T, Hq, d = q.shape
    Hkv, G = c["Hkv"], Hq // c["Hkv"]
    out, lse = torch.zeros_like(q), torch.full((B, Hq, T), -math.inf, device=DEV)
    for b in range(B):
        n, P = s["ns"][b], s["Ps"][b]
        page, at = _places(s, b, 0, P)
        rows = lambda codes, scales, t: torch.cat((_values(codes[0, page, :, at], scales[0, page, :, at]), t[b, :n].float())).transpose(0, 1).contiguous()
        K, V = rows(s["kc"], s["ks"], kt), rows(s["vc"], s["vs"], vt)                      # [Hkv, P + n, d]
        Q = q[b, :n].float().reshape(n, Hkv, G, d).permute(1, 2, 0, 3).reshape(Hkv, G * n, d)
        x = torch.matmul(Q, K.transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(d)).reshape(Hq, n, P + n)
        x[:, :, P:].masked_fill_(~s["vis"][b, :n, :n], -math.inf)
        m = x.amax(-1, keepdim=True)
        x = x.sub_(m).exp_()
        z = x.sum(-1, keepdim=True)
        o = torch.matmul(x.reshape(Hkv, G * n, P + n), V).reshape(Hq, n, d) / z
        out[b, :n] = o.permute(1, 0, 2).to(q.dtype)
        lse[b, :, :n] = (m + z.log())[..., 0]
    return out, lse


def _plain_read(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    shape = (c["layers"], c["B"], s["window"], c["Hkv"], c["d"])
    k, v = torch.zeros(shape, dtype=dt, device=DEV), torch.zeros(shape, dtype=dt, device=DEV)
    for b in range(c["B"]):
        page, at = _places(s, b, s["lo"][b], s["back"][b])
        k[:, b, :s["back"][b]] = _values(s["kc"][:, page, :, at], s["ks"][:, page, :, at]).transpose(0, 1).to(dt)
        v[:, b, :s["back"][b]] = _values(s["vc"][:, page, :, at], s["vs"][:, page, :, at]).transpose(0, 1).to(dt)
    return k, v


def _plain_write(s):
    c = s["case"]
    for b, n in enumerate(s["counts"]):
        page, at = _places(s, b, s["Ps"][b], n)
        for x, codes, scales in ((s["k"], s["kc"], s["ks"]), (s["v"], s["vc"], s["vs"])):
            rows = x[:, b, s["acc_nodes"][b, :n].long()] if c["kind"] == "commit" else x[:, b, :n]
            cq, sq = _quantise(rows)                                                       # [layers, n, Hkv, ...]
            codes[:, page, :, at], scales[:, page, :, at] = cq.transpose(0, 1), sq.transpose(0, 1)
    rest = [torch.zeros(c["B"], dtype=torch.int32, device=DEV)]
    if c["kind"] == "commit":
        slots = torch.full((c["B"], c["W"]), -1, dtype=torch.int32, device=DEV)
        for b, n in enumerate(s["counts"]):
            page, at = _places(s, b, s["Ps"][b], n)
            slots[b, :n] = (page * c["block"] if c["block"] else 0) + at
        rest = [slots] + rest
        added = s["accept_len"] + 1
    else:
        added = s["n_rows"]
    return (s["prefix_len"] + added, *rest, *_plain_read(s))


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"attn": _plain_attn, "read": _plain_read, "write": _plain_write, "commit": _plain_write}[c["kind"]](s)
    from paper_2603_08088_amd import api
    if c["kind"] == "attn":
        return api.tree_verify_attention_q4(s["q"], s["layer"], s["prefix_len"], s["kt"], s["vt"], s["bitmask"], s["n_nodes"],
                                            P_max=s["P_max"], block_table=s["block_table"], out=s["out"], lse=s["lse"],
                                            workspace=s["workspace"], desc=s["desc"])
    head = ()
    if c["kind"] == "write":
        r = api.quantize_kv_q4(s["k"], s["v"], s["cache"], s["prefix_len"], s["n_rows"], s["capacity"], block_table=s["block_table"])
        head = (r["prefix_len_out"], r["status"])
    elif c["kind"] == "commit":
        r = api.commit_accepted_kv_q4(s["k"], s["v"], s["cache"], s["prefix_len"], s["capacity"], s["n_nodes"], s["acc_nodes"],
                                      s["accept_len"], block_table=s["block_table"])
        head = (r["prefix_len_out"], r["slot_map"], r["status"])
    r = api.dequantize_kv_q4(s["cache"], s["first"], s["back_rows"], s["window"], block_table=s["block_table"],
                             out=dict(k=s["k_back"], v=s["v_back"]))
    return (*head, r["k"], r["v"])


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _nearest64(x):
    """What the cache holds for rows x [..., d]: of every group of 32 the nearest values on its grid, in float64."""
    g = x.double().reshape(*x.shape[:-1], -1, 32)
    top = g.abs().max(-1, keepdim=True).values
    _, e = torch.frexp(top)                                          # top = m * 2^e, m in [1/2, 1)
    e = e + (top >= torch.ldexp(torch.full_like(top, 0.875), e)).int()
    e = torch.where(top > 0, e, torch.full_like(e, -200)).clamp(-122, 128) - 3
    step = torch.ldexp(torch.ones_like(top), e)
    size = g.abs() / step
    best, gap = torch.zeros_like(size), size.clone()
    for i, v in enumerate(_GRID[1:], 1):
        new = (size - v).abs()
        closer = new < gap if i % 2 else new <= gap                  # a tie goes to the value with the even code
        best, gap = torch.where(closer, torch.full_like(best, v), best), torch.minimum(gap, new)
    return (best * step * torch.where(g < 0, -1.0, 1.0)).reshape(x.shape)


def _held64(s, codes, scales, layer, b, lo, n):
    """Positions lo .. lo + n - 1 of sequence b as the cache holds them: float64 [n, Hkv, d]."""
    pos = np.arange(lo, lo + n)
    size = s["case"]["block"]
    if size:
        page, at = _dev(s["table"][b][pos // size].astype(np.int64)), _dev(pos % size)
    else:
        page, at = _dev(np.full(n, b)), _dev(pos)
    both = np.array([[(-1.0 if h & 8 else 1.0) * _GRID[h & 7] for h in (byte & 15, byte >> 4)] for byte in range(256)])
    val = _dev(both)[codes[layer][page, :, at].int()].flatten(-2)
    return val * torch.pow(2.0, scales[layer][page, :, at].double() - 127).repeat_interleave(32, -1)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "attn":
        B, T, Hq, d = s["q"].shape
        G = Hq // c["Hkv"]
        out = torch.zeros((B, T, Hq, d), dtype=torch.float64, device=DEV)
        lse = torch.full((B, Hq, T), -math.inf, dtype=torch.float64, device=DEV)
        for b in range(B):
            n, P = s["ns"][b], s["Ps"][b]
            K = torch.cat((_held64(s, s["kc"], s["ks"], 0, b, 0, P), s["kt"][b, :n].double()))
            V = torch.cat((_held64(s, s["vc"], s["vs"], 0, b, 0, P), s["vt"][b, :n].double()))
            seen = torch.cat((torch.ones((n, P), dtype=torch.bool, device=DEV), s["vis"][b, :n, :n]), 1)
            for h in range(Hq):
                score = s["q"][b, :n, h].double() @ K[:, h // G].T.contiguous() / math.sqrt(d)
                score = torch.where(seen, score, -math.inf)
                lse[b, h, :n] = torch.logsumexp(score, 1)
                out[b, :n, h] = torch.exp(score - lse[b, h, :n, None]) @ V[:, h // G].contiguous()
        return out, lse
    back = []
    for codes, scales, new in ((s["kc"], s["ks"], s.get("k")), (s["vc"], s["vs"], s.get("v"))):
        y = torch.zeros((c["layers"], c["B"], s["window"], c["Hkv"], c["d"]), dtype=torch.float64, device=DEV)
        for b in range(c["B"]):
            for layer in range(c["layers"]):
                y[layer, b, :s["back"][b]] = _held64(s, codes, scales, layer, b, s["lo"][b], s["back"][b])
            if new is not None:
                rows = new[:, b][:, torch.as_tensor(s["acc"][b, :s["counts"][b]].astype(np.int64), device=DEV)] if c["kind"] == "commit" \
                    else new[:, b, :s["counts"][b]]
                y[:, b, MARGIN:MARGIN + s["counts"][b]] = _nearest64(rows)
        back.append(y)
    if c["kind"] == "read":
        return tuple(back)
    length = [P + n for P, n in zip(s["Ps"], s["counts"])]
    head = [torch.tensor(length, device=DEV, dtype=torch.int32)]
    if c["kind"] == "commit":
        slots = np.full((c["B"], c["W"]), -1, dtype=np.int32)
        for b, P in enumerate(s["Ps"]):
            for i in range(s["counts"][b]):
                slots[b, i] = s["table"][b][(P + i) // c["block"]] * c["block"] + (P + i) % c["block"] if c["block"] else P + i
        head.append(_dev(slots))
    head.append(torch.zeros(c["B"], dtype=torch.int32, device=DEV))
    return (*head, *back)
