"""The 4-bit prefix cache from its definition, in numpy and float64, and small seeded inputs for its tests."""
import math

import numpy as np
import torch

from paper_2603_08088_amd import api

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """x [..., d] -> codes uint8 [..., d/2], scales uint8 [..., d/32]."""
    g = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], -1, 32)
    finite = np.isfinite(g).all(-1)
    g = np.where(finite[..., None], g, 0.0)
    a = np.abs(g).max(-1)
    m, e = np.frexp(a)                                   # a = m * 2^e, 1/2 <= m < 1
    e = np.where(a > 0, e - 1 + (m >= 0.875), -1000)     # exponent after rounding to two significant bits
    s = np.clip(e + 127 - 2, 2, 252)
    y = np.abs(g) / np.ldexp(1.0, s - 127)[..., None]
    gap = np.abs(y[..., None] - GRID)                    # ties: the even code, which the added trifle prefers
    order = gap + 1e-9 * (np.arange(8) % 2)
    code = order.argmin(-1).astype(np.uint8) | (np.signbit(np.asarray(x, np.float64).reshape(g.shape)).astype(np.uint8) << 3)
    code = np.where(finite[..., None], code, 0).reshape(*x.shape).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), np.where(finite, s, 255).astype(np.uint8)


def values(codes, scales):
    nib = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1)
    v = GRID[nib & 7] * np.where(nib & 8, -1.0, 1.0)
    f = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (v.reshape(*scales.shape, 32) * f[..., None]).reshape(*codes.shape[:-1], -1)


def place(table, size, b, pos):
    """(page, offset) of a position: in block `table[b][pos // size]`, or in the sequence's own rows."""
    return (b, pos) if table is None else (int(table[b][pos // size]), pos % size)


def held(codes, scales, table, size, b, P):
    """Positions 0 .. P-1 of sequence b of one layer's tensors [blocks, Hkv, size, ...]: float64 [P, Hkv, d]."""
    if P == 0:
        return np.zeros((0, codes.shape[1], 2 * codes.shape[-1]))
    at = [place(table, size, b, j) for j in range(P)]
    page, off = np.array([a[0] for a in at]), np.array([a[1] for a in at])
    return values(codes[page, :, off], scales[page, :, off])


def attention(q, K, V, kt, vt, vis, n, scale):
    """One sequence: q [T,Hq,d], prefix K/V [P,Hkv,d], tree kt/vt [T,Hkv,d], vis bool [T,T].  Keys a row does not see are not
    touched.  Returns out [T,Hq,d], lse [Hq,T], and for the tolerances spread = sum of weight * |value| [T,Hq,d]."""
    T, Hq, d = q.shape
    P, G = K.shape[0], Hq // kt.shape[1]
    out, lse, spread = np.zeros((T, Hq, d)), np.full((Hq, T), -np.inf), np.zeros((T, Hq, d))
    for k in range(n):
        rows = np.flatnonzero(vis[k, :n])
        for h in range(Hq):
            Kk, Vv = np.concatenate((K[:, h // G], kt[rows, h // G])), np.concatenate((V[:, h // G], vt[rows, h // G]))
            if not len(Kk):
                continue
            with np.errstate(invalid="ignore", over="ignore"):
                s = Kk @ q[k, h] * scale
                m = s.max()
                w = np.exp(s - m)
                z = w.sum()
                out[k, h], spread[k, h] = w @ Vv / z, w @ np.abs(Vv) / z
                lse[h, k] = m + math.log(z) if np.isfinite(m) else np.nan
    return out, lse, spread


class Case:
    """A batch with a 4-bit prefix: host arrays, and the same on the GPU after .cuda()."""

    def __init__(self, seed, B, T, Hq, Hkv, d, dtype, Ps, block, ns=None, q_scale=1.0):
        rng = np.random.default_rng(seed)
        self.rng, self.B, self.T, self.Hq, self.Hkv, self.d, self.block = rng, B, T, Hq, Hkv, d, block
        self.dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
        self.Ps, self.ns = list(Ps), list(ns) if ns is not None else [T] * B
        self.P_max = max(self.Ps)
        real = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(self.dtype)
        self.q, self.kt, self.vt = real(B, T, Hq, d) * q_scale, real(B, T, Hkv, d), real(B, T, Hkv, d)
        room = max(self.P_max, 1) + 5
        if block:
            width = -(-room // block)
            pages, self.size = B * width + 3, block
            self.table = rng.permutation(pages)[:B * width].reshape(B, width).astype(np.int32)
        else:
            pages, self.size, self.table = B, room, None
        # positions behind a sequence hold codes with NaN scales: whoever reads them shows it
        shape = (pages, Hkv, self.size)
        self.codes = [rng.integers(0, 256, shape + (d // 2,)).astype(np.uint8) for _ in range(2)]
        self.scales = [np.full(shape + (d // 32,), 255, np.uint8) for _ in range(2)]
        for b, P in enumerate(self.Ps):
            if P:
                at = [place(self.table, self.size, b, j) for j in range(P)]
                page, off = np.array([a[0] for a in at]), np.array([a[1] for a in at])
                for x in range(2):
                    c, s = quantise(rng.standard_normal((P, Hkv, d)))
                    self.codes[x][page, :, off], self.scales[x][page, :, off] = c, s
        self.vis = np.zeros((B, T, T), bool)
        for b in range(B):
            for k in range(self.ns[b]):
                if k:
                    self.vis[b, k] = self.vis[b, int(rng.integers(max(0, k - 9), k))]
                self.vis[b, k, k] = True

    def words(self):
        bits = np.zeros((self.B, self.T, 64 * ((self.T + 63) // 64)), bool)
        bits[:, :, :self.T] = self.vis
        return np.packbits(bits, axis=2, bitorder="little").view(np.int64)

    def cache(self, layers=None):
        ts = [torch.from_numpy(a).cuda() for a in (self.codes[0], self.scales[0], self.codes[1], self.scales[1])]
        return api.KVCacheQ4(*(t if layers is None else t[None].repeat(layers, 1, 1, 1, 1) for t in ts))

    def tables(self):
        return None if self.table is None else torch.from_numpy(self.table).cuda()

    def ints(self, xs):
        return torch.tensor(xs, dtype=torch.int32, device="cuda")

    def run(self, scale=0.0, **kw):
        kw.setdefault("block_table", self.tables())
        P_max = kw.pop("P_max", self.P_max)
        return api.tree_verify_attention_q4(self.q.cuda(), self.cache(), self.ints(self.Ps), self.kt.cuda(), self.vt.cuda(),
                                            torch.from_numpy(self.words()).cuda(), self.ints(self.ns), P_max=P_max, scale=scale, **kw)

    def plain(self, scale=0.0):
        f, sc = (lambda t: t.double().numpy()), scale or 1 / math.sqrt(self.d)
        res = [attention(f(self.q[b]), *(held(self.codes[x], self.scales[x], self.table, self.size, b, self.Ps[b]) for x in range(2)),
                         f(self.kt[b]), f(self.vt[b]), self.vis[b], self.ns[b], sc) for b in range(self.B)]
        return tuple(np.stack(x) for x in zip(*res))

    def score_slack(self, scale=0.0):
        """How far a score may be off: the products of a row are exact or rounded to fp32 and added in fp32 (d + 8 roundings of at
        most 2^-24 of the sum of their magnitudes); q may enter them as a fixed-point number of 2^-18 (fp32: 2^-26) of its group's maximum."""
        G, sc = self.Hq // self.Hkv, abs(scale) or 1 / math.sqrt(self.d)
        q = np.abs(self.q.double().numpy())
        top = q.reshape(*q.shape[:-1], -1, 32).max(-1).repeat(32, -1)
        worst = 0.0
        for b in range(self.B):
            K = np.abs(np.nan_to_num(held(self.codes[0], self.scales[0], self.table, self.size, b, self.Ps[b])))
            for h in range(self.Hq):
                keys = np.concatenate((K[:, h // G], np.nan_to_num(np.abs(self.kt[b, :, h // G].double().numpy()), posinf=0)))
                if len(keys):
                    exactness = 2.0 ** (-18 if self.dtype == torch.bfloat16 else -26)
                    worst = max(worst, float((keys @ (top[b, :, h] * exactness + q[b, :, h] * (self.d + 8) * 2.0 ** -24).T).max()))
        return worst * sc

    def check(self, out, lse, scale=0.0):
        want, want_lse, spread = self.plain(scale)
        got, n = out.double().cpu().numpy(), self.P_max + self.T
        ds = self.score_slack(scale)
        half = torch.finfo(self.dtype).eps / 2
        # a weight is off by exp(2 ds), a rounding to the type (bf16: probabilities) and the fp32 sums over the keys; then the output is rounded
        weight = math.expm1(2 * ds) + (2 * half if self.dtype == torch.bfloat16 else 8 * 2.0 ** -24) + (n + 64) * 2.0 ** -24
        tol = weight * (spread + np.abs(want)) + half * np.abs(want) * 1.01 + 1e-30
        bad = ~(np.abs(got - want) <= tol) & ~(np.isnan(got) & np.isnan(want))
        assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], tol[bad][:3])
        for b in range(self.B):
            assert (got[b, self.ns[b]:] == 0).all()
        if lse is not None:
            g = lse.double().cpu().numpy()
            assert np.array_equal(np.isneginf(g), np.isneginf(want_lse))
            with np.errstate(invalid="ignore"):
                ok = np.isneginf(want_lse) | (np.isnan(g) & np.isnan(want_lse)) | (np.abs(g - want_lse) <= ds + weight + 2.0 ** -22 * (1 + np.abs(want_lse)))
            assert ok.all(), (np.argwhere(~ok)[:3], g[~ok][:3], want_lse[~ok][:3])
