"""rotary_write_kv on the GPU against its definition in extended precision."""
import numpy as np
import pytest
import torch

import beam_plain
from paper_2603_08088_amd import api

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def freqs(half):
    return (10000.0 ** (-np.arange(half) / half)).astype(np.float32)


class Case:
    def __init__(self, seed, B, T, Hq, Hkv, d, dtype, rot=None, axes=1, inter=False, far=4000, scale=1.0, fused=False):
        self.rng, self.scale, self.inter = np.random.default_rng(seed), scale, inter
        self.shape = B, T, Hq, Hkv, d
        rows = torch.from_numpy(self.rng.standard_normal((B, T, Hq + 2 * Hkv, d)).astype(np.float32)).to(DT[dtype])
        self.host = rows.split([Hq, Hkv, Hkv], 2)
        on = rows.cuda()
        self.q, self.k, self.v = on.split([Hq, Hkv, Hkv], 2) if fused else (t.contiguous() for t in on.split([Hq, Hkv, Hkv], 2))
        half = (rot or d) // 2
        self.inv_freq = freqs(half)
        self.axis_of = [int(a) for a in np.sort(self.rng.integers(0, axes, half))]
        self.positions = self.rng.integers(0, far, (axes, B, T))
        self.dtype, self.half = DT[dtype], half
        self.rotary = api.Rotary(dev(self.inv_freq, np.float32), axis_of=self.axis_of, interleaved=inter, scale=scale)

    def want(self, t, inverse=False):
        return beam_plain.rotate(t.double().numpy(), self.positions, self.inv_freq, self.axis_of, self.inter, self.scale, inverse)

    def close(self, got, t, inverse=False):
        """An angle is off by 2^-26 of a quarter turn (0.4 of 2^-24), the fp32 sine and cosine by two units in the last place (2^-24 each at most),
        the factor by a half, the two products and their sum by one: less than 5 * 2^-24 of |x| + |y|; then one rounding."""
        x = np.abs(t.double().numpy())
        pair = beam_plain.rotate(x, np.zeros_like(self.positions), self.inv_freq * 0, self.axis_of, self.inter)
        r = 2 * self.half
        if self.inter:
            pair[..., :r:2] = pair[..., 1:r:2] = x[..., :r:2] + x[..., 1:r:2]
        else:
            pair[..., :self.half] = pair[..., self.half:r] = x[..., :self.half] + x[..., self.half:r]
        want = self.want(t, inverse)
        slack = 5 * 2.0 ** -24 * pair * abs(self.scale)
        slack[..., r:] = 0
        slack += (torch.finfo(self.dtype).eps / 2 if self.dtype == torch.bfloat16 else 0) * (np.abs(want) + slack)
        off = np.abs(got.double().cpu().numpy() - want)
        assert (off <= slack).all(), (off - slack).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("B,T,Hq,Hkv,d,rot,axes,fused", [
    (1, 1, 1, 1, 16, None, 1, False), (8, 1, 32, 8, 128, None, 1, True), (2, 60, 32, 8, 128, None, 1, False), (3, 77, 12, 4, 128, 64, 3, True),
    (2, 33, 28, 4, 64, None, 2, False), (1, 130, 5, 1, 80, 32, 3, True), (2, 9, 3, 3, 256, 256, 3, False), (1, 1025, 4, 2, 64, 48, 1, True), (5, 2, 40, 10, 96, None, 1, False)])
def test_rows_turn_as_defined(dtype, inter, B, T, Hq, Hkv, d, rot, axes, fused):
    c = Case(B * T, B, T, Hq, Hkv, d, dtype, rot, axes, inter, fused=fused)
    v = torch.empty((B, T, Hkv, d), dtype=c.dtype, device="cuda")
    r = api.rotary_write_kv(c.q, c.k, c.v, dev(c.positions), c.rotary, out=dict(v=v))
    c.close(r["q"], c.host[0])
    c.close(r["k"], c.host[1])
    assert torch.equal(v, c.v)
    # and back
    r = api.rotary_write_kv(c.q, c.k, None, dev(c.positions), c.rotary, inverse=True)
    c.close(r["q"], c.host[0], True)
    c.close(r["k"], c.host[1], True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [0, 1, 16, 48])
@pytest.mark.parametrize("T", [1, 19, 300])
def test_rows_go_to_their_slots_and_nothing_else_changes(dtype, block, T):
    B, Hkv, d = 3, 2, 64
    c = Case(T, B, T, 4, Hkv, d, dtype, axes=3, fused=True)
    room = T + 40
    shape = (B * (-(-room // block)) + 2, Hkv, block, d) if block else (B, room, Hkv, d)
    rows = shape[0] * block if block else B * room
    slots = c.rng.permutation(rows)[:B * T].reshape(B, T).astype(np.int64)
    slots[c.rng.random((B, T)) < 0.2] = -1
    slots[0, 0], slots[1, 0] = rows, 2 ** 31 - 1                       # outside the cache
    n = [T, max(1, T // 2), 0]
    kc, vc = (torch.from_numpy(c.rng.standard_normal(shape).astype(np.float32)).to(c.dtype).cuda() for _ in range(2))
    kc0, vc0 = kc.clone(), vc.clone()
    q = torch.full((B, T, 4, d), 7, dtype=c.dtype, device="cuda")
    r = api.rotary_write_kv(c.q, c.k, c.v, dev(c.positions), c.rotary, n_rows=dev(n), slot_map=dev(slots), k_cache=kc, v_cache=vc, paged=block > 0, out=dict(q=q))
    assert r["k"] is None and r["v"] is None
    alone = api.rotary_write_kv(c.q, c.k, None, dev(c.positions), c.rotary)
    for b in range(B):
        assert torch.equal(q[b, :n[b]], alone["q"][b, :n[b]]) and bool((q[b, n[b]:] == 7).all())
        for t in range(n[b]):
            s = int(slots[b, t])
            if 0 <= s < rows:
                at = (s // block, slice(None), s % block) if block else (s // room, s % room)
                kc0[at], vc0[at] = alone["k"][b, t], c.v[b, t]
    assert torch.equal(kc, kc0) and torch.equal(vc, vc0)


@pytest.mark.parametrize("inter", [False, True])
def test_far_positions_of_either_sign(inter):
    """Angles of up to 2^31 radians: the definition's product is exact, and so is what is left of it."""
    c = Case(3, 2, 7, 2, 1, 64, "f32", axes=2, inter=inter)
    c.positions[:] = np.array([0, 1, -1, 10 ** 6 + 1, -(2 ** 31), 2 ** 31 - 1, 123456789])
    r = api.rotary_write_kv(c.q, c.k, None, dev(c.positions), c.rotary)
    # 53 of the product's 55 bits are kept: up to 2^-22 radians at 2^31
    want, got = c.want(c.host[0]), r["q"].double().cpu().numpy()
    assert np.abs(got - want).max() <= 2.0 ** -21 * np.abs(c.host[0].numpy()).max() * 2
    near = slice(0, 4)
    assert np.abs(got[:, near] - want[:, near]).max() <= 5 * 2.0 ** -24 * 2 * np.abs(c.host[0].numpy()).max()


def test_an_output_may_be_its_input_and_parts_may_be_left_out():
    c = Case(4, 2, 50, 6, 2, 128, "bf16", rot=64, axes=3, fused=True, scale=0.75)
    p = dev(c.positions)
    want = api.rotary_write_kv(c.q, c.k, None, p, c.rotary)
    c.close(want["q"], c.host[0])
    q, k = c.q.clone(), c.k
    api.rotary_write_kv(c.q, c.k, c.v, p, c.rotary, out=dict(q=c.q, k=c.k, v=c.v))       # within the projection's output
    assert torch.equal(c.q, want["q"]) and torch.equal(c.k, want["k"]) and c.k is k
    only = api.rotary_write_kv(q, None, None, p, c.rotary)
    assert torch.equal(only["q"], want["q"]) and only["k"] is None


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("scale", [1.0, -1.5])
def test_the_inverse_is_the_gradient(inter, scale):
    """<g, R(x + h) - R(x - h)> / 2 = <R^T(g), h>: R is linear, so differences are exact but for rounding."""
    c = Case(5, 2, 11, 3, 2, 64, "f32", rot=48, axes=3, inter=inter, scale=scale)
    p = dev(c.positions)
    turn = lambda x, **kw: api.rotary_write_kv(x, None, None, p, c.rotary, **kw)["q"].double()
    g, h = (torch.randn(c.q.shape, device="cuda") for _ in range(2))
    ahead = (turn(c.q + h) - turn(c.q - h)) / 2
    left, right = (g.double() * ahead).sum().item(), (turn(g, inverse=True) * h.double()).sum().item()
    size = (g.double().abs() * (c.q.abs() + h.abs()).double()).sum().item()
    assert abs(left - right) <= 16 * 2.0 ** -24 * abs(scale) * size
    # and by the formula: each entry of the gradient of sum(g * R(x))
    want = beam_plain.rotate(g.double().cpu().numpy(), c.positions, c.inv_freq, c.axis_of, inter, scale, True)
    assert np.abs(turn(g, inverse=True).cpu().numpy() - want).max() <= 5 * 2.0 ** -24 * abs(scale) * 2 * g.abs().max().item()


def test_positions_of_a_tree():
    """tensorize_tree's position_ids as they come: node k at prefix + depth."""
    parent = dev([[0, 0, 0, 1, 1, 2, 3, 0]])
    n, P = dev([7]), dev([1000])
    m = api.tensorize_tree(parent, n, P, 8, 8)
    c = Case(6, 1, 8, 4, 2, 64, "bf16")
    c.positions = np.array([[[1000, 1001, 1001, 1002, 1002, 1002, 1003, 1000]]])
    r = api.rotary_write_kv(c.q, c.k, None, m["position_ids"], c.rotary)
    c.close(r["q"], c.host[0])


def test_values_that_are_not_finite_stay_with_their_pairs():
    c = Case(7, 1, 4, 2, 1, 64, "f32")
    c.q[0, 1, 0, 3], c.q[0, 2, 1, 40] = float("nan"), float("inf")
    r = api.rotary_write_kv(c.q, None, None, dev(c.positions), c.rotary)["q"]
    bad = torch.zeros_like(r, dtype=torch.bool)
    bad[0, 1, 0, [3, 35]] = bad[0, 2, 1, [8, 40]] = True
    assert torch.equal(~torch.isfinite(r), bad)


def test_layouts_of_inputs_and_outputs():
    """Tokens before sequences, one row of a larger tensor, one sequence for all: any strides that keep rows apart."""
    c = Case(8, 3, 5, 4, 2, 64, "bf16", axes=2)
    p = dev(c.positions)
    want = api.rotary_write_kv(c.q, c.k, None, p, c.rotary)
    turned = torch.empty((5, 3, 4, 64), dtype=c.dtype, device="cuda").transpose(0, 1)
    r = api.rotary_write_kv(c.q.transpose(0, 1).contiguous().transpose(0, 1), None, None, p, c.rotary, out=dict(q=turned))
    assert torch.equal(r["q"], want["q"])
    r = api.rotary_write_kv(c.q[:1].expand(3, 5, 4, 64), None, None, p, c.rotary)
    for b in range(3):
        alone = api.rotary_write_kv(c.q[:1], None, None, p[:, b:b + 1].contiguous(), c.rotary)
        assert torch.equal(r["q"][b], alone["q"][0])
    one = c.q[1:2, 2:3].as_strided((1, 1, 4, 64), (1, 3, 64, 1))
    r = api.rotary_write_kv(one, None, None, p[:, 1:2, 2:3].contiguous(), c.rotary)
    assert torch.equal(r["q"][0, 0], want["q"][1, 2])
    with pytest.raises(api.EtvError):
        api.rotary_write_kv(c.q, None, None, p, c.rotary, out=dict(q=want["q"][:1].expand(3, 5, 4, 64)))
    with pytest.raises(ValueError):                       # channels of a head that are not side by side with the next head's
        api.rotary_write_kv(c.q[..., 8:40], None, None, p, api.Rotary(dev(freqs(16), np.float32)))


def test_an_empty_batch():
    q = torch.empty((0, 3, 2, 64), device="cuda")
    r = api.rotary_write_kv(q, None, None, torch.empty((0, 3), dtype=torch.int32, device="cuda"), api.Rotary(dev(freqs(32), np.float32)))
    assert r["q"].shape == q.shape


@pytest.mark.parametrize("paged", [True, False])
def test_a_cache_of_more_than_2_32_elements(paged):
    c = Case(23, 2, 5, 8, 8, 128, "bf16")
    rows = (1 << 22) + 4096
    shape = (rows // 16, 8, 16, 128) if paged else (2, rows // 2, 8, 128)
    k, v = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slots = np.array([[rows - 1, rows - 17, 0, 1 << 22, (1 << 22) - 1], [rows - 2, 5, rows, 1 << 21, rows // 2]])
    plain = api.rotary_write_kv(c.q, c.k, c.v, dev(c.positions), c.rotary)
    api.rotary_write_kv(c.q, c.k, c.v, dev(c.positions), c.rotary, slot_map=dev(slots), k_cache=k, v_cache=v, paged=paged)
    for cache, want in ((k, plain["k"]), (v, c.v)):
        for (b, t), s in np.ndenumerate(slots):
            if s < rows:
                got = cache[s // 16, :, s % 16] if paged else cache.view(rows, 8, 128)[s]
                assert torch.equal(got, want[b, t]), s
                got.zero_()
        assert not any(part.any() for part in cache.view(-1).split(1 << 30))


@pytest.mark.parametrize("T,Hq,Hkv,d,rot", [(900, 32, 8, 128, None), (10000, 3, 1, 64, 32), (2100, 1, 1, 16, None)])
@pytest.mark.parametrize("dtype,inter", [("bf16", False), ("f32", True)])
def test_padding_of_many_rows_is_left_alone(T, Hq, Hkv, d, rot, dtype, inter):
    """Batches large enough that padding is not even read; tokens that share a workgroup are of two sequences, of padding and of none."""
    B = 3
    c = Case(T, B, T, Hq, Hkv, d, dtype, rot=rot, inter=inter, axes=2)
    n = [T - 1, 0, T // 2 + 3]
    every = api.rotary_write_kv(c.q, c.k, None, dev(c.positions), c.rotary)
    c.close(every["q"], c.host[0])
    slots = c.rng.permutation(B * T).reshape(B, T)
    kc, vc = (torch.full((B, T, Hkv, d), 3, dtype=c.dtype, device="cuda") for _ in range(2))
    out = dict(q=torch.full_like(c.q, 7), k=torch.full_like(c.k, 7), v=torch.full_like(c.v, 7))
    api.rotary_write_kv(c.q, c.k, c.v, dev(c.positions), c.rotary, n_rows=dev(n), slot_map=dev(slots), k_cache=kc, v_cache=vc, paged=False, out=out)
    there = torch.zeros((B, T), dtype=torch.bool, device="cuda")
    for b in range(B):
        there[b, :n[b]] = True
    for name, want in (("q", every["q"]), ("k", every["k"]), ("v", c.v)):
        assert torch.equal(out[name], torch.where(there[..., None, None], want, torch.full_like(want, 7))), name
    at = torch.from_numpy(slots).cuda()[there]
    for cache, want in ((kc, every["k"]), (vc, c.v)):
        expect = torch.full_like(cache, 3)
        expect.view(B * T, Hkv, d)[at] = want[there]
        assert torch.equal(cache, expect)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("far", [2 ** 24, 2 ** 28, 2 ** 31])
def test_far_positions_are_good_to_fp32(far, dtype, inter):
    """The bound of near positions holds for all of them, of either sign, with frequencies of 24 bits: what 64 bits lose of the product and of 2 / pi is
    added again."""
    c = Case(9, 2, 601, 3, 2, 64, dtype, axes=2, inter=inter)
    c.positions = c.rng.integers(-far, far, (2, 2, 601))
    c.positions[:, 0, :4] = [-far, far - 1, far // 2 + 1, 1 - far]
    c.inv_freq = c.rng.uniform(0.5, 1.5, 32).astype(np.float32)
    c.rotary = api.Rotary(dev(c.inv_freq, np.float32), axis_of=c.axis_of, interleaved=inter)
    p = dev(c.positions)
    for inverse in (False, True):
        r = api.rotary_write_kv(c.q, c.k, None, p, c.rotary, inverse=inverse)
        c.close(r["q"], c.host[0], inverse)
        c.close(r["k"], c.host[1], inverse)
