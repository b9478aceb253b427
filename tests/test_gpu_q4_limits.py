"""tree_verify_attention_q4 on the GPU at the limits of what it takes: scores, lengths, layouts and every form of its kernel."""
import copy
import math

import numpy as np
import pytest
import torch

from paper_2603_08088_amd import api
from q4_plain import Case, place, quantise

pytestmark = pytest.mark.gpu


def call(c, cache, **kw):
    """The call of Case.run on a cache of the caller's (one layer)."""
    return api.tree_verify_attention_q4(c.q.cuda(), cache, c.ints(c.Ps), c.kt.cuda(), c.vt.cuda(), torch.from_numpy(c.words()).cuda(),
                                        c.ints(c.ns), P_max=c.P_max, block_table=c.tables(), **kw)


def hold(c, x, b, lo, rows):
    """Rows [n, Hkv, d] of K (x = 0) or V (1) into positions lo .. of sequence b."""
    codes, scales = quantise(rows)
    for i in range(len(rows)):
        page, off = place(c.table, c.size, b, lo + i)
        c.codes[x][page, :, off], c.scales[x][page, :, off] = codes[i], scales[i]


def scale_for(log2_scale):
    """The largest float32 whose product with log2(e) in float32 is `log2_scale`."""
    one, s = np.float32(1.4426950408889634), np.float32(log2_scale * math.log(2) * (1 + 2.0 ** -20))
    while s * one > np.float32(log2_scale):
        s = np.nextafter(s, np.float32(0))
    assert s * one == np.float32(log2_scale)
    return float(s)


@pytest.mark.parametrize("d,T,Hq", [(64, 16, 2), (128, 16, 2), (64, 128, 2), (128, 128, 4)])
@pytest.mark.parametrize("log2_scale", [2 - 2.0 ** -22, 0.125 - 2.0 ** -26, 2 - 2.0 ** -13, 1.0, 0.18])
def test_queries_just_under_a_power_of_two_keep_their_bits(d, T, Hq, log2_scale):
    """One key, one channel of q: lse is the score.  q comes as a number of four digits, off by at most 2^-17.95 of it; beside that
    are some twelve fp32 roundings (the scale's two, q's, one a product, the logarithm's)."""
    scale = scale_for(np.float32(log2_scale)) if log2_scale != 0.18 else 0.18 * math.log(2)
    for part in range(0, 128, T):
        c = Case(1, 1, T, Hq, 2, d, "bf16", [1], 0)
        c.vis[:] = False                             # the tree's keys are not seen
        c.q[:] = 0
        mantissas = 1 + torch.arange(part, part + T) / 128
        c.q[0, :, :, d - 3] = mantissas[:, None].to(torch.bfloat16)
        row = np.zeros((1, 2, d))
        row[0, :, d - 3] = 96
        hold(c, 0, 0, 0, row)
        _, lse = c.run(scale=scale)
        want = mantissas.double()[None, None] * 96 * float(np.float32(scale))
        off = ((lse.double().cpu() - want).abs() / want).max().item()
        assert off <= 2.0 ** -17.95 + 12 * 2.0 ** -24, off


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_layer_of_a_cache_of_odd_rows(dtype):
    """Scales of heads of 64 are two bytes a row: the second layer of 1003 rows starts at an odd pair."""
    c = Case(2, 1, 3, 4, 1, 64, dtype, [998], 0)
    assert c.size == 1003
    cache = c.cache(layers=3)
    assert cache.layer(1).k_scales.data_ptr() % 4 == 2
    for layer in range(3):
        for kw in (dict(), dict(kv_split=128), dict(flags=api.ATTN_FLAG_GENERIC)):
            c.check(*call(c, cache.layer(layer), **kw))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,Ps,kw", [(6, [0], {}), (70, [0], {}), (6, [0, 600], dict(kv_split=64)), (40, [0, 600], dict(kv_split=64)),
                                     (40, [0, 600], dict(flags=api.ATTN_FLAG_GENERIC))])
def test_rows_that_see_only_a_score_of_minus_infinity(dtype, T, Ps, kw):
    """They see a key, so they are NaN, as the definition's quotient is; a row that sees none is zeros and -inf."""
    c = Case(3, len(Ps), T, 8, 2, 64, dtype, Ps, 16)
    c.vis[0] = False
    c.vis[0, 3:, 4] = True                           # rows 0 .. 2 see nothing, the others this key
    c.kt[0, 4, 0, 9], c.kt[0, 4, 1, 9] = float("inf"), float("-inf")
    c.q[0, :, :4, 9], c.q[0, :, 4:, 9] = -1, 2
    out, lse = c.run(**kw)
    assert (out[0, :3] == 0).all() and torch.isneginf(lse[0, :, :3]).all()
    assert torch.isnan(out[0, 3:]).all() and torch.isnan(lse[0, :, 3:]).all()
    assert torch.isfinite(out[1:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,Hq,d", [(1, 8, 128), (5, 8, 64), (13, 8, 128), (40, 8, 128), (40, 8, 64)])
@pytest.mark.parametrize("P,low,tree_low", [(20, -200, -200), (300, -90, -90), (700, -200, -200), (700, -5000, -4990), (700, -150, -700), (40, -400, 30)])
def test_rows_whose_scores_are_all_far_below_zero(dtype, T, Hq, d, P, low, tree_low):
    """A softmax does not change when all scores fall by the same amount: those of the prefix about `low`, the tree's about `tree_low`;
    whole and in splits, where wavefronts and splits without keys stand beside those with."""
    c = Case(8, 2, T, Hq, 2, d, dtype, [P, P // 2], 16)
    K = c.rng.standard_normal((P, 2, d))
    K[:, :, d - 32:] = 0
    K[:, :, d - 1] = low / 4
    c.q[..., d - 32:], c.q[..., d - 1] = 0, 4 * math.sqrt(d)
    c.kt[..., d - 32:], c.kt[..., d - 1] = 0, tree_low / 4
    for b in range(2):
        hold(c, 0, b, 0, K[:c.Ps[b]])
    for kv_split in (4096, 128):
        c.check(*c.run(kv_split=kv_split))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,Hq,d", [(5, 8, 128), (13, 8, 64), (40, 8, 128), (40, 8, 64)])
@pytest.mark.parametrize("none,P,kv_split", [(300, 700, 4096), (300, 700, 512), (300, 300, 4096), (257, 1200, 4096)])
def test_tiles_whose_scores_overflow_to_minus_infinity_weigh_nothing(dtype, T, Hq, d, none, P, kv_split):
    """The first keys score -inf for every row, the others 2^-384: such keys weigh nothing, wherever a wavefront meets them.
    The scale is a power of two in base 2 and q's large value one too, so that its lower digits are zero."""
    c, scale = Case(4, 1, T, Hq, 2, d, dtype, [P], 16), scale_for(0.125)
    K = c.rng.standard_normal((P, 2, d))
    K[:, :, :32], K[:, :, 40], c.kt[..., :32], c.kt[..., 40] = 0, -384, 0, -384
    hold(c, 0, 0, 0, K)
    small = copy.deepcopy(c)                         # for the tolerance: without the keys that weigh nothing
    K[:none, :, 3] = -1e38
    hold(c, 0, 0, 0, K)
    for x in (c, small):
        x.q[..., :32], x.q[..., 3], x.q[..., 40] = 0, 2.0 ** 126, 8
    small.plain = c.plain
    small.check(*c.run(scale=scale, kv_split=kv_split), scale=scale)


@pytest.mark.parametrize("B,kv_split", [(1, 0), (1, 1 << 24), (65, 0)])
def test_prefixes_up_to_the_longest(B, kv_split):
    """2^31 - 4097 positions, all but the last 2^20 - 4097 in one block, which weighs nothing: what is out comes from those."""
    d, size, width = 64, 1 << 20, 2048
    P = 2 ** 31 - 4097
    kc, ks, vc, vs = (torch.zeros((2, 1, size, w), dtype=torch.uint8, device="cuda") for w in (d // 2, d // 32, d // 2, d // 32))
    kc[0], ks[:], vs[:] = 0xff, 127 + 3, 127                         # K: -48 throughout; V: 0
    vc[1] = 0x22                                                     # V: 1
    table = torch.zeros((B, width), dtype=torch.int32, device="cuda")
    table[:, -1] = 1
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    lens[B // 2] = P
    q, kt = torch.ones((B, 1, 1, d), dtype=torch.bfloat16, device="cuda"), torch.full((B, 1, 1, d), -48.0, dtype=torch.bfloat16, device="cuda")
    mask, n = torch.ones((B, 1, 1), dtype=torch.int64, device="cuda"), torch.ones(B, dtype=torch.int32, device="cuda")
    out, lse = api.tree_verify_attention_q4(q, api.KVCacheQ4(kc, ks, vc, vs), lens, kt, torch.full_like(kt, 3), mask, n, P_max=P, block_table=table,
                                            kv_split=kv_split)
    # sums and outputs of equal weights are whole numbers below 2^24 a lane
    assert torch.equal(out[B // 2], torch.ones_like(out[0])) and abs(lse[B // 2].item() - math.log(2 ** 20 - 4097)) <= 2.0 ** -20 * 14
    others = torch.arange(B, device="cuda") != B // 2
    assert (out[others] == 3).all() and (lse[others] + 48 * 8).abs().le(2.0 ** -10).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [3, 10, 40])
@pytest.mark.parametrize("rising", [False, True])
def test_references_move_in_the_middle_of_long_prefixes(dtype, d, T, rising):
    """Scores far apart, met at random or each tile far above the one before: rows get a new reference tile after tile."""
    c = Case(5, 1, T, 8, 2, d, dtype, [3000], 16, q_scale=12.0)
    if rising:
        K = c.rng.standard_normal((3000, 2, d))
        K[:, :, 7] = np.arange(3000)[:, None] / 8
        hold(c, 0, 0, 0, K)
        c.q[..., 7] = 16 * d / 64
    for kv_split in (4096, 1024):
        c.check(*c.run(kv_split=kv_split))


@pytest.mark.parametrize("kv_split", [4096, 256])
@pytest.mark.parametrize("block", [0, 48])
@pytest.mark.parametrize("T", [5, 13, 33])            # rows of one, two and four wavefronts
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_every_form_of_the_kernel_reads_a_prefix(d, dtype, T, block, kv_split):
    """Both head sizes and types, rows of one, two and four wavefronts, either layout, split and whole; prefixes end inside a tile."""
    c = Case(6, 3, T, 8, 2, d, dtype, [523, 70, 257], block, [T, T - 1, T])
    c.check(*c.run(kv_split=kv_split))


@pytest.mark.parametrize("T,Hq,d", [(6, 8, 128), (14, 8, 64), (40, 8, 128), (40, 4, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_finite_rows_beside_values_that_are_not(dtype, T, Hq, d):
    """Infinities and NaN in tree K and V that some rows see: the other rows, and the other columns, keep their precision."""
    c = Case(7, 1, T, Hq, 2, d, dtype, [37], 16)
    c.kt[0, 1, 0, 9], c.kt[0, 3, 1, d - 1] = float("nan"), float("inf")
    c.vt[0, 2, 0, 33], c.vt[0, 2, 1, 3], c.vt[0, 4, 1, 5] = float("inf"), float("nan"), float("-inf")
    c.vis[0] = c.rng.random((T, T)) < 0.3
    out, _ = c.run()
    want, _, spread = c.plain()
    got, fine = out.double().cpu().numpy(), np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isposinf(got), np.isposinf(want)) and fine.any() and not fine.all()
    # the bound of Case.check
    ds, half = c.score_slack(), torch.finfo(c.dtype).eps / 2
    weight = math.expm1(2 * ds) + (2 * half if dtype == "bf16" else 8 * 2.0 ** -24) + (37 + T + 64) * 2.0 ** -24
    off = np.abs(got[fine] - want[fine]) - weight * (spread[fine] + np.abs(want[fine])) - half * np.abs(want[fine]) * 1.01
    assert off.max() <= 1e-30, off.max()


@pytest.mark.parametrize("T,kv_split", [(3, 4096), (40, 64)])
def test_outputs_do_not_depend_on_lse_or_the_workspace(T, kv_split):
    c = Case(9, 2, T, 8, 2, 64, "bf16", [300, 41], 16)
    want, _ = c.run(kv_split=kv_split)
    used = torch.full((1 << 26,), 0xff, dtype=torch.uint8, device="cuda")        # larger than asked for, NaN throughout
    for kw in (dict(want_lse=False), dict(workspace=used), dict(want_lse=False, flags=api.ATTN_FLAG_GENERIC)):
        got, lse = c.run(kv_split=kv_split, **kw)
        assert (lse is None) == ("want_lse" in kw)
        assert "flags" in kw or torch.equal(got, want)
        c.check(got, lse)
