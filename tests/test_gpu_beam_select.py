"""beam_select on the GPU against its definition in 64 bits: the choices exactly, the scores to their rounding."""
import math

import numpy as np
import pytest
import torch

import beam_plain
from paper_2603_08088_amd import api

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def slack(x, parent):
    """How far a total may be off before its rounding: the relative error of its beam's sum.  A term exp(t) is an fp32 exponential of y = t log2(e):
    y is rounded twice (2^-24 |t| in exp(t) each time), and the function is good to a unit in the last place (2^-23); so 2^-23 (1 + |t|), weighted
    with the terms.  t is relative to a reference that may lie 1 below the row's maximum, which adds 1 to its size at most: 2^-23 (2 + |x - max|).  At
    most 10 fp32 additions lie between a term and the 64-bit sum (2^-24 each)."""
    off = np.zeros(parent.shape)
    with np.errstate(invalid="ignore", over="ignore"):
        t = x - x.max(-1, keepdims=True)
        p = np.exp(t)
        mean = np.where(p > 0, p * -t, 0).sum(-1) / p.sum(-1)
    for b in range(len(parent)):
        off[b] = np.nan_to_num(mean[b])[np.maximum(parent[b], 0)]
    return 2.0 ** -23 * (2 + off) + 10 * 2.0 ** -24


def check(logits, scores, M, n_beams=None, finished=None, end=-1, **kw):
    """logits: a host tensor [B, K, V]."""
    r = api.beam_select(kw.pop("on", None) if "on" in kw else logits.cuda(), dev(scores, np.float32), M, n_beams=None if n_beams is None else dev(n_beams),
                        finished=None if finished is None else dev(finished, np.uint8), end_token=end, **kw)
    with np.errstate(invalid="ignore"):
        best, parent, token, ended, status = beam_plain.select(logits.double().numpy(), np.asarray(scores, dtype=np.float32), M, n_beams, finished, end)
    assert np.array_equal(r["parent"].cpu().numpy(), parent) and np.array_equal(r["token"].cpu().numpy(), token)
    assert np.array_equal(r["finished"].cpu().numpy(), ended) and r["status"].tolist() == status
    got = r["scores"].double().cpu().numpy()
    fine = np.isfinite(best)
    assert np.array_equal(got[~fine], best[~fine])
    assert (np.abs(got[fine] - best[fine]) <= (slack(logits.double().numpy(), parent) + 2.0 ** -24 * np.abs(best) * (1 + 1e-6))[fine]).all()
    return r


def normal(rng, shape, dtype, spread=2.0):
    return torch.from_numpy((spread * rng.standard_normal(shape)).astype(np.float32)).to(DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,K,M,V", [(1, 1, 1, 1), (1, 1, 8, 5), (2, 3, 4, 7), (1, 4, 4, 1000), (3, 8, 8, 4097), (2, 10, 10, 32000), (1, 64, 64, 3001), (4, 5, 64, 8192),
                                     (1, 1, 60, 50021), (70, 2, 3, 300), (2, 64, 1, 2048)])
def test_the_best_continuations(B, K, M, V, dtype):
    rng = np.random.default_rng(V + M)
    check(normal(rng, (B, K, V), dtype), -5 * rng.random((B, K)), M)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [0, 1, 3, 8])
def test_rows_apart_and_odd_vocabularies(dtype, pad):
    """Rows that begin at any element; what lies between them is not looked at."""
    rng = np.random.default_rng(pad)
    B, K, V = 3, 5, 5003
    whole = torch.full((B + 1, K + 1, V + pad), float("nan"), dtype=DT[dtype])
    x = normal(rng, (B, K, V), dtype)
    whole[1:, 1:, :V] = x
    check(x, -rng.random((B, K)), 7, on=whole.cuda()[1:, 1:, :V])


def test_one_row_for_all_beams():
    rng = np.random.default_rng(21)
    x = normal(rng, (3, 1, 6001), "bf16")
    check(x.expand(3, 4, 6001), -rng.random((3, 4)), 9, on=x.cuda().expand(3, 4, 6001))
    check(x[:1].expand(3, 4, 6001), -rng.random((3, 4)), 9, on=x[:1].cuda().expand(3, 4, 6001))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 4, 33, 64])
def test_ties_go_to_the_lowest(dtype, M):
    """Equal logits everywhere, few different values, equal beams: the lower beam, then the lower token."""
    rng = np.random.default_rng(M)
    check(torch.zeros((2, 3, 9001), dtype=DT[dtype]), np.zeros((2, 3)), M)
    check(torch.from_numpy(rng.integers(0, 3, (2, 4, 8193)).astype(np.float32)).to(DT[dtype]), -np.tile(rng.integers(0, 2, (2, 1)), (1, 4)), M)
    x = normal(rng, (2, 1, 5001), dtype).expand(2, 6, 5001).contiguous()      # six beams alike, each row at another alignment
    check(x, np.full((2, 6), -1.25), M)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_logits_finished_and_missing_beams(dtype):
    rng = np.random.default_rng(9)
    B, K, V, M = 6, 7, 6007, 9
    x = normal(rng, (B, K, V), dtype)
    x[torch.from_numpy(rng.random((B, K, V)) < 0.995)] = -math.inf
    x[0, 2] = x[1] = -math.inf                                        # beams that offer nothing, a request that does not
    x[2, 1, :], x[2, 1, 4000] = -math.inf, 3.0                        # one token, of probability 1
    x[3, 0, 17] = torch.finfo(DT[dtype]).min                          # lowest value: an offer like any other
    n, done = rng.integers(0, K + 1, B), (rng.random((B, K)) < 0.3).astype(np.uint8)
    n[2], done[2, 1], scores = K, 0, -4 * rng.random((B, K))
    scores[4, :3] = -math.inf
    check(x, scores, M, n, done, 4000)
    check(x, scores, M, n, None, 4000)
    check(x, scores, M, None, done, 0)
    check(x, scores, M, [0] * B, done, 0)
    check(x, scores, M, None, np.ones((B, K), dtype=np.uint8), V - 1)
    lone = torch.full((1, 2, 5000), torch.finfo(DT[dtype]).min, dtype=DT[dtype])
    check(lone, [[0.0, -1.0]], 5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", [math.nan, math.inf])
def test_beams_that_are_not_finite_offer_nothing_and_are_reported(dtype, what):
    rng = np.random.default_rng(11)
    for at in (0, 4095, 4096, 8999):
        x = normal(rng, (3, 4, 9000), dtype)
        x[0, 1, at] = x[1, 3, at] = what
        x[2, 2, at] = what                                            # a finished beam's logits do not matter
        scores = -rng.random((3, 4))
        scores[1, 0] = what
        r = check(x, scores, 6, None, np.array([[0, 0, 0, 0], [0, 0, 0, 0], [0, 0, 1, 0]]), 7)
        assert r["status"].tolist() == [1, 3, 0]


@pytest.mark.parametrize("spread", [0.0, 0.3, 30.0, 1e4])
def test_totals_far_apart_and_close_together(spread):
    rng = np.random.default_rng(12)
    for dtype in DT:
        check(normal(rng, (2, 6, 20011), dtype, spread), -100 * rng.random((2, 6)), 16)
    big = torch.from_numpy((3e38 * rng.uniform(-1, 1, (1, 2, 5000))).astype(np.float32))
    check(big, [[0.0, -1.0]], 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [300.0, -3e5, 7e5, 1048576.0, -2e6, 1e9, -1e30, 3e38])
def test_logits_far_from_zero(offset, dtype):
    """Terms are relative to a reference whose product with log2(e) 32 bits round; masks of the type's lowest value are far from every reference."""
    rng = np.random.default_rng(17)
    x = (normal(rng, (2, 3, 9001), "f32", 2.0) + offset).to(DT[dtype])
    x[:, 1, ::3] = torch.finfo(DT[dtype]).min
    x[1, 2, :5000] = -math.inf
    x[0, 0, 8000] += x[0, 0].abs().max() * 0.01
    check(x, -rng.random((2, 3)), 5)


def test_close_calls_between_beams():
    """Totals of different beams that differ by a few 1e-8: decided as in 64 bits."""
    rng = np.random.default_rng(13)
    x = normal(rng, (4, 2, 30000), "f32", 3.0)
    f = x.double().numpy()
    lse = np.log(np.exp(f).sum(-1))
    top = f.max(-1) - lse
    # scores in fp32 that make the beams' best totals nearly equal; the nearest are some 1e-7 apart
    scores = np.stack((-top[:, 0] - 6, -top[:, 1] - 6), 1).astype(np.float32)
    totals = np.sort(top + scores, 1)
    gap = totals[:, 1] - totals[:, 0]
    assert (gap < 1e-6).all()
    if (gap > 2e-8).all():
        check(x, scores, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [7, 3000, 30001])
@pytest.mark.parametrize("M", [2, 5])
def test_calls_decided_by_the_last_bit_of_a_score(M, V, dtype):
    """Rows with the same logits in other orders, whose sums are equal but for their rounding, and scores 2^-24 apart: the later beams are better."""
    rng = np.random.default_rng(V)
    x = normal(rng, (40, 1, V), dtype, 3.0).expand(40, 3, V).clone()
    for b in range(40):
        for k in range(3):
            x[b, k] = x[b, k, torch.from_numpy(rng.permutation(V))]
    scores = np.full((40, 3), -0.75) + np.arange(3) * 2.0 ** -24
    r = check(x, scores, M)
    assert (r["parent"][:, 0] == 2).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["normal", "ramp", "three lanes", "odd end"])
def test_segments_of_many_steps(dtype, kind):
    """As many rows as give a wavefront eight steps of a row; the beams of a request share one row, so that the definition is quick: their totals
    are sums of a score and a logarithm, and the best are among the best of each."""
    rng = np.random.default_rng(31)
    B, K, M, step = 64, 64, 8, 2048 if dtype == "bf16" else 1024
    V = 16 * step + (77 if kind == "odd end" else 0)
    f = 2.0 * rng.standard_normal((B, V))
    if kind == "ramp":
        f = f * 1e-3 + np.linspace(6, -6, V) * rng.choice([-1, 1], (B, 1))
    if kind == "three lanes":                     # all that is large lies with three lanes, in every step
        lane = np.arange(V) // (8 if dtype == "bf16" else 4) % 64
        f = np.where((lane > 20) & (lane < 24), f + 30, f)
    x = torch.from_numpy(f.astype(np.float32)).to(DT[dtype])
    scores = (-6 * rng.random((B, K))).astype(np.float32)
    r = api.beam_select(x.cuda()[:, None].expand(B, K, V), dev(scores, np.float32), M)
    f = x.double().numpy()
    for b in range(B):
        top = np.argsort(-f[b], kind="stable")[:M]
        lse = f[b].max() + math.log(math.fsum(np.exp(f[b] - f[b].max())))
        totals = scores[b].astype(np.float64)[:, None] + (f[b, top] - lse)
        order = sorted(((-totals[k, i], k, int(top[i])) for k in range(K) for i in range(M)))[:M]
        assert r["parent"][b].tolist() == [k for _, k, _ in order] and r["token"][b].tolist() == [v for _, _, v in order], b
        want = np.array([-t for t, _, _ in order])
        off = np.abs(r["scores"][b].double().cpu().numpy() - want)
        assert (off <= slack(f[b][None, None], np.zeros((1, M), dtype=int))[0] + 2.0 ** -24 * np.abs(want) * (1 + 1e-6)).all()


@pytest.mark.parametrize("M", [3, 16, 64])
def test_logits_that_differ_in_their_last_bits(M):
    """fp32 logits that agree in their upper halves: no bound tells them apart."""
    rng = np.random.default_rng(41)
    x = torch.from_numpy((1 + rng.permuted(np.tile(np.arange(9000), (2, 3, 1)), axis=-1) * 2.0 ** -23).astype(np.float32))
    check(x, -rng.random((2, 3)) * 1e-3, M)


@pytest.mark.parametrize("B,K,V", [(4, 32, 28000), (2, 50, 17000), (1, 64, 9000)])
@pytest.mark.parametrize("alike", [0.0, 1e-3, 6.0])
def test_hundreds_of_candidates_above_the_first_bound(B, K, V, alike):
    """Many lists that are gone into at two places: beams alike, nearly alike and apart."""
    rng = np.random.default_rng(K)
    check(normal(rng, (B, K, V), "bf16", 2.0), -alike * rng.random((B, K)), 64)


@pytest.mark.parametrize("M", [5, 16, 40, 64])
def test_more_candidates_than_a_merge_holds(M):
    """Many lists, a few beams far ahead of the others; all totals alike."""
    rng = np.random.default_rng(51)
    x = normal(rng, (1, 64, 40000), "bf16")
    scores = np.full((1, 64), -50.0) - rng.random((1, 64))
    scores[0, [7, 20, 21]] = -rng.random(3)
    check(x, scores, M)
    check(torch.zeros((1, 64, 4100)), np.zeros((1, 64)), M)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_few_values_whose_totals_nearly_meet(dtype):
    """All terms of such a row are off by the same: scores bring the best totals of two beams to within an fp32 step of each other, either way."""
    rng = np.random.default_rng(61)
    B, V = 64, 20000
    x = torch.zeros((B, 2, V))
    for b in range(B):
        for k in range(2):
            low, n = -float(rng.uniform(1, 11)), int(rng.integers(1, 9))
            x[b, k] = low
            x[b, k, torch.from_numpy(rng.permutation(V)[:n])] = 0
    x = x.to(DT[dtype])
    f = x.double().numpy()
    lse = np.log(np.exp(f).sum(-1))
    scores = np.stack((np.full(B, -0.25), -0.25 + lse[:, 1] - lse[:, 0]), 1).astype(np.float32)
    gap = (scores[:, 0].astype(np.float64) - lse[:, 0]) - (scores[:, 1].astype(np.float64) - lse[:, 1])
    assert (np.abs(gap) < 1e-6).all() and (np.abs(gap) > 2.0 ** -39).all() and (gap > 0).any() and (gap < 0).any()
    check(x, scores, 12)


def test_totals_that_fp32_does_not_hold():
    x = torch.tensor([[[0.0, -1e37, -3e38, 1.0], [5.0, -math.inf, 4.0, -2e37]]])
    check(x, [[-3.4e38, -3.3e38]], 8)
    check(x, [[-3.4028235e38, -3.4028235e38]], 8)


def test_scores_and_flags_in_place():
    """A request's new scores take the place of its own old ones, also where sums are taken again."""
    rng = np.random.default_rng(71)
    x = normal(rng, (300, 1, 3000), "bf16", 3.0).expand(300, 4, 3000).clone()
    x[:, 1] = x[:, 1].flip(-1)
    scores = np.stack((np.full(300, -0.75), np.full(300, -0.75 + 2.0 ** -24), -9 * rng.random(300), -2 - rng.random(300)), 1)
    done = np.zeros((300, 4), dtype=np.uint8)
    done[:, 3] = 1
    s, f = dev(scores, np.float32), dev(done, np.uint8)
    want = api.beam_select(x.cuda(), s.clone(), 4, finished=f.clone(), end_token=7)
    r = api.beam_select(x.cuda(), s, 4, finished=f, end_token=7, out=dict(scores=s, finished=f))
    assert all(torch.equal(r[n], want[n]) for n in want) and r["scores"] is s
    with pytest.raises(api.EtvError):
        api.beam_select(x.cuda(), s, 3, out=dict(scores=s.view(-1)[:900].view(300, 3)))


def test_the_workspace_may_hold_anything():
    rng = np.random.default_rng(14)
    x = normal(rng, (3, 4, 7000), "bf16")
    n = api.beam_select_workspace_bytes(3, 4, 7000, 5, torch.bfloat16)
    for fill in (0, 255):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        check(x, -rng.random((3, 4)), 5, [4, 0, 2], workspace=ws)
    r = api.beam_select(x.cuda()[:0], dev(np.zeros((0, 4)), np.float32), 5)
    assert r["parent"].shape == (0, 5)


def test_rows_further_apart_than_32_bits_reach():
    rng = np.random.default_rng(81)
    x = normal(rng, (2, 4, 5001), "bf16")
    far = torch.empty((1 << 32) + 8 + 3 * ((1 << 30) + 1) + 5001, dtype=torch.bfloat16, device="cuda").as_strided((2, 4, 5001), ((1 << 32) + 8, (1 << 30) + 1, 1))
    far.copy_(x)
    check(x, -rng.random((2, 4)), 6, on=far)


def masked_steps(rng, B, K, V, dtype):
    """Rows in which whole steps of a wavefront hold nothing but a mask's finite value, before others that hold logits of ordinary size; a value and a
    layout for each request."""
    step = 2048 if dtype == "bf16" else 1024
    x, at = normal(rng, (B, K, V), dtype), np.arange(V) // step
    lows = [torch.finfo(DT[dtype]).min, -1e30, -1e12, -1e10, -3e9, -4e6, -1e4]
    climb = [-3e38, -1e30, -1e20, -1e10, -3e9, -2e9, -1e7, -2e6, -1.1e6, -1048579, -1048573, -1e6, -5e5, -900, -30, 0]
    for b in range(B):
        low, layout = lows[b % 7], b // 7 % 7
        for k in range(K):
            if layout == 0:                                           # some steps
                mask = (rng.random(at[-1] + 1) < 0.5)[at]
            elif layout == 1:                                         # all but the last logits
                mask = np.arange(V) < V - 100
            elif layout == 2:                                         # all but a few tokens that a grammar allows
                mask = np.ones(V, dtype=bool)
                mask[rng.integers(0, V, 12)] = False
            elif layout == 3:                                         # the first half
                mask = np.arange(V) < V // 2 + k
            elif layout == 4:                                         # all of a row, and steps that are masked in two ways
                mask = np.ones(V, dtype=bool) if k == 0 else at % 4 < 3
                x[b, k, torch.from_numpy(at % 4 == 1)] = -math.inf
            elif layout == 5:                                         # both masks side by side
                mask = (rng.random(at[-1] + 1) < 0.7)[at]
                x[b, k, torch.from_numpy(mask & (rng.random(V) < 0.5))] = -math.inf
            else:                                                     # every step's logits above those of the step before
                base = np.array(climb)[np.sort(rng.integers(0, len(climb), at[-1] + 1))]
                x[b, k] = (x[b, k].double() + torch.from_numpy(base)[at]).to(DT[dtype])
                continue
            x[b, k, torch.from_numpy(mask) & (x[b, k] > -math.inf)] = low
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [5, 20])
def test_steps_of_masked_logits_before_others(M, dtype):
    """72 requests of 4 beams: a wavefront's segment is three to eight steps of a row."""
    rng = np.random.default_rng(91)
    x = masked_steps(rng, 72, 4, 32000, dtype)
    check(x, -rng.random((72, 4)), M)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_masked_step_with_what_is_not_a_number(dtype):
    """The sum so far is of no weight behind a masked step, but for the news of a logit that is not finite."""
    rng = np.random.default_rng(92)
    B, K, V = 72, 4, 32000
    x = normal(rng, (B, K, V), dtype)
    x[:8, :, :16384] = torch.finfo(DT[dtype]).min
    x[4:8, :, 5:9000:2] = -math.inf
    for b, what in enumerate((math.nan, math.inf, -math.nan, math.nan) * 2):
        x[b, b % 3, int(rng.integers(0, 16384))] = what
    n = [K] * 8 + [0] * (B - 8)
    r = check(x, -rng.random((B, K)), 5, n)
    assert r["status"].tolist() == [1] * 8 + [4] * (B - 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("copies", [False, True])
@pytest.mark.parametrize("K", [3, 6])
@pytest.mark.parametrize("M", [4, 6, 12, 40])
def test_equal_beams_whose_best_tokens_lie_close(M, K, copies, dtype):
    """One row for all beams, or the same row at several places, and two best logits a step of their type apart: (0, A) (1, A) .. (0, B) (1, B) .."""
    rng = np.random.default_rng(101)
    for V in (600, 9001):
        x = torch.from_numpy(rng.uniform(-8, -1, (4, 1, V)).astype(np.float32)).to(DT[dtype])
        a, b = (2.0 ** -13 + 2.0 ** -20, 2.0 ** -13) if dtype == "bf16" else (5.0 + 2.0 ** -21, 5.0)
        for i in range(4):
            at = rng.permutation(V)[:2]
            x[i, 0, int(at[0])], x[i, 0, int(at[1])] = a, b
        x = x.expand(4, K, V)
        check(x, np.full((4, K), -1.25), M, on=(x.contiguous().cuda() if copies else x[:, :1].cuda().expand(4, K, V)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("third", [0, 1, 2])
@pytest.mark.parametrize("M", [1, 2, 3, 8, 30])
def test_equal_beams_and_one_close_by(M, third, dtype):
    """Two beams alike, and another row whose best total is an fp32 step above or below theirs."""
    rng = np.random.default_rng(102)
    B, V = 32, 5001
    x = normal(rng, (B, 2, V), dtype, 3.0)
    f = x.double().numpy()
    best = f.max(-1) - np.array([[f[b, k].max() + math.log(math.fsum(np.exp(f[b, k] - f[b, k].max()))) for k in range(2)] for b in range(B)])
    alike, other = np.full(B, -6.0, dtype=np.float32), (-6.0 + best[:, 0] - best[:, 1]).astype(np.float32)
    gap = other + best[:, 1] - (alike + best[:, 0])
    assert (np.abs(gap) < 1e-6).all() and (np.abs(gap) > 2.0 ** -39).all() and (gap > 0).any() and (gap < 0).any()
    order = [0, 0]
    order.insert(third, 1)
    check(x[:, order].contiguous(), np.stack((alike, other), 1)[:, order], M)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("third", [0, 1, 2])
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("M", [1, 2, 3, 20])
def test_equal_beams_and_one_closer_than_the_second_sum_tells(M, sign, third, dtype):
    """Two beams alike, and one with the same logits in another order whose score is 2^-28 off."""
    rng = np.random.default_rng(103)
    B, V = 32, 5001
    x = normal(rng, (B, 1, V), dtype, 3.0).expand(B, 3, V).clone()
    for b in range(B):
        x[b, third] = x[b, third, torch.from_numpy(rng.permutation(V))]
    scores = np.full((B, 3), np.float32(-0.05))
    scores[:, third] += sign * 2.0 ** -28
    assert (scores == scores.astype(np.float32)).all()
    check(x, scores, M)


@pytest.mark.parametrize("V", [2, 5000])
@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("M", [1, 2, 4, 20])
def test_sums_that_fp32_does_not_tell_apart(M, far, V):
    """Rows of two tokens a thread adds up, [0, -a] and [0, -a'] with a' an fp32 step behind a, or both so far that 1 + exp(-a) is 1: the totals differ in
    64 bits alone, the better beam first or second."""
    rng = np.random.default_rng(104)
    B = 64
    x = torch.full((B, 2, V), -math.inf)
    a = (rng.uniform(17.5, 22, B) if far else rng.uniform(1, 10, B)).astype(np.float32)
    behind = a + np.float32(0.5) if far else np.nextafter(a, np.float32(99))
    for b in range(B):
        at = 2 * int(rng.integers(0, V // 2))
        x[b, :, at] = 0
        x[b, b % 2, at + 1], x[b, 1 - b % 2, at + 1] = float(-a[b]), float(-behind[b])
    gap = np.log1p(np.exp(-a.astype(np.float64))) - np.log1p(np.exp(-behind.astype(np.float64)))
    assert (gap > 2.0 ** -39).all()
    r = check(x, np.full((B, 2), -0.5), M)
    assert (r["parent"][:, 0].cpu() == 1 - torch.arange(B) % 2).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_totals_of_finished_and_running_beams(dtype):
    """A finished beam's score against a running beam's best total: a row of one token has a probability of 1 whatever its logit is."""
    rng = np.random.default_rng(105)
    x = torch.full((40, 4, 3001), -math.inf, dtype=DT[dtype])
    for b in range(40):
        for k in range(4):
            x[b, k, int(rng.integers(3001))] = float(rng.normal())
    done = (rng.random((40, 4)) < 0.5).astype(np.uint8)
    for M in (2, 4):
        check(x, np.full((40, 4), -0.75), M, None, done, 17)


def test_one_workspace_for_every_batch():
    """Sized for the largest batch; the smaller ones leave what is behind it alone, and so does the largest."""
    rng = np.random.default_rng(107)
    x = normal(rng, (80, 4, 32000), "bf16")
    n = api.beam_select_workspace_bytes(80, 4, 32000, 4, torch.bfloat16)
    whole = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda")
    for B in (80, 72, 71, 64, 1):
        check(x[:B], -rng.random((B, 4)), 4, workspace=whole[:n])
        assert bool((whole[n:] == 77).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,M", [(2, 2), (2, 8), (5, 5), (5, 20)])
def test_close_calls_between_rows_of_any_kind(K, M, dtype):
    """Scores that bring the best totals of all beams to within an fp32 step of each other: whatever lies between them, the order is that of 64 bits."""
    rng = np.random.default_rng(106)
    B, V = 24, 20000
    x = normal(rng, (B, K, V), dtype, 3.0)
    f = x.double().numpy()
    top = np.array([[-math.log(math.fsum(np.exp(f[b, k] - f[b, k].max()))) for k in range(K)] for b in range(B)])
    scores = (-6 - top).astype(np.float32)
    totals = np.sort(top + scores, 1)
    assert (totals[:, -1] - totals[:, 0] < 1e-6).all() and (np.diff(totals) > 2.0 ** -39).all()
    check(x, scores, M)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [3, 5, 8, 9, 601, 4099, 8193, 16384, 16385, 16391, 33000])
def test_rows_that_differ_in_one_logit(V, dtype):
    """Copies of a row, and rows like it but for one place, where a logit is -18.5 instead of -18: better by 6e-9, wherever that place is."""
    rng = np.random.default_rng(V)
    for at in {0, 1, V - 1, V // 3}:
        x = torch.full((4, 4, V), -math.inf, dtype=DT[dtype])
        for b in range(4):
            top = int(rng.choice([v for v in (0, 1, 2, V - 2) if v != at]))
            x[b, :, top], x[b, :, at] = 0, -18
            x[b, torch.from_numpy(rng.random(4) < 0.5), at] = -18.5
        for M in (1, 4, 8):
            check(x, np.full((4, 4), -0.5), M)
