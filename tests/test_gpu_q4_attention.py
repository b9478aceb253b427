"""tree_verify_attention_q4 on the GPU against float64, at the sizes and masks where it can go wrong."""
import numpy as np
import pytest
import torch

from paper_2603_08088_amd import api
from q4_plain import Case

pytestmark = pytest.mark.gpu

# B, T, Hq, Hkv, d, dtype, prefix lengths, block size, node counts
SHAPES = [
    (1, 1, 4, 4, 64, "bf16", [0], 0, [1]),                   # a single token without a prefix sees itself
    (1, 1, 8, 2, 128, "bf16", [1], 0, [1]),
    (2, 1, 32, 8, 128, "bf16", [130, 64], 16, [1, 1]),
    (3, 1, 7, 1, 64, "bf16", [63, 65, 1000], 32, [1, 1, 0]),  # seven heads share one; a sequence without nodes
    (2, 5, 28, 4, 128, "bf16", [17, 300], 48, [5, 2]),
    (1, 33, 4, 2, 64, "bf16", [127], 16, [33]),
    (2, 8, 32, 8, 128, "bf16", [515, 31], 16, [8, 7]),
    (2, 16, 8, 2, 128, "bf16", [200, 0], 64, [16, 15]),
    (2, 60, 8, 2, 128, "bf16", [333, 96], 16, [60, 41]),
    (1, 129, 4, 1, 128, "bf16", [70], 0, [129]),
    (2, 256, 4, 4, 64, "bf16", [65, 128], 16, [256, 200]),
    (1, 256, 8, 1, 128, "bf16", [40], 256, [255]),
    (1, 65, 2, 2, 128, "bf16", [1029], 16, [65]),
    (1, 1, 4, 2, 128, "f32", [33], 16, [1]),
    (2, 3, 28, 4, 64, "f32", [0, 129], 16, [3, 3]),
    (2, 33, 8, 2, 128, "f32", [100, 257], 48, [29, 33]),
    (1, 130, 4, 2, 64, "f32", [500], 0, [130]),
    (1, 256, 2, 1, 128, "f32", [77], 64, [250]),
]


@pytest.mark.parametrize("kv_split", [0, 64, 192])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:6])))
def test_against_float64(shape, kv_split):
    B, T, Hq, Hkv, d, dtype, Ps, block, ns = shape
    c = Case(T + d, B, T, Hq, Hkv, d, dtype, Ps, block, ns)
    c.check(*c.run(kv_split=kv_split))


@pytest.mark.parametrize("shape", SHAPES[2::3], ids=lambda s: "-".join(map(str, s[:6])))
def test_generic_kernel_against_float64(shape):
    B, T, Hq, Hkv, d, dtype, Ps, block, ns = shape
    c = Case(T + d, B, T, Hq, Hkv, d, dtype, Ps, block, ns)
    c.check(*c.run(flags=api.ATTN_FLAG_GENERIC))


@pytest.mark.parametrize("splits", [2, 9, 16, 17, 31, 33, 64, 65, 130])
@pytest.mark.parametrize("T,Hq,Hkv,d,dtype", [(1, 8, 2, 128, "bf16"), (17, 2, 1, 64, "bf16"), (40, 4, 2, 128, "f32"), (80, 32, 16, 64, "bf16")])
def test_every_number_of_splits_is_joined(T, Hq, Hkv, d, dtype, splits):
    """Fewer and more partials than the lanes of a row take at once, few and many rows, lengths that leave the last split short."""
    step = 512                                       # of the largest round of a workgroup
    Ps = [splits * step - 37, splits * step // 3]
    c = Case(splits, 2, T, Hq, Hkv, d, dtype, [1, 1], 0)
    c.Ps, c.P_max, c.size = Ps, max(Ps), max(Ps)
    rng, shape = c.rng, (2, Hkv, max(Ps))
    c.codes = [rng.integers(0, 256, shape + (d // 2,)).astype(np.uint8) for _ in range(2)]
    c.scales = [rng.integers(122, 127, shape + (d // 32,)).astype(np.uint8) for _ in range(2)]
    want, want_lse = c.run(flags=api.ATTN_FLAG_GENERIC)
    got, lse = c.run(kv_split=step)
    # two roundings to the type in either, weights and result, and 2^-13 for scores and sums in another order
    tol = (4 * torch.finfo(c.dtype).eps / 2 + 2.0 ** -13) * want.float().abs().max().item()
    assert (got.float() - want.float()).abs().max().item() <= tol and (lse - want_lse).abs().max().item() <= 2.0 ** -13


@pytest.mark.parametrize("B,T,Hq,Hkv,d,kv_split", [(70, 3, 8, 2, 128, 0), (66, 1, 4, 4, 64, 128), (33, 40, 8, 2, 128, 256), (5, 90, 8, 1, 128, 0)])
def test_large_batches_of_ragged_sequences(B, T, Hq, Hkv, d, kv_split):
    """More sequences than a wavefront has lanes, sequences without a prefix and without nodes; against the generic kernel."""
    rng = np.random.default_rng(B)
    Ps, ns = [int(x) for x in rng.integers(0, 900, B)], [int(x) for x in rng.integers(0, T + 1, B)]
    Ps[1], Ps[2], ns[3], ns[0], Ps[0] = 0, 899, 0, T, 700
    c = Case(B, B, T, Hq, Hkv, d, "bf16", Ps, 16, ns)
    want, want_lse = c.run(flags=api.ATTN_FLAG_GENERIC)
    got, lse = c.run(kv_split=kv_split)
    assert (got.float() - want.float()).abs().max().item() <= (4 * 2.0 ** -8 + 2.0 ** -13) * want.float().abs().max().item()
    assert torch.equal(torch.isinf(lse), torch.isinf(want_lse)) and torch.nan_to_num(lse - want_lse).abs().max().item() <= 2.0 ** -13


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,Hq,P", [(2, 8, 60), (20, 8, 300), (50, 8, 200)])
def test_lse_keeps_fp32(dtype, T, Hq, P):
    """The sum is over unrounded weights, of scores that are right to 2^-18 of q's maximum."""
    c = Case(15, 1, T, Hq, 2, 128, dtype, [P], 16, [T])
    _, lse = c.run()
    want = c.plain()[1]
    assert np.abs(lse.double().cpu().numpy() - want).max() <= c.score_slack() + 2.0 ** -20


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1.0, -0.09, 2.0])
def test_scales_of_either_sign_and_peaked_rows(dtype, scale):
    c = Case(7, 2, 6, 8, 2, 128, dtype, [150, 40], 16, [6, 6])
    c.check(*c.run(scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_queries_of_mixed_magnitude(dtype, d):
    """Channels of a group that differ by powers of two in both directions, and whole groups that are zero."""
    c = Case(8, 1, 9, 8, 2, d, dtype, [90], 16, [9])
    f = np.exp2(c.rng.integers(-12, 3, c.q.shape)).astype(np.float32)
    f[0, 3] = 0
    c.q = (c.q * torch.from_numpy(f)).to(c.dtype)
    c.check(*c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,Hq,Hkv,d", [(5, 8, 2, 128), (70, 4, 2, 64), (130, 4, 2, 128)])
def test_rows_that_see_nothing_and_what_lies_behind_masks(dtype, T, Hq, Hkv, d):
    """Masks of any form; infinities, NaN and the largest values in tree rows that some rows see and others do not."""
    c = Case(9, 2, T, Hq, Hkv, d, dtype, [0, 37], 16, [T, T - 1])
    c.vis = c.rng.random((2, T, T)) < 0.4
    c.vis[:, 1] = False                              # sees no node: nothing at all in the first sequence
    c.vis[0, 2, :] = False
    c.vis[:, :, 3:5] = False
    c.vis[0, 2, 3] = True                            # sees only a NaN
    c.vis[1, T - 2, 4] = True                        # sees an infinity among others
    c.vt[0, 3, 0, 5], c.kt[0, 3, 1, 7] = float("nan"), float("nan")
    c.vt[1, 3, 1, 0], c.kt[1, 3, 0, 1] = float("inf"), float("-inf")
    c.vt[1, 4, 0, 33], c.vt[1, 4, 1, 2] = float("inf"), float("-inf")
    c.kt[1, 3, 1] = torch.finfo(c.dtype).max
    for b in range(2):                               # rows behind the last node
        c.kt[b, c.ns[b]:], c.vt[b, c.ns[b]:] = float("nan"), float("inf")
    out, lse = c.run()
    want, want_lse, _ = c.plain()
    got = out.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
    assert (got[0, 1] == 0).all() and np.isneginf(lse[0, :, 1].cpu().numpy()).all()
    fine = np.isfinite(want)
    assert np.abs(got[fine] - want[fine]).max() <= 2.0 ** -5     # values of a few units, rounded to 8 bits twice
    g = lse.double().cpu().numpy()
    assert np.array_equal(np.isnan(g), np.isnan(want_lse)) and np.array_equal(np.isneginf(g), np.isneginf(want_lse))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,Hq,P", [(6, 4, 0), (6, 4, 70), (40, 8, 200)])
def test_infinite_scores(dtype, T, Hq, P):
    """A tree key with an infinity: nothing where its score is -inf, NaN rows where it is +inf; a query with one: NaN."""
    c = Case(16, 1, T, Hq, 2, 64, dtype, [P], 16, [T])
    c.vis = np.tril(np.ones((1, T, T), bool))
    c.kt[0, 2, 0, 9] = float("inf")
    c.q[0, 4, Hq - 1, 3] = float("-inf")
    out, lse = c.run()
    want, want_lse, _ = c.plain()
    got, nan = out.double().cpu().numpy(), np.isnan(want)
    assert nan.any() and not nan.all() and np.array_equal(np.isnan(got), nan)
    assert np.abs(got - want)[~nan].max() <= 2.0 ** -5 and np.array_equal(np.isnan(lse.cpu().numpy()), np.isnan(want_lse))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_groups_of_the_prefix_show(dtype):
    c = Case(10, 1, 4, 4, 2, 128, dtype, [70], 16, [4])
    page, off = c.table[0][66 // 16], 66 % 16
    c.scales[1][page, 0, off, 2] = 255               # V of one key, one group: that group of that head's outputs
    out, _ = c.run()
    bad = torch.isnan(out).cpu().numpy()
    want = np.zeros_like(bad)
    want[:, :, :2, 64:96] = True
    assert np.array_equal(bad, want)
    c.scales[0][page, 1, off, 0] = 255               # K: whole rows of the other head
    bad = torch.isnan(c.run()[0]).cpu().numpy()
    want[:, :, 2:] = True
    assert np.array_equal(bad, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 100])
def test_blocks_outside_the_pool_read_as_nan(dtype, T):
    """One sequence of a batch names blocks that do not exist: its rows are NaN, the others keep their results."""
    c = Case(12, 3, T, 8, 2, 128, dtype, [200, 100, 150], 16, [T] * 3)
    want, _ = c.run()
    table = c.tables()
    table[1, 2], table[1, 4] = 2 ** 30, -7
    table[2, 12] = -1                                # behind the sequence's prefix: nobody looks
    got, _ = c.run(block_table=table)
    assert torch.isnan(got[1]).all() and torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])


def test_prefix_lengths_are_held_within_the_bound():
    c = Case(13, 2, 3, 4, 2, 64, "bf16", [50, 20], 16, [3, 3])
    out, _ = c.run(P_max=32)
    c.Ps[0], c.P_max = 32, 32
    c.check(out, None)
    c.Ps[1] = 0
    c.check(api.tree_verify_attention_q4(c.q.cuda(), c.cache(), c.ints([32, -4]), c.kt.cuda(), c.vt.cuda(), torch.from_numpy(c.words()).cuda(),
                                         c.ints([3, 9]), P_max=32, block_table=c.tables())[0], None)


@pytest.mark.parametrize("dtype,T", [("bf16", 1), ("bf16", 64), ("f32", 7)])
def test_same_bits_on_every_run_on_another_stream_and_in_a_graph(dtype, T):
    c = Case(14, 2, T, 8, 2, 128, dtype, [700, 260], 16, [T, T])
    cache, P, n, bt, mask = c.cache(), c.ints(c.Ps), c.ints(c.ns), c.tables(), torch.from_numpy(c.words()).cuda()
    q, kt, vt = c.q.cuda(), c.kt.cuda(), c.vt.cuda()
    dsc = api.attn_q4_desc(q, cache, kt, bt, c.P_max)
    ws = [torch.empty(max(256, api.tree_verify_attention_q4_workspace_bytes(dsc)), dtype=torch.uint8, device="cuda") for _ in range(2)]
    out, lse = torch.empty_like(q), torch.empty((2, 8, T), device="cuda")

    def call(w, o=None, l=None):
        return api.tree_verify_attention_q4(q, cache, P, kt, vt, mask, n, P_max=c.P_max, block_table=bt, out=o, lse=l, workspace=w, desc=dsc)
    want = call(ws[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = call(ws[1], out, lse)
    again = call(ws[0])                              # at the same time, in a workspace of its own
    torch.cuda.synchronize()
    for x in (other, again):
        assert torch.equal(x[0], want[0]) and torch.equal(x[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(ws[1], out, lse)
    for rep in range(4):
        q.copy_(torch.randn(q.shape, device="cuda"))
        P.copy_(c.ints([700 - 100 * rep, rep]))
        out.fill_(7)
        graph.replay()
        want = call(ws[0])
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), rep


def test_a_decoding_loop_over_a_4bit_cache():
    """As it is used: a prompt is written, then steps of draft trees (tree tensors, attention of both layers, acceptance, commit
    into the 4-bit cache) and single tokens; after each the cache holds what the same calls leave in plain arrays."""
    from paper_2603_08088_amd import synth
    import q4_plain
    rng = np.random.default_rng(21)
    Lyr, B, T, Hq, Hkv, d, W, V, block = 2, 2, 12, 8, 2, 128, 5, 50, 16
    dt, pages, S = torch.bfloat16, 24, 37
    cache = api.KVCacheQ4(*(torch.zeros((Lyr, pages, Hkv, block, d // n), dtype=torch.uint8, device="cuda") for n in (2, 32, 2, 32)))
    host = [t.cpu().numpy() for t in cache]
    table = rng.permutation(pages)[:2 * 10].reshape(2, 10).astype(np.int32)
    bt, cap = torch.from_numpy(table).cuda(), torch.tensor([160, 160], dtype=torch.int32, device="cuda")
    i32 = lambda xs: torch.tensor(xs, dtype=torch.int32, device="cuda")

    def note(rows_k, rows_v, b, P):                  # [Lyr, n, Hkv, d] into the plain arrays
        for x, rows in enumerate((rows_k, rows_v)):
            c, s = q4_plain.quantise(rows.double().cpu().numpy())
            for i in range(rows.shape[1]):
                page, off = q4_plain.place(table, block, b, P + i)
                host[2 * x][:, page, :, off], host[2 * x + 1][:, page, :, off] = c[:, i], s[:, i]
    k, v = (torch.randn((Lyr, B, S, Hkv, d), device="cuda").to(dt) for _ in range(2))
    ns = [37, 20]
    r = api.quantize_kv_q4(k, v, cache, i32([0, 0]), i32(ns), cap, block_table=bt)
    P, lens = r["prefix_len_out"], [37, 20]
    for b in range(B):
        note(k[:, b, :ns[b]], v[:, b, :ns[b]], b, 0)
    for step in range(4):
        n = T if step != 2 else 1                    # the third step has no draft: a single token
        parents = [synth.tree_bfs(rng, n, 4, 3) if n > 1 else np.zeros(1, np.int32) for _ in range(B)]
        parent = torch.from_numpy(np.stack(parents).astype(np.int32)).cuda()
        m = api.tensorize_tree(parent, i32([n, n]), P, n, W)
        kt, vt = (torch.randn((Lyr, B, n, Hkv, d), device="cuda").to(dt) for _ in range(2))
        q = torch.randn((Lyr, B, n, Hq, d), device="cuda").to(dt)
        for layer in range(Lyr):
            out, lse = api.tree_verify_attention_q4(q[layer], cache.layer(layer), P, kt[layer], vt[layer], m["bitmask"], i32([n, n]),
                                                    P_max=160, block_table=bt)
            c = Case(0, B, n, Hq, Hkv, d, "bf16", lens, block)
            c.table, c.codes, c.scales = table, [host[0][layer], host[2][layer]], [host[1][layer], host[3][layer]]
            c.q, c.kt, c.vt, c.vis = q[layer].cpu(), kt[layer].cpu(), vt[layer].cpu(), m["dense"][:, 0].bool().cpu().numpy()
            c.check(out, lse)
        tokens = torch.randint(0, 3, (B, n), dtype=torch.int32, device="cuda")
        logits = torch.randn((B, n, V), device="cuda")
        logits[:, :, :3] += 6
        post = api.evaluate_posterior(logits, tokens, m["retrieve"], i32([n, n]))
        r = api.commit_accepted_kv_q4(kt, vt, cache, P, cap, i32([n, n]), post["acc_nodes"], post["accept_len"], block_table=bt)
        assert r["status"].tolist() == [0, 0]
        for b in range(B):
            nodes = post["acc_nodes"][b, :int(post["accept_len"][b]) + 1].long()
            note(kt[:, b, nodes], vt[:, b, nodes], b, lens[b])
            lens[b] += len(nodes)
        P = r["prefix_len_out"]
        assert P.tolist() == lens
        for t, a in zip(cache, host):
            assert np.array_equal(t.cpu().numpy(), a)
