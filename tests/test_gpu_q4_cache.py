"""The 4-bit prefix cache on the GPU: rows written by quantize_kv_q4 and commit_accepted_kv_q4, byte for byte, and read back."""
import numpy as np
import pytest
import torch

import q4_plain
from paper_2603_08088_amd import api

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def i32(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def empty_cache(rng, layers, B, Hkv, d, block, room):
    """A cache of random bytes, its table (None: contiguous) and host copies of its four tensors."""
    width = -(-room // block) if block else 0
    pages, size = (B * width + 2, block) if block else (B, room)
    table = rng.permutation(pages)[:B * width].reshape(B, width).astype(np.int32) if block else None
    host = [rng.integers(0, 256, (layers, pages, Hkv, size, d // n)).astype(np.uint8) for n in (2, 32, 2, 32)]
    return api.KVCacheQ4(*(torch.from_numpy(a).cuda() for a in host)), table, host, size


def written(host, table, size, x, layer, b, pos, row):
    """Row [Hkv, d] of K (x = 0) or V (1) into the host copy."""
    page, off = q4_plain.place(table, size, b, pos)
    c, s = q4_plain.quantise(row)
    host[2 * x][layer, page, :, off], host[2 * x + 1][layer, page, :, off] = c, s


def same(cache, host):
    for t, a in zip(cache, host):
        assert np.array_equal(t.cpu().numpy(), a)


def dev(table):
    return None if table is None else torch.from_numpy(table).cuda()


WRITES = [  # layers, B, rows, Hkv, d, dtype, block, prefix lengths, rows of each sequence
    (1, 1, 1, 1, 64, "bf16", 0, [0], [1]),
    (3, 2, 1, 8, 128, "bf16", 16, [15, 16], [1, 1]),
    (2, 3, 40, 2, 128, "bf16", 16, [0, 7, 33], [40, 0, 17]),
    (1, 2, 70, 3, 64, "bf16", 48, [47, 1], [70, 3]),
    (2, 2, 33, 4, 64, "f32", 0, [5, 0], [33, 32]),
    (1, 3, 129, 1, 128, "f32", 32, [31, 64, 1], [129, 128, 1]),
    (1, 1, 1000, 2, 128, "bf16", 256, [513], [999]),
]


@pytest.mark.parametrize("layers,B,rows,Hkv,d,dtype,block,Ps,ns", WRITES)
def test_rows_are_written_as_defined_and_nothing_else_is(layers, B, rows, Hkv, d, dtype, block, Ps, ns):
    rng = np.random.default_rng(rows)
    room = max(Ps) + rows + 3
    cache, table, host, size = empty_cache(rng, layers, B, Hkv, d, block, room)
    k, v = (torch.from_numpy((rng.standard_normal((layers, B, rows, Hkv, d)) * np.exp(3 * rng.standard_normal((layers, B, rows, Hkv, 1))))
                             .astype(np.float32)).to(DT[dtype]) for _ in range(2))
    r = api.quantize_kv_q4(k.cuda(), v.cuda(), cache, i32(Ps), i32(ns), i32([room] * B), block_table=dev(table))
    assert r["status"].tolist() == [0] * B and r["prefix_len_out"].tolist() == [P + n for P, n in zip(Ps, ns)]
    for layer in range(layers):
        for b in range(B):
            for i in range(ns[b]):
                for x, t in enumerate((k, v)):
                    written(host, table, size, x, layer, b, Ps[b] + i, t[layer, b, i].double().numpy())
    same(cache, host)
    # and back, in both types: what the cache holds is exact in either
    for out in ("bf16", "f32"):
        r = api.dequantize_kv_q4(cache, i32(Ps), i32(ns), rows, block_table=dev(table), dtype=DT[out])
        assert r["status"].tolist() == [0] * B
        for layer in range(layers):
            for b in range(B):
                for x, got in enumerate((r["k"], r["v"])):
                    want = np.zeros((rows, Hkv, d))
                    for i in range(ns[b]):
                        page, off = q4_plain.place(table, size, b, Ps[b] + i)
                        want[i] = q4_plain.values(host[2 * x][layer, page, :, off], host[2 * x + 1][layer, page, :, off])
                    assert np.array_equal(got[layer, b].double().cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_values_at_every_border_of_the_format(dtype, d):
    """Ties, the step from one scale to the next, zeros of both signs, the smallest and largest magnitudes, infinities and NaN."""
    rng = np.random.default_rng(5)
    t = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 0, -0.0, 0.2490234375, 0.2509765625, 6.96875, 7.0, 7.9375, 4, 3.984375])
    rows = []
    for e in (-149, -140, -133, -130, -126, -125, -124, -123, -20, 0, 1, 60, 120, 123, 124, 125):
        for top in (4.0, 6.0, 6.96875, 7.0, 7.5, 7.96875):
            g = np.concatenate(([top], rng.choice(t[np.abs(t) <= top], 31)))
            rows.append(rng.permutation(g * rng.choice([-1.0, 1.0], 32)) * 2.0 ** e)
    for bad in (np.inf, -np.inf, np.nan):
        g = rng.standard_normal(32)
        g[rng.integers(32)] = bad
        rows.append(g)
    rows += [np.zeros(32), -np.zeros(32), np.full(32, -3.3e38), np.full(32, 2.0 ** -149)]
    with np.errstate(over="ignore"):
        x = torch.from_numpy(np.stack(rows).astype(np.float32)).to(DT[dtype])
    x = x[torch.arange(-(-len(rows) * 32 // d) * d // 32) % len(rows)].reshape(1, 1, -1, 1, d)
    n = x.shape[2]
    cache = api.KVCacheQ4.empty(1, 1, 1, n, d)
    r = api.quantize_kv_q4(x.cuda(), x.flip(2).cuda(), cache, i32([0]), i32([n]), i32([n]))
    assert r["status"].tolist() == [0]
    c, s = q4_plain.quantise(x[0, 0, :, 0].double().numpy())
    for got, want in zip(cache, (c, s, c[::-1], s[::-1])):
        assert np.array_equal(got[0, 0, 0].cpu().numpy(), want)
    back = api.dequantize_kv_q4(cache, i32([0]), i32([n]), n, dtype=DT[dtype])["k"][0, 0, :, 0].double().cpu().numpy()
    assert np.array_equal(back, q4_plain.values(c, s), equal_nan=True)


@pytest.mark.parametrize("layers,B,T,W,Hkv,d,dtype,block", [(1, 1, 1, 1, 1, 64, "bf16", 0), (4, 3, 60, 7, 8, 128, "bf16", 16),
                                                           (2, 2, 256, 40, 2, 64, "f32", 48), (3, 5, 33, 12, 4, 128, "f32", 0)])
def test_commit_matches_the_unquantised_commit_and_the_format(layers, B, T, W, Hkv, d, dtype, block):
    """Lengths, slots and status are commit_accepted_kv's on the same arguments; the rows are the tree's, quantised."""
    rng = np.random.default_rng(T + W)
    Ps = [int(x) for x in rng.integers(0, 70, B)]
    room = max(Ps) + W + 1
    cache, table, host, size = empty_cache(rng, layers, B, Hkv, d, block, room)
    kt, vt = (torch.from_numpy(rng.standard_normal((layers, B, T, Hkv, d)).astype(np.float32)).to(DT[dtype]) for _ in range(2))
    acc, A = rng.integers(0, T, (B, W)).astype(np.int32), [int(x) for x in rng.integers(0, W, B)]
    ns, cap = [T] * B, [room] * B
    if B > 2:
        acc[1, 0], A[1] = T, max(A[1], 1)     # not a node
        cap[2] = Ps[2] + A[2]                 # one row short
    args = (i32(Ps), i32(cap), i32(ns), torch.from_numpy(acc).cuda(), i32(A))
    r = api.commit_accepted_kv_q4(kt.cuda(), vt.cuda(), cache, *args, block_table=dev(table))
    shape = (layers, len(host[0][0]), Hkv, size, d) if block else (layers, B, size, Hkv, d)
    kc, vc = (torch.zeros(shape, dtype=DT[dtype], device="cuda") for _ in range(2))
    want = api.commit_accepted_kv(kt.cuda(), vt.cuda(), kc, vc, *args, block_table=dev(table))
    for key in ("prefix_len_out", "slot_map", "status"):
        assert torch.equal(r[key], want[key]), key
    for layer in range(layers):
        for b in range(B):
            for i in range(A[b] + 1 if not r["status"][b] else 0):
                for x, t in enumerate((kt, vt)):
                    written(host, table, size, x, layer, b, Ps[b] + i, t[layer, b, acc[b, i]].double().numpy())
    same(cache, host)


def test_sequences_that_fail_a_check_are_left_alone():
    rng = np.random.default_rng(11)
    layers, B, rows, Hkv, d, block = 2, 8, 20, 2, 64, 16
    cache, table, host, size = empty_cache(rng, layers, B, Hkv, d, block, 64)      # 4 blocks each
    pool = host[0].shape[1]
    table[2, 1], table[3, 0] = pool, -1
    Ps, ns, cap = [50, 3, 10, 1, -1, 5, 5, 2 ** 31 - 1], [14, 21, 8, 2, 1, -1, 20, 20], [63, 64, 64, 64, 64, 64, 64, 2 ** 31 - 1]
    want = [api.COMMIT_CAPACITY, api.COMMIT_BAD_LEN, api.COMMIT_BAD_BLOCK, api.COMMIT_BAD_BLOCK, api.COMMIT_CAPACITY, api.COMMIT_BAD_LEN, 0,
            api.COMMIT_CAPACITY]
    k = torch.randn((layers, B, rows, Hkv, d), device="cuda")
    r = api.quantize_kv_q4(k, -k, cache, i32(Ps), i32(ns), i32(cap), block_table=dev(table))
    assert r["status"].tolist() == want and r["prefix_len_out"].tolist() == Ps[:6] + [25] + Ps[7:]
    for layer in range(layers):
        for i in range(20):
            for x, t in enumerate((k, -k)):
                written(host, table, size, x, layer, 6, 5 + i, t[layer, 6, i].double().cpu().numpy())
    same(cache, host)
    # reading: beyond the table, a negative start or count, a bad block; zeros throughout, also where n is short
    out = dict(k=torch.full((layers, B, rows, Hkv, d), 7.0, device="cuda"), v=torch.full((layers, B, rows, Hkv, d), 7.0, device="cuda"))
    first, ns = [50, -3, 10, 1, 3, 5, 5, 2 ** 31 - 1], [15, 2, 8, 2, 21, -1, 20, 20]
    r = api.dequantize_kv_q4(cache, i32(first), i32(ns), rows, block_table=dev(table), out=out)
    assert r["status"].tolist() == [1, 4, 8, 8, 4, 4, 0, 1]
    assert not out["k"][:, [0, 1, 2, 3, 4, 5, 7]].any() and not out["v"][:, [0, 1, 2, 3, 4, 5, 7]].any()
    page, off = table[6, 1], 3
    assert np.array_equal(out["v"][1, 6, 14].double().cpu().numpy(), q4_plain.values(host[2][1, page, :, off], host[3][1, page, :, off]))


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB of codes: the last block is written, read and attended."""
    Hkv, d, block = 8, 128, 256
    blocks = (4 << 30) // (Hkv * block * d // 2) + 3
    cache = api.KVCacheQ4(*(torch.zeros((1, blocks, Hkv, block, d // n), dtype=torch.uint8, device="cuda") for n in (2, 32, 2, 32)))
    table = i32([[blocks - 1, 1]])
    k = torch.randn((1, 1, 300, Hkv, d), device="cuda", dtype=torch.bfloat16)
    assert api.quantize_kv_q4(k, -k, cache, i32([0]), i32([300]), i32([512]), block_table=table)["status"].item() == 0
    assert not cache.k_codes[0, :1].any() and not cache.k_codes[0, 2:-1].any()
    r = api.dequantize_kv_q4(cache, i32([0]), i32([300]), 300, block_table=table)
    assert torch.equal(r["k"], -r["v"]) and (r["k"] - k).abs().max() <= 0.25 * k.abs().max()
    q, kt = torch.randn((1, 2, 32, d), device="cuda", dtype=torch.bfloat16), torch.randn((1, 2, Hkv, d), device="cuda", dtype=torch.bfloat16)
    args = (i32([300]), kt, kt, torch.tensor([[[1], [3]]], device="cuda"), i32([2]))
    got, _ = api.tree_verify_attention_q4(q, cache.layer(0), *args, P_max=300, block_table=table)
    small = api.KVCacheQ4(*(t[:, [blocks - 1, 1]].contiguous() for t in cache))
    want, _ = api.tree_verify_attention_q4(q, small.layer(0), *args, P_max=300, block_table=i32([[0, 1]]))
    assert torch.equal(got, want)


def test_calls_follow_the_current_stream_and_replay_in_a_graph():
    """Written, read back: captured once, replayed with new rows and lengths in the same buffers, eager work in between."""
    layers, B, rows, Hkv, d, block = 2, 3, 9, 2, 128, 16
    rng = np.random.default_rng(3)
    cache, table, _, _ = empty_cache(rng, layers, B, Hkv, d, block, 64)
    other = api.KVCacheQ4(*(t.clone() for t in cache))
    k, P, n, cap, bt = torch.randn((layers, B, rows, Hkv, d), device="cuda"), i32([0, 0, 0]), i32([1, 1, 1]), i32([64] * 3), dev(table)
    out = dict(k=torch.empty_like(k), v=torch.empty_like(k), status=i32([0] * 3))
    wr = dict(prefix_len_out=i32([0] * 3), status=i32([0] * 3))

    def call():
        api.quantize_kv_q4(k, k, cache, P, n, cap, block_table=bt, out=wr)
        api.dequantize_kv_q4(cache, P, n, rows, block_table=bt, out=out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for rep in range(4):
        k.copy_(torch.randn(k.shape, device="cuda"))
        P.copy_(i32([rep * 9, 5, 40 - rep]))
        n.copy_(i32([9, rep, 1 + rep]))
        graph.replay()
        r = api.quantize_kv_q4(k, k, other, P, n, cap, block_table=bt)
        want = api.dequantize_kv_q4(other, P, n, rows, block_table=bt, dtype=torch.float32)
        torch.cuda.synchronize()
        assert torch.equal(r["prefix_len_out"], wr["prefix_len_out"]) and torch.equal(out["k"], want["k"]) and torch.equal(out["v"], want["v"])
