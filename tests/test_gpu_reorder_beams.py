"""reorder_beams on the GPU against its definition: tables, ring, state, status, and every byte of the caches."""
import numpy as np
import pytest
import torch

import beam_plain
from paper_2603_08088_amd import api

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def beams(rng, B, K, lens, size, width, spare, apart=3):
    """Tables of beams that share blocks up to some column and part from there on; the ring of all other blocks."""
    need = sum(beam_plain.cover(max(0, L), size) * K for L in lens)
    n = need + spare
    ids, at = rng.permutation(n).astype(np.int32), 0
    table = np.full((B, K, width), -1, dtype=np.int32)
    for b, L in enumerate(lens):
        cols = min(width, beam_plain.cover(max(0, L), size))
        group = np.zeros(K, dtype=int)
        for j in range(cols):
            last = j == cols - 1 and L % size
            if last:
                group = np.arange(K)
            elif j >= cols - 1 - apart:
                group = np.array([g if rng.random() < 0.6 else g + (k + 1) * 100 for k, g in enumerate(group)])
            names = {g: i for i, g in enumerate(dict.fromkeys(group.tolist()))}
            table[b, :, j] = ids[at:at + len(names)][[names[g] for g in group.tolist()]]
            at += len(names)
    free = ids[at:]
    first = int(rng.integers(n))
    ring = np.full(n, -5, dtype=np.int32)
    ring[(first + np.arange(len(free))) % n] = free
    return table, ring, [first, len(free)]


def cache_of(rng, layers, n, Hkv, size, d, dtype):
    if dtype == "q4":
        return [torch.from_numpy(rng.integers(0, 256, (layers, n, Hkv, size, d // w)).astype(np.uint8)) for w in (2, 32, 2, 32)]
    kind = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    return [torch.from_numpy(rng.standard_normal((layers, n, Hkv, size, d)).astype(np.float32)).to(kind) for _ in range(2)]


def check(rng, table, lens, parent, ring, state, size, dtype="bf16", layers=2, Hkv=2, d=64, **kw):
    parts = cache_of(rng, layers, len(ring), Hkv, size, d, dtype)
    on, blocks, before = [t.cuda() for t in parts], dev(ring), dev(table)
    free = api.FreeBlocks(blocks, dev(state))
    if dtype == "q4":
        r = api.reorder_beams_q4(api.KVCacheQ4(*on), before, dev(lens), dev(parent), free, **kw)
    else:
        r = api.reorder_beams(*on, before, dev(lens), dev(parent), free, **kw)
    out, want_ring, want_state, status, copies = beam_plain.reorder(table, lens, parent, ring, state, size)
    assert r["status"].tolist() == status
    assert np.array_equal(r["block_table"].cpu().numpy(), out)
    assert np.array_equal(blocks.cpu().numpy(), want_ring) and r["free_state"].tolist() == want_state
    assert np.array_equal(before.cpu().numpy(), table)
    for source, to, rows in copies:
        for t in parts:
            t[:, to, :, :rows] = t[:, source, :, :rows]
    for got, want in zip(on, parts):
        assert torch.equal(got.cpu().view(torch.uint8), want.view(torch.uint8))
    return out, want_state, status, copies


@pytest.mark.parametrize("dtype", ["bf16", "f32", "q4"])
@pytest.mark.parametrize("B,K,M,size", [(1, 1, 1, 16), (1, 4, 4, 16), (3, 1, 8, 16), (5, 8, 8, 32), (2, 8, 3, 16), (40, 3, 5, 16), (2, 64, 64, 48), (300, 2, 2, 16), (3, 5, 1, 128)])
def test_tables_copies_and_the_ring(B, K, M, size, dtype):
    rng = np.random.default_rng(B * K + M)
    lens = [int(x) for x in rng.integers(0, 10 * size, B)]
    lens[0] = 3 * size + 5
    table, ring, state = beams(rng, B, K, lens, size, 12, B * M)
    parent = rng.integers(0, K, (B, M))
    parent[rng.random((B, M)) < 0.1] = -1
    *_, status, copies = check(rng, table, lens, parent, ring, state, size, dtype, layers=3 if B < 10 else 1, Hkv=5 if B < 10 else 1, d=128 if K == 4 else 64)
    assert status == [0] * B


@pytest.mark.parametrize("L", [0, 1, 15, 16, 17, 2047, 2048, 2049, 4000])
@pytest.mark.parametrize("parent", [[0, 1, 2, 3], [3, 3, 3, 3], [-1, -1, -1, -1], [2, -1, 2, 0], [1, 0, 1, 0]])
def test_lengths_at_the_borders_of_blocks_and_chunks(L, parent):
    rng = np.random.default_rng(L + 1)
    table, ring, state = beams(rng, 1, 4, [L], 16, 260, 6)
    out, after, *_ = check(rng, table, [L], [parent], ring, state, 16, layers=1, Hkv=1)
    if parent == [-1] * 4:          # the request's end: all of its blocks are free again
        assert after[1] == state[1] + len(set(table[0][table[0] >= 0].tolist())) and (out == -1).all()


@pytest.mark.parametrize("K", [9, 20, 33, 64])
@pytest.mark.parametrize("apart,M", [(0, 5), (3, 64), (200, 3)])
@pytest.mark.parametrize("kept", [0, 2, 40])
def test_many_beams_that_part_early_or_late(K, apart, M, kept):
    """Columns that all beams share, that groups share and that each has to itself, over several chunks; few beams go on, or none."""
    rng = np.random.default_rng(K + apart)
    lens = [16 * 150 + 3, 16 * 70, 5, 0]
    table, ring, state = beams(rng, 4, K, lens, 16, 152, 4 * M, apart=apart)
    parent = rng.integers(0, min(K, kept), (4, M)) if kept else np.full((4, M), -1)
    table[1, K - 1, :3] = [-9, len(ring), 2 ** 30]               # of a beam that does not go on, unless all may
    *_, status, _ = check(rng, table, lens, parent, ring, state, 16, layers=1, Hkv=1)
    assert kept == 40 or status == [0] * 4


@pytest.mark.parametrize("refused", [(), (3,), (65, 300, 699)])
def test_many_requests_of_several_chunks(refused):
    """What the requests before a request need and give is added up over more of them than a workgroup takes at a time."""
    rng = np.random.default_rng(700)
    B, size = 700, 1
    lens = [int(rng.integers(70, 140)) if b % 50 == 0 else int(rng.integers(1, 10)) for b in range(B)]
    table, ring, state = beams(rng, B, 2, lens, size, 140, B)
    size = 16
    lens = [(L - 1) * size + 1 + L % size for L in lens]      # the same columns, most of them with a half-filled block
    parent = rng.integers(0, 2, (B, 2))
    for b in refused:
        if b % 2: parent[b, 1] = 2                            # no such beam
        else: table[b, 0, 0], table[b, 1, 0] = -7, -7         # no such block, in another chunk than the one being filled
    *_, status, copies = check(rng, table, lens, parent, ring, state, size, layers=1, Hkv=1)
    assert [b for b, st in enumerate(status) if st] == list(refused) and len(copies) > 200


def test_a_long_table():
    rng = np.random.default_rng(8)
    table, ring, state = beams(rng, 1, 3, [20000 * 2 + 1], 2, 20002, 9, apart=2500)
    *_, status, copies = check(rng, table, [40001], [[2, 2, -1]], ring, state, 2, layers=1, Hkv=1)
    assert status == [0] and len(copies) == 1


def test_beams_that_share_the_block_being_filled_part():
    """A table that was copied row by row: every beam but the first gets a block of its own, and rows without a beam do not count."""
    rng = np.random.default_rng(3)
    table = np.full((2, 4, 6), -1, dtype=np.int32)
    table[0, :, :3] = [4, 9, 2]
    table[1, 0, :2] = table[1, 2, :2] = [5, 6]
    ring = np.array([-1, 0, 1, 3, 7, 8, 10, 11, 12, -1, -1, -1, -1], dtype=np.int32)
    out, state, _, copies = check(rng, table, [40, 20], [[0, 1, 2, 3], [0, 2, 2, -1]], ring, [1, 8], 16)
    assert out[0, :, 2].tolist() == [2, 0, 1, 3] and out[1, :, 1].tolist() == [6, 7, 8, -1] and state == [6, 3]


@pytest.mark.parametrize("short", [0, 1, 2, 4])
def test_a_ring_that_is_short_serves_the_first_requests(short):
    rng = np.random.default_rng(4)
    lens, parent = [20, 32, 50, 7], [[0, 0, 1], [0, 0, 0], [2, 2, 2], [0, 0, 1]]
    table, ring, state = beams(rng, 4, 3, lens, 16, 5, 4)
    keep = [state[0], 4 - short]
    *_, status, _ = check(rng, table, lens, parent, ring, keep, 16)
    assert status == {0: [0, 0, 0, 0], 1: [0, 0, 0, 16], 2: [0, 0, 16, 16], 4: [16, 0, 16, 16]}[short]


def test_refusals_leave_requests_as_they_were():
    rng = np.random.default_rng(5)
    lens, parent = [20, -3, 200, 40, 33, 18, 30], [[0, 0], [0, 1], [1, 1], [0, 2], [-2, 1], [1, 1], [0, 0]]
    table, ring, state = beams(rng, 7, 2, [20, 0, 96, 40, 33, 18, 30], 16, 6, 9)
    table[5, 1, 0] = len(ring)           # a parent's block
    table[6, 1, 0] = -4                  # a block of a beam without children
    *_, status, _ = check(rng, table, lens, parent, ring, state, 16)
    assert status == [0, 4, 1, 2, 2, 8, 0]
    for place in range(4):               # bad entries of the ring: the beams that they were for
        table, ring, state = beams(rng, 2, 3, [20, 21], 16, 4, 5)
        ring[(state[0] + place) % len(ring)] = -1 - place
        *_, status, _ = check(rng, table, [20, 21], [[0, 0, 0], [1, 1, 0]], ring, state, 16)
        assert status == [[32, 0], [32, 0], [0, 32], [0, 0]][place]
    for room in range(8):                # no room for what is given back
        table, ring, state = beams(rng, 3, 2, [40, 16, 33], 16, 4, 3)
        check(rng, table, [40, 16, 33], [[-1, -1], [0, 0], [-1, -1]], ring, [state[0], len(ring) - room], 16)
    for bad in ([-1, 3], [len(ring), 3], [0, -1], [0, len(ring) + 1]):
        check(rng, table, [40, 16, 33], [[0, 0], [0, 0], [1, 1]], ring, bad, 16)


def test_the_workspace_and_the_outputs_may_hold_anything():
    rng = np.random.default_rng(6)
    table, ring, state = beams(rng, 3, 4, [100, 33, 16], 16, 9, 12)
    n = api.reorder_beams_workspace_bytes(3, 4, 5, 9)
    for fill in (0, 0xff):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        out = dict(block_table=torch.full((3, 5, 9), 12345, dtype=torch.int32, device="cuda"))
        check(rng, table, [100, 33, 16], [[0, 1, 1, 2, 2]] * 3, ring, state, 16, workspace=ws, out=out)
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    c = torch.zeros((1, 8, 1, 16, 64), device="cuda")
    r = api.reorder_beams(c, c, e.view(0, 2, 4), e, e.view(0, 2), api.FreeBlocks(dev(range(8)), dev([2, 6])))
    assert r["free_state"].tolist() == [2, 6]


def test_a_run_of_steps_keeps_every_block_once():
    """Beams part, die and grow over many steps: every block is in use or in the ring, the ring never twice, and each beam reads what its line wrote."""
    rng = np.random.default_rng(7)
    B, K, size, n, width = 3, 5, 16, 200, 14
    free = api.FreeBlocks.all(n)
    k, v = (torch.zeros((1, n, 1, size, 64), device="cuda") for _ in range(2))
    one = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    lens = np.array([37, 16, 1])
    r = api.resize_block_tables(one, dev([0] * B), dev(lens), free, size, 64)
    free, table, lines = free.after(r), one.view(B, 1, width), [[[float(100 * b + i) for i in range(L)]] for b, L in enumerate(lens)]
    for b, L in enumerate(lens):
        k.view(-1, 64)[r["slot_map"][b, :L].long()] = torch.tensor(lines[b][0], device="cuda")[:, None]
    for step in range(120):
        parent = rng.integers(0, table.shape[1], (B, K))
        r = api.reorder_beams(k, v, table, dev(lens), dev(parent), free)
        assert r["status"].tolist() == [0] * B
        free, table = free.after(r), r["block_table"]
        lines = [[list(lines[b][p]) for p in parent[b]] for b in range(B)]
        flat = table.view(B * K, width)
        r = api.resize_block_tables(flat, dev(np.repeat(lens, K)), dev(np.repeat(lens + 1, K)), free, size, 1)
        assert r["status"].tolist() == [0] * (B * K)
        free, lens = free.after(r), lens + 1
        new = rng.standard_normal((B, K)).astype(np.float32)
        k.view(-1, 64)[r["slot_map"].view(-1).long()] = torch.from_numpy(new).cuda().view(-1, 1)
        for b in range(B):
            for i in range(K):
                lines[b][i].append(float(new[b, i]))
        t, (first, count), ring = table.cpu().numpy(), free.state.tolist(), free.blocks.cpu().numpy()
        used = {int(x) for b in range(B) for x in t[b, :, :beam_plain.cover(int(lens[b]), size)].ravel()}
        spare = [int(ring[(first + i) % n]) for i in range(count)]
        assert len(set(spare)) == len(spare) and sorted(list(used) + spare) == list(range(n))
        for b in range(B):
            for i in range(K):
                at = [int(t[b, i, p // size]) * size + p % size for p in range(lens[b])]
                assert k.view(-1, 64)[at, 3].tolist() == pytest.approx(lines[b][i], abs=0)
        if step % 40 == 39:             # all but one request end, and begin again
            parent = np.full((B, 1), -1)
            parent[step % B] = 0
            r = api.reorder_beams(k, v, table, dev(lens), dev(parent), free)
            free, table = free.after(r), r["block_table"]
            gone = [b for b in range(B) if b != step % B]
            lines = [[lines[b][0]] if b not in gone else [[]] for b in range(B)]
            lens = np.array([0 if b in gone else int(lens[b]) for b in range(B)])
            if lens.max() > 150:
                r = api.resize_block_tables(table.view(B, width), dev(lens), dev([0] * B), free, size, 1)
                free, lens, lines = free.after(r), lens * 0, [[[]] for _ in range(B)]


def test_layers_of_more_than_2_32_bytes():
    n, size = (1 << 20) + 64, 16
    k, v = (torch.zeros((2, n, 2, size, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = np.array([[[n - 1, n - 2], [n - 1, n - 3]]])
    ring = np.full(n, -1, dtype=np.int32)
    ring[n - 1], ring[0] = 7, n - 4
    for i, t in enumerate((k, v)):
        t[:, n - 2] = 1 + i
        t[:, n - 3] = 3 + i
    free = api.FreeBlocks(dev(ring), dev([n - 1, 2]))
    r = api.reorder_beams(k, v, dev(table), dev([16 + 9]), dev([[1, 1, 1]]), free)
    assert r["status"].tolist() == [0] and r["block_table"].tolist() == [[[n - 1, n - 3], [n - 1, 7], [n - 1, n - 4]]]
    assert r["free_state"].tolist() == [1, 1] and free.blocks[1].item() == n - 2
    for i, t in enumerate((k, v)):
        for block in (7, n - 4):
            assert (t[:, block, :, :9] == 3 + i).all() and not t[:, block, :, 9:].any()
        t[:, [7, n - 2, n - 3, n - 4]] = 0
        assert not any(part.any() for part in t.view(-1).split(1 << 30))


@pytest.mark.parametrize("size,d", [((1 << 23) + 16, 128), ((1 << 15) + 100, 1 << 15)])
def test_a_head_s_rows_in_a_block_of_more_than_2_31_bytes(size, d):
    """Blocks may have up to 2^32 bytes, those of one head too: their offsets are unsigned."""
    k, v = (torch.zeros((1, 3, 1, size, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(3)
    for t in (k, v):
        t.view(torch.int16)[0, 1].random_(generator=gen)
    free, rows = api.FreeBlocks(dev([2, 0, -1]), dev([0, 2])), size - 5
    r = api.reorder_beams(k, v, dev([[[1]]]), dev([rows]), dev([[0, 0]]), free)
    assert r["status"].tolist() == [0] and r["block_table"].tolist() == [[[1], [2]]] and r["free_state"].tolist() == [1, 1]
    for t in (k, v):
        t = t.view(torch.int16)[0, :, 0]
        assert torch.equal(t[2, :rows], t[1, :rows]) and not t[2, rows:].any() and not t[0].any()
