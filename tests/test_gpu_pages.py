"""resize_block_tables on the GPU against its definition: every table entry, ring entry, slot, length and status bit."""
import numpy as np
import pytest
import torch

import beam_plain
from paper_2603_08088_amd import api

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def batch(rng, lens, news, size, spare, width=None, first=None):
    """Tables of their own blocks, and a ring of all others, `spare` of them free beyond what the growth takes."""
    have = [beam_plain.cover(max(0, int(L)), size) for L in lens]
    grow = sum(max(0, beam_plain.cover(max(0, int(N)), size) - h) for N, h in zip(news, have))
    n = max(1, sum(have) + max(0, grow + spare))
    width = width or max([beam_plain.cover(max(0, int(x)), size) for x in list(lens) + list(news)] + [1]) + 1
    ids = rng.permutation(n).astype(np.int32)
    table, at = np.full((len(lens), width), -7, dtype=np.int32), 0
    for b, h in enumerate(have):
        table[b, :min(h, width)] = ids[at:at + min(h, width)]
        at += h
    first = int(rng.integers(n)) if first is None else first
    ring = np.full(n, -9, dtype=np.int32)
    ring[(first + np.arange(n - at)) % n] = ids[at:]
    return table, ring, [first, n - at]


def check(table, lens, news, ring, state, size, S, **kw):
    t, blocks = dev(table), dev(ring)
    r = api.resize_block_tables(t, dev(lens), dev(news), api.FreeBlocks(blocks, dev(state)), size, S, **kw)
    want = beam_plain.resize(table, lens, news, ring, state, size, S)
    assert r["status"].tolist() == want[5]
    assert r["length"].tolist() == want[3]
    assert np.array_equal(t.cpu().numpy(), want[0])
    assert np.array_equal(blocks.cpu().numpy(), want[1])
    assert r["free_state"].tolist() == want[2]
    if r["slot_map"] is not None:
        assert np.array_equal(r["slot_map"].cpu().numpy(), want[4])
    return want


@pytest.mark.parametrize("size", [1, 16, 24, 64])
@pytest.mark.parametrize("B,S", [(1, 1), (3, 1), (64, 1), (300, 1), (2000, 1), (5, 40), (70, 63), (3, 700), (7, 1024), (4, 2500), (2, 9000)])
def test_growth_and_release(B, S, size):
    rng = np.random.default_rng(B + S)
    lens = rng.integers(0, 400, B)
    news = lens + rng.integers(0, S + 1, B)
    news = np.where(rng.random(B) < 0.25, (lens * rng.random(B)).astype(int), news)     # some shrink, some to nothing
    table, ring, state = batch(rng, lens, news, size, 3)
    want = check(table, lens, news, ring, state, size, S)
    assert want[5] == [0] * B


@pytest.mark.parametrize("lens,news", [([0], [0]), ([0], [1]), ([15, 16, 17], [16, 17, 18]), ([16, 1, 0], [0, 0, 16]), ([100, 100], [96, 97]), ([5], [5]),
                                       ([31, 32, 33, 0], [0, 31, 32, 33])])
def test_lengths_at_the_borders_of_blocks(lens, news):
    rng = np.random.default_rng(1)
    table, ring, state = batch(rng, lens, news, 16, 0)
    check(table, lens, news, ring, state, 16, 40)
    check(table, lens, news, ring, state, 16, 40, want_slots=False)


@pytest.mark.parametrize("short", [1, 2, 5, 9])
def test_a_ring_that_is_short_serves_the_first_sequences(short):
    rng = np.random.default_rng(2)
    lens, news = [20, 3, 40, 7, 16, 0, 90], [60, 3, 70, 12, 33, 50, 10]
    table, ring, state = batch(rng, lens, news, 16, -short)
    want = check(table, lens, news, ring, state, 16, 64)
    assert beam_plain.NO_BLOCKS in want[5] and want[5][6] == 0
    check(table, lens, news, ring, [0, 0], 16, 64)


def test_refusals_leave_sequences_as_they_were():
    rng = np.random.default_rng(3)
    lens, news = [20, -1, 5, 40, 33, 60, 10, 48, 64, 5], [30, 4, -2, 120, 40, 20, 11, 10, 16, 500]
    table, ring, state = batch(rng, [max(0, x) for x in lens], [min(120, max(0, x)) for x in news], 16, 4, width=6)
    table[4, 2] = 10 ** 6            # the block its new rows go on in
    table[5, 3] = -1                 # one to give back
    table[6, 0] = -1                 # the same, growing within the block
    want = check(table, lens, news, ring, state, 16, 100)
    assert want[5] == [0, 4, 4, 1, 8, 8, 8, 0, 0, 4]
    # bad entries of the ring: the sequences that would get them
    for place in range(4):
        lens, news = [16, 0, 32, 16], [40, 5, 33, 16]
        table, ring, state = batch(rng, lens, news, 16, 1)
        ring[(state[0] + place) % len(ring)] = len(ring) + place
        want = check(table, lens, news, ring, state, 16, 64)
        assert want[5].count(beam_plain.BAD_FREE) == 1
    # long rows, each of whose workgroups has to come to the same answer
    lens, news = [3, 0], [5000, 4000]
    table, ring, state = batch(rng, lens, news, 16, 0)
    ring[(state[0] + 300) % len(ring)] = -1
    assert check(table, lens, news, ring, state, 16, 5000)[5] == [beam_plain.BAD_FREE, 0]


def test_a_ring_without_room_and_states_that_are_none():
    rng = np.random.default_rng(4)
    lens, news = [64, 32, 10, 48], [0, 0, 40, 0]
    table, ring, state = batch(rng, lens, news, 16, 2)
    for room in range(0, 9):
        check(table, lens, news, ring, [state[0], len(ring) - room], 16, 64)
    for bad in ([-1, 3], [len(ring), 3], [0, -1], [0, len(ring) + 1], [2 ** 31 - 1, 2 ** 31 - 1]):
        want = check(table, lens, news, ring, bad, 16, 64)
        assert want[5] == [32, 32, 16, 32] and want[2] == bad


def test_many_sequences_give_back_across_the_scans_steps():
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 900, 1200)
    news = np.where(rng.random(1200) < 0.7, (lens * rng.random(1200)).astype(int), lens + rng.integers(0, 50, 1200))
    table, ring, state = batch(rng, lens, news, 16, 0)
    for b in rng.integers(0, 1200, 20):
        table[b, 0] = -1
    check(table, lens, news, ring, state, 16, 50)


def test_an_empty_batch_hands_the_state_on():
    blocks = torch.arange(8, dtype=torch.int32, device="cuda")
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    r = api.resize_block_tables(empty.view(0, 4), empty, empty, api.FreeBlocks(blocks, dev([3, 5])), 16, 1)
    assert r["free_state"].tolist() == [3, 5]


def test_lengths_to_the_end_of_31_bits():
    """Slots and positions near 2^31: one block of 2^30 rows after another."""
    size = 1 << 30
    table = np.array([[0, -1]], dtype=np.int32)
    want = check(table, [size - 3], [size], np.array([-1], dtype=np.int32), [0, 0], size, 8)
    assert want[4][0, :4].tolist() == [size - 3, size - 2, size - 1, -1]
    check(np.array([[0, -1]]), [2 ** 31 - 1], [2 ** 31 - 1], np.array([-1]), [0, 0], size, 8)


def test_a_run_of_steps_keeps_every_block_once():
    """Requests that come, grow and leave: a block is in one table or in the ring, never twice."""
    rng = np.random.default_rng(6)
    B, size, n = 12, 16, 150
    table, free, lens = torch.full((B, 40), -1, dtype=torch.int32, device="cuda"), api.FreeBlocks.all(n), np.zeros(B, dtype=int)
    for _ in range(60):
        news = np.where(rng.random(B) < 0.15, 0, np.minimum(lens + rng.integers(0, 60, B), 600))
        r = api.resize_block_tables(table, dev(lens), dev(news), free, size, 64)
        free, lens = free.after(r), r["length"].cpu().numpy()
        first, count = free.state.tolist()
        ring, t = free.blocks.cpu().numpy(), table.cpu().numpy()
        used = [int(x) for b in range(B) for x in t[b, :beam_plain.cover(int(lens[b]), size)]]
        assert sorted(used + [int(ring[(first + i) % n]) for i in range(count)]) == list(range(n))
