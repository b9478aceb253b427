"""The calls of beam decoding as plain definitions, entry by entry and in 64 bits: the oracle of their GPU tests."""
import math

import numpy as np

BAD_LEN, CAPACITY, BAD_NODE, BAD_BLOCK, NO_BLOCKS, BAD_FREE = 4, 1, 2, 8, 16, 32


class Ring:
    """The free blocks: what may be taken from the front, and where given-back ones go."""

    def __init__(self, blocks, state):
        self.blocks, self.n = np.array(blocks), len(blocks)
        self.first, self.count = (int(x) for x in state)
        self.valid = 0 <= self.first < self.n and 0 <= self.count <= self.n
        self.usable, self.room = (self.count, self.n - self.count) if self.valid else (0, 0)
        self.taken = self.given = 0

    def entry(self, i):
        return int(self.blocks[(self.first + i) % self.n])

    def put(self, ids):
        for block in ids:
            self.blocks[(self.first + self.count + self.given) % self.n] = block
            self.given += 1

    def state(self):
        if not self.valid:
            return [self.first, self.count]
        return [(self.first + self.taken) % self.n, self.count - self.taken + self.given]


def cover(length, size):
    return -(-length // size)


def resize(table, lens, news, blocks, state, size, S):
    """-> table, ring entries, state, lengths, slots [B, S], status"""
    table, ring, B = np.array(table), Ring(blocks, state), len(lens)
    new_len, slots, status = [int(x) for x in lens], np.full((B, S), -1, dtype=np.int32), [0] * B
    old_table, asked, giving = table.copy(), 0, 0
    for b, (L, N) in enumerate(zip(lens, news)):
        L, N = int(L), int(N)
        if L < 0 or N < 0 or N - L > S:
            status[b] = BAD_LEN
            continue
        have, want = cover(L, size), cover(N, size)
        if max(have, want) > table.shape[1]:
            status[b] = CAPACITY
            continue
        if want < have:
            ids = old_table[b, want:have]
            if ((ids < 0) | (ids >= ring.n)).any():
                status[b] = BAD_BLOCK
                continue
            giving += len(ids)
            if giving > ring.room:
                status[b] = BAD_FREE
                continue
            ring.put(ids)
        else:
            start, asked = asked, asked + want - have
            if want > have and asked > ring.usable:
                status[b] = NO_BLOCKS
                continue
            ring.taken = max(ring.taken, asked if want > have else 0)
            if N > L and L % size and not 0 <= old_table[b, have - 1] < ring.n:
                status[b] = BAD_BLOCK
                continue
            ids = [ring.entry(start + i) for i in range(want - have)]
            if any(not 0 <= x < ring.n for x in ids):
                status[b] = BAD_FREE
                continue
            table[b, have:want] = ids
            for i in range(max(0, N - L)):
                slots[b, i] = table[b, (L + i) // size] * size + (L + i) % size
        new_len[b] = N
    return table, ring.blocks, ring.state(), new_len, slots, status


def reorder(table, lens, parent, blocks, state, size):
    """-> table, ring entries, state, status, copies [(source block, destination block, rows)]"""
    table, parent, ring = np.array(table), np.array(parent), Ring(blocks, state)
    (B, K, width), M = table.shape, parent.shape[1]
    out, status, copies, asked, giving = np.full((B, M, width), -1, dtype=np.int32), [0] * B, [], 0, 0
    for b in range(B):
        L = int(lens[b])
        if L < 0:
            status[b] = BAD_LEN
        elif cover(L, size) > width:
            status[b] = CAPACITY
        if ((parent[b] < -1) | (parent[b] >= K)).any():
            status[b] |= BAD_NODE
        cols = 0 if status[b] & (BAD_LEN | CAPACITY) else cover(L, size)
        alive = sorted({int(p) for p in parent[b] if 0 <= p < K})
        if any(not 0 <= x < ring.n for p in alive for x in table[b, p, :cols]):
            status[b] |= BAD_BLOCK
        if status[b]:
            continue
        held, copied = set(), []
        if L % size:
            for i, p in enumerate(parent[b]):
                if p >= 0 and int(table[b, p, cols - 1]) in held:
                    copied.append(i)
                elif p >= 0:
                    held.add(int(table[b, p, cols - 1]))
        start, asked = asked, asked + len(copied)
        if copied and asked > ring.usable:
            status[b] = NO_BLOCKS
            continue
        if copied:
            ring.taken = asked
        back = []
        for j in range(cols):
            used = {int(table[b, p, j]) for p in alive}
            for k in range(K):
                x = int(table[b, k, j])
                if k not in alive and 0 <= x < ring.n and x not in used:
                    back.append(x)
                    used.add(x)
        for i, p in enumerate(parent[b]):
            if p >= 0:
                out[b, i, :cols] = table[b, p, :cols]
        for n, i in enumerate(copied):
            source, to = int(out[b, i, cols - 1]), ring.entry(start + n)
            if 0 <= to < ring.n:
                copies.append((source, to, L % size))
                out[b, i, cols - 1] = to
            else:
                out[b, i] = -1
                status[b] |= BAD_FREE
        giving += len(back)
        if giving > ring.room and back:
            status[b] |= BAD_FREE
            out[b] = -1
            continue
        ring.put(back)
    return out, ring.blocks, ring.state(), status, copies


def rotate(x, positions, inv_freq, axis_of, interleaved, scale=1.0, inverse=False):
    """x float64 [B, T, H, d], positions [n_axes, B, T] -> the turned rows.  The angle is an exact product of a 32-bit position and a 24-bit
    frequency, taken modulo a turn in extended precision."""
    half = len(inv_freq)
    turn = 2 * np.longdouble("3.14159265358979323846264338327950288")
    angle = np.stack([positions[axis_of[i]].astype(np.longdouble) * np.longdouble(inv_freq[i]) for i in range(half)], -1)[:, :, None]
    angle = angle - turn * np.rint(angle / turn)
    c, s = np.cos(angle).astype(np.float64) * scale, np.sin(angle).astype(np.float64) * scale * (-1 if inverse else 1)
    y = x.copy()
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


LEAST = float.fromhex("0x1.ffffffp127")      # half an fp32 step beyond the largest


def select(logits, scores, M, n_beams=None, finished=None, end=-1):
    """logits float64 [B, K, V] -> scores float64, parent, token, finished, status"""
    B, K, V = logits.shape
    best, parent, token = np.full((B, M), -math.inf), np.full((B, M), -1), np.full((B, M), -1)
    ended, status = np.zeros((B, M), dtype=int), [0] * B
    for b in range(B):
        totals = np.full((K, V), -math.inf)
        for k in range(K if n_beams is None else min(K, int(n_beams[b]))):
            s, x = float(scores[b, k]), logits[b, k]
            if math.isnan(s) or s == math.inf:
                status[b] |= 2
            elif s == -math.inf:
                continue
            elif finished is not None and finished[b, k]:
                totals[k, end] = s
            elif np.isnan(x).any() or (x == math.inf).any():
                status[b] |= 1
            elif (x > -math.inf).any():
                m = x.max()
                totals[k] = s + ((x - m) - math.log(math.fsum(np.exp(x - m))))     # m apart: it may be as large as fp32 goes
        order = np.argsort(-totals.ravel(), kind="stable")[:M]
        for i, at in enumerate(order):
            if totals.ravel()[at] > -LEAST:          # what rounds to less has no fp32 number
                best[b, i], parent[b, i], token[b, i] = totals.ravel()[at], at // V, at % V
                ended[b, i] = bool(finished is not None and finished[b, parent[b, i]]) or token[b, i] == end
        if (parent[b] < 0).any():
            status[b] |= 4
    return best, parent, token, ended, status
