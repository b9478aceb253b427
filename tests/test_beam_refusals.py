"""What the calls of beam decoding refuse on the host, before anything is launched, and the oracle of their GPU tests pinned by hand; needs no GPU."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import beam_plain
from paper_2603_08088_amd import api

A = 1 << 20      # an aligned address that nobody follows


def pages(d, len=A, new=2 * A, bt=A, fb=A, fs=A, fo=2 * A, lo=3 * A, slots=5 * A, st=4 * A):
    return api.lib().etv_resize_block_tables(C.byref(d), len, new, bt, fb, fs, fo, lo, slots, st, None)


def pages_desc(**kw):
    return api.PagesDesc(**{**dict(B=2, S=4, block_size=16, max_blocks=8, num_blocks=20), **kw})


@pytest.mark.parametrize("kw,rc", [(dict(B=-1), -1), (dict(S=0), -1), (dict(block_size=0), -1), (dict(block_size=-16), -1), (dict(max_blocks=0), -1), (dict(num_blocks=0), -1),
                                   (dict(B=1 << 16, S=1 << 16), -2), (dict(num_blocks=1 << 28), -2), (dict(max_blocks=(1 << 22) + 1), -2)])
def test_pages_descriptors(kw, rc):
    assert pages(pages_desc(**kw)) == rc


def test_pages_pointers_and_aliases():
    d = pages_desc()
    for name in ("len", "new", "bt", "fb", "fs", "fo", "lo", "st"):
        assert pages(d, **{name: None}) == -1, name
    assert pages(d, fo=A) == pages(d, lo=A) == pages(d, lo=2 * A) == -1
    assert pages(d, st=A + 4) == pages(d, st=2 * A - 4) == pages(d, slots=A) == pages(d, slots=2 * A - 28) == pages(d, lo=A - 4) == -1


def rotary_desc(**kw):
    d = api.RotaryDesc(**{**dict(B=2, T=3, Hq=4, Hkv=2, d=64, dtype=api.BF16, rot_dim=64, n_axes=3, flags=0, block_size=16, cache_rows=320, scale=1.0), **kw})
    d.strides[:] = [3 * 4 * 64, 4 * 64, 3 * 2 * 64, 2 * 64] * 3
    return d


def rotary(d, q=A, k=A, v=A, pos=A, freq=A, n=A, qo=A, ko=A, vo=A, slots=A, kc=A, vc=A):
    return api.lib().etv_rotary_write_kv(C.byref(d), q, k, v, pos, freq, n, qo, ko, vo, slots, kc, vc, None)


@pytest.mark.parametrize("kw,rc", [(dict(B=-1), -1), (dict(T=0), -1), (dict(Hq=-1), -1), (dict(Hq=0, Hkv=0), -1), (dict(n_axes=0), -1), (dict(flags=4), -1), (dict(block_size=-1), -1),
                                   (dict(scale=math.nan), -1), (dict(scale=math.inf), -1), (dict(dtype=2), -2), (dict(d=72), -2), (dict(d=272), -2), (dict(rot_dim=0), -2),
                                   (dict(rot_dim=80), -2), (dict(rot_dim=24), -2), (dict(cache_rows=-1), -1), (dict(B=1 << 12, T=1 << 12), -2), (dict(B=0), 0)])
def test_rotary_descriptors(kw, rc):
    assert rotary(rotary_desc(**kw)) == rc


def test_rotary_pointers_strides_and_axes():
    d = rotary_desc()
    for name in ("q", "k", "v", "pos", "freq", "qo", "slots", "kc", "vc"):
        assert rotary(d, **{name: None}) == -1, name
    for name in ("q", "k", "v", "qo", "ko", "vo", "kc", "vc"):
        assert rotary(d, **{name: A + 8}) == -1, name
    assert rotary(d, ko=None, slots=None, kc=None, vc=None) == -1                    # k would go nowhere
    assert rotary(rotary_desc(Hq=0)) == rotary(rotary_desc(Hkv=0)) == -1             # heads that are not there
    for i in range(12):
        for wrong in (4, -1 << 20):
            bad = rotary_desc()
            bad.strides[i] += wrong
            assert rotary(bad) == -1, i
        if i >= 6:                                                                   # rows of an output on one another
            bad = rotary_desc()
            bad.strides[i] = 0
            assert rotary(bad) == -1, i
    bad = rotary_desc(T=2)
    bad.strides[6:8] = [256, 264]
    assert rotary(bad) == -1
    moved = rotary_desc()                                                            # in place, but the rows somewhere else
    moved.strides[6] += 64
    assert rotary(moved) == -1
    one = rotary_desc(B=1, T=1, block_size=-1)                                       # one row: its strides are not looked at, the rest is
    one.strides[:] = [3] * 12
    assert rotary(one) == -1
    d.axis_of[31] = 3
    assert rotary(d) == -1
    d.axis_of[31], d.axis_of[32] = 2, 9                                              # behind the last pair: not looked at
    d.B = 0
    assert rotary(d) == 0


def beam_desc(**kw):
    return api.BeamDesc(**{**dict(B=2, K=4, V=1000, M=4, dtype=api.BF16, end_token=7, batch_stride=4000, row_stride=1000), **kw})


def select(d, x=A, s=A, n=A, f=2 * A, o=A, p=A, t=A, fo=2 * A, st=A, ws=A, size=1 << 40):
    return api.lib().etv_beam_select(C.byref(d), x, s, n, f, o, p, t, fo, st, ws, size, None)


@pytest.mark.parametrize("kw,rc", [(dict(B=-1), -1), (dict(K=0), -1), (dict(M=0), -1), (dict(V=0), -1), (dict(end_token=-2), -1), (dict(end_token=1000), -1), (dict(row_stride=-1), -1), (dict(batch_stride=-1), -1), (dict(B=1 << 20, K=64, V=1 << 20), -2), (dict(B=1 << 23, K=1, V=10), -2),
                                   (dict(K=65), -2), (dict(M=65), -2), (dict(dtype=3), -2), (dict(V=2 ** 31 - 1, row_stride=2 ** 31), -2), (dict(B=0), 0)])
def test_beam_descriptors(kw, rc):
    assert select(beam_desc(**kw)) == rc
    if rc:
        assert api.lib().etv_beam_select_workspace_bytes(C.byref(beam_desc(**kw))) == 0


def test_beam_pointers_and_workspace():
    d = beam_desc()
    for name in ("x", "s", "o", "p", "t", "st"):
        assert select(d, **{name: None}) == -1, name
    assert select(d, x=A + 1) == select(d, ws=A + 8) == select(beam_desc(end_token=-1)) == -1
    assert select(d, o=A + 4) == select(d, o=A - 28) == select(d, fo=2 * A + 7) == select(beam_desc(M=5)) == select(beam_desc(M=3), o=3 * A) == -1    # on old ones
    need = api.lib().etv_beam_select_workspace_bytes(C.byref(d))
    assert need > 0 and select(d, size=need - 1) == select(d, ws=None) == -3


def cache_desc(**kw):
    return api.CacheDesc(**{**dict(B=2, Hkv=2, d=64, elem_bytes=2, n_layers=2, block_size=16, max_blocks=8, num_blocks=20, P_cap=0, reserved=0, cache_layer_stride=20 * 2 * 16 * 64), **kw})


def reorder(d, k=A, v=A, bt=A, len=A, K=4, p=A, M=4, fb=A, fs=A, to=2 * A, fo=2 * A, st=3 * A, ws=A, size=1 << 40):
    return api.lib().etv_reorder_beams(C.byref(d), k, v, bt, len, K, p, M, fb, fs, to, fo, st, ws, size, None)


def reorder_q4(d, kc=A, ks=A, vc=A, vs=A, bt=A, to=2 * A, ws=A):
    return api.lib().etv_reorder_beams_q4(C.byref(d), kc, ks, vc, vs, bt, A, 4, A, 4, A, A, to, 2 * A, A, ws, 1 << 40, None)


@pytest.mark.parametrize("kw,rc", [(dict(B=-1), -1), (dict(Hkv=0), -1), (dict(d=0), -1), (dict(n_layers=0), -1), (dict(block_size=-1), -1), (dict(block_size=0), -5), (dict(max_blocks=0), -1),
                                   (dict(num_blocks=0), -1), (dict(elem_bytes=1), -2), (dict(d=12), -2), (dict(B=70000), -2), (dict(num_blocks=1 << 28), -2),
                                   (dict(cache_layer_stride=20 * 2 * 16 * 64 + 4), -2), (dict(max_blocks=(1 << 22) + 1), -2)])
def test_reorder_descriptors(kw, rc):
    assert reorder(cache_desc(**kw)) == rc


def test_reorder_pointers_beams_and_workspace():
    d = cache_desc()
    for name in ("k", "v", "bt", "len", "p", "fb", "fs", "to", "fo", "st"):
        assert reorder(d, **{name: None}) == -1, name
    assert reorder(d, to=A + 4 * 2 * 4 * 8 - 4) == reorder(d, to=A - 4 * 2 * 4 * 8 + 4) == -1          # overlapping tables
    assert reorder(cache_desc(Hkv=1 << 15, d=256, block_size=256, num_blocks=4)) == -2              # a block of a layer beyond 32 bits
    assert reorder(d, st=A) == reorder(d, st=A + 4) == reorder(d, st=A - 4) == -1
    assert reorder(d, k=A + 8) == reorder(d, to=A) == reorder(d, fo=A) == reorder(d, ws=A + 4) == -1
    assert reorder(d, K=0) == reorder(d, M=0) == -1 and reorder(d, K=65) == reorder(d, M=65) == -2
    assert reorder(cache_desc(B=1 << 13, max_blocks=1 << 16)) == -2 and api.reorder_beams_workspace_bytes(1 << 13, 4, 4, 1 << 16) == 0   # 2^31 entries
    need = api.reorder_beams_workspace_bytes(2, 4, 4, 8)
    assert need > 0 and reorder(d, size=need - 1) == reorder(d, ws=None) == -3
    assert api.reorder_beams_workspace_bytes(2, 65, 4, 8) == api.reorder_beams_workspace_bytes(-1, 4, 4, 8) == 0
    q = api.Q4Desc(B=2, rows=1, Hkv=2, d=64, n_layers=2, block_size=16, max_blocks=8, num_blocks=20, layer_rows=640)
    for name in ("kc", "ks", "vc", "vs", "bt", "to", "ws"):
        assert reorder_q4(q, **{name: None}) in (-1, -3), name
    assert reorder_q4(q, kc=A + 8) == reorder_q4(q, ks=A + 1) == -1
    for kw, rc in ((dict(block_size=0), -5), (dict(block_size=24), -2), (dict(d=96), -2), (dict(layer_rows=-1), -1)):
        q = api.Q4Desc(**{**dict(B=2, rows=1, Hkv=2, d=64, n_layers=2, block_size=16, max_blocks=8, num_blocks=20, layer_rows=640), **kw})
        assert reorder_q4(q) == rc


def test_struct_layouts_match_the_header():
    assert C.sizeof(api.PagesDesc) == 24 and C.sizeof(api.BeamDesc) == 40 and C.sizeof(api.RotaryDesc) == 40 + 8 + 8 + 96 + 128


def test_python_checks_shapes_before_the_library_is_called():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    free = api.FreeBlocks(i32(20), i32(2))
    good = [i32(2, 8), i32(2), i32(2), free, 16, 4]
    for at, other in ((0, i32(2, 8).long()), (0, i32(3, 8)), (1, i32(3)), (2, i32(2).long()), (3, api.FreeBlocks(i32(20, 1), i32(2))), (3, api.FreeBlocks(i32(20), i32(3)))):
        with pytest.raises(ValueError):
            api.resize_block_tables(*good[:at], other, *good[at + 1:])
    with pytest.raises(ValueError):
        api.resize_block_tables(*good, out=dict(slot_map=i32(2, 5)))
    with pytest.raises(AssertionError):                                # good shapes: refused as host memory
        api.resize_block_tables(*good)
    with pytest.raises(TypeError):
        api.resize_block_tables(*good[:4], 16.0, 4)

    rot = api.Rotary(torch.ones(32), axis_of=[0] * 16 + [2] * 16)
    q, k, pos = torch.zeros((2, 3, 4, 64)), torch.zeros((2, 3, 2, 64)), i32(3, 2, 3)
    cache = torch.zeros((20, 2, 16, 64))
    call = lambda **kw: api.rotary_write_kv(**{**dict(q=q, k=k, v=k, positions=pos, rotary=rot), **kw})
    for kw in (dict(q=q[0]), dict(k=k.bfloat16()), dict(v=k[:, :, :1]), dict(v=k[:, :2]), dict(q=q.transpose(1, 2)), dict(q=q.transpose(2, 3)), dict(positions=pos.long()),
               dict(positions=pos[:, :, :2]), dict(n_rows=i32(3)), dict(k_cache=cache, v_cache=cache), dict(slot_map=i32(2, 4), k_cache=cache, v_cache=cache),
               dict(slot_map=i32(2, 3), k_cache=cache, v_cache=cache.bfloat16()), dict(slot_map=i32(2, 3), k_cache=cache, v_cache=cache, paged=False), dict(out=dict(q=q[:, :, :2])),
               dict(q=None, out=dict(q=q)), dict(k=None), dict(q=None, k=None, v=None)):
        with pytest.raises((ValueError, TypeError)):
            call(**kw)
    with pytest.raises(api.EtvError):
        call(q=q.half(), k=None, v=None)
    for bad in (dict(axis_of=[0] * 31), dict(axis_of=[0] * 31 + [-1]), dict(scale=0.0), dict(scale=math.nan)):
        with pytest.raises(ValueError):
            api.Rotary(torch.ones(32), **bad)
    with pytest.raises(ValueError):
        api.Rotary(torch.ones(32, dtype=torch.float64))

    x, s = torch.zeros((2, 4, 50)), torch.zeros((2, 4))
    for kw in (dict(scores=s[:1]), dict(scores=s.double()), dict(n_beams=i32(3)), dict(finished=torch.zeros((2, 4))), dict(logits=x.transpose(1, 2)), dict(end_token=50),
               dict(end_token=-2), dict(out=dict(scores=torch.zeros((2, 4)))), dict(out=dict(parent=i32(2, 4)))):
        with pytest.raises(ValueError):
            api.beam_select(**{**dict(logits=x, scores=s, M=3), **kw})
    with pytest.raises(api.EtvError):
        api.beam_select(x.half(), s, 3)

    c, t = torch.zeros((2, 20, 2, 16, 64)), i32(2, 4, 8)
    good = [c, c, t, i32(2), i32(2, 4), free]
    for at, other in ((0, c[0]), (1, c.bfloat16()), (2, t[0]), (2, t.long()), (3, i32(3)), (4, i32(3, 4)), (4, i32(2)), (5, api.FreeBlocks(i32(19), i32(2)))):
        with pytest.raises(ValueError):
            api.reorder_beams(*good[:at], other, *good[at + 1:])
    with pytest.raises(ValueError):
        api.reorder_beams(*good, out=dict(block_table=i32(2, 4, 7)))
    with pytest.raises(AssertionError):
        api.reorder_beams(*good)
    q4 = api.KVCacheQ4.empty(2, 20, 2, 16, 64, device="cpu")
    with pytest.raises(ValueError):
        api.reorder_beams_q4(q4._replace(v_scales=q4.v_codes), *good[2:])
    with pytest.raises(AssertionError):
        api.reorder_beams_q4(q4, *good[2:])


def test_the_oracle_by_hand():
    # two sequences over blocks of four rows: one grows from 3 to 9, the other shrinks from 8 to 2
    table, ring, state, lens, slots, status = beam_plain.resize([[5, -1, -1], [2, 6, -1]], [3, 8], [9, 2], [-1, 0, 1, 3, 4, -1, -1], [1, 4], 4, 6)
    assert table.tolist() == [[5, 0, 1], [2, 6, -1]] and ring.tolist() == [-1, 0, 1, 3, 4, 6, -1] and state == [3, 3]
    assert lens == [9, 2] and slots[0].tolist() == [23, 0, 1, 2, 3, 4] and (slots[1] == -1).all() and status == [0, 0]
    # beams 0 and 2 of three go on, 0 twice: its block is copied into the ring's next, beam 1's own block is given back
    out, ring, state, status, copies = beam_plain.reorder([[[7, 1], [7, 2], [7, 3]]], [6], [[0, 2, 0]], [-1, -1, 0, 4, 5, 6, -1, -1], [2, 4], 4)
    assert out.tolist() == [[[7, 1], [7, 3], [7, 0]]] and copies == [(1, 0, 2)] and ring.tolist() == [-1, -1, 0, 4, 5, 6, 2, -1] and state == [3, 4] and status == [0]
    # a quarter turn
    x = np.arange(4.0).reshape(1, 1, 1, 4)
    q = math.pi / 2
    assert np.allclose(beam_plain.rotate(x, np.array([[[1]], [[2]]]), np.array([q, q]), [0, 1], False), [-2, -1, 0, -3])
    assert np.allclose(beam_plain.rotate(x, np.array([[[1]], [[2]]]), np.array([q, q]), [0, 1], True), [-1, 0, -2, -3])
    assert np.allclose(beam_plain.rotate(x, np.array([[[1]], [[2]]]), np.array([q, q]), [0, 1], True, 2.0, True), [2, 0, -4, -6])
    # two beams of probabilities (1/2, 1/2) and (1/4, 3/4), scores log 2 and log 4 below
    p = np.log(np.array([[[0.5, 0.5], [1.0, 3.0]]]))
    best, parent, token, ended, status = beam_plain.select(p, np.array([[0.0, math.log(0.5)]]), 5, None, None, 1)
    assert np.allclose(np.exp(best[0]), [0.5, 0.5, 0.375, 0.125, 0]) and parent[0].tolist() == [0, 0, 1, 1, -1] and token[0].tolist() == [0, 1, 1, 0, -1]
    assert ended[0].tolist() == [0, 1, 1, 0, 0] and status == [4]
    best, parent, token, ended, _ = beam_plain.select(p, np.array([[-1.0, -0.1]]), 2, None, np.array([[0, 1]]), 1)
    assert parent[0].tolist() == [1, 0] and token[0].tolist() == [1, 0] and ended[0].tolist() == [1, 0] and best[0, 0] == -0.1


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_workspace_for_the_largest_selection_fits_smaller_ones(dtype):
    """A program sizes it once: fewer requests, beams, logits or continuations need no more, although their rows are in more segments."""
    size = lambda B, K, V, M: api.beam_select_workspace_bytes(B, K, V, M, dtype)
    assert all(size(B, 4, 32000, 4) <= size(B + 1, 4, 32000, 4) for B in range(1, 300))
    assert all(size(B, 8, 128000, 20) <= size(B + 1, 8, 128000, 20) for B in range(1, 150))
    assert all(size(40, K, 50021, 17) <= size(40, K + 1, 50021, 17) for K in range(1, 64))
    assert all(size(30, 10, V, 10) <= size(30, 10, V + 700, 10) for V in range(1, 400000, 700))
    assert all(size(32, 8, 128000, M) <= size(32, 8, 128000, M + 1) for M in range(1, 64))
    rng = np.random.default_rng(5)
    for _ in range(2000):
        most = [int(np.exp(rng.uniform(0, np.log(n)))) for n in (2000, 64, 300000, 64)]
        assert size(*(int(rng.integers(1, n + 1)) for n in most)) <= size(*most), most


@pytest.mark.parametrize("by", [-4, 4])
def test_the_ring_s_new_state_beside_its_old_one(by):
    """Every workgroup reads the old state while one writes the new: half of one on the other is refused like all of it."""
    assert pages(pages_desc(), fs=2 * A, fo=2 * A + by) == pages(pages_desc(B=0), fs=2 * A, fo=2 * A + by) == -1
    assert reorder(cache_desc(), fs=2 * A, fo=2 * A + by) == reorder(cache_desc(B=0), fs=2 * A, fo=2 * A + by) == -1
    q = api.Q4Desc(B=2, rows=1, Hkv=2, d=64, n_layers=2, block_size=16, max_blocks=8, num_blocks=20, layer_rows=640)
    assert api.lib().etv_reorder_beams_q4(C.byref(q), A, A, A, A, A, A, 4, A, 4, A, 2 * A, 2 * A, 2 * A + by, A, A, 1 << 40, None) == -1
