"""What the calls of the 4-bit prefix cache refuse on the host, before anything is launched; needs no GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import q4_plain
from paper_2603_08088_amd import api

A = 1 << 20      # an aligned address that nobody follows


def q4_desc(**kw):
    return api.Q4Desc(**{**dict(B=2, rows=4, Hkv=2, d=64, dtype=api.BF16, n_layers=1, W=3, block_size=16, max_blocks=4, num_blocks=9, P_cap=0,
                                reserved=0, layer_rows=9 * 2 * 16), **kw})


def write(d, k=A, v=A, kc=A, ks=A, vc=A, vs=A, bt=A, P=A, n=A, cap=A, plo=2 * A, st=A):
    return api.lib().etv_quantize_kv_q4(C.byref(d), k, v, kc, ks, vc, vs, bt, P, n, cap, plo, st, None)


def commit(d, kt=A, ks=A, bt=A, P=A, plo=2 * A, acc=A, slot=A):
    return api.lib().etv_commit_accepted_kv_q4(C.byref(d), kt, A, A, ks, A, A, bt, P, A, A, acc, A, plo, slot, A, None)


def read(d, kc=A, bt=A, k=A, first=A):
    return api.lib().etv_dequantize_kv_q4(C.byref(d), kc, A, A, A, bt, first, A, k, A, A, None)


BAD = [(dict(d=96), -2), (dict(dtype=2), -2), (dict(block_size=24), -2), (dict(block_size=-16), -1), (dict(B=-1), -1), (dict(rows=0), -1),
       (dict(Hkv=0), -1), (dict(n_layers=0), -1), (dict(max_blocks=0), -1), (dict(num_blocks=0), -1), (dict(block_size=0, P_cap=0), -1),
       (dict(B=70000), -2), (dict(n_layers=70000), -2), (dict(max_blocks=1 << 28), -2), (dict(layer_rows=-1), -1)]


@pytest.mark.parametrize("kw,rc", BAD)
def test_descriptors(kw, rc):
    assert write(q4_desc(**kw)) == commit(q4_desc(**kw)) == read(q4_desc(**kw)) == rc


def test_pointers_alignment_and_aliases():
    d = q4_desc()
    for name in ("k", "v", "kc", "ks", "vc", "vs", "bt", "P", "n", "cap", "plo", "st"):
        assert write(d, **{name: None}) == -1, name
    for name in ("k", "v", "kc", "vc"):
        assert write(d, **{name: A + 8}) == -1, name
    assert write(d, ks=A + 2) == write(d, vs=A + 1) == -1
    assert write(d, plo=A) == commit(d, plo=A) == -1          # prefix_len_out is prefix_len
    assert commit(d, acc=None) == commit(d, slot=None) == commit(q4_desc(W=0)) == commit(d, bt=None) == commit(d, ks=None) == -1
    assert read(d, kc=None) == read(d, k=None) == read(d, first=None) == read(d, bt=None) == read(d, k=A + 4) == -1
    assert write(q4_desc(rows=1 << 30)) == read(q4_desc(rows=1 << 30)) == -2
    assert write(q4_desc(B=0)) == commit(q4_desc(B=0)) == read(q4_desc(B=0)) == 0      # nothing to do


def attend(d, q=A, kc=A, ks=A, vc=A, vs=A, bt=A, P=A, kt=A, vt=A, mask=A, n=A, out=A, ws=A, size=1 << 40):
    return api.lib().etv_tree_verify_attention_q4(C.byref(d), q, kc, ks, vc, vs, bt, P, kt, vt, mask, n, out, None, ws, size, None)


def attn_desc(**kw):
    return api.AttnDesc(**{**dict(B=1, T_max=8, Hq=8, Hkv=2, d=128, dtype=api.BF16, block_size=16, max_blocks=9, num_blocks=9, P_cap=0, P_max=100),
                           **kw})


@pytest.mark.parametrize("kw,rc", [(dict(B=-1), -1), (dict(T_max=0), -1), (dict(T_max=257), -2), (dict(Hq=9), -1), (dict(Hkv=0), -1), (dict(d=96), -2),
                                   (dict(dtype=7), -2), (dict(block_size=8), -2), (dict(block_size=-16), -1), (dict(num_blocks=0), -1),
                                   (dict(max_blocks=0), -1), (dict(P_max=145), -1), (dict(P_max=-1), -1), (dict(block_size=0, P_cap=99), -1),
                                   (dict(kv_split=-1), -1), (dict(flags=api.ATTN_FLAG_WIDE), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(scale=1e-38), -1),
                                   (dict(B=70000), -2), (dict(B=0), 0)])
def test_attention_descriptors(kw, rc):
    assert attend(attn_desc(**kw)) == rc


def test_attention_pointers_and_workspace():
    d = attn_desc()
    for name in ("q", "kc", "ks", "vc", "vs", "bt", "P", "kt", "vt", "mask", "n", "out"):
        assert attend(d, **{name: None}) == -1, name
    for name in ("q", "kc", "vc", "kt", "vt", "out", "ws"):
        assert attend(d, **{name: A + 8}) == -1, name
    assert attend(d, ks=A + 2) == -1
    d = attn_desc(P_max=8192, max_blocks=512, kv_split=64)
    need = api.tree_verify_attention_q4_workspace_bytes(d)
    if need > 256:
        assert attend(d, size=need - 1) == attend(d, ws=None) == -3
    assert api.tree_verify_attention_q4_workspace_bytes(attn_desc(T_max=0)) == 0


def test_python_checks_shapes_before_the_library_is_called():
    t8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    cache = api.KVCacheQ4(t8(1, 9, 2, 16, 32), t8(1, 9, 2, 16, 2), t8(1, 9, 2, 16, 32), t8(1, 9, 2, 16, 2))
    k = torch.zeros((1, 2, 4, 2, 64), dtype=torch.bfloat16)
    ok = (k, k, cache, i32(2), i32(2), i32(2))
    for args, kw in [((k[0], k[0]) + ok[2:], {}), ((k, k.float()) + ok[2:], {}), (ok, {}),     # no table: not one block per sequence
                     ((k, k, cache._replace(v_codes=t8(1, 9, 2, 16, 64))) + ok[3:], dict(block_table=i32(2, 4))),
                     ((k, k, cache._replace(k_scales=t8(1, 9, 2, 16, 4))) + ok[3:], dict(block_table=i32(2, 4))),
                     ((k, k, cache._replace(v_scales=i32(1, 9, 2, 16, 2))) + ok[3:], dict(block_table=i32(2, 4))),
                     (ok, dict(block_table=i32(3, 4))), (ok, dict(block_table=i32(2, 4).long())),
                     (ok[:3] + (i32(3),) + ok[4:], dict(block_table=i32(2, 4))), (ok[:4] + (i32(2).long(),) + ok[5:], dict(block_table=i32(2, 4)))]:
        with pytest.raises(ValueError):
            api.quantize_kv_q4(*args, **kw)
    with pytest.raises(api.EtvError):                   # a type that is neither
        api.quantize_kv_q4(k.half(), k.half(), *ok[2:], block_table=i32(2, 4))
    with pytest.raises(AssertionError):                 # good shapes: refused as host memory
        api.quantize_kv_q4(*ok, block_table=i32(2, 4))
    with pytest.raises(ValueError):
        api.commit_accepted_kv_q4(k, k, cache, i32(2), i32(2), i32(2), i32(3, 5), i32(2), block_table=i32(2, 4))
    with pytest.raises(ValueError):
        api.dequantize_kv_q4(cache, i32(2), i32(2), 4, block_table=i32(2, 4), out=dict(k=k[:, :, :3]))
    q, one, mask = torch.zeros((2, 4, 8, 64), dtype=torch.bfloat16), cache.layer(0), torch.zeros((2, 4, 1), dtype=torch.int64)
    good = dict(q=q, cache=one, prefix_len=i32(2), kt=k[0], vt=k[0], bitmask=mask, n_nodes=i32(2), P_max=20, block_table=i32(2, 4))
    for kw in (dict(q=q[0]), dict(kt=k[0].float()), dict(vt=k[0][:, :3]), dict(cache=cache), dict(bitmask=mask[:, :3]), dict(bitmask=mask.int()),
               dict(prefix_len=i32(1)), dict(block_table=None), dict(out=q.float()), dict(lse=torch.zeros((2, 4, 8))), dict(block_table=i32(2)),
               dict(desc=api.AttnDesc(B=2, T_max=5, Hq=8, Hkv=2, d=64, dtype=1))):
        with pytest.raises(ValueError):
            api.tree_verify_attention_q4(**{**good, **kw})
    with pytest.raises(AssertionError):
        api.tree_verify_attention_q4(**good)


def test_the_plain_format_is_what_the_header_says():
    """The oracle of the GPU tests, pinned by hand: one group worked out on paper."""
    x = np.zeros(64)
    x[:8] = [7, -3.5, 0.25, 0.26, -0.75, 5, 2.5, -0.0]         # 7 counts as 8: scale 2, so 3.5, -1.75, 0.125 ...
    x[32:36] = [6.9, 5, 1.25, -0.3]                            # scale 1: 6 (beyond), 4, 1, -0.5
    codes, scales = q4_plain.quantise(x)
    assert scales.tolist() == [128, 127]
    v = q4_plain.values(codes, scales)
    assert v[:8].tolist() == [8, -4, 0, 0, -1, 4, 2, 0] and v[32:36].tolist() == [6, 4, 1, -0.5]
    assert codes[0] == 0x6 | (0x8 | 0x4) << 4
    x[3] = np.inf
    codes, scales = q4_plain.quantise(x)
    assert scales[0] == 255 and not codes[:16].any() and np.isnan(q4_plain.values(codes, scales)[:32]).all()
