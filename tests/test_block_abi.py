"""The block cache calls without a GPU: what they refuse (before anything is launched), what they ask for as workspace, and
the formats' definition in the tests' own plain form."""
import ctypes

import numpy as np
import pytest
import torch

import block_cache_util as U
from paper_2506_19830_amd import binding as B

OK, INVALID, UNSUPPORTED, SMALL = 0, 1, 2, 3
P = 1 << 20   # an address that is aligned and never followed


def status(fn, *args):
    return getattr(B.load(), fn)(*args)


def cache(**kw):
    f = dict(k=P, v=P, k_exp=P, v_exp=P, k_bounds=P, exp_stride=0, bounds_stride=0)
    f.update(kw)
    return B.la_block_cache(*f.values())


def lens(*x):
    return (ctypes.c_int32 * len(x))(*x)


BAD_DESCS = [
    (dict(B_=0), INVALID), (dict(Hq=5, Hkv=2), INVALID), (dict(gamma=0), INVALID), (dict(L=0), INVALID), (dict(bs=8), INVALID),
    (dict(bs=48), INVALID), (dict(max_blocks=-1), INVALID), (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(D=32), UNSUPPORTED), (dict(D=96), UNSUPPORTED), (dict(max_blocks=1 << 27), UNSUPPORTED),
    (dict(gamma=1 << 15, L=1 << 15, Hq=8), UNSUPPORTED),
]


def calls(d, **kw):
    """Status of every call for a descriptor (none may get as far as a launch)."""
    a = dict(cache=cache(), sel=B.make_select_desc(group_len=1, max_blocks=2), lens=lens(10), ws=0)
    a.update(kw)
    dp, cp, sp = ctypes.byref(d), ctypes.byref(a["cache"]), ctypes.byref(a["sel"])
    n = ctypes.c_size_t()
    return {
        "store": status("la_kv_store", dp, cp, None, P, a["lens"], P, P, None, None, -1, None, None, None, 2 * P, None, None),
        "load": status("la_kv_load", dp, cp, None, P, None, 0, P, P, None, None),
        "select_ws": status("la_block_select_workspace", dp, sp, a["lens"], ctypes.byref(n)),
        "select": status("la_block_select", dp, sp, P, P, None, P, a["lens"], P, None, None, 0, None),
        "sparse_ws": status("la_verify_attention_sparse_workspace", dp, sp, a["lens"], ctypes.byref(n)),
        "sparse": status("la_verify_attention_sparse", dp, sp, P, cp, None, P, a["lens"], P, None, P, P, P, None, None, 0, None),
    }


@pytest.mark.parametrize("kw,want", BAD_DESCS)
def test_bad_descriptors(kw, want):
    for name, st in calls(U.desc("bf16", **kw)).items():
        assert st == want, name


def test_types():
    """Only the block cache's formats, bf16 queries and branches, bf16 or fp32 results; no forced split or shape."""
    for field, value, want in (("kv_dtype", B.LA_F32, UNSUPPORTED), ("kv_dtype", B.LA_FP8_E4M3, UNSUPPORTED), ("kv_dtype", 5, INVALID),
                               ("kv_dtype", -1, INVALID), ("q_dtype", B.LA_F32, UNSUPPORTED), ("q_dtype", 9, INVALID),
                               ("branch_kv_dtype", B.LA_MXFP8_E4M3, UNSUPPORTED), ("out_dtype", B.LA_FP8_E4M3, UNSUPPORTED),
                               ("kv_split_tokens", 64, INVALID), ("kernel_shape", 1, INVALID)):
        d = U.desc("mxfp8_e4m3")
        setattr(d, field, value)
        for name, st in calls(d).items():
            assert st == want, (field, value, name)
    # the other calls of the library do not take the block cache's formats
    for code in (B.LA_MXFP8_E4M3, B.LA_MXFP4_E2M1):
        d = U.desc("bf16", D=128)
        d.kv_dtype = code
        with pytest.raises(B.LaError) as err:
            B.la_verify_attention_workspace(d, [10])
        assert err.value.status == INVALID


def test_store_refuses():
    def call(fmt="mxfp4_e2m1", c=None, table=None, pl=P, host=lens(100, 3), kb=P, vb=P, kc=P, vc=P, C=7, new=2 * P, layers=None, **kw):
        d = U.desc(fmt, **dict(dict(B_=2, L=5, bs=16, max_blocks=7), **kw))
        return status("la_kv_store", ctypes.byref(d), None if c is False else ctypes.byref(c or cache()), table, pl, host, kb, vb, kc, vc,
                      C, None, None, None, new, None if layers is None else ctypes.byref(layers), None)
    full = lens(101, 3)                                        # 101 + 7 + 5 positions, 112 are mapped
    for kw in (dict(c=False), dict(c=cache(k=None)), dict(c=cache(v=None)), dict(c=cache(k_exp=None)), dict(c=cache(v_exp=None)),
               dict(c=cache(k=P + 8)), dict(c=cache(k_exp=P + 4)), dict(c=cache(k_bounds=P + 2)), dict(pl=None), dict(host=None),
               dict(kb=None), dict(vb=None), dict(kc=None), dict(vc=None), dict(C=-1), dict(new=None), dict(new=P), dict(kb=P + 8),
               dict(kc=P + 2), dict(host=full), dict(host=lens(-1, 0)),
               dict(layers=B.la_layer_strides(0, 0, 0, 0, 0)), dict(layers=B.la_layer_strides(65536, 0, 0, 0, 0)),
               dict(layers=B.la_layer_strides(2, 16, 0, 0, 0)),       # half a group
               dict(layers=B.la_layer_strides(2, -32, 0, 0, 0)), dict(layers=B.la_layer_strides(2, 64, 4, 0, 0)),
               dict(layers=B.la_layer_strides(2, 64, 64, 4, 0)),
               dict(layers=B.la_layer_strides(2, 64, 64, 64, 0), c=cache(exp_stride=8)),
               dict(layers=B.la_layer_strides(2, 64, 64, 64, 0), c=cache(bounds_stride=4))):
        assert call(**kw) == INVALID, kw
    assert call("bf16", c=cache(k_exp=None, v_exp=None), new=None) == INVALID


def test_load_refuses():
    def call(c=None, pl=P, n=4, k=P, v=P, layers=None, fmt="mxfp8_e4m3", **kw):
        d = U.desc(fmt, **kw)
        return status("la_kv_load", ctypes.byref(d), None if c is False else ctypes.byref(c or cache()), None, pl, None, n, k, v,
                      None if layers is None else ctypes.byref(layers), None)
    for kw in (dict(c=False), dict(c=cache(k=None)), dict(c=cache(v_exp=None)), dict(pl=None), dict(n=0), dict(n=-3), dict(k=None),
               dict(v=None), dict(k=P + 8), dict(layers=B.la_layer_strides(2, 64, 4, 0, 0))):
        assert call(**kw) == INVALID, kw
    assert call(n=2 ** 31 - 1, Hq=8, Hkv=8) == UNSUPPORTED


def test_select_refuses():
    d = U.desc("bf16", B_=2, L=5, bs=16, max_blocks=64)
    good = dict(group_len=2, max_blocks=4, keep_first=1, keep_last=1)

    def call(d=d, q=P, kb=P, pl=P, host=lens(900, 3), blocks=P, counts=P, ws=P, n=1 << 20, **kw):
        s = B.make_select_desc(**dict(good, **kw))
        return status("la_block_select", ctypes.byref(d), ctypes.byref(s), q, kb, None, pl, host, blocks, counts, ws, n, None)
    for kw in (dict(group_len=0), dict(group_len=6), dict(max_blocks=0), dict(keep_first=-1), dict(keep_last=-1),
               dict(keep_first=3, keep_last=2), dict(q=None), dict(kb=None), dict(pl=None), dict(host=None), dict(host=lens(1025, 0)),
               dict(host=lens(3, -1)), dict(blocks=None), dict(counts=None), dict(q=P + 8), dict(kb=P + 8), dict(ws=P + 8)):
        assert call(**kw) == INVALID, kw
    assert status("la_block_select", ctypes.byref(d), None, P, P, None, P, lens(900, 3), P, P, P, 1 << 20, None) == INVALID
    assert call(max_blocks=1 << 27) == UNSUPPORTED
    need = B.la_block_select_workspace(d, B.make_select_desc(**good), [900, 3])
    assert need > 0 and call(n=need - 1) == SMALL and call(ws=None) == SMALL
    assert B.la_block_select_workspace(d, B.make_select_desc(**dict(good, max_blocks=57)), [900, 3]) == 0    # nothing to choose
    with pytest.raises(B.LaError):
        B.la_block_select_workspace(d, None, [900, 3])
    many = U.desc("bf16", B_=1 << 12, L=1 << 10, Hq=8, Hkv=8, bs=16, max_blocks=1)
    with pytest.raises(B.LaError) as err:
        B.la_block_select_workspace(many, B.make_select_desc(group_len=1, max_blocks=1), [0] * (1 << 12))
    assert err.value.status == UNSUPPORTED


def test_sparse_refuses():
    d = U.desc("mxfp4_e2m1", B_=2, L=5, bs=16, max_blocks=64)
    s = B.make_select_desc(group_len=2, max_blocks=4)

    def call(sel=s, q=P, c=None, pl=P, host=lens(900, 3), blocks=P, counts=P, kb=P, vb=P, out=P, ws=P, n=1 << 30):
        return status("la_verify_attention_sparse", ctypes.byref(d), None if sel is None else ctypes.byref(sel), q,
                      None if c is False else ctypes.byref(c or cache()), None, pl, host, blocks, counts, kb, vb, out, None, ws, n, None)
    for kw in (dict(sel=None), dict(blocks=None), dict(counts=None), dict(sel=None, blocks=None), dict(q=None), dict(c=False),
               dict(c=cache(k=None)), dict(c=cache(k_exp=None)), dict(c=cache(v=P + 8)), dict(pl=None), dict(host=None),
               dict(host=lens(1025, 0)), dict(kb=None), dict(vb=None), dict(out=None), dict(q=P + 8), dict(out=P + 8), dict(ws=P + 8),
               dict(sel=B.make_select_desc(group_len=6, max_blocks=4)), dict(sel=B.make_select_desc(group_len=1, max_blocks=0))):
        assert call(**kw) == INVALID, kw
    long = U.desc("mxfp4_e2m1", L=1, bs=16, max_blocks=4096)
    need = B.la_verify_attention_sparse_workspace(long, None, [60000])
    assert need > 0
    st = status("la_verify_attention_sparse", ctypes.byref(long), None, P, ctypes.byref(cache()), None, P, lens(60000), None, None, P, P, P,
                None, P, need - 1, None)
    assert st == SMALL


def test_struct_layouts():
    assert ctypes.sizeof(B.la_block_cache) == 7 * 8 and ctypes.sizeof(B.la_select_desc) == 4 * 4


def test_make_block_cache():
    k = torch.zeros((2, 3, 4, 16, 64), dtype=torch.bfloat16)
    e = torch.zeros((2, 3, 4, 16, 2), dtype=torch.uint8)
    c = B.make_block_cache(k, k, e, e, torch.zeros((2, 3, 4, 2, 64), dtype=torch.bfloat16))
    assert (c.exp_stride, c.bounds_stride, c.k) == (3 * 4 * 32, 3 * 4 * 128, k.data_ptr())
    assert B.make_block_cache(k[0], k[0]).exp_stride == 0
    with pytest.raises(ValueError):
        B.make_block_cache(k.transpose(0, 1), k)


def test_the_formats_definition():
    """The plain quantiser on numbers worked out by hand."""
    x = np.zeros((1, 64))
    x[0, :8] = [6.0, -5.0, 2.5, 3.5, 0.25, -0.25, 0.75, 1.25]
    x[0, 32] = 7.0                                               # above 6: the group's power is 2, 7 / 2 = 3.5 goes to 4
    code, exps, values = U.quantise(x, "mxfp4_e2m1")
    assert exps.tolist() == [[0, 1]]
    assert values[0, :8].tolist() == [6.0, -4.0, 2.0, 4.0, 0.0, 0.0, 1.0, 1.0] and values[0, 32] == 8.0
    assert code[0, :8].tolist() == [7, 14, 4, 6, 0, 8, 2, 2]
    x[0, :2], x[0, 2:] = [448.0, 2.0 ** -10], 0.0
    x[0, 32:34] = [449.0, -17.0]
    code, exps, values = U.quantise(x, "mxfp8_e4m3")
    assert exps.tolist() == [[0, 1]] and code[0, :3].tolist() == [126, 0, 0]
    assert values[0, 32] == 448.0 and values[0, 33] == -16.0     # codes there are 16 and 1 apart: 224.5, 8.5 go to 224, 8
    assert U.quantise(np.zeros((1, 32)), "mxfp8_e4m3")[1].tolist() == [[-100]]
