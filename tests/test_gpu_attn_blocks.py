"""``la_verify_attention_sparse`` against the definition in 64 bits, with bounds counted from its roundings."""
import numpy as np
import pytest
import torch

import block_cache_util as U
from paper_2506_19830_amd import binding as B

pytestmark = pytest.mark.gpu


def random_lists(rng, prefix, gamma, groups, Hkv, bs, most):
    """[B][gamma][groups][Hkv] ascending distinct blocks: full lists, short ones and empty ones, with and without the last."""
    out = []
    for p in prefix:
        have = -(-p // bs)
        out.append([[[np.sort(rng.permutation(have)[:rng.integers(0, min(have, most) + 1) if rng.random() < 0.5 else min(have, most)])
                      for _ in range(Hkv)] for _ in range(groups)] for _ in range(gamma)])
    return out


def run_attend(rng, fmt, prefix, gamma, L, Hq, Hkv, D, bs, group, most, out="bf16", paged=True, lists="random", scale=None,
               size=1.0, want_lse=True, spare=1):
    n = len(prefix)
    max_blocks = -(-max(prefix) // bs) + spare
    c = U.Cache(rng, fmt, prefix, Hkv, D, bs, max_blocks, paged)
    q = U.bf16(size * rng.standard_normal((n, gamma, L, Hq, D)))
    kb, vb = (U.bf16(rng.standard_normal((n, gamma, L, Hkv, D))) for _ in "kv")
    d = U.desc(fmt, B_=n, Hq=Hq, Hkv=Hkv, D=D, gamma=gamma, L=L, bs=bs, max_blocks=max_blocks, out=out, scale=scale)
    groups, s, blocks, counts = -(-L // group), None, None, None
    if lists is not None:
        lists = random_lists(rng, prefix, gamma, groups, Hkv, bs, most) if isinstance(lists, str) else lists
        s = B.make_select_desc(group_len=group, max_blocks=most)
        host = np.full((n, gamma, groups, Hkv, most), -1, dtype=np.int32)
        num = np.zeros((n, gamma, groups, Hkv), dtype=np.int32)
        for at in np.ndindex(*num.shape):
            x = lists[at[0]][at[1]][at[2]][at[3]]
            host[at][:len(x)], num[at] = x, len(x)
        blocks, counts = torch.from_numpy(host).cuda(), torch.from_numpy(num).cuda()
    up = lambda x: torch.from_numpy(x).to(torch.bfloat16).cuda()  # noqa: E731
    o = torch.full((n, gamma, L, Hq, D), float("nan"), dtype=torch.bfloat16 if out == "bf16" else torch.float32, device="cuda")
    lse = torch.full((n, gamma, L, Hq), float("nan"), device="cuda") if want_lse else None
    ws = torch.full((max(16, B.la_verify_attention_sparse_workspace(d, s, list(prefix))),), 255, dtype=torch.uint8, device="cuda")
    B.la_verify_attention_sparse(d, s, up(q), c.desc, c.table, c.lens, list(prefix), blocks, counts, up(kb), up(vb), o, lse, ws)
    torch.cuda.synchronize()
    worst = 0.0
    for b in range(n):
        ref = U.ref_attend(q[b], c.k[b], c.v[b], kb[b], vb[b], None if lists is None else lists[b], bs, group,
                           np.float64(np.float32(D ** -0.5 if scale is None else scale)))
        worst = max(worst, U.check_attend(o[b].double().cpu().numpy(), None if lse is None else lse[b].double().cpu().numpy(),
                                          ref, D, out))
    return worst


SHAPES = [
    # prefix, gamma, L, Hq, Hkv, D, bs, group, most
    ((0,), 1, 1, 1, 1, 64, 16, 1, 1),                        # no prefix: a token sees itself
    ((1, 15, 16, 17), 1, 1, 5, 1, 128, 16, 1, 2),
    ((31, 33, 64, 65), 2, 3, 6, 2, 64, 32, 1, 3),
    ((300, 7), 2, 9, 10, 2, 128, 16, 4, 6),                  # the last group of a branch has one token
    ((500,), 3, 21, 8, 2, 128, 64, 21, 4),                   # 84 rows: tiles of 64
    ((500, 129), 1, 40, 7, 1, 64, 128, 13, 3),               # 91 rows
    ((260,), 2, 35, 3, 3, 256, 16, 35, 9),                   # own tokens over two tiles
    ((90, 0, 200), 2, 2, 32, 2, 256, 32, 2, 3),              # 32 rows
    ((1500,), 1, 1, 16, 1, 128, 16, 1, 90),                  # split over workgroups
    ((1111, 40), 4, 1, 8, 1, 64, 64, 1, 17),
]


@pytest.mark.parametrize("fmt", U.FORMATS)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda c: f"P{'-'.join(map(str, c[0]))}_g{c[1]}L{c[2]}_{c[3]}-{c[4]}_D{c[5]}_bs{c[6]}_grp{c[7]}")
def test_listed_blocks(fmt, shape):
    run_attend(np.random.default_rng(sum(shape[0]) + shape[2]), fmt, *shape)


@pytest.mark.parametrize("fmt", U.FORMATS)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda c: f"P{'-'.join(map(str, c[0]))}_g{c[1]}L{c[2]}_{c[3]}-{c[4]}_D{c[5]}_bs{c[6]}")
def test_whole_prefix(fmt, shape):
    """No lists: the rows of all branches share their tiles."""
    run_attend(np.random.default_rng(sum(shape[0]) + 77), fmt, *shape, lists=None)


@pytest.mark.parametrize("fmt", U.FORMATS)
def test_forms_of_the_call(fmt):
    """fp32 results, no lse, blocks in order without a table, another scale, large scores."""
    rng = np.random.default_rng(6)
    run_attend(rng, fmt, (200, 33), 2, 5, 8, 2, 128, 16, 5, 6, out="f32")
    run_attend(rng, fmt, (200, 33), 2, 5, 8, 2, 64, 16, 5, 6, want_lse=False, paged=False)
    run_attend(rng, fmt, (200,), 1, 3, 4, 2, 64, 32, 2, 4, scale=1.0)
    run_attend(rng, fmt, (900,), 1, 2, 4, 2, 128, 32, 2, 20, size=12.0, out="f32")
    run_attend(rng, fmt, (900,), 1, 2, 4, 2, 128, 32, 2, 20, lists=None, size=12.0)
    run_attend(rng, fmt, (64, 128), 1, 2, 4, 2, 128, 32, 2, 4, lists=None, spare=0)


def test_every_list_empty():
    rng = np.random.default_rng(1)
    empty = [[[[[] for _ in range(2)] for _ in range(3)] for _ in range(2)] for _ in range(2)]
    for fmt in U.FORMATS:
        run_attend(rng, fmt, (100, 0), 2, 7, 4, 2, 64, 16, 3, 5, lists=empty)


@pytest.mark.parametrize("fmt", U.FORMATS)
def test_long_lists_and_prefixes(fmt):
    """More blocks than a workgroup's table holds, in lists and without."""
    rng = np.random.default_rng(2)
    lists = [[[[np.sort(rng.permutation(5000)[:4500])]]]]
    run_attend(rng, fmt, (79995,), 1, 1, 2, 1, 64, 16, 1, 4500, lists=lists)
    run_attend(rng, fmt, (79995,), 2, 1, 2, 1, 64, 16, 1, 1, lists=None)


def test_counts_and_ids_outside_their_ranges():
    """Counts beyond the list's length and ids beyond the prefix are clamped: the call stays inside the prefix's blocks."""
    rng = np.random.default_rng(12)
    c = U.Cache(rng, "mxfp4_e2m1", [40], 1, 64, 16, 3)
    d = U.desc("mxfp4_e2m1", Hq=1, Hkv=1, D=64, bs=16, max_blocks=3)
    s = B.make_select_desc(group_len=1, max_blocks=2)
    q = torch.randn((1, 1, 1, 1, 64), device="cuda").to(torch.bfloat16)
    kb = torch.randn((1, 1, 1, 1, 64), device="cuda").to(torch.bfloat16)
    ws = torch.empty(max(16, B.la_verify_attention_sparse_workspace(d, s, [40])), dtype=torch.uint8, device="cuda")

    def call(ids, n):
        o = torch.empty((1, 1, 1, 1, 64), dtype=torch.bfloat16, device="cuda")
        B.la_verify_attention_sparse(d, s, q, c.desc, c.table, c.lens, [40], U.i32([[[[ids]]]]), U.i32([[[[n]]]]), kb, kb, o, None, ws)
        return o
    assert torch.equal(call([1, 2], 7), call([1, 2], 2))
    assert torch.equal(call([1, 99], 2), call([1, 2], 2))
    assert torch.equal(call([-5, 1], 2), call([0, 1], 2))
    assert torch.equal(call([1, 2], -3), call([1, 2], 0))


def test_results_repeat():
    rng = np.random.default_rng(14)
    c = U.Cache(rng, "mxfp8_e4m3", [1900], 2, 128, 16, 120)
    d = U.desc("mxfp8_e4m3", Hq=8, Hkv=2, D=128, gamma=2, L=2, bs=16, max_blocks=120)
    q = torch.randn((1, 2, 2, 8, 128), device="cuda").to(torch.bfloat16)
    kb = torch.randn((1, 2, 2, 2, 128), device="cuda").to(torch.bfloat16)
    ws = torch.empty(max(16, B.la_verify_attention_sparse_workspace(d, None, [1900])), dtype=torch.uint8, device="cuda")
    outs = []
    for _ in range(4):
        o = torch.empty_like(q)
        B.la_verify_attention_sparse(d, None, q, c.desc, c.table, c.lens, [1900], None, None, kb, kb, o, None, ws)
        outs.append(o)
    assert all(torch.equal(o, outs[0]) for o in outs)
