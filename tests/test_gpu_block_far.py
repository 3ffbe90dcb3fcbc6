"""A block cache whose rows, exponents and bounds lie more than 2^32 bytes behind their bases: every call gives to the bit what it gives
on a small cache, and the last block of the pool is as good as any."""
import numpy as np
import pytest
import torch

import block_cache_util as U
from paper_2506_19830_amd import binding as B

pytestmark = pytest.mark.gpu

D, BS, POOL = 128, 16, (1 << 23) + 64      # 2^32 bytes of bounds and up to 2^35 of rows lie below block 2^23


def results(fmt, pool, table):
    g = torch.Generator().manual_seed(5)
    rand = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).cuda()
    P, gamma, L, Hq, most = 37 * BS - 3, 2, 40, 4, 9
    dtype, width = {"bf16": (torch.bfloat16, D), "mxfp8_e4m3": (torch.float8_e4m3fn, D), "mxfp4_e2m1": (torch.uint8, D // 2)}[fmt]
    el = [torch.empty((pool, 1, BS, width), dtype=dtype, device="cuda") for _ in "kv"]
    ex = [None if fmt == "bf16" else torch.empty((pool, 1, BS, D // 32), dtype=torch.uint8, device="cuda") for _ in "kv"]
    bounds = torch.empty((pool, 1, 2, D), dtype=torch.bfloat16, device="cuda")
    cache = B.make_block_cache(*el, *ex, bounds)
    table = U.i32([table])
    kw = dict(Hq=Hq, Hkv=1, D=D, bs=BS, max_blocks=table.shape[1])
    lens = U.i32([0])
    kv = [rand(1, 1, P, 1, D) for _ in "kv"]
    B.la_kv_store(U.desc(fmt, L=P, **kw), cache, table, U.i32([0]), [0], *kv, None, None, None, None, None, lens)
    back = [torch.zeros((1, P, 1, D), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    B.la_kv_load(U.desc(fmt, **kw), cache, table, lens, None, *back)
    res = [lens, *back]
    q, kb, vb = rand(1, gamma, L, Hq, D), rand(1, gamma, L, 1, D), rand(1, gamma, L, 1, D)
    d = U.desc(fmt, gamma=gamma, L=L, **kw)
    for group in (1, 6, L):                    # few rows, up to 32, many
        sel = B.make_select_desc(group_len=group, max_blocks=most, keep_first=1, keep_last=1)
        shape = (1, gamma, -(-L // group), 1)
        blocks, counts = torch.zeros(shape + (most,), dtype=torch.int32, device="cuda"), torch.zeros(shape, dtype=torch.int32, device="cuda")
        ws = [torch.empty(max(16, n), dtype=torch.uint8, device="cuda") for n in (
            B.la_block_select_workspace(d, sel, [P]), B.la_verify_attention_sparse_workspace(d, sel, [P]))]
        out, lse = torch.zeros_like(q), torch.zeros(q.shape[:-1], device="cuda")
        B.la_block_select(d, sel, q, bounds, table, lens, [P], blocks, counts, ws[0])
        B.la_verify_attention_sparse(d, sel, q, cache, table, lens, [P], blocks, counts, kb, vb, out, lse, ws[1])
        res += [blocks, counts, out, lse]
    ws = torch.empty(max(16, B.la_verify_attention_sparse_workspace(d, None, [P])), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:-1], device="cuda")
    B.la_verify_attention_sparse(d, None, q, cache, table, lens, [P], None, None, kb, vb, out, lse, ws)
    res += [out, lse]
    return [U.raw(t) if t.dtype == torch.bfloat16 else t.cpu() for t in res]


@pytest.mark.parametrize("fmt", U.FORMATS)
def test_far_blocks(fmt):
    order = np.concatenate(([63], np.random.default_rng(3).permutation(63)[:39]))
    near = results(fmt, 64, order.tolist())
    far = results(fmt, POOL, (POOL - 64 + order).tolist())
    assert int(near[0]) == 37 * BS - 3
    for a, b in zip(near, far):
        assert torch.equal(a, b)
