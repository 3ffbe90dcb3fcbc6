"""Every kernel shape of ``la_verify_attention_sparse`` against the definition in 64 bits, on the same small calls: the shapes and
the splits are forced through a hook of the benchmark library, whose kernels are the product's."""
import numpy as np
import pytest
import torch

import block_cache_util as U
from paper_2506_19830_amd import binding as B
from test_gpu_attn_blocks import random_lists

pytestmark = pytest.mark.gpu

# (rows, wavefronts) of a workgroup
SHAPES = {64: [(16, 4), (16, 8), (32, 4), (32, 8), (64, 4), (96, 6), (128, 8)], 256: [(16, 4), (32, 4), (128, 4)]}
SHAPES[128] = SHAPES[64]


@pytest.fixture
def bench_library():
    B.select_library("bench")
    try:
        yield
    finally:
        B.la_selftest_sparse_plan()
        B.select_library("product")


class Call:
    """Inputs of a call and what the definition gives for them."""

    def __init__(self, seed, fmt, prefix, gamma, L, Hq, Hkv, D, bs, group, most, listed, out):
        rng = np.random.default_rng(seed)
        n, self.prefix, self.D, self.out_dtype = len(prefix), list(prefix), D, out
        max_blocks = -(-max(prefix) // bs) + 1
        self.c = U.Cache(rng, fmt, prefix, Hkv, D, bs, max_blocks)
        q = U.bf16(rng.standard_normal((n, gamma, L, Hq, D)))
        kb, vb = (U.bf16(rng.standard_normal((n, gamma, L, Hkv, D))) for _ in "kv")
        self.desc = U.desc(fmt, B_=n, Hq=Hq, Hkv=Hkv, D=D, gamma=gamma, L=L, bs=bs, max_blocks=max_blocks, out=out)
        self.sel = self.blocks = self.counts = lists = None
        if listed:
            groups = -(-L // group)
            lists = random_lists(rng, prefix, gamma, groups, Hkv, bs, most)
            self.sel = B.make_select_desc(group_len=group, max_blocks=most)
            host, num = np.full((n, gamma, groups, Hkv, most), -1, dtype=np.int32), np.zeros((n, gamma, groups, Hkv), dtype=np.int32)
            for at in np.ndindex(*num.shape):
                x = lists[at[0]][at[1]][at[2]][at[3]]
                host[at][:len(x)], num[at] = x, len(x)
            self.blocks, self.counts = torch.from_numpy(host).cuda(), torch.from_numpy(num).cuda()
        self.q, self.kb, self.vb = (torch.from_numpy(x).to(torch.bfloat16).cuda() for x in (q, kb, vb))
        self.ref = [U.ref_attend(q[b], self.c.k[b], self.c.v[b], kb[b], vb[b], None if lists is None else lists[b], bs, group,
                                 np.float64(np.float32(D ** -0.5))) for b in range(n)]

    def run(self):
        need = B.la_verify_attention_sparse_workspace(self.desc, self.sel, self.prefix)
        ws = torch.full((max(16, need),), 255, dtype=torch.uint8, device="cuda")
        out = torch.full(self.q.shape, float("nan"), dtype=torch.bfloat16 if self.out_dtype == "bf16" else torch.float32, device="cuda")
        lse = torch.full(self.q.shape[:-1], float("nan"), device="cuda")
        B.la_verify_attention_sparse(self.desc, self.sel, self.q, self.c.desc, self.c.table, self.c.lens, self.prefix, self.blocks, self.counts,
                                     self.kb, self.vb, out, lse, ws)
        torch.cuda.synchronize()
        for b, ref in enumerate(self.ref):
            U.check_attend(out[b].double().cpu().numpy(), lse[b].double().cpu().numpy(), ref, self.D, self.out_dtype)
        return need


# prefix, gamma, L, Hq, Hkv, bs, group, most
CALLS = [
    ((700, 33, 0), 2, 70, 6, 2, 16, 33, 30),      # 99 rows, and 12 in a branch's last group
    ((420, 97), 3, 3, 10, 2, 32, 3, 9),           # 15 rows; without lists 45, of three branches
]


@pytest.mark.parametrize("fmt", U.FORMATS)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("listed", [True, False], ids=["lists", "whole"])
@pytest.mark.parametrize("call", CALLS, ids=["steps", "tokens"])
def test_every_shape(bench_library, call, listed, D, fmt):
    prefix, gamma, L, Hq, Hkv, bs, group, most = call
    c = Call(D + len(prefix), fmt, prefix, gamma, L, Hq, Hkv, D, bs, group, most, listed, "f32" if listed else "bf16")
    for rows, waves in SHAPES[D]:
        for split in (1, 3, 11):
            B.la_selftest_sparse_plan(rows, waves, split)
            need = c.run()
            assert (need == 0) == (split == 1), f"{rows} rows, {waves} wavefronts, split {split}"


def test_more_workgroups_than_tiles(bench_library):
    """Most of a unit's workgroups have nothing to do; more than the merge takes at a time."""
    c = Call(3, "mxfp8_e4m3", (300, 0), 2, 40, 4, 2, 128, 16, 40, 9, True, "bf16")
    for rows, waves in SHAPES[128]:
        B.la_selftest_sparse_plan(rows, waves, 70)
        c.run()
