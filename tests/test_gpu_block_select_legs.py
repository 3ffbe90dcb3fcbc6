"""``la_block_select`` against the definition at sizes that reach every form of its two kernels: groups of few and of many rows,
several groups to a workgroup, candidates that a workgroup holds in registers and ones that it does not, ties and near ties in
each, and more (request, head) pairs than one dimension of a grid holds."""
import numpy as np
import pytest
import torch

import block_cache_util as U
from paper_2506_19830_amd import binding as B
from test_gpu_block_limits import near_ties
from test_gpu_block_select import inputs, run_select

pytestmark = pytest.mark.gpu

# prefix, gamma, L, Hq, Hkv, bs, group, most, first, last
GROUPS = [
    ((1700,), 1, 5, 8, 2, 16, 5, 9, 1, 1),                # 20 rows, 107 blocks
    ((2500, 90), 2, 14, 6, 2, 16, 11, 20, 0, 2),          # 33 rows, and 9 in the last group of a branch
    ((2100, 3300), 1, 47, 5, 1, 16, 33, 30, 1, 0),        # 165 rows, and 70
    ((1100,) * 4, 4, 31, 16, 8, 16, 9, 5, 1, 2),          # 18 rows; 16 groups to a request and head
    ((1300,), 1, 300, 2, 2, 16, 10, 7, 0, 0),             # 10 rows
]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("case", GROUPS, ids=lambda c: f"P{'-'.join(map(str, c[0]))}_g{c[1]}L{c[2]}_{c[3]}-{c[4]}_grp{c[6]}")
def test_groups_of_many_rows(case, D):
    prefix, gamma, L, Hq, Hkv, bs, group, most, first, last = case
    rng = np.random.default_rng(sum(prefix) + D)
    q, bounds = inputs(rng, prefix, gamma, L, Hq, Hkv, D, bs)
    run_select(q, bounds, list(prefix), Hkv, bs, group, most, first, last)


def test_several_groups_of_many_rows_to_a_workgroup():
    """64 (request, head) pairs: workgroups enough for the chip, which go through several groups each."""
    rng = np.random.default_rng(6)
    for D, L, group in ((128, 100, 5), (64, 90, 9)):       # 20 and 36 rows
        q, bounds = inputs(rng, [300] * 8, 3, L, 32, 8, D, 16)
        run_select(q, bounds, [300] * 8, 8, 16, group, 4, 0, 1)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("blocks,most,rows", [(2050, 100, 3), (2500, 1500, 20), (8192, 65, 1), (8193, 65, 1), (9000, 2000, 3)])
def test_many_blocks(D, blocks, most, rows):
    """More than four and more than sixteen wavefronts' registers hold."""
    rng = np.random.default_rng(blocks + D)
    prefix = [blocks * 16 - 5, 3000]
    q, bounds = inputs(rng, prefix, 1, 1, rows, 1, D, 16)
    run_select(q, bounds, prefix, 1, 16, 1, most, 1, 2)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("blocks", [3000, 9000])
def test_many_equal_scores(D, blocks):
    """Few different blocks many times over: thousands at the threshold, more than are listed, the lowest indices first."""
    rng = np.random.default_rng(blocks + D)
    for kinds in (1, 4):
        q, few = inputs(rng, [16 * kinds], 1, 2, 3, 1, D, 16)
        bounds = few[0][rng.integers(0, kinds, blocks)]
        run_select(q, [bounds], [blocks * 16], 1, 16, 2, 1500, 1, 1)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("rows,blocks", [(12, 600), (40, 600), (100, 700), (200, 2100), (12, 8500)])
def test_near_ties_of_groups_of_many_rows(D, rows, blocks):
    """Scores closer than fp32 can tell, with more than eight rows: in one part of the groups one row decides, in the others many
    rows are as good as the best."""
    rng = np.random.default_rng(rows + D)
    bounds = near_ties(rng, blocks, D)
    q = U.bf16(rng.standard_normal((1, 1, 2 * rows, 1, D)))
    same = U.bf16(rng.standard_normal(D))
    q[0, 0, rows:] = same
    q[0, 0, rows::3, :, 5] = U.bf16(same[5] * rng.choice([0.5, 1.0, 2.0, -1.0], (len(range(rows, 2 * rows, 3)), 1)))
    run_select(q, [bounds], [blocks * 16], 1, 16, rows, 50, 0, 1)


def test_a_channel_of_outliers():
    """One channel far from zero, as keys have them: the error of every rounded score is that of the large channel."""
    rng = np.random.default_rng(17)
    for D, L, Hq, group in ((128, 64, 5, 64), (64, 3, 4, 1), (256, 1, 8, 1)):
        q, bounds = inputs(rng, [32000], 1, L, Hq, 1, D, 16)
        bounds[0][..., 7] += 100.0
        run_select(q, [U.bf16(bounds[0])], [32000], 1, 16, group, 128, 1, 4)


def test_more_requests_and_heads_than_one_dimension_of_a_grid():
    """65600 (request, head) pairs over a pool that they share: unit 65535 and those behind it included."""
    n, H, D, N, pool = 8200, 8, 64, 3, 500
    g = torch.Generator(device="cuda").manual_seed(13)
    q = torch.randn((n, 1, 1, H, D), generator=g, device="cuda").to(torch.bfloat16)
    low = torch.randn((pool, H, 1, D), generator=g, device="cuda") - 1.0
    bounds = torch.cat((low, low + 1.0 + torch.rand(low.shape, generator=g, device="cuda")), 2).to(torch.bfloat16)
    table = torch.randint(0, pool, (n, N), generator=g, device="cuda").to(torch.int32)
    lens = torch.randint(1, 48 + 1, (n,), generator=g, device="cuda").to(torch.int32)
    d = U.desc("bf16", B_=n, Hq=H, Hkv=H, D=D, bs=16, max_blocks=N)
    s = B.make_select_desc(group_len=1, max_blocks=1)
    blocks, counts = torch.full((n, 1, 1, H, 1), -9, dtype=torch.int32, device="cuda"), torch.full((n, 1, 1, H), -9, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.la_block_select_workspace(d, s, lens.tolist()), dtype=torch.uint8, device="cuda")
    B.la_block_select(d, s, q, bounds, table, lens, lens.tolist(), blocks, counts, ws)
    x, b = q[:, 0, 0, None].double(), bounds[table.long()].double()                   # [n, 1, H, D], [n, N, H, 2, D]
    score = torch.where(x > 0, x * b[:, :, :, 1], x * b[:, :, :, 0]).sum(-1)          # [n, N, H]
    score = torch.where(torch.arange(N, device="cuda")[:, None] < ((lens.long() + 15) // 16)[:, None, None], score, -np.inf)
    want = score.cpu().numpy().argmax(1)                                              # (the first of equal ones)
    assert (counts == 1).all()
    assert np.array_equal(blocks[:, 0, 0, :, 0].cpu().numpy(), want)
