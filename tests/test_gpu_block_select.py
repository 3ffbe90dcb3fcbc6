"""``la_block_select`` against the definition in 64 bits: the lists are equal, index for index."""
import numpy as np
import pytest
import torch

import block_cache_util as U
from paper_2506_19830_amd import binding as B

pytestmark = pytest.mark.gpu


def run_select(q, bounds, prefix, Hkv, bs, group, most, first, last, paged=True, seed=0, poison=True):
    """q [B, gamma, L, Hq, D] and per request bounds [N, Hkv, 2, D], float64 holding bf16 numbers."""
    rng = np.random.default_rng(seed)
    n, gamma, L, Hq, D = q.shape
    max_blocks = max(1, -(-max(prefix) // bs))
    host, table, pool = U.tables(rng, n, max_blocks, paged)
    store = np.full((pool, Hkv, 2, D), np.nan if poison else 0.0)
    for b in range(n):
        have = -(-prefix[b] // bs)
        store[host[b, :have]] = bounds[b][:have]
    d = U.desc("bf16", B_=n, Hq=Hq, Hkv=Hkv, D=D, gamma=gamma, L=L, bs=bs, max_blocks=max_blocks)
    s = B.make_select_desc(group_len=group, max_blocks=most, keep_first=first, keep_last=last)
    groups = -(-L // group)
    blocks = torch.full((n, gamma, groups, Hkv, most), -9, dtype=torch.int32, device="cuda")
    counts = torch.full((n, gamma, groups, Hkv), -9, dtype=torch.int32, device="cuda")
    ws = torch.full((max(16, B.la_block_select_workspace(d, s, prefix)),), 255, dtype=torch.uint8, device="cuda")
    B.la_block_select(d, s, torch.from_numpy(q).to(torch.bfloat16).cuda(), torch.from_numpy(store).to(torch.bfloat16).cuda(),
                      table, U.i32(prefix), prefix, blocks, counts, ws)
    torch.cuda.synchronize()
    for b in range(n):
        want, want_n = U.ref_select(q[b], bounds[b], -(-prefix[b] // bs), group, most, first, last)
        assert np.array_equal(counts[b].cpu().numpy(), want_n)
        assert np.array_equal(blocks[b].cpu().numpy(), want), f"request {b}"


def inputs(rng, prefix, gamma, L, Hq, Hkv, D, bs, spread=0.3):
    q = U.bf16(rng.standard_normal((len(prefix), gamma, L, Hq, D)))
    bounds = []
    for p in prefix:
        c = rng.standard_normal((-(-p // bs), Hkv, D)) * 0.5
        w = 1.5 + spread * np.abs(rng.standard_normal((2,) + c.shape))
        bounds.append(U.bf16(np.stack((c - w[0], c + w[1]), 2)))
    return q, bounds


CASES = [
    # prefix, gamma, L, Hq, Hkv, D, bs, group, most, first, last
    ((700,), 1, 1, 5, 1, 128, 16, 1, 8, 1, 2),
    ((0, 1, 16, 17, 900), 1, 1, 4, 2, 64, 16, 1, 2, 0, 1),
    ((1000, 64), 2, 7, 6, 2, 128, 16, 3, 5, 1, 1),          # the last group of a branch has one token
    ((2100, 333), 3, 9, 14, 2, 64, 32, 9, 7, 0, 0),         # rows of a group: 63
    ((1300,), 2, 33, 16, 4, 256, 16, 16, 11, 2, 3),
    ((5000,), 1, 2, 16, 1, 64, 16, 1, 1, 0, 0),             # a single block
    ((5000,), 1, 2, 16, 1, 64, 16, 2, 1, 0, 1),             # the last one only: nothing to choose
    ((800, 801), 1, 1, 8, 8, 128, 16, 1, 49, 5, 40),        # all but one or two
    ((9000,), 1, 1, 3, 3, 256, 16, 1, 400, 1, 1),
    ((40000,), 1, 1, 2, 1, 64, 16, 1, 1500, 1, 1),          # 2500 blocks
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"P{'-'.join(map(str, c[0]))}_g{c[1]}L{c[2]}_D{c[5]}_most{c[8]}")
@pytest.mark.parametrize("paged", [True, False])
def test_select(case, paged):
    prefix, gamma, L, Hq, Hkv, D, bs, group, most, first, last = case
    rng = np.random.default_rng(sum(prefix) + most)
    q, bounds = inputs(rng, prefix, gamma, L, Hq, Hkv, D, bs)
    run_select(q, bounds, list(prefix), Hkv, bs, group, most, first, last, paged)


def test_equal_scores_go_to_the_lower_index():
    """Few different blocks, each many times over, and all blocks alike."""
    rng = np.random.default_rng(3)
    for kinds in (1, 2, 5):
        q = U.bf16(rng.standard_normal((1, 2, 3, 4, 64)))
        few = inputs(rng, [16 * kinds], 1, 1, 4, 2, 64, 16)[1][0]
        bounds = few[rng.integers(0, kinds, 1300)]
        run_select(q, [bounds], [1300 * 16 - 3], 2, 16, 2, 77, 1, 1)


def test_scores_closer_than_fp32_can_tell():
    """Blocks that differ in one channel by one bf16 step of a small number: the scores agree to far more digits than a sum
    in fp32 holds, and their order is that of the exact ones.  Channels of very different size, and a large common part."""
    rng = np.random.default_rng(8)
    for D in (64, 128, 256):
        n = 600
        q = U.bf16(rng.standard_normal((1, 1, 2, 4, D)))
        one = U.bf16(100.0 * rng.standard_normal((1, 1, D)))
        base = np.stack((one - 200.0, one + 200.0), 2)
        bounds = U.bf16(np.repeat(base, n, 0))
        small = int(rng.integers(0, D))
        bounds[:, 0, 0, small] = U.bf16(-2.0 ** -6 * (1 + rng.permutation(n) % 128 / 128.0))
        bounds[:, 0, 1, small] = U.bf16(2.0 ** -6 * (1 + rng.permutation(n) % 128 / 128.0))
        run_select(q, [bounds], [n * 16], 1, 16, 1, 50, 0, 0)
        run_select(q, [bounds], [n * 16], 1, 16, 2, 171, 1, 2)


def test_zeros_and_signs():
    """Queries of zeros (all scores equal), negative zeros, bounds of one sign, a group whose largest row is its last."""
    rng = np.random.default_rng(9)
    q, bounds = inputs(rng, [700], 1, 40, 4, 1, 64, 16)
    q[:, :, :39] *= 2.0 ** -20
    run_select(q, bounds, [700], 1, 16, 40, 9, 0, 1)
    run_select(np.zeros_like(q), bounds, [700], 1, 16, 7, 9, 2, 1)
    run_select(-np.zeros_like(q), bounds, [700], 1, 16, 7, 9, 2, 1)
    run_select(q, [np.abs(bounds[0]) + 1.0 - 1.0], [700], 1, 16, 7, 9, 2, 1)


def test_many_groups():
    """More groups than one dimension of a grid holds."""
    rng = np.random.default_rng(10)
    q, bounds = inputs(rng, [80], 1, 9000, 8, 8, 64, 16)
    run_select(q, bounds, [80], 8, 16, 1, 3, 0, 1)
