"""The block cache's calls at sizes where an index, a count or a sum could leave its type."""
import numpy as np
import pytest
import torch

import block_cache_util as U
from paper_2506_19830_amd import binding as B
from test_gpu_block_select import run_select

pytestmark = pytest.mark.gpu


def near_ties(rng, n, D):
    """Bounds [n, 1, 2, D] whose scores a sum in fp32 cannot tell apart: a large common part, and a small channel that differs."""
    one = U.bf16(100.0 * rng.standard_normal((1, 1, D)))
    bounds = U.bf16(np.repeat(np.stack((one - 200.0, one + 200.0), 2), n, 0))
    for which, sign in ((0, -1.0), (1, 1.0)):
        bounds[:, 0, which, 5] = U.bf16(sign * 2.0 ** -6 * (1 + rng.permutation(n) % 128 / 128.0))
    return bounds


def test_select_with_more_than_four_million_rows_to_a_group():
    """The row that decides lies 2^22 rows behind the group's first; the row with its number less 2^22 has another sign and would
    order the blocks otherwise."""
    rng = np.random.default_rng(31)
    G, D, n, most = 8, 64, 40, 9
    L = (1 << 19) + 40                                        # 2^22 + 320 rows
    bounds = near_ties(rng, n, D)
    row = U.bf16(rng.standard_normal((1, 1, 1, D)))
    q = torch.zeros((1, 1, L, G, D), dtype=torch.bfloat16, device="cuda")
    at = (1 << 22) + 77
    q[0, 0, at // G, at % G] = torch.from_numpy(row.ravel()).to(torch.bfloat16).cuda()
    q[0, 0, 77 // G, 77 % G] = torch.from_numpy(-0.5 * row.ravel()).to(torch.bfloat16).cuda()
    d = U.desc("bf16", Hq=G, Hkv=1, D=D, L=L, bs=16, max_blocks=n)
    s = B.make_select_desc(group_len=L, max_blocks=most)
    blocks = torch.full((1, 1, 1, 1, most), -9, dtype=torch.int32, device="cuda")
    counts = torch.full((1, 1, 1, 1), -9, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.la_block_select_workspace(d, s, [16 * n]), dtype=torch.uint8, device="cuda")
    B.la_block_select(d, s, q, torch.from_numpy(bounds).to(torch.bfloat16).cuda(), None, U.i32([16 * n]), [16 * n], blocks, counts, ws)
    # (the rows of zeros score nothing, below the two others)
    want = U.ref_select(np.concatenate((row, -0.5 * row), 2), bounds, n, 1, most, 0, 0)[0]
    assert U.ref_select(-0.5 * row, bounds, n, 1, most, 0, 0)[0].tolist() != want.tolist()
    assert counts.item() == most
    assert blocks.cpu().numpy().ravel().tolist() == want.ravel().tolist()


def test_attention_of_two_to_the_23_groups():
    """As many workgroups as a launch may have, a row each: eight wavefronts to a workgroup would be 2^32 threads."""
    gamma, H, D, bs, P = 1 << 20, 8, 64, 16, 13
    g = torch.Generator(device="cuda").manual_seed(11)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    k, v = rand(1, H, bs, D), rand(1, H, bs, D)
    q, kb, vb = rand(1, gamma, 1, H, D), rand(1, gamma, 1, H, D), rand(1, gamma, 1, H, D)
    d = U.desc("bf16", Hq=H, Hkv=H, D=D, gamma=gamma, L=1, bs=bs, max_blocks=1)
    s = B.make_select_desc(group_len=1, max_blocks=1)
    blocks = torch.zeros((1, gamma, 1, H, 1), dtype=torch.int32, device="cuda")
    counts = torch.ones((1, gamma, 1, H), dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:-1], float("nan"), device="cuda")
    ws = torch.empty(max(16, B.la_verify_attention_sparse_workspace(d, s, [P])), dtype=torch.uint8, device="cuda")
    B.la_verify_attention_sparse(d, s, q, B.make_block_cache(k, v), None, U.i32([P]), [P], blocks, counts, kb, vb, out, lse, ws)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    at = np.concatenate((np.arange(5), np.random.default_rng(2).integers(0, gamma, 200), gamma - 1 - np.arange(5)))
    up = lambda x: x.double().cpu().numpy()  # noqa: E731
    here = torch.from_numpy(at).cuda()
    ref = U.ref_attend(*(up(x) for x in (q[0, here], k[0, :, :P].transpose(0, 1), v[0, :, :P].transpose(0, 1), kb[0, here], vb[0, here])),
                       None, bs, 1, float(np.float32(D ** -0.5)))
    U.check_attend(up(out[0, here]), up(lse[0, here]), ref, D)


def test_a_row_that_sees_nothing_in_the_first_64_splits():
    """A prefix of more keys than 64 workgroups' tables hold, beside a request without a prefix and two long branches: tiles of rows
    reach over both branches, and the second one's rows see nothing of what the first 64 workgroups look at."""
    P, gamma, L, D, bs = 1_200_000, 2, 6000, 64, 16
    g = torch.Generator(device="cuda").manual_seed(7)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    n_blocks = P // bs
    k, v = rand(n_blocks, 1, bs, D), rand(n_blocks, 1, bs, D)
    table = torch.stack((torch.randperm(n_blocks, generator=g, device="cuda"), torch.zeros(n_blocks, device="cuda"))).to(torch.int32)
    q, kb, vb = rand(2, gamma, L, 1, D), rand(2, gamma, L, 1, D), rand(2, gamma, L, 1, D)
    d = U.desc("bf16", B_=2, Hq=1, Hkv=1, D=D, gamma=gamma, L=L, bs=bs, max_blocks=n_blocks)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:-1], device="cuda")
    need = B.la_verify_attention_sparse_workspace(d, None, [P, 0])
    assert need >= 65 * 2 * gamma * L * (D + 2) * 4           # more than 64 partial results of every row
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    B.la_verify_attention_sparse(d, None, q, B.make_block_cache(k, v), table, U.i32([P, 0]), [P, 0], None, None, kb, vb, out, lse, ws)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    scale = float(np.float32(D ** -0.5))
    for b, branch, rows in ((1, 0, slice(None)), (1, 1, slice(None)), (0, 0, [0, 5999]), (0, 1, [0, 17, 5999])):
        kk, vv = (x[b, branch, :, 0].double() for x in (kb, vb))
        at = torch.arange(L, device="cuda")[rows]
        seen = torch.arange(L, device="cuda") <= at[:, None]
        if b == 0:
            prefix = [x[table[0].long()].reshape(P, D).double() for x in (k, v)]
            kk, vv = torch.cat((prefix[0], kk)), torch.cat((prefix[1], vv))
            seen = torch.cat((torch.ones((len(at), P), dtype=torch.bool, device="cuda"), seen), 1)
        x = q[b, branch, at, 0].double()
        score = (x @ kk.T.contiguous() * scale).masked_fill(~seen, -np.inf)
        size = (x.abs() @ kk.abs().T.contiguous() * scale).masked_fill(~seen, 0.0).amax(1)
        p = torch.softmax(score, 1)
        ref = [t.cpu().numpy() for t in (p @ vv, torch.logsumexp(score, 1), p @ vv.abs(), size)]
        U.check_attend(out[b, branch, at, 0].double().cpu().numpy(), lse[b, branch, at, 0].double().cpu().numpy(), ref, D)


@pytest.mark.parametrize("rows,n", [(1, 60), (20, 60), (80, 300), (2, 8300)])
@pytest.mark.parametrize("where", ["everywhere", "one channel", "one block"])
def test_select_where_fp32_sums_overflow(rows, n, where):
    """Finite queries and bounds whose scores, or parts of them, lie beyond fp32: the order is still that of the exact scores, and
    the list is written whole."""
    rng = np.random.default_rng(rows + n)
    D, bs = 64, 16
    q = U.bf16(rng.standard_normal((1, 1, rows, 1, D)))
    c = rng.standard_normal((n, 1, D))
    bounds = U.bf16(np.stack((c - 1.0 - rng.random(c.shape), c + 1.0 + rng.random(c.shape)), 2))
    big = 2.0 ** 70
    if where == "everywhere":
        q, bounds = q * big, bounds * big
    elif where == "one channel":
        q[..., 3] *= big
        bounds[..., 3] *= big
    else:
        q *= big
        bounds[n // 2] *= big
        bounds[n // 2, :, 0] *= -1.0                          # (bounds that are no bounds: one sum of both infinities)
    run_select(q, [bounds], [n * bs], 1, bs, rows, 7, 1, 1)
    run_select(q, [bounds], [n * bs], 1, bs, rows, min(n - 1, 1100), 0, 0)
