"""``la_kv_store`` and ``la_kv_load``: codes, exponents, bounds and lengths are exact, byte for byte."""
import numpy as np
import pytest
import torch

import block_cache_util as U
from paper_2506_19830_amd import binding as B

pytestmark = pytest.mark.gpu


def run_store(seed, fmt, prefix, own, L, Hkv, D, bs, gamma=1, chain=0, kept=0, layers=1, paged=True, bounds=True, rows=None,
              decisions=True):
    rng = np.random.default_rng(seed)
    n = len(prefix)
    max_blocks = -(-(max(prefix) + chain + L) // bs)
    host_table, table, pool = U.tables(rng, n, max_blocks, paged)
    width = {"bf16": 2 * D, "mxfp8_e4m3": D, "mxfp4_e2m1": D // 2}[fmt]
    el = {w: torch.from_numpy(rng.integers(0, 256, (layers, pool, Hkv, bs, width), dtype=np.uint8)) for w in "kv"}
    ex = {w: torch.from_numpy(rng.integers(0, 256, (layers, pool, Hkv, bs, D // 32), dtype=np.uint8)) for w in "kv"}
    low = U.bf16(rng.standard_normal((layers, pool, Hkv, D)) - 1.0)
    old_bounds = np.stack((low, low + 2.0), 3)
    old_bounds = U.bf16(old_bounds)
    src = rng.integers(0, gamma, n)
    draw = (lambda shape: U.bf16(rng.standard_normal(shape) * np.exp2(rng.integers(-6, 7, shape[:-1] + (1,))))) if rows is None else rows
    new = {w + part: draw((layers, n) + shape) for w in "kv"
           for part, shape in (("_branch", (gamma, L, Hkv, D)), ("_chain", (chain, Hkv, D)))}

    # expected
    want_el, want_ex = {w: el[w].clone() for w in "kv"}, {w: ex[w].clone() for w in "kv"}
    want_bounds = old_bounds.copy()
    want_lens, back = [], {w: np.zeros((layers, n, chain + L, Hkv, D)) for w in "kv"}
    for b in range(n):
        take = kept + own[b]
        want_lens.append(prefix[b] + take)
        for w in "kv":
            x = np.concatenate((new[w + "_chain"][:, b, :kept], new[w + "_branch"][:, b, src[b], :own[b]]), 1)
            e, s, values = U.storage(x, fmt)
            back[w][:, b, :take] = values
            for t in range(take):
                pos = prefix[b] + t
                blk = int(host_table[b, pos // bs])
                want_el[w][:, blk, :, pos % bs] = U.raw(e[:, t]).contiguous().view(torch.uint8).reshape(layers, Hkv, width)
                if s is not None:
                    want_ex[w][:, blk, :, pos % bs] = s[:, t]
                if w == "k":
                    if pos % bs == 0:
                        want_bounds[:, blk, :, 0] = want_bounds[:, blk, :, 1] = values[:, t]
                    want_bounds[:, blk, :, 0] = np.minimum(want_bounds[:, blk, :, 0], values[:, t])
                    want_bounds[:, blk, :, 1] = np.maximum(want_bounds[:, blk, :, 1], values[:, t])

    view = {"bf16": torch.bfloat16, "mxfp8_e4m3": torch.float8_e4m3fn, "mxfp4_e2m1": torch.uint8}[fmt]
    dev = {w: el[w].cuda().view(view) for w in "kv"}
    exd = {w: None if fmt == "bf16" else ex[w].cuda() for w in "kv"}
    bd = torch.from_numpy(old_bounds).to(torch.bfloat16).cuda() if bounds else None
    cache = B.make_block_cache(dev["k"], dev["v"], exd["k"], exd["v"], bd)
    up = {k: torch.from_numpy(x).to(torch.bfloat16).cuda() for k, x in new.items()}
    d = U.desc(fmt, B_=n, Hq=Hkv, Hkv=Hkv, D=D, gamma=gamma, L=L, bs=bs, max_blocks=max_blocks)
    rows_of = n * Hkv * D
    strides = B.la_layer_strides(layers, pool * Hkv * bs * D, gamma * L * rows_of, chain * rows_of, 0)
    lens, new_lens = U.i32(prefix), U.i32([-7] * n)
    B.la_kv_store(d, cache, table, lens, prefix, up["k_branch"], up["v_branch"], up["k_chain"] if chain else None,
                  up["v_chain"] if chain else None, U.i32(src.tolist()) if decisions else None,
                  U.i32([kept] * n) if chain else None, U.i32(own) if decisions else None, new_lens,
                  strides if layers > 1 else None)
    torch.cuda.synchronize()
    assert new_lens.tolist() == want_lens
    for w in "kv":
        assert torch.equal(dev[w].view(torch.uint8).cpu(), want_el[w]), f"{w} elements"
        if fmt != "bf16":
            assert torch.equal(exd[w].cpu(), want_ex[w]), f"{w} exponents"
    if bounds:
        assert np.array_equal(bd.double().cpu().numpy(), want_bounds)

    # and back, into both types; rows that do not exist stay as they were
    for out, dtype in (("bf16", torch.bfloat16), ("f32", torch.float32)):
        d2 = U.desc(fmt, B_=n, Hq=Hkv, Hkv=Hkv, D=D, gamma=gamma, L=L, bs=bs, max_blocks=max_blocks, out=out)
        got = [torch.full((layers, n, chain + L, Hkv, D), 3.25, dtype=dtype, device="cuda") for _ in "kv"]
        s2 = B.la_layer_strides(layers, pool * Hkv * bs * D, (chain + L) * rows_of, 0, 0)
        B.la_kv_load(d2, cache, table, new_lens, lens, *got, s2)
        torch.cuda.synchronize()
        for w, t in zip("kv", got):
            for b in range(n):
                x = t[:, b].double().cpu().numpy()
                assert np.array_equal(x[:, :kept + own[b]], back[w][:, b, :kept + own[b]])
                assert (x[:, kept + own[b]:] == 3.25).all()


@pytest.mark.parametrize("fmt", U.FORMATS)
@pytest.mark.parametrize("kw", [
    dict(prefix=[0], own=[1], L=1, Hkv=1, D=64, bs=16),                                        # the first token of all
    dict(prefix=[15, 16, 17, 31], own=[1, 1, 1, 1], L=1, Hkv=3, D=128, bs=16),                 # around a block's end
    dict(prefix=[0, 5, 64], own=[130, 0, 77], L=130, Hkv=2, D=128, bs=64),                     # ragged prompts, one empty
    dict(prefix=[7, 40], own=[9, 4], L=9, Hkv=2, D=64, bs=32, gamma=3, chain=21, kept=13, layers=3),
    dict(prefix=[33], own=[0], L=5, Hkv=2, D=256, bs=16, gamma=2, chain=40, kept=40),          # the chain alone
    dict(prefix=[3], own=[70], L=70, Hkv=5, D=256, bs=128, paged=False, bounds=False),
    dict(prefix=[100], own=[0], L=1, Hkv=1, D=128, bs=128),                                    # nothing at all
    dict(prefix=[20, 0], own=[33, 33], L=33, Hkv=8, D=128, bs=16, decisions=False),            # no decisions: all of branch 0
], ids=lambda kw: f"P{'-'.join(map(str, kw['prefix']))}_L{kw['L']}_D{kw['D']}_bs{kw['bs']}")
def test_store_and_load(fmt, kw):
    run_store(11, fmt, **kw)


@pytest.mark.parametrize("fmt", U.FORMATS)
def test_values_where_rounding_decides(fmt):
    """Every middle between two codes, values one bf16 step beside it, zeros of both signs, groups of zeros, the largest
    magnitude exactly at and just above a power's reach, groups far below and far above the exponents' range."""
    grid = U.GRID[fmt if fmt != "bf16" else "mxfp8_e4m3"]
    middles = (grid[1:] + grid[:-1]) / 2

    def rows(shape):
        if np.prod(shape) == 0:
            return np.zeros(shape)
        rng = np.random.default_rng(5)
        x = np.empty(shape)
        flat = x.reshape(-1, 32)
        for i in range(flat.shape[0]):
            kind = i % 8
            e = float(rng.integers(-20, 20))
            base = rng.choice(np.concatenate((middles, grid)), 32)
            step = rng.choice([0.0, 2.0 ** -8, -2.0 ** -8], 32)
            flat[i] = base * (1 + step) * rng.choice([-1.0, 1.0], 32) * 2.0 ** e
            if kind == 1:
                flat[i] = rng.choice([0.0, -0.0], 32)
            if kind == 2:
                flat[i, 7] = grid[-1] * 2.0 ** e
            if kind == 3:
                flat[i, 31] = -grid[-1] * 2.0 ** e * (1 + 2.0 ** -7)
            if kind == 4:
                flat[i] *= 2.0 ** -90
            if kind == 5:
                flat[i] *= 2.0 ** -110
            if kind == 6:
                flat[i] = np.where(np.arange(32) == 3, 1.5 * 2.0 ** 120, flat[i])
            if kind == 7:
                flat[i] = 2.0 ** -126 * rng.choice([1.0, 0.5, -0.25, 0.0], 32)   # the smallest normal number and below
        return U.bf16(x)
    run_store(3, fmt, prefix=[5, 0], own=[40, 40], L=40, Hkv=2, D=128, bs=16, rows=rows)


def test_load_takes_what_exists():
    """Starts before, inside and behind the prefix, with and without a table; more tokens than there are."""
    rng = np.random.default_rng(2)
    for fmt in U.FORMATS:
        for paged in (True, False):
            c = U.Cache(rng, fmt, [37, 0, 16, 5], 2, 64, 16, 3, paged)
            first = [30, 0, -4, 9]
            out = [torch.full((4, 12, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
            d = U.desc(fmt, B_=4, Hkv=2, D=64, bs=16, max_blocks=3)
            B.la_kv_load(d, c.desc, c.table, c.lens, U.i32(first), *out)
            for t, rows in zip(out, (c.k, c.v)):
                got = t.double().cpu().numpy()
                for b in range(4):
                    for i in range(12):
                        pos = first[b] + i
                        if 0 <= pos < c.prefix[b]:
                            assert np.array_equal(got[b, i], rows[b][pos])
                        else:
                            assert (got[b, i] == 9.0).all()
            # without a start: from the first row
            B.la_kv_load(d, c.desc, c.table, c.lens, None, *out)
            assert np.array_equal(out[0].double().cpu().numpy()[0], c.k[0][:12])


def test_decisions_are_clamped():
    """Branch, chain and own counts outside their ranges are brought into them."""
    rng = np.random.default_rng(4)
    x = torch.from_numpy(rng.standard_normal((2, 2, 3, 1, 64))).to(torch.bfloat16).cuda()
    chain = torch.from_numpy(rng.standard_normal((2, 4, 1, 64))).to(torch.bfloat16).cuda()
    el = [torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    cache = B.make_block_cache(*el)
    d = U.desc("bf16", B_=2, Hq=1, Hkv=1, D=64, gamma=2, L=3, bs=16, max_blocks=1)
    new = U.i32([0, 0])
    B.la_kv_store(d, cache, None, U.i32([2, 1]), [2, 1], x, x, chain, chain, U.i32([99, -5]), U.i32([-3, 50]), U.i32([7, -1]), new)
    assert new.tolist() == [5, 5]
    assert torch.equal(el[0][0, 0, 2:5], x[0, 1, :, 0]) and torch.equal(el[1][1, 0, 1:5], chain[1, :, 0])
    assert not el[0][0, 0, 5:].any() and not el[0][1, 0, 5:].any()
