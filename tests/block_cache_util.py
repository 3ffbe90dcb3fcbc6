"""Plain 64-bit counterparts of the block cache calls, and what their tests share.  Everything is numpy in float64, written
from the definitions; nothing of the library's arithmetic is used."""
from __future__ import annotations

import numpy as np
import torch

from paper_2506_19830_amd import binding as B

FORMATS = ("bf16", "mxfp8_e4m3", "mxfp4_e2m1")
FP4 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
FP8 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])
GRID = {"mxfp8_e4m3": FP8, "mxfp4_e2m1": FP4}


def bf16(x):
    """Nearest bf16, as float64."""
    return torch.as_tensor(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).double().numpy()


def quantise(x, fmt):
    """Rows [.., D] of float64 -> (codes, exponents [.., D / 32], values)."""
    grid = GRID[fmt]
    g = np.asarray(x, dtype=np.float64).reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    top = np.abs(g).max(-1)
    exps = np.full(top.shape, -100, dtype=np.int64)
    for e in range(-100, 100):                       # the smallest exponent that holds the largest magnitude
        exps += top > grid[-1] * 2.0 ** e
    y = g / np.exp2(exps.astype(np.float64))[..., None]
    a = np.minimum(np.abs(y), grid[-1])
    up = np.searchsorted(grid, a)                    # grid[up - 1] < a <= grid[up]
    down = np.maximum(up - 1, 0)
    below, above = a - grid[down], grid[up] - a
    take_up = (above < below) | ((above == below) & (up % 2 == 0))
    code = np.where(take_up, up, down)
    sign = np.signbit(y)
    values = np.where(sign, -1.0, 1.0) * grid[code] * np.exp2(exps.astype(np.float64))[..., None]
    code = code + np.where(sign, 128 if fmt == "mxfp8_e4m3" else 8, 0)
    return code.reshape(x.shape), exps, values.reshape(x.shape)


def storage(x, fmt):
    """Rows [.., D] of bf16 numbers in float64 -> (elements, exponents or None: CPU tensors as the cache holds them, values)."""
    if fmt == "bf16":
        return torch.from_numpy(x).to(torch.bfloat16), None, x
    code, exps, values = quantise(x, fmt)
    code = code.astype(np.uint8)
    if fmt == "mxfp8_e4m3":
        el = torch.from_numpy(code).view(torch.float8_e4m3fn)
    else:
        el = torch.from_numpy(code[..., 0::2] | (code[..., 1::2] << 4))
    return el, torch.from_numpy((exps + 127).astype(np.uint8)), values


def raw(t):
    """A tensor's bytes (or words) for exact comparison."""
    t = t.detach().cpu().contiguous()
    return t.view(torch.int16) if t.dtype == torch.bfloat16 else t.view(torch.uint8) if t.element_size() == 1 else t


def desc(fmt, *, B_=1, Hq=4, Hkv=2, D=64, gamma=1, L=1, bs=16, max_blocks=8, out="bf16", scale=None):
    return B.make_attn_desc(num_requests=B_, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, gamma=gamma, branch_len=L,
                            block_size=bs, max_blocks_per_request=max_blocks, q_dtype="bf16", kv_dtype=fmt,
                            branch_kv_dtype="bf16", out_dtype=out, softmax_scale=D ** -0.5 if scale is None else scale)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def tables(rng, n, max_blocks, paged):
    """(host table [n, max_blocks], device table or None for the identity, blocks of the pool)."""
    pool = n * max_blocks + (3 if paged else 0)
    host = rng.permutation(pool)[:n * max_blocks] if paged else np.arange(pool)
    host = host.reshape(n, max_blocks).astype(np.int32)
    return host, (torch.from_numpy(host).cuda() if paged else None), pool


class Cache:
    """A block cache with the given prefixes in it; every byte that no prefix owns is set to all ones (NaN, or the largest
    code and exponent), so that whatever reads it shows."""

    def __init__(self, rng, fmt, prefix, Hkv, D, bs, max_blocks, paged=True, k_rows=None, v_rows=None):
        self.fmt, self.prefix, self.bs, self.max_blocks = fmt, list(prefix), bs, max_blocks
        n = len(prefix)
        self.host_table, self.table, pool = tables(rng, n, max_blocks, paged)
        es = {"bf16": (D, torch.int16), "mxfp8_e4m3": (D, torch.uint8), "mxfp4_e2m1": (D // 2, torch.uint8)}[fmt]
        self.k, self.v = [], []               # per request: values [P, Hkv, D], float64
        store = {}
        for w, given in (("k", k_rows), ("v", v_rows)):
            el = torch.full((pool, Hkv, bs, es[0]), -1 if es[1] == torch.int16 else 255, dtype=es[1])
            ex = None if fmt == "bf16" else torch.full((pool, Hkv, bs, D // 32), 255, dtype=torch.uint8)
            for b, p in enumerate(prefix):
                x = bf16(rng.standard_normal((p, Hkv, D))) if given is None else given[b]
                e, s, values = storage(x, fmt)
                getattr(self, w).append(values)
                for t in range(p):
                    blk = int(self.host_table[b, t // bs])
                    el[blk, :, t % bs] = raw(e[t])
                    if ex is not None:
                        ex[blk, :, t % bs] = s[t]
            el = el.cuda()
            store[w] = el.view(torch.bfloat16) if fmt == "bf16" else el.view(torch.float8_e4m3fn) if fmt == "mxfp8_e4m3" else el
            store[w + "_exp"] = None if ex is None else ex.cuda()
        self.t = store
        self.desc = B.make_block_cache(store["k"], store["v"], store["k_exp"], store["v_exp"])
        self.lens = i32(self.prefix)


def ref_select(q, bounds, have, group, most, first, last):
    """q [gamma, L, Hq, D], bounds [N, Hkv, 2, D], both float64 -> blocks [gamma, groups, Hkv, most], counts."""
    gamma, L, Hq, D = q.shape
    Hkv = bounds.shape[1]
    G, groups = Hq // Hkv, -(-L // group)
    blocks = np.full((gamma, groups, Hkv, most), -1, dtype=np.int32)
    counts = np.full((gamma, groups, Hkv), min(have, most), dtype=np.int32)
    for g in range(gamma):
        for i in range(groups):
            for h in range(Hkv):
                if have <= most:
                    blocks[g, i, h, :have] = np.arange(have)
                    continue
                rows = q[g, i * group:(i + 1) * group, h * G:(h + 1) * G].reshape(-1, D)
                lo, hi = bounds[:have, h, 0], bounds[:have, h, 1]
                score = (rows[:, None] * np.where(rows[:, None] > 0, hi, lo)).sum(-1).max(0)
                rest = np.arange(first, have - last)
                order = rest[np.argsort(-score[rest], kind="stable")][:most - first - last]
                blocks[g, i, h] = np.sort(np.concatenate((np.arange(first), order, np.arange(have - last, have))))
    return blocks, counts


def ref_attend(q, k, v, kb, vb, lists, bs, group, scale):
    """One request, float64: q [gamma, L, Hq, D], prefix k / v [P, Hkv, D], branch kb / vb [gamma, L, Hkv, D]; lists: None or
    [gamma][groups][Hkv] index arrays.  Returns out, lse, the mean of |v| under the probabilities, and a bound of |q.k| sums."""
    gamma, L, Hq, D = q.shape
    P, Hkv = k.shape[0], kb.shape[2]
    G = Hq // Hkv
    out, mass = np.empty(q.shape), np.empty(q.shape)
    lse, size = np.empty(q.shape[:3]), np.empty(q.shape[:3])
    for g in range(gamma):
        for i in range(L):
            for h in range(Hkv):
                if lists is None:
                    at = np.arange(P)
                else:
                    names = np.asarray(lists[g][i // group][h], dtype=np.int64)
                    at = (names[:, None] * bs + np.arange(bs)).reshape(-1)
                    at = at[at < P]
                kk = np.concatenate((k[at, h], kb[g, :i + 1, h]))
                vv = np.concatenate((v[at, h], vb[g, :i + 1, h]))
                rows = q[g, i, h * G:(h + 1) * G]
                x = rows @ kk.T * scale
                m = x.max(-1, keepdims=True)
                p = np.exp(x - m)
                total = p.sum(-1, keepdims=True)
                out[g, i, h * G:(h + 1) * G] = p @ vv / total
                mass[g, i, h * G:(h + 1) * G] = p @ np.abs(vv) / total
                lse[g, i, h * G:(h + 1) * G] = (m + np.log(total))[:, 0]
                size[g, i, h * G:(h + 1) * G] = (np.abs(rows) @ np.abs(kk).T * scale).max(-1)
    return out, lse, mass, size


def check_attend(got, got_lse, ref, D, out="bf16"):
    """Against the definition.  A probability is rounded to bf16 (relative 2^-8 at most), the result to bf16 again; a score is
    a sum of D exact products in fp32, scaled once (D + 2 roundings, counted at a whole unit of 2^-23 of the sum of
    magnitudes), and moves its probability by a factor of 1 + its error, the sum by as much.  The exponential and the fp32
    sums add less than 2^-12 to what the probabilities' rounding allows."""
    want, lse, mass, size = ref
    moved = (D + 2) * 2.0 ** -23 * size
    allowed = (2.0 ** -8 + 2.0 ** -12 + 2 * moved)[..., None] * mass
    if out == "bf16":
        allowed = allowed + 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -7)
    assert np.isfinite(got).all()
    worst = (np.abs(got - want) / allowed).max()
    assert worst <= 1.0, f"{worst:.3f} times what the roundings allow"
    if got_lse is not None:
        assert (np.abs(got_lse - lse) <= moved + 2.0 ** -18 * np.maximum(1, np.abs(lse))).all()
    return worst
