"""The block cache's calls together, as a program runs them: a prompt is stored, a pass selects blocks and attends to them, what
it accepted is stored, the next pass sees it; the same step captured into a graph, on a stream of its own."""
import numpy as np
import pytest
import torch

import block_cache_util as U
from paper_2506_19830_amd import binding as B

pytestmark = pytest.mark.gpu


class Program:
    """Buffers of a small model's one layer and its calls."""

    def __init__(self, fmt, seed, prompts=(150, 37), gamma=3, L=5, Hq=6, Hkv=2, D=64, bs=16, max_blocks=24, group=5, most=6):
        self.rng = np.random.default_rng(seed)
        self.fmt, self.gamma, self.L, self.Hq, self.Hkv, self.D, self.bs, self.group, self.most = fmt, gamma, L, Hq, Hkv, D, bs, group, most
        self.prompts, n = list(prompts), len(prompts)
        self.n, self.max_blocks = n, max_blocks
        self.host_table, self.table, pool = U.tables(self.rng, n, max_blocks, True)
        shape = (pool, Hkv, bs)
        dtype, width = {"bf16": (torch.bfloat16, D), "mxfp8_e4m3": (torch.float8_e4m3fn, D), "mxfp4_e2m1": (torch.uint8, D // 2)}[fmt]
        self.el = [torch.zeros(shape + (width,), dtype=torch.uint8, device="cuda").view(dtype) if fmt != "bf16" else
                   torch.zeros(shape + (width,), dtype=dtype, device="cuda") for _ in "kv"]
        self.ex = [None if fmt == "bf16" else torch.zeros(shape + (D // 32,), dtype=torch.uint8, device="cuda") for _ in "kv"]
        self.bounds = torch.full((pool, Hkv, 2, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.cache = B.make_block_cache(*self.el, *self.ex, self.bounds)
        self.kw = dict(B_=n, Hq=Hq, Hkv=Hkv, D=D, bs=bs, max_blocks=max_blocks)
        self.desc = U.desc(fmt, gamma=gamma, L=L, **self.kw)
        self.choice = B.make_select_desc(group_len=group, max_blocks=most, keep_first=1, keep_last=1)
        groups = -(-L // group)
        self.blocks = torch.zeros((n, gamma, groups, Hkv, most), dtype=torch.int32, device="cuda")
        self.counts = torch.zeros((n, gamma, groups, Hkv), dtype=torch.int32, device="cuda")
        self.q = torch.zeros((n, gamma, L, Hq, D), dtype=torch.bfloat16, device="cuda")
        self.kv = [torch.zeros((n, gamma, L, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        self.out, self.lse = torch.zeros_like(self.q), torch.zeros(self.q.shape[:-1], device="cuda")
        self.src, self.own = U.i32([0] * n), U.i32([0] * n)
        self.held = [[np.zeros((0, Hkv, D)) for _ in range(n)] for _ in "kv"]    # what the cache stands for

    def draw(self, t):
        t.copy_(torch.from_numpy(self.rng.standard_normal(tuple(t.shape))).to(torch.bfloat16).cuda())

    def prompt(self):
        longest = max(self.prompts)
        kv = [torch.zeros((self.n, 1, longest, self.Hkv, self.D), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        for t in kv:
            self.draw(t)
        zero, lens = U.i32([0] * self.n), U.i32([0] * self.n)
        B.la_kv_store(U.desc(self.fmt, L=longest, **self.kw), self.cache, self.table, zero, [0] * self.n, *kv, None, None, None, None,
                      U.i32(self.prompts), lens)
        assert lens.tolist() == self.prompts
        for w in (0, 1):
            for b, p in enumerate(self.prompts):
                self.grow(w, b, kv[w][b, 0, :p])
        return lens

    def grow(self, w, b, rows):
        x = rows.double().cpu().numpy()
        self.held[w][b] = np.concatenate((self.held[w][b], U.storage(x, self.fmt)[2] if x.shape[0] else x))

    def workspace(self, lens):
        return [torch.empty(max(16, n), dtype=torch.uint8, device="cuda") for n in (
            B.la_block_select_workspace(self.desc, self.choice, lens), B.la_verify_attention_sparse_workspace(self.desc, self.choice, lens))]

    def step(self, lens_dev, lens, new_lens, ws, out=None, lse=None):
        B.la_block_select(self.desc, self.choice, self.q, self.bounds, self.table, lens_dev, lens, self.blocks, self.counts, ws[0])
        B.la_verify_attention_sparse(self.desc, self.choice, self.q, self.cache, self.table, lens_dev, lens, self.blocks, self.counts,
                                     *self.kv, self.out if out is None else out, self.lse if lse is None else lse, ws[1])
        B.la_kv_store(self.desc, self.cache, self.table, lens_dev, lens, *self.kv, None, None, self.src, None, self.own, new_lens)

    def expected(self, lens):
        """(blocks, counts, attention's reference) of every request."""
        res = []
        for b, p in enumerate(lens):
            k, v = self.held[0][b], self.held[1][b]
            have = -(-p // self.bs)
            bounds = np.stack([np.stack((k[j * self.bs:(j + 1) * self.bs].min(0), k[j * self.bs:(j + 1) * self.bs].max(0)), 1) for j in range(have)])
            q = self.q[b].double().cpu().numpy()
            blocks, counts = U.ref_select(q, bounds, have, self.group, self.most, 1, 1)
            lists = [[[blocks[g, i, h, :counts[g, i, h]] for h in range(self.Hkv)] for i in range(blocks.shape[1])] for g in range(self.gamma)]
            kb, vb = (t[b].double().cpu().numpy() for t in self.kv)
            res.append((blocks, counts, U.ref_attend(q, k, v, kb, vb, lists, self.bs, self.group, float(np.float32(self.D ** -0.5)))))
        return res

    def check(self, lens, out=None, lse=None):
        out, lse = self.out if out is None else out, self.lse if lse is None else lse
        for b, (blocks, counts, ref) in enumerate(self.expected(lens)):
            assert np.array_equal(self.blocks[b].cpu().numpy(), blocks) and np.array_equal(self.counts[b].cpu().numpy(), counts)
            U.check_attend(out[b].double().cpu().numpy(), lse[b].double().cpu().numpy(), ref, self.D)


@pytest.mark.parametrize("fmt", U.FORMATS)
def test_passes_over_a_growing_cache(fmt):
    p = Program(fmt, 21)
    lens_dev = p.prompt()
    lens = list(p.prompts)
    for turn in range(4):
        for t in [p.q] + p.kv:
            p.draw(t)
        src, own = p.rng.integers(0, p.gamma, p.n).tolist(), p.rng.integers(0, p.L + 1, p.n).tolist()
        p.src.copy_(U.i32(src)), p.own.copy_(U.i32(own))
        new = U.i32([0] * p.n)
        p.step(lens_dev, lens, new, p.workspace(lens))
        torch.cuda.synchronize()
        p.check(lens)
        for w in (0, 1):
            for b in range(p.n):
                p.grow(w, b, p.kv[w][b, src[b], :own[b]])
        lens = [a + b for a, b in zip(lens, own)]
        assert new.tolist() == lens
        lens_dev = new
    # what was stored comes back
    most = max(lens)
    back = [torch.zeros((p.n, most, p.Hkv, p.D), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    B.la_kv_load(p.desc, p.cache, p.table, lens_dev, None, *back)
    for w in (0, 1):
        for b in range(p.n):
            assert np.array_equal(back[w][b, :lens[b]].double().cpu().numpy(), p.held[w][b])


@pytest.mark.parametrize("fmt", U.FORMATS)
def test_captured_step_replays_like_eager(fmt):
    """Two steps captured with workspaces of their own, replayed in turn with eager work between, on inputs that change in
    place; every replay equals an eager run."""
    p = Program(fmt, 22, prompts=(200, 90), most=4)
    lens_dev, lens = p.prompt(), list(p.prompts)
    p.own.copy_(U.i32([3, 5])), p.src.copy_(U.i32([2, 1]))
    p.draw(p.q)
    bufs = [dict(ws=p.workspace(lens), out=torch.zeros_like(p.out), lse=torch.zeros_like(p.lse), new=U.i32([0, 0])) for _ in range(3)]

    def run(b):
        p.step(lens_dev, lens, b["new"], b["ws"], b["out"], b["lse"])
    run(bufs[0])
    torch.cuda.synchronize()
    graphs = []
    for b in bufs[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(b)
        graphs.append(g)
    for replay in range(4):
        for t in [p.q] + p.kv:
            p.draw(t)
        for b in bufs:
            b["out"].zero_(), b["lse"].zero_(), b["new"].zero_()
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        run(bufs[2])
        torch.cuda.synchronize()
        p.check(lens, bufs[2]["out"], bufs[2]["lse"])   # (the last block, whose bounds only widen, is always taken)
        for b in bufs[:2]:
            for k in ("out", "lse", "new"):
                assert torch.equal(b[k], bufs[2][k]), f"replay {replay}: {k}"


def test_calls_follow_the_current_stream():
    """Work queued on a side stream comes after what fills its inputs there, and two streams run side by side."""
    ps = [Program("mxfp4_e2m1", 30 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in ps]
    todo = []
    for p, s in zip(ps, streams):
        lens_dev, lens = p.prompt(), list(p.prompts)
        fresh = [torch.from_numpy(p.rng.standard_normal(tuple(t.shape))).to(torch.bfloat16).cuda() for t in [p.q] + p.kv]
        big = torch.randn((2048, 2048), device="cuda")
        todo.append((p, s, lens_dev, lens, fresh, big, p.workspace(lens), U.i32([0, 0])))
    torch.cuda.synchronize()
    for p, s, lens_dev, lens, fresh, big, ws, new in todo:
        with torch.cuda.stream(s):
            for _ in range(10):
                big = big @ big * 1e-3
            for t, x in zip([p.q] + p.kv, fresh):
                t.copy_(x + 0 * big[0, 0].to(torch.bfloat16).nan_to_num(0.0, 0.0, 0.0))
            p.step(lens_dev, lens, new, ws)
    torch.cuda.synchronize()
    for p, s, lens_dev, lens, fresh, big, ws, new in todo:
        p.check(lens)
