"""The block cache of the verification path as measurable cases: writing it, reading it back, choosing its blocks, attending
over the chosen ones.

A block cache is the paged K/V cache whose rows are kept in bf16 or quantised as they are written (groups of 32 elements
share a power of two; the elements are fp8-e4m3 or fp4-e2m1), with the smallest and the largest key of every block beside
it.  Four operators work on it:

``store``   rows of accepted tokens are quantised into the cache, and the bounds of the blocks they touch widened
``load``    rows come back as the values the cache holds
``select``  for every group of query tokens and KV head, the blocks whose bounds allow the largest score
``attend``  verification attention over the selected blocks (or over all) and the branch's own tokens

``run`` computes them with elementary torch operations, and through the package's entry points where ``own`` is true.
"""
from __future__ import annotations

import math

import torch

own = False

_FORMATS = ("bf16", "mxfp8_e4m3", "mxfp4_e2m1")
_ROW_BYTES = {"bf16": lambda d: 2 * d, "mxfp8_e4m3": lambda d: d + d // 32, "mxfp4_e2m1": lambda d: d // 2 + d // 32}
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)   # magnitudes of the fp4 codes 0..7
_EXP_MIN, _EXP_MAX = -100, 100

# Upper bounds of what a drawn case may cost (see draw()): those of the largest listed ones.
_MAX_STORE_ROWS, _MAX_LOAD_ROWS = 2.0e6, 6.0e5
_MAX_SELECT_FLOPS, _MAX_SELECT_BYTES = 2.1e10, 7.0e7
_MAX_ATTEND_FLOPS, _MAX_ATTEND_BYTES, _MAX_ATTEND_GATHER = 2.3e10, 6.0e8, 5.0e8


def _text(values):
    return ",".join(str(int(v)) for v in values)


def _numbers(text):
    return tuple(int(v) for v in text.split(","))


def _ages(n, lo, hi):
    """n prefix lengths between lo and hi, geometrically spaced, all different from a multiple of a block."""
    return [int(lo * (hi / lo) ** ((i + 0.5) / n)) | 1 for i in range(n)]


def _store(fmt, prefix, own_len, L, hkv, d, block, gamma=1, chain=0, kept_chain=0, layers=1):
    return {"kind": "store", "fmt": fmt, "prefix": _text(prefix), "own_len": _text(own_len), "L": L, "Hkv": hkv, "D": d,
            "block": block, "gamma": gamma, "chain": chain, "kept_chain": kept_chain, "layers": layers}


def _load(fmt, prefix, first, tokens, hkv, d, block):
    return {"kind": "load", "fmt": fmt, "prefix": _text(prefix), "first": _text(first), "tokens": tokens, "Hkv": hkv, "D": d,
            "block": block}


def _select(prefix, gamma, L, group, hq, hkv, d, block, most, first, last):
    return {"kind": "select", "prefix": _text(prefix), "gamma": gamma, "L": L, "group": group, "Hq": hq, "Hkv": hkv, "D": d,
            "block": block, "most": most, "keep_first": first, "keep_last": last}


def _attend(fmt, prefix, gamma, L, group, hq, hkv, d, block, most):
    """most: blocks selected per group at most; 0: no selection, every block of the prefix."""
    return {"kind": "attend", "fmt": fmt, "prefix": _text(prefix), "gamma": gamma, "L": L, "group": group, "Hq": hq,
            "Hkv": hkv, "D": d, "block": block, "most": most}


def listed():
    cases = {
        # a decoding batch: every request's next token joins a 4-bit cache (one layer; latency counts)
        "store_token_fp4": _store("mxfp4_e2m1", _ages(32, 300, 16000), [1] * 32, 1, 8, 128, 64),
        # prompts of different length enter an 8-bit cache at once
        "store_prompt_fp8": _store("mxfp8_e4m3", [0] * 4, [8192, 5003, 7777, 1021], 8192, 8, 128, 64),
        # what survives a verification pass joins the 4-bit cache of all 64 layers: 192 drafted tokens and a step of 64
        "store_steps_fp4_layers": _store("mxfp4_e2m1", [4099], [64], 64, 8, 128, 16, gamma=8, chain=448, kept_chain=192,
                                         layers=64),
        # the tail of two short contexts in plain bf16, head dimension 64
        "load_tail_bf16": _load("bf16", [777, 131], [700, 64], 77, 8, 64, 16),
        # a long shared prefix comes back in bf16 for a dense pass of another model part
        "load_prefix_fp4": _load("mxfp4_e2m1", [32768], [0], 32768, 8, 128, 64),
        # the next token of a decoding batch chooses 32 blocks of 64 keys per KV head (first block and last two always)
        "select_decode": _select(_ages(32, 4096, 32768), 1, 1, 1, 40, 8, 128, 64, 32, 1, 2),
        # whole drafted steps choose 128 of 2048 small blocks together
        "select_steps": _select([32768], 8, 64, 64, 40, 8, 128, 16, 128, 1, 4),
        # speculative tokens of six steps choose one by one (the paper's operating point)
        "select_tokens": _select([20011], 6, 9, 1, 40, 8, 128, 32, 64, 1, 1),
        # the decoding batch attends over what it selected, 4-bit cache
        "attend_decode_fp4": _attend("mxfp4_e2m1", _ages(32, 4096, 32768), 1, 1, 1, 40, 8, 128, 64, 32),
        # whole drafted steps over 32 blocks of 64 keys each, bf16 cache
        "attend_steps_bf16": _attend("bf16", [32768], 8, 64, 64, 40, 8, 128, 64, 32),
        # speculative tokens that selected one by one, 8-bit cache
        "attend_tokens_fp8": _attend("mxfp8_e4m3", [20011], 6, 9, 1, 40, 8, 128, 32, 64),
        # plain decoding of a batch over everything an 8-bit cache holds, four continuations each
        "attend_all_fp8": _attend("mxfp8_e4m3", _ages(8, 8192, 32768), 4, 1, 1, 64, 8, 128, 64, 0),
    }
    return [dict(c, name=n) for n, c in cases.items()]


# ------------------------------------------------------------------------------------------------ drawing

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    return rng.choice(((40, 8), (64, 8), (32, 8), (32, 4), (16, 2), (8, 8)))


def _draw_store(rng):
    d = rng.choice((64, 128, 128, 128, 256))
    if rng.random() < 0.5:   # tokens that join a cache: next tokens of a batch, or prompts
        n, L = _log_int(rng, 1, 48), _log_int(rng, 1, 8192)
        prefix = [rng.choice((0, _log_int(rng, 1, 4096))) for _ in range(n)]
        return _store(rng.choice(_FORMATS), prefix, [rng.randint(0 if L > 1 else 1, L) for _ in range(n)], L, rng.choice((2, 4, 8)),
                      d, rng.choice((16, 32, 64, 128)))
    n, L, chain = rng.choice((1, 1, 2, 4)), _log_int(rng, 1, 64), rng.choice((0, _log_int(rng, 1, 448)))
    return _store(rng.choice(_FORMATS), [_log_int(rng, 16, 8192) for _ in range(n)], [rng.randint(0, L) for _ in range(n)], L,
                  rng.choice((2, 4, 8)), d, rng.choice((16, 16, 64)), gamma=rng.randint(1, 8), chain=chain,
                  kept_chain=rng.randint(0, chain), layers=_log_int(rng, 1, 64))


def _draw_load(rng):
    n = _log_int(rng, 1, 16)
    prefix = [_log_int(rng, 1, 32768) for _ in range(n)]
    first = [rng.choice((0, rng.randint(0, p - 1))) for p in prefix]
    return _load(rng.choice(_FORMATS), prefix, first, max(1, max(p - f for p, f in zip(prefix, first)) - rng.randint(0, 3)),
                 rng.choice((2, 4, 8)), rng.choice((64, 128, 128, 128, 256)), rng.choice((16, 32, 64, 128)))


def _draw_passes(rng):
    """Shape of a pass: decoding batches, speculative tokens, drafted steps."""
    what = rng.choice(("decode", "tokens", "steps"))
    if what == "decode":
        return [_log_int(rng, 64, 32768) for _ in range(_log_int(rng, 1, 48))], rng.choice((1, 1, 4)), 1, 1
    if what == "tokens":
        return [_log_int(rng, 256, 32768) for _ in range(rng.choice((1, 1, 2)))], rng.randint(1, 8), rng.randint(3, 12), rng.choice((1, 1, 3))
    L = _log_int(rng, 8, 64)
    return [_log_int(rng, 256, 32768) for _ in range(rng.choice((1, 1, 2)))], rng.randint(1, 8), L, rng.choice((L, L, min(L, 16)))


def _draw_select(rng):
    prefix, gamma, L, group = _draw_passes(rng)
    hq, hkv = _heads(rng)
    block = rng.choice((16, 32, 64, 64, 128))
    most = _log_int(rng, 4, max(8, 4096 // block))
    return _select(prefix, gamma, L, group, hq, hkv, rng.choice((64, 128, 128, 128, 256)), block, most, rng.choice((0, 1, 1)),
                   rng.choice((0, 1, 2)))


def _draw_attend(rng):
    prefix, gamma, L, group = _draw_passes(rng)
    hq, hkv = _heads(rng)
    block = rng.choice((16, 32, 64, 64, 128))
    most = _log_int(rng, 4, max(8, 4096 // block)) if rng.random() < 0.8 else 0
    return _attend(rng.choice(_FORMATS), prefix, gamma, L, group, hq, hkv, rng.choice((64, 128, 128, 128, 256)), block, most)


def _affordable(c):
    if c["kind"] == "store":
        rows = (len(_numbers(c["prefix"])) * (c["gamma"] * c["L"] + c["chain"])) * c["layers"] * c["Hkv"] * c["D"] / 128
        return rows <= _MAX_STORE_ROWS and work(c)["bytes"] <= 1.0e8
    if c["kind"] == "load":
        return len(_numbers(c["prefix"])) * c["tokens"] * c["Hkv"] * c["D"] / 128 <= _MAX_LOAD_ROWS
    w = work(c)
    if c["kind"] == "select":
        return w["flops"] <= _MAX_SELECT_FLOPS and w["bytes"] <= _MAX_SELECT_BYTES
    keys = c["most"] * c["block"] * c["gamma"] * -(-c["L"] // c["group"]) if c["most"] else max(_numbers(c["prefix"]))
    gathered = len(_numbers(c["prefix"])) * c["Hkv"] * c["D"] * keys
    return w["flops"] <= _MAX_ATTEND_FLOPS and w["bytes"] <= _MAX_ATTEND_BYTES and gathered <= _MAX_ATTEND_GATHER


def draw(rng):
    family = rng.choice((_draw_store, _draw_load, _draw_select, _draw_select, _draw_attend, _draw_attend, _draw_attend))
    while True:
        c = family(rng)
        if _affordable(c):
            return c


# ------------------------------------------------------------------------------------------------ the cache's formats

def _pow2(e):
    """2^e of whole numbers -126..127, in 32 bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(x, fmt):
    """fp32 rows [.., D] -> (signed element values, exponents [.., D / 32]); a group's exponent is the smallest at which its
    largest magnitude does not exceed the largest element."""
    g = x.unflatten(-1, (-1, 32))
    m, e = torch.frexp(g.abs().amax(-1))
    if fmt == "mxfp8_e4m3":      # 448 = 0.875 * 2^9
        e = torch.where(m > 0.875, e - 8, e - 9)
    else:                        # 6 = 0.75 * 2^3
        e = torch.where(m > 0.75, e - 2, e - 3)
    e = torch.where(m == 0, torch.full_like(e, _EXP_MIN), e).clamp(_EXP_MIN, _EXP_MAX)
    y = g * _pow2(-e)[..., None]
    if fmt == "mxfp8_e4m3":
        y = y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float()
    else:
        a = y.abs().clamp(max=6.0)
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        y = torch.copysign(torch.round(a / step) * step, y)
    return y.flatten(-2), e


def _values(y, e):
    return (y.unflatten(-1, (-1, 32)) * _pow2(e)[..., None]).flatten(-2)


def _pack(y, fmt):
    if fmt == "bf16":
        return y.to(torch.bfloat16)
    if fmt == "mxfp8_e4m3":
        return y.to(torch.float8_e4m3fn)
    grid = torch.tensor(_GRID, device=y.device)
    code = torch.bucketize(y.abs(), grid).to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _unpack(codes, exps, fmt):
    """Stored rows -> fp32 values."""
    if fmt == "bf16":
        return codes.float()
    if fmt == "mxfp8_e4m3":
        return _values(codes.float(), exps.to(torch.int32) - 127)
    table = torch.tensor(_GRID + tuple(-v for v in _GRID), device=codes.device)
    y = torch.stack((table[(codes & 15).long()], table[(codes >> 4).long()]), -1).flatten(-2)
    return _values(y, exps.to(torch.int32) - 127)


# ------------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _i32(rows):
    return torch.tensor(rows, dtype=torch.int32, device="cuda")


def _paged(case, capacity, gen):
    """Block tables of requests of `capacity` tokens at most, blocks scattered over the pool."""
    n, per = len(_numbers(case["prefix"])), -(-capacity // case["block"])
    return torch.randperm(n * per, generator=gen, device="cuda").to(torch.int32).view(n, per).contiguous(), n * per


def _cache(case, shape, gen):
    """A filled cache [.., blocks, Hkv, block, D] of keys with a mean of their own per channel, and values."""
    out = {}
    for w in "kv":
        x = torch.randn(shape, generator=gen, device="cuda")
        if w == "k":
            x += torch.randn(shape[-1], generator=gen, device="cuda")
        if case["fmt"] == "bf16":
            out[w], out[w + "_exp"] = x.to(torch.bfloat16), None
        else:
            y, e = _quantise(x.to(torch.bfloat16).float(), case["fmt"])
            out[w], out[w + "_exp"] = _pack(y, case["fmt"]), (e + 127).to(torch.uint8)
    return out


def _prepare_store(case, gen):
    prefix, L, C, n_layers = _numbers(case["prefix"]), case["L"], case["chain"], case["layers"]
    n, hkv, d = len(prefix), case["Hkv"], case["D"]
    table, blocks = _paged(case, max(prefix) + C + L, gen)
    s = _cache(case, (n_layers, blocks, hkv, case["block"], d), gen)
    mean = torch.randn(d, generator=gen, device="cuda")
    s["k_bounds"] = torch.stack((mean - 1, mean + 1)).to(torch.bfloat16).expand(n_layers, blocks, hkv, 2, d).contiguous()
    for w in "kv":
        add = mean if w == "k" else 0.0
        s[w + "_branch"] = (torch.randn((n_layers, n, case["gamma"], L, hkv, d), generator=gen, device="cuda") + add).to(torch.bfloat16)
        s[w + "_chain"] = (torch.randn((n_layers, n, C, hkv, d), generator=gen, device="cuda") + add).to(torch.bfloat16) if C else None
    s.update(table=table, blocks=blocks, prefix_lens=_i32(prefix),
             src=torch.randint(0, case["gamma"], (n,), generator=gen, device="cuda").to(torch.int32),
             n_chain=_i32([case["kept_chain"]] * n), n_own=_i32(_numbers(case["own_len"])))
    return s


def _prepare_load(case, gen):
    prefix = _numbers(case["prefix"])
    table, blocks = _paged(case, max(prefix), gen)
    s = _cache(case, (1, blocks, case["Hkv"], case["block"], case["D"]), gen)
    s.update(table=table, blocks=blocks, prefix_lens=_i32(prefix), first=_i32(_numbers(case["first"])))
    return s


def _queries(case, gen):
    n = len(_numbers(case["prefix"]))
    q = torch.randn((n, case["gamma"], case["L"], case["Hq"], case["D"]), generator=gen, device="cuda")
    return q.to(torch.bfloat16)


def _prepare_select(case, gen):
    prefix = _numbers(case["prefix"])
    table, blocks = _paged(case, max(prefix), gen)
    shape = (blocks, case["Hkv"], case["D"])
    centre = 0.5 * torch.randn(shape, generator=gen, device="cuda") + torch.randn(case["D"], generator=gen, device="cuda")
    low = centre - 1.5 - 0.3 * torch.randn(shape, generator=gen, device="cuda").abs()
    high = centre + 1.5 + 0.3 * torch.randn(shape, generator=gen, device="cuda").abs()
    return {"table": table, "blocks": blocks, "prefix_lens": _i32(prefix), "q": _queries(case, gen),
            "k_bounds": torch.stack((low, high), 2).to(torch.bfloat16).contiguous()}


def _prepare_attend(case, gen):
    prefix, block, most = _numbers(case["prefix"]), case["block"], case["most"]
    n, hkv, gamma, L = len(prefix), case["Hkv"], case["gamma"], case["L"]
    table, blocks = _paged(case, max(prefix), gen)
    s = _cache(case, (1, blocks, hkv, block, case["D"]), gen)
    s.update(table=table, blocks=blocks, prefix_lens=_i32(prefix), q=_queries(case, gen), sel=None, count=None)
    for w in "kv":
        s[w + "_branch"] = torch.randn((n, gamma, L, hkv, case["D"]), generator=gen, device="cuda").to(torch.bfloat16)
    if most:
        # the last block and others at random, in ascending order
        have = _i32([-(-p // block) for p in prefix])[:, None, None, None, None]
        groups, width = -(-L // case["group"]), max(most, table.shape[1])
        at = torch.arange(width, device="cuda")
        score = torch.rand((n, gamma, groups, hkv, width), generator=gen, device="cuda")
        score = torch.where(at == have - 1, 2.0, torch.where(at < have, score, -1.0 - at))
        sel = score.topk(most, dim=-1).indices.sort(-1).values.to(torch.int32)
        s["count"] = have[..., 0].clamp(max=most).expand(n, gamma, groups, hkv).contiguous()
        s["sel"] = torch.where(torch.arange(most, device="cuda") < s["count"][..., None], sel, -1).contiguous()
    return s


def prepare(case, seed):
    gen = _generator(seed)
    s = {"store": _prepare_store, "load": _prepare_load, "select": _prepare_select, "attend": _prepare_attend}[case["kind"]](case, gen)
    s["case"] = case
    if own:
        _handles(case, s)
    return s


# ------------------------------------------------------------------------------------------------ the package's calls

def _handles(case, s):
    """Descriptors, workspaces and output buffers, which a program makes once for its shapes."""
    from paper_2506_19830_amd import binding as B
    kind, n, d = case["kind"], len(_numbers(case["prefix"])), case["D"]
    s["lens"] = list(_numbers(case["prefix"]))
    s["desc"] = B.make_attn_desc(
        num_requests=n, num_q_heads=case.get("Hq", case["Hkv"]), num_kv_heads=case["Hkv"], head_dim=d,
        gamma=case.get("gamma", 1), branch_len=case.get("L", 1), block_size=case["block"],
        max_blocks_per_request=s["table"].shape[1], q_dtype="bf16", kv_dtype=case.get("fmt", "bf16"), branch_kv_dtype="bf16",
        out_dtype="bf16", softmax_scale=d ** -0.5)
    empty = lambda shape, dtype: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
    if kind != "select":
        s["cache"] = B.make_block_cache(s["k"], s["v"], s["k_exp"], s["v_exp"], s.get("k_bounds"))
    if kind == "store":
        n_layers, C, L = case["layers"], case["chain"], case["L"]
        rows = n * case["Hkv"] * d
        s["strides"] = B.la_layer_strides(n_layers, s["blocks"] * case["block"] * case["Hkv"] * d, case["gamma"] * L * rows, C * rows, 0)
        s["back"] = B.la_layer_strides(n_layers, s["blocks"] * case["block"] * case["Hkv"] * d, (C + L) * rows, 0, 0)
        s["new_lens"] = empty(n, torch.int32)
        s["out"] = [empty((n_layers, n, C + L, case["Hkv"], d), torch.bfloat16) for _ in "kv"]
    elif kind == "load":
        s["out"] = [empty((n, case["tokens"], case["Hkv"], d), torch.bfloat16) for _ in "kv"]
    elif kind == "select":
        s["choice"] = B.make_select_desc(group_len=case["group"], max_blocks=case["most"], keep_first=min(case["keep_first"], case["most"]),
                                         keep_last=min(case["keep_last"], case["most"]))
        shape = (n, case["gamma"], -(-case["L"] // case["group"]), case["Hkv"])
        s["sel"], s["count"] = empty(shape + (case["most"],), torch.int32), empty(shape, torch.int32)
        s["workspace"] = empty(max(16, B.la_block_select_workspace(s["desc"], s["choice"], s["lens"])), torch.uint8)
    else:
        s["choice"] = B.make_select_desc(group_len=case["group"], max_blocks=case["most"]) if case["most"] else None
        s["out"] = empty(s["q"].shape, torch.bfloat16)
        s["lse"] = empty(s["q"].shape[:-1], torch.float32)
        s["workspace"] = empty(max(16, B.la_verify_attention_sparse_workspace(s["desc"], s["choice"], s["lens"])), torch.uint8)


def _run_own(s):
    from paper_2506_19830_amd import binding as B
    kind = s["case"]["kind"]
    if kind == "store":
        # the new rows join the cache and come back as it holds them (what a dense pass over the chunk itself attends to)
        B.la_kv_store(s["desc"], s["cache"], s["table"], s["prefix_lens"], s["lens"], s["k_branch"], s["v_branch"], s["k_chain"],
                      s["v_chain"], s["src"], s["n_chain"], s["n_own"], s["new_lens"], s["strides"])
        B.la_kv_load(s["desc"], s["cache"], s["table"], s["new_lens"], s["prefix_lens"], *s["out"], s["back"])
        return _stored(s, s["out"], s["new_lens"])
    if kind == "load":
        B.la_kv_load(s["desc"], s["cache"], s["table"], s["prefix_lens"], s["first"], *s["out"])
        return {"k": s["out"][0], "v": s["out"][1]}
    if kind == "select":
        B.la_block_select(s["desc"], s["choice"], s["q"], s["k_bounds"], s["table"], s["prefix_lens"], s["lens"], s["sel"], s["count"],
                          s["workspace"])
        return {"blocks": s["sel"], "count": s["count"]}
    B.la_verify_attention_sparse(s["desc"], s["choice"], s["q"], s["cache"], s["table"], s["prefix_lens"], s["lens"], s["sel"],
                                 s["count"], s["k_branch"], s["v_branch"], s["out"], s["lse"], s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


def _stored(s, values, new_lens):
    got = {"k": values[0], "v": values[1], "k_bounds": s["k_bounds"], "new_prefix_lens": new_lens}
    if s["k_exp"] is not None:
        got.update(k_exp=s["k_exp"], v_exp=s["v_exp"])
    return got


# ------------------------------------------------------------------------------------------------ the plain forms

def _appended(s, w):
    """The rows a store appends, [layers, B, C + L, Hkv, D] bf16, and which of them are real, [B, C + L]."""
    case, n = s["case"], len(_numbers(s["case"]["prefix"]))
    C, L = case["chain"], case["L"]
    t = torch.arange(C + L, device="cuda")
    kept, own_len = s["n_chain"].long()[:, None], s["n_own"].long()[:, None]
    real = t < kept + own_len
    each = torch.arange(n, device="cuda")[:, None]
    rows = s[w + "_branch"][:, each, s["src"].long()[:, None], (t - kept).clamp(0, L - 1)]
    if C:
        chain = s[w + "_chain"][:, each, t.clamp(max=C - 1).expand(n, -1)]
        rows = torch.where((t < kept)[..., None, None], chain, rows)
    return rows, real


def _plain_store(s):
    case, block = s["case"], s["case"]["block"]
    n_layers, hkv, d = case["layers"], case["Hkv"], case["D"]
    P, n = s["prefix_lens"].long(), len(_numbers(case["prefix"]))
    out, real = [], None
    for w in "kv":
        rows, real = _appended(s, w)
        b, t = real.nonzero(as_tuple=True)
        pos = P[b] + t
        phys = s["table"][b, pos // block].long()
        x = rows[:, b, t]                                                # [layers, tokens, Hkv, D]
        if case["fmt"] == "bf16":
            s[w][:, phys, :, pos % block] = x.transpose(0, 1)
            value = x.float()
        else:
            y, e = _quantise(x.float(), case["fmt"])
            store = s[w].view(torch.uint8) if case["fmt"] == "mxfp8_e4m3" else s[w]
            store[:, phys, :, pos % block] = _pack(y, case["fmt"]).view(torch.uint8).transpose(0, 1)
            s[w + "_exp"][:, phys, :, pos % block] = (e + 127).to(torch.uint8).transpose(0, 1)
            value = _values(y, e)
        back = torch.zeros_like(rows)
        back[:, b, t] = value.to(torch.bfloat16)
        out.append(back)
        if w == "k":
            # blocks that begin with a new token start afresh, the one the prefix ends in is widened
            starts = pos % block == 0
            s["k_bounds"][:, phys[starts], :, 0] = math.inf
            s["k_bounds"][:, phys[starts], :, 1] = -math.inf
            low, high = (s["k_bounds"][:, :, :, i].float().transpose(0, 1).contiguous() for i in (0, 1))
            low.index_reduce_(0, phys, value.transpose(0, 1).contiguous(), "amin")
            high.index_reduce_(0, phys, value.transpose(0, 1).contiguous(), "amax")
            s["k_bounds"].copy_(torch.stack((low, high), 3).transpose(0, 1))
    return _stored(s, out, (P + real.sum(-1)).to(torch.int32))


def _plain_load(s):
    case, block = s["case"], s["case"]["block"]
    pos = s["first"].long()[:, None] + torch.arange(case["tokens"], device="cuda")
    real = pos < s["prefix_lens"].long()[:, None]
    at = torch.where(real, pos, 0)
    phys = s["table"].gather(1, at // block).long()
    out = {}
    for w in "kv":
        exps = None if s[w + "_exp"] is None else s[w + "_exp"][0][phys, :, at % block]
        codes = s[w][0].view(torch.uint8) if case["fmt"] == "mxfp8_e4m3" else s[w][0]
        codes = codes[phys, :, at % block]
        codes = codes.view(torch.float8_e4m3fn) if case["fmt"] == "mxfp8_e4m3" else codes
        rows = _unpack(codes, exps, case["fmt"])
        out[w] = torch.where(real[..., None, None], rows, 0.0).to(torch.bfloat16)
    return out


def _grouped(case, q):
    """Queries [B, gamma, L, Hq, D] -> [B, gamma, groups, Hkv, rows, D], short last groups filled with their first token."""
    L, g, hkv = case["L"], case["group"], case["Hkv"]
    groups = -(-L // g)
    t = torch.arange(groups * g, device="cuda")
    t = torch.where(t < L, t, (groups - 1) * g)
    x = q[:, :, t].unflatten(2, (groups, g)).unflatten(4, (hkv, -1))    # [B, gamma, groups, g, Hkv, G, D]
    return x.permute(0, 1, 2, 4, 3, 5, 6).flatten(4, 5)


def _ungrouped(case, x):
    """The way back, [B, gamma, groups, Hkv, rows, ..] -> [B, gamma, L, Hq, ..]."""
    x = x.unflatten(4, (case["group"], -1))
    order = (0, 1, 2, 4, 3, 5) + tuple(range(6, x.dim()))
    return x.permute(order).flatten(2, 3)[:, :, :case["L"]].flatten(3, 4)


def _choose(case, score, have):
    """score [B, gamma, groups, Hkv, N] -> the chosen blocks in ascending order (-1 behind the last), and their number."""
    most = case["most"]
    first, last = min(case["keep_first"], most), min(case["keep_last"], most)
    have = have[:, None, None, None, None]
    at = torch.arange(score.shape[-1], device="cuda")
    score = torch.where((at < first) | (at >= have - last), math.inf, score)
    score = torch.where(at < have, score, -math.inf)
    if score.shape[-1] < most:
        score = torch.nn.functional.pad(score, (0, most - score.shape[-1]), value=-math.inf)
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :most]
    count = have[..., 0].clamp(max=most).expand(score.shape[:-1])
    chosen = torch.where(torch.arange(most, device="cuda") < count[..., None], order, 1 << 30).sort(-1).values
    return torch.where(chosen == 1 << 30, -1, chosen).to(torch.int32), count.to(torch.int32).contiguous()


def _plain_select(s):
    case = s["case"]
    # the score of a block decides between neighbours: 64 bits
    q = _grouped(case, s["q"]).double()                                  # [B, gamma, groups, Hkv, rows, D]
    bounds = s["k_bounds"][s["table"].long()].double()                   # [B, N, Hkv, 2, D]
    bounds = bounds.permute(0, 2, 3, 4, 1).flatten(2, 3).contiguous()    # [B, Hkv, 2 D, N]
    signed = torch.cat((q.clamp(max=0), q.clamp(min=0)), -1)             # below 0 with the smallest, above with the largest key
    B, gamma, groups, hkv, rows, _ = q.shape
    signed = signed.permute(0, 3, 1, 2, 4, 5).flatten(2, 4).contiguous()
    score = torch.matmul(signed, bounds).unflatten(2, (gamma, groups, rows)).amax(4)
    have = -(-s["prefix_lens"].long() // case["block"])
    chosen, count = _choose(case, score.permute(0, 2, 3, 1, 4), have)
    return {"blocks": chosen, "count": count}


def _softmax_part(q, k, v, seen, scale):
    """(maximum, sum, weighted values) of rows q over keys k where `seen`; nothing seen: (-inf, 0, 0)."""
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()) * scale
    x = torch.where(seen, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    return m, p.sum(-1, keepdim=True), torch.matmul(p, v)


def _plain_attend(s):
    case, block, scale = s["case"], s["case"]["block"], s["case"]["D"] ** -0.5
    n, gamma, L, hkv = len(_numbers(case["prefix"])), case["gamma"], case["L"], case["Hkv"]
    P = s["prefix_lens"].long()
    heads = torch.arange(hkv, device="cuda")
    off = torch.arange(block, device="cuda")
    q = s["q"].float()
    if case["most"]:
        rows = _grouped(case, q)
        sel = s["sel"].long()                                            # [B, gamma, groups, Hkv, most]
        phys = s["table"].long()[torch.arange(n, device="cuda")[:, None, None, None, None], sel.clamp(min=0)]
        seen = ((sel >= 0)[..., None] & (sel[..., None] * block + off < P[:, None, None, None, None, None])).flatten(-2)
        at = (phys, heads[:, None])
    else:                                                                # every block, rows of all branches together
        rows = q.unflatten(3, (hkv, -1)).permute(0, 3, 1, 2, 4, 5).flatten(2, 4)
        blocks = torch.arange(s["table"].shape[1], device="cuda")
        seen = (blocks[:, None] * block + off < P[:, None, None]).flatten(-2)[:, None]
        at = (s["table"].long()[:, None], heads[:, None])
    parts = []
    for w in "kv":
        exps = None if s[w + "_exp"] is None else s[w + "_exp"][0][at]
        codes = s[w][0].view(torch.uint8) if case["fmt"] == "mxfp8_e4m3" else s[w][0]
        codes = codes[at]
        codes = codes.view(torch.float8_e4m3fn) if case["fmt"] == "mxfp8_e4m3" else codes
        parts.append(_unpack(codes, exps, case["fmt"]).flatten(-3, -2))
    prefix = _softmax_part(rows, parts[0], parts[1], seen[..., None, :], scale)
    if case["most"]:
        prefix = [_ungrouped(case, x) for x in prefix]
    else:
        prefix = [x.unflatten(2, (gamma, L, -1)).permute(0, 2, 3, 1, 4, 5).flatten(3, 4) for x in prefix]
    # the branch's own tokens, up to the query's own
    mine = q.unflatten(3, (hkv, -1)).permute(0, 1, 3, 2, 4, 5).flatten(3, 4)     # [B, gamma, Hkv, L * G, D]
    k, v = (s[w + "_branch"].float().transpose(2, 3).contiguous() for w in "kv")
    i = torch.arange(L, device="cuda")
    causal = (i <= i[:, None]).repeat_interleave(case["Hq"] // hkv, 0)
    own_part = _softmax_part(mine, k, v, causal, scale)
    own_part = [x.unflatten(3, (L, -1)).permute(0, 1, 3, 2, 4, 5).flatten(3, 4) for x in own_part]
    m = torch.maximum(prefix[0], own_part[0])
    a, b = torch.exp(prefix[0] - m), torch.exp(own_part[0] - m)
    total = a * prefix[1] + b * own_part[1]
    return {"out": ((a * prefix[2] + b * own_part[2]) / total).to(torch.bfloat16), "lse": (m + torch.log(total))[..., 0].contiguous()}


def run(state):
    if own:
        return _run_own(state)
    return {"store": _plain_store, "load": _plain_load, "select": _plain_select, "attend": _plain_attend}[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------ what it takes

def work(case):
    prefix, hkv, d = _numbers(case["prefix"]), case["Hkv"], case["D"]
    if case["kind"] == "store":
        tokens = sum(_numbers(case["own_len"])) + len(prefix) * case["kept_chain"]
        rows = case["layers"] * hkv * tokens
        # written from bf16 rows, and read back into bf16 rows; bounds of whole blocks
        per = 2 * (2 * d + 2 * _ROW_BYTES[case["fmt"]](d) + 2 * d)
        return {"bytes": float(rows * per + 4 * d * rows / case["block"]), "flops": 0.0}
    if case["kind"] == "load":
        tokens = sum(max(0, min(case["tokens"], p - f)) for p, f in zip(prefix, _numbers(case["first"])))
        return {"bytes": float(2 * tokens * hkv * (_ROW_BYTES[case["fmt"]](d) + 2 * d)), "flops": 0.0}
    n, gamma, L, hq, block = len(prefix), case["gamma"], case["L"], case["Hq"], case["block"]
    groups, most = gamma * -(-L // case["group"]), case["most"]
    have = [-(-p // block) for p in prefix]
    if case["kind"] == "select":
        scored = [h if h > most else 0 for h in have]   # a prefix that fits is taken whole, unseen
        return {"bytes": float(sum(scored) * hkv * 4 * d + n * gamma * L * hq * 2 * d + 4 * n * groups * hkv * (most + 1)),
                "flops": 2.0 * sum(scored) * gamma * L * hq * 2 * d}
    rows = n * gamma * L * hq
    keys = [min(p, most * block) if most else p for p in prefix]
    if most:   # distinct blocks that `groups` selections name between them
        read = [hkv * min(p, block * h * (1.0 - (1.0 - min(most, h) / h) ** groups)) for p, h in zip(prefix, have)]
    else:
        read = [hkv * p for p in prefix]
    flops = 4.0 * d * hq * gamma * (L * sum(keys) + n * L * (L + 1) / 2)
    return {"bytes": float(2 * sum(read) * _ROW_BYTES[case["fmt"]](d) + 4 * n * gamma * L * hkv * d + rows * (4 * d + 4) +
                           (4 * n * groups * hkv * most)), "flops": flops}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits

def _power(e):
    """2^e in 64 bits, from a table: a device's pow() may be off in the last place."""
    return torch.tensor([2.0 ** k for k in range(-160, 161)], dtype=torch.float64, device=e.device)[e.long() + 160]


def _nearest(x, fmt):
    """Group by group: the power of two, then the nearest element, ties to the one with the even code.  x: float64 [.., D]."""
    grid = torch.tensor(_GRID, dtype=torch.float64, device=x.device)
    if fmt == "mxfp8_e4m3":
        code = torch.arange(127, device=x.device)
        e, m = (code >> 3).double(), (code & 7).double()
        grid = torch.where(code < 8, m * 2.0 ** -9, (1 + m / 8) * _power(e - 7))
    g = x.reshape(x.shape[:-1] + (-1, 32))
    top = g.abs().amax(-1)
    powers = torch.arange(_EXP_MIN, _EXP_MAX, device=x.device)
    limits = grid[-1] * _power(powers)
    e = _EXP_MIN + torch.searchsorted(limits, top.contiguous())
    y = g / _power(e)[..., None]
    a = y.abs().contiguous()
    middle = (grid[1:] + grid[:-1]) / 2
    code = torch.searchsorted(middle, a)             # values on a middle go down here
    tie = (code < middle.numel()) & (a == middle[code.clamp(max=middle.numel() - 1)])
    code = torch.where(tie & (code % 2 == 1), code + 1, code)
    return (torch.sign(y) * grid[code] * _power(e)[..., None]).reshape(x.shape), e


def _exact_store(s):
    case, block, n = s["case"], s["case"]["block"], len(_numbers(s["case"]["prefix"]))
    C, L, src = case["chain"], case["L"], s["src"].tolist()
    shape = (case["layers"], n, C + L, case["Hkv"], case["D"])
    out = {"k": torch.zeros(shape, dtype=torch.float64, device="cuda"), "v": torch.zeros(shape, dtype=torch.float64, device="cuda")}
    bounds, lens = s["k_bounds"].double(), []
    for b, (p, own_len) in enumerate(zip(_numbers(case["prefix"]), _numbers(case["own_len"]))):
        kept = case["kept_chain"]
        lens.append(p + kept + own_len)
        for w in "kv":
            rows = s[w + "_branch"][:, b, src[b], :own_len]
            if kept:
                rows = torch.cat((s[w + "_chain"][:, b, :kept], rows), 1)
            rows = rows.double()
            if rows.shape[1]:
                out[w][:, b, :kept + own_len] = rows if case["fmt"] == "bf16" else _nearest(rows, case["fmt"])[0]
        for j in range(p // block, -(-lens[-1] // block)):
            phys, first = int(s["table"][b, j]), max(p, j * block)
            held = out["k"][:, b, first - p:min(lens[-1], (j + 1) * block) - p]
            if not held.shape[1]:
                continue
            low, high = held.amin(1), held.amax(1)
            if first > j * block:
                low, high = torch.minimum(low, bounds[:, phys, :, 0]), torch.maximum(high, bounds[:, phys, :, 1])
            bounds[:, phys, :, 0], bounds[:, phys, :, 1] = low, high
    return {**out, "k_bounds": bounds, "new_prefix_lens": torch.tensor(lens), "k_exp": None, "v_exp": None}


def _held(s, w, phys):
    """The values of whole blocks, float64, decoded element by element from a table of the codes."""
    fmt, codes = s["case"]["fmt"], s[w][0][phys] if s["case"]["fmt"] != "mxfp8_e4m3" else s[w][0].view(torch.uint8)[phys]
    if fmt == "bf16":
        return codes.double()
    if fmt == "mxfp8_e4m3":
        c = torch.arange(256)
        e, m = ((c >> 3) & 15).double(), (c & 7).double()
        table = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7)) * torch.where(c > 127, -1.0, 1.0)
        y = table.double().cuda()[codes.long()]
    else:
        table = torch.tensor([[(-1 if c & 8 else 1) * _GRID[c & 7] for c in (b & 15, b >> 4)] for b in range(256)], dtype=torch.float64, device="cuda")
        y = table[codes.long()].flatten(-2)
    return y * _power(s[w + "_exp"][0][phys].long() - 127).repeat_interleave(32, -1)


def _exact_load(s):
    case, block = s["case"], s["case"]["block"]
    out = {w: torch.zeros((len(_numbers(case["prefix"])), case["tokens"], case["Hkv"], case["D"]), dtype=torch.float64, device="cuda") for w in "kv"}
    for b, (p, f) in enumerate(zip(_numbers(case["prefix"]), _numbers(case["first"]))):
        end = min(p, f + case["tokens"])
        phys = s["table"][b, f // block:-(-end // block)].long()
        for w in "kv":
            rows = _held(s, w, phys).transpose(1, 2).flatten(0, 1)       # [tokens, Hkv, D]
            out[w][b, :end - f] = rows[f % block:f % block + end - f]
    return out


def _exact_select(s):
    case = s["case"]
    if work(case)["flops"] > 3e10:
        return None
    groups, most = -(-case["L"] // case["group"]), case["most"]
    n, gamma, hkv = len(_numbers(case["prefix"])), case["gamma"], case["Hkv"]
    first, last = min(case["keep_first"], most), min(case["keep_last"], most)
    blocks = torch.full((n, gamma, groups, hkv, most), -1, dtype=torch.int32, device="cuda")
    count = torch.zeros((n, gamma, groups, hkv), dtype=torch.int32, device="cuda")
    per = case["Hq"] // hkv
    for b, p in enumerate(_numbers(case["prefix"])):
        have = -(-p // case["block"])
        count[b] = min(have, most)
        if have <= most:
            blocks[b, ..., :have] = torch.arange(have, device="cuda")
            continue
        bounds = s["k_bounds"][s["table"][b, :have].long()].double()     # [N, Hkv, 2, D]
        for g in range(gamma):
            q = s["q"][b, g].double().unflatten(1, (hkv, per))           # [L, Hkv, G, D]
            best = torch.full((groups, hkv, have), -math.inf, dtype=torch.float64, device="cuda")
            for t in range(case["L"]):
                for h in range(per):
                    x = q[t, :, h]                                       # [Hkv, D]
                    score = torch.maximum(x * bounds[:, :, 0], x * bounds[:, :, 1]).sum(-1).T
                    best[t // case["group"]] = torch.maximum(best[t // case["group"]], score)
            best[..., :first] = math.inf
            if last:
                best[..., have - last:] = math.inf
            order = torch.argsort(-best, dim=-1, stable=True)[..., :most]
            blocks[b, g] = order.sort(-1).values.to(torch.int32)
    return {"blocks": blocks, "count": count}


def _exact_attend(s):
    case, block, scale = s["case"], s["case"]["block"], s["case"]["D"] ** -0.5
    hkv, most, group = case["Hkv"], case["most"], case["group"]
    per = case["Hq"] // hkv
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:-1], dtype=torch.float64, device="cuda")
    for b, p in enumerate(_numbers(case["prefix"])):
        have = -(-p // block)
        at = torch.arange(have * block, device="cuda").view(have, block)
        k, v = (_held(s, w, s["table"][b, :have].long()) for w in "kv")  # [N, Hkv, block, D]
        for g in range(case["gamma"]):
            for h in range(hkv):
                mine = [s[w + "_branch"][b, g, :, h].double() for w in "kv"]
                for first in range(0, case["L"], group if most else case["L"]):
                    last = min(case["L"], first + group) if most else case["L"]
                    names = s["sel"][b, g, first // group, h] if most else torch.arange(have, device="cuda")
                    names = names[names >= 0].long()
                    real = (at[names] < p).flatten()
                    kk = torch.cat((k[names, h].flatten(0, 1)[real], mine[0]))
                    vv = torch.cat((v[names, h].flatten(0, 1)[real], mine[1]))
                    x = s["q"][b, g, first:last, h * per:(h + 1) * per].double().flatten(0, 1) @ kk.T.contiguous() * scale
                    n_own = torch.arange(first, last, device="cuda").repeat_interleave(per) + 1
                    behind = torch.arange(kk.shape[0], device="cuda") - int(real.sum())
                    x = x.masked_fill(behind >= n_own[:, None], -math.inf)
                    lse[b, g, first:last, h * per:(h + 1) * per] = torch.logsumexp(x, -1).view(last - first, per)
                    out[b, g, first:last, h * per:(h + 1) * per] = (torch.softmax(x, -1) @ vv).view(last - first, per, -1)
    return {"out": out, "lse": lse}


def exact(case, seed):
    gen = _generator(seed)
    s = {"store": _prepare_store, "load": _prepare_load, "select": _prepare_select, "attend": _prepare_attend}[case["kind"]](case, gen)
    s["case"] = case
    return {"store": _exact_store, "load": _exact_load, "select": _exact_select, "attend": _exact_attend}[case["kind"]](s)
