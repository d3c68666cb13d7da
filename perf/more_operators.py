"""Operators beside the decode step: a KV cache held in 4 bits, and the attention of whole prompts, as cases that can
be timed and compared.

A cache in 4 bits holds 3.2 times the tokens of one in 16: new tokens are normed, rotated, rounded to codes and
written to their slots, and read back ("append4": what a later chunk of the prompt will see of them), slots' values
are brought back to 16 bits ("read4"), and single queries attend over the codes ("attend4").  "prompt" is the
attention of the tokens that a step's bulk append has just written: whole prompts or chunks of them, packed one after
another, each query over the earlier tokens of its own request.

`run` computes them in plain torch where `own` is false and through paper_2608_02244_gb300.kv where it is true.
Lengths are quantiles of the lognormals of paper_2608_02244_gb300/workloads.py, so that the multiset (and with it
the work) goes by the case alone; their order, the blocks and all values go by the seed.

The format: 32 neighbouring values of a head are a group with a scale S and an offset B of the cache's type T; the
code c of a value stands for T(B + (1 + c / 16) S).  Two codes make a byte, the first in its low bits.
"""
from __future__ import annotations

import math
import statistics

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-6
GROUP = 32


# ------------------------------------------------------------------- cases
def _append4(name, tokens, heads, kv_heads, dim, rot, pairs, norm, block, kind, order, positions):
    """`tokens` new tokens; `rot` of the `dim` values of a head are rotated, as neighbours ("pairs") or as halves;
    `order` is the cache's: tokens of a block outermost ("token") or heads ("head")."""
    c = {"op": "append4", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rot": rot, "pairs": pairs,
         "norm": norm, "block": block, "kind": kind, "order": order, "positions": positions}
    return dict(c, name=name) if name else c


def _read4(name, tokens, kv_heads, dim, block, kind, order):
    c = {"op": "read4", "tokens": tokens, "heads": kv_heads, "kv_heads": kv_heads, "dim": dim, "block": block, "kind": kind,
         "order": order}
    return dict(c, name=name) if name else c


def _attend4(name, rows, heads, kv_heads, dim, block, kind, order, median, sigma, longest, idle, window, sinks, prefix):
    """One query for each of `rows` requests, `idle` of them empty; `prefix` tokens are shared by all and come before
    each request's own."""
    c = {"op": "attend4", "rows": rows, "heads": heads, "kv_heads": kv_heads, "dim": dim, "block": block, "kind": kind,
         "order": order, "median": median, "sigma": sigma, "longest": longest, "idle": idle, "window": window, "sinks": sinks,
         "prefix": prefix}
    return dict(c, name=name) if name else c


def _prompt(name, rows, heads, kv_heads, dim, block, kind, order, median, sigma, longest, idle, before, window, sinks, prefix):
    """`rows` requests of which each brings a prompt's tokens, but `idle` bring none; `before` tokens of each are in the
    cache from earlier chunks (at least half of that, spread evenly), `prefix` tokens are shared by all."""
    c = {"op": "prompt", "rows": rows, "heads": heads, "kv_heads": kv_heads, "dim": dim, "block": block, "kind": kind,
         "order": order, "median": median, "sigma": sigma, "longest": longest, "idle": idle, "before": before,
         "window": window, "sinks": sinks, "prefix": prefix}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decode step of the online workload's batch: 256 slots
        _append4("append4_256", 256, 32, 8, 128, 128, False, True, 16, "bf16", "head", 4096),
        # a prefill's worth of tokens at odd sizes: seven query heads on each key head, half of each head turned as pairs
        _append4("append4_20011_pairs", 20011, 28, 4, 64, 32, True, True, 8, "fp16", "token", 16384),
        # one request's tokens, before its next chunk
        _read4("read4_777", 777, 8, 128, 16, "bf16", "head"),
        # many requests' tokens: a batch of chunks goes on
        _read4("read4_98309", 98309, 8, 128, 32, "bf16", "token"),
        # a single short request: latency counts
        _attend4("attend4_1", 1, 32, 8, 128, 16, "bf16", "head", 777, 0.0, 777, 0, 0, 0, 0),
        # odd sizes: seven query heads on each key head, an odd window and first tokens, small blocks
        _attend4("attend4_61_odd", 61, 28, 4, 64, 8, "fp16", "token", 2000, 1.0, 16384, 2, 1777, 5, 0),
        # the online workload's batch, all of its tokens
        _attend4("attend4_256", 256, 32, 8, 128, 16, "bf16", "head", 640, 1.0, 6144, 3, 0, 0, 0),
        # the long-context batch: 512 slots with more than a million tokens
        _attend4("attend4_512", 512, 64, 8, 128, 32, "bf16", "head", 2048, 0.6, 8192, 5, 0, 0, 0),
        # one short prompt: latency counts
        _prompt("prompt_1", 1, 32, 8, 128, 16, "bf16", "token", 23, 0.0, 23, 0, 0, 0, 0, 0),
        # a refill of many slots at odd sizes: ragged prompts, seven query heads on each key head, a window
        _prompt("prompt_37_odd", 37, 28, 4, 64, 8, "fp16", "head", 300, 1.0, 2048, 2, 0, 777, 5, 0),
        # chunks of long prompts: few queries for each over tens of thousands of tokens, a shared system prompt
        _prompt("prompt_4_chunks", 4, 32, 8, 128, 64, "bf16", "token", 512, 0.0, 512, 0, 32000, 0, 0, 1024),
        # one long document
        _prompt("prompt_16384", 1, 32, 8, 128, 32, "bf16", "token", 16384, 0.0, 16384, 0, 0, 0, 0, 0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more step of the listed ranges: one token to 49,152 of append4 and 98,309 of read4, one to 512 single queries
    over one token to 16,384, prompts of one token to 16,384 over up to 32,768 earlier ones."""
    op = rng.choice(["append4", "read4", "attend4", "attend4", "prompt", "prompt", "prompt"])
    block = rng.choice([8, 16, 32, 64, 128])
    kind, order = rng.choice(["bf16", "bf16", "fp16"]), rng.choice(["head", "token"])
    kv_heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16])
    while kv_heads * group > 64:
        group = max(1, group // 2)
    dim = rng.choice([64, 128, 128, 256])
    heads, size = kv_heads * group, kv_heads * dim
    if op == "append4":
        tokens = _log(rng, 1, max(1, min(49152, 98309 * 1024 // (heads * dim + 4 * size))))
        return _append4(None, tokens, heads, kv_heads, dim, rng.choice([dim, dim, dim // 2]), rng.random() < 0.3,
                        rng.random() < 0.8, block, kind, order, _log(rng, 64, 49152))
    if op == "read4":
        return _read4(None, _log(rng, 1, min(98309, 98309 * 1024 // size)), kv_heads, dim, block, kind, order)
    if op == "attend4":
        rows = _log(rng, 1, 512)
        longest = _log(rng, 1, min(16384, max(64, 512 * 8192 * 1024 // (rows * size * 2))))
        window = rng.choice([0, 0, _log(rng, 16, 4096)])
        prefix = rng.choice([0, 0, 0, block * rng.randint(1, 16)])
        return _attend4(None, rows, heads, kv_heads, dim, block, kind, order, max(1, longest // rng.randint(1, 12)),
                        round(rng.uniform(0.0, 1.2), 2), longest, min(rows - 1, rng.randint(0, 5)), window,
                        rng.choice([0, 1, 4, 33]) if window else 0, prefix)
    rows = _log(rng, 1, 64)
    most = 16384 * 16384 * 32 * 128 // (rows * heads * dim)          # queries times tokens of each row
    before = rng.choice([0, 0, _log(rng, 1, 32768)])
    prefix = rng.choice([0, 0, 0, block * rng.randint(1, 16)])
    longest = max(1, min(16384, int(math.sqrt(most / 2)), most // (2 * (before + prefix + 1))))
    longest = _log(rng, 1, longest)
    window = rng.choice([0, 0, _log(rng, 16, 4096)])
    return _prompt(None, rows, heads, kv_heads, dim, block, kind, order, max(1, longest // rng.randint(1, 8)),
                   round(rng.uniform(0.0, 1.2), 2), longest, min(rows - 1, rng.randint(0, 3)), before, window,
                   rng.choice([0, 1, 4, 33]) if window else 0, prefix)


# ------------------------------------------------------------------- inputs
def _lengths(n, median, sigma, longest):
    """The n quantiles of a lognormal, rounded, in 1..longest."""
    normal = statistics.NormalDist()
    return [min(longest, max(1, round(median * math.exp(sigma * normal.inv_cdf((i + 0.5) / n))))) for i in range(n)]


def _blocks(n, block):
    return -(-n // block)


def _own_lengths(case):
    """Of each row: the tokens of an attend4 case, the new tokens of a prompt."""
    return _lengths(case["rows"] - case["idle"], case["median"], case["sigma"], case["longest"]) + [0] * case["idle"]


def _before(case):
    """Of each row of a prompt case, tokens of earlier chunks."""
    b, n = case["before"], case["rows"]
    return [b - (b // 2) * i // n for i in range(n)]


def _ordered(shape, order, make):
    """[blocks, block, kv_heads, ...] in the case's order of axes."""
    if order == "token":
        return make(shape)
    return make((shape[0], shape[2], shape[1]) + shape[3:]).transpose(1, 2)


def _cache(case, blocks, g):
    return _ordered((blocks, case["block"], case["kv_heads"], case["dim"]), case["order"],
                    lambda s: torch.randn(s, generator=g, device="cuda", dtype=TYPES[case["kind"]]))


def _cache4(case, blocks, g, filled):
    """Codes of keys and values, and their scales and offsets; filled: values of about normal size."""
    dim, dt = case["dim"], TYPES[case["kind"]]
    shape = (blocks, case["block"], case["kv_heads"])

    def codes(s):
        if not filled:
            return torch.zeros(s, device="cuda", dtype=torch.uint8)
        x, y = (torch.randint(0, 256, s, generator=g, device="cuda", dtype=torch.uint8) & 0x77 for _ in range(2))
        return x + y                                    # both codes of a byte are sums of two of 0..7

    def scales(s):
        if not filled:
            return torch.zeros(s, device="cuda", dtype=dt)
        x = 4.8 * (1 + 0.1 * torch.randn(s[:-1], generator=g, device="cuda")).clamp(0.5, 1.5)
        b = -(1 + 7 / 16) * x + 0.1 * torch.randn(s[:-1], generator=g, device="cuda")
        return torch.stack((x, b), -1).to(dt)

    return tuple(_ordered(shape + tail, case["order"], make)
                 for tail, make in (((dim // 2,), codes), ((dim // 2,), codes), ((dim // GROUP, 2), scales),
                                    ((dim // GROUP, 2), scales)))


def _rope(positions, rot):
    """cos then sin of each position's angles, [positions, rot] in 32 bits."""
    inv = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * inv
    return torch.cat((angle.cos(), angle.sin()), 1).float().contiguous()


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def prepare(case, seed):
    rng = np.random.Generator(np.random.PCG64(np.random.SeedSequence([seed, 78])))
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, bs, dt, dim, hq, hkv = case["op"], case["block"], TYPES[case["kind"]], case["dim"], case["heads"], case["kv_heads"]
    s = {"case": case}
    if op in ("append4", "read4"):
        n = case["tokens"]
        blocks = _blocks(n + n // 8, bs) + 1
        slots = rng.permutation(blocks * bs)[:n].astype(np.int64)
        if n > 8:                                   # a few places of the step's slot map are empty
            slots[rng.integers(1, n, size=n // 50)] = -1
        s.update(slots=torch.from_numpy(slots).cuda(), cache4=_cache4(case, blocks, g, op == "read4"))
        if op == "append4":
            s.update(qkv=torch.randn(n, (hq + 2 * hkv) * dim, generator=g, device="cuda", dtype=dt),
                     positions=_i32(rng.integers(0, case["positions"], size=n)), rope=_rope(case["positions"], case["rot"]),
                     q_weight=None, k_weight=None)
            if case["norm"]:
                s["q_weight"] = (1 + 0.2 * torch.randn(dim, generator=g, device="cuda")).to(dt)
                s["k_weight"] = (1 + 0.2 * torch.randn(dim, generator=g, device="cuda")).to(dt)
        return s
    order = rng.permutation(case["rows"])
    new = np.array(_own_lengths(case), np.int32)[order]
    lens = new + np.array(_before(case), np.int32)[order] if op == "prompt" else new
    own_blocks = -(-lens // bs)
    held, shared = int(own_blocks.sum()), case["prefix"] // bs
    blocks = held + shared + 3
    ids = rng.permutation(blocks).astype(np.int32)
    width = max(1, int(own_blocks.max()))
    table = np.full((case["rows"], width), -1, np.int32)
    table[np.arange(width)[None, :] < own_blocks[:, None]] = ids[:held]
    s.update(lens=_i32(lens), table=_i32(table), shared=_i32(ids[held:held + shared]) if shared else None)
    if op == "attend4":
        s.update(q=torch.randn(case["rows"], hq, dim, generator=g, device="cuda", dtype=dt),
                 cache4=_cache4(case, blocks, g, True))
    else:
        s.update(q=torch.randn(int(new.sum()), hq, dim, generator=g, device="cuda", dtype=dt),
                 starts=_i32(np.concatenate(([0], np.cumsum(new)))), k=_cache(case, blocks, g), v=_cache(case, blocks, g))
    return s


# ------------------------------------------------------------------- one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return {"append4": _own_append4, "read4": _own_read4, "attend4": _own_attend4, "prompt": _own_prompt}[op](s)
    return {"append4": _plain_append4, "read4": _plain_read4, "attend4": _plain_attend4, "prompt": _plain_prompt}[op](s)


_decoders = {}


def _decoder(s):
    """The handle that a serving program keeps for its cache's shape."""
    c = s["case"]
    blocks = (s["cache4"][0] if "cache4" in s else s["k"]).shape[0]
    key = (blocks, c["block"], c["heads"], c["kv_heads"], c["dim"], TYPES[c["kind"]], c.get("rows", 1))
    if key not in _decoders:
        from paper_2608_02244_gb300 import kv
        _decoders[key] = kv.Decoder(*key[:5], dtype=key[5], max_rows=key[6])
    return _decoders[key]


def _own_append4(s):
    d = _decoder(s)
    q = d.append4(s["qkv"], s["positions"], s["slots"], s["cache4"], s["rope"], s["q_weight"], s["k_weight"], eps=EPS,
                  pairs=s["case"]["pairs"])
    k, v = d.read4(s["slots"], s["cache4"])
    return {"q": q, "k": k, "v": v}


def _own_read4(s):
    k, v = _decoder(s).read4(s["slots"], s["cache4"])
    return {"k": k, "v": v}


def _own_attend4(s):
    c = s["case"]
    out, lse = _decoder(s).attend4(s["q"], s["cache4"], s["table"], s["lens"], prefix=s["shared"], window=c["window"],
                                   sinks=c["sinks"], lse=True)
    return {"out": out, "lse": lse}


def _own_prompt(s):
    c = s["case"]
    out, lse = _decoder(s).prompt(s["q"], s["k"], s["v"], s["table"], s["starts"], s["lens"], prefix=s["shared"],
                                  window=c["window"], sinks=c["sinks"], lse=True)
    return {"out": out, "lse": lse}


def _values(codes, scales):
    """What codes [..., dim / 2] with scales and offsets [..., dim / 32, 2] stand for, in 32 bits rounded to their type."""
    c = torch.stack((codes & 15, codes >> 4), -1).reshape(scales.shape[:-1] + (GROUP,))
    x = scales.float()
    return (x[..., 1:] + (1 + c.float() / 16) * x[..., :1]).to(scales.dtype).flatten(-2)


def _coded(x, dt):
    """Codes, and scales with offsets, of values [..., dim] in 32 bits."""
    x = x.reshape(x.shape[:-1] + (-1, GROUP))
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale = ((hi - lo) * (16 / 15)).to(dt).float()
    offset = (lo - scale).to(dt).float()
    c = torch.round((x - offset) / torch.where(scale > 0, scale, 1) * 16 - 16)
    c = torch.where(scale > 0, c.clamp(0, 15), 0).to(torch.uint8).flatten(-2)
    return c[..., ::2] | c[..., 1::2] << 4, torch.cat((scale, offset), -1).to(dt)


def _plain_append4(s):
    c = s["case"]
    n, hq, hkv, dim, rot = c["tokens"], c["heads"], c["kv_heads"], c["dim"], c["rot"]
    dt = s["qkv"].dtype
    x = s["qkv"].view(n, hq + 2 * hkv, dim).float()
    qk, v = x[:, :hq + hkv], x[:, hq + hkv:]
    if s["q_weight"] is not None:
        w = torch.cat((s["q_weight"].float().expand(hq, dim), s["k_weight"].float().expand(hkv, dim)))
        qk = qk * torch.rsqrt(qk.square().mean(-1, keepdim=True) + EPS) * w
    angle = s["rope"][s["positions"].long()][:, None]
    cos, sin = angle[..., :rot // 2], angle[..., rot // 2:]
    if c["pairs"]:
        a, b = qk[..., 0:rot:2], qk[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = qk[..., :rot // 2], qk[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    qk = torch.cat((turned, qk[..., rot:]), -1)
    real = s["slots"] >= 0
    put = real[:, None, None]
    q = torch.where(put, qk[:, :hq], 0).to(dt)
    # an empty place writes what the first token (never empty) writes, where it does
    slot = torch.where(real, s["slots"], s["slots"][0])
    at = slot // c["block"], slot % c["block"]
    k, v = torch.where(put, qk[:, hq:], qk[:1, hq:]), torch.where(put, v, v[:1])
    s["cache4"][0][at], s["cache4"][2][at] = _coded(k, dt)
    s["cache4"][1][at], s["cache4"][3][at] = _coded(v, dt)
    return dict(_plain_read4(s), q=q)


def _plain_read4(s):
    bs = s["case"]["block"]
    real = s["slots"] >= 0
    slot = torch.where(real, s["slots"], 0)
    at = slot // bs, slot % bs
    k, v, ks, vs = s["cache4"]
    return {"k": torch.where(real[:, None, None], _values(k[at], ks[at]), 0),
            "v": torch.where(real[:, None, None], _values(v[at], vs[at]), 0)}


def _seen(c, place, pos):
    """Whether the query at `place` sees the token at `pos` (both count the prefix)."""
    seen = pos <= place
    if c["window"]:
        seen = seen & ((pos > place - c["window"]) | (pos < c["sinks"]))
    return seen


def _at(s, pos, real):
    """Block and slot of tokens `pos` [rows, n] (prefix first)."""
    bs, shared = s["case"]["block"], s["shared"]
    table = s["table"].long()
    if shared is not None:
        table = torch.cat((shared.long().expand(table.shape[0], -1), table), 1)
    return torch.where(real, torch.gather(table, 1, pos // bs), 0), pos % bs


def _softmax_sums(score, p_v):
    """Weighted sums and log-sum-exps of scores [..., tokens], in place."""
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, 0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    lse = torch.where(total > 0, top + total.log(), -math.inf)
    return p_v(p), torch.where(total > 0, total, 1), lse[..., 0]


def _plain_attend4(s):
    c = s["case"]
    n, hkv, group, dim = c["rows"], c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"]
    lens = s["lens"].long()[:, None]
    ends = torch.where(lens > 0, lens + c["prefix"], 0)
    pos = torch.arange(c["longest"] + c["prefix"], device=lens.device).expand(n, -1)
    seen = _seen(c, ends - 1, pos)
    pos = torch.where(seen, pos, 0)
    at = _at(s, pos, seen)
    codes_k, codes_v, scales_k, scales_v = s["cache4"]
    k = _values(codes_k[at], scales_k[at]).float()
    score = torch.einsum("nhgd,nlhd->nhgl", s["q"].float().view(n, hkv, group, dim) * dim ** -0.5, k)
    del k
    score = score.masked_fill_(~seen[:, None, None], -math.inf)
    v = torch.where(seen[:, :, None, None], _values(codes_v[at], scales_v[at]), 0).float()
    out, total, lse = _softmax_sums(score, lambda p: torch.einsum("nhgl,nlhd->nhgd", p, v))
    return {"out": (out / total).reshape(n, -1, dim).to(s["q"].dtype), "lse": lse.reshape(n, -1)}


def _plain_prompt(s):
    """Queries and tokens of each row padded to the longest."""
    c = s["case"]
    n, hkv, group, dim = c["rows"], c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"]
    starts, lens = s["starts"].long(), s["lens"].long()
    count = starts[1:] - starts[:-1]
    i = torch.arange(min(c["longest"], s["q"].shape[0]), device=lens.device)
    real = i < count[:, None]
    index = torch.where(real, starts[:-1, None] + i, 0)
    q = s["q"].float()[index].view(n, -1, hkv, group, dim) * dim ** -0.5
    place = c["prefix"] + (lens - count)[:, None] + i
    pos = torch.arange(c["longest"] + c["before"] + c["prefix"], device=lens.device).expand(n, -1)
    held = pos < c["prefix"] + lens[:, None]
    at = _at(s, torch.where(held, pos, 0), held)
    seen = _seen(c, place[:, :, None], pos[:, None]) & held[:, None]
    score = torch.einsum("nqhgd,nlhd->nhgql", q, s["k"][at].float()).masked_fill_(~seen[:, None, None], -math.inf)
    v = torch.where(held[:, :, None, None], s["v"][at], 0).float()
    out, total, lse = _softmax_sums(score, lambda p: torch.einsum("nhgql,nlhd->nhgqd", p, v))
    out = (out / total).permute(0, 3, 1, 2, 4).reshape(n, -1, hkv * group, dim).to(s["q"].dtype)
    lse = lse.permute(0, 3, 1, 2).reshape(n, -1, hkv * group)
    return {"out": out[real], "lse": lse[real]}


# ------------------------------------------------------------------- what a pass cannot do without
def _sum_seen(c, first, count):
    """Tokens seen by `count` queries at places first, first + 1, ..., and how many different ones."""
    place = np.arange(first, first + count, dtype=np.int64)
    if not c["window"] or not count:
        return int((place + 1).sum()), first + count if count else 0
    low = np.maximum(0, place + 1 - c["window"])
    return int((place + 1 - low + np.minimum(low, c["sinks"])).sum()), \
        int(first + count - low[0] + min(low[0], c["sinks"]))


def work(case):
    bs, dim, hq, hkv = case["block"], case["dim"], case["heads"], case["kv_heads"]
    packed = dim // 2 + 4 * dim // GROUP                     # bytes of a token's key (or value) in one head
    if case["op"] == "append4":
        n = case["tokens"]
        # projections in, queries, codes and the codes' values out; slots, positions and angles
        return {"bytes": n * (2 * (hq + 2 * hkv) * dim + 2 * hq * dim + 2 * hkv * (packed + 2 * dim) + 12)
                + min(n, case["positions"]) * 4 * case["rot"],
                "flops": n * ((hq + hkv) * (4 * dim * case["norm"] + 3 * case["rot"]) + 2 * hkv * dim * 8)}
    if case["op"] == "read4":
        n = case["tokens"]
        return {"bytes": n * (2 * hkv * (packed + 2 * dim) + 8), "flops": n * 2 * hkv * dim * 2}
    if case["op"] == "attend4":
        c = case
        each = [_sum_seen(c, c["prefix"] + x - 1, 1) for x in _own_lengths(c) if x]
        seen, live = sum(x for x, _ in each), len(each)
        # a prefix is read once for all where no window hides it
        read = seen - (live - 1) * c["prefix"] if c["prefix"] and not c["window"] else seen
        return {"bytes": 2 * packed * hkv * read + 4 * c["rows"] * hq * dim + 4 * c["rows"] * (hq + 1) + 4 * _blocks(read, bs),
                "flops": 4 * dim * hq * seen}
    each = [_sum_seen(case, case["prefix"] + b, n) for n, b in zip(_own_lengths(case), _before(case))]
    seen, read, tokens = sum(x for x, _ in each), sum(x for _, x in each), sum(_own_lengths(case))
    if case["prefix"] and not case["window"]:
        read -= (sum(x > 0 for x in _own_lengths(case)) - 1) * case["prefix"]
    return {"bytes": 4 * dim * hkv * read + 4 * tokens * hq * dim + 4 * tokens * hq + 4 * _blocks(read, bs),
            "flops": 4 * dim * hq * seen}


# ------------------------------------------------------------------- in 64 bits, from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    return {"append4": _exact_append4, "read4": _exact_read4, "attend4": _exact_attend4, "prompt": _exact_prompt}[case["op"]](s)


def _exact_values(codes, scales):
    """Value by value of a group: the even ones are a byte's low code."""
    b = codes.reshape(scales.shape[:-1] + (GROUP // 2,)).long()
    s, o = scales.double().unbind(-1)
    out = torch.empty(b.shape[:-1] + (GROUP,), dtype=torch.float64, device=b.device)
    out[..., 0::2] = o[..., None] + s[..., None] * (16 + b % 16) / 16
    out[..., 1::2] = o[..., None] + s[..., None] * (16 + b // 16) / 16
    return out.to(scales.dtype).double().flatten(-2)


def _exact_round(x, dt):
    """Values [..., dim] as the nearest of their group's sixteen."""
    y = x.unflatten(-1, (-1, GROUP))
    lo, hi = y.min(-1).values, y.max(-1).values
    scale = ((hi - lo) * 16 / 15).to(dt).double()
    offset = (lo - scale).to(dt).double()
    step = (scale / 16)[..., None]
    code = torch.where(step > 0, ((y - (offset + scale)[..., None]) / step).round().clamp(0, 15), 0.0)
    return ((offset + scale)[..., None] + code * step).to(dt).double().flatten(-2)


def _exact_append4(s):
    c = s["case"]
    n, hq, hkv, dim, half = c["tokens"], c["heads"], c["kv_heads"], c["dim"], c["rot"] // 2
    x = s["qkv"].double().reshape(n, hq + 2 * hkv, dim)
    first = torch.arange(half, device=x.device)
    first, second = (2 * first, 2 * first + 1) if c["pairs"] else (first, first + half)
    z = torch.complex(*(s["rope"].double()[s["positions"].long()][:, None, i * half:(i + 1) * half] for i in (0, 1)))

    def turned(y, w):
        if w is not None:
            y = y / (y.pow(2).sum(-1, keepdim=True) / dim + EPS).sqrt() * w.double()
        r = torch.complex(y[..., first], y[..., second]) * z
        y = y.clone()
        y[..., first], y[..., second] = r.real, r.imag
        return y

    real = (s["slots"] >= 0).double()[:, None, None]
    dt = s["qkv"].dtype
    return {"q": turned(x[:, :hq], s["q_weight"]) * real,
            "k": _exact_round(turned(x[:, hq:hq + hkv], s["k_weight"]), dt) * real,
            "v": _exact_round(x[:, hq + hkv:], dt) * real}


def _exact_read4(s):
    bs, out = s["case"]["block"], {}
    real = (s["slots"] >= 0).nonzero()[:, 0]
    at = s["slots"][real] // bs, s["slots"][real] % bs
    for name, codes, scales in (("k", s["cache4"][0], s["cache4"][2]), ("v", s["cache4"][1], s["cache4"][3])):
        x = torch.zeros(s["case"]["tokens"], s["case"]["kv_heads"], s["case"]["dim"], dtype=torch.float64, device="cuda")
        x[real] = _exact_values(codes[at], scales[at])
        out[name] = x
    return out


def _exact_places(s, i, tokens):
    """Block and slot of the first `tokens` tokens of row i, prefix first."""
    bs = s["case"]["block"]
    blocks = s["table"][i].long()
    if s["shared"] is not None:
        blocks = torch.cat((s["shared"].long(), blocks))
    at = torch.arange(tokens, device="cuda")
    return blocks[at // bs], at % bs


def _exact_attend4(s):
    """Request by request."""
    c = s["case"]
    n, hkv, dim = c["rows"], c["kv_heads"], c["dim"]
    out = torch.zeros(n, c["heads"], dim, dtype=torch.float64, device="cuda")
    lse = torch.full((n, c["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    ck, cv, sk, sv = s["cache4"]
    for i, length in enumerate(s["lens"].tolist()):
        if not length:
            continue
        end = length + c["prefix"]
        block, place = _exact_places(s, i, end)
        if c["window"]:
            pos = torch.arange(end, device="cuda")
            pos = pos[(pos < c["sinks"]) | (pos >= end - c["window"])]
            block, place = block[pos], place[pos]
        k, v = _exact_values(ck[block, place], sk[block, place]), _exact_values(cv[block, place], sv[block, place])
        score = torch.matmul(s["q"][i].double().view(hkv, -1, dim), k.permute(1, 2, 0)) / math.sqrt(dim)
        out[i] = torch.matmul(score.softmax(-1), v.transpose(0, 1)).reshape(-1, dim)
        lse[i] = score.logsumexp(-1).reshape(-1)
    return {"out": out, "lse": lse}


def _exact_prompt(s):
    """Request by request, 512 queries at a time, over the tokens up to the last of them."""
    c = s["case"]
    hkv, dim = c["kv_heads"], c["dim"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    for i, length in enumerate(lens):
        a, b = starts[i], starts[i + 1]
        first = c["prefix"] + length - (b - a)                 # the place of the row's first query
        for x in range(a, b, 512):
            y = min(b, x + 512)
            end = first + y - a
            block, place = _exact_places(s, i, end)
            k, v = s["k"][block, place].double(), s["v"][block, place].double()
            q = s["q"][x:y].double().view(y - x, hkv, -1, dim).permute(1, 2, 0, 3)       # [hkv, group, queries, dim]
            score = torch.matmul(q, k.permute(1, 2, 0)[:, None]) / math.sqrt(dim)
            at, pos = torch.arange(first + x - a, end, device="cuda")[:, None], torch.arange(end, device="cuda")
            hidden = pos > at
            if c["window"]:
                hidden |= (pos <= at - c["window"]) & (pos >= c["sinks"])
            score.masked_fill_(hidden, -math.inf)
            out[x:y] = torch.matmul(score.softmax(-1), v.transpose(0, 1)[:, None]).permute(2, 0, 1, 3).reshape(y - x, -1, dim)
            lse[x:y] = score.logsumexp(-1).permute(2, 0, 1).reshape(y - x, -1)
    return {"out": out, "lse": lse}
