"""The operators of a decode step over a paged KV cache, as cases that can be timed and compared.

A serving step of the token-step model gives every running request one token.
On the machine below the schedule that step is: cache blocks for the new tokens
("assign": block tables and slot maps from request lengths), norms and position
rotation of the new queries and keys, written to their slots ("append"), and
attention of each query over its request's cached tokens, with a sliding window
and a few first tokens that stay visible ("window"), or over a prefix that the
whole batch shares ("prefix").

`run` computes them in plain torch where `own` is false and through
paper_2608_02244_gb300.kv where it is true.  Request lengths are quantiles of
the lognormals of paper_2608_02244_gb300/workloads.py, so that the multiset (and
with it the work) goes by the case alone; their order, the blocks and all values
go by the seed.
"""
from __future__ import annotations

import math
import statistics

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-6


# ------------------------------------------------------------------- cases
def _assign(name, rows, median, sigma, longest, block, kv, fresh, ended, idle, prefix, spare):
    """`rows` batch slots over a pool of `kv` tokens in blocks of `block`; of them the
    share `fresh` starts with its whole prompt, `ended` gives its blocks back,
    `idle` does nothing and all others get one token; room for `spare` more tokens
    than that in the slot map."""
    c = {"op": "assign", "rows": rows, "median": median, "sigma": sigma, "longest": longest, "block": block, "kv": kv,
         "fresh": fresh, "ended": ended, "idle": idle, "prefix": prefix, "spare": spare}
    return dict(c, name=name) if name else c


def _append(name, tokens, heads, kv_heads, dim, rot, pairs, norm, block, kind, order, positions):
    """`tokens` new tokens; `rot` of the `dim` values of a head are rotated, as
    neighbours ("pairs") or as halves; `order` is the cache's: tokens of a block
    outermost ("token") or heads ("head")."""
    c = {"op": "append", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rot": rot, "pairs": pairs,
         "norm": norm, "block": block, "kind": kind, "order": order, "positions": positions}
    return dict(c, name=name) if name else c


def _attend(name, rows, heads, kv_heads, dim, block, kind, order, median, sigma, longest, idle, window, sinks, prefix):
    """One query for each of `rows` requests, `idle` of them empty; `prefix` tokens
    are shared by all and come before each request's own."""
    c = {"op": "prefix" if prefix else "window", "rows": rows, "heads": heads, "kv_heads": kv_heads, "dim": dim,
         "block": block, "kind": kind, "order": order, "median": median, "sigma": sigma, "longest": longest, "idle": idle,
         "window": window, "sinks": sinks, "prefix": prefix}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decode step of the online workload's batch: 256 slots, 200,000 tokens of cache
        _assign("assign_step_256", 256, 512, 1.0, 4096, 16, 200_000, 0.0, 0.05, 0.05, 0, 0),
        # a refill of many slots: two thousand prompts at once among running requests, a slot map of millions
        _assign("assign_fill_2999", 2999, 1024, 1.0, 32768, 32, 8_000_000, 0.66, 0.1, 0.01, 64, 4099),
        # one decode step of the same batch through its norms and rotation
        _append("append_256", 256, 32, 8, 128, 128, False, True, 16, "bf16", "token", 4096),
        # prompts in chunks: odd head groups, half of each head rotated as pairs, heads outermost
        _append("append_1021_pairs", 1021, 28, 4, 64, 32, True, True, 8, "fp16", "head", 6144),
        # a whole prefill's worth of tokens
        _append("append_49152", 49152, 32, 8, 128, 128, False, True, 64, "bf16", "token", 49152),
        # a single short request: latency counts
        _attend("window_1", 1, 32, 8, 128, 16, "bf16", "token", 777, 0.0, 777, 0, 512, 4, 0),
        # the online workload's batch, a window shorter than its long requests
        _attend("window_256", 256, 32, 8, 128, 16, "bf16", "token", 640, 1.0, 6144, 3, 1024, 4, 0),
        # odd sizes: seven query heads on each key head, an odd window, heads outermost
        _attend("window_61_odd", 61, 28, 4, 64, 8, "fp16", "head", 2000, 1.0, 16384, 2, 1777, 5, 0),
        # the long-context batch: 512 slots, most of a million tokens in the window
        _attend("window_512", 512, 64, 8, 128, 32, "bf16", "token", 1536, 1.2, 49152, 5, 4096, 4, 0),
        # a few requests that share a system prompt
        _attend("prefix_17", 17, 32, 8, 128, 16, "bf16", "token", 256, 1.0, 2048, 1, 0, 0, 2048),
        # odd sizes: a prefix that ends inside a tile, seven query heads on each key head
        _attend("prefix_61_odd", 61, 28, 4, 64, 8, "fp16", "head", 300, 1.2, 2048, 2, 0, 0, 8136),
        # the largest batch over a long shared document
        _attend("prefix_512", 512, 64, 8, 128, 64, "bf16", "token", 256, 1.2, 2048, 4, 0, 0, 32768),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more step of the listed ranges: one to 512 queries (to 49,152 tokens of
    append, 2,999 slots of assign), contexts of one token to tens of thousands."""
    op = rng.choice(["assign", "append", "window", "prefix"])
    block = rng.choice([8, 16, 32, 64, 128])
    kind, order = rng.choice(["bf16", "bf16", "fp16"]), rng.choice(["token", "token", "head"])
    if op == "assign":
        rows = _log(rng, 1, 2999)
        median, longest = _log(rng, 16, 1024), 32768
        fresh = round(rng.choice([0.0, rng.uniform(0, 0.66)]), 3)
        # now and then the pool is too small for all that is asked
        kv = max(block * 4, int(rows * median * 1.65 * rng.uniform(0.8, 3.0)), int(rows * block * 1.2))
        return _assign(None, rows, median, 1.0, longest, block, min(kv | 1, 8_000_000), fresh, round(rng.uniform(0, 0.2), 3),
                       round(rng.uniform(0, 0.1), 3), rng.choice([0, 0, block * 4]), rng.choice([0, 0, rng.randint(1, 4099)]))
    kv_heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16])
    while kv_heads * group > 64:
        group = max(1, group // 2)
    dim = rng.choice([64, 128, 128, 256])
    if op == "append":
        cost = 49152 * 40 * 128
        tokens = _log(rng, 1, max(1, min(49152, cost // ((group + 1) * kv_heads * dim))))
        rot = rng.choice([dim, dim, dim // 2])
        return _append(None, tokens, kv_heads * group, kv_heads, dim, rot, rng.random() < 0.3, rng.random() < 0.8, block,
                       kind, order, _log(rng, 64, 49152))
    rows = _log(rng, 1, 512)
    size = kv_heads * dim
    if op == "window":
        window = rng.choice([0, _log(rng, 64, 4096), _log(rng, 64, 4096)])
        longest = min(49152, max(64, 512 * 4096 * 1024 // (rows * size))) if window else min(49152, max(64, 4096 * 512 * 1024 // (rows * size * 2)))
        longest = _log(rng, 32, longest)
        return _attend(None, rows, kv_heads * group, kv_heads, dim, block, kind, order, max(1, longest // rng.randint(1, 12)),
                       round(rng.uniform(0.0, 1.2), 2), longest, min(rows - 1, rng.randint(0, 5)), window,
                       rng.choice([0, 1, 4, 33]) if window else 0, 0)
    longest = _log(rng, 1, 2048)
    most = 32768 * 512 * 8192 // (rows * kv_heads * group * dim)
    prefix = block * (_log(rng, 64, max(64, min(32768, most))) // block | 1)
    return _attend(None, rows, kv_heads * group, kv_heads, dim, block, kind, order, max(1, longest // rng.randint(1, 8)),
                   round(rng.uniform(0.0, 1.2), 2), longest, min(rows - 1, rng.randint(0, 4)), 0, 0, prefix)


# ------------------------------------------------------------------- inputs
def _lengths(n, median, sigma, longest):
    """The n quantiles of a lognormal, rounded, in 1..longest."""
    normal = statistics.NormalDist()
    return [min(longest, max(1, round(median * math.exp(sigma * normal.inv_cdf((i + 0.5) / n))))) for i in range(n)]


def _spread(values, n, k):
    """k of the n values, evenly spread over them."""
    return [values[(2 * i + 1) * n // (2 * k)] for i in range(k)]


def _parts(case):
    """The requests of an assign case by kind: lengths held by those that end, that idle
    and that go on, and the prompts of those that start."""
    n = case["rows"]
    lens = _lengths(n, case["median"], case["sigma"], case["longest"])
    k = [int(case[f] * n) for f in ("fresh", "ended", "idle")]
    mixed = [lens[(i * 7919 + 13) % n] for i in range(n)]   # 7919 is prime and more than n
    at = [0, k[0], k[0] + k[1], k[0] + k[1] + k[2], n]
    return [mixed[a:b] for a, b in zip(at, at[1:])]        # fresh, ended, idle, going on


def _blocks(n, block):
    return -(-n // block)


def _pool(case):
    """Blocks of an assign case's pool: those held and what is left of `kv`, at least none."""
    fresh, ended, idle, rest = _parts(case)
    held = sum(_blocks(x, case["block"]) for x in ended + idle + rest)
    return held, max(held, case["kv"] // case["block"])


def _own_lengths(case):
    lens = _lengths(case["rows"] - case["idle"], case["median"], case["sigma"], case["longest"])
    return lens + [0] * case["idle"]


def _cache(case, blocks, g):
    """A cache [blocks, block, kv_heads, dim] in the case's order of axes, filled."""
    shape = (blocks, case["block"], case["kv_heads"], case["dim"])
    if case["order"] == "head":
        shape = (shape[0], shape[2], shape[1], shape[3])
    x = torch.randn(shape, generator=g, device="cuda", dtype=TYPES[case["kind"]])
    return x.transpose(1, 2) if case["order"] == "head" else x


def _rope(positions, rot):
    """cos then sin of each position's angles, [positions, rot] in 32 bits."""
    inv = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * inv
    return torch.cat((angle.cos(), angle.sin()), 1).float().contiguous()


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def prepare(case, seed):
    rng = np.random.Generator(np.random.PCG64(np.random.SeedSequence([seed, 77])))
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, bs = case["op"], case["block"]
    s = {"case": case}
    if op == "assign":
        fresh, ended, idle, rest = _parts(case)
        lens = np.array([0] * len(fresh) + ended + idle + rest, np.int32)
        new = np.array(fresh + [-1] * len(ended) + [0] * len(idle) + [1] * len(rest), np.int32)
        order = rng.permutation(case["rows"])
        lens, new = lens[order], new[order]
        held, blocks = _pool(case)
        width = _blocks(case["longest"] + 1, bs)
        ids = rng.permutation(blocks).astype(np.int32)
        own_blocks = -(-lens // bs)
        table = np.full((case["rows"], width), -1, np.int32)
        table[np.arange(width)[None, :] < own_blocks[:, None]] = ids[:held]
        free = np.full(blocks, -1, np.int32)
        free[:blocks - held] = ids[held:]
        s.update(lens=_i32(lens), new=_i32(new), table=_i32(table), free=_i32(free), n_free=_i32([blocks - held]),
                 blocks=blocks, tokens=max(1, sum(fresh) + len(rest) + case["spare"]))
        return s
    dt, dim, hq, hkv = TYPES[case["kind"]], case["dim"], case["heads"], case["kv_heads"]
    if op == "append":
        n = case["tokens"]
        blocks = _blocks(n + n // 8, bs) + 1
        slots = rng.permutation(blocks * bs)[:n].astype(np.int64)
        if n > 8:                                   # a few places of the step's slot map are empty
            slots[rng.integers(1, n, size=n // 50)] = -1
        positions = rng.integers(0, case["positions"], size=n)
        s.update(qkv=torch.randn(n, (hq + 2 * hkv) * dim, generator=g, device="cuda", dtype=dt),
                 positions=_i32(positions), slots=torch.from_numpy(slots).cuda(), rope=_rope(case["positions"], case["rot"]),
                 k=_cache(case, blocks, g), v=_cache(case, blocks, g), q_weight=None, k_weight=None)
        if case["norm"]:
            s["q_weight"] = (1 + 0.2 * torch.randn(dim, generator=g, device="cuda")).to(dt)
            s["k_weight"] = (1 + 0.2 * torch.randn(dim, generator=g, device="cuda")).to(dt)
        return s
    lens = rng.permutation(np.array(_own_lengths(case), np.int32))
    own_blocks = -(-lens // bs)
    held, shared = int(own_blocks.sum()), case["prefix"] // bs
    ids = rng.permutation(held + shared + 3).astype(np.int32)
    width = max(1, int(own_blocks.max()))
    table = np.full((case["rows"], width), -1, np.int32)
    table[np.arange(width)[None, :] < own_blocks[:, None]] = ids[:held]
    q = torch.randn(case["rows"], hq, dim, generator=g, device="cuda", dtype=dt)
    s.update(q=q, lens=_i32(lens), table=_i32(table), k=_cache(case, held + shared + 3, g),
             v=_cache(case, held + shared + 3, g), shared=_i32(ids[held:held + shared]) if shared else None)
    return s


# ------------------------------------------------------------------- one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return {"assign": _own_assign, "append": _own_append, "window": _own_attend, "prefix": _own_attend}[op](s)
    return {"assign": _plain_assign, "append": _plain_append, "window": _plain_attend, "prefix": _plain_attend}[op](s)


_decoders = {}


def _decoder(s):
    """The handle that a serving program keeps for its cache's shape."""
    c = s["case"]
    if c["op"] == "assign":
        key = (s["blocks"], c["block"], 1, 1, 64, torch.bfloat16, c["rows"])
    else:
        key = (s["k"].shape[0], c["block"], c["heads"], c["kv_heads"], c["dim"], TYPES[c["kind"]], c.get("rows", 1))
    if key not in _decoders:
        from paper_2608_02244_gb300 import kv
        _decoders[key] = kv.Decoder(*key[:5], dtype=key[5], max_rows=key[6])
    return _decoders[key]


def _own_assign(s):
    p = _decoder(s).assign(s["lens"], s["new"], s["table"], s["free"], s["n_free"], s["tokens"],
                           prefix_len=s["case"]["prefix"])
    return {"slots": p.slots, "positions": p.positions, "rows": p.rows, "visible": p.visible, "starts": p.starts,
            "granted": p.granted, "lens": p.lens, "n_free": p.n_free, "table": s["table"], "free": s["free"]}


def _own_append(s):
    q = _decoder(s).append(s["qkv"], s["positions"], s["slots"], s["k"], s["v"], s["rope"], s["q_weight"], s["k_weight"],
                           eps=EPS, pairs=s["case"]["pairs"])
    return {"q": q, "k": s["k"], "v": s["v"]}


def _own_attend(s):
    c = s["case"]
    out, lse = _decoder(s).attend(s["q"], s["k"], s["v"], s["table"], s["lens"], prefix=s["shared"], window=c["window"],
                                  sinks=c["sinks"], lse=True)
    return {"out": out, "lse": lse}


def _plain_assign(s):
    """Blocks are taken from the top of the free list, rows in order; a row gets all its
    new tokens or none.  Rows that end push theirs first."""
    bs, room, prefix = s["case"]["block"], s["tokens"], s["case"]["prefix"]
    lens, new, table, free = s["lens"].long(), s["new"].long(), s["table"], s["free"]
    n, width = table.shape
    ends = new < 0
    ask = new.clamp(min=0)
    held = (lens + bs - 1) // bs
    fits = lens + ask <= width * bs
    ask = torch.where(fits, ask, 0)
    need = (lens + ask + bs - 1) // bs - held
    back = torch.where(ends, held, 0)
    avail = s["n_free"].long() + back.sum()
    granted = torch.where(((need == 0) | (need.cumsum(0) <= avail)) & (ask.cumsum(0) <= room), ask, 0)
    lens_out = torch.where(ends, 0, lens + granted)
    takes = torch.where(granted > 0, need, 0)
    # blocks given back, in order of rows and places, go on top of the free list
    place = torch.arange(width, device=lens.device)
    gives = place < back[:, None]
    to = torch.where(gives, s["n_free"] + (back.cumsum(0) - back)[:, None] + place, free.shape[0])
    stack = torch.cat((free, free.new_zeros(1)))
    stack[to.reshape(-1)] = torch.where(gives, table, 0).reshape(-1)
    free.copy_(stack[:-1])
    # and are taken from there
    gets = (place >= held[:, None]) & (place < (held + takes)[:, None])
    index = avail - 1 - (takes.cumsum(0) - takes)[:, None] - (place - held[:, None])
    table.copy_(torch.where(gets, free[torch.where(gets, index, 0)], table))
    # the new tokens, rows one after another
    starts = torch.cat((granted.new_zeros(1), granted.cumsum(0)))
    t = torch.arange(room, device=lens.device)
    row = torch.searchsorted(starts[1:].contiguous(), t, right=True).clamp(max=n - 1)
    real = t < starts[-1]
    at = torch.where(real, lens[row] + t - starts[row], 0)
    slot = table[row, at // bs].long() * bs + at % bs
    i32 = torch.int32
    return {"slots": torch.where(real, slot, -1), "positions": torch.where(real, prefix + at, 0).to(i32),
            "rows": torch.where(real, row, -1).to(i32), "visible": torch.where(real, at + 1, 0).to(i32),
            "starts": starts.to(i32), "granted": granted.to(i32), "lens": lens_out.to(i32),
            "n_free": (avail - takes.sum()).to(i32).reshape(1), "table": table, "free": free}


def _plain_append(s):
    c = s["case"]
    n, hq, hkv, dim, rot = c["tokens"], c["heads"], c["kv_heads"], c["dim"], c["rot"]
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
    qk = torch.cat((turned, qk[..., rot:]), -1).to(s["qkv"].dtype)
    real = s["slots"] >= 0
    q = torch.where(real[:, None, None], qk[:, :hq], 0)
    # an empty place writes what the first token (never empty) writes, where it does
    slot = torch.where(real, s["slots"], s["slots"][0])
    put = real[:, None, None]
    s["k"][slot // c["block"], slot % c["block"]] = torch.where(put, qk[:, hq:], qk[:1, hq:])
    s["v"][slot // c["block"], slot % c["block"]] = torch.where(put, v, v[:1]).to(s["qkv"].dtype)
    return {"q": q, "k": s["k"], "v": s["v"]}


def _plain_attend(s):
    c = s["case"]
    n, hkv, group, dim, bs = c["rows"], c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"], c["block"]
    lens = s["lens"].long()[:, None]
    q = s["q"].float().view(n, hkv, group, dim) * dim ** -0.5
    if c["window"]:
        # the first tokens, then the window's
        j = torch.arange(min(c["longest"], c["sinks"] + c["window"]), device=q.device)
        pos = torch.where(j < c["sinks"], j, lens - c["window"] + j - c["sinks"])
        seen = (pos < lens) & ((j < c["sinks"]) | (pos >= c["sinks"]))
        if c["longest"] <= c["sinks"] + c["window"]:
            pos, seen = j.expand(n, -1), j < lens
    else:
        pos = torch.arange(c["longest"], device=q.device).expand(n, -1)
        seen = pos < lens
    pos = torch.where(seen, pos, 0)
    block = torch.where(seen, torch.gather(s["table"].long(), 1, pos // bs), 0)
    score = torch.einsum("nhgd,nlhd->nhgl", q, s["k"][block, pos % bs].float())
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    if s["shared"] is not None:
        b = s["shared"].long()
        k, v = s["k"][b].float().reshape(-1, hkv, dim), s["v"][b].float().reshape(-1, hkv, dim)
        first = torch.einsum("nhgd,lhd->nhgl", q, k).masked_fill(lens[:, :, None, None] == 0, -math.inf)
        score = torch.cat((first, score), -1)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0, top))
    total = p.sum(-1, keepdim=True)
    lse = torch.where(total > 0, top + total.log(), -math.inf)
    p = p / torch.where(total > 0, total, 1)
    split = score.shape[-1] - pos.shape[1]
    value = torch.where(seen[:, :, None, None], s["v"][block, pos % bs].float(), 0)
    out = torch.einsum("nhgl,nlhd->nhgd", p[..., split:], value)
    if s["shared"] is not None:
        out = out + torch.einsum("nhgl,lhd->nhgd", p[..., :split], v)
    return {"out": out.reshape(n, -1, dim).to(s["q"].dtype), "lse": lse.reshape(n, -1)}


# ------------------------------------------------------------------- what a pass cannot do without
def work(case):
    bs = case["block"]
    if case["op"] == "assign":
        fresh, ended, idle, rest = _parts(case)
        held, blocks = _pool(case)
        given = sum(_blocks(x, bs) for x in ended)
        left = blocks - held + given
        taken = sum(_blocks(x, bs) for x in fresh) + sum(x % bs == 0 for x in rest)
        tokens = max(1, sum(fresh) + len(rest) + case["spare"])
        # lengths, new tokens, grants and row starts; blocks given back and taken, read and written; the maps
        return {"bytes": 16 * case["rows"] + 8 * given + 8 * min(left, taken) + 20 * tokens, "flops": 0}
    dim, hq, hkv = case["dim"], case["heads"], case["kv_heads"]
    if case["op"] == "append":
        n = case["tokens"]
        # projections in, queries and slots out, positions, slots and angles
        return {"bytes": n * (4 * (hq + 2 * hkv) * dim + 12) + min(n, case["positions"]) * 4 * case["rot"],
                "flops": n * (hq + hkv) * (4 * dim * case["norm"] + 3 * case["rot"])}
    seen = [min(x, case["window"] + min(case["sinks"], max(0, x - case["window"]))) if case["window"] else x
            for x in _own_lengths(case)]
    live = case["rows"] - case["idle"]
    return {"bytes": 4 * dim * hkv * (sum(seen) + case["prefix"]) + 4 * case["rows"] * hq * dim + 4 * case["rows"] * (hq + 1)
            + 4 * sum(_blocks(x, bs) for x in seen),
            "flops": 4 * dim * hq * (sum(seen) + live * case["prefix"])}


# ------------------------------------------------------------------- in 64 bits, from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    return {"assign": _exact_assign, "append": _exact_append, "window": _exact_attend, "prefix": _exact_attend}[case["op"]](s)


def _exact_assign(s):
    """One row after another, a stack of blocks."""
    bs, room, prefix = s["case"]["block"], s["tokens"], s["case"]["prefix"]
    lens, new, table = s["lens"].tolist(), s["new"].tolist(), s["table"].cpu().numpy()
    free, top = s["free"].cpu().numpy(), int(s["n_free"])
    for i, (x, k) in enumerate(zip(lens, new)):
        if k < 0:
            b = _blocks(x, bs)
            free[top:top + b] = table[i, :b]
            top += b
    asked_blocks = asked_tokens = 0
    avail, granted, starts, out = top, [], [0], []
    slots, positions, rows, visible = (np.full(room, x, t) for x, t in ((-1, np.int64), (0, np.int32), (-1, np.int32), (0, np.int32)))
    for i, (x, k) in enumerate(zip(lens, new)):
        k = 0 if k < 0 or x + k > table.shape[1] * bs else k
        old, b = _blocks(x, bs), _blocks(x + k, bs) - _blocks(x, bs)
        asked_blocks, asked_tokens = asked_blocks + b, asked_tokens + k
        if (b and asked_blocks > avail) or asked_tokens > room:
            k = b = 0
        table[i, old:old + b] = free[top - b:top][::-1]
        top -= b
        at, a = np.arange(x, x + k), starts[-1]
        slots[a:a + k] = table[i, at // bs].astype(np.int64) * bs + at % bs
        positions[a:a + k], rows[a:a + k], visible[a:a + k] = prefix + at, i, at + 1
        granted.append(k)
        starts.append(a + k)
        out.append(0 if new[i] < 0 else x + k)
    i32 = lambda v: np.array(v, np.int32)  # noqa: E731
    return {"slots": slots, "positions": positions, "rows": rows, "visible": visible, "starts": i32(starts),
            "granted": i32(granted), "lens": i32(out), "n_free": i32([top]), "table": table, "free": free}


def _exact_append(s):
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

    real = (s["slots"] >= 0).nonzero()[:, 0]
    q = torch.zeros(n, hq, dim, dtype=torch.float64, device=x.device)
    q[real] = turned(x[:, :hq], s["q_weight"])[real]
    k, v = s["k"].double(), s["v"].double()
    block, place = s["slots"][real] // c["block"], s["slots"][real] % c["block"]
    k[block, place] = turned(x[:, hq:hq + hkv], s["k_weight"])[real]
    v[block, place] = x[real, hq + hkv:]
    return {"q": q, "k": k, "v": v}


def _exact_attend(s):
    """Request by request."""
    c = s["case"]
    n, hkv, dim, bs = c["rows"], c["kv_heads"], c["dim"], c["block"]
    out = torch.zeros(n, c["heads"], dim, dtype=torch.float64, device="cuda")
    lse = torch.full((n, c["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    first = [s[x][s["shared"].long()].double().reshape(-1, hkv, dim) for x in "kv"] if s["shared"] is not None else None
    for i, length in enumerate(s["lens"].tolist()):
        if not length:
            continue
        pos = torch.arange(length, device="cuda")
        if c["window"]:
            pos = pos[(pos < c["sinks"]) | (pos >= length - c["window"])]
        at = s["table"][i].long()[pos // bs]
        k, v = (s[x][at, pos % bs].double() for x in "kv")
        if first:
            k, v = torch.cat((first[0], k)), torch.cat((first[1], v))
        score = torch.matmul(s["q"][i].double().view(hkv, -1, dim), k.permute(1, 2, 0)) / math.sqrt(dim)
        out[i] = torch.matmul(score.softmax(-1), v.transpose(0, 1)).reshape(-1, dim)
        lse[i] = score.logsumexp(-1).reshape(-1)
    return {"out": out, "lse": lse}
