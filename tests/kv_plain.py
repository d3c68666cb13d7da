"""Plain 64-bit forms of the decode step's parts, row by row, for the tests."""
import math

import torch


def assign(lens, new, table, free, n_free, block, room, prefix=0):
    """Lists in and out: a stack of free blocks, one row after another."""
    table, stack = [list(r) for r in table], list(free[:n_free])
    held = [-(-x // block) for x in lens]
    for i, k in enumerate(new):
        if k < 0:
            stack += table[i][:held[i]]
    avail = len(stack)
    used = list(stack) + list(free[len(stack):])
    asked = tokens = 0
    maps, granted, after, starts = [], [], [], [0]
    for i, (x, k) in enumerate(zip(lens, new)):
        ends, k = k < 0, max(k, 0)
        if x + k > len(table[i]) * block:
            k = 0
        need = 0 if ends else -(-(x + k) // block) - held[i]
        asked, tokens = asked + need, tokens + k
        if (need and asked > avail) or tokens > room:
            k = need = 0
        for j in range(need):
            table[i][held[i] + j] = stack.pop()
        for at in range(x, x + k):
            maps.append((table[i][at // block] * block + at % block, prefix + at, i, at + 1))
        granted.append(k)
        after.append(0 if ends else x + k)
        starts.append(starts[-1] + k)
    maps += [(-1, 0, -1, 0)] * (room - len(maps))
    return {"slots": [m[0] for m in maps], "positions": [m[1] for m in maps], "rows": [m[2] for m in maps],
            "visible": [m[3] for m in maps], "starts": starts, "granted": granted, "lens": after,
            "n_free": [len(stack)], "table": table, "free": used}


def append(qkv, positions, slots, rope, q_weight, k_weight, eps, pairs, hq, hkv, dim):
    """q, k, v of each token in 64 bits and, for q and k, the sum of magnitudes of each value's terms."""
    x = qkv.double().reshape(qkv.shape[0], hq + 2 * hkv, dim)
    out, mags = x.clone(), x.abs()
    for h in range(hq + hkv):
        y = x[:, h]
        w = q_weight if h < hq else k_weight
        if w is not None:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double()
        z, mag = y.clone(), y.abs()
        if rope is not None:
            half = rope.shape[1] // 2
            a = rope.double()[positions.long()]
            c, s = a[:, :half], a[:, half:]
            i = torch.arange(half, device=x.device)
            i, j = (2 * i, 2 * i + 1) if pairs else (i, i + half)
            z[:, i], z[:, j] = y[:, i] * c - y[:, j] * s, y[:, j] * c + y[:, i] * s
            mag[:, i] = (y[:, i] * c).abs() + (y[:, j] * s).abs()
            mag[:, j] = (y[:, j] * c).abs() + (y[:, i] * s).abs()
        out[:, h], mags[:, h] = z, mag
    return out, mags


def seen(total, window, sinks):
    """Places that a query at the end of `total` tokens sees."""
    return [p for p in range(total) if not window or p >= total - window or p < sinks]


def attend(q, k, v, table, lens, rows=None, prefix=None, window=0, sinks=0, scale=None):
    """out, lse and the weighted mean of |v| (what errors of the weights act on), in 64 bits."""
    n, hq, dim = q.shape
    block, hkv = k.shape[1], k.shape[2]
    scale = dim ** -0.5 if scale is None else scale
    out = torch.zeros(n, hq, dim, dtype=torch.float64, device=q.device)
    size = torch.zeros_like(out)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device=q.device)
    first = [] if prefix is None else prefix.tolist()
    for t in range(n):
        row, own = (t if rows is None else int(rows[t])), int(lens[t])
        if row < 0 or own <= 0:
            continue
        blocks = torch.tensor(first + table[row, :-(-own // block)].tolist(), device=q.device)
        pos = torch.tensor(seen(len(first) * block + own, window, sinks), device=q.device)
        kk, vv = (c[blocks[pos // block], pos % block].double() for c in (k, v))
        s = torch.einsum("hgd,lhd->hgl", q[t].double().view(hkv, hq // hkv, dim), kk) * scale
        p = s.softmax(-1)
        out[t] = torch.einsum("hgl,lhd->hgd", p, vv).reshape(hq, dim)
        size[t] = torch.einsum("hgl,lhd->hgd", p, vv.abs()).reshape(hq, dim)
        lse[t] = s.logsumexp(-1).reshape(hq)
    return out, lse, size


# Unit roundoff of the 16-bit types.  An output is a weighted mean with weights rounded once to the type (each off
# by at most `unit` of itself), rounded once more; scores and sums are in 32 bits, off by at most
# dim * 2^-24 * sum|q k| scale, about 1.5e-4 for 256 values of unit variance, hence the 2^-12.
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
REST = 2.0 ** -12


def check_attend(got, lse, want, want_lse, size):
    assert torch.isfinite(got.double()).all()
    bound = (2 * UNIT[got.dtype] + REST) * size + 2.0 ** -24
    assert ((got.double() - want).abs() <= bound).all(), ((got.double() - want).abs() / bound).max()
    dead = want_lse == -math.inf
    assert torch.equal(lse == -math.inf, dead)
    off = (lse.double() - want_lse).abs()[~dead]
    assert (off <= REST + 2.0 ** -20 * want_lse.abs()[~dead]).all(), off.max()
