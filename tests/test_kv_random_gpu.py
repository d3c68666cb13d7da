"""Random decode steps through all three operators against 64 bits: shapes, types, orders, windows, prefixes and row maps
drawn together, each step's maps feeding the next part."""
import math
import random

import numpy as np
import pytest

import kv_plain
from conftest import cuda_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]
EPS = 1e-5


@pytest.mark.parametrize("seed", range(40))
def test_step(seed):
    import torch
    from paper_2608_02244_gb300 import kv
    rng = random.Random(seed)
    dim, block = rng.choice([64, 64, 128, 128, 256]), rng.choice([8, 16, 16, 32, 64, 128, 256])
    hkv = rng.choice([1, 1, 2, 3, 8])
    hq = hkv * rng.choice([1, 2, 3, 4, 7, 8, 16, 19])
    dtype = rng.choice([torch.bfloat16, torch.float16])
    n = rng.choice([1, 2, 9, 33, 64, 130])
    longest = rng.choice([3, 40, 300, 1500])
    shared = rng.choice([0, 0, 1, 5, 40, 300]) if block <= 32 else rng.choice([0, 0, 1, 9])
    window = rng.choice([0, 0, 0, 1, 30, 500])
    sinks = rng.choice([0, 2, 40])
    rot, pairs = rng.choice([0, 16, dim // 2, dim]), rng.random() < 0.5
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731

    # lengths before the step, and its new tokens: some rows idle, some end, some get several
    lens = np.array([rng.choice([0, 1, block - 1, block, rng.randint(0, longest)]) for _ in range(n)])
    new = np.array([rng.choice([1, 1, 1, 1, 0, -1, rng.randint(2, 9)]) for _ in range(n)])
    width = -(-(int(lens.max()) + 9) // block)
    held = -(-lens // block)
    pool = int(held.sum()) + n + 3
    total = pool + shared
    ids = np.random.default_rng(seed).permutation(total)
    table = np.full((n, width), -1)
    table[np.arange(width)[None] < held[:, None]] = ids[:held.sum()]
    free = np.full(total, -1)
    free[:pool - held.sum()] = ids[held.sum():pool]
    prefix = i32(ids[pool:]) if shared else None
    tokens = int(new.clip(0).sum()) + rng.choice([0, 0, 5])
    if tokens == 0:
        tokens = 1
    order = rng.choice(["token", "head", "apart"])
    shape = {"token": (total, block, hkv, dim), "head": (total, hkv, block, dim), "apart": (block, total, hkv, dim)}[order]
    caches = []
    for _ in range(2):
        c = torch.full(shape, math.nan, device="cuda", dtype=dtype)
        c = {"token": c, "head": c.transpose(1, 2), "apart": c.transpose(0, 1)}[order]
        for i in range(n):
            at = torch.arange(int(lens[i]), device="cuda")
            if len(at):
                c[torch.tensor(table[i], device="cuda")[at // block], at % block] = rn(len(at), hkv, dim)
        for b in ids[pool:]:
            c[int(b)] = rn(block, hkv, dim)
        caches.append(c)
    k, v = caches
    d = kv.Decoder(total, block, hq, hkv, dim, dtype=dtype, max_rows=max(n, tokens))

    want = kv_plain.assign(lens.tolist(), new.tolist(), table.tolist(), free.tolist(), int(pool - held.sum()), block, tokens,
                           shared * block)
    t = i32(table)
    plan = d.assign(i32(lens), i32(new), t, i32(free), i32([pool - held.sum()]), tokens, prefix_len=shared * block)
    for f in plan._fields:
        assert getattr(plan, f).tolist() == want[f], f
    assert t.tolist() == want["table"]

    positions = int(plan.positions.max()) + 1
    angle = torch.rand(positions, max(1, rot // 2), generator=g, device="cuda") * 6.3
    rope = torch.cat((angle.cos(), angle.sin()), 1) if rot else None
    w = [rn(dim) if rng.random() < 0.7 else None for _ in range(2)]
    qkv = rn(tokens, (hq + 2 * hkv) * dim)
    wanted, mags = kv_plain.append(qkv, plan.positions, plan.slots, rope, *w, EPS, pairs, hq, hkv, dim)
    q = d.append(qkv, plan.positions, plan.slots, k, v, rope, *w, eps=EPS, pairs=pairs)
    real = plan.slots >= 0
    tol = kv_plain.UNIT[dtype] * wanted.abs() * (1 + 2.0 ** -6) + 2.0 ** -20 * mags + 2.0 ** -24
    assert ((q.double() - wanted[:, :hq]).abs() <= tol[:, :hq])[real].all() and (q[~real] == 0).all()
    at = plan.slots[real]
    assert ((k[at // block, at % block].double() - wanted[real, hq:hq + hkv]).abs() <= tol[real, hq:hq + hkv]).all()

    kw = dict(rows=plan.rows, prefix=prefix, window=window, sinks=sinks)
    out, lse = d.attend(q, k, v, t, plan.visible, lse=True, **kw)
    assert d.status() == 0
    kv_plain.check_attend(out, lse, *kv_plain.attend(q, k, v, t, plan.visible, **kw))
