"""A cache in 4 bits: codes against the format's definition, values read back bit for bit, attention against 64 bits
over what the codes stand for (bounds: kv4_plain.py and kv_plain.py)."""
import math

import numpy as np
import pytest

import kv4_plain
import kv_plain
from conftest import cuda_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]
EPS = 1e-6


# ---- append4 and read4
def new_tokens(n, hq, hkv, dim, rot, dtype, norm, block, seed, positions=300, order="token"):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    blocks = -(-n // block) + 2
    s = dict(qkv=rn(n, (hq + 2 * hkv) * dim).to(dtype),
             positions=torch.randint(0, positions, (n,), generator=g, device="cuda", dtype=torch.int32),
             slots=torch.randperm(blocks * block, generator=g, device="cuda")[:n],
             cache=kv4_plain.cache(blocks, block, hkv, dim, dtype, order, math.nan))
    if rot:
        angle = torch.rand(positions, rot // 2, generator=g, device="cuda") * 6.3
        s["rope"] = torch.cat((angle.cos(), angle.sin()), 1)
    if norm:
        s["q_weight"], s["k_weight"] = rn(dim).to(dtype), rn(dim).to(dtype)
    return s


def same_bits(a, b):
    import torch
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def check_append(s, hq, hkv, dim, pairs=False, **kw):
    import torch
    from paper_2608_02244_gb300 import kv
    c, n, dtype = s["cache"], s["qkv"].shape[0], s["qkv"].dtype
    block = c.k.shape[1]
    d = kv.Decoder(c.k.shape[0], block, hq, hkv, dim, dtype=dtype, max_rows=1)
    want, mags = kv_plain.append(s["qkv"], s["positions"], s["slots"], s.get("rope"), s.get("q_weight"), s.get("k_weight"), EPS,
                                 pairs, hq, hkv, dim)
    old, qkv = [t.clone() for t in c], s["qkv"].clone()
    q = d.append4(**s, eps=EPS, pairs=pairs, **kw)
    k, v = d.read4(s["slots"], c)
    assert d.status() == 0
    real = s["slots"] >= 0
    tol = kv_plain.UNIT[dtype] * want.abs() * (1 + 2.0 ** -6) + 2.0 ** -20 * mags + 2.0 ** -24
    assert ((q.double() - want[:, :hq]).abs() <= tol[:, :hq])[real].all()
    assert (q[~real] == 0).all() and (k[~real] == 0).all() and (v[~real] == 0).all()
    at = s["slots"][real]
    b, p = at // block, at % block
    # values: their codes and scales are the definition's, bit for bit (their inputs are exact)
    codes, scales = kv4_plain.coded(qkv.view(n, -1, dim)[real, hq + hkv:], dtype)
    assert torch.equal(c.v[b, p].cpu(), codes) and same_bits(c.v_scale[b, p].cpu(), scales)
    # both: read back as the codes say, and as near to what was written as the format allows
    for got, x, y, lo in ((k, c.k, c.k_scale, hq), (v, c.v, c.v_scale, hq + hkv)):
        assert torch.equal(got[real], kv4_plain.values(x[b, p], y[b, p]))
        off = (got.double() - want[:, lo:lo + hkv]).abs()[real]
        assert (off <= kv4_plain.bound(want[:, lo:lo + hkv], mags[:, lo:lo + hkv], dtype)[real]).all()
    for x, o in zip(c, old):                          # nothing else was written
        x, o = x.clone(), o.clone()
        x[b, p] = 0
        o[b, p] = 0
        assert same_bits(x, o)
    return q


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("rot", ["all", "half", 16, 0])
def test_append_values(dim, dtype, pairs, rot):
    import torch
    rot = {"all": dim, "half": dim // 2}.get(rot, rot)
    check_append(new_tokens(37, 6, 2, dim, rot, getattr(torch, dtype), rot != 16, 16, dim + rot), 6, 2, dim, pairs)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 5), (7, 1), (28, 4), (64, 8), (33, 11)])
@pytest.mark.parametrize("n", [1, 2, 130])
@pytest.mark.parametrize("dim", [64, 128])
def test_append_heads(hq, hkv, n, dim):
    import torch
    check_append(new_tokens(n, hq, hkv, dim, dim, torch.bfloat16, True, 8, n), hq, hkv, dim)


@pytest.mark.parametrize("order", ["token", "head", "apart"])
@pytest.mark.parametrize("block", [8, 64, 256])
@pytest.mark.parametrize("dim", [64, 256])
def test_append_orders(order, block, dim):
    import torch
    check_append(new_tokens(200, 8, 4, dim, dim, torch.float16, True, block, block, order=order), 8, 4, dim)


@pytest.mark.parametrize("n", [3647, 3648, 9001])
@pytest.mark.parametrize("dim,hq,hkv", [(64, 3, 1), (128, 6, 2), (256, 2, 1)])
def test_append_many(n, dim, hq, hkv):
    """Both sides of the number of tokens from which a token has one warp."""
    import torch
    check_append(new_tokens(n, hq, hkv, dim, dim, torch.bfloat16, True, 16, n), hq, hkv, dim)


def test_append_padding_and_bad_slots():
    import torch
    from paper_2608_02244_gb300 import kv
    s = new_tokens(50, 4, 2, 64, 64, torch.bfloat16, True, 16, 3)
    s["slots"][[0, 7, 49]] = -1
    check_append(s, 4, 2, 64)
    s = new_tokens(20, 4, 2, 64, 64, torch.bfloat16, False, 16, 4)
    d = kv.Decoder(s["cache"].k.shape[0], 16, 4, 2, 64, max_rows=1)
    total = s["cache"].k.shape[0] * 16
    s["slots"][3] = total
    s["positions"][5] = 300
    q = d.append4(**s)
    assert d.status() == kv.ISJL_ERR_INVALID_ARG and d.status() == 0
    assert (q[[3, 5]] == 0).all() and (q[[2, 4]] != 0).any()
    k, v = d.read4(s["slots"], s["cache"])
    assert d.status() == kv.ISJL_ERR_INVALID_ARG
    assert (k[3] == 0).all() and (v[3] == 0).all() and v[5].isnan().all()      # token 5 was not written
    s["slots"][3] = 2**62
    d.read4(s["slots"], s["cache"])
    assert d.status() == kv.ISJL_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_append_extreme_groups(dtype):
    """Groups of one value throughout, of two, of tiny numbers, far from 0; undefined and infinite values."""
    import torch
    from paper_2608_02244_gb300 import kv
    dtype = getattr(torch, dtype)
    n, dim = 12, 64
    x = torch.zeros(n, 3, dim, device="cuda")
    x[1] = 0.37
    x[2, :, ::2] = -1.5
    x[3] = torch.linspace(-1, 1, dim, device="cuda") * (2.0 ** -20 if dtype == torch.float16 else 2.0 ** -120)
    x[4] = 1000 + torch.arange(dim, device="cuda") % 7
    x[5] = -20000 + 40000 * (torch.arange(dim, device="cuda") % 2)
    x[6] = torch.arange(dim, device="cuda") - 31.5
    x[7] = 2.0 ** -24
    x = x.to(dtype)
    fine = x.clone()
    x[8, :, 3] = math.nan
    x[9, :, 40] = math.inf
    x[10, :, 63] = -math.inf
    d = kv.Decoder(1, 16, 1, 1, dim, dtype=dtype, max_rows=1)
    c = d.cache4()
    slots = torch.arange(n, device="cuda")
    d.append4(x.view(n, -1), None, slots, c)
    k, v = d.read4(slots, c)
    assert d.status() == 0
    for got, head in ((k[:, 0], 1), (v[:, 0], 2)):
        want = fine[:, head]
        off = (got.double() - want.double()).abs()
        live = torch.ones(n, dim, dtype=torch.bool, device="cuda")
        live[8, :32] = live[9, 32:] = live[10, 32:] = False
        assert (off <= kv4_plain.bound(want.double(), want.double().abs(), dtype))[live].all()
        assert got[~live].isnan().all()
        assert torch.equal(got[[0, 1, 7]], want[[0, 1, 7]])                    # one value: exact
    codes, scales = kv4_plain.coded(fine[:8, 2], dtype)
    assert torch.equal(c.v[0, :8, 0].cpu(), codes) and same_bits(c.v_scale[0, :8, 0].cpu(), scales)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_read_all_codes(dtype, dim):
    """Every code with many scales, in each order of axes, into strided outputs, with slots twice and none."""
    import torch
    from paper_2608_02244_gb300 import kv
    dtype, g = getattr(torch, dtype), torch.Generator(device="cuda").manual_seed(dim)
    for order in ("token", "head", "apart"):
        c = kv4_plain.cache(9, 32, 3, dim, dtype, order, math.nan)
        at = torch.arange(9 * 32, device="cuda")
        kv4_plain.fill(c, at // 32, at % 32, g)
        slots = torch.randint(-2, 9 * 32, (1001,), generator=g, device="cuda")
        d = kv.Decoder(9, 32, 3, 3, dim, dtype=dtype, max_rows=1)
        out = [torch.full((1001, 5, dim + 8), 7.0, device="cuda", dtype=dtype) for _ in range(2)]
        k, v = d.read4(slots, c, k=out[0][:, 1:4, :dim], v=out[1][:, 1:4, :dim])
        assert d.status() == 0
        for got, whole, want in zip((k, v), out, kv4_plain.in_16_bits(c)):
            want = torch.where((slots >= 0)[:, None, None], want[slots // 32, slots % 32], 0)
            assert torch.equal(got, want)
            assert (whole[:, [0, 4]] == 7).all() and (whole[..., dim:] == 7).all()
    k, v = d.read4(slots[:0], c)
    assert k.shape == (0, 3, dim) and d.status() == 0


# ---- attend4
def requests(lens, hq, hkv, dim, block, dtype="bfloat16", shared=0, order="token", seed=0, rows=None):
    """Queries and a cache whose places that no request has stand for NaN."""
    import torch
    dtype = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens)
    held = -(-lens // block)
    total = int(held.sum()) + shared + 2
    ids = rng.permutation(total)
    table = np.full((len(lens), max(1, int(held.max(initial=1)))), -1)
    table[np.arange(table.shape[1])[None] < held[:, None]] = ids[:held.sum()]
    first = ids[held.sum():held.sum() + shared]
    c = kv4_plain.cache(total, block, hkv, dim, dtype, order, math.nan)
    at = [(table[i, j // block], j % block) for i, x in enumerate(lens) for j in range(int(x))] + [
        (b, j) for b in first for j in range(block)]
    if at:
        b, p = torch.tensor(np.array(at), device="cuda").T
        kv4_plain.fill(c, b, p, g)
    n = len(lens) if rows is None else len(rows)
    q = torch.randn(n, hq, dim, generator=g, device="cuda").to(dtype)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(q=q, cache=c, table=i32(table), lens=i32(lens), prefix=i32(first) if shared else None)


def decoder4(s, max_rows=None):
    from paper_2608_02244_gb300 import kv
    c = s["cache"]
    return kv.Decoder(c.k.shape[0], c.k.shape[1], s["q"].shape[1], c.k.shape[2], s["q"].shape[2], dtype=s["q"].dtype,
                      max_rows=max_rows or max(1, s["q"].shape[0]))


def check_attend4(s, d=None, **kw):
    d = d or decoder4(s)
    out, lse = d.attend4(**s, lse=True, **kw)
    assert d.status() == 0
    plain = {x: y for x, y in s.items() if x != "cache"}
    k, v = kv4_plain.in_16_bits(s["cache"])
    kv_plain.check_attend(out, lse, *kv_plain.attend(**plain, k=k, v=v, **kw))
    return out, lse


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 0, 127, 128, 129, 300, 1000, 1]


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("block", [8, 16, 32, 64, 128, 256])
def test_attend_lengths(dim, dtype, block):
    check_attend4(requests(LENS, 8, 2, dim, block, dtype, seed=block))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (2, 1), (15, 5), (7, 1), (8, 1), (9, 1), (28, 4), (64, 8), (16, 1), (17, 1), (48, 1), (66, 2)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_heads(hq, hkv, dim):
    check_attend4(requests([5, 0, 200, 77], hq, hkv, dim, 16, seed=hq))


@pytest.mark.parametrize("order", ["token", "head", "apart"])
@pytest.mark.parametrize("block", [8, 32, 256])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_orders(order, block, dim):
    check_attend4(requests([400, 3, 130, 33], 8, 4, dim, block, order=order, seed=block))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (50, 4), (64, 64), (100, 33), (127, 200), (500, 3), (1000, 4), (5000, 9)])
@pytest.mark.parametrize("block", [8, 64])
def test_attend_windows(window, sinks, block):
    check_attend4(requests(LENS + [555, 3001], 6, 2, 64, block, seed=window), window=window, sinks=sinks)


@pytest.mark.parametrize("shared,block", [(1, 8), (3, 8), (17, 8), (5, 16), (1, 64), (3, 128), (2, 256)])
@pytest.mark.parametrize("dim,dtype", [(64, "float16"), (128, "bfloat16"), (256, "bfloat16")])
def test_attend_prefixes(shared, block, dim, dtype):
    s = requests(LENS, 8, 2, dim, block, dtype, shared=shared, seed=shared)
    check_attend4(s)
    check_attend4(s, window=60, sinks=3)


def test_attend_rows():
    """Several queries of a request, requests in any order, rows that are none."""
    import torch
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    rows = [3, 0, 0, 2, -1, 1, 3]
    s = requests([50, 3, 200, 90], 4, 2, 128, 16, rows=rows, seed=5)
    s["lens"] = i32([90, 50, 17, 200, 5, 0, 1])
    check_attend4(s, rows=i32(rows))


@pytest.mark.parametrize("n,longest,hq,hkv,dim", [(300, 700, 8, 2, 128), (1, 30000, 4, 1, 128), (3, 9000, 16, 1, 64),
                                                  (700, 40, 9, 3, 64), (40, 3001, 4, 4, 256), (2000, 9, 5, 1, 128)])
def test_attend_many(n, longest, hq, hkv, dim):
    """Items cut by the ends of the grid's runs, and runs of many items; the same bits every time."""
    import torch
    rng = np.random.default_rng(n)
    s = requests(np.where(rng.random(n) < 0.1, 0, rng.integers(1, longest + 1, n)) if n > 3 else [longest] * n, hq, hkv, dim, 16,
                 order="head", seed=n)
    d = decoder4(s)
    want, lse = check_attend4(s, d)
    for _ in range(5):
        out, again = d.attend4(**s, lse=True)
        assert torch.equal(out, want) and torch.equal(again, lse)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("shape", ["rising", "falling", "steps"])
def test_attend_maxima_that_move(dtype, shape):
    import torch
    s = requests([3000, 0, 1, 700], 4, 1, 128, 16, dtype, seed=1)
    x = torch.linspace(0, 1, 3000, device="cuda")
    size = {"rising": 5 * x, "falling": 5 * (1 - x), "steps": 7 * (x * 5).floor() / 5}[shape]
    at = torch.arange(3000, device="cuda")
    b = s["table"][0].long()[at // 16]
    s["cache"].k_scale[b, at % 16] = (s["cache"].k_scale[b, at % 16] * size[:, None, None, None]).to(s["q"].dtype)
    check_attend4(s)


def test_attend_small_weights_count():
    """fp16: thousands of tokens far below the largest score."""
    import torch
    s = requests([40000], 1, 1, 64, 16, "float16", seed=3)
    c, at = s["cache"], torch.arange(40000, device="cuda")
    b = s["table"][0].long()[at // 16]
    c.k[b, at % 16] = 0
    c.k_scale[b, at % 16] = 0
    s["q"][:] = 1
    c.k_scale[int(s["table"][0, 0]), 0, :, :, 1] = 2.0          # a score of 2 * 64 / 8 = 16 for the first token
    c.v_scale[b, at % 16, :, :, 1] = 1.0
    c.v_scale[b, at % 16, :, :, 0] = 0
    c.v_scale[int(s["table"][0, 0]), 0] = 0
    check_attend4(s)


def test_attend_undefined_values():
    """What is seen shows, what is not seen does not."""
    import torch
    s = requests([100, 100, 100], 4, 2, 128, 16, seed=4)
    c, t = s["cache"], s["table"].long()
    want, _ = check_attend4(s, window=20, sinks=2)
    c.v_scale[t[0, 1], 3] = math.nan                  # place 19: behind the window
    c.k_scale[t[0, 1], 4] = math.inf
    c.v_scale[t[1, 6], 0, 0, 1, 0] = math.nan         # place 96: seen
    out, lse = decoder4(s).attend4(**s, window=20, sinks=2, lse=True)
    assert torch.equal(out[0], want[0]) and torch.equal(out[2], want[2])
    assert out[1, :2, 32:64].isnan().all() and not out[1, :2, :32].isnan().any() and torch.equal(out[1, 2:], want[1, 2:])
    c.k_scale[t[2, 6], 1, 1] = math.nan
    out, lse = decoder4(s).attend4(**s, window=20, sinks=2, lse=True)
    assert out[2, 2:].isnan().all() and lse[2, 2:].isnan().all() and torch.equal(out[2, :2], want[2, :2])


def test_attend_bad_blocks_and_lengths():
    import torch
    from paper_2608_02244_gb300 import kv
    s = requests([40, 40, 40, 40], 4, 2, 64, 16, seed=6)
    d = decoder4(s)
    s["table"][1, 1] = s["cache"].k.shape[0]
    s["table"][2, 0] = -7
    s["lens"][3] = 3 * 16 + 1
    out, lse = d.attend4(**s, lse=True)
    assert d.status() == kv.ISJL_ERR_INVALID_ARG and d.status() == 0
    assert (out[3] == 0).all() and (lse[3] == -math.inf).all()
    # a block outside the cache reads as zeros
    z = [torch.cat((x, torch.zeros_like(x[:1]))) for x in kv4_plain.in_16_bits(s["cache"])]
    last = s["cache"].k.shape[0]
    table = torch.where((s["table"] < 0) | (s["table"] >= last), last, s["table"])
    kv_plain.check_attend(out[:3], lse[:3], *kv_plain.attend(s["q"][:3], z[0], z[1], table[:3], s["lens"][:3]))


@pytest.mark.parametrize("hq,hkv,dim", [(100, 100, 64), (700, 700, 64), (1024, 1024, 64), (1024, 256, 64), (305, 305, 256), (1000, 8, 64)])
def test_attend_many_heads(hq, hkv, dim):
    """Key heads in numbers that do not divide the grid's warps."""
    check_attend4(requests([70, 0, 200, 1, 33], hq, hkv, dim, 16, seed=hkv))


@pytest.mark.parametrize("number", ["n_blocks", -1, 2**31 - 1, -2**31])
def test_attend_any_bad_block_is_reported(number):
    """One block number outside the cache, whatever it is: reported, and its tokens read as zeros."""
    import torch
    from paper_2608_02244_gb300 import kv
    s = requests([70], 4, 2, 128, 16, seed=7)
    d = decoder4(s)
    last = s["cache"].k.shape[0]
    s["table"][0, 3] = last if number == "n_blocks" else number
    out, lse = d.attend4(**s, lse=True)
    assert d.status() == kv.ISJL_ERR_INVALID_ARG and d.status() == 0
    z = [torch.cat((x, torch.zeros_like(x[:1]))) for x in kv4_plain.in_16_bits(s["cache"])]
    table = torch.where((s["table"] < 0) | (s["table"] >= last), last, s["table"])
    kv_plain.check_attend(out, lse, *kv_plain.attend(s["q"], z[0], z[1], table, s["lens"]))


def test_attend_strided_and_given_outputs():
    import torch
    s = requests([70, 5, 300], 6, 2, 64, 16, seed=7)
    want, lse = check_attend4(s)
    q = torch.zeros(3, 9, 80, device="cuda", dtype=torch.bfloat16)
    q[:, 2:8, 8:72] = s["q"]
    out = torch.full((3, 7, 72), 5.0, device="cuda", dtype=torch.bfloat16)
    got = decoder4(s).attend4(**dict(s, q=q[:, 2:8, 8:72]), out=out[:, :6, :64])
    assert torch.equal(got, want) and (out[:, 6] == 5).all() and (out[..., 64:] == 5).all()
    got, again = decoder4(s).attend4(**s, scale=0.03, lse=True)
    plain = {x: y for x, y in s.items() if x != "cache"}
    k, v = kv4_plain.in_16_bits(s["cache"])
    kv_plain.check_attend(got, again, *kv_plain.attend(**plain, k=k, v=v, scale=0.03))


def test_attend_beyond_32_bits():
    """Codes and scales beyond 2^31 bytes and numbers."""
    import torch
    from paper_2608_02244_gb300 import kv
    blocks, block, hkv, dim = 300_000, 16, 8, 128
    d = kv.Decoder(blocks, block, 8, hkv, dim, max_rows=2)
    codes = torch.zeros(blocks, hkv, block, dim // 2, dtype=torch.uint8, device="cuda").transpose(1, 2)
    scales = torch.zeros(blocks, hkv, block, dim // 32, 2, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    c = kv.Cache4(codes, codes.clone(), scales, scales.clone())
    table = torch.tensor([[blocks - 1, 3, blocks - 2], [0, blocks // 2 + 9, 7]], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    at = torch.arange(48, device="cuda")
    for row in table.long():
        kv4_plain.fill(c, row[at // 16], at % 16, g)
    q = torch.randn(2, 8, dim, generator=g, device="cuda").bfloat16()
    lens = torch.tensor([48, 41], dtype=torch.int32, device="cuda")
    out, lse = d.attend4(q, c, table, lens, lse=True)
    slots = (table.long()[:, :, None] * 16 + torch.arange(16, device="cuda")).view(-1)
    k, v = d.read4(slots, c)
    assert d.status() == 0
    b, p = slots // 16, slots % 16
    assert torch.equal(k, kv4_plain.values(c.k[b, p], c.k_scale[b, p])) and torch.equal(v, kv4_plain.values(c.v[b, p], c.v_scale[b, p]))
    small = torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3)
    kv_plain.check_attend(out, lse, *kv_plain.attend(q, k.view(6, 16, hkv, dim), v.view(6, 16, hkv, dim), small, lens))
    qkv = torch.randn(96, 24 * dim, generator=g, device="cuda").bfloat16()
    d.append4(qkv, None, slots, c)
    k, v = d.read4(slots, c)
    want, sc = kv4_plain.coded(qkv.view(96, 24, dim)[:, 8:], torch.bfloat16)
    want = kv4_plain.values(want, sc)
    assert torch.equal(k.cpu(), want[:, :8]) and torch.equal(v.cpu(), want[:, 8:])


def test_graph_and_stream():
    """A step captured once and replayed with other inputs; a call on another stream."""
    import torch
    s = requests([70, 5, 300, 33], 8, 2, 128, 16, seed=8)
    d = decoder4(s)
    g = torch.Generator(device="cuda").manual_seed(2)
    qkv = torch.randn(4, 12 * 128, generator=g, device="cuda").bfloat16()
    slots = torch.tensor([int(s["table"][i, (n - 1) // 16]) * 16 + (n - 1) % 16 for i, n in enumerate(s["lens"].tolist())], device="cuda")

    def step():
        q = d.append4(qkv, None, slots, s["cache"])
        return d.attend4(**dict(s, q=q), lse=True) + d.read4(slots, s["cache"])

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in (3, 4):
        qkv.copy_(torch.randn(4, 12 * 128, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        graph.replay()
        got = [t.clone() for t in held]
        assert all(torch.equal(a, b) for a, b in zip(got, step()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    want, lse = d.attend4(**s, lse=True)
    torch.cuda.synchronize()
    out, again = d.attend4(**s, lse=True, stream=side)
    k, v = d.read4(slots, s["cache"], stream=side)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(again, lse) and torch.equal(k, got[2]) and torch.equal(v, got[3])


def test_refusals():
    import torch
    from paper_2608_02244_gb300 import kv
    s = requests([40, 3], 4, 2, 64, 16, seed=9)
    d, c = decoder4(s), s["cache"]

    def refused(call, *a, **kw):
        with pytest.raises(kv.IsjlError) as e:
            call(*a, **kw)
        assert e.value.status == kv.ISJL_ERR_INVALID_ARG

    slots = torch.zeros(2, dtype=torch.int64, device="cuda")
    shifted = torch.zeros(c.k.numel() + 16, dtype=torch.uint8, device="cuda")[8:8 + c.k.numel()].view(c.k.shape)
    wide = torch.zeros(c.k.shape[:3] + (40,), dtype=torch.uint8, device="cuda")[..., :32]      # strides of 40 bytes
    half = c.k_scale.half()
    for bad in (c[:3], (c.k, c.v, c.k_scale), c._replace(k=c.k.float()), c._replace(v=c.v[:1]), c._replace(k=shifted),
                c._replace(v=wide), c._replace(k_scale=half), c._replace(v_scale=c.v_scale.cpu()),
                c._replace(v_scale=c.v_scale.transpose(3, 4).contiguous().transpose(3, 4)), c._replace(k=c.k.expand(c.k.shape).as_strided(c.k.shape, (0, 0, 0, 1)))):
        refused(d.attend4, s["q"], bad, s["table"], s["lens"])
        refused(d.read4, slots, bad)
        refused(d.append4, torch.zeros(2, 8 * 64, device="cuda", dtype=torch.bfloat16), None, slots, bad)
    refused(d.attend4, s["q"].half(), c, s["table"], s["lens"])
    refused(d.attend4, s["q"], c, s["table"].long(), s["lens"])
    refused(d.attend4, s["q"], c, s["table"], s["lens"][:1])
    refused(d.attend4, s["q"], c, s["table"], s["lens"], window=-1)
    refused(d.attend4, s["q"], c, s["table"], s["lens"], scale=0.0)
    refused(d.attend4, s["q"], c, s["table"], s["lens"], scale=math.nan)
    refused(d.read4, slots.int(), c)
    refused(d.read4, slots, c, k=torch.zeros(2, 2, 32, device="cuda", dtype=torch.bfloat16))
    refused(d.read4, slots, c, v=torch.zeros(2, 2, 65, device="cuda", dtype=torch.bfloat16)[..., 1:])
    refused(d.append4, torch.zeros(2, 8 * 64 + 1, device="cuda", dtype=torch.bfloat16), None, slots, c)
    refused(d.append4, torch.zeros(2, 8 * 64, device="cuda", dtype=torch.bfloat16), None, slots, c, eps=-1.0)
    assert d.status() == 0
    d.close()
    refused(d.read4, slots, c)
