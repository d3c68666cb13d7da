"""Attention over paged tokens against 64 bits, request by request (bounds: kv_plain.py)."""
import math

import numpy as np
import pytest

import kv_plain
from conftest import cuda_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]


def inputs(lens, hq, hkv, dim, block, dtype="bfloat16", shared=0, order="token", seed=0, rows=None):
    """Queries and a cache whose places that no request has are NaN."""
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
    shape = {"token": (total, block, hkv, dim), "head": (total, hkv, block, dim), "apart": (block, total, hkv, dim)}[order]
    caches = []
    for _ in range(2):
        c = torch.full(shape, math.nan, device="cuda", dtype=dtype)
        c = {"token": c, "head": c.transpose(1, 2), "apart": c.transpose(0, 1)}[order]
        for i, x in enumerate(lens):
            at = torch.arange(int(x), device="cuda")
            b = torch.tensor(table[i], device="cuda")[at // block]
            c[b, at % block] = torch.randn(int(x), hkv, dim, generator=g, device="cuda").to(dtype)
        for b in first:
            c[int(b)] = torch.randn(block, hkv, dim, generator=g, device="cuda").to(dtype)
        caches.append(c)
    n = len(lens) if rows is None else len(rows)
    q = torch.randn(n, hq, dim, generator=g, device="cuda").to(dtype)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(q=q, k=caches[0], v=caches[1], table=i32(table), lens=i32(lens), prefix=i32(first) if shared else None)


def decoder(s, max_rows=None):
    from paper_2608_02244_gb300 import kv
    return kv.Decoder(s["k"].shape[0], s["k"].shape[1], s["q"].shape[1], s["k"].shape[2], s["q"].shape[2], dtype=s["q"].dtype,
                      max_rows=max_rows or max(1, s["q"].shape[0]))


def check(s, d=None, **kw):
    d = d or decoder(s)
    out, lse = d.attend(**s, lse=True, **kw)
    assert d.status() == 0
    kv_plain.check_attend(out, lse, *kv_plain.attend(**s, **kw))
    return out, lse


LENS = [0, 1, 2, 15, 16, 17, 63, 64, 65, 0, 127, 128, 129, 300, 1000, 1]


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("block", [8, 16, 32, 64, 128, 256])
def test_lengths(dim, dtype, block):
    check(inputs(LENS, 8, 2, dim, block, dtype, seed=block))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (2, 1), (15, 5), (7, 1), (28, 4), (64, 8), (16, 1), (17, 1), (48, 1), (66, 2)])
def test_heads(hq, hkv):
    check(inputs([5, 0, 200, 77], hq, hkv, 64 if hq > 32 else 128, 16, seed=hq))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (50, 4), (64, 64), (100, 33), (127, 200), (500, 3), (1000, 4), (5000, 9)])
@pytest.mark.parametrize("block", [8, 64])
def test_windows(window, sinks, block):
    check(inputs(LENS + [555, 3001], 6, 2, 64, block, seed=window), window=window, sinks=sinks)


@pytest.mark.parametrize("shared,block", [(1, 8), (3, 8), (17, 8), (5, 16), (1, 64), (3, 128), (2, 256)])
@pytest.mark.parametrize("dim,dtype", [(64, "float16"), (128, "bfloat16"), (256, "bfloat16")])
def test_prefixes(shared, block, dim, dtype):
    check(inputs(LENS, 8, 2, dim, block, dtype, shared=shared, seed=shared))


@pytest.mark.parametrize("window,sinks", [(3, 2), (60, 4), (100, 300), (400, 7), (4000, 1)])
def test_prefix_with_window(window, sinks):
    check(inputs(LENS, 4, 1, 128, 16, shared=9, seed=window), window=window, sinks=sinks)


def test_window_that_hides_nothing():
    """A window of at least the table's and the prefix's tokens is none; one token less is one."""
    import torch
    s = inputs([128, 100, 1] * 10, 4, 1, 64, 16, shared=60)
    whole = 16 * (60 + s["table"].shape[1])
    want = check(s)[0]
    assert torch.equal(decoder(s).attend(**s, window=whole, sinks=3), want)
    assert torch.equal(decoder(s).attend(**s, window=2**31 - 1), want)
    check(s, window=whole - 1)


@pytest.mark.parametrize("n,hq,hkv,shared,block", [(100, 8, 1, 40, 16), (33, 28, 4, 130, 8), (300, 4, 4, 9, 64), (129, 16, 2, 33, 32),
                                                   (17, 64, 8, 7, 256), (260, 7, 1, 65, 8)])
@pytest.mark.parametrize("dim,dtype", [(64, "bfloat16"), (128, "float16"), (256, "bfloat16")])
def test_prefix_of_many(n, hq, hkv, shared, block, dim, dtype):
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 90, n)
    check(inputs(lens, hq, hkv, dim, block, dtype, shared=shared, seed=n))


@pytest.mark.parametrize("n,shared", [(7, 1023), (7, 1024), (8, 219), (8, 220), (9, 191), (9, 192)])
def test_around_prefix_apart(n, shared):
    """Both sides of the sizes from which a prefix has its own kernel."""
    check(inputs([20 + 7 * i for i in range(n)], 8, 2, 64, 8, shared=shared, seed=n))


@pytest.mark.parametrize("n,hq,hkv,dim,shared,block", [(40, 2, 2, 64, 500, 8), (500, 3, 1, 128, 60, 32), (70, 20, 10, 64, 300, 16),
                                                       (150, 128, 1, 64, 20, 128), (16, 130, 1, 128, 40, 64), (9, 8, 8, 128, 200, 64)])
def test_prefix_items_and_blocks(n, hq, hkv, dim, shared, block):
    """Row tiles with rows left over, one or two to an item, items cut by blocks and blocks of several items; more
    query heads on a key head than rows in a tile (not apart)."""
    check(inputs([1 + i % 9 for i in range(n)], hq, hkv, dim, block, shared=shared, seed=n))


@pytest.mark.parametrize("dim,dtype", [(64, "float16"), (128, "bfloat16")])
@pytest.mark.parametrize("shape", ["rising", "falling", "steps"])
def test_prefix_maxima_that_move(dim, dtype, shape):
    """Scores that grow along the prefix: the running maximum moves often, by little and by much."""
    import torch
    s = inputs([30, 0, 1, 5] * 8, 4, 1, dim, 16, dtype, shared=80, seed=1)
    x = torch.linspace(0, 1, 80 * 16, device="cuda")
    size = {"rising": 6 * x, "falling": 6 * (1 - x), "steps": 8 * (x * 5).floor() / 5}[shape].view(80, 16, 1, 1)
    s["k"][s["prefix"].long()] = (s["k"][s["prefix"].long()] * size).to(s["k"].dtype)
    check(s)


def test_prefix_extreme_keys():
    """Keys of -infinite score in whole tiles, and an undefined one, which every query sees."""
    import torch
    s = inputs([30, 2, 90, 1] * 16, 2, 1, 128, 64, shared=40, seed=2)
    s["q"] = s["q"].abs()
    b = s["prefix"].long()
    s["k"][b[:10]] = -math.inf
    s["k"][b[30]] = -math.inf
    out, lse = decoder(s).attend(**s, lse=True)
    want, want_lse, size = kv_plain.attend(**s)
    kv_plain.check_attend(out, lse, want, want_lse, size)
    s["k"][b[20], 3, 0, 5] = math.nan
    out, lse = decoder(s).attend(**s, lse=True)
    assert out.isnan().all() and lse.isnan().all()


@pytest.mark.parametrize("n", [1700, 1900, 2600])
def test_many_queries_of_128(n):
    """Both sides of the query count from which one block less fits an SM."""
    check(inputs(np.arange(n) % 50, 2, 1, 128, 16, seed=n))


@pytest.mark.parametrize("order", ["token", "head", "apart"])
@pytest.mark.parametrize("shared", [0, 20, 200])
def test_cache_orders(order, shared):
    check(inputs([100] * 40 + [0, 3], 8, 2, 128, 16, order=order, shared=shared))


@pytest.mark.parametrize("n", [1, 3, 500, 2000, 4096])
def test_many_queries(n):
    """Short ragged requests: items that end inside runs, more than one wave's worth."""
    rng = np.random.default_rng(n)
    check(inputs(np.minimum(rng.integers(0, 140, n), rng.integers(0, 140, n)), 4, 2, 64, 8, seed=n))


def test_one_long_request():
    check(inputs([70001], 8, 1, 128, 64))
    check(inputs([40000, 1, 0, 39999], 2, 2, 128, 16))


def test_large_scores_and_extreme_values():
    """Scores far apart, values at the type's ends, and a scale of the caller's."""
    import torch
    s = inputs([300, 40, 7], 4, 2, 128, 16, "float16")
    s["q"] *= 30
    check(s, scale=0.11)
    s = inputs([300, 40, 7], 4, 2, 128, 16, "bfloat16")
    s["v"][s["table"][0, 0]] = 3e38
    out, lse = decoder(s).attend(**s, lse=True)
    want = kv_plain.attend(**s)
    assert torch.equal(torch.isfinite(out[1:]), torch.isfinite(want[0][1:])) and torch.isfinite(lse).all()


def test_infinite_keys_and_values():
    """An infinite value that is seen shows; one that is not seen (beyond a length, outside a window) does not."""
    import torch
    s = inputs([200, 150, 90], 2, 1, 64, 16)
    s["v"][s["table"][1, 0], 3] = math.inf
    out = decoder(s).attend(**s)
    assert (out[1] == math.inf).all() and torch.isfinite(out[0]).all() and torch.isfinite(out[2]).all()
    out = decoder(s).attend(**s, window=100, sinks=3)
    assert torch.isfinite(out).all()
    s["k"][s["table"][0, 1], 5] = math.nan
    out, lse = decoder(s).attend(**s, lse=True)
    assert out[0].isnan().all() and lse[0].isnan().all() and torch.isfinite(out[2]).all()
    # keys whose score is -infinity get no weight
    s = inputs([64, 64], 2, 1, 64, 16)
    s["q"][0] = 1
    s["k"][s["table"][0, :2].long()] = -math.inf
    got, _ = decoder(s).attend(**s, lse=True)
    assert torch.isfinite(got[0]).all()


def test_rows_of_one_request():
    """Several new tokens of a request: each sees the tokens up to itself; entries without a row see nothing."""
    import torch
    s = inputs([300, 40], 8, 2, 128, 16, rows=range(10))
    rows = torch.tensor([0, 0, 0, 1, -1, 0, 1, 1, 0, -1], dtype=torch.int32, device="cuda")
    s["lens"] = torch.tensor([298, 299, 300, 40, 9, 1, 17, 0, 130, 0], dtype=torch.int32, device="cuda")
    out, lse = check(s, rows=rows)
    assert (out[4] == 0).all() and (lse[9] == -math.inf).all()


def test_strided_queries_and_outputs():
    import torch
    s = inputs([30, 0, 200], 6, 2, 64, 8)
    want = check(s)[0]
    wide = torch.full((3, 10, 72), math.nan, device="cuda", dtype=torch.bfloat16)
    q = wide[:, 2:8, :64]
    q.copy_(s["q"])
    out = torch.full((6, 3, 64), math.nan, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    assert decoder(s).attend(**dict(s, q=q), out=out) is out
    assert torch.equal(out, want)


def test_repeats_and_handles():
    """The same bits every time, on another stream, from a graph, and with a handle for more rows."""
    import torch
    rng = np.random.default_rng(0)
    s = inputs(rng.integers(0, 3000, 40), 16, 2, 128, 16, shared=30)
    d = decoder(s)
    want = check(s, d)[0]
    for _ in range(5):
        assert torch.equal(d.attend(**s), want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = d.attend(**s, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = d.attend(**s)
    out.zero_()
    graph.replay()
    assert torch.equal(out, want)
    check(s, decoder(s, max_rows=4096))
    small = dict(s, q=s["q"][:1], lens=s["lens"][:1])
    check(small, d)


def test_cache_beyond_32_bits():
    """Blocks whose elements lie past 2^31."""
    import torch
    from paper_2608_02244_gb300 import kv
    block, hkv, dim = 256, 8, 256
    blocks = 2**31 // (block * hkv * dim) + 5
    k = torch.empty(blocks, block, hkv, dim, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    ids = [blocks - 1, 0, blocks - 2]
    for b in ids:
        k[b].normal_()
        v[b].normal_()
    s = dict(q=torch.randn(3, 16, dim, device="cuda").bfloat16(), k=k, v=v, lens=torch.tensor([700, 256, 1], dtype=torch.int32, device="cuda"),
             table=torch.tensor([ids, ids, ids], dtype=torch.int32, device="cuda"), prefix=torch.tensor(ids[:1], dtype=torch.int32, device="cuda"))
    check(s)
    d = kv.Decoder(blocks, block, 16, hkv, dim, max_rows=4)
    qkv = torch.randn(1, 32 * dim, device="cuda").bfloat16()
    d.append(qkv, None, torch.tensor([(blocks - 1) * block + 9], device="cuda"), k, v)
    assert torch.equal(v[blocks - 1, 9].flatten(), qkv[0, 24 * dim:])


def test_reports_invalid_values():
    """Block numbers outside the cache and lengths beyond the table are reported; other requests are as before."""
    import torch
    from paper_2608_02244_gb300 import kv
    for name, at, value in (("table", (1, 2), -5), ("table", (1, 2), 10**6), ("lens", 1, 10**6), ("prefix", 1, 10**6)):
        s = inputs([100, 100, 100], 8, 2, 128, 16, shared=3)
        d = decoder(s)
        want = d.attend(**s)
        s[name][at] = value
        got = d.attend(**s)
        assert d.status() == kv.ISJL_ERR_INVALID_ARG and d.status() == 0
        if name != "prefix":
            assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
        if name == "lens":
            assert (got[1] == 0).all()
    s = inputs([9] * 100, 8, 2, 128, 16, shared=60)            # a prefix done apart
    d = decoder(s)
    assert torch.isfinite(d.attend(**s)).all() and d.status() == 0
    for value in (-1, s["k"].shape[0]):
        s["prefix"][59] = value
        assert torch.isfinite(d.attend(**s)).all()
        assert d.status() == kv.ISJL_ERR_INVALID_ARG and d.status() == 0
    s = inputs([100, 100], 8, 2, 128, 16)
    d = decoder(s)
    rows = torch.tensor([0, 7], dtype=torch.int32, device="cuda")
    out = d.attend(**s, rows=rows)
    assert d.status() == kv.ISJL_ERR_INVALID_ARG and (out[1] == 0).all()


def test_refusals():
    import torch
    from paper_2608_02244_gb300 import kv
    s = inputs([100, 30, 2], 8, 2, 64, 16)
    d = decoder(s)
    d.attend(**s)
    assert d.attend(**dict(s, q=s["q"][:0], lens=s["lens"][:0])).shape == (0, 8, 64)
    odd = torch.zeros(3 * 8 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(3, 8, 64)
    for bad in (dict(q=s["q"].float()), dict(q=odd), dict(q=s["q"][:, :4]), dict(q=torch.cat([s["q"]] * 2)), dict(k=s["k"].float()),
                dict(v=s["v"][:-1]), dict(table=s["table"].long()), dict(table=s["table"][:2]), dict(lens=s["lens"][:2]),
                dict(lens=s["lens"].long()), dict(rows=s["lens"][:2]), dict(prefix=s["table"].long()[0]), dict(window=-1), dict(sinks=-1),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(out=s["q"].float()), dict(out=odd)):
        with pytest.raises(kv.IsjlError) as e:
            d.attend(**dict(s, **bad))
        assert e.value.status == kv.ISJL_ERR_INVALID_ARG
    torch.cuda.synchronize()
