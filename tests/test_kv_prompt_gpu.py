"""Attention of packed prompts against 64 bits, query by query (bounds: kv_plain.py)."""
import math

import numpy as np
import pytest

import kv_plain
from conftest import cuda_available
from test_kv_attend_gpu import inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]


def prompts(counts, before, hq, hkv, dim, block, dtype="bfloat16", shared=0, order="token", seed=0, spare=0):
    """Packed queries of `counts` new tokens after `before` earlier ones of each row, and `spare` behind them."""
    import torch
    counts = np.asarray(counts)
    lens = counts + np.asarray(before)
    s = inputs(lens, hq, hkv, dim, block, dtype, shared, order, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    s["q"] = torch.randn(int(counts.sum()) + spare, hq, dim, generator=g, device="cuda").to(s["q"].dtype)
    s["starts"] = torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32, device="cuda")
    return s


def decoder(s, max_rows=None):
    from paper_2608_02244_gb300 import kv
    return kv.Decoder(s["k"].shape[0], s["k"].shape[1], s["q"].shape[1], s["k"].shape[2], s["q"].shape[2], dtype=s["q"].dtype,
                      max_rows=max_rows or max(1, s["lens"].shape[0]))


def plain(s, **kw):
    """Each query as a single one (64 bits, all queries of a row together)."""
    import torch
    q, k, v, table = s["q"], s["k"], s["v"], s["table"]
    hq, dim = q.shape[1:]
    block, hkv = k.shape[1], k.shape[2]
    window, sinks, scale = kw.get("window", 0), kw.get("sinks", 0), kw.get("scale") or dim ** -0.5
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    first = [] if s["prefix"] is None else s["prefix"].tolist()
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    size, lse = torch.zeros_like(out), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for i, length in enumerate(lens):
        a, b = starts[i], starts[i + 1]
        if a == b:
            continue
        end = len(first) * block + length
        blocks = torch.tensor(first + table[i, :-(-length // block)].tolist(), device="cuda")
        pos = torch.arange(end, device="cuda")
        kk, vv = (c[blocks[pos // block], pos % block].double() for c in (k, v))
        place = torch.arange(end - (b - a), end, device="cuda")[:, None]
        hidden = pos > place
        if window:
            hidden |= (pos <= place - window) & (pos >= sinks)
        x = torch.einsum("qhgd,lhd->hgql", q[a:b].double().view(b - a, hkv, hq // hkv, dim), kk) * scale
        x = x.masked_fill(hidden, -math.inf)
        p = x.softmax(-1)
        out[a:b] = torch.einsum("hgql,lhd->qhgd", p, vv).reshape(b - a, hq, dim)
        size[a:b] = torch.einsum("hgql,lhd->qhgd", p, vv.abs()).reshape(b - a, hq, dim)
        lse[a:b] = x.logsumexp(-1).permute(2, 0, 1).reshape(b - a, hq)
    return out, lse, size


def check(s, d=None, **kw):
    d = d or decoder(s)
    out, lse = d.prompt(**s, lse=True, **kw)
    assert d.status() == 0
    n = int(s["starts"][-1])
    want, want_lse, size = plain(s, **kw)
    kv_plain.check_attend(out[:n], lse[:n], want[:n], want_lse[:n], size[:n])
    return out, lse


COUNTS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 0, 127, 128, 129, 300, 1]


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("block", [8, 16, 32, 64, 128, 256])
def test_lengths(dim, dtype, block):
    check(prompts(COUNTS, [0] * len(COUNTS), 8, 2, dim, block, dtype, seed=block))


@pytest.mark.parametrize("count", [1, 2, 3, 8, 127, 128, 129, 255, 256, 257, 700])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_one_prompt(count, dim):
    check(prompts([count], [0], 4, 1, dim, 16, seed=count))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (2, 1), (15, 5), (3, 1), (7, 1), (28, 4), (64, 8), (16, 1), (17, 1), (48, 1), (100, 1),
                                    (128, 1), (129, 1), (66, 2), (300, 1)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_heads(hq, hkv, dim):
    check(prompts([5, 0, 200, 77], [3, 9, 0, 130], hq, hkv, dim, 16, seed=hq))


@pytest.mark.parametrize("before", [1, 7, 64, 127, 128, 129, 1000])
@pytest.mark.parametrize("dim,dtype", [(64, "float16"), (128, "bfloat16"), (256, "bfloat16")])
def test_chunks(before, dim, dtype):
    """Later chunks: queries after tokens that are in the cache already; single ones among them."""
    check(prompts([1, 40, 129, 1], [before, before, 2 * before, 0], 6, 2, dim, 16, dtype, seed=before))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (50, 4), (64, 64), (100, 33), (127, 200), (128, 128), (300, 3), (500, 129),
                                          (5000, 9)])
@pytest.mark.parametrize("dim,block", [(64, 8), (128, 64), (256, 16)])
def test_windows(window, sinks, dim, block):
    check(prompts([1, 40, 300, 0, 555, 700, 130], [0, 700, 0, 5, 3, 400, 129], 6, 2, dim, block, seed=window), window=window, sinks=sinks)


@pytest.mark.parametrize("shared,block", [(1, 8), (3, 8), (17, 8), (5, 16), (1, 64), (3, 128), (2, 256)])
@pytest.mark.parametrize("dim,dtype", [(64, "float16"), (128, "bfloat16"), (256, "bfloat16")])
def test_prefixes(shared, block, dim, dtype):
    s = prompts(COUNTS, [3] * len(COUNTS), 8, 2, dim, block, dtype, shared=shared, seed=shared)
    check(s)
    check(s, window=90, sinks=17)


@pytest.mark.parametrize("order", ["token", "head", "apart"])
@pytest.mark.parametrize("block", [8, 128, 256])
def test_orders(order, block):
    check(prompts([130, 20, 1], [0, 300, 40], 8, 4, 128, block, order=order, seed=block))


@pytest.mark.parametrize("counts,before,hq,hkv,dim", [([3000], [0], 8, 2, 128), ([64] * 3, [20000] * 3, 8, 2, 128), ([1], [50000], 4, 1, 64),
                                                      ([900, 1, 2500, 40] * 5, [0, 7000, 100, 0] * 5, 4, 2, 64),
                                                      ([2] * 700, [30] * 700, 7, 1, 128), ([1500, 20], [0, 9000], 4, 2, 256)])
def test_items_cut(counts, before, hq, hkv, dim):
    """Items cut by the ends of the grid's runs, many items in a run, one item in many; the same bits every time."""
    import torch
    s = prompts(counts, before, hq, hkv, dim, 32, seed=len(counts))
    d = decoder(s)
    want, lse = check(s, d)
    for _ in range(5):
        out, again = d.prompt(**s, lse=True)
        assert torch.equal(out, want) and torch.equal(again, lse)


def test_many_rows():
    """As many rows as a call takes, most of them empty."""
    import torch
    rng = np.random.default_rng(1)
    counts = np.where(rng.random(4096) < 0.7, 0, rng.integers(1, 20, 4096))
    check(prompts(counts, rng.integers(0, 30, 4096), 2, 1, 64, 8, seed=1))


@pytest.mark.parametrize("dim,dtype", [(64, "float16"), (128, "bfloat16"), (256, "float16")])
@pytest.mark.parametrize("shape", ["rising", "falling", "steps"])
def test_maxima_that_move(dim, dtype, shape):
    import torch
    s = prompts([900, 30], [600, 0], 4, 1, dim, 16, dtype, seed=1)
    x = torch.linspace(0, 1, 1500, device="cuda")
    size = {"rising": 6 * x, "falling": 6 * (1 - x), "steps": 8 * (x * 5).floor() / 5}[shape]
    at = torch.arange(1500, device="cuda")
    b = s["table"][0].long()[at // 16]
    s["k"][b, at % 16] = (s["k"][b, at % 16] * size[:, None, None]).to(s["k"].dtype)
    check(s)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 1, 20, 65, 130])
def test_maxima_that_move_in_short_items(dim, window):
    """Many items of one to seven tiles in a run, with maxima that grow from tile to tile; the same bits every time."""
    import torch
    s = prompts([400] * 30, [0] * 30, 48, 1, dim, 16, seed=2)
    d = decoder(s)
    at = torch.arange(400, device="cuda")
    for row in s["table"].long():
        b = row[at // 16]
        s["k"][b, at % 16] = (s["k"][b, at % 16] * (at[:, None, None] / 60)).to(s["k"].dtype)
    want, lse = check(s, d, window=window)
    for _ in range(5):
        out, again = d.prompt(**s, window=window, lse=True)
        assert torch.equal(out, want) and torch.equal(again, lse)


def test_small_weights_count():
    """fp16: thousands of tokens far below the largest score."""
    import torch
    s = prompts([2], [40000], 1, 1, 64, 16, "float16", seed=3)
    s["q"][:], s["k"][:], s["v"][:] = 1, 0, 1
    b = int(s["table"][0, 0])
    s["k"][b, 0], s["v"][b, 0] = 2, 0                 # a score of 16 for the first token
    check(s)


def test_behind_the_last_row():
    """What lies behind the last row's queries is neither read nor written."""
    import torch
    s = prompts([70, 5, 0, 130], [0, 40, 3, 0], 6, 2, 64, 16, seed=7, spare=60)
    s["q"][205:] = math.nan
    d = decoder(s)
    out = torch.full_like(s["q"], 5.0)
    got, lse = d.prompt(**s, out=out, lse=True)
    want, want_lse, size = plain(s)
    kv_plain.check_attend(got[:205], lse[:205], want[:205], want_lse[:205], size[:205])
    assert (out[205:] == 5).all()


def test_strided():
    import torch
    s = prompts([70, 5], [0, 40], 6, 2, 64, 16, seed=8)
    want, lse = check(s)
    q = torch.zeros(75, 9, 80, device="cuda", dtype=torch.bfloat16)
    q[:, 2:8, 8:72] = s["q"]
    out = torch.full((75, 7, 72), 5.0, device="cuda", dtype=torch.bfloat16)
    got = decoder(s).prompt(**dict(s, q=q[:, 2:8, 8:72]), out=out[:, :6, :64])
    assert torch.equal(got, want) and (out[:, 6] == 5).all() and (out[..., 64:] == 5).all()
    check(s, scale=0.03)
    turned = s["q"].transpose(0, 1).contiguous().transpose(0, 1)       # heads outermost
    assert torch.equal(decoder(s).prompt(**dict(s, q=turned)), want)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 3)])
def test_undefined_values(dim, bad, window, sinks):
    """A value that is undefined or infinite shows in the queries that see it and in no other, dimension by dimension."""
    import torch
    s = prompts([300, 40], [50, 0], 4, 2, dim, 16, seed=dim)
    d = decoder(s)
    want, want_lse = d.prompt(**s, window=window, sinks=sinks, lse=True)
    at = 50 + 170                                      # of row 0: the 171st query's own
    b = int(s["table"][0, at // 16])
    s["v"][b, at % 16, 1, 5] = bad
    out, lse = d.prompt(**s, window=window, sinks=sinks, lse=True)
    assert d.status() == 0
    seen = torch.zeros(340, dtype=torch.bool, device="cuda")
    seen[170:300 if not window else 170 + window] = True
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[seen, 2:, 5] = True
    assert torch.equal(lse, want_lse) and torch.equal(out[~hit], want[~hit])
    assert (out[hit].isnan() if math.isnan(bad) else (out[hit] == bad) | out[hit].isnan()).all()
    assert math.isnan(bad) or (out[170, 2:, 5] == bad).all() or out[170, 2:, 5].isnan().any()


def test_undefined_keys():
    import torch
    s = prompts([300, 40], [50, 0], 4, 2, 128, 16, seed=2)
    d = decoder(s)
    want, want_lse = d.prompt(**s, lse=True)
    at = 50 + 170
    s["k"][int(s["table"][0, at // 16]), at % 16, 1, 5] = math.nan
    out, lse = d.prompt(**s, lse=True)
    assert out[170:300, 2:].isnan().all() and lse[170:300, 2:].isnan().all()
    out[170:300, 2:], lse[170:300, 2:] = want[170:300, 2:], want_lse[170:300, 2:]
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_keys_of_no_weight():
    """Scores of -infinity: tokens that are seen and count nothing, whole tiles of them, and all of a query's."""
    import torch
    s = prompts([300, 40], [300, 0], 2, 1, 128, 16, seed=3)
    s["q"] = s["q"].abs() + 0.1
    at = torch.arange(256, device="cuda")
    s["k"][s["table"][0].long()[at // 16], at % 16] = -math.inf
    check(s)
    at = torch.arange(40, device="cuda")
    s["k"][s["table"][1].long()[at // 16], at % 16] = -math.inf
    out, lse = decoder(s).prompt(**s, lse=True)
    assert (out[300:] == 0).all() and (lse[300:] == -math.inf).all()


def test_bad_rows_and_blocks():
    import torch
    from paper_2608_02244_gb300 import kv
    s = prompts([40, 20, 30, 25, 10], [0, 10, 0, 5, 0], 4, 2, 64, 16, seed=6)
    d = decoder(s)
    good, good_lse = d.prompt(**s, lse=True)
    s["lens"][1] = 19                                  # fewer own tokens than queries
    s["lens"][2] = 16 * s["table"].shape[1] + 1        # more than the table holds
    out, lse = d.prompt(**s, lse=True)
    assert d.status() == kv.ISJL_ERR_INVALID_ARG and d.status() == 0
    assert (out[40:90] == 0).all() and (lse[40:90] == -math.inf).all()
    assert torch.equal(out[:40], good[:40]) and torch.equal(out[90:], good[90:]) and torch.equal(lse[90:], good_lse[90:])
    s["lens"][1], s["lens"][2] = 30, 30
    s["table"][0, 1], s["table"][3, 0] = s["k"].shape[0], -9
    out, lse = d.prompt(**s, lse=True)
    assert d.status() == kv.ISJL_ERR_INVALID_ARG
    last = s["k"].shape[0]
    k, v = (torch.cat((x, torch.zeros_like(x[:1]))) for x in (s["k"], s["v"]))
    table = torch.where((s["table"] < 0) | (s["table"] >= last), last, s["table"])
    want, want_lse, size = plain(dict(s, k=k, v=v, table=table))
    kv_plain.check_attend(out, lse, want, want_lse, size)


@pytest.mark.parametrize("number", ["n_blocks", -1, 2**31 - 1, -2**31])
def test_any_bad_block_is_reported(number):
    """One block number outside the cache, whatever it is: reported, and its tokens read as zeros."""
    import torch
    from paper_2608_02244_gb300 import kv
    s = prompts([50], [20], 4, 2, 128, 16, seed=7)
    d = decoder(s)
    last = s["k"].shape[0]
    s["table"][0, 3] = last if number == "n_blocks" else number
    out, lse = d.prompt(**s, lse=True)
    assert d.status() == kv.ISJL_ERR_INVALID_ARG and d.status() == 0
    k, v = (torch.cat((x, torch.zeros_like(x[:1]))) for x in (s["k"], s["v"]))
    table = torch.where((s["table"] < 0) | (s["table"] >= last), last, s["table"])
    want, want_lse, size = plain(dict(s, k=k, v=v, table=table))
    kv_plain.check_attend(out, lse, want, want_lse, size)


def test_bad_starts():
    """Rows whose starts descend or leave the queries are skipped, the others are not."""
    import torch
    from paper_2608_02244_gb300 import kv
    s = prompts([40, 20, 30], [0, 10, 0], 4, 2, 64, 16, seed=6)
    d = decoder(s)
    good = d.prompt(**s)
    for starts in ([0, 40, 60, 91], [0, 40, 60, 2**31 - 1], [0, 40, 60, 50], [0, 40, 60, -1]):
        s["starts"].copy_(torch.tensor(starts))
        out = torch.full_like(good, 5.0)
        d.prompt(**s, out=out)
        assert d.status() == kv.ISJL_ERR_INVALID_ARG and d.status() == 0
        assert torch.equal(out[:60], good[:60]) and (out[60:] == 5).all()
    s["starts"].copy_(torch.tensor([-1, 40, 60, 90]))
    out = torch.full_like(good, 5.0)
    d.prompt(**s, out=out)
    assert d.status() == kv.ISJL_ERR_INVALID_ARG
    assert (out[:40] == 5).all() and torch.equal(out[40:], good[40:])


def test_nothing_to_do():
    import torch
    s = prompts([0, 0], [5, 0], 4, 2, 64, 16)
    assert decoder(s).prompt(**s).shape == (0, 4, 64)
    s = prompts([0, 0], [5, 0], 4, 2, 64, 16, spare=9)
    out = torch.full_like(s["q"], 5.0)
    d = decoder(s)
    d.prompt(**s, out=out)
    assert (out == 5).all() and d.status() == 0
    i32 = dict(dtype=torch.int32, device="cuda")
    d.prompt(s["q"], s["k"], s["v"], torch.zeros(0, 1, **i32), torch.zeros(1, **i32), torch.zeros(0, **i32), out=out)
    assert (out == 5).all() and d.status() == 0


def test_beyond_32_bits():
    """A cache of more than 2^32 bytes."""
    import torch
    from paper_2608_02244_gb300 import kv
    blocks, hkv, dim = 300_000, 8, 64
    d = kv.Decoder(blocks, 16, 16, hkv, dim, max_rows=2)
    k, v = (torch.zeros(blocks, 16, hkv, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.tensor([[blocks - 1, 3, blocks - 2], [0, blocks // 2 + 9, 7]], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    for b in table.view(-1).tolist():
        k[b], v[b] = (torch.randn(16, hkv, dim, generator=g, device="cuda").bfloat16() for _ in range(2))
    s = dict(q=torch.randn(60, 16, dim, generator=g, device="cuda").bfloat16(), k=k, v=v, table=table,
             starts=torch.tensor([0, 40, 60], dtype=torch.int32, device="cuda"),
             lens=torch.tensor([48, 41], dtype=torch.int32, device="cuda"), prefix=None)
    check(s, d)


def test_graph_and_stream():
    """A call captured once and replayed with other rows and queries; a call on another stream; two handles at once."""
    import torch
    s = prompts([70, 5, 300, 33], [0, 10, 0, 90], 8, 2, 128, 16, seed=8)
    other = prompts([90, 200, 0, 118], [9, 0, 3, 7], 8, 2, 128, 16, seed=9)
    width = max(s["table"].shape[1], other["table"].shape[1])
    total = max(s["k"].shape[0], other["k"].shape[0])
    import torch.nn.functional as F
    for x in (s, other):
        x["table"] = F.pad(x["table"], (0, width - x["table"].shape[1]), value=-1)
        x["k"], x["v"] = (F.pad(x[y], (0, 0, 0, 0, 0, 0, 0, total - x[y].shape[0])) for y in "kv")
    d = decoder(s)
    held = {x: y.clone() if y is not None else None for x, y in s.items()}
    wants = [d.prompt(**x, lse=True) for x in (s, other)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = d.prompt(**held, lse=True)
    for x, want in ((other, wants[1]), (s, wants[0]), (other, wants[1])):
        for y in ("q", "k", "v", "table", "lens", "starts"):
            held[y].copy_(x[y])
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    side = torch.cuda.Stream()
    e = decoder(s)
    torch.cuda.synchronize()
    first = d.prompt(**s, lse=True)
    second = e.prompt(**other, lse=True, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, wants[0])) and all(torch.equal(a, b) for a, b in zip(second, wants[1]))


def test_refusals():
    import torch
    from paper_2608_02244_gb300 import kv
    s = prompts([40, 3], [0, 9], 4, 2, 64, 16, seed=9)
    d = decoder(s)

    def refused(**kw):
        with pytest.raises(kv.IsjlError) as e:
            d.prompt(**dict(s, **kw))
        assert e.value.status == kv.ISJL_ERR_INVALID_ARG

    refused(q=s["q"].half())
    refused(q=s["q"][:, :3])
    refused(q=s["q"].cpu())
    refused(k=s["k"].half())
    refused(v=s["v"][:1])
    refused(table=s["table"][:1])
    refused(table=s["table"].long())
    refused(starts=s["starts"][:2])
    refused(starts=s["starts"].long())
    refused(lens=s["lens"][:1])
    refused(lens=s["lens"].repeat_interleave(2)[::2])
    refused(window=-1)
    refused(sinks=2**31)
    refused(scale=0.0)
    refused(scale=math.inf)
    refused(out=torch.zeros(43, 4, 32, device="cuda", dtype=torch.bfloat16))
    refused(out=torch.zeros(43, 4, 72, device="cuda", dtype=torch.bfloat16)[..., 1:65])
    refused(q=torch.zeros(43, 4, 68, device="cuda", dtype=torch.bfloat16)[..., :64])
    refused(table=torch.zeros(2, 2**27, dtype=torch.int32, device="cuda"))
    many = torch.zeros(3, dtype=torch.int32, device="cuda")
    refused(lens=many, starts=torch.zeros(4, dtype=torch.int32, device="cuda"), table=torch.zeros(3, 4, dtype=torch.int32, device="cuda"))
    assert d.status() == 0
    d.close()
    refused()
