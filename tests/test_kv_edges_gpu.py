"""Places where the decode step's kernels can go wrong, beside the sizes of the other tests: lanes that part ways,
memory and streams, ends of number ranges, handles of other devices."""
import math

import numpy as np
import pytest

import kv_plain
from conftest import cuda_available
from test_kv_attend_gpu import check, decoder, inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]


@pytest.mark.parametrize("hq,hkv,dim,shared", [(3, 1, 64, 0), (5, 1, 128, 0), (11, 1, 256, 0), (34, 2, 128, 0), (9, 3, 64, 300),
                                               (13, 1, 128, 160)])
def test_lanes_that_part_ways(hq, hkv, dim, shared):
    """An item ends in almost every slice, and its queries keep some lanes longer than others: prefetches, stores of
    live rows, waits.  The same bits every time."""
    import torch
    rng = np.random.default_rng(hq)
    s = inputs(np.where(rng.random(700) < 0.5, rng.integers(1, 40, 700), 32), hq, hkv, dim, 16, shared=shared, seed=hq)
    d = decoder(s)
    want, lse = check(s, d)
    for _ in range(20):
        out, again = d.attend(**s, lse=True)
        assert torch.equal(out, want) and torch.equal(again, lse)


def _results_of(call, want, side):
    """The call's results on another stream, asked for while the current one still has work to do on memory of
    their sizes that it has given back."""
    import torch
    torch.cuda.synchronize()
    left = [torch.empty_like(t) for t in want]
    at = [t.data_ptr() for t in left]
    torch.cuda._sleep(200_000_000)                   # a tenth of a second
    for t in left:
        t.view(torch.uint8).fill_(255)
    del t
    left.clear()
    again = [torch.empty_like(t) for t in want]
    assert {t.data_ptr() for t in again} & set(at)   # the current stream would get that memory
    again.clear()
    got = call(side)
    side.synchronize()
    early = [t.cpu() for t in got]                   # copies on the current stream: after its work
    torch.cuda.synchronize()
    assert all(torch.equal(a, b.cpu()) for a, b in zip(early, want))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    return got


def test_results_on_another_stream():
    """Their memory is not what the current stream still uses, and stays theirs while the current stream uses them."""
    import torch
    from paper_2608_02244_gb300 import kv
    side = torch.cuda.Stream()
    s = inputs([40] * 300 + [0], 32, 4, 128, 16)
    d = decoder(s)
    want = d.attend(**s, lse=True)
    _results_of(lambda stream: d.attend(**s, lse=True, stream=stream), want, side)

    n = 1000
    g = torch.Generator(device="cuda").manual_seed(1)
    qkv = torch.randn(n, 40 * 128, generator=g, device="cuda").bfloat16()
    slots = torch.randperm(s["k"].shape[0] * 16, generator=g, device="cuda")[:n]
    k, v = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
    want = [d.append(qkv, None, slots, k, v)]
    _results_of(lambda stream: [d.append(qkv, None, slots, k, v, stream=stream)], want, side)

    rows, m = 200, 300_000
    i32 = dict(dtype=torch.int32, device="cuda")
    lens, new, table = torch.arange(rows, **i32) % 50, torch.full((rows,), 3, **i32), torch.arange(rows * 8, **i32).view(rows, 8)
    d = kv.Decoder(rows * 8 + 1000, 16, 1, 1, 64, max_rows=rows)
    free, n_free = torch.zeros(rows * 8 + 1000, **i32), torch.tensor([1000], **i32)
    free[:1000] = torch.arange(rows * 8, rows * 8 + 1000, **i32)
    want = d.assign(lens, new, table, free, n_free, m)
    got = _results_of(lambda stream: d.assign(lens, new, table, free, n_free, m, stream=stream), want, side)
    # dropped after use on the current stream: the other stream does not get the memory before that use is over
    out = got.slots
    at, before = out.data_ptr(), out.clone()
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    kept = out + 0
    del out, got
    with torch.cuda.stream(side):
        other = torch.empty_like(before)
        other.fill_(7)
    assert other.data_ptr() != at
    torch.cuda.synchronize()
    assert torch.equal(kept, before)


def test_handle_of_another_device():
    """With another device current than the handle's, calls are refused on the host and nothing is launched.  One GPU is
    enough for that: the number of the device that the handle keeps, after its configuration, is changed."""
    import ctypes

    import torch
    from paper_2608_02244_gb300 import kv
    s = inputs([30, 1], 4, 2, 64, 16)
    d = decoder(s)
    i32 = dict(dtype=torch.int32, device="cuda")
    qkv = torch.randn(2, 8 * 64, device="cuda").bfloat16()
    slots = torch.tensor([-1, -1], device="cuda")
    free = torch.zeros(d.n_blocks, **i32)
    n_free, new = torch.zeros(1, **i32), torch.zeros(2, **i32)
    out = torch.full_like(s["q"], math.nan)
    calls = [lambda: d.assign(s["lens"], new, s["table"], free, n_free, 4), lambda: d.append(qkv, None, slots, s["k"], s["v"]),
             lambda: d.attend(**s, out=out)]
    kept = ctypes.c_int32.from_address(d.handle.value + ctypes.sizeof(kv.isjl_kv_config))
    assert kept.value == torch.cuda.current_device()
    kept.value += 1
    try:
        for call in calls:
            with pytest.raises(kv.IsjlError) as e:
                call()
            assert e.value.status == kv.ISJL_ERR_INVALID_ARG
        assert d.status() == kv.ISJL_ERR_INVALID_ARG
    finally:
        kept.value -= 1
    assert out.isnan().all()
    for call in calls:
        call()
    assert d.status() == 0 and torch.isfinite(out).all()


def test_most_tokens():
    """Tables and prefixes of up to 2^31 - 256 tokens: places are rounded up to whole tiles in 32 bits.  The tables
    repeat one block; what a call does not see is not read."""
    import torch
    from paper_2608_02244_gb300 import kv
    for block in (8, 256):
        most = (2**31 - 256) // block
        s = inputs([300], 2, 1, 64, block, seed=block)
        want = check(s)
        wide = torch.full((1, most + 1), -1, dtype=torch.int32, device="cuda")
        wide[0, :s["table"].shape[1]] = s["table"][0]
        d = decoder(s)
        for more in (dict(table=wide), dict(table=wide[:, :most - 4].contiguous(), prefix=wide[0, :5])):
            with pytest.raises(kv.IsjlError) as e:
                d.attend(**dict(s, **more))
            assert e.value.status == kv.ISJL_ERR_INVALID_ARG
        out, lse = d.attend(**dict(s, table=wide[:, :most].contiguous()), lse=True)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        # the longest request there can be, in a window at its end
        table = s["table"][:, :1].expand(1, most).contiguous()
        lens = torch.full((1,), most * block, dtype=torch.int32, device="cuda")
        out, lse = d.attend(**dict(s, table=table, lens=lens), window=block, lse=True)
        assert d.status() == 0
        one = dict(s, table=s["table"][:, :1].contiguous(), lens=torch.full((1,), block, dtype=torch.int32, device="cuda"))
        kv_plain.check_attend(out, lse, *kv_plain.attend(**one))


def test_misaligned_pointers_are_refused():
    """Each array of numbers of the three calls, a byte beside its place: INVALID_ARG on the host, nothing launched."""
    import ctypes

    import torch
    from paper_2608_02244_gb300 import kv
    L, d = kv.lib(), kv.Decoder(20, 8, 2, 1, 64, max_rows=3)
    memory = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    base = memory.data_ptr()
    cache = kv.isjl_kv_cache(base, base, (ctypes.c_int64 * 3)(512, 64, 8), (ctypes.c_int64 * 3)(512, 64, 8))
    stream = torch.cuda.current_stream().cuda_stream

    def args(cls, numbers, pointers, other):
        a = cls(**numbers, **other)
        for i, f in enumerate(pointers):
            setattr(a, f, base + 4096 + 1024 * i)
        return a

    ints = ("lens", "new_tokens", "table", "free_list", "n_free", "lens_out", "n_free_out", "granted", "starts", "slots", "positions",
            "rows", "visible")
    assign = args(kv.isjl_kv_assign_args, dict(n_rows=3, table_width=4, max_tokens=4), ints, {})
    append = args(kv.isjl_kv_append_args, dict(n_tokens=2, n_positions=2, rot=16), ("positions", "slots"),
                  dict(qkv=base, qkv_stride=256, q_out=base + 32768, q_out_stride=128, rope=base))
    attend = args(kv.isjl_kv_attend_args, dict(n=2, n_table_rows=2, table_width=2, n_prefix_blocks=1, scale=1.0),
                  ("lse", "lens", "rows", "table", "prefix"),
                  dict(q=base, q_stride=(128, 64), out=base + 32768, out_stride=(128, 64)))
    for a, fields, call in ((assign, ints, lambda a: L.isjl_kv_assign(d.handle, ctypes.byref(a), stream)),
                            (append, ("positions", "slots"), lambda a: L.isjl_kv_append(d.handle, ctypes.byref(a), ctypes.byref(cache), stream)),
                            (attend, ("lse", "lens", "rows", "table", "prefix"),
                             lambda a: L.isjl_kv_attend(d.handle, ctypes.byref(a), ctypes.byref(cache), stream))):
        assert call(a) == kv.ISJL_OK
        for f in fields:
            for by in (1, 2, 4) if f == "slots" else (1, 2):
                setattr(a, f, getattr(a, f) + by)
                assert call(a) == kv.ISJL_ERR_INVALID_ARG, f
                setattr(a, f, getattr(a, f) - by)
    torch.cuda.synchronize()


def long_runs(dim, dtype="bfloat16", seed=0):
    """Enough queries that a block of the prefix's kernel has runs of ten token tiles of an item: 32 items of 20 tiles on
    64 blocks."""
    return inputs([30, 2, 90, 1] * 128, 16, 8, dim, 64, dtype, shared=40, seed=seed)


@pytest.mark.parametrize("dim", [64, 128])
def test_prefix_row_of_minus_infinity_beside_growing_ones(dim):
    """A row whose scores are -infinity in the first tiles, in a warp where other rows' maxima grow: its later tiles
    give it a result all the same."""
    s = long_runs(dim, seed=3)
    first = s["prefix"].long()
    s["k"][first[:2]] *= 0.1
    s["k"][first[2:6]] *= 8
    s["k"][..., 0] = 0
    s["k"][first[:6], :, :, 0] = -1e20
    s["q"][..., 0] = 0
    s["q"][1::2, :, 0] = 1e20                        # times -1e20: beyond 32 bits
    check(s)


def test_errors_do_not_outlive_their_call():
    """A call that fails in the CUDA runtime (a report asked for during a capture, a launch into a capture that this
    broke) leaves nothing behind that a later call reports as its own."""
    import ctypes

    import torch
    from paper_2608_02244_gb300 import kv, sim
    rt = ctypes.CDLL("libcudart.so.%s" % torch.version.cuda.split(".")[0])
    s = inputs([30, 1], 4, 2, 64, 16)
    d = decoder(s)
    qkv = torch.randn(2, 8 * 64, device="cuda").bfloat16()
    slots = torch.tensor([-1, -1], device="cuda")
    q, out = torch.empty_like(s["q"]), torch.empty_like(s["q"])
    side = torch.cuda.Stream()
    for fails in (False, True):
        d.append(qkv, None, slots, s["k"], s["v"], out=q)
        torch.cuda.synchronize()
        graph = ctypes.c_void_p()
        assert rt.cudaStreamBeginCapture(ctypes.c_void_p(side.cuda_stream), 1) == 0
        assert d.status() == sim.ISJL_ERR_CUDA
        if fails:
            with pytest.raises(kv.IsjlError) as e:
                d.attend(**s, out=out, stream=side)
            assert e.value.status == sim.ISJL_ERR_CUDA
        assert rt.cudaStreamEndCapture(ctypes.c_void_p(side.cuda_stream), ctypes.byref(graph)) != 0
        rt.cudaGetLastError()
        d.append(qkv, None, slots, s["k"], s["v"], out=q)
        assert d.status() == 0 and (q == 0).all()


def tail(got, lse, s, **kw):
    """All queries are the same: each is compared with the first one's 64 bits."""
    want, want_lse, size = kv_plain.attend(**dict(s, q=s["q"][:1], lens=s["lens"][:1]), **kw)
    kv_plain.check_attend(got, lse, want.expand(got.shape), want_lse.expand(lse.shape), size.expand(got.shape))


@pytest.mark.parametrize("dim", [64, 128])
def test_many_small_weights_of_fp16(dim):
    """Tens of thousands of weights 2^-24 or less of the largest, which together count, since the largest's value is 0:
    no weight is lost to the range of 16 bits.  Enough queries that one warp has the whole of a request."""
    import torch
    n = 1300
    s = inputs([49152], 1, 1, dim, 64, "float16", rows=range(n), seed=4)
    s["q"][:] = 0
    s["q"][..., 0] = dim ** 0.5
    own = s["table"][0].long()
    s["k"][..., 0] = 0.4
    s["v"][:] = 1
    s["k"][own[0], 7, 0, 0] = 18                     # 25.4 powers of two above the others
    s["v"][own[0], 7] = 0
    s["lens"] = s["lens"].expand(n).contiguous()
    rows = torch.zeros_like(s["lens"])
    d = decoder(s)
    got, lse = d.attend(**s, rows=rows, lse=True)
    assert d.status() == 0
    tail(got, lse, s, rows=rows)


@pytest.mark.parametrize("dim", [64, 128])
def test_many_small_weights_of_fp16_in_a_prefix(dim):
    s = inputs([1] * 512, 16, 8, dim, 64, "float16", shared=512, seed=5)
    s["q"][:] = 0
    s["q"][..., 0] = dim ** 0.5
    s["k"][..., 0] = 0.4
    s["v"][:] = 1
    first = s["prefix"].long()
    s["k"][first[0], 7, :, 0] = 17                   # 23.9 powers of two above the others
    s["v"][first[0], 7] = 0
    s["k"][first[100], 9, :, 0] = 17.9               # and one that comes later, 25.2
    s["v"][first[100], 9] = 0
    d = decoder(s)
    got, lse = d.attend(**s, lse=True)
    assert d.status() == 0
    tail(got, lse, s)


@pytest.mark.parametrize("rows,room", [(3, 16), (3, 5000), (1200, 1300)])
@pytest.mark.parametrize("number", [-3, 40])
@pytest.mark.parametrize("where", ["held", "free", "ends"])
def test_blocks_outside_the_cache(rows, room, number, where):
    """A block number outside the cache, in the place where a row's next token goes, on the free list or among those
    given back, is reported; no token gets a slot in it."""
    import torch
    from paper_2608_02244_gb300 import kv
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    d = kv.Decoder(40, 8, 1, 1, 64, max_rows=rows)
    lens, new = [0] * rows, [0] * rows
    table = np.full((rows, 2), -1)
    lens[0], lens[1], lens[2], new[0], new[1], new[2] = 3, 8, 5, 2, 1, -1 if where == "ends" else 1
    table[0, 0], table[1, 0], table[2, 0] = 10, 11, 12
    free = np.arange(40)
    if where == "held":
        table[0, 0] = number
    elif where == "free":
        free[6] = number
    else:
        table[2, 0], new[1] = number, 0
    p = d.assign(i32(lens), i32(new), i32(table), i32(free), i32([7]), room)
    assert d.status() == kv.ISJL_ERR_INVALID_ARG and d.status() == 0
    want = {"held": [-1, -1, 6 * 8, 12 * 8 + 5], "free": [10 * 8 + 3, 10 * 8 + 4, -1, 12 * 8 + 5], "ends": [10 * 8 + 3, 10 * 8 + 4]}[where]
    assert p.slots.tolist() == want + [-1] * (room - len(want))
    assert p.granted.tolist()[:3] == [2, 0 if where == "ends" else 1, 0 if where == "ends" else 1]
