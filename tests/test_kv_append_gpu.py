"""Norms, rotation and cache write against 64 bits.  A value is its terms' sum in 32 bits (a few roundings of
2^-24, taken as 2^-20 of the terms' magnitudes) rounded once to the cache's type."""
import pytest

import kv_plain
from conftest import cuda_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]
EPS = 1e-6


def inputs(n, hq, hkv, dim, rot, dtype, norm, block, seed, positions=300, order="token"):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    blocks = -(-n // block) + 2
    shape = {"token": (blocks, block, hkv, dim), "head": (blocks, hkv, block, dim), "apart": (block, blocks, hkv, dim)}[order]
    cache = [rn(*shape).to(dtype) for _ in range(2)]
    if order != "token":
        cache = [c.transpose(1, 2) if order == "head" else c.transpose(0, 1) for c in cache]
    s = dict(qkv=rn(n, (hq + 2 * hkv) * dim).to(dtype), positions=torch.randint(0, positions, (n,), generator=g, device="cuda", dtype=torch.int32),
             slots=torch.randperm(blocks * block, generator=g, device="cuda")[:n], k=cache[0], v=cache[1])
    if rot:
        angle = torch.rand(positions, rot // 2, generator=g, device="cuda") * 6.3
        s["rope"] = torch.cat((angle.cos(), angle.sin()), 1)
    if norm:
        s["q_weight"], s["k_weight"] = rn(dim).to(dtype), rn(dim).to(dtype)
    return s


def check(s, hq, hkv, dim, pairs=False, **kw):
    import torch
    from paper_2608_02244_gb300 import kv
    n, block, dtype = s["qkv"].shape[0], s["k"].shape[1], s["qkv"].dtype
    d = kv.Decoder(s["k"].shape[0], block, hq, hkv, dim, dtype=dtype, max_rows=1)
    want, mags = kv_plain.append(s["qkv"], s["positions"], s["slots"], s.get("rope"), s.get("q_weight"), s.get("k_weight"), EPS,
                                 pairs, hq, hkv, dim)
    old = s["k"].clone(), s["v"].clone()
    qkv = s["qkv"].clone()
    torch.cuda.synchronize()
    q = d.append(**s, eps=EPS, pairs=pairs, **kw)
    assert d.status() == 0
    tol = kv_plain.UNIT[dtype] * want.abs() * (1 + 2.0 ** -6) + 2.0 ** -20 * mags + 2.0 ** -24
    real = s["slots"] >= 0
    assert ((q.double() - want[:, :hq]).abs() <= tol[:, :hq])[real].all()
    assert (q[~real] == 0).all()
    at = s["slots"][real]
    b, p = at // block, at % block
    assert ((s["k"][b, p].double() - want[real, hq:hq + hkv]).abs() <= tol[real, hq:hq + hkv]).all()
    if n:
        assert torch.equal(s["v"][b, p], qkv.view(n, -1, dim)[real, hq + hkv:])
    for c, o in zip((s["k"], s["v"]), old):           # nothing else was written
        c, o = c.clone(), o.clone()
        c[b, p] = 0
        o[b, p] = 0
        assert torch.equal(c, o)
    return q


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("rot", ["all", "half", 16, 0])
def test_values(dim, dtype, pairs, rot):
    import torch
    rot = {"all": dim, "half": dim // 2}.get(rot, rot)
    check(inputs(37, 6, 2, dim, rot, getattr(torch, dtype), rot != 16, 16, dim + rot), 6, 2, dim, pairs)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 5), (7, 1), (28, 4), (64, 8), (33, 11)])
@pytest.mark.parametrize("n", [1, 2, 130])
def test_heads(hq, hkv, n):
    import torch
    check(inputs(n, hq, hkv, 64, 64, torch.bfloat16, True, 8, n), hq, hkv, 64)


@pytest.mark.parametrize("order", ["token", "head", "apart"])
@pytest.mark.parametrize("block", [8, 64, 256])
def test_cache_orders(order, block):
    import torch
    check(inputs(200, 8, 4, 128, 128, torch.bfloat16, True, block, block, order=order), 8, 4, 128)


def test_many_tokens():
    import torch
    check(inputs(20011, 8, 2, 128, 128, torch.bfloat16, True, 16, 1), 8, 2, 128)


@pytest.mark.parametrize("n", [3647, 3648, 4999])
@pytest.mark.parametrize("dim,hq,hkv", [(64, 3, 1), (128, 6, 2), (256, 2, 1)])
def test_around_many_tokens(n, dim, hq, hkv):
    """Both sides of the token count from which a token is one warp's."""
    import torch
    s = inputs(n, hq, hkv, dim, dim // 2, torch.bfloat16, True, 32, n)
    s["slots"][5::97] = -1
    check(s, hq, hkv, dim, pairs=n % 2 == 0)


def test_infinite_values_stay_in_their_place():
    """A value outside the rotated part, or a v value, is copied whatever it is; a rotated pair shows it."""
    import math

    import torch
    from paper_2608_02244_gb300 import kv
    s = inputs(3, 2, 1, 64, 16, torch.bfloat16, False, 8, 11)
    s["qkv"][0, 40], s["qkv"][1, 3 * 64 + 5] = math.inf, math.nan          # q head 0 beyond rot; v
    q = kv.Decoder(s["k"].shape[0], 8, 2, 1, 64, max_rows=1).append(**s)
    bad = ~torch.isfinite(q)
    assert bad.sum() == 1 and q[0, 0, 40] == math.inf
    at = s["slots"][1]
    assert torch.isnan(s["v"][at // 8, at % 8]).sum() == 1


def test_padding_one_weight_and_large_values():
    import torch
    s = inputs(50, 4, 2, 64, 32, torch.float16, True, 8, 5)
    s["slots"][::3] = -1
    s["positions"][::3] = -7                       # not looked at
    check(s, 4, 2, 64)
    s = inputs(20, 4, 2, 64, 64, torch.float16, True, 8, 6)
    s["qkv"] *= 200                                # squares beyond the type's range
    s["q_weight"] = None
    s["qkv"][3] = 0                                # a head of zeros stays one
    check(s, 4, 2, 64)


def test_in_place_strided_and_other_stream():
    import torch
    s = inputs(40, 8, 2, 128, 128, torch.bfloat16, True, 16, 7)
    wide = torch.zeros(40, 12 * 128 + 24, dtype=torch.bfloat16, device="cuda")
    wide[:, :12 * 128] = s["qkv"]
    want = check(dict(s, k=s["k"].clone(), v=s["v"].clone()), 8, 2, 128).clone()
    s["qkv"] = wide[:, :12 * 128]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    q = check(s, 8, 2, 128, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(q, want)
    from paper_2608_02244_gb300 import kv
    d = kv.Decoder(s["k"].shape[0], 16, 8, 2, 128, max_rows=1)
    rest = s["qkv"][:, 8 * 128:].clone()
    out = s["qkv"][:, :8 * 128].unflatten(1, (8, 128))
    assert d.append(**s, eps=EPS, out=out) is out and torch.equal(out, want) and torch.equal(s["qkv"][:, 8 * 128:], rest)


def test_reports_invalid_values():
    import torch
    from paper_2608_02244_gb300 import kv
    for name, value in (("slots", 10**9), ("positions", 300), ("positions", -1)):
        s = inputs(5, 4, 2, 64, 64, torch.bfloat16, False, 8, 8)
        s[name][2] = value
        d = kv.Decoder(s["k"].shape[0], 8, 4, 2, 64, max_rows=1)
        old = s["k"].clone()
        slot = s["slots"].tolist()
        q = d.append(**s)
        assert d.status() == kv.ISJL_ERR_INVALID_ARG and d.status() == 0
        assert (q[2] == 0).all() and (q[1] != 0).any()
        if name == "positions":
            assert torch.equal(s["k"][slot[2] // 8, slot[2] % 8], old[slot[2] // 8, slot[2] % 8])


def test_refusals():
    import torch
    from paper_2608_02244_gb300 import kv
    s = inputs(6, 4, 2, 64, 64, torch.bfloat16, True, 8, 9)
    d = kv.Decoder(s["k"].shape[0], 8, 4, 2, 64, max_rows=1)
    d.append(**s)
    assert d.append(**dict(s, qkv=s["qkv"][:0], positions=s["positions"][:0], slots=s["slots"][:0])).shape == (0, 4, 64)
    f = s["qkv"].float()
    odd = torch.zeros(6 * 512 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(6, 512)
    for bad in (dict(qkv=f), dict(qkv=s["qkv"][:, :-8]), dict(qkv=odd), dict(positions=s["positions"].long()), dict(slots=s["slots"].int()),
                dict(slots=s["slots"][:5]), dict(k=s["k"].half()), dict(k=s["k"][:-1]), dict(v=s["v"].transpose(0, 1)),
                dict(rope=s["rope"].double()), dict(rope=s["rope"][:, :24].contiguous()), dict(rope=torch.zeros(4, 128, device="cuda")),
                dict(q_weight=s["q_weight"].float()), dict(k_weight=s["k_weight"][:32]), dict(eps=-1.0), dict(eps=float("nan")),
                dict(out=torch.zeros(6, 4, 64, device="cuda"))):
        with pytest.raises(kv.IsjlError) as e:
            d.append(**dict(s, **bad))
        assert e.value.status == kv.ISJL_ERR_INVALID_ARG
    torch.cuda.synchronize()
