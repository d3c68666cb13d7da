"""Plain forms of a cache in 4 bits, for the tests: the groups' values, codes and bounds."""
import torch

import kv_plain

GROUP = 32


def values(codes, scales):
    """What codes [..., dim / 2] with scales and offsets [..., dim / 32, 2] stand for, in their type.  B + (1 + c / 16) S
    has at most 5 + 11 bits before the sum, so that 64 bits hold it exactly and it is rounded once."""
    c = torch.stack((codes & 15, codes >> 4), -1).reshape(scales.shape[:-1] + (GROUP,)).double()
    x = scales.double()
    return (x[..., 1:] + (1 + c / 16) * x[..., :1]).to(scales.dtype).flatten(-2)


def coded(x, dtype):
    """Codes, and scales with offsets, of values [..., dim] in 32 bits; on the CPU, whose divisions are exact."""
    x = x.float().cpu().unflatten(-1, (-1, GROUP))
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale = ((hi - lo) * torch.tensor(16 / 15, dtype=torch.float32)).to(dtype).float()
    offset = (lo - scale).to(dtype).float()
    c = torch.round((x - offset) / torch.where(scale > 0, scale, 1) * 16 - 16)
    c = torch.where(scale > 0, c.clamp(0, 15), 0).to(torch.uint8).flatten(-2)
    return c[..., ::2] | c[..., 1::2] << 4, torch.cat((scale, offset), -1).to(dtype)


def bound(x, mags, dtype):
    """Of the distance between values [..., dim] (64 bits) and what their codes stand for.  With T's unit roundoff u: S
    is off by u S, B by u |lo - S|, so that the least and largest value lie at most u (|lo| + S) + u S outside of what
    the codes reach; half a step is S / 32; the value is rounded once more, by u (|lo| + S).  Together S / 32 +
    u (2 |lo| + 4 S).  The values themselves are 32-bit sums, off by 2^-20 of their terms' magnitudes, which moves a
    group's ends as well; numbers below the type's normal ones are off by at most their spacing."""
    u = kv_plain.UNIT[dtype]
    g, m = x.unflatten(-1, (-1, GROUP)), mags.unflatten(-1, (-1, GROUP)).amax(-1, keepdim=True)
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    s = (hi - lo) * 16 / 15 * (1 + u)
    return (s / 32 + u * (2 * lo.abs() + 4 * s) + 2.0 ** -18 * m + 2.0 ** -24).expand(g.shape).flatten(-2)


def cache(total, block, hkv, dim, dtype, order="token", fill=0.0):
    """A cache on the GPU whose places all hold codes of 15 with scale and offset `fill`."""
    from paper_2608_02244_gb300 import kv
    axes = {"token": (0, 1, 2), "head": (0, 2, 1), "apart": (1, 0, 2)}[order]
    lead = [(total, block, hkv)[i] for i in axes]

    def make(inner, x, t):
        c = torch.full(lead + list(inner), x, dtype=t, device="cuda")
        return c.permute([axes.index(i) for i in range(3)] + list(range(3, 3 + len(inner))))

    return kv.Cache4(make((dim // 2,), 255, torch.uint8), make((dim // 2,), 255, torch.uint8),
                     make((dim // GROUP, 2), fill, dtype), make((dim // GROUP, 2), fill, dtype))


def fill(c, block, place, g, size=1.0):
    """Random tokens at [block, place]: codes of all values, offsets on both sides of 0."""
    n, (hkv, half), dtype = len(block), c.k.shape[2:], c.k_scale.dtype
    for codes, scales in ((c.k, c.k_scale), (c.v, c.v_scale)):
        codes[block, place] = torch.randint(0, 256, (n, hkv, half), generator=g, device="cuda", dtype=torch.uint8)
        s = torch.rand(n, hkv, half // 16, generator=g, device="cuda") * 6 * size
        b = -1.47 * s + 0.3 * size * torch.randn(s.shape, generator=g, device="cuda")
        scales[block, place] = torch.stack((s, b), -1).to(dtype)


def in_16_bits(c):
    """Keys and values of all of a cache's places."""
    return values(c.k, c.k_scale), values(c.v, c.v_scale)
