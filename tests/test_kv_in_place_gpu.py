"""Results written where the queries are (out is q): the bits of a call with an output of its own."""
import math

import pytest

import test_kv_attend_gpu as single
import test_kv_four_gpu as four
import test_kv_prompt_gpu as packed
from conftest import cuda_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]


def check(call, s, **kw):
    import torch
    want, want_lse = call(**s, lse=True, **kw)
    q = s["q"].clone()
    out, lse = call(**dict(s, q=q), out=q, lse=True, **kw)
    assert out is q
    bits = lambda t: t.contiguous().view(torch.uint8)  # noqa: E731
    assert torch.equal(bits(out), bits(want)) and torch.equal(bits(lse), bits(want_lse))


# items of many lengths, cut ones, heads in parts, a prefix read by each query and one done apart
ROWS = [([0, 5, 200, 77, 1], 8, 2, 128, 0), ([30000], 4, 1, 128, 0), ([300, 0, 900], 66, 2, 64, 0), ([70] * 40, 8, 2, 64, 60), ([70] * 3, 4, 4, 256, 5)]


@pytest.mark.parametrize("lens,hq,hkv,dim,shared", ROWS)
def test_attend(lens, hq, hkv, dim, shared):
    s = single.inputs(lens, hq, hkv, dim, 16, shared=shared, seed=1)
    check(single.decoder(s).attend, s)


@pytest.mark.parametrize("lens,hq,hkv,dim,shared", ROWS)
def test_attend4(lens, hq, hkv, dim, shared):
    s = four.requests(lens, hq, hkv, dim, 16, shared=shared, seed=1)
    check(four.decoder4(s).attend4, s)


@pytest.mark.parametrize("counts,before,hq,hkv", [([300, 0, 40, 1], [50, 3, 0, 0], 8, 2), ([64] * 3, [20000] * 3, 8, 2), ([130] * 20, [0] * 20, 7, 1),
                                                  ([60, 5], [0, 9], 300, 1)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_prompt(counts, before, hq, hkv, dim):
    s = packed.prompts(counts, before, hq, hkv, dim, 16, seed=2)
    check(packed.decoder(s).prompt, s)
    check(packed.decoder(s).prompt, s, window=90, sinks=3)


@pytest.mark.parametrize("dim", [64, 128, 256])
# items in pieces, and (in many rows) whole ones, whose results are written at once
@pytest.mark.parametrize("counts,before", [([300, 40], [50, 0]), ([64, 64], [20000, 0]), ([300, 40] * 80, [50, 0] * 80)])
def test_prompt_with_infinities(dim, counts, before):
    """Of values that are not finite the weights are computed again, from the queries."""
    s = packed.prompts(counts, before, 4, 2, dim, 16, seed=3)
    for column, x in ((5, math.inf), (dim // 2 + 1, -math.inf), (dim - 1, math.inf), (dim - 2, math.nan)):
        for row in range(0, len(counts), 2):
            at = before[row] + counts[row] // 2
            s["v"][int(s["table"][row, at // 16]), at % 16, :, column] = x
    check(packed.decoder(s).prompt, s)
    check(packed.decoder(s).prompt, s, window=60)
