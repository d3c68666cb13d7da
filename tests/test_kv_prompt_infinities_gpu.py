"""Infinite and undefined values in prompts: exactly the queries that see one have it in exactly its dimension, with its
sign; two of opposite signs, and one of weight 0, make it undefined.  All other results keep their bits."""
import math

import pytest

from conftest import cuda_available
from test_kv_prompt_gpu import decoder, prompts

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]


def place_of(s, row, token):
    block = s["k"].shape[1]
    return int(s["table"][row, token // block]), token % block


def check(s, values, weightless=(), **sight):
    """values: (row, own token, key head, dimension, value).  No weight of a token that is seen rounds to 0 (scores of
    independent normal values, some +-6, and their differences are far from 2^-25), but that of the `weightless`."""
    import torch
    d = decoder(s)
    group = s["q"].shape[1] // s["k"].shape[2]
    for row, token, head in weightless:
        s["k"][place_of(s, row, token)][head] = -math.inf
    want, want_lse = d.prompt(**s, lse=True, **sight)
    assert torch.isfinite(want.double()).all()
    sums = torch.zeros(want.shape, dtype=torch.float64, device="cuda")         # of what the values add
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    window, sinks = sight.get("window", 0), sight.get("sinks", 0)
    for row, token, head, column, x in values:
        s["v"][place_of(s, row, token)][head, column] = x
        a, b = starts[row], starts[row + 1]
        at = torch.arange(lens[row] - (b - a), lens[row], device="cuda")       # the queries' places
        sees = at >= token
        if window:
            sees &= (at < token + window) | (token < sinks)
        assert sees.any()
        add = math.nan if (row, token, head) in weightless else x
        sums[a:b, head * group:(head + 1) * group, column] += torch.where(sees, add, 0.0)[:, None]
    out, lse = d.prompt(**s, lse=True, **sight)
    assert d.status() == 0
    expected = torch.where(sums == 0, want.double(), sums)
    assert torch.equal(out.double().nan_to_num(7e7, 8e7, -8e7), expected.nan_to_num(7e7, 8e7, -8e7))
    assert torch.equal(lse, want_lse)


SIGHTS = [dict(), dict(window=60, sinks=3), dict(window=130)]


# behind the first query; the last of a tile; where windows begin; a first token; the last query's own
@pytest.mark.parametrize("token", [50, 130, 220, 255, 256, 300, 349, 55, 60])
@pytest.mark.parametrize("dim,dtype", [(64, "bfloat16"), (64, "float16"), (128, "bfloat16"), (128, "float16"), (256, "bfloat16"), (256, "float16")])
@pytest.mark.parametrize("sight", SIGHTS)
def test_one_infinity(dim, dtype, token, sight):
    for x in (math.inf, -math.inf, math.nan):
        check(prompts([300, 40], [50, 0], 4, 2, dim, 16, dtype, seed=dim), [(0, token, 1, 5, x)], **sight)


def test_a_first_token_beside_a_window():
    check(prompts([300, 40], [0, 5], 4, 2, 128, 16, seed=1), [(0, 1, 0, 127, math.inf), (1, 2, 1, 0, -math.inf)], window=60, sinks=3)


@pytest.mark.parametrize("dim,dtype", [(64, "float16"), (128, "bfloat16"), (256, "bfloat16")])
@pytest.mark.parametrize("sight", SIGHTS)
def test_infinities_of_both_signs(dim, dtype, sight):
    """In one dimension: the queries that see one of them, and those that see both; in others and other heads, one each."""
    check(prompts([300, 40], [50, 0], 4, 2, dim, 16, dtype, seed=3),
          [(0, 220, 1, 5, math.inf), (0, 225, 1, 5, -math.inf), (0, 225, 1, 6, -math.inf), (0, 225, 0, 5, math.inf), (1, 17, 1, 5, -math.inf),
           (0, 320, 1, dim - 1, math.inf), (0, 320, 1, 17, -math.inf)], **sight)


@pytest.mark.parametrize("dim,dtype", [(64, "bfloat16"), (128, "float16"), (128, "bfloat16"), (256, "float16")])
@pytest.mark.parametrize("sight", SIGHTS)
def test_an_infinity_of_weight_zero(dim, dtype, sight):
    """A score of -infinity: 0 times infinity; another token's infinity beside it keeps its sign."""
    s = prompts([300, 40], [50, 0], 4, 2, dim, 16, dtype, seed=4)
    s["q"] = s["q"].abs() + 0.1
    check(s, [(0, 220, 1, 5, math.inf), (0, 222, 1, 6, math.inf), (0, 340, 0, 40, -math.inf)], weightless=[(0, 220, 1), (0, 340, 0)], **sight)


@pytest.mark.parametrize("counts,before,hq,hkv,dim,dtype", [([64], [20000], 8, 2, 128, "bfloat16"), ([64], [20000], 8, 2, 64, "float16"),
                                                            ([30], [20000], 8, 2, 256, "bfloat16"), ([1], [9000], 4, 1, 128, "bfloat16"),
                                                            ([700, 64], [3000, 20000], 8, 2, 128, "float16")])
def test_infinities_in_items_in_pieces(counts, before, hq, hkv, dim, dtype):
    """Items that the ends of runs cut: the values lie in one piece, in the last tile, or in two of them."""
    row = len(counts) - 1
    n, b = counts[row], before[row]
    s = prompts(counts, before, hq, hkv, dim, 32, dtype, seed=5)
    check(s, [(row, b + n // 2, 0, 5, math.inf), (row, b, 0, 6, -math.inf), (row, 40, 0, 7, math.inf), (row, b - 300, 0, 8, -math.inf),
              (row, b + n // 2, 0, 8, math.inf)])
    s = prompts(counts, before, hq, hkv, dim, 32, dtype, seed=5)
    check(s, [(row, b - 4000 + (n + 1) // 2, 0, 5, math.inf), (row, b, 0, 6, -math.inf)], window=4000)


@pytest.mark.parametrize("dim,dtype", [(64, "float16"), (128, "bfloat16"), (128, "float16"), (256, "bfloat16")])
@pytest.mark.parametrize("sight", SIGHTS)
def test_infinities_in_whole_items(dim, dtype, sight):
    """So many items that most lie whole in a block's run."""
    rows = 160
    s = prompts([300, 40] * (rows // 2), [50, 0] * (rows // 2), 4, 2, dim, 16, dtype, seed=6)
    check(s, [x for row in range(0, rows, 2) for x in ((row, 51 + row, row // 2 % 2, 5, math.inf), (row, 60 + row, 1, dim - 1, -math.inf),
                                                       (row, 225, 0, 7, math.inf), (row, 230, 0, 7, -math.inf),
                                                       (row + 1, row // 4, 1, 33, math.inf))], **sight)


@pytest.mark.parametrize("hq,hkv,dim", [(1, 1, 64), (2, 2, 128), (4, 1, 128), (1, 1, 256)])
@pytest.mark.parametrize("sight", [dict(), dict(window=700, sinks=3)])
def test_all_values_undefined(hq, hkv, dim, sight):
    """The slowest that such values can be, in the longest items: a result all the same, and no wait that gives up."""
    s = prompts([2048, 300], [700, 0], hq, hkv, dim, 16, seed=8)
    s["v"].fill_(math.nan)
    d = decoder(s)
    out, lse = d.prompt(**s, lse=True, **sight)
    assert d.status() == 0
    assert out.isnan().all() and lse.isfinite().all()
