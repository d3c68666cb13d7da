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
