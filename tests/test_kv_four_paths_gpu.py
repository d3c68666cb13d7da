"""attend4 on both sides of the number of queries with which one block less fits an SM: what is launched, and results."""
import numpy as np
import pytest

import kv4_plain
import kv_plain
from conftest import cuda_available
from test_kv_four_gpu import decoder4, requests
from test_kv_paths_gpu import blocks_of, launches, sms

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]


@pytest.mark.parametrize("n", [3000, 4096])
@pytest.mark.parametrize("hq,hkv,dim,blocks", [(8, 2, 128, (3, 2)), (16, 1, 128, (2, 2)), (4, 1, 256, (2, 1)), (5, 1, 64, (3, 3))])
def test_blocks_by_queries(n, hq, hkv, dim, blocks):
    """More places before queries lie in each block's shared memory: the grid is what fits, not a part of it twice."""
    rng = np.random.default_rng(n)
    s = requests(np.where(rng.random(n) < 0.1, 0, rng.integers(1, 60, n)), hq, hkv, dim, 16, seed=n)
    d = decoder4(s)
    out, lse = d.attend4(**s, lse=True)
    assert d.status() == 0
    k, v = kv4_plain.in_16_bits(s["cache"])
    plain = {x: y for x, y in s.items() if x != "cache"}
    kv_plain.check_attend(out, lse, *kv_plain.attend(**plain, k=k, v=v))
    found = launches(lambda: d.attend4(**s, lse=True))
    assert blocks_of(found, "attend4_kernel") == blocks[n > 3200] * sms()


@pytest.mark.parametrize("hq,hkv", [(700, 700)])
def test_a_warp_for_each_head_where_few_blocks_fit(hq, hkv):
    rng = np.random.default_rng(5)
    n = 3500
    s = requests(np.where(rng.random(n) < 0.9, 0, rng.integers(1, 3, n)), hq, hkv, 256, 8, seed=5)
    d = decoder4(s)
    out, lse = d.attend4(**s, lse=True)
    assert d.status() == 0
    k, v = kv4_plain.in_16_bits(s["cache"])
    plain = {x: y for x, y in s.items() if x != "cache"}
    kv_plain.check_attend(out, lse, *kv_plain.attend(**plain, k=k, v=v))
    assert blocks_of(launches(lambda: d.attend4(**s, lse=True)), "attend4_kernel") == max(sms(), hkv // 4)
