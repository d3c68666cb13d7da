"""Groups of a cache in 4 bits whose values are finite and whose scale or offset is beyond the type stand for NaN; within
the bounds that the header names none does."""
import pytest

import kv4_plain
from conftest import cuda_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]


# least, largest; whether S = (hi - lo) 16/15 and B = lo - S are numbers of the type (largest: bf16 3.39e38, fp16 65,504)
GROUPS = {"bfloat16": [(-1e38, 1e38, True), (1e38, 1e38, True), (-1e38, -1e38, True), (0.0, 3.3e38, False), (-3e38, 3e38, False),
                       (-3e38, -2e38, False), (2e38, 3e38, True), (-3.3e38, -3.3e38, True)],
          "float16": [(-20000.0, 20000.0, True), (20000.0, 20000.0, True), (0.0, 65504.0, False), (-65504.0, 65504.0, False),
                      (-60000.0, -50000.0, False), (50000.0, 60000.0, True), (-65504.0, -65504.0, True)]}


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_groups_beyond_the_type(dtype):
    import torch
    from paper_2608_02244_gb300 import kv
    groups, dtype = GROUPS[dtype], getattr(torch, dtype)
    n, dim = len(groups), 64
    x = torch.zeros(n, 3, dim)
    for i, (lo, hi, _) in enumerate(groups):
        x[i, :, :32] = torch.linspace(0, 1, 32).double().mul(hi / 4 - lo / 4).add(lo / 4).mul(4).float()      # the other group is 0
    x = x.to(dtype).cuda()
    d = kv.Decoder(1, 16, 1, 1, dim, dtype=dtype, max_rows=1)
    c = d.cache4()
    slots = torch.arange(n, device="cuda")
    d.append4(x.view(n, -1), None, slots, c)
    k, v = d.read4(slots, c)
    assert d.status() == 0
    want = x[:, 2].double()
    bound = kv4_plain.bound(want, want.abs(), dtype)
    for got in (k[:, 0], v[:, 0]):
        assert (got[:, 32:] == 0).all()
        for i, (lo, hi, held) in enumerate(groups):
            if held:
                assert ((got[i].double() - want[i]).abs() <= bound[i]).all(), (lo, hi)
            else:
                assert got[i, :32].isnan().all(), (lo, hi)
