"""A block number outside the cache is reported whatever it is, by each kernel that meets it, and its tokens read as zeros."""
import pytest

import kv_plain
from conftest import cuda_available
from test_kv_attend_gpu import decoder, inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]


# own tokens; a prefix that each query reads; one that is done apart, with heads of one and two halves
@pytest.mark.parametrize("n,shared,dim,where", [(1, 0, 128, "table"), (3, 4, 64, "table"), (3, 4, 256, "prefix"), (17, 80, 128, "prefix"),
                                                (17, 80, 64, "prefix"), (17, 80, 128, "table")])
@pytest.mark.parametrize("number", ["n_blocks", -1, 2**31 - 1, -2**31, -2**31 + 1])
def test_any_bad_block_is_reported(n, shared, dim, where, number):
    import torch
    from paper_2608_02244_gb300 import kv
    s = inputs([70] * n, 4, 2, dim, 16, shared=shared, seed=7)
    d = decoder(s)
    last = s["k"].shape[0]
    (s["table"][0] if where == "table" else s["prefix"])[3] = last if number == "n_blocks" else number
    out, lse = d.attend(**s, lse=True)
    assert d.status() == kv.ISJL_ERR_INVALID_ARG and d.status() == 0
    inside = lambda t: torch.where((t < 0) | (t >= last), last, t)  # noqa: E731
    k, v = (torch.cat((x, torch.zeros_like(x[:1]))) for x in (s["k"], s["v"]))
    plain = dict(s, k=k, v=v, table=inside(s["table"]), prefix=None if s["prefix"] is None else inside(s["prefix"]))
    kv_plain.check_attend(out, lse, *kv_plain.attend(**plain))
