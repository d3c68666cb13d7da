"""A request's life as a server runs it: prompts in chunks through assign, append and prompt, their tokens kept in 4
bits, then single tokens through append4 and attend4; each step against 64 bits over what the caches hold."""
import pytest

import kv4_plain
import kv_plain
import test_kv_prompt_gpu as prompt_tests
from conftest import cuda_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]


@pytest.mark.parametrize("hq,hkv,dim,block,dtype", [(8, 2, 128, 16, "bfloat16"), (7, 1, 64, 8, "float16"), (6, 3, 256, 32, "bfloat16")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 2)])
def test_chain(hq, hkv, dim, block, dtype, window, sinks):
    import torch
    from paper_2608_02244_gb300 import kv
    dtype, rows, width = getattr(torch, dtype), 5, 24
    g = torch.Generator(device="cuda").manual_seed(dim)
    i32 = dict(dtype=torch.int32, device="cuda")
    blocks = rows * width
    d = kv.Decoder(blocks, block, hq, hkv, dim, dtype=dtype, max_rows=rows)
    k, v = (torch.zeros(blocks, block, hkv, dim, dtype=dtype, device="cuda") for _ in range(2))
    cache = d.cache4()
    lens, table = torch.zeros(rows, **i32), torch.full((rows, width), -1, **i32)
    free, n_free = torch.arange(blocks - 1, -1, -1, **i32), torch.tensor([blocks], **i32)
    angle = torch.rand(400, dim // 2, generator=g, device="cuda") * 6.3
    rope = torch.cat((angle.cos(), angle.sin()), 1)
    weights = [torch.randn(dim, generator=g, device="cuda").to(dtype) for _ in range(2)]
    sight = dict(window=window, sinks=sinks)

    for chunk in ([50, 0, 1, 33, 17], [20, 64, 0, 1, 40]):
        tokens = sum(chunk) + 3                            # some places of the step's map stay empty
        plan = d.assign(lens, torch.tensor(chunk, **i32), table, free, n_free, tokens, in_place=True)
        qkv = torch.randn(tokens, (hq + 2 * hkv) * dim, generator=g, device="cuda").to(dtype)
        # the earlier chunks' tokens come back from 4 bits, the new ones are exact
        q = d.append(qkv, plan.positions, plan.slots, k, v, rope, *weights)
        out, lse = d.prompt(q, k, v, table, plan.starts, plan.lens, lse=True, **sight)
        again = d.append4(qkv, plan.positions, plan.slots, cache, rope, *weights)
        back = d.read4(plan.slots, cache)
        assert torch.equal(q, again)
        n = int(plan.starts[-1])
        assert n == sum(chunk)
        s = dict(q=q, k=k, v=v, table=table, starts=plan.starts, lens=plan.lens, prefix=None)
        want, want_lse, size = prompt_tests.plain(s, **sight)
        kv_plain.check_attend(out[:n], lse[:n], want[:n], want_lse[:n], size[:n])
        at = plan.slots[:n]
        k[at // block, at % block], v[at // block, at % block] = back[0][:n], back[1][:n]
    for _ in range(3):
        plan = d.assign(lens, torch.tensor([1, 1, 0, 1, 1], **i32), table, free, n_free, rows, in_place=True)
        qkv = torch.randn(rows, (hq + 2 * hkv) * dim, generator=g, device="cuda").to(dtype)
        q = d.append4(qkv, plan.positions, plan.slots, cache, rope, *weights)
        out, lse = d.attend4(q, cache, table, plan.visible, rows=plan.rows, lse=True, **sight)
        kk, vv = kv4_plain.in_16_bits(cache)
        kv_plain.check_attend(out, lse, *kv_plain.attend(q, kk, vv, table, plan.visible, rows=plan.rows, **sight))
    assert d.status() == 0
