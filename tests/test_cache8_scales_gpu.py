"""The scale bytes that the header names, all of them: a read gives what attention sees, and an append behind rows at either
end of the range keeps them as they were."""

import numpy as np
import pytest
import torch

from oracle import cache8
from paper_2605_05819_amd import cl

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("dtype,lo,hi", [(F16, 112, 135), (BF16, 10, 247)], ids=["fp16", "bf16"])
def test_reads_and_attention_agree_on_every_scale(dtype, lo, hi):
    """One key a sequence: attention gives its value, whatever the query (softmax over one key is 1).  A page a scale."""
    n, D = hi - lo + 1, 64
    g = torch.Generator().manual_seed(lo)
    codes = torch.randint(0, 256, (n, 1, 1, D), generator=g, dtype=torch.int32).to(torch.uint8)
    codes[codes & 0x7f == 0x7f] = 0x7e                      # no NaN
    codes[-1].bitwise_and_(0xf7)                            # the largest scale: 240 2^8 and 240 2^120 are the types' largest, 448 would pass them
    scales = torch.arange(lo, hi + 1).to(torch.uint8).view(n, 1, 1)
    cache = cl.KvCache8(codes.cuda(), codes.cuda(), scales.cuda(), scales.cuda(), dtype)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = cl.KvBatch(i32([1] * n), i32(list(range(n))).view(n, 1), n, max_kv_len=1)
    k, v = cl.kv_read(cache, batch)
    out = cl.attention(cache, batch, torch.zeros((n, 1, D), dtype=dtype, device="cuda"), out_dtype=dtype)
    torch.cuda.synchronize()
    want = cache8.decode(codes.numpy()).reshape(n, 1, D) * 2.0 ** (scales.numpy().astype(np.float64).reshape(n, 1, 1) - 127)
    assert np.array_equal(k.double().cpu().numpy(), want) and torch.equal(k, v) and torch.equal(out.abs(), v.abs())
    assert np.array_equal(out.double().cpu().numpy(), want)
