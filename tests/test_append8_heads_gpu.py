"""Appends to an 8-bit cache with one, three and five key heads whose first sequence begins with token 0: the waves beyond
the last head have nothing of k and v to read there (their addresses: tests/test_append8_addresses.py)."""

import numpy as np
import pytest
import torch

from paper_2605_05819_amd import cl
from tests.test_cache8_gpu import BF16, F16, Pool, turned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hkv", [1, 3, 5])
@pytest.mark.parametrize("D,page,block", [(64, 64, 64), (128, 16, 16), (128, 32, 1), (256, 64, 32), (64, 256, 256)])
def test_odd_key_heads_from_the_first_token(Hkv, D, page, block):
    """Single tokens and prompts, of tensors that are all of their allocation and of views with other rows around them."""
    g = np.random.default_rng(Hkv + D)
    dtype = F16 if D == 128 else BF16
    freq = cl.rope_frequencies(D, 10000.0)[0]
    rope = cl.Rope(freq.cuda())
    for view in (False, True):
        p = Pool([640, 40], Hkv, D, page, block, dtype, seed=Hkv)
        lens = np.zeros(2, np.int64)
        for counts in ([1, 1], [600, 13], [7, 0], [1, 1]):
            lens += counts
            N = sum(counts)
            k, v = (torch.from_numpy(g.standard_normal((N, Hkv, D))).to(dtype).cuda() for _ in range(2))
            if view:
                wide = torch.full((N + 2, 2, Hkv, D), float("nan"), dtype=dtype, device="cuda")
                wide[1:-1, 0], wide[1:-1, 1] = k, v
                k, v = wide[1:-1, 0], wide[1:-1, 1]
            cl.kv_append(p.cache, p.batch(list(lens), counts), k, v, rope=rope)
            torch.cuda.synchronize()
            p.check(lens, counts, turned(k.double().cpu().numpy(), lens, counts, freq.double().numpy()), v.double().cpu().numpy())
