"""Attention weights far below their row's largest one, in fp16 (GPU).

The weights are rounded to the dtype for the products with the values, and
fp16's subnormals end at 2^-24: keys that weigh less one by one still count
together.
"""

import numpy as np
import pytest
import torch

from cache_side import AttnCase, bounds
from gpu_side import say
from oracle import cache as oracle_cache

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]

LATENT, D128, D64 = (576, 512), (128, 128), (64, 64)


def one_key_ahead(dims, gap, n, rows, whole, dtype):
    """A prompt whose key 0 scores `gap` and has values 0; all other keys score 0 and have values 1.

    The score lies in a dimension that is no value's.  ``whole``: as many tiles
    as are not cut, by documents that all begin at 0.
    """
    heads = 128
    c = AttnCase("prompt", [n], [rows], heads, 1, dims, dtype, block=64, scale=1.0,
                 documents=[0] * rows if whole else None)
    at = dims[0] - 1
    rec = torch.zeros(n, c.values, dtype=torch.float32)
    values = slice(0, dims[1]) if c.latent else slice(c.dk, c.dk + c.dv)
    rec[1:, values] = 1
    rec[0, at] = gap
    blocks = c.pool.view(c.pool_blocks, c.block, -1)
    for j in range(0, n, c.block):
        blocks[int(c.tables[0, j // c.block]), :min(c.block, n - j)] = rec[j:j + c.block].to(c.dtype)
    c.q_wide.zero_()
    c.q_wide[..., at] = 1
    return c


@pytest.mark.parametrize("dims,rows", [(D128, 600), (D64, 800), (LATENT, 300)])
@pytest.mark.parametrize("gap", [10.0, 17.0, 17.5, 21.0])   # e^-17.5 = 2^-25.2
@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_keys_far_below_the_first(dims, rows, gap, whole, dtype):
    n = 4096
    say("case: keys far below the first", dims, gap, whole, dtype)
    c = one_key_ahead(dims, gap, n, rows, whole, dtype).run()
    out, lse = c.d["out"].double().cpu().numpy(), c.d["lse"].double().cpu().numpy()
    k, v = np.zeros((n, dims[0])), np.ones((n, dims[1]))
    k[0, -1], v[0] = gap, 0
    q = np.zeros(dims[0])
    q[-1] = 1
    for i in (0, 1, rows // 2, rows - 1):
        see, p = oracle_cache.visible("prompt", n, rows, i)
        o, l, a, dot = oracle_cache.attend(q, k, v, see, p, 1.0)
        bound, lb = bounds(o, l, a, dot, c.dtype, dims[0], int(see.sum()))
        if dtype == "f16":
            # each key's weight is off by half of fp16's last subnormal step, 2^-25, where the largest one is held as
            # 2^7 at least: 2^-32 of the sum
            bound = bound + see.sum() * 2.0 ** -32
        for h in (0, 77):
            err = np.abs(out[i, h, :dims[1]] - o)
            assert np.all(err <= bound), (i, h, float(err.max()), float(bound.min()), float(o[0]))
            assert abs(lse[i, h] - l) <= lb, (i, h)
