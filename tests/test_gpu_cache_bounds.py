"""The paged cache's operators at the ends of their ranges (GPU)."""

import numpy as np
import pytest
import torch

from cache_side import AttnCase, context, ints, stream
from gpu_side import say
from paper_2608_17826_amd import bsr

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]
C = bsr.BSR_KIND_CONTIG
MOST = 2 ** 31 - 1


@pytest.mark.parametrize("added,admitted", [([MOST, 1, 3], 1), ([2 ** 30, 2 ** 30 - 1, 0, 1], 3), ([2 ** 30] * 5, 1),
                                            ([MOST, MOST], 1), ([5, MOST, 7], 1), ([7] + [0] * 70 + [MOST - 7, 1], 72),
                                            ([MOST - 1] + [0] * 80 + [2] * 100, 81)])
def test_rows_past_31_bits(added, admitted):
    """A batch with room for 2^31 - 1 rows (no tables, no slots): the request that would pass it gets nothing."""
    say("case: rows past 31 bits", added[:5], admitted)
    n = len(added)
    d = dict(cached=ints(np.zeros(n)), added=ints(added), starts=ints(np.full(n + 1, 77)), lens=ints(np.full(n, 77)),
             result=ints(np.full(2, 77)))
    a = bsr.tables_args(n, d["cached"].data_ptr(), d["added"].data_ptr(), [bsr.table_group(0, 0, 0, 0)], MOST,
                        d["starts"].data_ptr(), d["lens"].data_ptr(), d["result"].data_ptr())
    bsr.bsr_tables_build(context((16, 1, 64, C, 0)), a, stream())
    torch.cuda.synchronize()
    assert d["result"].tolist() == [admitted, 0]
    sums = np.concatenate([[0], np.cumsum(np.asarray(added[:admitted], np.int64))])
    assert d["starts"].tolist() == list(sums) + [sums[-1]] * (n - admitted)
    assert d["lens"].tolist() == added[:admitted] + [0] * (n - admitted)


@pytest.mark.parametrize("mode", ["tree", "prompt"])
@pytest.mark.parametrize("dims,heads,kv", [((64, 64), 2, 1), ((128, 128), 4, 2), ((576, 512), 16, 1)])
def test_lengths_past_the_tables(mode, dims, heads, kv):
    """lens above what a table holds, where max_len would allow them: the table's last token is the request's."""
    say("case: lengths past the tables", mode, dims)
    rows = [1, 3]
    c = AttnCase(mode, [96, 96], rows, heads, kv, dims, masks=[1, 1, 3, 7] if mode == "tree" else None, seed=31, max_len=5000)
    c.stride = 6                       # 96 tokens in blocks of 16: all that the tables hold
    c.tables = c.tables[:, :6].contiguous()
    c.place()
    for far in (97, 4000, MOST):
        c.d["lens"].fill_(far)
        c.d["out"].fill_(7)
        c.d["lse"].fill_(7)
        c.call(c.prepare())
        torch.cuda.synchronize()
        c.check()


@pytest.mark.parametrize("dims,heads,kv", [((64, 64), 2, 1), ((576, 512), 16, 1)])
def test_starts_past_the_rows(dims, heads, kv):
    """starts beyond n_tokens and below zero end at the rows there are."""
    say("case: starts past the rows", dims)
    # rows 0..4 in both; the kernel reads starts [-9, 2, 1000, 2^31 - 1]: rows 0 and 1, 2 to 4, none
    c = AttnCase("prompt", [40, 77, 9], [2, 3, 0], heads, kv, dims, seed=32).place()
    c.d["starts"].copy_(torch.tensor([-9, 2, 1000, MOST], dtype=torch.int32))
    c.call()
    torch.cuda.synchronize()
    c.check()


@pytest.mark.parametrize("mode", ["tree", "prompt"])
@pytest.mark.parametrize("dims,heads,kv,dtype", [((64, 64), 4, 2, "f16"), ((128, 128), 4, 2, "bf16"), ((128, 128), 32, 1, "bf16")])
@pytest.mark.parametrize("n", [70, 3000])
def test_keys_and_values_in_two_pools(mode, dims, heads, kv, dtype, n):
    """K and V in two tensors of a group, at offsets of their own."""
    say("case: two pools", mode, dims, kv, n)
    rows = [5, 1]
    c = AttnCase(mode, [n, 33], rows, heads, kv, dims, dtype, lead=16,
                 masks=[1, 3, 5, 11, 19, 1] if mode == "tree" else None, seed=33).place()
    k_at, v_at, width = c.lead, c.lead + kv * c.dk, kv * c.dk
    # the first pool holds the keys where they were and nothing else, the second the values from 8 on
    other = torch.full_like(c.d["pool"], float("nan"))
    other[:, 8:8 + width] = c.d["pool"][:, v_at:v_at + width]
    c.d["pool"][:, v_at:] = float("nan")
    c.d["other"] = other
    c.call(c.prepare(v_pool=other.data_ptr(), v_offset=16, k_offset=2 * k_at))
    torch.cuda.synchronize()
    c.check(sample=60)
