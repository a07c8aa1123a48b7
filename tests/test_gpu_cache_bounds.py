"""The paged cache's operators at the ends of their ranges (GPU)."""

import numpy as np
import pytest
import torch

from cache_side import context, ints, stream
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
