"""Where a paged cache's blocks are: none is lost, none is given out twice (GPU)."""

import numpy as np
import pytest
import torch

from gpu_side import say
from paper_2608_17826_amd import bsr
from paper_2608_17826_amd.cache import PagedCache
from test_gpu_cache_session import W, Engine

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.fixture
def engine():
    e = Engine()
    yield e
    torch.cuda.synchronize()
    bsr.bsr_ctx_destroy(e.ctx)


def free_ids(c):
    """Per group, the free block ids."""
    return [sorted(f[t:].tolist()) for f, t in zip(c.free, c.taken)]


def code(call):
    with pytest.raises(bsr.BsrError) as x:
        call()
    return x.value.code


def test_refused_binds_give_their_blocks_back(engine):
    e, c = engine, engine.cache
    n, _, _ = bsr.bsr_probe(e.ctx, 20, e.wi.salt, e.wi.tokens)
    c.extend([0], [320])
    torch.cuda.synchronize()
    e.session.bind(20, n, c.dsts(0))   # holds the bounded-retrieve lock
    bsr.bsr_probe(e.ctx, 21, e.wi.salt, e.wi.tokens)
    before = free_ids(c)
    say("case: binds refused as busy")
    for _ in range(8):                  # (a prefix takes 20 to 40 of 90 blocks)
        assert code(lambda: e.session.restore_into(21, n, c, row=1)) == bsr.BSR_E_BUSY
        assert free_ids(c) == before
    bsr.bsr_invalidate(e.ctx, 20, bsr.BSR_FAIL_ABORT)
    bsr.bsr_commit(e.ctx, 20)
    bsr.bsr_request_end(e.ctx, 20)
    say("case: a bind of a request that was not probed")
    assert code(lambda: e.session.restore_into(22, n, c, row=1)) == bsr.BSR_E_STATE
    assert free_ids(c) == before
    say("case: the retry")
    out = e.session.restore_into(21, n, c, row=1)
    assert out.fallback == 0 and out.exposed_tokens == 320
    for g, s in enumerate(W.groups):
        for t in range(s.n_tensors):
            np.testing.assert_array_equal(e.records(g, t, 1, 320), e.restored(g, t, n))
        held = c.tables[g][1, :c.blocks(g, 320)].tolist()
        assert sorted(held + free_ids(c)[g]) == before[g]
    bsr.bsr_request_end(e.ctx, 21)


def test_a_hook_that_raises_keeps_the_blocks(engine):
    """Past the bind the GPU may still write to them."""
    e, c = engine, engine.cache
    n, _, _ = bsr.bsr_probe(e.ctx, 23, e.wi.salt, e.wi.tokens)
    calls = []

    def hook():
        calls.append(1)
        raise ValueError("the caller's own")
    say("case: a hook that raises")
    before = free_ids(c)
    with pytest.raises(ValueError):
        e.session.restore_into(23, n, c, row=0, after_bind=hook)
    assert calls == [1]
    assert [len(f) for f in free_ids(c)] == [len(b) - c.blocks(g, 320) for g, b in enumerate(before)]
    bsr.bsr_invalidate(e.ctx, 23, bsr.BSR_FAIL_ABORT)
    bsr.bsr_commit(e.ctx, 23)
    bsr.bsr_request_end(e.ctx, 23)


def test_released_blocks_are_not_valid(engine):
    """Blocks of a restored prefix that hold something else next."""
    e, c = engine, engine.cache
    n, _, _ = bsr.bsr_probe(e.ctx, 24, e.wi.salt, e.wi.tokens)
    e.session.restore_into(24, n, c, row=2)
    bsr.bsr_request_end(e.ctx, 24)
    b = c.extend([0, 0, 320], [50, 0, 9])
    assert [int(v.sum()) for v in c.valid] == [c.blocks(g, 320) for g in range(3)]
    say("case: a restored request ends")
    c.release(2, 329)
    assert not any(v.any() for v in c.valid)
    c.extend([50], [500])
    assert not any(v.any() for v in c.valid)
    assert b.result.tolist()[0] == 3


def test_block_ids_outside_the_pool_are_released_too(engine):
    """As many as a list of free ids has; nothing is written for them."""
    e = engine
    say("case: free ids outside the pool")
    free = [torch.tensor([90, 3, -1, 2 ** 31 - 1, 89, 0], dtype=torch.int32, device="cuda") for _ in W.groups]
    c = PagedCache(e.ctx, e.cache.pools, max_requests=2, max_tokens=600, free=free)
    for v in c.valid:
        v.fill_(1)
    c.extend([0], [32])     # 2, 1 and 4 blocks
    c.release(0, 32)
    got = [v.cpu().numpy() for v in c.valid]
    for v, ids in zip(got, ([90, 3], [90], [90, 3, -1, 2 ** 31 - 1])):
        want = np.ones(90, np.uint8)
        want[[i for i in ids if 0 <= i < 90]] = 0
        np.testing.assert_array_equal(v, want)
