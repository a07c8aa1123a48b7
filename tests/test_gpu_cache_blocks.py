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


def check_whole(c, tokens):
    """Every block id is free or one row's, once; the rows hold what their tokens need."""
    for g in range(len(W.groups)):
        held = [c.tables[g][r, :c.blocks(g, n)].tolist() for r, n in enumerate(tokens)]
        assert sorted(sum(held, free_ids(c)[g])) == list(range(90)), g


def test_rejected_drafts_keep_no_blocks(engine):
    """A tree's tokens of which the next call keeps fewer."""
    c = engine.cache
    say("case: drafts rejected")
    c.extend([0], [7])
    for at in (7, 8, 9, 10, 13, 16, 30, 31, 64):
        c.extend([at], [40])
        check_whole(c, [at + 40])
        c.extend([at], [1 if at != 30 else 0])     # (a request that adds nothing is left alone)
        check_whole(c, [at + (1 if at != 30 else 40)])
        if at != 64:
            c.extend([at], [40])
    say("case: none kept")
    c.extend([0], [3])
    check_whole(c, [3])
    c.release(0, 1)     # the request ends: the blocks of what it did not keep go too
    check_whole(c, [0])


def test_blocks_given_back_are_there_to_take(engine):
    c = engine.cache
    say("case: the pool's last blocks")
    c.extend([0, 0], [8, 600])      # 1 + 75 of the last group's 90 blocks
    c.release(1, 600)
    c.extend([0, 0], [0, 560])
    c.extend([8], [8 * 19])         # 1 + 19 + 70: all of them
    assert free_ids(c)[2] == []
    before = [t.clone() for t in c.tables], list(c.taken), free_ids(c)
    assert code(lambda: c.extend([8 * 20], [1])) == bsr.BSR_E_NOMEM
    assert code(lambda: c.extend([8, 560], [8 * 19, 1])) == bsr.BSR_E_NOMEM
    assert all(torch.equal(a, t) for a, t in zip(before[0], c.tables)) and (c.taken, free_ids(c)) == before[1:]
    b = c.extend([8, 560], [8 * 18, 1])     # the first gives 19 back and takes 18
    assert b.result.tolist()[0] == 2
    check_whole(c, [8 * 19, 561])


def test_rows_that_do_not_hold_what_a_call_says(engine):
    """A second release, a release or a request of more than a row holds, a restore into a row in use."""
    e, c = engine, engine.cache
    n, _, _ = bsr.bsr_probe(e.ctx, 25, e.wi.salt, e.wi.tokens)
    c.extend([0, 0], [5, 40])
    say("case: rows that do not hold what a call says")
    for call in (lambda: c.release(0, 9), lambda: c.release(2, 1), lambda: c.extend([0, 0, 1], [0, 0, 1]),
                 lambda: c.extend([17, 40], [1, 1]), lambda: e.session.restore_into(25, n, c, row=1)):
        assert code(call) == bsr.BSR_E_ARG
        check_whole(c, [5, 40])
    c.release(0, 5)
    for call in (lambda: c.release(0, 5), lambda: c.release(0, 1), lambda: c.extend([5], [1])):
        assert code(call) == bsr.BSR_E_ARG
        check_whole(c, [0, 40])
    c.release(0, 0)
    c.release(1, 40)
    check_whole(c, [0, 0])
    out = e.session.restore_into(25, n, c, row=1)
    assert out.exposed_tokens == 320
    check_whole(c, [0, 320])
    bsr.bsr_request_end(e.ctx, 25)


def test_blocks_through_random_calls(engine):
    c = engine.cache
    rng = np.random.default_rng(7)
    tokens = [0, 0, 0]      # that the rows' blocks were laid out for
    say("case: random calls")
    for step in range(60):
        if rng.random() < 0.25:
            r = int(rng.integers(3))
            c.release(r, int(rng.integers(tokens[r] + 1)))
            tokens[r] = 0
        else:
            k = int(rng.integers(1, 4))
            cached = [int(rng.integers(max(0, t - 30), t + 1)) for t in tokens[:k]]
            added = [int(rng.integers(0, 70)) for _ in range(k)]
            then = [x + y if y else t for x, y, t in zip(cached, added, tokens)] + tokens[k:]
            if max(then) > 600 or any(sum(c.blocks(g, t) for t in then) > 90 for g in range(3)):
                continue
            b = c.extend(cached, added)
            tokens = then
            assert b.result.tolist()[0] == k
            for g, s in enumerate(W.groups):
                want = [int(c.tables[g][r, p // s.block_tokens]) * s.block_tokens + p % s.block_tokens
                        for r in range(k) for p in range(cached[r], cached[r] + added[r])]
                assert b.slots[g].tolist() == want
        check_whole(c, tokens)
