"""What a paged cache refuses before it would answer wrongly (GPU)."""

import pytest
import torch

from gpu_side import say
from paper_2608_17826_amd import bsr
from test_gpu_cache_session import Engine

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.fixture
def engine():
    e = Engine()
    yield e
    torch.cuda.synchronize()
    bsr.bsr_ctx_destroy(e.ctx)


def code(call):
    with pytest.raises(bsr.BsrError) as x:
        call()
    return x.value.code


def new_tokens(c, n=4, dtype=torch.bfloat16):
    """A request of n tokens; its K/V records' sources and queries."""
    g = torch.Generator(device="cuda").manual_seed(1)
    b = c.extend([0], [n])
    return b, torch.randn(n, 256, generator=g, device="cuda").to(dtype), torch.randn(n, 2, 128, generator=g, device="cuda").to(dtype)


def attend(c, q, b, **kw):
    kw = dict(dict(max_len=600, offsets=(0, 256)), **kw)
    return c.attend_prompt(2, (0, 0), q, b, (128, 128), 1, **kw)


def test_numbers_past_32_bits_are_refused(engine):
    """They would come out as others in the library's fields."""
    c = engine.cache
    b, kv, q = new_tokens(c)
    c.append(2, 0, b.slots[2], [kv])
    say("case: numbers past 32 bits")
    for kw in (dict(max_len=2 ** 32 + 2), dict(max_len=-1), dict(window=2 ** 32 + 1), dict(window=-(2 ** 32) + 1),
               dict(offsets=(2 ** 32, 256)), dict(offsets=(0, 2 ** 32 + 256)), dict(offsets=(-(2 ** 32), 256))):
        assert code(lambda: attend(c, q, b, **kw)) == bsr.BSR_E_ARG, kw
    assert code(lambda: c.attend_prompt(2, (0, 0), q, b, (128, 128), 2 ** 32 + 1, 600, (0, 256))) == bsr.BSR_E_ARG
    before = list(c.taken)
    assert code(lambda: c.extend([0, 0], [0, 1], n_slots=2 ** 32 + 1)) == bsr.BSR_E_ARG
    assert c.taken == before and c.held[2][1] == 0


def test_gradients_are_refused(engine):
    c = engine.cache
    b, kv, q = new_tokens(c)
    say("case: gradients")
    c.append(2, 0, b.slots[2], [kv])
    out = attend(c, q, b)
    one = torch.ones(4, 1, dtype=torch.int64, device="cuda")
    leaf, rows = q.clone().requires_grad_(), kv.clone().requires_grad_()
    for call in (lambda: attend(c, leaf, b), lambda: attend(c, leaf * 1, b), lambda: c.append(2, 0, b.slots[2], [rows]),
                 lambda: attend(c, q, b, slopes=torch.zeros(2, device="cuda").requires_grad_()),
                 lambda: c.attend_tree(2, (0, 0), leaf, b, one, (128, 128), 1, 600, (0, 256))):
        assert code(call) == bsr.BSR_E_ARG
    with torch.no_grad():
        c.append(2, 0, b.slots[2], [rows])
        assert torch.equal(attend(c, leaf, b), out)
    assert torch.equal(attend(c, leaf.detach(), b), out)


@pytest.mark.parametrize("dtype,other", [(torch.bfloat16, torch.float16), (torch.float16, torch.bfloat16)])
def test_a_cache_read_or_written_as_another_type(engine, dtype, other):
    c = engine.cache
    b, kv, q = new_tokens(c, dtype=dtype)
    say("case: another type than the cache's", dtype)
    attend(c, q, b), attend(c, q.to(other), b)      # nothing has been appended: either may be what was restored
    c.append(2, 0, b.slots[2], [kv], dtype=dtype)
    out = attend(c, q, b)
    assert code(lambda: attend(c, q.to(other), b)) == bsr.BSR_E_ARG
    assert code(lambda: c.append(2, 0, b.slots[2], [kv], dtype=other)) == bsr.BSR_E_ARG
    c.append(2, 0, b.slots[2], [kv.float()], dtype=dtype)    # (the source's type is another matter)
    assert torch.equal(attend(c, q, b), out)
    x = torch.zeros(4, 576, device="cuda")
    c.append(0, 0, b.slots[0], [x], dtype=other)     # another tensor
    c.append(0, 1, b.slots[0], [x], dtype=dtype)
    c.types.pop((2, 0))                              # the pool starts over
    c.append(2, 0, b.slots[2], [kv], dtype=other)
    attend(c, q.to(other), b)
