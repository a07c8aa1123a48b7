"""A restore and what follows it in an engine, over one paged cache (GPU).

Blocks laid out on the GPU, a prefix restored into them, new tokens appended
and attended to, as prompt and as drafted trees, in groups of latent records,
index keys and K/V records: every cached byte against what was stored or
appended, and attention against its definition in 64 bits.
"""

import numpy as np
import pytest
import torch

from cache_side import bounds
from gpu_side import layout_of, say
from oracle import cache as oracle_cache
from paper_2608_17826_amd import bsr
from paper_2608_17826_amd.cache import Batch, PagedCache
from paper_2608_17826_amd.session import RestoreSession
from workloads import generate
from workloads.configs import GroupSpec, Workload

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]

W = Workload(index=40, name="serve", n_tokens=64 * 5 + 9, chunk_tokens=64, windows=(2,), groups=(
    GroupSpec("latent", 16, 2, 1152), GroupSpec("index", 32, 1, 132, kind="planar", split_bytes=128, value_kind="fp8_scaled"),
    GroupSpec("swa", 8, 1, 512)))


class Engine:
    def __init__(self):
        self.wi = generate(W)
        self.ctx = bsr.bsr_ctx_create(layout_of(self.wi), 2, hip_device=0)
        bsr.bsr_store_reserve(self.ctx, 16 << 20)
        keys = bsr.bsr_chunk_keys(self.wi.salt, self.wi.tokens, W.chunk_tokens)
        bsr.bsr_store_put_chunks(self.ctx, [int(k) for k in keys], [self.wi.payloads(i) for i in range(len(keys))])
        self.keys = keys
        g = torch.Generator().manual_seed(3)
        pools = [[torch.randint(0, 255, (90, s.block_tokens * s.record_bytes), generator=g, dtype=torch.uint8).cuda()
                  for _ in range(s.n_tensors)] for s in W.groups]
        for group in pools:      # what no token has written yet
            for p in group:
                p.fill_(0xFF)
        free = [torch.randperm(90, generator=g).to(torch.int32).cuda() for _ in W.groups]
        self.cache = PagedCache(self.ctx, pools, max_requests=3, max_tokens=600, free=free)
        self.session = RestoreSession(self.ctx)

    def records(self, g, t, row, tokens):
        """uint8 [tokens, record_bytes] of table row `row`."""
        s, c = W.groups[g], self.cache
        tab = c.tables[g][row].cpu().numpy()
        pool = c.pools[g][t].cpu().numpy()
        out = np.empty((tokens, s.record_bytes), np.uint8)
        for j in range(tokens):
            b, o = tab[j // s.block_tokens], j % s.block_tokens
            if s.kind == "contig":
                out[j] = pool[b, o * s.record_bytes:(o + 1) * s.record_bytes]
            else:
                out[j, :s.split_bytes] = pool[b, o * s.split_bytes:(o + 1) * s.split_bytes]
                at, rest = s.block_tokens * s.split_bytes, s.record_bytes - s.split_bytes
                out[j, s.split_bytes:] = pool[b, at + o * rest:at + (o + 1) * rest]
        return out

    def restored(self, g, t, n):
        out = []
        for i in range(n):
            s = W.groups[g]
            e = self.wi.payload(i, g).reshape(s.n_tensors, W.chunk_tokens, s.record_bytes)
            out.append(e[t])
        return np.concatenate(out)


def bf16(records):
    return torch.from_numpy(np.ascontiguousarray(records)).view(torch.bfloat16).double().numpy()


def check_rows(out, lse, q, k, v, rows, see_of, scale, **kw):
    out, lse, q = out.double().cpu().numpy(), lse.double().cpu().numpy(), q.double().cpu().numpy()
    for i, row in enumerate(rows):
        see, p = see_of(i)
        for h in range(q.shape[1]):
            o, l, a, d = oracle_cache.attend(q[row, h], k, v, see, p, scale, **kw)
            bound, lb = bounds(o, l, a, d, torch.bfloat16, q.shape[2], int(see.sum()))
            assert np.all(np.abs(out[row, h] - o) <= bound) and abs(lse[row, h] - l) <= lb, (i, h)


def test_restore_append_and_attend():
    e = Engine()
    c = e.cache
    gen = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    try:
        n, _, _ = bsr.bsr_probe(e.ctx, 7, e.wi.salt, e.wi.tokens)
        assert n == 5
        say("case: restore into blocks laid out on the GPU")
        out = e.session.restore_into(7, n, c, row=1)
        assert out.exposed_tokens == 320 and out.fallback == 0
        for g, s in enumerate(W.groups):
            for t in range(s.n_tensors):
                np.testing.assert_array_equal(e.records(g, t, 1, 320), e.restored(g, t, n))
            held = set(c.tables[g][1, :c.blocks(g, 320)].tolist())
            assert set(np.nonzero(c.valid[g].cpu().numpy())[0]) == held and len(held) == c.blocks(g, 320)
        bsr.bsr_request_end(e.ctx, 7)

        say("case: the prompt's tail, beside a new request")
        cached, added = [0, 320, 0], [21, 9, 0]
        b = c.extend(cached, added, n_slots=33)
        assert b.result.tolist() == [3] + [sum(c.blocks(g, x + y) - c.blocks(g, x) for x, y in zip(cached, added))
                                           for g in range(3)]
        latent, rope, keys = rand(33, 512).bfloat16(), rand(33, 64).bfloat16(), rand(33, 128)
        kv = rand(33, 256).bfloat16()
        for t in range(2):
            c.append(0, t, b.slots[0], [latent * (t + 1), rope])
        c.append(1, 0, b.slots[1], [keys])
        c.append(2, 0, b.slots[2], [kv[:, :128], kv[:, 128:]])
        for row, first, (x, y) in ((0, 0, (0, 21)), (1, 21, (320, 9))):
            for t in range(2):
                want = torch.cat([latent * (t + 1), rope], 1)[first:first + y].view(torch.uint8).cpu().numpy()
                np.testing.assert_array_equal(e.records(0, t, row, x + y)[x:], want)
            np.testing.assert_array_equal(e.records(2, 0, row, x + y)[x:], kv[first:first + y].view(torch.uint8).cpu().numpy())
            got = e.records(1, 0, row, x + y)[x:]
            scale = keys[first:first + y].abs().amax(1).cpu() / 448
            assert torch.equal(torch.from_numpy(got[:, 128:].copy()).view(torch.float32)[:, 0], scale)
            back = torch.from_numpy(got[:, :128].copy()).view(torch.float8_e4m3fn).float() * scale[:, None]
            # half a step of e4m3 is 2^-4 of the value, and at the bottom 2^-10 of the scale
            off = (back - keys[first:first + y].cpu()).abs()
            assert bool((off <= back.abs() * 2.0 ** -4 * (1 + 2.0 ** -3) + scale[:, None] * 2.0 ** -10).all())
        for g, s in enumerate(W.groups):    # the restored prefix is as it was
            np.testing.assert_array_equal(e.records(g, 0, 1, 320), e.restored(g, 0, n))
        q = rand(33, 16, 576).bfloat16()
        o, lse = c.attend_prompt(0, (1, 1), q, b, (576, 512), 1, max_len=600, scale=0.1, lse=True)
        for row, first, (x, y) in ((0, 0, (0, 21)), (1, 21, (320, 9))):
            k = bf16(e.records(0, 1, row, x + y))
            check_rows(o, lse, q, k, k[:, :512], range(first, first + y),
                       lambda i: oracle_cache.visible("prompt", x + y, y, i), float(np.float32(0.1)))

        say("case: a drafted tree and a single token")
        cached, added = [21, 329, 0], [1, 4, 0]
        b = c.extend(cached, added)
        kv = rand(5, 256).bfloat16()
        c.append(2, 0, b.slots[2], [kv])
        masks = [1, 0b1, 0b11, 0b101, 0b1011]
        q = rand(5, 8, 128).bfloat16()
        o, lse = c.attend_tree(2, (0, 0), q, b, torch.tensor(masks, device="cuda")[:, None], (128, 128), 1, max_len=600,
                               offsets=(0, 256), window=100, lse=True)
        for row, first, (x, y) in ((0, 0, (21, 1)), (1, 1, (329, 4))):
            r = bf16(e.records(2, 0, row, x + y))
            check_rows(o, lse, q, r[:, :128], r[:, 128:], range(first, first + y),
                       lambda i: oracle_cache.visible("tree", x + y, y, i, mask=[masks[first + i]], window=100),
                       float(np.float32(128 ** -0.5)))
    finally:
        bsr.bsr_ctx_destroy(e.ctx)


def test_fallback_gives_its_blocks_back():
    e = Engine()
    c = e.cache
    try:
        n, _, _ = bsr.bsr_probe(e.ctx, 8, e.wi.salt, e.wi.tokens)
        bsr.bsr_store_remove(e.ctx, int(e.keys[3]), 2)
        say("case: a restore that falls back")
        before = [sorted(f[t:].tolist()) for f, t in zip(c.free, c.taken)]
        out = e.session.restore_into(8, n, c, row=0)
        assert out.fallback == 1 and out.exposed_tokens == 0
        assert [sorted(f[t:].tolist()) for f, t in zip(c.free, c.taken)] == before
        bsr.bsr_request_end(e.ctx, 8)
        with pytest.raises(bsr.BsrError) as x:
            c.extend([0, 0], [600, 600])
        assert x.value.code == bsr.BSR_E_NOMEM
        with pytest.raises(bsr.BsrError) as x:
            c.extend([0], [700])
        assert x.value.code == bsr.BSR_E_ARG
    finally:
        bsr.bsr_ctx_destroy(e.ctx)


def test_captured_decode_step():
    """Append and attention in one graph, replayed over new tokens."""
    e = Engine()
    c = e.cache
    try:
        gen = torch.Generator(device="cuda").manual_seed(6)
        n, _, _ = bsr.bsr_probe(e.ctx, 9, e.wi.salt, e.wi.tokens)
        e.session.restore_into(9, n, c, row=0)
        say("case: a decode step in a graph")
        b = c.extend([320], [1])
        x, q = torch.zeros(1, 576, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 16, 576, dtype=torch.bfloat16, device="cuda")
        one = torch.ones(1, 1, dtype=torch.int64, device="cuda")

        def step():
            c.append(0, 0, b.slots[0], [x])
            return c.attend_tree(0, (0, 0), q, b, one, (576, 512), 1, max_len=600, lse=True)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o, lse = step()
        for at in range(320, 324):
            if at > 320:
                nb = c.extend([at], [1])
                for dst, src in zip([b.starts, b.lens, b.result] + b.slots, [nb.starts, nb.lens, nb.result] + nb.slots):
                    dst.copy_(src)
            x.normal_(generator=gen)
            q.normal_(generator=gen)
            graph.replay()
            torch.cuda.synchronize()
            k = bf16(e.records(0, 0, 0, at + 1))
            np.testing.assert_array_equal(k[at], x[0].double().cpu().numpy())
            check_rows(o, lse, q, k, k[:, :512], [0], lambda i: oracle_cache.visible("tree", at + 1, 1, 0, mask=[1]),
                       float(np.float32(576 ** -0.5)))
        bsr.bsr_request_end(e.ctx, 9)
    finally:
        bsr.bsr_ctx_destroy(e.ctx)


def test_the_cache_checks_rows_and_batches():
    """Rows outside the tables, blocks that a row cannot hold, and batches that are not the tables'."""
    e = Engine()
    c = e.cache
    try:
        b = c.extend([0], [4])
        before = [t.clone() for t in c.tables], list(c.taken)
        q = torch.zeros(4, 2, 128, dtype=torch.bfloat16, device="cuda")
        i32 = dict(dtype=torch.int32, device="cuda")
        attend = lambda starts, lens: c.attend_prompt(2, (0, 0), q, Batch(starts, lens, b.slots, b.result),  # noqa: E731
                                                      (128, 128), 1, 600, (0, 256))
        say("case: rows and batches that are not the cache's")
        for call in [lambda: c.dsts(-1), lambda: c.dsts(3), lambda: c.release(3, 4), lambda: c.release(-1, 4),
                     lambda: c.release(0, -1), lambda: c.release(0, 601 + 16), lambda: e.session.restore_into(5, 1, c, -1),
                     lambda: e.session.restore_into(5, 1, c, 3),
                     lambda: attend(torch.zeros(5, **i32), torch.zeros(4, **i32)), lambda: attend(b.starts[:1], b.lens),
                     lambda: attend(b.starts.long(), b.lens), lambda: attend(b.starts, b.lens.long()),
                     lambda: attend(b.starts.cpu(), b.lens), lambda: attend(torch.zeros(4, **i32)[::2], b.lens)]:
            with pytest.raises(bsr.BsrError) as x:
                call()
            assert x.value.code == bsr.BSR_E_ARG
        assert c.taken == before[1] and all(torch.equal(a, t) for a, t in zip(before[0], c.tables))
        attend(b.starts, b.lens)
    finally:
        bsr.bsr_ctx_destroy(e.ctx)


def test_the_cache_checks_its_tensors():
    e = Engine()
    c = e.cache
    try:
        b = c.extend([0], [4])
        q = torch.zeros(4, 2, 128, dtype=torch.bfloat16, device="cuda")
        say("case: tensors of the wrong type or shape")
        bad = [lambda: c.append(2, 0, b.slots[2].int(), [q[:, 0]]), lambda: c.append(2, 0, b.slots[2], [q[:3, 0]]),
               lambda: c.append(2, 0, b.slots[2], [q[:, 0], q[:, 1].float()]),
               lambda: c.append(2, 0, b.slots[2], [q[:, 0].double(), q[:, 1].double()]),
               lambda: c.attend_prompt(2, (0, 0), q.float(), b, (128, 128), 1, 600, (0, 256)),
               lambda: c.attend_prompt(2, (0, 0), q, b, (64, 64), 1, 600, (0, 256)),
               lambda: c.attend_prompt(2, (0, 0), q, b, (128, 128), 1, 600, (0, 256), documents=torch.zeros(3, dtype=torch.int32, device="cuda")),
               lambda: c.attend_prompt(2, (0, 0), q, b, (128, 128), 1, 600, (0, 256), slopes=torch.zeros(2, device="cuda").double()),
               lambda: c.attend_tree(2, (0, 0), q, b, torch.zeros(4, dtype=torch.int64, device="cuda"), (128, 128), 1, 600),
               lambda: c.attend_prompt(2, (0, 0), q, b, (128, 128), 1, 600, (0, 256), out=torch.empty(4, 2, 64, dtype=torch.bfloat16, device="cuda")),
               lambda: c.attend_prompt(1, (0, 0), q, b, (128, 128), 1, 600)]
        for call in bad:
            with pytest.raises(bsr.BsrError) as x:
                call()
            assert x.value.code == bsr.BSR_E_ARG
    finally:
        bsr.bsr_ctx_destroy(e.ctx)
