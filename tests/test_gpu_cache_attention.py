"""Attention over the paged cache against its definition in 64 bits (GPU)."""

import numpy as np
import pytest
import torch

from cache_side import AttnCase, stream
from gpu_side import say
from paper_2608_17826_amd import bsr

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]

LATENT, D128, D64 = (576, 512), (128, 128), (64, 64)
FAR = 2 ** 31 - 1


def chain(T):
    return [(1 << (i + 1)) - 1 for i in range(T)]


def random_tree(T, rng):
    m = []
    for i in range(T):
        m.append((m[rng.integers(max(0, i - 5), i)] if i else 0) | 1 << i)
    return m


def words_of(masks, words):
    return [[m >> 64 * k & (2 ** 64 - 1) for k in range(words)] for m in masks]


@pytest.mark.parametrize("dims,heads,kv", [(LATENT, 16, 1), (LATENT, 128, 1), (LATENT, 5, 1), (D128, 8, 2),
                                           (D128, 3, 3), (D64, 14, 2), (D64, 1, 1), (D128, 160, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_single_tokens(dims, heads, kv, dtype):
    """A decode step: lengths from the token alone to over a few tiles."""
    lens = [1, 2, 31, 33, 64, 65, 200, 517]
    say("case: single tokens", dims, heads, kv, dtype)
    c = AttnCase("tree", lens, [1] * len(lens), heads, kv, dims, dtype, masks=[1] * len(lens), seed=heads)
    c.run().check(sample=200)


@pytest.mark.parametrize("dims,heads,kv,block", [(LATENT, 16, 1, 64), (LATENT, 128, 1, 16), (D128, 32, 8, 32),
                                                 (D64, 6, 2, 5), (D128, 7, 1, 128), (LATENT, 3, 1, 1)])
def test_trees(dims, heads, kv, block):
    """Trees behind ragged prefixes; a padded node that sees no node; a request without rows, one without tokens."""
    rng = np.random.default_rng(heads)
    lens, rows = [70, 0, 300, 33, 90, 4], [17, 0, 64, 1, 0, 4]
    masks = []
    for T in rows:
        m = random_tree(T, rng)
        if T > 10:
            m[-1] = 0
        masks += m
    masks[-1] = 0    # the last request's last node sees nothing but ...
    masks[-4] = 0    # ... its rows are all there is: an empty row
    say("case: trees", dims, heads, kv, block)
    c = AttnCase("tree", lens, rows, heads, kv, dims, block=block, masks=masks, tail_rows=3, lead=8, q_pad=8, seed=1)
    c.run().check(sample=300)


@pytest.mark.parametrize("words,T", [(2, 100), (4, 256), (2, 150)])
def test_wide_trees(words, T):
    """Masks of several words; rows past the words are seen by none."""
    rng = np.random.default_rng(T)
    masks = words_of([m & ((1 << 64 * words) - 1) for m in random_tree(T, rng)], words)
    say("case: wide trees", words, T)
    c = AttnCase("tree", [T + 40, T], [T, T], 4, 2, D128, masks=masks + masks, words=words, seed=2)
    c.run().check(sample=300)


@pytest.mark.parametrize("dims,heads,kv", [(D128, 4, 1), (LATENT, 16, 1)])
def test_tree_window_and_cap(dims, heads, kv):
    say("case: tree window and cap", dims)
    c = AttnCase("tree", [500, 90, 64], [9, 5, 64], heads, kv, dims, masks=chain(9) + chain(5) + chain(64), window=64,
                 cap=3.0, seed=3)
    c.run().check(sample=300)


@pytest.mark.parametrize("dims,heads,kv,dtype", [(D128, 4, 2, "bf16"), (D64, 3, 1, "f16"), (LATENT, 16, 1, "bf16"),
                                                 (D64, 2, 2, "bf16"), (LATENT, 200, 1, "f16")])
@pytest.mark.parametrize("cached", [0, 1, 250])
def test_prompts(dims, heads, kv, dtype, cached):
    lens = [cached + T for T in (150, 1, 0, 37)]
    say("case: prompts", dims, heads, kv, dtype, cached)
    c = AttnCase("prompt", lens, [150, 1, 0, 37], heads, kv, dims, dtype, block=16, seed=4, tail_rows=2)
    c.run().check(sample=300)


@pytest.mark.parametrize("dims,heads,kv", [(D128, 4, 2), (D64, 5, 1), (LATENT, 8, 1)])
@pytest.mark.parametrize("what", ["documents", "prefix", "slopes", "window", "all"])
def test_prompt_masks(dims, heads, kv, what):
    lens, rows = [210, 90, 64, 700], [130, 90, 3, 200]
    rng = np.random.default_rng(5)
    kw = {}
    if what in ("documents", "all"):
        docs = []
        for n, T in zip(lens, rows):
            at = 0
            for i in range(T):
                if rng.random() < 0.05:
                    at = n - T + i
                docs.append(at)
        docs[7] = FAR       # padding: sees nothing
        docs[130] = -5      # before the first position: the first
        kw["documents"] = docs
    if what in ("prefix", "all"):
        kw["prefix"] = [100, 1000, 0, 640]
    if what in ("slopes", "all"):
        kw["slopes"] = [2.0 ** -(i + 1) for i in range(heads)]
    if what in ("window", "all"):
        kw["window"] = 33
    if what == "all":
        kw["cap"] = 5.0
    say("case: prompt masks", dims, what)
    c = AttnCase("prompt", lens, rows, heads, kv, dims, block=32, seed=6, **kw)
    c.run().check(sample=400)


@pytest.mark.parametrize("dims,heads,kv,dtype", [(D128, 4, 2, "f16"), (D64, 2, 1, "bf16"), (LATENT, 16, 1, "f16")])
@pytest.mark.parametrize("cap,scale", [(63.0, None), (65.0, None), (65.0, 4.0), (1e4, None), (1e6, 40.0), (1e30, None),
                                       (3e38, 1e-3), (1e-30, None)])
def test_caps_of_every_width(dims, heads, kv, dtype, cap, scale):
    """Caps far above the scores leave them alone; scores on both sides of 0.4 caps; a cap that leaves them all zero."""
    say("case: caps", dims, cap, scale)
    c = AttnCase("prompt", [150, 40], [70, 1], heads, kv, dims, dtype, cap=cap, scale=scale, seed=12)
    c.run().check(sample=200)


def test_more_rows_than_tokens():
    """Rows before the first position see nothing (of a prompt), or what the tree still has."""
    say("case: more rows than tokens")
    c = AttnCase("prompt", [3, 0], [8, 2], 2, 1, D64, seed=7)
    c.run().check()
    c = AttnCase("tree", [3], [8], 2, 1, D64, masks=chain(8), seed=7)
    c.run().check()


@pytest.mark.parametrize("dims,heads,kv", [(D128, 2, 1), (LATENT, 4, 1)])
def test_non_finite_keys_and_values(dims, heads, kv):
    """What a row does not see counts for nothing; what it sees goes through."""
    docs = [0] * 40 + [40] * 40 + [0] * 20
    c = AttnCase("prompt", [100], [100], heads, kv, dims, documents=docs, seed=8)
    say("case: NaN in one document", dims)
    t = 10
    b = int(c.tables[0, t // 16])
    rec = c.pool.view(c.pool_blocks, 16, -1)[b, t % 16]
    rec[:] = float("nan")
    c.run().check()
    say("case: an infinite value", dims)
    rec[:] = 0.5
    rec[5 if c.latent else kv * c.dk + 5] = float("inf")
    if not c.latent:   # (of a latent record the value is the key, whose score is then infinite too)
        c.run().check()
    masks = [1, 3, 5, 0]
    say("case: NaN in another branch", dims)
    c = AttnCase("tree", [50], [4], heads, kv, dims, masks=masks, seed=9)
    t = 47
    c.pool.view(c.pool_blocks, 16, -1)[int(c.tables[0, t // 16]), t % 16] = float("nan")
    c.run().check()


def test_blocks_outside_the_pool():
    for dims, heads in ((D128, 2), (LATENT, 4)):
        say("case: block ids outside the pool", dims)
        c = AttnCase("prompt", [150, 60], [30, 60], heads, 1, dims, seed=10)
        c.tables[0, 2] = -1
        c.tables[0, 5] = c.pool_blocks
        c.tables[1, :] = 2 ** 31 - 1
        c.run().check()


def test_lengths_past_their_bounds():
    """lens above max_len or the table, below zero, and starts past the rows are taken as the nearest that holds."""
    say("case: lengths past their bounds")
    c = AttnCase("tree", [100, 60], [1, 1], 2, 1, D64, masks=[1, 1], seed=11)
    c.place()
    c.d["lens"][0] = 10 ** 9
    c.max_len = 100
    c.call(c.prepare())
    torch.cuda.synchronize()
    c.check()
    c.d["lens"][1] = -3
    c.call(c.prepare())
    torch.cuda.synchronize()
    assert bool((c.d["out"][1, :, :64] == 0).all()) and bool((c.d["lse"][1] == -float("inf")).all())


@pytest.mark.parametrize("mode,dims,heads,kv,lens,rows", [
    ("tree", LATENT, 16, 1, [9000, 11, 4000], [4, 1, 8]),
    ("tree", D128, 8, 1, [20_000, 300], [1, 1]),
    ("tree", D64, 8, 8, [5000], [33]),
    ("prompt", D128, 8, 2, [6000, 900], [300, 900]),
    ("prompt", LATENT, 16, 1, [5000], [100]),
    ("prompt", D64, 4, 4, [3000], [700])])
def test_long(mode, dims, heads, kv, lens, rows):
    say("case: long", mode, dims, lens)
    masks = sum((chain(T) for T in rows), []) if mode == "tree" else None
    c = AttnCase(mode, lens, rows, heads, kv, dims, block=64, masks=masks, seed=12)
    c.run().check(sample=60)


def test_large_scores():
    """Scores in the hundreds: the running maximum rises from tile to tile, weights underflow."""
    for dims, heads in ((D128, 4), (LATENT, 16)):
        say("case: large scores", dims)
        c = AttnCase("tree", [700], [1], heads, 1, dims, masks=[1], seed=13, scale=2.0)
        c.pool *= torch.linspace(0.1, 4, c.pool.shape[0])[:, None].to(c.pool.dtype)
        c.pool.view(c.pool_blocks, 16, -1)[int(c.tables[0, 43])][12:] = float("nan")
        c.run().check()


def test_same_results_twice_and_on_another_stream():
    say("case: twice, and on another stream")
    c = AttnCase("tree", [3000, 70], [4, 4], 16, 1, LATENT, masks=chain(4) * 2, seed=14).run()
    out, lse = c.d["out"].clone(), c.d["lse"].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.d["out"].fill_(7)
        c.call()
    s.synchronize()
    assert torch.equal(out, c.d["out"]) and torch.equal(lse, c.d["lse"])


def test_captured_and_replayed_with_new_lengths():
    """A graph follows the lengths, queries and tables of each replay."""
    say("case: graph")
    c = AttnCase("tree", [900, 500, 64], [4, 2, 1], 16, 1, LATENT, masks=chain(4) + chain(2) + chain(1), seed=15).place()
    a = c.prepare()
    c.call(a)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.call(a)
    full = list(c.lens)
    for lens in (full, [100, 500, 64], [4, 2, 1], full):
        c.lens = lens
        c.d["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        c.d["q"].mul_(-1)
        c.q_wide = -c.q_wide
        c.d["out"].fill_(7)
        c.d["lse"].fill_(7)
        g.replay()
        torch.cuda.synchronize()
        c.check(sample=60)
        (torch.ones(1000, device="cuda") * 2).sum().item()


@pytest.mark.parametrize("dims,heads,kv,dtype", [(LATENT, 16, 1, "bf16"), (D128, 4, 2, "f16"), (D64, 2, 2, "bf16")])
@pytest.mark.parametrize("n", [64, 65, 130, 700])
def test_many_requests(dims, heads, kv, dtype, n):
    """Batches around and past a wave's 64 requests, some without rows or tokens."""
    rng = np.random.default_rng(n)
    rows = rng.integers(0, 4, n)
    lens = [int(r) + int(rng.integers(0, 400)) * int(rng.random() < 0.8) for r in rows]
    say("case: many requests", dims, n)
    c = AttnCase("tree", lens, rows, heads, kv, dims, dtype, block=32, masks=sum((chain(int(r)) for r in rows), []), seed=n)
    c.run().check(sample=200)


@pytest.mark.parametrize("dims,heads,kv", [(LATENT, 16, 1), (D128, 8, 1)])
def test_one_long_request_among_short_ones(dims, heads, kv):
    """Parts of one length for all: the long one's are many."""
    lens = [50] * 30 + [20_000] + [130] * 40
    say("case: one long request", dims)
    c = AttnCase("tree", lens, [1] * 71, heads, kv, dims, block=64, masks=[1] * 71, seed=16).run()
    c.check(sample=80)
    c2 = AttnCase("tree", lens + [3] * 60, [1] * 131, heads, kv, dims, block=64, masks=[1] * 131, seed=16).run()
    c2.check(sample=80)


def test_more_tiles_than_the_gpu_holds_at_once():
    """300 tiles of 128 latent heads, cut twice; the same with documents, left whole."""
    say("case: 300 latent tiles")
    c = AttnCase("prompt", [12_000], [300], 128, 1, LATENT, block=64, seed=17)
    c.run().check(sample=24)
    c.documents = [5000 + i for i in range(300)]
    c.run().check(sample=24)


def test_two_streams_with_workspaces_of_their_own():
    say("case: two streams")
    a = AttnCase("tree", [5000, 900], [4, 2], 16, 1, LATENT, masks=chain(4) + chain(2), seed=18).place()
    b = AttnCase("prompt", [4000], [50], 8, 2, D128, seed=19).place()
    args = a.prepare(), b.prepare()
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        for c, x, s in zip((a, b), args, streams):
            with torch.cuda.stream(s):
                c.call(x)
    torch.cuda.synchronize()
    a.check(sample=40)
    b.check(sample=40)


def test_two_graphs_share_a_workspace():
    """One after the other, with eager calls on the same workspace between."""
    say("case: two graphs, one workspace")
    a = AttnCase("tree", [5000, 900], [4, 2], 16, 1, LATENT, masks=chain(4) + chain(2), seed=20).place()
    b = AttnCase("tree", [7000], [1], 16, 1, LATENT, masks=[1], seed=21).place()
    xa, xb = a.prepare(), b.prepare()
    big = max((xa, xb), key=lambda x: x.workspace_bytes)
    for x in (xa, xb):
        x.workspace, x.workspace_bytes = big.workspace, big.workspace_bytes
    a.call(xa), b.call(xb)
    torch.cuda.synchronize()
    graphs = []
    for c, x in ((a, xa), (b, xb)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.call(x)
        graphs.append(g)
    for _ in range(3):
        for c, x, g, other, y in ((a, xa, graphs[0], b, xb), (b, xb, graphs[1], a, xa)):
            c.d["out"].fill_(7)
            c.d["lse"].fill_(7)
            g.replay()
            other.call(y)
            torch.cuda.synchronize()
            c.check(sample=20)


@pytest.mark.parametrize("dims,heads,kv", [(LATENT, 16, 1), (D128, 4, 2)])
def test_blocks_past_32_bits(dims, heads, kv):
    """Records that lie behind 2^32 bytes of their pool."""
    say("case: blocks past 32 bits", dims)
    c = AttnCase("tree", [700, 40], [4, 1], heads, kv, dims, masks=chain(4) + [1], seed=22).place()
    far = (1 << 32) // (c.block * 2 * c.values) + 1
    pool = torch.zeros((far + c.pool_blocks) * c.block, c.values, dtype=c.dtype, device="cuda")
    pool[far * c.block:] = c.d["pool"]
    c.d["pool"] = pool
    c.d["tables"] = torch.where(c.d["tables"] >= 0, c.d["tables"] + far, c.d["tables"])
    c.call(c.prepare(pool_blocks=far + c.pool_blocks))
    torch.cuda.synchronize()
    c.check(sample=60)
