"""The paged cache's operators refuse what they cannot run (CPU).

A host-only context is enough: arguments are checked before the device, so a
call with good arguments gets as far as BSR_E_DEVICE.  Addresses are made up;
nothing is read through them.
"""

import numpy as np
import pytest

from oracle import cache as oracle_cache
from paper_2608_17826_amd import bsr

C, P = bsr.BSR_KIND_CONTIG, bsr.BSR_KIND_PLANAR
A = 1 << 20  # an aligned address


@pytest.fixture(scope="module")
def ctx():
    # latent records; index keys; K and V of one head of 128; 2 KV heads of 64; odd records
    c = bsr.bsr_ctx_create(bsr.make_layout(256, [(64, 1, 1152, C, 0), (128, 1, 132, P, 128), (32, 1, 512, C, 0),
                                                 (16, 1, 512, C, 0), (16, 1, 36, C, 0), (16, 1, 40, P, 32)]), 1,
                           hip_device=-1)
    yield c
    bsr.bsr_ctx_destroy(c)


def code(call, *args):
    with pytest.raises(bsr.BsrError) as e:
        call(*args)
    return e.value.code


def attn(mode="tree", **other):
    f = dict(group=0, dtype=bsr.BSR_TYPE_BF16, n_requests=2, n_tokens=2, n_heads=16, n_kv_heads=1, k_dim=576,
             v_dim=512, q=A, q_strides=(16 * 576, 576), out=A, out_strides=(16 * 512, 512), lse=A, k_pool=A, v_pool=A,
             k_offset=0, v_offset=0, pool_blocks=10, tables=A, table_stride=4, starts=A, lens=A, max_len=64,
             scale=0.1, softcap=0.0, window=0, workspace=A, workspace_bytes=1 << 40)
    if mode == "tree":
        f.update(tree=A, tree_words=1)
    f.update(other)
    return bsr.attn_args(**f)


HEADS = dict(group=2, n_heads=8, k_dim=128, v_dim=128, v_offset=256, q_strides=(1024, 128), out_strides=(1024, 128))


def test_good_arguments_reach_the_device(ctx):
    for mode, call in (("tree", bsr.bsr_attend_tree), ("prompt", bsr.bsr_attend_prompt)):
        assert code(call, ctx, attn(mode), 0) == bsr.BSR_E_DEVICE
        assert code(call, ctx, attn(mode, **HEADS), 0) == bsr.BSR_E_DEVICE
        assert code(call, ctx, attn(mode, n_tokens=0, q=0, out=0), 0) == bsr.BSR_E_DEVICE
        assert code(call, ctx, attn(mode, dtype=bsr.BSR_TYPE_F16, window=64), 0) == bsr.BSR_E_DEVICE
    assert code(bsr.bsr_attend_prompt, ctx, attn("prompt", slopes=A, prefix=A, documents=A), 0) == bsr.BSR_E_DEVICE


@pytest.mark.parametrize("other", [
    dict(group=6), dict(group=1), dict(group=4), dict(dtype=bsr.BSR_TYPE_F32), dict(k_dim=576, v_dim=576),
    dict(k_dim=512, v_dim=512), dict(k_dim=96, v_dim=96), dict(k_dim=128, v_dim=64), dict(n_heads=0), dict(n_kv_heads=0),
    dict(n_kv_heads=2), dict(v_pool=A + 64), dict(v_offset=16), dict(k_offset=8), dict(k_offset=16, v_offset=16),
    dict(n_requests=1 << 20), dict(n_tokens=1 << 24), dict(max_len=1 << 30), dict(window=1 << 30), dict(scale=0.0),
    dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(softcap=-1.0),
    dict(softcap=float("nan")), dict(softcap=float("inf")), dict(softcap=1e-44), dict(q_strides=(100, 576)),
    dict(q_strides=(9216, 577)), dict(out_strides=(9217, 512)), dict(out_strides=(9216, 500)), dict(reserved=1),
    dict(q=0), dict(out=0), dict(k_pool=0, v_pool=0), dict(tables=0), dict(starts=0), dict(lens=0), dict(q=A + 8),
    dict(out=A + 2), dict(k_pool=A + 8, v_pool=A + 8), dict(tables=A + 2), dict(lse=A + 1), dict(starts=A + 3),
    dict(pool_blocks=0), dict(pool_blocks=1 << 31), dict(table_stride=0),
    dict(max_len=1000, table_stride=100, workspace=0), dict(max_len=1000, table_stride=100, workspace_bytes=100),
    dict(max_len=1000, table_stride=100, workspace=A + 4),
    dict(HEADS, group=3, n_kv_heads=2, v_offset=512), dict(HEADS, n_kv_heads=2), dict(HEADS, v_offset=272),
    dict(HEADS, n_heads=4097, n_kv_heads=1)])
def test_attention_refuses(ctx, other):
    assert code(bsr.bsr_attend_tree, ctx, attn(**other), 0) == bsr.BSR_E_ARG
    assert code(bsr.bsr_attend_prompt, ctx, attn("prompt", **other), 0) == bsr.BSR_E_ARG
    assert bsr.bsr_last_error()


def test_attention_refuses_the_other_calls_masks(ctx):
    for other in (dict(slopes=A), dict(prefix=A), dict(documents=A), dict(tree=0), dict(tree_words=0),
                  dict(tree_words=17), dict(tree=A + 4), dict(window=63), dict(window=127, tree_words=2)):
        assert code(bsr.bsr_attend_tree, ctx, attn(**other), 0) == bsr.BSR_E_ARG
    for other in (dict(tree=A), dict(tree_words=1), dict(slopes=A + 2), dict(prefix=A + 1), dict(documents=A + 2)):
        assert code(bsr.bsr_attend_prompt, ctx, attn("prompt", **other), 0) == bsr.BSR_E_ARG


def test_workspace_bytes(ctx):
    assert bsr.bsr_attn_workspace_bytes(ctx, attn(max_len=64)) == 0           # nothing is ever cut
    n = bsr.bsr_attn_workspace_bytes(ctx, attn(max_len=1 << 20))
    assert n == bsr.bsr_attn_workspace_bytes(ctx, attn(max_len=1 << 20, q=0, tables=0, workspace=0))  # sizes alone
    assert 0 < n <= 2 * 256 * 128 * 514 * 4
    assert bsr.bsr_attn_workspace_bytes(ctx, attn(n_requests=0, n_tokens=0)) == 0
    assert code(bsr.bsr_attn_workspace_bytes, ctx, attn(scale=0.0)) == bsr.BSR_E_ARG


@pytest.mark.parametrize("n_requests", [0, 1, 2])
@pytest.mark.parametrize("heads", [1, 16, 33, 128, 300])
def test_workspace_bytes_without_rows(ctx, heads, n_requests):
    """More heads than the smallest tile has rows, and no rows at all."""
    assert bsr.bsr_attn_workspace_bytes(ctx, attn(n_heads=heads, n_requests=n_requests, n_tokens=0, max_len=1 << 20)) == 0
    assert code(bsr.bsr_attend_tree, ctx, attn(n_heads=heads, n_requests=n_requests, n_tokens=0), 0) == bsr.BSR_E_DEVICE


def append(**other):
    f = dict(group=0, n_tokens=3, slots=A, pool=A, pool_blocks=4, src_type=bsr.BSR_TYPE_BF16,
             cache_type=bsr.BSR_TYPE_BF16, sources=[(A, 512, 512), (A, 64, 64)])
    f.update(other)
    return bsr.append_args(**f)


PLANAR = dict(group=1, cache_type=bsr.BSR_TYPE_E4M3_SCALED, sources=[(A, 128, 128)])


def test_append_reaches_the_device(ctx):
    for other in ({}, PLANAR, dict(n_tokens=0, slots=0, pool=0, sources=[(0, 576, 576)]), dict(sources=[(A + 2, 576, 577)]),
                  dict(src_type=bsr.BSR_TYPE_F32, cache_type=bsr.BSR_TYPE_F16, sources=[(A + 4, 576, 600)])):
        assert code(bsr.bsr_cache_append, ctx, append(**other), 0) == bsr.BSR_E_DEVICE


@pytest.mark.parametrize("other", [
    dict(group=6), dict(src_type=3), dict(cache_type=bsr.BSR_TYPE_F32), dict(cache_type=bsr.BSR_TYPE_E4M3_SCALED),
    dict(sources=[]), dict(sources=[(A, 512, 512)]), dict(sources=[(A, 512, 512), (A, 65, 65)]),
    dict(sources=[(A, 576, 576), (A, 0, 0)]), dict(sources=[(A, 192, 192)] * 3), dict(sources=[(0, 576, 576)]),
    dict(sources=[(A + 1, 576, 576)]), dict(sources=[(A, 576, 575)]), dict(sources=[(A, 576, -576)]), dict(slots=0),
    dict(slots=A + 4), dict(pool=0), dict(pool=A + 8), dict(n_tokens=1 << 24), dict(n_tokens=10_000_000, sources=[(A + 2, 576, 576)]),
    dict(src_type=bsr.BSR_TYPE_F32, sources=[(A + 2, 576, 576)]),
    dict(PLANAR, cache_type=bsr.BSR_TYPE_BF16), dict(PLANAR, sources=[(A, 64, 64), (A, 64, 64)]),
    dict(PLANAR, group=5, sources=[(A, 32, 32)]), dict(PLANAR, sources=[(A, 132, 132)])])
def test_append_refuses(ctx, other):
    assert code(bsr.bsr_cache_append, ctx, append(**other), 0) == bsr.BSR_E_ARG


def tables(groups=None, **other):
    f = dict(n_requests=3, cached_ptr=A, added_ptr=A + 64, n_slots=10, starts_ptr=A + 128, lens_ptr=A + 256, result_ptr=A + 512)
    f.update(other)
    if groups is None:
        groups = [bsr.table_group(A, 5, A, 4, A)] * 6
    return bsr.tables_args(groups=groups, **f)


def test_tables_reach_the_device(ctx):
    ok = bsr.table_group(A, 5, A, 4, A)
    for a in (tables(), tables([ok] * 5 + [bsr.table_group(0, 0, 0, 0)]), tables(n_requests=bsr.BSR_MAX_TABLE_REQUESTS, cached_ptr=A + (1 << 20), added_ptr=A + (2 << 20), lens_ptr=A + (3 << 20)),
              tables(n_requests=0, cached_ptr=0, added_ptr=0, lens_ptr=0), tables([bsr.table_group(0, 0, A, 4)] * 6)):
        assert code(bsr.bsr_tables_build, ctx, a, 0) == bsr.BSR_E_DEVICE


@pytest.mark.parametrize("other", [
    dict(n_requests=4097), dict(n_slots=1 << 31), dict(cached_ptr=0), dict(added_ptr=0), dict(starts_ptr=0),
    dict(lens_ptr=0), dict(result_ptr=0), dict(cached_ptr=A + 2), dict(lens_ptr=A), dict(lens_ptr=A + 4),
    dict(lens_ptr=A + 72), dict(starts_ptr=A + 8), dict(starts_ptr=A + 60), dict(result_ptr=A + 513)])
def test_tables_refuse(ctx, other):
    assert code(bsr.bsr_tables_build, ctx, tables(**other), 0) == bsr.BSR_E_ARG


@pytest.mark.parametrize("group", [
    bsr.table_group(A, 5, 0, 4, A), bsr.table_group(A, 5, A, 0, A), bsr.table_group(0, 5, A, 4, A),
    bsr.table_group(A + 2, 5, A, 4, A), bsr.table_group(A, 5, A + 1, 4, A), bsr.table_group(A, 5, A, 4, A + 4),
    bsr.table_group(A, 1 << 31, A, 4, A)])
def test_tables_refuse_a_group(ctx, group):
    ok = bsr.table_group(A, 5, A, 4, A)
    assert code(bsr.bsr_tables_build, ctx, tables([ok] * 5 + [group]), 0) == bsr.BSR_E_ARG


def test_tables_want_every_group(ctx):
    assert code(bsr.bsr_tables_build, ctx, tables([bsr.table_group(A, 5, A, 4, A)] * 5), 0) == bsr.BSR_E_ARG


# ---- the oracle's own pins ----------------------------------------------------------
def test_oracle_tables_by_hand():
    g = [dict(block_tokens=4, free=np.array([9, 8, 7]), tables=np.full((3, 3), -1), slots=True)]
    g[0]["tables"][0, 0] = 5
    starts, lens, result, ((t, s),) = oracle_cache.tables_build([3, 0, 0], [2, 5, 1], 9, g)
    assert list(starts) == [0, 2, 7, 7] and list(lens) == [5, 5, 0] and list(result) == [2, 3]
    assert t.tolist() == [[5, 9, -1], [8, 7, -1], [-1, -1, -1]]
    assert s.tolist() == [23, 36, 32, 33, 34, 35, 28, -1, -1]


def test_oracle_attention_by_hand():
    see, p = oracle_cache.visible("tree", 5, 3, 2, mask=[0b101])
    assert see.tolist() == [True, True, True, False, True] and p == 3
    see, p = oracle_cache.visible("prompt", 6, 4, 1, window=2, prefix=5)
    assert see.tolist() == [False, False, True, True, True, False] and p == 3
    assert oracle_cache.visible("prompt", 6, 4, 1, document=4)[0].sum() == 0
    q, k, v = np.array([1.0, 0]), np.array([[0.0, 0], [np.log(3), 5]]), np.array([[4.0], [8.0]])
    o, l, a, d = oracle_cache.attend(q, k, v, np.array([True, True]), 1, 1.0)
    assert np.allclose(o, [7.0]) and np.isclose(l, np.log(4)) and np.allclose(a, [7.0]) and np.isclose(d, np.log(3))
    o, l, _, _ = oracle_cache.attend(q, k, v, np.array([True, True]), 1, 1.0, cap=1e9, slope=np.log(3))
    assert np.allclose(o, [4 * 0.1 + 8 * 0.9])
