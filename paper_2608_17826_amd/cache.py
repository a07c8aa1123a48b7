"""The paged cache around a restore, over the C ABI, with torch as the memory plumbing.

A :class:`PagedCache` holds what an engine keeps for a context's allocator
groups: the pools of every tensor, valid bytes, free block ids and the batch's
block tables.  It lays blocks out from request lengths on the GPU, gives the
destinations that a restore binds, appends new tokens' records and runs
attention over what is cached.  All device work runs inside libbsr.so on the
stream that is current where a method is called; no method waits for the GPU.
Append and attention may be captured into a graph; extend and release keep
their books on the host and may not.

Shapes and types of tensors are checked here, everything else by the library.
"""

from __future__ import annotations

from dataclasses import dataclass
from typing import Dict, List, Optional, Sequence, Tuple

import torch

from . import bsr

_TYPES = {torch.bfloat16: bsr.BSR_TYPE_BF16, torch.float16: bsr.BSR_TYPE_F16, torch.float32: bsr.BSR_TYPE_F32}


@dataclass
class Batch:
    """New tokens of a batch, as :meth:`PagedCache.extend` laid them out (device tensors)."""

    starts: torch.Tensor         # int32 [n_requests + 1]: first row of each request
    lens: torch.Tensor           # int32 [n_requests]: tokens in the cache, the new ones included
    slots: List[torch.Tensor]    # per group, int64 [n_slots]: block * block_tokens + position, -1 behind the last row
    result: torch.Tensor         # int32 [1 + n_groups]: requests admitted, blocks taken per group


def _check(ok: bool, what: str) -> None:
    if not ok:
        raise bsr.BsrError(bsr.BSR_E_ARG, what)


def _check_no_grad(*tensors: Optional[torch.Tensor]) -> None:
    _check(not (torch.is_grad_enabled() and any(x is not None and x.requires_grad for x in tensors)),
           "append and attention have no backward pass: detach the tensors, or call under torch.no_grad()")


class PagedCache:
    """Pools and block tables of a batch of up to ``max_requests`` requests of ``max_tokens`` tokens.

    ``pools[g][t]``: uint8 tensor of tensor t of group g, [pool_blocks, block
    bytes].  ``free[g]``: int32 ids of the group's free blocks, all of them by
    default.  The cache takes blocks from the front of ``free`` and puts them
    back behind the others: at :meth:`release`, and where :meth:`extend` is given fewer
    tokens than a row's blocks were laid out for (drafted ones that were rejected).
    ``held[g][row]``: how many blocks of group g a table row holds; a program
    that moves rows of ``tables`` moves these with them.  ``types[g, t]``: what
    :meth:`append` has written into tensor t of group g, bfloat16 or float16; only
    that is appended to it or read as such from then on.
    """

    def __init__(self, ctx: bsr.Ctx, pools: Sequence[Sequence[torch.Tensor]], max_requests: int, max_tokens: int,
                 free: Optional[Sequence[torch.Tensor]] = None):
        L = ctx.layout
        _check(len(pools) == L.n_groups, "pools of every group of the layout")
        _check(0 < max_requests <= bsr.BSR_MAX_TABLE_REQUESTS and max_tokens > 0, "max_requests or max_tokens out of range")
        self.ctx, self.pools, self.max_requests = ctx, [list(p) for p in pools], max_requests
        self.device = pools[0][0].device
        self.groups = [L.groups[g] for g in range(L.n_groups)]
        self.pool_blocks, self.bases, self.valid, self.tables, self.free, self.taken = [], [], [], [], [], []
        self.held = [[0] * max_requests for _ in self.groups]
        self.types: Dict[Tuple[int, int], torch.dtype] = {}
        self._valid = []       # valid, and a byte more for block ids outside the pool
        for g, (d, ts) in enumerate(zip(self.groups, self.pools)):
            _check(len(ts) == d.n_tensors, f"group {g} has {d.n_tensors} tensors")
            n = ts[0].shape[0]
            for t in ts:
                _check(t.dtype == torch.uint8 and t.device == self.device and t.is_contiguous() and
                       tuple(t.shape) == (n, d.block_tokens * d.record_bytes),
                       f"group {g}: a pool is a contiguous uint8 [pool_blocks, {d.block_tokens * d.record_bytes}] tensor")
            self.pool_blocks.append(n)
            self.bases.append(torch.tensor([t.data_ptr() for t in ts], dtype=torch.int64, device=self.device))
            self._valid.append(torch.zeros(n + 1, dtype=torch.uint8, device=self.device))
            self.valid.append(self._valid[g][:n])
            self.tables.append(torch.full((max_requests, -(-max_tokens // d.block_tokens)), -1, dtype=torch.int32,
                                          device=self.device))
            ids = torch.arange(n, dtype=torch.int32, device=self.device) if free is None else free[g]
            _check(ids.dtype == torch.int32 and ids.dim() == 1 and ids.device == self.device, f"group {g}: free ids are int32")
            self.free.append(ids.contiguous())
            self.taken.append(0)   # of the front of free

    def _stream(self) -> int:
        return torch.cuda.current_stream(self.device).cuda_stream

    def blocks(self, g: int, tokens: int) -> int:
        return -(-tokens // self.groups[g].block_tokens)

    def _check_row(self, row: int) -> None:
        _check(0 <= row < self.max_requests, f"table row {row} of {self.max_requests}")

    # ---- block tables --------------------------------------------------------------
    def _give_back(self, g: int, ids: Sequence[torch.Tensor]) -> None:
        """Block ids behind the free ones; they read as not valid until a restore commits into them."""
        ids = torch.cat(list(ids))
        n = self.pool_blocks[g]
        self._valid[g].index_fill_(0, torch.where((ids >= 0) & (ids < n), ids, n).long(), 0)
        self.free[g] = torch.cat([self.free[g][self.taken[g]:], ids])
        self.taken[g] = 0

    def extend(self, cached: Sequence[int], added: Sequence[int], n_slots: Optional[int] = None) -> Batch:
        """Blocks and slots for ``added[r]`` more tokens of request r (table row r), which has ``cached[r]``.

        A row that gets tokens first gives back the blocks that it holds behind
        the cached ones'; a row that gets none is left alone.  Raises where a row
        does not hold its cached tokens' blocks, or the free blocks or a table have no room
        for all of them, before anything is enqueued.
        """
        n = len(cached)
        _check(n <= self.max_requests and len(added) == n and all(c >= 0 and a >= 0 for c, a in zip(cached, added)),
               "lengths of up to max_requests requests, none negative")
        n_slots = sum(added) if n_slots is None else n_slots
        _check(sum(added) <= n_slots < 1 << 31, "n_slots is fewer than the new tokens, or not below 2^31")
        rows = [r for r in range(n) if added[r]]
        at, to = [cached[r] for r in rows], [cached[r] + added[r] for r in rows]
        take, back, then = [], [], []
        for g, d in enumerate(self.groups):
            B, held = d.block_tokens, [self.held[g][r] for r in rows]
            have, need = [-(-t // B) for t in at], [-(-t // B) for t in to]
            short = next((r for r, h, k in zip(rows, have, held) if h > k), None)
            if short is not None:
                raise bsr.BsrError(bsr.BSR_E_ARG, f"group {g}: table row {short} holds {self.held[g][short]} blocks, "
                                   f"fewer than {cached[short]} tokens take")
            if max(need, default=0) > self.tables[g].shape[1]:
                raise bsr.BsrError(bsr.BSR_E_ARG, f"group {g}: a request outgrows its table")
            take.append(sum(need) - sum(have))
            left = self.free[g].numel() - self.taken[g] + sum(held) - sum(have)
            if take[g] > left:
                raise bsr.BsrError(bsr.BSR_E_NOMEM, f"group {g}: {take[g]} blocks wanted, {left} free")
            back.append([x for x in zip(rows, have, held) if x[1] < x[2]] if sum(held) > sum(have) else [])
            then.append(need)
        for g, rests in enumerate(back):
            if rests:
                self._give_back(g, [self.tables[g][r, h:k] for r, h, k in rests])
                for r, h, _ in rests:
                    self.held[g][r] = h
        i32 = dict(dtype=torch.int32, device=self.device)
        lengths = torch.tensor([list(cached), list(added)], dtype=torch.int32, pin_memory=True).to(self.device, non_blocking=True)
        b = Batch(torch.empty(n + 1, **i32), torch.empty(n, **i32),
                  [torch.empty(n_slots, dtype=torch.int64, device=self.device) for _ in self.groups],
                  torch.empty(1 + len(self.groups), **i32))
        groups = [bsr.table_group(f.data_ptr() + 4 * t, f.numel() - t, tab.data_ptr(), tab.shape[1], s.data_ptr())
                  for f, t, tab, s in zip(self.free, self.taken, self.tables, b.slots)]
        bsr.bsr_tables_build(self.ctx, bsr.tables_args(n, lengths.data_ptr(), lengths.data_ptr() + 4 * n, groups, n_slots,
                                                       b.starts.data_ptr(), b.lens.data_ptr(), b.result.data_ptr()),
                             self._stream())
        self.taken = [t + k for t, k in zip(self.taken, take)]
        for held, need in zip(self.held, then):
            for r, k in zip(rows, need):
                held[r] = k
        return b

    def release(self, row: int, tokens: int) -> None:
        """The request of table row ``row``, of ``tokens`` tokens, is over: all blocks of the row go behind the free ones.

        (Those of drafted tokens that it did not keep among them.)  Raises where
        the row holds fewer blocks than its tokens take, so where it was released before.
        """
        self._check_row(row)
        _check(tokens >= 0 and all(self.blocks(g, tokens) <= held[row] for g, held in enumerate(self.held)),
               f"table row {row} does not hold {tokens} tokens")
        for g, held in enumerate(self.held):
            if held[row]:
                self._give_back(g, [self.tables[g][row, :held[row]]])
                held[row] = 0

    def dsts(self, row: int) -> List[bsr.bsr_group_dst]:
        """Destinations of a restore into table row ``row`` (for bsr_request_bind)."""
        self._check_row(row)
        return [bsr.group_dst(tab.data_ptr() + 4 * row * tab.shape[1], base.data_ptr(), v.data_ptr(), tab.shape[1], n)
                for tab, base, v, n in zip(self.tables, self.bases, self.valid, self.pool_blocks)]

    def _check_type(self, group: int, tensor: int, dtype: torch.dtype) -> Tuple[int, int]:
        key = group, tensor % len(self.pools[group])
        _check(self.types.get(key, dtype) == dtype, f"group {group}: tensor {tensor} holds {self.types.get(key)}")
        return key

    # ---- append -----------------------------------------------------------------------
    def append(self, group: int, tensor: int, slots: torch.Tensor, sources: Sequence[torch.Tensor],
               dtype: Optional[torch.dtype] = None) -> None:
        """Rows of ``sources`` (one or two [n, width] tensors, side by side a record) into their slots.

        ``dtype``: of a CONTIG group's values, bfloat16 by default.
        """
        x = sources[0]
        n = slots.numel()
        _check(slots.dtype == torch.int64 and slots.is_contiguous() and slots.device == self.device, "slots are int64")
        for s in sources:
            _check(s.dim() == 2 and s.shape[0] == n and s.dtype == x.dtype and s.device == self.device and
                   (s.stride(1) == 1 or s.shape[1] == 1), "sources are [n, width] rows of one type")
        _check(x.dtype in _TYPES, "sources are bfloat16, float16 or float32")
        _check_no_grad(*sources)
        planar = self.groups[group].kind == bsr.BSR_KIND_PLANAR
        dtype = torch.bfloat16 if dtype is None else dtype
        _check(planar or dtype in (torch.bfloat16, torch.float16), "a cache holds bfloat16 or float16")
        key = None if planar else self._check_type(group, tensor, dtype)
        a = bsr.append_args(group, n, slots.data_ptr(), self.pools[group][tensor].data_ptr(), self.pool_blocks[group],
                            _TYPES[x.dtype], bsr.BSR_TYPE_E4M3_SCALED if planar else _TYPES[dtype],
                            [(s.data_ptr(), s.shape[1], max(s.stride(0), s.shape[1]) if n < 2 else s.stride(0)) for s in sources])
        bsr.bsr_cache_append(self.ctx, a, self._stream())
        if key is not None:
            self.types[key] = dtype

    # ---- attention -----------------------------------------------------------------------
    def _attend(self, call, group: int, tensors: Tuple[int, int], q: torch.Tensor, batch: Batch, dims, kv_heads: int,
                max_len: int, offsets: Tuple[int, int], scale: Optional[float], softcap: float, window: int, arrays,
                out, lse: bool):
        _check(q.dim() == 3 and q.dtype in (torch.bfloat16, torch.float16) and q.device == self.device and
               q.stride(2) == 1 and q.shape[2] == dims[0], f"q is [tokens, heads, {dims[0]}] of bfloat16 or float16")
        _check_no_grad(q, out, *(x for x, _, _ in arrays.values()))
        _check(all(0 <= x < 1 << 32 for x in (group, kv_heads, max_len, window, *offsets)),
               "group, kv_heads, max_len, window and offsets are of 32 bits")
        n, heads, _ = q.shape
        if out is None:
            out = torch.empty(n, heads, dims[1], dtype=q.dtype, device=self.device)
        _check(tuple(out.shape) == (n, heads, dims[1]) and out.dtype == q.dtype and out.device == self.device and
               out.stride(2) == 1, f"out is [tokens, heads, {dims[1]}] of q's type")
        for x, size in ((batch.starts, batch.lens.numel() + 1), (batch.lens, batch.lens.numel())):
            _check(x.dtype == torch.int32 and x.is_contiguous() and x.device == self.device and x.numel() == size,
                   "a batch's starts and lens are int32 [n_requests + 1] and [n_requests]")
        _check(batch.lens.numel() <= self.max_requests, "the batch has more requests than the tables have rows")
        sums = torch.empty(n, heads, dtype=torch.float32, device=self.device) if lse else None
        for x, dtype, size in arrays.values():
            _check(x is None or (x.dtype == dtype and x.is_contiguous() and x.device == self.device and x.numel() == size),
                   "a mask's array has another type or size")
        for t in tensors:
            self._check_type(group, t, q.dtype)
        tab = self.tables[group]
        ptr = lambda x: 0 if x is None else x.data_ptr()  # noqa: E731
        a = bsr.attn_args(group=group, dtype=_TYPES[q.dtype], n_requests=batch.lens.numel(), n_tokens=n, n_heads=heads,
                          n_kv_heads=kv_heads, k_dim=dims[0], v_dim=dims[1], q=q.data_ptr(),
                          q_strides=(q.stride(0), q.stride(1)), out=out.data_ptr(),
                          out_strides=(out.stride(0), out.stride(1)), lse=ptr(sums),
                          k_pool=self.pools[group][tensors[0]].data_ptr(), v_pool=self.pools[group][tensors[1]].data_ptr(),
                          k_offset=offsets[0], v_offset=offsets[1], pool_blocks=self.pool_blocks[group],
                          tables=tab.data_ptr(), table_stride=tab.shape[1], starts=batch.starts.data_ptr(),
                          lens=batch.lens.data_ptr(), max_len=max_len,
                          scale=dims[0] ** -0.5 if scale is None else scale, softcap=softcap, window=window,
                          **{k: ptr(x) for k, (x, _, _) in arrays.items()})
        if "tree" in arrays:
            a.tree_words = arrays["tree"][0].shape[1]
        # a workspace of the call's own: torch gives its memory to later work of the same stream alone, and a graph
        # that captures the call keeps it
        size = bsr.bsr_attn_workspace_bytes(self.ctx, a)
        workspace = torch.empty(size, dtype=torch.uint8, device=self.device)
        a.workspace, a.workspace_bytes = workspace.data_ptr(), size
        call(self.ctx, a, self._stream())
        return (out, sums) if lse else out

    def attend_tree(self, group: int, tensors: Tuple[int, int], q: torch.Tensor, batch: Batch, tree: torch.Tensor,
                    dims: Tuple[int, int], kv_heads: int, max_len: int, offsets: Tuple[int, int] = (0, 0),
                    scale: Optional[float] = None, softcap: float = 0.0, window: int = 0,
                    out: Optional[torch.Tensor] = None, lse: bool = False):
        """Attention of drafted trees, or of single tokens; ``tree``: int64 [tokens, words] masks.

        ``tensors``: the group's tensors that hold K and V, at ``offsets``
        bytes of their records.  ``scale``: k_dim ** -0.5 by default; a model with
        latent records scales by the width that its heads had before, not by 576,
        and passes that.  Rows behind the batch's last are not written: of an output
        that the call makes they hold anything.  See bsr_attend_tree.
        """
        _check(tree.dim() == 2 and 1 <= tree.shape[1] <= bsr.BSR_MAX_TREE_WORDS, "tree is [tokens, words]")
        return self._attend(bsr.bsr_attend_tree, group, tensors, q, batch, dims, kv_heads, max_len, offsets, scale,
                            softcap, window, {"tree": (tree, torch.int64, q.shape[0] * tree.shape[1])}, out, lse)

    def attend_prompt(self, group: int, tensors: Tuple[int, int], q: torch.Tensor, batch: Batch, dims: Tuple[int, int],
                      kv_heads: int, max_len: int, offsets: Tuple[int, int] = (0, 0), scale: Optional[float] = None,
                      softcap: float = 0.0, window: int = 0, slopes: Optional[torch.Tensor] = None,
                      prefix: Optional[torch.Tensor] = None, documents: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None, lse: bool = False):
        """Attention of prompt tokens, with a bias by distance (``slopes``, fp32 per head), bidirectional
        prefixes (int32 per request) and packed documents (int32 first position per token).

        A prefix that reaches past a row's document shows the row later ones' keys
        too.  ``tensors``, ``offsets`` and ``scale`` as in :meth:`attend_tree`.  See bsr_attend_prompt.
        """
        arrays = {"slopes": (slopes, torch.float32, q.shape[1]), "prefix": (prefix, torch.int32, batch.lens.numel()),
                  "documents": (documents, torch.int32, q.shape[0])}
        return self._attend(bsr.bsr_attend_prompt, group, tensors, q, batch, dims, kv_heads, max_len, offsets, scale,
                            softcap, window, arrays, out, lse)
