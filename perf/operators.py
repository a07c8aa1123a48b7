"""Timed calls of the operators that an engine uses around a restore.

A case is a plain dict; "op" says which operator it calls:

  tables   block tables and slot maps of a batch, built from its requests'
           lengths (bsr_tables_build)
  append   new tokens' records written into their slots (bsr_cache_append)
  tree     attention of drafted token trees, or of single tokens, over the
           paged cache (bsr_attend_tree)
  prompt   attention of new prompt tokens over the paged cache, with document
           and prefix masks, a distance bias, a window, capped scores
           (bsr_attend_prompt)

A case's lengths, trees and documents come from its own "shape" number, its
values from the seed.  The cache layouts are this repository's: MLA latent
records of 576 values whose first 512 are the value, fp8 index keys with a
scale, and records of K and V side by side.
"""

import math
import random

import numpy as np
import torch

own = False

BF16, F16, F32 = "bf16", "f16", "f32"
TYPES = {BF16: torch.bfloat16, F16: torch.float16, F32: torch.float32}
# tokens per block of the 512K workload's four groups
MTP_BLOCKS = (64, 128, 32, 64)
FAR = 2 ** 31 - 1  # a document that no token of the request belongs to


def listed():
    return [
        # one decode step of a batch: 32 requests get a token each in all four groups
        _tables("tables-decode", 32, 30_000, 1, 1),
        # prompts of a full batch are admitted: some 256K new tokens behind nothing or a restored prefix
        _tables("tables-prompts", 64, 8192, 8192, 2),
        # a decode step's latent records, one layer
        _append("append-latent-decode", "latent", 64, BF16, 3),
        # a long prompt's latent records, one layer
        _append("append-latent-prompt", "latent", 32_768, BF16, 4),
        # a prompt's index keys, from fp32 projections to fp8 values and scales
        _append("append-index-8k", "index", 8200, F32, 5),
        # one token over a short prefix, the heads of one rank of eight: latency
        _tree("tree-latent-one", "latent", 1, 1000, 1, 16, 1, 6),
        # a batch with eight drafted nodes each behind ragged prefixes, the same heads
        _tree("tree-latent-batch", "latent", 16, 33_000, 8, 16, 1, 7),
        # four drafted nodes over the 512K workload's context, every head
        _tree("tree-latent-512k", "latent", 1, 524_288, 4, 128, 1, 8),
        # trees of up to 64 nodes over grouped heads, capped scores
        _tree("tree-heads-64", "kv128", 8, 9000, 64, 32, 8, 9, dtype=F16, cap=50.0),
        # a short turn behind a system prompt whose tokens see one another
        _prompt("prompt-turn", "kv128", 1, 1003, 37, 16, 2, 10, dtype=F16, prefix=True, cap=30.0),
        # packed documents with a bias by distance, nothing restored
        _prompt("prompt-documents", "kv64", 4, 0, 4096, 16, 4, 11, docs=True, slopes=True),
        # the tail of a 128K prompt of which all but 1,024 tokens were restored
        _prompt("prompt-tail-128k", "kv128", 1, 131_072, 1024, 16, 2, 12),
    ]


def _tables(name, requests, cached, added, shape):
    return {"name": name, "op": "tables", "requests": requests, "cached": cached, "added": added, "shape": shape}


def _append(name, layout, tokens, source, shape):
    return {"name": name, "op": "append", "layout": layout, "tokens": tokens, "source": source, "shape": shape}


def _tree(name, layout, requests, cached, nodes, heads, kv_heads, shape, dtype=BF16, cap=0.0, window=0, block=64):
    return {"name": name, "op": "tree", "layout": layout, "requests": requests, "cached": cached, "nodes": nodes,
            "heads": heads, "kv_heads": kv_heads, "shape": shape, "dtype": dtype, "cap": cap, "window": window,
            "block": block}


def _prompt(name, layout, requests, cached, added, heads, kv_heads, shape, dtype=BF16, cap=0.0, window=0, block=64,
            docs=False, prefix=False, slopes=False):
    return {"name": name, "op": "prompt", "layout": layout, "requests": requests, "cached": cached, "added": added,
            "heads": heads, "kv_heads": kv_heads, "shape": shape, "dtype": dtype, "cap": cap, "window": window,
            "block": block, "docs": docs, "prefix": prefix, "slopes": slopes}


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["tables", "append", "tree", "tree", "prompt", "prompt"])
    shape = rng.randrange(1000, 1_000_000)
    if op == "tables":
        requests = _log(rng, 1, 512)
        case = _tables("", requests, _log(rng, 1, 30_000), _log(rng, 1, max(2, 262_144 // requests)), shape)
    elif op == "append":
        layout = rng.choice(["latent", "index", "kv128", "kv64"])
        case = _append("", layout, _log(rng, 1, 32_768), rng.choice([BF16, F16, F32]), shape)
    else:
        layout = rng.choice(["latent", "latent", "kv128", "kv64"])
        kv_heads = 1 if layout == "latent" else rng.choice([1, 2, 4, 8])
        heads = rng.choice([16, 32, 128]) if layout == "latent" else kv_heads * rng.choice([1, 3, 4, 8])
        dtype = rng.choice([BF16, BF16, F16])
        cap = rng.choice([0.0, 0.0, 50.0])
        block = rng.choice([16, 32, 64, 128])
        window = rng.choice([0, 0, 128, 4096])
        if op == "tree":
            nodes = rng.choice([1, 1, 4, 8, 17, 64])
            requests = _log(rng, 1, 64)
            most = min(131_072, 2_000_000 // requests, 200_000_000 // (requests * nodes * heads))
            cached = _log(rng, 1, max(2, most))
            case = _tree("", layout, requests, cached, nodes, heads, kv_heads, shape, dtype, cap, window, block)
        else:
            requests = _log(rng, 1, 16)
            added = _log(rng, 1, 4096)
            most = 400_000_000 if layout == "latent" else 1_000_000_000  # score entries
            cached = min(65_536, most // (requests * added * heads)) - added
            cached = _log(rng, 1, cached) if cached > 1 else 0
            added = min(added, max(1, most // (requests * heads * (cached + added))))
            case = _prompt("", layout, requests, cached, added, heads, kv_heads, shape, dtype, cap, window, block,
                           docs=rng.random() < 0.4, prefix=rng.random() < 0.3, slopes=rng.random() < 0.4)
    del case["name"]
    return case


# ---- shapes, from the case alone ------------------------------------------------
LAYOUTS = {"latent": (576, 512), "kv128": (128, 128), "kv64": (64, 64)}


def _lengths(case):
    """(cached, added) of every request: the first has the largest, the others a share of it, down to nothing."""
    r = random.Random(case["shape"])
    most = case["nodes"] if case["op"] == "tree" else case["added"]
    cached, added = [case["cached"]], [most]
    for _ in range(case["requests"] - 1):
        cached.append(int(case["cached"] * r.random()))
        added.append(1 if most == 1 else int((most + 1) * r.random()))
    return cached, added


def _trees(case, added):
    """One mask of ancestors (and itself) per node, in the order of the nodes; a padded node sees none of them."""
    r = random.Random(case["shape"] + 1)
    masks = []
    for n in added:
        own_masks = []
        for i in range(n):
            parent = r.randrange(max(0, i - 8), i) if i else None
            m = (own_masks[parent] if i else 0) | 1 << i
            own_masks.append(m)
        if n > 8:
            own_masks[-1] = 0
        masks += own_masks
    return masks


def _documents(case, cached, added):
    """Where each new token's document begins in its request; the last token of a long request is padding."""
    r = random.Random(case["shape"] + 2)
    starts = []
    for c, a in zip(cached, added):
        at = 0
        own_starts = []
        left = r.randrange(1, 1200)
        for i in range(a):
            if left == 0:
                at, left = c + i, r.randrange(1, 1200)
            left -= 1
            own_starts.append(at)
        if a > 16:
            own_starts[-1] = FAR
        starts += own_starts
    return starts


def _prefixes(case, cached, added):
    r = random.Random(case["shape"] + 3)
    return [int((c + a) * r.random()) for c, a in zip(cached, added)]


def _ranges(case):
    """Per new token: (keys before the tree that it sees, first of them) for work()."""
    cached, added = _lengths(case)
    seen = read = 0
    if case["op"] == "tree":
        for c, a in zip(cached, added):
            w = min(c, case["window"]) if case["window"] else c
            seen += a * w
            read += w + a
        seen += sum(bin(m).count("1") for m in _trees(case, added))
        return seen, read, sum(added)
    docs = _documents(case, cached, added) if case["docs"] else [0] * sum(added)
    prefixes = _prefixes(case, cached, added) if case["prefix"] else [0] * len(added)
    k = 0
    for c, a, pre in zip(cached, added, prefixes):
        first = c + a
        for i in range(a):
            p = c + i
            lo = max(docs[k], p + 1 - case["window"] if case["window"] else 0)
            hi = max(p + 1, pre)
            if lo < hi:
                seen += hi - lo
                first = min(first, lo)
            k += 1
        read += c + a - first
    return seen, read, sum(added)


def work(case):
    if case["op"] == "tables":
        cached, added = _lengths(case)
        taken = sum(-(-(c + a) // b) - -(-c // b) for c, a in zip(cached, added) for b in MTP_BLOCKS)
        return {"bytes": 16 * case["requests"] + 8 * taken + 8 * len(MTP_BLOCKS) * sum(added), "flops": 0}
    if case["op"] == "append":
        size = {BF16: 2, F16: 2, F32: 4}[case["source"]]
        values = _values(case["layout"])
        record = 132 if case["layout"] == "index" else 2 * values
        return {"bytes": case["tokens"] * (8 + values * size + record), "flops": 0}
    dk, dv = LAYOUTS[case["layout"]]
    seen, read, rows = _ranges(case)
    record = dk if case["layout"] == "latent" else case["kv_heads"] * (dk + dv)
    return {"bytes": 2 * read * record + rows * case["heads"] * (2 * (dk + dv) + 4),
            "flops": 2 * (dk + dv) * seen * case["heads"]}


# ---- inputs -------------------------------------------------------------------------
class _State:
    pass


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = _State()
    s.case, s.op = case, case["op"]
    {"tables": _prepare_tables, "append": _prepare_append}.get(s.op, _prepare_attention)(s, case, gen)
    s.call = _framework_call(s) if own else None
    return s


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _prepare_tables(s, case, gen):
    cached, added = _lengths(case)
    s.cached, s.added = _ints(cached), _ints(added)
    s.n_slots = sum(added) + 5  # a padded batch: a few rows behind the last request
    s.free, s.tables, s.stride, s.slots = [], [], [], []
    for b in MTP_BLOCKS:
        most = max(-(-(c + a) // b) for c, a in zip(cached, added))
        held = sum(-(-c // b) for c in cached)
        taken = sum(-(-(c + a) // b) - -(-c // b) for c, a in zip(cached, added))
        ids = torch.randperm(held + taken + 100, generator=gen, device="cuda", dtype=torch.int32)
        table = torch.full((case["requests"], most), -1, dtype=torch.int32, device="cuda")
        blocks = _ints([-(-c // b) for c in cached])
        mine = torch.arange(most, device="cuda")[None, :] < blocks[:, None]
        table[mine] = ids[:held]
        s.tables.append(table)
        s.free.append(ids[held:].contiguous())
        s.slots.append(torch.zeros(s.n_slots, dtype=torch.int64, device="cuda"))
    s.starts = torch.zeros(case["requests"] + 1, dtype=torch.int32, device="cuda")
    s.lens = torch.zeros(case["requests"], dtype=torch.int32, device="cuda")
    s.result = torch.zeros(1 + len(MTP_BLOCKS), dtype=torch.int32, device="cuda")


def _values(layout):
    return {"latent": 576, "index": 128, "kv128": 256, "kv64": 128}[layout]


def _prepare_append(s, case, gen):
    n, values = case["tokens"], _values(case["layout"])
    s.planar = case["layout"] == "index"
    s.block = 128 if s.planar else 64
    s.record = 132 if s.planar else 2 * values
    s.type = TYPES[F16 if case["source"] == F16 and not s.planar else BF16]
    blocks = -(-n // s.block) + 2
    s.pool = torch.zeros((blocks, s.block * s.record), dtype=torch.uint8, device="cuda")
    # a prompt's tokens follow one another in blocks in any order; every 97th row is padding
    order = torch.randperm(blocks, generator=gen, device="cuda")
    t = torch.arange(n, device="cuda") + 3
    s.slots = order[t // s.block] * s.block + t % s.block
    s.slots[96::97] = -1
    width = {"latent": (512, 64), "index": (128,), "kv128": (128, 128), "kv64": (64, 64)}[case["layout"]]
    # projections come out beside others: rows wider than what is stored
    s.src = [(torch.randn(n, w + 64, generator=gen, device="cuda") * 2).to(TYPES[case["source"]])[:, :w] for w in width]


def _prepare_attention(s, case, gen):
    dk, dv = LAYOUTS[case["layout"]]
    latent = case["layout"] == "latent"
    s.dk, s.dv, s.latent = dk, dv, latent
    s.type = TYPES[case["dtype"]]
    s.cached_host, s.added_host = _lengths(case)
    s.block = case["block"]
    lens = [c + a for c, a in zip(s.cached_host, s.added_host)]
    s.max_len, s.max_added, rows = max(lens), max(s.added_host), sum(s.added_host)
    s.lens, s.added = _ints(lens), _ints(s.added_host)
    s.starts = _ints([0] + list(np.cumsum(s.added_host)))
    s.record_values = dk if latent else case["kv_heads"] * (dk + dv)
    need = [-(-n // s.block) for n in lens]
    s.pool_blocks = sum(need) + 3
    s.pool = torch.empty((s.pool_blocks * s.block, s.record_values), dtype=s.type, device="cuda")
    s.pool.normal_(generator=gen)
    ids = torch.randperm(s.pool_blocks, generator=gen, device="cuda", dtype=torch.int32)
    s.tables = torch.zeros((case["requests"], max(need)), dtype=torch.int32, device="cuda")
    mine = torch.arange(max(need), device="cuda")[None, :] < _ints(need)[:, None]
    s.tables[mine] = ids[:sum(need)]
    s.q = torch.randn(rows, case["heads"], dk, generator=gen, device="cuda").to(s.type)
    s.out = torch.zeros(rows, case["heads"], dv, dtype=s.type, device="cuda")
    s.lse = torch.zeros(rows, case["heads"], dtype=torch.float32, device="cuda")
    s.scale = (192 if latent else dk) ** -0.5  # a latent head stands for 128 + 64 dimensions
    s.tree = s.docs = s.prefix = s.slopes = None
    if case["op"] == "tree":
        s.tree = _ints([m - (1 << 64) if m >> 63 else m for m in _trees(case, s.added_host)], torch.int64)
    else:
        if case["docs"]:
            s.docs = _ints(_documents(case, s.cached_host, s.added_host))
        if case["prefix"]:
            s.prefix = _ints(_prefixes(case, s.cached_host, s.added_host))
        if case["slopes"]:
            h = case["heads"]
            s.slopes = _ints([2.0 ** (-8.0 * (i + 1) / h) for i in range(h)], torch.float32)


# ---- the framework's calls -------------------------------------------------------------
_contexts = {}


def _context(groups):
    """The program's one context for a layout."""
    from paper_2608_17826_amd import bsr
    if groups not in _contexts:
        _contexts[groups] = bsr.bsr_ctx_create(bsr.make_layout(256, groups), 1, hip_device=0)
    return _contexts[groups]


def _framework_call(s):
    """What a program keeps for an operator's calls: the context and the call's arguments."""
    from paper_2608_17826_amd import bsr
    stream = torch.cuda.current_stream().cuda_stream
    if s.op == "tables":
        ctx = _context(tuple((b, 1, 1152, bsr.BSR_KIND_CONTIG, 0) for b in MTP_BLOCKS))
        groups = [bsr.table_group(f.data_ptr(), f.numel(), t.data_ptr(), t.shape[1], m.data_ptr())
                  for f, t, m in zip(s.free, s.tables, s.slots)]
        args = bsr.tables_args(s.cached.numel(), s.cached.data_ptr(), s.added.data_ptr(), groups, s.n_slots,
                               s.starts.data_ptr(), s.lens.data_ptr(), s.result.data_ptr())
        return lambda: bsr.bsr_tables_build(ctx, args, stream)
    if s.op == "append":
        kind, split = (bsr.BSR_KIND_PLANAR, 128) if s.planar else (bsr.BSR_KIND_CONTIG, 0)
        ctx = _context(((s.block, 1, s.record, kind, split),))
        types = {torch.bfloat16: bsr.BSR_TYPE_BF16, torch.float16: bsr.BSR_TYPE_F16, torch.float32: bsr.BSR_TYPE_F32}
        args = bsr.append_args(group=0, n_tokens=s.slots.numel(), slots=s.slots.data_ptr(), pool=s.pool.data_ptr(),
                               pool_blocks=s.pool.shape[0], src_type=types[s.src[0].dtype],
                               cache_type=bsr.BSR_TYPE_E4M3_SCALED if s.planar else types[s.type],
                               sources=[(x.data_ptr(), x.shape[1], x.stride(0)) for x in s.src])
        return lambda: bsr.bsr_cache_append(ctx, args, stream)
    case = s.case
    ctx = _context(((s.block, 1, 2 * s.record_values, bsr.BSR_KIND_CONTIG, 0),))
    kv = 2 * case["kv_heads"] * s.dk
    args = bsr.attn_args(group=0, dtype=bsr.BSR_TYPE_BF16 if s.type == torch.bfloat16 else bsr.BSR_TYPE_F16,
                         n_requests=s.lens.numel(), n_tokens=s.q.shape[0], n_heads=case["heads"],
                         n_kv_heads=case["kv_heads"], k_dim=s.dk, v_dim=s.dv,
                         q=s.q.data_ptr(), q_strides=(s.q.stride(0), s.q.stride(1)),
                         out=s.out.data_ptr(), out_strides=(s.out.stride(0), s.out.stride(1)), lse=s.lse.data_ptr(),
                         k_pool=s.pool.data_ptr(), v_pool=s.pool.data_ptr(), k_offset=0,
                         v_offset=0 if s.latent else kv, pool_blocks=s.pool_blocks,
                         tables=s.tables.data_ptr(), table_stride=s.tables.shape[1],
                         starts=s.starts.data_ptr(), lens=s.lens.data_ptr(), max_len=s.max_len,
                         scale=s.scale, softcap=case["cap"], window=case["window"],
                         tree=s.tree.data_ptr() if s.tree is not None else 0, tree_words=1 if s.tree is not None else 0,
                         slopes=s.slopes.data_ptr() if s.slopes is not None else 0,
                         prefix=s.prefix.data_ptr() if s.prefix is not None else 0,
                         documents=s.docs.data_ptr() if s.docs is not None else 0)
    s.workspace = torch.empty(max(16, bsr.bsr_attn_workspace_bytes(ctx, args)), dtype=torch.uint8, device="cuda")
    args.workspace, args.workspace_bytes = s.workspace.data_ptr(), s.workspace.numel()
    attend = bsr.bsr_attend_tree if s.op == "tree" else bsr.bsr_attend_prompt
    return lambda: attend(ctx, args, stream)


# ---- the plain forms --------------------------------------------------------------------
def run(state):
    if own:
        state.call()
    else:
        {"tables": _plain_tables, "append": _plain_append}.get(state.op, _plain_attention)(state)
    if state.op == "tables":
        return {"starts": state.starts, "lens": state.lens, "result": state.result, "tables": state.tables,
                "slots": state.slots}
    if state.op == "append":
        return _pool_values(state.pool, state)
    return {"out": state.out, "lse": state.lse}


def _pool_values(pool, s):
    """The pool as the values it holds."""
    if not s.planar:
        return {"records": pool.view(s.type)}
    at = 128 * s.block
    return {"values": pool[:, :at].view(torch.float8_e4m3fn), "scales": pool[:, at:].view(torch.float32)}


def _plain_tables(s):
    cached, added = s.cached.long(), s.added.long()
    ends = added.cumsum(0)
    s.starts[1:] = ends
    s.lens.copy_(cached + added)
    s.result[0] = cached.numel()  # every request of these batches finds its blocks
    row = torch.arange(s.n_slots, device="cuda")
    r = torch.searchsorted(ends, row, right=True).clamp_(max=cached.numel() - 1)
    t = cached[r] + row - (ends[r] - added[r])
    for g, (b, free, table, slots) in enumerate(zip(MTP_BLOCKS, s.free, s.tables, s.slots)):
        held, need = (cached + b - 1) // b, (cached + added + b - 1) // b
        taken = need - held
        at = taken.cumsum(0) - taken
        k = torch.arange(table.shape[1], device="cuda")[None, :]
        new = (k >= held[:, None]) & (k < need[:, None])
        ids = free[(at[:, None] + k - held[:, None]).clamp_(0, free.numel() - 1)]
        table.copy_(torch.where(new, ids, table))
        s.result[1 + g] = taken.sum()
        slot = table[r, (t // b).clamp_(max=table.shape[1] - 1)].long() * b + t % b
        slots.copy_(torch.where(row < ends[-1], slot, -1))


def _plain_append(s):
    keep = s.slots >= 0
    at = s.slots[keep]
    x = torch.cat([x.float() for x in s.src], 1)[keep]
    if s.planar:
        scale = x.abs().amax(1) / 448.0
        q = (x / torch.where(scale > 0, scale, 1.0)[:, None]).to(torch.float8_e4m3fn)
        values = _pool_values(s.pool, s)
        values["values"].view(torch.uint8).view(-1, s.block, 128)[at // s.block, at % s.block] = q.view(torch.uint8)
        values["scales"][at // s.block, at % s.block] = scale
    else:
        s.pool.view(s.type).view(-1, s.record // 2)[at] = x.to(s.type)


def _gathered(s, dtype):
    """K and V of every request, [requests, kv_heads, max_len, dim], zeros behind each one's length."""
    j = torch.arange(s.max_len, device="cuda")
    rows = s.tables.long()[:, j // s.block] * s.block + j % s.block
    x = s.pool[rows].to(dtype) * (j[None, :] < s.lens[:, None])[..., None]
    n, hk = x.shape[0], s.case["kv_heads"]
    if s.latent:
        x = x[:, None]
        return x, x[..., :s.dv]
    k, v = x.split([hk * s.dk, hk * s.dv], 2)
    return (k.reshape(n, -1, hk, s.dk).transpose(1, 2).contiguous(),
            v.reshape(n, -1, hk, s.dv).transpose(1, 2).contiguous())


def _visible(s):
    """bool [requests, max_added, max_len]: which keys each padded query row sees; and each row's position."""
    i = torch.arange(s.max_added, device="cuda")
    j = torch.arange(s.max_len, device="cuda")
    base = (s.lens - s.added).long()
    real = i[None, :] < s.added[:, None]
    row = (s.starts[:-1, None].long() + i).clamp_(max=s.q.shape[0] - 1)
    if s.tree is not None:
        mask = s.tree[row]
        bits = mask[:, :, None] >> torch.arange(64, device="cuda") & 1
        depth = bits.sum(2) - 1
        p = base[:, None] + depth
        node = j[None, :] - base[:, None]
        inside = (node >= 0) & (node < s.added[:, None])
        branch = bits.gather(2, node.clamp(0, 63)[:, None, :].expand(-1, s.max_added, -1)) > 0
        see = torch.where(inside[:, None, :], branch, (node < 0)[:, None, :])
        if s.case["window"]:
            see &= (node >= 0)[:, None, :] | (j > p[..., None] - s.case["window"])
    else:
        p = base[:, None] + i
        hi = p + 1
        if s.prefix is not None:
            hi = torch.maximum(hi, torch.minimum(s.prefix, s.lens)[:, None])
        see = j < hi[..., None]
        if s.case["window"]:
            see &= j > p[..., None] - s.case["window"]
        if s.docs is not None:
            see &= j >= s.docs[row][..., None]
    return see & real[..., None], p, row, real


def _plain_attention(s):
    heads, hk = s.case["heads"], s.case["kv_heads"]
    k, v = _gathered(s, torch.float32)
    see, p, row, real = _visible(s)
    n, t = row.shape
    q = s.q[row].float().view(n, t, hk, heads // hk, s.dk).permute(0, 2, 3, 1, 4).reshape(n, hk, -1, s.dk)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(s.scale)
    if s.case["cap"]:
        x = x.div_(s.case["cap"]).tanh_().mul_(s.case["cap"])
    x = x.view(n, hk, heads // hk, t, -1)
    if s.slopes is not None:
        away = (p[..., None] - torch.arange(s.max_len, device="cuda")).abs().float()
        x -= s.slopes.view(hk, -1, 1, 1) * away[:, None, None]
    x.masked_fill_(~see[:, None, None], -math.inf)
    top = x.amax(4, keepdim=True)
    x.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = x.sum(4, keepdim=True)
    lse = (top + total.log())[..., 0]
    o = torch.matmul(x.view(n, hk, -1, s.max_len), v).view(n, hk, heads // hk, t, s.dv)
    o = o / torch.where(total > 0, total, 1.0)
    s.out.copy_(o.permute(0, 3, 1, 2, 4).reshape(n, t, heads, s.dv)[real])
    s.lse.copy_(lse.permute(0, 3, 1, 2).reshape(n, t, heads)[real])


# ---- the definitions in 64 bits ---------------------------------------------------------
def exact(case, seed):
    """Each operator by its definition: one request, and one head, at a time."""
    if case["op"] == "tables":
        return None  # whole numbers: equal, or wrong
    s = _State()
    s.case, s.op = case, case["op"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "append":
        _prepare_append(s, case, gen)
        x = torch.cat([a.double() for a in s.src], 1)
        at, held = s.slots, s.slots >= 0
        n = s.pool.shape[0] * s.block
        if not s.planar:
            records = torch.zeros(n, x.shape[1], dtype=torch.float64, device="cuda")
            records[at[held]] = x[held]
            return {"records": records.view(s.pool.shape[0], -1)}
        scales = torch.zeros(n, dtype=torch.float64, device="cuda")
        scales[at[held]] = x[held].abs().amax(1) / 448
        return {"values": None, "scales": scales.view(-1, s.block)}
    _prepare_attention(s, case, gen)
    heads, hk = case["heads"], case["kv_heads"]
    out = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s.lse.shape, dtype=torch.float64, device="cuda")
    trees = _trees(case, s.added_host) if case["op"] == "tree" else None
    docs = _documents(case, s.cached_host, s.added_host) if case.get("docs") else None
    prefixes = _prefixes(case, s.cached_host, s.added_host) if case.get("prefix") else None
    first = 0
    for r, (c, a) in enumerate(zip(s.cached_host, s.added_host)):
        n = c + a
        blocks = s.tables[r, :-(-n // s.block)].long()
        rec = s.pool.view(s.pool_blocks, s.block, -1)[blocks].reshape(-1, s.record_values)[:n]
        j = torch.arange(n, device="cuda", dtype=torch.float64)
        see = torch.zeros(a, n, dtype=torch.bool, device="cuda")
        if trees is not None:
            mine = trees[first:first + a]
            see[:, c:] = torch.tensor([[m >> k & 1 for k in range(a)] for m in mine], device="cuda") > 0
            p = torch.tensor([c - 1 + bin(m).count("1") for m in mine], device="cuda")
            see[:, :c] = True if not case["window"] else j[:c] > p[:, None] - case["window"]
        else:
            p = torch.arange(c, n, device="cuda")
            upto = p if prefixes is None else p.clamp(min=min(prefixes[r], n) - 1)
            see = j <= upto[:, None]
            if case["window"]:
                see &= j > p[:, None] - case["window"]
            if docs is not None:
                see &= j >= torch.tensor(docs[first:first + a], device="cuda")[:, None]
        away = (p[:, None] - j).abs()
        for h in range(heads):
            g = h // (heads // hk)
            k = rec[:, g * s.dk:(g + 1) * s.dk].double()
            v = rec[:, :s.dv].double() if s.latent else rec[:, hk * s.dk + g * s.dv:hk * s.dk + (g + 1) * s.dv].double()
            x = s.q[first:first + a, h].double() @ k.T * s.scale
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            if s.slopes is not None:
                x = x - s.slopes[h].double() * away
            x = torch.where(see, x, -math.inf)
            total = torch.logsumexp(x, 1)
            lse[first:first + a, h] = total
            w = torch.exp(x - torch.where(total > -math.inf, total, 0.0)[:, None])
            out[first:first + a, h] = w @ v
        first += a
    return {"out": out, "lse": lse}
