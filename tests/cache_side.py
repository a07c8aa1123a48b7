"""Drive the paged cache's operators through the binding, beside the oracle (GPU tests only)."""

from __future__ import annotations

import numpy as np
import torch

from oracle import cache as oracle_cache
from paper_2608_17826_amd import bsr

TYPE = {"bf16": (torch.bfloat16, bsr.BSR_TYPE_BF16), "f16": (torch.float16, bsr.BSR_TYPE_F16),
        "f32": (torch.float32, bsr.BSR_TYPE_F32)}
_ctx = {}


def context(*groups):
    """One context per layout for the whole run; groups: (block_tokens, n_tensors, record_bytes, kind, split)."""
    if groups not in _ctx:
        _ctx[groups] = bsr.bsr_ctx_create(bsr.make_layout(256, groups), 1, hip_device=0)
    return _ctx[groups]


def stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def ints(x, dtype=torch.int32):
    return torch.as_tensor(np.asarray(x), dtype=dtype).cuda()


def bounds(o, l, a, dot, dtype, dk, n, bias=0.0):
    """How far an attention row may be off: (out, lse), from what oracle.cache.attend gives.

    ``n``: keys that the row sees; ``bias``: the largest distance bias.  In
    fp32 (half a unit f = 2^-24) a score's product of dk terms is off by (dk + 8) f
    of its sum of magnitudes, and scaling, cap, bias, log2(e), running
    maximum and exponent round it some eight times more.  A weight is off by its
    score's error and the maximum's, and by the exponential and the sums.  The
    weights are rounded to the dtype (u relative; below fp16's subnormals
    absolutely), and so is the result.
    """
    f, u = 2.0 ** -24, torch.finfo(dtype).eps / 2
    ds = f * (dk + 8) * dot + 8 * f * (dot + bias)
    dw = 2 * ds + (8 + np.log2(max(2, n)) + 64) * f
    a = np.where(np.isfinite(a), a, 0)   # (not looked at there)
    small = 2.0 ** -25 if dtype == torch.float16 else 0
    return (u + dw) * a * (1 + u) + u * np.abs(o) + 1e-30 + small * (1 + a), 2 * ds + (80 + abs(l)) * 2 * f


class AttnCase:
    """A paged cache, queries and their call.

    lens, rows: per request; dims (k, v); the record holds the KV heads' keys,
    then their values (latent records: the key alone), behind ``lead`` values
    that belong to something else.
    """

    def __init__(self, mode, lens, rows, heads, kv_heads, dims, dtype="bf16", block=16, seed=0, window=0, cap=0.0,
                 masks=None, words=1, slopes=None, prefix=None, documents=None, lead=0, tail_rows=0, q_pad=0,
                 scale=None, max_len=None, spread=1.0):
        self.mode, self.lens, self.rows = mode, list(lens), list(rows)
        self.heads, self.kv_heads, (self.dk, self.dv) = heads, kv_heads, dims
        self.latent = dims == (576, 512)
        self.dtype, self.code = TYPE[dtype]
        self.block, self.window, self.cap = block, window, cap
        self.scale = dims[0] ** -0.5 if scale is None else scale
        g = torch.Generator().manual_seed(seed)
        self.values = lead + (self.dk if self.latent else kv_heads * (self.dk + self.dv))
        self.values += -self.values % 8
        self.lead = lead
        need = [-(-n // block) for n in self.lens]
        self.pool_blocks = sum(need) + 2
        self.pool = (torch.randn(self.pool_blocks * block, self.values, generator=g) * spread).to(self.dtype)
        ids = torch.randperm(self.pool_blocks, generator=g).to(torch.int32)
        self.stride = max(need + [1]) + 1
        self.tables = torch.full((len(self.lens), self.stride), -7, dtype=torch.int32)
        at = 0
        for r, k in enumerate(need):
            self.tables[r, :k] = ids[at:at + k]
            at += k
        # blocks that no request holds carry what must not be read into any result
        self.pool.view(self.pool_blocks, block, -1)[ids[at:].long()] = float("nan")
        for r, n in enumerate(self.lens):  # so does the end of the last block
            if n % block:
                b = int(self.tables[r, n // block])
                self.pool.view(self.pool_blocks, block, -1)[b, n % block:] = float("nan")
        total = sum(self.rows)
        self.n_tokens = total + tail_rows
        wide = torch.randn(self.n_tokens, heads, self.dk + q_pad, generator=g).to(self.dtype)
        self.q_wide = wide
        self.starts = np.concatenate([[0], np.cumsum(self.rows)])
        self.words = words
        self.masks, self.slopes, self.prefix, self.documents = masks, slopes, prefix, documents
        self.max_len = max(self.lens + [1]) if max_len is None else max_len

    def place(self):
        self.d = dict(pool=self.pool.cuda(), tables=self.tables.cuda(), q=self.q_wide.cuda()[..., :self.dk],
                      out=torch.full((self.n_tokens, self.heads, self.dv + 8), 7.0, dtype=self.dtype).cuda(),
                      lse=torch.full((self.n_tokens, self.heads), 7.0).cuda(),
                      starts=ints(self.starts), lens=ints(self.lens))
        if self.mode == "tree":
            m = np.asarray(self.masks, dtype=np.uint64).reshape(-1, self.words)
            m = np.concatenate([m, np.full((self.n_tokens - len(m), self.words), 2 ** 64 - 1, np.uint64)])
            self.d["tree"] = torch.from_numpy(m.view(np.int64).copy()).cuda()
        if self.slopes is not None:
            self.d["slopes"] = torch.tensor(self.slopes, dtype=torch.float32).cuda()
        if self.prefix is not None:
            self.d["prefix"] = ints(self.prefix)
        if self.documents is not None:
            self.d["documents"] = ints(list(self.documents) + [0] * (self.n_tokens - len(self.documents)))
        return self

    def args(self, **other):
        d = self.d
        p = lambda k: d[k].data_ptr() if k in d else 0  # noqa: E731
        kv = 2 * (self.lead + (0 if self.latent else self.kv_heads * self.dk))
        f = dict(group=0, dtype=self.code, n_requests=len(self.lens), n_tokens=self.n_tokens, n_heads=self.heads,
                 n_kv_heads=self.kv_heads, k_dim=self.dk, v_dim=self.dv, q=p("q"),
                 q_strides=(d["q"].stride(0), d["q"].stride(1)), out=p("out"),
                 out_strides=(d["out"].stride(0), d["out"].stride(1)), lse=p("lse"), k_pool=p("pool"),
                 v_pool=p("pool"), k_offset=2 * self.lead, v_offset=kv, pool_blocks=self.pool_blocks,
                 tables=p("tables"), table_stride=self.stride, starts=p("starts"), lens=p("lens"),
                 max_len=self.max_len, window=self.window, scale=self.scale, softcap=self.cap, tree=p("tree"),
                 tree_words=self.words if self.mode == "tree" else 0, slopes=p("slopes"), prefix=p("prefix"),
                 documents=p("documents"))
        f.update(other)
        return bsr.attn_args(**f)

    def ctx(self):
        return context((self.block, 1, 2 * self.values, bsr.BSR_KIND_CONTIG, 0))

    def prepare(self, **other):
        """The call's args with a workspace of its own."""
        a = self.args(**other)
        n = bsr.bsr_attn_workspace_bytes(self.ctx(), a)
        self.d["workspace"] = torch.full((n + 16,), 0xFF, dtype=torch.uint8, device="cuda")
        a.workspace, a.workspace_bytes = self.d["workspace"].data_ptr(), n
        return a

    def call(self, a=None):
        a = self.prepare() if a is None else a
        (bsr.bsr_attend_tree if self.mode == "tree" else bsr.bsr_attend_prompt)(self.ctx(), a, stream())
        return a

    def run(self):
        self.place()
        self.call()
        torch.cuda.synchronize()
        return self

    # ---- against the oracle ----------------------------------------------------
    def row_case(self, r, i):
        first = int(self.starts[r])
        kw = dict(window=self.window)
        if self.mode == "tree":
            kw["mask"] = [int(x) for x in np.asarray(self.masks, dtype=np.uint64).reshape(-1, self.words)[first + i]]
        else:
            kw["prefix"] = 0 if self.prefix is None else self.prefix[r]
            kw["document"] = 0 if self.documents is None else self.documents[first + i]
        return oracle_cache.visible(self.mode, self.lens[r], self.rows[r], i, **kw)

    def check(self, sample=None, seed=0):
        """Every row and head (or `sample` drawn ones) against the oracle, within the derived bound; untouched rows."""
        out, lse = self.d["out"].double().cpu().numpy(), self.d["lse"].double().cpu().numpy()
        assert np.all(out[..., self.dv:] == 7), "beside the output"
        total = int(self.starts[-1])
        assert np.all(out[total:] == 7) and np.all(lse[total:] == 7), "rows behind the last request"
        todo = [(r, i, h) for r, T in enumerate(self.rows) for i in range(T) for h in range(self.heads)]
        if sample is not None and sample < len(todo):
            rng = np.random.default_rng(seed)
            todo = [todo[k] for k in sorted(rng.choice(len(todo), sample, replace=False))]
        pool = self.pool.double().numpy()
        q = self.q_wide[..., :self.dk].double().numpy()
        recs = {}
        worst = 0.0
        for r, i, h in todo:
            n, row = self.lens[r], int(self.starts[r]) + i
            if r not in recs:
                j = np.arange(n)
                ids = self.tables[r].numpy()[j // self.block].astype(np.int64) if n else np.zeros(0, np.int64)
                bad = (ids < 0) | (ids >= self.pool_blocks)
                recs[r] = pool[np.where(bad, 0, ids) * self.block + j % self.block], bad
            x, bad = recs[r]
            g = h // (self.heads // self.kv_heads)
            k = x[:, self.lead + g * self.dk:][:, :self.dk]
            v = k[:, :self.dv] if self.latent else x[:, self.lead + self.kv_heads * self.dk + g * self.dv:][:, :self.dv]
            see, p = self.row_case(r, i)
            slope = 0.0 if self.slopes is None else float(np.float32(self.slopes[h]))
            o, l, a, dot = oracle_cache.attend(q[row, h], k, v, see & ~bad, p, float(np.float32(self.scale)),
                                               float(np.float32(self.cap)), slope)
            where = f"request {r} row {i} head {h}"
            got = out[row, h, :self.dv]
            fine = np.isfinite(o)
            np.testing.assert_array_equal(got[~fine], o[~fine], err_msg=where)
            if not np.isfinite(l) or not np.isfinite(dot):   # nothing seen, or a score that is no number
                assert lse[row, h] == l or (np.isnan(lse[row, h]) and np.isnan(l)), (where, lse[row, h], l)
                assert not fine.any() or l == -np.inf, where
                np.testing.assert_array_equal(got[fine], o[fine], err_msg=where)
                continue
            bound, lb = bounds(o, l, a, dot, self.dtype, self.dk, int(see.sum()), abs(slope) * len(see))
            with np.errstate(invalid="ignore"):
                err, bound = np.abs(got - o)[fine], bound[fine]
            assert np.all(err <= bound), (where, float((err / bound).max()), got[:4], o[:4])
            worst = max(worst, float((err / bound).max(initial=0)))
            assert abs(lse[row, h] - l) <= lb, (where, lse[row, h], l, lb)
        return worst
