// What a query row of the paged cache's attention sees, where its keys lie and
// how a batch's work is cut: the kernels' own functions, host-callable too, so
// that a CPU test checks them.
#pragma once

#include "bsr_cache.h"

#define BSR_ROWS_FN __host__ __device__ __forceinline__

namespace bsr {

template <typename T>
BSR_ROWS_FN T lesser(T a, T b) { return a < b ? a : b; }
template <typename T>
BSR_ROWS_FN T greater(T a, T b) { return a < b ? b : a; }

// One request of the batch: its rows [first, first + rows) and its keys [0, n);
// row i stands at base + i.
struct Request {
  int first, rows, n, base;
  const int32_t* table;
};

BSR_ROWS_FN Request request_of(const AttnParams& p, uint32_t r) {
  Request q;
  const int cap = static_cast<int>(p.n_tokens);
  q.first = lesser(greater(p.starts[r], 0), cap);
  q.rows = lesser(greater(p.starts[r + 1], q.first), cap) - q.first;
  q.n = lesser(greater(p.lens[r], 0), static_cast<int>(p.max_len));
  q.base = q.n - q.rows;
  q.table = p.tables + static_cast<uint64_t>(r) * p.table_stride;
  return q;
}

// What row i of a request sees: keys [lo, hi), those from base on by the bits
// of its mask in a tree; and its position, from which distances count.
struct Row {
  int lo, hi, pos;
  const uint64_t* mask;
};

BSR_ROWS_FN Row row_of(const AttnParams& p, const Request& q, uint32_t r, int i) {
  Row w;
  w.mask = nullptr;
  if (p.tree) {
    w.mask = p.tree + static_cast<uint64_t>(q.first + i) * p.tree_words;
    int bits = 0;
    if (p.window)
      for (uint32_t k = 0; k < p.tree_words; ++k) bits += __builtin_popcountll(w.mask[k]);
    w.pos = q.base + bits - 1;
    w.hi = q.n;
  } else {
    w.pos = q.base + i;
    w.hi = w.pos + 1;
    if (p.prefix) w.hi = greater(w.hi, lesser(p.prefix[r], q.n));
  }
  w.lo = 0;
  if (p.window) w.lo = greater(0, w.pos - static_cast<int>(p.window) + 1);
  if (p.documents) w.lo = greater(w.lo, p.documents[q.first + i]);
  return w;
}

BSR_ROWS_FN bool sees(const AttnParams& p, const Request& q, const Row& w, int j) {
  if (j < w.lo || j >= w.hi) return false;
  if (!w.mask || j < q.base) return true;
  const uint32_t k = static_cast<uint32_t>(j - q.base);
  return k < 64 * p.tree_words && (w.mask[k >> 6] >> (k & 63) & 1);
}

// Byte offset of token j's record in a pool, or -1 where its block lies outside.
BSR_ROWS_FN int64_t record_at(const AttnParams& p, const Request& q, int j) {
  const uint32_t b = p.div_block.div(j);
  const int32_t id = q.table[b];
  if (id < 0 || static_cast<uint32_t>(id) >= p.pool_blocks) return -1;
  return static_cast<int64_t>(static_cast<uint64_t>(id) * p.block_bytes + (j - b * p.div_block.d) * p.record_bytes);
}

// The bits of a row's tree mask from key offset `off` of the request's rows on,
// ones before them.
BSR_ROWS_FN uint64_t tree_bits(const AttnParams& p, const uint64_t* mask, int off) {
  if (off <= -64) return ~0ull;
  if (off < 0) return (mask[0] << -off) | ((1ull << -off) - 1);
  const uint32_t w = off >> 6, sh = off & 63;
  if (w >= p.tree_words) return 0;
  uint64_t bits = mask[w] >> sh;
  if (sh && w + 1 < p.tree_words) bits |= mask[w + 1] << (64 - sh);
  return bits;
}

// Bits [lo, hi) of 64, both taken into 0..64.
BSR_ROWS_FN uint64_t bit_range(int lo, int hi) {
  lo = lesser(greater(lo, 0), 64);
  hi = lesser(greater(hi, 0), 64);
  if (lo >= hi) return 0;
  const uint64_t to = hi == 64 ? ~0ull : (1ull << hi) - 1;
  return to & (~0ull << lo);
}

// One part of a tile's keys for one KV head.
struct Work {
  uint32_t r;       // request
  uint32_t tile;    // of the request's tokens
  uint32_t unit;    // KV head x chunk of its heads
  uint32_t split, n_splits;
  uint32_t slot;    // first partial result of the item's parts
};

// Whether an item's parts lie in the workspace and can be joined.  Always, but
// for starts that decrease: their tiles may number past 32 bits.
BSR_ROWS_FN bool parts_fit(const AttnParams& p, const Work& w) {
  return w.n_splits < 2 || (w.n_splits <= p.parts && w.n_splits <= kMaxTarget && w.slot <= p.parts - w.n_splits);
}

// What a lane knows of its request: tiles of tokens, and the keys that one of
// them can see at most.
struct RequestWork {
  Request q;
  uint32_t tiles, range;
};

BSR_ROWS_FN RequestWork request_work(const AttnParams& p, uint32_t r) {
  RequestWork w{};
  if (r >= p.n_requests) return w;
  w.q = request_of(p, r);
  const uint32_t rows = w.q.rows;
  w.tiles = (rows + p.tile_tokens - 1) / p.tile_tokens;
  w.range = w.q.n;
  if (p.window && !p.prefix) w.range = lesser(w.range, p.window + (p.tree ? rows : lesser(rows, p.tile_tokens)));
  return w;
}

BSR_ROWS_FN uint32_t splits_of(uint32_t range, uint32_t part) { return range > part ? (range + part - 1) / part : 1; }

// Keys [lo, hi) that a tile's rows see any of; documents are looked at by the
// caller.
BSR_ROWS_FN void tile_range(const AttnParams& p, const Request& q, const Work& w, int* lo, int* hi) {
  const int i0 = w.tile * p.tile_tokens, i1 = lesser(i0 + static_cast<int>(p.tile_tokens), q.rows);
  *lo = 0;
  if (p.tree) {
    *hi = q.n;
    if (p.window) *lo = greater(0, q.base - static_cast<int>(p.window));  // a row that sees no row stands at base - 1
  } else {
    *hi = q.base + i1;
    if (p.prefix) *hi = greater(*hi, lesser(p.prefix[w.r], q.n));
    *hi = greater(*hi, 0);
    if (p.window) *lo = greater(0, q.base + i0 - static_cast<int>(p.window) + 1);
  }
}

// Part `split` of the keys [lo, hi): whole steps of 64 keys.
BSR_ROWS_FN void cut(const Work& w, int lo, int hi, int* k0, int* k1) {
  if (hi < lo) hi = lo;
  const uint32_t len = hi - lo;
  const uint32_t per = ((len + w.n_splits - 1) / w.n_splits + 63) & ~63u;
  const uint64_t at = static_cast<uint64_t>(per) * w.split;
  *k0 = at < len ? lo + static_cast<int>(at) : hi;
  *k1 = at + per < len ? lo + static_cast<int>(at + per) : hi;
}

// The record offset of a key, and whether its block lies in the pool; keys past the
// part's last are read as that one (the rows do not see them).
struct KeyLoad {
  int j;
  uint32_t block;
  int32_t id;
};
BSR_ROWS_FN KeyLoad key_load(const AttnParams& p, const Request& q, int j, int last) {
  KeyLoad k;
  k.j = lesser(j, last);
  k.block = p.div_block.div(k.j);
  k.id = q.table[k.block];
  return k;
}
BSR_ROWS_FN bool key_offset(const AttnParams& p, const KeyLoad& k, int64_t* off) {
  const bool ok = static_cast<uint32_t>(k.id) < p.pool_blocks;  // (fewer than 2^31)
  const uint32_t keep = 0u - static_cast<uint32_t>(ok);  // no branch: latent steps do this beside their products
  const uint32_t id = k.id & keep, at = (k.j - k.block * p.div_block.d) & keep;
  *off = static_cast<int64_t>(static_cast<uint64_t>(id) * p.block_bytes + at * p.record_bytes);  // a block is smaller than 2^31 bytes
  return ok;
}

}  // namespace bsr
