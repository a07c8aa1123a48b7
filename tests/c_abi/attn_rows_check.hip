// The paged attention's own functions for what a row sees, where a key lies and
// how a tile's keys are cut, on the host, against the definitions: random
// requests, trees, windows, documents and prefixes, and lengths, starts and
// block ids that are out of their ranges.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "bsr_attn_rows.h"

using namespace bsr;

static std::mt19937_64 rng(1);
static int pick(int lo, int hi) { return lo + static_cast<int>(rng() % static_cast<uint64_t>(hi - lo + 1)); }

#define EXPECT(x) \
  do { \
    if (!(x)) { std::printf("line %d: %s (case %d)\n", __LINE__, #x, number); std::exit(1); } \
  } while (0)

int main() {
  for (int number = 0; number < 4000; ++number) {
    AttnParams p{};
    const bool tree = number & 1, wild = number % 5 == 0;
    const uint32_t block = pick(1, 40);
    p.n_requests = pick(1, 4);
    p.table_stride = pick(1, 20);
    p.max_len = lesser<uint32_t>(p.table_stride * block, pick(0, 700));
    p.div_block = make_fastdiv(block);
    p.record_bytes = 16 * pick(1, 80);
    p.block_bytes = static_cast<uint64_t>(block) * p.record_bytes;
    p.pool_blocks = number % 7 ? pick(1, 50) : 0x7fffffff;
    p.tree_words = tree ? pick(1, 3) : 0;
    p.window = number % 3 ? 0 : tree ? 64 * p.tree_words + pick(0, 30) : pick(1, 200);
    std::vector<int32_t> starts{0}, lens, prefix, docs, tables(p.n_requests * p.table_stride);
    for (uint32_t r = 0; r < p.n_requests; ++r) {
      const int n = pick(0, p.max_len), rows = pick(0, tree ? 64 * p.tree_words + 9 : 90);
      lens.push_back(wild && pick(0, 2) == 0 ? (pick(0, 1) ? -pick(1, 1 << 30) : 0x7fffffff) : n);
      starts.push_back(wild && pick(0, 2) == 0 ? pick(-1000, 1000) : starts.back() + rows);
      prefix.push_back(pick(0, 3) ? pick(-5, 800) : 0);
    }
    p.n_tokens = wild ? pick(0, 200) : static_cast<uint32_t>(starts.back() + pick(0, 3));
    for (uint32_t i = 0; i < p.n_tokens; ++i) docs.push_back(pick(0, 9) ? pick(-3, 300) : 0x7fffffff);
    std::vector<uint64_t> masks(static_cast<size_t>(p.n_tokens) * p.tree_words);
    for (auto& m : masks) m = pick(0, 4) ? rng() : 0;
    for (auto& b : tables) b = pick(0, 9) ? pick(0, 60) : static_cast<int32_t>(rng());
    p.starts = starts.data();
    p.lens = lens.data();
    p.tables = tables.data();
    p.tree = tree ? masks.data() : nullptr;
    if (tree && masks.empty()) continue;
    p.prefix = !tree && number % 4 < 2 ? prefix.data() : nullptr;
    p.documents = !tree && number % 8 < 4 && p.n_tokens ? docs.data() : nullptr;
    p.tile_tokens = pick(1, 40);
    for (uint32_t r = 0; r < p.n_requests; ++r) {
      const Request q = request_of(p, r);
      EXPECT(q.first >= 0 && q.rows >= 0 && q.first + q.rows <= static_cast<int>(p.n_tokens));
      EXPECT(q.n >= 0 && q.n <= static_cast<int>(p.max_len) && q.base == q.n - q.rows);
      const RequestWork rw = request_work(p, r);
      for (uint32_t tile = 0; tile < rw.tiles; ++tile) {
        Work w{r, tile, 0, 0, 1, 0};
        int lo, hi;
        tile_range(p, q, w, &lo, &hi);
        EXPECT(lo >= 0 && hi <= q.n && hi >= 0);
        EXPECT(static_cast<uint32_t>(greater(hi - lo, 0)) <= rw.range);
        // the parts follow one another and are all of it
        w.n_splits = pick(1, 9);
        int at = lo;
        for (w.split = 0; w.split < w.n_splits; ++w.split) {
          int k0, k1;
          cut(w, lo, hi, &k0, &k1);
          EXPECT(k0 <= k1);
          if (k0 < k1) {
            EXPECT(k0 == at && (w.split == 0 || (k0 - lo) % 64 == 0) && k1 <= hi);
            at = k1;
          }
        }
        EXPECT(at == greater(lo, hi));
        for (uint32_t t = 0; t < p.tile_tokens; ++t) {
          const int i = static_cast<int>(tile * p.tile_tokens + t);
          if (i >= q.rows) break;
          const Row row = row_of(p, q, r, i);
          // by the definition
          int bits = 0;
          if (tree)
            for (uint32_t k = 0; k < 64 * p.tree_words; ++k)
              bits += masks[static_cast<size_t>(q.first + i) * p.tree_words + k / 64] >> (k % 64) & 1;
          const long pos = tree ? (p.window ? q.base + bits - 1L : 0) : q.base + i;
          for (int j0 = 0; j0 < q.n + 64; j0 += 64) {  // (a step starts at a key)
            uint64_t see = bit_range(greater(row.lo, 0) - j0, lesser(row.hi, q.n) - j0);
            if (tree) see &= tree_bits(p, row.mask, j0 - q.base);
            for (int e = 0; e < 64; ++e) {
              const long j = j0 + e;
              bool want = j >= 0 && j < q.n;
              if (tree) {
                const long k = j - q.base;
                if (p.window) want = want && (k >= 0 || j > pos - static_cast<long>(p.window));
                if (k >= 0)
                  want = want && k < 64L * p.tree_words &&
                         (masks[static_cast<size_t>(q.first + i) * p.tree_words + k / 64] >> (k % 64) & 1);
              } else {
                want = want && (j <= pos || (p.prefix && j < lesser(prefix[r], q.n)));
                if (p.window) want = want && j > pos - static_cast<long>(p.window);
                if (p.documents) want = want && j >= docs[q.first + i];
              }
              EXPECT((see >> e & 1) == want);
              if (j >= 0 && j < q.n) EXPECT(sees(p, q, row, static_cast<int>(j)) == want);
              if (want) EXPECT(j >= lo && j < hi);
            }
          }
        }
      }
      for (int j = 0; j < q.n; ++j) {
        const KeyLoad k = key_load(p, q, j, q.n - 1);
        const int32_t id = tables[r * p.table_stride + j / block];
        int64_t off;
        const bool ok = key_offset(p, k, &off);
        EXPECT(ok == (id >= 0 && static_cast<uint32_t>(id) < p.pool_blocks));
        const int64_t want = static_cast<int64_t>(id) * block * p.record_bytes + static_cast<int64_t>(j % block) * p.record_bytes;
        EXPECT(off == (ok ? want : 0) && record_at(p, q, j) == (ok ? want : -1));
      }
    }
  }
  // items whose parts the workspace holds, and no others, whatever the sums wrapped to
  for (int number = 0; number < 4000; ++number) {
    AttnParams p{};
    p.parts = pick(0, 3) ? pick(0, 2 * kMaxTarget) : 0;
    Work w{};
    w.n_splits = pick(0, 3) ? pick(1, 2 * kMaxTarget) : static_cast<uint32_t>(rng()) | 1;
    w.slot = pick(0, 3) ? pick(0, 2 * kMaxTarget) : static_cast<uint32_t>(rng());
    const uint64_t end = static_cast<uint64_t>(w.slot) + w.n_splits;
    EXPECT(parts_fit(p, w) == (w.n_splits == 1 || (end <= p.parts && w.n_splits <= kMaxTarget)));
  }
  std::puts("ok");
  return 0;
}
