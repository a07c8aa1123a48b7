// Attention over the paged cache, for drafted trees and for prompt tokens.
//
// A query row (token, head) sees the keys lo <= j < hi of its request, and of
// those in a drafted tree's rows the ones whose bit its mask has.  Its scores
// pass the softmax in one go over the keys, with a running maximum m and sum
// l: new keys scale what was summed so far by exp(m - m').
#include <hip/hip_runtime.h>

#include "bsr_attn_rows.h"

namespace bsr {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Score times log2(e) of a product.
__device__ __forceinline__ float score2(const AttnParams& p, float qk, float slope, int away) {
  float s = qk * p.scale;
  if (p.softcap > 0) {
    const float z = s / p.softcap;
    if (!(fabsf(z) < 1e-4f)) s = p.softcap * tanhf(z);  // (below, the cap takes z^2 / 3 of it, less than a rounding)
  }
  return (s - slope * static_cast<float>(abs(away))) * kLog2e;
}

// One row over the keys [lo, hi) by one wave: 64 keys at a time, a lane each
// for the scores, then every lane VD / 64 dimensions of the values.  Only what
// the row sees is read.  m and l are the wave's, acc the lane's.  (For rows whose
// matrix products met an infinity or a NaN: right, not fast.)
template <typename T, int KD, int VD>
__device__ void attend_row(const AttnParams& p, const Request& q, const Row& w, int i, uint32_t head, int lo, int hi,
                           float& m, float& l, float (&acc)[VD / 64]) {
  constexpr int kPer = VD / 64;
  const int lane = threadIdx.x & 63;
  const uint32_t kv = head / (p.n_heads / p.n_kv_heads);
  const T* qr = reinterpret_cast<const T*>(p.q + (q.first + i) * p.q_token + head * p.q_head);
  const float slope = p.slopes ? p.slopes[head] : 0.0f;
  m = -__builtin_inff();
  l = 0;
  for (int d = 0; d < kPer; ++d) acc[d] = 0;
  for (int j0 = lo; j0 < hi; j0 += 64) {
    const int j = j0 + lane;
    int64_t at = -1;
    if (j < hi && sees(p, q, w, j)) at = record_at(p, q, j);
    float s = -__builtin_inff();
    if (at >= 0) {
      const T* k = reinterpret_cast<const T*>(p.k_pool + at + kv * (2 * KD));
      float dot = 0;
#pragma unroll 2
      for (int d = 0; d < KD; d += 8) {
        T x[8];
        __builtin_memcpy(x, __builtin_assume_aligned(k + d, 16), 16);
        for (int e = 0; e < 8; ++e) dot += static_cast<float>(x[e]) * static_cast<float>(qr[d + e]);
      }
      s = score2(p, dot, slope, w.pos - j);
    }
    const uint64_t seen = __ballot(at >= 0);
    if (!seen) continue;
    float top = at >= 0 ? s : -__builtin_inff();
    bool odd = at >= 0 && s != s;
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float m1 = fmaxf(m, top);
    const float back = m > -__builtin_inff() ? exp2_(m - m1) : 0.0f;
    float e = at >= 0 ? (m1 > -__builtin_inff() || odd ? exp2_(s - m1) : 0.0f) : 0.0f;
    float sum = e;
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    l = l * back + sum;
    m = m1;
    for (int d = 0; d < kPer; ++d) acc[d] *= back;
    for (uint64_t left = seen; left; left &= left - 1) {
      const int k = __builtin_ctzll(left);
      const float e1 = __shfl(e, k);
      const int64_t a1 = __shfl(at, k);
      const T* v = reinterpret_cast<const T*>(p.v_pool + a1 + kv * (2 * VD)) + lane * kPer;
      for (int d = 0; d < kPer; ++d) acc[d] += e1 * static_cast<float>(v[d]);
    }
  }
}


// ---------------------------------------------------------------------------
// The work: a tile is up to tile_rows query rows, tile_tokens tokens times
// tile_heads heads of one KV head, so that a key read once serves them all.
// Where a batch has few tiles its key ranges are cut into parts, and a second
// kernel joins them.  Every workgroup finds its item from the lengths alone:
// nothing about them is known to the host.
// ---------------------------------------------------------------------------
// What is the same in every lane, into a scalar register.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
  return static_cast<uint64_t>(uniform(static_cast<uint32_t>(x >> 32))) << 32 | uniform(static_cast<uint32_t>(x));
}

// A lane's value from another lane of its row of 16, or from the last lane of
// the rows before, 0 where there is none; an inclusive sum over the wave of them.
template <int kCtrl, int kRows>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return __builtin_amdgcn_update_dpp(0, static_cast<int>(x), kCtrl, kRows, 0xf, false);
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x += dpp<0x111, 0xf>(x);
  x += dpp<0x112, 0xf>(x);
  x += dpp<0x114, 0xf>(x);
  x += dpp<0x118, 0xf>(x);
  x += dpp<0x142, 0xa>(x);
  x += dpp<0x143, 0xc>(x);
  return x;
}
__device__ __forceinline__ float wave_total(float x) {
  const auto add = [](float v, uint32_t u) { return v + __uint_as_float(u); };
  x = add(x, dpp<0x111, 0xf>(__float_as_uint(x)));
  x = add(x, dpp<0x112, 0xf>(__float_as_uint(x)));
  x = add(x, dpp<0x114, 0xf>(__float_as_uint(x)));
  x = add(x, dpp<0x118, 0xf>(__float_as_uint(x)));
  x = add(x, dpp<0x142, 0xa>(__float_as_uint(x)));
  x = add(x, dpp<0x143, 0xc>(__float_as_uint(x)));
  return __shfl(x, 63);
}

// Over the requests of a batch of up to 64.
__device__ __forceinline__ uint32_t wave_sum(const AttnParams& p, uint32_t x) {
  return p.n_requests > 1 ? static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(wave_scan(x)), 63)) : uniform(x);
}

// Keys of a part.  Where the batch has no more tiles x units than the GPU holds
// workgroups (target), its ranges are cut into as many parts as those, so that
// all run at once and end together; up to twice as many tiles are cut into twice
// as many parts if those are long (kLongPart) and no documents make the ranges
// uncertain; more are left whole.  All parts have the same length, which starts
// at their share of the batch's (tile, key) pairs and grows until the parts, each
// range's rounded up, are no more than that.  Past six rounds, and for batches of
// over 64 requests, it is the length that no rounding makes too many of.
//
// One token of 64 heads (8 KV heads of 128) of 70 requests, 560 tiles: up to 20K
// keys 571 us cut, 613 whole; up to 2K 81 and 78; up to 500 33.4 and 30.0.
//
// The rule goes by the batch's tiles and its sum, so one long range among many short
// ones is cut the less the nearer the tiles come to target: such a token over
// 131,072 keys among others over 1,000 takes 152 us of 32 requests, 252 of 48 and, whole,
// 2,360 of 63 to 100 (the bytes 137 to 195); with latent records of 16 heads 105 us of 100
// requests, 308 of 200, 6,300 of 255 and 300 (55 to 104).
constexpr float kLongPart = 2048;  // keys
__device__ __forceinline__ uint32_t part_keys(const AttnParams& p, const RequestWork& first) {
  constexpr uint32_t kWhole = 0x7fffffffu;
  if (!p.target) return kWhole;
  const uint32_t lane = threadIdx.x & 63;
  uint32_t base;
  float total = static_cast<float>(first.tiles) * static_cast<float>(first.range);
  if (p.n_requests <= 64) {
    base = wave_sum(p, first.tiles) * p.units;
    total = p.n_requests > 1 ? wave_total(total) : __shfl(total, 0);
  } else {
    uint32_t tiles = first.tiles;
    for (uint32_t r0 = 64; r0 < p.n_requests; r0 += 64) {
      const RequestWork w = request_work(p, r0 + lane);
      tiles += w.tiles;
      total += static_cast<float>(w.tiles) * static_cast<float>(w.range);
    }
    base = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(wave_scan(tiles)), 63)) * p.units;
    total = wave_total(total);
  }
  // (p.parts is what the workspace holds, whatever the lengths say)
  const uint32_t limit = lesser(base <= p.target ? p.target : 2 * p.target, p.parts);
  total *= static_cast<float>(p.units);
  if (base >= limit || (base > p.target && (p.documents || total < kLongPart * static_cast<float>(limit)))) return kWhole;
  const auto length = [&](float keys) {  // whole steps; the sum is off by less than a thousandth (2^14 additions a lane)
    const uint32_t k = static_cast<uint32_t>(fminf(keys * 1.002f, 2e9f)) + 1;
    return uniform(((k > p.min_part ? k : p.min_part) + 63) & ~63u);
  };
  if (p.n_requests <= 64) {
    uint32_t part = length(total / static_cast<float>(limit));
    for (int i = 0; i < 6; ++i) {
      const uint32_t n = wave_sum(p, first.tiles * splits_of(first.range, part)) * p.units;
      if (n <= limit) return part;
      part = length(static_cast<float>(part) * static_cast<float>(n) / static_cast<float>(limit));
    }
  }
  return length(total / static_cast<float>(limit - base));
}

// Item `b` of the batch (every wave finds it for itself); kBase: b counts tiles
// x units, and the item is its first part.
template <bool kBase>
__device__ __forceinline__ bool find_work(const AttnParams& p, uint32_t b, Work* out, Request* q) {
  const uint32_t lane = threadIdx.x & 63;
  RequestWork w = request_work(p, lane);
  const uint32_t part = part_keys(p, w);
  uint32_t items_before = 0, slots_before = 0;
  for (uint32_t r0 = 0; r0 < p.n_requests; r0 += 64) {
    if (r0) w = request_work(p, r0 + lane);
    const uint32_t s = splits_of(w.range, part), base = w.tiles * p.units;
    const uint32_t items = kBase ? base : base * s, slots = s > 1 ? base * s : 0;
    uint32_t ends = items, slot_ends = slots;
    if (p.n_requests > 1) {
      ends = wave_scan(ends);
      slot_ends = wave_scan(slot_ends);
    }
    ends += items_before;
    slot_ends += slots_before;
    const uint64_t past = __ballot(ends > b);
    if (past) {
      const int l = __builtin_ctzll(past);
      const auto of = [&](uint32_t x) { return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), l)); };
      const uint32_t local = b - of(ends - items);
      out->r = r0 + l;
      out->n_splits = of(s);
      const uint32_t rest = kBase ? local : local / out->n_splits;
      out->split = kBase ? 0 : local - rest * out->n_splits;
      const uint32_t t = rest / p.units;
      out->unit = rest - t * p.units;
      out->tile = of(w.tiles) - 1 - t;  // the last tokens see the most keys: first
      out->slot = of(slot_ends - slots) + rest * out->n_splits;
      q->first = of(w.q.first);
      q->rows = of(w.q.rows);
      q->n = of(w.q.n);
      q->base = q->n - q->rows;
      q->table = p.tables + static_cast<uint64_t>(out->r) * p.table_stride;
      return parts_fit(p, *out);
    }
    items_before = __builtin_amdgcn_readlane(ends, 63);
    slots_before = __builtin_amdgcn_readlane(slot_ends, 63);
  }
  return false;
}

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// C[32 x 32] += A[32 x 16] B[16 x 32].  Lane l = 32 h + c holds row c of A and
// column c of B at k = 8 h .. 8 h + 7, and column c of C at rows
// 8 (e / 4) + 4 h + e % 4 for e = 0..15.
template <typename T>
__device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c);
template <>
__device__ __forceinline__ f32x16 mfma<__bf16>(s16x8 a, s16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x16 mfma<_Float16>(s16x8 a, s16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// The same with the results in vector registers whatever the rest of the
// kernel uses: the compiler keeps all of a kernel's results in accumulator
// registers once it needs any of them, and the latent attention has none left.
// It sees no matrix instruction here: the wait before each covers an operand that
// it has just computed, and the last product's result is read after mfma_done (a
// product of 8 passes needs 11 wait states; the waits are 20).
template <typename T>
__device__ __forceinline__ void mfma_first(f32x16& c, s16x8 a, s16x8 b) {
  if (__is_same(T, __bf16)) asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(c) : "v"(a), "v"(b));
  else asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_f16 %0, %1, %2, 0" : "=&v"(c) : "v"(a), "v"(b));
}
template <typename T>
__device__ __forceinline__ void mfma_next(f32x16& c, s16x8 a, s16x8 b) {
  if (__is_same(T, __bf16)) asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "v"(b));
  else asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_done(f32x16& c) { asm volatile("s_nop 15\n\ts_nop 3" : "+v"(c)); }
__device__ __forceinline__ void mfma_done(f32x16& a, f32x16& b) { asm volatile("s_nop 15\n\ts_nop 3" : "+v"(a), "+v"(b)); }

template <typename T>
__device__ __forceinline__ s16x8 to_half(const float* x) {
  typedef T T8 __attribute__((ext_vector_type(8)));
  T8 y;
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = static_cast<T>(x[i]);
  return __builtin_bit_cast(s16x8, y);
}

// c *= f with c in accumulator registers throughout, which vector instructions
// do not take: the plain product makes the compiler move and spill all of the
// latent attention's sums at every step, though few steps need it.  The first wait
// lets products that write c end, the last keeps the next one off a register just
// written.
__device__ __forceinline__ void scale_accumulators(f32x16& c, float f) {
  asm volatile("s_nop 15\n\ts_nop 3" : "+a"(c));
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    float x = c[e], y;
    asm volatile("v_accvgpr_read_b32 %1, %0\n\ts_nop 1\n\tv_mul_f32 %1, %1, %2\n\ts_nop 1\n\tv_accvgpr_write_b32 %0, %1" : "+a"(x), "=&v"(y) : "v"(f));
    c[e] = x;
  }
  asm volatile("s_nop 3" : "+a"(c));
}

#define BSR_INLINE __attribute__((always_inline))
#define BSR_LDS __attribute__((address_space(3)))
__device__ __forceinline__ uint32_t lds_at(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((BSR_LDS const uint8_t*)p));
}

// 64 lanes x 16 bytes from memory to LDS, lane after lane from `lds` on
// (wave-uniform), past the registers.  The compiler does not see it: it is waited
// for by loads_done, and every reader lies behind that and a barrier.
__device__ __forceinline__ void load_to_lds(const uint8_t* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(src) : "memory", "m0");
}
// The same from a scalar address plus a lane's offset.  (A load must not follow
// closely on a vector instruction that wrote its scalar address, and the compiler
// sees no load here: the address comes from two scalar additions.)
__device__ __forceinline__ void load_to_lds(const uint8_t* base, uint32_t lo, uint32_t hi, uint32_t offset, uint32_t lds) {
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  uint32_t x, y;
  asm volatile("s_add_u32 %0, %2, %4\n\ts_addc_u32 %1, %3, %5"
               : "=&s"(x), "=s"(y)
               : "s"(static_cast<uint32_t>(b)), "s"(static_cast<uint32_t>(b >> 32)), "s"(lo), "s"(hi)
               : "scc");
  const uint64_t at = static_cast<uint64_t>(y) << 32 | x;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(at) : "memory", "m0");
}
// 64 lanes x 4 bytes likewise.
__device__ __forceinline__ void load_words_to_lds(const void* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(src) : "memory", "m0");
}
// Waits until at most `left` of the wave's loads are under way (they end in order).
template <int left = 0>
__device__ __forceinline__ void loads_done() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(left) : "memory");
}
__device__ __forceinline__ void barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ s16x8 lds_row16(uint32_t at) {
  return *(const BSR_LDS s16x8*)(uintptr_t)at;
}
// Transposed read: every 16 lanes read a block of four rows (keys) of 16
// 16-bit values, lane i the four at row i / 4, column 4 (i % 4); lane i gets column i.
__device__ __forceinline__ s16x4 lds_columns(uint32_t at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((BSR_LDS s16x4*)(uintptr_t)at);
}

// A lane's value and that of the same lane of the other half, in either order.
struct Halves {
  float a, b;
};
__device__ __forceinline__ Halves halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ float max_halves(float x) {
  const Halves h = halves(x);
  return fmaxf(h.a, h.b);
}
__device__ __forceinline__ float sum_halves(float x) {
  const Halves h = halves(x);
  return h.a + h.b;
}

// A wave's 32 query rows, one per lane of either half.
struct TileRows {
  bool real;         // the row exists
  int i;             // of the request
  uint32_t head;
  Row see;
  float slope2;      // slope x log2(e)
};

__device__ __forceinline__ TileRows tile_row(const AttnParams& p, const Request& q, const Work& w, uint32_t row) {
  TileRows t;
  const uint32_t per_kv = p.n_heads / p.n_kv_heads, chunks = p.units / p.n_kv_heads;
  const uint32_t kv = w.unit / chunks, chunk = w.unit - kv * chunks;
  const uint32_t tok = row / p.tile_heads, hd = chunk * p.tile_heads + row - tok * p.tile_heads;
  t.i = static_cast<int>(w.tile * p.tile_tokens + tok);
  t.real = tok < p.tile_tokens && hd < per_kv && t.i < q.rows;
  t.head = kv * per_kv + hd;
  t.see = Row{0x7fffffff, 0, 0, nullptr};
  t.slope2 = 0;
  if (t.real) {
    t.see = row_of(p, q, w.r, t.i);
    t.see.lo = max(t.see.lo, 0);
    t.see.hi = min(t.see.hi, q.n);
    if (p.slopes) t.slope2 = p.slopes[t.head] * kLog2e;
  }
  return t;
}

__device__ __forceinline__ int wave_min(int x) {
  for (int d = 32; d; d >>= 1) x = min(x, __shfl_xor(x, d));
  return x;
}
__device__ __forceinline__ int wave_max(int x) {
  for (int d = 32; d; d >>= 1) x = max(x, __shfl_xor(x, d));
  return x;
}

// Scores (times log2(e)) of a lane's keys j0 + 8 (e / 4) + e % 4, j0 = the
// first key of the 32 plus 4 h, from their products.  Without cap and bias the
// products stay as they are, and `unit` (scale x log2(e)) goes into the exponent.
constexpr int kCap = 1, kSlopes = 2;  // what is done to a score
struct ScoreMods {
  float unit;       // scale x log2(e)
  float cap2;       // softcap x log2(e), 0 without
  float in_cap;     // 2 log2(e) scale / softcap: tanh(x) = 1 - 2 / (2^(2 x log2 e) + 1)
  float over;       // scale / softcap where the cap is wide, else 0
  bool ahead;       // rows see keys behind their own position
};
// That tanh is off by 2^-23 or so however small x is, which a cap c makes c 2^-23 or
// more of a score: from here on scores below 0.4 c take the first terms of its
// series (the next one is 0.0036 x^12, under 2^-23).  8 trees of 64 nodes behind 9,000
// tokens, 32 heads: 67.5 us with a cap of 64, 78.2 with one of 100.
constexpr float kWideCap = 64;

__device__ __forceinline__ ScoreMods score_mods(const AttnParams& p) {
  ScoreMods m;
  m.unit = p.scale * kLog2e;
  m.cap2 = p.softcap * kLog2e;
  m.in_cap = p.softcap > 0 ? 2 * kLog2e * (p.scale / p.softcap) : 0;
  m.over = p.softcap > kWideCap ? p.scale / p.softcap : 0;
  m.ahead = p.prefix != nullptr;
  return m;
}

template <int kMods>
__device__ __forceinline__ void modify(const ScoreMods& m, float slope2, int pos, int j0, f32x16& s) {
  if (kMods & kCap) {
    if (m.cap2 > kWideCap * kLog2e) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float z = s[e] * m.over, z2 = z * z;
        float y = __builtin_fmaf(z2, -1382.0f / 155925, 62.0f / 2835);
        y = __builtin_fmaf(z2, y, -17.0f / 315);
        y = __builtin_fmaf(z2, y, 2.0f / 15);
        y = __builtin_fmaf(z2, y, -1.0f / 3);
        const float x = s[e] * m.unit;
        const float far = m.cap2 - 2 * m.cap2 * __builtin_amdgcn_rcpf(exp2_(s[e] * m.in_cap) + 1);
        s[e] = fabsf(z) < 0.4f ? __builtin_fmaf(x, z2 * y, x) : far;
        if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // (all at once take more registers than there are)
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[e] = m.cap2 - 2 * m.cap2 * __builtin_amdgcn_rcpf(exp2_(s[e] * m.in_cap) + 1);
        if (e % 8 == 7) __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  if (!(kMods & kSlopes)) return;
  const float unit = kMods & kCap ? 1.0f : m.unit, away = static_cast<float>(pos - j0);
  if (m.ahead) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      s[e] = __builtin_fmaf(-slope2, fabsf(away - static_cast<float>(8 * (e / 4) + e % 4)), s[e] * unit);
  } else {  // two instructions a score: the distance of a key that is seen has one sign
    const float from = -slope2 * away;
#pragma unroll
    for (int e = 0; e < 16; ++e)
      s[e] = __builtin_fmaf(s[e], unit, __builtin_fmaf(slope2, static_cast<float>(8 * (e / 4) + e % 4), from));
  }
}

// The running maximum m follows a rise of more than kRise (weights grow by up to
// 2^8 until then, which the sums in fp32 and the weights in 16 bits hold alike):
// past a row's first steps its sums are rescaled hardly ever.  Following every
// rise: 16 latent trees of 8 nodes 179 us for 94, causal 8192 382 for 372.
//
// m is the maximum less kLift, so that the largest weight is 2^kLift.  fp16's
// weights are rounded to steps of 2^-24 at the least: with 1 for the largest, a key
// below half of one would count for nothing, though enough of them matter (each off by
// 2^-25 of the sum, 2^17 of them by 2^-8).  With 2^7 to 2^15 (65,504 is the
// type's most) a key is off by 2^-32 of the sum, 2^20 of them by 2^-12.  The same
// trees in fp16: 87 us with a lift of 0 or 7; 90 with a lift of 9 and a
// rise of 6, 100 with 11 and 4, which leave less.
constexpr float kRise = 8;
template <typename T>
constexpr float kLift = __is_same(T, _Float16) ? 7 : 0;

// The compiler's own maximum first multiplies each operand by one, against a
// signalling NaN: half of the instructions of a maximum (rows that meet a NaN are
// done again).  It does not know that this reads a matrix product's result:
// mfma_done or modify comes before.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float x;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(x) : "v"(a), "v"(b), "v"(c));
  return x;
}

// The running maximum m and sum l of a lane's row after 16 kSubs more scores
// (`unit` is what is left to multiply them by).  Returns whether any row of the
// wave rescales what it has summed, and the lane's factor in *back.
template <typename T, int kSubs>
__device__ __forceinline__ bool raise(const f32x16 (&s)[kSubs], float unit, float& m, float& l, float* back) {
  float tops[4];  // four in a row, since each waits for the last one of its own
#pragma unroll
  for (int i = 0; i < 4; ++i) tops[i] = max3(s[0][i], s[0][4 + i], s[0][8 + i]);
#pragma unroll
  for (int e = 12; e < 16 * kSubs; e += 8)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = e + 4 < 16 * kSubs ? e + 4 : e;
      tops[i] = max3(tops[i], s[e / 16][e % 16 + i], s[n / 16][n % 16 + i]);
    }
  const float top = max_halves(fmaxf(max3(tops[0], tops[1], tops[2]), tops[3])) * unit;
  *back = 1;
  if (!__any(top > m + (kLift<T> + kRise))) return false;
  const float m1 = fmaxf(m, top - kLift<T>);
  *back = m > -__builtin_inff() ? exp2_(m - m1) : 0.0f;
  l *= *back;
  m = m1;
  return true;
}

// 16 scores to weights, and their sum.
__device__ __forceinline__ float weigh(f32x16& s, float unit, float from) {
  float sum[2] = {};
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    s[e] = exp2_(__builtin_fmaf(s[e], unit, -from));
    sum[e & 1] += s[e];
  }
  return sum[0] + sum[1];
}

// A score where bit n of `see` is set, else -infinity.
__device__ __forceinline__ float seen(float s, uint32_t see, int n) {
  const int keep = static_cast<int>(see << (31 - n)) >> 31;
  return __uint_as_float((__float_as_uint(s) & keep) | (0xff800000u & ~keep));
}

// Where a tile's row goes: the output, or a partial result.
struct Sink {
  bool part;
  uint32_t slot;
};

template <typename T>
__device__ __forceinline__ void put4(const AttnParams& p, const Request& q, const TileRows& t, const Sink& k, uint32_t row,
                                     uint32_t d, f32x4 x) {
  if (k.part) {
    *reinterpret_cast<f32x4*>(p.part + (static_cast<uint64_t>(k.slot) * p.tile_rows + row) * p.v_dim + d) = x;
  } else {
    typedef T T4 __attribute__((ext_vector_type(4)));
    T4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = static_cast<T>(x[i]);
    *reinterpret_cast<T4*>(p.out + (q.first + t.i) * p.out_token + t.head * p.out_head + d * sizeof(T)) = y;
  }
}

__device__ __forceinline__ void put_stats(const AttnParams& p, const Request& q, const TileRows& t, const Sink& k,
                                          uint32_t row, float m, float l) {
  if (k.part) {
    float* at = p.part_ml + (static_cast<uint64_t>(k.slot) * p.tile_rows + row) * 2;
    at[0] = m;
    at[1] = l;
  } else if (p.lse) {
    p.lse[static_cast<uint64_t>(q.first + t.i) * p.n_heads + t.head] = l == 0 ? -__builtin_inff() : (m + __log2f(l)) * kLn2;
  }
}

// Rows whose result is not finite saw an infinity or a NaN, or it lay where they
// see nothing and met a weight of zero: these are done again over the keys
// [lo, hi), reading what they see alone.
template <typename T, int KD, int VD>
__device__ void redo_row(const AttnParams& p, const Request& q, const Work& w, const Sink& k, uint32_t row, int lo, int hi) {
  constexpr int kPer = VD / 64;
  const TileRows t = tile_row(p, q, w, row);
  if (!t.real) return;
  float m, l, acc[kPer];
  attend_row<T, KD, VD>(p, q, t.see, t.i, t.head, max(lo, t.see.lo), min(hi, t.see.hi), m, l, acc);
  const uint32_t d0 = (threadIdx.x & 63) * kPer;
  for (int d = 0; d < kPer; ++d) {
    if (k.part) p.part[(static_cast<uint64_t>(k.slot) * p.tile_rows + row) * VD + d0 + d] = acc[d];
    else
      reinterpret_cast<T*>(p.out + (q.first + t.i) * p.out_token + t.head * p.out_head)[d0 + d] =
          static_cast<T>(l == 0 ? 0.0f : acc[d] / l);
  }
  if ((threadIdx.x & 63) == 0) put_stats(p, q, t, k, row, m, l);
}

// ---------------------------------------------------------------------------
// KV heads of 64 or 128: four waves of 32 query rows each, 64 keys a step.
//
// S^T = K Q^T, so a lane holds one query row's scores of 32 keys: the softmax
// stays in the lane but for one exchange with the other half.  The
// weights then are the B operand of O^T = V^T P^T as they lie, since the order
// of the keys within a product is free: lane half h takes keys 4 h .. 4 h + 3
// and 8 + 4 h .. of every 16, and V^T, read transposed from LDS, follows.
// O^T keeps a query row per lane too, so rescaling is a product with a lane's
// own factor.
//
// K and V lie in LDS row by row, their 16-byte units permuted by the row, so
// that neither the reads of 16 rows at one place nor the transposed reads of 8
// rows meet in a bank (no conflict is counted).  Two buffers: step t + 1 is loaded,
// past the registers, while t is computed.
//
// The weights are rounded to T for the products with V: products of fp32 run at a
// sixteenth of the rate, and two halves of a weight would double the products.  It
// costs at most 2^-8 (fp16 2^-11) of a row's sum of weight x |value|; measured, off from 64
// bits by 0.0019-0.0024 for 0.0016-0.0017 with weights in fp32 (bf16, whose result alone is
// rounded by as much), 2.7e-4 for 2.1e-4 (fp16).
//
// Heads of 128 leave registers for 2 workgroups a CU, heads of 64 for 3 (which with a
// cap spill 15 to 21 registers).  What bounds it: with many rows the matrix and
// the vector unit in turn (a step's 32 products of a wave take 1,090 cycles, its 32
// scores a lane some 900 without mask, cap or bias), and the clock, 1.8 GHz under this
// load; with few rows the cache's bytes; in between neither, but too few waves at
// work: ramps, uneven tiles, waves without rows.  1,024 tokens of 16 heads behind
// 128K: 1,110-1,170 us, 940-990 TFLOP/s (vector unit busy 55% of the time, matrix
// unit 48%, 1.7 of 2 waves a SIMD); one token of 32 heads over 128K: 115 us with the
// join, 4.7 TB/s; 8 trees of 64 nodes, 32 heads, capped, over 9,000: 52-54 us
// (35%, 15%, 1.3 of 2); 10.7K packed tokens of 16 heads of 64 with a bias: 50 us (41%,
// 11%, 1.5 of 3; 5.4 steps a tile, behind some 6 us to the first).
// ---------------------------------------------------------------------------
constexpr int kAttnThreads = 256;

template <int D>
__device__ __forceinline__ uint32_t unit_swap(uint32_t row) {
  if (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
  return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

template <typename T, int D, int kMods>
__global__ __launch_bounds__(kAttnThreads, D == 64 ? 3 : 2) void k_attend_heads(AttnParams p) {
  constexpr int kStep = 64, kUnits = D / 8, kTileBytes = kStep * D * 2;
  constexpr int kRowsPerLoad = 64 / kUnits, kLoads = kStep / 4 / kRowsPerLoad;  // per wave, K and V each
  __shared__ __attribute__((aligned(1024))) uint8_t kv_tiles[2][2][kTileBytes];
  __shared__ int64_t offsets[2][kStep];
  __shared__ uint64_t outside[4];
  __shared__ int ranges[4];

  Work w;
  Request q;
  if (!find_work<false>(p, blockIdx.x, &w, &q)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const uint32_t kv = w.unit / (p.units / p.n_kv_heads);
  const uint32_t row = wave * 32 + col;
  const TileRows t = tile_row(p, q, w, row);
  const bool active = __any(t.real);
  // keys that all of the wave's rows see without a look at their masks
  const int open_lo = uniform(wave_max(t.real ? t.see.lo : 0));
  const int open_hi = uniform(wave_min(!t.real ? 0x7fffffff : p.tree ? min(t.see.hi, q.base) : t.see.hi));
  const int wave_lo = wave_min(t.see.lo);
  int lo, hi, k0, k1;
  tile_range(p, q, w, &lo, &hi);
  if (p.documents) {  // a tile of late documents starts late
    if (lane == 0) ranges[wave] = wave_lo;
    barrier();
    lo = uniform(max(lo, min(min(ranges[0], ranges[1]), min(ranges[2], ranges[3]))));
  }
  cut(w, lo, hi, &k0, &k1);
  const int steps = (k1 - k0 + kStep - 1) / kStep;

  f32x16 o[D / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d) o[d] = f32x16{};
  float m = -__builtin_inff(), l = 0;
  const ScoreMods mods = score_mods(p);

  const uint8_t* k_base = p.k_pool + kv * (2 * D);
  const uint8_t* v_base = p.v_pool + kv * (2 * D);
  const uint32_t tiles_at = lds_at(&kv_tiles[0][0][0]);
  // loading: the wave's rows of a step, kRowsPerLoad at a time
  const uint32_t load_row = wave * (kStep / 4) + lane / kUnits;
  auto load_part = [&](int i, int buf, int64_t at) BSR_INLINE {  // load i of 2 kLoads: keys, then values of the same rows
    const int n = i / 2;
    const int64_t off = at + (((lane % kUnits) ^ unit_swap<D>(load_row + n * kRowsPerLoad)) * 16);
    const uint32_t to = tiles_at + buf * (2 * kTileBytes) + (wave * (kStep / 4) + n * kRowsPerLoad) * (D * 2);
    load_to_lds((i & 1 ? v_base : k_base) + off, to + (i & 1) * kTileBytes);
  };
  auto offset_at = [&](int slot, int i) BSR_INLINE { return offsets[slot][load_row + i / 2 * kRowsPerLoad]; };
  auto load_step = [&](int buf, int slot) BSR_INLINE {
#pragma unroll
    for (int i = 0; i < 2 * kLoads; ++i) load_part(i, buf, offset_at(slot, i));
  };
  KeyLoad next{}, k_first{}, k_second{};
  if (wave == 0 && steps > 0) {  // (steps past the last read its last key's block id)
    k_first = key_load(p, q, k0 + lane, k1 - 1);
    k_second = key_load(p, q, k0 + kStep + lane, k1 - 1);
    next = key_load(p, q, k0 + 2 * kStep + lane, k1 - 1);
  }
  s16x8 qf[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    qf[s] = s16x8{};
    if (t.real)
      qf[s] = *reinterpret_cast<const s16x8*>(p.q + (q.first + t.i) * p.q_token + t.head * p.q_head + s * 32 + half * 16);
  }
  auto put_offsets = [&](int step, const KeyLoad& k) BSR_INLINE {  // by wave 0
    int64_t off;
    const bool ok = key_offset(p, k, &off);
    offsets[step & 1][lane] = off;
    const uint64_t bad = ~__ballot(ok);
    if (lane == 0) outside[step & 3] = bad;
  };
  if (steps > 0) {
    if (wave == 0) {
      put_offsets(0, k_first);
      put_offsets(1, k_second);
    }
    barrier();
    load_step(0, 0);
  }

  // read positions: K, row col of 32; V transposed, row 4 h + (lane % 16) / 4
  const uint32_t k_at = col * (D * 2), k_swap = unit_swap<D>(col);
  const uint32_t v_row = 4 * half + ((lane & 15) >> 2);
  const uint32_t v_unit = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  uint32_t v_at[2];
#pragma unroll
  for (int e = 0; e < 2; ++e)
    v_at[e] = (v_row + 8 * e) * (D * 2) + ((v_unit ^ unit_swap<D>(v_row + 8 * e)) * 16) + (lane & 1) * 8;

  // waits for a step, and sends the loads of the next
  auto turn = [&](int step, bool load) BSR_INLINE {
    loads_done();
    barrier();
    const int buf = step & 1;
    if (wave == 0) put_offsets(step + 2, next);  // (of the last key, past the last step)
    if (load && step + 1 < steps) load_step(buf ^ 1, buf ^ 1);
    if (wave == 0) next = key_load(p, q, k0 + (step + 3) * kStep + lane, k1 - 1);
  };
  // a wave without rows loads its share all the same (in a loop of its own: a
  // way round the sums' products would have them copied at every step)
  if (!active)
    for (int step = 0; step < steps; ++step) turn(step, true);
  else
  for (int step = 0; step < steps; ++step) {
    turn(step, false);
    const int buf = step & 1, j0 = k0 + step * kStep;
    const uint32_t k_tile = tiles_at + buf * (2 * kTileBytes), v_tile = k_tile + kTileBytes;
    constexpr int kN = D / 16, kD = D / 32;
    auto k_row = [&](int u, int n) BSR_INLINE {
      return lds_row16(k_tile + u * 32 * (D * 2) + k_at + (((2 * n + half) ^ k_swap) * 16));
    };
    // values of 16 keys g, dimensions 32 d ..
    auto v_cols = [&](int g, int d) BSR_INLINE {
      const uint32_t at = v_tile + 16 * g * (D * 2);
      const s16x4 a = lds_columns(at + (v_at[0] ^ (d * 64))), b = lds_columns(at + (v_at[1] ^ (d * 64)));
      return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // reads of LDS run kAhead products ahead, into the registers that a product has
    // just left; the first values are read before the softmax
    constexpr int kAhead = 4;
    f32x16 s[2] = {};
    s16x8 kf[kAhead], vf[kD];
    int64_t off[2];
    off[0] = offset_at(buf ^ 1, 0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) kf[i] = k_row(i % 2, i / 2);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 2 * kN; ++i) {
      s[i % 2] = mfma<T>(kf[i % kAhead], qf[i / 2], s[i % 2]);
      if (i + kAhead < 2 * kN) kf[i % kAhead] = k_row((i + kAhead) % 2, (i + kAhead) / 2);
      else if (i + kAhead - 2 * kN < kD) vf[i + kAhead - 2 * kN] = v_cols(0, i + kAhead - 2 * kN);
      // the next step's loads (past the last step, of its last key's record), one
      // beside every second product: a load holds its wave up
      if (i % 2 == 0 && i / 2 < 2 * kLoads) {
        load_part(i / 2, buf ^ 1, off[i / 4 % 2]);
        if (i % 4 == 0 && i / 4 + 1 < kLoads) off[(i / 4 + 1) % 2] = offset_at(buf ^ 1, i / 2 + 2);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    float unit = mods.unit;
    if (!kMods) {
      mfma_done(s[0], s[1]);
    } else {
      unit = 1;
#pragma unroll
      for (int u = 0; u < 2; ++u) modify<kMods>(mods, t.slope2, t.see.pos, j0 + 32 * u + 4 * half, s[u]);
    }
    const uint64_t bad = uniform(outside[step & 3]);
    if (j0 < open_lo || j0 + kStep > open_hi || bad || j0 + kStep > k1) {
      uint64_t see = bit_range(t.see.lo - j0, min(t.see.hi, k1) - j0) & ~bad;
      if (p.tree && t.real) see &= tree_bits(p, t.see.mask, j0 - q.base);
      see >>= 4 * half;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[u][e] = seen(s[u][e], static_cast<uint32_t>(see >> (32 * u)), 8 * (e / 4) + e % 4);
    }
    float back;
    if (raise<T, 2>(s, unit, m, l, &back)) {
#pragma unroll
      for (int d = 0; d < kD; ++d) o[d] *= back;
    }
    const float from = m > -__builtin_inff() ? m : 0.0f;
#pragma unroll
    for (int g = 0; g < 4; ++g) {  // 16 keys each
      if (g % 2 == 0) l += weigh(s[g / 2], unit, from);
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = s[g / 2][8 * (g % 2) + e];
      const s16x8 pf = to_half<T>(x);
#pragma unroll
      for (int d = 0; d < kD; ++d) {
        o[d] = mfma<T>(vf[d], pf, o[d]);
        if (g < 3) vf[d] = v_cols(g + 1, d);
      }
    }
  }

  loads_done();  // none may reach LDS that is no longer the workgroup's
  const Sink sink{w.n_splits > 1, w.slot + w.split};
  l = sum_halves(l);
  const float inv = sink.part ? 1.0f : l == 0 ? 0.0f : 1.0f / l;
  float zero = 0;  // NaN where a result is not finite
#pragma unroll
  for (int d = 0; d < D / 32; ++d) {
    o[d] *= inv;
#pragma unroll
    for (int e = 0; e < 16; ++e) zero += o[d][e] * 0.0f;
  }
  zero = sum_halves(zero) + l * 0.0f;
  const bool again = t.real && !(zero == 0);
  const uint32_t mine = static_cast<uint32_t>(__ballot(again));
  if (t.real && !again) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        put4<T>(p, q, t, sink, row, 32 * d + 8 * e + 4 * half, f32x4{o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]});
    if (half == 0) put_stats(p, q, t, sink, row, m, l);
  }
  for (uint32_t left = mine; left; left &= left - 1)
    redo_row<T, D, D>(p, q, w, sink, wave * 32 + __builtin_ctz(left), k0, k1);
}

// ---------------------------------------------------------------------------
// Latent records of 576, the first 512 the value: one tile serves K and V.
//
// Four waves; 32 keys a step.  Wave w scores query rows 32 w .. 32 w + 31, its
// queries in registers, and leaves their weights in LDS; then it sums values
// 128 w .. 128 w + 127 of all 128 rows, so that a record is read for the products
// with V once.  Scores of step t + 1 and values of step t share a stretch between
// two barriers, and steps t + 2 on are loaded meanwhile.
//
// The sums of 128 rows are 256 accumulator registers, so a CU holds one
// workgroup; tiles of 32 or 64 rows (kBlocks 1, 2) score with one or two waves and
// have a buffer more.  What bounds it: a step of 128 rows takes 5,000 cycles, of
// which the products 2,310; a load holds its wave 80 cycles, 9 of them a step, and
// the softmax of a step has only the products of the step before beside it.  4
// nodes of 128 heads over 512K: 607-615 us with the join, 950-960 TFLOP/s (vector unit busy
// 22% of the time, matrix unit 41%); 16 trees of 8 nodes, 16 heads, over up to 33K: 79-82
// us, 3.2-3.3 TB/s (18%, 24%, 0.76 of a wave a SIMD); one token of 16 heads over 1,000:
// 12-13 us, of which 6 until the first records are there.  Tiles of 128 rows
// spill 5 vector registers, 27 with cap and bias.
// ---------------------------------------------------------------------------
template <typename T, int kMods, int kBlocks>
__global__ __attribute__((amdgpu_waves_per_eu(1, 1))) __launch_bounds__(kAttnThreads, 1) void k_attend_latent(AttnParams p) {
  constexpr int KD = 576, VD = 512, kStep = 32, kTileBytes = kStep * KD * 2;
  // LDS of a step: the eight records of each wave, their values (1,024 bytes
  // each) and then the rest of their keys (128 bytes each), so that a load of 64
  // lanes takes a record's values, at a scalar address, or the rest of all eight
  constexpr int kValueBytes = VD * 2, kRestBytes = (KD - VD) * 2, kWaveBytes = kTileBytes / 4;
  // steps loaded or in use at once: three where there is LDS for no more
  constexpr int kBufs = kBlocks == 4 ? 3 : 4, kLoads = 9;  // of a wave and step
  constexpr int kKeys = kStep / 4, kIdSteps = 64 / kKeys;  // keys that a wave loads at a step; steps of one load of block ids
  constexpr int kN = KD / 16, kAhead = 5;
  constexpr int kHeld = kBlocks == 4 ? 32 : kN;  // products whose queries lie in registers; the others' are read from LDS
  __shared__ __attribute__((aligned(1024))) uint8_t tiles[kBufs][kTileBytes];
  __shared__ __attribute__((aligned(16))) uint8_t weights[2][kBlocks][2][1024];  // [step][rows / 32][16 keys][lane]
  __shared__ float backs[2][32 * kBlocks];
  __shared__ __attribute__((aligned(16))) uint32_t rises[2][4];
  __shared__ float stats[2][32 * kBlocks];
  __shared__ __attribute__((aligned(16))) uint8_t queries[kBlocks == 4 ? 4 : 1][kN - kHeld + 1][1024];  // [wave][n - kHeld][lane]
  __shared__ int32_t block_ids[4][2][64];
  __shared__ __attribute__((aligned(4))) uint8_t outside[8][4];
  __shared__ int ranges[4];
  __shared__ uint32_t redo[4];

  Work w;
  Request q;
  if (!find_work<false>(p, blockIdx.x, &w, &q)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const bool scores = kBlocks == 4 || wave < kBlocks;  // waves with query rows of their own
  const uint32_t row = wave * 32 + col;
  const TileRows t = tile_row(p, q, w, row);
  const int open_lo = uniform(wave_max(t.real ? t.see.lo : 0));
  const int open_hi = uniform(wave_min(!t.real ? 0x7fffffff : p.tree ? min(t.see.hi, q.base) : t.see.hi));
  const int wave_lo = wave_min(t.see.lo);
  if (lane == 0) {
    rises[0][wave] = rises[1][wave] = 0;
    redo[wave] = 0;
    for (int i = 0; i < 8; ++i) outside[i][wave] = 0;
  }
  int lo, hi, k0, k1;
  tile_range(p, q, w, &lo, &hi);
  if (p.documents) {  // a tile of late documents starts late
    if (lane == 0) ranges[wave] = wave_lo;
    barrier();
    lo = uniform(max(lo, min(min(ranges[0], ranges[1]), min(ranges[2], ranges[3]))));
  }
  cut(w, lo, hi, &k0, &k1);
  const int steps = (k1 - k0 + kStep - 1) / kStep;

  s16x8 qf[kHeld];
  f32x16 o[kBlocks][4];
#pragma unroll
  for (int b = 0; b < kBlocks; ++b)
#pragma unroll
    for (int d = 0; d < 4; ++d) o[b][d] = f32x16{};
  float m = -__builtin_inff(), l = 0;
  const ScoreMods mods = score_mods(p);

  const uint32_t tiles_at = lds_at(&tiles[0][0]), weights_at = lds_at(&weights[0][0][0][0]);
  // A wave loads keys 8 wave .. 8 wave + 7 of a step, and their block ids
  // kIdSteps steps at a time: it waits for its own loads alone.
  auto key_at = [&](int step, int key) BSR_INLINE { return min(k0 + step * kStep + wave * kKeys + key, k1 - 1); };
  auto load_ids = [&](int first_step) BSR_INLINE {
    const int j = key_at(first_step + lane / kKeys, lane % kKeys);
    load_words_to_lds(q.table + p.div_block.div(j), lds_at(&block_ids[wave][first_step / kIdSteps & 1][0]));
  };
  // The offset of the lane's record, key lane % 8 of a step, in strides (the block
  // id is read from LDS, the others are a few instructions each).
  KeyLoad key{};
  int64_t offset = 0;
  bool marks = false;
  auto find_offset = [&](int step, int stride) BSR_INLINE {
    if (stride == 0) key.id = block_ids[wave][step / kIdSteps & 1][step % kIdSteps * kKeys + lane % kKeys];
    if (stride == 1) key.j = key_at(step, lane % kKeys);
    if (stride == 2) key.block = p.div_block.div(key.j);
    if (stride == 3) {
      const uint32_t bad = static_cast<uint8_t>(~__ballot(key_offset(p, key, &offset)));
      marks |= bad != 0;  // nothing is written before the first block that lies outside
      if (marks && lane == 0) outside[step & 7][wave] = static_cast<uint8_t>(bad);
    }
  };
  // load n of a step: the values of record n, or the rest of all; units of 16
  // bytes are permuted by the record's row
  auto load_unit = [&](int n, int buf) BSR_INLINE {
    const uint32_t to = tiles_at + buf * kTileBytes + wave * kWaveBytes + n * 1024;
    const uint32_t lo = static_cast<uint32_t>(offset), hi = static_cast<uint32_t>(offset >> 32);
    if (n < kKeys) {
      load_to_lds(p.k_pool, __builtin_amdgcn_readlane(lo, n), __builtin_amdgcn_readlane(hi, n),
                  (lane ^ unit_swap<128>(wave * kKeys + n)) * 16, to);
    } else {
      const int r = lane >> 3;
      const uint64_t off = static_cast<uint64_t>(__shfl(hi, r)) << 32 | __shfl(lo, r);
      load_to_lds(p.k_pool + off + kValueBytes + (((lane & 7) ^ unit_swap<64>(wave * kKeys + r)) * 16), to);
    }
  };
  auto load_step = [&](int buf) BSR_INLINE {
#pragma unroll
    for (int n = 0; n < kLoads; ++n) load_unit(n, buf);
  };

  // read positions: the key of row col, 8 dimensions of it; four values of row
  // 4 h + (lane % 16) / 4, transposed
  const uint32_t k_at = (col >> 3) * kWaveBytes + (col & 7) * kValueBytes + ((half ^ unit_swap<128>(col)) * 16);
  const uint32_t k_rest = (col >> 3) * kWaveBytes + kKeys * kValueBytes + (col & 7) * kRestBytes + ((half ^ unit_swap<64>(col)) * 16);
  const uint32_t v_row = 4 * half + ((lane & 15) >> 2);
  const uint32_t v_unit = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  uint32_t v_at[2];
#pragma unroll
  for (int e = 0; e < 2; ++e)
    v_at[e] = e * kWaveBytes + v_row * kValueBytes + wave * 256 + ((v_unit ^ unit_swap<128>(v_row + 8 * e)) * 16) + (lane & 1) * 8;

  // Products of the wave's rows with the 32 keys in buffer `buf`.  Reads of LDS run
  // kAhead products ahead; beside(n) goes on beside them, after() while the last
  // ones end; the order is pinned.
  auto score = [&](int buf, f32x16& s, auto beside, auto after) BSR_INLINE {
    const uint32_t at = tiles_at + buf * kTileBytes;
    auto k_row = [&](int n) BSR_INLINE {
      return n < VD / 16 ? lds_row16(at + (k_at ^ (n % 8 * 32)) + n / 8 * 256) : lds_row16(at + (k_rest ^ ((n - VD / 16) * 32)));
    };
    s16x8 kf[kAhead], q_next{};
#pragma unroll
    for (int n = 0; n < kAhead; ++n) kf[n] = k_row(n);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      if (n == 0) mfma_first<T>(s, kf[n], qf[n]);
      else mfma_next<T>(s, kf[n % kAhead], n < kHeld ? qf[n < kHeld ? n : 0] : q_next);
      if (n + 1 >= kHeld && n + 1 < kN) q_next = *reinterpret_cast<const s16x8*>(&queries[wave][n + 1 - kHeld][lane * 16]);
      if (n + kAhead < kN) kf[n % kAhead] = k_row(n + kAhead);
      beside(n);
      __builtin_amdgcn_sched_barrier(0);
    }
    after();
    __builtin_amdgcn_sched_barrier(0);
    mfma_done(s);
  };
  auto outside_of = [&](int step) BSR_INLINE { return uniform(*reinterpret_cast<const uint32_t*>(&outside[step & 7][0])); };
  // their scores, what the rows see of them, and the running maximum
  auto settle = [&](int step, f32x16 (&s)[1], float* unit, uint32_t bad) BSR_INLINE {
    const int j0 = k0 + step * kStep;
    *unit = mods.unit;
    if (kMods) {
      *unit = 1;
      modify<kMods>(mods, t.slope2, t.see.pos, j0 + 4 * half, s[0]);
    }
    if (j0 < open_lo || j0 + kStep > open_hi || bad || j0 + kStep > k1) {
      uint64_t see = bit_range(t.see.lo - j0, min(t.see.hi, k1) - j0) & ~static_cast<uint64_t>(bad);
      if (p.tree && t.real) see &= tree_bits(p, t.see.mask, j0 - q.base);
      see >>= 4 * half;
#pragma unroll
      for (int e = 0; e < 16; ++e)
        s[0][e] = seen(s[0][e], static_cast<uint32_t>(see), 8 * (e / 4) + e % 4);
    }
    float back;
    const bool rise = raise<T, 1>(s, *unit, m, l, &back);
    if (rise && half == 0) backs[step & 1][row] = back;
    if (lane == 0) rises[step & 1][wave] = rise;
  };
  // scores [from, to) to weights; each eight of them then go to LDS
  auto leave_weights = [&](int step, f32x16& s, float unit, float base, int from, int to) BSR_INLINE {
#pragma unroll
    for (int e = from; e < to; ++e) {
      s[e] = exp2_(__builtin_fmaf(s[e], unit, -base));
      l += s[e];
      if (e % 8 != 7) continue;
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = s[e - 7 + i];
      *(BSR_LDS s16x8*)(uintptr_t)(weights_at + (((step & 1) * kBlocks + wave) * 2 + e / 8) * 1024 + lane * 16) = to_half<T>(x);
    }
  };
  auto rescale = [&](int step) BSR_INLINE {
    const u32x4 rise = *reinterpret_cast<const u32x4*>(&rises[step & 1][0]);
    if (!uniform(rise[0] | rise[1] | rise[2] | rise[3])) return;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
      if (uniform(rise[b])) {
        const float back = backs[step & 1][b * 32 + col];
#pragma unroll
        for (int d = 0; d < 4; ++d) scale_accumulators(o[b][d], back);
      }
  };
  // The value products of a step, 8 kBlocks of them: 16 keys g, 32 dimensions d, 32
  // rows b, the last fastest.  The weights of all rows stay in registers over the
  // dimensions; the values of the next dimensions, and at the last of them the
  // weights of the next keys, are read ahead.
  constexpr int kValueProducts = 8 * kBlocks;
  s16x8 vf[2], pf[kBlocks];
  auto v_cols = [&](int buf, int g, int d) BSR_INLINE {
    const uint32_t at = tiles_at + buf * kTileBytes + 2 * g * kWaveBytes;
    const s16x4 a = lds_columns(at + (v_at[0] ^ (d * 64))), b = lds_columns(at + (v_at[1] ^ (d * 64)));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto p_cols = [&](int step, int g, int b) BSR_INLINE {
    return lds_row16(weights_at + (((step & 1) * kBlocks + b) * 2 + g) * 1024 + lane * 16);
  };
  auto start_values = [&](int step, int buf) BSR_INLINE {
    vf[0] = v_cols(buf, 0, 0);
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) pf[b] = p_cols(step, 0, b);
  };
  auto value_product = [&](int step, int buf, int i) BSR_INLINE {
    const int b = i % kBlocks, d = i / kBlocks % 4, g = i / (4 * kBlocks), next = i / kBlocks + 1;
    if (b == 0 && next < 8) vf[next & 1] = v_cols(buf, next / 4, next % 4);
    o[b][d] = mfma<T>(vf[d & 1], pf[b], o[b][d]);
    if (g == 0 && d == 3) pf[b] = p_cols(step, 1, b);
  };
  auto values = [&](int step, int buf) BSR_INLINE {
    start_values(step, buf);
#pragma unroll
    for (int i = 0; i < kValueProducts; ++i) value_product(step, buf, i);
  };

  if (steps > 0) {
    load_ids(0);
    load_ids(kIdSteps);
  }
#pragma unroll
  for (int n = 0; n < kN; ++n) {
    s16x8 x{};
    if (t.real) x = *reinterpret_cast<const s16x8*>(p.q + (q.first + t.i) * p.q_token + t.head * p.q_head + n * 32 + half * 16);
    if (n < kHeld) qf[n] = x;
    else *reinterpret_cast<s16x8*>(&queries[wave][n - kHeld][lane * 16]) = x;
  }
  if (steps > 0) {
    loads_done();
#pragma unroll
    for (int i = 0; i < kBufs; ++i) {
      for (int stride = 0; stride < 4; ++stride) find_offset(i, stride);
      if (i < kBufs - 1) load_step(i);
    }
    loads_done<(kBufs - 2) * kLoads>();
    barrier();
    if (scores) {
      f32x16 s[1];
      float unit;
      score(0, s[0], [](int) {}, [] {});
      settle(0, s, &unit, outside_of(0));
      leave_weights(0, s[0], unit, m > -__builtin_inff() ? m : 0.0f, 0, 16);
    }
  }
  // Waits until step + 1 lies in LDS, and the weights of this step; the buffer of
  // step - 1 is free.  Loads go on past the last step, of its last key's record, so
  // that as many are always under way.
  auto turn = [&](int step) BSR_INLINE {
    loads_done<(kBufs - 3) * kLoads>();
    barrier();
    if (step % kIdSteps == 0 && step) load_ids(step + kIdSteps);
    rescale(step);
  };
  int buf = 0;
  if (scores) {
    for (int step = 0; step + 1 < steps; ++step) {
      turn(step);
      const int buf1 = buf + 1 == kBufs ? 0 : buf + 1, last = buf == 0 ? kBufs - 1 : buf - 1;
      f32x16 s[1];
      float unit;
      const uint32_t bad = outside_of(step + 1);
      // the scores of step + 1, with the next loads beside them; then the values of
      // this step, with the softmax of the next beside them
      score(buf1, s[0], [&](int n) BSR_INLINE {
        if (n < kLoads) load_unit(n, last);
        if (n == 1) find_offset(step + kBufs, 0);
        if (n == kN - 3) start_values(step, buf);
      }, [&]() BSR_INLINE {
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) value_product(step, buf, i);
      });
      settle(step + 1, s, &unit, bad);
      const float base = m > -__builtin_inff() ? m : 0.0f;
      constexpr int kRest = kValueProducts - kBlocks;
#pragma unroll
      for (int i = 0; i < kRest; ++i) {
        value_product(step, buf, kBlocks + i);
        leave_weights(step + 1, s[0], unit, base, i * 16 / kRest, (i + 1) * 16 / kRest);
        if (i < 3) find_offset(step + kBufs, i + 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      buf = buf1;
    }
  } else {  // (in a loop of its own: two ways round the value products would have the sums copied)
    for (int step = 0; step + 1 < steps; ++step) {
      turn(step);
      load_step(buf == 0 ? kBufs - 1 : buf - 1);
      values(step, buf);
      for (int stride = 0; stride < 4; ++stride) find_offset(step + kBufs, stride);
      buf = buf + 1 == kBufs ? 0 : buf + 1;
    }
  }
  if (steps > 0) {
    loads_done();  // none may reach LDS that is no longer the workgroup's
    barrier();
    rescale(steps - 1);
    values(steps - 1, buf);
  }

  const Sink sink{w.n_splits > 1, w.slot + w.split};
  l = sum_halves(l);
  if (scores && half == 0) {
    stats[0][row] = m;
    stats[1][row] = l;
  }
  barrier();
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) {
    const float lb = stats[1][b * 32 + col];
    const float inv = sink.part ? 1.0f : lb == 0 ? 0.0f : 1.0f / lb;
    float zero = lb * 0.0f;  // NaN where a result is not finite
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      o[b][d] *= inv;
#pragma unroll
      for (int e = 0; e < 16; ++e) zero += o[b][d][e] * 0.0f;
    }
    const uint32_t odd = static_cast<uint32_t>(__ballot(!(sum_halves(zero) == 0)));
    if (lane == 0 && odd) atomicOr(&redo[b], odd);
  }
  barrier();
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) {
    const uint32_t at = b * 32 + col;
    const TileRows tb = tile_row(p, q, w, at);
    if (!tb.real || (redo[b] >> col & 1)) continue;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        put4<T>(p, q, tb, sink, at, 128 * wave + 32 * d + 8 * e + 4 * half,
                f32x4{o[b][d][4 * e], o[b][d][4 * e + 1], o[b][d][4 * e + 2], o[b][d][4 * e + 3]});
    if (half == 0 && wave == 0) put_stats(p, q, tb, sink, at, stats[0][at], stats[1][at]);
  }
  for (int b = 0; b < kBlocks; ++b)
    for (uint32_t left = uniform(redo[b]); left; left &= left - 1) {
      const uint32_t c = __builtin_ctz(left);
      if ((c & 3) == static_cast<uint32_t>(wave)) redo_row<T, KD, VD>(p, q, w, sink, b * 32 + c, k0, k1);
    }
}

// ---------------------------------------------------------------------------
// Joins the parts of a row: sums and maxima as the running softmax would have
// joined them, in an order that the sizes alone decide.  Bounded by the parts' bytes
// and by finding the work: 512 parts of 128 rows of 128 (34 MB) 14 us; 4.5 us
// where the lengths, which the host does not know, leave nothing to join.
// ---------------------------------------------------------------------------
// Parts of a range, at most: of `target` for up to as many ranges, or of twice
// that for more than `target` ranges, every other of which has a part too.
constexpr uint32_t kJoinParts = kMaxTarget;
constexpr uint32_t kJoinRun = 8;  // parts that a thread sums, about

__host__ __device__ __forceinline__ uint32_t teams_of(uint64_t parts, uint32_t most) {
  uint32_t teams = 1;
  while (teams < most && teams * kJoinRun < parts) teams *= 2;
  return teams;
}

// A team of kSlice / 4 threads holds four dimensions each of a row (of kSlice of
// them) and sums every teams-th part; the teams of a row meet in LDS.  One row
// takes all teams from 8 parts a team on; fewer parts leave room for several rows.
// A team's first sums are read beside the maxima.
template <typename T, int VD, int kSlice, uint32_t kJoinThreads>
__global__ __launch_bounds__(kJoinThreads) void k_attend_join(AttnParams p, uint32_t rows_per) {
  constexpr uint32_t kVecs = kSlice / 4, kTeams = kJoinThreads / kVecs;
  constexpr uint32_t kStats = kJoinParts > kTeams * kJoinRun ? kJoinParts : kTeams * kJoinRun;  // of all rows at once
  __shared__ __attribute__((aligned(16))) float part_m[kStats], part_l[kStats];
  __shared__ f32x4 sums[kJoinThreads];
  __shared__ float sums_l[kTeams];
  Work w;
  Request q;
  if (!find_work<true>(p, blockIdx.x, &w, &q) || w.n_splits < 2) return;
  const uint32_t n = w.n_splits, team = threadIdx.x / kVecs, at = threadIdx.x % kVecs, d = (blockIdx.z * kVecs + at) * 4;
  const uint32_t teams = teams_of(n, kTeams);  // of a row
  const uint32_t side = kTeams / teams, mine = team / teams, first = team % teams;
  const uint64_t step = static_cast<uint64_t>(p.tile_rows) * VD;
  const uint32_t n4 = (n + 3) & ~3u, stats = mine * n4;  // (at most kJoinRun parts a row where several rows are side by side)
  for (uint32_t r0 = blockIdx.y * rows_per; r0 < (blockIdx.y + 1) * rows_per; r0 += side) {
    const uint32_t row = r0 + mine;
    TileRows t = tile_row(p, q, w, row);
    t.real = t.real && row < (blockIdx.y + 1) * rows_per;
    const float* ml = p.part_ml + (static_cast<uint64_t>(w.slot) * p.tile_rows + row) * 2;
    const float* part = p.part + (static_cast<uint64_t>(w.slot) * p.tile_rows + row) * VD + d;
    f32x4 ahead[kJoinRun];
    if (t.real) {
#pragma unroll
      for (uint32_t i = 0; i < kJoinRun; ++i)
        ahead[i] = *reinterpret_cast<const f32x4*>(part + min(first + i * teams, n - 1) * step);
      for (uint32_t s = first * kVecs + at; s < n4; s += teams * kVecs) {
        part_m[stats + s] = s < n ? ml[static_cast<uint64_t>(s) * p.tile_rows * 2] : -__builtin_inff();
        part_l[stats + s] = s < n ? ml[static_cast<uint64_t>(s) * p.tile_rows * 2 + 1] : 0.0f;
      }
    }
    __syncthreads();
    float m = -__builtin_inff(), l = 0;
    f32x4 x{};
    if (t.real) {
#pragma unroll 4
      for (uint32_t s = 0; s < n4; s += 4) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(&part_m[stats + s]);
        m = fmaxf(fmaxf(fmaxf(m, v[0]), fmaxf(v[1], v[2])), v[3]);
      }
      const float from = m > -__builtin_inff() ? m : 0.0f;
      const auto add = [&](uint32_t s, f32x4 part_sums) BSR_INLINE {
        const float ls = part_l[stats + s];
        const float f = ls == 0 ? 0.0f : exp2_(part_m[stats + s] - from);  // a part without a seen key weighs nothing
        l += f * ls;
        x += f * part_sums;
      };
#pragma unroll
      for (uint32_t i = 0; i < kJoinRun; ++i)
        if (first + i * teams < n) add(first + i * teams, ahead[i]);
#pragma unroll 4
      for (uint32_t s = first + kJoinRun * teams; s < n; s += teams) add(s, *reinterpret_cast<const f32x4*>(part + s * step));
    }
    sums[threadIdx.x] = x;
    if (at == 0) sums_l[team] = l;
    __syncthreads();
    if (t.real && first == 0) {
      for (uint32_t i = 1; i < teams; ++i) {
        x += sums[threadIdx.x + i * kVecs];
        l += sums_l[team + i];
      }
      const Sink sink{false, 0};
      x *= l == 0 ? 0.0f : 1.0f / l;
      put4<T>(p, q, t, sink, row, d, x);
      if (d == 0) put_stats(p, q, t, sink, row, m, l);
    }
    __syncthreads();
  }
}

template <typename T, int VD, int kSlice, uint32_t kThreads>
hipError_t launch_join(const AttnParams& p, const AttnTiling& t, hipStream_t s) {
  const uint32_t rows = p.tile_tokens * p.tile_heads, teams = kThreads / (kSlice / 4);
  // rows of a workgroup: as many as its teams take at once if the parts spread
  // evenly over the tiles there may be, more where the tiles alone fill the GPU
  uint32_t per = teams / teams_of(t.slots / t.base, teams);
  while (per < rows && t.base * ((rows + per - 1) / per) > 8192) per *= 2;
  hipLaunchKernelGGL((k_attend_join<T, VD, kSlice, kThreads>), dim3(static_cast<uint32_t>(t.base), (rows + per - 1) / per, VD / kSlice),
                     dim3(kThreads), 0, s, p, per);
  return hipGetLastError();
}

// Few tiles, each in many parts: 16 teams for 128 dimensions of a row.  One
// latent token over 128K (16 rows, 256 parts): 21.2 us with the teams of the
// others, 9.3 so; 22 latent tiles in 256 parts: 13.2 and 17.8.
template <typename T, int VD>
hipError_t launch_join(const AttnParams& p, const AttnTiling& t, hipStream_t s) {
  if (t.base <= 4) return launch_join<T, VD, (VD < 128 ? VD : 128), 512>(p, t, s);
  return launch_join<T, VD, VD, 128>(p, t, s);
}

template <typename T, int kMods>
hipError_t launch_tiles(const AttnParams& p, hipStream_t s) {
  const AttnTiling t = attn_tiling(p.n_requests, p.n_tokens, p.n_heads, p.n_kv_heads, p.v_dim, p.max_len);
  const dim3 grid(static_cast<uint32_t>(t.items)), block(kAttnThreads);
  if (p.k_dim == 64) hipLaunchKernelGGL((k_attend_heads<T, 64, kMods>), grid, block, 0, s, p);
  else if (p.k_dim == 128) hipLaunchKernelGGL((k_attend_heads<T, 128, kMods>), grid, block, 0, s, p);
  else if (p.tile_rows == 32) hipLaunchKernelGGL((k_attend_latent<T, kMods, 1>), grid, block, 0, s, p);
  else if (p.tile_rows == 64) hipLaunchKernelGGL((k_attend_latent<T, kMods, 2>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((k_attend_latent<T, kMods, 4>), grid, block, 0, s, p);
  if (hipError_t e = hipGetLastError()) return e;
  if (!p.target) return hipSuccess;
  return p.v_dim == 64 ? launch_join<T, 64>(p, t, s) : p.v_dim == 128 ? launch_join<T, 128>(p, t, s) : launch_join<T, 512>(p, t, s);
}

template <typename T>
hipError_t launch_typed(const AttnParams& p, hipStream_t s) {
  if (p.softcap > 0) return p.slopes ? launch_tiles<T, kCap | kSlopes>(p, s) : launch_tiles<T, kCap>(p, s);
  return p.slopes ? launch_tiles<T, kSlopes>(p, s) : launch_tiles<T, 0>(p, s);
}

}  // namespace

hipError_t launch_attention(const AttnParams& p, hipStream_t s) {
  return p.f16 ? launch_typed<_Float16>(p, s) : launch_typed<__bf16>(p, s);
}

}  // namespace bsr
