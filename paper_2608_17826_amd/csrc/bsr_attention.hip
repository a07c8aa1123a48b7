// Attention over the paged cache, for drafted trees and for prompt tokens.
//
// A query row (token, head) sees the keys lo <= j < hi of its request, and of
// those in a drafted tree's rows the ones whose bit its mask has.  Its scores
// pass the softmax in one go over the keys, with a running maximum m and sum
// l: new keys scale what was summed so far by exp(m - m').
#include <hip/hip_runtime.h>

#include "bsr_cache.h"

namespace bsr {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// One request of the batch: its rows [first, first + rows) and its keys [0, n);
// row i stands at base + i.
struct Request {
  int first, rows, n, base;
  const int32_t* table;
};

__device__ __forceinline__ Request request_of(const AttnParams& p, uint32_t r) {
  Request q;
  const int cap = static_cast<int>(p.n_tokens);
  q.first = min(max(p.starts[r], 0), cap);
  q.rows = min(max(p.starts[r + 1], q.first), cap) - q.first;
  q.n = min(max(p.lens[r], 0), static_cast<int>(p.max_len));
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

__device__ __forceinline__ Row row_of(const AttnParams& p, const Request& q, uint32_t r, int i) {
  Row w;
  w.mask = nullptr;
  if (p.tree) {
    w.mask = p.tree + static_cast<uint64_t>(q.first + i) * p.tree_words;
    int bits = 0;
    if (p.window)
      for (uint32_t k = 0; k < p.tree_words; ++k) bits += __popcll(w.mask[k]);
    w.pos = q.base + bits - 1;
    w.hi = q.n;
  } else {
    w.pos = q.base + i;
    w.hi = w.pos + 1;
    if (p.prefix) w.hi = max(w.hi, min(p.prefix[r], q.n));
  }
  w.lo = 0;
  if (p.window) w.lo = max(0, w.pos - static_cast<int>(p.window) + 1);
  if (p.documents) w.lo = max(w.lo, p.documents[q.first + i]);
  return w;
}

__device__ __forceinline__ bool sees(const AttnParams& p, const Request& q, const Row& w, int j) {
  if (j < w.lo || j >= w.hi) return false;
  if (!w.mask || j < q.base) return true;
  const uint32_t k = static_cast<uint32_t>(j - q.base);
  return k < 64 * p.tree_words && (w.mask[k >> 6] >> (k & 63) & 1);
}

// Score times log2(e) of a product.
__device__ __forceinline__ float score2(const AttnParams& p, float qk, float slope, int away) {
  float s = qk * p.scale;
  if (p.softcap > 0) s = p.softcap * tanhf(s / p.softcap);
  return (s - slope * static_cast<float>(abs(away))) * kLog2e;
}

// Byte offset of token j's record in a pool, or -1 where its block lies outside.
__device__ __forceinline__ int64_t record_at(const AttnParams& p, const Request& q, int j) {
  const uint32_t b = p.div_block.div(j);
  const int32_t id = q.table[b];
  if (id < 0 || static_cast<uint32_t>(id) >= p.pool_blocks) return -1;
  return static_cast<int64_t>(id) * p.block_bytes + static_cast<int64_t>(j - b * p.div_block.d) * p.record_bytes;
}

// One row over the keys [lo, hi) by one wave: 64 keys at a time, a lane each
// for the scores, then every lane VD / 64 dimensions of the values.  Only what
// the row sees is read.  m and l are the wave's, acc the lane's.
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

constexpr int kRowThreads = 256;

// A wave per row and head.
template <typename T, int KD, int VD>
__global__ __launch_bounds__(kRowThreads) void k_attend_rows(AttnParams p) {
  const uint32_t row = blockIdx.x, head = blockIdx.y * (kRowThreads / 64) + threadIdx.x / 64;
  if (head >= p.n_heads || static_cast<int>(row) >= p.starts[p.n_requests]) return;
  uint32_t lo = 0, hi = p.n_requests;  // the last request that starts at or before the row
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (p.starts[mid] <= static_cast<int>(row)) lo = mid;
    else hi = mid;
  }
  const Request q = request_of(p, lo);
  const int i = static_cast<int>(row) - q.first;
  if (i < 0 || i >= q.rows) return;
  const Row w = row_of(p, q, lo, i);
  float m, l, acc[VD / 64];
  attend_row<T, KD, VD>(p, q, w, i, head, max(w.lo, 0), min(w.hi, q.n), m, l, acc);
  T* o = reinterpret_cast<T*>(p.out + row * p.out_token + head * p.out_head) + (threadIdx.x & 63) * (VD / 64);
  const bool none = l == 0;
  for (int d = 0; d < VD / 64; ++d) o[d] = static_cast<T>(none ? 0.0f : acc[d] / l);
  if (p.lse && (threadIdx.x & 63) == 0)
    p.lse[static_cast<uint64_t>(row) * p.n_heads + head] = none ? -__builtin_inff() : (m + __log2f(l)) * kLn2;
}

template <typename T>
hipError_t launch_rows(const AttnParams& p, hipStream_t s) {
  const dim3 grid(p.n_tokens, (p.n_heads + kRowThreads / 64 - 1) / (kRowThreads / 64));
  if (p.k_dim == 64) hipLaunchKernelGGL((k_attend_rows<T, 64, 64>), grid, dim3(kRowThreads), 0, s, p);
  else if (p.k_dim == 128) hipLaunchKernelGGL((k_attend_rows<T, 128, 128>), grid, dim3(kRowThreads), 0, s, p);
  else hipLaunchKernelGGL((k_attend_rows<T, 576, 512>), grid, dim3(kRowThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attention(const AttnParams& p, hipStream_t s) {
  return p.f16 ? launch_rows<_Float16>(p, s) : launch_rows<__bf16>(p, s);
}

}  // namespace bsr
