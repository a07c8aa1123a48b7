// Block tables and slot maps from request lengths, and the append of new
// tokens' records into their slots.
#include <hip/hip_runtime.h>

#include "bsr_cache.h"

namespace bsr {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------
// Block tables and slot maps
//
// Prefix sums over the requests (of rows, and of blocks taken per group) say
// where every row and block goes; each workgroup computes them all for itself in
// LDS, so one launch does and nothing is handed from workgroup to workgroup.
// A wave takes every fourth sum, a lane the requests of 1/64 of the batch, so a
// sum is one scan within the wave and the waves meet once.  Sums saturate at
// 2^32 - 1, which no admitted request reaches (n_slots and n_free are below 2^31).
// Then a thread finds its row's request by bisection and writes its slot in every
// group; the row that is the first of a block writes the block's table entry.
// ---------------------------------------------------------------------------
constexpr int kTablesThreads = 256;
constexpr uint32_t kMostTokens = 0x7fffffffu;
__device__ const int32_t kNoBlock = 0;

__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

template <int kCtrl, int kRows>
__device__ __forceinline__ uint32_t sat_step(uint32_t x) {
  return sat_add(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), kCtrl, kRows, 0xf, false)));
}
// Inclusive saturating sum over a wave.
__device__ __forceinline__ uint32_t sat_scan(uint32_t x) {
  x = sat_step<0x111, 0xf>(x);  // lanes 1, 2, 4, 8 before, of the row of 16
  x = sat_step<0x112, 0xf>(x);
  x = sat_step<0x114, 0xf>(x);
  x = sat_step<0x118, 0xf>(x);
  x = sat_step<0x142, 0xa>(x);  // the last lane of the row before, and of the half before
  return sat_step<0x143, 0xc>(x);
}

__device__ __forceinline__ uint32_t blocks_of(const FastDiv& d, uint32_t tokens) {
  return tokens ? d.div(tokens - 1) + 1 : 0;
}

// A request's tokens held and added; nothing where its lengths or its tables'
// room rule it out.
struct Lengths {
  uint32_t have, add;
  bool fits;
};
__device__ __forceinline__ Lengths lengths_of(const TablesBuildParams& p, int32_t c, int32_t a) {
  Lengths x;
  x.fits = c >= 0 && a >= 0 && static_cast<uint32_t>(c) + static_cast<uint32_t>(a) <= kMostTokens;
  for (uint32_t g = 0; g < p.n_groups; ++g)
    if (p.g[g].tables && x.fits && blocks_of(p.g[g].div_block, c + a) > p.g[g].table_stride) x.fits = false;
  x.have = x.fits ? c : 0;
  x.add = x.fits ? a : 0;
  return x;
}

// What bounds it is the launch and three loads one behind the other (the lengths, a
// row's request's own once more, out of the cache, and the block ids), 5 of the 6 us
// that 37 rows of four groups take; 268K rows (64 requests) take 8.7, with four rows
// a thread and a quarter of the workgroups 12.6.
__global__ __launch_bounds__(kTablesThreads) void k_tables_build(TablesBuildParams p) {
  // [1 + n_groups][n_requests + 1]: rows, then blocks taken, before each request
  extern __shared__ uint32_t before[];
  __shared__ uint32_t s_admitted;
  const uint32_t n = p.n_requests, line = n + 1, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) s_admitted = n;
  __syncthreads();
  const uint32_t per = (n + 63) / 64, r0 = min(lane * per, n), r1 = min(r0 + per, n);
  Lengths only{};  // of the lane's request, where it has no more than one
  if (per == 1 && r0 < r1) only = lengths_of(p, p.cached[r0], p.added[r0]);
  for (uint32_t sum = wave; sum <= p.n_groups; sum += kTablesThreads / 64) {
    const bool rows = sum == 0;
    const TablesBuildGroup& g = p.g[rows ? 0 : sum - 1];
    if (!rows && !g.tables) continue;
    const uint32_t limit = rows ? p.n_slots : g.n_free;
    const auto share = [&](const Lengths& x) {
      return rows ? x.add : blocks_of(g.div_block, x.have + x.add) - blocks_of(g.div_block, x.have);
    };
    uint32_t mine = per == 1 ? share(only) : 0;
    if (per > 1) {
#pragma unroll 4
      for (uint32_t r = r0; r < r1; ++r) mine = sat_add(mine, share(lengths_of(p, p.cached[r], p.added[r])));
    }
    const uint32_t upto = sat_scan(mine);
    if (lane == 63) before[sum * line + n] = upto;
    // before the lane's first request: what the lanes before it have
    uint32_t at = __shfl_up(upto, 1), stop = n;
    if (lane == 0) at = 0;
    for (uint32_t r = r0; r < r1; ++r) {
      const Lengths x = per == 1 ? only : lengths_of(p, p.cached[r], p.added[r]);
      before[sum * line + r] = at;
      at = sat_add(at, share(x));
      if (stop == n && !(x.fits && at <= limit)) stop = r;
    }
    if (stop < n) atomicMin(&s_admitted, stop);
  }
  __syncthreads();
  const uint32_t admitted = s_admitted, total = before[admitted];
  if (blockIdx.x == 0) {
    for (uint32_t r = threadIdx.x; r <= n; r += kTablesThreads) p.starts[r] = min(before[r], total);
    for (uint32_t r = threadIdx.x; r < n; r += kTablesThreads) {
      const int32_t c = p.cached[r];
      p.lens[r] = r < admitted ? c + p.added[r] : max(c, 0);
    }
    if (threadIdx.x == 0) p.result[0] = admitted;
    if (threadIdx.x < p.n_groups)
      p.result[1 + threadIdx.x] = p.g[threadIdx.x].tables ? before[(1 + threadIdx.x) * line + admitted] : 0;
  }
  const uint64_t s = static_cast<uint64_t>(blockIdx.x) * kTablesThreads + threadIdx.x;
  if (s >= p.n_slots) return;
  const bool real = s < total;
  // the last request that starts at or before the row (one without rows starts
  // where the next does)
  uint32_t lo = 0, hi = real ? admitted : 0;
  while (hi - lo > 1 && hi) {
    const uint32_t mid = (lo + hi) / 2;
    if (before[mid] <= s) lo = mid;
    else hi = mid;
  }
  const uint32_t have = *(real ? p.cached + lo : &kNoBlock);
  const uint32_t t = real ? have + static_cast<uint32_t>(s) - before[lo] : 0;
  // the row's block ids in all groups, their loads under way together (no
  // branch round any: a row without one reads a zero)
  int32_t id[BSR_MAX_GROUPS];
#pragma unroll
  for (uint32_t g = 0; g < BSR_MAX_GROUPS; ++g) {
    if (g >= p.n_groups) break;
    const TablesBuildGroup& q = p.g[g];
    const uint32_t k = q.div_block.div(t), held = blocks_of(q.div_block, have);
    const int32_t* from = k < held ? q.tables + static_cast<uint64_t>(lo) * q.table_stride + k
                                   : q.free_blocks + (before[(1 + g) * line + lo] + k - held);
    id[g] = *(q.tables && real ? from : &kNoBlock);
  }
#pragma unroll
  for (uint32_t g = 0; g < BSR_MAX_GROUPS; ++g) {
    if (g >= p.n_groups) break;
    const TablesBuildGroup& q = p.g[g];
    const uint32_t k = q.div_block.div(t), o = t - k * q.div_block.d;
    const bool in = q.tables && real;
    if (in && o == 0 && k >= blocks_of(q.div_block, have)) q.tables[static_cast<uint64_t>(lo) * q.table_stride + k] = id[g];
    if (q.slots) q.slots[s] = in && id[g] >= 0 ? static_cast<int64_t>(id[g]) * q.div_block.d + o : -1;
  }
}

// ---------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------
__device__ __forceinline__ float load_value(const uint8_t* row, uint32_t i, uint32_t type) {
  if (type == BSR_TYPE_F32) return reinterpret_cast<const float*>(row)[i];
  if (type == BSR_TYPE_F16) return static_cast<float>(reinterpret_cast<const _Float16*>(row)[i]);
  return static_cast<float>(reinterpret_cast<const __bf16*>(row)[i]);
}

// Eight values of 16-byte aligned memory.
template <typename S>
__device__ __forceinline__ void load8(const uint8_t* at, float (&x)[8]) {
  typedef S S8 __attribute__((ext_vector_type(8)));
  const S8 v = *reinterpret_cast<const S8*>(at);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(v[i]);
}
template <typename C>
__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
  typedef C C8 __attribute__((ext_vector_type(8)));
  C8 y;
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = static_cast<C>(x[i]);
  return __builtin_bit_cast(u32x4, y);
}

constexpr int kAppendThreads = 256;
constexpr uint32_t kAppendUnits = 4;  // of a thread, kAppendThreads apart: their loads are under way together

__device__ __forceinline__ bool append_unit(const AppendParams& p, uint64_t i, uint32_t per, const uint8_t** row, uint32_t* v,
                                            uint8_t** record, uint32_t* at) {
  if (i >= static_cast<uint64_t>(p.n_tokens) * p.units) return false;
  const uint32_t t = p.div_units.div(static_cast<uint32_t>(i));  // (all units number below 2^32)
  *at = (static_cast<uint32_t>(i) - t * p.units) * per;
  const int64_t slot = p.slots[t];
  if (slot < 0 || static_cast<uint64_t>(slot) >= p.n_slots) return false;
  const uint32_t which = *at >= p.width[0];
  *v = which ? *at - p.width[0] : *at;
  *row = p.src[which] + static_cast<int64_t>(t) * p.src_stride[which];
  *record = p.pool + static_cast<uint64_t>(slot) * p.record_bytes;
  return true;
}

// CONTIG records in units of eight values, from S to C (the same: copied bit by
// bit).  Bounded by memory: 32,768 latent records of two sources (75.8 MB moved)
// 13.0 us, 5.8 TB/s (part of the sources comes out of the caches); 64 records 2.9
// us, the launch and two ways to memory.  One unit a thread, in turn on one
// box: 64 records the same, 8,192 of them 4.6 us for 6.0, 32,768 12.5-13.0 for
// 13.0, and with inputs that stay in the caches 13.0 for 15.7.
template <typename S, typename C>
__global__ __launch_bounds__(kAppendThreads) void k_append(AppendParams p) {
  const uint64_t i0 = static_cast<uint64_t>(blockIdx.x) * (kAppendThreads * kAppendUnits) + threadIdx.x;
  u32x4 out[kAppendUnits];
  uint8_t* to[kAppendUnits];
#pragma unroll
  for (uint32_t k = 0; k < kAppendUnits; ++k) {
    const uint8_t* row;
    uint8_t* record;
    uint32_t v, at;
    to[k] = nullptr;
    if (!append_unit(p, i0 + k * kAppendThreads, 8, &row, &v, &record, &at)) continue;
    to[k] = record + at * 2;
    if (__is_same(S, C)) {
      out[k] = *reinterpret_cast<const u32x4*>(row + v * sizeof(S));
    } else {
      float x[8];
      load8<S>(row + v * sizeof(S), x);
      out[k] = pack8<C>(x);
    }
  }
#pragma unroll
  for (uint32_t k = 0; k < kAppendUnits; ++k)
    if (to[k]) *reinterpret_cast<u32x4*>(to[k]) = out[k];
}

// CONTIG records value by value, where sizes or alignment leave no units.
__global__ __launch_bounds__(kAppendThreads) void k_append_values(AppendParams p) {
  const uint64_t i = static_cast<uint64_t>(blockIdx.x) * kAppendThreads + threadIdx.x;
  const uint8_t* row;
  uint8_t* record;
  uint32_t v, at;
  if (!append_unit(p, i, 1, &row, &v, &record, &at)) return;
  if (p.src_type == p.cache_type) {
    reinterpret_cast<uint16_t*>(record)[at] = reinterpret_cast<const uint16_t*>(row)[v];
  } else {
    const float x = load_value(row, v, p.src_type);
    if (p.cache_type == BSR_TYPE_F16) reinterpret_cast<_Float16*>(record)[at] = static_cast<_Float16>(x);
    else reinterpret_cast<__bf16*>(record)[at] = static_cast<__bf16>(x);
  }
}

// Four values to fp8-e4m3fn (round to nearest even; they are at most 448).
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

// A value over its record's scale: zero where that is zero or not a number.
__device__ __forceinline__ float scaled(float x, float scale) {
  const float y = scale > 0 ? x / scale : 0.0f;
  return fminf(fmaxf(y, -448.0f), 448.0f);
}

struct ScaledSlot {
  uint8_t* values;
  float* scale;
};
__device__ __forceinline__ bool scaled_slot(const AppendParams& p, uint32_t t, ScaledSlot* s) {
  if (t >= p.n_tokens) return false;
  const int64_t slot = p.slots[t];
  if (slot < 0 || static_cast<uint64_t>(slot) >= p.n_slots) return false;
  // most pools have fewer than 2^32 records: no division in 64 bits
  const uint64_t at = static_cast<uint64_t>(slot);
  const uint64_t block = at >> 32 ? at / p.block_tokens : p.div_block.div(static_cast<uint32_t>(at));
  const uint64_t o = at - block * p.block_tokens;
  uint8_t* base = p.pool + block * p.block_tokens * p.record_bytes;
  s->values = base + o * p.split_bytes;
  s->scale = reinterpret_cast<float*>(base + static_cast<uint64_t>(p.block_tokens) * p.split_bytes) + o;
  return true;
}

// PLANAR records of 128 values in aligned rows: 16 lanes a token, eight values
// each.  8,200 fp32 rows (5.3 MB moved) 3.2 us: the launch and three ways to memory.
template <typename S>
__global__ __launch_bounds__(kAppendThreads) void k_append_scaled128(AppendParams p) {
  const uint32_t t = blockIdx.x * (kAppendThreads / 16) + threadIdx.x / 16, lane = threadIdx.x & 15;
  ScaledSlot to;
  if (!scaled_slot(p, t, &to)) return;  // (all 16 lanes or none)
  float x[8], most = 0;
  load8<S>(p.src[0] + static_cast<int64_t>(t) * p.src_stride[0] + lane * 8 * sizeof(S), x);
  bool odd = false;  // an infinity or a NaN
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    odd |= !(fabsf(x[i]) < __builtin_inff());
    most = fmaxf(most, fabsf(x[i]));
  }
  if (odd) most = __builtin_inff();  // (the maximum skips a NaN)
#pragma unroll
  for (int d = 8; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
  const float scale = most < __builtin_inff() ? most / 448.0f : __builtin_nanf("");
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(4)));  // (a block of an odd number of tokens)
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = scaled(x[i], scale);
  *reinterpret_cast<u32x2*>(to.values + lane * 8) = u32x2{pack_e4m3(x[0], x[1], x[2], x[3]), pack_e4m3(x[4], x[5], x[6], x[7])};
  if (lane == 0) *to.scale = scale;
}

// PLANAR records of any size: a wave a token.
__global__ __launch_bounds__(kAppendThreads) void k_append_scaled(AppendParams p) {
  const uint32_t t = blockIdx.x * (kAppendThreads / 64) + threadIdx.x / 64, lane = threadIdx.x & 63;
  ScaledSlot to;
  if (!scaled_slot(p, t, &to)) return;
  const uint8_t* row = p.src[0] + static_cast<int64_t>(t) * p.src_stride[0];
  float most = 0;
  for (uint32_t v = lane; v < p.split_bytes; v += 64) {
    const float x = fabsf(load_value(row, v, p.src_type));
    most = x < __builtin_inff() ? fmaxf(most, x) : __builtin_inff();
  }
  for (int d = 32; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
  const float scale = most < __builtin_inff() ? most / 448.0f : __builtin_nanf("");
  for (uint32_t w = lane; w < p.split_bytes / 4; w += 64) {
    float x[4];
    for (int k = 0; k < 4; ++k) x[k] = scaled(load_value(row, 4 * w + k, p.src_type), scale);
    reinterpret_cast<uint32_t*>(to.values)[w] = pack_e4m3(x[0], x[1], x[2], x[3]);
  }
  if (lane == 0) *to.scale = scale;
}

template <typename S>
void append_from(const AppendParams& p, uint32_t grid, hipStream_t s) {
  if (p.cache_type == BSR_TYPE_F16) hipLaunchKernelGGL((k_append<S, _Float16>), dim3(grid), dim3(kAppendThreads), 0, s, p);
  else hipLaunchKernelGGL((k_append<S, __bf16>), dim3(grid), dim3(kAppendThreads), 0, s, p);
}

}  // namespace

hipError_t launch_tables_build(const TablesBuildParams& p, hipStream_t s) {
  const uint32_t lds = (1 + p.n_groups) * (p.n_requests + 1) * sizeof(uint32_t);
  const uint32_t grid = p.n_slots ? (p.n_slots - 1) / kTablesThreads + 1 : 1;
  hipLaunchKernelGGL(k_tables_build, dim3(grid), dim3(kTablesThreads), lds, s, p);
  return hipGetLastError();
}

hipError_t launch_append(const AppendParams& p, hipStream_t s) {
  const auto grid = [](uint64_t n, uint32_t per) { return static_cast<uint32_t>((n + per - 1) / per); };
  const uint64_t n = static_cast<uint64_t>(p.n_tokens) * p.units;
  if (p.split_bytes == 128 && p.vector) {
    const dim3 g(grid(p.n_tokens, kAppendThreads / 16)), b(kAppendThreads);
    if (p.src_type == BSR_TYPE_F32) hipLaunchKernelGGL(k_append_scaled128<float>, g, b, 0, s, p);
    else if (p.src_type == BSR_TYPE_F16) hipLaunchKernelGGL(k_append_scaled128<_Float16>, g, b, 0, s, p);
    else hipLaunchKernelGGL(k_append_scaled128<__bf16>, g, b, 0, s, p);
  } else if (p.split_bytes) {
    hipLaunchKernelGGL(k_append_scaled, dim3(grid(p.n_tokens, kAppendThreads / 64)), dim3(kAppendThreads), 0, s, p);
  } else if (!p.vector) {
    hipLaunchKernelGGL(k_append_values, dim3(grid(n, kAppendThreads)), dim3(kAppendThreads), 0, s, p);
  } else {
    const uint32_t g = grid(n, kAppendThreads * kAppendUnits);
    if (p.src_type == BSR_TYPE_F32) append_from<float>(p, g, s);
    else if (p.src_type == BSR_TYPE_F16) append_from<_Float16>(p, g, s);
    else append_from<__bf16>(p, g, s);
  }
  return hipGetLastError();
}

}  // namespace bsr
