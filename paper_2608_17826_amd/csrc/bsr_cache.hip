// Block tables and slot maps from request lengths, and the append of new
// tokens' records into their slots.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "bsr_cache.h"

namespace bsr {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------------------
// Block tables and slot maps
//
// Three prefix sums over the requests (rows, and blocks taken per group) say
// where every row and block goes; each workgroup computes them all for itself
// in LDS, so one launch does and nothing is handed from workgroup to
// workgroup.  Sums saturate at 2^31 - 1, which no admitted request reaches
// (n_slots and n_free are smaller).  Then a thread per row finds its request by
// bisection and writes its slot in every group; the row that is the first of a
// block writes the block's table entry.
// ---------------------------------------------------------------------------
constexpr int kTablesThreads = 256;
constexpr uint32_t kSat = 0x7fffffffu;

__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) {
  const uint32_t s = a + b;  // both at most 2^31 - 1
  return s < kSat ? s : kSat;
}

// Inclusive saturating sum over the workgroup's threads; *total gets all of it.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* wave_sums, uint32_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t u = __shfl_up(v, d);
    if (lane >= d) v = sat_add(v, u);
  }
  __syncthreads();  // the sums of the scan before have been read
  if (lane == 63) wave_sums[wave] = v;
  __syncthreads();
  uint32_t before = 0, all = 0;
  for (int w = 0; w < kTablesThreads / 64; ++w) {
    const uint32_t s = wave_sums[w];
    if (w < wave) before = sat_add(before, s);
    all = sat_add(all, s);
  }
  *total = all;
  return sat_add(before, v);
}

__device__ __forceinline__ uint32_t blocks_of(const FastDiv& d, uint32_t tokens) {
  return tokens ? d.div(tokens - 1) + 1 : 0;
}

__global__ __launch_bounds__(kTablesThreads) void k_tables_build(TablesBuildParams p) {
  // [1 + n_groups][n_requests + 1]: rows, then blocks taken, before each request
  extern __shared__ uint32_t before[];
  __shared__ uint32_t wave_sums[kTablesThreads / 64];
  __shared__ uint32_t s_admitted;
  const uint32_t n = p.n_requests, row = n + 1;
  if (threadIdx.x == 0) s_admitted = n;
  uint32_t carry[1 + BSR_MAX_GROUPS] = {};
  for (uint32_t r0 = 0; r0 < n; r0 += kTablesThreads) {
    const uint32_t r = r0 + threadIdx.x;
    int32_t c = 0, a = 0;
    if (r < n) {
      c = p.cached[r];
      a = p.added[r];
    }
    bool fits = c >= 0 && a >= 0 && static_cast<uint32_t>(c) + static_cast<uint32_t>(a) <= kSat;
    const uint32_t have = fits ? c : 0, len = fits ? have + a : 0;
    for (uint32_t g = 0; g < p.n_groups; ++g)
      if (p.g[g].tables && blocks_of(p.g[g].div_block, len) > p.g[g].table_stride) fits = false;
    uint32_t all;
    const uint32_t add = fits ? len - have : 0;
    const uint32_t upto = sat_add(carry[0], block_scan(add, wave_sums, &all));
    if (r < n) before[r] = upto - add;
    bool room = upto <= p.n_slots;
    carry[0] = sat_add(carry[0], all);
#pragma unroll
    for (uint32_t g = 0; g < BSR_MAX_GROUPS; ++g) {
      if (g >= p.n_groups || !p.g[g].tables) continue;
      const uint32_t take = fits ? blocks_of(p.g[g].div_block, len) - blocks_of(p.g[g].div_block, have) : 0;
      const uint32_t at = sat_add(carry[1 + g], block_scan(take, wave_sums, &all));
      if (r < n) before[(1 + g) * row + r] = at - take;
      room = room && at <= p.g[g].n_free;
      carry[1 + g] = sat_add(carry[1 + g], all);
    }
    if (r < n && !(fits && room)) atomicMin(&s_admitted, r);
  }
  if (threadIdx.x == 0) {
    before[n] = carry[0];
#pragma unroll
    for (uint32_t g = 0; g < BSR_MAX_GROUPS; ++g)
      if (g < p.n_groups) before[(1 + g) * row + n] = carry[1 + g];
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
    if (threadIdx.x < p.n_groups) {
      const bool in = p.g[threadIdx.x].tables;
      p.result[1 + threadIdx.x] = in ? before[(1 + threadIdx.x) * row + admitted] : 0;
    }
  }
  for (uint64_t s = blockIdx.x * kTablesThreads + threadIdx.x; s < p.n_slots; s += gridDim.x * kTablesThreads) {
    if (s >= total) {
      for (uint32_t g = 0; g < p.n_groups; ++g)
        if (p.g[g].slots) p.g[g].slots[s] = -1;
      continue;
    }
    uint32_t lo = 0, hi = admitted;  // the last request that starts at or before the row (those without rows start where the next does)
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (before[mid] <= s) lo = mid;
      else hi = mid;
    }
    const uint32_t c = p.cached[lo], t = c + static_cast<uint32_t>(s) - before[lo];
    for (uint32_t g = 0; g < p.n_groups; ++g) {
      const TablesBuildGroup& q = p.g[g];
      if (!q.tables) continue;
      const uint32_t k = q.div_block.div(t), o = t - k * q.div_block.d, held = blocks_of(q.div_block, c);
      int32_t* entry = q.tables + static_cast<uint64_t>(lo) * q.table_stride + k;
      int32_t id;
      if (k < held) {
        if (!q.slots) continue;
        id = *entry;
      } else {
        id = q.free_blocks[before[(1 + g) * row + lo] + k - held];
        if (o == 0) *entry = id;
      }
      if (q.slots) q.slots[s] = id < 0 ? -1 : static_cast<int64_t>(id) * q.div_block.d + o;
    }
  }
}

// ---------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ float as_float(const uint8_t* p) {
  return static_cast<float>(*reinterpret_cast<const T*>(p));
}
__device__ __forceinline__ float load_value(const uint8_t* row, uint32_t i, uint32_t type) {
  if (type == BSR_TYPE_F32) return reinterpret_cast<const float*>(row)[i];
  if (type == BSR_TYPE_F16) return static_cast<float>(reinterpret_cast<const _Float16*>(row)[i]);
  return static_cast<float>(reinterpret_cast<const __bf16*>(row)[i]);
}

constexpr int kAppendThreads = 256;

// CONTIG: a thread per unit of a record: 8 values, or one where sizes or
// alignment leave no 16-byte units.
__global__ __launch_bounds__(kAppendThreads) void k_append(AppendParams p) {
  const uint64_t i = static_cast<uint64_t>(blockIdx.x) * kAppendThreads + threadIdx.x;
  if (i >= static_cast<uint64_t>(p.n_tokens) * p.units) return;
  const uint32_t t = static_cast<uint32_t>(i / p.units);
  uint32_t u = static_cast<uint32_t>(i - static_cast<uint64_t>(t) * p.units);
  const int64_t slot = p.slots[t];
  if (slot < 0 || static_cast<uint64_t>(slot) >= p.n_slots) return;
  uint8_t* record = p.pool + static_cast<uint64_t>(slot) * p.record_bytes;
  const uint32_t per = p.vector ? 8 : 1;
  uint32_t v = u * per;
  const uint32_t which = v >= p.width[0];
  const uint8_t* row = p.src[which] + static_cast<int64_t>(t) * p.src_stride[which];
  if (which) v -= p.width[0];
  for (uint32_t k = 0; k < per; ++k) {
    const uint32_t at = u * per + k;
    if (p.src_type == p.cache_type) {
      reinterpret_cast<uint16_t*>(record)[at] = reinterpret_cast<const uint16_t*>(row)[v + k];
    } else {
      const float x = load_value(row, v + k, p.src_type);
      if (p.cache_type == BSR_TYPE_F16) reinterpret_cast<_Float16*>(record)[at] = static_cast<_Float16>(x);
      else reinterpret_cast<__bf16*>(record)[at] = static_cast<__bf16>(x);
    }
  }
}

// Four values to fp8-e4m3fn (round to nearest even; they are at most 448).
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

// PLANAR: a wave per token.
__global__ __launch_bounds__(kAppendThreads) void k_append_scaled(AppendParams p) {
  const uint32_t t = blockIdx.x * (kAppendThreads / 64) + threadIdx.x / 64, lane = threadIdx.x & 63;
  if (t >= p.n_tokens) return;
  const int64_t slot = p.slots[t];
  if (slot < 0 || static_cast<uint64_t>(slot) >= p.n_slots) return;
  const uint64_t block = static_cast<uint64_t>(slot) / p.block_tokens;
  const uint64_t o = static_cast<uint64_t>(slot) - block * p.block_tokens;
  uint8_t* base = p.pool + block * p.block_tokens * p.record_bytes;
  const uint8_t* row = p.src[0] + static_cast<int64_t>(t) * p.src_stride[0];
  float most = 0;
  bool odd = false;  // an infinity or a NaN
  for (uint32_t v = lane; v < p.split_bytes; v += 64) {
    const float x = fabsf(load_value(row, v, p.src_type));
    odd |= !(x < __builtin_inff());
    most = fmaxf(most, x);
  }
  for (int d = 32; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
  odd = __any(odd);
  const float scale = odd ? __builtin_nanf("") : most / 448.0f;
  for (uint32_t w = lane; w < p.split_bytes / 4; w += 64) {
    float x[4];
    for (int k = 0; k < 4; ++k) {
      const float y = odd || scale == 0 ? 0.0f : load_value(row, 4 * w + k, p.src_type) / scale;
      x[k] = fminf(fmaxf(y, -448.0f), 448.0f);
    }
    reinterpret_cast<uint32_t*>(base + o * p.split_bytes)[w] = pack_e4m3(x[0], x[1], x[2], x[3]);
  }
  if (lane == 0) reinterpret_cast<float*>(base + static_cast<uint64_t>(p.block_tokens) * p.split_bytes)[o] = scale;
}

}  // namespace

hipError_t launch_tables_build(const TablesBuildParams& p, hipStream_t s) {
  const uint64_t want = (static_cast<uint64_t>(p.n_slots) + kTablesThreads - 1) / kTablesThreads;
  const uint32_t grid = static_cast<uint32_t>(want < 1 ? 1 : want > 1024 ? 1024 : want);
  const uint32_t lds = (1 + p.n_groups) * (p.n_requests + 1) * sizeof(uint32_t);
  hipLaunchKernelGGL(k_tables_build, dim3(grid), dim3(kTablesThreads), lds, s, p);
  return hipGetLastError();
}

hipError_t launch_append(const AppendParams& p, hipStream_t s) {
  if (p.split_bytes) {
    const uint32_t per = kAppendThreads / 64;
    hipLaunchKernelGGL(k_append_scaled, dim3((p.n_tokens + per - 1) / per), dim3(kAppendThreads), 0, s, p);
  } else {
    const uint64_t n = static_cast<uint64_t>(p.n_tokens) * p.units;
    hipLaunchKernelGGL(k_append, dim3(static_cast<uint32_t>((n + kAppendThreads - 1) / kAppendThreads)),
                       dim3(kAppendThreads), 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace bsr
