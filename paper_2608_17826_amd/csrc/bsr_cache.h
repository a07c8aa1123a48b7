// Internal interface of the paged cache's operators (block tables and slot
// maps, append, attention): what bsr_cache.cpp hands to the kernels in
// bsr_cache.hip and bsr_attention.hip.
#pragma once

#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "bsr.h"
#include "bsr_device.h"

namespace bsr {

// of bsr_runtime.cpp
const bsr_layout* ctx_layout(const bsr_ctx* c);
int ctx_device(const bsr_ctx* c);
int set_error(int code, const char* message);

// ---- block tables and slot maps ------------------------------------------------
struct TablesBuildGroup {
  const int32_t* free_blocks;
  int32_t* tables;  // null: the group is left out
  int64_t* slots;   // may be null
  uint32_t n_free;
  uint32_t table_stride;
  FastDiv div_block;
};
struct TablesBuildParams {
  uint32_t n_requests;
  uint32_t n_slots;
  uint32_t n_groups;
  const int32_t* cached;
  const int32_t* added;
  int32_t* starts;
  int32_t* lens;
  uint32_t* result;
  TablesBuildGroup g[BSR_MAX_GROUPS];
};
hipError_t launch_tables_build(const TablesBuildParams& p, hipStream_t s);

// ---- append --------------------------------------------------------------------
struct AppendParams {
  const int64_t* slots;
  uint8_t* pool;
  const uint8_t* src[2];
  int64_t src_stride[2];  // bytes
  uint32_t width[2];
  uint32_t n_tokens;
  uint32_t record_bytes;
  uint32_t block_tokens;
  uint32_t split_bytes;   // 0: CONTIG
  uint32_t src_type, cache_type;
  uint64_t n_slots;       // pool_blocks * block_tokens
  FastDiv div_units;      // CONTIG: by the units of a record
  uint32_t units;         // CONTIG: 8-value units of a record, or its values
  uint32_t vector;        // whole units of 8 values, 16-byte aligned everywhere (PLANAR: in the source)
  FastDiv div_block;      // by block_tokens
};
hipError_t launch_append(const AppendParams& p, hipStream_t s);

// ---- attention -------------------------------------------------------------------
struct AttnParams {
  const uint8_t* q;
  uint8_t* out;
  float* lse;
  const uint8_t* k_pool;  // at the first KV head's key (value)
  const uint8_t* v_pool;
  const int32_t* tables;
  const int32_t* starts;
  const int32_t* lens;
  const uint64_t* tree;   // null: prompt
  const float* slopes;
  const int32_t* prefix;
  const int32_t* documents;
  int64_t q_token, q_head, out_token, out_head;  // strides in bytes
  uint64_t block_bytes;
  uint32_t n_requests, n_tokens, n_heads, n_kv_heads;
  uint32_t k_dim, v_dim;
  uint32_t f16;           // 1: fp16, 0: bf16
  uint32_t record_bytes, pool_blocks, table_stride;
  uint32_t max_len;       // min(max_len, what a table holds)
  uint32_t window, tree_words;
  float scale, softcap;
  FastDiv div_block;      // by block_tokens
  // the tiling (attn_tiling)
  uint32_t tile_rows;     // query rows of a tile
  uint32_t tile_heads;    // query heads of a KV head that a tile takes: min(its heads, tile_rows)
  uint32_t tile_tokens;   // tokens of a tile: tile_rows / tile_heads
  uint32_t units;         // tiles beside one another of the same tokens: KV heads x chunks of their heads
  uint32_t target;        // parts that the batch's key ranges are cut into, about; 0: never cut
  uint32_t min_part;      // keys of a part, at least
  uint32_t parts;         // parts that the workspace holds
  float* part;            // workspace: sums of parts [slot][tile_rows][v_dim], then their (maximum, sum)
  float* part_ml;
};

// An attention tile is up to kTileRows query rows (tokens x heads of one KV head).
constexpr uint32_t kTileRows = 128;
constexpr uint32_t kMaxTarget = 768;

struct AttnTiling {
  uint32_t tile_rows, tile_heads, tile_tokens, units, target, min_part;
  uint64_t base;      // tiles x units of the batch, at most
  uint64_t items;     // parts of them, at most
  uint64_t slots;     // partial results, at most
  uint64_t workspace; // bytes
};
AttnTiling attn_tiling(uint32_t n_requests, uint32_t n_tokens, uint32_t n_heads, uint32_t n_kv_heads, uint32_t v_dim,
                       uint32_t max_len);
hipError_t launch_attention(const AttnParams& p, hipStream_t s);

}  // namespace bsr
