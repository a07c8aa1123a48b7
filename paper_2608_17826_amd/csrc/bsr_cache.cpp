// Host side of the paged cache's operators: argument checks and launches
// behind include/bsr.h.  Nothing is allocated, no device memory is read and no
// lock is taken; the context gives the layout and the device alone.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "bsr_cache.h"

namespace {

int refuse(int code, const char* fmt, ...) {
  char buf[400];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return bsr::set_error(code, buf);
}

// Makes the context's device current while a call enqueues its work.
class OnDevice {
 public:
  explicit OnDevice(int device) {
    err_ = hipGetDevice(&before_);
    if (err_ == hipSuccess && before_ != device) {
      err_ = hipSetDevice(device);
      moved_ = err_ == hipSuccess;
    }
  }
  ~OnDevice() {
    if (moved_) (void)hipSetDevice(before_);
  }
  hipError_t error() const { return err_; }

 private:
  int before_ = 0;
  bool moved_ = false;
  hipError_t err_;
};

// Refusals come before the device, so that a host-only context tells them too.
int check_device(const bsr_ctx* c) {
  if (bsr::ctx_device(c) < 0) return refuse(BSR_E_DEVICE, "operation needs a GPU context (hip_device >= 0)");
  return BSR_OK;
}

template <typename Launch>
int enqueue(const bsr_ctx* c, const char* what, Launch launch) {
  if (int rc = check_device(c)) return rc;
  OnDevice on(bsr::ctx_device(c));
  hipError_t e = on.error();
  if (e == hipSuccess) e = launch();
  if (e != hipSuccess) return refuse(BSR_E_TRANSFER, "%s: %s", what, hipGetErrorString(e));
  return BSR_OK;
}

int check_ctx(const bsr_ctx* c, const void* args) {
  if (!c || !args) return refuse(BSR_E_ARG, "context or args is NULL");
  return BSR_OK;
}

bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
  const auto x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

bool aligned(const void* p, uint64_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// A stride of values in bytes; one that 64 bits do not hold wraps round, as addresses would.
int64_t bytes_of(int64_t stride, uint32_t size) { return static_cast<int64_t>(static_cast<uint64_t>(stride) * size); }

// Whether rows of `width` values that begin at t * st + h * sh (t < nt, h < nh) overlap.
bool rows_overlap(int64_t st, int64_t nt, int64_t sh, int64_t nh, int64_t width) {
  if (nt < 1 || nh < 1) return false;
  const __int128 at = st < 0 ? -static_cast<__int128>(st) : st, ah = sh < 0 ? -static_cast<__int128>(sh) : sh;
  // one within the other, as tensors and their views have it
  if ((nt == 1 || at >= (nh - 1) * ah + width) && (nh == 1 || ah >= width)) return false;
  if ((nh == 1 || ah >= (nt - 1) * at + width) && (nt == 1 || at >= width)) return false;
  // any other two strides: for each distance of heads the distances of tokens that come closest
  for (int64_t dh = 0; dh < nh; ++dh) {
    const __int128 h = static_cast<__int128>(dh) * sh, near = st ? -h / st : 0;
    for (int i = -1; i <= 1; ++i) {
      const __int128 dt = near + i < 1 - nt ? 1 - nt : near + i > nt - 1 ? nt - 1 : near + i;
      const __int128 gap = dt * st + h;
      if ((dt || dh) && gap < width && -gap < width) return true;
    }
  }
  return false;
}

int check_attn(const bsr_ctx* c, const bsr_attn_args* a, bsr::AttnParams* p) {
  const bsr_layout* L = bsr::ctx_layout(c);
  if (a->group >= L->n_groups) return refuse(BSR_E_ARG, "group %u of %u", a->group, L->n_groups);
  const bsr_group_desc& d = L->groups[a->group];
  if (d.kind != BSR_KIND_CONTIG || d.record_bytes % 16)
    return refuse(BSR_E_ARG, "attention reads CONTIG groups with records of a multiple of 16 bytes");
  if (a->dtype != BSR_TYPE_BF16 && a->dtype != BSR_TYPE_F16) return refuse(BSR_E_ARG, "dtype is bf16 or f16");
  const bool latent = a->k_dim == 576 && a->v_dim == 512;
  if (!latent && !((a->k_dim == 64 || a->k_dim == 128) && a->v_dim == a->k_dim))
    return refuse(BSR_E_ARG, "(k_dim, v_dim) = (%u, %u): (64, 64), (128, 128) or (576, 512)", a->k_dim, a->v_dim);
  if (a->n_heads == 0 || a->n_kv_heads == 0 || a->n_heads % a->n_kv_heads || a->n_heads > 4096)
    return refuse(BSR_E_ARG, "n_heads (1..4096) must be a multiple of n_kv_heads");
  if (latent && (a->n_kv_heads != 1 || a->k_pool != a->v_pool || a->k_offset != a->v_offset))
    return refuse(BSR_E_ARG, "latent records have one KV head, and their value lies in the key");
  if (a->k_offset % 16 || a->v_offset % 16) return refuse(BSR_E_ARG, "record offsets must be multiples of 16");
  if (a->k_offset + 2ull * a->n_kv_heads * a->k_dim > d.record_bytes ||
      a->v_offset + 2ull * a->n_kv_heads * a->v_dim > d.record_bytes)
    return refuse(BSR_E_ARG, "the heads reach past a record of %u bytes", d.record_bytes);
  if (a->n_requests >= (1u << 20) || a->n_tokens >= (1u << 24) || a->max_len >= (1u << 30) || a->window >= (1u << 30))
    return refuse(BSR_E_ARG, "n_requests below 2^20, n_tokens below 2^24, max_len and window below 2^30");
  if (!(a->scale > 0) || !std::isfinite(a->scale)) return refuse(BSR_E_ARG, "scale must be positive and finite");
  if (!(a->softcap >= 0) || !std::isfinite(a->softcap) || (a->softcap > 0 && !std::isfinite(4 * (a->scale / a->softcap))))
    return refuse(BSR_E_ARG, "softcap must be 0, or positive and finite, and so must scale / softcap");
  if (a->q_token_stride % 8 || a->q_head_stride % 8 || a->out_token_stride % 8 || a->out_head_stride % 8)
    return refuse(BSR_E_ARG, "strides must be multiples of 8 values");
  if (a->reserved) return refuse(BSR_E_ARG, "reserved must be 0");
  if (!p || a->n_requests == 0 || a->n_tokens == 0) return BSR_OK;  // (nothing is launched without rows)
  if (!a->q || !a->out || !a->k_pool || !a->v_pool || !a->tables || !a->starts || !a->lens)
    return refuse(BSR_E_ARG, "NULL pointer");
  if (!aligned(a->q, 16) || !aligned(a->out, 16) || !aligned(a->k_pool, 16) || !aligned(a->v_pool, 16))
    return refuse(BSR_E_ARG, "q, out and the pools must be 16-byte aligned");
  if (!aligned(a->tables, 4) || !aligned(a->starts, 4) || !aligned(a->lens, 4) || !aligned(a->lse, 4) ||
      !aligned(a->tree, 8) || !aligned(a->slopes, 4) || !aligned(a->prefix, 4) || !aligned(a->documents, 4))
    return refuse(BSR_E_ARG, "an array is not aligned to its type");
  if (a->pool_blocks == 0 || a->pool_blocks >= (1u << 31)) return refuse(BSR_E_ARG, "pool_blocks must be in 1..2^31-1");
  if (a->table_stride == 0) return refuse(BSR_E_ARG, "table_stride is 0");
  if (rows_overlap(a->out_token_stride, a->n_tokens, a->out_head_stride, a->n_heads, a->v_dim))
    return refuse(BSR_E_ARG, "rows of out overlap");
  p->q = static_cast<const uint8_t*>(a->q);
  p->out = static_cast<uint8_t*>(a->out);
  p->lse = a->lse;
  p->k_pool = static_cast<const uint8_t*>(a->k_pool) + a->k_offset;
  p->v_pool = static_cast<const uint8_t*>(a->v_pool) + a->v_offset;
  p->tables = a->tables;
  p->starts = a->starts;
  p->lens = a->lens;
  p->q_token = bytes_of(a->q_token_stride, 2);
  p->q_head = bytes_of(a->q_head_stride, 2);
  p->out_token = bytes_of(a->out_token_stride, 2);
  p->out_head = bytes_of(a->out_head_stride, 2);
  p->block_bytes = static_cast<uint64_t>(d.block_tokens) * d.record_bytes;
  p->n_requests = a->n_requests;
  p->n_tokens = a->n_tokens;
  p->n_heads = a->n_heads;
  p->n_kv_heads = a->n_kv_heads;
  p->k_dim = a->k_dim;
  p->v_dim = a->v_dim;
  p->f16 = a->dtype == BSR_TYPE_F16;
  p->record_bytes = d.record_bytes;
  p->pool_blocks = a->pool_blocks;
  p->table_stride = a->table_stride;
  const uint64_t holds = static_cast<uint64_t>(a->table_stride) * d.block_tokens;
  p->max_len = holds < a->max_len ? static_cast<uint32_t>(holds) : a->max_len;
  p->window = a->window;
  p->scale = a->scale;
  p->softcap = a->softcap;
  p->div_block = bsr::make_fastdiv(d.block_tokens);
  return BSR_OK;
}

bsr::AttnTiling tiling_of(const bsr_attn_args* a) {
  return bsr::attn_tiling(a->n_requests, a->n_tokens, a->n_heads, a->n_kv_heads, a->v_dim, a->max_len);
}

int check_tiling(const bsr::AttnTiling& t) {
  if (t.items >= (1ull << 24)) return refuse(BSR_E_ARG, "too many rows and heads for one launch");
  return BSR_OK;
}

int attend(const bsr_ctx* c, const bsr_attn_args* a, bsr::AttnParams* p, void* stream) {
  if (a->n_requests == 0 || a->n_tokens == 0) return check_device(c);
  const bsr::AttnTiling t = tiling_of(a);
  if (int rc = check_tiling(t)) return rc;
  if (t.workspace && (!a->workspace || !aligned(a->workspace, 16) || a->workspace_bytes < t.workspace))
    return refuse(BSR_E_ARG, "workspace is NULL, not 16-byte aligned or smaller than %llu bytes",
                  static_cast<unsigned long long>(t.workspace));
  p->tile_rows = t.tile_rows;
  p->tile_heads = t.tile_heads;
  p->tile_tokens = t.tile_tokens;
  p->units = t.units;
  p->target = t.target;
  p->min_part = t.min_part;
  p->parts = static_cast<uint32_t>(t.slots);
  p->part = static_cast<float*>(a->workspace);
  p->part_ml = p->part + t.slots * t.tile_rows * a->v_dim;
  return enqueue(c, "attention", [&] { return bsr::launch_attention(*p, static_cast<hipStream_t>(stream)); });
}

}  // namespace

namespace bsr {

AttnTiling attn_tiling(uint32_t n_requests, uint32_t n_tokens, uint32_t n_heads, uint32_t n_kv_heads, uint32_t v_dim,
                       uint32_t max_len) {
  AttnTiling t{};
  const uint32_t per_kv = n_heads / n_kv_heads;
  t.tile_heads = per_kv < kTileRows ? per_kv : kTileRows;
  t.tile_rows = kTileRows;
  if (v_dim == 512 && n_requests && n_tokens && n_tokens % n_requests == 0) {
    // requests of as many rows each, it seems (and at least one): no more row blocks
    // than those need (16 rows over 128K: 52 us in a tile of 32, 69 in one of 128).
    // A padded row more, or rows that do not divide evenly, and all tiles have 128.
    const uint64_t rows = static_cast<uint64_t>(n_tokens) / n_requests * t.tile_heads;
    t.tile_rows = rows <= 32 ? 32 : rows <= 64 ? 64 : kTileRows;
  }
  t.tile_tokens = t.tile_rows / t.tile_heads;
  t.units = n_kv_heads * ((per_kv + t.tile_heads - 1) / t.tile_heads);
  // every request may end a tile early; none has a tile without a token
  const uint64_t tiles = (n_tokens / t.tile_tokens) + static_cast<uint64_t>(n_requests < n_tokens ? n_requests : n_tokens);
  t.base = t.items = tiles * t.units;
  // two steps: one latent token over 1,000 keys takes 17.5 us, 20.7 with parts of 128
  // at least; 20 tokens of heads of 128 14.6, 15.9 with 256, 15.2 with 64
  t.min_part = v_dim == 512 ? 64 : 128;
  if (max_len > t.min_part) {
    t.target = v_dim == 512 ? 256 : v_dim == 128 ? 512 : kMaxTarget;  // workgroups that the GPU holds at once
    const uint64_t parts = t.base <= t.target ? t.target : 2 * t.target;
    const uint64_t most = t.base * ((max_len + t.min_part - 1) / t.min_part);
    t.slots = most < parts ? most : parts;
    if (t.items < t.slots) t.items = t.slots;
    t.workspace = t.slots * t.tile_rows * (v_dim + 2) * sizeof(float);
  }
  return t;
}

}  // namespace bsr

extern "C" {

int bsr_tables_build(bsr_ctx* c, const bsr_tables_args* a, void* stream) {
  if (int rc = check_ctx(c, a)) return rc;
  const bsr_layout* L = bsr::ctx_layout(c);
  if (a->n_requests > BSR_MAX_TABLE_REQUESTS)
    return refuse(BSR_E_ARG, "n_requests must be at most %d", BSR_MAX_TABLE_REQUESTS);
  if (a->n_slots >= (1u << 31)) return refuse(BSR_E_ARG, "n_slots below 2^31");
  if (!a->groups || !a->starts || !a->result || (a->n_requests && (!a->cached || !a->added || !a->lens)))
    return refuse(BSR_E_ARG, "NULL pointer");
  if (!aligned(a->cached, 4) || !aligned(a->added, 4) || !aligned(a->starts, 4) || !aligned(a->lens, 4) ||
      !aligned(a->result, 4))
    return refuse(BSR_E_ARG, "an array is not aligned to its type");
  const uint64_t n4 = 4ull * a->n_requests;
  for (const int32_t* in : {a->cached, a->added})
    if (overlap(in, n4, a->lens, n4) || overlap(in, n4, a->starts, n4 + 4))
      return refuse(BSR_E_ARG, "lens and starts must not overlap cached or added");
  bsr::TablesBuildParams p{};
  p.n_requests = a->n_requests;
  p.n_slots = a->n_slots;
  p.n_groups = L->n_groups;
  p.cached = a->cached;
  p.added = a->added;
  p.starts = a->starts;
  p.lens = a->lens;
  p.result = a->result;
  for (uint32_t g = 0; g < L->n_groups; ++g) {
    const bsr_table_group& t = a->groups[g];
    if (!t.tables && t.slots && a->n_requests) return refuse(BSR_E_ARG, "group %u: slots without tables", g);
    if (t.tables && (t.table_stride == 0 || (t.n_free && !t.free_blocks)))
      return refuse(BSR_E_ARG, "group %u: table_stride is 0 or free_blocks is NULL", g);
    if (!aligned(t.tables, 4) || !aligned(t.free_blocks, 4) || !aligned(t.slots, 8))
      return refuse(BSR_E_ARG, "group %u: an array is not aligned to its type", g);
    if (t.n_free >= (1u << 31)) return refuse(BSR_E_ARG, "group %u: n_free below 2^31", g);
    p.g[g] = {t.free_blocks, t.tables, t.slots, t.n_free, t.table_stride, bsr::make_fastdiv(L->groups[g].block_tokens)};
  }
  return enqueue(c, "bsr_tables_build", [&] { return bsr::launch_tables_build(p, static_cast<hipStream_t>(stream)); });
}

int bsr_cache_append(bsr_ctx* c, const bsr_append_args* a, void* stream) {
  if (int rc = check_ctx(c, a)) return rc;
  const bsr_layout* L = bsr::ctx_layout(c);
  if (a->group >= L->n_groups) return refuse(BSR_E_ARG, "group %u of %u", a->group, L->n_groups);
  const bsr_group_desc& d = L->groups[a->group];
  const bool planar = d.kind == BSR_KIND_PLANAR;
  if (a->src_type != BSR_TYPE_BF16 && a->src_type != BSR_TYPE_F16 && a->src_type != BSR_TYPE_F32)
    return refuse(BSR_E_ARG, "src_type is bf16, f16 or f32");
  if (planar ? a->cache_type != BSR_TYPE_E4M3_SCALED : a->cache_type != BSR_TYPE_BF16 && a->cache_type != BSR_TYPE_F16)
    return refuse(BSR_E_ARG, "cache_type is bf16 or f16 of a CONTIG group, scaled e4m3 of a PLANAR one");
  if (a->n_sources < 1 || a->n_sources > 2 || (planar && a->n_sources != 1))
    return refuse(BSR_E_ARG, "one or two sources, one of a PLANAR group");
  if (planar && d.record_bytes != d.split_bytes + 4)
    return refuse(BSR_E_ARG, "a scaled record is split_bytes values and an fp32 scale");
  const uint32_t size = a->src_type == BSR_TYPE_F32 ? 4 : 2;
  uint64_t values = 0;
  for (uint32_t i = 0; i < a->n_sources; ++i) {
    if (a->width[i] == 0) return refuse(BSR_E_ARG, "source %u has no values", i);
    values += a->width[i];
    if (a->n_tokens && (!a->src[i] || !aligned(a->src[i], size))) return refuse(BSR_E_ARG, "source %u is NULL or not aligned", i);
    if (a->src_stride[i] < 0 || static_cast<uint64_t>(a->src_stride[i]) < a->width[i])
      return refuse(BSR_E_ARG, "source %u: rows overlap", i);
  }
  if (values != (planar ? d.split_bytes : d.record_bytes / 2))
    return refuse(BSR_E_ARG, "the sources' %llu values are not a record's", static_cast<unsigned long long>(values));
  if (a->n_tokens >= (1u << 24)) return refuse(BSR_E_ARG, "n_tokens below 2^24");
  if (a->n_tokens == 0) return check_device(c);
  if (!a->slots || !a->pool || !aligned(a->slots, 8) || !aligned(a->pool, 16))
    return refuse(BSR_E_ARG, "slots or pool is NULL or not aligned");
  bsr::AppendParams p{};
  p.slots = a->slots;
  p.pool = static_cast<uint8_t*>(a->pool);
  p.vector = planar || d.record_bytes % 16 == 0;
  for (uint32_t i = 0; i < a->n_sources; ++i) {
    p.src[i] = static_cast<const uint8_t*>(a->src[i]);
    p.src_stride[i] = bytes_of(a->src_stride[i], size);
    p.width[i] = a->width[i];
    p.vector &= aligned(a->src[i], 16) && p.src_stride[i] % 16 == 0 && p.width[i] % 8 == 0;
  }
  p.n_tokens = a->n_tokens;
  p.record_bytes = d.record_bytes;
  p.block_tokens = d.block_tokens;
  p.split_bytes = planar ? d.split_bytes : 0;
  p.src_type = a->src_type;
  p.cache_type = a->cache_type;
  p.n_slots = static_cast<uint64_t>(a->pool_blocks) * d.block_tokens;
  p.units = static_cast<uint32_t>(p.vector ? values / 8 : values);
  p.div_units = bsr::make_fastdiv(p.units);
  p.div_block = bsr::make_fastdiv(d.block_tokens);
  if (!planar && static_cast<uint64_t>(a->n_tokens) * p.units >= (1ull << 32) - 256)
    return refuse(BSR_E_ARG, "too many values for one launch");
  return enqueue(c, "bsr_cache_append", [&] { return bsr::launch_append(p, static_cast<hipStream_t>(stream)); });
}

uint64_t bsr_attn_workspace_bytes(bsr_ctx* c, const bsr_attn_args* a) {
  if (check_ctx(c, a) || check_attn(c, a, nullptr)) return BSR_ATTN_REFUSED;
  const bsr::AttnTiling t = tiling_of(a);
  return check_tiling(t) ? BSR_ATTN_REFUSED : t.workspace;
}

int bsr_attend_tree(bsr_ctx* c, const bsr_attn_args* a, void* stream) {
  if (int rc = check_ctx(c, a)) return rc;
  bsr::AttnParams p{};
  if (int rc = check_attn(c, a, &p)) return rc;
  if (a->slopes || a->prefix || a->documents) return refuse(BSR_E_ARG, "slopes, prefix and documents belong to bsr_attend_prompt");
  if (a->tree_words < 1 || a->tree_words > BSR_MAX_TREE_WORDS)
    return refuse(BSR_E_ARG, "tree_words must be in 1..%d", BSR_MAX_TREE_WORDS);
  if (a->n_requests && a->n_tokens && !a->tree) return refuse(BSR_E_ARG, "tree is NULL");
  if (a->window && a->window < 64 * a->tree_words)
    return refuse(BSR_E_ARG, "a window must hold a whole tree (64 * tree_words = %u)", 64 * a->tree_words);
  p.tree = a->tree;
  p.tree_words = a->tree_words;
  return attend(c, a, &p, stream);
}

int bsr_attend_prompt(bsr_ctx* c, const bsr_attn_args* a, void* stream) {
  if (int rc = check_ctx(c, a)) return rc;
  bsr::AttnParams p{};
  if (int rc = check_attn(c, a, &p)) return rc;
  if (a->tree || a->tree_words) return refuse(BSR_E_ARG, "tree belongs to bsr_attend_tree");
  p.slopes = a->slopes;
  p.prefix = a->prefix;
  p.documents = a->documents;
  return attend(c, a, &p, stream);
}

}  // extern "C"
