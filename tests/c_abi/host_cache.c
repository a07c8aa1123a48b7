/* The paged cache's entry points from plain C11, on a host-only context: sizes
 * of their structs, refusals, and sizes and strides at the ends of their ranges.
 * Addresses are made up; nothing is read through them.  Exits non-zero on the
 * first violated expectation. */
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "bsr.h"

#define CHECK(cond)                                                                         \
  do {                                                                                      \
    if (!(cond)) {                                                                          \
      fprintf(stderr, "FAILED %s:%d: %s (%s)\n", __FILE__, __LINE__, #cond, bsr_last_error()); \
      return 1;                                                                             \
    }                                                                                       \
  } while (0)

static char* const A = (char*)(uintptr_t)(1 << 20); /* an aligned address */

static bsr_attn_args heads(void) {
  bsr_attn_args a;
  memset(&a, 0, sizeof a);
  a.group = 1;
  a.dtype = BSR_TYPE_BF16;
  a.n_requests = a.n_tokens = 2;
  a.n_heads = 8;
  a.n_kv_heads = 1;
  a.k_dim = a.v_dim = 128;
  a.q = a.out = a.lse = (void*)A;
  a.q_token_stride = a.out_token_stride = 1024;
  a.q_head_stride = a.out_head_stride = 128;
  a.k_pool = a.v_pool = A;
  a.v_offset = 256;
  a.pool_blocks = 10;
  a.table_stride = 4;
  a.tables = a.starts = a.lens = (const int32_t*)A;
  a.max_len = 64;
  a.scale = 0.1f;
  a.workspace = A;
  a.workspace_bytes = UINT64_MAX;
  return a;
}

int main(void) {
  CHECK(bsr_struct_size(BSR_STRUCT_TABLE_GROUP) == sizeof(bsr_table_group));
  CHECK(bsr_struct_size(BSR_STRUCT_TABLES_ARGS) == sizeof(bsr_tables_args));
  CHECK(bsr_struct_size(BSR_STRUCT_APPEND_ARGS) == sizeof(bsr_append_args));
  CHECK(bsr_struct_size(BSR_STRUCT_ATTN_ARGS) == sizeof(bsr_attn_args));

  bsr_layout L;
  memset(&L, 0, sizeof L);
  L.chunk_tokens = 256;
  L.n_groups = 3;
  L.groups[0] = (bsr_group_desc){64, 1, 1152, BSR_KIND_CONTIG, 0};
  L.groups[1] = (bsr_group_desc){32, 1, 512, BSR_KIND_CONTIG, 0};
  L.groups[2] = (bsr_group_desc){128, 1, 132, BSR_KIND_PLANAR, 128};
  bsr_config cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.window_chunks = 1;
  cfg.hip_device = -1;
  bsr_ctx* c = NULL;
  CHECK(bsr_ctx_create(&L, &cfg, &c) == BSR_OK);

  /* attention */
  bsr_attn_args a = heads(), t = heads();
  t.tree = (const uint64_t*)A;
  t.tree_words = 1;
  CHECK(bsr_attend_prompt(NULL, &a, NULL) == BSR_E_ARG && bsr_attend_prompt(c, NULL, NULL) == BSR_E_ARG);
  CHECK(bsr_attend_tree(NULL, &t, NULL) == BSR_E_ARG && bsr_attend_tree(c, NULL, NULL) == BSR_E_ARG);
  CHECK(bsr_attn_workspace_bytes(NULL, &a) == BSR_ATTN_REFUSED && bsr_attn_workspace_bytes(c, NULL) == BSR_ATTN_REFUSED);
  CHECK(bsr_attend_prompt(c, &a, NULL) == BSR_E_DEVICE && bsr_attend_tree(c, &t, NULL) == BSR_E_DEVICE);
  CHECK(bsr_attend_prompt(c, &t, NULL) == BSR_E_ARG && bsr_attend_tree(c, &a, NULL) == BSR_E_ARG);
  /* no rows: no pointer is needed, whatever else is set */
  a = heads();
  a.n_tokens = 0;
  a.q = a.out = a.lse = a.workspace = NULL;
  a.k_pool = a.v_pool = NULL;
  a.tables = a.starts = a.lens = NULL;
  a.workspace_bytes = 0;
  CHECK(bsr_attn_workspace_bytes(c, &a) == 0 && bsr_attend_prompt(c, &a, NULL) == BSR_E_DEVICE);
  a.n_requests = 0;
  CHECK(bsr_attend_prompt(c, &a, NULL) == BSR_E_DEVICE);
  /* strides to the ends of 64 bits */
  static const int64_t far[] = {INT64_MIN, INT64_MIN + 8, -(INT64_C(1) << 62), INT64_C(1) << 62, INT64_MAX - 7, 0, 8, -8};
  for (unsigned i = 0; i < sizeof far / sizeof *far; ++i)
    for (unsigned k = 0; k < sizeof far / sizeof *far; ++k) {
      a = heads();
      a.q_token_stride = far[i];
      a.q_head_stride = far[k];
      CHECK(bsr_attend_prompt(c, &a, NULL) == BSR_E_DEVICE);
      a.out_token_stride = far[i];
      a.out_head_stride = far[k];
      a.n_tokens = 5;
      const int rc = bsr_attend_prompt(c, &a, NULL);
      CHECK(rc == BSR_E_DEVICE || rc == BSR_E_ARG);
      a.n_tokens = a.n_heads = 1;
      CHECK(bsr_attend_prompt(c, &a, NULL) == BSR_E_DEVICE);
    }
  /* every workspace size, or a refusal, without a division by zero or an overflow */
  static const uint32_t some[] = {0, 1, 2, 3, 31, 64, 65, 300, 4096, (1u << 20) - 1, (1u << 24) - 1, (1u << 30) - 1, UINT32_MAX};
  enum { N = sizeof some / sizeof *some };
  for (unsigned latent = 0; latent < 2; ++latent)
    for (unsigned r = 0; r < N; ++r)
      for (unsigned n = 0; n < N; ++n)
        for (unsigned h = 0; h < N; ++h)
          for (unsigned m = 0; m < N; ++m) {
            a = heads();
            if (latent) a.group = 0, a.k_dim = 576, a.v_dim = 512, a.v_offset = 0;
            a.n_requests = some[r];
            a.n_tokens = some[n];
            a.n_heads = some[h];
            a.max_len = some[m];
            const uint64_t bytes = bsr_attn_workspace_bytes(c, &a);
            CHECK(bytes == BSR_ATTN_REFUSED || bytes <= (UINT64_C(1) << 32));
          }

  /* append */
  bsr_append_args p;
  memset(&p, 0, sizeof p);
  p.group = 1;
  p.n_tokens = 3;
  p.slots = (const int64_t*)A;
  p.pool = A;
  p.pool_blocks = 4;
  p.n_sources = 2;
  p.src[0] = p.src[1] = A;
  p.width[0] = p.width[1] = 128;
  p.src_stride[0] = p.src_stride[1] = INT64_MAX;
  CHECK(bsr_cache_append(NULL, &p, NULL) == BSR_E_ARG && bsr_cache_append(c, NULL, NULL) == BSR_E_ARG);
  CHECK(bsr_cache_append(c, &p, NULL) == BSR_E_DEVICE);
  p.src_type = BSR_TYPE_F32;
  p.pool_blocks = UINT32_MAX;
  CHECK(bsr_cache_append(c, &p, NULL) == BSR_E_DEVICE);
  p.src_stride[1] = INT64_MIN;
  CHECK(bsr_cache_append(c, &p, NULL) == BSR_E_ARG);
  p.src_stride[1] = 128;
  p.width[1] = UINT32_MAX;
  CHECK(bsr_cache_append(c, &p, NULL) == BSR_E_ARG);
  p.group = UINT32_MAX;
  CHECK(bsr_cache_append(c, &p, NULL) == BSR_E_ARG);

  /* tables */
  bsr_table_group g[3];
  for (int i = 0; i < 3; ++i) g[i] = (bsr_table_group){(const int32_t*)A, (int32_t*)A, (int64_t*)A, 0x7fffffff, UINT32_MAX};
  bsr_tables_args b;
  memset(&b, 0, sizeof b);
  b.n_requests = 3;
  b.n_slots = 0x7fffffff;
  b.cached = (const int32_t*)A;
  b.added = (const int32_t*)(A + 64);
  b.starts = (int32_t*)(A + 128);
  b.lens = (int32_t*)(A + 192);
  b.result = (uint32_t*)(A + 256);
  b.groups = g;
  CHECK(bsr_tables_build(NULL, &b, NULL) == BSR_E_ARG && bsr_tables_build(c, NULL, NULL) == BSR_E_ARG);
  CHECK(bsr_tables_build(c, &b, NULL) == BSR_E_DEVICE);
  b.lens = (int32_t*)(uintptr_t)(UINTPTR_MAX - 3); /* the last word there is */
  CHECK(bsr_tables_build(c, &b, NULL) == BSR_E_DEVICE);
  b.lens = (int32_t*)(A + 8);
  CHECK(bsr_tables_build(c, &b, NULL) == BSR_E_ARG);
  b.lens = (int32_t*)(A + 192);
  b.groups = NULL;
  CHECK(bsr_tables_build(c, &b, NULL) == BSR_E_ARG);
  CHECK(bsr_ctx_destroy(c) == BSR_OK);
  puts("ok");
  return 0;
}
