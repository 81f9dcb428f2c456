/*
 * Host-side paths of every rdf2v.h entry point, for a library built with
 * AddressSanitizer and UndefinedBehaviorSanitizer on its host code: the
 * workspace-size functions at extreme sizes, and each call with arguments
 * that the host rejects before any HIP call (so no device is needed and the
 * fake device pointers are never dereferenced). Any undefined behaviour in the
 * size arithmetic or the checks ends the run with an error.
 */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "rdf2v.h"

#define EXPECT(cond)                                                  \
  do {                                                                \
    if (!(cond)) {                                                    \
      fprintf(stderr, "failed: %s (line %d)\n", #cond, __LINE__);     \
      exit(1);                                                        \
    }                                                                 \
  } while (0)

static void *fake(uintptr_t addr) { return (void *)addr; }

/* The operators of a sequence model over walk tokens. */
static size_t model_entries(const int64_t *big64, size_t n64, const int32_t *big32, size_t n32) {
  size_t sink = 0;
  void *F = fake((uintptr_t)1 << 40), *W = fake((uintptr_t)1 << 44);
  float *FF = (float *)F, *WF = (float *)W;
  int32_t *FI = (int32_t *)F, *WI = (int32_t *)W;
  const int64_t lengths[] = {0, 1, 448, 449, 1024, ((int64_t)1 << 31) - 1, INT64_MAX, INT64_MIN};
  for (size_t i = 0; i < n64; ++i) {
    for (size_t j = 0; j < sizeof(lengths) / sizeof(lengths[0]); ++j)
      for (size_t k = 0; k < n32; ++k)
        for (size_t l = 0; l < n32; ++l) {
          const rdf2v_attention a = {big64[i], lengths[j], big32[k], big32[l], 1 + (int32_t)(l % 128), 128, RDF2V_F32,
                                     1.0f, NULL, NULL};
          rdf2v_attention b = a;
          b.kv_heads = b.heads;
          b.dk = big32[l];
          sink += rdf2v_decay_attention_workspace_size(&a) + rdf2v_decay_attention_backward_workspace_size(&a);
          sink += rdf2v_decay_attention_workspace_size(&b) + rdf2v_decay_attention_backward_workspace_size(&b);
        }
    for (size_t j = 0; j < n64; ++j)
      for (size_t k = 0; k < n32; ++k) {
        sink += rdf2v_beam_select_workspace_size(big64[i], big32[k], big64[j], 64);
        sink += rdf2v_beam_select_workspace_size(big64[i], 64, big64[j], big32[k]);
        sink += rdf2v_distill_workspace_size(big64[i], big64[j], big32[k], RDF2V_BF16);
        sink += rdf2v_distill_workspace_size(big64[i], big64[j], 512, big32[k]);
      }
  }

  /* decay attention */
  const rdf2v_attention ok = {4, 10, 4, 2, 16, 24, RDF2V_F32, 1.0f, FF, NULL};
  const rdf2v_heads_view v = {F, 640, 64, 16}, none = {NULL, 640, 64, 16}, far = {F, INT64_MIN, INT64_MAX, INT64_MIN};
  rdf2v_attention a = ok;
  EXPECT(rdf2v_decay_attention(NULL, &v, &v, &v, NULL, W, NULL, NULL, 0, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_decay_attention(&ok, &v, &far, &v, NULL, W, NULL, NULL, 0, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_decay_attention(&ok, &v, &none, &v, NULL, W, NULL, NULL, 0, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_decay_attention_backward(&ok, &v, &v, &v, &v, NULL, NULL, W, W, W, NULL, NULL, 0, NULL, NULL) ==
         RDF2V_ERR_WORKSPACE);
  EXPECT(rdf2v_decay_attention_step(&ok, &v, &v, &v, FF, INT64_MAX, FI, W, WF, NULL, NULL) == RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_decay_attention_step(&ok, &v, &v, &v, FF, INT64_MIN, FI, W, WF, NULL, NULL) ==
         RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_decay_attention_step(&ok, &v, &v, &v, FF, 4, FI, W, FF, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  a.rows = ((int64_t)1 << 31) - 1;
  a.length = a.rows;
  EXPECT(rdf2v_decay_attention(&a, &v, &v, &v, NULL, W, NULL, NULL, 0, NULL, NULL) == RDF2V_ERR_TOO_LARGE);
  for (size_t i = 0; i < sizeof(lengths) / sizeof(lengths[0]); ++i) {
    a = ok;
    a.rows = 0;
    a.length = lengths[i];
    const rdf2v_status want = a.length < 0                   ? RDF2V_ERR_INVALID_ARGUMENT
                              : a.length >= (int64_t)1 << 31 ? RDF2V_ERR_TOO_LARGE
                                                             : RDF2V_OK;
    EXPECT(rdf2v_decay_attention(&a, &v, &v, &v, NULL, W, NULL, NULL, 0, NULL, NULL) == want);
    EXPECT(rdf2v_decay_attention_backward(&a, &v, &v, &v, &v, NULL, NULL, W, W, W, NULL, NULL, 0, NULL, NULL) == want);
  }

  /* beam selection and reordering */
  EXPECT(rdf2v_beam_select(F, INT64_MAX, RDF2V_F32, FF, NULL, 2, 3, 100, 4, WF, WI, WI, NULL, 0, NULL, NULL) ==
         RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_beam_select(F, INT64_MIN, RDF2V_F32, FF, NULL, 2, 3, 100, 4, WF, WI, WI, NULL, 0, NULL, NULL) ==
         RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_beam_select(F, 100, RDF2V_F32, FF, NULL, 2, 3, 100, 4, WF, WI, WI, NULL, 0, NULL, NULL) ==
         RDF2V_ERR_WORKSPACE);
  EXPECT(rdf2v_beam_reorder(F, INT64_MAX, INT64_MAX, FI, 1, W, NULL, NULL) == RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_beam_reorder(F, 1, INT64_MAX, FI, 1, W, NULL, NULL) == RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_beam_reorder(F, 1, INT64_MIN, FI, 1, W, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_beam_reorder(F, 4, 64, FI, 4, (char *)F + 255, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);

  /* distillation */
  EXPECT(rdf2v_distill_loss(F, INT64_MAX, RDF2V_F32, FI, FF, 8, 100, 4, 1.0f, WF, WF, NULL, NULL, 0, NULL, 0, NULL,
                            NULL) == RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_distill_loss(F, 100, RDF2V_F32, FI, FF, INT64_MIN, 100, 4, 1.0f, WF, WF, NULL, NULL, 0, NULL, 0, NULL,
                            NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_distill_loss(F, (int64_t)1 << 30, RDF2V_F32, FI, FF, 8, (int64_t)1 << 30, 4, 1.0f, WF, WF, NULL, NULL,
                            0, NULL, 0, NULL, NULL) == RDF2V_ERR_WORKSPACE);
  EXPECT(rdf2v_distill_loss_backward(F, 100, RDF2V_F32, FI, FF, 8, 100, 4, 1.0f, FF, FF, W, INT64_MIN, NULL, 0, NULL,
                                     NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_distill_loss_backward(F, 100, RDF2V_F32, FI, FF, 8, 100, 4, 1.0f, FF, FF, W, INT64_MAX, NULL, 0, NULL,
                                     NULL) == RDF2V_ERR_TOO_LARGE);
  return sink;
}

int main(void) {
  const int64_t big64[] = {0, 1, 4095, 4096, 4097, (int64_t)1 << 30, ((int64_t)1 << 31) - 1, (int64_t)1 << 31,
                           (int64_t)1 << 40, INT64_MAX, -1, INT64_MIN};
  const int32_t big32[] = {0, 1, 2, 255, 256, 1 << 17, (1 << 18) + 1, 1 << 26, INT32_MAX, -1, INT32_MIN};
  const size_t n64 = sizeof(big64) / sizeof(big64[0]), n32 = sizeof(big32) / sizeof(big32[0]);
  size_t sink = 0;
  for (size_t i = 0; i < n64; ++i) {
    for (size_t j = 0; j < n32; ++j) {
      sink += rdf2v_build_csr_workspace_size(big64[i], big32[j]);
      sink += rdf2v_bfs_walks_workspace_size(big32[j], big64[i]);
      sink += (size_t)rdf2v_walk_edges_recommended(big32[j], big64[i]);
      for (size_t k = 0; k < n64; ++k) sink += rdf2v_build_vocabulary_workspace_size(big64[i], big64[k], big64[k]);
    }
    sink += rdf2v_skipgram_pairs_workspace_size(big64[i]);
    sink += rdf2v_cbow_examples_workspace_size(big64[i]);
    sink += rdf2v_unique_walks_workspace_size(big64[i]);
  }
  for (size_t j = 0; j < n32; ++j) sink += rdf2v_nonsink_starts_workspace_size(big32[j]);
  EXPECT(rdf2v_build_csr_workspace_size(INT64_MAX, INT32_MAX) == 0);

  void *F = fake((uintptr_t)1 << 40);
  int32_t *FI = (int32_t *)F;
  rdf2v_csr csr = {10, 3, 20, FI, FI, NULL};
  rdf2v_csr bad = {-1, 3, 20, FI, FI, NULL};

  /* CSR build */
  EXPECT(rdf2v_build_csr(FI, FI, FI, -1, 10, 3, FI, FI, F, 1 << 20, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_build_csr(FI, FI, FI, (int64_t)1 << 31, 10, 3, FI, FI, F, 1 << 20, NULL, NULL) == RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_build_csr(FI, FI, FI, 100, INT32_MAX, INT32_MAX, FI, FI, F, 1 << 20, NULL, NULL) == RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_build_csr(FI, FI, FI, 100, 10, 3, FI, FI, NULL, 0, NULL, NULL) == RDF2V_ERR_WORKSPACE);
  EXPECT(rdf2v_build_walk_edges(&bad, FI, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_nonsink_starts(&bad, FI, (int64_t *)F, F, 1 << 20, NULL) == RDF2V_ERR_INVALID_ARGUMENT);

  /* walks */
  EXPECT(rdf2v_random_walks(&csr, FI, INT64_MAX, INT32_MAX, 4, 42, 0, 1, FI, FI, NULL, NULL) == RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_random_walks(&csr, FI, 5, 2, 65, 42, 0, 1, FI, FI, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_random_walks(&csr, FI, 5, 2, 4, 42, INT64_MAX, INT64_MAX, FI, FI, NULL, NULL) ==
         RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_random_walks(&csr, FI, (int64_t)1 << 61, 4, 64, 42, 0, (int64_t)1 << 62, FI, FI, NULL, NULL) ==
         RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_random_walks_tokens(&csr, FI, 5, 2, 4, 42, 0, 10, 7, FI, FI, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);

  /* skip-gram pairs, duplicate-free walks, BFS walks */
  EXPECT(rdf2v_skipgram_pairs(FI, FI, INT64_MAX, 129, 5, FI, 1, (int64_t *)F, F, 1 << 20, NULL, NULL) ==
         RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_skipgram_pairs(FI, FI, 10, 0, 5, FI, 1, (int64_t *)F, F, 1 << 20, NULL, NULL) ==
         RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_skipgram_pairs_noalloc(FI, FI, INT64_MAX, 9, 5, FI, 1, (int64_t *)F, NULL, NULL) ==
         RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_skipgram_pairs_noalloc(FI, FI, RDF2V_NOALLOC_MAX_WALKS + 1, 9, 5, FI, 1, (int64_t *)F, NULL, NULL) ==
         RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_skipgram_pairs_noalloc(FI, FI, 10, 0, 5, FI, 1, (int64_t *)F, NULL, NULL) ==
         RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_cbow_examples(FI, FI, INT64_MAX, 129, 5, FI, FI, 1, (int64_t *)F, F, 1 << 20, NULL, NULL) ==
         RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_cbow_examples(FI, FI, 10, 9, 5, FI, FI, INT64_MAX, (int64_t *)F, F, 1 << 20, NULL, NULL) ==
         RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_cbow_examples(FI, FI, 10, 9, 0, FI, FI, 1, (int64_t *)F, F, 1 << 20, NULL, NULL) ==
         RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_unique_walks(FI, FI, INT64_MAX, 3, INT32_MAX, FI, FI, (int64_t *)F, F, 1 << 20, NULL, NULL) ==
         RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_unique_walks(FI, FI, 10, 0, 9, FI, FI, (int64_t *)F, F, 1 << 20, NULL, NULL) ==
         RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_bfs_walks(&csr, FI, INT64_MAX, 64, INT32_MAX, FI, FI, FI, F, 1 << 20, NULL, NULL) ==
         RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_bfs_walks(&csr, FI, 10, 2, 0, FI, FI, FI, F, 1 << 20, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_bfs_fill_unused(FI, INT64_MAX, INT32_MAX, 129, FI, FI, NULL) == RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_bfs_fill_unused(FI, INT64_MIN, 4, 9, FI, FI, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_bfs_fill_unused(FI, 10, INT32_MIN, 9, FI, FI, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_bfs_fill_unused(FI, 10, 4, INT32_MAX, FI, FI, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_bfs_fill_unused(FI, 10, 4, 9, NULL, FI, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_bfs_fill_unused(NULL, 0, 4, 9, NULL, NULL, NULL) == RDF2V_OK);

  /* vocabulary */
  const uint8_t *C = (const uint8_t *)F;
  const int64_t *O = (const int64_t *)F;
  int64_t *counts = (int64_t *)F;
  EXPECT(rdf2v_build_vocabulary(C, O, 10, C, O, 10, C, O, 10, INT64_MAX, 10, 10, FI, FI, FI, counts, F, 1 << 20,
                                NULL, NULL) == RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_build_vocabulary(C, O, -1, C, O, 10, C, O, 10, 5, 10, 10, FI, FI, FI, counts, F, 1 << 20, NULL,
                                NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_build_vocabulary(C, O, 10, C, O, 10, C, O, 10, 5, 10, 10, FI, FI, FI, counts, NULL, 0, NULL,
                                NULL) == RDF2V_ERR_WORKSPACE);

  sink += model_entries(big64, n64, big32, n32);

  for (int s = -1; s < 7; ++s) EXPECT(rdf2v_status_string(s) != NULL);
  printf("abi sanitize: ok (%zu)\n", sink % 7);
  return 0;
}
