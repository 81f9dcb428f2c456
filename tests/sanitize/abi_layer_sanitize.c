/*
 * Host-side paths of the layer operators' entry points, for objects built with
 * AddressSanitizer and UndefinedBehaviorSanitizer on their host code: the
 * workspace-size functions at extreme sizes, and calls with arguments that the
 * host rejects before any HIP call (the fake device pointers are never
 * dereferenced).
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

#define COUNT(a) (sizeof(a) / sizeof((a)[0]))

static void *fake(int i) { return (void *)(((uintptr_t)1 << 44) + ((uintptr_t)i << 36)); }
static float *fakef(int i) { return (float *)fake(i); }

int main(void) {
  const int64_t big64[] = {0, 1, 7, 8, 9, 16, 17, 4095, ((int64_t)1 << 31) - 1, (int64_t)1 << 31, (int64_t)1 << 53,
                           INT64_MAX, INT64_MIN, -1};
  const int32_t big32[] = {0, 1, 3, 8, 16, 63, 64, 65, 16384, 1 << 24, 1 << 28, INT32_MAX, INT32_MIN, -1};
  size_t sink = 0;
  for (size_t i = 0; i < COUNT(big64); ++i)
    for (size_t j = 0; j < COUNT(big64); ++j)
      for (size_t k = 0; k < COUNT(big32); ++k)
        for (size_t l = 0; l < COUNT(big32); ++l)
          for (int type = -1; type < 3; ++type) {
            const rdf2v_conv conv = {big64[i], big64[j], big32[k], big32[l], type, 1, NULL, NULL, NULL};
            const rdf2v_scan one = {big64[i], big64[j], big32[k], 1, big32[l], type, NULL, NULL, NULL, NULL};
            const rdf2v_scan many = {big64[i], big64[j], big32[k], big32[l], 64, type, NULL, NULL, NULL, NULL};
            rdf2v_norm norm = {0};
            norm.rows = big64[i];
            norm.length = big64[j];
            norm.channels = big32[k];
            norm.dtype = type;
            norm.residual_dtype = big32[l];
            norm.drop = 0.5;
            sink += rdf2v_causal_conv_backward_workspace_size(&conv);
            sink += rdf2v_selective_scan_workspace_size(&one) + rdf2v_selective_scan_backward_workspace_size(&one);
            sink += rdf2v_selective_scan_workspace_size(&many) + rdf2v_selective_scan_backward_workspace_size(&many);
            sink += rdf2v_residual_norm_backward_workspace_size(&norm);
          }
  EXPECT(rdf2v_causal_conv_backward_workspace_size(NULL) == 0);
  EXPECT(rdf2v_selective_scan_workspace_size(NULL) == 0);
  EXPECT(rdf2v_residual_norm_backward_workspace_size(NULL) == 0);

  /* views of extreme strides beside outputs, and extreme sizes */
  const rdf2v_tokens_view x = {fake(1), 640, 64}, y = {fake(2), -640, -64}, none = {NULL, 0, 0};
  const rdf2v_heads_view b = {fake(3), 640, 64, 16}, wide = {fake(4), INT64_MAX, INT64_MIN, 1};
  const int64_t most = ((int64_t)1 << 56) - 1;
  const rdf2v_tokens_view far = {fake(5), most, -most}, over = {fake(6), 10, 10};
  const rdf2v_conv conv = {4, 10, 48, 4, RDF2V_F32, 1, fakef(7), NULL, NULL};
  EXPECT(rdf2v_causal_conv(&conv, &none, NULL, fake(10), NULL, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_causal_conv(&conv, &x, NULL, fake(1), NULL, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_causal_conv(&conv, &y, NULL, fake(2), NULL, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_causal_conv(&conv, &over, NULL, fake(6), NULL, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_causal_conv(&conv, &far, NULL, fake(5), NULL, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_causal_conv_step(&conv, &x, fake(8), INT64_MAX, (const int32_t *)fake(9), fake(10), fake(11), NULL,
                                NULL) == RDF2V_ERR_TOO_LARGE);
  EXPECT(rdf2v_causal_conv_step(&conv, &x, fake(8), INT64_MIN, (const int32_t *)fake(9), fake(10), fake(11), NULL,
                                NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  const rdf2v_scan scan = {4, 10, 48, 2, 16, RDF2V_BF16, fakef(7), NULL, NULL, NULL};
  EXPECT(rdf2v_selective_scan(&scan, &x, &y, &b, &wide, NULL, NULL, fake(10), NULL, fake(20), 0, NULL, NULL) ==
         RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_selective_scan(&scan, &x, &far, &b, &b, &x, NULL, fake(1), NULL, fake(20), 0, NULL, NULL) ==
         RDF2V_ERR_INVALID_ARGUMENT);
  const rdf2v_scan_gradients nothing = {0};
  EXPECT(rdf2v_selective_scan_backward(&scan, &x, &x, &b, &b, NULL, &x, NULL, NULL, &nothing, NULL, 0, NULL, NULL) ==
         RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_selective_scan_backward(&scan, &x, &x, &b, &b, NULL, &x, NULL, NULL, NULL, NULL, 0, NULL, NULL) ==
         RDF2V_ERR_INVALID_ARGUMENT);
  EXPECT(rdf2v_selective_scan_step(&scan, &x, &x, &b, &b, NULL, fakef(8), INT64_MAX, (const int32_t *)fake(9), fake(10),
                                   fakef(11), NULL, NULL) == RDF2V_ERR_TOO_LARGE);
  rdf2v_norm norm = {4, 10, 48, RDF2V_F32, RDF2V_F32, 1, 1e-5f, fakef(7), NULL, NULL, 0.1, UINT64_MAX, NULL, 0, NULL};
  EXPECT(rdf2v_residual_norm(&norm, &x, &far, fake(5), NULL, NULL, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  norm.row_begin = INT64_MAX;
  EXPECT(rdf2v_residual_norm(&norm, &x, NULL, fake(10), NULL, NULL, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  norm.row_begin = INT64_MIN;
  EXPECT(rdf2v_residual_norm(&norm, &x, NULL, fake(10), NULL, NULL, NULL, NULL) == RDF2V_ERR_INVALID_ARGUMENT);
  printf("abi layer sanitize: ok (%zu)\n", sink % 7);
  return 0;
}
