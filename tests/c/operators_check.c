/*
 * operators_check.c -- a plain C (C11) consumer of the calls around the path in
 * include/zq.h: embedding and its gradient, gradient norm and clipping, INT4 product, on
 * device buffers it allocates with the HIP runtime, against plain loops.  Every sum's
 * terms are small multiples of a power of two, so any order gives the same bits.
 * Exit status 0 when everything matches, 1 otherwise.
 */
#include <hip/hip_runtime_api.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "zq.h"

static int failures = 0;

#define HIP_OK(call)                                                                           \
  do {                                                                                         \
    hipError_t e_ = (call);                                                                    \
    if (e_ != hipSuccess) {                                                                    \
      fprintf(stderr, "%s:%d %s: %s\n", __FILE__, __LINE__, #call, hipGetErrorString(e_));     \
      exit(2);                                                                                 \
    }                                                                                          \
  } while (0)

static void expect(int got, int want, const char* what) {
  if (got != want) {
    fprintf(stderr, "%s: status %d (%s), want %d\n", what, got, zq_status_string(got), want);
    ++failures;
  }
}

/* host memory of at least one byte */
static void* host(size_t bytes) {
  void* p = calloc(bytes ? bytes : 1, 1);
  if (!p) exit(2);
  return p;
}

/* device memory: a copy of h, or bytes that no result has */
static void* dev(const void* h, size_t bytes) {
  void* p = NULL;
  HIP_OK(hipMalloc(&p, bytes ? bytes : 1));
  HIP_OK(hipMemset(p, 0xA5, bytes ? bytes : 1));
  if (h) HIP_OK(hipMemcpy(p, h, bytes, hipMemcpyHostToDevice));
  return p;
}

static void compare(const void* d, const float* want, int64_t n, const char* what) {
  float* got = host(n * sizeof(float));
  HIP_OK(hipMemcpy(got, d, n * sizeof(float), hipMemcpyDeviceToHost));
  for (int64_t i = 0; i < n; ++i)
    if (got[i] != want[i]) {
      fprintf(stderr, "%s: element %lld of %lld is %g, want %g\n", what, (long long)i, (long long)n, got[i], want[i]);
      ++failures;
      break;
    }
  free(got);
}

static uint64_t rng = 0x9E3779B97F4A7C15ull;
static int pick(int lo, int hi) { /* lo .. hi */
  rng ^= rng >> 12;
  rng ^= rng << 25;
  rng ^= rng >> 27;
  return lo + (int)((rng * 0x2545F4914F6CDD1Dull >> 33) % (uint64_t)(hi - lo + 1));
}

static int64_t nscales(int64_t n, int32_t b) { return (n + b - 1) / b; }
static int code(const uint8_t* packed, int64_t i) {
  const int u = packed[i / 2] >> (4 * (i % 2)) & 15;
  return u < 8 ? u : u - 16;
}
static float power(int e) { return ldexpf(1.0f, e); }

/* the lookup from a dense and an INT8 table, and the gradient: few tokens (one launch)
 * and many (with a workspace), written and added to what is there */
static void embeddings(hipStream_t st, int64_t T) {
  enum { V = 77, D = 45, B = 32 };
  int32_t* ids = host(T * 4);
  float *table = host(V * D * 4), *dy = host(T * D * 4), *want = host((T > V ? T : V) * D * 4), *scales = host(V * D * 4);
  int8_t* codes = host(V * D);
  for (int64_t t = 0; t < T; ++t) ids[t] = t % 7 == 3 ? -1 : t % 11 == 5 ? V : pick(0, V - 1);
  for (int i = 0; i < V * D; ++i) table[i] = (float)pick(-64, 64) / 8, codes[i] = (int8_t)pick(-127, 127);
  for (int i = 0; i < nscales(V * D, B); ++i) scales[i] = power(-pick(0, 6));
  for (int64_t i = 0; i < T * D; ++i) dy[i] = (float)pick(-16, 16) / 4;
  void *d_ids = dev(ids, T * 4), *d_table = dev(table, V * D * 4), *d_codes = dev(codes, V * D);
  void *d_scales = dev(scales, nscales(V * D, B) * 4), *d_dy = dev(dy, T * D * 4), *d_y = dev(NULL, T * D * 4);

  for (int64_t t = 0; t < T; ++t)
    for (int d = 0; d < D; ++d) want[t * D + d] = ids[t] < 0 || ids[t] >= V ? 0 : 0.5f * table[ids[t] * D + d];
  expect(zq_embedding(d_ids, ZQ_I32, T, d_table, ZQ_F32, V, D, 0.5f, d_y, ZQ_F32, st), ZQ_OK, "zq_embedding");
  HIP_OK(hipStreamSynchronize(st));
  compare(d_y, want, T * D, "zq_embedding");
  for (int64_t t = 0; t < T; ++t)
    for (int d = 0; d < D; ++d) {
      const int64_t f = (int64_t)ids[t] * D + d;
      want[t * D + d] = ids[t] < 0 || ids[t] >= V ? 0 : 2.0f * ((float)codes[f] * scales[f / B]);
    }
  expect(qwz_embedding(d_ids, ZQ_I32, T, d_codes, d_scales, V, D, B, 2.0f, d_y, ZQ_F32, st), ZQ_OK, "qwz_embedding");
  HIP_OK(hipStreamSynchronize(st));
  compare(d_y, want, T * D, "qwz_embedding");
  expect(qwz_embedding(d_ids, ZQ_I32, T, d_codes, d_scales, V, D, 48, 2.0f, d_y, ZQ_F32, st), ZQ_E_BLOCK, "block 48");

  const int64_t need = zq_embedding_grad_bytes(T, V, D);
  void *d_dw = dev(NULL, V * D * 4), *ws = need > 0 ? dev(NULL, need) : NULL;
  memset(want, 0, V * D * 4);
  for (int64_t t = 0; t < T; ++t)
    for (int d = 0; d < D; ++d)
      if (ids[t] >= 0 && ids[t] < V) want[ids[t] * D + d] += 0.25f * dy[t * D + d];
  expect(zq_embedding_grad(d_ids, ZQ_I32, T, d_dy, ZQ_F32, V, D, 0.25f, 0, d_dw, ZQ_F32, ws, need, st), ZQ_OK,
         "zq_embedding_grad");
  HIP_OK(hipStreamSynchronize(st));
  compare(d_dw, want, V * D, "zq_embedding_grad");
  for (int i = 0; i < V * D; ++i) want[i] *= 2;
  expect(zq_embedding_grad(d_ids, ZQ_I32, T, d_dy, ZQ_F32, V, D, 0.25f, 1, d_dw, ZQ_F32, ws, need, st), ZQ_OK,
         "zq_embedding_grad, added");
  HIP_OK(hipStreamSynchronize(st));
  compare(d_dw, want, V * D, "zq_embedding_grad, added");
  if (need > 0)
    expect(zq_embedding_grad(d_ids, ZQ_I32, T, d_dy, ZQ_F32, V, D, 1.0f, 0, d_dw, ZQ_F32, ws, need - 1, st), ZQ_E_SIZE,
           "a workspace that is too small");
  HIP_OK(hipFree(d_ids)); HIP_OK(hipFree(d_table)); HIP_OK(hipFree(d_codes)); HIP_OK(hipFree(d_scales));
  HIP_OK(hipFree(d_dy)); HIP_OK(hipFree(d_y)); HIP_OK(hipFree(d_dw));
  if (ws) HIP_OK(hipFree(ws));
  free(ids); free(table); free(dy); free(want); free(scales); free(codes);
}

/* a dense tensor in place, an INT4 shard into an output and one in place by its scales */
static void norm_and_clip(hipStream_t st) {
  enum { N0 = 50001, N1 = 70003, N2 = 1000, B = 64 };
  float *g = host(N0 * 4), *s1 = host(N1 * 4), *s2 = host(N2 * 4), *want = host(N1 * 4), norm = 0;
  uint8_t *p1 = host(N1), *p2 = host(N2);
  double sum = 0;
  for (int i = 0; i < N0; ++i) g[i] = (float)pick(-8, 8) / 16, sum += (double)g[i] * g[i];
  for (int i = 0; i < N1; ++i) p1[i] = (uint8_t)pick(0, 255);
  for (int i = 0; i < N2; ++i) p2[i] = (uint8_t)pick(0, 255);
  for (int i = 0; i < nscales(N1, B); ++i) s1[i] = power(-pick(2, 6));
  for (int i = 0; i < nscales(N2, B); ++i) s2[i] = power(-pick(2, 6));
  for (int i = 0; i < N1; ++i) sum += (double)(code(p1, i) * s1[i / B]) * (code(p1, i) * s1[i / B]);
  for (int i = 0; i < N2; ++i) sum += (double)(code(p2, i) * s2[i / B]) * (code(p2, i) * s2[i / B]);
  void *d_g = dev(g, N0 * 4), *d_p1 = dev(p1, (N1 + 1) / 2), *d_p2 = dev(p2, (N2 + 1) / 2);
  void *d_s1 = dev(s1, nscales(N1, B) * 4), *d_s2 = dev(s2, nscales(N2, B) * 4), *d_out = dev(NULL, N1 * 4);
  float* d_norm = dev(NULL, 4);
  const zq_grad grads[3] = {{d_g, NULL, NULL, N0, ZQ_F32, 0, 0, 0},
                            {d_p1, d_s1, d_out, N1, ZQ_INT4, ZQ_F32, B, 0},
                            {d_p2, d_s2, NULL, N2, ZQ_INT4, 0, B, 0}};
  zq_grad_plan plan;
  expect(zq_grad_plan_make(grads, 3, &plan), ZQ_OK, "zq_grad_plan_make");
  void* table = host(plan.bytes);
  expect(zq_grad_plan_table(grads, &plan, table), ZQ_OK, "zq_grad_plan_table");
  void* d_table = dev(table, plan.bytes);
  expect(zq_grad_norm(&plan, d_table, -0.5f, d_norm, st), ZQ_OK, "zq_grad_norm");
  HIP_OK(hipStreamSynchronize(st));
  HIP_OK(hipMemcpy(&norm, d_norm, 4, hipMemcpyDeviceToHost));
  const float exact = (float)(0.5 * sqrt(sum));
  if (norm != exact) {
    fprintf(stderr, "zq_grad_norm: %.9g, want %.9g\n", norm, exact);
    ++failures;
  }
  /* clipped by scale * max / (norm + 1e-6), in binary32 */
  const float ratio = 1.0f / (norm + 1e-6f), c = 0.5f * (ratio > 1.0f ? 1.0f : ratio);
  expect(zq_grad_clip(&plan, d_table, d_norm, 1.0f, 0.5f, st), ZQ_OK, "zq_grad_clip");
  expect(zq_grad_clip(&plan, d_table, d_norm, -1.0f, 0.5f, st), ZQ_E_SIZE, "a negative largest norm");
  HIP_OK(hipStreamSynchronize(st));
  for (int i = 0; i < N0; ++i) want[i] = g[i] * c;
  compare(d_g, want, N0, "a dense tensor clipped in place");
  for (int i = 0; i < N1; ++i) {
    const float s = s1[i / B] * c;
    want[i] = (float)code(p1, i) * s;
  }
  compare(d_out, want, N1, "an INT4 shard clipped into its output");
  for (int i = 0; i < nscales(N2, B); ++i) want[i] = s2[i] * c;
  compare(d_s2, want, nscales(N2, B), "an INT4 shard's scales clipped");
  HIP_OK(hipFree(d_g)); HIP_OK(hipFree(d_p1)); HIP_OK(hipFree(d_p2)); HIP_OK(hipFree(d_s1)); HIP_OK(hipFree(d_s2));
  HIP_OK(hipFree(d_out)); HIP_OK(hipFree(d_norm)); HIP_OK(hipFree(d_table));
  free(g); free(s1); free(s2); free(want); free(p1); free(p2); free(table);
}

/* M rows of bf16 x with an N x K weight; K long enough for slices at few weight rows */
static void product(hipStream_t st, int64_t M, int64_t N, int64_t K, int32_t B) {
  uint16_t* x = host(M * K * 2);
  float *xf = host(M * K * 4), *scales = host(nscales(N * K, B) * 4), *want = host(M * N * 4);
  uint8_t* packed = host(N * K / 2);
  for (int64_t i = 0; i < M * K; ++i) {
    uint32_t bits;
    xf[i] = pick(0, 7) ? 0.0f : (float)pick(-8, 8) / 4;
    memcpy(&bits, &xf[i], 4);
    x[i] = (uint16_t)(bits >> 16);
  }
  for (int64_t i = 0; i < N * K / 2; ++i) packed[i] = (uint8_t)pick(0, 255);
  for (int64_t i = 0; i < nscales(N * K, B); ++i) scales[i] = power(-pick(0, 4));
  for (int64_t m = 0; m < M; ++m)
    for (int64_t n = 0; n < N; ++n) {
      double v = 0;
      for (int64_t k = 0; k < K; ++k) v += (double)xf[m * K + k] * code(packed, n * K + k) * scales[(n * K + k) / B];
      want[m * N + n] = (float)v;
    }
  const int64_t need = zq_int4_dequant_gemm_bytes(M, N, K);
  void *d_x = dev(x, M * K * 2), *d_p = dev(packed, N * K / 2), *d_s = dev(scales, nscales(N * K, B) * 4);
  void *d_y = dev(NULL, M * N * 4), *ws = need > 0 ? dev(NULL, need) : NULL;
  expect(zq_int4_dequant_gemm(d_x, ZQ_BF16, d_p, d_s, M, N, K, B, d_y, ws, need, st), ZQ_OK, "zq_int4_dequant_gemm");
  HIP_OK(hipStreamSynchronize(st));
  compare(d_y, want, M * N, "zq_int4_dequant_gemm");
  expect(zq_int4_dequant_gemm(d_x, ZQ_F32, d_p, d_s, M, N, K, B, d_y, ws, need, st), ZQ_E_DTYPE, "x in binary32");
  HIP_OK(hipFree(d_x)); HIP_OK(hipFree(d_p)); HIP_OK(hipFree(d_s)); HIP_OK(hipFree(d_y));
  if (ws) HIP_OK(hipFree(ws));
  free(x); free(xf); free(scales); free(want); free(packed);
}

int main(void) {
  hipStream_t st;
  HIP_OK(hipStreamCreate(&st));
  embeddings(st, 300);
  embeddings(st, 5000);
  norm_and_clip(st);
  product(st, 1, 100, 320, 64);
  product(st, 20, 77, 640, 128);
  product(st, 3, 33, 24576, 128);
  product(st, 8, 33, 24576, 32);
  HIP_OK(hipStreamDestroy(st));
  if (failures) return 1;
  printf("operators_check ok\n");
  return 0;
}
