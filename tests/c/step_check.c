/*
 * step_check.c -- a plain C (C11) consumer of the optimizer's step, the RMS norm and the
 * policy loss in include/zq.h, on device buffers it allocates with the HIP runtime, against
 * plain loops: the optimizer bit for bit, the others to a few binary32 roundings.
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
/* within `tol` of the larger of a value and `least`; 0: the same bits */
static void compare(const void* d, const float* want, int64_t n, double tol, double least, const char* what) {
  float* got = host(n * sizeof(float));
  HIP_OK(hipMemcpy(got, d, n * sizeof(float), hipMemcpyDeviceToHost));
  for (int64_t i = 0; i < n; ++i) {
    const double off = fabs((double)got[i] - want[i]), size = fabs((double)want[i]);
    if (tol == 0 ? memcmp(got + i, want + i, 4) != 0 : !(off <= tol * (size > least ? size : least))) {
      fprintf(stderr, "%s: element %lld of %lld is %.9g, want %.9g\n", what, (long long)i, (long long)n, got[i], want[i]);
      ++failures;
      break;
    }
  }
  free(got);
}
static uint64_t rng = 0x9E3779B97F4A7C15ull;
static float uniform(void) { /* -1 .. 1 */
  rng ^= rng >> 12;
  rng ^= rng << 25;
  rng ^= rng >> 27;
  return (float)(int32_t)(rng * 0x2545F4914F6CDD1Dull >> 32) / 2147483648.0f;
}

/* two tensors, one with an INT8 copy; the count on the host and on the device */
static void optimizer(hipStream_t st) {
  enum { N0 = 5003, N1 = 77, B = 64, S0 = (N0 + B - 1) / B };
  const int64_t sizes[2] = {N0, N1};
  float *p[2], *g[2], *m[2], *v[2];
  zq_adamw t[2];
  memset(t, 0, sizeof t);
  for (int k = 0; k < 2; ++k) {
    const int64_t n = sizes[k];
    p[k] = host(n * 4), g[k] = host(n * 4), m[k] = host(n * 4), v[k] = host(n * 4);
    for (int64_t i = 0; i < n; ++i) {
      p[k][i] = uniform(), g[k][i] = 1e-2f * uniform(), m[k][i] = 1e-3f * uniform(), v[k][i] = 1e-5f * fabsf(uniform());
    }
    t[k].param = dev(p[k], n * 4), t[k].grad = dev(g[k], n * 4), t[k].m = dev(m[k], n * 4), t[k].v = dev(v[k], n * 4);
    t[k].n = n, t[k].weight_decay = 0.1 * k, t[k].lr_scale = 1.0;
    t[k].param_dtype = t[k].grad_dtype = t[k].state_dtype = ZQ_F32;
  }
  t[0].out = dev(NULL, N0), t[0].out_scales = dev(NULL, S0 * 4), t[0].out_dtype = ZQ_INT8, t[0].out_block = B;
  zq_adamw_plan plan;
  expect(zq_adamw_plan_make(t, 2, &plan), ZQ_OK, "zq_adamw_plan_make");
  void* h_table = host(plan.bytes);
  expect(zq_adamw_plan_table(t, &plan, h_table), ZQ_OK, "zq_adamw_plan_table");
  void* table = dev(h_table, plan.bytes);
  const float norm = 3.0f;
  const int64_t three = 3;
  void *d_norm = dev(&norm, 4), *d_step = dev(&three, 8);
  zq_adamw_args a = {1e-3, 0.9, 0.99, 1e-8, 2, 1.5f, 0.5f};
  for (int step = 2; step <= 3; ++step) {
    expect(zq_adamw_step(&plan, table, &a, step == 2 ? NULL : d_step, NULL, d_norm, st), ZQ_OK, "zq_adamw_step");
    HIP_OK(hipStreamSynchronize(st));
    const float ratio = 1.5f / (norm + 1e-6f), c = 0.5f * (ratio > 1.0f ? 1.0f : ratio);
    const float root = (float)(1.0 / sqrt(1.0 - pow(0.99, step))), alpha = (float)(1e-3 / (1.0 - pow(0.9, step)));
    for (int k = 0; k < 2; ++k) {
      const float decay = (float)(1.0 - 1e-3 * (0.1 * k));
      for (int64_t i = 0; i < sizes[k]; ++i) {
        const float x = g[k][i] * c;
        m[k][i] = m[k][i] * 0.9f + x * (float)(1.0 - 0.9);
        v[k][i] = v[k][i] * 0.99f + (x * x) * (float)(1.0 - 0.99);
        const float d = sqrtf(v[k][i]) * root + 1e-8f;
        p[k][i] = p[k][i] * decay - (m[k][i] / d) * alpha;
      }
      compare(t[k].param, p[k], sizes[k], 0, 0, "weights");
      compare(t[k].m, m[k], sizes[k], 0, 0, "m");
      compare(t[k].v, v[k], sizes[k], 0, 0, "v");
    }
    float* s = host(S0 * 4);
    int8_t* q = host(N0);
    HIP_OK(hipMemcpy(q, t[0].out, N0, hipMemcpyDeviceToHost));
    for (int b = 0; b < S0; ++b) {
      float most = 0;
      for (int i = b * B; i < N0 && i < (b + 1) * B; ++i) most = fmaxf(most, fabsf(p[0][i]));
      s[b] = most / 127.0f;
      for (int i = b * B; i < N0 && i < (b + 1) * B; ++i)
        if (q[i] != (int8_t)rintf(p[0][i] * (127.0f / most))) {
          fprintf(stderr, "INT8 copy: code %d is %d\n", i, q[i]);
          ++failures;
          b = S0;
          break;
        }
    }
    compare(t[0].out_scales, s, failures ? 0 : S0, 0, 0, "INT8 copy's scales");
    free(s), free(q);
  }
  a.step = 0;
  expect(zq_adamw_step(&plan, table, &a, NULL, NULL, d_norm, st), ZQ_E_SIZE, "step 0");
  t[1].param = t[0].param;
  expect(zq_adamw_plan_make(t, 2, &plan), ZQ_E_ALIAS, "a parameter twice");
}

static void norm(hipStream_t st, int64_t T, int64_t D) {
  const int64_t n = T * D;
  float *x = host(n * 4), *r = host(n * 4), *w = host(D * 4), *h = host(n * 4), *y = host(n * 4), *s = host(T * 4);
  float *dy = host(n * 4), *dx = host(n * 4), *dw = host(D * 4);
  for (int64_t i = 0; i < n; ++i) x[i] = uniform(), r[i] = 2 * uniform(), dy[i] = uniform();
  for (int64_t d = 0; d < D; ++d) w[d] = 1 + 0.5f * uniform();
  double* sums = host(D * 8);
  for (int64_t t = 0; t < T; ++t) {
    double q = 0, c = 0;
    for (int64_t d = 0; d < D; ++d) h[t * D + d] = x[t * D + d] + r[t * D + d], q += (double)h[t * D + d] * h[t * D + d];
    const double rstd = 1 / sqrt(q / D + 1e-5);
    s[t] = (float)rstd;
    for (int64_t d = 0; d < D; ++d) {
      const double xh = h[t * D + d] * rstd;
      y[t * D + d] = (float)(xh * w[d]);
      c += (double)dy[t * D + d] * w[d] * xh;
      sums[d] += dy[t * D + d] * xh;
    }
    for (int64_t d = 0; d < D; ++d)
      dx[t * D + d] = (float)(rstd * ((double)dy[t * D + d] * w[d] - h[t * D + d] * rstd * c / D) + r[t * D + d]);
  }
  for (int64_t d = 0; d < D; ++d) dw[d] = (float)sums[d];
  void *d_x = dev(x, n * 4), *d_r = dev(r, n * 4), *d_w = dev(w, D * 4), *d_h = dev(NULL, n * 4), *d_y = dev(NULL, n * 4);
  void *d_s = dev(NULL, T * 4), *d_dy = dev(dy, n * 4), *d_dx = dev(NULL, n * 4), *d_dw = dev(NULL, D * 4);
  const int64_t need = zq_rms_norm_grad_bytes(T, D);
  void* ws = dev(NULL, need);
  expect(zq_rms_norm(d_x, d_r, ZQ_F32, d_w, ZQ_F32, T, D, 1e-5, d_h, d_y, ZQ_F32, d_s, st), ZQ_OK, "zq_rms_norm");
  expect(zq_rms_norm_grad(d_dy, ZQ_F32, d_h, ZQ_F32, d_w, ZQ_F32, d_s, d_r, T, D, d_dx, 0, d_dw, ZQ_F32, ws, need, st), ZQ_OK,
         "zq_rms_norm_grad");
  expect(zq_rms_norm_grad(d_dy, ZQ_F32, d_h, ZQ_F32, d_w, ZQ_F32, d_s, d_r, T, D, d_dx, 0, d_dw, ZQ_F32, ws, need - 4, st),
         ZQ_E_SIZE, "a workspace that is too small");
  HIP_OK(hipStreamSynchronize(st));
  compare(d_h, h, n, 0, 0, "x + residual");
  compare(d_s, s, T, 1.2e-7, 0, "rstd");
  compare(d_y, y, n, 3e-7, 0, "y");
  compare(d_dx, dx, n, 1e-5, 1, "dx");
  compare(d_dw, dw, D, 1e-5, (double)T, "dw");
  if (D % 32 == 0) { /* the same as codes: half a step off at most */
    void *q = dev(NULL, n), *sc = dev(NULL, n / 32 * 4);
    expect(qwz_rms_norm(d_x, d_r, ZQ_F32, d_w, ZQ_F32, T, D, 1e-5, d_h, q, sc, 32, d_s, st), ZQ_OK, "qwz_rms_norm");
    expect(qwz_dequantize(q, sc, n, 32, d_y, ZQ_F32, st), ZQ_OK, "qwz_dequantize");
    HIP_OK(hipStreamSynchronize(st));
    float most = 0;
    for (int64_t i = 0; i < n; ++i) most = fmaxf(most, fabsf(y[i]));
    compare(d_y, y, n, 0.501 / 127, most, "INT8 y");
  }
}

static void loss(hipStream_t st, int64_t T, int64_t V, int64_t ld) {
  float *z = host(T * ld * 4), *old = host(T * 4), *adv = host(T * 4), *lp = host(T * 4), *grad = host(T * ld * 4), sums[4];
  int32_t* ids = host(T * 4);
  double total[4] = {0, 0, 0, 0};
  for (int64_t i = 0; i < T * ld; ++i) z[i] = 3 * uniform(), grad[i] = -1;
  for (int64_t t = 0; t < T; ++t) {
    ids[t] = (int32_t)((t * 7919) % (V + 1)); /* V: no token */
    adv[t] = uniform();
    double m = -INFINITY, s = 0;
    for (int64_t v = 0; v < V; ++v) m = fmax(m, z[t * ld + v]);
    for (int64_t v = 0; v < V; ++v) s += exp(z[t * ld + v] - m);
    const double logp = ids[t] < V ? z[t * ld + ids[t]] - m - log(s) : 0;
    old[t] = (float)(logp + 0.3 * uniform());
    lp[t] = (float)logp;
    const double r = exp(logp - old[t]), A = adv[t], lo = 1 - (double)0.2f, hi = 1 + (double)0.2f;
    const int clipped = (A > 0 && r > hi) || (A < 0 && r < lo);
    const double slope = clipped || ids[t] == V ? 0 : -r * A;
    if (ids[t] < V) total[1] += -(clipped ? (A > 0 ? hi : lo) * A : r * A), total[3] += clipped;
    for (int64_t v = 0; v < V; ++v) grad[t * ld + v] = (float)(slope * ((v == ids[t]) - exp(z[t * ld + v] - m) / s));
  }
  total[0] = total[1];
  for (int k = 0; k < 4; ++k) sums[k] = (float)total[k];
  void *d_z = dev(z, T * ld * 4), *d_ids = dev(ids, T * 4), *d_old = dev(old, T * 4), *d_adv = dev(adv, T * 4);
  float* minus = host(T * ld * 4);
  for (int64_t i = 0; i < T * ld; ++i) minus[i] = -1;
  void *d_g = dev(minus, T * ld * 4), *d_lp = dev(NULL, T * 4), *d_lp2 = dev(NULL, T * 4), *d_s = dev(NULL, 16);
  const int64_t need = zq_policy_loss_bytes(T);
  void* ws = dev(NULL, need);
  zq_policy p;
  memset(&p, 0, sizeof p);
  p.old_logp = d_old, p.advantages = d_adv, p.clip_low = p.clip_high = 0.2f, p.scale = p.grad_scale = 1.0f;
  expect(zq_policy_loss(d_z, ZQ_F32, T, V, ld, d_ids, ZQ_I32, &p, d_s, d_lp, d_g, ZQ_F32, ld, ws, need, st), ZQ_OK, "zq_policy_loss");
  expect(zq_token_logp(d_z, ZQ_F32, T, V, ld, d_ids, ZQ_I32, 1.0f, d_lp2, st), ZQ_OK, "zq_token_logp");
  HIP_OK(hipStreamSynchronize(st));
  compare(d_lp, lp, T, 1e-6, 1, "logp");
  compare(d_lp2, lp, T, 1e-6, 1, "logp alone");
  compare(d_s, sums, 4, 1e-5, 1, "sums");
  compare(d_g, grad, T * ld, 2e-6, 1, "gradient, and what lies between its rows");
  p.kl = 0.1f;
  expect(zq_policy_loss(d_z, ZQ_F32, T, V, ld, d_ids, ZQ_I32, &p, d_s, d_lp, d_g, ZQ_F32, ld, ws, need, st), ZQ_E_NULL,
         "a KL term without a reference");
}

int main(void) {
  hipStream_t st;
  HIP_OK(hipStreamCreate(&st));
  optimizer(st);
  norm(st, 3, 100);
  norm(st, 300, 2048);
  norm(st, 5, 17001);
  loss(st, 50, 333, 340);
  loss(st, 7, 20011, 20011);
  HIP_OK(hipStreamDestroy(st));
  if (failures) return 1;
  printf("step_check ok\n");
  return 0;
}
