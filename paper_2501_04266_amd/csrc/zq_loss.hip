// zq_loss.hip -- log-probabilities of given tokens, and the clipped policy loss with its
// gradient, from rows of logits, on gfx950.
//
//   logp = scale (z[a] - m) - log S      m = max z, S = sum exp(scale (z - m))
//   r = exp(logp - old)   loss = -min(r A, clip(r) A) + kl (exp(u) - u - 1)   u = ref - logp
//   grad[v] = w scale (dloss/dlogp) ((v == a) - exp(scale (z[v] - m)) / S)
//
// Bound by memory: a row of logits is read once, kept in the registers of one workgroup
// (64 to 1,024 threads, up to 16 vectors of 16 bytes each), and its gradient written once
// (8,192 rows of 50,000 of bf16, a tenth of them without a token: 282 us, 5.5 TB/s).  exp is
// v_exp_f32 of a binary32 difference; it is taken twice, for the sum and for the gradient,
// since a row's exponentials in binary32 would need twice the registers of
// 16-bit logits.  Sums of a vector's 4 or 8 exponentials are binary32 (but for a likely token's
// vector, whose others are what its logarithm is made of), sums over vectors and threads and what
// follows binary64: whether a token is clipped is decided at 1 +- clip, and its logarithm
// is what the binary32 terms allow.  Rows too long for the registers are read again.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>
#include <type_traits>

#include "zq.h"
#include "zq_device.h"
#include "zq_host.h"
#include "zq_lanes.h"
#include "zq_vec.h"

#pragma clang fp contract(off)

namespace zq {
namespace {

constexpr int64_t kMaxVocab = 1 << 24;
constexpr int64_t kMaxPlaces = (int64_t)1 << 59;  // T * ld: bytes of all rows within 63 bits
constexpr float kMaxScale = 0x1p127f;  // times log2 e a binary32 number
constexpr float kInf = __builtin_inff();

struct Loss {
  const void* logits;
  const void* ids;
  int64_t T, V, ld;
  float scale;
  int it;
  float* logp;
  // the loss's: rows is NULL for log-probabilities alone
  double* rows;  // [T][4]: the terms of the sums
  void* grad;
  int64_t ldg;
  int gt;
  const float* old_logp;
  const float* advantages;
  const float* weights;
  const float* ref_logp;
  float clip_low, clip_high, kl, grad_scale;
};

template <int DT>
constexpr int per_vec() { return 16 / dt_size<DT>(); }

// A 16-byte vector of logits from element i of n; -infinity behind the end.  A row's last,
// partial vector is read as the 16 bytes up to its end and moved down.
template <int DT>
__device__ __forceinline__ void load_vec(const char* row, int i, int n, uint32_t (&w)[4]) {
  constexpr int E = per_vec<DT>(), S = dt_size<DT>();
  constexpr uint32_t none = DT == ZQ_F32 ? 0xff800000u : DT == ZQ_BF16 ? 0xff80ff80u : 0xfc00fc00u;
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = none;
  if (n >= E) {
    const int at = min(i, n - E);
    if (i < n) load_words_any<false>(row + (uint32_t)at * S, w);
    if (i == at || i >= n) return;
    const int words = (i - at) * S / 4;
#pragma unroll
    for (int b = 2; b >= 1; b /= 2) {
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = words & b ? (k + b < 4 ? w[k + b] : none) : w[k];
    }
    if (S == 2 && (i - at) & 1) {
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = w[k] >> 16 | (k + 1 < 4 ? w[k + 1] : none) << 16;
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < E - 1; ++k) {
    if (i + k >= n) continue;
    if constexpr (DT == ZQ_F32) {
      w[k] = reinterpret_cast<const uint32_t*>(row)[i + k];
    } else {
      const uint32_t h = reinterpret_cast<const uint16_t*>(row)[i + k];
      w[k / 2] = k & 1 ? (w[k / 2] & 0xffffu) | h << 16 : (w[k / 2] & 0xffff0000u) | h;
    }
  }
}

// The words are what they were, but the compiler does not know: what it has derived from
// them (their widened values) is not kept in registers across this point.
__device__ __forceinline__ void forget(uint32_t (&w)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(w[k]));
}

template <int GT, int E>
__device__ __forceinline__ void store_vec(char* row, int i, int n, const float (&v)[E]) {
  if (i + E <= n) {
    store_elems<GT, E, true>(row + (uint32_t)i * dt_size<GT>(), 0, v);
    return;
  }
#pragma unroll
  for (int k = 0; k < E; ++k) {
    const float t[1] = {v[k]};
    if (i + k < n) store_elems<GT, 1>(row, i + k, t);
  }
}
// f<type>() for the type that dt names
template <typename F>
__device__ __forceinline__ void for_type(int dt, F f) {
  if (dt == ZQ_F32) f(std::integral_constant<int, ZQ_F32>());
  else if (dt == ZQ_BF16) f(std::integral_constant<int, ZQ_BF16>());
  else f(std::integral_constant<int, ZQ_F16>());
}

template <int R>
__device__ __forceinline__ float group_max(float v, float* slot) {
  v = over_lanes<64>(v, [](float a, float b) { return fmaxf(a, b); });
  if constexpr (R == 64) return v;
  if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
  __syncthreads();
  float m = slot[0];
#pragma unroll
  for (int w = 1; w < R / 64; ++w) m = fmaxf(m, slot[w]);
  return m;
}
template <int R>
__device__ __forceinline__ double group_sum(double v, double* slot) {
  v = lanes_sum<64>(v);
  if constexpr (R == 64) return v;
  if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = slot[0];
#pragma unroll
  for (int w = 1; w < R / 64; ++w) s += slot[w];
  return s;
}

// exp and log of a token's few binary64 numbers, by their series: they run while a row
// waits in the vector registers, and the library's functions take some 40 of those.  Relative
// errors below 2^-50 of the logarithm; of exp 2^-48 up to |x| = 100, 2^-45 up to 700, where log 2
// rounded once, times k, counts.  (As loops with the coefficients read in turn they held a row of 50,000
// up for 6% of its time; a token's own values loaded when wanted, for 2%.)
__device__ __forceinline__ double exp64(double x) {
  if (!(fabs(x) <= 700.0)) return x > 0.0 ? (double)kInf : x < 0.0 ? 0.0 : x;
  // x = k log 2 + r, |r| <= 0.35: the series to r^13 / 13!
  constexpr double c[14] = {1.0,         1.0,          1.0 / 2,       1.0 / 6,        1.0 / 24,        1.0 / 120,       1.0 / 720,
                            1.0 / 5040., 1.0 / 40320., 1.0 / 362880., 1.0 / 3628800., 1.0 / 39916800., 1.0 / 479001600.,
                            1.0 / 6227020800.};
  const double k = rint(x * 1.4426950408889634), r = __builtin_fma(k, -0x1.62e42fefa39efp-1, x);
  double p = c[13];
#pragma unroll
  for (int n = 12; n >= 0; --n) p = __builtin_fma(p, r, c[n]);
  return ldexp(p, (int)k);
}
// of s from 1 to 2^24 (or NaN)
__device__ __forceinline__ double log64(double s) {
  int k;
  double f = frexp(s, &k);
  if (f < 0.70710678118654752) f *= 2.0, --k;
  // log f = 2 (q + q^3 / 3 + ... + q^23 / 23), q = (f - 1) / (f + 1), |q| <= 0.172
  const double q = (f - 1.0) / (f + 1.0), q2 = q * q;
  double p = 1.0 / 23;
#pragma unroll
  for (int n = 21; n >= 1; n -= 2) p = __builtin_fma(p, q2, 1.0 / n);
  return __builtin_fma((double)k, 0x1.62e42fefa39efp-1, 2.0 * q * p);
}

// What a token brings beside its logits; loaded with them, not when it is wanted.
struct Token {
  float weight, advantage, old_logp, ref_logp;
};
__device__ __forceinline__ Token token_of(const Loss& a, int64_t t) {
  Token k = {1.0f, 0.0f, 0.0f, 0.0f};
  if (!a.rows) return k;
  if (a.weights) k.weight = a.weights[t];
  k.advantage = a.advantages[t];
  k.old_logp = a.old_logp[t];
  if (a.ref_logp) k.ref_logp = a.ref_logp[t];
  return k;
}

// The terms of a token, and the factor of its row of gradients.
__device__ __forceinline__ double token_terms(const Loss& a, const Token& k, double logp, double* rows) {
  const double w = k.weight;
  if (w == 0.0) {
    rows[0] = rows[1] = rows[2] = rows[3] = 0.0;
    return 0.0;
  }
  const bool never = logp == -(double)kInf;  // a token that cannot occur, whatever the other policies say of it
  const double A = k.advantage, r = never ? 0.0 : exp64(logp - (double)k.old_logp);
  const double lo = 1.0 - (double)a.clip_low, hi = 1.0 + (double)a.clip_high;
  const bool clipped = (A > 0.0 && r > hi) || (A < 0.0 && r < lo);
  const double pg = -(clipped ? (A > 0.0 ? hi : lo) * A : r * A);
  double slope = clipped ? 0.0 : -r * A, kl = 0.0;
  if (a.ref_logp) {
    const double u = never ? (double)kInf : (double)k.ref_logp - logp, e = exp64(u);
    kl = e == (double)kInf ? e : e - u - 1.0;  // not infinity less infinity
    if (a.kl != 0.0f) slope += (double)a.kl * (1.0 - e);
  }
  rows[0] = w * (a.kl != 0.0f ? pg + (double)a.kl * kl : pg);
  rows[1] = w * pg;
  rows[2] = w * kl;
  rows[3] = clipped ? w : 0.0;
  return (double)a.grad_scale * w * (double)a.scale * slope;
}

// R threads a row, NV vectors each; NV = 0: rows of any length, read again
template <int LT, int R, int NV>
__global__ void __launch_bounds__(R, NV > 8 ? 4 : NV == 8 && R < 1024 ? 7 : 8) k_loss(unsigned first, Loss a) {
  constexpr int E = per_vec<LT>();
  __shared__ float top[R / 64];
  __shared__ double total[R / 64];
  __shared__ double factor;
  const int64_t t = first + blockIdx.x;
  const int64_t id = a.it == ZQ_I64 ? static_cast<const int64_t*>(a.ids)[t] : static_cast<const int32_t*>(a.ids)[t];
  const char* row = static_cast<const char*>(a.logits) + t * a.ld * dt_size<LT>();
  char* grow = a.grad ? static_cast<char*>(a.grad) + t * a.ldg * (a.gt == ZQ_F32 ? 4 : 2) : nullptr;
  const float k2 = a.scale * 1.44269504088896340736f;  // exp(scale d) = 2^(k2 d)
  const int V = (int)a.V;  // up to 2^24: places in a row are 32-bit numbers
  constexpr int STEP = R * E;

  auto zeros = [&]() {
    for_type(a.gt, [&](auto gt) {
      const float zero[E] = {};
      for (int i = threadIdx.x * E; i < V; i += STEP) store_vec<gt>(grow, i, V, zero);
    });
  };
  auto none = [&]() {  // no token: no loss, a gradient of zeros
    if (threadIdx.x == 0) {
      if (a.logp) a.logp[t] = 0.0f;
      if (a.rows) a.rows[4 * t] = a.rows[4 * t + 1] = a.rows[4 * t + 2] = a.rows[4 * t + 3] = 0.0;
    }
    if (grow) zeros();
  };
  if (id < 0 || id >= V) {
    none();
    return;
  }

  uint32_t z[NV > 0 ? NV : 1][4];
  float m = -kInf;
  auto max_of = [&](const uint32_t(&w)[4]) {
    float v[E];
    widen<LT>(w, v);
#pragma unroll
    for (int k = 0; k < E; ++k) m = fmaxf(m, v[k]);
  };
  const int beside = (int)id & -E;  // the vector that the token's logit is in
  float own[1] = {-kInf};           // one of its elements
  const Token token = token_of(a, t);  // not beside the id, which the row's loads wait for
  auto load_own = [&]() {
    const int i = beside + (int)(threadIdx.x & (E - 1));
    if (i < V) load_elems<LT, 1>(row + (uint32_t)i * dt_size<LT>(), 0, own);
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) load_vec<LT>(row, (j * R + (int)threadIdx.x) * E, V, z[j]);
    load_own();
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      max_of(z[j]);
      forget(z[j]);
    }
  } else {
    load_own();
    for (int i = threadIdx.x * E; i < V; i += STEP) {
      load_vec<LT>(row, i, V, z[0]);
      max_of(z[0]);
    }
  }
  m = group_max<R>(m, top);
  if (m == -kInf) {  // no logit above -infinity, or none but NaNs
    int nan = 0;
    for (int i = threadIdx.x; i < V; i += R) {
      float v[1];
      load_elems<LT, 1>(row, i, v);
      nan |= v[0] != v[0];
    }
    if (!__syncthreads_or(nan)) {
      none();
      return;
    }
  }

  double sum = 0.0;
  auto add = [&](const uint32_t(&w)[4]) {
    float v[E];
    widen<LT>(w, v);
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = __builtin_amdgcn_exp2f((v[k] - m) * k2);
#pragma unroll
    for (int o = 1; o < E; o *= 2) {  // in the order of lanes_sum
#pragma unroll
      for (int k = 0; k < E; k += 2 * o) v[k] += v[k + o];
    }
    sum += (double)v[0];
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      add(z[j]);
      forget(z[j]);
    }
  } else {
    for (int i = threadIdx.x * E; i < V; i += STEP) {
      load_vec<LT>(row, i, V, z[0]);
      add(z[0]);
    }
  }
  sum = group_sum<R>(sum, total);

  // one wave's work, the others wait for it if they have a gradient to write
  if (threadIdx.x < 64) {
    const float za = u2f((uint32_t)__builtin_amdgcn_readlane((int)f2u(own[0]), (int)id - beside));
    double S = sum;
    if (za == m && sum < 2.0) {  // a likely token: its exponential is 1, and those of its vector were lost beside it
      const float e = __builtin_amdgcn_exp2f((own[0] - m) * k2);
      S += lanes_sum<E>((double)e) - (double)lanes_sum<E>(e);  // the vector's sum again, for what it was
    }
    const double logp = (double)a.scale * ((double)za - (double)m) - log64(S);
    double rows[4];
    const double g = a.rows ? token_terms(a, token, logp, rows) : 0.0;
    if (threadIdx.x == 0) {
      if (a.logp) a.logp[t] = (float)logp;
      if (a.rows) {
#pragma unroll
        for (int k = 0; k < 4; ++k) a.rows[4 * t + k] = rows[k];
      }
      factor = g;
    }
  }
  if (!grow) return;
  __syncthreads();
  const float g = (float)factor, c = (float)(-factor / sum);
  if (g == 0.0f) {  // masked, or clipped without a KL term
    zeros();
    return;
  }
  int thread = threadIdx.x;
  asm volatile("" : "+v"(thread));  // places computed anew: those of the loads are not kept
  if (fabsf(g) == kInf) {  // an infinite KL term, mostly: 0 where there is no probability, not 0 times infinity
    const double f = factor;
    for_type(a.gt, [&](auto gt) {
      for (int i = thread; i < V; i += R) {
        float v[1];
        load_elems<LT, 1>(row, i, v);
        const double p = (double)__builtin_amdgcn_exp2f((v[0] - m) * k2) / sum;
        const float t[1] = {v[0] == -kInf ? 0.0f : (float)(i == (int)id ? f * (1.0 - p) : p == 0.0 ? 0.0 : -f * p)};
        store_elems<gt, 1>(grow, i, t);
      }
    });
    return;
  }
  for_type(a.gt, [&](auto gt) {
    auto put = [&](const uint32_t(&w)[4], int i) {
      float v[E];
      widen<LT>(w, v);
#pragma unroll
      for (int k = 0; k < E; ++k) v[k] = __builtin_amdgcn_exp2f((v[k] - m) * k2) * c;
      const uint32_t at = (uint32_t)((int)id - i);
      if (at < (uint32_t)E) {
#pragma unroll
        for (int k = 0; k < E; ++k) v[k] = at == (uint32_t)k ? v[k] + g : v[k];
      }
      store_vec<gt>(grow, i, V, v);
    };
    if constexpr (NV > 0) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int i = (j * R + thread) * E;
        if (i < V) put(z[j], i);
      }
    } else {
      for (int i = threadIdx.x * E; i < V; i += STEP) {
        load_vec<LT>(row, i, V, z[0]);
        put(z[0], i);
      }
    }
  });
}

// A sum over the rows a workgroup: each thread its rows in their order, 8 loads in flight,
// then the threads in theirs.
__global__ void __launch_bounds__(1024) k_loss_sums(const double* __restrict__ rows, int64_t T, float* __restrict__ sums) {
  __shared__ double part[16];
  const int k = blockIdx.x;
  double s = 0.0;
  int64_t t = threadIdx.x;
  for (; t + 7 * 1024 < T; t += 8 * 1024) {
    double v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = rows[4 * (t + 1024 * u) + k];
#pragma unroll
    for (int u = 0; u < 8; ++u) s += v[u];
  }
  for (; t < T; t += 1024) s += rows[4 * t + k];
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  double v = 0.0;
  for (int w = 0; w < 16; ++w) v += part[w];
  sums[k] = (float)v;
}

// Threads of a row and their vectors, by the row's vectors of 16 bytes: the fewest
// threads that hold them in 8 each, then 1,024 with more.  Up to 7 vectors fit the 64
// registers of 8 waves a SIMD; 8 vectors take 7 waves, or with 1,024 threads 8 words of
// scratch a thread.  Against the next more threads, loss with its gradient and log-probabilities
// alone (us): 100,000 rows of 1,000 of bf16 112 and 42 with 64 threads, 212 and 104 with 256;
// 32,768 of 2,500 66 and 31, 95 and 51; of 4,096 97 and 42, 110 and 52; 16,384 of 10,000 124
// and 57 with 256, 129 and 74 with 512, of 16,384 202 and 89, 185 and 88; 8,192 of 20,000 120
// and 55 with 512, 138 and 80 with 1,024, of 32,768 220 and 92, 195 and 96 (rows that fill 8
// vectors would be better with more threads if they are written, not if they are only read).
// Against 1,024 threads of 7 vectors, rows of 50,000 of bf16 took 1% longer with 512 of 13 and
// with 256 of 25; of 16,411 of binary32, against 1,024 of 5, 4% with 512 of 9, 7% with 256 of 17.
template <int LT, int R, int NV>
int rows_in(const Loss& a, hipStream_t st) {
  return launch_parts(&k_loss<LT, R, NV>, a.T, R, st, a);
}
template <int LT>
int rows_of(const Loss& a, hipStream_t st) {
  const int64_t vecs = (a.V + per_vec<LT>() - 1) / per_vec<LT>();
  const auto per = [&](int64_t threads) { return (vecs + threads - 1) / threads; };
  if (per(64) <= 2) return rows_in<LT, 64, 2>(a, st);
  if (per(64) <= 4) return rows_in<LT, 64, 4>(a, st);
  if (per(64) <= 6) return rows_in<LT, 64, 6>(a, st);
  if (per(64) <= 8) return rows_in<LT, 64, 8>(a, st);
  if (per(256) <= 2) return rows_in<LT, 256, 2>(a, st);
  if (per(256) <= 3) return rows_in<LT, 256, 3>(a, st);
  if (per(256) <= 4) return rows_in<LT, 256, 4>(a, st);
  if (per(256) <= 6) return rows_in<LT, 256, 6>(a, st);
  if (per(256) <= 8) return rows_in<LT, 256, 8>(a, st);
  if (per(512) <= 5) return rows_in<LT, 512, 5>(a, st);
  if (per(512) <= 6) return rows_in<LT, 512, 6>(a, st);
  if (per(512) <= 7) return rows_in<LT, 512, 7>(a, st);
  if (per(512) <= 8) return rows_in<LT, 512, 8>(a, st);
  if (per(1024) <= 5) return rows_in<LT, 1024, 5>(a, st);
  if (per(1024) <= 6) return rows_in<LT, 1024, 6>(a, st);
  if (per(1024) <= 7) return rows_in<LT, 1024, 7>(a, st);
  if (per(1024) <= 8) return rows_in<LT, 1024, 8>(a, st);
  if (per(1024) <= 10) return rows_in<LT, 1024, 10>(a, st);
  if (per(1024) <= 13) return rows_in<LT, 1024, 13>(a, st);
  if (per(1024) <= 16) return rows_in<LT, 1024, 16>(a, st);
  return rows_in<LT, 1024, 0>(a, st);
}

int run(const Loss& a, int lt, hipStream_t st) {
  return lt == ZQ_F32 ? rows_of<ZQ_F32>(a, st) : lt == ZQ_F16 ? rows_of<ZQ_F16>(a, st) : rows_of<ZQ_BF16>(a, st);
}

// bytes of T rows of V elements, `ld` apart
int64_t span(int64_t T, int64_t V, int64_t ld, int64_t e) { return T > 0 ? ((T - 1) * ld + V) * e : 0; }

int check_logits(const void* logits, int lt, int64_t T, int64_t V, int64_t ld, const void* ids, int it, float scale) {
  if (!dtype_ok(lt) || (it != ZQ_I32 && it != ZQ_I64)) return ZQ_E_DTYPE;
  if (T < 0 || T > (1 << 30) || V < 1 || V > kMaxVocab || ld < V || (T > 0 && ld > kMaxPlaces / T)) return ZQ_E_SIZE;
  if (!(scale > 0.0f && scale <= kMaxScale)) return ZQ_E_SIZE;
  if (T == 0) return ZQ_OK;
  if (!logits || !ids) return ZQ_E_NULL;
  if (!aligned(logits, elem_bytes(lt)) || !aligned(ids, it == ZQ_I64 ? 8 : 4)) return ZQ_E_ALIGN;
  return ZQ_OK;
}

}  // namespace
}  // namespace zq

extern "C" {

using namespace zq;

int zq_token_logp(const void* logits, zq_dtype lt, int64_t T, int64_t V, int64_t ld, const void* ids, zq_dtype it,
                  float scale, float* logp, void* stream) {
  const int rc = check_logits(logits, lt, T, V, ld, ids, it, scale);
  if (rc != ZQ_OK || T == 0) return rc;
  if (!logp) return ZQ_E_NULL;
  if (!aligned(logp, 4)) return ZQ_E_ALIGN;
  if (any_overlap({{logp, 4 * T}}, {{logits, span(T, V, ld, elem_bytes(lt))}, {ids, T * (it == ZQ_I64 ? 8 : 4)}}))
    return ZQ_E_ALIAS;
  Loss a = {};
  a.logits = logits, a.ids = ids, a.T = T, a.V = V, a.ld = ld, a.scale = scale, a.it = it, a.logp = logp;
  return run(a, lt, static_cast<hipStream_t>(stream));
}

int64_t zq_policy_loss_bytes(int64_t T) { return T < 0 || T > (1 << 30) ? -1 : 32 * T; }

int zq_policy_loss(const void* logits, zq_dtype lt, int64_t T, int64_t V, int64_t ld, const void* ids, zq_dtype it,
                   const zq_policy* policy, float* sums, float* logp, void* grad, zq_dtype gt, int64_t ldg,
                   void* workspace, int64_t workspace_bytes, void* stream) {
  if (!policy) return ZQ_E_NULL;
  const zq_policy& p = *policy;
  const int rc = check_logits(logits, lt, T, V, ld, ids, it, p.scale);
  if (rc != ZQ_OK) return rc;
  if (grad && !dtype_ok(gt)) return ZQ_E_DTYPE;
  if (!(p.clip_low >= 0.0f && p.clip_low <= 1.0f) || !(p.clip_high >= 0.0f) || !(p.kl >= 0.0f) ||
      !std::isfinite(p.clip_high) || !std::isfinite(p.kl) || !std::isfinite(p.grad_scale))
    return ZQ_E_SIZE;
  if (grad && (ldg < V || (T > 0 && ldg > kMaxPlaces / T))) return ZQ_E_SIZE;
  const int64_t need = zq_policy_loss_bytes(T);
  if (workspace_bytes < need) return ZQ_E_SIZE;
  if (!sums || (T > 0 && (!workspace || !p.old_logp || !p.advantages || (p.kl != 0.0f && !p.ref_logp)))) return ZQ_E_NULL;
  const int64_t ge = grad ? elem_bytes(gt) : 1;
  if (!aligned(sums, 4) || !aligned(logp, 4) || !aligned(grad, ge) || (T > 0 && !aligned(workspace, 16)) ||
      !aligned(p.old_logp, 4) || !aligned(p.advantages, 4) || !aligned(p.weights, 4) || !aligned(p.ref_logp, 4))
    return ZQ_E_ALIGN;
  const bool in_place = grad && grad == logits && gt == lt && ldg == ld;
  const Range g = {grad, grad ? span(T, V, ldg, ge) : 0};
  const Range z = {in_place ? nullptr : logits, in_place ? 0 : span(T, V, ld, elem_bytes(lt))};
  const Range old = {p.old_logp, 4 * T}, adv = {p.advantages, 4 * T};
  const Range w = {p.weights, p.weights ? 4 * T : 0}, ref = {p.ref_logp, p.ref_logp ? 4 * T : 0};
  if (any_overlap({g, {sums, 16}, {logp, logp ? 4 * T : 0}, {need ? workspace : nullptr, need}},
                  {z, {ids, T * (it == ZQ_I64 ? 8 : 4)}, old, adv, w, ref}))
    return ZQ_E_ALIAS;
  hipStream_t st = static_cast<hipStream_t>(stream);
  Loss a = {};
  a.logits = logits, a.ids = ids, a.T = T, a.V = V, a.ld = ld, a.scale = p.scale, a.it = it, a.logp = logp;
  a.rows = static_cast<double*>(workspace);
  a.grad = grad, a.ldg = ldg, a.gt = gt;
  a.old_logp = p.old_logp, a.advantages = p.advantages, a.weights = p.weights, a.ref_logp = p.ref_logp;
  a.clip_low = p.clip_low, a.clip_high = p.clip_high, a.kl = p.kl, a.grad_scale = p.grad_scale;
  if (T > 0) {
    const int rc2 = run(a, lt, st);
    if (rc2 != ZQ_OK) return rc2;
  }
  return launch(&k_loss_sums, 4u, 1024u, st, static_cast<const double*>(workspace), T, sums);
}

}  // extern "C"
