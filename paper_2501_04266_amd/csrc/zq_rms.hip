// zq_rms.hip -- root-mean-square norm of rows after the residual's addition, its output
// dense or as INT8 blocks, and its gradient, on gfx950.
//
//   h = cvt(fl(x + residual))   rstd = fl(1 / sqrt(sum h^2 / D + eps))   y = fl(fl(h rstd) w)
//   dx = rstd (dy w - xh sum(dy w xh) / D) + dh      dw = sum over rows of dy xh      xh = fl(h rstd)
//
// Bound by memory: a row is read once, held in its threads' registers between the sum and
// the output, and written once (16,384 rows of 6,144 of bf16 with a residual: 134 us, 6.0
// TB/s; their gradient 137, 5.9 TB/s).  Squares and their sum are binary64: the sum's order does
// not show in rstd except by one rounding, so INT8 codes next to a border do not depend on
// how a row is cut.
//
// A row belongs to 16 to 1,024 threads with up to 2 vectors of 8 elements each (in the
// gradient up to 4), by its length; longer rows are read a second time.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "zq.h"
#include "zq_device.h"
#include "zq_host.h"
#include "zq_lanes.h"
#include "zq_vec.h"

#pragma clang fp contract(off)

namespace zq {
namespace {

constexpr int kInt8 = 3;  // y's type code beside ZQ_F32 / ZQ_F16 / ZQ_BF16
constexpr int64_t kMaxWidth = 1 << 24;
constexpr int64_t kUnits = 256;  // CUs of the chip

// ---------------------------------------------------------------- rows

// Places in a row are 32-bit numbers of bytes: rows have up to 2^24 elements.  Threads hold
// vectors of 8 elements of the first D - D % 8; the row's last D % 8 are held one each by its
// first threads, so that no vector needs moving or splitting (a partial vector's words moved
// into place cost the gradient of 16,384 x 2,056 twice its time: the wave waited for them).

// Which accesses pass the caches by, measured in turns on 16,384 x 6,144 of bf16, outputs in
// new memory each time: the norm 140 us with its stores past them, 137 with its loads too
// (but 37 and 35 us on 8,192 x 2,048 into INT8), 147 with neither; its gradient 137 with
// both, 148 with its loads alone, 153 with neither.  The gradient's do so only where rows are
// whole lines of 128 bytes, or with 16-bit elements alone whole halves of one: else two rows
// share a line (5,003 rows of 2,051 of fp16: loads past them 39 us, through them 32, with stores
// past them 4% more).  Whole halves, past them and through them: of bf16 a million rows of 96
// 132 and 144 us, 24,000 of 4,128 140 and 147; of binary32 95,000 rows of 528 194 and 161,
// 24,000 of 2,064 193 and 171.  Where dx starts does not matter as much as that its rows are
// written whole (16,384 x 6,144 of bf16 from any element 138 us, through the caches 153).
constexpr bool kNormLoadsPast = false, kNormStoresPast = true;

// the words of 8 elements from element i on; zeros from element n on, a multiple of 8
template <int DT, bool PAST>
__device__ __forceinline__ void load8(const char* row, int i, int n, uint32_t (&w)[2 * dt_size<DT>()]) {
#pragma unroll
  for (int k = 0; k < 2 * dt_size<DT>(); ++k) w[k] = 0u;
  if (i < n) load_words_any<PAST>(row + (uint32_t)i * dt_size<DT>(), w);
}
// of a type that is known when the kernel runs: in the first 4 or in all 8 words
template <bool PAST>
__device__ __forceinline__ void load8(int dt, const char* row, int i, int n, uint32_t (&w)[8]) {
  if (dt == ZQ_F32) {
    load8<ZQ_F32, PAST>(row, i, n, w);
    return;
  }
  uint32_t t[4];
  load8<ZQ_BF16, PAST>(row, i, n, t);
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = t[k], w[k + 4] = 0u;
}
// one element
template <int DT>
__device__ __forceinline__ float load1(const char* row, int i) {
  float v[1];
  load_elems<DT, 1>(row + (uint32_t)i * dt_size<DT>(), 0, v);
  return v[0];
}
__device__ __forceinline__ float load1(int dt, const char* row, int i) {
  return dt == ZQ_F32 ? load1<ZQ_F32>(row, i) : dt == ZQ_BF16 ? load1<ZQ_BF16>(row, i) : load1<ZQ_F16>(row, i);
}
template <int DT>
__device__ __forceinline__ void store1(char* row, int i, float v) {
  const float t[1] = {v};
  store_elems<DT, 1>(row + (uint32_t)i * dt_size<DT>(), 0, t);
}
__device__ __forceinline__ void store1(int dt, char* row, int i, float v) {
  if (dt == ZQ_F32) store1<ZQ_F32>(row, i, v);
  else if (dt == ZQ_BF16) store1<ZQ_BF16>(row, i, v);
  else store1<ZQ_F16>(row, i, v);
}
__device__ __forceinline__ void widen8(int dt, const uint32_t (&w)[8], float (&v)[8]) {
  if (dt == ZQ_F32) widen<ZQ_F32>(w, v);
  else if (dt == ZQ_BF16) widen<ZQ_BF16>(w, v);
  else widen<ZQ_F16>(w, v);
}
template <int DT, bool PAST>
__device__ __forceinline__ void store8(char* row, int i, int n, const float (&v)[8]) {
  if (i < n) store_elems<DT, 8, PAST>(row + (uint32_t)i * dt_size<DT>(), 0, v);
}
template <bool PAST>
__device__ __forceinline__ void store8(int dt, char* row, int i, int n, const float (&v)[8]) {
  if (dt == ZQ_F32) store8<ZQ_F32, PAST>(row, i, n, v);
  else if (dt == ZQ_BF16) store8<ZQ_BF16, PAST>(row, i, n, v);
  else store8<ZQ_F16, PAST>(row, i, n, v);
}
template <int DT>
__device__ __forceinline__ float as_stored(float v) {
  if constexpr (DT == ZQ_BF16) return u2f(bf16x2_bits(v, 0.0f) << 16);
  else if constexpr (DT == ZQ_F16) return h2f(f2h(v));
  else return v;
}
// the words of 8 values as a type holds them
template <int DT>
__device__ __forceinline__ void narrow8(const float (&v)[8], uint32_t (&w)[2 * dt_size<DT>()]) {
#pragma unroll
  for (int k = 0; k < 2 * dt_size<DT>(); ++k) {
    if constexpr (DT == ZQ_F32) w[k] = f2u(v[k]);
    else if constexpr (DT == ZQ_BF16) w[k] = bf16x2_bits(v[2 * k], v[2 * k + 1]);
    else w[k] = f2h(v[2 * k]) | (f2h(v[2 * k + 1]) << 16);
  }
}
// The words are what they were, but the compiler does not know: what it has derived from
// them (their widened values) is not kept in registers across this point.
template <int N>
__device__ __forceinline__ void forget(uint32_t (&w)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) asm volatile("" : "+v"(w[k]));
}

constexpr int kind_bytes(int dt) { return dt == ZQ_F32 ? 4 : 2; }

// ---------------------------------------------------------------- sums over a row's threads

// the sum over a row's R threads, in all of them; `slot`: R / 64 values of LDS, written
// again only after a barrier
template <int R, typename F>
__device__ __forceinline__ F row_sum(F v, F* slot) {
  if constexpr (R <= 64) return lanes_sum<R>(v);
  v = lanes_sum<64>(v);
  if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
  __syncthreads();
  F s = slot[0];
#pragma unroll
  for (int w = 1; w < R / 64; ++w) s += slot[w];
  return s;
}

// The largest of `v` (bits of non-negative numbers) over each group of `lanes` lanes.
__device__ __forceinline__ uint32_t lanes_max(uint32_t v, int lanes) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));                    // quad_perm 1,0,3,2
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));                    // quad_perm 2,3,0,1
  if (lanes >= 8) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false));   // row_half_mirror
  if (lanes >= 16) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, false));  // row_mirror
  if (lanes >= 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16, 64));
  if (lanes >= 64) v = max(v, (uint32_t)__shfl_xor((int)v, 32, 64));
  return v;
}

// 1 / sqrt(x) to the last bits of binary64: v_rsq_f64 (good to some 2^-26) and one step of
// third order, y + y e (1/2 + 3/8 e) with e = 1 - x y^2, whose error is about e^3.  Every thread
// of a row computes it: with a division and a square root in its place, 8,192 rows of 2,048
// into INT8 (and dequantised) take 34.6 us and not 33.2.
__device__ __forceinline__ double inverse_root(double x) {
  if (!(x > 0.0 && x < (double)__builtin_inff())) return 1.0 / sqrt(x);
  const double y = __builtin_amdgcn_rsq(x), e = __builtin_fma(-x * y, y, 1.0);
  return __builtin_fma(y * e, __builtin_fma(0.375, e, 0.5), y);
}

// ---------------------------------------------------------------- forward

struct Norm {
  const void* x;
  const void* residual;
  const void* weight;
  void* h;
  void* y;
  float* scales;
  float* rstd;
  int64_t T, D;
  double eps, share;  // share = 1 / D
  int8_t wt, yt, lgB;
};

// 8 values of a row as codes of the INT8 format.  All threads of the row's waves call it;
// a block of 1,024 is two waves', whose halves meet in `half` (LDS, R / 64 values).
template <int R>
__device__ __forceinline__ void put_int8(const Norm& a, int64_t at, int i, const float (&v)[8], uint32_t* half) {
  uint32_t t = 0u;
#pragma unroll
  for (int k = 0; k < 8; ++k) t = max(t, f2u(v[k]) & 0x7fffffffu);
  t = lanes_max(t, a.lgB < 9 ? 1 << (a.lgB - 3) : 64);
  if (R > 64 && a.lgB == 10) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) half[threadIdx.x >> 6] = t;
    __syncthreads();
    t = max(t, half[(threadIdx.x >> 6) ^ 1]);
  }
  const float m = u2f(t);
  const bool fits = m >= 0x1p-119f;
  // m / 127 is a binary32 number or further than 2^-32 of it from the middle of two: its product
  // with 1 / 127 in binary64, rounded, is the rounded quotient
  const float s = fits ? (float)((double)m * (1.0 / 127.0)) : 0.0f, r = fits ? 127.0f / m : 0.0f;
  if (i >= (int)a.D) return;
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int k = 0; k < 8; ++k) w[k / 4] |= ((uint32_t)(int)rintf(v[k] * r) & 0xffu) << (8 * (k & 3));
  store_words_any<true>(static_cast<char*>(a.y) + at + i, w);
  if ((i & ((1 << a.lgB) - 1)) == 0) a.scales[(at + i) >> a.lgB] = s;
}

// NV vectors of 8 elements a thread; NV = 0: rows of any length, h read again.
// Everything a row needs is loaded before the first store: loads would wait behind stores
// that might be to their memory.
template <int XT, int R, int NV>
__device__ __forceinline__ void norm_row(const Norm& a, int64_t t, int lane, double* slot, uint32_t* half) {
  constexpr int W = 2 * dt_size<XT>(), N = NV > 0 ? NV : 1;
  const int D = (int)a.D & ~7, last = D + lane;  // vectors up to D, then one element a thread
  const bool has_last = last < (int)a.D;
  const int64_t at = t * a.D;  // the row's first element
  const char* x = static_cast<const char*>(a.x) + at * dt_size<XT>();
  const char* res = a.residual ? static_cast<const char*>(a.residual) + at * dt_size<XT>() : nullptr;
  const char* weight = static_cast<const char*>(a.weight);
  char* h = a.residual ? static_cast<char*>(a.h) + at * dt_size<XT>() : nullptr;
  char* y = static_cast<char*>(a.y) + at * kind_bytes(a.yt);

  double sum = 0.0;
  uint32_t xw[N][W], rw[N][W], ww[N][8];
  float x1 = 0.0f, r1 = 0.0f, w1 = 1.0f;
  auto load = [&](int j, int i) {
    load8<XT, kNormLoadsPast>(x, i, D, xw[j]);
    if (res) load8<XT, kNormLoadsPast>(res, i, D, rw[j]);
  };
  auto load_last = [&]() {
    if (!has_last) return;
    x1 = load1<XT>(x, last);
    if (res) r1 = load1<XT>(res, last);
    if (weight) w1 = load1(a.wt, weight, last);
  };
  auto add = [&](int j, int i) {  // xw becomes h's words
    float v[8];
    widen<XT>(xw[j], v);
    if (res) {
      float b[8];
      widen<XT>(rw[j], b);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = v[k] + b[k];
      narrow8<XT>(v, xw[j]);
      widen<XT>(xw[j], v);
      store8<XT, kNormStoresPast>(h, i, D, v);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) sum = __builtin_fma((double)v[k], (double)v[k], sum);
    forget(xw[j]);
  };
  auto add_last = [&]() {  // x1 becomes h's element
    if (!has_last) return;
    if (res) {
      x1 = as_stored<XT>(x1 + r1);
      store1<XT>(h, last, x1);
    }
    sum = __builtin_fma((double)x1, (double)x1, sum);
  };
  auto put = [&](int j, int i, float rstd) {
    float v[8], w[8];
    widen<XT>(xw[j], v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = v[k] * rstd;
    if (weight) {
      widen8(a.wt, ww[j], w);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = v[k] * w[k];
    }
    if (a.yt == kInt8) put_int8<R>(a, at, i, v, half);
    else store8<kNormStoresPast>(a.yt, y, i, D, v);
  };
  auto finish = [&]() {
    sum = row_sum<R>(sum, slot);
    const float rstd = (float)inverse_root(sum * a.share + a.eps);
    if (a.rstd && lane == 0) a.rstd[t] = rstd;
    if (has_last) store1(a.yt, y, last, weight ? (x1 * rstd) * w1 : x1 * rstd);
    return rstd;
  };

  if constexpr (NV > 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) load(j, (j * R + lane) * 8);
    if (weight) {
#pragma unroll
      for (int j = 0; j < NV; ++j) load8<false>(a.wt, weight, (j * R + lane) * 8, D, ww[j]);
    }
    load_last();
#pragma unroll
    for (int j = 0; j < NV; ++j) add(j, (j * R + lane) * 8);
    add_last();
    const float rstd = finish();
#pragma unroll
    for (int j = 0; j < NV; ++j) put(j, (j * R + lane) * 8, rstd);
  } else {
    const int end = (D + 8 * R - 1) / (8 * R) * (8 * R);  // all threads take every turn
    load_last();
    for (int i = lane * 8; i < end; i += 8 * R) {
      load(0, i);
      add(0, i);
    }
    add_last();
    const float rstd = finish();
    for (int i = lane * 8; i < end; i += 8 * R) {
      load8<XT, kNormLoadsPast>(res ? h : x, i, D, xw[0]);  // h: this thread's own writes
      if (weight) load8<false>(a.wt, weight, i, D, ww[0]);
      put(0, i, rstd);
    }
  }
}

template <int XT, int R, int NV>
__global__ void __launch_bounds__(R <= 64 ? 256 : R) k_rms(unsigned first, Norm a) {
  constexpr int THREADS = R <= 64 ? 256 : R;
  __shared__ double slot[(R + 63) / 64];
  __shared__ uint32_t half[(R + 63) / 64];
  const int lane = threadIdx.x % R;
  const int64_t t = (int64_t)(first + blockIdx.x) * (THREADS / R) + threadIdx.x / R;
  if (R <= 64 && t >= a.T) return;  // rows within a wave: the others go on
  norm_row<XT, R, NV>(a, t, lane, slot, half);
}

// ---------------------------------------------------------------- gradient

struct NormGrad {
  const void* dy;
  const void* h;
  const void* weight;
  const float* rstd;
  const void* dh;
  void* dx;
  float* part;  // [parts][D] sums of dw, or NULL
  int64_t T, D;
  int groups;   // of rows: group g has the rows g, g + groups, ...
  int8_t gt, wt;
  bool lines;   // rows of whole cache lines (or halves), from the first byte of one
};

// The rows of group g.  A thread keeps its columns' weight and sums of dw; AHEAD: the next
// row's h and dy are loaded before the present row's sum is taken.  LINES: rows are whole
// cache lines or halves of them.  Where a workgroup has several groups (R <= 64) it adds their sums of dw, in the
// groups' order and in binary64, and writes one: with each group's own, 16,384 of them at
// D <= 128, 65,536 rows of 16 took 76 us and not 17, of 128 84 and not 20, of 512 67 and not 53.
template <int XT, int R, int NV, bool SAME, bool AHEAD, bool LINES>
__device__ __forceinline__ void grad_rows(const NormGrad& a, int g, int lane, float (*slot)[(R + 63) / 64],
                                          float* sums) {
  constexpr int W = 2 * dt_size<XT>(), WY = SAME ? W : 8;
  const int D = (int)a.D & ~7, last = D + lane;  // vectors up to D, then one element a thread
  const bool has_last = !LINES && last < (int)a.D;
  const int64_t row_bytes = a.D * dt_size<XT>(), dy_bytes = a.D * (SAME ? dt_size<XT>() : kind_bytes(a.gt));
  float w[NV][8], dw[NV][8], w1 = 1.0f, dw1 = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
#pragma unroll
    for (int k = 0; k < 8; ++k) dw[j][k] = 0.0f, w[j][k] = 1.0f;
    if (a.weight) {
      uint32_t t[8];
      load8<false>(a.wt, static_cast<const char*>(a.weight), (j * R + lane) * 8, D, t);
      widen8(a.wt, t, w[j]);
    }
  }
  if (has_last && a.weight) w1 = load1(a.wt, static_cast<const char*>(a.weight), last);
  uint32_t hw[NV][W], yw[NV][WY], dhw[NV][W], hn[AHEAD ? NV : 1][W], yn[AHEAD ? NV : 1][WY];
  float h1 = 0.0f, y1 = 0.0f, hn1 = 0.0f, yn1 = 0.0f;
  auto load = [&](int64_t t, auto& hw_, auto& yw_, float& h1_, float& y1_) {
    const char* hr = static_cast<const char*>(a.h) + t * row_bytes;
    const char* yr = static_cast<const char*>(a.dy) + t * dy_bytes;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      load8<XT, LINES>(hr, (j * R + lane) * 8, D, hw_[j]);
      if constexpr (SAME) load8<XT, LINES>(yr, (j * R + lane) * 8, D, yw_[j]);
      else load8<LINES>(a.gt, yr, (j * R + lane) * 8, D, yw_[j]);
    }
    if (has_last) {
      h1_ = load1<XT>(hr, last);
      y1_ = SAME ? load1<XT>(yr, last) : load1(a.gt, yr, last);
    }
  };
  auto dy_of = [&](int j, float (&v)[8]) {
    if constexpr (SAME) widen<XT>(yw[j], v);
    else widen8(a.gt, yw[j], v);
  };
  int turn = 0;
  const bool rows = R > 64 || g < a.groups;
  float rstd_next = 0.0f;
  if (rows) {
    if constexpr (AHEAD) load(g, hw, yw, h1, y1);
    rstd_next = a.rstd[g];
  }
  for (int64_t t = rows ? g : a.T; t < a.T; t += a.groups, turn ^= 1) {
    const char* dhr = a.dh ? static_cast<const char*>(a.dh) + t * row_bytes : nullptr;
    char* dxr = static_cast<char*>(a.dx) + t * row_bytes;
    const float rstd = rstd_next;
    float d1 = 0.0f;
    if constexpr (!AHEAD) load(t, hw, yw, h1, y1);
    if (dhr) {
#pragma unroll
      for (int j = 0; j < NV; ++j) load8<XT, LINES>(dhr, (j * R + lane) * 8, D, dhw[j]);
      if (has_last) d1 = load1<XT>(dhr, last);
    }
    if (t + a.groups < a.T) {
      rstd_next = a.rstd[t + a.groups];
      if constexpr (AHEAD) load(t + a.groups, hn, yn, hn1, yn1);
    }
    const float xh1 = h1 * rstd, gw1 = y1 * w1;
    float c = gw1 * xh1;
    dw1 += y1 * xh1;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float h[8], dy[8];
      widen<XT>(hw[j], h);
      dy_of(j, dy);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float xh = h[k] * rstd;
        dw[j][k] += dy[k] * xh;
        c += (dy[k] * w[j][k]) * xh;
      }
      forget(hw[j]);
      forget(yw[j]);
    }
    c = row_sum<R>(c, slot[turn]) / (float)a.D;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float h[8], dy[8], d[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
      widen<XT>(hw[j], h);
      dy_of(j, dy);
      if (dhr) widen<XT>(dhw[j], d);
#pragma unroll
      for (int k = 0; k < 8; ++k) d[k] += (dy[k] * w[j][k] - (h[k] * rstd) * c) * rstd;
      store8<XT, LINES>(dxr, (j * R + lane) * 8, D, d);
    }
    if (has_last) store1<XT>(dxr, last, d1 + (gw1 - xh1 * c) * rstd);
    if constexpr (AHEAD) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int k = 0; k < W; ++k) hw[j][k] = hn[j][k];
#pragma unroll
        for (int k = 0; k < WY; ++k) yw[j][k] = yn[j][k];
      }
      h1 = hn1, y1 = yn1;
    }
  }
  if (!a.part) return;
  if constexpr (R <= 64) {
    float* own = sums + (threadIdx.x / R) * (8 * R);
    if (lane * 8 < D) {
#pragma unroll
      for (int k = 0; k < 8; ++k) own[lane * 8 + k] = dw[0][k];
    }
    if (has_last) own[last] = dw1;
    __syncthreads();
    for (int d = threadIdx.x; d < (int)a.D; d += 256) {
      double v = 0.0;
      for (int r = 0; r < 256 / R; ++r) v += (double)sums[r * (8 * R) + d];
      a.part[(int64_t)blockIdx.x * a.D + d] = (float)v;
    }
    return;
  }
  char* part = reinterpret_cast<char*>(a.part + (int64_t)g * a.D);
#pragma unroll
  for (int j = 0; j < NV; ++j) store8<ZQ_F32, false>(part, (j * R + lane) * 8, D, dw[j]);
  if (has_last) store1<ZQ_F32>(part, last, dw1);
}

template <int XT, int R, int NV, bool SAME, bool AHEAD>
__global__ void __launch_bounds__(R <= 64 ? 256 : R) k_rms_grad(NormGrad a) {
  constexpr int THREADS = R <= 64 ? 256 : R;
  static_assert(R > 64 || NV == 1, "8 R columns a group's sums");
  __shared__ float slot[2][(R + 63) / 64], sums[R <= 64 ? 8 * THREADS : 1];
  const int lane = threadIdx.x % R;
  const int g = blockIdx.x * (THREADS / R) + threadIdx.x / R;  // R <= 64: the last may have no rows
  if (a.lines) grad_rows<XT, R, NV, SAME, AHEAD, true>(a, g, lane, slot, sums);
  else grad_rows<XT, R, NV, SAME, AHEAD, false>(a, g, lane, slot, sums);
}

// rows of any length: dx, a row a workgroup, read twice
template <int XT>
__global__ void __launch_bounds__(1024) k_rms_grad_long(unsigned first, NormGrad a) {
  __shared__ double slot[16];
  const int D = (int)a.D & ~7, last = D + (int)threadIdx.x;
  const bool has_last = last < (int)a.D;
  const int64_t t = first + blockIdx.x, at = t * a.D;
  const char* hr = static_cast<const char*>(a.h) + at * dt_size<XT>();
  const char* dyr = static_cast<const char*>(a.dy) + at * kind_bytes(a.gt);
  const char* dhr = a.dh ? static_cast<const char*>(a.dh) + at * dt_size<XT>() : nullptr;
  const char* weight = static_cast<const char*>(a.weight);
  char* dxr = static_cast<char*>(a.dx) + at * dt_size<XT>();
  const float rstd = a.rstd[t];
  auto take = [&](int i, float (&xh)[8], float (&gw)[8]) {
    uint32_t hw[2 * dt_size<XT>()], yw[8], ww[8];
    load8<XT, false>(hr, i, D, hw);
    load8<false>(a.gt, dyr, i, D, yw);
    widen<XT>(hw, xh);
    widen8(a.gt, yw, gw);
    if (weight) {
      float w[8];
      load8<false>(a.wt, weight, i, D, ww);
      widen8(a.wt, ww, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) gw[k] = gw[k] * w[k];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) xh[k] = xh[k] * rstd;
  };
  const float xh1 = has_last ? load1<XT>(hr, last) * rstd : 0.0f;
  const float gw1 = has_last ? load1(a.gt, dyr, last) * (weight ? load1(a.wt, weight, last) : 1.0f) : 0.0f;
  double sum = (double)(gw1 * xh1);
  for (int i = threadIdx.x * 8; i < D; i += 8192) {
    float xh[8], gw[8], c = 0.0f;
    take(i, xh, gw);
#pragma unroll
    for (int k = 0; k < 8; ++k) c += gw[k] * xh[k];
    sum += (double)c;
  }
  const float c = (float)(row_sum<1024>(sum, slot) / (double)a.D);
  for (int i = threadIdx.x * 8; i < D; i += 8192) {
    float xh[8], gw[8], d[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    take(i, xh, gw);
    if (dhr) {
      uint32_t dw[2 * dt_size<XT>()];
      load8<XT, false>(dhr, i, D, dw);
      widen<XT>(dw, d);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) d[k] += (gw[k] - xh[k] * c) * rstd;
    store8<XT, false>(dxr, i, D, d);
  }
  if (has_last) store1<XT>(dxr, last, (dhr ? load1<XT>(dhr, last) : 0.0f) + (gw1 - xh1 * c) * rstd);
}

// and their part of dw: 256 x 8 columns of a group of rows a workgroup, the row's last
// D % 8 columns with the first 8's
template <int XT>
__global__ void __launch_bounds__(256) k_rms_grad_columns(unsigned first, NormGrad a, unsigned tiles) {
  const unsigned b = first + blockIdx.x;
  const int g = (int)(b / tiles), D = (int)a.D & ~7, i = (int)((b % tiles) * 256 + threadIdx.x) * 8, last = D + i / 8;
  const bool has_last = last < (int)a.D;
  if (i >= D && !has_last) return;
  float dw[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f}, dw1 = 0.0f;
  for (int64_t t = g; t < a.T; t += a.groups) {
    const char* hr = static_cast<const char*>(a.h) + t * a.D * dt_size<XT>();
    const char* yr = static_cast<const char*>(a.dy) + t * a.D * kind_bytes(a.gt);
    uint32_t hw[2 * dt_size<XT>()], yw[8];
    float h[8], dy[8];
    load8<XT, false>(hr, i, D, hw);
    load8<false>(a.gt, yr, i, D, yw);
    const float rstd = a.rstd[t];
    if (has_last) dw1 += load1(a.gt, yr, last) * (load1<XT>(hr, last) * rstd);
    widen<XT>(hw, h);
    widen8(a.gt, yw, dy);
#pragma unroll
    for (int k = 0; k < 8; ++k) dw[k] += dy[k] * (h[k] * rstd);
  }
  char* part = reinterpret_cast<char*>(a.part + (int64_t)g * a.D);
  store8<ZQ_F32, false>(part, i, D, dw);
  if (has_last) store1<ZQ_F32>(part, last, dw1);
}

// dw from the sums of the groups, or of the workgroups that have several: 64 columns a
// workgroup, 16 slices of the sums, each in its order, and then the slices in theirs, in binary64
__global__ void __launch_bounds__(1024)
    k_rms_grad_join(const float* __restrict__ part, int groups, int64_t D, int accumulate, void* dw, int dwt) {
  __shared__ double slice[16][64];
  const int64_t d = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
  const int s = threadIdx.x >> 6;
  double v = 0.0;
  if (d < D) {
    const int g0 = (int)((int64_t)groups * s / 16), g1 = (int)((int64_t)groups * (s + 1) / 16);
    int g = g0;
    for (; g + 16 <= g1; g += 16) {
      float t[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) t[k] = part[(int64_t)(g + k) * D + d];
#pragma unroll
      for (int k = 0; k < 16; ++k) v += (double)t[k];
    }
    for (; g < g1; ++g) v += (double)part[(int64_t)g * D + d];
  }
  slice[s][threadIdx.x & 63] = v;
  __syncthreads();
  if (s != 0 || d >= D) return;
  for (int k = 1; k < 16; ++k) v += slice[k][threadIdx.x];
  float t[1] = {(float)v};
  if (dwt == ZQ_F32) {
    float o[1];
    if (accumulate) load_elems<ZQ_F32, 1>(dw, d, o), t[0] = o[0] + t[0];
    store_elems<ZQ_F32, 1>(dw, d, t);
  } else if (dwt == ZQ_BF16) {
    float o[1];
    if (accumulate) load_elems<ZQ_BF16, 1>(dw, d, o), t[0] = o[0] + t[0];
    store_elems<ZQ_BF16, 1>(dw, d, t);
  } else {
    float o[1];
    if (accumulate) load_elems<ZQ_F16, 1>(dw, d, o), t[0] = o[0] + t[0];
    store_elems<ZQ_F16, 1>(dw, d, t);
  }
}

// ---------------------------------------------------------------- choice of kernel

// Threads of a row and vectors of each, by the row's length.  A block of 1,024 elements is
// two waves of one turn of a row's threads: where D can be a multiple of 1,024, R is one of 128.
template <int XT, int R, int NV>
int norm_in(const Norm& a, hipStream_t st) {
  return launch_parts(&k_rms<XT, R, NV>, a.T, R, st, a);
}
template <int XT>
int forward(const Norm& a, hipStream_t st) {
  if (a.D <= 128) return launch_parts(&k_rms<XT, 16, 1>, (a.T + 15) / 16, 256, st, a);
  if (a.D <= 256) return launch_parts(&k_rms<XT, 32, 1>, (a.T + 7) / 8, 256, st, a);
  if (a.D <= 512) return launch_parts(&k_rms<XT, 64, 1>, (a.T + 3) / 4, 256, st, a);
  if (a.D <= 1024) return norm_in<XT, 128, 1>(a, st);
  if (a.D <= 1536) return norm_in<XT, 192, 1>(a, st);
  if (a.D <= 2048) return norm_in<XT, 256, 1>(a, st);
  if (a.D <= 2560) return norm_in<XT, 320, 1>(a, st);
  if (a.D <= 4096) return norm_in<XT, 512, 1>(a, st);
  // 16,384 rows of 6,144: 140 us so, 145 with 256 threads of 3 vectors
  if (a.D <= 6144) return norm_in<XT, 384, 2>(a, st);
  if (a.D <= 8192) return norm_in<XT, 512, 2>(a, st);
  if (a.D <= 12288) return norm_in<XT, 768, 2>(a, st);
  if (a.D <= 16384) return norm_in<XT, 1024, 2>(a, st);
  return norm_in<XT, 1024, 0>(a, st);
}

int check_forward(const Norm& a, int xt, const void* weight, int wt, bool int8, int yt, int32_t block) {
  if (!dtype_ok(xt) || (weight && !dtype_ok(wt)) || (!int8 && !dtype_ok(yt))) return ZQ_E_DTYPE;
  if (int8 && log2_block(block) < 0) return ZQ_E_BLOCK;
  if (a.T < 0 || a.D < 1 || a.D > kMaxWidth || a.T > kMaxGrid || !(a.eps >= 0.0)) return ZQ_E_SIZE;
  if (int8 && a.D % block) return ZQ_E_SIZE;
  if (a.T == 0) return ZQ_OK;
  if (!a.x || !a.y || (a.residual && !a.h) || (int8 && !a.scales)) return ZQ_E_NULL;
  const int64_t e = elem_bytes(xt), n = a.T * a.D;
  if (!aligned(a.x, e) || !aligned(a.residual, e) || !aligned(a.h, e) || (weight && !aligned(weight, elem_bytes(wt))) ||
      (!int8 && !aligned(a.y, elem_bytes(yt))) || !aligned(a.scales, 4) || !aligned(a.rstd, 4))
    return ZQ_E_ALIGN;
  const Range x = {a.x, n * e}, res = {a.residual, a.residual ? n * e : 0};
  const Range w = {weight, weight ? a.D * elem_bytes(wt) : 0};
  const Range y = {a.y, int8 ? n : n * elem_bytes(yt)}, sc = {a.scales, int8 ? 4 * (n / block) : 0};
  const Range rs = {a.rstd, a.rstd ? 4 * a.T : 0}, h = {a.h, a.residual ? n * e : 0};
  if (any_overlap({y, sc, rs}, {x, res, w, h})) return ZQ_E_ALIAS;
  // h in the place of x or of residual, or apart from both
  if (a.residual && (overlap(h, w) || (a.h != a.x && overlap(h, x)) || (a.h != a.residual && overlap(h, res))))
    return ZQ_E_ALIAS;
  return ZQ_OK;
}

int rms_norm(const void* x, const void* residual, int xt, const void* weight, int wt, int64_t T, int64_t D, double eps,
             void* h, void* y, int yt, float* scales, int32_t block, float* rstd, void* stream, bool int8) {
  const Norm a = {x, residual, weight, h, y, scales, rstd, T, D, eps, 1.0 / (double)(D > 0 ? D : 1), (int8_t)wt, (int8_t)(int8 ? kInt8 : yt),
                  (int8_t)(int8 ? log2_block(block) : 0)};
  const int rc = check_forward(a, xt, weight, wt, int8, yt, block);
  if (rc != ZQ_OK || T == 0) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  return xt == ZQ_F32 ? forward<ZQ_F32>(a, st) : xt == ZQ_F16 ? forward<ZQ_F16>(a, st) : forward<ZQ_BF16>(a, st);
}

// Threads of a row in the gradient's kernels; 256 with up to 4 vectors each, as far as that
// goes, are better than more with fewer: 16,384 rows of 6,144 took 134 us with 256 threads of
// 3 vectors, 155 with 768 of one, 165 with 384 of 2.
// From 8,193 to 16,384 elements 1,024 threads hold a row only with words in scratch (49 a thread
// of 16 bits, 88 of unlike types, 170 of binary32): 6,144 rows of 16,384 take 145 us of bf16 (1.2
// of their floor), 3,072 of binary32 198 (1.6), of bf16 with a binary32 dy 112 (1.5).
int row_threads(int64_t D) {
  for (int r : {16, 32, 64, 128, 192, 256})
    if (D <= 8 * r) return r;
  return D <= 8192 ? 256 : 1024;
}
// Rows are dealt to groups, whose sums of dw are joined: the same number of groups for each
// CU, by D alone (the workspace's size knows no types) and as far as the sums stay within 16 MB:
// 16 waves' up to 2,048 elements a row, 12 to 4,096, 8 beyond.  The registers of a CU hold as
// many at once of 16-bit rows with dy of their type up to 6,144 elements.  Of others they hold one
// group fewer (binary32 and unlike types from 2,049 to 4,096, binary32 rows of 1,537 to 2,048
// with dy of another type) or one of two (16-bit rows from 6,145 to 8,192; binary32 and unlike
// types from 4,097, in 512 threads), and the rest run after them: 24,576 rows of 4,096 of
// binary32 take 306 us, 1.25 of their floor.
int64_t groups_for(int64_t T, int64_t D) {
  const int waves = D <= 2048 ? 16 : D <= 4096 ? 12 : 8;
  const int64_t g = kUnits * std::max(1, waves * 64 / row_threads(D));
  const int64_t most = std::max<int64_t>(1, (1 << 22) / D);
  return std::max<int64_t>(1, std::min(std::min(g, most), T));
}
// Sums of dw, 4 D bytes each: one a group, or one a workgroup of 256 threads with several.
int64_t parts_for(int64_t T, int64_t D) {
  const int r = row_threads(D), each = r <= 64 ? 256 / r : 1;
  return (groups_for(T, D) + each - 1) / each;
}

template <int XT, int R, int NV, bool SAME, bool AHEAD = true>
int grad_in(const NormGrad& a, hipStream_t st) {
  return launch(&k_rms_grad<XT, R, NV, SAME, AHEAD>, (unsigned)a.groups, R, st, a);
}
template <int XT, bool SAME>
int backward_short(const NormGrad& a, hipStream_t st) {
  constexpr bool WIDE = XT == ZQ_F32 || !SAME;  // vectors of up to 8 words: not more than 2 a thread
  switch (row_threads(a.D)) {
    case 16: return launch(&k_rms_grad<XT, 16, 1, SAME, true>, (unsigned)(a.groups + 15) / 16, 256u, st, a);
    case 32: return launch(&k_rms_grad<XT, 32, 1, SAME, true>, (unsigned)(a.groups + 7) / 8, 256u, st, a);
    case 64: return launch(&k_rms_grad<XT, 64, 1, SAME, true>, (unsigned)(a.groups + 3) / 4, 256u, st, a);
    case 128: return grad_in<XT, 128, 1, SAME>(a, st);
    case 192: return grad_in<XT, 192, 1, SAME>(a, st);
    case 1024: return grad_in<XT, 1024, 2, SAME, false>(a, st);
    default: break;
  }
  if (a.D <= 2048) return grad_in<XT, 256, 1, SAME>(a, st);
  if (a.D <= 4096) return grad_in<XT, 256, 2, SAME>(a, st);
  if constexpr (WIDE) return grad_in<XT, 512, 2, SAME>(a, st);
  else return a.D <= 6144 ? grad_in<XT, 256, 3, SAME>(a, st) : grad_in<XT, 256, 4, SAME>(a, st);
}

template <int XT>
int backward(const NormGrad& a, hipStream_t st) {
  if (a.D <= 16384) return a.gt == XT ? backward_short<XT, true>(a, st) : backward_short<XT, false>(a, st);
  int rc = launch_parts(&k_rms_grad_long<XT>, a.T, 1024, st, a);
  if (rc != ZQ_OK || !a.part) return rc;
  const unsigned tiles = (unsigned)((a.D + 2047) / 2048);
  return launch_parts(&k_rms_grad_columns<XT>, (int64_t)tiles * a.groups, 256, st, a, tiles);
}

bool grad_sizes_ok(int64_t T, int64_t D) { return T >= 0 && T <= kMaxGrid && D >= 1 && D <= kMaxWidth; }

}  // namespace
}  // namespace zq

extern "C" {

using namespace zq;

int zq_rms_norm(const void* x, const void* residual, zq_dtype xt, const void* weight, zq_dtype wt, int64_t T,
                int64_t D, double eps, void* h, void* y, zq_dtype yt, float* rstd, void* stream) {
  return rms_norm(x, residual, xt, weight, wt, T, D, eps, h, y, yt, nullptr, 0, rstd, stream, false);
}

int qwz_rms_norm(const void* x, const void* residual, zq_dtype xt, const void* weight, zq_dtype wt, int64_t T,
                 int64_t D, double eps, void* h, int8_t* codes, float* scales, int32_t block, float* rstd,
                 void* stream) {
  return rms_norm(x, residual, xt, weight, wt, T, D, eps, h, codes, 0, scales, block, rstd, stream, true);
}

int64_t zq_rms_norm_grad_bytes(int64_t T, int64_t D) {
  return grad_sizes_ok(T, D) ? 4 * parts_for(T, D) * D : -1;
}

int zq_rms_norm_grad(const void* dy, zq_dtype gt, const void* h, zq_dtype xt, const void* weight, zq_dtype wt,
                     const float* rstd, const void* dh, int64_t T, int64_t D, void* dx, int accumulate, void* dw,
                     zq_dtype dwt, void* workspace, int64_t workspace_bytes, void* stream) {
  if (!dtype_ok(gt) || !dtype_ok(xt) || (weight && !dtype_ok(wt)) || (dw && !dtype_ok(dwt))) return ZQ_E_DTYPE;
  if (!grad_sizes_ok(T, D)) return ZQ_E_SIZE;
  const int64_t need = dw ? zq_rms_norm_grad_bytes(T, D) : 0;
  if (workspace_bytes < need) return ZQ_E_SIZE;
  if (T == 0 && (!dw || accumulate)) return ZQ_OK;
  if ((need && !workspace) || (T > 0 && (!dy || !h || !rstd || !dx))) return ZQ_E_NULL;
  const int64_t e = elem_bytes(xt), n = T * D;
  if (!aligned(dy, elem_bytes(gt)) || !aligned(h, e) || (weight && !aligned(weight, elem_bytes(wt))) ||
      !aligned(rstd, 4) || !aligned(dh, e) || !aligned(dx, e) || (dw && !aligned(dw, elem_bytes(dwt))) ||
      (need && !aligned(workspace, 16)))
    return ZQ_E_ALIGN;
  const Range rdy = {dy, n * elem_bytes(gt)}, rh = {h, n * e}, rw = {weight, weight ? D * elem_bytes(wt) : 0};
  const Range rr = {rstd, 4 * T}, rdh = {dh, dh && dh != dx ? n * e : 0}, rdx = {dx, n * e};
  const Range rdw = {dw, dw ? D * elem_bytes(dwt) : 0}, ws = {need ? workspace : nullptr, need};
  if (any_overlap({rdx, rdw, ws}, {rdy, rh, rw, rr, rdh})) return ZQ_E_ALIAS;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int64_t line = xt == ZQ_F32 || gt == ZQ_F32 ? 128 : 64;
  const NormGrad a = {dy, h, weight, rstd, dh, dx, dw ? static_cast<float*>(workspace) : nullptr, T, D,
                      (int)groups_for(T, D), (int8_t)gt, (int8_t)wt,
                      D * e % line == 0 && D * elem_bytes(gt) % line == 0 && aligned(h, line) && aligned(dy, line) &&
                          aligned(dh, line)};
  if (T > 0) {
    const int rc = xt == ZQ_F32 ? backward<ZQ_F32>(a, st) : xt == ZQ_F16 ? backward<ZQ_F16>(a, st) : backward<ZQ_BF16>(a, st);
    if (rc != ZQ_OK) return rc;
  }
  if (!dw) return ZQ_OK;
  return launch(&k_rms_grad_join, (unsigned)((D + 63) / 64), 1024u, st, static_cast<const float*>(workspace),
                T > 0 ? (int)parts_for(T, D) : 0, D, accumulate, dw, (int)dwt);
}

}  // extern "C"
