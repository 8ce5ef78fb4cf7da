// zq_adamw.hip -- one AdamW step over many tensors, on gfx950.
//
//   g = fl(grad * c)      m = fl(fl(b1 m) + fl(om1 g))      v = fl(fl(b2 v) + fl(om2 fl(g g)))
//   p = cvt(fl(fl(p decay) - fl(alpha fl(m / fl(fl(sqrt(v) root) + eps)))))
//
// with c the clipping factor from a norm on the device, and the step's numbers alpha,
// decay, root computed in binary64.  Gradients are dense or INT4 shards (read as they
// are), moments binary32 or 8-bit floats with a scale a block, and the new weight can go
// out a second time in 16 bits or as INT8 codes and scales.
//
// Bound by memory: with binary32 weights and moments, bf16 gradients and a bf16 copy an
// element moves 28 bytes, with INT4 gradients, 8-bit moments and an INT8 copy 13.7.  One
// pass: the moments' scales and the INT8 copy's need the largest value of a block that is
// only known after the update, so a wave holds whole blocks (1,024 elements, the largest
// block) in registers, updates them, and takes the blocks' maxima across its lanes.
//
// A launch covers all tensors of a kind, a workgroup a piece: 4,096 elements where there are
// blocks, 1,024 where moments are binary32 and the copy is dense (fewer registers, twice the
// waves: in turns the step of 0.8 million elements took 5.5 us so and 7.6 in pieces of 4,096,
// that of 1.2 billion 6,040 and 6,080).  A map in the table says which tensor a piece belongs to.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "zq.h"
#include "zq_device.h"
#include "zq_host.h"
#include "zq_spans.h"
#include "zq_vec.h"

#pragma clang fp contract(off)

namespace zq {
namespace {

constexpr int kAdamThreads = 256;
constexpr int kSteps = 4;  // of a wave with blocks, 256 elements each: whole blocks of any size
constexpr int kPlainSteps = 1;
__host__ __device__ constexpr int piece_elems(bool blocks) { return (blocks ? kSteps : kPlainSteps) * 4 * kAdamThreads; }
constexpr int kInt4 = 3, kInt8 = 4;      // type codes beside ZQ_F32 / ZQ_F16 / ZQ_BF16
constexpr int kNone = -1;

// One tensor of the table.
struct Entry {
  char* p;
  const char* g;
  const float* gs;
  char* m;
  float* ms;
  char* v;
  float* vs;
  char* out;
  float* outs;
  int64_t n;
  int64_t piece0;  // pieces of the tensors of its kind before it
  double decay, lr_scale;
  int8_t pt, gt, ot, state8;
  int8_t lgG, lgS, lgO, pad;
};
static_assert(sizeof(Entry) == 112, "table layout");

// The step's numbers.
struct Coef {
  double lr, rate;  // rate = lr / (1 - b1^t)
  float b1, om1, b2, om2, root, eps, max_norm, scale;
  uint32_t key, pad;
};
static_assert(sizeof(Coef) == 56, "table layout");

// Table: the numbers of a step whose count or rate is on the device, the entries, the
// entry of each piece without blocks and of each with.
constexpr int64_t kEntriesAt = 64;
__host__ __device__ inline int64_t map_at(int entries) { return kEntriesAt + (int64_t)entries * (int64_t)sizeof(Entry); }

// ---------------------------------------------------------------- numbers of a step

// 32 bits to 32 that look drawn: every bit of x reaches every bit of the result (two
// multiplications by odd numbers, shifted halves folded in between).
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0x3B67AE85u;
  return x ^ (x >> 16);
}

__host__ __device__ inline Coef coef_of(const zq_adamw_args& a, int64_t step, double lr) {
  Coef c = {};
  if (step < 1) step = 1;
  c.lr = lr;
  c.rate = lr / (1.0 - pow(a.beta1, (double)step));
  c.b1 = (float)a.beta1;
  c.om1 = (float)(1.0 - a.beta1);
  c.b2 = (float)a.beta2;
  c.om2 = (float)(1.0 - a.beta2);
  c.root = (float)(1.0 / sqrt(1.0 - pow(a.beta2, (double)step)));
  c.eps = (float)a.eps;
  c.max_norm = a.max_norm;
  c.scale = a.scale;
  c.key = mix((uint32_t)step);
  return c;
}

__global__ void k_adamw_numbers(char* __restrict__ table, zq_adamw_args a, const int64_t* __restrict__ step,
                                const float* __restrict__ lr) {
  if (threadIdx.x == 0) *reinterpret_cast<Coef*>(table) = coef_of(a, step ? *step : a.step, lr ? (double)*lr : a.lr);
}

// ---------------------------------------------------------------- 8-bit floats and blocks

// A code's bits are the top of a binary32 number's exponent and mantissa, times a power of
// two: value = number(code << shift) / unit.
template <bool SIGNED>
struct F8 {
  static constexpr int shift = SIGNED ? 20 : 21;
  static constexpr float top = SIGNED ? 448.0f : 57344.0f;
  static constexpr float unit = SIGNED ? 0x1p-120f : 0x1p-112f;
  static constexpr uint32_t last = SIGNED ? 126u : 123u;  // the code of top
};

// 4 codes, exactly
template <bool SIGNED>
__device__ __forceinline__ void decode8(uint32_t w, float (&v)[4]) {
  f32x2_t lo, hi;
  if constexpr (SIGNED) {
    lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  } else {
    lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, false);
    hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, true);
  }
  v[0] = lo.x, v[1] = lo.y, v[2] = hi.x, v[3] = hi.y;
}

// The code of x * r in the top byte of the result.  drawn: 16 bits of m's in the low half of
// a word, of v's in the high half; they are scaled and added below the code in one instruction.
template <bool SIGNED>
__device__ __forceinline__ uint32_t code_on_top(float x, float r, uint32_t drawn) {
  const uint32_t y = f2u((fabsf(x) * r) * F8<SIGNED>::unit);
  uint32_t t;
  if constexpr (SIGNED) asm("v_mad_u32_u16 %0, %1, 16, %2" : "=v"(t) : "v"(drawn), "v"(y));
  else asm("v_mad_u32_u16 %0, %1, 32, %2 op_sel:[1,0,0,0]" : "=v"(t) : "v"(drawn), "v"(y));
  t = (t + (1u << (F8<SIGNED>::shift - 17))) << (24 - F8<SIGNED>::shift);
  t = min(t, F8<SIGNED>::last << 24 | 0xffffffu);
  return SIGNED ? (t & 0x7fffffffu) | (f2u(x) & 0x80000000u) : t;
}
// the top bytes of 4 words, or their lowest
__device__ __forceinline__ uint32_t pack_top(const uint32_t (&t)[4]) {
  return __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0703u) | __builtin_amdgcn_perm(t[3], t[2], 0x07030c0cu);
}
__device__ __forceinline__ uint32_t pack_low(const uint32_t (&t)[4]) {
  return __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0400u) | __builtin_amdgcn_perm(t[3], t[2], 0x04000c0cu);
}

// 32 drawn bits of each of 4 elements from element i on, a multiple of 4: mix(key ^ (i + k)).
// The first product's factors differ in their two lowest bits alone, so 3 of the 4 are the
// first plus or minus the constant and its double (a 32-bit product takes 4 cycles of any other).
__device__ __forceinline__ void draw4(uint32_t key, uint32_t i, uint32_t (&w)[4]) {
  constexpr uint32_t C = 0x6A09E667u;
  uint32_t x = key ^ i;
  x ^= x >> 16;
  const uint32_t d1 = x & 1u ? 0u - C : C, d2 = x & 2u ? 0u - 2u * C : 2u * C;
  w[0] = x * C;
  w[1] = w[0] + d1;
  w[2] = w[0] + d2;
  w[3] = w[1] + d2;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    w[k] ^= w[k] >> 15;
    w[k] *= 0x3B67AE85u;
    w[k] ^= w[k] >> 16;
  }
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kRor4 = 0x124, kRor8 = 0x128;  // lanes of a quad, of 16

// The largest magnitude of the blocks (2^lgB elements, 32 to 1,024) that a lane's elements
// of the 4 steps are in: lane l gets that of step l % 4.  The 4 maxima are reduced side by
// side: each exchange between lanes halves what a lane still has to carry.
__device__ __forceinline__ float block_max(const float (&x)[kSteps][4], int lgB) {
  static_assert(kSteps == 4, "a step for each lane of a quad");
  uint32_t w[4];
#pragma unroll
  for (int u = 0; u < 4; ++u)
    w[u] = f2u(fmaxf(fmaxf(fabsf(x[u][0]), fabsf(x[u][1])), fmaxf(fabsf(x[u][2]), fabsf(x[u][3]))));
  const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
  const uint32_t a = max(odd ? w[1] : w[0], dpp<kSwap1>(odd ? w[0] : w[1]));
  const uint32_t b = max(odd ? w[3] : w[2], dpp<kSwap1>(odd ? w[2] : w[3]));
  uint32_t v = max(high ? b : a, dpp<kSwap2>(high ? a : b));
  if (lgB == 5) return u2f(max(v, (uint32_t)__shfl_xor((int)v, 4, 64)));  // 8 lanes
  v = max(v, dpp<kRor4>(v));
  v = max(v, dpp<kRor8>(v));
  if (lgB >= 7) {
    const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(s[0], s[1]);
  }
  if (lgB >= 8) {
    const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = max(s[0], s[1]);
  }
  if (lgB >= 9) v = max(v, dpp<kSwap1>(v));
  if (lgB >= 10) v = max(v, dpp<kSwap2>(v));
  return u2f(v);
}
// what lane l has of step l % 4, for each step
__device__ __forceinline__ void of_steps(float v, float (&all)[4]) {
  all[0] = u2f(dpp<0x00>(f2u(v)));
  all[1] = u2f(dpp<0x55>(f2u(v)));
  all[2] = u2f(dpp<0xAA>(f2u(v)));
  all[3] = u2f(dpp<0xFF>(f2u(v)));
}
// The scales of a wave's blocks, from lanes that have them as block_max does.  e0: the
// wave's first element.
template <bool FULL>
__device__ __forceinline__ void store_scales(float* scales, float s, int lgB, int64_t e0, int64_t n) {
  const int lane = threadIdx.x & 63, lanes = lgB < 8 ? 1 << (lgB - 2) : 64;
  const int step = lane & 3;
  if ((lane & (lanes - 1)) >= 4 || (lgB > 8 && (step & ((1 << (lgB - 8)) - 1)) != 0)) return;
  const int64_t block = (e0 + step * 256 + lane * 4) >> lgB;
  if (FULL || block << lgB < n) scales[block] = s;
}

// ---------------------------------------------------------------- loads and stores of 4 elements

template <int DT, bool FULL>
__device__ __forceinline__ void load4(const char* base, int64_t i, int64_t n, uint32_t (&w)[4]) {
  constexpr int S = dt_size<DT>();
  if (FULL || i + 4 <= n) {
    uint32_t t[S];
    load_words_any<true>(base + i * S, t);
#pragma unroll
    for (int k = 0; k < S; ++k) w[k] = t[k];
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = 0u;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    if (i + k >= n) continue;
    if constexpr (S == 4) w[k] = reinterpret_cast<const uint32_t*>(base)[i + k];
    else w[k / 2] |= (uint32_t) reinterpret_cast<const uint16_t*>(base)[i + k] << (16 * (k & 1));
  }
}

template <int DT>
__device__ __forceinline__ void widen4(const uint32_t (&w)[4], float (&x)[4]) {
  widen<DT>(w, x);
}

template <int DT, bool FULL>
__device__ __forceinline__ void store4(char* base, int64_t i, int64_t n, const float (&x)[4]) {
  if (FULL || i + 4 <= n) {
    store_elems<DT, 4, true>(base, i, x);
    return;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const float t[1] = {x[k]};
    if (i + k < n) store_elems<DT, 1>(base, i + k, t);
  }
}

// 4 bytes at byte i of n
template <bool FULL>
__device__ __forceinline__ uint32_t load4b(const char* base, int64_t i, int64_t n) {
  if (FULL || i + 4 <= n) return *reinterpret_cast<const u32_any*>(base + i);
  uint32_t w = 0u;
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (i + k < n) w |= (uint32_t)(uint8_t)base[i + k] << (8 * k);
  return w;
}
template <bool FULL>
__device__ __forceinline__ void store4b(char* base, int64_t i, int64_t n, uint32_t w) {
  if (FULL || i + 4 <= n) {
    *reinterpret_cast<u32_any*>(base + i) = w;
    return;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (i + k < n) base[i + k] = (char)(w >> (8 * k));
}

// 4 INT4 codes from element i, a multiple of 4, in the low 16 bits
template <bool FULL>
__device__ __forceinline__ uint32_t load_int4(const char* base, int64_t i, int64_t n) {
  if (FULL || i + 4 <= n) return *reinterpret_cast<const u16_any*>(base + i / 2);
  uint32_t w = 0u;
  if (i < n) w = (uint8_t)base[i / 2];
  if (i + 2 < n) w |= (uint32_t)(uint8_t)base[i / 2 + 1] << 8;
  // the high half of the last byte of an odd count is no code
  return n > i && ((n - i) & 1) ? w & ((1u << (4 * (n - i))) - 1u) : w;
}

// Writes x as 8-bit floats and their blocks' scales.  a / top is a / 7 times a power of two,
// which is a binary32 number or further than 2^-29 of it from the middle of two, so its
// product with 1 / top in binary64, rounded, is the rounded quotient.
template <bool SIGNED, bool FULL>
__device__ __forceinline__ void store_state8(const float (&x)[kSteps][4], const uint32_t (&drawn)[kSteps][4], char* codes,
                                             float* scales, int lgB, int64_t i0, int64_t n) {
  const float a = block_max(x, lgB);
  const bool fits = a >= 0x1p-110f;
  store_scales<FULL>(scales, fits ? (float)((double)a * (1.0 / F8<SIGNED>::top)) : 0.0f, lgB,
                     i0 - (threadIdx.x & 63) * 4, n);
  float r[kSteps];
  of_steps(fits ? F8<SIGNED>::top / a : 0.0f, r);
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    uint32_t t[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) t[k] = code_on_top<SIGNED>(x[u][k], r[u], drawn[u][k]);
    store4b<FULL>(codes, i0 + u * 256, n, pack_top(t));
  }
}

// Writes x as INT8 codes and scales, as the weights' quantiser does: a code is in the low
// byte of x r + 1.5 * 2^23, a / 127 as above.
template <bool FULL>
__device__ __forceinline__ void store_int8(const float (&x)[kSteps][4], char* codes, float* scales, int lgB, int64_t i0,
                                           int64_t n) {
  const float a = block_max(x, lgB);
  const bool fits = a >= 0x1p-119f;
  store_scales<FULL>(scales, fits ? (float)((double)a * (1.0 / 127.0)) : 0.0f, lgB, i0 - (threadIdx.x & 63) * 4, n);
  float r[kSteps];
  of_steps(fits ? 127.0f / a : 0.0f, r);
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    uint32_t t[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) t[k] = f2u(x[u][k] * r[u] + 12582912.0f);
    store4b<FULL>(codes, i0 + u * 256, n, pack_low(t));
  }
}

// ---------------------------------------------------------------- a wave's elements

// BLOCKS: 8-bit moments or an INT8 copy, or both
template <int PT, int GT, bool BLOCKS, bool S8, bool FULL>
__device__ __forceinline__ void update(const Entry& en, const Coef& c, float clip, int tensor, int64_t i0) {
  static_assert(BLOCKS || !S8, "8-bit moments are in blocks");
  constexpr int N = BLOCKS ? kSteps : kPlainSteps;
  const int64_t n = en.n;
  // all loads first
  uint32_t pw[N][4], gw[N][4], mw[N][4], vw[N][4];
  float gs[N], ms[N], vs[N];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int64_t i = i0 + u * 256;
    load4<PT, FULL>(en.p, i, n, pw[u]);
    if constexpr (GT == kInt4) {
      gw[u][0] = load_int4<FULL>(en.g, i, n);
      gs[u] = FULL || i < n ? en.gs[i >> en.lgG] : 0.0f;
    } else {
      load4<GT, FULL>(en.g, i, n, gw[u]);
    }
    if constexpr (S8) {
      mw[u][0] = load4b<FULL>(en.m, i, n);
      vw[u][0] = load4b<FULL>(en.v, i, n);
      ms[u] = FULL || i < n ? en.ms[i >> en.lgS] : 0.0f;
      vs[u] = FULL || i < n ? en.vs[i >> en.lgS] : 0.0f;
    } else {
      load4<ZQ_F32, FULL>(en.m, i, n, mw[u]);
      load4<ZQ_F32, FULL>(en.v, i, n, vw[u]);
    }
  }
  const float alpha = (float)(c.rate * en.lr_scale), decay = (float)(1.0 - c.lr * en.lr_scale * en.decay);

  float p[N][4], m[N][4], v[N][4];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    float g[4];
    widen4<PT>(pw[u], p[u]);
    if constexpr (GT == kInt4) {
      const float s = gs[u] * clip;
#pragma unroll
      for (int k = 0; k < 4; ++k) g[k] = (float)((int32_t)(gw[u][0] << (28 - 4 * k)) >> 28) * s;
    } else {
      widen4<GT>(gw[u], g);
#pragma unroll
      for (int k = 0; k < 4; ++k) g[k] = g[k] * clip;
    }
    float m0[4], v0[4];
    if constexpr (S8) {
      decode8<true>(mw[u][0], m0);
      decode8<false>(vw[u][0], v0);
#pragma unroll
      for (int k = 0; k < 4; ++k) m0[k] = m0[k] * ms[u], v0[k] = v0[k] * vs[u];
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) m0[k] = u2f(mw[u][k]), v0[k] = u2f(vw[u][k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[u][k] = m0[k] * c.b1 + g[k] * c.om1;
      v[u][k] = v0[k] * c.b2 + (g[k] * g[k]) * c.om2;
      const float d = sqrtf(v[u][k]) * c.root + c.eps;
      p[u][k] = p[u][k] * decay - (m[u][k] / d) * alpha;
    }
  }

#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int64_t i = i0 + u * 256;
    store4<PT, FULL>(en.p, i, n, p[u]);
    if constexpr (!S8) {
      store4<ZQ_F32, FULL>(en.m, i, n, m[u]);
      store4<ZQ_F32, FULL>(en.v, i, n, v[u]);
    }
  }
  if constexpr (S8) {
    uint32_t key = mix(c.key + (uint32_t)tensor * 0x9E3779B9u);
    if ((i0 >> 32) != 0) key = mix(key + (uint32_t)(i0 >> 32));  // the same for a piece
    uint32_t drawn[N][4];
#pragma unroll
    for (int u = 0; u < N; ++u) draw4(key, (uint32_t)i0 + (uint32_t)(u * 256), drawn[u]);
    store_state8<true, FULL>(m, drawn, en.m, en.ms, en.lgS, i0, n);
    store_state8<false, FULL>(v, drawn, en.v, en.vs, en.lgS, i0, n);
  }
  if (en.ot == kNone) return;
  if constexpr (PT != ZQ_F32) {  // the copy is of the weight as stored
#pragma unroll
    for (int u = 0; u < N; ++u) {
#pragma unroll
      for (int k = 0; k < 4; ++k) p[u][k] = PT == ZQ_BF16 ? u2f(bf16x2_bits(p[u][k], 0.0f) << 16) : h2f(f2h(p[u][k]));
    }
  }
  if constexpr (BLOCKS) if (en.ot == kInt8) {
    if constexpr (!FULL) {  // what lies behind the end counts in no block
#pragma unroll
      for (int u = 0; u < N; ++u) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i0 + u * 256 + k >= n) p[u][k] = 0.0f;
      }
    }
    store_int8<FULL>(p, en.out, en.outs, en.lgO, i0, n);
    return;
  }
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int64_t i = i0 + u * 256;
    if (en.ot == ZQ_BF16) store4<ZQ_BF16, FULL>(en.out, i, n, p[u]);
    else if (en.ot == ZQ_F16) store4<ZQ_F16, FULL>(en.out, i, n, p[u]);
    else store4<ZQ_F32, FULL>(en.out, i, n, p[u]);
  }
}

template <int PT, int GT, bool BLOCKS>
__device__ __forceinline__ void update_any(const Entry& en, const Coef& c, float clip, int tensor, int64_t i0, bool full) {
  if constexpr (BLOCKS) {
    if (en.state8) {
      if (full) update<PT, GT, true, true, true>(en, c, clip, tensor, i0);
      else update<PT, GT, true, true, false>(en, c, clip, tensor, i0);
      return;
    }
  }
  if (full) update<PT, GT, BLOCKS, false, true>(en, c, clip, tensor, i0);
  else update<PT, GT, BLOCKS, false, false>(en, c, clip, tensor, i0);
}

template <int PT, bool BLOCKS>
__device__ __forceinline__ void update_grad(const Entry& en, const Coef& c, float clip, int tensor, int64_t i0, bool full) {
  switch (en.gt) {
    case ZQ_F32: update_any<PT, ZQ_F32, BLOCKS>(en, c, clip, tensor, i0, full); break;
    case ZQ_F16: update_any<PT, ZQ_F16, BLOCKS>(en, c, clip, tensor, i0, full); break;
    case ZQ_BF16: update_any<PT, ZQ_BF16, BLOCKS>(en, c, clip, tensor, i0, full); break;
    default: update_any<PT, kInt4, BLOCKS>(en, c, clip, tensor, i0, full); break;
  }
}

// With blocks 4 waves a SIMD (128 registers): 453 million elements with 8-bit moments take
// 1,315 us, with the 136 registers that the compiler would take 1,385.
template <bool BLOCKS>
__global__ void __launch_bounds__(kAdamThreads, 4)
    k_adamw(unsigned first, const char* __restrict__ table, const int* __restrict__ entry_of, Coef given, int from_table,
            const float* __restrict__ norm) {
  const unsigned piece = first + blockIdx.x;
  const int tensor = entry_of[piece];
  const Entry en = reinterpret_cast<const Entry*>(table + kEntriesAt)[tensor];
  const Coef c = from_table ? *reinterpret_cast<const Coef*>(table) : given;
  float clip = c.scale;
  if (norm) {
    const float t = *norm;
    if (!(fabsf(t) <= 0x1.fffffep127f)) return;  // infinite or NaN
    const float ratio = c.max_norm / (t + 1e-6f);
    clip = c.scale * (ratio > 1.0f ? 1.0f : ratio);
  }
  constexpr int PIECE = piece_elems(BLOCKS), WAVE = PIECE / (kAdamThreads / 64);
  static_assert(WAVE == (BLOCKS ? kSteps : kPlainSteps) * 256, "a wave's elements");
  const int64_t e0 = ((int64_t)piece - en.piece0) * PIECE;
  const int64_t i0 = e0 + (threadIdx.x >> 6) * WAVE + (threadIdx.x & 63) * 4;
  const bool full = e0 + PIECE <= en.n;
  switch (en.pt) {
    case ZQ_F32: update_grad<ZQ_F32, BLOCKS>(en, c, clip, tensor, i0, full); break;
    case ZQ_F16: update_grad<ZQ_F16, BLOCKS>(en, c, clip, tensor, i0, full); break;
    default: update_grad<ZQ_BF16, BLOCKS>(en, c, clip, tensor, i0, full); break;
  }
}

// ---------------------------------------------------------------- table

bool has_blocks(const zq_adamw& t) { return t.state_dtype == ZQ_F8 || (t.out && t.out_dtype == ZQ_INT8); }
int64_t pieces_of(const zq_adamw& t) {
  const int64_t per = piece_elems(has_blocks(t));
  return (t.n + per - 1) / per;
}

int check(const zq_adamw& t) {
  if (t.n < 0 || t.n > INT64_MAX / 16) return ZQ_E_SIZE;
  const bool int4 = t.grad_dtype == ZQ_INT4, s8 = t.state_dtype == ZQ_F8, int8 = t.out_dtype == ZQ_INT8;
  if (!dtype_ok(t.param_dtype) || !(int4 || dtype_ok(t.grad_dtype)) || !(s8 || t.state_dtype == ZQ_F32)) return ZQ_E_DTYPE;
  if (t.out && !(int8 || dtype_ok(t.out_dtype))) return ZQ_E_DTYPE;
  if ((int4 && log2_block(t.grad_block) < 0) || (s8 && log2_block(t.state_block) < 0)) return ZQ_E_BLOCK;
  if (t.out && int8 && log2_block(t.out_block) < 0) return ZQ_E_BLOCK;
  if (!std::isfinite(t.weight_decay) || !std::isfinite(t.lr_scale)) return ZQ_E_SIZE;
  if (t.n == 0) return ZQ_OK;
  if (!t.param || !t.grad || !t.m || !t.v || (int4 && !t.grad_scales) || (s8 && (!t.m_scales || !t.v_scales))) return ZQ_E_NULL;
  if (t.out && int8 && !t.out_scales) return ZQ_E_NULL;
  if (!aligned(t.param, elem_bytes(t.param_dtype)) || (!int4 && !aligned(t.grad, elem_bytes(t.grad_dtype)))) return ZQ_E_ALIGN;
  if (int4 && !aligned(t.grad_scales, 4)) return ZQ_E_ALIGN;
  if (s8 ? !aligned(t.m_scales, 4) || !aligned(t.v_scales, 4) : !aligned(t.m, 4) || !aligned(t.v, 4)) return ZQ_E_ALIGN;
  if (t.out && (int8 ? !aligned(t.out_scales, 4) : !aligned(t.out, elem_bytes(t.out_dtype)))) return ZQ_E_ALIGN;
  return ZQ_OK;
}

int check_overlaps(const zq_adamw* tensors, int32_t count) {
  std::vector<Span> spans;
  spans.reserve(9 * (size_t)count);
  for (int32_t i = 0; i < count; ++i) {
    const zq_adamw& t = tensors[i];
    const int64_t n = t.n;
    const bool s8 = t.state_dtype == ZQ_F8;
    put_span(spans, t.param, n * elem_bytes(t.param_dtype), true);
    if (t.grad_dtype == ZQ_INT4) {
      put_span(spans, t.grad, (n + 1) / 2, false);
      put_span(spans, t.grad_scales, 4 * num_scales(n, t.grad_block), false);
    } else {
      put_span(spans, t.grad, n * elem_bytes(t.grad_dtype), false);
    }
    put_span(spans, t.m, s8 ? n : 4 * n, true);
    put_span(spans, t.v, s8 ? n : 4 * n, true);
    if (s8) {
      put_span(spans, t.m_scales, 4 * num_scales(n, t.state_block), true);
      put_span(spans, t.v_scales, 4 * num_scales(n, t.state_block), true);
    }
    if (t.out && t.out_dtype == ZQ_INT8) {
      put_span(spans, t.out, n, true);
      put_span(spans, t.out_scales, 4 * num_scales(n, t.out_block), true);
    } else if (t.out) {
      put_span(spans, t.out, n * elem_bytes(t.out_dtype), true);
    }
  }
  return check_spans(spans);
}

Entry entry_for(const zq_adamw& t) {
  Entry e = {};
  const bool int4 = t.grad_dtype == ZQ_INT4, s8 = t.state_dtype == ZQ_F8, int8 = t.out && t.out_dtype == ZQ_INT8;
  e.p = static_cast<char*>(t.param);
  e.g = static_cast<const char*>(t.grad);
  e.gs = t.grad_scales;
  e.m = static_cast<char*>(t.m);
  e.ms = t.m_scales;
  e.v = static_cast<char*>(t.v);
  e.vs = t.v_scales;
  e.out = static_cast<char*>(t.out);
  e.outs = t.out_scales;
  e.n = t.n;
  e.decay = t.weight_decay;
  e.lr_scale = t.lr_scale;
  e.pt = (int8_t)t.param_dtype;
  e.gt = (int8_t)(int4 ? kInt4 : t.grad_dtype);
  e.ot = (int8_t)(!t.out ? kNone : int8 ? kInt8 : t.out_dtype);
  e.state8 = s8;
  e.lgG = (int8_t)(int4 ? log2_block(t.grad_block) : 0);
  e.lgS = (int8_t)(s8 ? log2_block(t.state_block) : 0);
  e.lgO = (int8_t)(int8 ? log2_block(t.out_block) : 0);
  return e;
}

int plan_table(const zq_adamw* tensors, int32_t count, zq_adamw_plan* plan) {
  if (!plan || (count > 0 && !tensors)) return ZQ_E_NULL;
  if (count < 0) return ZQ_E_SIZE;
  zq_adamw_plan p = {};
  p.count = count;
  for (int32_t i = 0; i < count; ++i) {
    const int rc = check(tensors[i]);
    if (rc != ZQ_OK) return rc;
    (has_blocks(tensors[i]) ? p.block_pieces : p.pieces) += pieces_of(tensors[i]);
    if (p.pieces > kMaxGrid || p.block_pieces > kMaxGrid) return ZQ_E_SIZE;
  }
  const int rc = check_overlaps(tensors, count);
  if (rc != ZQ_OK) return rc;
  p.bytes = map_at(count) + 4 * (p.pieces + p.block_pieces);
  *plan = p;
  return ZQ_OK;
}

}  // namespace
}  // namespace zq

extern "C" {

using namespace zq;

int zq_adamw_plan_make(const zq_adamw* tensors, int32_t count, zq_adamw_plan* plan) {
  try {
    return plan_table(tensors, count, plan);
  } catch (...) {  // more tensors than the host has memory to check for overlaps
    return ZQ_E_SIZE;
  }
}

int zq_adamw_plan_table(const zq_adamw* tensors, const zq_adamw_plan* plan, void* host_table) {
  if (!plan || !host_table || (plan->count > 0 && !tensors)) return ZQ_E_NULL;
  char* t = static_cast<char*>(host_table);
  std::fill(t, t + kEntriesAt, (char)0);
  Entry* entries = reinterpret_cast<Entry*>(t + kEntriesAt);
  int* map = reinterpret_cast<int*>(t + map_at(plan->count));
  int64_t at[2] = {0, 0};
  for (int32_t i = 0; i < plan->count; ++i) {
    const bool blocks = has_blocks(tensors[i]);
    entries[i] = entry_for(tensors[i]);
    entries[i].piece0 = at[blocks];
    const int64_t pieces = pieces_of(tensors[i]);
    int* of = map + (blocks ? plan->pieces : 0) + at[blocks];
    std::fill(of, of + pieces, i);
    at[blocks] += pieces;
  }
  return ZQ_OK;
}

int zq_adamw_step(const zq_adamw_plan* plan, void* table, const zq_adamw_args* args, const int64_t* step,
                  const float* lr, const float* norm, void* stream) {
  if (!plan || !table || !args) return ZQ_E_NULL;
  if (!aligned(table, 16) || (step && !aligned(step, 8)) || (lr && !aligned(lr, 4)) || (norm && !aligned(norm, 4)))
    return ZQ_E_ALIGN;
  const auto share = [](double b) { return b >= 0.0 && b < 1.0; };
  if (!share(args->beta1) || !share(args->beta2) || !(args->eps >= 0.0) || (!step && args->step < 1) ||
      (!lr && !std::isfinite(args->lr)) || (norm && !(args->max_norm >= 0.0f)))
    return ZQ_E_SIZE;
  if (plan->pieces == 0 && plan->block_pieces == 0) return ZQ_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  Coef c = {};
  if (step || lr) {
    const int rc = launch(&k_adamw_numbers, 1u, 64u, st, static_cast<char*>(table), *args, step, lr);
    if (rc != ZQ_OK) return rc;
  } else {
    c = coef_of(*args, args->step, args->lr);
  }
  const char* t = static_cast<const char*>(table);
  const int* map = reinterpret_cast<const int*>(t + map_at(plan->count));
  const int from_table = step || lr ? 1 : 0;
  const int rc = launch_parts(&k_adamw<false>, plan->pieces, kAdamThreads, st, t, map, c, from_table, norm);
  if (rc != ZQ_OK) return rc;
  return launch_parts(&k_adamw<true>, plan->block_pieces, kAdamThreads, st, t, map + plan->pieces, c, from_table, norm);
}

}  // extern "C"
