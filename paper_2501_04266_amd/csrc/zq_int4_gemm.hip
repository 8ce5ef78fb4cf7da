// zq_int4_gemm.hip -- products of a few rows with a weight held as INT4 codes
// and block scales, for gfx950 MFMA.
//
//   y[m][n] = sum_k x[m][k] * q[n][k] * s[(n K + k) / B]
//
// The weight is streamed once: a wave loads 16 bytes (32 codes) a lane, turns
// them into bf16 / fp16 values q / 16 in registers (exact: 4 bits of
// significand) and multiplies on 16 x 16 x 32 MFMAs.  The sums over a block's
// codes stay apart from its scale, which multiplies them in binary32: no
// weight is rounded.  The factor 16 goes into the finished sum.
//
// A workgroup of W waves takes 16 NT weight rows and all of K, the waves 256
// codes a row in turn (whole 128-byte lines); their partial sums are added in
// LDS in the order of the waves.  x passes through LDS, a range of K at a time.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "zq.h"
#include "zq_device.h"
#include "zq_host.h"

#pragma clang fp contract(off)

namespace zq {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef __fp16 fp16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// buffer resource word 3 for raw (untyped) buffer loads on gfx9-family targets
constexpr int kRawBuffer = 0x00020000;
constexpr uint32_t kOutside = 0x7fff0000u;  // an offset past every resource: reads zeros

template <int XT>
__device__ __forceinline__ f32x4_t mfma(u32x4 a, u32x4 b, f32x4_t c) {
  if constexpr (XT == ZQ_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0,
                                                  0, 0);
}

// q / 16 for the low nibble (two's complement) of byte BYTE of w: one
// instruction, exact
template <int BYTE>
__device__ __forceinline__ float sixteenth(uint32_t w) {
  float f;
  if constexpr (BYTE == 0)
    asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(f) : "v"(w));
  else if constexpr (BYTE == 1)
    asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(f) : "v"(w));
  else if constexpr (BYTE == 2)
    asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(f) : "v"(w));
  else
    asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(f) : "v"(w));
  return f;
}

// two values of at most 8 significant bits as XT, packed low-first (exact)
template <int XT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (XT == ZQ_BF16) return __builtin_amdgcn_perm(f2u(b), f2u(a), 0x07060302u);
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
}

// the 8 codes of a word as an MFMA operand, in sixteenths
template <int XT>
__device__ __forceinline__ u32x4 operand(uint32_t w) {
  const uint32_t h = w >> 4;
  return u32x4{pack2<XT>(sixteenth<0>(w), sixteenth<0>(h)), pack2<XT>(sixteenth<1>(w), sixteenth<1>(h)),
               pack2<XT>(sixteenth<2>(w), sixteenth<2>(h)), pack2<XT>(sixteenth<3>(w), sixteenth<3>(h))};
}

// Lane (c, g) (c = lane % 16, g = lane / 16) holds words 0 .. 3 of its 16 bytes:
// word j of lane (c, g) becomes word g of lane (c, j).  A 4 x 4 transposition
// between the quarters of the wave, so that MFMA j reads 32 codes in a row.
__device__ __forceinline__ u32x4 transposed(u32x4 w) {
  auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
  auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
  auto p = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
  auto q = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  return u32x4{p[0], p[1], q[0], q[1]};
}

// MT, NT: 16-row tiles of x and of the weight; W: waves; D: pieces (256 codes of
// each of the wave's rows) in flight; G: codes summed before their scale is
// applied (they lie in one block).  `range`: codes of K whose x is in LDS at a
// time, those of `per` rounds of the waves, or all of K.
template <int XT, int MT, int NT, int W, int D, int G>
__global__ void __launch_bounds__(64 * W)
    k_int4_rows(const uint16_t* __restrict__ x, const uint8_t* __restrict__ packed, const float* __restrict__ scales,
                int64_t M, int64_t N, int64_t K, int lgB, int range, int per,
                float* __restrict__ y) {
  extern __shared__ u32x4 lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * (16 * NT), m0 = (int64_t)blockIdx.y * (16 * MT);
  const int rows = (int)(N - n0 < 16 * NT ? N - n0 : 16 * NT);
  const int mrows = (int)(M - m0 < 16 * MT ? M - m0 : 16 * MT);
  const int kk = (int)K;
  const __amdgpu_buffer_rsrc_t wres = __builtin_amdgcn_make_buffer_rsrc(
      (void*)(packed + n0 * (K / 2)), (short)0, rows * (kk / 2), kRawBuffer);
  const int64_t s0 = (n0 * K) >> lgB, s1 = ((n0 + rows) * K + (1 << lgB) - 1) >> lgB;
  const __amdgpu_buffer_rsrc_t sres =
      __builtin_amdgcn_make_buffer_rsrc((void*)(scales + s0), (short)0, (int)((s1 - s0) * 4), kRawBuffer);
  const uint32_t fbase = (uint32_t)((n0 * K) & ((1ll << lgB) - 1));  // of the first row in its block

  constexpr int SC = 256 / G;  // scales of a row's piece
  const int pieces = (kk + 255) / 256;
  u32x4 wr[D][NT][2];
  float sr[D][NT][SC];
  auto load = [&](int d, int piece) {
    const int k0 = piece * 256;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int row = 16 * t + c;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = k0 + 128 * h + 32 * g;
        const uint32_t off = k < kk && row < rows ? (uint32_t)(row * (kk / 2) + k / 2) : kOutside;
        wr[d][t][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(wres, (int)off, 0, 0));
      }
#pragma unroll
      for (int q = 0; q < SC; ++q) {
        const int k = k0 + G * q;
        const uint32_t off =
            k < kk && row < rows ? (((uint32_t)row * (uint32_t)kk + (uint32_t)k + fbase) >> lgB) * 4 : kOutside;
        sr[d][t][q] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(sres, (int)off, 0, 0));
      }
    }
  };
  // x[m0 ..][k0 .. k0 + range) into LDS, rows 16 bytes apart beyond their length
  // (so that 8 lanes' 16-byte reads of one column fall into distinct banks)
  const int stride = range / 8 + 1;
  auto stage = [&](int k0) {
    const int len = (kk - k0 < range ? kk - k0 : range) / 8;
    for (int m = wave; m < mrows; m += W) {
      const uint16_t* row = x + (m0 + m) * K + k0;
      for (int i = lane; i < len; i += 64) lds[m * stride + i] = *reinterpret_cast<const u32x4*>(row + 8 * i);
      // what the last, half step of K multiplies with zero codes
      if (len * 8 < range)
        for (int i = len + lane; i < len + 32 && i < range / 8; i += 64) lds[m * stride + i] = u32x4{0u, 0u, 0u, 0u};
    }
  };

  f32x4_t acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[i][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  int xrow[MT];  // rows past M repeat the last one; their sums are not stored
#pragma unroll
  for (int i = 0; i < MT; ++i) xrow[i] = (16 * i + c < mrows ? 16 * i + c : mrows - 1) * stride + g;

  auto multiply = [&](int d, int k0) {  // k0: in the staged range
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 wt[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) wt[t] = transposed(wr[d][t][h]);
      f32x4_t part[MT][NT];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u32x4 xf[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) xf[i] = lds[xrow[i] + (k0 + 128 * h + 32 * j) / 8];
        const bool first = (32 * j) % G == 0, done = (32 * j + 32) % G == 0;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const u32x4 wf = operand<XT>(wt[t][j]);
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            part[i][t] = mfma<XT>(xf[i], wf, first ? f32x4_t{0.0f, 0.0f, 0.0f, 0.0f} : part[i][t]);
            if (done) {
              const float s = sr[d][t][(128 * h + 32 * j) / G];
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][t][e] = __builtin_fmaf(part[i][t][e], s, acc[i][t][e]);
            }
          }
        }
      }
    }
  };

  const int rounds = (pieces + W - 1) / W;
#pragma unroll
  for (int d = 0; d < D; ++d) load(d, d * W + wave);
  for (int r0 = 0; r0 < rounds; r0 += D) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const int r = r0 + d;
      if (r < rounds) {
        if (r % per == 0) {
          if (r > 0) __syncthreads();
          stage(r * W * 256);
          __syncthreads();
        }
        const int k0 = (r * W + wave) * 256;
        if (k0 < kk) multiply(d, k0 - r / per * per * (256 * W));
        load(d, (r + D) * W + wave);
      }
    }
  }

  // the waves' sums, in the order of the waves; D element e of lane (c, g): row
  // 4 g + e of x, weight row c
  __syncthreads();
  float* part = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        part[((wave * MT + i) * 16 + 4 * g + e) * (16 * NT) + 16 * t + c] = acc[i][t][e];
  __syncthreads();
  for (int o = threadIdx.x; o < 256 * MT * NT; o += 64 * W) {
    const int m = o / (16 * NT), n = o % (16 * NT);
    if (m >= mrows || n >= rows) continue;
    float v = 0.0f;
    for (int w = 0; w < W; ++w) v += part[(w * MT * 16 + m) * (16 * NT) + n];
    y[(m0 + m) * N + n0 + n] = 16.0f * v;
  }
}

using Int4Kernel = void (*)(const uint16_t*, const uint8_t*, const float*, int64_t, int64_t, int64_t, int, int, int,
                            float*);

template <int XT, int MT, int NT, int W, int D>
Int4Kernel int4_kernel_for(int G) {
  return G == 128  ? &k_int4_rows<XT, MT, NT, W, D, 128>
         : G == 64 ? &k_int4_rows<XT, MT, NT, W, D, 64>
                   : &k_int4_rows<XT, MT, NT, W, D, 32>;
}

constexpr int64_t kInt4MaxK = 1 << 22;  // 64 rows of codes stay below 2^31 bytes
constexpr int kInt4Waves = 8;

}  // namespace
}  // namespace zq

extern "C" int zq_int4_dequant_gemm(const void* x, zq_dtype xt, const uint8_t* packed, const float* scales, int64_t M,
                                    int64_t N, int64_t K, int32_t block, float* y, void* stream) {
  using namespace zq;
  if (M < 0 || N < 0 || K < 0 || K % 64 != 0 || K > kInt4MaxK) return ZQ_E_SIZE;
  const int lgB = log2_block(block);
  if (lgB < 0) return ZQ_E_BLOCK;
  if (xt != ZQ_BF16 && xt != ZQ_F16) return ZQ_E_DTYPE;
  if (M == 0 || N == 0) return ZQ_OK;
  if (!y || (K > 0 && (!x || !packed || !scales))) return ZQ_E_NULL;
  if (!aligned(x, 16) || !aligned(packed, 16) || !aligned(scales, 4) || !aligned(y, 4)) return ZQ_E_ALIGN;
  if (N > INT64_MAX / 8 / (K + 1) || M > INT64_MAX / 8 / (K + 1) || M > INT64_MAX / 8 / N) return ZQ_E_SIZE;
  if (any_overlap({{y, 4 * M * N}}, {{x, 2 * M * K}, {packed, N * K / 2}, {scales, 4 * num_scales(N * K, block)}}))
    return ZQ_E_ALIAS;

  constexpr int W = kInt4Waves;
  const int MT = 1, NT = 1;
  const int G = block >= 128 && K % 128 == 0 ? 128 : block >= 64 ? 64 : 32;
  const int64_t mrows = M < 16 * MT ? M : 16 * MT;
  // all of K in LDS where it fits 64 KiB, else whole rounds of it
  int64_t range = (K + 255) / 256 * 256, per = (K + 256 * W - 1) / (256 * W);
  if (mrows * (2 * range + 16) > 65536) {
    per = (65536 / mrows - 16) / 2 / (256 * W);
    if (per < 1) per = 1;
    range = per * 256 * W;
  }
  int64_t lds = mrows * (2 * range + 16);
  if (lds < 4 * 256 * MT * NT * W) lds = 4 * 256 * MT * NT * W;
  const int64_t grid = (N + 16 * NT - 1) / (16 * NT), gridm = (M + 16 * MT - 1) / (16 * MT);
  if (grid > kMaxGrid || gridm > 65535) return ZQ_E_SIZE;
  Int4Kernel k = xt == ZQ_BF16 ? int4_kernel_for<ZQ_BF16, 1, 1, W, 3>(G) : int4_kernel_for<ZQ_F16, 1, 1, W, 3>(G);
  return launch_grid(k, dim3((unsigned)grid, (unsigned)gridm), 64u * W, (unsigned)lds, static_cast<hipStream_t>(stream),
                   static_cast<const uint16_t*>(x), packed, scales, M, N, K, lgB, (int)range, (int)per, y);
}
