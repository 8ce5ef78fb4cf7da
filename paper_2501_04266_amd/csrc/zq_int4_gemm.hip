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
// A workgroup of 8 waves takes 16 weight rows at a time (or some times 16), its
// waves 256 codes a row in turn (whole 128-byte lines) over a slice of K, which
// is all of K unless x or the grid asks for less; the waves' sums are added in
// LDS in the order of the waves, the slices' sums in a second launch.
//
// What bounds it: the weight's bytes where they are many and the rows of x few
// (5 rows, 50,001 x 6,144: 37 us, 4.5 TB/s of the 6.4 of a plain copy; 16 rows,
// 40,000 x 6,144: 38 us), close behind it the instructions that turn codes into
// operands (about 330 cycles of a SIMD for 2,048 codes: 13 a word for 8 codes,
// the moves between lanes, the addresses).  Up to about 8 MiB of weight a launch
// and one round of loads take longer than its bytes: 6 to 8 us.  With more than
// 16 rows the conversion and x bind, which k_int4_wide shares in LDS (64 rows,
// 24,576 x 6,144: 50 us).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "zq.h"
#include "zq_device.h"
#include "zq_host.h"
#include "zq_int4_plan.h"

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

// q / 16 for the low nibble (two's complement) of byte BYTE of w: one instruction,
// exact.  The builtin and no inline asm: the compiler has to know of these writes to
// keep them off the registers that an MFMA still in flight will write.
template <int BYTE>
__device__ __forceinline__ float sixteenth(uint32_t w) {
  return __builtin_amdgcn_cvt_off_f32_i4((int)(w >> (8 * BYTE) & 0xffu));
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
  uint32_t h = w >> 4;
  asm("" : "+v"(h));  // one shift: left to itself the compiler takes each upper nibble out of w by one of its own
  return u32x4{pack2<XT>(sixteenth<0>(w), sixteenth<0>(h)), pack2<XT>(sixteenth<1>(w), sixteenth<1>(h)),
               pack2<XT>(sixteenth<2>(w), sixteenth<2>(h)), pack2<XT>(sixteenth<3>(w), sixteenth<3>(h))};
}

// v of another lane
__device__ __forceinline__ uint32_t from_lane(int lane, uint32_t v) {
  return (uint32_t)__builtin_amdgcn_ds_bpermute(4 * lane, (int)v);
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

// The part of K that a workgroup sums over: slices of `each` (a multiple of kPiece)
// codes by blockIdx.z, the sums of slice z in plane z of `y` (M x N each).
struct Slice {
  int from, count;
  __device__ __forceinline__ Slice(int64_t K, int each) {
    from = (int)blockIdx.z * each;
    count = (int)K - from < each ? (int)K - from : each;
  }
};

// The weight as a wave streams it.  A load takes half a piece (128 codes) of 16 rows:
// lane l has 32 codes of row l / 4, from code 32 (l % 4) on, so that 4 lanes in a row
// read 64 bytes in a row (with a row for each of 16 lanes in a row the same loads take
// four times as long in the address unit), and the scale of those codes, which lie in
// one block.  Slots of D pieces of NT x 16 rows are in flight.
template <int T, int S>
struct Weight {
  u32x4 codes[S][2];
  float scale[S][2];

  const uint8_t* packed;
  const float* scales;
  int64_t N, K;
  int lgB, groups;
  // of the group being loaded
  __amdgpu_buffer_rsrc_t wres, sres;
  uint32_t first;  // its first row's place in its block
  uint32_t row0;   // this lane's first code, in the group's flat order
  int end;         // pieces of the slice that start before this have codes for the lane

  __device__ __forceinline__ Weight(const uint8_t* p, const float* s, int64_t n, int64_t k, Slice sl, int lg, int gr)
      : packed(p), scales(s), N(n), K(k), lgB(lg), groups(gr) {
    const int lane = threadIdx.x & 63;
    row0 = (uint32_t)(lane >> 2) * (uint32_t)k + (uint32_t)sl.from + 32u * (lane & 3);
    end = sl.count - 32 * (lane & 3);
  }
  __device__ __forceinline__ void turn_to(int group) {
    // past the last group: empty resources; the same loads go out, so that the number
    // of loads in flight is known at every wait, and bring zeros
    const bool any = group < groups;
    const int64_t n0 = any ? (int64_t)group * (16 * T) : 0;
    const int rows = any ? (int)(N - n0 < 16 * T ? N - n0 : 16 * T) : 0;
    wres = __builtin_amdgcn_make_buffer_rsrc((void*)(packed + n0 * (K / 2)), (short)0, rows * (int)(K / 2), kRawBuffer);
    const int64_t f0 = n0 * K, s0 = f0 >> lgB, s1 = (f0 + (int64_t)rows * K + (1 << lgB) - 1) >> lgB;
    sres = __builtin_amdgcn_make_buffer_rsrc((void*)(scales + s0), (short)0, (int)((s1 - s0) * 4), kRawBuffer);
    first = (uint32_t)(f0 & ((1ll << lgB) - 1));
  }
  // half h of the piece from code k0 of the slice on of the group's tile t, into slot s; rows
  // past the last, and codes past the slice, are outside the resources: zeros
  __device__ __forceinline__ void load(int s, int h, int t, uint32_t k0) {
    const uint32_t f = row0 + 16 * t * (uint32_t)K + k0;
    const bool in = (int)k0 < end - 128 * h;
    const uint32_t off = in ? f / 2 + 64u * h : kOutside;
    codes[s][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(wres, (int)off, 0, 0));
    const uint32_t soff = in ? ((f + first + 128u * h) >> lgB) * 4 : kOutside;
    scale[s][h] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(sres, (int)soff, 0, 0));
  }
};

// A slice of x rows m0 .. m0 + mrows in LDS, whole; elements past it, which meet zero codes, are
// zeros.  Rows are an odd number of 16-byte units long, so that lanes that read one
// column of 8 rows meet distinct banks.  `between` runs once the first loads are out.
// What there is no place for goes to the unit after the last row: a load whose result
// is left in its registers makes the compiler wait for all loads wherever these are
// used again, in each turn of the loops below.
template <typename F>
__device__ __forceinline__ void stage_x(u32x4* lds, __amdgpu_buffer_rsrc_t xres, int mrows, int64_t K, Slice sl,
                                        F between) {
  constexpr int U = 4;
  const int stride = x_stride(sl.count);
  const unsigned row = (unsigned)stride - 1, units = (unsigned)mrows * row;  // 16-byte units: below 2^14
  // a unit's row: the quotient is a half over the row length or more away from the next
  // whole number, the product off by 2^-23 of it
  const float inv = 1.0f / (float)row;
  auto row_of = [&](unsigned i) { return (unsigned)(((float)i + 0.5f) * inv); };
  u32x4 v[U];
  auto read = [&](unsigned at) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const unsigned i = at + u * kGemmThreads, m = row_of(i), k = 8 * (i - m * row);
      const uint32_t off =
          i < units && k < (unsigned)sl.count ? (m * (unsigned)K + (unsigned)sl.from + k) * 2 : kOutside;
      v[u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xres, (int)off, 0, 0));
    }
  };
  auto write = [&](unsigned at) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const unsigned i = at + u * kGemmThreads;
      lds[i < units ? i + row_of(i) : (unsigned)(mrows * stride)] = v[u];
    }
  };
  read(threadIdx.x);
  between();
  write(threadIdx.x);
  for (unsigned at = threadIdx.x + U * kGemmThreads; at < units; at += U * kGemmThreads) {
    read(at);
    write(at);
  }
}

// ---------------------------------------------------------------- few rows of x
//
// The transposed words of a half piece make 4 operands w of 16 columns: column c is row
// 4 w + c / 4 of the weight and its codes 32 (c % 4) .. + 32.  The other operand holds 4
// rows of x for each of the four ranges of codes: row 4 s + m is x[m] at 32 s .. + 32.  Of
// the product's 16 x 16 sums those with s = c % 4 count, a quarter: lane (c, g) has them,
// elements m, where g = c % 4.  The matrix cores have room for that (16 cycles of about
// 150 per operand), and no lane needs codes that another one loaded, beyond the
// transposition.  Each column has one scale, whatever the block size.  Two pieces in
// flight (3 and 4 measured no faster).  One row, 18,432 x 6,144: 16 us; 24,576 x 6,144:
// 20 us, 4.0 TB/s; 6,144 x 24,576: 24 us.
// MR: rows of x, 1, 2 or 4.
template <int XT, int MR, int D>
__global__ void __launch_bounds__(kGemmThreads)
    k_int4_few(const uint16_t* __restrict__ x, const uint8_t* __restrict__ packed, const float* __restrict__ scales,
               int64_t M, int64_t N, int64_t K, int each, int lgB, int groups, float* __restrict__ y) {
  extern __shared__ u32x4 lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15;
  const int g = lane >> 4;
  const Slice sl(K, each);
  const int mrows = (int)M, stride = x_stride(sl.count);
  const int rounds = (pieces_of(sl.count) + kWaves - 1) / kWaves;
  y += blockIdx.z * (M * N);
  Weight<1, D> wt(packed, scales, N, K, sl, lgB, groups);
  int load_group = blockIdx.x, load_round = 0;
  wt.turn_to(load_group);
  auto load = [&](int d) {
    const uint32_t k0 = (uint32_t)((load_round * kWaves + wave) * kPiece);
    wt.load(d, 0, 0, k0), wt.load(d, 1, 0, k0);
    if (++load_round == rounds) load_round = 0, wt.turn_to(load_group += gridDim.x);
  };
  const __amdgpu_buffer_rsrc_t xres =
      __builtin_amdgcn_make_buffer_rsrc((void*)x, (short)0, mrows * (int)K * 2, kRawBuffer);
  stage_x(lds, xres, mrows, K, sl, [&] {
#pragma unroll
    for (int d = 0; d < D; ++d) load(d);
  });
  // rows past M repeat the last one; their sums are not stored
  const u32x4* const xat = lds + ((lane & 3) < mrows ? lane & 3 : mrows - 1) * stride + 4 * (c >> 2) + g;

  float acc[4][MR];
  auto clear = [&] {
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int m = 0; m < MR; ++m) acc[w][m] = 0.0f;
  };
  auto multiply = [&](int d, int h, int k0) {
    const u32x4 xf = xat[k0 / 8];
    const u32x4 words = transposed(wt.codes[d][h]);
    float s[4];  // the scale of lane 16 w + c
#pragma unroll
    for (int w = 0; w < 4; ++w)
      s[w] = u2f(from_lane(16 * w + c, f2u(wt.scale[d][h])));
    f32x4_t part[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) part[w] = mfma<XT>(xf, operand<XT>(words[w]), f32x4_t{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int m = 0; m < MR; ++m) acc[w][m] = __builtin_fmaf(part[w][m], s[w], acc[w][m]);
  };

  float* const sums = reinterpret_cast<float*>(lds + mrows * stride);
  constexpr int kOne = few_sums(MR);
  int group = blockIdx.x, round = 0, turn = 0;
  auto finish = [&] {
    float* const part = sums + turn * (kWaves * kOne);
    if (g == (c & 3)) {
#pragma unroll
      for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int w = 0; w < 4; ++w) part[wave * kOne + (g * MR + m) * 16 + 4 * w + (c >> 2)] = acc[w][m];
    }
    __syncthreads();
    const int64_t n = (int64_t)group * 16 + (threadIdx.x & 15);
    const int m = threadIdx.x >> 4;
    if (m < mrows && n < N) {
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int s = 0; s < 4; ++s) v += part[w * kOne + s * MR * 16 + threadIdx.x];
      y[m * N + n] = 16.0f * v;
    }
    turn ^= 1;  // the next group's sums go beside these, which may still be read
    clear();
  };

  clear();
  __syncthreads();
  // The D steps have one way out, after the last: with one after each the compiler
  // waits for all loads in every turn.  Steps past the last group multiply zeros.
  do {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const int k0 = (round * kWaves + wave) * kPiece;
      if (k0 < sl.count) multiply(d, 0, k0), multiply(d, 1, k0 + 128);
      load(d);
      if (++round == rounds) {
        if (group < groups) finish();
        round = 0;
        group += gridDim.x;
      }
    }
  } while (group < groups);
}

// ---------------------------------------------------------------- 5 to 16 rows
//
// All of x, or a slice, is in LDS from before the first group of 16 weight rows on, and
// the workgroups that are resident at once share the groups.  The codes and scales go to
// the lanes that need them through LDS (permutations of the wave): lane (c, g) takes the
// 32 codes of row c from 32 g on.  (Loads that bring them there directly, a row to each
// of 16 lanes in a row, take longer in the address unit: 76 us for 5 rows of 50,001 x
// 6,144, 35 this way.)
// G: codes summed before their scale is applied (they lie in one block).
template <int XT, int D, int G>
__global__ void __launch_bounds__(kGemmThreads)
    k_int4_lds(const uint16_t* __restrict__ x, const uint8_t* __restrict__ packed, const float* __restrict__ scales,
               int64_t M, int64_t N, int64_t K, int each, int lgB, int groups, float* __restrict__ y) {
  extern __shared__ u32x4 lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15;
  const int g = lane >> 4;
  const Slice sl(K, each);
  const int mrows = (int)M, stride = x_stride(sl.count);
  const int rounds = (pieces_of(sl.count) + kWaves - 1) / kWaves;
  y += blockIdx.z * (M * N);
  Weight<1, D> wt(packed, scales, N, K, sl, lgB, groups);
  int load_group = blockIdx.x, load_round = 0;
  wt.turn_to(load_group);
  auto load = [&](int d) {
    const uint32_t k0 = (uint32_t)((load_round * kWaves + wave) * kPiece);
    wt.load(d, 0, 0, k0), wt.load(d, 1, 0, k0);
    if (++load_round == rounds) load_round = 0, wt.turn_to(load_group += gridDim.x);
  };
  const __amdgpu_buffer_rsrc_t xres =
      __builtin_amdgcn_make_buffer_rsrc((void*)x, (short)0, mrows * (int)K * 2, kRawBuffer);
  stage_x(lds, xres, mrows, K, sl, [&] {
#pragma unroll
    for (int d = 0; d < D; ++d) load(d);
  });
  // Lane (c, g) multiplies in MFMA j of a half piece elements 32 g + 8 j on, where the
  // codes may stay as they are loaded; else, with the words transposed, 32 j + 8 g on.
  constexpr bool kAsLoaded = G == 128;
  constexpr int XG = kAsLoaded ? 32 : 8, XJ = kAsLoaded ? 8 : 32;
  // rows past M repeat the last one; their sums are not stored
  const u32x4* const xat = lds + (c < mrows ? c : mrows - 1) * stride + XG * g / 8;

  f32x4_t acc;
  auto multiply = [&](int d, int h, int k0) {  // half h of the piece in slot d; k0: its first code
    u32x4 xf[4], words;
#pragma unroll
    for (int j = 0; j < 4; ++j) xf[j] = xat[(k0 + XJ * j) / 8];
#pragma unroll
    for (int q = 0; q < 4; ++q) words[q] = from_lane(4 * c + g, wt.codes[d][h][q]);
    if constexpr (!kAsLoaded) words = transposed(words);
    float s[128 / G];
#pragma unroll
    for (int q = 0; q < 128 / G; ++q) s[q] = u2f(from_lane(4 * c + q * (G / 32), f2u(wt.scale[d][h])));
    f32x4_t part;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool first = (32 * j) % G == 0, done = (32 * j + 32) % G == 0;
      part = mfma<XT>(xf[j], operand<XT>(words[j]), first ? f32x4_t{0.0f, 0.0f, 0.0f, 0.0f} : part);
      if (done) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(part[e], s[32 * j / G], acc[e]);
      }
    }
  };

  // the waves' sums, in the order of the waves; element e of lane (c, g): row 4 g + e of
  // x, weight row c
  float* const sums = reinterpret_cast<float*>(lds + mrows * stride);
  int group = blockIdx.x, round = 0, turn = 0;
  auto finish = [&] {
    float* const part = sums + turn * (kWaves * 16 * mrows);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (4 * g + e < mrows) part[(wave * mrows + 4 * g + e) * 16 + c] = acc[e];
    __syncthreads();
    const int64_t n = (int64_t)group * 16 + (threadIdx.x & 15);
    const int m = threadIdx.x >> 4;
    if (m < mrows && n < N) {
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) v += part[w * mrows * 16 + threadIdx.x];
      y[m * N + n] = 16.0f * v;
    }
    turn ^= 1;  // the next group's sums go beside these, which may still be read
    acc = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  };

  acc = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  __syncthreads();
  // one way out, after the last of the D steps, as above
  do {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const int k0 = (round * kWaves + wave) * kPiece;
      if (k0 < sl.count) multiply(d, 0, k0), multiply(d, 1, k0 + 128);
      load(d);
      if (++round == rounds) {
        if (group < groups) finish();
        round = 0;
        group += gridDim.x;
      }
    }
  } while (group < groups);
}

// ---------------------------------------------------------------- more rows, small weights
//
// A wave takes the half pieces of its part of K; x of a half piece (16 MT rows) comes from
// the caches, moved between lanes like the codes, and is multiplied with the codes of GB
// tiles of 16 weight rows, whose sums stay in registers over the slice.  Nothing waits for
// a staged x, and no workgroup has more than its share of K to read: a 2,048 x 8,192
// product of 16 rows takes 8 us, 11 with x passed through LDS.  What it costs is x, read
// again by every workgroup, at 10 TB/s from the L2s in all: GB tiles of the weight share a
// read.  The codes of a whole
// piece, GB tiles of it, are in flight, and one half piece of x (two where GB is 1).
// G: codes summed before their scale is applied.
template <int XT, int MT, int GB, int G>
__global__ void __launch_bounds__(kGemmThreads, MT == 1 ? 4 : 2)
    k_int4_regs(const uint16_t* __restrict__ x, const uint8_t* __restrict__ packed, const float* __restrict__ scales,
                int64_t M, int64_t N, int64_t K, int each, int lgB, int groups, float* __restrict__ y) {
  extern __shared__ u32x4 lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15;
  const int g = lane >> 4;
  const int64_t m0 = (int64_t)blockIdx.y * (16 * MT);
  const int mrows = (int)(M - m0 < 16 * MT ? M - m0 : 16 * MT);
  const Slice sl(K, each);
  y += blockIdx.z * (M * N);
  const __amdgpu_buffer_rsrc_t xres =
      __builtin_amdgcn_make_buffer_rsrc((void*)(x + m0 * K), (short)0, mrows * (int)K * 2, kRawBuffer);
  Weight<GB, GB> wt(packed, scales, N, K, sl, lgB, groups);
  const int rounds = (pieces_of(sl.count) + kWaves - 1) / kWaves;

  // In MFMA j of a half piece lane (c, g) multiplies elements 32 j + 8 g on.
  constexpr int XB = GB == 1 ? 2 : 1;  // half pieces of x in flight
  u32x4 xv[XB][MT][4];
  auto read_x = [&](int buf, int k0) {  // the half piece from k0 on; lane l: row l / 4
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = k0 + 32 * j + 8 * (lane & 3);
        const uint32_t off =
            k < sl.count ? ((uint32_t)(16 * i + (lane >> 2)) * (uint32_t)K + (uint32_t)(sl.from + k)) * 2 : kOutside;
        xv[buf][i][j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xres, (int)off, 0, 0));
      }
  };

  f32x4_t acc[MT][GB];
  auto clear = [&] {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int t = 0; t < GB; ++t) acc[i][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  };
  u32x4 xf[MT][4];
  auto turn_x = [&](int buf) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) xf[i][j][q] = from_lane(4 * c + g, xv[buf][i][j][q]);
  };
  auto multiply = [&](int t, int h) {  // half h of tile t's piece
    u32x4 words;
#pragma unroll
    for (int q = 0; q < 4; ++q) words[q] = from_lane(4 * c + g, wt.codes[t][h][q]);
    words = transposed(words);
    float s[128 / G];
#pragma unroll
    for (int q = 0; q < 128 / G; ++q) s[q] = u2f(from_lane(4 * c + q * (G / 32), f2u(wt.scale[t][h])));
    f32x4_t part[MT];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool first = (32 * j) % G == 0, done = (32 * j + 32) % G == 0;
      const u32x4 wf = operand<XT>(words[j]);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        part[i] = mfma<XT>(xf[i][j], wf, first ? f32x4_t{0.0f, 0.0f, 0.0f, 0.0f} : part[i]);
        if (done) {
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][t][e] = __builtin_fmaf(part[i][e], s[32 * j / G], acc[i][t][e]);
        }
      }
    }
  };

  // ---- the waves' sums, in the order of the waves; D element e of lane (c, g): row
  // 4 g + e of x, weight row c
  float* const sums = reinterpret_cast<float*>(lds);
  auto finish = [&](int group) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = 16 * i + 4 * g + e;
        if (m < mrows)
#pragma unroll
          for (int t = 0; t < GB; ++t) sums[(wave * mrows + m) * (16 * GB) + 16 * t + c] = acc[i][t][e];
      }
    __syncthreads();
    const int64_t n0 = (int64_t)group * (16 * GB);
    for (int o = threadIdx.x; o < mrows * 16 * GB; o += kGemmThreads) {
      const int m = o / (16 * GB), n = o % (16 * GB);
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) v += sums[w * mrows * (16 * GB) + o];
      if (n0 + n < N) y[(m0 + m) * N + n0 + n] = 16.0f * v;
    }
    __syncthreads();  // the next group's sums go where these are
    clear();
  };

  int group = blockIdx.x, round = 0, k0 = wave * kPiece;
  wt.turn_to(group);
#pragma unroll
  for (int b = 0; b < XB; ++b) read_x(b, k0 + 128 * b);
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int t = 0; t < GB; ++t) wt.load(t, h, t, (uint32_t)k0);
  clear();
  do {
    const bool last = round + 1 == rounds;
    const int next = last ? wave * kPiece : k0 + kWaves * kPiece;
    if (last) wt.turn_to(group + gridDim.x);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      turn_x(h % XB);
      read_x(h % XB, XB == 2 ? next + 128 * h : h == 0 ? k0 + 128 : next);
#pragma unroll
      for (int t = 0; t < GB; ++t) {
        if (k0 + 128 * h < sl.count) multiply(t, h);
        wt.load(t, h, t, (uint32_t)next);
      }
    }
    k0 = next;
    ++round;
    if (last) {
      finish(group);
      round = 0;
      group += gridDim.x;
    }
  } while (group < groups);
}

// ---------------------------------------------------------------- more than 16 rows
//
// Each wave has a tile of 16 weight rows to itself over the slice of K, and the 8 waves
// share x: a piece of 16 MT rows is in LDS while the next one is on its way there through
// registers, so that x is read once for 128 weight rows.  Bound by LDS and the codes'
// conversion in turn: 64 rows, 65,536 x 2,048 34 us (k_int4_regs 69, most of it reads of x);
// 24,576 x 6,144 51 (57).
// MT: 16-row tiles of x.  G: codes summed before their scale is applied.
template <int XT, int MT, int G>
__global__ void __launch_bounds__(kGemmThreads, 4)
    k_int4_wide(const uint16_t* __restrict__ x, const uint8_t* __restrict__ packed, const float* __restrict__ scales,
                int64_t M, int64_t N, int64_t K, int each, int lgB, int tiles, float* __restrict__ y) {
  constexpr int D = 2;                                  // pieces of the weight in flight, and of x in LDS
  constexpr int kRow = kPiece / 8 + 1;                  // 16-byte units of a row: odd, as above
  constexpr int kBuffer = 16 * MT * kRow;
  static_assert(kGemmThreads * MT * 8 == 16 * MT * kPiece, "a piece of x is MT units a thread");
  __shared__ u32x4 lds[D * kBuffer];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15;
  const int g = lane >> 4;
  const int64_t m0 = (int64_t)blockIdx.y * (16 * MT);
  const int mrows = (int)(M - m0 < 16 * MT ? M - m0 : 16 * MT);
  const Slice sl(K, each);
  const int pieces = pieces_of(sl.count);
  const __amdgpu_buffer_rsrc_t xres =
      __builtin_amdgcn_make_buffer_rsrc((void*)(x + m0 * K), (short)0, mrows * (int)K * 2, kRawBuffer);
  const int tile = (int)blockIdx.x * kWaves + wave;
  Weight<1, D> wt(packed, scales, N, K, sl, lgB, tiles);
  wt.turn_to(tile);

  // of the thread's first unit; the next ones are 16 rows on each
  const int xrow = threadIdx.x / (kPiece / 8), xcol = threadIdx.x % (kPiece / 8);
  u32x4 xv[MT];
  auto read_x = [&](int p) {  // rows past M are outside the resource: zeros
    const int k = p * kPiece + 8 * xcol;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const uint32_t off =
          k < sl.count ? ((uint32_t)(16 * i + xrow) * (uint32_t)K + (uint32_t)(sl.from + k)) * 2 : kOutside;
      xv[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xres, (int)off, 0, 0));
    }
  };
  auto write_x = [&](int buf) {
#pragma unroll
    for (int i = 0; i < MT; ++i) lds[buf * kBuffer + (16 * i + xrow) * kRow + xcol] = xv[i];
  };

  constexpr bool kAsLoaded = G == 128;
  constexpr int XG = kAsLoaded ? 32 : 8, XJ = kAsLoaded ? 8 : 32;
  const u32x4* const xat = lds + c * kRow + XG * g / 8;
  f32x4_t acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  auto multiply = [&](int d, int h) {  // half h of the piece in slot d and buffer d
    u32x4 words;
#pragma unroll
    for (int q = 0; q < 4; ++q) words[q] = from_lane(4 * c + g, wt.codes[d][h][q]);
    if constexpr (!kAsLoaded) words = transposed(words);
    float s[128 / G];
#pragma unroll
    for (int q = 0; q < 128 / G; ++q) s[q] = u2f(from_lane(4 * c + q * (G / 32), f2u(wt.scale[d][h])));
    f32x4_t part[MT];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool first = (32 * j) % G == 0, done = (32 * j + 32) % G == 0;
      const u32x4 wf = operand<XT>(words[j]);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const u32x4 xf = xat[d * kBuffer + 16 * i * kRow + (128 * h + XJ * j) / 8];
        part[i] = mfma<XT>(xf, wf, first ? f32x4_t{0.0f, 0.0f, 0.0f, 0.0f} : part[i]);
        if (done) {
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][e] = __builtin_fmaf(part[i][e], s[32 * j / G], acc[i][e]);
        }
      }
    }
  };

  read_x(0);
#pragma unroll
  for (int d = 0; d < D; ++d) wt.load(d, 0, 0, (uint32_t)(d * kPiece)), wt.load(d, 1, 0, (uint32_t)(d * kPiece));
  write_x(0);
  read_x(1);
  for (int p = 0; p < pieces; p += D) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      __syncthreads();  // x of this piece is there, and no wave reads the last one any more
      if (p + d < pieces) multiply(d, 0), multiply(d, 1);
      const uint32_t next = (uint32_t)((p + d + D) * kPiece);
      wt.load(d, 0, 0, next), wt.load(d, 1, 0, next);
      write_x(d ^ 1);
      read_x(p + d + 2);
    }
  }

  // element e of lane (c, g): row 4 g + e of x, weight row c
  y += blockIdx.z * (M * N);
  const int64_t n = (int64_t)tile * 16 + c;
  if (n >= N) return;
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int m = 16 * i + 4 * g + e;
      if (m < mrows) y[(m0 + m) * N + n] = 16.0f * acc[i][e];
    }
}

// The slices' sums, in the order of the slices.  16 rows of 6,144 columns, 2 slices: 2 us.
constexpr int kJoinThreads = 256;
__global__ void __launch_bounds__(kJoinThreads)
    k_int4_join(unsigned first, const float* __restrict__ planes, int64_t n, int count, float* __restrict__ y) {
  const int64_t i = (int64_t)(first + blockIdx.x) * kJoinThreads + threadIdx.x;
  if (i >= n) return;
  float v = 0.0f;
  for (int z = 0; z < count; ++z) v += planes[z * n + i];
  y[i] = v;
}

using Int4Kernel = void (*)(const uint16_t*, const uint8_t*, const float*, int64_t, int64_t, int64_t, int, int, int,
                            float*);

template <int XT>
Int4Kernel int4_few_kernel(int MR) {
  return MR == 1 ? &k_int4_few<XT, 1, 2> : MR == 2 ? &k_int4_few<XT, 2, 2> : &k_int4_few<XT, 4, 2>;
}
template <int XT>
Int4Kernel int4_lds_kernel(int G) {
  return G == 128 ? &k_int4_lds<XT, 2, 128> : G == 64 ? &k_int4_lds<XT, 2, 64> : &k_int4_lds<XT, 2, 32>;
}
template <int XT, int MT>
Int4Kernel int4_wide_kernel_of(int G) {
  return G == 128 ? &k_int4_wide<XT, MT, 128> : G == 64 ? &k_int4_wide<XT, MT, 64> : &k_int4_wide<XT, MT, 32>;
}
template <int XT>
Int4Kernel int4_wide_kernel(int MT, int G) {
  return MT == 2   ? int4_wide_kernel_of<XT, 2>(G)
         : MT == 3 ? int4_wide_kernel_of<XT, 3>(G)
                   : int4_wide_kernel_of<XT, 4>(G);
}
template <int XT, int MT, int GB>
Int4Kernel int4_regs_kernel_for(int G) {
  return G == 128  ? &k_int4_regs<XT, MT, GB, 128>
         : G == 64 ? &k_int4_regs<XT, MT, GB, 64>
                   : &k_int4_regs<XT, MT, GB, 32>;
}
template <int XT, int GB>
Int4Kernel int4_regs_kernel_of(int MT, int G) {
  return MT == 1   ? int4_regs_kernel_for<XT, 1, GB>(G)
         : MT == 2 ? int4_regs_kernel_for<XT, 2, GB>(G)
                   : int4_regs_kernel_for<XT, 4, GB>(G);
}
template <int XT>
Int4Kernel int4_regs_kernel(int MT, int GB, int G) {
  return GB == 1   ? int4_regs_kernel_of<XT, 1>(MT, G)
         : GB == 2 ? int4_regs_kernel_of<XT, 2>(MT, G)
                   : int4_regs_kernel_of<XT, 3>(MT, G);
}

}  // namespace
}  // namespace zq

extern "C" int64_t zq_int4_dequant_gemm_bytes(int64_t M, int64_t N, int64_t K) {
  using namespace zq;
  if (!int4_sizes_ok(M, N, K)) return -1;
  if (M == 0 || N == 0) return 0;
  return workspace_of(int4_plan(M, N, K), M, N);
}

extern "C" int zq_int4_dequant_gemm(const void* x, zq_dtype xt, const uint8_t* packed, const float* scales, int64_t M,
                                    int64_t N, int64_t K, int32_t block, float* y, void* workspace,
                                    int64_t workspace_bytes, void* stream) {
  using namespace zq;
  if (!int4_sizes_ok(M, N, K)) return ZQ_E_SIZE;
  const int lgB = log2_block(block);
  if (lgB < 0) return ZQ_E_BLOCK;
  if (xt != ZQ_BF16 && xt != ZQ_F16) return ZQ_E_DTYPE;
  if (M == 0 || N == 0) return ZQ_OK;
  const Int4Plan p = int4_plan(M, N, K);
  const int64_t need = workspace_of(p, M, N);
  if (workspace_bytes < need) return ZQ_E_SIZE;
  if (!y || (need > 0 && !workspace) || (K > 0 && (!x || !packed || !scales))) return ZQ_E_NULL;
  if (!aligned(x, 16) || !aligned(packed, 16) || !aligned(scales, 4) || !aligned(y, 4) ||
      (need > 0 && !aligned(workspace, 4)))
    return ZQ_E_ALIGN;
  if (any_overlap({{y, 4 * M * N}, {workspace, need}},
                  {{x, 2 * M * K}, {packed, N * K / 2}, {scales, 4 * num_scales(N * K, block)}}))
    return ZQ_E_ALIAS;

  const int G = int4_codes_a_scale(K, block);
  const bool bf = xt == ZQ_BF16;
  const Int4Kernel k = p.way == Int4Way::few   ? (bf ? int4_few_kernel<ZQ_BF16>(p.MR) : int4_few_kernel<ZQ_F16>(p.MR))
                       : p.way == Int4Way::wide ? (bf ? int4_wide_kernel<ZQ_BF16>(p.MT, G)
                                                      : int4_wide_kernel<ZQ_F16>(p.MT, G))
                       : p.way == Int4Way::lds ? (bf ? int4_lds_kernel<ZQ_BF16>(G) : int4_lds_kernel<ZQ_F16>(G))
                                               : (bf ? int4_regs_kernel<ZQ_BF16>(p.MT, p.GB, G)
                                                     : int4_regs_kernel<ZQ_F16>(p.MT, p.GB, G));
  const int64_t joins = grid_for(M * N, kJoinThreads);
  if (p.slices > 1 && joins == 0) return ZQ_E_SIZE;
  const auto st = static_cast<hipStream_t>(stream);
  float* out = p.slices > 1 ? static_cast<float*>(workspace) : y;
  const uint16_t* xs = static_cast<const uint16_t*>(x);
  int each = (int)p.each, lg = lgB, groups = (int)p.groups;
  void* args[] = {&xs, &packed, &scales, &M, &N, &K, &each, &lg, &groups, &out};
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(k),
                                       dim3((unsigned)p.grid, (unsigned)p.mgroups, (unsigned)p.slices),
                                       dim3(kGemmThreads), args, (size_t)p.lds, st);
  if (e != hipSuccess) return ZQ_E_HIP;
  if (p.slices == 1) return ZQ_OK;
  return launch_parts(&k_int4_join, joins, (unsigned)kJoinThreads, st, out, M * N, (int)p.slices, y);
}
