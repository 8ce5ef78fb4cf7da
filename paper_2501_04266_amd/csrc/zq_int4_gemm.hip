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

constexpr int kWaves = 8;
constexpr int kPiece = 256;  // codes of a weight row that a wave takes at a time: a 128-byte line
constexpr int kGemmThreads = 64 * kWaves;
__host__ __device__ inline int pieces_of(int64_t K) { return K == 0 ? 1 : (int)((K + kPiece - 1) / kPiece); }

// The weight as a wave streams it.  A load takes half a piece (128 codes) of 16 rows:
// lane l has 32 codes of row l / 4, from code 32 (l % 4) on, so that 4 lanes in a row
// read 64 bytes in a row (with a row for each of 16 lanes in a row the same loads take
// four times as long in the address unit), and the scale of those codes, which lie in
// one block.  Slots of D pieces of NT x 16 rows are in flight.
template <int NT, int D>
struct Weight {
  u32x4 codes[D][NT][2];
  float scale[D][NT][2];

  const uint8_t* packed;
  const float* scales;
  int64_t N, K;
  int lgB, groups;
  // of the group being loaded
  __amdgpu_buffer_rsrc_t wres, sres;
  uint32_t first;  // its first row's place in its block
  uint32_t row0;   // this lane's first code, in the group's flat order
  int end;         // pieces that start before this have codes for the lane

  __device__ __forceinline__ Weight(const uint8_t* p, const float* s, int64_t n, int64_t k, int lg, int gr)
      : packed(p), scales(s), N(n), K(k), lgB(lg), groups(gr) {
    const int lane = threadIdx.x & 63;
    row0 = (uint32_t)(lane >> 2) * (uint32_t)k + 32u * (lane & 3);
    end = (int)k - 32 * (lane & 3);
  }
  __device__ __forceinline__ void turn_to(int group) {
    // past the last group: empty resources; the same loads go out, so that the number
    // of loads in flight is known at every wait, and bring zeros
    const bool any = group < groups;
    const int64_t n0 = any ? (int64_t)group * (16 * NT) : 0;
    const int rows = any ? (int)(N - n0 < 16 * NT ? N - n0 : 16 * NT) : 0;
    wres = __builtin_amdgcn_make_buffer_rsrc((void*)(packed + n0 * (K / 2)), (short)0, rows * (int)(K / 2), kRawBuffer);
    const int64_t f0 = n0 * K, s0 = f0 >> lgB, s1 = (f0 + (int64_t)rows * K + (1 << lgB) - 1) >> lgB;
    sres = __builtin_amdgcn_make_buffer_rsrc((void*)(scales + s0), (short)0, (int)((s1 - s0) * 4), kRawBuffer);
    first = (uint32_t)(f0 & ((1ll << lgB) - 1));
  }
  // the piece from code k0 of the group's rows on; rows past the last, and codes past K,
  // are outside the resources: zeros
  __device__ __forceinline__ void load(int d, uint32_t k0) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const uint32_t f = row0 + 16 * t * (uint32_t)K + k0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool in = (int)k0 < end - 128 * h;
        const uint32_t off = in ? f / 2 + 64u * h : kOutside;
        codes[d][t][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(wres, (int)off, 0, 0));
        const uint32_t soff = in ? ((f + first + 128u * h) >> lgB) * 4 : kOutside;
        scale[d][t][h] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(sres, (int)soff, 0, 0));
      }
    }
  }
};

// x rows m0 .. m0 + mrows in LDS, whole; elements past K, which meet zero codes, are
// zeros.  Rows are an odd number of 16-byte units long, so that lanes that read one
// column of 8 rows meet distinct banks.  `between` runs once the first loads are out.
// What there is no place for goes to the unit after the last row: a load whose result
// is left in its registers makes the compiler wait for all loads wherever these are
// used again, in each turn of the loops below.
__device__ __forceinline__ int x_stride(int64_t K) { return pieces_of(K) * (kPiece / 8) + 1; }
template <typename F>
__device__ __forceinline__ void stage_x(u32x4* lds, __amdgpu_buffer_rsrc_t xres, int mrows, int64_t K, F between) {
  constexpr int U = 4;
  const int stride = x_stride(K), kk = (int)K;
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
      const uint32_t off = i < units && k < (unsigned)kk ? (m * (unsigned)kk + k) * 2 : kOutside;
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
// transposition.  Each column has one scale, whatever the block size.
// MR: rows of x, 1, 2 or a multiple of 4.
__host__ __device__ constexpr int few_sums(int MR) { return 4 * MR * 16; }  // a wave's: MR x 16 of each range
__host__ __device__ constexpr int few_buffers(int MR) { return MR <= 4 ? 2 : 1; }
template <int XT, int MR, int D>
__global__ void __launch_bounds__(kGemmThreads)
    k_int4_few(const uint16_t* __restrict__ x, const uint8_t* __restrict__ packed, const float* __restrict__ scales,
               int64_t M, int64_t N, int64_t K, int lgB, int groups, float* __restrict__ y) {
  constexpr int MG = MR <= 4 ? 1 : MR / 4, MQ = MR < 4 ? MR : 4;
  extern __shared__ u32x4 lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15;
  const int g = lane >> 4;
  const int kk = (int)K, mrows = (int)M, stride = x_stride(K);
  const int rounds = (pieces_of(K) + kWaves - 1) / kWaves;
  Weight<1, D> wt(packed, scales, N, K, lgB, groups);
  int load_group = blockIdx.x, load_round = 0;
  wt.turn_to(load_group);
  auto load = [&](int d) {
    wt.load(d, (uint32_t)((load_round * kWaves + wave) * kPiece));
    if (++load_round == rounds) load_round = 0, wt.turn_to(load_group += gridDim.x);
  };
  stage_x(lds, __builtin_amdgcn_make_buffer_rsrc((void*)x, (short)0, mrows * kk * 2, kRawBuffer), mrows, K, [&] {
#pragma unroll
    for (int d = 0; d < D; ++d) load(d);
  });
  const u32x4* xat[MG];  // rows past M repeat the last one; their sums are not stored
#pragma unroll
  for (int q = 0; q < MG; ++q) {
    const int m = 4 * q + (lane & 3);
    xat[q] = lds + (m < mrows ? m : mrows - 1) * stride + 4 * (c >> 2) + g;
  }

  float acc[4][MR];
  auto clear = [&] {
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int m = 0; m < MR; ++m) acc[w][m] = 0.0f;
  };
  auto multiply = [&](int d, int h, int k0) {
    u32x4 xf[MG];
#pragma unroll
    for (int q = 0; q < MG; ++q) xf[q] = xat[q][k0 / 8];
    const u32x4 words = transposed(wt.codes[d][0][h]);
    float s[4];  // the scale of lane 16 w + c
#pragma unroll
    for (int w = 0; w < 4; ++w)
      s[w] = u2f((uint32_t)__builtin_amdgcn_ds_bpermute(4 * (16 * w + c), (int)f2u(wt.scale[d][0][h])));
    f32x4_t part[4][MG];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const u32x4 wf = operand<XT>(words[w]);
#pragma unroll
      for (int q = 0; q < MG; ++q) part[w][q] = mfma<XT>(xf[q], wf, f32x4_t{0.0f, 0.0f, 0.0f, 0.0f});
    }
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int q = 0; q < MG; ++q)
#pragma unroll
        for (int m = 0; m < MQ; ++m) acc[w][4 * q + m] = __builtin_fmaf(part[w][q][m], s[w], acc[w][4 * q + m]);
  };

  float* const sums = reinterpret_cast<float*>(lds + mrows * stride);
  constexpr int kOne = few_sums(MR);
  int group = blockIdx.x, round = 0, turn = 0;
  auto finish = [&] {
    float* const part = sums + turn * (kWaves * kOne);
    if (few_buffers(MR) == 1) __syncthreads();
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
    if (few_buffers(MR) == 2) turn ^= 1;  // the next group's sums go beside these, which may still be read
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
      if (k0 < kk) multiply(d, 0, k0), multiply(d, 1, k0 + 128);
      load(d);
      if (++round == rounds) {
        if (group < groups) finish();
        round = 0;
        group += gridDim.x;
      }
    }
  } while (group < groups);
}

// ---------------------------------------------------------------- more rows
//
// MT: 16-row tiles of x.  G: codes summed before their scale is applied (they lie in one
// block).  The codes and scales go to the lanes that need them through LDS (one
// permutation of the wave): lane (c, g) takes the 32 codes of row c from 32 g on.
// XL: all of x is in LDS, from before the first group on.  Otherwise it is read from
// the caches, half a piece ahead, permuted like the codes; a group then has several
// tiles, which share it.
template <int XT, int MT, int NT, int D, int G, bool XL>
__global__ void __launch_bounds__(kGemmThreads)
    k_int4_rows(const uint16_t* __restrict__ x, const uint8_t* __restrict__ packed, const float* __restrict__ scales,
                int64_t M, int64_t N, int64_t K, int lgB, int groups, float* __restrict__ y) {
  extern __shared__ u32x4 lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15;
  const int g = lane >> 4;
  const int64_t m0 = (int64_t)blockIdx.y * (16 * MT);
  const int mrows = (int)(M - m0 < 16 * MT ? M - m0 : 16 * MT);
  const int kk = (int)K, stride = x_stride(K);
  const __amdgpu_buffer_rsrc_t xres =
      __builtin_amdgcn_make_buffer_rsrc((void*)(x + m0 * K), (short)0, mrows * kk * 2, kRawBuffer);
  Weight<NT, D> wt(packed, scales, N, K, lgB, groups);
  const int rounds = (pieces_of(K) + kWaves - 1) / kWaves;
  int load_group = blockIdx.x, load_round = 0;
  wt.turn_to(load_group);
  auto load = [&](int d) {
    wt.load(d, (uint32_t)((load_round * kWaves + wave) * kPiece));
    if (++load_round == rounds) load_round = 0, wt.turn_to(load_group += gridDim.x);
  };
  auto from = [&](int source, uint32_t v) {
    return (uint32_t)__builtin_amdgcn_ds_bpermute(4 * source, (int)v);
  };

  // Lane (c, g) multiplies in MFMA j of a half piece: elements 32 g + 8 j on, where the
  // codes may stay as they are loaded; else, with the words transposed, 32 j + 8 g on.
  constexpr bool kAsLoaded = G == 128 && XL;
  constexpr int XG = kAsLoaded ? 32 : 8, XJ = kAsLoaded ? 8 : 32;
  int xrow[MT];  // rows past M repeat the last one; their sums are not stored
#pragma unroll
  for (int i = 0; i < MT; ++i) xrow[i] = 16 * i + c < mrows ? 16 * i + c : mrows - 1;
  u32x4 xv[XL ? 1 : 2][MT][4];
  auto read_x = [&](int buf, int k0) {  // the half piece from k0 on; lane l: row l / 4, 8 elements at 32 j + 8 (l % 4)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = k0 + 32 * j + 8 * (lane & 3);
        const uint32_t off = k < kk ? ((uint32_t)(16 * i + (lane >> 2)) * (uint32_t)kk + (uint32_t)k) * 2 : kOutside;
        xv[buf][i][j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xres, (int)off, 0, 0));
      }
  };
  auto load_all = [&] {
#pragma unroll
    for (int d = 0; d < D; ++d) load(d);
  };
  if constexpr (XL) stage_x(lds, xres, mrows, K, load_all);
  else load_all();

  f32x4_t acc[MT][NT];
  auto clear = [&] {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[i][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  };
  auto multiply = [&](int d, int h, int k0) {  // half h of the piece in slot d; k0: its first code
    u32x4 xf[MT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (XL) {
          xf[i][j] = lds[xrow[i] * stride + (k0 + XG * g + XJ * j) / 8];
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) xf[i][j][q] = from(4 * c + g, xv[h][i][j][q]);
        }
      }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      u32x4 words;
#pragma unroll
      for (int q = 0; q < 4; ++q) words[q] = from(4 * c + g, wt.codes[d][t][h][q]);
      if constexpr (!kAsLoaded) words = transposed(words);
      float s[128 / G];
#pragma unroll
      for (int q = 0; q < 128 / G; ++q) s[q] = u2f(from(4 * c + q * (G / 32), f2u(wt.scale[d][t][h])));
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
    }
  };

  // ---- the waves' sums, in the order of the waves; D element e of lane (c, g): row
  // 4 g + e of x, weight row c
  float* const sums = reinterpret_cast<float*>(lds + (XL ? mrows * stride : 0));
  int group = blockIdx.x, round = 0, turn = 0;
  auto finish = [&] {
    float* const part = sums + turn * (kWaves * mrows * 16 * NT);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = 16 * i + 4 * g + e;
        if (m < mrows)
#pragma unroll
          for (int t = 0; t < NT; ++t) part[(wave * mrows + m) * (16 * NT) + 16 * t + c] = acc[i][t][e];
      }
    __syncthreads();
    const int64_t n0 = (int64_t)group * (16 * NT);
    for (int o = threadIdx.x; o < mrows * 16 * NT; o += kGemmThreads) {
      const int m = o / (16 * NT), n = o % (16 * NT);
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) v += part[w * mrows * (16 * NT) + o];
      if (n0 + n < N) y[(m0 + m) * N + n0 + n] = 16.0f * v;
    }
    turn ^= 1;  // the next group's sums go beside these, which may still be read
    clear();
  };

  clear();
  if constexpr (XL) __syncthreads();
  else read_x(0, wave * kPiece);
  // The D steps have one way out, after the last: with one after each the compiler
  // waits for all loads in every turn.  Steps past the last group multiply zeros.
  do {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const int k0 = (round * kWaves + wave) * kPiece;
      if constexpr (XL) {
        if (k0 < kk) multiply(d, 0, k0), multiply(d, 1, k0 + 128);
      } else {
        read_x(1, k0 + 128);
        if (k0 < kk) multiply(d, 0, k0);
        read_x(0, round + 1 == rounds ? wave * kPiece : k0 + kWaves * kPiece);
        if (k0 < kk) multiply(d, 1, k0 + 128);
      }
      load(d);
      if (++round == rounds) {
        if (group < groups) finish();
        round = 0;
        group += gridDim.x;
      }
    }
  } while (group < groups);
}

using Int4Kernel = void (*)(const uint16_t*, const uint8_t*, const float*, int64_t, int64_t, int64_t, int, int, float*);

template <int XT, int MT, int NT, int D, bool XL>
Int4Kernel int4_kernel_for(int G) {
  return G == 128  ? &k_int4_rows<XT, MT, NT, D, 128, XL>
         : G == 64 ? &k_int4_rows<XT, MT, NT, D, 64, XL>
                   : &k_int4_rows<XT, MT, NT, D, 32, XL>;
}
template <int XT>
Int4Kernel int4_few_kernel(int few) {
  return few == 1   ? &k_int4_few<XT, 1, 2>
         : few == 2 ? &k_int4_few<XT, 2, 2>
                    : &k_int4_few<XT, 4, 2>;
}
template <int XT>
Int4Kernel int4_kernel(bool xl, int MT, int NT, int G) {
  if (xl) return MT == 1 ? int4_kernel_for<XT, 1, 1, 2, true>(G) : int4_kernel_for<XT, 2, 1, 2, true>(G);
  if (MT == 1) return NT == 1 ? int4_kernel_for<XT, 1, 1, 3, false>(G) : int4_kernel_for<XT, 1, 2, 2, false>(G);
  return NT == 1 ? int4_kernel_for<XT, 2, 1, 3, false>(G) : int4_kernel_for<XT, 2, 2, 2, false>(G);
}

constexpr int64_t kInt4MaxK = 1 << 22;  // 32 rows of x and 16 of codes stay below 2^31 bytes
constexpr int64_t kLds = 160 * 1024, kCus = 256;

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

  const int MT = M <= 16 ? 1 : 2;
  const int64_t mrows = M < 16 * MT ? M : 16 * MT, mgroups = (M + 16 * MT - 1) / (16 * MT);
  // codes under one scale: 128 from a multiple of 128 on lie in one block only where
  // rows start at multiples of 128
  const int G = block >= 128 && K % 128 == 0 ? 128 : block >= 64 ? 64 : 32;
  // x in LDS where it leaves room for the waves' sums
  const int few = M <= 2 ? (int)M : M <= 4 ? 4 : 0;
  const int64_t xbytes = mrows * (pieces_of(K) * (kPiece / 8) + 1) * 16;
  const int64_t sbytes = few ? few_buffers(few) * kWaves * few_sums(few) * 4 : 2 * kWaves * 16 * mrows * 4;
  const bool xl = xbytes + sbytes <= kLds;
  const int64_t tiles = (N + 15) / 16;
  const int NT = xl || tiles <= 512 ? 1 : 2;
  const int64_t groups = (tiles + NT - 1) / NT;
  if (groups > kMaxGrid / 2 || mgroups > 65535) return ZQ_E_SIZE;
  const int64_t lds = xl ? xbytes + sbytes : 2 * kWaves * 16 * 4 * mrows * NT;
  // x in LDS: as many workgroups as are resident at once
  const int64_t room = (lds <= kLds / 2 ? 2 : 1) * kCus, grid = xl && groups > room ? room : groups;
  const Int4Kernel k = xl && few ? (xt == ZQ_BF16 ? int4_few_kernel<ZQ_BF16>(few) : int4_few_kernel<ZQ_F16>(few))
                                 : (xt == ZQ_BF16 ? int4_kernel<ZQ_BF16>(xl, MT, NT, G) : int4_kernel<ZQ_F16>(xl, MT, NT, G));
  return launch_grid(k, dim3((unsigned)grid, (unsigned)mgroups), (unsigned)kGemmThreads, (unsigned)lds,
                     static_cast<hipStream_t>(stream), static_cast<const uint16_t*>(x), packed, scales, M, N, K, lgB,
                     (int)groups, y);
}
