// zq_int4_plan.h -- which kernel of the products with INT4 weights runs a product, in
// which tiles and slices: host arithmetic on the sizes alone, without HIP, so that a
// test on the CPU can ask it.  The kernels take their tile sizes from here.
#pragma once

#include <stdint.h>

#include "zq_limits.h"

namespace zq {

constexpr int kWaves = 8;
constexpr int kPiece = 256;  // codes of a weight row that a wave takes at a time: a 128-byte line
constexpr int kGemmThreads = 64 * kWaves;
constexpr int pieces_of(int64_t K) { return K == 0 ? 1 : (int)((K + kPiece - 1) / kPiece); }
// 16-byte units of a row of x in LDS: an odd number
constexpr int x_stride(int64_t K) { return pieces_of(K) * (kPiece / 8) + 1; }
constexpr int few_sums(int MR) { return 4 * MR * 16; }  // a wave's of k_int4_few: MR x 16 of each range

constexpr int64_t kInt4MaxK = 1 << 22;  // 64 rows of x and 48 of codes stay below 2^31 bytes
constexpr int64_t kLds = 160 * 1024, kCus = 256;

// How a product is cut.
enum class Int4Way { few, lds, regs, wide };
struct Int4Plan {
  Int4Way way;
  int MR, MT, GB;        // few: rows of sums; regs: 16-row tiles of x, tiles of the weight
  int64_t each, slices;  // of K
  int64_t groups, grid, mgroups, lds;
};

// codes of a slice where there are `slices` at most
inline int64_t slice_of(int64_t K, int64_t slices) {
  const int64_t each = ((K + slices - 1) / slices + kPiece - 1) / kPiece * kPiece;
  return each < kPiece ? kPiece : each;
}

// Up to 4 rows k_int4_few; up to 16 and more than two tiles a CU k_int4_lds, whose
// reads of x cost least once its LDS is filled (5 rows, 50,001 x 6,144: 35 us, k_int4_regs
// 52; 16 rows, 24,576 x 4,096: 16 and 19; but 16 rows, 6,144 x 6,144: 14 and 9).  Both
// take x in slices where it is too long for LDS.  Else k_int4_regs or k_int4_wide.
inline Int4Plan int4_plan(int64_t M, int64_t N, int64_t K) {
  Int4Plan p{};
  const int64_t tiles = (N + 15) / 16;
  p.MR = M <= 2 ? (int)M : 4;
  p.MT = M <= 16 ? 1 : M <= 32 ? 2 : 4;
  p.GB = 1, p.mgroups = 1, p.slices = 1;
  p.way = M <= 4 ? Int4Way::few : M <= 16 && tiles > 2 * kCus ? Int4Way::lds : Int4Way::regs;
  if (p.way != Int4Way::regs) {
    const int64_t sums = 2 * kWaves * 4 * (p.way == Int4Way::few ? few_sums(p.MR) : 16 * M);
    auto lds_of = [&](int64_t k) { return M * x_stride(k) * 16 + sums; };
    // slices: the largest that fit; with up to 4 rows two workgroups a CU (3 rows, 4,096 x
    // 49,152: 34 us, 44 with one; 16 rows, 24,576 x 6,144: 31, with one 27)
    const int64_t most = p.way == Int4Way::few && lds_of(K) > kLds ? kLds / 2 : kLds;
    while (lds_of(slice_of(K, p.slices)) > most) ++p.slices;
    p.each = slice_of(K, p.slices);
    p.lds = lds_of(p.each);
    p.groups = tiles;
    // as many workgroups as are resident at once, each with all slices' share
    const int64_t room = (p.lds <= kLds / 2 ? 2 : 1) * kCus;
    p.grid = room / p.slices > 1 ? room / p.slices : 1;
  } else {
    p.mgroups = (M + 16 * p.MT - 1) / (16 * p.MT);
    // The least load of the busiest CU, in quarters of a tile's code (about 7,000 a us): a
    // workgroup's tiles and its reads of x (3/4 of a tile's time for 16 rows), for its
    // codes and 1,024 more to begin and end; slices cost the second launch, and their sums'
    // bytes.  Of the choices tried at 96 sizes (8 to 64 rows, 1,000 to 40,000 x 2,048 to
    // 24,576) it takes the fastest or one within 10% of it at 89, within 26% at all.  16
    // rows, 6,144 x 24,576: 30 us by two slices of 3 tiles, 47 by single tiles.
    double least = 0;
    for (int GB = 3; GB >= 1; --GB)
      for (int64_t S = 1; S == 1 || (S <= 16 && S <= K / 2048); ++S) {
        const double wgs = (double)((tiles + GB - 1) / GB) * (double)(p.mgroups * S);
        const double load = __builtin_ceil(wgs / kCus) * (double)(slice_of(K, S) + 1024) * (4 * GB + 3 * p.MT) +
                            (S > 1 ? 49152.0 + (double)M * (double)N * (double)S / 64 : 0.0);
        if (least == 0 || load < least) least = load, p.GB = GB, p.slices = S;
      }
    // k_int4_wide for more than 16 rows: a workgroup's 8 tiles take 1.2, 1.4 or 1.9 us a
    // piece (2, 3 and 4 tiles of x), and one and a half pieces to begin and end; two
    // workgroups on a CU take nearly twice that, and a few more than the CUs hold one of
    // take half as long again, not twice as long.  32 rows: 65,536 x 2,048 23 us, k_int4_regs 37; 20,000 x
    // 12,288 in three slices 45 and 64; but 4,096 x 4,096 12 and 8.
    if (p.MT > 1) {
      const int MT = M <= 32 ? 2 : M <= 48 ? 3 : 4;
      const double piece = 7000 * (MT == 2 ? 1.15 : MT == 3 ? 1.44 : 1.87);
      const int64_t grid = (tiles + kWaves - 1) / kWaves, mgroups = (M + 16 * MT - 1) / (16 * MT);
      // k_int4_regs, whose workgroups share the tiles out, where one launch has no room for a tile a wave
      for (int64_t S = 1; grid <= most_groups(kGemmThreads) && (S == 1 || (S <= 16 && S <= K / 512)); ++S) {
        const double w = (double)grid * (double)(mgroups * S) / kCus, even = 0.45 + 0.9 * w;
        const double turns = even < 1.0 ? 1.0 : even < __builtin_ceil(w) ? even : __builtin_ceil(w);
        const double load = turns * (double)(slice_of(K, S) / kPiece + 1.5) * piece +
                            (S > 1 ? 35000.0 + (double)M * (double)N * (double)S / 375 : 0.0);
        if (load < least) {
          least = load, p.way = Int4Way::wide, p.slices = S;
          p.MT = MT, p.mgroups = mgroups, p.grid = grid, p.groups = tiles, p.lds = 0;
        }
      }
    }
    p.each = slice_of(K, p.slices);
    if (p.way == Int4Way::regs) {
      p.groups = (tiles + p.GB - 1) / p.GB;
      p.grid = (p.MT == 1 ? 2 : 1) * kCus;
      p.lds = kWaves * 16 * 4 * (M < 16 * p.MT ? M : 16 * p.MT) * p.GB;
    }
  }
  if (p.way != Int4Way::wide && p.grid > p.groups) p.grid = p.groups;
  p.slices = K ? (K + p.each - 1) / p.each : 1;
  return p;
}

// bytes: the slices' sums
inline int64_t workspace_of(const Int4Plan& p, int64_t M, int64_t N) {
  return p.slices == 1 ? 0 : 4 * M * N * p.slices;
}

inline bool int4_sizes_ok(int64_t M, int64_t N, int64_t K) {
  return M >= 0 && N >= 0 && K >= 0 && K % 64 == 0 && K <= kInt4MaxK && M <= 64 * 65535 &&
         N <= INT64_MAX / 16 / (K + 1) && (N + 15) / 16 <= kMaxGrid / 2 && (M == 0 || N <= INT64_MAX / 1024 / M);
}

// Codes under one scale that the kernels sum before they apply it: 128 from a multiple
// of 128 on lie in one block only where rows start at multiples of 128.
inline int int4_codes_a_scale(int64_t K, int32_t block) {
  return block >= 128 && K % 128 == 0 ? 128 : block >= 64 ? 64 : 32;
}

}  // namespace zq
