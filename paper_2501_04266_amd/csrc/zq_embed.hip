// zq_embed.hip -- the embedding layer on gfx950: rows of the table by token id,
// and the table's gradient.
//
//   y[t][d]  = cvt(fl(scale * w[id_t][d]))           zeros where id_t is not a row
//   dw[v][d] = cvt(fl(scale * sum_{t: id_t = v} dy[t][d]))
//
// with w the table's elements, or fl(q * s) of its INT8 codes and block scales:
// the values qwz_dequantize writes, without writing them.
//
// Both are bound by memory: the lookup by the rows it reads and writes, the
// gradient by the dense result (V x D, most of it zeros) and the rows of dy.
// 16,384 tokens, 50,000 x 6,144 in binary32: 274 us, 5.2 TB/s (sorting the ids 14,
// the rows 255, the long rows' join 5; writing the zeros alone would take 178).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "zq.h"
#include "zq_device.h"
#include "zq_host.h"
#include "zq_vec.h"

#pragma clang fp contract(off)

namespace zq {
namespace {

constexpr int kEmbedThreads = 256;
constexpr int kInt8 = -1;  // WT of the lookup: INT8 codes and block scales

// The (row, piece) pairs of a matrix of C pieces a row, 256 consecutive ones a
// workgroup: this thread's row and piece.  The workgroup's first row comes from
// one binary64 product (its first pair is below 2^39, so the quotient is off by
// one at most), the thread's own from there in 32 bits.
struct Piece {
  int64_t row;
  int piece;
};
__device__ __forceinline__ Piece locate(unsigned wg, int C, double inv_c) {
  const int64_t u0 = (int64_t)wg * kEmbedThreads;
  int64_t row = (int64_t)((double)u0 * inv_c);
  int64_t rest = u0 - row * C;
  if (rest < 0) --row, rest += C;
  else if (rest >= C) ++row, rest -= C;
  const unsigned local = (unsigned)rest + threadIdx.x;
  const unsigned q = local / (unsigned)C;
  return {row + q, (int)(local - q * C)};
}

__device__ __forceinline__ int64_t id_at(const void* ids, bool wide, int64_t t) {
  return wide ? static_cast<const int64_t*>(ids)[t] : (int64_t)static_cast<const int32_t*>(ids)[t];
}

// A thread moves E elements of one token's row, 16 or 32 bytes of y.  The last piece of a
// row starts E before its end (it repeats elements of the piece before it where E does
// not divide D); E = 1 serves rows shorter than 8.  y is written past the caches, which
// are left to the table's rows: tokens repeat (16,384 tokens of 6,144 bf16 elements, ids
// of frequency 1 / rank, three sets of inputs in turn: 57 us, 4.8 TB/s, 64 with plain stores;
// from INT8 44 and 68; one set again and again 47).  Slices of the columns by XCD, so that
// each XCD's L2 holds other columns, measured slower (65).
template <int WT, int YT, int E>
__global__ void __launch_bounds__(kEmbedThreads)
    k_embed(unsigned first, const void* __restrict__ ids, bool wide, const void* __restrict__ table,
            const float* __restrict__ scales, int64_t T, int64_t V, int64_t D, int C, double inv_c, int lgB, float scale,
            void* __restrict__ y) {
  const Piece p = locate(first + blockIdx.x, C, inv_c);
  if (p.row >= T) return;
  const int64_t id = id_at(ids, wide, p.row);
  const int64_t d0 = (int64_t)p.piece * E;
  const int64_t d = d0 + E > D ? D - E : d0;
  float v[E];
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] = 0.0f;
  if ((uint64_t)id < (uint64_t)V) {
    const int64_t f = id * D + d;
    if constexpr (WT == kInt8) {
      const int8_t* codes = static_cast<const int8_t*>(table) + f;
      // E <= 32 elements meet two blocks at most
      const int64_t b = f >> lgB, b1 = (f + E - 1) >> lgB;
      const float s0 = scales[b], s1 = scales[b1];
      const int64_t turn = (b + 1) << lgB;  // the second block's first element
      if constexpr (E == 1) {
        v[0] = (float)codes[0] * s0;
      } else {
        uint32_t w[E / 4];
        load_words_any<false>(codes, w);
#pragma unroll
        for (int i = 0; i < E; ++i)
          v[i] = (float)(int32_t)(int8_t)(w[i / 4] >> (8 * (i % 4))) * (f + i < turn ? s0 : s1);
      }
    } else {
      load_elems<WT, E>(table, f, v);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = scale * v[i];
  }
  store_elems<YT, E, true>(y, p.row * D + d, v);
}

// ---------------------------------------------------------------- gradient
//
// 1. k_sort_ids (14 us for 16,384 tokens and 50,000 rows, 18 for 40,001 and 16,411:
//    latency of the loads and the LDS counts): the tokens in the order of their ids, ties in
//    the order of the tokens, and each row's first position in that order.  A workgroup owns a
//    range of rows and a part of the tokens, and reads all ids: first it counts its
//    rows' tokens, in its part and before and after it, and those of the rows before
//    its own, which gives its place in the order without another workgroup's count;
//    then it writes its tokens.
// 2. k_grad_rows: the sums of a row's tokens, and zeros for rows without any.  The
//    tokens of long rows (those that hold 64 positions from a multiple of 64 on) are
//    summed a segment of 64 positions at a time, by as many waves as there are
//    segments, beside the other rows.
// 3. k_grad_join: the long rows from their segments' sums.
// The order of every sum follows from the ids alone: no atomics on sums.
// Up to 512 tokens take k_grad_few instead, one launch.

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kRangeBits = 9, kMaxRange = 1 << kRangeBits;  // rows of a workgroup's range at most (48 KiB of LDS)
constexpr int kPart = 64;        // positions of a segment
constexpr int64_t kMaxTokens = 1 << 30;
// Ids that the sorting workgroups read in all, every one of a range of rows the T ids:
// 2^37 take about 0.1 s, so the most a call takes is about 2 s of the GPU.
constexpr int64_t kMaxReads = int64_t(1) << 41;

// What this wave's lanes wrote and read in LDS before comes before what they do after.
__device__ __forceinline__ void order_lds() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// This lane's place among the tokens of its row: the row's count so far (in the
// wave's `counts`) and the lanes of the same row before it; the counts move on.
// The lanes of one row are found by comparing the rows bit by bit.  Lanes that are not
// `in` give row 0 and get a place of no meaning.
__device__ __forceinline__ int take_place(int* counts, bool in, int row) {
  const uint64_t all = __ballot(in);
  uint32_t lo = (uint32_t)all, hi = (uint32_t)(all >> 32);
#pragma unroll
  for (int b = 0; b < kRangeBits; ++b) {
    const uint32_t mine = (uint32_t)((int32_t)((uint32_t)row << (31 - b)) >> 31);
    const uint64_t set = __ballot(mine != 0);
    lo &= ~((uint32_t)set ^ mine);
    hi &= ~((uint32_t)(set >> 32) ^ mine);
  }
  const int before = __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
  // All lanes of a row read its count before the first of them moves it on, and the next
  // group's lanes read it after that: lanes of one wave, so the fence costs no wait of its own.
  const int base = counts[row];
  order_lds();
  if (in && before == 0) counts[row] = base + __popc(lo) + __popc(hi);
  order_lds();
  return base + before;
}

constexpr int kSortSteps = 8;   // groups of 64 ids that a wave loads at a time
constexpr int kCopies = 4;      // of a row's counts: lanes that count the same row meet less often
constexpr int kSortLds = (kSortWaves + 2 * kCopies) * kMaxRange * 4;

// Workgroup (r, p) writes the tokens of part p that belong to rows [r kMaxRange, (r +
// 1) kMaxRange).  It counts its rows' tokens in all parts by itself.
template <typename Id>
__global__ void __launch_bounds__(kSortThreads)
    k_sort_ids(const Id* __restrict__ ids, int T, int64_t V, int parts, int* __restrict__ start,
               int* __restrict__ order) {
  // counts of the own part's tokens by wave, of those of the parts before it and after it
  __shared__ int counts[kSortLds / 4];
  __shared__ int less_of[kSortWaves], sums[kSortWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int* const mine = counts + wave * kMaxRange;
  int* const before = counts + kSortWaves * kMaxRange;  // [row][copy]
  int* const after = before + kCopies * kMaxRange;
  const int p = blockIdx.x % parts;
  const int lo = (int)(blockIdx.x / parts) * kMaxRange;
  const int rows = (int)(V - lo < kMaxRange ? V - lo : kMaxRange);
  for (int i = threadIdx.x; i < kSortLds / 16; i += kSortThreads)
    reinterpret_cast<u32x4*>(counts)[i] = u32x4{0u, 0u, 0u, 0u};
  __syncthreads();

  // part q: tokens [16 q sub, 16 (q + 1) sub), wave w its w-th sixteenth, of whole groups
  const int sub = ((T + parts * kSortWaves - 1) / (parts * kSortWaves) + 63) & ~63;
  const int groups = sub / 64;
  // The rows of kSortSteps groups, those of part q from group f on and then those of
  // the next parts.  All loads go out before the first id is looked at (where there is
  // no token the last one is read).  What is no row, or no token, compares above every row.
  auto read = [&](int q, int f, int(&row)[kSortSteps], int(&part)[kSortSteps]) {
    Id id[kSortSteps];
    unsigned at[kSortSteps];
#pragma unroll
    for (int u = 0; u < kSortSteps; ++u) {
      at[u] = q < parts ? (unsigned)((q * kSortWaves + wave) * sub + f * 64) + lane : ~0u;
      id[u] = ids[at[u] < (unsigned)T ? at[u] : (unsigned)T - 1];
      part[u] = q;
      if (++f == groups) f = 0, ++q;
    }
#pragma unroll
    for (int u = 0; u < kSortSteps; ++u)
      row[u] = at[u] < (unsigned)T && (uint64_t)(int64_t)id[u] < (uint64_t)V ? (int)id[u] : 0x7fffffff;
  };
  int less = 0;
  for (int g = 0; g < parts * groups && T > 0; g += kSortSteps) {
    int row[kSortSteps], part[kSortSteps];
    read(g / groups, g % groups, row, part);
#pragma unroll
    for (int u = 0; u < kSortSteps; ++u) {
      less += row[u] < lo;
      const unsigned rel = (unsigned)(row[u] - lo);
      const bool own = part[u] == p;
      const int from = own ? wave * kMaxRange : kSortWaves * kMaxRange + (part[u] < p ? 0 : kCopies * kMaxRange);
      if (rel < (unsigned)rows) atomicAdd(&counts[from + (own ? rel : rel * kCopies + lane % kCopies)], 1);
    }
  }
  for (int o = 32; o; o >>= 1) less += __shfl_xor(less, o);
  if (lane == 0) less_of[wave] = less;
  __syncthreads();

  // counts -> places: rows in order, and within a row the parts, then the waves
  const int i = threadIdx.x;
  int own[kSortWaves], earlier = 0, total = 0;
  if (i < rows) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) own[w] = counts[w * kMaxRange + i], total += own[w];
#pragma unroll
    for (int k = 0; k < kCopies; ++k) earlier += before[i * kCopies + k], total += after[i * kCopies + k];
    total += earlier;
  }
  int upto = total;
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int place = upto - total;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    place += less_of[w];
    if (w < wave) place += sums[w];
  }
  if (i < rows) {
    if (p == 0) {
      start[lo + i] = place;
      if (lo + i == V - 1) start[V] = place + total;
    }
    place += earlier;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      counts[w * kMaxRange + i] = place;
      place += own[w];
    }
  }
  __syncthreads();

  for (int f = 0; f < groups && T > 0; f += kSortSteps) {
    int row[kSortSteps], part[kSortSteps];
    read(p, f, row, part);
#pragma unroll
    for (int u = 0; u < kSortSteps; ++u) {
      const unsigned rel = (unsigned)(row[u] - lo);
      const bool in = rel < (unsigned)rows && part[u] == p;
      if (__ballot(in)) {
        const int at = take_place(mine, in, in ? (int)rel : 0);
        if (in) order[at] = (p * kSortWaves + wave) * sub + (f + u) * 64 + lane;
      }
    }
  }
}

// A wave of the two kernels below works on 64 pieces of E columns of one row.  Which
// row and which of its `per` waves: one binary64 product, as in locate().
struct WaveRow {
  int64_t row;
  int sub;
};
__device__ __forceinline__ WaveRow wave_row(unsigned group, int per, double inv_per) {
  const int64_t w = (int64_t)group * (kEmbedThreads / 64) + (threadIdx.x >> 6);
  int64_t row = (int64_t)((double)w * inv_per);
  int64_t sub = w - row * per;
  if (sub < 0) --row, sub += per;
  else if (sub >= per) ++row, sub -= per;
  return {__builtin_amdgcn_readfirstlane((int)row), __builtin_amdgcn_readfirstlane((int)sub)};
}

// First column of piece c of C: the row's last piece starts E before its end.
// Lanes past the last piece repeat it and store nothing.
template <int E>
__device__ __forceinline__ int64_t piece_column(int c, int C, int64_t D) {
  return c < C - 1 ? (int64_t)c * E : D - E;
}

// acc += the elements of N rows, in their order; all loads go out before the first
// addition.  The rows' addresses are the same in all lanes, `at` is the lane's own.
template <int DT, int E, int N>
__device__ __forceinline__ void add_rows(const char* const (&rows)[N], unsigned at, float (&acc)[E]) {
  float v[N][E];
#pragma unroll
  for (int u = 0; u < N; ++u) load_elems<DT, E>(rows[u] + at * dt_size<DT>(), 0, v[u]);
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] += v[u][i];
}

// Adds the rows of dy at positions [p, end) of the order to acc, in this order.  The
// wave reads its positions' tokens 64 at a time, one a lane, and has the rows of up to 32
// registers in flight.  p and end are the same in all lanes.
template <int GT, int E>
__device__ __forceinline__ void add_tokens(const char* dy, const int* order, int p, int end, int64_t D, unsigned d,
                                           float (&acc)[E]) {
  constexpr int kMost = E == 8 ? 4 : 8;
  const int lane = threadIdx.x & 63;
  for (; p < end; p += 64) {
    const int n = end - p < 64 ? end - p : 64;
    const int tokens = lane < n ? order[p + lane] : 0;
    auto batch = [&](int b, auto count) {
      constexpr int N = decltype(count)::value;
      const char* rows[N];
#pragma unroll
      for (int u = 0; u < N; ++u)
        rows[u] = dy + (int64_t)__builtin_amdgcn_readlane(tokens, b + u) * (D * dt_size<GT>());
      add_rows<GT, E, N>(rows, d, acc);
    };
    int b = 0;
    for (; b + kMost <= n; b += kMost) batch(b, std::integral_constant<int, kMost>{});
    if constexpr (kMost > 4)
      if (n - b >= 4) batch(b, std::integral_constant<int, 4>{}), b += 4;
    if (n - b >= 2) batch(b, std::integral_constant<int, 2>{}), b += 2;
    if (n - b >= 1) batch(b, std::integral_constant<int, 1>{});
  }
}

// Writes E columns of row `row` of the result: scale * acc, or that added to what is
// there.  The result goes past the caches: it is read again only once it is whole, and
// its writing otherwise costs the reads of dy their place (50,000 x 6,144 in binary32,
// 16,384 tokens, dy in the cache: 348 us with plain stores, 215 so; with two or four
// pieces a lane 248 and 264).
template <int YT, int E, bool ADD>
__device__ __forceinline__ void put_row(void* dw, int64_t row, int64_t D, int c, int C, unsigned d, float scale,
                                        float (&acc)[E]) {
#pragma unroll
  for (int i = 0; i < E; ++i) acc[i] = scale * acc[i];
  if (c >= C) return;
  if constexpr (ADD) {
    // where E does not divide D the row's last piece overlaps the one before it: the
    // shared elements are that one's to add
    const int skip = c == C - 1 ? (int)((int64_t)C * E - D) : 0;
    float old[E];
    load_elems<YT, E>(dw, row * D + d, old);
    if (skip == 0) {
#pragma unroll
      for (int i = 0; i < E; ++i) acc[i] = old[i] + acc[i];
      store_elems<YT, E>(dw, row * D + d, acc);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        if (i < skip) continue;
        const float one[1] = {old[i] + acc[i]};
        store_elems<YT, 1>(dw, row * D + d + i, one);
      }
    }
  } else {
    store_elems<YT, E, true>(dw, row * D + d, acc);
  }
}

// Segment j of the order: kPart positions from j kPart on.  A row that holds a whole
// segment is a long row: its sum is that of its first segment's part, its whole
// segments and its last segment's part, each summed apart: the whole ones and last parts
// in parts[2 j], first parts in parts[2 j + 1].
__device__ __forceinline__ bool is_long(int s, int e) { return (s + kPart - 1) / kPart < e / kPart; }

// Waves of the first seg_groups workgroups sum the long rows' segments, the others
// write the rows that are not long.
template <int GT, int YT, int E, bool ADD>
__global__ void __launch_bounds__(kEmbedThreads)
    k_grad_rows(unsigned first, const void* __restrict__ ids, bool wide, const char* __restrict__ dy,
                const int* __restrict__ start, const int* __restrict__ order, int segs, unsigned seg_groups,
                float* __restrict__ parts, int64_t V, int64_t D, int C, int per, double inv_per, float scale,
                void* __restrict__ dw) {
  const unsigned group = first + blockIdx.x;
  const bool seg = group < seg_groups;
  const WaveRow w = wave_row(seg ? group : group - seg_groups, per, inv_per);
  const int c = w.sub * 64 + (threadIdx.x & 63);
  const unsigned d = (unsigned)piece_column<E>(c, C, D);
  if (seg) {
    const int p0 = (int)w.row * kPart, all = start[V];
    if (w.row >= segs || p0 >= all) return;
    const int p1 = p0 + kPart < all ? p0 + kPart : all;
    const int64_t a = id_at(ids, wide, order[p0]), b = id_at(ids, wide, order[p1 - 1]);
    const int sa = start[a], ea = start[a + 1], sb = start[b], eb = start[b + 1];
    float* out = parts + 2 * w.row * D + d;
    if (is_long(sa, ea)) {  // the whole segment, or what row a has left in it
      float acc[E] = {};
      add_tokens<GT, E>(dy, order, p0, ea < p1 ? ea : p1, D, d, acc);
      if (c < C) store_elems<ZQ_F32, E>(out, 0, acc);
    }
    if (a != b && is_long(sb, eb)) {  // the beginning of row b
      float acc[E] = {};
      add_tokens<GT, E>(dy, order, sb, p1, D, d, acc);
      if (c < C) store_elems<ZQ_F32, E>(out + D, 0, acc);
    }
    return;
  }
  if (w.row >= V) return;
  const int s = start[w.row], e = start[w.row + 1];
  if ((ADD && s == e) || is_long(s, e)) return;
  float acc[E] = {};
  add_tokens<GT, E>(dy, order, s, e, D, d, acc);
  put_row<YT, E, ADD>(dw, w.row, D, c, C, d, scale, acc);
}

// The long rows' sums, each by the waves of its first whole segment.
template <int YT, int E, bool ADD>
__global__ void __launch_bounds__(kEmbedThreads)
    k_grad_join(unsigned first, const void* __restrict__ ids, bool wide, const int* __restrict__ start,
                const int* __restrict__ order, int segs, const float* __restrict__ parts, int64_t V, int64_t D, int C,
                int per, double inv_per, float scale, void* __restrict__ dw) {
  const WaveRow w = wave_row(first + blockIdx.x, per, inv_per);
  const int j = (int)w.row, p0 = j * kPart;
  if (j >= segs || p0 + kPart > start[V]) return;
  const int64_t row = id_at(ids, wide, order[p0]);
  const int s = start[row], e = start[row + 1], j1 = e / kPart;
  if ((s + kPart - 1) / kPart != j || j >= j1) return;
  const int c = w.sub * 64 + (threadIdx.x & 63);
  const unsigned d = (unsigned)piece_column<E>(c, C, D);
  float acc[E] = {};
  auto add_parts = [&](int64_t k, auto count) {  // parts[k], parts[k + 2], ..
    constexpr int N = decltype(count)::value;
    const char* rows[N];
#pragma unroll
    for (int u = 0; u < N; ++u) rows[u] = reinterpret_cast<const char*>(parts + (k + 2 * u) * D);
    add_rows<ZQ_F32, E, N>(rows, d, acc);
  };
  if (s < p0) add_parts(2 * (int64_t)j - 1, std::integral_constant<int, 1>{});
  int k = j;
  const int end = e > j1 * kPart ? j1 + 1 : j1;  // with the last part
  for (; k + 16 <= end; k += 16) add_parts(2 * (int64_t)k, std::integral_constant<int, 16>{});
  for (; k + 4 <= end; k += 4) add_parts(2 * (int64_t)k, std::integral_constant<int, 4>{});
  for (; k < end; ++k) add_parts(2 * (int64_t)k, std::integral_constant<int, 1>{});
  put_row<YT, E, ADD>(dw, row, D, c, C, d, scale, acc);
}

// ---- few tokens: one launch
//
// A workgroup has up to kFewRows rows and the columns of 4 waves' pieces, 8 KiB or a little
// more of the result: it is written fastest in the order of its addresses, and workgroups
// are few enough to look through all ids each (512 tokens, 8,000 x 1,024 in binary32: 9 us,
// in 16 KiB 13.7, in 32 KiB 20; in three launches 15.5).  It marks its rows' tokens, a bit
// each, in LDS: the bits of a row in their order are its tokens in theirs.
constexpr int kFewTokens = 512, kFewWords = kFewTokens / 32;
constexpr int kFewRows = 64;
constexpr int64_t kFewBytes = 8192;
constexpr int kEmbedWaves = kEmbedThreads / 64;
template <int GT, int YT, int E, bool ADD>
__global__ void __launch_bounds__(kEmbedThreads)
    k_grad_few(const void* __restrict__ ids, bool wide, int T, const char* __restrict__ dy, int64_t V, int64_t D, int C,
               int per, unsigned cols, int rb, float scale, void* __restrict__ dw) {
  __shared__ uint32_t marks[kFewRows * kFewWords];
  __shared__ int counts[kFewRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned block = blockIdx.x / cols, col = blockIdx.x - block * cols;
  const int64_t row0 = (int64_t)block * rb;
  const int n = (int)(V - row0 < rb ? V - row0 : rb);
  int64_t id[kFewTokens / kEmbedThreads];
#pragma unroll
  for (int u = 0; u < kFewTokens / kEmbedThreads; ++u) {
    const int t = u * kEmbedThreads + (int)threadIdx.x;
    id[u] = t < T ? id_at(ids, wide, t) : -1;
  }
  for (int i = threadIdx.x; i < n * kFewWords; i += kEmbedThreads) marks[i] = 0;
  if (threadIdx.x < kFewRows) counts[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kFewTokens / kEmbedThreads; ++u) {
    const uint64_t rel = (uint64_t)(id[u] - row0);
    if (id[u] >= 0 && rel < (uint64_t)n) {
      const int t = u * kEmbedThreads + (int)threadIdx.x;
      atomicOr(&marks[(int)rel * kFewWords + t / 32], 1u << (t & 31));
      atomicAdd(&counts[(int)rel], 1);
    }
  }
  __syncthreads();
  const int tokens_of = counts[lane];

  // the 4 waves take the (row, piece) pairs in turn
  const int first = (int)col * kEmbedWaves, subs = per - first < kEmbedWaves ? per - first : kEmbedWaves;
  const unsigned inv = 65536u / (unsigned)subs + 1u;  // exact for the 256 pairs
  for (int i = wave; i < n * subs; i += kEmbedWaves) {
    const int row = (int)((unsigned)i * inv >> 16), sub = i - row * subs;
    const int c = (first + sub) * 64 + lane;
    const unsigned d = (unsigned)piece_column<E>(c, C, D);
    int left = __builtin_amdgcn_readlane(tokens_of, row);
    if (ADD && left == 0) continue;
    float acc[E] = {};
    if (left > 0) {
      const uint32_t word = lane < kFewWords ? marks[row * kFewWords + lane] : 0u;
      uint64_t words = __ballot(word != 0);
      uint32_t bits = 0;
      int at = 0;
      auto next = [&] {  // the next token of the row
        if (bits == 0) {
          at = __builtin_ctzll(words);
          words &= words - 1;
          bits = (uint32_t)__builtin_amdgcn_readlane((int)word, at);
        }
        const int t = at * 32 + __builtin_ctz(bits);
        bits &= bits - 1;
        return t;
      };
      auto batch = [&](auto size) {
        constexpr int N = decltype(size)::value;
        const char* rows[N];
#pragma unroll
        for (int u = 0; u < N; ++u) rows[u] = dy + (int64_t)next() * (D * dt_size<GT>());
        add_rows<GT, E, N>(rows, d, acc);
        left -= N;
      };
      if constexpr (E < 8)
        while (left >= 16) batch(std::integral_constant<int, 16>{});
      while (left >= 8) batch(std::integral_constant<int, 8>{});
      if (left >= 4) batch(std::integral_constant<int, 4>{});
      if (left >= 2) batch(std::integral_constant<int, 2>{});
      if (left >= 1) batch(std::integral_constant<int, 1>{});
    }
    put_row<YT, E, ADD>(dw, row0 + row, D, c, C, d, scale, acc);
  }
}

// ---------------------------------------------------------------- dispatch

using EmbedKernel = void (*)(unsigned, const void*, bool, const void*, const float*, int64_t, int64_t, int64_t, int,
                             double, int, float, void*);
// columns of a piece: 16 bytes of the result (1 column where rows are shorter than 8)
template <int YT>
constexpr int piece_of() {
  return 16 / dt_size<YT>();
}
// of the lookup: 32 bytes where both sides are binary32 (16,384 x 6,144: 108 us, 126 with 16)
constexpr int lookup_piece(int wt, int yt) { return wt == ZQ_F32 || yt != ZQ_F32 ? 8 : 4; }
template <int WT, int YT>
EmbedKernel embed_kernel_for(bool short_rows) {
  return short_rows ? &k_embed<WT, YT, 1> : &k_embed<WT, YT, lookup_piece(WT, YT)>;
}
template <int WT>
EmbedKernel embed_kernel_to(int yt, bool short_rows) {
  return yt == ZQ_F32   ? embed_kernel_for<WT, ZQ_F32>(short_rows)
         : yt == ZQ_F16 ? embed_kernel_for<WT, ZQ_F16>(short_rows)
                        : embed_kernel_for<WT, ZQ_BF16>(short_rows);
}
EmbedKernel embed_kernel(int wt, int yt, bool short_rows) {
  return wt == kInt8    ? embed_kernel_to<kInt8>(yt, short_rows)
         : wt == ZQ_F32 ? embed_kernel_to<ZQ_F32>(yt, short_rows)
         : wt == ZQ_F16 ? embed_kernel_to<ZQ_F16>(yt, short_rows)
                        : embed_kernel_to<ZQ_BF16>(yt, short_rows);
}

using RowsKernel = void (*)(unsigned, const void*, bool, const char*, const int*, const int*, int, unsigned, float*,
                            int64_t, int64_t, int, int, double, float, void*);
using JoinKernel = void (*)(unsigned, const void*, bool, const int*, const int*, int, const float*, int64_t, int64_t,
                            int, int, double, float, void*);
template <int GT, int YT, int E>
RowsKernel rows_kernel_add(bool add) {
  return add ? &k_grad_rows<GT, YT, E, true> : &k_grad_rows<GT, YT, E, false>;
}
template <int YT, int E>
JoinKernel join_kernel_add(bool add) {
  return add ? &k_grad_join<YT, E, true> : &k_grad_join<YT, E, false>;
}
template <int GT, int YT>
RowsKernel rows_kernel_for(bool short_rows, bool add) {
  return short_rows ? rows_kernel_add<GT, YT, 1>(add) : rows_kernel_add<GT, YT, piece_of<YT>()>(add);
}
template <int GT>
RowsKernel rows_kernel_to(int yt, bool short_rows, bool add) {
  return yt == ZQ_F32   ? rows_kernel_for<GT, ZQ_F32>(short_rows, add)
         : yt == ZQ_F16 ? rows_kernel_for<GT, ZQ_F16>(short_rows, add)
                        : rows_kernel_for<GT, ZQ_BF16>(short_rows, add);
}
RowsKernel rows_kernel(int gt, int yt, bool short_rows, bool add) {
  return gt == ZQ_F32   ? rows_kernel_to<ZQ_F32>(yt, short_rows, add)
         : gt == ZQ_F16 ? rows_kernel_to<ZQ_F16>(yt, short_rows, add)
                        : rows_kernel_to<ZQ_BF16>(yt, short_rows, add);
}

using FewKernel = void (*)(const void*, bool, int, const char*, int64_t, int64_t, int, int, unsigned, int, float, void*);
template <int GT, int YT, int E>
FewKernel few_kernel_add(bool add) {
  return add ? &k_grad_few<GT, YT, E, true> : &k_grad_few<GT, YT, E, false>;
}
template <int GT, int YT>
FewKernel few_kernel_for(bool short_rows, bool add) {
  return short_rows ? few_kernel_add<GT, YT, 1>(add) : few_kernel_add<GT, YT, piece_of<YT>()>(add);
}
template <int GT>
FewKernel few_kernel_to(int yt, bool short_rows, bool add) {
  return yt == ZQ_F32   ? few_kernel_for<GT, ZQ_F32>(short_rows, add)
         : yt == ZQ_F16 ? few_kernel_for<GT, ZQ_F16>(short_rows, add)
                        : few_kernel_for<GT, ZQ_BF16>(short_rows, add);
}
FewKernel few_kernel(int gt, int yt, bool short_rows, bool add) {
  return gt == ZQ_F32   ? few_kernel_to<ZQ_F32>(yt, short_rows, add)
         : gt == ZQ_F16 ? few_kernel_to<ZQ_F16>(yt, short_rows, add)
                        : few_kernel_to<ZQ_BF16>(yt, short_rows, add);
}

template <int YT>
JoinKernel join_kernel_for(bool short_rows, bool add) {
  return short_rows ? join_kernel_add<YT, 1>(add) : join_kernel_add<YT, piece_of<YT>()>(add);
}
JoinKernel join_kernel(int yt, bool short_rows, bool add) {
  return yt == ZQ_F32   ? join_kernel_for<ZQ_F32>(short_rows, add)
         : yt == ZQ_F16 ? join_kernel_for<ZQ_F16>(short_rows, add)
                        : join_kernel_for<ZQ_BF16>(short_rows, add);
}

constexpr int64_t kMaxRow = 1 << 24;  // elements of a table row

int embed(const void* ids, int it, int64_t T, const void* table, const float* scales, int wt, int64_t V, int64_t D,
          int32_t block, float scale, void* y, int yt, void* stream) {
  if (T < 0 || V < 0 || D < 0 || D > kMaxRow) return ZQ_E_SIZE;
  const int lgB = wt == kInt8 ? log2_block(block) : 0;
  if (lgB < 0) return ZQ_E_BLOCK;
  if ((it != ZQ_I32 && it != ZQ_I64) || (wt != kInt8 && !dtype_ok(wt)) || !dtype_ok(yt)) return ZQ_E_DTYPE;
  if (T == 0 || D == 0) return ZQ_OK;
  if (!ids || !y || (V > 0 && (!table || (wt == kInt8 && !scales)))) return ZQ_E_NULL;
  const int64_t ib = it == ZQ_I64 ? 8 : 4, wb = wt == kInt8 ? 1 : elem_bytes(wt);
  if (!aligned(ids, ib) || !aligned(table, wb) || !aligned(scales, 4) || !aligned(y, elem_bytes(yt))) return ZQ_E_ALIGN;
  if (V > INT64_MAX / 8 / D || T > INT64_MAX / 8 / D) return ZQ_E_SIZE;
  if (any_overlap({{y, T * D * elem_bytes(yt)}},
                  {{ids, T * ib}, {table, V * D * wb}, {scales, wt == kInt8 ? 4 * num_scales(V * D, block) : 0}}))
    return ZQ_E_ALIAS;
  const bool short_rows = D < 8;
  const int64_t E = short_rows ? 1 : lookup_piece(wt, yt), C = (D + E - 1) / E;
  const int64_t grid = grid_for(T * C, kEmbedThreads);
  if (grid == 0) return ZQ_E_SIZE;
  return launch_parts(embed_kernel(wt, yt, short_rows), grid, kEmbedThreads, static_cast<hipStream_t>(stream), ids,
                      it == ZQ_I64, table, scales, T, V, D, (int)C, 1.0 / (double)C, lgB, scale, y);
}

// One launch for few tokens, unless the result is so large that the order it is written
// in outweighs two launches (512 tokens, three launches and one: 400 MB in binary32 67 and
// 64 us, 524 MB 112 and 103; 1.2 GB 179 and 208, 614 MB in bf16 94 and 107).  A row's
// tokens are added by the same lanes one after the other: 512 tokens of one row of 6,144
// columns 45 us, 38 in three launches; 1,024 tokens took 100.
bool in_one_launch(int64_t T, int64_t V, int64_t D) { return T <= kFewTokens && (D == 0 || V <= (1 << 27) / D); }

int64_t ranges_of(int64_t V) { return (V + kMaxRange - 1) / kMaxRange; }

// Workspace of the gradient: first positions (V + 1), the order (T), the segments'
// sums (2 rows of D each), each from a 16-byte boundary on.
int64_t up16(int64_t b) { return (b + 15) & ~(int64_t)15; }
int64_t start_bytes(int64_t V) { return up16(4 * (V + 1)); }
int64_t order_bytes(int64_t T) { return up16(4 * T); }

}  // namespace
}  // namespace zq

extern "C" {

using namespace zq;

int zq_embedding(const void* ids, zq_dtype it, int64_t T, const void* table, zq_dtype wt, int64_t V, int64_t D,
                 float scale, void* y, zq_dtype yt, void* stream) {
  if (!dtype_ok(wt)) return ZQ_E_DTYPE;
  return embed(ids, it, T, table, nullptr, wt, V, D, 0, scale, y, yt, stream);
}

int qwz_embedding(const void* ids, zq_dtype it, int64_t T, const int8_t* codes, const float* scales, int64_t V,
                  int64_t D, int32_t block, float scale, void* y, zq_dtype yt, void* stream) {
  return embed(ids, it, T, codes, scales, kInt8, V, D, block, scale, y, yt, stream);
}

int64_t zq_embedding_grad_bytes(int64_t T, int64_t V, int64_t D) {
  if (T < 0 || T > kMaxTokens || V < 0 || V > kMaxTokens || D < 0 || D > kMaxRow) return -1;
  if (in_one_launch(T, V, D)) return 0;
  if (T * ranges_of(V) > kMaxReads) return -1;
  return start_bytes(V) + order_bytes(T) + (T < kPart ? 0 : 8 * ((T + kPart - 1) / kPart) * D);
}

int zq_embedding_grad(const void* ids, zq_dtype it, int64_t T, const void* dy, zq_dtype gt, int64_t V, int64_t D,
                      float scale, int accumulate, void* dw, zq_dtype wt, void* workspace, int64_t workspace_bytes,
                      void* stream) {
  const int64_t need = zq_embedding_grad_bytes(T, V, D);
  if (need < 0) return ZQ_E_SIZE;
  if ((it != ZQ_I32 && it != ZQ_I64) || !dtype_ok(gt) || !dtype_ok(wt)) return ZQ_E_DTYPE;
  if (V == 0 || D == 0 || (accumulate && T == 0)) return ZQ_OK;
  if (!dw || (need > 0 && !workspace) || (T > 0 && (!ids || !dy))) return ZQ_E_NULL;
  const int64_t ib = it == ZQ_I64 ? 8 : 4;
  if (!aligned(ids, ib) || !aligned(dy, elem_bytes(gt)) || !aligned(dw, elem_bytes(wt)) ||
      (need > 0 && !aligned(workspace, 16)))
    return ZQ_E_ALIGN;
  if (workspace_bytes < need) return ZQ_E_SIZE;
  if (any_overlap({{dw, V * D * elem_bytes(wt)}, {workspace, need}}, {{ids, T * ib}, {dy, T * D * elem_bytes(gt)}}))
    return ZQ_E_ALIAS;

  char* ws = static_cast<char*>(workspace);
  int* start = reinterpret_cast<int*>(ws);
  int* order = reinterpret_cast<int*>(ws + start_bytes(V));
  float* sums = reinterpret_cast<float*>(ws + start_bytes(V) + order_bytes(T));
  // waves of a row: 64 pieces each
  const bool short_rows = D < 8, add = accumulate != 0;
  const int64_t E = short_rows ? 1 : wt == ZQ_F32 ? 4 : 8, C = (D + E - 1) / E, per = (C + 63) / 64;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (in_one_launch(T, V, D)) {
    const int64_t cols = (per + kEmbedWaves - 1) / kEmbedWaves;
    const int64_t bytes = (D < 64 * kEmbedWaves * E ? D : 64 * kEmbedWaves * E) * elem_bytes(wt);  // of a row
    int64_t rb = kFewBytes / bytes;
    if (rb < 1) rb = 1;
    if (rb > kFewRows) rb = kFewRows;
    const int64_t grid = (V + rb - 1) / rb * cols;
    return launch(few_kernel(gt, wt, short_rows, add), (unsigned)grid, kEmbedThreads, st, ids, it == ZQ_I64, (int)T,
                  static_cast<const char*>(dy), V, D, (int)C, (int)per, (unsigned)cols, (int)rb, scale, dw);
  }
  // no row is long with fewer tokens than a segment
  const int64_t segs = T < kPart ? 0 : (T + kPart - 1) / kPart;
  const int64_t seg_groups = segs ? grid_for(segs * per, kEmbedThreads / 64) : 0;
  const int64_t row_groups = grid_for(V * per, kEmbedThreads / 64);
  if (row_groups == 0 || (segs && seg_groups == 0) || row_groups + seg_groups > kMaxGrid) return ZQ_E_SIZE;
  // Sorting workgroups: ranges of 512 rows, times parts of the tokens.  Every
  // workgroup reads all ids (about T ranges parts 4e-7 us; 8.5e-7 for millions of ids,
  // which come from further away), while the parts share out
  // the work on the tokens of a range that most tokens fall into (T / parts 6e-4 us):
  // the least sum is at the square root of 1,700 / ranges.
  const int64_t ranges = ranges_of(V);
  int parts = 1;
  while (parts < 16 && (int64_t)(parts + 1) * 1024 <= T && (2 * parts + 1) * (2 * parts + 1) * ranges < 4 * 1700) ++parts;
  const int64_t sorts = ranges * parts;
  if (sorts > kMaxGrid) return ZQ_E_SIZE;
  int rc = it == ZQ_I64 ? launch(&k_sort_ids<int64_t>, (unsigned)sorts, kSortThreads, st,
                                 static_cast<const int64_t*>(ids), (int)T, V, parts, start, order)
                        : launch(&k_sort_ids<int32_t>, (unsigned)sorts, kSortThreads, st,
                                 static_cast<const int32_t*>(ids), (int)T, V, parts, start, order);
  if (rc != ZQ_OK) return rc;
  rc = launch_parts(rows_kernel(gt, wt, short_rows, add), row_groups + seg_groups, kEmbedThreads, st, ids, it == ZQ_I64,
                    static_cast<const char*>(dy), start, order, (int)segs, (unsigned)seg_groups, sums, V, D, (int)C,
                    (int)per, 1.0 / (double)per, scale, dw);
  if (rc != ZQ_OK || segs == 0) return rc;
  return launch_parts(join_kernel(wt, short_rows, add), seg_groups, kEmbedThreads, st, ids, it == ZQ_I64, start, order,
                      (int)segs, sums, V, D, (int)C, (int)per, 1.0 / (double)per, scale, dw);
}

}  // extern "C"
