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
#include <hip/hip_runtime.h>
#include <stdint.h>

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

// A thread moves E elements of one token's row.  The last piece of a row starts
// E before its end (it repeats elements of the piece before it where E does not
// divide D); E = 1 serves rows shorter than 8.
template <int WT, int YT, int E>
__global__ void __launch_bounds__(kEmbedThreads)
    k_embed(const void* __restrict__ ids, bool wide, const void* __restrict__ table, const float* __restrict__ scales,
            int64_t T, int64_t V, int64_t D, int C, double inv_c, int lgB, float scale, void* __restrict__ y) {
  const Piece p = locate(blockIdx.x, C, inv_c);
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
  store_elems<YT, E>(y, p.row * D + d, v);
}

// ---------------------------------------------------------------- gradient
//
// 1. k_sort_ids: the tokens in the order of their ids, ties in the order of the
//    tokens, and each row's first position in that order.  A workgroup owns a
//    range of rows and reads all ids twice (they come from L2: 16,384 of them
//    are 128 KiB): first it counts its rows' tokens, and those of the rows
//    before its own, which gives its place in the order without another
//    workgroup's count; then it writes its tokens.  Wave w takes the w-th
//    sixteenth of the tokens in both, so waves need no order among themselves
//    but their counts'.
// 2. k_grad_parts: the sums of 64 consecutive positions, where all of them
//    belong to one row.  Rows of frequent tokens are thus summed by as many
//    workgroups as they have 64s of tokens.
// 3. k_grad_rows: each row's tokens up to a multiple of 64, the sums of its
//    64s, the tokens after them, in this order; rows without tokens are zero.
// The order of every sum follows from the ids alone: no atomics on sums.

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMaxRange = 512;   // rows of a workgroup's range (counts: 32 KiB of LDS)
constexpr int kPart = 64;        // positions of a partial sum
constexpr int64_t kMaxTokens = 1 << 30;

// Adds this lane's row to the wave's counts: the lanes of one row in one step.
// Returns the row's count before this group's, plus the lanes of the row
// before this one (the lane's place among the row's tokens of this wave).
__device__ __forceinline__ int take_place(int* counts, bool in, int row, int bits) {
  const int lane = threadIdx.x & 63;
  uint64_t peers = __ballot(in);
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot(row >> b & 1);
    peers &= row >> b & 1 ? set : ~set;
  }
  int place = 0;
  if (in) {
    const int before = __popcll(peers & ((1ull << lane) - 1));
    const int base = counts[row];
    place = base + before;
    if (before == 0) counts[row] = base + __popcll(peers);
  }
  // the next group's reads come after this group's writes
  __builtin_amdgcn_wave_barrier();
  return place;
}

__global__ void __launch_bounds__(kSortThreads)
    k_sort_ids(const void* __restrict__ ids, bool wide, int T, int64_t V, int range, int bits, int* __restrict__ start,
               int* __restrict__ order) {
  extern __shared__ int counts[];  // kSortWaves x range
  __shared__ int before[kSortWaves], sums[kSortWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t lo = (int64_t)blockIdx.x * range;
  const int rows = (int)(V - lo < range ? V - lo : range);
  int* mine = counts + wave * range;
  for (int i = threadIdx.x; i < kSortWaves * range; i += kSortThreads) counts[i] = 0;
  __syncthreads();

  const int part = ((T + kSortWaves - 1) / kSortWaves + 63) & ~63;
  const int64_t t0 = (int64_t)wave * part, t1 = t0 + part < T ? t0 + part : T;
  int less = 0;
  for (int64_t t = t0 + lane; t - lane < t1; t += 64) {
    const int64_t id = t < t1 ? id_at(ids, wide, t) : -1;
    const bool in = id >= lo && id < lo + rows;
    less += id >= 0 && id < lo;
    if (__ballot(in)) take_place(mine, in, in ? (int)(id - lo) : 0, bits);
  }
  for (int o = 32; o; o >>= 1) less += __shfl_xor(less, o);
  if (lane == 0) before[wave] = less;
  __syncthreads();

  // counts -> places: rows in order, and within a row the waves
  int total = 0;
  if (threadIdx.x < (unsigned)rows)
    for (int w = 0; w < kSortWaves; ++w) total += counts[w * range + threadIdx.x];
  int upto = total;
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int place = upto - total;
  for (int w = 0; w < kSortWaves; ++w) {
    place += before[w];
    if (w < wave) place += sums[w];
  }
  if (threadIdx.x < (unsigned)rows) {
    start[lo + threadIdx.x] = place;
    if (lo + threadIdx.x == V - 1) start[V] = place + total;
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = counts[w * range + threadIdx.x];
      counts[w * range + threadIdx.x] = place;
      place += c;
    }
  }
  __syncthreads();

  for (int64_t t = t0 + lane; t - lane < t1; t += 64) {
    const int64_t id = t < t1 ? id_at(ids, wide, t) : -1;
    const bool in = id >= lo && id < lo + rows;
    if (__ballot(in)) {
      const int at = take_place(mine, in, in ? (int)(id - lo) : 0, bits);
      if (in) order[at] = (int)t;
    }
  }
}

// sum of the rows of dy at positions [p, end) of the order, from `acc` on
template <int GT, int E>
__device__ __forceinline__ void add_tokens(const void* dy, const int* order, int p, int end, int64_t D, int64_t d,
                                           float (&acc)[E]) {
  for (; p < end; ++p) {
    float v[E];
    load_elems<GT, E>(dy, (int64_t)order[p] * D + d, v);
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] += v[i];
  }
}

template <int GT, int E>
__global__ void __launch_bounds__(kEmbedThreads)
    k_grad_parts(const void* __restrict__ ids, bool wide, const void* __restrict__ dy, const int* __restrict__ start,
                 const int* __restrict__ order, int64_t V, int64_t D, int C, int cols, float* __restrict__ parts) {
  const int64_t j = blockIdx.x / cols;
  const int c = (int)(blockIdx.x % cols) * kEmbedThreads + threadIdx.x;
  const int64_t p0 = j * kPart;
  if (p0 + kPart > start[V]) return;
  if (id_at(ids, wide, order[p0]) != id_at(ids, wide, order[p0 + kPart - 1])) return;
  if (c >= C) return;
  const int64_t d0 = (int64_t)c * E, d = d0 + E > D ? D - E : d0;
  float acc[E];
#pragma unroll
  for (int i = 0; i < E; ++i) acc[i] = 0.0f;
  add_tokens<GT, E>(dy, order, (int)p0, (int)p0 + kPart, D, d, acc);
  store_elems<ZQ_F32, E>(parts, j * D + d, acc);
}

template <int GT, int YT, int E, bool ADD>
__global__ void __launch_bounds__(kEmbedThreads)
    k_grad_rows(const void* __restrict__ dy, const int* __restrict__ start, const int* __restrict__ order,
                const float* __restrict__ parts, int64_t V, int64_t D, int C, double inv_c, float scale,
                void* __restrict__ dw) {
  const Piece p = locate(blockIdx.x, C, inv_c);
  if (p.row >= V) return;
  const int s = start[p.row], e = start[p.row + 1];
  if (ADD && s == e) return;
  const int64_t d0 = (int64_t)p.piece * E;
  const int64_t d = d0 + E > D ? D - E : d0;
  float acc[E];
#pragma unroll
  for (int i = 0; i < E; ++i) acc[i] = 0.0f;
  if (s < e) {
    const int j0 = (s + kPart - 1) / kPart, j1 = e / kPart;
    if (j0 < j1) {
      add_tokens<GT, E>(dy, order, s, j0 * kPart, D, d, acc);
      for (int j = j0; j < j1; ++j) {
        float v[E];
        load_elems<ZQ_F32, E>(parts, (int64_t)j * D + d, v);
#pragma unroll
        for (int i = 0; i < E; ++i) acc[i] += v[i];
      }
      add_tokens<GT, E>(dy, order, j1 * kPart, e, D, d, acc);
    } else {
      add_tokens<GT, E>(dy, order, s, e, D, d, acc);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] = scale * acc[i];
  }
  if constexpr (ADD) {
    float old[E];
    // the row's last piece overlaps the one before it where E does not divide D:
    // the shared elements are the earlier piece's to add
    const int skip = (int)(d0 - d);
    load_elems<YT, E>(dw, p.row * D + d, old);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      if (i < skip) continue;
      float one[1] = {old[i] + acc[i]};
      store_elems<YT, 1>(dw, p.row * D + d + i, one);
    }
  } else {
    store_elems<YT, E>(dw, p.row * D + d, acc);
  }
}

// ---------------------------------------------------------------- dispatch

using EmbedKernel = void (*)(const void*, bool, const void*, const float*, int64_t, int64_t, int64_t, int, double, int,
                             float, void*);
template <int WT, int E>
EmbedKernel embed_kernel_to(int yt) {
  return yt == ZQ_F32 ? &k_embed<WT, ZQ_F32, E> : yt == ZQ_F16 ? &k_embed<WT, ZQ_F16, E> : &k_embed<WT, ZQ_BF16, E>;
}
template <int E>
EmbedKernel embed_kernel(int wt, int yt) {
  return wt == kInt8    ? embed_kernel_to<kInt8, E>(yt)
         : wt == ZQ_F32 ? embed_kernel_to<ZQ_F32, E>(yt)
         : wt == ZQ_F16 ? embed_kernel_to<ZQ_F16, E>(yt)
                        : embed_kernel_to<ZQ_BF16, E>(yt);
}

using PartsKernel = void (*)(const void*, bool, const void*, const int*, const int*, int64_t, int64_t, int, int,
                             float*);
template <int E>
PartsKernel parts_kernel(int gt) {
  return gt == ZQ_F32 ? &k_grad_parts<ZQ_F32, E> : gt == ZQ_F16 ? &k_grad_parts<ZQ_F16, E> : &k_grad_parts<ZQ_BF16, E>;
}
using RowsKernel = void (*)(const void*, const int*, const int*, const float*, int64_t, int64_t, int, double, float,
                            void*);
template <int GT, int YT, int E>
RowsKernel rows_kernel_add(bool add) {
  return add ? &k_grad_rows<GT, YT, E, true> : &k_grad_rows<GT, YT, E, false>;
}
template <int GT, int E>
RowsKernel rows_kernel_to(int yt, bool add) {
  return yt == ZQ_F32   ? rows_kernel_add<GT, ZQ_F32, E>(add)
         : yt == ZQ_F16 ? rows_kernel_add<GT, ZQ_F16, E>(add)
                        : rows_kernel_add<GT, ZQ_BF16, E>(add);
}
template <int E>
RowsKernel rows_kernel(int gt, int yt, bool add) {
  return gt == ZQ_F32   ? rows_kernel_to<ZQ_F32, E>(yt, add)
         : gt == ZQ_F16 ? rows_kernel_to<ZQ_F16, E>(yt, add)
                        : rows_kernel_to<ZQ_BF16, E>(yt, add);
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
  const int E = D < 8 ? 1 : 8;
  const int64_t C = (D + E - 1) / E;
  const int64_t grid = grid_for(T * C, kEmbedThreads);
  if (grid == 0) return ZQ_E_SIZE;
  return launch(E == 8 ? embed_kernel<8>(wt, yt) : embed_kernel<1>(wt, yt), (unsigned)grid, kEmbedThreads,
                static_cast<hipStream_t>(stream), ids, it == ZQ_I64, table, scales, T, V, D, (int)C, 1.0 / (double)C,
                lgB, scale, y);
}

// Workspace of the gradient: first positions (V + 1), the order (T), partial
// sums (T / 64 rows of D), each from a 16-byte boundary on.
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
  return start_bytes(V) + order_bytes(T) + 4 * (T / kPart) * D;
}

int zq_embedding_grad(const void* ids, zq_dtype it, int64_t T, const void* dy, zq_dtype gt, int64_t V, int64_t D,
                      float scale, int accumulate, void* dw, zq_dtype wt, void* workspace, int64_t workspace_bytes,
                      void* stream) {
  const int64_t need = zq_embedding_grad_bytes(T, V, D);
  if (need < 0) return ZQ_E_SIZE;
  if ((it != ZQ_I32 && it != ZQ_I64) || !dtype_ok(gt) || !dtype_ok(wt)) return ZQ_E_DTYPE;
  if (V == 0 || D == 0 || (accumulate && T == 0)) return ZQ_OK;
  if (!dw || !workspace || (T > 0 && (!ids || !dy))) return ZQ_E_NULL;
  const int64_t ib = it == ZQ_I64 ? 8 : 4;
  if (!aligned(ids, ib) || !aligned(dy, elem_bytes(gt)) || !aligned(dw, elem_bytes(wt)) || !aligned(workspace, 16))
    return ZQ_E_ALIGN;
  if (workspace_bytes < need) return ZQ_E_SIZE;
  if (any_overlap({{dw, V * D * elem_bytes(wt)}, {workspace, need}}, {{ids, T * ib}, {dy, T * D * elem_bytes(gt)}}))
    return ZQ_E_ALIAS;

  char* ws = static_cast<char*>(workspace);
  int* start = reinterpret_cast<int*>(ws);
  int* order = reinterpret_cast<int*>(ws + start_bytes(V));
  float* parts = reinterpret_cast<float*>(ws + start_bytes(V) + order_bytes(T));
  const int E = D < 8 ? 1 : 8;
  const int64_t C = (D + E - 1) / E, cols = (C + kEmbedThreads - 1) / kEmbedThreads;
  // rows of a sorting workgroup: a power of two that gives about 256 of them
  int range = 1, bits = 0;
  while (range < kMaxRange && (int64_t)range * 256 < V) range *= 2, ++bits;
  const int64_t sorts = (V + range - 1) / range, segs = T / kPart;
  const int64_t grid = grid_for(V * C, kEmbedThreads);
  if (grid == 0 || segs * cols > kMaxGrid) return ZQ_E_SIZE;

  hipStream_t st = static_cast<hipStream_t>(stream);
  int rc = launch_grid(&k_sort_ids, dim3((unsigned)sorts), kSortThreads, kSortWaves * range * 4, st, ids, it == ZQ_I64, (int)T,
                      V, range, bits, start, order);
  if (rc != ZQ_OK) return rc;
  if (segs > 0) {
    rc = launch(E == 8 ? parts_kernel<8>(gt) : parts_kernel<1>(gt), (unsigned)(segs * cols), kEmbedThreads, st, ids,
                it == ZQ_I64, dy, start, order, V, D, (int)C, (int)cols, parts);
    if (rc != ZQ_OK) return rc;
  }
  return launch(E == 8 ? rows_kernel<8>(gt, wt, accumulate != 0) : rows_kernel<1>(gt, wt, accumulate != 0),
                (unsigned)grid, kEmbedThreads, st, dy, start, order, parts, V, D, (int)C, 1.0 / (double)C, scale, dw);
}

}  // extern "C"
