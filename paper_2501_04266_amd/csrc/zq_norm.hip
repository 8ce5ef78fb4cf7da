// zq_norm.hip -- the norm of a rank's gradients and their clipping, on gfx950.
//
//   norm = |scale| * sqrt(sum over all tensors of sum g^2)
//   c    = fl(scale * min(1, fl(max_norm / fl(norm + 1e-6))))
//   out  = cvt(fl(g * c))
//
// g are the elements of dense tensors, or q * s of INT4 shards as the reduce
// levels leave them.  An INT4 shard needs no dequantised copy for either: its
// sum is sum_b s_b^2 sum_{i in b} q_i^2, the inner sum in whole numbers (one
// v_dot8_i32_i4 for 8 codes), and clipping it means scaling its scales.
//
// Bound by memory: each byte is read once (and, clipping, written once).  The norm
// of 1.2 billion bf16 elements takes 360 us (6.7 TB/s), of 906 million INT4 codes 75
// (6.4 TB/s); a second launch of 2 to 4 us adds the workgroups' sums.  The
// squares are summed in binary64, exactly squared binary32 values, so neither
// overflow nor underflow of a square is met and the order of the sums does not
// show in the binary32 result except by one rounding; the order is fixed all
// the same.
//
// One launch covers all tensors: the table holds an entry per tensor with the
// index of its first chunk (16 KiB of data), workgroup w takes the chunks [w n / W,
// (w + 1) n / W) of all n and finds its first tensor by comparing against all entries
// at once.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "zq.h"
#include "zq_device.h"
#include "zq_host.h"
#include "zq_spans.h"
#include "zq_vec.h"

#pragma clang fp contract(off)

namespace zq {
namespace {

constexpr int kNormThreads = 256;
constexpr int kNormGroups = 2048;     // workgroups at most: 8 a CU
constexpr int64_t kChunkBytes = 16384;  // data of a chunk
constexpr int kInt4 = 3;              // type code of an entry's INT4 data

// One tensor of the table.  Read by every workgroup, so 48 bytes.
struct Entry {
  const char* data;
  const float* scales;
  char* out;
  int64_t n;        // elements
  int64_t chunk0;   // chunks (clipping: pieces) of the entries before it
  int8_t type, out_type, lgB, pad;
  int32_t pad4;
};
static_assert(sizeof(Entry) == 48, "table layout");

// elements of a chunk of `type`
__host__ __device__ constexpr int64_t chunk_elems(int type) {
  return type == kInt4 ? 2 * kChunkBytes : type == ZQ_F32 ? kChunkBytes / 4 : kChunkBytes / 2;
}

// Table: the workgroups' sums, the entries of the norm, the entries of clipping (an
// INT4 shard clipped in place is its scales there), the entry of each piece of clipping.
constexpr int64_t kSumsAt = 0, kEntriesAt = kSumsAt + 8 * kNormGroups;
__host__ __device__ inline int64_t clip_at(int entries) { return kEntriesAt + (int64_t)entries * (int64_t)sizeof(Entry); }
__host__ __device__ inline int64_t map_at(int entries) { return clip_at(entries) + (int64_t)entries * (int64_t)sizeof(Entry); }

// index of the entry that holds chunk c (every thread gets it)
__device__ __forceinline__ int find_entry(const Entry* entries, int count, int64_t c) {
  __shared__ int found;
  for (int i = threadIdx.x; i < count; i += kNormThreads) {
    const int64_t a = entries[i].chunk0;
    const int64_t b = i + 1 < count ? entries[i + 1].chunk0 : INT64_MAX;
    if (a <= c && c < b) found = i;
  }
  __syncthreads();
  return found;
}

// Loads in flight: a thread issues those of kSteps pieces (16 bytes each, the
// workgroup's 4 KiB apart) before it uses the first.
constexpr int kSteps = 4;

template <int DT>
__device__ __forceinline__ double sum_squares(const Entry& en, int64_t e0, int64_t e1) {
  constexpr int E = 16 / dt_size<DT>(), STEP = kNormThreads * E;
  double a = 0.0, b = 0.0;
  auto add = [&](const uint32_t(&w)[4]) {
    float v[E];
    widen<DT>(w, v);
#pragma unroll
    for (int k = 0; k < E; k += 2) {
      a = __builtin_fma((double)v[k], (double)v[k], a);
      b = __builtin_fma((double)v[k + 1], (double)v[k + 1], b);
    }
  };
  int64_t i = e0 + (int64_t)threadIdx.x * E;
  for (; i + (kSteps - 1) * STEP + E <= e1; i += kSteps * STEP) {
    uint32_t w[kSteps][4];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) load_words_any<true>(en.data + (i + u * STEP) * dt_size<DT>(), w[u]);
#pragma unroll
    for (int u = 0; u < kSteps; ++u) add(w[u]);
  }
  for (; i + E <= e1; i += STEP) {
    uint32_t w[4];
    load_words_any<true>(en.data + i * dt_size<DT>(), w);
    add(w);
  }
  for (; i < e1; ++i) {  // one thread: the elements of the last, short piece
    float v[1];
    load_elems<DT, 1>(en.data, i, v);
    a = __builtin_fma((double)v[0], (double)v[0], a);
  }
  return a + b;
}

// 32 codes a thread and step: within one block, as blocks are multiples of 32
__device__ __forceinline__ double sum_squares_int4(const Entry& en, int64_t e0, int64_t e1) {
  constexpr int E = 32, STEP = kNormThreads * E;
  double a = 0.0;
  auto add = [&](const uint32_t(&w)[4], float scale) {
    int q2 = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) q2 = __builtin_amdgcn_sdot8((int)w[k], (int)w[k], q2, false);
    const double s = (double)scale;
    a = __builtin_fma(s * s, (double)q2, a);
  };
  int64_t i = e0 + (int64_t)threadIdx.x * E;
  for (; i + (kSteps - 1) * STEP + E <= e1; i += kSteps * STEP) {
    uint32_t w[kSteps][4];
    float s[kSteps];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      load_words_any<true>(en.data + (i + u * STEP) / 2, w[u]);
      s[u] = en.scales[(i + u * STEP) >> en.lgB];
    }
#pragma unroll
    for (int u = 0; u < kSteps; ++u) add(w[u], s[u]);
  }
  for (; i < e1; i += STEP) {
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    const char* p = en.data + i / 2;
    if (i + E <= e1) {
      load_words_any<true>(p, w);
    } else {
      for (int k = 0; i + k < e1; ++k) {
        const uint32_t q = (uint8_t)p[k / 2] >> (4 * (k & 1)) & 15u;
        w[k / 8] |= q << (4 * (k % 8));
      }
    }
    add(w, en.scales[i >> en.lgB]);
  }
  return a;
}

__device__ __forceinline__ double wave_sum(double v) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// sum over the workgroup, in thread 0
__device__ __forceinline__ double group_sum(double v) {
  __shared__ double part[kNormThreads / 64];
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
  for (int w = 0; w < kNormThreads / 64; ++w) s += part[w];
  __syncthreads();
  return s;
}

__global__ void __launch_bounds__(kNormThreads)
    k_grad_norm(char* __restrict__ table, int count, int64_t chunks, float scale, float* __restrict__ norm) {
  const Entry* entries = reinterpret_cast<const Entry*>(table + kEntriesAt);
  double* sums = reinterpret_cast<double*>(table + kSumsAt);
  const int64_t W = gridDim.x, w = blockIdx.x;
  int64_t c = w * chunks / W;
  const int64_t c1 = (w + 1) * chunks / W;
  double a = 0.0;
  if (c < c1) {
    int i = find_entry(entries, count, c);
    while (c < c1) {
      const Entry en = entries[i];
      const int64_t per = chunk_elems(en.type);
      const int64_t e0 = (c - en.chunk0) * per;
      const int64_t last = en.chunk0 + (en.n + per - 1) / per;  // the next entry's first chunk
      const int64_t to = c1 < last ? c1 : last;
      int64_t e1 = (to - en.chunk0) * per;
      if (e1 > en.n) e1 = en.n;
      switch (en.type) {
        case ZQ_F32: a += sum_squares<ZQ_F32>(en, e0, e1); break;
        case ZQ_F16: a += sum_squares<ZQ_F16>(en, e0, e1); break;
        case ZQ_BF16: a += sum_squares<ZQ_BF16>(en, e0, e1); break;
        default: a += sum_squares_int4(en, e0, e1); break;
      }
      c = to;
      ++i;
    }
  }
  a = group_sum(a);
  if (threadIdx.x != 0) return;
  if (W == 1) *norm = (float)(fabs((double)scale) * sqrt(a));
  else sums[w] = a;
}

// the workgroups' sums, in their order
__global__ void __launch_bounds__(kNormThreads)
    k_norm_finish(const char* __restrict__ table, int groups, float scale, float* __restrict__ norm) {
  const double* sums = reinterpret_cast<const double*>(table + kSumsAt);
  double v[kNormGroups / kNormThreads], t = 0.0;
#pragma unroll
  for (int u = 0; u < kNormGroups / kNormThreads; ++u) {
    const int k = u * kNormThreads + threadIdx.x;
    v[u] = k < groups ? sums[k] : 0.0;
  }
#pragma unroll
  for (int u = 0; u < kNormGroups / kNormThreads; ++u) t += v[u];
  t = group_sum(t);
  if (threadIdx.x == 0) *norm = (float)(fabs((double)scale) * sqrt(t));
}

// ---- clipping: a workgroup per piece of kClipElems elements.  Pieces are small and
// workgroups start in their order, so that the result is written nearly in address
// order (50 million bf16 elements into binary32: 51 us, 5.9 TB/s; in 2,048 streams far
// apart, as the norm reads, 60).
constexpr int kClipElems = 4096;
constexpr int kClipSteps = kClipElems / kNormThreads / 4;

// 4 elements a thread and step, so that a binary32 store of the wave covers whole lines
template <int DT, int YT>
__device__ __forceinline__ void scale_elems(const Entry& en, int64_t e0, float c) {
  constexpr int N = dt_size<DT>();  // words of 4 elements
  auto put = [&](int64_t i, const uint32_t(&w)[N]) {
    float v[4];
    widen<DT>(w, v);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = v[k] * c;
    store_elems<YT, 4, true>(en.out, i, v);
  };
  const int64_t i = e0 + threadIdx.x * 4;
  if (e0 + kClipElems <= en.n) {
    uint32_t w[kClipSteps][N];
#pragma unroll
    for (int u = 0; u < kClipSteps; ++u)
      load_words_any<false>(en.data + (i + u * (4 * kNormThreads)) * dt_size<DT>(), w[u]);
#pragma unroll
    for (int u = 0; u < kClipSteps; ++u) put(i + u * (4 * kNormThreads), w[u]);
    return;
  }
  for (int u = 0; u < kClipSteps; ++u) {
    int64_t k = i + u * (4 * kNormThreads);
    if (k + 4 <= en.n) {
      uint32_t w[N];
      load_words_any<false>(en.data + k * dt_size<DT>(), w);
      put(k, w);
    } else {
      for (; k < en.n && k < i + u * (4 * kNormThreads) + 4; ++k) {
        float v[1];
        load_elems<DT, 1>(en.data, k, v);
        v[0] = v[0] * c;
        store_elems<YT, 1>(en.out, k, v);
      }
    }
  }
}

// the INT4 shard dequantised with its scales times c: fl(q * fl(s * c))
template <int YT>
__device__ __forceinline__ void scale_int4(const Entry& en, int64_t e0, float c) {
  auto value = [](uint32_t q, int k, float s) { return (float)((int32_t)(q << (28 - 4 * k)) >> 28) * s; };
  const int64_t i = e0 + threadIdx.x * 4;
  if (e0 + kClipElems <= en.n) {
    uint32_t q[kClipSteps];
    float s[kClipSteps];
#pragma unroll
    for (int u = 0; u < kClipSteps; ++u) {
      const int64_t k = i + u * (4 * kNormThreads);
      q[u] = *reinterpret_cast<const u16_any*>(en.data + k / 2);
      s[u] = en.scales[k >> en.lgB];
    }
#pragma unroll
    for (int u = 0; u < kClipSteps; ++u) {
      const float t = s[u] * c;
      const float v[4] = {value(q[u], 0, t), value(q[u], 1, t), value(q[u], 2, t), value(q[u], 3, t)};
      store_elems<YT, 4, true>(en.out, i + u * (4 * kNormThreads), v);
    }
    return;
  }
  for (int u = 0; u < kClipSteps; ++u) {
    const int64_t k0 = i + u * (4 * kNormThreads);
    for (int64_t k = k0; k < en.n && k < k0 + 4; ++k) {
      const float v[1] = {value((uint8_t)en.data[k / 2] >> (4 * (k & 1)), 0, en.scales[k >> en.lgB] * c)};
      store_elems<YT, 1>(en.out, k, v);
    }
  }
}

template <int YT>
__device__ __forceinline__ void scale_to(const Entry& en, int64_t e0, float c) {
  switch (en.type) {
    case ZQ_F32: scale_elems<ZQ_F32, YT>(en, e0, c); break;
    case ZQ_F16: scale_elems<ZQ_F16, YT>(en, e0, c); break;
    case ZQ_BF16: scale_elems<ZQ_BF16, YT>(en, e0, c); break;
    default: scale_int4<YT>(en, e0, c); break;
  }
}

__global__ void __launch_bounds__(kNormThreads)
    k_grad_clip(unsigned first, const char* __restrict__ table, int count, const float* __restrict__ norm,
                float max_norm, float scale) {
  const int* entry_of = reinterpret_cast<const int*>(table + map_at(count));
  const unsigned piece = first + blockIdx.x;
  const Entry en = reinterpret_cast<const Entry*>(table + clip_at(count))[entry_of[piece]];
  const float ratio = max_norm / (*norm + 1e-6f);
  // a NaN ratio stays: min would drop it
  const float c = scale * (ratio > 1.0f ? 1.0f : ratio);
  // in place and nothing to scale: the tensor stays as it is
  if (en.out == en.data && c == 1.0f) return;
  const int64_t e0 = ((int64_t)piece - en.chunk0) * kClipElems;
  switch (en.out_type) {
    case ZQ_F32: scale_to<ZQ_F32>(en, e0, c); break;
    case ZQ_F16: scale_to<ZQ_F16>(en, e0, c); break;
    default: scale_to<ZQ_BF16>(en, e0, c); break;
  }
}

// ---------------------------------------------------------------- table

int64_t data_bytes(int64_t n, int type) { return type == kInt4 ? (n + 1) / 2 : n * elem_bytes(type); }

int check(const zq_grad& g) {
  if (g.n < 0 || g.n > INT64_MAX / 16) return ZQ_E_SIZE;
  const bool int4 = g.dtype == ZQ_INT4;
  if (!int4 && !dtype_ok(g.dtype)) return ZQ_E_DTYPE;
  if (g.out && !dtype_ok(g.out_dtype)) return ZQ_E_DTYPE;
  if (int4 && log2_block(g.block) < 0) return ZQ_E_BLOCK;
  if (g.n == 0) return ZQ_OK;
  if (!g.data || (int4 && !g.scales)) return ZQ_E_NULL;
  if (!int4 && !aligned(g.data, elem_bytes(g.dtype))) return ZQ_E_ALIGN;
  if (int4 && !aligned(g.scales, 4)) return ZQ_E_ALIGN;
  if (g.out && !aligned(g.out, elem_bytes(g.out_dtype))) return ZQ_E_ALIGN;
  // in place, the type stays
  if (!int4 && g.out == g.data && g.out_dtype != g.dtype) return ZQ_E_ALIAS;
  return ZQ_OK;
}

Entry norm_entry(const zq_grad& g) {
  Entry e = {};
  e.data = static_cast<const char*>(g.data);
  e.scales = g.scales;
  e.n = g.n;
  e.type = (int8_t)(g.dtype == ZQ_INT4 ? kInt4 : g.dtype);
  e.lgB = (int8_t)(g.dtype == ZQ_INT4 ? log2_block(g.block) : 0);
  return e;
}
Entry clip_entry(const zq_grad& g) {
  Entry e = norm_entry(g);
  if (g.out) {
    e.out = static_cast<char*>(g.out);
    e.out_type = (int8_t)g.out_dtype;
  } else if (g.dtype == ZQ_INT4) {
    e.data = reinterpret_cast<const char*>(g.scales);
    e.out = reinterpret_cast<char*>(g.scales);
    e.scales = nullptr;
    e.n = num_scales(g.n, g.block);
    e.type = e.out_type = ZQ_F32;
  } else {
    e.out = static_cast<char*>(g.data);
    e.out_type = e.type;
  }
  return e;
}
int64_t chunks_of(const Entry& e) { return (e.n + chunk_elems(e.type) - 1) / chunk_elems(e.type); }
int64_t pieces_of(const Entry& e) { return (e.n + kClipElems - 1) / kClipElems; }

// Outputs must not overlap each other nor another tensor's data.
int check_overlaps(const zq_grad* grads, int32_t count) {
  std::vector<Span> spans;
  spans.reserve(3 * (size_t)count);
  for (int32_t i = 0; i < count; ++i) {
    const zq_grad& g = grads[i];
    const Entry n = norm_entry(g), c = clip_entry(g);
    if (g.n == 0) continue;
    const bool in_place = c.out == (g.dtype == ZQ_INT4 && !g.out ? (const char*)g.scales : (const char*)g.data);
    put_span(spans, c.out, c.n * elem_bytes(c.out_type), true);
    if (!(in_place && g.dtype != ZQ_INT4)) put_span(spans, n.data, data_bytes(n.n, n.type), false);
    if (g.dtype == ZQ_INT4 && g.out) put_span(spans, g.scales, 4 * num_scales(g.n, g.block), false);
  }
  return check_spans(spans);
}

int plan_table(const zq_grad* grads, int32_t count, zq_grad_plan* plan) {
  if (!plan || (count > 0 && !grads)) return ZQ_E_NULL;
  if (count < 0) return ZQ_E_SIZE;
  zq_grad_plan p = {};
  p.count = count;
  for (int32_t i = 0; i < count; ++i) {
    const int rc = check(grads[i]);
    if (rc != ZQ_OK) return rc;
    p.norm_chunks += chunks_of(norm_entry(grads[i]));
    p.clip_chunks += pieces_of(clip_entry(grads[i]));
    if (p.clip_chunks > kMaxGrid) return ZQ_E_SIZE;
  }
  const int rc = check_overlaps(grads, count);
  if (rc != ZQ_OK) return rc;
  p.bytes = map_at(count) + 4 * p.clip_chunks;
  *plan = p;
  return ZQ_OK;
}

// A workgroup a chunk, up to kNormGroups of them.
unsigned groups_for(int64_t chunks) {
  return (unsigned)(chunks < kNormGroups ? (chunks < 1 ? 1 : chunks) : kNormGroups);
}

}  // namespace
}  // namespace zq

extern "C" {

using namespace zq;

int zq_grad_plan_make(const zq_grad* grads, int32_t count, zq_grad_plan* plan) {
  try {
    return plan_table(grads, count, plan);
  } catch (...) {  // more tensors than the host has memory to check for overlaps
    return ZQ_E_SIZE;
  }
}

int zq_grad_plan_table(const zq_grad* grads, const zq_grad_plan* plan, void* host_table) {
  if (!plan || !host_table || (plan->count > 0 && !grads)) return ZQ_E_NULL;
  char* t = static_cast<char*>(host_table);
  std::fill(t, t + kEntriesAt, (char)0);
  Entry* norm = reinterpret_cast<Entry*>(t + kEntriesAt);
  Entry* clip = reinterpret_cast<Entry*>(t + clip_at(plan->count));
  int* map = reinterpret_cast<int*>(t + map_at(plan->count));
  int64_t n = 0, c = 0;
  for (int32_t i = 0; i < plan->count; ++i) {
    norm[i] = norm_entry(grads[i]);
    clip[i] = clip_entry(grads[i]);
    norm[i].chunk0 = n;
    clip[i].chunk0 = c;
    n += chunks_of(norm[i]);
    const int64_t pieces = pieces_of(clip[i]);
    std::fill(map + c, map + c + pieces, i);
    c += pieces;
  }
  return ZQ_OK;
}

int zq_grad_norm(const zq_grad_plan* plan, void* table, float scale, float* norm, void* stream) {
  if (!plan || !table || !norm) return ZQ_E_NULL;
  if (!aligned(table, 16) || !aligned(norm, 4)) return ZQ_E_ALIGN;
  // One launch up to 4 chunks (one workgroup reads them), else a second one that
  // adds the workgroups' sums.  (The last workgroup to finish adding them in the same
  // launch needs a release and an acquire by every workgroup: 60 us for 2,048.)
  const unsigned groups = plan->norm_chunks <= 4 ? 1u : groups_for(plan->norm_chunks);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int rc = launch(&k_grad_norm, groups, kNormThreads, st, static_cast<char*>(table), plan->count,
                        plan->norm_chunks, scale, norm);
  if (rc != ZQ_OK || groups == 1) return rc;
  return launch(&k_norm_finish, 1u, kNormThreads, st, static_cast<const char*>(table), (int)groups, scale, norm);
}

int zq_grad_clip(const zq_grad_plan* plan, const void* table, const float* norm, float max_norm, float scale,
                 void* stream) {
  if (!plan || !table || !norm) return ZQ_E_NULL;
  if (!aligned(table, 16) || !aligned(norm, 4)) return ZQ_E_ALIGN;
  if (!(max_norm >= 0.0f)) return ZQ_E_SIZE;
  if (plan->clip_chunks == 0) return ZQ_OK;
  return launch_parts(&k_grad_clip, plan->clip_chunks, kNormThreads, static_cast<hipStream_t>(stream),
                      static_cast<const char*>(table), plan->count, norm, max_norm, scale);
}

}  // extern "C"
