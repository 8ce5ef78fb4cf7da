// zq_vec.h -- vectors of elements of a storage type, read into binary32 and
// written from it, at any element address: the gfx9 ABI runs with unaligned
// global access, so a 16-byte load or store is one instruction wherever it
// starts, and rows of odd lengths need no second path.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "zq.h"
#include "zq_device.h"

namespace zq {

typedef uint16_t u16_any __attribute__((aligned(1)));
typedef uint32_t u32_any __attribute__((aligned(1)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));

template <int DT>
constexpr int dt_size() {
  return DT == ZQ_F32 ? 4 : 2;
}

// N 32-bit words from any address; NT: not kept in the caches
template <bool NT, int N>
__device__ __forceinline__ void load_words_any(const void* p, uint32_t (&w)[N]) {
  static_assert(N == 1 || N == 2 || N % 4 == 0, "16-byte pieces");
  const char* b = static_cast<const char*>(p);
  if constexpr (N == 1) {
    w[0] = *reinterpret_cast<const u32_any*>(b);
  } else if constexpr (N == 2) {
    const u32x2_any* q = reinterpret_cast<const u32x2_any*>(b);
    const u32x2 t = NT ? __builtin_nontemporal_load(q) : *q;
    w[0] = t[0], w[1] = t[1];
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const u32x4_any* q = reinterpret_cast<const u32x4_any*>(b + 16 * i);
      const u32x4 t = NT ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[4 * i + j] = t[j];
    }
  }
}

template <bool NT, int N>
__device__ __forceinline__ void store_words_any(void* p, const uint32_t (&w)[N]) {
  static_assert(N == 1 || N == 2 || N % 4 == 0, "16-byte pieces");
  char* b = static_cast<char*>(p);
  if constexpr (N == 1) {
    *reinterpret_cast<u32_any*>(b) = w[0];
  } else if constexpr (N == 2) {
    u32x2_any* q = reinterpret_cast<u32x2_any*>(b);
    const u32x2_any t = {w[0], w[1]};
    if constexpr (NT) __builtin_nontemporal_store(t, q);
    else *q = t;
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      u32x4_any* q = reinterpret_cast<u32x4_any*>(b + 16 * i);
      const u32x4_any t = {w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
      if constexpr (NT) __builtin_nontemporal_store(t, q);
      else *q = t;
    }
  }
}

// words of a storage type <-> binary32 values
template <int DT, int E, int N>
__device__ __forceinline__ void widen(const uint32_t (&w)[N], float (&v)[E]) {
#pragma unroll
  for (int i = 0; i < E; ++i) {
    if constexpr (DT == ZQ_F32) v[i] = u2f(w[i]);
    else if constexpr (DT == ZQ_BF16) v[i] = u2f(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    else v[i] = h2f((w[i / 2] >> (16 * (i & 1))) & 0xffffu);
  }
}

// E elements of type DT from element i of `base` on (E = 1, 4 or 8)
template <int DT, int E, bool NT = false>
__device__ __forceinline__ void load_elems(const void* base, int64_t i, float (&v)[E]) {
  const char* p = static_cast<const char*>(base) + i * dt_size<DT>();
  if constexpr (E == 1 && DT != ZQ_F32) {
    const uint32_t h = *reinterpret_cast<const uint16_t*>(p);
    v[0] = DT == ZQ_BF16 ? u2f(h << 16) : h2f(h);
  } else {
    uint32_t w[E * dt_size<DT>() / 4];
    load_words_any<NT>(p, w);
    widen<DT>(w, v);
  }
}

template <int DT, int E, bool NT = false>
__device__ __forceinline__ void store_elems(void* base, int64_t i, const float (&v)[E]) {
  char* p = static_cast<char*>(base) + i * dt_size<DT>();
  if constexpr (E == 1 && DT != ZQ_F32) {
    *reinterpret_cast<uint16_t*>(p) = (uint16_t)(DT == ZQ_BF16 ? bf16x2_bits(v[0], 0.0f) & 0xffffu : f2h(v[0]));
  } else {
    uint32_t w[E * dt_size<DT>() / 4];
#pragma unroll
    for (int j = 0; j < E * dt_size<DT>() / 4; ++j) {
      if constexpr (DT == ZQ_F32) w[j] = f2u(v[j]);
      else if constexpr (DT == ZQ_BF16) w[j] = bf16x2_bits(v[2 * j], v[2 * j + 1]);
      else w[j] = f2h(v[2 * j]) | (f2h(v[2 * j + 1]) << 16);
    }
    store_words_any<NT>(p, w);
  }
}

}  // namespace zq
