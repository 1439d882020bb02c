// ae_rows.h — pieces of eight elements of a row, at any alignment of the element's own, of which `left` lie inside the row.
#pragma once

#include "ae_device.h"

namespace ae {

// eight elements as numbers, zeros behind the row's end; whole pieces with one load (bf16) or two
// (binary32) at any alignment of the element's own
template <typename T>
__device__ __forceinline__ void load8(const T* p, int left, float (&v)[8]) {
  if (left >= 8) {
    if constexpr (sizeof(T) == 2) {
      uint32_t w[4];
      __builtin_memcpy(w, p, 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    } else {
      __builtin_memcpy(v, p, 32);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? Store<T>::ld(p + i) : 0.0f;
  }
}

// eight elements as they lie in memory, so that a load can be in flight while its registers are not looked at
template <typename T>
struct Eight {
  uint32_t w[2 * sizeof(T)];
};
template <typename T>
__device__ __forceinline__ void fetch8(const T* p, int left, Eight<T>& e) {
  if (left >= 8) {
    __builtin_memcpy(e.w, p, sizeof(e.w));
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) e.w[i] = i < left ? __float_as_uint(p[i]) : 0u;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) e.w[i] = (2 * i < left ? (uint32_t)p[2 * i] : 0u) | (2 * i + 1 < left ? (uint32_t)p[2 * i + 1] << 16 : 0u);
  }
}
template <typename T>
__device__ __forceinline__ float value(const Eight<T>& e, int i) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(e.w[i]);
  return __uint_as_float(i & 1 ? e.w[i >> 1] & 0xFFFF0000u : e.w[i >> 1] << 16);
}
template <typename T>
__device__ __forceinline__ void put8(T* p, int left, const float (&v)[8]) {
  if (left >= 8) {
    if constexpr (sizeof(T) == 4) {
      __builtin_memcpy(p, v, 32);
    } else {
      const uint32_t w[4] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
      __builtin_memcpy(p, w, 16);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) Store<T>::st(p + i, v[i]);
  }
}

}  // namespace ae
