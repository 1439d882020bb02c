// ae_rows.h — pieces of a few elements of a row, at any alignment of the element's own, of which `left` lie inside the row.
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

// N elements as they lie in memory, so that a load can be in flight while its registers are not looked at
template <typename T, int N>
struct Piece {
  static constexpr int WORDS = N * sizeof(T) / 4;
  uint32_t w[WORDS];
};
template <typename T> using Eight = Piece<T, 8>;
// One access of a whole piece (or of 16 bytes of it), at the element's alignment.  A vector type and not a copy of bytes: the
// compiler takes copies apart, finds the first element in the path of a row's end too, and loads or stores it on its own.
template <typename T, int N>
struct Words {
  static constexpr int PER = Piece<T, N>::WORDS < 4 ? Piece<T, N>::WORDS : 4, COUNT = Piece<T, N>::WORDS / PER;
  typedef uint32_t type __attribute__((ext_vector_type(PER), aligned(sizeof(T))));
};
// A whole piece.  STREAM: with the hint that it is not wanted again soon; a read of 512 MB runs at 7.0 TB/s with it and at 6.1 without,
// a copy at 6.4 and 5.6, a fill is slower with it (5.4 and 5.7).
template <bool STREAM, typename T, int N>
__device__ __forceinline__ void fetch_whole(const T* p, Piece<T, N>& e) {
  typedef typename Words<T, N>::type words;
  constexpr int PER = Words<T, N>::PER;
#pragma unroll
  for (int i = 0; i < Words<T, N>::COUNT; ++i) {
    const words* at = reinterpret_cast<const words*>(p) + i;
    const words w = STREAM ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
    for (int k = 0; k < PER; ++k) e.w[i * PER + k] = w[k];
  }
}
template <typename T, int N>
__device__ __forceinline__ void fetch(const T* p, int left, Piece<T, N>& e) {
  if (left >= N) {
    fetch_whole<false>(p, e);
  } else if (left > 0) {                         // all of them in flight: a lane's last element stands in for what is not there
    T u[N];
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] = p[i < left ? i : left - 1];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) e.w[i] = i < left ? __float_as_uint(u[i]) : 0u;
    } else {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) e.w[i] = (2 * i < left ? (uint32_t)u[2 * i] : 0u) | (2 * i + 1 < left ? (uint32_t)u[2 * i + 1] << 16 : 0u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < Piece<T, N>::WORDS; ++i) e.w[i] = 0u;
  }
}
// The piece of a row of `len` elements that begins at column col, in two steps: the load, which is the same for all lanes (one that
// reaches over the row's end, or lies behind it, takes the row's last N elements), and, when it has come, their shift into
// place with zeros behind.  So a row of any length keeps its loads in flight.  SHORT: rows may be shorter than a piece, and go
// element by element then.
template <bool STREAM, bool SHORT, typename T, int N>
__device__ __forceinline__ void fetch_row(const T* row, int col, int len, Piece<T, N>& e) {
  if (SHORT && len < N) fetch(row + col, len - col, e);
  else fetch_whole<STREAM>(row + (col <= len - N ? col : len - N), e);
}
template <bool SHORT, typename T, int N>
__device__ __forceinline__ void settle(int col, int len, Piece<T, N>& e) {
  constexpr int W = Piece<T, N>::WORDS;
  int over = col - (len - N);
  if ((SHORT && len < N) || over <= 0) return;
  if (over > N) over = N;
  if constexpr (sizeof(T) == 2) {
    if (over & 1) {
#pragma unroll
      for (int i = 0; i < W; ++i) e.w[i] = e.w[i] >> 16 | (i + 1 < W ? e.w[i + 1] << 16 : 0u);
    }
    over >>= 1;
  }
#pragma unroll
  for (int b = 1; b <= W; b *= 2)
    if (over & b) {
#pragma unroll
      for (int i = 0; i < W; ++i) e.w[i] = i + b < W ? e.w[i + b] : 0u;
    }
}
// A call that moves more than this reads and writes as a stream: less than half of the 256 MB cache may well be there from the call
// before, or be wanted from there by the next.
constexpr int64_t kStreamBytes = (int64_t)96 << 20;

template <typename T, int N>
__device__ __forceinline__ float value(const Piece<T, N>& e, int i) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(e.w[i]);
  return __uint_as_float(i & 1 ? e.w[i >> 1] & 0xFFFF0000u : e.w[i >> 1] << 16);
}
// rounded to nearest, ties to even
template <typename T, int N>
__device__ __forceinline__ void make_piece(const float (&v)[N], Piece<T, N>& e) {
#pragma unroll
  for (int i = 0; i < Piece<T, N>::WORDS; ++i) {
    if constexpr (sizeof(T) == 4) e.w[i] = __float_as_uint(v[i]);
    else e.w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
  }
}
template <bool STREAM, typename T, int N>
__device__ __forceinline__ void put_piece(T* p, const Piece<T, N>& e) {
  typedef typename Words<T, N>::type words;
  constexpr int PER = Words<T, N>::PER;
#pragma unroll
  for (int i = 0; i < Words<T, N>::COUNT; ++i) {
    words w;
#pragma unroll
    for (int k = 0; k < PER; ++k) w[k] = e.w[i * PER + k];
    words* at = reinterpret_cast<words*>(p) + i;
    if constexpr (STREAM) __builtin_nontemporal_store(w, at);
    else *at = w;
  }
}
template <bool STREAM, typename T, int N>
__device__ __forceinline__ void put_whole(T* p, const float (&v)[N]) {
  Piece<T, N> e;
  make_piece(v, e);
  put_piece<STREAM>(p, e);
}
// STREAM is no argument: of two branches that differ in the hint alone the compiler makes one without it
template <bool STREAM = false, typename T, int N>
__device__ __forceinline__ void put(T* p, int left, const float (&v)[N]) {
  if (left >= N) {
    put_whole<STREAM>(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < left) Store<T>::st(p + i, v[i]);
  }
}

}  // namespace ae
