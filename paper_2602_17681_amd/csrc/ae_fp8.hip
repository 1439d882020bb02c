// ae_fp8.hip — matrices of E4M3 codes with a binary32 scale for each block of 128: the quantiser and the product
//   y[i][j] = bias[j] + sum_c sa[c][i] sb[c; j] sum_{k in c} a[i][k] b[j][k].
// A block is as long as K of the widest 8-bit matrix instruction (16 x 16 x 128): one instruction gives the sum over a
// block in its four result registers, which are scaled and added to the accumulators in binary32.
#include <hip/hip_runtime.h>
#include <float.h>
#include <string.h>

#include <type_traits>

#include "ae_device.h"
#include "ae_internal.h"

namespace ae {
namespace {

constexpr int BLK = 128;                 // elements that share a scale
constexpr float kCodeMax = 448.0f;       // largest magnitude of an E4M3 code
constexpr float kScaleMin = 1.17549435e-38f;

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

// Infinities are rare and cost the common case nothing: the maximum over all magnitudes (which passes NaN by) tells whether
// a block holds any.  If not, x * (1 / scale) is at most 448 (1 + 2^-23), which the conversion rounds to 448, and a NaN
// becomes the NaN code by itself; if so, the maximum is taken again over what is finite, and the products are cut off at 448.
__device__ __forceinline__ float finite_abs(float v) {
  const float a = fabsf(v);
  return a <= FLT_MAX ? a : 0.0f;
}
__device__ __forceinline__ float block_scale(float amax) { return fmaxf(amax / kCodeMax, kScaleMin); }
template <bool INF>
__device__ __forceinline__ float code_value(float v, float inv) {
  const float y = v * inv;
  if constexpr (!INF) return y;
  return y != y ? y : fminf(fmaxf(y, -kCodeMax), kCodeMax);
}
template <bool INF>
__device__ __forceinline__ float magnitude(float v) { return INF ? finite_abs(v) : fabsf(v); }
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

// eight elements of a row from column c on, zeros behind the row's end; whole pieces with one load (bf16) or two
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

// ---- quantiser -----------------------------------------------------------------------------------------------------
// One workgroup of 256 threads per 128 x 128 tile of x: thread t holds rows 8 (t / 16) .. + 7 of columns 8 (t % 16) .. + 7
// in registers, so that a block maximum along a row is a reduction over 16 neighbouring lanes, along a column over the 16
// row groups, and both orientations come from one read.  Transposed codes go through LDS to be written as whole 16-byte
// pieces of a row of x^T.
constexpr int QT_STRIDE = BLK / 4 + 1;    // words of a transposed row in LDS: eight rows on, as far as neighbouring lanes write, are 8 banks on
struct QuantizeArgs {
  int rows, cols, tiles_c;
  int first;                              // the launch's first workgroup (row blocks alone)
  uint8_t* q;
  int64_t ldq;
  float* scale;
  uint8_t* qt;
  int64_t ldqt;
  float* scale_t;
};
template <bool TILES, bool Q, bool QT, bool INF>
__device__ __forceinline__ void quantize_tile(const float (&v)[8][8], const QuantizeArgs& p, int tr_i, int tc_i, float* red, uint32_t* tr) {
  const int r0 = tr_i * BLK, c0 = tc_i * BLK, rows = p.rows, cols = p.cols;
  const int t = threadIdx.x, cg = t & 15, rg = t >> 4, wave = t >> 6;
  const int row = r0 + rg * 8, col = c0 + cg * 8;
  float inv_r[8], inv_c[8];               // what the elements of a row / column are multiplied with
  if constexpr (TILES) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaxf(m, magnitude<INF>(v[i][j]));
    m = max_rows(max16(m));
    if ((t & 63) == 0) red[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float s = block_scale(m), inv = 1.0f / s;
    if (t == 0) {
      if constexpr (Q) p.scale[(int64_t)tr_i * p.tiles_c + tc_i] = s;
      if constexpr (QT) p.scale_t[(int64_t)tc_i * ((rows + BLK - 1) / BLK) + tr_i] = s;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) inv_r[i] = inv_c[i] = inv;
  } else {
    if constexpr (Q) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = fmaxf(m, magnitude<INF>(v[i][j]));
        const float s = block_scale(max16(m));
        inv_r[i] = 1.0f / s;
        if (cg == 0 && row + i < rows) p.scale[(int64_t)tc_i * rows + row + i] = s;
      }
    }
    if constexpr (QT) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, magnitude<INF>(v[i][j]));
        m = max_rows(m);
        if ((t & 63) < 16) red[wave * BLK + cg * 8 + j] = m;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = cg * 8 + j;
        const float s = block_scale(fmaxf(fmaxf(red[c], red[BLK + c]), fmaxf(red[2 * BLK + c], red[3 * BLK + c])));
        inv_c[j] = 1.0f / s;
        if (rg == 0 && c0 + c < cols) p.scale_t[(int64_t)tr_i * cols + c0 + c] = s;
      }
    }
  }
  if constexpr (Q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (row + i >= rows || col >= cols) continue;
      uint8_t* at = p.q + (int64_t)(row + i) * p.ldq + col;
      float u[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = code_value<INF>(v[i][j], inv_r[i]);
      const uint32_t lo = codes4(u[0], u[1], u[2], u[3]), hi = codes4(u[4], u[5], u[6], u[7]);
      if (col + 8 <= cols) {
        *reinterpret_cast<uint2*>(at) = make_uint2(lo, hi);
      } else {
        for (int j = 0; j < cols - col; ++j) at[j] = (uint8_t)((j < 4 ? lo : hi) >> (8 * (j & 3)));
      }
    }
  }
  if constexpr (QT) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = code_value<INF>(v[i][j], inv_c[j]);
      uint32_t* w = tr + (cg * 8 + j) * QT_STRIDE + rg * 2;
      w[0] = codes4(u[0], u[1], u[2], u[3]);
      w[1] = codes4(u[4], u[5], u[6], u[7]);
    }
    __syncthreads();
#pragma unroll
    for (int pass = 0; pass < 4; ++pass) {
      const int c = pass * 32 + (t >> 3), ch = (t & 7) * 16;
      const int left = rows - r0 - ch;
      if (c0 + c >= cols || left <= 0) continue;
      uint8_t* at = p.qt + (int64_t)(c0 + c) * p.ldqt + r0 + ch;
      const uint32_t* s = tr + c * QT_STRIDE + ch / 4;
      if (left >= 16) {
        *reinterpret_cast<uint4*>(at) = make_uint4(s[0], s[1], s[2], s[3]);
      } else {
        for (int i = 0; i < left; ++i) at[i] = (uint8_t)(s[i >> 2] >> (8 * (i & 3)));
      }
    }
  }
}
template <typename T, bool TILES, bool Q, bool QT>
__global__ __launch_bounds__(256) void k_fp8_quantize(const T* __restrict__ x, int64_t ldx, QuantizeArgs p) {
  __shared__ float red[4 * BLK];
  __shared__ uint32_t tr[QT ? BLK * QT_STRIDE : 1];
  const int tr_i = blockIdx.x / p.tiles_c, tc_i = blockIdx.x - tr_i * p.tiles_c;
  const int row = tr_i * BLK + (threadIdx.x >> 4) * 8, col = tc_i * BLK + (threadIdx.x & 15) * 8;
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (row + i < p.rows) {
      load8<T>(x + (int64_t)(row + i) * ldx + col, p.cols - col, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    }
  }
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(v[i][j]));
  if (__syncthreads_or(m > FLT_MAX)) quantize_tile<TILES, Q, QT, true>(v, p, tr_i, tc_i, red, tr);
  else quantize_tile<TILES, Q, QT, false>(v, p, tr_i, tc_i, red, tr);
}

// Codes in row blocks alone need no tile: 16 lanes take a block, a workgroup 16 R rows of one column of blocks, so that
// also few rows make many workgroups.
template <typename T, int R>
__global__ __launch_bounds__(256) void k_fp8_quantize_rows(const T* __restrict__ x, int64_t ldx, QuantizeArgs p) {
  const int at = p.first + (int)blockIdx.x, rt = at / p.tiles_c, tc = at - rt * p.tiles_c;
  const int row = rt * 16 * R + (threadIdx.x >> 4), cg = threadIdx.x & 15, col = tc * BLK + cg * 8;
  float v[R][8], m[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = row + 16 * i;
    if (r < p.rows) {
      load8<T>(x + (int64_t)r * ldx + col, p.cols - col, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    }
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    m[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) m[i] = fmaxf(m[i], fabsf(v[i][j]));
    m[i] = max16(m[i]);
    const bool inf = __any(m[i] > FLT_MAX);
    if (inf) {
      m[i] = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) m[i] = fmaxf(m[i], finite_abs(v[i][j]));
      m[i] = max16(m[i]);
    }
    const float s = block_scale(m[i]), inv = 1.0f / s;
    const int r = row + 16 * i;
    float u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = inf ? code_value<true>(v[i][j], inv) : code_value<false>(v[i][j], inv);
    if (r >= p.rows) continue;
    if (cg == 0) p.scale[(int64_t)tc * p.rows + r] = s;
    if (col >= p.cols) continue;
    uint8_t* at = p.q + (int64_t)r * p.ldq + col;
    const uint32_t lo = codes4(u[0], u[1], u[2], u[3]), hi = codes4(u[4], u[5], u[6], u[7]);
    if (col + 8 <= p.cols) {
      *reinterpret_cast<uint2*>(at) = make_uint2(lo, hi);
    } else {
      for (int j = 0; j < p.cols - col; ++j) at[j] = (uint8_t)((j < 4 ? lo : hi) >> (8 * (j & 3)));
    }
  }
}

// ---- product -------------------------------------------------------------------------------------------------------
// 32 codes of a row from k0 on as a matrix operand: two aligned 16-byte loads; TAIL: zeros behind the row's end k.
template <bool TAIL>
__device__ __forceinline__ v8i load_codes(const uint8_t* row, int k0, int k) {
  v8i r;
  if constexpr (!TAIL) {
    __builtin_memcpy(&r, __builtin_assume_aligned(row + k0, 16), 32);
    return r;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int left = k - (k0 + 16 * h);
    uint4 w = make_uint4(0, 0, 0, 0);
    if (left > 0) w = *reinterpret_cast<const uint4*>(row + k0 + 16 * h);
    uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const int n = left - 4 * d;        // valid bytes of this word
      r[4 * h + d] = (int)(n >= 4 ? u[d] : n <= 0 ? 0u : u[d] & ((1u << (8 * n)) - 1u));
    }
  }
  return r;
}

// Sum over a block of 128 of the products of two fragments of 16 rows.  The 8-bit instruction adds the products of eight
// neighbouring k at the exponent of the largest with 14 bits below it (measured: 2^16 + 2^s keeps s >= 3 within the eight,
// s >= -7 outside): about 2^-16 of the result, 1/100 of a bfloat16 rounding, but far from binary32.  So binary32 results take
// the codes as bfloat16, which holds them exactly, through the bfloat16 instruction at half the rate: 2^-26 of the result.
template <bool EXACT>
struct Frag {
  v8i c;                                 // 32 codes
};
template <>
struct Frag<true> {
  v8bf w[4];                             // the same, in eights
};
__device__ __forceinline__ v8bf exact_eight(const v8i& c, int s) {
  v8bf w;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const v2bf lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * s + h], 1.0f, false);
    const v2bf hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * s + h], 1.0f, true);
    w[4 * h] = lo[0]; w[4 * h + 1] = lo[1]; w[4 * h + 2] = hi[0]; w[4 * h + 3] = hi[1];
  }
  return w;
}
template <bool EXACT>
__device__ __forceinline__ Frag<EXACT> make_frag(v8i c) {
  Frag<EXACT> f;
  if constexpr (EXACT) {
#pragma unroll
    for (int s = 0; s < 4; ++s) f.w[s] = exact_eight(c, s);
  } else {
    f.c = c;
  }
  return f;
}
template <bool EXACT>
__device__ __forceinline__ v4f block_product(const Frag<EXACT>& a, const Frag<EXACT>& b) {
  v4f p = {0, 0, 0, 0};
  if constexpr (EXACT) {
#pragma unroll
    for (int s = 0; s < 4; ++s) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.w[s], b.w[s], p, 0, 0, 0);
  } else {
    p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.c, b.c, p, 0, 0, 0, 0, 0, 0);
  }
  return p;
}

template <typename T> __device__ __forceinline__ void store_out(T* p, float v) { Store<T>::st(p, v); }
// four neighbouring results, of which `left` lie inside the row
template <typename T>
__device__ __forceinline__ void store4(T* p, const float (&o)[4], int left) {
  if (left >= 4) {
    if constexpr (sizeof(T) == 4) {
      __builtin_memcpy(p, o, 16);
    } else {
      const uint32_t w[2] = {pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
      __builtin_memcpy(p, w, 8);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) store_out<T>(p + e, o[e]);
  }
}

// ---- product of few rows ---------------------------------------------------------------------------------------------
// Bound by the reading of b, and at 16 MB of it by the latency of two rounds of loads: 1 x 4 096 x 4 096 with the quantiser
// 6.5 us, 16 x 8 192 x 4 096 10.8.  A workgroup makes 16 MT rows x 16 NT columns, its wavefronts take every WAVES-th block of K
// with fragments straight from memory (lane l of a fragment: row l % 16, 32 codes from 32 (l / 16) on, so four lanes read
// the 128 bytes of a row), UNROLL blocks in flight, and add up through LDS.  b is the first matrix operand, so a lane holds
// row l % 16 of the result and columns 4 (l / 16) .. + 3.
// X: a is not there in codes: x is quantised on the way, each lane 32 elements of its row, the block's maximum over the
// row's four lanes (every workgroup does so for itself: the rows are few).
template <typename T>
struct Elements {                        // 32 elements of a row as they lie in memory
  uint32_t w[8 * sizeof(T)];
};
template <typename T, bool TAIL>
__device__ __forceinline__ Elements<T> load_elements(const T* row, int left, bool there) {
  Elements<T> x;
  if constexpr (!TAIL) {
    if (there) {
      __builtin_memcpy(x.w, row, sizeof(x.w));
    } else {
#pragma unroll
      for (int i = 0; i < (int)(8 * sizeof(T)); ++i) x.w[i] = 0u;
    }
  } else {
    T e[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) e[i] = there && i < left ? row[i] : (T)0;
    __builtin_memcpy(x.w, e, sizeof(x.w));
  }
  return x;
}
template <bool INF>
__device__ __forceinline__ float row_maximum(const float (&v)[32]) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 32; ++i) m = fmaxf(m, magnitude<INF>(v[i]));
  return max_rows(m);
}
template <bool INF>
__device__ __forceinline__ v8i codes_of(const float (&v)[32], float inv) {
  v8i c;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    c[i] = (int)codes4(code_value<INF>(v[4 * i], inv), code_value<INF>(v[4 * i + 1], inv), code_value<INF>(v[4 * i + 2], inv), code_value<INF>(v[4 * i + 3], inv));
  return c;
}
template <typename T>
__device__ __forceinline__ v8i quantize_elements(const Elements<T>& x, float& scale) {
  float v[32];
#pragma unroll
  for (int i = 0; i < 32; ++i)
    v[i] = sizeof(T) == 4 ? __uint_as_float(x.w[i % (8 * sizeof(T))]) : __uint_as_float(i & 1 ? x.w[i / 2] & 0xFFFF0000u : x.w[i / 2] << 16);
  float m = row_maximum<false>(v);
  if (__any(m > FLT_MAX)) {
    m = row_maximum<true>(v);
    scale = block_scale(m);
    return codes_of<true>(v, 1.0f / scale);
  }
  scale = block_scale(m);
  return codes_of<false>(v, 1.0f / scale);
}

template <typename T, bool X, bool BROWS, int MT, int NT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_fp8_few(const void* __restrict__ a, int64_t lda, const float* __restrict__ sa,
                                                        const uint8_t* __restrict__ b, int64_t ldb, const float* __restrict__ sb,
                                                        const float* __restrict__ bias, int m, int n, int k, T* __restrict__ y,
                                                        int64_t ldy, int tiles_n, int first) {
  constexpr bool EXACT = sizeof(T) == 4;
  constexpr int UNROLL = MT * NT >= 4 ? 2 : 4;
  __shared__ __align__(16) float red[WAVES][MT * NT][64][4];
  const int tile = first + (int)blockIdx.x, tm = tile / tiles_n, tn = tile - tm * tiles_n;
  const int m0 = tm * 16 * MT, n0 = tn * 16 * NT;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kb = (k + BLK - 1) / BLK;
  int64_t a_off[MT], b_off[NT];
  int a_row[MT], n_blk[NT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    a_row[i] = m0 + 16 * i + l16 < m ? m0 + 16 * i + l16 : m - 1;      // rows behind the end repeat the last one, and are not stored
    a_off[i] = (int64_t)a_row[i] * lda;
  }
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int r = n0 + 16 * j + l16;
    b_off[j] = (int64_t)(r < n ? r : n - 1) * ldb;
    n_blk[j] = (n0 + 16 * j < n ? n0 + 16 * j : n - 1) / BLK;
  }
  v4f acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = (v4f){0, 0, 0, 0};
  auto blocks = [&](int c0, auto count, auto end) {
    constexpr int U = decltype(count)::value;
    constexpr bool TAIL = decltype(end)::value;
    v8i rb[U][NT], rx[U][MT];
    Elements<T> ex[X ? U : 1][MT];
    float s[U][MT];
    v4f cs[U][NT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * WAVES, at = c * BLK + 32 * g;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        rb[u][j] = load_codes<TAIL>(b + b_off[j], at, k);
        if constexpr (BROWS) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int col = n0 + 16 * j + 4 * g + e;
            cs[u][j][e] = sb[(int64_t)c * n + (col < n ? col : n - 1)];
          }
        } else {
          const float f = sb[(int64_t)n_blk[j] * kb + c];
          cs[u][j] = (v4f){f, f, f, f};
        }
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        if constexpr (!X) {
          rx[u][i] = load_codes<TAIL>((const uint8_t*)a + a_off[i], at, k);
          s[u][i] = sa[(int64_t)c * m + a_row[i]];
        } else {
          ex[u][i] = load_elements<T, TAIL>((const T*)a + a_off[i] + at, k - at, m0 + 16 * i + l16 < m);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (X) {
#pragma unroll
        for (int i = 0; i < MT; ++i) rx[u][i] = quantize_elements<T>(ex[u][i], s[u][i]);
      }
      Frag<EXACT> fb[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) fb[j] = make_frag<EXACT>(rb[u][j]);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const Frag<EXACT> fa = make_frag<EXACT>(rx[u][i]);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const v4f p = block_product<EXACT>(fb[j], fa);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[e], s[u][i] * cs[u][j][e], acc[i][j][e]);
        }
      }
    }
  };
  const int whole = k / BLK;
  int c = wave;
  for (; c + (UNROLL - 1) * WAVES < whole; c += UNROLL * WAVES) blocks(c, std::integral_constant<int, UNROLL>(), std::false_type());
  if constexpr (UNROLL > 1)
    for (; c < whole; c += WAVES) blocks(c, std::integral_constant<int, 1>(), std::false_type());
  if (c < kb) blocks(c, std::integral_constant<int, 1>(), std::true_type());
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) *reinterpret_cast<v4f*>(red[wave][i * NT + j][lane]) = acc[i][j];
  __syncthreads();
  for (int at = threadIdx.x; at < MT * NT * 64; at += WAVES * 64) {
    const int tile = at >> 6, l = at & 63;
    v4f v = *reinterpret_cast<const v4f*>(red[0][tile][l]);
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += *reinterpret_cast<const v4f*>(red[w][tile][l]);
    const int row = m0 + 16 * (tile / NT) + (l & 15), col = n0 + 16 * (tile % NT) + 4 * (l >> 4);
    if (row >= m || col >= n) continue;
    float o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = v[e] + (bias && col + e < n ? bias[col + e] : 0.0f);
    store4<T>(y + (int64_t)row * ldy + col, o, n - col);
  }
}

// ---- product of many rows: tiles staged in LDS -----------------------------------------------------------------------
// A group of WGM x WGN wavefronts makes a tile of BM x BN results, a wavefront 16 MI x 16 NJ of them, in steps of one
// block (128 codes) of K.  Where tiles are few, KG groups of a workgroup share K: more loads in flight on a compute unit.
// The codes of a step go from memory straight into LDS (16 bytes a lane, a row of 128 in eight pieces) while the step before
// is multiplied; two such stages.  The first matrix operand is b and the second a, so that a
// lane's results are four neighbouring columns of one row: the row's scale is one register, and with the order of b's rows
// below a lane's NJ fragments are 4 NJ columns in a row, which it stores in 16-byte pieces.
//   piece c of row r lies at piece c ^ key(r) of that row, eight keys among the 16 rows of a fragment, and lane group g reads
//   pieces g and g + 4 (any order of K will do, as long as it is b's too): 5.8 cycles a read, as for consecutive addresses;
//   pieces 2 g and 2 g + 1 take 8.0
// Bound by the matrix cores and by what of a tile's first load and last store nothing runs beside (one workgroup of
// 256 x 256 fills a compute unit): 16 384 x 4 096 x 4 096 in bfloat16 247 - 268 us by box and operands, 2.05 - 2.2 PFLOP/s (under
// the profiler 251 at least, 281 in the mean); 4 096 x 4 096 x 4 096 63.  b in row blocks, 256 x 128 tiles: 355 and 84.
// Binary32 results: by turning codes into bfloat16 (an instruction of half rate for two codes, 16 times a fragment) beside
// the bfloat16 products: 4 096 x 4 096 x 4 096 145 us, 950 TFLOP/s, b in row blocks 153 (alone; after the other launches of a
// backward pass, under the profiler, 164 - 178).
template <int NJ> __device__ __forceinline__ int b_row(int i, int j) { return (i >> 2) * (4 * NJ) + j * 4 + (i & 3); }   // row of b in fragment j, place i
__device__ __forceinline__ int a_key(int r) { return (r >> 1) & 7; }
template <int NJ> __device__ __forceinline__ int b_key(int r) { return ((r / (4 * NJ)) & 3) << 1 | ((r >> 1) & 1); }

// 16 bytes of each lane from a buffer straight into LDS: lane l writes at lds + 16 l; offsets past the buffer's range deliver
// zeros.  In assembly, because the compiler would wait for every such load before the next read of LDS, whichever part
// of it that reads; the kernel waits itself (vmcnt) where it needs the data.  There is no register result.  (The instruction
// may read m0 one wait state after it was written, which the compiler does not see here: s_nop.)
typedef int v4i __attribute__((ext_vector_type(4)));
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"      // m0 is a reserved register: the compiler keeps nothing in it from one of its own instructions to another
__device__ __forceinline__ void load_to_lds(v4i rsrc, unsigned lds, unsigned voffset, unsigned soffset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(voffset), "s"(rsrc), "s"(soffset) : "memory", "m0");
}
#pragma clang diagnostic pop
// a raw buffer of `bytes` bytes, at most 2^31 - 1 of them, from p on
__device__ __forceinline__ v4i buffer_of(const void* p, int64_t bytes) {
  const uint64_t a = (uint64_t)(uintptr_t)p;
  const int n = bytes < 0x7FFFFFFF ? (int)bytes : 0x7FFFFFFF;
  const v4i r = {__builtin_amdgcn_readfirstlane((int)(uint32_t)a), __builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xFFFF)),
                 __builtin_amdgcn_readfirstlane(n), 0x00020000};
  return r;
}

// Tiles in an order in which workgroups that run at the same time share rows of a and b: consecutive workgroups go to
// different dies (8, each with its own L2), so each die takes a contiguous run of tiles, and a run walks columns of 6 tiles:
// its 32 tiles at a time read few different rows of a and of b (16 384 x 4 096 x 4 096: 250 us; columns of 4 254, of 8 258;
// 8 192 x 8 192 x 2 048 143, 149, 151; binary32 16 384 x 4 096 x 1 024 228, 236, 245, 2 048 x 32 768 x 4 096 with b in rows 617, 622, 635;
// 4 096 x 16 384 x 4 096, 2 048 x 32 768 x 4 096, 4 352 x 4 096 x 4 096, 1 500 x 4 096 x 4 096 within 1 % or 6 the least).
constexpr int GROUP = 6;
__device__ __forceinline__ void tile_of(int b, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int total = tiles_m * tiles_n, xcd = b & 7, per = total >> 3, more = total & 7;
  const int id = xcd * per + (xcd < more ? xcd : more) + (b >> 3);
  const int group = GROUP * tiles_n, gi = id / group, first = gi * GROUP, in = id - gi * group;
  const int height = tiles_m - first < GROUP ? tiles_m - first : GROUP;
  tm = first + in % height;
  tn = in / height;
}

template <typename T, bool BROWS, int WGM, int WGN, int MI, int NJ, int KG>
__global__ __launch_bounds__(WGM * WGN * KG * 64) void k_fp8_tile(const uint8_t* __restrict__ a, int64_t lda, const float* __restrict__ sa,
                                                             const uint8_t* __restrict__ b, int64_t ldb, const float* __restrict__ sb,
                                                             const float* __restrict__ bias, int m, int n, int k, T* __restrict__ y,
                                                             int64_t ldy, int tiles_m, int tiles_n, int first_tile) {
  constexpr bool EXACT = sizeof(T) == 4;
  constexpr int NTH = WGM * WGN * 64, NWV = WGM * WGN;         // threads and wavefronts of a group
  constexpr int BM = WGM * MI * 16, BN = WGN * NJ * 16;
  constexpr int STAGE = (BM + BN) * BLK;                       // bytes of codes of a step
  constexpr int CB = BN >= BLK ? BN / BLK : 1;                 // column blocks of a tile
  constexpr int NS = BROWS ? BM + BN : CB * BM;                // scales of a step: rows' and columns', or rows' times the block's
  constexpr int SPT = (NS + NTH - 1) / NTH;
  constexpr int LA = BM / 8 / NWV, LB = BN / 8 / NWV, LOADS = LA + LB;      // a wavefront's loads of a step
  static_assert(BM % (16 * NWV) == 0 && BN % (16 * NWV) == 0 && NJ == 4, "whole loads, keys as the loads assume them");
  static_assert(MI * NJ >= LOADS, "a load beside a product");
  __shared__ __align__(1024) uint8_t all_codes[KG][2][STAGE];
  __shared__ __align__(16) float all_scales[KG][2][NS];
  const int kg = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NTH);
  uint8_t (*codes)[STAGE] = all_codes[kg];
  float (*scales)[NS] = all_scales[kg];
  const int t = threadIdx.x - kg * NTH, lane = t & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6), wm = wave / WGN, wn = wave - wm * WGN;
  int tm, tn;
  tile_of(first_tile + (int)blockIdx.x, tiles_m, tiles_n, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int kb = (k + BLK - 1) / BLK;
  const int per = (kb + KG - 1) / KG, first = kg * per;        // blocks of K of a group; behind the last one they are zeros

  // loads: an instruction moves eight rows, lane l piece l % 8 (before the keys) of row l / 8; rows behind the end lie
  // outside the buffer's range and become zeros (eight rows all behind it: the last row and zeros; they are not stored).
  // So a range is never shorter than a row, and a step's offset, which the hardware takes off the range, never longer.
  // Eight rows that begin at a multiple of 8 share all of the key but what l / 8 gives, and the two addends are bits of
  // their own.
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)codes[0];
  const int l8 = lane >> 3;
  const int a_piece = (lane & 7) ^ a_key(l8), b_piece = (lane & 7) ^ b_key<NJ>(l8);
  v4i ra[LA], rb[LB];
#pragma unroll
  for (int i = 0; i < LA; ++i) {
    const int r0 = m0 + (wave * LA + i) * 8, r = r0 < m ? r0 : m - 1;
    ra[i] = buffer_of(a + (int64_t)r * lda, (m - r) * lda);
  }
#pragma unroll
  for (int i = 0; i < LB; ++i) {
    const int r0 = n0 + (wave * LB + i) * 8, r = r0 < n ? r0 : n - 1;
    rb[i] = buffer_of(b + (int64_t)r * ldb, (n - r) * ldb);
  }
  // instruction i of the loads of step c; TAIL: pieces behind the rows' end become zeros too
  auto load_part = [&](int c, int i, bool tail) {
    const bool is_a = i < LA;
    const int r = is_a ? (wave * LA + i) * 8 : (wave * LB + (i - LA) / 2 * 2) * 8;       // two instructions share a key of b
    const int piece = is_a ? a_piece ^ (i & 1 ? 4 : 0) : b_piece ^ b_key<NJ>(r);
    unsigned o = l8 * (unsigned)(is_a ? lda : ldb) + piece * 16;
    if (tail && c * BLK + piece * 16 >= k) o = 0x80000000u;
    load_to_lds(is_a ? ra[i < LA ? i : 0] : rb[i < LA ? 0 : i - LA],
                lds0 + ((c - first) & 1) * STAGE + (is_a ? wave * LA + i : BM / 8 + wave * LB + i - LA) * 1024, o, (unsigned)__builtin_amdgcn_readfirstlane((KG > 1 && c >= kb ? kb - 1 : c) * BLK));
  };
  auto load_scales = [&](int at_c, float (&v)[SPT]) {
    const int c = at_c < kb ? at_c : kb - 1;
#pragma unroll
    for (int i = 0; i < SPT; ++i) {
      const int at = t + i * NTH;
      if (NS % NTH != 0 && at >= NS) break;
      if constexpr (BROWS) {
        const bool is_a = at < BM;
        const int r = is_a ? m0 + at : n0 + at - BM, end = is_a ? m : n;
        v[i] = (is_a ? sa : sb)[(int64_t)c * end + (r < end ? r : end - 1)];
        if (KG > 1 && at_c >= kb) v[i] = 0.0f;
      } else {
        const int cb = at / BM, r = m0 + at - cb * BM;
        int blk = n0 / BLK + cb;
        if (blk > (n - 1) / BLK) blk = (n - 1) / BLK;
        v[i] = sa[(int64_t)c * m + (r < m ? r : m - 1)] * sb[(int64_t)blk * kb + c];
        if (KG > 1 && at_c >= kb) v[i] = 0.0f;
      }
    }
  };
  auto store_scales = [&](int buf, const float (&v)[SPT]) {
#pragma unroll
    for (int i = 0; i < SPT; ++i) {
      const int at = t + i * NTH;
      if (NS % NTH != 0 && at >= NS) break;
      scales[buf][at] = v[i];
    }
  };

  // this wavefront's loads are in LDS, then everybody's, and nobody reads what the next ones will overwrite
  auto arrive = [&] {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };
  // the piece that holds the end of the rows, in the last block: zeros behind it.  Every group comes here at the same step.
  auto cut_tail = [&](int c) {
    const int cut = (k % BLK) >> 4, keep = k & 15, buf = (c - first) & 1;
    for (int r = t; r < BM + BN && c == kb - 1; r += NTH) {
      const int key = r < BM ? a_key(r) : b_key<NJ>(r - BM);
      uint32_t* w = reinterpret_cast<uint32_t*>(codes[buf] + r * BLK + (cut ^ key) * 16);
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const int left = keep - 4 * d;
        w[d] = left >= 4 ? w[d] : left <= 0 ? 0u : w[d] & ((1u << (8 * left)) - 1u);
      }
    }
    __syncthreads();
  };

  v4f acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = (v4f){0, 0, 0, 0};

  // a lane's two 16-byte pieces of a fragment
  const int arow = wm * MI * 16 + l16;
  auto raw = [&](const uint8_t* row, int key) {
    union { uint4 h[2]; v8i v; } u;
    u.h[0] = *reinterpret_cast<const uint4*>(row + (g ^ key) * 16);
    u.h[1] = *reinterpret_cast<const uint4*>(row + ((g + 4) ^ key) * 16);
    return u.v;
  };
  auto raw_a = [&](int buf, int i) { return raw(codes[buf] + (arow + i * 16) * BLK, a_key(arow)); };
  auto raw_b = [&](int buf, int j) {
    const int r = wn * NJ * 16 + b_row<NJ>(l16, j);
    return raw(codes[buf] + (BM + r) * BLK, b_key<NJ>(r));
  };
  auto row_scale = [&](int buf, int i) { return scales[buf][(BROWS ? 0 : (wn * NJ * 16 / BLK) * BM) + arow + i * 16]; };
  constexpr int AHEAD = MI > 2 ? 2 : 1;          // fragments of a that are on their way from LDS
  // Binary32 results: the next fragment of a is turned into bfloat16 a quarter at a time beside the products of the present
  // one (fn), a fragment of b before the first product that takes it (LATE_B).  All where a step begins they took 551 us at
  // 16 384 x 4 096 x 4 096, so 522, and held registers for longer (1 000 x 1 000 x 1 024, b in row blocks, 13.2 and 10.1).  Only
  // 256 x 128 tiles with b in row blocks gain nothing (in a backward pass of 4 096 x 4 096 x 4 096 167 and, late, 169).
  constexpr bool LATE_B = EXACT && !(BROWS && NWV == 8);
  Frag<EXACT> fb[NJ], fn;
  v4f cs[NJ];
  v8i ahead[AHEAD], raw_fb[LATE_B ? NJ : 1];
  float s_ahead[AHEAD];
  auto begin_step = [&](int buf) {
    if constexpr (LATE_B) raw_fb[0] = raw_b(buf, 0);
    else fb[0] = make_frag<EXACT>(raw_b(buf, 0));
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      ahead[i] = raw_a(buf, i);
      s_ahead[i] = row_scale(buf, i);
    }
#pragma unroll
    for (int j = 1; j < NJ; ++j) {
      if constexpr (LATE_B) raw_fb[j] = raw_b(buf, j);
      else fb[j] = make_frag<EXACT>(raw_b(buf, j));
    }
    if constexpr (BROWS) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) cs[j] = *reinterpret_cast<const v4f*>(&scales[buf][BM + wn * NJ * 16 + g * 4 * NJ + j * 4]);
    }
  };
  auto add_scaled = [&](int i, int j, const v4f& p, float s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[e], BROWS ? s * cs[j][e] : s, acc[i][j][e]);
  };
  // The codes of step c: rows 16 i .. + 15 are multiplied while the sums of those before are scaled and added, two fragments
  // of a are on their way, and the next step's codes are asked for, a load beside a product (all at once they would stand in
  // front of the reads of LDS; later ones would not be there in time).  When the last rows' products are issued, everything
  // that the step reads from LDS has been read: the wait for the next step's codes, the barrier and the first reads of that
  // step run beside them.
  enum { LAST = 0, MORE = 1, MORE_TAIL = 2 };
  auto step = [&](int c, auto what) {
    constexpr int W = decltype(what)::value;
    const int buf = (c - first) & 1;
    v4f p[2][NJ];
    float s_at[2], sv[SPT];
    if constexpr (W != LAST) load_scales(c + 1, sv);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const Frag<EXACT> fa = EXACT && i > 0 ? fn : make_frag<EXACT>(ahead[i % AHEAD]);
      s_at[i & 1] = s_ahead[i % AHEAD];
      if (i + AHEAD < MI) {
        ahead[i % AHEAD] = raw_a(buf, i + AHEAD);
        s_ahead[i % AHEAD] = row_scale(buf, i + AHEAD);
      }
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if constexpr (LATE_B) {
          if (i == 0) fb[j] = make_frag<EXACT>(raw_fb[j]);
        }
        p[i & 1][j] = block_product<EXACT>(fb[j], fa);
        if constexpr (EXACT) {
          if (i + 1 < MI) fn.w[j] = exact_eight(ahead[(i + 1) % AHEAD], j);
        }
        if (i > 0) add_scaled(i - 1, j, p[(i - 1) & 1][j], s_at[(i - 1) & 1]);
        if constexpr (W != LAST) {
          if (i * NJ + j < LOADS) load_part(c + 1, i * NJ + j, W == MORE_TAIL);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    // held here: below the branches that follow, the addends would need registers of their own
#pragma unroll
    for (int i = 0; i + 1 < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) asm volatile("" : "+v"(acc[i][j]));
    if constexpr (W != LAST) {
      store_scales(buf ^ 1, sv);
      arrive();
      if constexpr (W == MORE_TAIL) {
        if ((k & 15) != 0 && (KG == 1 || c + 1 - first == (kb - 1) % per)) cut_tail(c + 1);
      }
    }
    float s_last = s_at[(MI - 1) & 1];
    v4f c_last[NJ];
    if constexpr (BROWS) {                       // the next step's column scales are read over these
#pragma unroll
      for (int j = 0; j < NJ; ++j) c_last[j] = s_last * cs[j];
    }
    if constexpr (W != LAST) begin_step(buf ^ 1);
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[MI - 1][j][e] = fmaf(p[(MI - 1) & 1][j][e], BROWS ? c_last[j][e] : s_last, acc[MI - 1][j][e]);
#pragma unroll
    for (int j = 0; j < NJ; ++j) asm volatile("" : "+v"(acc[MI - 1][j]));
  };
  {
    float sv[SPT];
    load_scales(first, sv);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load_part(first, i, KG > 1 || kb == 1);
    store_scales(0, sv);
    arrive();
    if ((k & 15) != 0 && (kb - 1) % per == 0) cut_tail(first);
    begin_step(0);
  }
  int c = first;
  const int end = first + per;
  if constexpr (KG == 1) {
    for (; c + 2 < end; ++c) step(c, std::integral_constant<int, MORE>());
    if (c + 1 < end) {
      step(c, std::integral_constant<int, MORE_TAIL>());
      ++c;
    }
  } else {
    for (; c + 1 < end; ++c) step(c, std::integral_constant<int, MORE_TAIL>());
  }
  step(c, std::integral_constant<int, LAST>());
  if constexpr (KG > 1) {                        // the groups' sums, added up in their order through LDS
    static_assert((KG - 1) * BM * BN * 4 <= (int)sizeof(all_codes), "room for the sums");
    v4f* sums = reinterpret_cast<v4f*>(&all_codes[0][0][0]);
    __syncthreads();
    if (kg > 0) {
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) sums[((kg - 1) * MI * NJ + i * NJ + j) * NTH + t] = acc[i][j];
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int q = 0; q < KG - 1; ++q)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] += sums[(q * MI * NJ + i * NJ + j) * NTH + t];
  }
  // results: lane: row l16 of each 16, columns 4 NJ g .. of the wavefront's
  const int col = n0 + wn * NJ * 16 + g * 4 * NJ;
  if (col >= n) return;
  float bb[4 * NJ];
#pragma unroll
  for (int j = 0; j < 4 * NJ; ++j) bb[j] = bias && col + j < n ? bias[col + j] : 0.0f;
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int row = m0 + arow + i * 16;
    if (row >= m) continue;
    T* p = y + (int64_t)row * ldy + col;
    float o[4 * NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[4 * j + e] = acc[i][j][e] + bb[4 * j + e];
    if (col + 4 * NJ <= n) {
      if constexpr (EXACT) {
        __builtin_memcpy(p, o, sizeof(o));
      } else {
        uint32_t w[2 * NJ];
#pragma unroll
        for (int j = 0; j < 2 * NJ; ++j) w[j] = pack_bf16(o[2 * j], o[2 * j + 1]);
        __builtin_memcpy(p, w, sizeof(w));
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4 * NJ; ++j)
        if (col + j < n) store_out<T>(p + j, o[j]);
    }
  }
}

constexpr int64_t kSizeMax = 0x7FFFFFFF - 512;   // the end of the last tile is an int
bool sizes_ok(int64_t m, int64_t n, int64_t k) { return m >= 0 && n >= 0 && k >= 1 && m <= kSizeMax && n <= kSizeMax && k <= kSizeMax; }
bool codes_ok(const void* p, int64_t ld, int64_t cols) { return ((uintptr_t)p & 15) == 0 && ld >= cols && ld % 16 == 0 && ld < ((int64_t)1 << 40); }

struct Product {
  const void* a; int64_t lda; const float* sa;
  const uint8_t* b; int64_t ldb; const float* sb;
  int b_blocks;
  const float* bias;
  int64_t m, n, k;
  int dtype;
  void* y; int64_t ldy;
};

// everything but a, which the caller may make itself
int check_product(const char* who, const Product& p) {
  if (!p.b || !p.sb || !p.y) return fail(AE_EINVAL, "%s: null argument", who);
  if (!codes_ok(p.b, p.ldb, p.k)) return fail(AE_EINVAL, "%s: rows of codes must begin on 16-byte borders and not overlap", who);
  if (((uintptr_t)p.sb | (uintptr_t)p.bias) & 3) return fail(AE_EINVAL, "%s: misaligned scales or bias", who);
  if (p.ldy < p.n || p.ldy >= ((int64_t)1 << 40) || (uintptr_t)p.y % dtype_size(p.dtype)) return fail(AE_EINVAL, "%s: bad y", who);
  return AE_OK;
}

template <typename T, bool BROWS, int WGM, int WGN, int MI, int NJ, int KG>
int launch_tile(const Product& p, hipStream_t s) {
  constexpr int BM = WGM * MI * 16, BN = WGN * NJ * 16;
  const int64_t tm = (p.m + BM - 1) / BM, tn = (p.n + BN - 1) / BN;
  if (tm * tn > 0x7FFFFFFF) return fail(AE_EINVAL, "model_fp8_matmul: result too large");
  const int64_t most = launch_blocks(WGM * WGN * KG * 64);
  for (int64_t first = 0; first < tm * tn; first += most) {
    const int64_t left = tm * tn - first;
    hipLaunchKernelGGL((k_fp8_tile<T, BROWS, WGM, WGN, MI, NJ, KG>), dim3((unsigned)(left < most ? left : most)), dim3(WGM * WGN * KG * 64), 0, s, (const uint8_t*)p.a, p.lda,
                       p.sa, p.b, p.ldb, p.sb, p.bias, (int)p.m, (int)p.n, (int)p.k, (T*)p.y, p.ldy, (int)tm, (int)tn, (int)first);
  }
  return launch_status("fp8_matmul");
}
// The largest tiles that still leave no compute unit idle, by the number of tiles (256 compute units; times with the quantiser):
//   up to 256 of 64 x 64     four groups of K    200 x 4 096 x 4 096 in bfloat16 22 us (two groups 26, one 34; 128 x 128 in two groups 33)
//   up to 512                two groups          400 x 4 096 x 4 096 30 us (four 36, one 35; 128 x 128 in two groups 33); binary32: 128 x 64, the product 32.8 us (64 x 64 34.2)
//   up to 256 of 128 x 128   two groups of K     777 x 4 096 x 4 096 36 us (one 44; 64 x 64 39; 256 x 256 57)
//   more                     one group, two workgroups to a compute unit    1 500 x 4 096 x 4 096 49 us (256 x 256 59; 64 x 64 63)
//   from 192 of 256 x 256    1 500 x 8 192 x 2 048 41 us (128 x 128 48).  Binary32 results and b in row blocks need more registers:
//                            256 x 128, and only where it is a whole round or many (1 500 x 4 096 x 4 096 78 us, 128 x 128 83; 1 500 x 8 192 x 2 048 88, 78).
// Products alone at K = 2 048, in us.  bfloat16, b in tiles, by the number of 256 x 256 tiles: 128 29 (128 x 128: 25), 176 31 (38), 208 32 (45),
// 272 59 (58), 512 69 (89).  By the number of 256 x 128 tiles, binary32 with b in tiles / in rows, bfloat16 with b in rows:
//   160 39 / 44 / 23 (128 x 128: 42 / 46 / 23)   320 76 / 82 / 44 (66 / 70 / 37)    416 82 / 87 / 45 (82 / 85 / 45)   480 86 / 92 / 47 (86 / 89 / 47)
//   576 116 / 124 / 66 (104 / 107 / 58)          768 128 / 136 / 70 (128 / 133 / 71)   896 160 / 172 / 88 (148 / 153 / 81)   1 024 165 / 178 / 93 (168 / 172 / 93)
template <typename T, bool BROWS>
int launch_tiles(const Product& p, hipStream_t s) {
  auto tiles = [&](int64_t bm, int64_t bn) { return ((p.m + bm - 1) / bm) * ((p.n + bn - 1) / bn); };
  constexpr bool WIDE = sizeof(T) == 4 || BROWS;
  if constexpr (WIDE) {
    const int64_t t = tiles(256, 128);
    if ((t >= 192 && t <= 256) || (t > 448 && t <= 512) || t >= 1024) return launch_tile<T, BROWS, 4, 2, 4, 4, 1>(p, s);
  } else {
    if (tiles(256, 256) >= 192) return launch_tile<T, BROWS, 2, 4, 8, 4, 1>(p, s);
  }
  if (tiles(64, 64) <= 256) return launch_tile<T, BROWS, 4, 1, 1, 4, 4>(p, s);
  if (tiles(64, 64) <= 512) return launch_tile<T, BROWS, 4, 1, WIDE ? 2 : 1, 4, 2>(p, s);
  if (tiles(128, 128) <= 256) return launch_tile<T, BROWS, 2, 2, 4, 4, 2>(p, s);
  return launch_tile<T, BROWS, 2, 2, 4, 4, 1>(p, s);
}
template <typename T, bool X, bool BROWS, int MT, int NT, int WAVES>
int launch_few(const Product& p, hipStream_t s) {
  const int64_t tm = (p.m + 16 * MT - 1) / (16 * MT), tn = (p.n + 16 * NT - 1) / (16 * NT);
  if (tm * tn > 0x7FFFFFFF) return fail(AE_EINVAL, "model_fp8_matmul: result too large");
  const int64_t most = launch_blocks(WAVES * 64);
  for (int64_t first = 0; first < tm * tn; first += most) {
    const int64_t left = tm * tn - first;
    hipLaunchKernelGGL((k_fp8_few<T, X, BROWS, MT, NT, WAVES>), dim3((unsigned)(left < most ? left : most)), dim3(WAVES * 64), 0, s, (const void*)p.a, p.lda, p.sa, p.b,
                       p.ldb, p.sb, p.bias, (int)p.m, (int)p.n, (int)p.k, (T*)p.y, p.ldy, (int)tn, (int)first);
  }
  return launch_status("fp8_matmul");
}
// x quantised on the way: every workgroup reads and quantises all of x, so it takes as many columns as leave 256 workgroups
constexpr int64_t kQuantizeOnTheWay = 16;        // rows
template <typename T>
int launch_few_elements(const Product& p, hipStream_t s) {
  if (p.n >= 64 * 256) return launch_few<T, true, false, 1, 4, 8>(p, s);
  if (p.n >= 32 * 256) return launch_few<T, true, false, 1, 2, 8>(p, s);
  return launch_few<T, true, false, 1, 1, 8>(p, s);
}
template <typename T, bool BROWS>
int launch_rows(const Product& p, hipStream_t s) {
  // the tiles' offsets are 31 bits: longer rows, of which there are then few, go through the kernel of few rows at any m
  if (p.m > 64 && p.lda < (1 << 23) && p.ldb < (1 << 23)) return launch_tiles<T, BROWS>(p, s);
  if (p.m <= 16) return launch_few<T, false, BROWS, 1, 1, 8>(p, s);
  if (p.m <= 32) return launch_few<T, false, BROWS, 2, 1, 8>(p, s);
  return launch_few<T, false, BROWS, 4, 1, 8>(p, s);
}

int launch_product(const Product& p, hipStream_t s) {
  if (p.dtype == AE_BF16) return p.b_blocks == AE_FP8_ROWS ? launch_rows<bf16_t, true>(p, s) : launch_rows<bf16_t, false>(p, s);
  return p.b_blocks == AE_FP8_ROWS ? launch_rows<float, true>(p, s) : launch_rows<float, false>(p, s);
}

template <typename T>
int launch_quantize(const void* x, int64_t rows, int64_t cols, int64_t ldx, int blocks, void* q, int64_t ldq, float* scale, void* qt,
                    int64_t ldqt, float* scale_t, hipStream_t s) {
  const int64_t tr = (rows + BLK - 1) / BLK, tc = (cols + BLK - 1) / BLK;
  constexpr int QROWS = 2;                       // 16 384 x 4 096 in bfloat16: 37 us, 5.4 TB/s (one 38, four 45; 128 x 128 tiles 46)
  const int64_t row_blocks = (rows + 16 * QROWS - 1) / (16 * QROWS) * tc, most = launch_blocks(256);
  const bool rows_alone = blocks == AE_FP8_ROWS && !qt;
  if (rows_alone ? row_blocks > 0x7FFFFFFF : tr * tc > most) return fail(AE_EINVAL, "model_fp8_quantize: matrix too large");      // over 288 GB in any case
  QuantizeArgs p = {(int)rows, (int)cols, (int)tc, 0, (uint8_t*)q, ldq, scale, (uint8_t*)qt, ldqt, scale_t};
#define QUANT(TI, A, B)                                                                                                         \
  hipLaunchKernelGGL((k_fp8_quantize<T, TI, A, B>), dim3((unsigned)(tr * tc)), dim3(256), 0, s, (const T*)x, ldx, p)
  if (blocks == AE_FP8_TILES) {
    if (q && qt) QUANT(true, true, true);
    else if (q) QUANT(true, true, false);
    else QUANT(true, false, true);
  } else {
    if (q && qt) QUANT(false, true, true);
    else if (qt) QUANT(false, false, true);
    else
      for (int64_t first = 0; first < row_blocks; first += most) {
        const int64_t left = row_blocks - first;
        p.first = (int)first;
        hipLaunchKernelGGL((k_fp8_quantize_rows<T, QROWS>), dim3((unsigned)(left < most ? left : most)), dim3(256), 0, s, (const T*)x, ldx, p);
      }
  }
#undef QUANT
  return launch_status("fp8_quantize");
}

int64_t align16(int64_t v) { return (v + 15) / 16 * 16; }

}  // namespace
}  // namespace ae

extern "C" int model_fp8_quantize(const void* x, int64_t rows, int64_t cols, int64_t ldx, int dtype, int blocks, void* q, int64_t ldq,
                                  float* scale, void* qt, int64_t ldqt, float* scale_t, void* stream) {
  using namespace ae;
  if (dtype != AE_F32 && dtype != AE_BF16) return fail(AE_EINVAL, "model_fp8_quantize: bad dtype");
  if (blocks != AE_FP8_ROWS && blocks != AE_FP8_TILES) return fail(AE_EINVAL, "model_fp8_quantize: blocks must be AE_FP8_ROWS or AE_FP8_TILES");
  if (rows < 0 || cols < 0 || rows > kSizeMax || cols > kSizeMax || ldx < cols || ldx >= ((int64_t)1 << 40)) return fail(AE_EINVAL, "model_fp8_quantize: bad size");
  if (rows == 0 || cols == 0) return AE_OK;
  if ((!q) != (!scale) || (!qt) != (!scale_t)) return fail(AE_EINVAL, "model_fp8_quantize: codes and their scales go together");
  if (!q && !qt) return fail(AE_EINVAL, "model_fp8_quantize: no output");
  if (!x || (uintptr_t)x % dtype_size(dtype)) return fail(AE_EINVAL, "model_fp8_quantize: x is null or not on an element's border");
  if ((q && !codes_ok(q, ldq, cols)) || (qt && !codes_ok(qt, ldqt, rows)))
    return fail(AE_EINVAL, "model_fp8_quantize: rows of codes must begin on 16-byte borders and not overlap");
  if (((uintptr_t)scale | (uintptr_t)scale_t) & 3) return fail(AE_EINVAL, "model_fp8_quantize: misaligned scales");
  hipStream_t s = (hipStream_t)stream;
  return dtype == AE_BF16 ? launch_quantize<bf16_t>(x, rows, cols, ldx, blocks, q, ldq, scale, qt, ldqt, scale_t, s)
                          : launch_quantize<float>(x, rows, cols, ldx, blocks, q, ldq, scale, qt, ldqt, scale_t, s);
}

extern "C" int model_fp8_matmul_workspace(int64_t m, int64_t n, int64_t k, int64_t* bytes) {
  using namespace ae;
  if (!bytes || !sizes_ok(m, n, k)) return fail(AE_EINVAL, "model_fp8_matmul_workspace: bad argument");
  *bytes = 0;
  return AE_OK;
}

extern "C" int model_fp8_matmul(const void* a, int64_t lda, const float* a_scale, const void* b, int64_t ldb, const float* b_scale,
                                int b_blocks, const float* bias, int64_t m, int64_t n, int64_t k, int dtype, void* y, int64_t ldy,
                                void* workspace, void* stream) {
  using namespace ae;
  if (!sizes_ok(m, n, k)) return fail(AE_EINVAL, "model_fp8_matmul: bad size");
  if (b_blocks != AE_FP8_ROWS && b_blocks != AE_FP8_TILES) return fail(AE_EINVAL, "model_fp8_matmul: b_blocks must be AE_FP8_ROWS or AE_FP8_TILES");
  if (dtype != AE_F32 && dtype != AE_BF16) return fail(AE_EINVAL, "model_fp8_matmul: bad dtype");
  if (m == 0 || n == 0) return AE_OK;
  if (!a || !a_scale) return fail(AE_EINVAL, "model_fp8_matmul: null argument");
  if (!codes_ok(a, lda, k) || ((uintptr_t)a_scale & 3)) return fail(AE_EINVAL, "model_fp8_matmul: rows of codes must begin on 16-byte borders and not overlap, scales must not be misaligned");
  const Product p = {a, lda, a_scale, (const uint8_t*)b, ldb, b_scale, b_blocks, bias, m, n, k, dtype, y, ldy};
  AE_TRY(check_product("model_fp8_matmul", p));
  return launch_product(p, (hipStream_t)stream);
}

extern "C" int model_fp8_linear_workspace(int64_t m, int64_t n, int64_t k, int64_t* bytes) {
  using namespace ae;
  if (!bytes || !sizes_ok(m, n, k)) return fail(AE_EINVAL, "model_fp8_linear_workspace: bad argument");
  *bytes = m <= kQuantizeOnTheWay ? 0 : m * align16(k) + align16(m * ((k + BLK - 1) / BLK) * 4);
  return AE_OK;
}

extern "C" int model_fp8_linear(const void* x, int64_t ldx, const void* w, int64_t ldw, const float* w_scale, const float* bias,
                                int64_t m, int64_t n, int64_t k, int dtype, void* y, int64_t ldy, void* workspace, void* stream) {
  using namespace ae;
  int64_t need = 0;
  if (!sizes_ok(m, n, k)) return fail(AE_EINVAL, "model_fp8_linear: bad size");
  if (dtype != AE_F32 && dtype != AE_BF16) return fail(AE_EINVAL, "model_fp8_linear: bad dtype");
  if (m == 0 || n == 0) return AE_OK;
  if (!x || (uintptr_t)x % dtype_size(dtype)) return fail(AE_EINVAL, "model_fp8_linear: x is null or not on an element's border");
  if (ldx < k || ldx >= ((int64_t)1 << 40)) return fail(AE_EINVAL, "model_fp8_linear: bad size");
  AE_TRY(model_fp8_linear_workspace(m, n, k, &need));
  if (need && (!workspace || ((uintptr_t)workspace & 15))) return fail(AE_EINVAL, "model_fp8_linear: workspace is null or not on a 16-byte border");
  uint8_t* q = (uint8_t*)workspace;
  float* sx = (float*)(q + m * align16(k));
  const Product p = {q, align16(k), sx, (const uint8_t*)w, ldw, w_scale, AE_FP8_TILES, bias, m, n, k, dtype, y, ldy};
  AE_TRY(check_product("model_fp8_linear", p));
  if (m <= kQuantizeOnTheWay) {
    Product f = p;
    f.a = x;
    f.lda = ldx;
    return dtype == AE_BF16 ? launch_few_elements<bf16_t>(f, (hipStream_t)stream) : launch_few_elements<float>(f, (hipStream_t)stream);
  }
  AE_TRY(model_fp8_quantize(x, m, k, ldx, dtype, AE_FP8_ROWS, q, align16(k), sx, nullptr, 0, nullptr, stream));
  return launch_product(p, (hipStream_t)stream);
}
