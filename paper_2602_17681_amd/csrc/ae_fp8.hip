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

// magnitude that counts for a block's scale: infinities and NaN do not
__device__ __forceinline__ float finite_abs(float v) {
  const float a = fabsf(v);
  return a <= FLT_MAX ? a : 0.0f;
}
__device__ __forceinline__ float block_scale(float amax) { return fmaxf(amax / kCodeMax, kScaleMin); }
// what is encoded: saturated (the conversion would make a NaN of anything over 448), NaN kept
__device__ __forceinline__ float code_value(float v, float inv) {
  const float y = v * inv;
  return y != y ? y : fminf(fmaxf(y, -kCodeMax), kCodeMax);
}
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
constexpr int QT_STRIDE = BLK + 16;      // bytes of a transposed row in LDS: whole 16-byte pieces, banks shifted from row to row
template <typename T, bool TILES, bool Q, bool QT>
__global__ __launch_bounds__(256) void k_fp8_quantize(const T* __restrict__ x, int rows, int cols, int64_t ldx, int tiles_c,
                                                      uint8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale,
                                                      uint8_t* __restrict__ qt, int64_t ldqt, float* __restrict__ scale_t) {
  __shared__ float red[4 * BLK];
  __shared__ __align__(16) uint8_t tr[QT ? BLK * QT_STRIDE : 16];
  const int tr_i = blockIdx.x / tiles_c, tc_i = blockIdx.x - tr_i * tiles_c;
  const int r0 = tr_i * BLK, c0 = tc_i * BLK;
  const int t = threadIdx.x, cg = t & 15, rg = t >> 4, wave = t >> 6;
  const int row = r0 + rg * 8, col = c0 + cg * 8;
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (row + i < rows) {
      load8<T>(x + (int64_t)(row + i) * ldx + col, cols - col, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    }
  }
  float inv_r[8], inv_c[8];               // what the elements of a row / column are multiplied with
  if constexpr (TILES) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaxf(m, finite_abs(v[i][j]));
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    if ((t & 63) == 0) red[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float s = block_scale(m), inv = 1.0f / s;
    if (t == 0) {
      if constexpr (Q) scale[(int64_t)tr_i * tiles_c + tc_i] = s;
      if constexpr (QT) scale_t[(int64_t)tc_i * ((rows + BLK - 1) / BLK) + tr_i] = s;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) inv_r[i] = inv_c[i] = inv;
  } else {
    if constexpr (Q) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = fmaxf(m, finite_abs(v[i][j]));
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
        const float s = block_scale(m);
        inv_r[i] = 1.0f / s;
        if (cg == 0 && row + i < rows) scale[(int64_t)tc_i * rows + row + i] = s;
      }
    }
    if constexpr (QT) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_abs(v[i][j]));
        m = fmaxf(m, __shfl_xor(m, 16, 64));
        m = fmaxf(m, __shfl_xor(m, 32, 64));
        if ((t & 63) < 16) red[wave * BLK + cg * 8 + j] = m;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = cg * 8 + j;
        const float s = block_scale(fmaxf(fmaxf(red[c], red[BLK + c]), fmaxf(red[2 * BLK + c], red[3 * BLK + c])));
        inv_c[j] = 1.0f / s;
        if (rg == 0 && c0 + c < cols) scale_t[(int64_t)tr_i * cols + c0 + c] = s;
      }
    }
  }
  if constexpr (Q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (row + i >= rows || col >= cols) continue;
      uint8_t* p = q + (int64_t)(row + i) * ldq + col;
      float u[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = code_value(v[i][j], inv_r[i]);
      const uint32_t lo = codes4(u[0], u[1], u[2], u[3]), hi = codes4(u[4], u[5], u[6], u[7]);
      if (col + 8 <= cols) {
        *reinterpret_cast<uint2*>(p) = make_uint2(lo, hi);
      } else {
        for (int j = 0; j < cols - col; ++j) p[j] = (uint8_t)((j < 4 ? lo : hi) >> (8 * (j & 3)));
      }
    }
  }
  if constexpr (QT) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = code_value(v[i][j], inv_c[j]);
      *reinterpret_cast<uint2*>(tr + (cg * 8 + j) * QT_STRIDE + rg * 8) =
          make_uint2(codes4(u[0], u[1], u[2], u[3]), codes4(u[4], u[5], u[6], u[7]));
    }
    __syncthreads();
#pragma unroll
    for (int pass = 0; pass < 4; ++pass) {
      const int c = pass * 32 + (t >> 3), ch = (t & 7) * 16;
      const int left = rows - r0 - ch;
      if (c0 + c >= cols || left <= 0) continue;
      uint8_t* p = qt + (int64_t)(c0 + c) * ldqt + r0 + ch;
      const uint8_t* s = tr + c * QT_STRIDE + ch;
      if (left >= 16) {
        *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(s);
      } else {
        for (int i = 0; i < left; ++i) p[i] = s[i];
      }
    }
  }
}

// ---- product -------------------------------------------------------------------------------------------------------
// 32 codes of a row from k0 on as a matrix operand: two aligned 16-byte loads, zeros behind the row's end k.
__device__ __forceinline__ v8i load_codes(const uint8_t* row, int k0, int k) {
  v8i r;
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
template <bool EXACT>
__device__ __forceinline__ Frag<EXACT> make_frag(v8i c) {
  Frag<EXACT> f;
  if constexpr (EXACT) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const v2bf lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * s + h], 1.0f, false);
        const v2bf hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * s + h], 1.0f, true);
        f.w[s][4 * h] = lo[0]; f.w[s][4 * h + 1] = lo[1]; f.w[s][4 * h + 2] = hi[0]; f.w[s][4 * h + 3] = hi[1];
      }
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

// Four wavefronts, 64 x 64 results: each takes 64 rows and 16 columns, fragments straight from global memory.  Lane l of
// a fragment holds row l % 16 and 32 codes from 32 (l / 16) on (both operands alike, so any order of K would do); of a
// result it holds column l % 16 and rows 4 (l / 16) .. + 3.
template <typename T, bool BROWS>
__global__ __launch_bounds__(256) void k_fp8_direct(const uint8_t* __restrict__ a, int64_t lda, const float* __restrict__ sa,
                                                    const uint8_t* __restrict__ b, int64_t ldb, const float* __restrict__ sb,
                                                    const float* __restrict__ bias, int m, int n, int k, T* __restrict__ y, int64_t ldy,
                                                    int tiles_n) {
  constexpr bool EXACT = sizeof(T) == 4;
  const int tm = blockIdx.x / tiles_n, tn = blockIdx.x - tm * tiles_n;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
  const int col = tn * 64 + (threadIdx.x >> 6) * 16 + l16;
  const int kb = (k + BLK - 1) / BLK;
  const uint8_t* bp = b + (int64_t)(col < n ? col : n - 1) * ldb;
  const uint8_t* ap[4];
  int row[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = tm * 64 + 16 * i + l16;
    ap[i] = a + (int64_t)(r < m ? r : m - 1) * lda;
    row[i] = tm * 64 + 16 * i + 4 * g;
  }
  v4f acc[4] = {};
  for (int c = 0; c < kb; ++c) {
    const Frag<EXACT> fb = make_frag<EXACT>(load_codes(bp, c * BLK + 32 * g, k));
    const float s_col = BROWS ? sb[(int64_t)c * n + (col < n ? col : n - 1)] : sb[(int64_t)((col < n ? col : n - 1) / BLK) * kb + c];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const v4f p = block_product<EXACT>(make_frag<EXACT>(load_codes(ap[i], c * BLK + 32 * g, k)), fb);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][e] = fmaf(p[e], sa[(int64_t)c * m + (row[i] + e < m ? row[i] + e : m - 1)] * s_col, acc[i][e]);
    }
  }
  if (col >= n) return;
  const float bb = bias ? bias[col] : 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (row[i] + e < m) store_out<T>(y + (int64_t)(row[i] + e) * ldy + col, acc[i][e] + bb);
}

// ---- product of many rows: tiles staged in LDS -----------------------------------------------------------------------
// A workgroup of WGM x WGN wavefronts makes a tile of BM x BN results, a wavefront 16 MI x 16 NJ of them, in steps of one
// block (128 codes) of K.  The codes of a step go from memory straight into LDS (16 bytes a lane, a row of 128 in eight
// pieces) while the step before is multiplied; two such stages.  The first matrix operand is b and the second a, so that a
// lane's results are four neighbouring columns of one row: the row's scale is one register, and with the order of b's rows
// below a lane's NJ fragments are 4 NJ columns in a row, which it stores in 16-byte pieces.
//   piece c of row r lies at piece c ^ key(r) of that row, eight keys among the 16 rows of a fragment, and lane group g reads
//   pieces g and g + 4 (any order of K will do, as long as it is b's too): 5.8 cycles a read, as for consecutive addresses;
//   pieces 2 g and 2 g + 1 take 8.0
template <int NJ> __device__ __forceinline__ int b_row(int i, int j) { return (i >> 2) * (4 * NJ) + j * 4 + (i & 3); }   // row of b in fragment j, place i
__device__ __forceinline__ int a_key(int r) { return (r >> 1) & 7; }
template <int NJ> __device__ __forceinline__ int b_key(int r) { return ((r / (4 * NJ)) & 3) << 1 | ((r >> 1) & 1); }

// 16 bytes of each lane from a buffer straight into LDS: lane l writes at lds + 16 l; offsets past the buffer's range deliver
// zeros.  In assembly, because the compiler would wait for every such load before the next read of LDS, whichever part
// of it that reads; the kernel waits itself (vmcnt) where it needs the data.  There is no register result.  (The instruction
// may read m0 one wait state after it was written, which the compiler does not see here: s_nop.)
typedef int v4i __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void load_to_lds(v4i rsrc, unsigned lds, unsigned voffset, unsigned soffset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(voffset), "s"(rsrc), "s"(soffset) : "memory", "m0");
}
// a raw buffer of `bytes` bytes, 0 to 2^31 - 1, from p on
__device__ __forceinline__ v4i buffer_of(const void* p, int64_t bytes) {
  const uint64_t a = (uint64_t)(uintptr_t)p;
  const int n = bytes <= 0 ? 0 : bytes < 0x7FFFFFFF ? (int)bytes : 0x7FFFFFFF;
  const v4i r = {__builtin_amdgcn_readfirstlane((int)(uint32_t)a), __builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xFFFF)),
                 __builtin_amdgcn_readfirstlane(n), 0x00020000};
  return r;
}

// Tiles in an order in which workgroups that run at the same time share rows of a and b: consecutive workgroups go to
// different dies (8, each with its own L2), so each die takes a contiguous run of tiles, and a run walks columns of 6 tiles:
// its 32 tiles at a time read few different rows of a and of b (16 384 x 4 096 x 4 096: 250 us; columns of 4 254, of 8 258).
constexpr int GROUP = 6;
__device__ __forceinline__ void tile_of(int b, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int total = tiles_m * tiles_n, xcd = b & 7, per = total >> 3, more = total & 7;
  const int id = xcd * per + (xcd < more ? xcd : more) + (b >> 3);
  const int group = GROUP * tiles_n, gi = id / group, first = gi * GROUP, in = id - gi * group;
  const int height = tiles_m - first < GROUP ? tiles_m - first : GROUP;
  tm = first + in % height;
  tn = in / height;
}

template <typename T, bool BROWS, int WGM, int WGN, int MI, int NJ>
__global__ __launch_bounds__(WGM * WGN * 64) void k_fp8_tile(const uint8_t* __restrict__ a, int64_t lda, const float* __restrict__ sa,
                                                             const uint8_t* __restrict__ b, int64_t ldb, const float* __restrict__ sb,
                                                             const float* __restrict__ bias, int m, int n, int k, T* __restrict__ y,
                                                             int64_t ldy, int tiles_m, int tiles_n) {
  constexpr bool EXACT = sizeof(T) == 4;
  constexpr int NTH = WGM * WGN * 64, NWV = WGM * WGN;
  constexpr int BM = WGM * MI * 16, BN = WGN * NJ * 16;
  constexpr int STAGE = (BM + BN) * BLK;                       // bytes of codes of a step
  constexpr int CB = BN >= BLK ? BN / BLK : 1;                 // column blocks of a tile
  constexpr int NS = BROWS ? BM + BN : CB * BM;                // scales of a step: rows' and columns', or rows' times the block's
  constexpr int SPT = (NS + NTH - 1) / NTH;
  constexpr int LA = BM / 8 / NWV, LB = BN / 8 / NWV, LOADS = LA + LB;      // a wavefront's loads of a step
  static_assert(BM % (16 * NWV) == 0 && BN % (16 * NWV) == 0 && NJ == 4, "whole loads, keys as the loads assume them");
  __shared__ __align__(1024) uint8_t codes[2][STAGE];
  __shared__ __align__(16) float scales[2][NS];
  const int t = threadIdx.x, lane = t & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6), wm = wave / WGN, wn = wave - wm * WGN;
  int tm, tn;
  tile_of(blockIdx.x, tiles_m, tiles_n, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int kb = (k + BLK - 1) / BLK;

  // loads: an instruction moves eight rows, lane l piece l % 8 (before the keys) of row l / 8; rows behind the end lie
  // outside the buffer's range and become zeros.  Eight rows that begin at a multiple of 8 share all of the key but what
  // l / 8 gives, and the two addends are bits of their own.
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&codes[0][0];
  const int l8 = lane >> 3;
  const int a_piece = (lane & 7) ^ a_key(l8), b_piece = (lane & 7) ^ b_key<NJ>(l8);
  v4i ra[LA], rb[LB];
#pragma unroll
  for (int i = 0; i < LA; ++i) {
    const int r = m0 + (wave * LA + i) * 8;
    ra[i] = buffer_of(a + (int64_t)r * lda, (m - r) * lda);
  }
#pragma unroll
  for (int i = 0; i < LB; ++i) {
    const int r = n0 + (wave * LB + i) * 8;
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
                lds0 + (c & 1) * STAGE + (is_a ? wave * LA + i : BM / 8 + wave * LB + i - LA) * 1024, o, c * BLK);
  };
  auto load_scales = [&](int c, float (&v)[SPT]) {
#pragma unroll
    for (int i = 0; i < SPT; ++i) {
      const int at = t + i * NTH;
      if (NS % NTH != 0 && at >= NS) break;
      if constexpr (BROWS) {
        const bool is_a = at < BM;
        const int r = is_a ? m0 + at : n0 + at - BM, end = is_a ? m : n;
        v[i] = (is_a ? sa : sb)[(int64_t)c * end + (r < end ? r : end - 1)];
      } else {
        const int cb = at / BM, r = m0 + at - cb * BM;
        int blk = n0 / BLK + cb;
        if (blk > (n - 1) / BLK) blk = (n - 1) / BLK;
        v[i] = sa[(int64_t)c * m + (r < m ? r : m - 1)] * sb[(int64_t)blk * kb + c];
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
  // the piece that holds the end of the rows, in the last step: zeros behind it
  auto cut_tail = [&](int buf) {
    const int cut = (k % BLK) >> 4, keep = k & 15;
    for (int r = t; r < BM + BN; r += NTH) {
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
  Frag<EXACT> fb[NJ];
  v4f cs[NJ];
  v8i ahead[AHEAD];
  float s_ahead[AHEAD];
  auto begin_step = [&](int buf) {
    fb[0] = make_frag<EXACT>(raw_b(buf, 0));
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      ahead[i] = raw_a(buf, i);
      s_ahead[i] = row_scale(buf, i);
    }
#pragma unroll
    for (int j = 1; j < NJ; ++j) fb[j] = make_frag<EXACT>(raw_b(buf, j));
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
  // front of the reads of LDS; later ones would not be there in time).  When the last rows' products are issued, everything that the step reads from LDS has been
  // read: the wait for the next step's codes, the barrier and the first reads of that step run beside them.
  enum { LAST = 0, MORE = 1, MORE_TAIL = 2 };
  auto step = [&](int c, auto what) {
    constexpr int W = decltype(what)::value;
    const int buf = c & 1;
    v4f p[2][NJ];
    float s_at[2], sv[SPT];
    if constexpr (W != LAST) load_scales(c + 1, sv);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const Frag<EXACT> fa = make_frag<EXACT>(ahead[i % AHEAD]);
      s_at[i & 1] = s_ahead[i % AHEAD];
      if (i + AHEAD < MI) {
        ahead[i % AHEAD] = raw_a(buf, i + AHEAD);
        s_ahead[i % AHEAD] = row_scale(buf, i + AHEAD);
      }
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        p[i & 1][j] = block_product<EXACT>(fb[j], fa);
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
        if ((k & 15) != 0) cut_tail(buf ^ 1);
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
    load_scales(0, sv);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load_part(0, i, kb == 1);
    store_scales(0, sv);
    arrive();
    if (kb == 1 && (k & 15) != 0) cut_tail(0);
    begin_step(0);
  }
  int c = 0;
  for (; c + 2 < kb; ++c) step(c, std::integral_constant<int, MORE>());
  if (c + 1 < kb) {
    step(c, std::integral_constant<int, MORE_TAIL>());
    ++c;
  }
  step(c, std::integral_constant<int, LAST>());
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

bool sizes_ok(int64_t m, int64_t n, int64_t k) { return m >= 0 && n >= 0 && k >= 1 && m < 0x7FFFFFFF && n < 0x7FFFFFFF && k < 0x7FFFFFFF; }
bool codes_ok(const void* p, int64_t ld, int64_t cols) { return ((uintptr_t)p & 15) == 0 && ld >= cols && ld % 16 == 0 && ld < ((int64_t)1 << 40); }

struct Product {
  const uint8_t* a; int64_t lda; const float* sa;
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

template <typename T, bool BROWS, int WGM, int WGN, int MI, int NJ>
int launch_tile(const Product& p, hipStream_t s) {
  constexpr int BM = WGM * MI * 16, BN = WGN * NJ * 16;
  const int64_t tm = (p.m + BM - 1) / BM, tn = (p.n + BN - 1) / BN;
  if (tm * tn > 0x7FFFFFFF) return fail(AE_EINVAL, "model_fp8_matmul: result too large");
  hipLaunchKernelGGL((k_fp8_tile<T, BROWS, WGM, WGN, MI, NJ>), dim3((unsigned)(tm * tn)), dim3(WGM * WGN * 64), 0, s, p.a, p.lda, p.sa, p.b, p.ldb,
                     p.sb, p.bias, (int)p.m, (int)p.n, (int)p.k, (T*)p.y, p.ldy, (int)tm, (int)tn);
  return launch_status("fp8_matmul");
}
template <typename T, bool BROWS>
int launch_tiles(const Product& p, hipStream_t s) {
  const int64_t big = ((p.m + 255) / 256) * ((p.n + 255) / 256);
  if constexpr (sizeof(T) == 4 || BROWS) {      // bfloat16 operands, or column scales in registers: 64 rows a wavefront are what fits
    if (((p.m + 255) / 256) * ((p.n + 127) / 128) >= 192) return launch_tile<T, BROWS, 4, 2, 4, 4>(p, s);
  } else {
    if (big >= 192) return launch_tile<T, BROWS, 2, 4, 8, 4>(p, s);
  }
  return launch_tile<T, BROWS, 2, 2, 4, 4>(p, s);
}

int launch_product(const Product& p, hipStream_t s) {
  // offsets inside a tile are 31 bits
  if (p.m > 64 && p.lda < (1 << 23) && p.ldb < (1 << 23)) {
    if (p.dtype == AE_BF16) return p.b_blocks == AE_FP8_ROWS ? launch_tiles<bf16_t, true>(p, s) : launch_tiles<bf16_t, false>(p, s);
    return p.b_blocks == AE_FP8_ROWS ? launch_tiles<float, true>(p, s) : launch_tiles<float, false>(p, s);
  }
  const int64_t tn = (p.n + 63) / 64, tm = (p.m + 63) / 64;
  if (tn * tm > 0x7FFFFFFF) return fail(AE_EINVAL, "model_fp8_matmul: result too large");
#define DIRECT(T, R)                                                                                                            \
  hipLaunchKernelGGL((k_fp8_direct<T, R>), dim3((unsigned)(tn * tm)), dim3(256), 0, s, p.a, p.lda, p.sa, p.b, p.ldb, p.sb, p.bias, \
                     (int)p.m, (int)p.n, (int)p.k, (T*)p.y, p.ldy, (int)tn)
  if (p.dtype == AE_BF16) { if (p.b_blocks == AE_FP8_ROWS) DIRECT(bf16_t, true); else DIRECT(bf16_t, false); }
  else { if (p.b_blocks == AE_FP8_ROWS) DIRECT(float, true); else DIRECT(float, false); }
#undef DIRECT
  return launch_status("fp8_matmul");
}

template <typename T>
int launch_quantize(const void* x, int64_t rows, int64_t cols, int64_t ldx, int blocks, void* q, int64_t ldq, float* scale, void* qt,
                    int64_t ldqt, float* scale_t, hipStream_t s) {
  const int64_t tr = (rows + BLK - 1) / BLK, tc = (cols + BLK - 1) / BLK;
  if (tr * tc > 0x7FFFFFFF) return fail(AE_EINVAL, "model_fp8_quantize: matrix too large");
#define QUANT(TI, A, B)                                                                                                         \
  hipLaunchKernelGGL((k_fp8_quantize<T, TI, A, B>), dim3((unsigned)(tr * tc)), dim3(256), 0, s, (const T*)x, (int)rows, (int)cols, ldx, \
                     (int)tc, (uint8_t*)q, ldq, scale, (uint8_t*)qt, ldqt, scale_t)
  if (blocks == AE_FP8_TILES) {
    if (q && qt) QUANT(true, true, true);
    else if (q) QUANT(true, true, false);
    else QUANT(true, false, true);
  } else {
    if (q && qt) QUANT(false, true, true);
    else if (q) QUANT(false, true, false);
    else QUANT(false, false, true);
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
  if (rows < 0 || cols < 0 || rows >= 0x7FFFFFFF || cols >= 0x7FFFFFFF || ldx < cols || ldx >= ((int64_t)1 << 40)) return fail(AE_EINVAL, "model_fp8_quantize: bad size");
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
  const Product p = {(const uint8_t*)a, lda, a_scale, (const uint8_t*)b, ldb, b_scale, b_blocks, bias, m, n, k, dtype, y, ldy};
  AE_TRY(check_product("model_fp8_matmul", p));
  return launch_product(p, (hipStream_t)stream);
}

extern "C" int model_fp8_linear_workspace(int64_t m, int64_t n, int64_t k, int64_t* bytes) {
  using namespace ae;
  if (!bytes || !sizes_ok(m, n, k)) return fail(AE_EINVAL, "model_fp8_linear_workspace: bad argument");
  *bytes = m * align16(k) + align16(m * ((k + BLK - 1) / BLK) * 4);
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
  AE_TRY(model_fp8_quantize(x, m, k, ldx, dtype, AE_FP8_ROWS, q, align16(k), sx, nullptr, 0, nullptr, stream));
  return launch_product(p, (hipStream_t)stream);
}
