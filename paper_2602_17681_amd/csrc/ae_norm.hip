// ae_norm.hip — root-mean-square norm of rows with the residual's addition, and its adjoint.
//   h = x + residual,   y = h r w,   r = 1 / sqrt(mean h^2 + eps);   y in dtype and / or as E4M3 codes in blocks of 128
//   g = dy w,   u = h r:   dh = d_h + r (g - u mean(g u)),   dw = sum over rows of dy u
// Both are bound by memory: a row is read once and stays in registers between its sum and its results.  16 384 x 4 096 in bfloat16 with
// residual into codes 80 us (472 MB, 5.9 TB/s); the adjoint of 4 096 x 4 096 with the residual path's gradient 29.4 us (134 MB,
// 4.6 TB/s, of which the sum of the weight's gradient over workgroups 4 us).  Sums are binary32.  Where a row's sum of squares leaves binary32's range
// (|h| from 2^54 on), that of h 2^-76 is taken instead: what becomes subnormal there has no part in it.  The row itself stays as it is, since its
// small elements would lose bits: u = (h r) 2^-76 with the r of that sum, and h r is at most 2^76 sqrt(d).
#include <hip/hip_runtime.h>
#include <float.h>

#include "ae_device.h"
#include "ae_fp8.h"
#include "ae_rows.h"
#include "ae_internal.h"

namespace ae {
namespace {

constexpr float kDown = 1.3234889800848443e-23f;   // 2^-76

// eight elements as numbers, zeros behind the row's end
template <typename T>
__device__ __forceinline__ void numbers(const T* p, int left, float (&v)[8]) {
  Eight<T> e;
  fetch(p, left, e);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = value(e, i);
}

// sum over the lanes that share a row: 8, 16, 32 or 64 of a wavefront, or several wavefronts; sm is not written again before the
// workgroup's next barrier but one
template <int LANES>
__device__ __forceinline__ float team_sum(float v, float* sm) {
  if constexpr (LANES == 8) {
    v += __shfl_xor(v, 4, 64);
    v += __shfl_xor(v, 2, 64);
    return v + __shfl_xor(v, 1, 64);
  }
  v = sum16(v);
  if constexpr (LANES == 32) return v + __shfl_xor(v, 16, 64);
  if constexpr (LANES >= 64) v = sum_rows(v);
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sum_of<LANES / 64>(sm);
  }
  return v;
}

struct NormArgs {
  const void* x;
  int64_t ldx;
  const void* residual;
  int64_t ldr;
  const float* weight;
  int64_t rows;
  int d;
  float eps;
  void* h;
  int64_t ldh;
  void* y;
  int64_t ldy;
  uint8_t* q;
  int64_t ldq;
  float* scale;
  bool stream;
};

// the largest value of the 16 lanes that hold a block of 128, or of 8 that hold a row of 64
template <int LANES>
__device__ __forceinline__ float block_max(float v) {
  if constexpr (LANES != 8) return max16(v);
  v = fmaxf(v, __shfl_xor(v, 4, 64));
  v = fmaxf(v, __shfl_xor(v, 2, 64));
  return fmaxf(v, __shfl_xor(v, 1, 64));
}
// eight results of a row from column col on (behind the row's end: none); the lanes of a block of 128 come here together
template <typename T, int LANES>
__device__ __forceinline__ void emit(const NormArgs& p, int64_t row, int col, const float (&y)[8]) {
  const int left = p.d - col;
  if (p.y && left > 0) put((T*)p.y + row * p.ldy + col, left, y);
  if (!p.q) return;
  float m = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(y[j]));
  m = block_max<LANES>(m);
  const bool inf = __any(m > FLT_MAX);
  if (inf) {
    m = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, finite_abs(y[j]));
    m = block_max<LANES>(m);
  }
  const float s = block_scale(m), inv = 1.0f / s;
  float u[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) u[j] = inf ? code_value<true>(y[j], inv) : code_value<false>(y[j], inv);
  if (left <= 0) return;
  if (threadIdx.x % (LANES == 8 ? 8 : 16) == 0) p.scale[(int64_t)(col / BLK) * p.rows + row] = s;
  uint8_t* at = p.q + row * p.ldq + col;
  const uint32_t lo = codes4(u[0], u[1], u[2], u[3]), hi = codes4(u[4], u[5], u[6], u[7]);
  if (left >= 8) {
    *reinterpret_cast<uint2*>(at) = make_uint2(lo, hi);
  } else {
    for (int j = 0; j < left; ++j) at[j] = (uint8_t)((j < 4 ? lo : hi) >> (8 * (j & 3)));
  }
}

// 1 / sqrt(mean + eps) of a row; down: of the row times 2^-76, whose mean was so large that eps plays no part
__device__ __forceinline__ float rms_inverse(float sum, int d, float eps, bool down) { return 1.0f / sqrtf(sum / (float)d + (down ? 0.0f : eps)); }

// LANES lanes hold a row in NV pieces of eight elements each; a workgroup has 256 / LANES rows at a time, or one, and many
// workgroups come after each other: their stores go beside the others' loads (16 384 x 4 096 80 us; 2 048 workgroups that stay 94,
// with the next row asked for early 96).
template <typename T, int LANES, int NV, bool STREAM>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void k_rms_norm(NormArgs p) {
  constexpr int TEAMS = LANES < 256 ? 256 / LANES : 1, W = LANES / 64 ? LANES / 64 : 1;
  constexpr bool SHORT = LANES == 8;
  __shared__ float sm[3][W];
  const int t = threadIdx.x % LANES, team = threadIdx.x / LANES, step = (int)gridDim.x * TEAMS;
  const T* x = (const T*)p.x;
  const T* res = (const T*)p.residual;
  constexpr bool LATE = NV > 2;                  // the weights behind the sum: two workgroups to a compute unit
  Eight<float> w[LATE ? 1 : NV];
  if (!LATE && p.weight) {
#pragma unroll
    for (int v = 0; v < NV; ++v) fetch_row<false, SHORT>(p.weight, (v * LANES + t) * 8, p.d, w[LATE ? 0 : v]);
#pragma unroll
    for (int v = 0; v < NV; ++v) settle<SHORT>((v * LANES + t) * 8, p.d, w[LATE ? 0 : v]);
  }
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * TEAMS; row0 < p.rows; row0 += step, turn ^= 1) {
    const int64_t row = row0 + team;
    const bool live = row < p.rows;                // the rows of a wavefront go together
    Eight<T> xe[NV], re[NV];
    const int64_t at = live ? row : p.rows - 1;
#pragma unroll
    for (int v = 0; v < NV; ++v) fetch_row<STREAM, SHORT>(x + at * p.ldx, (v * LANES + t) * 8, p.d, xe[v]);
    if (res) {
#pragma unroll
      for (int v = 0; v < NV; ++v) fetch_row<STREAM, SHORT>(res + at * p.ldr, (v * LANES + t) * 8, p.d, re[v]);
    }
    float h[NV][8], sum = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * LANES + t) * 8;
      settle<SHORT>(col, p.d, xe[v]);
      if (res) settle<SHORT>(col, p.d, re[v]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[v][j] = value(xe[v], j);
        if (res) h[v][j] += value(re[v], j);
        sum = fmaf(h[v][j], h[v][j], sum);
      }
    }
    if (p.h && live) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int col = (v * LANES + t) * 8;
        if (col < p.d) put<STREAM>((T*)p.h + row * p.ldh + col, p.d - col, h[v]);
      }
    }
    sum = team_sum<LANES>(sum, sm[turn]);
    const bool down = !(sum <= FLT_MAX);           // the same in all threads of the row
    const bool any = LANES <= 64 ? __any(down) : down;
    const float by = down ? kDown : 1.0f;          // of several rows in a wavefront the others are multiplied by one
    if (any) {
      sum = 0.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fmaf(h[v][j] * by, h[v][j] * by, sum);
      if constexpr (LANES > 64) __syncthreads();
      sum = team_sum<LANES>(sum, sm[2]);
      if constexpr (LANES > 64) __syncthreads();
    }
    const float r = rms_inverse(sum, p.d, p.eps, down);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = h[v][j] * r;
      if (any) {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] *= by;
      }
      if (p.weight) {
        if (LATE) {
          fetch_row<false, SHORT>(p.weight, (v * LANES + t) * 8, p.d, w[0]);
          settle<SHORT>((v * LANES + t) * 8, p.d, w[0]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] *= value(w[LATE ? 0 : v], j);
      }
      emit<T, LANES>(p, row, live ? (v * LANES + t) * 8 : p.d, y);
    }
  }
}

// Rows that registers do not hold are read twice; each element's results are written by the thread that reads it, behind
// its second read, so that h may take the place of x or of the residual here too.  1 676 x 20 000 72 us, 670 x 50 021 88; with
// more pieces of a thread in flight fewer wavefronts fit: 512 threads of four 80 and 93, of two 70 and 95, 1 024 of three 75 and 96, of two 82 and 91.
constexpr int WIDE = 1024;
template <typename T>
__global__ __launch_bounds__(WIDE) void k_rms_norm_wide(NormArgs p) {
  __shared__ float sm[2][WIDE / 64];
  const T* x = (const T*)p.x;
  const T* res = (const T*)p.residual;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    auto load = [&](int col, float by, float (&h)[8]) {
      float r8[8];
      numbers(x + row * p.ldx + col, p.d - col, h);
      if (res) numbers(res + row * p.ldr + col, p.d - col, r8);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[j] = (res ? h[j] + r8[j] : h[j]) * by;
    };
    auto squares = [&](float by) {
      float sum = 0.0f, h[8];
      for (int col = threadIdx.x * 8; col < p.d; col += WIDE * 8) {
        load(col, by, h);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fmaf(h[j], h[j], sum);
      }
      return sum;
    };
    float sum = team_sum<WIDE>(squares(1.0f), sm[0]);
    const bool down = !(sum <= FLT_MAX);
    if (down) sum = team_sum<WIDE>(squares(kDown), sm[1]);
    const float r = rms_inverse(sum, p.d, p.eps, down);
    for (int c0 = 0; c0 < p.d; c0 += WIDE * 8) {           // all threads: a block's lanes meet in emit
      const int col = c0 + threadIdx.x * 8;
      float h[8], w[8], y[8];
      load(col, 1.0f, h);
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = 1.0f;
      if (p.weight) numbers(p.weight + col, p.d - col, w);
      if (p.h && col < p.d) put((T*)p.h + row * p.ldh + col, p.d - col, h);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = (down ? h[j] * r * kDown : h[j] * r) * w[j];
      emit<T, WIDE>(p, row, col, y);
    }
    __syncthreads();
  }
}

template <typename T, int LANES, int NV>
int launch_norm_row(const NormArgs& p, hipStream_t s) {
  constexpr int TEAMS = LANES < 256 ? 256 / LANES : 1;
  const int64_t want = (p.rows + TEAMS - 1) / TEAMS, most = 1 << 20;
  hipLaunchKernelGGL((p.stream ? k_rms_norm<T, LANES, NV, true> : k_rms_norm<T, LANES, NV, false>), dim3((unsigned)(want < most ? want : most)), dim3(LANES < 256 ? 256 : LANES), 0, s, p);
  return launch_status("rms_norm");
}
// Lanes by the row's length.  524 288 x 64 in bfloat16 8 lanes 44 us, 16 lanes 86; 262 144 x 128 16 lanes 43, 64 lanes 116; 131 072 x 256 32 lanes 43, 64 lanes 60;
// 16 384 x 4 096 256 lanes of two pieces 81, 512 of one 83, 64 of eight 155; 2 730 x 12 288 512 lanes of three
// pieces 50, 1 024 of two 58, of which only one workgroup fits into a compute unit; 1 676 x 20 000 read twice 72, 1 024 lanes of four pieces (which spill) 147.
template <typename T>
int launch_norm(const NormArgs& p, hipStream_t s) {
  if (p.d <= 64) return launch_norm_row<T, 8, 1>(p, s);
  if (p.d <= 128) return launch_norm_row<T, 16, 1>(p, s);
  if (p.d <= 256) return launch_norm_row<T, 32, 1>(p, s);
  if (p.d <= 512) return launch_norm_row<T, 64, 1>(p, s);
  if (p.d <= 1024) return launch_norm_row<T, 64, 2>(p, s);
  if (p.d <= 2048) return launch_norm_row<T, 256, 1>(p, s);
  if (p.d <= 4096) return launch_norm_row<T, 256, 2>(p, s);
  if (p.d <= 8192) return launch_norm_row<T, 512, 2>(p, s);
  if (p.d <= 12288) return launch_norm_row<T, 512, 3>(p, s);
  if (p.d <= 16384) return launch_norm_row<T, 512, 4>(p, s);
  const int64_t most = 512;
  hipLaunchKernelGGL((k_rms_norm_wide<T>), dim3((unsigned)(p.rows < most ? p.rows : most)), dim3(WIDE), 0, s, p);
  return launch_status("rms_norm");
}

// ---- adjoint -------------------------------------------------------------------------------------------------------
struct NormGradArgs {
  const void* dy;
  int64_t ldy;
  const void* h;
  int64_t ldh;
  const float* weight;
  const void* d_h;
  int64_t ldg;
  int64_t rows;
  int d;
  float eps;
  void* dx;
  int64_t lddx;
  float* part;                            // [workgroups][d]: each one's sum of dy u over its rows; null: not wanted
  struct RowStat* stat;                   // [rows], rows that registers do not hold
  bool stream;
};

// What a row's gradients take:  u = h r down,   dh = d_h + (dy part w - u mean) t.  In an ordinary row down and part are 1, t is r and mean that of g u.
// Three kinds of rows have their sums taken once more, that of h^2 with h times by, that of g h with g times scale and h times lift:
//   down  the sum of h^2 leaves binary32: by = lift = down = 2^-76, and r is that of h 2^-76
//   far   r times the sum of g h leaves 2^90, or the sum itself binary32 (in all other rows the part along h is less than the rounding of binary32's largest number):
//         scale = 2^-90
//   near  r is large and the sum of g h so small that products in it are subnormal: lift = 2^120 (h is less than 1 there)
// In these rows `part` has (most of) r in it, so that what is subnormal on the way is so in the result, and what leaves the range, too.
struct RowStat {
  float r, down, part, mean, t;
};
constexpr float kFar = 1.2379400392853803e27f;        // 2^90
constexpr float kNear = 7.8886090522101181e-31f;      // 2^-100
constexpr float kLift = 1.3292279957849159e36f;       // 2^120
struct Again {
  bool down, far, near;
  __device__ __forceinline__ Again(float hh, float gh, float r) {
    down = !(hh <= FLT_MAX);
    far = !(fabsf(r * gh) <= kFar && fabsf(gh) <= FLT_MAX);
    // products are off by 2^-150, u mean too, and a gradient by r^2 u or r times that: with u up to 2^5 below 2^-126 up to r = 2^10.  Where the sum of h^2 is 0, h is
    // below 2^-75, and u below r 2^-75: up to r = 2^24.  So rows of zeros (padding) are ordinary for every eps from 2^-48 on
    near = r > (hh > 0.0f ? 1024.0f : 16777216.0f) && fabsf(gh) < kNear;
  }
  __device__ __forceinline__ bool any() const { return down || far || near; }
  __device__ __forceinline__ float by() const { return down ? kDown : 1.0f; }
  __device__ __forceinline__ float scale() const { return far ? 1.0f / kFar : 1.0f; }
  __device__ __forceinline__ float lift() const { return near ? kLift : by(); }
};
__device__ __forceinline__ RowStat row_stat(float gh, float r, int d) { return {r, 1.0f, 1.0f, r * gh / (float)d, r}; }
// from the second sums; first: that of an ordinary row.  Large products that cancel leave the range in 2^120 of them: then there is nothing subnormal to lose
__device__ __forceinline__ RowStat row_stat(const Again& a, float hh, float gh, int d, float eps, const RowStat& first) {
  if (a.near) return fabsf(gh) <= FLT_MAX ? RowStat{first.r, 1.0f, first.r, gh / (float)d * first.r * (first.r * (1.0f / kLift)), 1.0f} : first;
  const float r = rms_inverse(hh, d, eps, a.down), c = gh / (float)d * r;            // mean(g u) times scale
  // r = part t but for down: 2^-64 2^-12 there, and where h is as it is min(r, 1) 2^-12 and max(r, 1) 2^12
  const float part = a.down ? r * 5.4210108624275222e-20f : fminf(r, 1.0f) * 0.000244140625f, t = a.down ? 0.000244140625f : fmaxf(r, 1.0f) * 4096.0f;
  return {r, a.by(), part, a.far ? c * (part * kFar) : c * part, t};
}

template <typename T, int LANES, int NV, bool STREAM>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void k_rms_norm_grad(NormGradArgs p) {
  constexpr int TEAMS = LANES < 256 ? 256 / LANES : 1, W = LANES / 64 ? LANES / 64 : 1;
  constexpr bool SHORT = LANES == 8;
  __shared__ float sm[3][2][W];
  __shared__ float join[TEAMS > 1 ? TEAMS - 1 : 1][TEAMS > 1 ? NV * LANES * 8 : 1];
  const int t = threadIdx.x % LANES, team = threadIdx.x / LANES, step = (int)gridDim.x * TEAMS;
  float w[NV][8], acc[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int col = (v * LANES + t) * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) { w[v][j] = 1.0f; acc[v][j] = 0.0f; }
    if (p.weight) numbers(p.weight + col, p.d - col, w[v]);
  }
  Eight<T> he[NV], ge[NV], re[NV];
  auto ask = [&](int64_t row) {
    const int64_t at = row < p.rows ? row : p.rows - 1;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      fetch_row<STREAM, SHORT>((const T*)p.h + at * p.ldh, (v * LANES + t) * 8, p.d, he[v]);
      fetch_row<STREAM, SHORT>((const T*)p.dy + at * p.ldy, (v * LANES + t) * 8, p.d, ge[v]);
    }
    if (p.d_h) {
#pragma unroll
      for (int v = 0; v < NV; ++v) fetch_row<STREAM, SHORT>((const T*)p.d_h + at * p.ldg, (v * LANES + t) * 8, p.d, re[v]);
    }
  };
  int64_t row0 = (int64_t)blockIdx.x * TEAMS;
  if (row0 < p.rows) ask(row0 + team);
  int turn = 0;
  for (; row0 < p.rows; row0 += step, turn ^= 1) {
    const int64_t row = row0 + team;
    const bool live = row < p.rows;                // the rows of a wavefront go together
    float h[NV][8], dy[NV][8], add[NV][8], hh = 0.0f, gh = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * LANES + t) * 8;
      settle<SHORT>(col, p.d, he[v]);
      settle<SHORT>(col, p.d, ge[v]);
      if (p.d_h) settle<SHORT>(col, p.d, re[v]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[v][j] = value(he[v], j);
        dy[v][j] = live ? value(ge[v], j) : 0.0f;
        add[v][j] = p.d_h ? value(re[v], j) : 0.0f;
        hh = fmaf(h[v][j], h[v][j], hh);
        gh = fmaf(dy[v][j] * w[v][j], h[v][j], gh);
      }
    }
    if (row0 + step < p.rows) ask(row + step);
    // both sums at one barrier
    auto sums = [&](float (&s2)[2][W]) {
      if constexpr (LANES <= 64) {
        hh = team_sum<LANES>(hh, nullptr);
        gh = team_sum<LANES>(gh, nullptr);
      } else {
        hh = sum_rows(sum16(hh));
        gh = sum_rows(sum16(gh));
        if ((threadIdx.x & 63) == 0) { s2[0][threadIdx.x >> 6] = hh; s2[1][threadIdx.x >> 6] = gh; }
        __syncthreads();
        hh = sum_of<W>(s2[0]);
        gh = sum_of<W>(s2[1]);
      }
    };
    sums(sm[turn]);
    const float r1 = rms_inverse(hh, p.d, p.eps, false);
    RowStat st = row_stat(gh, r1, p.d);
    const Again again(hh, gh, r1);
    if (LANES <= 64 ? __any(again.any()) : again.any()) {      // of several rows in a wavefront the others keep what they have
      const float by = again.by(), scale = again.scale(), lift = again.lift();
      hh = gh = 0.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          hh = fmaf(h[v][j] * by, h[v][j] * by, hh);
          gh = fmaf(dy[v][j] * scale * w[v][j], h[v][j] * lift, gh);
        }
      if constexpr (LANES > 64) __syncthreads();
      sums(sm[2]);
      if constexpr (LANES > 64) __syncthreads();
      if (again.any()) st = row_stat(again, hh, gh, p.d, p.eps, st);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * LANES + t) * 8;
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float u = h[v][j] * st.r * st.down;
        if (live) acc[v][j] = fmaf(dy[v][j], u, acc[v][j]);
        o[j] = (dy[v][j] * st.part * w[v][j] - u * st.mean) * st.t + add[v][j];
      }
      if (p.dx && live && col < p.d) put((T*)p.dx + row * p.lddx + col, p.d - col, o);
    }
  }
  if (!p.part) return;
  // the rows that a workgroup has at a time: added in their order
  if constexpr (TEAMS > 1) {
    if (team) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) join[team - 1][(v * 8 + j) * LANES + t] = acc[v][j];
    }
    __syncthreads();
    if (team) return;
#pragma unroll
    for (int k = 0; k < TEAMS - 1; ++k)
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[v][j] += join[k][(v * 8 + j) * LANES + t];
  }
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int col = (v * LANES + t) * 8;
    if (col < p.d) put(p.part + (int64_t)blockIdx.x * p.d + col, p.d - col, acc[v]);
  }
}

// Rows that registers do not hold: the RowStat of every row first, then the gradients by columns.
template <typename T>
__global__ __launch_bounds__(WIDE, 8) void k_rms_norm_stat(NormGradArgs p) {       // 64 registers: two workgroups to a compute unit
  __shared__ float sm[4][WIDE / 64];
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    float hh, gh;
    auto sums = [&](float by, float scale, float lift) {
      hh = gh = 0.0f;
      for (int col = threadIdx.x * 8; col < p.d; col += WIDE * 8) {
        float h[8], g[8], w[8];
        numbers((const T*)p.h + row * p.ldh + col, p.d - col, h);
        numbers((const T*)p.dy + row * p.ldy + col, p.d - col, g);
        if (p.weight) numbers(p.weight + col, p.d - col, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          hh = fmaf(h[j] * by, h[j] * by, hh);
          gh = fmaf(p.weight ? g[j] * scale * w[j] : g[j] * scale, h[j] * lift, gh);
        }
      }
    };
    sums(1.0f, 1.0f, 1.0f);
    hh = team_sum<WIDE>(hh, sm[0]);
    gh = team_sum<WIDE>(gh, sm[1]);
    const float r = rms_inverse(hh, p.d, p.eps, false);
    RowStat st = row_stat(gh, r, p.d);
    const Again again(hh, gh, r);
    if (again.any()) {
      sums(again.by(), again.scale(), again.lift());
      hh = team_sum<WIDE>(hh, sm[2]);
      gh = team_sum<WIDE>(gh, sm[3]);
      st = row_stat(again, hh, gh, p.d, p.eps, st);
    }
    if (threadIdx.x == 0) p.stat[row] = st;
    __syncthreads();
  }
}
// blockIdx.x: 2 048 columns, blockIdx.y: every gridDim.y-th row
template <typename T>
__global__ __launch_bounds__(256) void k_rms_norm_grad_columns(NormGradArgs p) {
  const int col = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 8, left = p.d - col;
  if (left <= 0) return;
  float w[8], acc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) { w[j] = 1.0f; acc[j] = 0.0f; }
  if (p.weight) numbers(p.weight + col, left, w);
  for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
    const RowStat st = p.stat[row];
    float h[8], dy[8], add[8], o[8];
    numbers((const T*)p.h + row * p.ldh + col, left, h);
    numbers((const T*)p.dy + row * p.ldy + col, left, dy);
    if (p.d_h) numbers((const T*)p.d_h + row * p.ldg + col, left, add);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float u = h[j] * st.r * st.down;
      acc[j] = fmaf(dy[j], u, acc[j]);
      o[j] = (dy[j] * st.part * w[j] - u * st.mean) * st.t + (p.d_h ? add[j] : 0.0f);
    }
    if (p.dx) put((T*)p.dx + row * p.lddx + col, left, o);
  }
  if (p.part) put(p.part + (int64_t)blockIdx.y * p.d + col, left, acc);
}

// dw[j] = sum of n parts in a fixed order: 64 groups of 16 lanes take every 64th part of 16 columns
__global__ __launch_bounds__(1024) void k_sum_parts(const float* __restrict__ part, int64_t n, int d, float* __restrict__ out) {
  __shared__ float sm[64][17];
  const int lane = threadIdx.x & 15, g = threadIdx.x >> 4, col = (int)blockIdx.x * 16 + lane;
  float acc = 0.0f;
  if (col < d) {
    constexpr int U = 8;
    for (int64_t i0 = g; i0 < n; i0 += 64 * U) {
      float v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = i0 + 64 * u < n ? part[(i0 + 64 * u) * d + col] : 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u) acc += v[u];
    }
  }
  sm[g][lane] = acc;
  __syncthreads();
  if (threadIdx.x >= 256) return;
  const int c = threadIdx.x >> 4, k = threadIdx.x & 15;        // 16 lanes to a column
  acc = sum16(sm[4 * k][c] + sm[4 * k + 1][c] + (sm[4 * k + 2][c] + sm[4 * k + 3][c]));
  if (k == 0 && (int)blockIdx.x * 16 + c < d) out[blockIdx.x * 16 + c] = acc;
}

// columns of a row that registers hold beside its gradient, the next row and the sums of the weight's (four binary32 pieces spill: 1 024 x
// 16 384 60 us, in two passes 44)
int64_t in_registers(int dtype) { return dtype == AE_BF16 ? 16384 : 12288; }
// workgroups of a launch, each with a part of the weight's gradient: as many as the registers of 256 compute units hold.  16.8 M elements in
// bfloat16, us with 256 / 512 / 1 024: rows of 512 50 / 32 / 33, of 2 048 55 / 36 / 35, of 4 096 33 / 32 / 39, of 8 192 33 / 39 / 50.  Rows of
// 12 288 and 16 384 in 512 lanes 35 and 36, in two passes 50 and 44, in 1 024 lanes without the next row 110 and 103.
int64_t grad_groups(int64_t rows, int64_t d, int dtype) {
  if (d > in_registers(dtype)) return rows < 64 ? rows : 64;
  const int64_t teams = d <= 64 ? 32 : d <= 128 ? 16 : d <= 256 ? 8 : d <= 1024 ? 4 : 1;
  const int64_t want = (rows + teams - 1) / teams, most = d <= 512 || (d > 1024 && d <= 2048) ? 1024 : d <= 4096 ? 512 : 256;
  return want < most ? want : most;
}
int64_t align16(int64_t v) { return (v + 15) / 16 * 16; }

template <typename T, int LANES, int NV>
int launch_grad_row(const NormGradArgs& p, int64_t groups, hipStream_t s) {
  hipLaunchKernelGGL((p.stream ? k_rms_norm_grad<T, LANES, NV, true> : k_rms_norm_grad<T, LANES, NV, false>), dim3((unsigned)groups), dim3(LANES < 256 ? 256 : LANES), 0, s, p);
  return launch_status("rms_norm_backward");
}
template <typename T>
int launch_grad(const NormGradArgs& p, int64_t groups, hipStream_t s) {
  if (p.d <= 64) return launch_grad_row<T, 8, 1>(p, groups, s);
  if (p.d <= 128) return launch_grad_row<T, 16, 1>(p, groups, s);
  if (p.d <= 256) return launch_grad_row<T, 32, 1>(p, groups, s);
  if (p.d <= 512) return launch_grad_row<T, 64, 1>(p, groups, s);
  if (p.d <= 1024) return launch_grad_row<T, 64, 2>(p, groups, s);
  if (p.d <= 2048) return launch_grad_row<T, 256, 1>(p, groups, s);
  if (p.d <= 4096) return launch_grad_row<T, 256, 2>(p, groups, s);
  if (p.d <= 8192) return launch_grad_row<T, 512, 2>(p, groups, s);
  if (p.d <= 12288) return launch_grad_row<T, 512, 3>(p, groups, s);
  if constexpr (sizeof(T) == 2)
    if (p.d <= 16384) return launch_grad_row<T, 512, 4>(p, groups, s);
  hipLaunchKernelGGL((k_rms_norm_stat<T>), dim3((unsigned)(p.rows < 512 ? p.rows : 512)), dim3(WIDE), 0, s, p);
  hipLaunchKernelGGL((k_rms_norm_grad_columns<T>), dim3((unsigned)((p.d + 2047) / 2048), (unsigned)groups), dim3(256), 0, s, p);
  return launch_status("rms_norm_backward");
}

constexpr int64_t kRowsMax = 0x7FFFFFFF - 512;
constexpr int64_t kWidthMax = 1 << 20;
constexpr float kEpsMax = 1152921504606846976.0f;     // 2^60: beside a mean of squares near binary32's end it plays no part
int check_norm(const char* who, int64_t rows, int64_t d, float eps, int dtype) {
  if (dtype != AE_F32 && dtype != AE_BF16) return fail(AE_EINVAL, "%s: bad dtype", who);
  if (rows < 0 || rows > kRowsMax) return fail(AE_EINVAL, "%s: rows must be 0 .. 2^31 - 513", who);
  if (d < 1 || d > kWidthMax) return fail(AE_EINVAL, "%s: d must be 1 .. 2^20", who);
  if (!(eps >= FLT_MIN && eps <= kEpsMax)) return fail(AE_EINVAL, "%s: eps must be 2^-126 .. 2^60", who);
  return AE_OK;
}
// a matrix of rows that do not overlap, on its elements' borders; null is no matrix
bool rows_ok(const void* p, int64_t ld, int64_t d, int dtype) {
  return !p || (ld >= d && ld < ((int64_t)1 << 40) && (uintptr_t)p % dtype_size(dtype) == 0);
}

}  // namespace
}  // namespace ae

extern "C" int model_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* weight, int64_t rows, int64_t d,
                              float eps, int dtype, void* h, int64_t ldh, void* y, int64_t ldy, void* q, int64_t ldq, float* scale,
                              void* stream) {
  using namespace ae;
  AE_TRY(check_norm("model_rms_norm", rows, d, eps, dtype));
  if (rows == 0) return AE_OK;                       // a matrix without rows may have no address
  if ((!q) != (!scale)) return fail(AE_EINVAL, "model_rms_norm: codes and their scales go together");
  if (!h && !y && !q) return fail(AE_EINVAL, "model_rms_norm: no output");
  if (!x) return fail(AE_EINVAL, "model_rms_norm: null argument");
  if (!rows_ok(x, ldx, d, dtype) || !rows_ok(residual, ldr, d, dtype) || !rows_ok(h, ldh, d, dtype) || !rows_ok(y, ldy, d, dtype))
    return fail(AE_EINVAL, "model_rms_norm: rows must not overlap and must lie on their elements' borders");
  if (((uintptr_t)weight | (uintptr_t)scale) & 3) return fail(AE_EINVAL, "model_rms_norm: misaligned weight or scales");
  if (q && (((uintptr_t)q & 15) || ldq < d || ldq % 16 || ldq >= ((int64_t)1 << 40)))
    return fail(AE_EINVAL, "model_rms_norm: rows of codes must begin on 16-byte borders and not overlap");
  if ((h && ((h == x && ldh != ldx) || (h == residual && ldh != ldr))) || (y && ((y == x && ldy != ldx) || (y == residual && ldy != ldr))) || (h && h == y))
    return fail(AE_EINVAL, "model_rms_norm: an output in an input's place has its stride, and h and y have places of their own");
  const int64_t es = dtype_size(dtype);
  const bool stream_norm = rows * d * (es * (1 + !!residual + !!h + !!y) + !!q) > kStreamBytes;
  const NormArgs p = {x, ldx, residual, ldr, weight, rows, (int)d, eps, h, ldh, y, ldy, (uint8_t*)q, ldq, scale, stream_norm};
  return dtype == AE_BF16 ? launch_norm<bf16_t>(p, (hipStream_t)stream) : launch_norm<float>(p, (hipStream_t)stream);
}

extern "C" int model_rms_norm_backward_workspace(int64_t rows, int64_t d, int dtype, int64_t* bytes) {
  using namespace ae;
  if (!bytes) return fail(AE_EINVAL, "model_rms_norm_backward_workspace: null argument");
  AE_TRY(check_norm("model_rms_norm_backward_workspace", rows, d, 1.0f, dtype));
  *bytes = align16(grad_groups(rows, d, dtype) * d * 4) + (d > in_registers(dtype) ? align16(rows * (int64_t)sizeof(RowStat)) : 0);
  return AE_OK;
}

extern "C" int model_rms_norm_backward(const void* dy, int64_t ldy, const void* h, int64_t ldh, const float* weight, const void* d_h,
                                       int64_t ldg, int64_t rows, int64_t d, float eps, int dtype, void* dx, int64_t lddx,
                                       float* d_weight, void* workspace, void* stream) {
  using namespace ae;
  AE_TRY(check_norm("model_rms_norm_backward", rows, d, eps, dtype));
  if (rows == 0 && !d_weight) return AE_OK;          // a matrix without rows may have no address
  if (!dx && !d_weight) return fail(AE_EINVAL, "model_rms_norm_backward: no output");
  if (((uintptr_t)weight | (uintptr_t)d_weight) & 3) return fail(AE_EINVAL, "model_rms_norm_backward: misaligned weight");
  int64_t need = 0;
  AE_TRY(model_rms_norm_backward_workspace(rows, d, dtype, &need));
  if (need && (!workspace || ((uintptr_t)workspace & 15))) return fail(AE_EINVAL, "model_rms_norm_backward: workspace is null or not on a 16-byte border");
  hipStream_t s = (hipStream_t)stream;
  const int64_t groups = grad_groups(rows, d, dtype);
  if (rows > 0) {
    if (!dy || !h) return fail(AE_EINVAL, "model_rms_norm_backward: null argument");
    if (!rows_ok(dy, ldy, d, dtype) || !rows_ok(h, ldh, d, dtype) || !rows_ok(d_h, ldg, d, dtype) || !rows_ok(dx, lddx, d, dtype))
      return fail(AE_EINVAL, "model_rms_norm_backward: rows must not overlap and must lie on their elements' borders");
    if (dx && ((dx == dy && lddx != ldy) || (dx == h && lddx != ldh) || (dx == d_h && lddx != ldg)))
      return fail(AE_EINVAL, "model_rms_norm_backward: a gradient in an input's place has its stride");
    NormGradArgs p = {dy, ldy, h, ldh, weight, d_h, ldg, rows, (int)d, eps, dx, lddx, nullptr, nullptr, rows * d * (int64_t)dtype_size(dtype) * (2 + !!d_h + !!dx) > kStreamBytes};
    if (d_weight) p.part = (float*)workspace;
    p.stat = (RowStat*)((char*)workspace + align16(groups * d * 4));
    AE_TRY(dtype == AE_BF16 ? launch_grad<bf16_t>(p, groups, s) : launch_grad<float>(p, groups, s));
  }
  if (d_weight) hipLaunchKernelGGL(k_sum_parts, dim3((unsigned)((d + 15) / 16)), dim3(1024), 0, s, (const float*)workspace, groups, (int)d, d_weight);
  return launch_status("rms_norm_backward");
}
