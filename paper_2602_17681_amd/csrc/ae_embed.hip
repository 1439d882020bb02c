// ae_embed.hip — rows of a table picked by tokens, and the gradient of the table.
//   out[i] = scale * table[ids[i]];   d_table[v] = scale * sum of d_out[i] over the places i with ids[i] = v, in the order of i
// The gradient sorts the places by token (stable, so that a sum's order does not change from call to call), cuts the sorted
// list into runs of equal length and adds up each run's rows: a token that fills half the batch takes as many workgroups
// as its places need, and what a token has in several runs is joined in their order.
// Both are bound by memory.  16 384 tokens of 4 096 bfloat16 columns, tokens as in text: the lookup 27 us (repeated rows come from the
// cache; its results written as a stream, 39 without), the gradient over 32 768 tokens of vocabulary 141 us: sort 9.5, sums and the zeros of 27 000 tokens that do not
// occur 126 (690 MB at 5.5 TB/s), join 5.7.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "ae_device.h"
#include "ae_internal.h"
#include "ae_rows.h"

namespace ae {
namespace {

// LANES threads take a row in pieces of eight elements, 256 / LANES rows at a time and U of them in flight; the scaled value
// is rounded once.
template <typename T, int LANES, int U, bool STREAM>
__global__ __launch_bounds__(256) void k_embedding(const T* __restrict__ table, int64_t ldt, int64_t vocab, int d, const int* __restrict__ ids,
                                                   int64_t n, float scale, T* __restrict__ out, int64_t ldo, int64_t first) {
  constexpr int ROWS = 256 / LANES;
  constexpr bool SHORT = LANES == 16;
  const int t = threadIdx.x % LANES;
  const int64_t i0 = (first + blockIdx.x) * (ROWS * U) + threadIdx.x / LANES;
  int64_t at[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = i0 + u * ROWS;
    const int id = i < n ? ids[i] : -1;
    at[u] = id >= 0 && id < vocab ? (int64_t)id * ldt : -1;
  }
  for (int col = (blockIdx.y * LANES + t) * 8; col < d; col += gridDim.y * LANES * 8) {
    const int left = d - col;
    Eight<T> e[U];
#pragma unroll
    for (int u = 0; u < U; ++u) fetch_row<false, SHORT>(table + (at[u] < 0 ? 0 : at[u]), col, d, e[u]);       // no token: the first row, not used
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * ROWS >= n) continue;
      settle<SHORT>(col, d, e[u]);
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = at[u] < 0 ? 0.0f : value(e[u], j) * scale;
      put<STREAM>(out + (i0 + u * ROWS) * ldo + col, left, v);
    }
  }
}

// ---- the gradient ------------------------------------------------------------------------------------------------
// Places in the order of their tokens, without a pass over global counters: each workgroup owns a range of tokens, reads
// all ids twice (they are few bytes beside the rows) and keeps its tokens' counters in LDS.  The first pass counts its
// tokens and what lies below its range; the second puts its places down in their order.
constexpr int SORT_NT = 1024, SORT_WAVES = SORT_NT / 64, SORT_RANGE = 4096;    // tokens of a range at most
struct EmbedSort {
  int* place;                             // [n]: places in the order of their tokens
  int* token;                             // [n]: the token at each position of that order
  int* start;                             // [vocab + 1]: each token's first position; null: no token occurs
};
// LOADS times four neighbouring ids are in a thread's registers at a time.
template <int LOADS>
__global__ __launch_bounds__(SORT_NT) void k_embed_sort(const int* __restrict__ ids, int64_t n, int vocab, int range, EmbedSort out) {
  constexpr int IDS = SORT_NT * 4 * LOADS, LANES = LOADS * SORT_WAVES;
  __shared__ int at[SORT_RANGE];
  __shared__ uint32_t queue[IDS];                // token within the range << 14 | place within the ids at hand
  __shared__ int sums[LANES < 2 * SORT_WAVES ? 2 * SORT_WAVES : LANES];
  static_assert(IDS <= 1 << 14 && SORT_RANGE <= 1 << 18, "a queue entry holds both");
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int v0 = (int)blockIdx.x * range, mine = vocab - v0 < range ? vocab - v0 : range;
  int id[LOADS][4];
  auto load = [&](int64_t base) {
#pragma unroll
    for (int l = 0; l < LOADS; ++l) {
      const int64_t i = base + (l * SORT_NT + t) * 4;
      if (i + 4 <= n) {
        __builtin_memcpy(id[l], ids + i, 16);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) id[l][k] = i + k < n ? ids[i + k] : -1;
      }
    }
  };
  load(0);
  for (int v = t; v < mine; v += SORT_NT) at[v] = 0;
  __syncthreads();
  int below = 0;
  for (int64_t base = 0; base < n; base += IDS) {
    if (base) load(base);
#pragma unroll
    for (int l = 0; l < LOADS; ++l)
#pragma unroll
      for (int k = 0; k < 4; ++k) {              // a negative id is a large unsigned number
        below += (unsigned)id[l][k] < (unsigned)v0;
        const unsigned v = (unsigned)id[l][k] - (unsigned)v0;
        if (v < (unsigned)mine) atomicAdd(&at[v], 1);
      }
  }
  // exclusive sums: of `below` over the threads, then of the counters
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) below += __shfl_xor(below, o, 64);
  if (lane == 0) sums[wave] = below;
  __syncthreads();
  const int each = (range + SORT_NT - 1) / SORT_NT, c0 = t * each;
  int run = 0, count = 0;
  for (int w = 0; w < SORT_WAVES; ++w) run += sums[w];
  for (int v = c0; v < c0 + each && v < mine; ++v) count += at[v];
  int incl = count;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(incl, o, 64);
    if (lane >= o) incl += up;
  }
  if (lane == 63) sums[SORT_WAVES + wave] = incl;
  __syncthreads();
  run += incl - count;
  for (int w = 0; w < wave; ++w) run += sums[SORT_WAVES + w];
  for (int v = c0; v < c0 + each && v < mine; ++v) {
    const int c = at[v];
    at[v] = run;
    out.start[v0 + v] = run;
    run += c;
  }
  if (v0 + mine == vocab && c0 < mine && c0 + each >= mine) out.start[vocab] = run;
  for (int64_t base = 0; base < n; base += IDS) {
    __syncthreads();
    if (n > IDS) load(base);
    // this range's tokens among these ids, in order
    int before[LOADS];
#pragma unroll
    for (int l = 0; l < LOADS; ++l) {
      int total = 0;
      before[l] = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint64_t m = __ballot((unsigned)id[l][k] - (unsigned)v0 < (unsigned)mine);
        before[l] += __popcll(m & (((uint64_t)1 << lane) - 1));
        total += __popcll(m);
      }
      if (lane == 0) sums[l * SORT_WAVES + wave] = total;
    }
    __syncthreads();
    // the sums one to a lane: all wavefronts scan them alike
    static_assert(LANES <= 64, "a sum to a lane");
    int scan = lane < LANES ? sums[lane] : 0;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(scan, o, 64);
      if (lane >= o) scan += up;
    }
    const int all = __builtin_amdgcn_readlane(scan, 63);
#pragma unroll
    for (int l = 0; l < LOADS; ++l) {
      const int slot = l * SORT_WAVES + wave;
      int q = before[l] + (slot ? __shfl(scan, slot - 1, 64) : 0);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const unsigned v = (unsigned)id[l][k] - (unsigned)v0;
        if (v < (unsigned)mine) queue[q++] = v << 14 | ((l * SORT_NT + t) * 4 + k);
      }
    }
    __syncthreads();
    for (int q0 = 0; q0 < all; q0 += SORT_NT) {
      const bool live = q0 + t < all;
      const uint32_t e = live ? queue[q0 + t] : 0;
      const int mv = live ? (int)(e >> 14) : -1;
      // among the wavefront's 64: how many equal ones come before, and who of them stands for all
      int rank = 0, leader = 0, equal = 0;
      uint64_t todo = __ballot(live);
      while (todo) {
        const int first = __ffsll((unsigned long long)todo) - 1, fv = __builtin_amdgcn_readlane(mv, first);
        const uint64_t m = __ballot(mv == fv);
        if (mv == fv) {
          rank = __popcll(m & (((uint64_t)1 << lane) - 1));
          leader = first;
          equal = __popcll(m);
        }
        todo &= ~m;
      }
      const int waves = (all - q0 + 63) / 64;
      int from = 0;
      for (int w = 0; w < SORT_WAVES && w < waves; ++w) {       // one wavefront after the other
        if (w == wave && live && rank == 0) {
          from = at[mv];
          at[mv] = from + equal;
        }
        __syncthreads();
      }
      from = __shfl(from, leader, 64);
      if (live) {
        out.place[from + rank] = (int)(base + (e & ((1 << 14) - 1)));
        out.token[from + rank] = v0 + mv;
      }
    }
  }
}

struct EmbedGrad {
  const void* d_out;
  int64_t ldo;
  EmbedSort sort;
  int vocab, d, run;                      // run: positions of the sorted list that are added up by one team (few places: rows of zeros to a workgroup)
  int64_t n, runs;
  int cols, sums;                         // pieces of a row, and workgroups that add up; the others write zeros
  float scale;
  float* d_table;
  int64_t ldt;
  int accumulate;
  bool stream;                            // the table is large, and whole lines are written
  int* owner;                             // [runs]: the token that begins in a run and goes on behind it, or -1
  float* part;                            // [runs][2][d]: a run's share of a token that begins before it, of one that goes on behind it
};
__device__ __forceinline__ void add_row(const EmbedGrad& p, int v, int col, const float (&acc)[4]) {
  float* at = p.d_table + (int64_t)v * p.ldt + col;
  const int left = p.d - col;
  Piece<float, 4> old;
  if (p.accumulate) fetch(at, left, old);
  float o[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] = p.accumulate ? value(old, j) + acc[j] * p.scale : acc[j] * p.scale;
  put(at, left, o);
}
// W wavefronts add up the rows of a run of sorted places, NV times four neighbouring columns to a lane (16 bytes of the result, so
// that a wavefront's stores are whole lines).  The workgroups behind `sums` write the zeros of tokens that do not occur (among the sums,
// one for one: 228 us against 162, since every second workgroup is on the same four of the eight dies; by eights 166 against 150).
constexpr int ZERO_ROWS = 4;                     // (embed gradient above 150 us with 4 rows or 2, 152 with 16; beside the join instead of the sums no faster)
template <typename T, int W, int NV, bool SHORT>
__global__ __launch_bounds__(256) void k_embed_sum(EmbedGrad p) {
  constexpr int TEAM = 64 * W, TEAMS = 4 / W;
  if ((int)blockIdx.x >= p.sums) {
    const int lane = threadIdx.x & 63, v0 = ((int)blockIdx.x - p.sums) * ZERO_ROWS, v = v0 + lane;
    const uint64_t todo = __ballot(lane < ZERO_ROWS && v < p.vocab && (!p.sort.start || p.sort.start[v] == p.sort.start[v + 1]));
    // a large table's zeros as a stream: 16 384 tokens into 32 768 x 4 096 149 us without, 141 with, its sums too 150; 6 022 tokens into
    // 22 088 x 4 555, whose rows begin on 4-byte borders, 120 without and 124 with
    auto write = [&](auto stream) {
      const float zero[4] = {0, 0, 0, 0};
      for (uint64_t left = todo; left; left &= left - 1) {
        float* at = p.d_table + (int64_t)(v0 + __ffsll((unsigned long long)left) - 1) * p.ldt;
        for (int col = threadIdx.x * 4; col < p.d; col += 1024) put<stream>(at + col, p.d - col, zero);
      }
    };
    if (p.stream) write(std::true_type());
    else write(std::false_type());
    return;
  }
  const int t = threadIdx.x % TEAM, lane = threadIdx.x & 63;
  const int group = (int)blockIdx.x / p.cols, c0 = ((int)blockIdx.x - group * p.cols) * (TEAM * 4 * NV) + t * 4;
  const int64_t run = (int64_t)group * TEAMS + (TEAMS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM) : 0);
  if (run >= p.runs) return;
  // what the run depends on is asked for at once: behind `all` the lists hold nothing, but there is room up to n
  const int64_t from = run * p.run;
  const int all = p.sort.start[p.vocab], earlier = from ? p.sort.token[from - 1] : -1;
  int place = from + lane < p.n ? p.sort.place[from + lane] : 0, token = from + lane < p.n ? p.sort.token[from + lane] : -1;
  const int64_t to = from + p.run < all ? from + p.run : all;
  if (from >= to) {
    if (c0 == 0) p.owner[run] = -1;
    return;
  }
  const int behind = to < all ? p.sort.token[to] : -1;
  constexpr int U = NV * sizeof(T) > 4 ? 8 : 16;               // rows in flight
  float acc[NV][4];
  auto clear = [&] {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[k][j] = 0.0f;
  };
  auto give = [&](int v) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (c0 + k * TEAM * 4 < p.d) add_row(p, v, c0 + k * TEAM * 4, acc[k]);
  };
  auto keep = [&](int slot) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int col = c0 + k * TEAM * 4;
      if (col < p.d) put(p.part + (run * 2 + slot) * p.d + col, p.d - col, acc[k]);
    }
  };
  clear();
  const bool edge = __any(c0 + (NV - 1) * TEAM * 4 > p.d - 4);   // the rows' end lies in this wavefront's columns
  int v = __builtin_amdgcn_readfirstlane(token);
  bool begun = earlier == v;                     // the sum at hand is of a token that began before the run
  for (int64_t s0 = from; s0 < to; s0 += 64) {
    const int here = to - s0 < 64 ? (int)(to - s0) : 64;
    if (s0 > from) {
      place = lane < here ? p.sort.place[s0 + lane] : 0;
      token = lane < here ? p.sort.token[s0 + lane] : -1;
    }
    for (int u0 = 0; u0 < here; u0 += U) {
      Piece<T, 4> e[U][NV];
#pragma unroll
      for (int u = 0; u < U; ++u) {                // behind the run's end: its last row again
        const T* row = (const T*)p.d_out + (int64_t)__builtin_amdgcn_readlane(place, u0 + u < here ? u0 + u : here - 1) * p.ldo;
#pragma unroll
        for (int k = 0; k < NV; ++k) fetch_row<true, SHORT>(row, c0 + k * TEAM * 4, p.d, e[u][k]);
      }
      if (edge) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int k = 0; k < NV; ++k) settle<SHORT>(c0 + k * TEAM * 4, p.d, e[u][k]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u0 + u >= here) break;
        const int tok = __builtin_amdgcn_readlane(token, u0 + u);
        if (tok != v) {
          if (begun) keep(0);
          else give(v);
          begun = false;
          v = tok;
          clear();
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[k][j] += value(e[u][k], j);
        }
      }
    }
  }
  const bool on = !begun && behind == v;
  if (begun) keep(0);
  else if (on) keep(1);
  else give(v);
  if (c0 == 0) p.owner[run] = on ? v : -1;
}
// A token that begins in a run and goes on: the shares of the runs that follow, a quarter of them to a wavefront, joined in their
// order.  A workgroup has 256 columns of one run's token.
__global__ __launch_bounds__(256) void k_embed_join(EmbedGrad p) {
  __shared__ float sm[3][256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = (int)blockIdx.y * 256 + lane * 4, left = p.d - col;
  const int64_t r = blockIdx.x;
  const int v = p.owner[r];
  if (v < 0) return;
  const int64_t n = (p.sort.start[v + 1] - 1) / p.run - r;
  const int64_t begin = r + 1 + n * wave / 4, end = r + 1 + n * (wave + 1) / 4;
  float acc[4];
  Piece<float, 4> own;
  fetch(p.part + (r * 2 + 1) * p.d + col, wave == 0 ? left : 0, own);
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = value(own, j);
  constexpr int U = 8;
  for (int64_t i = begin; i < end; i += U) {
    Piece<float, 4> e[U];
#pragma unroll
    for (int u = 0; u < U; ++u) fetch(p.part + (i + u) * 2 * p.d + col, i + u < end ? left : 0, e[u]);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] += value(e[u], j);
  }
  if (wave) {
#pragma unroll
    for (int j = 0; j < 4; ++j) sm[wave - 1][lane * 4 + j] = acc[j];
  }
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int w = 0; w < 3; ++w)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] += sm[w][lane * 4 + j];
  if (left > 0) add_row(p, v, col, acc);
}

// Few places: one launch without sorting.  Every place has a team, which compares its token with all ids at once; the first
// place of a token goes on and adds up the rows of all its places in their order.  Against the three launches below, in us, bfloat16,
// tokens as in text / all different / all the same, 4 000 tokens of vocabulary: 256 places of 1 024 columns 6.3 / 6.0 / 17 (three launches
// 15.7 / 14.4 / 13), 512 6.6 / 6.9 / 30 (15.6 / 15.7 / 14), 1 024 9 / 9 / 58 (16 / 16 / 17); 512 of 4 096 columns 15 / 17 / 38 (21 / 21 / 21), 1 024
// 22 / 24 / 67 (24 / 23 / 24): what one token costs a single team ends the rule at 512.
constexpr int FEW = 512, FEW_ZERO_ROWS = 16;     // at most: as many rows of zeros to a workgroup as leave 1 024 of them
template <typename T, int W, int NV, bool SHORT>
__global__ __launch_bounds__(256) void k_embed_few(EmbedGrad p, const int* __restrict__ ids) {
  constexpr int TEAM = 64 * W, TEAMS = 4 / W;
  __shared__ int places[4][FEW];                 // each wavefront's own list
  const int n = (int)p.n, lane = threadIdx.x & 63;
  if ((int)blockIdx.x >= p.sums) {
    const int v0 = ((int)blockIdx.x - p.sums) * p.run, rows = p.vocab - v0 < p.run ? p.vocab - v0 : p.run;
    int* there = places[0];
    if (threadIdx.x < FEW_ZERO_ROWS) there[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < FEW / 256; ++k) {
      const int i = k * 256 + (int)threadIdx.x;
      const unsigned v = i < n ? (unsigned)ids[i] - (unsigned)v0 : ~0u;
      if (v < (unsigned)rows) there[v] = 1;      // whoever writes, writes the same
    }
    __syncthreads();
    const float zero[4] = {0, 0, 0, 0};
    for (int v = 0; v < rows; ++v) {               // (500 tokens into 24 576 x 4 096 81 us, as a stream 84: nothing beside them)
      if (there[v]) continue;
      float* at = p.d_table + (int64_t)(v0 + v) * p.ldt;
      for (int col = threadIdx.x * 4; col < p.d; col += 1024) put(at + col, p.d - col, zero);
    }
    return;
  }
  const int t = threadIdx.x % TEAM, wave = threadIdx.x >> 6;
  const int group = (int)blockIdx.x / p.cols, c0 = ((int)blockIdx.x - group * p.cols) * (TEAM * 4 * NV) + t * 4;
  const int mine = group * TEAMS + (TEAMS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM) : 0);
  if (mine >= n) return;
  int id[FEW / 64];
#pragma unroll
  for (int k = 0; k < FEW / 64; ++k) id[k] = k * 64 + lane < n ? ids[k * 64 + lane] : -1;
  const int v = ids[mine];
  if (v < 0 || v >= p.vocab) return;
  int count = 0;
#pragma unroll
  for (int k = 0; k < FEW / 64; ++k) {
    const uint64_t m = __ballot(id[k] == v);
    if (id[k] == v) places[wave][count + __popcll(m & (((uint64_t)1 << lane) - 1))] = k * 64 + lane;
    count += __popcll(m);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");         // the list is written and read by this wavefront alone
  if (__builtin_amdgcn_readfirstlane(places[wave][0]) != mine) return;
  constexpr int U = NV * sizeof(T) > 4 ? 8 : 16;               // rows in flight
  const bool edge = __any(c0 + (NV - 1) * TEAM * 4 > p.d - 4);   // the rows' end lies in this wavefront's columns
  float acc[NV][4];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[k][j] = 0.0f;
  for (int at = 0; at < count; at += U) {
    Piece<T, 4> e[U][NV];
    const int place = places[wave][at + lane < count ? at + lane : count - 1];           // behind the list's end: its last row again
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const T* row = (const T*)p.d_out + (int64_t)__builtin_amdgcn_readlane(place, u) * p.ldo;
#pragma unroll
      for (int k = 0; k < NV; ++k) fetch_row<false, SHORT>(row, c0 + k * TEAM * 4, p.d, e[u][k]);
    }
    if (edge) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < NV; ++k) settle<SHORT>(c0 + k * TEAM * 4, p.d, e[u][k]);
    }
    if (at + U <= count) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[k][j] += value(e[u][k], j);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[k][j] = at + u < count ? acc[k][j] + value(e[u][k], j) : acc[k][j];
    }
  }
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (c0 + k * TEAM * 4 < p.d) add_row(p, v, c0 + k * TEAM * 4, acc[k]);
}

// Wavefronts and four-column pieces of a lane that share a run, and from them its positions: at least 16, and as many as leave
// 1 024 workgroups (16 384 x 4 096 150 us, with 2 048 148 and twice the workspace; 16 positions always 228: more partial sums; all before the
// zeros went as a stream).
int team_of(int64_t d) { return d <= 512 ? 1 : 4; }
int pieces_of(int64_t d) { return d > 256 && d <= 512 ? 2 : 1; }
int64_t run_of(int64_t n, int64_t d) {
  const int64_t cols = 256 * team_of(d) * pieces_of(d), groups = 1024 * (4 / team_of(d)) / ((d + cols - 1) / cols);
  const int64_t r = (n + groups - 1) / (groups < 1 ? 1 : groups);
  return r < 16 ? 16 : r;
}
int64_t runs_of(int64_t n, int64_t d) { return (n + run_of(n, d) - 1) / run_of(n, d); }

template <typename T, int W, int NV, bool SHORT = false>
int launch_embed_sum(EmbedGrad p, hipStream_t s) {
  constexpr int TEAMS = 4 / W, COLS = 64 * W * 4 * NV;
  p.cols = (p.d + COLS - 1) / COLS;
  p.sums = (int)((p.runs + TEAMS - 1) / TEAMS) * p.cols;
  const int zeros = p.accumulate ? 0 : (p.vocab + ZERO_ROWS - 1) / ZERO_ROWS;
  hipLaunchKernelGGL((k_embed_sum<T, W, NV, SHORT>), dim3((unsigned)(p.sums + zeros)), dim3(256), 0, s, p);
  return launch_status("embedding_backward");
}
template <typename T, int W, int NV, bool SHORT = false>
int launch_embed_few_team(EmbedGrad p, const int* ids, hipStream_t s) {
  constexpr int TEAMS = 4 / W, COLS = 64 * W * 4 * NV;
  p.cols = (p.d + COLS - 1) / COLS;
  p.sums = (int)((p.n + TEAMS - 1) / TEAMS) * p.cols;
  p.run = p.vocab < 2048 ? 1 : p.vocab / 1024 < FEW_ZERO_ROWS ? p.vocab / 1024 : FEW_ZERO_ROWS;
  const int zeros = p.accumulate ? 0 : (p.vocab + p.run - 1) / p.run;
  hipLaunchKernelGGL((k_embed_few<T, W, NV, SHORT>), dim3((unsigned)(p.sums + zeros)), dim3(256), 0, s, p, ids);
  return launch_status("embedding_backward");
}
template <typename T>
int launch_embed_few(const EmbedGrad& p, const int* ids, hipStream_t s) {
  if (p.d < 4) return launch_embed_few_team<T, 1, 1, true>(p, ids, s);       // rows shorter than a piece
  if (team_of(p.d) == 1) return pieces_of(p.d) == 1 ? launch_embed_few_team<T, 1, 1>(p, ids, s) : launch_embed_few_team<T, 1, 2>(p, ids, s);
  return launch_embed_few_team<T, 4, 1>(p, ids, s);
}
template <typename T>
int launch_embed_sums(const EmbedGrad& p, hipStream_t s) {
  if (p.d < 4) return launch_embed_sum<T, 1, 1, true>(p, s);       // rows shorter than a piece
  if (team_of(p.d) == 1) return pieces_of(p.d) == 1 ? launch_embed_sum<T, 1, 1>(p, s) : launch_embed_sum<T, 1, 2>(p, s);
  return launch_embed_sum<T, 4, 1>(p, s);
}

constexpr int64_t kTokensMax = 1 << 30, kVocabMax = 1 << 20, kWidthMax = 1 << 20;
int64_t align16(int64_t v) { return (v + 15) / 16 * 16; }
int check_embedding(const char* who, int64_t n, int64_t vocab, int64_t d, int dtype) {
  if (dtype != AE_F32 && dtype != AE_BF16) return fail(AE_EINVAL, "%s: bad dtype", who);
  if (n < 0 || n > kTokensMax) return fail(AE_EINVAL, "%s: tokens must be 0 .. 2^30", who);
  if (vocab < 1 || vocab > kVocabMax) return fail(AE_EINVAL, "%s: vocab must be 1 .. 2^20", who);
  if (d < 1 || d > kWidthMax) return fail(AE_EINVAL, "%s: d must be 1 .. 2^20", who);
  return AE_OK;
}
bool stride_ok(int64_t ld, int64_t d) { return ld >= d && ld < ((int64_t)1 << 40); }

template <typename T, int LANES, int U, bool STREAM = false>
int launch_embedding(const void* table, int64_t ldt, int64_t vocab, int64_t d, const int* ids, int64_t n, float scale, void* out, int64_t ldo,
                     hipStream_t s) {
  const int64_t rows = 256 / LANES * U, want = (n + rows - 1) / rows, pieces = (d + LANES * 8 - 1) / (LANES * 8);
  const int64_t cols = pieces < 64 ? pieces : 64, most = launch_blocks(256) / cols;
  for (int64_t first = 0; first < want; first += most) {
    const int64_t left = want - first;
    hipLaunchKernelGGL((k_embedding<T, LANES, U, STREAM>), dim3((unsigned)(left < most ? left : most), (unsigned)cols), dim3(256), 0, s, (const T*)table, ldt, vocab,
                       (int)d, ids, n, scale, (T*)out, ldo, first);
  }
  return launch_status("embedding");
}
template <typename T>
int launch_embedding_rows(const void* table, int64_t ldt, int64_t vocab, int64_t d, const int* ids, int64_t n, float scale, void* out, int64_t ldo,
                          hipStream_t s) {
  if (d <= 128) return launch_embedding<T, 16, 1>(table, ldt, vocab, d, ids, n, scale, out, ldo, s);
  if (d <= 512) return launch_embedding<T, 64, 1>(table, ldt, vocab, d, ids, n, scale, out, ldo, s);
  if (n < 1024) return launch_embedding<T, 256, 1>(table, ldt, vocab, d, ids, n, scale, out, ldo, s);
  if (2 * n * d * (int64_t)sizeof(T) > kStreamBytes) return launch_embedding<T, 256, 4, true>(table, ldt, vocab, d, ids, n, scale, out, ldo, s);
  return launch_embedding<T, 256, 4>(table, ldt, vocab, d, ids, n, scale, out, ldo, s);
}

}  // namespace
}  // namespace ae

extern "C" int model_embedding(const void* table, int64_t ldt, int64_t vocab, int64_t d, const int* ids, int64_t n, float scale, int dtype,
                               void* out, int64_t ldo, void* stream) {
  using namespace ae;
  AE_TRY(check_embedding("model_embedding", n, vocab, d, dtype));
  if (!stride_ok(ldt, d) || !stride_ok(ldo, d)) return fail(AE_EINVAL, "model_embedding: rows must not overlap");
  if (n == 0) return AE_OK;
  if (!table || !ids || !out) return fail(AE_EINVAL, "model_embedding: null argument");
  if (((uintptr_t)table | (uintptr_t)out) % dtype_size(dtype) || ((uintptr_t)ids & 3)) return fail(AE_EINVAL, "model_embedding: misaligned argument");
  if (table == out) return fail(AE_EINVAL, "model_embedding: the rows cannot take the table's place");
  return dtype == AE_BF16 ? launch_embedding_rows<bf16_t>(table, ldt, vocab, d, ids, n, scale, out, ldo, (hipStream_t)stream)
                          : launch_embedding_rows<float>(table, ldt, vocab, d, ids, n, scale, out, ldo, (hipStream_t)stream);
}

extern "C" int model_embedding_backward_workspace(int64_t n, int64_t vocab, int64_t d, int dtype, int64_t* bytes) {
  using namespace ae;
  if (!bytes) return fail(AE_EINVAL, "model_embedding_backward_workspace: null argument");
  AE_TRY(check_embedding("model_embedding_backward_workspace", n, vocab, d, dtype));
  *bytes = n <= FEW ? 0 : 2 * align16(n * 4) + align16((vocab + 1) * 4) + align16(runs_of(n, d) * 4) + runs_of(n, d) * 2 * d * 4;
  return AE_OK;
}

extern "C" int model_embedding_backward(const void* d_out, int64_t ldo, const int* ids, int64_t n, int64_t vocab, int64_t d, float scale,
                                        int dtype, float* d_table, int64_t ldt, int accumulate, void* workspace, void* stream) {
  using namespace ae;
  int64_t need = 0;
  AE_TRY(check_embedding("model_embedding_backward", n, vocab, d, dtype));
  if (!stride_ok(ldo, d) || !stride_ok(ldt, d)) return fail(AE_EINVAL, "model_embedding_backward: rows must not overlap");
  if (!d_table || ((uintptr_t)d_table & 3)) return fail(AE_EINVAL, "model_embedding_backward: d_table is null or misaligned");
  AE_TRY(model_embedding_backward_workspace(n, vocab, d, dtype, &need));
  hipStream_t s = (hipStream_t)stream;
  if (n > 0) {
    if (!d_out || !ids) return fail(AE_EINVAL, "model_embedding_backward: null argument");
    if ((uintptr_t)d_out % dtype_size(dtype) || ((uintptr_t)ids & 3)) return fail(AE_EINVAL, "model_embedding_backward: misaligned argument");
    if (need && (!workspace || ((uintptr_t)workspace & 15))) return fail(AE_EINVAL, "model_embedding_backward: workspace is null or not on a 16-byte border");
  } else if (accumulate) {
    return AE_OK;
  }
  char* ws = (char*)workspace;
  EmbedGrad p = {d_out, ldo, {}, (int)vocab, (int)d, (int)run_of(n, d), n, runs_of(n, d), 0, 0, scale, d_table, ldt, accumulate ? 1 : 0,
                 vocab * d * 4 > kStreamBytes && ldt % 4 == 0 && ((uintptr_t)d_table & 15) == 0, nullptr, nullptr};
  if (n == 0) return launch_embed_sums<float>(p, s);       // zeros alone
  if (n <= FEW) return dtype == AE_BF16 ? launch_embed_few<bf16_t>(p, ids, s) : launch_embed_few<float>(p, ids, s);
  p.sort.place = (int*)ws;
  p.sort.token = (int*)(ws + align16(n * 4));
  p.sort.start = (int*)(ws + 2 * align16(n * 4));
  p.owner = (int*)(ws + 2 * align16(n * 4) + align16((vocab + 1) * 4));
  p.part = (float*)((char*)p.owner + align16(p.runs * 4));
  const int range = (int)((vocab + 255) / 256);
  static_assert(kVocabMax / 256 <= SORT_RANGE, "a range's counters fit into LDS");
  // 1 024 places in one batch of four each 15.8 us with the sums, 17.8 in the kernel for four batches; 4 097 in two 18.2 and 19.4
  const auto sort = n <= 4 * SORT_NT ? k_embed_sort<1> : n <= 8 * SORT_NT ? k_embed_sort<2> : k_embed_sort<4>;
  hipLaunchKernelGGL(sort, dim3((unsigned)((vocab + range - 1) / range)), dim3(SORT_NT), 0, s, ids, n, (int)vocab, range, p.sort);
  AE_TRY(dtype == AE_BF16 ? launch_embed_sums<bf16_t>(p, s) : launch_embed_sums<float>(p, s));
  if (p.runs > 1)
    hipLaunchKernelGGL(k_embed_join, dim3((unsigned)(p.runs - 1), (unsigned)((d + 255) / 256)), dim3(256), 0, s, p);
  return launch_status("embedding_backward");
}
