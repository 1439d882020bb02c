// ae_embed.hip — rows of a table picked by tokens, and the gradient of the table.
//   out[i] = scale * table[ids[i]];   d_table[v] = scale * sum of d_out[i] over the places i with ids[i] = v, in the order of i
// The gradient sorts the places by token (stable, so that a sum's order does not change from call to call), cuts the sorted
// list into runs of equal length and adds up each run's rows: a token that fills half the batch takes as many workgroups
// as its places need, and what a token has in several runs is joined in their order.
#include <hip/hip_runtime.h>

#include "ae_device.h"
#include "ae_internal.h"
#include "ae_rows.h"

namespace ae {
namespace {

// LANES threads take a row in pieces of eight elements, 256 / LANES rows at a time and U of them in flight; the scaled value
// is rounded once.
template <typename T, int LANES, int U>
__global__ __launch_bounds__(256) void k_embedding(const T* __restrict__ table, int64_t ldt, int64_t vocab, int d, const int* __restrict__ ids,
                                                   int64_t n, float scale, T* __restrict__ out, int64_t ldo, int64_t first) {
  constexpr int ROWS = 256 / LANES;
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
    for (int u = 0; u < U; ++u) fetch8(table + (at[u] < 0 ? 0 : at[u]) + col, at[u] < 0 ? 0 : left, e[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * ROWS >= n) continue;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = at[u] < 0 ? 0.0f : value(e[u], j) * scale;
      put8(out + (i0 + u * ROWS) * ldo + col, left, v);
    }
  }
}

// ---- the gradient ------------------------------------------------------------------------------------------------
// Places in the order of their tokens, without a pass over global counters: each workgroup owns a range of tokens, reads
// all ids twice (they are few bytes beside the rows) and keeps its tokens' counters in LDS.  The first pass counts its
// tokens and what lies below its range; the second puts its places down in their order.
constexpr int SORT_NT = 1024, SORT_WAVES = SORT_NT / 64, SORT_RANGE = 4096, SORT_IDS = 4;    // tokens of a range at most; ids of a thread at a time
struct EmbedSort {
  int* place;                             // [n]: places in the order of their tokens
  int* token;                             // [n]: the token at each position of that order
  int* start;                             // [vocab + 1]: each token's first position; null: no token occurs
};
__global__ __launch_bounds__(SORT_NT) void k_embed_sort(const int* __restrict__ ids, int64_t n, int vocab, int range, EmbedSort out) {
  __shared__ int at[SORT_RANGE];
  __shared__ int queue_v[SORT_NT * SORT_IDS], queue_i[SORT_NT * SORT_IDS];
  __shared__ int wave_sum_of[SORT_WAVES + 1];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int v0 = (int)blockIdx.x * range, mine = vocab - v0 < range ? vocab - v0 : range;
  for (int v = t; v < mine; v += SORT_NT) at[v] = 0;
  __syncthreads();
  int below = 0;
  for (int64_t i = t; i < n; i += SORT_NT) {
    const int id = ids[i];
    below += id >= 0 && id < v0;
    if ((unsigned)(id - v0) < (unsigned)mine && id >= 0) atomicAdd(&at[id - v0], 1);
  }
  // exclusive sums: of `below` over the threads, then of the counters
  auto wave_total = [&](int v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
  };
  below = wave_total(below);
  if (lane == 0) wave_sum_of[wave] = below;
  __syncthreads();
  int base = 0;
  for (int w = 0; w < SORT_WAVES; ++w) base += wave_sum_of[w];
  const int each = (range + SORT_NT - 1) / SORT_NT, c0 = t * each;
  int count = 0;
  for (int v = c0; v < c0 + each && v < mine; ++v) count += at[v];
  int incl = count;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(incl, o, 64);
    if (lane >= o) incl += up;
  }
  __syncthreads();
  if (lane == 63) wave_sum_of[wave] = incl;
  __syncthreads();
  int run = base + incl - count;
  for (int w = 0; w < wave; ++w) run += wave_sum_of[w];
  for (int v = c0; v < c0 + each && v < mine; ++v) {
    const int c = at[v];
    at[v] = run;
    out.start[v0 + v] = run;
    run += c;
  }
  if (v0 + mine == vocab && c0 < mine && c0 + each >= mine) out.start[vocab] = run;
  __syncthreads();
  for (int64_t i0 = 0; i0 < n; i0 += SORT_NT * SORT_IDS) {
    // this range's tokens among the next ids, in order
    int v[SORT_IDS], total = 0, before = 0;
    bool hit[SORT_IDS];
#pragma unroll
    for (int k = 0; k < SORT_IDS; ++k) {
      const int64_t i = i0 + t * SORT_IDS + k;
      const int id = i < n ? ids[i] : -1;
      v[k] = id - v0;
      hit[k] = id >= 0 && (unsigned)v[k] < (unsigned)mine;
      const uint64_t m = __ballot(hit[k]);
      before += __popcll(m & (((uint64_t)1 << lane) - 1));
      total += __popcll(m);
    }
    if (lane == 0) wave_sum_of[wave] = total;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < SORT_WAVES; ++w) {
      if (w < wave) before += wave_sum_of[w];
      all += wave_sum_of[w];
    }
#pragma unroll
    for (int k = 0; k < SORT_IDS; ++k)
      if (hit[k]) {
        queue_v[before] = v[k];
        queue_i[before++] = (int)(i0 + t * SORT_IDS + k);
      }
    __syncthreads();
    for (int q0 = 0; q0 < all; q0 += SORT_NT) {
      const bool live = q0 + t < all;
      const int mv = live ? queue_v[q0 + t] : -1;
      // among the wavefront's 64: how many equal ones come before, and who of them stands for all
      int rank = 0, leader = 0, equal = 0;
      uint64_t todo = __ballot(live);
      while (todo) {
        const int first = __ffsll((unsigned long long)todo) - 1, fv = __shfl(mv, first, 64);
        const uint64_t m = __ballot(live && mv == fv);
        if (live && mv == fv) {
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
        out.place[from + rank] = queue_i[q0 + t];
        out.token[from + rank] = v0 + mv;
      }
    }
    __syncthreads();
  }
}

struct EmbedGrad {
  const void* d_out;
  int64_t ldo;
  EmbedSort sort;
  int vocab, d, run;                      // run: positions of the sorted list that a workgroup takes
  int64_t runs;
  float scale;
  float* d_table;
  int64_t ldt;
  int accumulate;
  float* part;                            // [runs][2][d]: a run's share of a token that begins before it, of one that goes on behind it
};
__device__ __forceinline__ void add_row(const EmbedGrad& p, int v, int col, const float (&acc)[8]) {
  float* at = p.d_table + (int64_t)v * p.ldt + col;
  const int left = p.d - col;
  float o[8];
  if (p.accumulate) load8<float>(at, left, o);
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = p.accumulate ? o[j] + acc[j] * p.scale : acc[j] * p.scale;
  put8(at, left, o);
}
// Workgroups below `runs` add up a run of the sorted places each, the others write the zeros of tokens that do not occur.
// blockIdx.y: 2 048 columns.
template <typename T>
__global__ __launch_bounds__(256) void k_embed_sum(EmbedGrad p) {
  const int col = ((int)blockIdx.y * 256 + (int)threadIdx.x) * 8, left = p.d - col;
  if ((int64_t)blockIdx.x >= p.runs) {
    if (left <= 0) return;
    const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const int stride = (int)(gridDim.x - p.runs);
    for (int v = (int)(blockIdx.x - p.runs); v < p.vocab; v += stride)
      if (!p.sort.start || p.sort.start[v] == p.sort.start[v + 1]) put8(p.d_table + (int64_t)v * p.ldt + col, left, zero);
    return;
  }
  const int all = p.sort.start[p.vocab];
  const int64_t from = (int64_t)blockIdx.x * p.run, to = from + p.run < all ? from + p.run : all;
  if (from >= to || left <= 0) return;
  constexpr int U = sizeof(T) == 2 ? 8 : 4;        // rows in flight
  float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  float* const mine = p.part + (int64_t)blockIdx.x * 2 * p.d + col;
  int v = p.sort.token[from];
  const bool begun = p.sort.start[v] < from;       // the run's first token began before it
  bool first = true;
  for (int64_t s0 = from; s0 < to; s0 += U) {
    Eight<T> e[U];
    int tok[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = s0 + u < to;
      tok[u] = in ? p.sort.token[s0 + u] : -1;
      const int64_t i = in ? p.sort.place[s0 + u] : 0;
      fetch8((const T*)p.d_out + i * p.ldo + col, in ? left : 0, e[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (tok[u] < 0) continue;
      if (tok[u] != v) {
        if (first && begun) put8(mine, left, acc);
        else add_row(p, v, col, acc);
        first = false;
        v = tok[u];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = 0.0f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += value(e[u], j);
    }
  }
  const bool on = p.sort.start[v + 1] > to;        // the last one goes on behind the run
  if (first && begun) put8(mine, left, acc);
  else if (on) put8(mine + p.d, left, acc);
  else add_row(p, v, col, acc);
}
// A token that began in this run and goes on: the shares of the runs that follow, in their order.
__global__ __launch_bounds__(256) void k_embed_join(EmbedGrad p) {
  const int all = p.sort.start[p.vocab], col = ((int)blockIdx.y * 256 + (int)threadIdx.x) * 8, left = p.d - col;
  const int64_t from = (int64_t)blockIdx.x * p.run, to = from + p.run;
  if (to >= all || left <= 0) return;
  const int v = p.sort.token[to - 1];
  if (p.sort.start[v] < from || p.sort.start[v + 1] <= to) return;
  const int64_t last = (p.sort.start[v + 1] - 1) / p.run;
  float acc[8];
  load8<float>(p.part + ((int64_t)blockIdx.x * 2 + 1) * p.d + col, left, acc);
  constexpr int U = 4;
  for (int64_t r0 = blockIdx.x + 1; r0 <= last; r0 += U) {
    float e[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) load8<float>(p.part + (r0 + u) * 2 * p.d + col, r0 + u <= last ? left : 0, e[u]);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += e[u][j];
  }
  add_row(p, v, col, acc);
}

constexpr int64_t kTokensMax = 1 << 30, kVocabMax = 1 << 20, kWidthMax = 1 << 20;
int64_t align16(int64_t v) { return (v + 15) / 16 * 16; }
// positions of a run, and runs: at least 16 rows, at most 2 048 runs
int run_of(int64_t n) {
  const int64_t r = (n + 2047) / 2048;
  return (int)(r < 16 ? 16 : r);
}
int64_t runs_of(int64_t n) { return (n + run_of(n) - 1) / run_of(n); }

int check_embedding(const char* who, int64_t n, int64_t vocab, int64_t d, int dtype) {
  if (dtype != AE_F32 && dtype != AE_BF16) return fail(AE_EINVAL, "%s: bad dtype", who);
  if (n < 0 || n > kTokensMax) return fail(AE_EINVAL, "%s: tokens must be 0 .. 2^30", who);
  if (vocab < 1 || vocab > kVocabMax) return fail(AE_EINVAL, "%s: vocab must be 1 .. 2^20", who);
  if (d < 1 || d > kWidthMax) return fail(AE_EINVAL, "%s: d must be 1 .. 2^20", who);
  return AE_OK;
}
bool stride_ok(int64_t ld, int64_t d) { return ld >= d && ld < ((int64_t)1 << 40); }

template <typename T, int LANES, int U>
int launch_embedding(const void* table, int64_t ldt, int64_t vocab, int64_t d, const int* ids, int64_t n, float scale, void* out, int64_t ldo,
                     hipStream_t s) {
  const int64_t rows = 256 / LANES * U, want = (n + rows - 1) / rows, pieces = (d + LANES * 8 - 1) / (LANES * 8);
  const int64_t cols = pieces < 64 ? pieces : 64, most = launch_blocks(256) / cols;
  for (int64_t first = 0; first < want; first += most) {
    const int64_t left = want - first;
    hipLaunchKernelGGL((k_embedding<T, LANES, U>), dim3((unsigned)(left < most ? left : most), (unsigned)cols), dim3(256), 0, s, (const T*)table, ldt, vocab,
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
  *bytes = n == 0 ? 0 : 2 * align16(n * 4) + align16((vocab + 1) * 4) + runs_of(n) * 2 * d * 4;
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
    if (!workspace || ((uintptr_t)workspace & 15)) return fail(AE_EINVAL, "model_embedding_backward: workspace is null or not on a 16-byte border");
  } else if (accumulate) {
    return AE_OK;
  }
  char* ws = (char*)workspace;
  EmbedGrad p = {d_out, ldo, {}, (int)vocab, (int)d, run_of(n), runs_of(n), scale, d_table, ldt, accumulate ? 1 : 0, nullptr};
  const unsigned cols = (unsigned)((d + 2047) / 2048);
  const int64_t zeros = accumulate ? 0 : (vocab < 4096 ? vocab : 4096);
  if (n == 0) {
    p.runs = 0;
    hipLaunchKernelGGL((k_embed_sum<float>), dim3((unsigned)zeros, cols), dim3(256), 0, s, p);
    return launch_status("embedding_backward");
  }
  p.sort.place = (int*)ws;
  p.sort.token = (int*)(ws + align16(n * 4));
  p.sort.start = (int*)(ws + 2 * align16(n * 4));
  p.part = (float*)(ws + 2 * align16(n * 4) + align16((vocab + 1) * 4));
  const int range = (int)((vocab + 255) / 256);
  static_assert(kVocabMax / 256 <= SORT_RANGE, "a range's counters fit into LDS");
  hipLaunchKernelGGL(k_embed_sort, dim3((unsigned)((vocab + range - 1) / range)), dim3(SORT_NT), 0, s, ids, n, (int)vocab, range, p.sort);
  if (dtype == AE_BF16) hipLaunchKernelGGL((k_embed_sum<bf16_t>), dim3((unsigned)(p.runs + zeros), cols), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((k_embed_sum<float>), dim3((unsigned)(p.runs + zeros), cols), dim3(256), 0, s, p);
  if (p.runs > 1) hipLaunchKernelGGL(k_embed_join, dim3((unsigned)(p.runs - 1), cols), dim3(256), 0, s, p);
  return launch_status("embedding_backward");
}
