// ae_vocab.hip — passes over rows of logits: log probabilities of given tokens with entropy and top alternatives, and
// the distillation loss against a teacher's top logits with its gradient.
//   x_j = z_j / T,  lse = log sum_j exp x_j,  q_j = exp(x_j - lse).
// Everything is taken relative to the row's maximum m: e_j = exp((z_j - m) / T) and S = sum e_j, held as running values
// (when a larger logit comes along, what has been summed so far is scaled down), so that one read of the row gives them.
// A row is cut into `splits` pieces where there are few rows; a second launch joins the pieces.
#include <hip/hip_runtime.h>
#include <float.h>

#include "ae_device.h"
#include "ae_internal.h"

namespace ae {
namespace {

constexpr int NT = 512;                  // threads of a workgroup
constexpr int NW = NT / 64;
constexpr int CAND = 1024;               // candidates for the top list that LDS holds
constexpr int MAX_SPLITS = 64;           // a wavefront joins them, a piece per lane
constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// 16 bytes of elements at any alignment of the element's own
template <typename T>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[Store<T>::VEC]) {
  uint32_t w[4];
  __builtin_memcpy(w, p, 16);
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
  }
}
template <typename T>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[Store<T>::VEC]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = sizeof(T) == 2 ? pack_bf16(v[(2 * i) % Store<T>::VEC], v[(2 * i + 1) % Store<T>::VEC]) : __float_as_uint(v[i]);
  __builtin_memcpy(p, w, 16);
}
// the same for a vector that may cross the end: `left` elements are there, -infinity stands for the others
template <typename T>
__device__ __forceinline__ void load_vec_tail(const T* p, int left, float (&v)[Store<T>::VEC]) {
#pragma unroll
  for (int i = 0; i < Store<T>::VEC; ++i) v[i] = i < left ? Store<T>::ld(p + i) : -INFINITY;
}

// what the exponents of a row are taken relative to: the maximum, or 0 where there is nothing but -infinity
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.0f : m; }

// order of the logits as unsigned integers: NaN lowest, -0 equal to +0
__device__ __forceinline__ uint32_t order_key(float z) {
  if (z != z) return 0u;
  const uint32_t u = __float_as_uint(z + 0.0f);
  return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ uint64_t order_key(float z, int index) { return ((uint64_t)order_key(z) << 32) | (0xFFFFFFFFu - (uint32_t)index); }
__device__ __forceinline__ float key_logit(uint64_t k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return u == 0 ? __uint_as_float(0x7FC00000u) : __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ int key_index(uint64_t k) { return (int)(0xFFFFFFFFu - (uint32_t)k); }

// running statistics of a set of logits: maximum, sum of e_j, sum of e_j (z_j - m)
struct Stats {
  float m, s, a;
};
// the sum a after the maximum has grown by -d; f = the factor of the sums.  Nothing is left of what f = 0 scales (s d may overflow)
__device__ __forceinline__ float shifted(float a, float s, float d, float f) { return f == 0.0f ? 0.0f : f * (a + s * d); }
__device__ __forceinline__ Stats wave_join(Stats v, float c2) {
  Stats r;
  r.m = max_rows(max16(v.m));
  // the difference of -infinity (a side without entries) is cut off at the lowest number, so that 0 times it is 0
  const float d = fmaxf(v.m - reference(r.m), -FLT_MAX), f = fast_exp2(d * c2);
  r.s = sum_rows(sum16(f * v.s));
  r.a = sum_rows(sum16(shifted(v.a, v.s, d, f)));
  return r;
}
__device__ __forceinline__ Stats block_join(Stats v, float c2, Stats* sm /* NW */) {
  v = wave_join(v, c2);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
  __syncthreads();
  float m = sm[0].m;
#pragma unroll
  for (int i = 1; i < NW; ++i) m = fmaxf(m, sm[i].m);
  Stats r = {m, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    const float d = fmaxf(sm[i].m - reference(m), -FLT_MAX), f = fast_exp2(d * c2);
    r.s += f * sm[i].s;
    r.a += shifted(sm[i].a, sm[i].s, d, f);
  }
  return r;
}

constexpr int UNROLL = 4;                // vectors in flight

// Calls f(values of a vector, its first column) for the thread's vectors of columns [0, n) of a row piece, UNROLL at a time.
template <typename T, typename F>
__device__ __forceinline__ void for_vectors(const T* p, int n, F f) {
  constexpr int V = Store<T>::VEC;
  constexpr int STEP = NT * V;
  int base = 0;
  for (; base + UNROLL * STEP <= n; base += UNROLL * STEP) {
    float v[UNROLL][V];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) load_vec<T>(p + base + u * STEP + threadIdx.x * V, v[u]);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) f(v[u], base + u * STEP + (int)threadIdx.x * V, V);
  }
  for (int c = base + (int)threadIdx.x * V; c < n; c += STEP) {
    float v[V];
    if (c + V <= n) load_vec<T>(p + c, v);
    else load_vec_tail<T>(p + c, n - c, v);
    f(v, c, n - c < V ? n - c : V);
  }
}

// ---- top list ------------------------------------------------------------------------------------------------------
constexpr int GROUPS = 8;                // parts of a thread's share whose maxima are kept
struct TopShared {
  uint64_t cand[CAND];
  uint32_t tmax[NT];
  uint16_t gmax[GROUPS][NT];             // upper halves of the keys of the parts' maxima, 0: no elements
  uint32_t pairs[CAND];
  int hist[256];
  int sums[NW];
  int count, n_pairs, digit, before;
  uint32_t threshold;
};

// adds the keys of the lanes that want it; lanes of a wavefront take their places with one atomic
__device__ __forceinline__ void push(TopShared& sh, bool want, uint64_t key) {
  const uint64_t m = __ballot(want);
  if (!want) return;
  const int lane = threadIdx.x & 63, first = __ffsll((unsigned long long)m) - 1;
  int at = 0;
  if (lane == first) at = atomicAdd(&sh.count, __popcll(m));
  at = __shfl(at, first, 64) + __popcll(m & ((1ull << lane) - 1));
  if (at < CAND) sh.cand[at] = key;
}

// The k-th largest of the threads' maxima, which is at most the k-th largest key, since those maxima are k keys
// themselves, and not much less, since the largest keys lie in different shares for the most part.  The leading bits will
// do: all that a positive bfloat16 has, nine of a binary32 number's fraction.
constexpr int BOUND_BITS = 18;
// by the first wavefront: the largest number that k of the maxima reach, its bits from `high` to `low` found, those above given
__device__ uint32_t bound_bits(const TopShared& sh, int k, uint32_t bound, int high, int low) {
  const int lane = threadIdx.x & 63;
  uint32_t v[NW];
#pragma unroll
  for (int i = 0; i < NW; ++i) v[i] = sh.tmax[lane + 64 * i];
  for (int bit = high; bit >= low; --bit) {
    const uint32_t c = bound | (1u << bit);
    int n = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) n += __popcll(__ballot(v[i] >= c));
    if (n >= k) bound = c;
    if (n == k) break;
  }
  return bound;
}
__device__ uint32_t top_bound(TopShared& sh, int k, uint32_t tmax) {
  const int t = threadIdx.x;
  __syncthreads();
  sh.tmax[t] = tmax;
  if (t == 0) sh.count = sh.n_pairs = 0;
  __syncthreads();
  if (t < 64) {
    const uint32_t bound = bound_bits(sh, k, 0, 31, 32 - BOUND_BITS);
    if (t == 0) sh.threshold = bound;
  }
  __syncthreads();
  return sh.threshold;
}

// Where more keys reach the bound than LDS holds (long runs of equal logits, many large ones in one share): the exact value
// of the k-th largest, by its digits if the bound is not it already; then what is larger, in any order, and of what
// is equal the first ones in the order of the index.  There are enough of them, since k maxima of shares, which are keys, reach
// the bound.  A source gives its keys in steps of W to a thread, in that order.
template <typename Src, typename F>
__device__ __forceinline__ void for_steps(const Src& src, F f) {          // f(keys, how many) for the thread's steps, four loads in flight
  constexpr int W = Src::W;
  for (int s = 0; s < src.steps(); s += 4) {
    uint64_t key[4][W];
    int n[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) n[u] = src.load(s + u, key[u]);
#pragma unroll
    for (int u = 0; u < 4; ++u) f(key[u], n[u]);
  }
}
template <typename Src>
__device__ void top_exact(TopShared& sh, int k, uint32_t bound, const Src& src) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  constexpr int W = Src::W;
  uint64_t key[W];
  __syncthreads();
  if (t < 64) {                          // the bound to its last bit: one that equals the k-th largest saves its search
    const uint32_t b = bound_bits(sh, k, bound, 31 - BOUND_BITS, 0);
    if (t == 0) sh.threshold = b;
  }
  if (t == 0) sh.count = 0;
  __syncthreads();
  bound = sh.threshold;
  int more = 0;
  for_steps(src, [&](const uint64_t (&v)[W], int n) {
#pragma unroll
    for (int i = 0; i < W; ++i) more += i < n && (uint32_t)(v[i] >> 32) > bound ? 1 : 0;
  });
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) more += __shfl_xor(more, off, 64);
  if (lane == 0) atomicAdd(&sh.count, more);
  __syncthreads();
  uint32_t value = bound;
  int larger = sh.count;
  if (larger >= k) {
    value = 0;
    larger = 0;                          // keys known to be larger than every one with the prefix `value`
    for (int d = 3; d >= 0; --d) {
      __syncthreads();
      if (t < 256) sh.hist[t] = 0;
      __syncthreads();
      for_steps(src, [&](const uint64_t (&keys)[W], int n) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const uint32_t v = (uint32_t)(keys[i] >> 32);
          if (i < n && (d == 3 || (v >> (8 * d + 8)) == (value >> (8 * d + 8)))) {
            const int digit = (int)(v >> (8 * d)) & 255;
            const int first = __builtin_amdgcn_readfirstlane(digit);
            const uint64_t same = __ballot(digit == first);        // lanes of equal digits add once, not one after the other
            if (digit != first) atomicAdd(&sh.hist[digit], 1);
            else if (lane == __ffsll((unsigned long long)same) - 1) atomicAdd(&sh.hist[digit], __popcll(same));
          }
        }
      });
      __syncthreads();
      if (t == 0) {
        int above = larger, at = 255;
        while (at > 0 && above + sh.hist[at] < k) above += sh.hist[at--];
        sh.digit = at;
        sh.before = above;
      }
      __syncthreads();
      value |= (uint32_t)sh.digit << (8 * d);
      larger = sh.before;
    }
  }
  __syncthreads();
  if (t == 0) sh.count = 0;
  __syncthreads();
  if (larger > 0) {
    for_steps(src, [&](const uint64_t (&v)[W], int n) {
#pragma unroll
      for (int i = 0; i < W; ++i) push(sh, i < n && (uint32_t)(v[i] >> 32) > value, v[i]);
    });
  }
  __syncthreads();
  int have = larger;                     // fewer than k <= CAND
  for (int s = 0; s < src.steps() && have < k; ++s) {
    const int n = src.load(s, key);
    int mine = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) mine += i < n && (uint32_t)(key[i] >> 32) == value ? 1 : 0;
    int upto = mine;                     // in the lanes up to this one
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int o = __shfl_up(upto, off, 64);
      if (lane >= off) upto += o;
    }
    if (lane == 63) sh.sums[wave] = upto;
    __syncthreads();
    int at = have + upto - mine, total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      if (w < wave) at += sh.sums[w];
      total += sh.sums[w];
    }
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (i < n && (uint32_t)(key[i] >> 32) == value) {
        if (at < k) sh.cand[at] = key[i];
        ++at;
      }
    have += total;
    __syncthreads();
  }
  if (t == 0) sh.count = have < k ? have : k;
  __syncthreads();
}

// Calls f(rank, key) for the k largest candidates; keys differ, so a key's rank is the number of larger ones.  A few lanes
// share a candidate while there are more lanes than candidates.
template <typename F>
__device__ void top_ranked(TopShared& sh, int k, F f) {
  const int count = sh.count, t = threadIdx.x;
  const int lanes = count <= NT / 8 ? 8 : count <= NT / 4 ? 4 : count <= NT / 2 ? 2 : 1;
  const int step = 4 * lanes, whole = (count + step - 1) / step * step;
  for (int i = count + t; i < whole; i += NT) sh.cand[i] = 0;          // room for them: CAND is a multiple of 32
  __syncthreads();
  for (int i0 = 0; i0 < count; i0 += NT / lanes) {
    const int i = i0 + t / lanes;
    const uint64_t key = i < count ? sh.cand[i] : ~0ull;
    int rank = 0;
    for (int j = 4 * (t & (lanes - 1)); j < whole; j += step) {
#pragma unroll
      for (int u = 0; u < 4; ++u) rank += sh.cand[j + u] > key ? 1 : 0;
    }
    for (int off = 1; off < lanes; off <<= 1) rank += __shfl_xor(rank, off, 64);
    if (i < count && rank < k && (t & (lanes - 1)) == 0) f(rank, key);
  }
}

// the logits of a row piece as a source of keys
template <typename T>
struct RowKeys {
  static constexpr int W = Store<T>::VEC;
  const T* z;
  int n, c0;
  __device__ int steps() const { return (n + NT * W - 1) / (NT * W); }
  __device__ int load(int s, uint64_t (&key)[W]) const {
    const int c = (s * NT + (int)threadIdx.x) * W, left = n - c;
    float v[W];
    if (left >= W) load_vec<T>(z + c, v);
    else load_vec_tail<T>(z + c, left, v);
#pragma unroll
    for (int i = 0; i < W; ++i) key[i] = order_key(v[i], c0 + c + i);
    return left < 0 ? 0 : left < W ? left : W;
  }
};
// the lists of a row's pieces, each in falling order
struct ListKeys {
  static constexpr int W = 1;
  const uint64_t* keys;
  int n, lists, len;
  // a thread's share: one list, every (NT / lists)-th rank of it, so that the largest keys are maxima of different shares
  __device__ int rounds() const { return (len + NT / lists - 1) / (NT / lists); }
  __device__ uint64_t share(int j) const {
    const int ranks = NT / lists, t = threadIdx.x, list = t % lists, rank = t / lists + j * ranks;
    return t < ranks * lists && rank < len ? keys[list * len + rank] : 0;
  }
  __device__ int steps() const { return (n + NT - 1) / NT; }
  __device__ int load(int s, uint64_t (&key)[1]) const {
    const int i = s * NT + (int)threadIdx.x;
    key[0] = i < n ? keys[i] : 0;
    return key[0] != 0 ? 1 : 0;
  }
};

struct LogprobArgs {
  const void* logits;
  int64_t row0, rows, ld;                // the launch's first row
  int vocab, splits, chunk;              // columns of a piece
  float temp;
  const int* tokens;
  int n_tokens, top_k;
  float *logprob, *entropy, *lse;
  int* top_id;
  float *top_logit, *top_logprob;
  Stats* part;                           // [rows][splits]
  uint64_t* part_top;                    // [rows][splits][top_k]
};

// what a row's statistics give
struct RowLog {
  float m, log_s;
  bool empty;
};
__device__ __forceinline__ RowLog row_log(const Stats& st) { return {st.m, st.s == 0.0f ? 0.0f : logf(st.s), st.s == 0.0f}; }
__device__ __forceinline__ float log_prob(float z, const RowLog& r, float temp) { return r.empty ? -INFINITY : (z - r.m) / temp - r.log_s; }

template <typename T>
__device__ void write_row(const LogprobArgs& p, int64_t row, const Stats& st) {
  const RowLog r = row_log(st);
  const T* z = (const T*)p.logits + row * p.ld;
  if (threadIdx.x == 0) {
    if (p.lse) p.lse[row] = r.empty ? -INFINITY : st.m / p.temp + r.log_s;
    if (p.entropy) p.entropy[row] = r.empty ? 0.0f : r.log_s - (st.a / p.temp) / st.s;
  }
  for (int i = threadIdx.x; i < p.n_tokens; i += NT) {
    const int id = p.tokens[row * p.n_tokens + i];
    p.logprob[row * p.n_tokens + i] = id >= 0 && id < p.vocab ? log_prob(Store<T>::ld(z + id), r, p.temp) : 0.0f;
  }
}
__device__ __forceinline__ void write_top(const LogprobArgs& p, int64_t row, const RowLog& r, int rank, uint64_t key) {
  const float z = key_logit(key);
  const int64_t at = row * p.top_k + rank;
  if (p.top_id) p.top_id[at] = key_index(key);
  if (p.top_logit) p.top_logit[at] = z;
  if (p.top_logprob) p.top_logprob[at] = log_prob(z, r, p.temp);
}

// One workgroup per row piece; with one piece per row it writes the results, otherwise what k_logprob_join needs.  Bound by
// reading the logits: 2 048 x 131 072 in bfloat16 93 us without entropy and list, 5.8 TB/s, 99 with entropy.  A list costs
// what its threads do while a row's loads have ended and the next row's have not begun: 116 us with 64 entries.  Three
// workgroups to a compute unit, so that others load meanwhile: 80 registers (4 096 x 32 000 with 64 entries 93 us, two 118).
template <typename T, bool TOP, bool ENT>
__global__ __launch_bounds__(NT, 6) void k_logprob(LogprobArgs p) {
  constexpr int V = Store<T>::VEC, STEP = NT * V;
  __shared__ Stats sm[NW];
  __shared__ TopShared sh;
  const unsigned at_row = blockIdx.x / p.splits;
  const int64_t row = p.row0 + at_row;
  const int split = (int)(blockIdx.x - at_row * p.splits), t = threadIdx.x;
  const int c0 = split * p.chunk;
  const int n = p.vocab - c0 < p.chunk ? p.vocab - c0 : p.chunk;
  const T* z = (const T*)p.logits + row * p.ld + c0;
  const float c2 = kLog2e / p.temp;
  const int rounds = (n + UNROLL * STEP - 1) / (UNROLL * STEP), per = (rounds + GROUPS - 1) / GROUPS;      // rounds of loads, and to a group
  Stats st = {-INFINITY, 0.0f, 0.0f};
  float gm = -INFINITY;
  for (int r = 0; r < rounds; ++r) {
    const int base = r * UNROLL * STEP + t * V;
    float v[UNROLL][V];
    if ((r + 1) * UNROLL * STEP <= n) {
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) load_vec<T>(z + base + u * STEP, v[u]);
    } else {
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int c = base + u * STEP;
        if (c + V <= n) load_vec<T>(z + c, v[u]);
        else load_vec_tail<T>(z + c, n - c, v[u]);
      }
    }
    float cm = v[0][0];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
#pragma unroll
      for (int i = 0; i < V; ++i) cm = fmaxf(cm, v[u][i]);
    if (cm > st.m) {
      const float d = fmaxf(st.m - cm, -FLT_MAX), f = fast_exp2(d * c2);
      st.a = shifted(st.a, st.s, d, f);
      st.s *= f;
      st.m = cm;
    }
    const float ref = reference(st.m);
    float a = 0.0f;
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = v[u][i] - ref, e = fast_exp2(d * c2);
        st.s += e;
        if constexpr (ENT) a = fmaf(e, d, a);
      }
    if constexpr (ENT) {
      if (a != a) {                      // 0 times -infinity among them: those have no part in the sum
        a = 0.0f;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float d = v[u][i] - ref, e = fast_exp2(d * c2);
            a = fmaf(e, fmaxf(d, -FLT_MAX), a);
          }
      }
      st.a += a;
    }
    if constexpr (TOP) {
      gm = fmaxf(gm, cm);
      if (r % per == per - 1 || r == rounds - 1) {
        sh.gmax[r / per][t] = r / per * per * UNROLL * STEP + t * V < n ? (uint16_t)(order_key(gm) >> 16) : (uint16_t)0;
        gm = -INFINITY;
      }
    }
  }
  // the share's largest key; -infinity is none of its keys for sure if there are NaN, so for the bound such a share has the lowest
  const uint32_t tmax = t * V < n ? order_key(st.m) : 0u, sure = st.m == -INFINITY && st.s != st.s ? 0u : tmax;
  const Stats all = block_join(st, c2, sm);
  if (p.splits > 1 && t == 0) p.part[row * p.splits + split] = all;
  if constexpr (TOP) {
    const int k = p.top_k < n ? p.top_k : n;
    const uint32_t bound = top_bound(sh, k, sure);
    // the parts of shares that reach the bound, then their vectors, one to a thread
    if (tmax >= bound) {
      for (int g = 0; g * per < rounds; ++g)
        if (sh.gmax[g][t] >= (bound >> 16)) {
          const int at = atomicAdd(&sh.n_pairs, 1);
          if (at < CAND) sh.pairs[at] = (uint32_t)(g << 16 | t);
        }
    }
    __syncthreads();
    const int pairs = sh.n_pairs, width = per * UNROLL;
    if (pairs <= CAND) {
      for (int i = t; i < pairs * width; i += NT) {
        const int pair = i / width;
        const uint32_t g = sh.pairs[pair] >> 16, owner = sh.pairs[pair] & 0xFFFF;
        const int c = ((int)g * width + (i - pair * width)) * STEP + (int)owner * V, left = n - c;
        if (left <= 0) continue;
        float v[V];
        if (left >= V) load_vec<T>(z + c, v);
        else load_vec_tail<T>(z + c, left, v);
#pragma unroll
        for (int j = 0; j < V; ++j) push(sh, j < left && order_key(v[j]) >= bound, order_key(v[j], c0 + c + j));
      }
    }
    __syncthreads();
    const int found = sh.count;
    if (pairs > CAND || found > CAND) top_exact(sh, k, bound, RowKeys<T>{z, n, c0});
    if (p.splits == 1) {
      const RowLog r = row_log(all);
      top_ranked(sh, k, [&](int rank, uint64_t key) { write_top(p, row, r, rank, key); });
    } else {
      uint64_t* out = p.part_top + (row * p.splits + split) * p.top_k;
      top_ranked(sh, k, [&](int rank, uint64_t key) { out[rank] = key; });
      for (int i = k + t; i < p.top_k; i += NT) out[i] = 0;
    }
  }
  if (p.splits == 1) write_row<T>(p, row, all);
}

// One workgroup per row: joins its pieces.
template <typename T, bool TOP>
__global__ __launch_bounds__(NT) void k_logprob_join(LogprobArgs p) {
  __shared__ Stats sm;
  __shared__ TopShared sh;
  const int64_t row = blockIdx.x;
  const float c2 = kLog2e / p.temp;
  const ListKeys src = {p.part_top + row * p.splits * p.top_k, p.splits * p.top_k, p.splits, p.top_k};
  uint32_t tmax = 0;
  if constexpr (TOP) {
    for (int j = 0; j < src.rounds(); ++j) {
      const uint32_t h = (uint32_t)(src.share(j) >> 32);
      tmax = h > tmax ? h : tmax;
    }
  }
  if (threadIdx.x < 64) {
    Stats st = {-INFINITY, 0.0f, 0.0f};
    if ((int)threadIdx.x < p.splits) st = p.part[row * p.splits + threadIdx.x];
    st = wave_join(st, c2);
    if (threadIdx.x == 0) sm = st;
  }
  __syncthreads();
  const Stats all = sm;
  if constexpr (TOP) {
    const uint32_t bound = top_bound(sh, p.top_k, tmax);
    if (tmax >= bound) {
      for (int j = 0; j < src.rounds(); ++j) {
        const uint64_t key = src.share(j);
        push(sh, key != 0 && (uint32_t)(key >> 32) >= bound, key);
      }
    }
    __syncthreads();
    const int found = sh.count;
    if (found > CAND) top_exact(sh, p.top_k, bound, src);
    const RowLog r = row_log(all);
    top_ranked(sh, p.top_k, [&](int rank, uint64_t k) { write_top(p, row, r, rank, k); });
  }
  write_row<T>(p, row, all);
}

// ---- distillation --------------------------------------------------------------------------------------------------
// Statistics of a row piece.  What lies outside the teacher's list has a maximum of its own, so that its sum, by which the
// teacher's remaining mass is divided, neither vanishes nor loses bits where the list lies far above it.
struct DistillPart {
  float m_out, s_out, m_in, s_in;        // outside and inside the list: maximum, and sum of exp((z_j - that maximum) / T)
  double p, l;                           // sums over the list's entries in the piece: p_i, and p_i (log p_i - (z_i - m) / T), m = the larger maximum
};
__device__ __forceinline__ float maximum(const DistillPart& st) { return fmaxf(st.m_out, st.m_in); }
// a logit joins a sum with its running maximum
__device__ __forceinline__ void add_logit(float& m, float& s, float z, float c2) {
  if (z > m) {
    s *= fast_exp2((m - z) * c2);
    m = z;
  }
  s += fast_exp2((z - reference(m)) * c2);
}
// Other tokens with all their logits more than 708 T below the row's maximum (their probabilities are no normal binary64
// numbers any more; masks like -10^4) are ones that the student does not have.
constexpr double kFarthest = 708.0;
struct DistillArgs {
  const void* logits;
  int64_t row0, rows, ld;                // the launch's first row
  int vocab, splits, chunk;
  float temp;
  const int* top_id;
  const float* top_logit;
  int top_k;
  const float *teacher_lse, *weight;
  float *loss_rows, *loss;               // loss: null where another launch adds up the rows
  void* d_logits;
  int64_t ldd;
  DistillPart* part;                     // [rows][splits]
};

// exp(x) to binary32 precision of an x in binary64 (whose binary32 rounding would cost |x| 2^-24): whole powers of two taken
// out.  The teacher's binary32 numbers define its probabilities no better.
__device__ __forceinline__ double exp_of(double x) {
  const double y = x * 1.4426950408889634074, i = rint(y);
  const float f = (float)(y - i);                // |f| <= 1/2; NaN for infinities
  const float e = fast_exp2(f == f ? f : x < 0.0 ? -INFINITY : (float)x);
  return (double)ldexpf(e, (int)fmaxf(fminf((float)i, 300.0f), -300.0f));
}

// log(x) of an x in binary64, likewise: off by binary32 roundings of a number below 0.35, not of the logarithm's size
__device__ __forceinline__ double log_of(double x) {
  int i;
  const double h = frexp(x, &i);                 // in [1/2, 1)
  const bool low = h < 0.70710678118654752440;
  return (double)logf((float)(low ? 2.0 * h : h)) + (double)(low ? i - 1 : i) * 0.69314718055994530942;
}

// the logarithm of the sum that the teacher's probabilities are divided by
template <int NTH>
__device__ double list_norm(const DistillArgs& p, int64_t row, double* sm /* NTH / 64 + 1 */) {
  if (p.teacher_lse) return (double)p.teacher_lse[row];
  const int* id = p.top_id + row * p.top_k;
  const float* t = p.top_logit + row * p.top_k;
  float m = -INFINITY;
  for (int i = threadIdx.x; i < p.top_k; i += NTH)
    if (id[i] >= 0 && id[i] < p.vocab) m = fmaxf(m, t[i]);
  m = max_rows(max16(m));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = (double)m;
  __syncthreads();
  double dm = sm[0];
  for (int i = 1; i < NTH / 64; ++i) dm = sm[i] > dm ? sm[i] : dm;
  if (dm == -INFINITY) dm = 0.0;
  double s = 0.0;
  for (int i = threadIdx.x; i < p.top_k; i += NTH)
    if (id[i] >= 0 && id[i] < p.vocab) s += exp_of(((double)t[i] - dm) / (double)p.temp);
  __syncthreads();
  s = block_sum<NTH>(s, sm);
  return dm / (double)p.temp + log_of(s);
}
// a norm of -infinity: a teacher without any outcome (-infinity less -infinity would be NaN)
__device__ __forceinline__ double list_log_p(const DistillArgs& p, int64_t at, double norm) {
  return norm == -INFINITY ? -INFINITY : (double)p.top_logit[at] / (double)p.temp - norm;
}
__device__ __forceinline__ bool has_rest(const DistillArgs& p, double norm) { return p.teacher_lse && norm != -INFINITY; }

// marks the list's tokens that lie in columns [c0, c0 + n): a bit for each column
template <int NTH>
__device__ void mark_list(const DistillArgs& p, int64_t row, int c0, int n, uint32_t* bits) {
  for (int i = threadIdx.x; i < (n + 31) / 32; i += NTH) bits[i] = 0u;
  __syncthreads();
  for (int i = threadIdx.x; i < p.top_k; i += NTH) {
    const int id = p.top_id[row * p.top_k + i];
    if (id >= c0 && id < c0 + n) atomicOr(&bits[(id - c0) >> 5], 1u << ((id - c0) & 31));
  }
  __syncthreads();
}
template <int V> __device__ __forceinline__ uint32_t marks_of(const uint32_t* bits, int c) { return (bits[c >> 5] >> (c & 31)) & ((1u << V) - 1u); }

template <typename T>
__device__ DistillPart piece_stats(const DistillArgs& p, int64_t row, int c0, int n, const uint32_t* bits, double norm, float c2,
                                   float (*smf)[NW] /* 4 */, double (*smd)[NW] /* 2 */) {
  constexpr int V = Store<T>::VEC;
  const T* z = (const T*)p.logits + row * p.ld + c0;
  float m_out = -INFINITY, s_out = 0.0f, m_in = -INFINITY, s_in = 0.0f;
  // the list: its part of the sum, and the loss's terms, relative to the thread's maximum as long as the row's is not known
  const double inv_t = 1.0 / (double)p.temp;
  double sp = 0.0, sl = 0.0;
  for (int i = threadIdx.x; i < p.top_k; i += NT) {
    const int id = p.top_id[row * p.top_k + i];
    if (id < c0 || id >= c0 + n) continue;
    const float z_i = Store<T>::ld(z + id - c0);
    const double before = (double)reference(m_in);
    add_logit(m_in, s_in, z_i, c2);
    const double ref_t = (double)reference(m_in);
    if (sp != 0.0) sl += sp * (ref_t - before) * inv_t;
    const double lp = list_log_p(p, row * p.top_k + i, norm), pi = exp_of(lp);
    sp += pi;
    if (pi != 0.0) sl += pi * (lp - ((double)z_i - ref_t) * inv_t);
  }
  for_vectors<T>(z, n, [&](const float (&all)[V], int c, int) {
    float v[V];
    const uint32_t mk = marks_of<V>(bits, c);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = all[i];
    if (mk) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = mk >> i & 1 ? -INFINITY : v[i];
    }
    float cm = v[0];
#pragma unroll
    for (int i = 1; i < V; ++i) cm = fmaxf(cm, v[i]);
    if (cm > m_out) {
      s_out *= fast_exp2((m_out - cm) * c2);
      m_out = cm;
    }
    const float ref = reference(m_out);
#pragma unroll
    for (int i = 0; i < V; ++i) s_out += fast_exp2((v[i] - ref) * c2);
  });
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  float w_out = max_rows(max16(m_out)), w_in = max_rows(max16(m_in));
  s_out = sum_rows(sum16(fast_exp2((m_out - reference(w_out)) * c2) * s_out));
  s_in = sum_rows(sum16(fast_exp2((m_in - reference(w_in)) * c2) * s_in));
  __syncthreads();
  if (lane == 0) {
    smf[0][wave] = w_out;
    smf[1][wave] = s_out;
    smf[2][wave] = w_in;
    smf[3][wave] = s_in;
  }
  __syncthreads();
  const int i8 = lane & 15;
  const bool there = i8 < NW;
  const float o_i = there ? smf[0][i8] : -INFINITY, i_i = there ? smf[2][i8] : -INFINITY;
  DistillPart st = {max16(o_i), 0.0f, max16(i_i), 0.0f, 0.0, 0.0};
  st.s_out = sum16(there ? fast_exp2((o_i - reference(st.m_out)) * c2) * smf[1][i8] : 0.0f);
  st.s_in = sum16(there ? fast_exp2((i_i - reference(st.m_in)) * c2) * smf[3][i8] : 0.0f);
  if (sp != 0.0) sl -= sp * ((double)reference(m_in) - (double)reference(maximum(st))) * inv_t;
  if (p.top_k > 64 || wave == 0) {               // whose lanes have entries
    sp = wave_sum(sp);
    sl = wave_sum(sl);
  }
  if (lane == 0) {
    smd[0][wave] = sp;
    smd[1][wave] = sl;
  }
  __syncthreads();
  st.p = sum_of<NW>(smd[0]);
  st.l = sum_of<NW>(smd[1]);
  return st;
}

// What the statistics of a whole row give.  The loss, with its logarithms in binary64, is for one wavefront to compute.
struct RowGrad {
  float ref, ref_out, s_all;             // what exponents are relative to, outside the list; sum of e_j relative to ref
  float f_out;                           // the gradient outside the list is f_out exp((z_j - ref_out) / T)
  double mass, rest, scale;              // P, p_r, w / T
  double s_sum, gap;                     // the sum once more; (ref - ref_out) / T
  bool empty;
};
__device__ __forceinline__ RowGrad row_grad(const DistillArgs& p, const DistillPart& st, float w, float c2, bool tail) {
  RowGrad r;
  const float m = maximum(st);
  r.ref = reference(m);
  r.ref_out = reference(st.m_out);
  const float a = fast_exp2((st.m_out - r.ref) * c2), b = fast_exp2((st.m_in - r.ref) * c2);
  r.s_all = a * st.s_out + b * st.s_in;
  r.s_sum = (double)a * (double)st.s_out + (double)b * (double)st.s_in;
  r.empty = r.s_all == 0.0f;
  r.rest = tail ? 1.0 - st.p : 0.0;
  if (!(r.rest > 0.0) && r.rest == r.rest) r.rest = 0.0;
  r.gap = ((double)r.ref - (double)r.ref_out) / (double)p.temp;
  if (st.s_out == 0.0f || r.gap > kFarthest) r.rest = 0.0;
  r.mass = st.p + r.rest;
  const float scale = w / p.temp;
  r.scale = (double)scale;
  // P - p_r / q_r, over the sum; of each, a is left where the exponents are relative to the outside's maximum
  const float outside = r.rest != 0.0 ? (float)(r.mass * (double)a - r.rest * (double)(r.s_all / st.s_out)) : (float)r.mass * a;
  r.f_out = r.empty ? 0.0f : outside * scale / r.s_all;
  return r;
}
// off: the sums are 2^off times those of exponents relative to the maximum
__device__ float row_loss(const DistillPart& st, const RowGrad& r, float off = 0.0f) {
  if (r.empty) return 0.0f;
  if (r.s_all != r.s_all) return r.s_all;        // a NaN or +infinity in the row, also where the teacher gives no probability to anything
  double loss = st.l + (st.p != 0.0 ? st.p * (log_of(r.s_sum) - (double)off * 0.69314718055994530942) : 0.0);
  if (r.rest != 0.0) loss += r.rest * (log_of(r.rest * r.s_sum / (double)st.s_out) + r.gap);
  return (float)loss;
}
// stores the gradient of a vector's columns: those of the list are left as they are, since g may be z, which they still need
template <typename T>
__device__ __forceinline__ void store_outside(T* g, const float (&o)[Store<T>::VEC], uint32_t marks, int len) {
  if (marks == 0 && len >= Store<T>::VEC) {
    store_vec<T>(g, o);
  } else {
#pragma unroll
    for (int i = 0; i < Store<T>::VEC; ++i)
      if (i < len && !(marks >> i & 1)) Store<T>::st(g + i, o[i]);
  }
}
// the gradient of the list's entries in columns [c0, c0 + n)
template <typename T, int NTH>
__device__ void list_gradient(const DistillArgs& p, int64_t row, int c0, int n, double norm, float c2, const RowGrad& r) {
  const T* z = (const T*)p.logits + row * p.ld;
  T* g = (T*)p.d_logits + row * p.ldd;
  for (int i = threadIdx.x; i < p.top_k; i += NTH) {
    const int id = p.top_id[row * p.top_k + i];
    if (id < c0 || id >= c0 + n) continue;
    const double q = (double)(fast_exp2((Store<T>::ld(z + id) - r.ref) * c2) / r.s_all);
    const double pi = exp_of(list_log_p(p, row * p.top_k + i, norm));
    Store<T>::st(g + id, r.empty ? 0.0f : (float)((r.mass * q - pi) * r.scale));
  }
}

// The gradient of columns [c0, c0 + n) from the statistics of the whole row.
template <typename T>
__device__ void piece_gradient(const DistillArgs& p, int64_t row, int c0, int n, const uint32_t* bits, double norm, float c2, const RowGrad& r) {
  constexpr int V = Store<T>::VEC;
  const T* z = (const T*)p.logits + row * p.ld + c0;
  T* g = (T*)p.d_logits + row * p.ldd + c0;
  for_vectors<T>(z, n, [&](const float (&v)[V], int c, int len) {
    float o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = r.f_out * fast_exp2((v[i] - r.ref_out) * c2);
    store_outside<T>(g + c, o, marks_of<V>(bits, c), len);
  });
  list_gradient<T, NT>(p, row, c0, n, norm, c2, r);
}

// The statistics of a row from those of its pieces, one to a lane; in every lane.
__device__ DistillPart joined(const DistillArgs& p, int64_t row, float c2) {
  const int lane = threadIdx.x & 63;
  DistillPart v = {-INFINITY, 0.0f, -INFINITY, 0.0f, 0.0, 0.0};
  if (lane < p.splits) v = p.part[row * p.splits + lane];
  DistillPart st = {max_rows(max16(v.m_out)), 0.0f, max_rows(max16(v.m_in)), 0.0f, 0.0, 0.0};
  st.s_out = sum_rows(sum16(fast_exp2((v.m_out - reference(st.m_out)) * c2) * v.s_out));
  st.s_in = sum_rows(sum16(fast_exp2((v.m_in - reference(st.m_in)) * c2) * v.s_in));
  // the piece's own maximum in the terms of l becomes the row's
  if (v.p != 0.0) v.l -= v.p * ((double)reference(maximum(v)) - (double)reference(maximum(st))) / (double)p.temp;
  st.p = wave_sum(v.p);
  st.l = wave_sum(v.l);
  return st;
}

template <typename T>
__device__ void piece_zero(const DistillArgs& p, int64_t row, int c0, int n) {
  constexpr int V = Store<T>::VEC;
  T* g = (T*)p.d_logits + row * p.ldd + c0;
  const float o[V] = {};
  for (int c = threadIdx.x * V; c < n; c += NT * V) {
    if (c + V <= n) store_vec<T>(g + c, o);
    else
      for (int i = c; i < n; ++i) Store<T>::st(g + i, 0.0f);
  }
}

// The weighted sum of the losses of a few rows in pieces, by one workgroup: it forms every row's loss for itself.
constexpr int64_t kTotalHere = 2 * NW;           // rows: two to a wavefront
__device__ void total_of_pieces(const DistillArgs& p, float c2, double* sm /* NW + 1 */) {
  double acc = 0.0;
  for (int64_t row = threadIdx.x >> 6; row < p.rows; row += NW) {
    const float w = p.weight ? p.weight[row] : 1.0f;
    if (w == 0.0f) continue;
    const DistillPart st = joined(p, row, c2);
    if ((threadIdx.x & 63) == 0) acc += (double)w * (double)row_loss(st, row_grad(p, st, w, c2, has_rest(p, p.teacher_lse ? (double)p.teacher_lse[row] : 0.0)));
  }
  acc = block_sum<NT>(acc, sm);
  if (threadIdx.x == 0) *p.loss = (float)acc;
}

// Rows that the registers do not hold, or without a gradient, or with long lists: a row is read once for its statistics and
// again for its gradient (1 024 x 131 072 in binary32 332 us, 3.2 TB/s of one reading and one writing; loss alone 104, 5.2).
// MODE 0: statistics and gradient of whole rows; 1: statistics of row pieces; 2: gradient of row pieces from joined statistics
template <typename T, int MODE>
__global__ __launch_bounds__(NT) void k_distill(DistillArgs p) {
  extern __shared__ uint32_t bits[];
  __shared__ float smf[4][NW];
  __shared__ double smp[2][NW], smd[NW + 1];
  const unsigned at_row = blockIdx.x / p.splits;
  const int64_t row = p.row0 + at_row;
  const int split = (int)(blockIdx.x - at_row * p.splits);
  const int c0 = split * p.chunk;
  const int n = p.vocab - c0 < p.chunk ? p.vocab - c0 : p.chunk;
  const float w = p.weight ? p.weight[row] : 1.0f;
  const float c2 = kLog2e / p.temp;
  if (w == 0.0f) {
    if (MODE != 1) {
      if (threadIdx.x == 0 && split == 0) p.loss_rows[row] = 0.0f;
      if (MODE == 2 && p.loss && blockIdx.x == gridDim.x - 1) total_of_pieces(p, c2, smd);
      if (p.d_logits) piece_zero<T>(p, row, c0, n);
    }
    return;
  }
  mark_list<NT>(p, row, c0, n, bits);
  const double norm = list_norm<NT>(p, row, smd);
  DistillPart st;
  if constexpr (MODE != 2) {
    st = piece_stats<T>(p, row, c0, n, bits, norm, c2, smf, smp);
    if constexpr (MODE == 1) {
      if (threadIdx.x == 0) p.part[row * p.splits + split] = st;
      return;
    }
  } else {
    st = joined(p, row, c2);
  }
  const RowGrad r = row_grad(p, st, w, c2, has_rest(p, norm));
  if (threadIdx.x == 0 && split == 0) p.loss_rows[row] = row_loss(st, r);
  if (MODE == 2 && p.loss && blockIdx.x == gridDim.x - 1) total_of_pieces(p, c2, smd);
  if (p.d_logits) piece_gradient<T>(p, row, c0, n, bits, norm, c2, r);
}

// Whole rows that fit the registers: a workgroup of NTH threads holds a row, NV vectors to a thread, so that it is read
// once: 16 vectors in 1 024 threads are 256 KiB, half of a compute unit's registers.  As no more than one or a few
// workgroups then fit a compute unit, they stay, and ask for a vector of their next row as soon as the gradient of the
// present one's is stored.  Bound by memory: 8 192 x 131 072 in bfloat16 1 010 us, 4.25 TB/s read and written (a copy: 4.9),
// the difference being barriers that nothing is loaded beside.  A thread also holds its entry of the list, which is no
// longer than there are threads.
template <typename T, int NTH, int NV>
__global__ __launch_bounds__(NTH, 4) void k_distill_row(DistillArgs p) {
  constexpr int V = Store<T>::VEC, STEP = NTH * V, NWV = NTH / 64;
  extern __shared__ uint32_t bits[];
  __shared__ float smf[4][NWV];
  __shared__ double smd[3][NWV];
  const int n = p.vocab, k = p.top_k, t = threadIdx.x, wave = t >> 6;
  const float c2 = kLog2e / p.temp;
  const double inv_t = 1.0 / (double)p.temp;
  const int whole = n / V * V;                   // whole vectors, and what is left an element to a thread
  const int c_tail = whole + t;
  auto valid = [&](int id) { return id >= 0 && id < n; };
  auto weight_of = [&](int64_t row) { return row >= p.rows ? 0.0f : p.weight ? p.weight[row] : 1.0f; };
  int tv = t * V;
  uint32_t raw[NV][4];
  // the compiler must not keep what it makes of the row, or of its columns, in one pass for the next: that would take twice
  // the registers and more
  auto forget = [&] {
    asm volatile("" : "+v"(tv));
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(raw[u][i]));
  };
  auto load_vector = [&](const T* z, int u, int limit) {
    const int c = u * STEP + tv;
    if (c < limit) {
      __builtin_memcpy(raw[u], reinterpret_cast<const char*>(z) + (uint32_t)c * (uint32_t)sizeof(T), 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) raw[u][i] = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;      // -infinity
    }
  };
  auto element = [&](int u, int i) {
    return sizeof(T) == 4 ? __uint_as_float(raw[u][i % 4]) : __uint_as_float(i & 1 ? raw[u][i / 2] & 0xFFFF0000u : raw[u][i / 2] << 16);
  };
  auto exclude = [&](int u, int i) {
    if constexpr (sizeof(T) == 4) raw[u][i % 4] = 0xFF800000u;
    else raw[u][i / 2] = i & 1 ? (raw[u][i / 2] & 0xFFFFu) | 0xFF800000u : (raw[u][i / 2] & 0xFFFF0000u) | 0xFF80u;
  };
  int id_next = -1;
  float top_next = 0.0f, tail_next = 0.0f, lse_next = 0.0f;
  auto ask_for_rest = [&](int64_t r) {           // what a row needs beside its vectors
    const T* z = (const T*)p.logits + r * p.ld;
    id_next = t < k ? p.top_id[r * k + t] : -1;
    top_next = t < k ? p.top_logit[r * k + t] : 0.0f;
    tail_next = c_tail < n ? Store<T>::ld(z + c_tail) : -INFINITY;
    lse_next = p.teacher_lse ? p.teacher_lse[r] : 0.0f;
  };
  float w = weight_of(blockIdx.x);
  if (w != 0.0f) ask_for_rest(blockIdx.x);
  {
    const T* z = (const T*)p.logits + (int64_t)blockIdx.x * p.ld;
    const int limit = w != 0.0f ? whole : 0;     // a row without weight is not read
#pragma unroll
    for (int u = 0; u < NV; ++u) load_vector(z, u, limit);
  }
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T* z = (const T*)p.logits + row * p.ld;
    T* g = (T*)p.d_logits + row * p.ldd;
    const float w_next = weight_of(row + gridDim.x);
    const T* z_next = z + (int64_t)gridDim.x * p.ld;
    const int limit = w_next != 0.0f ? whole : 0;
    if (w == 0.0f) {
      if (t == 0) p.loss_rows[row] = 0.0f;
      const float o[V] = {};
      for (int c = t * V; c < n; c += STEP) store_outside<T>(g + c, o, 0u, n - c);
      if (w_next != 0.0f) ask_for_rest(row + gridDim.x);
#pragma unroll
      for (int u = 0; u < NV; ++u) load_vector(z_next, u, limit);
      w = w_next;
      continue;
    }
    const int id0 = id_next;
    const float top0 = top_next, z_tail = tail_next;
    const float z0 = valid(id0) ? Store<T>::ld(z + id0) : 0.0f;
    for (int i = t; i < (n + 31) / 32; i += NTH) bits[i] = 0u;
    float tm = valid(id0) ? top0 : -INFINITY;
    tm = max_rows(max16(tm));
    if ((t & 63) == 0) smf[0][wave] = tm;
    __syncthreads();
    if (valid(id0)) atomicOr(&bits[id0 >> 5], 1u << (id0 & 31));
    // the logarithm of what the teacher's probabilities are divided by
    double norm = (double)lse_next;
    if (!p.teacher_lse) {
      tm = max_of<NWV>(smf[0]);
      const double ref_t = tm == -INFINITY ? 0.0 : (double)tm;
      double s = 0.0;
      if (valid(id0)) s = exp_of(((double)top0 - ref_t) * inv_t);
      s = wave_sum(s);
      if ((t & 63) == 0) smd[0][wave] = s;
      norm = ref_t * inv_t;                      // and the sum's logarithm, below
    }
    float m = z_tail;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
#pragma unroll
      for (int i = 0; i < V; ++i) m = fmaxf(m, element(u, i));
      __builtin_amdgcn_sched_barrier(0);
    }
    m = max_rows(max16(m));
    forget();
    if ((t & 63) == 0) smf[1][wave] = m;
    __syncthreads();
    const bool tail = has_rest(p, norm);
    if (!p.teacher_lse && wave * 64 < k) norm += log_of(sum_of<NWV>(smd[0]));      // for wavefronts with entries of the list
    m = max_of<NWV>(smf[1]);
    // e_j = 2^(z_j c2 + k2) in one operation, k2 = -m c2.  What k2 is rounded by, |k2| 2^-25 at most, is a factor of all e_j, of
    // their sums too; the loss takes it out again (`off`).  That will do while the factor is near 1.  From |k2| = 2^20 on (a
    // large maximum, a low temperature; the same for all threads) the row becomes z_j - m before that, with k2 = 0: a
    // difference that the type does not hold is off by its last place, but of bfloat16 numbers it is then 0 or over
    // 2^20 2^-8 / c2, of which nothing is left anyway.  (A choice in every exponent takes 2 % longer.)
    float k2 = -reference(m) * c2, shift = 0.0f;
    if (!(fabsf(k2) < 0x1p20f)) {
      shift = reference(m);
      k2 = 0.0f;
#pragma unroll
      for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (sizeof(T) == 4) raw[u][i] = __float_as_uint(element(u, i) - shift);
          else raw[u][i] = pack_bf16(element(u, 2 * i) - shift, element(u, 2 * i + 1) - shift);
        }
    }
    const float off = fmaf(reference(m) - shift, c2, k2);     // 0 after that
    // e_j of a vector's columns
    auto exponentials = [&](int u, float (&e)[V]) {
#pragma unroll
      for (int i = 0; i < V; ++i) e[i] = fast_exp2(fmaf(element(u, i), c2, k2));
    };
    // the list's logits are its threads'; in the row, -infinity stands for them
    const bool in_tail = c_tail < n && (bits[c_tail >> 5] >> (c_tail & 31) & 1);
    const float x_tail = in_tail ? -INFINITY : z_tail - shift;
    const float e0 = valid(id0) ? fast_exp2(fmaf(z0 - shift, c2, k2)) : 0.0f;
    float e_tail = fast_exp2(fmaf(x_tail, c2, k2)), s_out = e_tail, s_in = e0;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int c = u * STEP + tv;
      if (u * STEP < whole) {
        const uint32_t mk = c < whole ? marks_of<V>(bits, c) : 0u;
        if (mk) {
#pragma unroll
          for (int i = 0; i < V; ++i)
            if (mk >> i & 1) exclude(u, i);
        }
        float e[V];
        exponentials(u, e);
        float sum = e[0];
#pragma unroll
        for (int i = 1; i < V; ++i) sum += e[i];
        s_out += sum;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    forget();
    double pi0 = 0.0, sp, sl = 0.0;
    if (valid(id0)) {
      const double lp = norm == -INFINITY ? -INFINITY : (double)top0 * inv_t - norm;
      pi0 = exp_of(lp);
      if (pi0 != 0.0) sl = pi0 * (lp - ((double)z0 - (double)reference(m)) * inv_t);
    }
    s_out = sum_rows(sum16(s_out));
    s_in = sum_rows(sum16(s_in));
    sp = wave_sum(pi0);
    sl = wave_sum(sl);
    if ((t & 63) == 0) {
      smf[2][wave] = s_out;
      smf[3][wave] = s_in;
      smd[1][wave] = sp;
      smd[2][wave] = sl;
    }
    __syncthreads();
    const float ref = reference(m) - shift;                    // in the row's present numbers
    DistillPart st = {ref, sum_of<NWV>(smf[2]), ref, sum_of<NWV>(smf[3]), sum_of<NWV>(smd[1]), sum_of<NWV>(smd[2])};
    float back = 1.0f;
    // One maximum will do for both sums while the outside's keeps its bits.  Where the teacher has a rest and that sum is small
    // (the same for all threads), it is taken again, relative to a maximum of its own; so is the gradient outside.
    if (tail && st.p < 1.0 && st.s_out < 0x1p-40f) {
      float mo = x_tail;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
#pragma unroll
        for (int i = 0; i < V; ++i) mo = fmaxf(mo, element(u, i));
        __builtin_amdgcn_sched_barrier(0);
      }
      mo = max_rows(max16(mo));
      forget();
      if ((t & 63) == 0) smf[0][wave] = mo;
      __syncthreads();
      st.m_out = mo = max_of<NWV>(smf[0]);
      if (((double)ref - (double)mo) * inv_t <= kFarthest) {     // so mo is hardly larger than the maximum, and k2 as small as before
        k2 = -mo * c2;
        float so = e_tail = fast_exp2(fmaf(x_tail, c2, k2));
#pragma unroll
        for (int u = 0; u < NV; ++u) {
          float e[V];
          exponentials(u, e);
#pragma unroll
          for (int i = 0; i < V; ++i) so += e[i];
          __builtin_amdgcn_sched_barrier(0);
        }
        so = sum_rows(sum16(so));
        forget();
        if ((t & 63) == 0) smf[1][wave] = so;
        __syncthreads();
        // in the measure of the other sum, 2^off
        back = fast_exp2(off - fmaf(mo, c2, k2));
        st.s_out = sum_of<NWV>(smf[1]) * back;
      }
    }
    RowGrad r = row_grad(p, st, w, c2, tail);
    r.f_out *= back;
    // the list's gradient and the loss first: what they are made of need not be held beside the row
    if (valid(id0)) {
      const double q = (double)(e0 / r.s_all);
      Store<T>::st(g + id0, r.empty ? 0.0f : (float)((r.mass * q - pi0) * r.scale));
    }
    if (t == NTH - 64) p.loss_rows[row] = row_loss(st, r, off);      // the last wavefront: the list is the first ones'
    if (w_next != 0.0f) ask_for_rest(row + gridDim.x);
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int c = u * STEP + tv;
      if (c < whole) {
        float o[V];
        exponentials(u, o);
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] *= r.f_out;
        store_outside<T>(g + c, o, marks_of<V>(bits, c), V);
      }
      load_vector(z_next, u, limit);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (c_tail < n && !in_tail) Store<T>::st(g + c_tail, r.f_out * e_tail);
    w = w_next;
    __syncthreads();                             // the marks and sums have been read
  }
}

// loss = sum of w_r L_r in a fixed order
__global__ __launch_bounds__(NT) void k_distill_total(const float* __restrict__ loss_rows, const float* __restrict__ weight, int64_t rows,
                                                      float* __restrict__ loss) {
  __shared__ double sm[NW + 1];
  double acc = 0.0;
  constexpr int U = 8;                           // loads in flight: 8 192 rows 24 us one by one
  for (int64_t r0 = threadIdx.x; r0 < rows; r0 += NT * U) {
    float w[U], l[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = r0 + u * NT;
      l[u] = r < rows ? loss_rows[r] : 0.0f;
      w[u] = r >= rows ? 0.0f : weight ? weight[r] : 1.0f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (w[u] != 0.0f) acc += (double)w[u] * (double)l[u];
  }
  acc = block_sum<NT>(acc, sm);
  if (threadIdx.x == 0) *loss = (float)acc;
}

template <typename T, int NTH, int NV>
int launch_distill_row(const DistillArgs& p, size_t lds, hipStream_t s) {
  // 16 vectors: workgroups that stay, as many as the registers of 256 compute units hold (128 to a thread).  Fewer: a row
  // each, since more of them run at a time (4 096 x 32 000 in bfloat16 124 us, with staying ones 145; 8 192 x 131 072 1 010, a
  // row each 1 071; 4 096 x 50 021 230 and 243)
  const int64_t stay = NV == 16 ? 256 * (1024 / NTH) : launch_blocks(NTH);
  hipLaunchKernelGGL((k_distill_row<T, NTH, NV>), dim3((unsigned)(p.rows < stay ? p.rows : stay)), dim3(NTH), lds, s, p);
  return launch_status("loss_distill");
}
template <typename T>
int launch_distill_rows(const DistillArgs& p, size_t lds, hipStream_t s) {
  const int vecs = (p.vocab + Store<T>::VEC - 1) / Store<T>::VEC;
  if (p.d_logits && p.top_k <= 256) {
    if (vecs <= 256 * 4) return launch_distill_row<T, 256, 4>(p, lds, s);
    if (vecs <= 256 * 8) return launch_distill_row<T, 256, 8>(p, lds, s);
    if (vecs <= 512 * 8) return launch_distill_row<T, 512, 8>(p, lds, s);
    if (vecs <= 512 * 16) return launch_distill_row<T, 512, 16>(p, lds, s);
    if (vecs <= 1024 * 16) return launch_distill_row<T, 1024, 16>(p, lds, s);
  }
  DistillArgs q = p;
  for (; q.row0 < p.rows; q.row0 += launch_blocks(NT)) {
    const int64_t left = p.rows - q.row0, most = launch_blocks(NT);
    hipLaunchKernelGGL((k_distill<T, 0>), dim3((unsigned)(left < most ? left : most)), dim3(NT), lds, s, q);
  }
  return launch_status("loss_distill");
}
template <typename T>
int launch_distill_pieces(const DistillArgs& p, size_t lds, hipStream_t s) {
  const dim3 grid((unsigned)(p.rows * p.splits));
  hipLaunchKernelGGL((k_distill<T, 1>), grid, dim3(NT), lds, s, p);
  hipLaunchKernelGGL((k_distill<T, 2>), grid, dim3(NT), lds, s, p);
  return launch_status("loss_distill");
}

// Rows in pieces of at least 4 096 columns, where whole rows would leave compute units idle for longer than the second launch takes.
constexpr int64_t kMaxVocab = 1 << 20;
void cut_rows(int64_t rows, int64_t vocab, bool cut, int* splits, int* chunk) {
  int64_t want = cut ? ((rows < 64 ? 256 : 512) + rows - 1) / rows : 1, most = (vocab + 4095) / 4096;
  if (want > most) want = most;
  if (want > MAX_SPLITS) want = MAX_SPLITS;
  const int64_t c = ((vocab + want - 1) / want + 63) / 64 * 64;
  *chunk = (int)c;
  *splits = (int)((vocab + c - 1) / c);
}
// log probabilities with a list of 20, 4 rows: 131 072 bfloat16 columns 16 us in pieces, 20 whole; 65 536 17 and 13; 50 021 binary32
// 15 and 13; 100 rows of 131 072 24 and 20
void cut_logprob(int64_t rows, int64_t vocab, int* splits, int* chunk) { cut_rows(rows, vocab, rows < 64 && vocab > 65536, splits, chunk); }
// The room that is asked for: from 32 769 columns on, as when rows were cut from there on.  Up to 65 536 no launch uses it; the
// query's answer, and that the call refuses less, stay as they were (4 rows of 65 536 with a list of 20: 11 KB).
void room_logprob(int64_t rows, int64_t vocab, int* splits, int* chunk) { cut_rows(rows, vocab, rows < 64 && vocab > 32768, splits, chunk); }
// distillation: 64 rows of 131 072 17 us in pieces, 28 whole; 100 of 50 021 16 and 19, 130 23 and 20; 4 rows
// of 32 768 in binary32 with the sum 11 and 14, of 17 000 11 and 9; 8 000 columns 10 and 8.  Rows that fill a compute
// unit's registers take twice as long from 257 rows on: 300 rows of 131 072 57 and 72 us, 511 91 and 78
void cut_distill(int64_t rows, int64_t vocab, int dtype, int* splits, int* chunk) {
  const bool alone = vocab > 512 * 16 * (dtype == AE_BF16 ? 8 : 4);
  cut_rows(rows, vocab, (rows < 128 && vocab > 24576) || (alone && rows > 256 && rows <= 384), splits, chunk);
}
int64_t align16(int64_t v) { return (v + 15) / 16 * 16; }

int check_rows(const char* who, int64_t rows, int64_t vocab, int dtype) {
  if (dtype != AE_F32 && dtype != AE_BF16) return fail(AE_EINVAL, "%s: bad dtype", who);
  if (rows < 0 || rows > ((int64_t)1 << 24)) return fail(AE_EINVAL, "%s: rows must be 0 .. 2^24", who);
  if (vocab < 1 || vocab > kMaxVocab) return fail(AE_EINVAL, "%s: vocab must be 1 .. 2^20", who);
  return AE_OK;
}
bool temp_ok(float t) { return t >= FLT_MIN && t <= FLT_MAX; }          // log2 e / t is finite

}  // namespace
}  // namespace ae

extern "C" int model_token_logprobs_workspace(int64_t rows, int64_t vocab, int top_k, int dtype, int64_t* bytes) {
  using namespace ae;
  if (!bytes) return fail(AE_EINVAL, "model_token_logprobs_workspace: null argument");
  AE_TRY(check_rows("model_token_logprobs_workspace", rows, vocab, dtype));
  if (top_k < 0 || top_k > 256 || top_k > vocab) return fail(AE_EINVAL, "model_token_logprobs_workspace: top_k must be 0 .. 256 and at most vocab");
  *bytes = 0;
  if (rows == 0) return AE_OK;
  int splits, chunk;
  room_logprob(rows, vocab, &splits, &chunk);
  if (splits > 1) *bytes = align16(rows * splits * (int64_t)sizeof(Stats)) + rows * splits * (int64_t)top_k * 8;
  return AE_OK;
}

extern "C" int model_token_logprobs(const void* logits, int64_t rows, int64_t vocab, int64_t ld, int dtype, float temperature,
                                    const int* tokens, int n_tokens, int top_k, float* logprob, float* entropy, float* lse,
                                    int* top_id, float* top_logit, float* top_logprob, void* workspace, void* stream) {
  using namespace ae;
  int64_t need = 0;
  AE_TRY(check_rows("model_token_logprobs", rows, vocab, dtype));
  if (ld < vocab || ld >= ((int64_t)1 << 40)) return fail(AE_EINVAL, "model_token_logprobs: rows must not overlap");
  if (!temp_ok(temperature)) return fail(AE_EINVAL, "model_token_logprobs: the temperature must be a positive normal number");
  if (n_tokens < 0 || n_tokens > 1024) return fail(AE_EINVAL, "model_token_logprobs: n_tokens must be 0 .. 1024");
  AE_TRY(model_token_logprobs_workspace(rows, vocab, top_k, dtype, &need));
  if (rows == 0) return AE_OK;
  if (!logits || (n_tokens && (!tokens || !logprob))) return fail(AE_EINVAL, "model_token_logprobs: null argument");
  if ((uintptr_t)logits % dtype_size(dtype)) return fail(AE_EINVAL, "model_token_logprobs: misaligned logits");
  if (need && (!workspace || ((uintptr_t)workspace & 15))) return fail(AE_EINVAL, "model_token_logprobs: workspace is null or not on a 16-byte border");
  LogprobArgs p = {};
  p.logits = logits; p.rows = rows; p.ld = ld; p.vocab = (int)vocab; p.temp = temperature;
  p.tokens = tokens; p.n_tokens = n_tokens; p.top_k = top_k;
  p.logprob = logprob; p.entropy = entropy; p.lse = lse; p.top_id = top_id; p.top_logit = top_logit; p.top_logprob = top_logprob;
  cut_logprob(rows, vocab, &p.splits, &p.chunk);
  p.part = (Stats*)workspace;
  p.part_top = (uint64_t*)((char*)workspace + align16(rows * p.splits * (int64_t)sizeof(Stats)));
  const bool top = top_k > 0 && (top_id || top_logit || top_logprob);
  hipStream_t s = (hipStream_t)stream;
  // rows in pieces are few: one launch takes them all
  const int64_t most = p.splits > 1 ? rows : launch_blocks(NT);
#define LOGPROB(T, TOP)                                                        \
  for (; p.row0 < rows; p.row0 += most) {                                      \
    const dim3 grid((unsigned)((rows - p.row0 < most ? rows - p.row0 : most) * p.splits));    \
    if (entropy) hipLaunchKernelGGL((k_logprob<T, TOP, true>), grid, dim3(NT), 0, s, p);      \
    else hipLaunchKernelGGL((k_logprob<T, TOP, false>), grid, dim3(NT), 0, s, p);             \
    if (p.splits > 1) hipLaunchKernelGGL((k_logprob_join<T, TOP>), dim3((unsigned)rows), dim3(NT), 0, s, p); \
  }
  if (dtype == AE_BF16) { if (top) LOGPROB(bf16_t, true) else LOGPROB(bf16_t, false) }
  else { if (top) LOGPROB(float, true) else LOGPROB(float, false) }
#undef LOGPROB
  return launch_status("token_logprobs");
}

extern "C" int model_loss_distill_workspace(int64_t rows, int64_t vocab, int dtype, int64_t* bytes) {
  using namespace ae;
  if (!bytes) return fail(AE_EINVAL, "model_loss_distill_workspace: null argument");
  AE_TRY(check_rows("model_loss_distill_workspace", rows, vocab, dtype));
  *bytes = 0;
  if (rows == 0) return AE_OK;
  int splits, chunk;
  cut_distill(rows, vocab, dtype, &splits, &chunk);
  *bytes = align16(rows * 4) + (splits > 1 ? rows * splits * (int64_t)sizeof(DistillPart) : 0);
  return AE_OK;
}

extern "C" int model_loss_distill(const void* logits, int64_t rows, int64_t vocab, int64_t ld, int dtype, float temperature,
                                  const int* top_id, const float* top_logit, int top_k, const float* teacher_lse,
                                  const float* weight, float* loss_rows, float* loss, void* d_logits, int64_t ldd,
                                  void* workspace, void* stream) {
  using namespace ae;
  int64_t need = 0;
  AE_TRY(check_rows("model_loss_distill", rows, vocab, dtype));
  if (ld < vocab || ld >= ((int64_t)1 << 40) || (d_logits && (ldd < vocab || ldd >= ((int64_t)1 << 40)))) return fail(AE_EINVAL, "model_loss_distill: rows must not overlap");
  if (!temp_ok(temperature)) return fail(AE_EINVAL, "model_loss_distill: the temperature must be a positive normal number");
  if (top_k < 1 || top_k > vocab) return fail(AE_EINVAL, "model_loss_distill: top_k must be 1 .. vocab");
  if (!loss_rows && !loss && !d_logits) return fail(AE_EINVAL, "model_loss_distill: no output");
  hipStream_t s = (hipStream_t)stream;
  if (rows > 0) {
    if (!logits || !top_id || !top_logit) return fail(AE_EINVAL, "model_loss_distill: null argument");
    if ((uintptr_t)logits % dtype_size(dtype) || (uintptr_t)d_logits % dtype_size(dtype)) return fail(AE_EINVAL, "model_loss_distill: misaligned logits");
    if (d_logits == logits && ldd != ld) return fail(AE_EINVAL, "model_loss_distill: a gradient in the logits' place has their stride");
    AE_TRY(model_loss_distill_workspace(rows, vocab, dtype, &need));
    if (!workspace || ((uintptr_t)workspace & 15)) return fail(AE_EINVAL, "model_loss_distill: workspace is null or not on a 16-byte border");
    DistillArgs p = {};
    p.logits = logits; p.rows = rows; p.ld = ld; p.vocab = (int)vocab; p.temp = temperature;
    p.top_id = top_id; p.top_logit = top_logit; p.top_k = top_k; p.teacher_lse = teacher_lse; p.weight = weight;
    p.loss_rows = loss_rows = loss_rows ? loss_rows : (float*)workspace;
    p.d_logits = d_logits; p.ldd = ldd;
    cut_distill(rows, vocab, dtype, &p.splits, &p.chunk);
    p.part = (DistillPart*)((char*)workspace + align16(rows * 4));
    const size_t lds = (size_t)(p.chunk + 31) / 32 * 4;
    if (p.splits > 1 && rows <= kTotalHere) {
      p.loss = loss;
      loss = nullptr;
    }
    if (p.splits == 1) AE_TRY(dtype == AE_BF16 ? launch_distill_rows<bf16_t>(p, lds, s) : launch_distill_rows<float>(p, lds, s));
    else AE_TRY(dtype == AE_BF16 ? launch_distill_pieces<bf16_t>(p, lds, s) : launch_distill_pieces<float>(p, lds, s));
  }
  if (loss) hipLaunchKernelGGL(k_distill_total, dim3(1), dim3(NT), 0, s, loss_rows, weight, rows, loss);
  return launch_status("loss_distill");
}
