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
__device__ __forceinline__ int key_index(uint64_t k) { return (int)(0xFFFFFFFFu - (uint32_t)k); }

// running statistics of a set of logits: maximum, sum of e_j, sum of e_j (z_j - m)
struct Stats {
  float m, s, a;
};
// the sum a after the maximum has grown by -d; f = the factor of the sums.  Nothing is left of what f = 0 scales (s d may overflow)
__device__ __forceinline__ float shifted(float a, float s, float d, float f) { return f == 0.0f ? 0.0f : f * (a + s * d); }
__device__ __forceinline__ Stats join(const Stats& x, const Stats& y, float c2) {
  Stats r;
  r.m = fmaxf(x.m, y.m);
  const float ref = reference(r.m);
  // differences of -infinity (a side without entries) are cut off at the lowest number, so that 0 times them is 0
  const float dx = fmaxf(x.m - ref, -FLT_MAX), dy = fmaxf(y.m - ref, -FLT_MAX);
  const float fx = fast_exp2(dx * c2), fy = fast_exp2(dy * c2);
  r.s = fx * x.s + fy * y.s;
  r.a = shifted(x.a, x.s, dx, fx) + shifted(y.a, y.s, dy, fy);
  return r;
}
__device__ __forceinline__ Stats wave_join(Stats v, float c2) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const Stats o = {__shfl_xor(v.m, off, 64), __shfl_xor(v.s, off, 64), __shfl_xor(v.a, off, 64)};
    v = join(v, o, c2);
  }
  return v;
}
__device__ __forceinline__ Stats block_join(Stats v, float c2, Stats* sm /* NW */) {
  v = wave_join(v, c2);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
  __syncthreads();
  v = sm[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) v = join(v, sm[i], c2);
  return v;
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
struct TopShared {
  uint64_t cand[CAND];
  uint32_t tmax[NT];
  int hist[256];
  int count, digit, before;
  uint32_t threshold;
};

// Leaves in sh.cand the sh.count >= min(k, all) largest keys, unordered, at most CAND.  `each(f)` calls f(key) for the
// thread's share of the keys; tmax is the upper half of the share's largest key, 0 for an empty share.
// The k-th largest of the threads' maxima is a lower bound of the k-th largest key, since those maxima are k keys
// themselves; as the largest keys lie in different shares for the most part, few others pass it.  Only threads whose
// maximum passes go over their share again.  Where more keys pass than LDS holds (long runs of equal logits, maxima in
// one share), the bound is sharpened by digits of the whole key.
template <typename E>
__device__ void top_select(TopShared& sh, int k, uint32_t tmax, E each) {
  const int t = threadIdx.x, lane = t & 63;
  __syncthreads();
  sh.tmax[t] = tmax;
  if (t == 0) sh.count = 0;
  __syncthreads();
  if (t < 64) {
    uint32_t v[NT / 64];
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) v[i] = sh.tmax[lane + 64 * i];
    uint32_t bound = 0;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t c = bound | (1u << bit);
      int n = 0;
#pragma unroll
      for (int i = 0; i < NT / 64; ++i) n += __popcll(__ballot(v[i] >= c));
      if (n >= k) bound = c;
      if (n == k) break;
    }
    if (lane == 0) sh.threshold = bound;
  }
  __syncthreads();
  const uint32_t bound = sh.threshold;
  if (tmax >= bound) {
    each([&](uint64_t key) {
      if ((uint32_t)(key >> 32) >= bound) {
        const int at = atomicAdd(&sh.count, 1);
        if (at < CAND) sh.cand[at] = key;
      }
    });
  }
  __syncthreads();
  int count = sh.count;
  if (count >= k && count <= CAND) return;
  uint64_t prefix = 0;
  int want = k;                          // how many of the keys that share the prefix belong to the list
  for (int d = 7; d >= 0; --d) {
    __syncthreads();
    if (t < 256) sh.hist[t] = 0;
    __syncthreads();
    each([&](uint64_t key) {
      if (d == 7 || (key >> (8 * d + 8)) == (prefix >> (8 * d + 8))) {
        const int digit = (int)(key >> (8 * d)) & 255;
        const int first = __builtin_amdgcn_readfirstlane(digit);
        const uint64_t same = __ballot(digit == first);          // lanes of equal digits add once, not one after the other
        if (digit == first) {
          if (lane == __ffsll((unsigned long long)same) - 1) atomicAdd(&sh.hist[digit], __popcll(same));
        } else {
          atomicAdd(&sh.hist[digit], 1);
        }
      }
    });
    __syncthreads();
    if (t == 0) {
      int above = 0, at = 255;
      while (at > 0 && above + sh.hist[at] < want) above += sh.hist[at--];
      sh.digit = at;
      sh.before = above;
    }
    __syncthreads();
    prefix |= (uint64_t)sh.digit << (8 * d);
    want -= sh.before;
    if (k - want + sh.hist[sh.digit] <= CAND) break;             // everything from the prefix on fits
  }
  __syncthreads();
  if (t == 0) sh.count = 0;
  __syncthreads();
  each([&](uint64_t key) {
    if (key >= prefix) {
      const int at = atomicAdd(&sh.count, 1);
      if (at < CAND) sh.cand[at] = key;
    }
  });
  __syncthreads();
}
// Calls f(rank, key) for the k largest candidates; keys differ, so a key's rank is the number of larger ones.
template <typename F>
__device__ void top_ranked(const TopShared& sh, int k, F f) {
  const int count = sh.count < CAND ? sh.count : CAND;
  for (int i = threadIdx.x; i < count; i += NT) {
    const uint64_t key = sh.cand[i];
    int rank = 0;
    for (int j = 0; j < count; ++j) rank += sh.cand[j] > key ? 1 : 0;
    if (rank < k) f(rank, key);
  }
}

struct LogprobArgs {
  const void* logits;
  int64_t rows, ld;
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
template <typename T>
__device__ void write_top(const LogprobArgs& p, int64_t row, const RowLog& r, int rank, uint64_t key) {
  const int id = key_index(key);
  const float z = Store<T>::ld((const T*)p.logits + row * p.ld + id);
  const int64_t at = row * p.top_k + rank;
  if (p.top_id) p.top_id[at] = id;
  if (p.top_logit) p.top_logit[at] = z;
  if (p.top_logprob) p.top_logprob[at] = log_prob(z, r, p.temp);
}

// One workgroup per row piece; with one piece per row it writes the results, otherwise what k_logprob_join needs.
template <typename T, bool TOP>
__global__ __launch_bounds__(NT) void k_logprob(LogprobArgs p) {
  constexpr int V = Store<T>::VEC;
  __shared__ Stats sm[NW];
  __shared__ TopShared sh;
  const int64_t row = blockIdx.x / p.splits;
  const int split = (int)(blockIdx.x - row * p.splits);
  const int c0 = split * p.chunk;
  const int n = p.vocab - c0 < p.chunk ? p.vocab - c0 : p.chunk;
  const T* z = (const T*)p.logits + row * p.ld + c0;
  const float c2 = kLog2e / p.temp;
  Stats st = {-INFINITY, 0.0f, 0.0f};
  bool some = false;
  for_vectors<T>(z, n, [&](const float (&v)[V], int, int) {
    float cm = v[0];
#pragma unroll
    for (int i = 1; i < V; ++i) cm = fmaxf(cm, v[i]);
    some = true;
    if (cm > st.m) {
      const float d = fmaxf(st.m - cm, -FLT_MAX), f = fast_exp2(d * c2);
      st.a = shifted(st.a, st.s, d, f);
      st.s *= f;
      st.m = cm;
    }
    const float ref = reference(st.m);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float d = v[i] - ref, e = fast_exp2(d * c2);
      st.s += e;
      st.a += e * fmaxf(d, -FLT_MAX);
    }
  });
  const uint32_t tmax = some ? order_key(st.m) : 0u;
  const Stats all = block_join(st, c2, sm);
  if (p.splits == 1) write_row<T>(p, row, all);
  else if (threadIdx.x == 0) p.part[row * p.splits + split] = all;
  if constexpr (TOP) {
    const int k = p.top_k < n ? p.top_k : n;
    top_select(sh, k, tmax, [&](auto f) {
      for_vectors<T>(z, n, [&](const float (&v)[V], int c, int len) {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (i < len) f(order_key(v[i], c0 + c + i));
      });
    });
    if (p.splits == 1) {
      const RowLog r = row_log(all);
      top_ranked(sh, k, [&](int rank, uint64_t key) { write_top<T>(p, row, r, rank, key); });
    } else {
      uint64_t* out = p.part_top + (row * p.splits + split) * p.top_k;
      top_ranked(sh, k, [&](int rank, uint64_t key) { out[rank] = key; });
      for (int i = k + (int)threadIdx.x; i < p.top_k; i += NT) out[i] = 0;
    }
  }
}

// One workgroup per row: joins its pieces.
template <typename T, bool TOP>
__global__ __launch_bounds__(NT) void k_logprob_join(LogprobArgs p) {
  __shared__ Stats sm;
  __shared__ TopShared sh;
  const int64_t row = blockIdx.x;
  const float c2 = kLog2e / p.temp;
  if (threadIdx.x < 64) {
    Stats st = {-INFINITY, 0.0f, 0.0f};
    if ((int)threadIdx.x < p.splits) st = p.part[row * p.splits + threadIdx.x];
    st = wave_join(st, c2);
    if (threadIdx.x == 0) sm = st;
  }
  __syncthreads();
  const Stats all = sm;
  write_row<T>(p, row, all);
  if constexpr (TOP) {
    const uint64_t* keys = p.part_top + row * p.splits * p.top_k;
    const int n = p.splits * p.top_k;
    uint32_t tmax = 0;
    for (int i = threadIdx.x; i < n; i += NT) {
      const uint32_t h = (uint32_t)(keys[i] >> 32);
      tmax = h > tmax ? h : tmax;
    }
    top_select(sh, p.top_k, tmax, [&](auto f) {
      for (int i = threadIdx.x; i < n; i += NT) {
        const uint64_t key = keys[i];
        if (key != 0) f(key);
      }
    });
    const RowLog r = row_log(all);
    top_ranked(sh, p.top_k, [&](int rank, uint64_t key) { write_top<T>(p, row, r, rank, key); });
  }
}

// ---- distillation --------------------------------------------------------------------------------------------------
struct DistillPart {                     // of a row piece
  float m, s_out, s_in, pad;             // maximum; sums of e_j outside and inside the teacher's list
  double p, l;                           // sums over the list's entries in the piece: p_i, and p_i (log p_i - z_i / T)
};
struct DistillArgs {
  const void* logits;
  int64_t rows, ld;
  int vocab, splits, chunk;
  float temp;
  const int* top_id;
  const float* top_logit;
  int top_k;
  const float *teacher_lse, *weight;
  float* loss_rows;
  void* d_logits;
  int64_t ldd;
  DistillPart* part;                     // [rows][splits]
};

__device__ __forceinline__ DistillPart join(const DistillPart& x, const DistillPart& y, float c2) {
  DistillPart r;
  r.m = fmaxf(x.m, y.m);
  const float ref = reference(r.m);
  const float fx = fast_exp2((x.m - ref) * c2), fy = fast_exp2((y.m - ref) * c2);
  r.s_out = fx * x.s_out + fy * y.s_out;
  r.s_in = fx * x.s_in + fy * y.s_in;
  r.pad = 0.0f;
  r.p = x.p + y.p;
  r.l = x.l + y.l;
  return r;
}

// the logarithm of the sum that the teacher's probabilities are divided by
__device__ double list_norm(const DistillArgs& p, int64_t row, double* sm /* NW + 1 */) {
  if (p.teacher_lse) return (double)p.teacher_lse[row];
  const int* id = p.top_id + row * p.top_k;
  const float* t = p.top_logit + row * p.top_k;
  float m = -INFINITY;
  for (int i = threadIdx.x; i < p.top_k; i += NT)
    if (id[i] >= 0 && id[i] < p.vocab) m = fmaxf(m, t[i]);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = (double)m;
  __syncthreads();
  double dm = sm[0];
  for (int i = 1; i < NW; ++i) dm = sm[i] > dm ? sm[i] : dm;
  if (dm == -INFINITY) dm = 0.0;
  double s = 0.0;
  for (int i = threadIdx.x; i < p.top_k; i += NT)
    if (id[i] >= 0 && id[i] < p.vocab) s += exp(((double)t[i] - dm) / (double)p.temp);
  __syncthreads();
  s = block_sum<NT>(s, sm);
  return dm / (double)p.temp + log(s);
}
__device__ __forceinline__ double list_log_p(const DistillArgs& p, int64_t at, double norm) { return (double)p.top_logit[at] / (double)p.temp - norm; }

// marks the list's tokens that lie in columns [c0, c0 + n): a bit for each column
__device__ void mark_list(const DistillArgs& p, int64_t row, int c0, int n, uint32_t* bits) {
  for (int i = threadIdx.x; i < (n + 31) / 32; i += NT) bits[i] = 0u;
  __syncthreads();
  for (int i = threadIdx.x; i < p.top_k; i += NT) {
    const int id = p.top_id[row * p.top_k + i];
    if (id >= c0 && id < c0 + n) atomicOr(&bits[(id - c0) >> 5], 1u << ((id - c0) & 31));
  }
  __syncthreads();
}
template <int V> __device__ __forceinline__ uint32_t marks_of(const uint32_t* bits, int c) { return (bits[c >> 5] >> (c & 31)) & ((1u << V) - 1u); }

template <typename T>
__device__ DistillPart piece_stats(const DistillArgs& p, int64_t row, int c0, int n, const uint32_t* bits, double norm, float c2,
                                   DistillPart* sm /* NW */) {
  constexpr int V = Store<T>::VEC;
  const T* z = (const T*)p.logits + row * p.ld + c0;
  DistillPart st = {-INFINITY, 0.0f, 0.0f, 0.0f, 0.0, 0.0};
  for_vectors<T>(z, n, [&](const float (&v)[V], int c, int) {
    float cm = v[0];
#pragma unroll
    for (int i = 1; i < V; ++i) cm = fmaxf(cm, v[i]);
    if (cm > st.m) {
      const float f = fast_exp2((st.m - cm) * c2);
      st.s_out *= f;
      st.s_in *= f;
      st.m = cm;
    }
    const float ref = reference(st.m);
    const uint32_t mk = marks_of<V>(bits, c);
    float e[V];
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = fast_exp2((v[i] - ref) * c2);
    if (mk) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (mk >> i & 1) st.s_in += e[i];
        else st.s_out += e[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) st.s_out += e[i];
    }
  });
  for (int i = threadIdx.x; i < p.top_k; i += NT) {
    const int id = p.top_id[row * p.top_k + i];
    if (id < c0 || id >= c0 + n) continue;
    const double lp = list_log_p(p, row * p.top_k + i, norm), pi = exp(lp);
    st.p += pi;
    if (pi != 0.0) st.l += pi * (lp - (double)Store<T>::ld(z + id - c0) / (double)p.temp);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const DistillPart o = {__shfl_xor(st.m, off, 64), __shfl_xor(st.s_out, off, 64), __shfl_xor(st.s_in, off, 64), 0.0f,
                           __shfl_xor(st.p, off, 64), __shfl_xor(st.l, off, 64)};
    st = join(st, o, c2);
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = st;
  __syncthreads();
  st = sm[0];
  for (int i = 1; i < NW; ++i) st = join(st, sm[i], c2);
  return st;
}

// The loss of a row and the gradient of columns [c0, c0 + n) from the statistics of the whole row.
template <typename T>
__device__ void piece_gradient(const DistillArgs& p, int64_t row, int c0, int n, const uint32_t* bits, double norm, float c2, float w,
                               const DistillPart& st, bool write_loss) {
  constexpr int V = Store<T>::VEC;
  const double s_all = (double)st.s_out + (double)st.s_in;
  const bool empty = s_all == 0.0;
  const double q_out = (double)st.s_out / s_all;
  double rest = p.teacher_lse ? 1.0 - st.p : 0.0;
  if (!(rest > 0.0) && rest == rest) rest = 0.0;
  if (st.s_out == 0.0f) rest = 0.0;
  const double mass = st.p + rest;
  if (write_loss && threadIdx.x == 0) {
    const double lse = (double)st.m / (double)p.temp + log(s_all);
    double loss = st.l + (st.p != 0.0 ? st.p * lse : 0.0);
    if (rest != 0.0) loss += rest * (log(rest) - log(q_out));
    p.loss_rows[row] = empty ? 0.0f : (float)loss;
  }
  if (!p.d_logits) return;
  const T* z = (const T*)p.logits + row * p.ld + c0;
  T* g = (T*)p.d_logits + row * p.ldd + c0;
  const double scale = (double)w / (double)p.temp;
  const float f_out = empty ? 0.0f : (float)((mass - (rest != 0.0 ? rest / q_out : 0.0)) * scale / s_all);
  const float ref = reference(st.m);
  for_vectors<T>(z, n, [&](const float (&v)[V], int c, int len) {
    float o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = f_out * fast_exp2((v[i] - ref) * c2);
    const uint32_t mk = marks_of<V>(bits, c);
    if (mk == 0 && len == V) {
      store_vec<T>(g + c, o);
    } else {
      // the list's entries are left as they are: g may be z, which they still need
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i < len && !(mk >> i & 1)) Store<T>::st(g + c + i, o[i]);
    }
  });
  for (int i = threadIdx.x; i < p.top_k; i += NT) {
    const int id = p.top_id[row * p.top_k + i];
    if (id < c0 || id >= c0 + n) continue;
    const double q = (double)fast_exp2((Store<T>::ld(z + id - c0) - ref) * c2) / s_all;
    const double pi = exp(list_log_p(p, row * p.top_k + i, norm));
    Store<T>::st(g + id - c0, empty ? 0.0f : (float)((mass * q - pi) * scale));
  }
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

// MODE 0: statistics and gradient of whole rows; 1: statistics of row pieces; 2: gradient of row pieces from joined statistics
template <typename T, int MODE>
__global__ __launch_bounds__(NT) void k_distill(DistillArgs p) {
  extern __shared__ uint32_t bits[];
  __shared__ DistillPart sm[NW];
  __shared__ double smd[NW + 1];
  const int64_t row = blockIdx.x / p.splits;
  const int split = (int)(blockIdx.x - row * p.splits);
  const int c0 = split * p.chunk;
  const int n = p.vocab - c0 < p.chunk ? p.vocab - c0 : p.chunk;
  const float w = p.weight ? p.weight[row] : 1.0f;
  if (w == 0.0f) {
    if (MODE != 1) {
      if (threadIdx.x == 0 && split == 0) p.loss_rows[row] = 0.0f;
      if (p.d_logits) piece_zero<T>(p, row, c0, n);
    }
    return;
  }
  const float c2 = kLog2e / p.temp;
  mark_list(p, row, c0, n, bits);
  const double norm = list_norm(p, row, smd);
  DistillPart st;
  if constexpr (MODE != 2) {
    st = piece_stats<T>(p, row, c0, n, bits, norm, c2, sm);
    if constexpr (MODE == 1) {
      if (threadIdx.x == 0) p.part[row * p.splits + split] = st;
      return;
    }
  } else {
    st = p.part[row * p.splits];
    for (int i = 1; i < p.splits; ++i) st = join(st, p.part[row * p.splits + i], c2);
  }
  piece_gradient<T>(p, row, c0, n, bits, norm, c2, w, st, split == 0);
}

// loss = sum of w_r L_r in a fixed order
__global__ __launch_bounds__(NT) void k_distill_total(const float* __restrict__ loss_rows, const float* __restrict__ weight, int64_t rows,
                                                      float* __restrict__ loss) {
  __shared__ double sm[NW + 1];
  double acc = 0.0;
  for (int64_t r = threadIdx.x; r < rows; r += NT) {
    const float w = weight ? weight[r] : 1.0f;
    if (w != 0.0f) acc += (double)w * (double)loss_rows[r];
  }
  acc = block_sum<NT>(acc, sm);
  if (threadIdx.x == 0) *loss = (float)acc;
}

// Pieces of a row: enough workgroups for the chip where rows alone are too few, none shorter than 4 096 columns.
constexpr int64_t kMaxVocab = 1 << 20;
void cut_rows(int64_t rows, int64_t vocab, int* splits, int* chunk) {
  int64_t want = rows >= 256 ? 1 : (512 + rows - 1) / rows, most = (vocab + 4095) / 4096;
  if (want > most) want = most;
  if (want > MAX_SPLITS) want = MAX_SPLITS;
  const int64_t c = ((vocab + want - 1) / want + 63) / 64 * 64;
  *chunk = (int)c;
  *splits = (int)((vocab + c - 1) / c);
}
int64_t align16(int64_t v) { return (v + 15) / 16 * 16; }

int check_rows(const char* who, int64_t rows, int64_t vocab, int dtype) {
  if (dtype != AE_F32 && dtype != AE_BF16) return fail(AE_EINVAL, "%s: bad dtype", who);
  if (rows < 0 || rows > ((int64_t)1 << 24)) return fail(AE_EINVAL, "%s: rows must be 0 .. 2^24", who);
  if (vocab < 1 || vocab > kMaxVocab) return fail(AE_EINVAL, "%s: vocab must be 1 .. 2^20", who);
  return AE_OK;
}
bool temp_ok(float t) { return t > 0.0f && t <= FLT_MAX; }

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
  cut_rows(rows, vocab, &splits, &chunk);
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
  if (!temp_ok(temperature)) return fail(AE_EINVAL, "model_token_logprobs: the temperature must be positive and finite");
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
  cut_rows(rows, vocab, &p.splits, &p.chunk);
  p.part = (Stats*)workspace;
  p.part_top = (uint64_t*)((char*)workspace + align16(rows * p.splits * (int64_t)sizeof(Stats)));
  const bool top = top_k > 0 && (top_id || top_logit || top_logprob);
  hipStream_t s = (hipStream_t)stream;
  const dim3 grid((unsigned)(rows * p.splits)), grid_j((unsigned)rows);
#define LOGPROB(T, TOP)                                                        \
  do {                                                                         \
    hipLaunchKernelGGL((k_logprob<T, TOP>), grid, dim3(NT), 0, s, p);          \
    if (p.splits > 1) hipLaunchKernelGGL((k_logprob_join<T, TOP>), grid_j, dim3(NT), 0, s, p); \
  } while (0)
  if (dtype == AE_BF16) { if (top) LOGPROB(bf16_t, true); else LOGPROB(bf16_t, false); }
  else { if (top) LOGPROB(float, true); else LOGPROB(float, false); }
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
  cut_rows(rows, vocab, &splits, &chunk);
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
  if (!temp_ok(temperature)) return fail(AE_EINVAL, "model_loss_distill: the temperature must be positive and finite");
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
    cut_rows(rows, vocab, &p.splits, &p.chunk);
    p.part = (DistillPart*)((char*)workspace + align16(rows * 4));
    const dim3 grid((unsigned)(rows * p.splits));
    const size_t lds = (size_t)(p.chunk + 31) / 32 * 4;
#define DISTILL(T)                                                                   \
  do {                                                                               \
    if (p.splits == 1) {                                                             \
      hipLaunchKernelGGL((k_distill<T, 0>), grid, dim3(NT), lds, s, p);              \
    } else {                                                                         \
      hipLaunchKernelGGL((k_distill<T, 1>), grid, dim3(NT), lds, s, p);              \
      hipLaunchKernelGGL((k_distill<T, 2>), grid, dim3(NT), lds, s, p);              \
    }                                                                                \
  } while (0)
    if (dtype == AE_BF16) DISTILL(bf16_t);
    else DISTILL(float);
#undef DISTILL
    AE_TRY(launch_status("loss_distill"));
  }
  if (loss) hipLaunchKernelGGL(k_distill_total, dim3(1), dim3(NT), 0, s, loss_rows, weight, rows, loss);
  return launch_status("loss_distill");
}
