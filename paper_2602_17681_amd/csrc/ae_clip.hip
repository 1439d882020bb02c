// ae_clip.hip — the norm of many gradients taken together, and the gradients scaled down to a largest norm.
//   norm = sqrt(sum over all elements of g^2);   out = g min(1, max_norm / norm)
// Two passes bound by memory.  The tensors' addresses are arguments of the kernels, so that nothing is copied to the device
// and a captured call keeps them; a list longer than the arguments' room takes several launches.  Squares are added up
// in binary64, whose range the squares of binary32 numbers do not leave.  134 M binary32 gradients: the norm 83 us (6.5 TB/s), clipped into other
// tensors 253 - 258 (1.6 GB through both passes at 6.3 TB/s, part of the second read from the cache); 128 tensors of 1 M in all 10 us in two launches.
#include <hip/hip_runtime.h>
#include <float.h>

#include <algorithm>
#include <new>
#include <utility>
#include <vector>

#include "ae_device.h"
#include "ae_internal.h"
#include "ae_rows.h"

namespace ae {
namespace {

constexpr int NT = 256;
constexpr int64_t CHUNK = 8192;                  // elements that a workgroup takes at a time
constexpr int LIST = 128;                        // tensors of a launch: 3.8 of the 4 KB that arguments may have
template <typename T> constexpr int VEC = 16 / (int)sizeof(T);
template <typename T> constexpr int PIECES = (int)(CHUNK / NT / VEC<T>);          // 16-byte pieces of a thread, all in flight
struct GradArgs {
  const void* in[LIST];
  void* out[LIST];
  int64_t size[LIST];
  int end[LIST];                                 // chunks of the tensors up to this one; behind the last: the largest int
  uint8_t bf16[LIST];
  int count, chunks;
  float keep;                                    // part of a share, at its end, that is read to stay in the cache
};
// the tensor that a chunk belongs to: the first whose end lies behind it, all compared at once
__device__ __forceinline__ int tensor_of(const GradArgs& p, int chunk) {
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int i = 0; i < LIST; i += 64) n += __popcll(__ballot(p.end[i + lane] <= chunk));
  return n;
}
template <typename T, bool STREAM>
__device__ __forceinline__ void chunk_load(const T* p, int64_t left, Piece<T, VEC<T>> (&e)[PIECES<T>]) {
  if (left >= CHUNK) {                            // whole chunks: nothing between the loads
#pragma unroll
    for (int u = 0; u < PIECES<T>; ++u) fetch_whole<STREAM>(p + (u * NT + (int)threadIdx.x) * VEC<T>, e[u]);
  } else {
#pragma unroll
    for (int u = 0; u < PIECES<T>; ++u) {
      const int at = (u * NT + (int)threadIdx.x) * VEC<T>, l = (int)left - at;
      fetch(p + at, l < 0 ? 0 : l, e[u]);
    }
  }
}
template <typename T, bool STREAM>
__device__ __forceinline__ double chunk_squares(const T* p, int64_t left) {
  Piece<T, VEC<T>> e[PIECES<T>];
  chunk_load<T, STREAM>(p, left, e);
  double acc = 0.0;
#pragma unroll
  for (int u = 0; u < PIECES<T>; ++u)
#pragma unroll
    for (int j = 0; j < VEC<T>; ++j) {
      const double v = (double)value(e[u], j);
      acc = fma(v, v, acc);
    }
  return acc;
}
// Workgroup g takes the g-th of gridDim.x equal shares of the chunks, in order.
__device__ __forceinline__ int share(const GradArgs& p, int g) { return (int)((int64_t)p.chunks * g / (int)gridDim.x); }
__global__ __launch_bounds__(NT) void k_grad_squares(GradArgs p, double* __restrict__ part) {
  __shared__ double sm[NT / 64 + 1];
  const int from = share(p, blockIdx.x), to = share(p, blockIdx.x + 1);
  const int stay = to - (int)ceilf((float)(to - from) * p.keep);
  double acc = 0.0;
  int k = tensor_of(p, from);
  for (int c = from; c < to; ++c) {
    while (c >= p.end[k]) ++k;
    const int64_t at = (int64_t)(c - (k ? p.end[k - 1] : 0)) * CHUNK, left = p.size[k] - at;
    if (c >= stay) acc += p.bf16[k] ? chunk_squares<bf16_t, false>((const bf16_t*)p.in[k] + at, left) : chunk_squares<float, false>((const float*)p.in[k] + at, left);
    else acc += p.bf16[k] ? chunk_squares<bf16_t, true>((const bf16_t*)p.in[k] + at, left) : chunk_squares<float, true>((const float*)p.in[k] + at, left);
  }
  acc = block_sum<NT>(acc, sm);
  if (threadIdx.x == 0) part[blockIdx.x] = acc;
}

// The product is binary64's and rounded once: max_norm / norm may be less than any binary32 number while the product is an ordinary one.
template <typename T>
__device__ __forceinline__ void chunk_scale(const T* p, T* out, int64_t left, double factor) {
  Piece<T, VEC<T>> e[PIECES<T>];
  chunk_load<T, true>(p, left, e);
#pragma unroll
  for (int u = 0; u < PIECES<T>; ++u) {
    const int at = (u * NT + (int)threadIdx.x) * VEC<T>;
    float v[VEC<T>];
#pragma unroll
    for (int j = 0; j < VEC<T>; ++j) v[j] = (float)((double)value(e[u], j) * factor);
    if (left >= CHUNK) put_whole<true>(out + at, v);
    else if (left > at) put(out + at, (int)left - at, v);
  }
}
// the sum of all shares' sums, and the norm; eight loads of a thread in flight, added in order
__device__ __forceinline__ double sum_of_parts(const double* __restrict__ part, int parts, double* sm) {
  constexpr int U = 8;
  double sum = 0.0;
  for (int i = threadIdx.x; i < parts; i += U * NT) {
    double v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = i + u * NT < parts ? part[i + u * NT] : 0.0;
#pragma unroll
    for (int u = 0; u < U; ++u) sum += v[u];
  }
  return block_sum<NT>(sum, sm);
}
__global__ __launch_bounds__(NT) void k_grad_norm(const double* __restrict__ part, int parts, float* __restrict__ norm, double* __restrict__ total) {
  __shared__ double sm[NT / 64 + 1];
  const double sum = sum_of_parts(part, parts, sm);
  if (threadIdx.x) return;
  if (norm) *norm = (float)sqrt(sum);
  if (total) *total = sum;
}
// Every workgroup adds up the shares' sums itself, in the same order (8 KB a launch of sums, from L2), so that no launch stands in between; of long
// lists, where each of many launches would read those of all, the one sum that k_grad_norm has made of them.
__global__ __launch_bounds__(NT) void k_grad_scale(GradArgs p, const double* __restrict__ part, int parts, float max_norm, float* __restrict__ norm) {
  __shared__ double sm[NT / 64 + 1];
  const double all = sqrt(sum_of_parts(part, parts, sm));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)all;
  // no number or infinite: an element is; nothing is scaled.  Finite gradients whose norm binary32 does not hold are
  const double factor = all > (double)max_norm && all <= DBL_MAX ? (double)max_norm / all : 1.0;
  const bool same = (float)factor == 1.0f;         // from 1 - 2^-25 on every product rounds to its gradient
  const int from = share(p, blockIdx.x), to = share(p, blockIdx.x + 1);
  int k = from < to ? tensor_of(p, to - 1) : 0;
  for (int c = to - 1; c >= from; --c) {           // backwards: what the first pass read last is still in the cache
    while (k > 0 && c < p.end[k - 1]) --k;
    if (same && p.in[k] == p.out[k]) continue;
    const int64_t at = (int64_t)(c - (k ? p.end[k - 1] : 0)) * CHUNK, left = p.size[k] - at;
    if (p.bf16[k]) chunk_scale((const bf16_t*)p.in[k] + at, (bf16_t*)p.out[k] + at, left, factor);
    else chunk_scale((const float*)p.in[k] + at, (float*)p.out[k] + at, left, factor);
  }
}

constexpr int kShares = 1024;                    // workgroups of a launch at most (512 MB, norm alone / clipped: 83 / 253 us; 2 048 83 / 258, 4 096 86 / 266)
// What the second pass finds in the cache, beginning with what the first read last; the first reads the rest of a list, and all
// where there is no second, as a stream.  512 MB clipped: 253 us with 256 MB kept, 261 with 192, 278 with 64, 257 with all; 1 024 MB 529, 537, 555, 547.
constexpr int64_t kKeep = (int64_t)256 << 20;
int64_t chunks_of(int64_t size) { return (size + CHUNK - 1) / CHUNK; }
// the tensors [from, *next) of one launch: *next is behind the last, chunks are counted
int64_t launch_range(const int64_t* sizes, int count, int from, int* next) {
  int64_t chunks = 0;
  int n = 0, k = from;
  for (; k < count && n < LIST; ++k) {
    const int64_t c = chunks_of(sizes[k]);
    if (c == 0) continue;
    if (chunks + c > 0x7FFFFFFF) break;
    chunks += c;
    ++n;
  }
  *next = k;
  return chunks;
}
int shares_of(int64_t chunks) { return (int)(chunks < kShares ? chunks : kShares); }
// Launches from which on the sum is made once.  Tensors of 8 192, in us, by every workgroup / once: 500 (4 launches) 31.0 / 32.1, 1 000 (8) 70.1 / 71.2, of 131 072
// each 331 / 316, 5 000 of 1 000 354 / 321, 20 000 1 877 / 1 344, 100 000 of 100 20 800 / 6 630 (2 000 launches of sums and scaling).
constexpr int kAlone = 4;
constexpr int64_t kSizeMax = (int64_t)1 << 40;   // elements of a tensor: 2^27 chunks
int check_sizes(const char* who, const int64_t* sizes, int count) {
  if (count < 0 || count > (1 << 20) || (count && !sizes)) return fail(AE_EINVAL, "%s: count must be 0 .. 2^20, with a size for each", who);
  for (int k = 0; k < count; ++k)
    if (sizes[k] < 0 || sizes[k] > kSizeMax) return fail(AE_EINVAL, "%s: sizes must be 0 .. 2^40", who);
  return AE_OK;
}
int64_t parts_of(const int64_t* sizes, int count) {
  int64_t parts = 0;
  for (int k = 0; k < count;) parts += shares_of(launch_range(sizes, count, k, &k));
  return parts;
}

// Whether no output overlaps another, or a gradient other than the one that it is the place of.
typedef std::pair<uintptr_t, uintptr_t> Range;
bool apart(void* const* grads, void* const* out, const int64_t* sizes, const int* dtypes, int count) {
  std::vector<Range> w, r;
  w.reserve(count);
  r.reserve(count);
  for (int k = 0; k < count; ++k) {
    const uintptr_t bytes = (uintptr_t)sizes[k] * dtype_size(dtypes[k]);
    if (!bytes) continue;
    w.emplace_back((uintptr_t)out[k], (uintptr_t)out[k] + bytes);
    if (out[k] != grads[k]) r.emplace_back((uintptr_t)grads[k], (uintptr_t)grads[k] + bytes);
  }
  if (!std::is_sorted(w.begin(), w.end())) std::sort(w.begin(), w.end());
  if (!std::is_sorted(r.begin(), r.end())) std::sort(r.begin(), r.end());
  for (size_t i = 1; i < w.size(); ++i)
    if (w[i].first < w[i - 1].second) return false;
  size_t j = 0;
  for (const Range& a : r) {
    while (j < w.size() && w[j].second <= a.first) ++j;
    if (j < w.size() && w[j].first < a.second) return false;
  }
  return true;
}

}  // namespace
}  // namespace ae

extern "C" int model_grad_clip_workspace(const int64_t* sizes, int count, int64_t* bytes) {
  using namespace ae;
  if (!bytes) return fail(AE_EINVAL, "model_grad_clip_workspace: null argument");
  AE_TRY(check_sizes("model_grad_clip_workspace", sizes, count));
  const int64_t parts = parts_of(sizes, count);
  *bytes = parts ? (parts + 1) * 8 : 0;            // and their sum
  return AE_OK;
}

extern "C" int model_grad_clip(void* const* grads, const int64_t* sizes, const int* dtypes, int count, float max_norm, float* norm,
                               void* const* out, void* workspace, void* stream) {
  using namespace ae;
  AE_TRY(check_sizes("model_grad_clip", sizes, count));
  if (!norm && !out) return fail(AE_EINVAL, "model_grad_clip: no output");
  if ((uintptr_t)norm & 3) return fail(AE_EINVAL, "model_grad_clip: misaligned norm");
  if (!(max_norm > 0.0f)) return fail(AE_EINVAL, "model_grad_clip: max_norm must be positive");
  if (count && (!grads || !dtypes)) return fail(AE_EINVAL, "model_grad_clip: null argument");
  for (int k = 0; k < count; ++k) {
    if (dtypes[k] != AE_F32 && dtypes[k] != AE_BF16) return fail(AE_EINVAL, "model_grad_clip: bad dtype of tensor %d", k);
    if (!sizes[k]) continue;
    if (!grads[k] || (out && !out[k])) return fail(AE_EINVAL, "model_grad_clip: tensor %d is null", k);
    if (((uintptr_t)grads[k] | (uintptr_t)(out ? out[k] : nullptr)) % dtype_size(dtypes[k])) return fail(AE_EINVAL, "model_grad_clip: tensor %d is misaligned", k);
  }
  if (out) {
    bool ok = false;
    try {
      ok = apart(grads, out, sizes, dtypes, count);
    } catch (const std::bad_alloc&) {
      return fail(AE_ENOMEM, "model_grad_clip: out of host memory");
    }
    if (!ok) return fail(AE_EINVAL, "model_grad_clip: an output overlaps another, or the gradient of another tensor");
  }
  const int64_t parts = parts_of(sizes, count);
  if (parts > 0x7FFFFFFF) return fail(AE_EINVAL, "model_grad_clip: too many tensors");
  if (parts && (!workspace || ((uintptr_t)workspace & 15))) return fail(AE_EINVAL, "model_grad_clip: workspace is null or not on a 16-byte border");
  hipStream_t s = (hipStream_t)stream;
  double* part = (double*)workspace;
  GradArgs p;
  auto fill = [&](int from, int next) {
    p.count = 0;
    p.chunks = 0;
    for (int k = from; k < next; ++k) {
      if (!sizes[k]) continue;
      const int n = p.count++;
      p.in[n] = grads[k];
      p.out[n] = out ? out[k] : nullptr;
      p.size[n] = sizes[k];
      p.bf16[n] = dtypes[k] == AE_BF16;
      p.end[n] = p.chunks += (int)chunks_of(sizes[k]);
    }
    for (int n = p.count; n < LIST; ++n) p.end[n] = 0x7FFFFFFF;
  };
  int64_t bytes = 0;
  for (int k = 0; k < count; ++k) bytes += sizes[k] * (int64_t)dtype_size(dtypes[k]);
  p.keep = !out ? 0.0f : bytes <= kKeep ? 1.0f : (float)kKeep / (float)bytes;
  int64_t done = 0;
  int launches = 0;
  for (int k = 0; k < count;) {
    int next;
    const int shares = shares_of(launch_range(sizes, count, k, &next));
    if (shares) {
      fill(k, next);
      hipLaunchKernelGGL(k_grad_squares, dim3((unsigned)shares), dim3(NT), 0, s, p, part + done);
      done += shares;
      ++launches;
    }
    k = next;
  }
  AE_TRY(launch_status("grad_clip"));
  if (!out || !launches) {
    if (norm) hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(NT), 0, s, part, (int)parts, norm, (double*)nullptr);
    return launch_status("grad_clip");
  }
  const bool once = launches > kAlone;
  if (once) hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(NT), 0, s, part, (int)parts, norm, part + parts);
  if (once) norm = nullptr;
  for (int k = 0; k < count;) {
    int next;
    const int shares = shares_of(launch_range(sizes, count, k, &next));
    if (shares) {
      if (launches > 1) fill(k, next);
      hipLaunchKernelGGL(k_grad_scale, dim3((unsigned)shares), dim3(NT), 0, s, p, once ? part + parts : part, once ? 1 : (int)parts, max_norm, norm);
      norm = nullptr;
    }
    k = next;
  }
  return launch_status("grad_clip");
}
