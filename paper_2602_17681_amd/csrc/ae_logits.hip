// ae_logits.hip — what comes between an output layer's logits and the choice of a token: penalties for tokens that occurred,
// biases of given tokens, and a mask of what a grammar allows.
// A workgroup takes a slice of a row.  Every column of the slice has a word in LDS: how often the token was answered, whether
// it occurred at all, and which bias it has.  The row's history and list of biases are read by each slice (they are short
// beside it, and in the cache), then the slice passes through registers once.  Bound by memory: 333 x 50 021 in binary32 with mask, 777 tokens
// of history and 5 biases 29.3 us (136 MB, 4.7 TB/s); 256 x 131 072 in bfloat16 without lists 25 us, with 1 024 tokens of history, 16 biases and mask 34, with
// 8 192 tokens 46 (with one of a thread's tokens asked for after the other 53); four rows 4.3 us.
#include <hip/hip_runtime.h>

#include "ae_device.h"
#include "ae_internal.h"
#include "ae_rows.h"

namespace ae {
namespace {

constexpr int NT = 512;
// a column's word: bits 0 .. 19 how often among the answers, bit 20 in the prompt, bits 21 .. 31 place in the list of biases + 1
constexpr uint32_t kCount = (1u << 20) - 1, kPrompt = 1u << 20, kSeen = kCount | kPrompt;
constexpr int AHEAD = 4;                          // tokens of the history that a thread asks for at once
constexpr int kBiasAt = 21, kMaxHistory = kCount, kMaxBias = 2047;

struct AdjustArgs {
  const void* logits;
  int64_t ld, rows;
  int vocab;
  const int* history;
  int n_history;
  const int* n_prompt;
  const float *repetition, *presence, *frequency;
  const int* bias_id;
  const float* bias;
  int n_bias;
  const uint32_t* allowed;
  void* out;
  int64_t ldo;
  int slices;
  int64_t first;
};

// -infinity in the place of the elements whose bit is 0, in the elements' own form
template <typename T, int N>
__device__ __forceinline__ void forbid(uint32_t ok, Piece<T, N>& e) {
#pragma unroll
  for (int i = 0; i < Piece<T, N>::WORDS; ++i) {
    if constexpr (sizeof(T) == 4) {
      e.w[i] = ok >> i & 1 ? e.w[i] : 0xFF800000u;
    } else {
      const uint32_t lo = (uint32_t)((int)(ok << (31 - 2 * i)) >> 31), hi = (uint32_t)((int)(ok << (30 - 2 * i)) >> 31);      // all bits or none
      const uint32_t keep = (lo & 0xFFFFu) | (hi & 0xFFFF0000u);
      e.w[i] = (e.w[i] & keep) | (0xFF80FF80u & ~keep);
    }
  }
}

template <typename T, int NP, bool LISTS>
__global__ __launch_bounds__(NT) void k_logits_adjust(AdjustArgs p) {
  constexpr int VEC = 16 / sizeof(T), S = NT * VEC * NP;       // elements of a piece, columns of a slice
  constexpr uint32_t ALL = (1u << VEC) - 1;
  __shared__ uint4 word4[LISTS ? S / 4 : 1];
  uint32_t* const word = (uint32_t*)word4;
  const int64_t at = p.first + blockIdx.x, row = at / p.slices;
  const int s0 = (int)(at - row * p.slices) * S, mine = p.vocab - s0 < S ? p.vocab - s0 : S;
  const T* z = (const T*)p.logits + row * p.ld + s0;
  Piece<T, VEC> e[NP];
  uint32_t ok[NP];
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int c = (k * NT + (int)threadIdx.x) * VEC;
    if (mine == S) fetch_whole<true>(z + c, e[k]);
    else fetch_row<true, true>(z - s0, s0 + c, p.vocab, e[k]);
    ok[k] = ALL;
    if (p.allowed && c < mine) ok[k] = p.allowed[row * ((p.vocab + 31) / 32) + (s0 + c) / 32] >> (c & 31) & ALL;
  }
  float repetition = 1.0f, presence = 0.0f, frequency = 0.0f;
  if constexpr (LISTS) {
    // the lists' first entries are asked for with the logits
    const int t = threadIdx.x, prompt = p.n_prompt ? p.n_prompt[row] : 0;
    const int bias0 = t < p.n_bias ? p.bias_id[row * p.n_bias + t] : -1;
    const int* const history = p.history + row * p.n_history;
    int token[AHEAD];
    auto ask = [&](int base) {
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) token[k] = base + k * NT + t < p.n_history ? history[base + k * NT + t] : -1;
    };
    ask(0);
    for (int i = threadIdx.x; i < S / 4; i += NT) word4[i] = make_uint4(0, 0, 0, 0);
    if (p.repetition) repetition = p.repetition[row];
    if (p.presence) presence = p.presence[row];
    if (p.frequency) frequency = p.frequency[row];
    __syncthreads();
    auto set_bias = [&](int i, int id) {
      const unsigned c = (unsigned)id - (unsigned)s0;
      if (c < (unsigned)mine) atomicMax(&word[c], (uint32_t)(i + 1) << kBiasAt);       // the last entry of a token counts
    };
    auto count = [&](int i, int id) {
      const unsigned c = (unsigned)id - (unsigned)s0;
      if (c >= (unsigned)mine) return;
      if (i < prompt) atomicOr(&word[c], kPrompt);
      else atomicAdd(&word[c], 1u);
    };
    if (p.n_bias) {
      set_bias(t, bias0);
      for (int i = t + NT; i < p.n_bias; i += NT) set_bias(i, p.bias_id[row * p.n_bias + i]);
      __syncthreads();
    }
    for (int base = 0; base < p.n_history; base += AHEAD * NT) {
      if (base) ask(base);
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) count(base + k * NT + t, token[k]);
    }
    __syncthreads();
  }
  const bool in_place = p.logits == p.out;
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int c = (k * NT + (int)threadIdx.x) * VEC;
    if (c >= mine) continue;
    if (mine < S) settle<true>(s0 + c, p.vocab, e[k]);
    T* const at_out = (T*)p.out + row * p.ldo + s0 + c;
    uint32_t w[VEC], touched = 0;
    if constexpr (LISTS) {
#pragma unroll
      for (int j = 0; j < VEC; j += 4) {
        const uint4 a = word4[(c + j) / 4];
        w[j] = a.x; w[j + 1] = a.y; w[j + 2] = a.z; w[j + 3] = a.w;
        touched |= a.x | a.y | a.z | a.w;
      }
    }
    if (in_place && !touched && ok[k] == ALL) continue;        // stays as it is
    if (touched) {
      float v[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[j] = value(e[k], j);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        if (w[j] & kSeen) v[j] = v[j] > 0.0f ? v[j] / repetition : v[j] * repetition;
        if (w[j] & kCount) v[j] = v[j] - frequency * (float)(w[j] & kCount) - presence;
        if (w[j] >> kBiasAt) v[j] += p.bias[row * p.n_bias + (w[j] >> kBiasAt) - 1];
      }
      make_piece(v, e[k]);
    }
    forbid(ok[k], e[k]);
    if (mine - c >= VEC) put_piece<false>(at_out, e[k]);
    else
      for (int j = 0; j < VEC; ++j)
        if (j < mine - c) Store<T>::st(at_out + j, value(e[k], j));
  }
}

template <typename T, int NP, bool LISTS>
int launch_adjust(AdjustArgs p, hipStream_t s) {
  constexpr int S = NT * 16 / (int)sizeof(T) * NP;
  p.slices = (p.vocab + S - 1) / S;
  const int64_t all = p.rows * p.slices, most = launch_blocks(NT);
  for (; p.first < all; p.first += most) {
    const int64_t left = all - p.first;
    hipLaunchKernelGGL((k_logits_adjust<T, NP, LISTS>), dim3((unsigned)(left < most ? left : most)), dim3(NT), 0, s, p);
  }
  return launch_status("logits_adjust");
}
template <typename T>
int launch_adjust_rows(const AdjustArgs& p, hipStream_t s) {
  constexpr int E = sizeof(T) / 2;               // pieces for 4 096 columns
  if (!p.n_history && !p.n_bias) return launch_adjust<T, 2 * E, false>(p, s);
  // slices of 4 096 columns where they are fewer than 1 024, as measured when 4 rows of 131 072 took 5.2 us (8 192 columns 5.6): 64 of 50 021 8.7
  // (9.9), 32 of 131 072 7.3 (7.2), 128 of 131 072 23 (21), 128 of 50 021 14.6 (13.8), 512 of 32 000 25 (21); 333 x 50 021 by 256 threads 40 (2 048 columns), 38 (4 096), 48 (8 192), by 512 37
  if (p.rows * ((p.vocab + 4095) / 4096) < 1024) return launch_adjust<T, E, true>(p, s);
  return launch_adjust<T, 2 * E, true>(p, s);
}

}  // namespace
}  // namespace ae

extern "C" int model_logits_adjust(const void* logits, int64_t rows, int64_t vocab, int64_t ld, int dtype, const int* history, int64_t n_history,
                                   const int* n_prompt, const float* repetition, const float* presence, const float* frequency,
                                   const int* bias_id, const float* bias, int n_bias, const uint32_t* allowed, void* out, int64_t ldo,
                                   void* stream) {
  using namespace ae;
  if (dtype != AE_F32 && dtype != AE_BF16) return fail(AE_EINVAL, "model_logits_adjust: bad dtype");
  if (rows < 0 || rows > ((int64_t)1 << 24)) return fail(AE_EINVAL, "model_logits_adjust: rows must be 0 .. 2^24");
  if (vocab < 1 || vocab > ((int64_t)1 << 20)) return fail(AE_EINVAL, "model_logits_adjust: vocab must be 1 .. 2^20");
  if (ld < vocab || ldo < vocab || ld >= ((int64_t)1 << 40) || ldo >= ((int64_t)1 << 40)) return fail(AE_EINVAL, "model_logits_adjust: rows must not overlap");
  if (n_history < 0 || n_history > kMaxHistory) return fail(AE_EINVAL, "model_logits_adjust: n_history must be 0 .. 2^20 - 1");
  if (n_bias < 0 || n_bias > kMaxBias) return fail(AE_EINVAL, "model_logits_adjust: n_bias must be 0 .. 2047");
  if (rows == 0) return AE_OK;
  if (!logits || !out || (n_history && !history) || (n_bias && (!bias_id || !bias))) return fail(AE_EINVAL, "model_logits_adjust: null argument");
  if (((uintptr_t)logits | (uintptr_t)out) % dtype_size(dtype)) return fail(AE_EINVAL, "model_logits_adjust: misaligned logits");
  if (((uintptr_t)history | (uintptr_t)n_prompt | (uintptr_t)repetition | (uintptr_t)presence | (uintptr_t)frequency | (uintptr_t)bias_id | (uintptr_t)bias |
       (uintptr_t)allowed) & 3)
    return fail(AE_EINVAL, "model_logits_adjust: misaligned list");
  if (logits == out && ld != ldo) return fail(AE_EINVAL, "model_logits_adjust: a result in the logits' place has their stride");
  const AdjustArgs p = {logits, ld, rows, (int)vocab, history, (int)n_history, n_prompt, repetition, presence, frequency,
                        bias_id, bias, n_bias, allowed, out, ldo, 0, 0};
  return dtype == AE_BF16 ? launch_adjust_rows<bf16_t>(p, (hipStream_t)stream) : launch_adjust_rows<float>(p, (hipStream_t)stream);
}
