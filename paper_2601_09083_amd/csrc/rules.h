// The sampling rules of a sequence as the walks apply them: the penalties of a
// logit, and the tokens of a row that differ from row to row (emitted on this
// walk, or with a bias), which are marked together with the masked ones.
#pragma once

#include "accept.h"

namespace {

constexpr int kPrompt = 0x8000;                       // bit of a count word: in the prompt
constexpr int kCount = 0x7fff;                        // its other bits: times in the output

struct RulesArgs : AcceptArgs {
  const uint16_t* seen;
  const float* repetition;
  const float* frequency;
  const float* presence;
  const int32_t* bias_offsets;
  const int32_t* bias_tokens;
  const float* bias_values;
  const uint32_t* mask;
  int32_t n_bias, mask_words;
};

// The rules of one sequence, then those of the node that it stands on.
struct Row {
  const float* logits;
  const float* noise;    // nullptr: greedy
  const uint16_t* seen;  // nullptr: no counts
  const uint32_t* mask;  // nullptr: everything allowed
  float r, f, p, invT;
  int bias0, bias1;      // its entries of the bias list
};

__device__ inline Row rules_of(const RulesArgs& a, int b, int level) {
  Row w;
  w.noise = a.gumbel ? a.gumbel + (static_cast<int64_t>(b) * (a.Dmax + 1) + level) * a.V : nullptr;
  w.seen = a.seen ? a.seen + static_cast<int64_t>(b) * a.V : nullptr;
  w.r = a.repetition ? a.repetition[b] : 1.f;
  w.f = a.frequency ? a.frequency[b] : 0.f;
  w.p = a.presence ? a.presence[b] : 0.f;
  w.invT = a.invT;
  w.bias0 = w.bias1 = 0;
  if (a.bias_offsets) {
    w.bias0 = min(max(a.bias_offsets[b], 0), a.n_bias);
    w.bias1 = min(max(a.bias_offsets[b + 1], w.bias0), a.n_bias);
  }
  return w;
}

__device__ inline void stand_on(const RulesArgs& a, Row& w, int b, int u) {
  w.logits = a.logits + (static_cast<int64_t>(b) * a.N + u) * a.V;
  w.mask = a.mask ? a.mask + (static_cast<int64_t>(b) * a.N + u) * a.mask_words : nullptr;
}

// The penalised logit; every operation rounded by itself.
__device__ inline float penalised(const Row& w, float y, bool prompt, int count) {
  if (prompt || count > 0) y = y > 0.f ? __fdiv_rn(y, w.r) : mul_rounded(y, w.r);
  y = add_rounded(y, -mul_rounded(w.f, static_cast<float>(count)));
  return count > 0 ? add_rounded(y, -w.p) : y;
}

template <bool kNoise>
__device__ inline float noisy(const Row& w, float y, float g) {
  return kNoise ? add_rounded(mul_rounded(y, w.invT), g) : y;
}

// The best so far in ascending order of the index: a NaN or -inf is never taken.
struct Top {
  float v = -INFINITY;
  int i = 0;
  __device__ void ascending(float x, int j) {
    if (x > v) {
      v = x;
      i = j;
    }
  }
  __device__ unsigned long long key() const { return v > -INFINITY ? pack_key(v, i) : 0ull; }
};

typedef uint16_t u16x4 __attribute__((ext_vector_type(4), aligned(2)));

// Tokens emitted on this walk, and whether the bias list has an entry of them.
struct Path {
  int32_t tok[kMaxLevels];
  int32_t biased[kMaxLevels];
};

// Marks of the tokens of the path and of those with a bias in the chunk [lo, hi),
// whose other marks are written; `bias` is the token at the thread's first entry `at`
// of the bias list (-1: none).  All threads; synchronises, before as well.
__device__ inline void mark_special(const RulesArgs& a, const Row& w, Path& path, int n, int lo, int hi,
                                    uint32_t* skip, int threads, int at, int bias) {
  if (static_cast<int>(threadIdx.x) < n) path.biased[threadIdx.x] = 0;
  __syncthreads();
  auto set = [&](int t) { atomicOr(&skip[(t - lo) >> 5], 1u << ((t - lo) & 31)); };
  auto set_bias = [&](int t) {
    if (t < lo || t >= hi) return;
    set(t);
    for (int i = 0; i < n; ++i)
      if (path.tok[i] == t) path.biased[i] = 1;
  };
  if (static_cast<int>(threadIdx.x) < n) {  // n < 64 <= threads
    const int t = path.tok[threadIdx.x];
    if (t >= lo && t < hi) set(t);
  }
  set_bias(bias);
  for (int i = at + threads; i < w.bias1; i += threads) set_bias(a.bias_tokens[i]);
  __syncthreads();
}

// Marks of the chunk [lo, hi) (lo a multiple of 32) in `skip`: masked entries,
// tokens of the path (n of them) and tokens with a bias.  All threads; synchronises.
__device__ inline void mark(const RulesArgs& a, const Row& w, Path& path, int n, int lo, int hi, uint32_t* skip,
                            int threads) {
  const int words = (hi - lo + 31) / 32;
  const int at = w.bias0 + static_cast<int>(threadIdx.x);
  const int bias = at < w.bias1 ? a.bias_tokens[at] : -1;  // (under way together with the mask)
  for (int i = threadIdx.x; i < words; i += threads) skip[i] = w.mask ? ~w.mask[lo / 32 + i] : 0u;
  mark_special(a, w, path, n, lo, hi, skip, threads, at, bias);
}

// The logit l of one marked token under the rules, its count word given: its path count
// and, where `from` >= 0, the run of its biases that starts at that entry of the list.
__device__ inline float special_logit(const RulesArgs& a, const Row& w, const Path& path, int n, int t, int from,
                                      float l, int word) {
  int count = word & kCount;
  for (int i = 0; i < n; ++i) count += path.tok[i] == t;
  float y = penalised(w, l, word & kPrompt, count);
  if (from >= 0)
    for (int i = from; i < w.bias1 && a.bias_tokens[i] == t; ++i) y = add_rounded(y, a.bias_values[i]);
  return y;
}

// Calls f(token, from) for the marked tokens of [lo, hi) that this thread scores:
// those of the path that the bias list does not have, and the list's.
template <typename F>
__device__ inline void for_special(const RulesArgs& a, const Row& w, const Path& path, int n, int lo, int hi,
                                   int threads, F f) {
  const int tid = threadIdx.x;
  if (tid < n) {  // (one that the bias list has is scored there)
    const int t = path.tok[tid];
    if (t >= lo && t < hi && !path.biased[tid]) f(t, -1);
  }
  for (int k = w.bias0 + tid; k < w.bias1; k += threads) {
    const int t = a.bias_tokens[k];
    if (t >= lo && t < hi && (k == w.bias0 || a.bias_tokens[k - 1] != t)) f(t, k);
  }
}

__device__ inline bool allowed_token(const Row& w, int t) { return !w.mask || ((w.mask[t >> 5] >> (t & 31)) & 1u); }

__device__ inline unsigned long long wave_max(unsigned long long key) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const unsigned long long o = shfl_xor_u64(key, off);
    key = o > key ? o : key;
  }
  return key;
}

// Host side: the rules' own checks, and their place in a walk's arguments.
int check_rules(const srt_rules& r) {
  if (r.reserved != 0 || r.n_bias < 0) return SRT_ERR_INVALID;
  const bool bias = r.bias_offsets || r.bias_tokens || r.bias_values;
  if (bias && (!r.bias_offsets || (r.n_bias > 0 && (!r.bias_tokens || !r.bias_values)))) return SRT_ERR_INVALID;
  return SRT_OK;
}

void take_rules(RulesArgs& a, const srt_rules& r) {
  a.seen = r.seen;
  a.repetition = r.repetition;
  a.frequency = r.frequency;
  a.presence = r.presence;
  a.bias_offsets = r.bias_offsets;
  a.bias_tokens = r.bias_tokens;
  a.bias_values = r.bias_values;
  a.mask = r.mask;
  a.n_bias = r.n_bias;
  a.mask_words = (a.V + 31) / 32;
}

}  // namespace
