// Sampling rules in the acceptance walk: penalties for repeated tokens, biases
// and masks, and the token counts that the penalties read.
//
// Method: the walk of accept.hip (Sections 1 and 3 of the paper: the policy's
// own choice at every node, which keeps its distribution) where the policy
// decodes under per-request rules.  What a token has been said before depends
// on the path that the walk has taken, so the rules belong to the walk: they are
// applied to the rows that it visits and to nothing else, and no modified
// logits are stored.
//
// GPU design.  A level kernel as accept.hip's: a visited row is split into up
// to 32 chunks, one workgroup each, which first takes the step of the level
// before.  Per entry it streams the logit, the noise and a 16-bit count word
// (10 bytes with noise, where the plain walk reads 8); the mask is a bit per
// entry.  The tokens that differ from row to row of a sequence -- those emitted
// on this walk, those with a bias -- are few: the workgroup marks them together
// with the masked entries in a bitmap of its chunk in LDS, the streaming pass
// skips marked entries (a quartet of them is not read), and a thread per marked
// token then scores it with its path count and bias.  Entries that were never
// said (count word 0) take no arithmetic of the penalties.
#include "accept.h"

namespace {

constexpr int kMaxChunk = 65536;                      // entries of a chunk, at most
constexpr int64_t kMaxVocab = int64_t(kMaxChunk) * kMaxChunks;
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

// Marks of the chunk [lo, hi) (lo a multiple of 32) in `skip`: masked entries,
// tokens of the path (n of them) and tokens with a bias.  All threads; synchronises.
__device__ inline void mark(const RulesArgs& a, const Row& w, Path& path, int n, int lo, int hi, uint32_t* skip,
                            int threads) {
  const int words = (hi - lo + 31) / 32;
  const int at = w.bias0 + static_cast<int>(threadIdx.x);
  const int bias = at < w.bias1 ? a.bias_tokens[at] : -1;  // (under way together with the mask)
  for (int i = threadIdx.x; i < words; i += threads) skip[i] = w.mask ? ~w.mask[lo / 32 + i] : 0u;
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

// Score of one marked token that is allowed, with its path count and, where
// `from` >= 0, the run of its biases that starts at that entry of the list.
template <bool kNoise>
__device__ inline void special(const RulesArgs& a, const Row& w, const Path& path, int n, int t, int from,
                               unsigned long long& key) {
  const uint32_t allowed = w.mask ? w.mask[t >> 5] >> (t & 31) : 1u;
  const int word = w.seen ? w.seen[t] : 0;
  const float l = w.logits[t], g = kNoise ? w.noise[t] : 0.f;
  int count = word & kCount;
  for (int i = 0; i < n; ++i) count += path.tok[i] == t;
  float y = penalised(w, l, word & kPrompt, count);
  if (from >= 0)
    for (int i = from; i < w.bias1 && a.bias_tokens[i] == t; ++i) y = add_rounded(y, a.bias_values[i]);
  const float x = noisy<kNoise>(w, y, g);
  if ((allowed & 1u) && x > -INFINITY) key = max(key, pack_key(x, t));
}

// This thread's best entry of [lo, hi) of one row, packed (0: none).  kUnroll
// quartets are read at a time: 5 make a chunk of a 152k vocabulary (4752 entries,
// 256 threads) one batch (10% less time than 4).
template <bool kNoise, int kUnroll>
__device__ inline unsigned long long part_best(const RulesArgs& a, const Row& w, const Path& path, int n,
                                               const uint32_t* skip, int lo, int hi, int threads) {
  const int tid = threadIdx.x;
  const f32x4u* r4 = reinterpret_cast<const f32x4u*>(w.logits);
  const f32x4u* g4 = reinterpret_cast<const f32x4u*>(w.noise);
  const u16x4* s4 = reinterpret_cast<const u16x4*>(w.seen);
  Top best;
  auto one = [&](float l, float g, int word, bool out, int j) {
    if (word) l = penalised(w, l, word & kPrompt, word & kCount);
    const float x = noisy<kNoise>(w, l, g);
    best.ascending(out ? -INFINITY : x, j);
  };
  auto four = [&](const f32x4& x, const f32x4& g, const u16x4& s, uint32_t out, int j) {
    one(x.x, g.x, s.x, out & 1u, j);
    one(x.y, g.y, s.y, out & 2u, j + 1);
    one(x.z, g.z, s.z, out & 4u, j + 2);
    one(x.w, g.w, s.w, out & 8u, j + 3);
  };
  auto marks = [&](int i) { return (skip[(4 * i - lo) >> 5] >> ((4 * i) & 31)) & 15u; };
  const int e4 = hi / 4;
  int i = lo / 4 + tid;
  for (; i < e4; i += kUnroll * threads) {
    f32x4 x[kUnroll], g[kUnroll];
    u16x4 s[kUnroll];
    uint32_t out[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int at = i + k * threads;
      out[k] = at < e4 ? marks(at) : 15u;
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      // a quartet of which nothing is left is not read (the first one's line is)
      const int at = out[k] == 15u ? i : i + k * threads;
      x[k] = __builtin_nontemporal_load(&r4[at]);
      g[k] = f32x4{0.f, 0.f, 0.f, 0.f};
      s[k] = u16x4{0, 0, 0, 0};
      if (kNoise) g[k] = __builtin_nontemporal_load(&g4[at]);
      if (w.seen) s[k] = s4[at];
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) four(x[k], g[k], s[k], out[k], 4 * (i + k * threads));
  }
  const int j = 4 * e4 + tid;  // the row's last one to three entries
  unsigned long long key = best.key();
  if (j < hi && !((skip[(j - lo) >> 5] >> ((j - lo) & 31)) & 1u)) {
    float y = w.logits[j];
    const int word = w.seen ? w.seen[j] : 0;
    if (word) y = penalised(w, y, word & kPrompt, word & kCount);
    const float x = noisy<kNoise>(w, y, kNoise ? w.noise[j] : 0.f);
    if (x > -INFINITY) key = max(key, pack_key(x, j));
  }
  if (tid < n) {  // (one that the bias list has is scored there)
    const int t = path.tok[tid];
    if (t >= lo && t < hi && !path.biased[tid]) special<kNoise>(a, w, path, n, t, -1, key);
  }
  for (int k = w.bias0 + tid; k < w.bias1; k += threads) {
    const int t = a.bias_tokens[k];
    if (t >= lo && t < hi && (k == w.bias0 || a.bias_tokens[k - 1] != t)) special<kNoise>(a, w, path, n, t, k, key);
  }
  return key;
}

__device__ inline unsigned long long wave_max(unsigned long long key) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const unsigned long long o = shfl_xor_u64(key, off);
    key = o > key ? o : key;
  }
  return key;
}

// decide() of accept.h; a row of which nothing is left gives token -1 and no child.
__device__ inline Step decide_rules(const RulesArgs& a, int b, int u, int level, int lane) {
  Step st = decide(a, b, u, level, lane);
  if (st.tok < 0) st.child = -1;
  return st;
}

__device__ inline void record_rules(const RulesArgs& a, int b, int level, const Step& st) {
  const int64_t orow = static_cast<int64_t>(b) * (a.Dmax + 1);
  a.out_tokens[orow + level] = st.tok;
  if (st.child >= 0) {
    a.out_nodes[orow + level] = st.child;
    a.cur[((level + 1) & 1) * a.B + b] = st.child;
    const int pos = atomicAdd(&a.n_act[level + 1], 1);
    a.act[((level + 1) & 1) * a.B + pos] = b;
  } else {
    a.n_accepted[b] = level;
    if (a.n_emitted) a.n_emitted[b] = level + (st.tok >= 0);
  }
}

// As accept_level_kernel: one chunk of the visited row of one walker.  (Later
// levels on 1024 to 4096 workgroups that stride over the chunks: 423 to 433 us
// for the batch that takes 371 with a workgroup for every chunk.)
template <bool kNoise>
__global__ __launch_bounds__(kThreads) void rules_level_kernel(RulesArgs a, int level) {
  __shared__ uint32_t skip[kMaxChunk / 32];
  __shared__ Path path;
  __shared__ unsigned long long s_key[kThreads / SRT_WAVE];
  __shared__ int s_child;
  const int g = blockIdx.x, tid = threadIdx.x, lv = level - 1;
  const int slot = g / a.n_chunks, c = g - slot * a.n_chunks;
  if (level > 0 && slot >= a.n_act[lv]) return;
  const int b = level == 0 ? slot : min(max(a.act[(lv & 1) * a.B + slot], 0), a.B - 1);
  Row w = rules_of(a, b, level);  // (under way together with what the step reads)
  int u = 0;
  if (level == 0) {  // every sequence; the walk's state is reset here
    if (g == 0 && tid <= kMaxLevels) a.n_act[tid] = tid == 0 ? a.B : 0;
    if (c == 0) {
      const int64_t orow = static_cast<int64_t>(b) * (a.Dmax + 1);
      for (int k = tid; k <= a.Dmax; k += kThreads) {
        a.out_tokens[orow + k] = -1;
        a.out_nodes[orow + k] = -1;
      }
      if (tid == 0) {
        a.act[b] = b;  // level 0, parity 0
        a.cur[b] = 0;
      }
    }
  } else {
    if (tid < SRT_WAVE) {
      const int prev = min(max(a.cur[(lv & 1) * a.B + b], 0), a.N - 1);
      // the path: earlier launches have written all of it but the last token
      if (tid < lv) path.tok[tid] = a.out_tokens[static_cast<int64_t>(b) * (a.Dmax + 1) + tid];
      const Step st = decide_rules(a, b, prev, lv, tid);
      if (tid == 0) {
        path.tok[lv] = st.tok;
        if (c == 0) record_rules(a, b, lv, st);
        s_child = st.child;
      }
    }
    __syncthreads();
    u = s_child;
    if (u < 0) return;
  }
  const int lo = c * a.chunk, hi = min(a.V, lo + a.chunk);
  stand_on(a, w, b, u);
  mark(a, w, path, level, lo, hi, skip, kThreads);
  unsigned long long key = wave_max(part_best<kNoise, 5>(a, w, path, level, skip, lo, hi, kThreads));
  if (tid % SRT_WAVE == 0) s_key[tid / SRT_WAVE] = key;
  __syncthreads();
  if (tid == 0) {
#pragma unroll
    for (int i = 0; i < kThreads / SRT_WAVE; ++i) key = max(key, s_key[i]);
    a.cand[(static_cast<int64_t>(level & 1) * a.B + b) * kMaxChunks + c] = key;
  }
}

// The step of the last level (Dmax), one wave per walker.
__global__ __launch_bounds__(kWalkWaves * SRT_WAVE) void rules_walk_kernel(RulesArgs a, int level) {
  const int lane = threadIdx.x % SRT_WAVE;
  const int slot = blockIdx.x * kWalkWaves + threadIdx.x / SRT_WAVE;
  if (slot >= a.n_act[level]) return;
  const int b = min(max(a.act[(level & 1) * a.B + slot], 0), a.B - 1);
  const int u = min(max(a.cur[(level & 1) * a.B + b], 0), a.N - 1);
  const Step st = decide_rules(a, b, u, level, lane);
  if (lane == 0) record_rules(a, b, level, st);
}

// Short rows: a workgroup walks one sequence in one launch, as accept_short_kernel.
template <bool kNoise>
__global__ __launch_bounds__(1024) void rules_short_kernel(RulesArgs a) {
  __shared__ uint32_t skip[(kShortRow + 31) / 32];
  __shared__ Path path;
  __shared__ int32_t s_par[kMaxN], s_tok[kMaxN];
  __shared__ unsigned long long s_key[1024 / SRT_WAVE];
  const int b = blockIdx.x, tid = threadIdx.x, threads = blockDim.x;
  const int lane = tid % SRT_WAVE, wave = tid / SRT_WAVE;
  const int64_t tr = static_cast<int64_t>(b) * a.N, orow = static_cast<int64_t>(b) * (a.Dmax + 1);
  const int n = min(max(a.n_nodes[b], 1), a.N);
  for (int c = tid; c < n; c += threads) {
    s_par[c] = a.tree_parent[tr + c];
    s_tok[c] = a.tree_tokens[tr + c];
  }
  int u = 0, k = 0, tok;
  for (;; ++k) {
    Row w = rules_of(a, b, k);
    stand_on(a, w, b, u);
    mark(a, w, path, k, 0, a.V, skip, threads);  // (also orders the staged tree and the path)
    unsigned long long key = wave_max(part_best<kNoise, 2>(a, w, path, k, skip, 0, a.V, threads));
    if (lane == 0) s_key[wave] = key;
    __syncthreads();
    key = wave_max(lane < threads / SRT_WAVE ? s_key[lane] : 0ull);
    tok = key ? key_token(key) : -1;
    int child = -1;
    if (k < a.Dmax && tok >= 0) {  // children of u have larger indices
      for (int c0 = u + 1; c0 < n && child < 0; c0 += SRT_WAVE) {
        const int c = c0 + lane;
        const unsigned long long hit = __ballot(c < n && s_par[c] == u && s_tok[c] == tok);
        if (hit) child = c0 + __ffsll(static_cast<long long>(hit)) - 1;
      }
    }
    if (tid == 0) {
      a.out_tokens[orow + k] = tok;
      a.out_nodes[orow + k] = child;  // -1 at the last step
      if (child >= 0) path.tok[k] = tok;
    }
    if (child < 0) break;
    u = child;
  }
  if (tid == 0) {
    a.n_accepted[b] = k;
    if (a.n_emitted) a.n_emitted[b] = k + (tok >= 0);
  }
  for (int j = k + 1 + tid; j <= a.Dmax; j += threads) {
    a.out_tokens[orow + j] = -1;
    a.out_nodes[orow + j] = -1;
  }
}

// ---------------------------------------------------------------------------
// Token counts
// ---------------------------------------------------------------------------
struct SeenArgs {
  uint16_t* seen;
  const int32_t* tokens;
  const int32_t* lengths;
  int32_t B, V, T, prompt;
};

__device__ inline uint16_t counted(uint16_t old, int n, bool prompt) {
  if (prompt) return old | kPrompt;
  return static_cast<uint16_t>((old & kPrompt) | min((old & kCount) + n, kCount));
}

constexpr int kSeenStep = SRT_WAVE;  // tokens of a sequence up to which one wave enters them

// Few tokens: a wave per sequence, a lane per token; the first lane of those
// with the same token writes its word.
__global__ __launch_bounds__(256) void seen_step_kernel(SeenArgs a) {
  const int b = blockIdx.x * (256 / SRT_WAVE) + threadIdx.x / SRT_WAVE;
  if (b >= a.B) return;
  const int lane = threadIdx.x % SRT_WAVE;
  const int len = min(max(a.lengths[b], 0), a.T);
  int t = lane < len ? a.tokens[static_cast<int64_t>(b) * a.T + lane] : -1;
  if (t >= a.V) t = -1;
  uint16_t* word = a.seen + static_cast<int64_t>(b) * a.V + max(t, 0);
  const uint16_t old = t >= 0 ? *word : uint16_t(0);
  int n = 0, first = -1;
  for (int j = 0; j < len; ++j) {
    const bool same = __builtin_amdgcn_readlane(t, j) == t;
    n += same;
    if (same && first < 0) first = j;
  }
  if (t >= 0 && first == lane) *word = counted(old, n, a.prompt);
}

// Many tokens, or rows built anew: a workgroup per chunk of a row counts the
// sequence's tokens `from` .. `from` + kSeenTokens - 1 of its chunk in LDS, two
// 16-bit counters a word (which hold that many), and writes the chunk: all of it,
// eight words of the row a store, or the words that a token touched.  A row is
// written at 3.4 TB/s with 32-bit counters and a store for every word, 5.1 so (256
// rows of 152064 words, prompts of up to 4096 tokens: 24.1 and 15.8 us).
constexpr int kSeenChunk = 32768;
constexpr int kSeenTokens = 65535;
constexpr int kSeenThreads = 1024;
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef uint16_t u16x8u __attribute__((ext_vector_type(8), aligned(2)));  // rows start at any word

template <bool kReset>
__global__ __launch_bounds__(kSeenThreads) void seen_rows_kernel(SeenArgs a, int chunks, int from) {
  __shared__ u16x8 cnt[kSeenChunk / 8];
  uint32_t* const pairs = reinterpret_cast<uint32_t*>(cnt);
  const int b = blockIdx.x / chunks, lo = (blockIdx.x - b * chunks) * kSeenChunk;
  const int n = min(a.V - lo, kSeenChunk), n8 = (n + 7) / 8;
  for (int i = threadIdx.x; i < n8; i += kSeenThreads) cnt[i] = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
  __syncthreads();
  const int len = min(min(max(a.lengths[b], 0), a.T) - from, kSeenTokens);
  const int32_t* tok = a.tokens + static_cast<int64_t>(b) * a.T + from;
  for (int i = threadIdx.x; i < len; i += kSeenThreads) {
    const int t = tok[i];
    const uint32_t at = static_cast<uint32_t>(t) - static_cast<uint32_t>(lo);
    if (t >= 0 && at < static_cast<uint32_t>(n)) atomicAdd(&pairs[at >> 1], 1u << (16 * (at & 1)));
  }
  __syncthreads();
  uint16_t* row = a.seen + static_cast<int64_t>(b) * a.V + lo;
  for (int i = threadIdx.x; i < n8; i += kSeenThreads) {
    const u16x8 c = cnt[i];
    if (kReset && 8 * i + 8 <= n) {
      const u16x8 most = {kCount, kCount, kCount, kCount, kCount, kCount, kCount, kCount};
      u16x8 w = __builtin_elementwise_min(c, most);
      if (a.prompt) {
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = c[k] ? kPrompt : 0;
      }
      *reinterpret_cast<u16x8u*>(row + 8 * i) = w;
      continue;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int at = 8 * i + k;
      if (at < n && (kReset || c[k])) row[at] = c[k] ? counted(kReset ? uint16_t(0) : row[at], c[k], a.prompt) : uint16_t(0);
    }
  }
}

}  // namespace

extern "C" int srt_accept_rules(int32_t B, int32_t N, int32_t V, int32_t Dmax, const float* logits,
                                const float* gumbel, float inv_temperature, const srt_rules* rules,
                                const int32_t* tree_tokens, const int32_t* tree_parent, const int32_t* n_nodes,
                                int32_t* n_accepted, int32_t* out_tokens, int32_t* out_nodes, int32_t* n_emitted,
                                void* scratch, size_t scratch_bytes, void* stream) {
  if (!rules || rules->reserved != 0 || rules->n_bias < 0) return SRT_ERR_INVALID;
  const bool bias = rules->bias_offsets || rules->bias_tokens || rules->bias_values;
  if (bias && (!rules->bias_offsets || (rules->n_bias > 0 && (!rules->bias_tokens || !rules->bias_values))))
    return SRT_ERR_INVALID;
  int st = check_args(B, N, V, Dmax, logits, inv_temperature, tree_tokens, tree_parent, n_nodes, n_accepted,
                      out_tokens, out_nodes);
  if (st != SRT_OK || B == 0) return st;
  if (V > kMaxVocab) return SRT_ERR_UNSUPPORTED;
  const bool short_rows = static_cast<int64_t>(V) * (gumbel ? 2 : 1) <= kShortRow;
  const unsigned short_threads = V <= kNarrowRow ? 256 : 1024;
  if (!scratch || scratch_bytes < srt_accept_scratch_bytes(B)) return SRT_ERR_CAPACITY;
  if (reinterpret_cast<uintptr_t>(scratch) % 256) return SRT_ERR_INVALID;

  RulesArgs a;
  static_cast<AcceptArgs&>(a) =
      walk_args(B, N, V, Dmax, logits, gumbel, inv_temperature, tree_tokens, tree_parent, n_nodes, n_accepted,
                out_tokens, out_nodes, n_emitted, static_cast<char*>(scratch), 32);
  a.seen = rules->seen;
  a.repetition = rules->repetition;
  a.frequency = rules->frequency;
  a.presence = rules->presence;
  a.bias_offsets = rules->bias_offsets;
  a.bias_tokens = rules->bias_tokens;
  a.bias_values = rules->bias_values;
  a.mask = rules->mask;
  a.n_bias = rules->n_bias;
  a.mask_words = (V + 31) / 32;
  const int64_t grid = static_cast<int64_t>(B) * a.n_chunks;
  if (!(short_rows ? launchable(B, short_threads) : launchable(grid, kThreads))) return SRT_ERR_UNSUPPORTED;

  hipStream_t s = as_stream(stream);
  if (short_rows) {
    if (gumbel) rules_short_kernel<true><<<static_cast<unsigned>(B), short_threads, 0, s>>>(a);
    else rules_short_kernel<false><<<static_cast<unsigned>(B), short_threads, 0, s>>>(a);
    return launch_status();
  }
  for (int level = 0; level <= Dmax && st == SRT_OK; ++level) {
    if (gumbel) rules_level_kernel<true><<<static_cast<unsigned>(grid), kThreads, 0, s>>>(a, level);
    else rules_level_kernel<false><<<static_cast<unsigned>(grid), kThreads, 0, s>>>(a, level);
    st = launch_status();
  }
  if (st == SRT_OK) {
    rules_walk_kernel<<<static_cast<unsigned>((B + kWalkWaves - 1) / kWalkWaves), kWalkWaves * SRT_WAVE, 0, s>>>(a,
                                                                                                               Dmax);
    st = launch_status();
  }
  return st;
}

extern "C" int srt_seen_add(uint16_t* seen, int32_t B, int32_t V, const int32_t* tokens, const int32_t* lengths,
                            int32_t stride, int32_t prompt, int32_t reset, void* stream) {
  if (B < 0 || V < 1 || stride < 1 || (prompt & ~1) || (reset & ~1)) return SRT_ERR_INVALID;
  if (B == 0) return SRT_OK;
  if (!seen || !tokens || !lengths) return SRT_ERR_INVALID;
  const int64_t chunks = (static_cast<int64_t>(V) + kSeenChunk - 1) / kSeenChunk;
  const bool few = !reset && stride <= kSeenStep;
  const int64_t step_grid = (static_cast<int64_t>(B) + 3) / 4;
  if (!(few ? launchable(step_grid, 256) : launchable(chunks * B, kSeenThreads))) return SRT_ERR_UNSUPPORTED;
  const SeenArgs a = {seen, tokens, lengths, B, V, stride, prompt};
  hipStream_t s = as_stream(stream);
  if (few) {
    seen_step_kernel<<<static_cast<unsigned>(step_grid), 256, 0, s>>>(a);
    return launch_status();
  }
  // (longer rows of tokens than a counter holds enter in pieces)
  for (int64_t from = 0; from < stride; from += kSeenTokens) {
    const unsigned grid = static_cast<unsigned>(chunks * B);
    if (reset && from == 0)
      seen_rows_kernel<true><<<grid, kSeenThreads, 0, s>>>(a, static_cast<int>(chunks), 0);
    else
      seen_rows_kernel<false><<<grid, kSeenThreads, 0, s>>>(a, static_cast<int>(chunks), static_cast<int>(from));
  }
  return launch_status();
}
