// Acceptance walk where the policy samples with a temperature, top-k, top-p and
// min-p of each sequence's own, from given Gumbel noise.
//
// Method: the walk of accept.hip (Sections 1 and 3 of the paper: the policy's own
// choice at every node, which keeps its distribution).  The policy's distribution
// is the softmax of the scores z = y * inv_temperature (y: the logit under the
// rules), cut off behind the first top_k tokens of the order (score descending,
// token ascending), behind the smallest set of them whose mass reaches top_p of
// theirs, and below min_p of the largest probability.  Each cut leaves a prefix of
// that order, so the kept set is all tokens from some last one up, and the choice
// is arg-max of z + noise over it, which needs no normalisation and is exact
// whatever order the sums are taken in -- only the place of the top-p cut depends
// on sums, and those are held in 64 bits.
//
// GPU design.  One workgroup walks one sequence, and its levels follow one another, so
// what bounds a batch is one CU's time for a row times the longest walk's levels: of a
// 152k vocabulary (608 KB) 18 us a row for the arg-max with noise, 14 with min-p, 16 with
// a top-k, 20 with a top-p or a top-k of 200 and a top-p, and under rules 5 to 15 more;
// 256 sequences of up to 13 rows 310 to 370 us, which goes by the inputs.  A CU's loads
// come at 75 to 80 GB/s, with one batch under way as with seven, which is 8 us of a row;
// the sum for a top-p is bound by the vector unit (one operation of every entry takes 1
// us).  A row is read from HBM once: its maximum, its sum of exp(z - max), and the
// maximum of every thread's every few entries (a segment) are taken in one pass.  A count
// and a lower bound of the mass over the segments' maxima give a score below which
// nothing can be kept; segments that reach it are read again, which a row that is sure of
// its tokens has few of, and their entries from that score up are listed in LDS, most
// often a hundred.
//
// The choice from a list or from the row is drawn: the best of all of them is the choice
// if it is kept itself, which takes the mass before it in the order, a sum without a
// sort; if it is not, the kept ones lie before it, and the best of those is next.  A list
// is sorted only where it is long and the mass of its first top_k is asked for.  Noise is
// read at the listed tokens alone, or once a draw.  (Long lists narrowed down by
// histograms of LDS atomics: flat rows of 64 sequences 226 us a pass; 111 to 128 now.)
// Sequences that cut nothing, or without noise, take the plain arg-max in one pass.
#include "rules.h"

namespace {

constexpr int kList = 4096;       // candidates that are listed in LDS
constexpr int kDraws = 12;        // of a long list's choice, before the last kept token is searched for
constexpr int kSegs = 16;         // segments of a thread, at most
constexpr int kSegsAt = 4;        // of them looked at together
constexpr int kUnroll = 4;        // quartets of a thread in a batch
// Batches whose registers are loaded or used (256 walks of 152k entries, 64 under rules,
// 64 of flat rows, 4 of 1024 entries, the same inputs: 309, 377, 119, 33.1 us a pass; 3:
// 317, 380, 123, 33.3; 4 of them, or 3 where there is noise: 321, 386, 123, 34.5.  The code
// has a copy of a batch's work for each).
constexpr int kAhead = 2;
constexpr int kAgain = 4;         // quartets of a thread that are read again together
// Batches after which a sum over a row is looked at (64 flat rows of 152k with a top-p of
// 0.999, 0.9, 0.5: 60, 117, 230 us; at the row's end alone 71, 123, 231).
constexpr int kStage = 4;
constexpr int kMost = 512;        // threads
constexpr int kSegBins = 512;     // of the segments' maxima, 1 / 8 of the score wide
constexpr int kMassBits = 44;     // of a bin's word: mass in units of 2^-24 below, count above
constexpr int64_t kMaxVocab = int64_t(1) << 21;
constexpr int64_t kMaxRuled = int64_t(1) << 18;  // a row's marks are held in LDS
constexpr int kSaid = 4096;       // tokens with a count word that are scored apart from the stream
constexpr int kApart = kSaid + 512;  // and with them those of the path and of the bias list
constexpr int kStaged = 512;      // entries of a bias list that are held in LDS
// Rows up to which 256 threads walk (the same inputs: 4 walks of 1024 entries 33 us a pass,
// 38 with 512 threads; 256 of 152k 371, 309 with 512).
constexpr int kShortVocab = 4096;
constexpr float kLog2e = 1.44269504088896341f;
constexpr double kUnit = 1125899906842624.0;  // 2^50 units a weight of 1: a list of 4096 stays below 2^63
static_assert(kList <= 4096, "sums of units");

struct SampleArgs : RulesArgs {
  const float* inv_temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
};

typedef unsigned long long u64;

// The larger of two that are no NaN (fmaxf would quiet each operand first).
__device__ __forceinline__ float larger_of(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// The weight of a score at distance x from the largest.  In 32 bits: the product is off by
// half a unit in its last place, the weight by up to 1e-6 of itself (from a distance of 11 on;
// nearer by less); a power in 64 bits is many operations, of which one for every entry of a
// 152k row takes 1 us.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// Reductions and prefix sums over the wave by DPP moves, as wave_sum of common.h (a
// few cycles a step, where a shuffle of 64 bits goes through the LDS crossbar twice).
template <int kCtrl, int kRows>
__device__ __forceinline__ u64 from_lane(u64 x) {  // 0 where there is none
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(x), kCtrl, kRows, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(x >> 32), kCtrl, kRows, 0xf, false);
  return static_cast<u64>(hi) << 32 | lo;
}
template <typename Fn>
__device__ __forceinline__ u64 wave_steps(u64 x, Fn join) {  // inclusive over the lanes up to each
  x = join(x, from_lane<0x111, 0xf>(x));  // row_shr:1
  x = join(x, from_lane<0x112, 0xf>(x));
  x = join(x, from_lane<0x114, 0xf>(x));
  x = join(x, from_lane<0x118, 0xf>(x));
  x = join(x, from_lane<0x142, 0xa>(x));  // row_bcast:15
  return join(x, from_lane<0x143, 0xc>(x));  // row_bcast:31
}
__device__ __forceinline__ u64 last_lane(u64 x) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(x), SRT_WAVE - 1);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(x >> 32), SRT_WAVE - 1);
  return static_cast<u64>(hi) << 32 | lo;
}
__device__ __forceinline__ u64 wave_top(u64 x) {
  return last_lane(wave_steps(x, [](u64 p, u64 q) { return p > q ? p : q; }));
}
__device__ __forceinline__ u64 wave_scan(u64 x) {
  return wave_steps(x, [](u64 p, u64 q) { return p + q; });
}
__device__ __forceinline__ double wave_scan(double x) {
  return __builtin_bit_cast(double, wave_steps(__builtin_bit_cast(u64, x), [](u64 p, u64 q) {
    return __builtin_bit_cast(u64, __builtin_bit_cast(double, p) + __builtin_bit_cast(double, q));
  }));
}
__device__ __forceinline__ double last_lane(double x) {
  return __builtin_bit_cast(double, last_lane(__builtin_bit_cast(u64, x)));
}
template <int kCtrl, int kRows>
__device__ __forceinline__ float larger_of_lane(float x) {  // (where there is none, x)
  const int y = __float_as_int(x);
  return larger_of(x, __int_as_float(__builtin_amdgcn_update_dpp(y, y, kCtrl, kRows, 0xf, false)));
}
__device__ __forceinline__ float wave_largest(float x) {
  x = larger_of_lane<0x111, 0xf>(x);
  x = larger_of_lane<0x112, 0xf>(x);
  x = larger_of_lane<0x114, 0xf>(x);
  x = larger_of_lane<0x118, 0xf>(x);
  x = larger_of_lane<0x142, 0xa>(x);
  x = larger_of_lane<0x143, 0xc>(x);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), SRT_WAVE - 1));
}

__device__ __forceinline__ float score_of(u64 key) {
  const uint32_t u = static_cast<uint32_t>(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}

// Loads past the buffer's bytes read 0.  (`base` is the same for all lanes.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const float* base, int bytes) {
  const uint64_t at = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<int>(at));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<int>(at >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(static_cast<uint64_t>(hi) << 32 | lo), 0, bytes, 0x00020000);
}
__device__ __forceinline__ f32x4 load_quartet(__amdgpu_buffer_rsrc_t row, uint32_t at) {
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  const i32x4 x = __builtin_amdgcn_raw_buffer_load_b128(row, at, 0, 0);
  return __builtin_bit_cast(f32x4, x);
}

// What the workgroup shares.
struct Lds {
  u64 list[kList];  // packed candidates (score, token)
  float seg[kSegs * kMost];
  u64 segbin[kSegBins];
  Path path;
  int32_t par[kMaxN], tok[kMaxN];
  u64 red[2][kMost / SRT_WAVE];
  double redd[2][kMost / SRT_WAVE];
  float redm[kMost / SRT_WAVE];
  u64 found;
  uint16_t work[kList];  // segments that are read again
  int32_t n, m;
};

template <bool kRules>
struct Walker {
  const SampleArgs& a;
  Lds& s;
  // Under rules: marked entries; the marked tokens and their scores, first n_said
  // with a count word (-1: more than there is room for, and the stream reads the
  // words), then those of the path and of the bias list (-1: too long a list).
  uint32_t* skip;
  int32_t* apart;
  float* apart_z;
  uint16_t* said_word;
  int n_said, n_special;
  Row w;
  int n;                 // tokens emitted on this walk
  int tid, threads, lane, wave, waves;
  int e4, full;          // quartets of a row; batches that are whole
  int seg_batches, batch_segs;  // batches of a segment, or segments of a batch
  int parity;            // of the reductions' arrays: the next one's writes meet no reads of the last one's
  float M;               // largest score of the row

  // The best of a set of tokens by score and noise (packed, 0 if there is none), and
  // its place in the order.
  struct Draw {
    u64 best = 0, at = 0;
    float most = -INFINITY;
    __device__ __forceinline__ void any(float z, float x, int j) {
      const u64 key = pack_key(x, j);
      if (!(x > -INFINITY) || key <= best) return;
      most = x;
      best = key;
      at = pack_key(z, j);
    }
  };

  // Score of a logit under the rules; a NaN counts as -inf.
  __device__ __forceinline__ float scored_raw(float l, int word) const {  // (may be a NaN, but a quiet one)
    if (kRules && word) l = penalised(w, l, word & kPrompt, word & kCount);
    return mul_rounded(l, w.invT);
  }
  __device__ __forceinline__ float scored(float l, int word) const {
    return __builtin_fmaxf(scored_raw(l, word), -INFINITY);
  }
  __device__ __forceinline__ bool streams_words() const { return w.seen && n_said < 0; }
  __device__ __forceinline__ bool marked(int j) const { return kRules && ((skip[j >> 5] >> (j & 31)) & 1u); }

  // A batch: quartets i, i + threads, .. of a row, i the thread's first.
  struct Batch {
    f32x4 x[kUnroll], g[kUnroll];
  };
  __device__ __forceinline__ int first_of(int b) const { return b * kUnroll * threads + tid; }
  __device__ __forceinline__ int batches() const { return full + (full * kUnroll * threads < e4); }

  // Calls f(batch number, batch, on(batch number)) for the row's batches in turn until it
  // returns true, the loads of the next kAhead - 1 under way: each in registers of its
  // own, the loop unrolled over them (to move a batch from one to the next would wait for
  // its loads).  Only threads with on() load.  Quartets behind the row's end read as 0.
  template <bool kNoise, typename On, typename Fn>
  __device__ __forceinline__ void stream(On on, Fn f) const {
    const int n_b = batches(), bytes = 16 * e4;
    const uint32_t step = 16 * threads;
    const __amdgpu_buffer_rsrc_t row = buffer_of(w.logits, bytes);
    const __amdgpu_buffer_rsrc_t noise = buffer_of(kNoise ? w.noise : w.logits, bytes);
    Batch t[kAhead];
    bool mine[kAhead];
    auto load = [&](int b, int r) {
      mine[r] = b < n_b && on(b);
      const uint32_t at = mine[r] ? 16 * tid + b * kUnroll * step : 1u << 30;
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        t[r].x[k] = load_quartet(row, at + k * step);
        if (kNoise) t[r].g[k] = load_quartet(noise, at + k * step);
      }
      __builtin_amdgcn_sched_barrier(0);  // (loads end in their order: one that is moved back is waited for with all)
    };
#pragma unroll
    for (int r = 0; r < kAhead; ++r) load(r, r);
    bool stop = false;
    for (int b = 0; b < n_b && !stop; b += kAhead) {
#pragma unroll
      for (int r = 0; r < kAhead; ++r) {  // (no way out of the middle, which would be one of another order of loads)
        if (b + r < n_b && !stop) stop = f(b + r, t[r], mine[r]);
        load(b + r + kAhead, r);
      }
    }
  }
  // Its scores (-inf or a NaN: none, or marked).
  __device__ __forceinline__ void raw_scores(int b, const Batch& t, float (&z)[4 * kUnroll]) const {
    if (kRules && streams_words()) scores_of<true>(b, t, z);
    else scores_of<false>(b, t, z);
  }
  // The same without a NaN.
  __device__ __forceinline__ void scores(int b, const Batch& t, float (&z)[4 * kUnroll]) const {
    raw_scores(b, t, z);
#pragma unroll
    for (int q = 0; q < 4 * kUnroll; ++q) z[q] = __builtin_fmaxf(z[q], -INFINITY);
  }
  template <bool kWords>
  __device__ __forceinline__ void scores_of(int b, const Batch& t, float (&z)[4 * kUnroll]) const {
    const int i = first_of(b);
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int at = i + k * threads;
      uint32_t out = b < full || at < e4 ? 0u : 15u;
      if (kRules && out == 0) out = (skip[at >> 3] >> ((4 * at) & 31)) & 15u;
      u16x4 c = {0, 0, 0, 0};
      if (kWords && out != 15u) c = reinterpret_cast<const u16x4*>(w.seen)[at];
      f32x4 x = t.x[k];
      if (!kRules && b < full) {
      } else if (__ballot(out != 0)) {  // (all bits set are a NaN, which counts as -inf)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          x[e] = __uint_as_float(__float_as_uint(x[e]) |
                                 static_cast<uint32_t>(__builtin_amdgcn_sbfe(static_cast<int>(out), e, 1)));
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) z[4 * k + e] = scored_raw(x[e], kWords ? c[e] : 0);
    }
  }
  __device__ __forceinline__ int token(int b, int q) const { return 4 * (first_of(b) + q / 4 * threads) + q % 4; }

  // f(score, token) for the entries outside the quartets: the row's last one to
  // three and, under rules, the marked ones that are allowed.
  template <typename Fn>
  __device__ __forceinline__ void extras(Fn f) const {
    const int j = 4 * e4 + tid;
    if (j < a.V && !marked(j)) f(scored(w.logits[j], kRules && streams_words() ? w.seen[j] : 0), j);
    if constexpr (kRules) {
      const int listed = max(n_said, 0) + max(n_special, 0);
      for (int i = tid; i < listed; i += threads) f(apart_z[i], apart[i]);
      if (n_special < 0)
        for_special(a, w, s.path, n, 0, a.V, threads, [&](int t, int from) { f(special_score(t, from), t); });
    }
  }
  __device__ __forceinline__ float special_score(int t, int from) const {
    if (!allowed_token(w, t)) return -INFINITY;
    const int word = w.seen ? w.seen[t] : 0;
    return __builtin_fmaxf(mul_rounded(special_logit(a, w, s.path, n, t, from, w.logits[t], word), w.invT), -INFINITY);
  }

  // Lists the tokens with a count word.  A penalty costs a division, which one such
  // token in a wave's 64 entries makes it take for all, and the words are half as much
  // to read as the logits: with them in the stream 64 walks of a 152k vocabulary, one
  // token in 50 said, take 669 us, and 377 so.  A thread's place in the list decides
  // with which others its tokens' weights are added, so the places follow from the words
  // alone: each wave counts its batches, and lists them behind all that come before.
  __device__ __forceinline__ void list_said() {
    const u16x4* s4 = reinterpret_cast<const u16x4*>(w.seen);
    constexpr int kWords = 8;  // quartets of a thread in a batch
    constexpr int kMostBatches = kMaxRuled / 4 / (kWords * kMost);
    static_assert(kMostBatches * kMost * sizeof(uint32_t) <= sizeof(s.list) && kShortVocab <= 4 * kWords * 256,
                  "a bit of every entry, in the place of the candidates");
    static_assert(kMostBatches * (kMost / SRT_WAVE) <= 2 * SRT_WAVE && 2 * SRT_WAVE * sizeof(int32_t) <= sizeof(s.segbin),
                  "two counts a lane");
    uint32_t* said_bits = reinterpret_cast<uint32_t*>(s.list);
    int32_t* counts = reinterpret_cast<int32_t*>(s.segbin);
    const int step = kWords * threads, n_b = (e4 + step - 1) / step;
    auto load = [&](int i0, u16x4 (&c)[kWords]) {
      if (i0 >= e4) return;
#pragma unroll
      for (int k = 0; k < kWords; ++k) c[k] = s4[min(i0 + tid + k * threads, e4 - 1)];
    };
    auto count = [&](int b, const u16x4 (&c)[kWords]) {
      uint32_t said = 0;  // bit 4 k + e: the batch's entry has a word
#pragma unroll
      for (int k = 0; k < kWords; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) said |= (b * step + tid + k * threads < e4 && c[k][e] ? 1u : 0u) << (4 * k + e);
      said_bits[b * threads + tid] = said;
      const int m = static_cast<int>(wave_scan(static_cast<u64>(__popc(said))));
      if (lane == SRT_WAVE - 1) counts[b * waves + wave] = m;
    };
    u16x4 c0[kWords], c1[kWords];
    load(0, c0);
    for (int b = 0; b < n_b; b += 2) {  // (each in registers of its own)
      load((b + 1) * step, c1);
      count(b, c0);
      if (b + 1 >= n_b) break;
      load((b + 2) * step, c0);
      count(b + 1, c1);
    }
    __syncthreads();
    const int parts = n_b * waves;
    const int x0 = 2 * lane < parts ? counts[2 * lane] : 0, x1 = 2 * lane + 1 < parts ? counts[2 * lane + 1] : 0;
    const int upto = static_cast<int>(wave_scan(static_cast<u64>(x0 + x1)));
    const int in_quartets = __builtin_amdgcn_readlane(upto, SRT_WAVE - 1);
    const int j = 4 * e4 + lane;  // (the row's last one to three, which every wave counts)
    const u64 rest = __ballot(j < a.V && w.seen[min(j, a.V - 1)]);
    n_said = in_quartets + __popcll(rest);
    if (n_said > kSaid) n_said = -1;
    if (n_said > 0) {
      for (int b = 0; b < n_b; ++b) {
        const int part = b * waves + wave;
        uint32_t said = said_bits[b * threads + tid];
        const int m = __popc(said);
        const int first = __builtin_amdgcn_readlane(part & 1 ? upto - x1 : upto - x1 - x0, part / 2);
        int at = first + static_cast<int>(wave_scan(static_cast<u64>(m))) - m;
        for (; said; said &= said - 1, ++at) {
          const int q = __ffs(said) - 1;
          apart[at] = 4 * (b * step + tid + q / 4 * threads) + q % 4;
        }
      }
      if (wave == 0 && ((rest >> lane) & 1)) apart[in_quartets + __popcll(rest & ((1ull << lane) - 1))] = j;
    }
    __syncthreads();
    for (int i = tid; i < n_said; i += threads) said_word[i] = w.seen[apart[i]];
  }

  // Marks the row's entries that the stream passes over.
  __device__ __forceinline__ void mark_row() {
    const int words = (a.V + 31) / 32, at = w.bias0 + tid, bias = at < w.bias1 ? a.bias_tokens[at] : -1;
    typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(4)));
    for (int i0 = 4 * tid; i0 < words; i0 += 4 * kUnroll * threads) {
      u32x4u x[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const int i = i0 + 4 * k * threads;
        if (w.mask && i + 4 <= words) x[k] = *reinterpret_cast<const u32x4u*>(w.mask + i);
      }
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const int i = i0 + 4 * k * threads;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (i + e < words) skip[i + e] = !w.mask ? 0u : i + 4 <= words ? ~x[k][e] : ~w.mask[i + e];
      }
    }
    mark_special(a, w, s.path, n, 0, a.V, skip, threads, at, bias);
    // One with a count word that is marked by now is forbidden, or scored as a special one.
    for (int i0 = tid; i0 < n_said; i0 += kUnroll * threads) {
      uint32_t t[kUnroll], was[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) t[k] = apart[min(i0 + k * threads, n_said - 1)];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
        if (i0 + k * threads < n_said) was[k] = atomicOr(&skip[t[k] >> 5], 1u << (t[k] & 31));
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
        if (i0 + k * threads < n_said) apart_z[i0 + k * threads] = (was[k] >> (t[k] & 31)) & 1u ? -INFINITY : 0.f;
    }
    __syncthreads();
  }

  // Scores the marked tokens that are allowed.  After the stream: read before it, these
  // few entries bring most of the row's lines out of HBM, one at a time (64 walks of a
  // 152k vocabulary with one token in 50 said: 478 us, and 418 behind it).
  __device__ __forceinline__ void score_apart() {
    if constexpr (!kRules) return;
    constexpr int kGather = 8;
    for (int i0 = tid; i0 < n_said; i0 += kGather * threads) {
      float l[kGather];
#pragma unroll
      for (int k = 0; k < kGather; ++k) l[k] = w.logits[apart[min(i0 + k * threads, n_said - 1)]];
#pragma unroll
      for (int k = 0; k < kGather; ++k) {
        const int i = i0 + k * threads;
        if (i < n_said && apart_z[i] == 0.f) apart_z[i] = scored(l[k], said_word[i]);
      }
    }
    const int room = kApart - max(n_said, 0), first = max(n_said, 0);
    n_special = n + w.bias1 - w.bias0 <= room ? n + w.bias1 - w.bias0 : -1;
    if (n_special >= 0) {
      // (a thread's own places: its token of the path, its entries of the list)
      if (tid < n) apart_z[first + tid] = -INFINITY;
      for (int k = w.bias0 + tid; k < w.bias1; k += threads) apart_z[first + n + k - w.bias0] = -INFINITY;
      for_special(a, w, s.path, n, 0, a.V, threads, [&](int t, int from) {
        const int i = first + (from < 0 ? tid : n + from - w.bias0);
        apart[i] = t;
        apart_z[i] = special_score(t, from);
      });
    }
    __syncthreads();
  }

  // Whether the thread has an entry of score `least` or more in a batch.
  __device__ __forceinline__ bool reaches(int b, float least) const {
    if (first_of(b) >= e4) return false;
    bool any = false;
    for (int g = 0; g < batch_segs; ++g) any |= s.seg[(b / seg_batches * batch_segs + g) * threads + tid] >= least;
    return any;
  }

  // The maxima of the thread's segments from i0 on (-inf: none).
  __device__ __forceinline__ void segments(int i0, int segs, float (&x)[kSegsAt]) const {
#pragma unroll
    for (int k = 0; k < kSegsAt; ++k) x[k] = i0 + k < segs ? s.seg[(i0 + k) * threads + tid] : -INFINITY;
  }

  // The tokens of score `least` and more as the list, and how many there are (more
  // than kList: at least that many).  The segments that reach it are listed first and
  // their quartets dealt out to all threads: where a thread reads its own ones again,
  // nearly every wave has one in each batch, and waits for each in turn (of a 152k row's
  // 27 us that took 15).  s.n and s.m have been cleared.
  __device__ __forceinline__ int collect(float least) {
    const int per = kUnroll * seg_batches / batch_segs;  // quartets of a segment
    const int segs = (batches() + seg_batches - 1) / seg_batches * batch_segs;
    for (int i0 = 0; i0 < segs; i0 += kSegsAt) {
      float top[kSegsAt];
      segments(i0, segs, top);
      u64 lanes[kSegsAt];
      int total = 0;
#pragma unroll
      for (int k = 0; k < kSegsAt; ++k) {
        lanes[k] = __ballot(top[k] >= least && top[k] > -INFINITY);
        total += __popcll(lanes[k]);
      }
      if (!total) continue;
      int at = 0;
      if (lane == 0) at = atomicAdd(&s.m, total);
      at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
      for (int k = 0; k < kSegsAt; ++k) {
        const int to = at + static_cast<int>(__builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(lanes[k] >> 32),
                                                                       __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(lanes[k]), 0)));
        if (((lanes[k] >> lane) & 1) && to < kList) s.work[to] = static_cast<uint16_t>((i0 + k) * threads + tid);
        at += __popcll(lanes[k]);
      }
    }
    __syncthreads();
    const int m = s.m;
    if (m > kList) return m;  // (each has a token)
    const f32x4u* r4 = reinterpret_cast<const f32x4u*>(w.logits);
    for (int i0 = 0; i0 < m * per; i0 += kAgain * threads) {
      f32x4 x[kAgain];
      int at[kAgain];
#pragma unroll
      for (int k = 0; k < kAgain; ++k) {
        const int i = i0 + k * threads + tid;
        at[k] = e4;
        if (i < m * per) {
          const int id = s.work[i / per], o = id / threads;
          at[k] = (o * per + i % per) * threads + (id - o * threads);
        }
        if (at[k] < e4) x[k] = r4[at[k]];
      }
      float z[4 * kAgain];
      int mine = 0;
#pragma unroll
      for (int k = 0; k < kAgain; ++k) {
        const bool on = at[k] < e4;
        const uint32_t out = kRules && on ? skip[at[k] >> 3] >> ((4 * at[k]) & 31) : 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool in = on && !((out >> e) & 1u);
          z[4 * k + e] = in ? scored(x[k][e], kRules && streams_words() ? w.seen[4 * at[k] + e] : 0) : -INFINITY;
          mine += z[4 * k + e] >= least && z[4 * k + e] > -INFINITY;
        }
      }
      const int upto = static_cast<int>(wave_scan(static_cast<u64>(mine)));
      int to = 0;
      if (lane == SRT_WAVE - 1 && upto > 0) to = atomicAdd(&s.n, upto);
      to = __builtin_amdgcn_readlane(to, SRT_WAVE - 1) + upto - mine;
#pragma unroll
      for (int q = 0; q < 4 * kAgain; ++q)
        if (z[q] >= least && z[q] > -INFINITY) {
          if (to < kList) s.list[to] = pack_key(z[q], 4 * at[q / 4] + q % 4);
          ++to;
        }
      if (*const_cast<volatile int32_t*>(&s.n) > kList) break;  // (each wave by itself)
    }
    extras([&](float z, int j) {
      if (!(z >= least) || z == -INFINITY) return;
      const int at = atomicAdd(&s.n, 1);
      if (at < kList) s.list[at] = pack_key(z, j);
    });
    __syncthreads();
    return s.n;
  }

  // The workgroup's largest.
  __device__ __forceinline__ u64 all_max(u64 key) {
    key = wave_top(key);
    if (lane == 0) s.red[parity][wave] = key;
    __syncthreads();
    key = wave_top(lane < waves ? s.red[parity][lane] : 0ull);
    parity ^= 1;
    return key;
  }
  // The workgroup's sum, of whole units, and of terms that are added in the same order always.
  __device__ __forceinline__ u64 all_units(u64 x) {
    x = last_lane(wave_scan(x));
    if (lane == 0) s.red[parity][wave] = x;
    __syncthreads();
    x = lane < waves ? s.red[parity][lane] : 0ull;
    parity ^= 1;
    return last_lane(wave_scan(x));
  }
  __device__ __forceinline__ double all_sum(double x) {
    x = last_lane(wave_scan(x));
    if (lane == 0) s.redd[parity][wave] = x;
    __syncthreads();
    x = lane < waves ? s.redd[parity][lane] : 0.0;
    parity ^= 1;
    return last_lane(wave_scan(x));
  }

  __device__ __forceinline__ void take(u64& key, float z, int j) const {
    const float x = w.noise ? add_rounded(z, w.noise[j]) : z;
    if (x > -INFINITY) key = max(key, pack_key(x, j));
  }

  // arg-max of score (or of the logit, without noise) plus noise over the row.
  template <bool kNoise>
  __device__ __forceinline__ u64 plain() {
    Top best;
    u64 key = 0;
    stream<kNoise>([](int) { return true; }, [&](int b, const Batch& t, bool) {
      float z[4 * kUnroll];
      raw_scores(b, t, z);
#pragma unroll
      for (int q = 0; q < 4 * kUnroll; ++q) best.ascending(kNoise ? add_rounded(z[q], t.g[q / 4][q % 4]) : z[q], token(b, q));
      return false;
    });
    score_apart();
    extras([&](float z, int j) {
      if (z > -INFINITY) take(key, z, j);
    });
    return all_max(max(key, best.key()));
  }

  // The pass over the row: M (-inf where nothing is left), the segments' maxima and,
  // if it is asked for, the row's mass in units of the largest weight.
  template <bool kMass>
  __device__ __forceinline__ double first_pass() {
    float m = -INFINITY, seg = -INFINITY;
    double sum = 0.0;  // of parts of a batch each
    auto add = [&](float top) {  // the running maximum goes up to `top`
      if (top > m) {
        if (kMass) sum *= exp_of(m - top);
        m = top;
      }
    };
    const int n_b = batches();
    int seg_at = tid, seg_left = seg_batches;  // the segment's place; its batches that are to come
    stream<false>([](int) { return true; }, [&](int b, const Batch& t, bool) {
      float z[4 * kUnroll], four[kUnroll], top = -INFINITY;
      raw_scores(b, t, z);
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {  // (a maximum passes over a NaN)
        four[k] = __builtin_fmaxf(__builtin_fmaxf(z[4 * k], z[4 * k + 1]), __builtin_fmaxf(z[4 * k + 2], z[4 * k + 3]));
        top = __builtin_fmaxf(top, four[k]);
      }
      add(top);
      if (kMass) {
        // exp(z - ref) as 2^(z log2(e) - c), one operation before the power; c is rounded,
        // which all terms share and the last factor takes back.
        const float ref = m == -INFINITY ? 0.f : m, c = ref * kLog2e, off = __builtin_fmaf(ref, kLog2e, -c);
        float part[2] = {0.f, 0.f};
#pragma unroll
        for (int q = 0; q < 4 * kUnroll; ++q) part[q & 1] += __builtin_amdgcn_exp2f(__builtin_fmaf(z[q], kLog2e, -c));
        float both = (part[0] + part[1]) * __builtin_amdgcn_exp2f(-off);
        if (!(both < INFINITY) || !(__builtin_fabsf(ref) < 65536.f)) {
          // a NaN, or a score whose product with log2(e) has lost what parts it from the maximum
          both = 0.f;
#pragma unroll
          for (int q = 0; q < 4 * kUnroll; ++q) both += exp_of(__builtin_fmaxf(z[q], -INFINITY) - ref);
        }
        sum += both;
      }
      if (batch_segs == 1) {
        seg = larger_of(seg, top);
        if (--seg_left == 0 || b + 1 == n_b) {
          s.seg[seg_at] = seg;
          seg_at += threads;
          seg_left = seg_batches;
          seg = -INFINITY;
        }
      } else {
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
          seg = __builtin_fmaxf(seg, four[k]);
          if ((k + 1) * batch_segs % kUnroll == 0) {
            s.seg[seg_at] = seg;
            seg_at += threads;
            seg = -INFINITY;
          }
        }
      }
      return false;
    });
    score_apart();
    extras([&](float z, int j) {
      add(z);
      if (kMass && z > -INFINITY) sum += exp_of(z - m);
    });
    // Join: first the wave's lanes, then the waves.
    const float top = wave_largest(m);
    double part = 0.0;
    if (kMass) part = last_lane(wave_scan(m > -INFINITY ? sum * exp_of(m - top) : 0.0));
    if (lane == 0) {
      s.redm[wave] = top;
      if (kMass) s.redd[0][wave] = part;
    }
    __syncthreads();
    const float mine = lane < waves ? s.redm[lane] : -INFINITY;
    M = wave_largest(mine);
    if (!kMass) return 0.0;
    return last_lane(wave_scan(mine > -INFINITY ? s.redd[0][lane] * exp_of(mine - M) : 0.0));
  }

  // A score that no kept token is below, from the segments' maxima: `k` of them
  // are at least it, or together weigh at least `mass`.  -inf if neither is found.
  // The bins have been cleared; every wave takes the sums by itself.
  __device__ __forceinline__ float least_kept(int k, double mass) {
    const int segs = (batches() + seg_batches - 1) / seg_batches * batch_segs;
    for (int i0 = 0; i0 < segs; i0 += kSegsAt) {
      float x[kSegsAt];
      segments(i0, segs, x);
#pragma unroll
      for (int k = 0; k < kSegsAt; ++k) {
        const float d = (M - x[k]) * 8.f;
        if (d < kSegBins)  // (not where x is -inf)
          atomicAdd(&s.segbin[static_cast<int>(d)], (1ull << kMassBits) + static_cast<u64>(exp_of(x[k] - M) * 16777216.f));
      }
    }
    __syncthreads();
    constexpr int kPer = kSegBins / SRT_WAVE;
    constexpr u64 kMassMask = (1ull << kMassBits) - 1;
    u64 x[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      x[i] = s.segbin[lane * kPer + i];
      sum += x[i];  // (16 segments of 512 threads: neither field runs over)
    }
    const u64 before = wave_scan(sum) - sum;
    // (a margin for the weights' roundings)
    const u64 want = mass < 1e6 ? static_cast<u64>(mass * 16777216.0 * 1.00001) + 1 : ~0ull;
    int found = kSegBins;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i) {
      const u64 upto = before + sum;
      if (static_cast<int64_t>(upto >> kMassBits) >= k || (upto & kMassMask) >= want) found = lane * kPer + i;
      sum -= x[i];
    }
    const u64 lanes = __ballot(found < kSegBins);
    if (!lanes) return -INFINITY;
    found = __builtin_amdgcn_readlane(found, __ffsll(static_cast<long long>(lanes)) - 1);
    return M - (found + 1.01f) * 0.125f;
  }

  // Sorts the list's first `count` entries, largest first.  A wave's 64 pairs at a
  // distance of up to 64 lie in 128 entries of its own: such steps need no barrier.
  __device__ __forceinline__ void sort(int count) const {
    int size = 4 * SRT_WAVE;
    while (size < count) size *= 2;
    for (int i = count + tid; i < size; i += threads) s.list[i] = 0;
    __syncthreads();
    volatile u64* list = s.list;
    for (int run = 2; run <= size; run *= 2) {
      for (int d = run / 2; d >= 1; d /= 2) {
        if (d > SRT_WAVE) __syncthreads();
        for (int t = tid; t < size / 2; t += threads) {
          const int i = 2 * t - (t & (d - 1)), j = i + d;
          const u64 x = list[i], y = list[j];
          if ((x < y) == ((i & run) == 0)) {
            list[i] = y;
            list[j] = x;
          }
        }
        if (d > SRT_WAVE) __syncthreads();
      }
    }
    __syncthreads();
  }

  __device__ __forceinline__ double weight(float z) const { return exp(static_cast<double>(z) - static_cast<double>(M)); }
  // The same in whole units, whose sums are the same in any order: a list's places are
  // as its waves came.
  __device__ __forceinline__ u64 units(float z) const { return static_cast<u64>(weight(z) * kUnit); }

  // The choice from a list of up to 64 R tokens, by wave 0 in registers: R a lane,
  // place 64 r + lane, drawn from as a long list is (weighs_less) until a draw is kept.
  template <int R>
  __device__ __forceinline__ u64 from_short(int count, int k, double p, double row_mass, float least) {
    if (wave == 0) {
      u64 x[R], best = 0;
#pragma unroll
      for (int r = 0; r < R; ++r) x[r] = SRT_WAVE * r + lane < count ? s.list[SRT_WAVE * r + lane] : 0ull;
      if (k < count && p < 1.0) {  // the k-th place, bit by bit until k tokens lie up to one
        u64 kth = 0;
        for (int bit = 63; bit >= 0; --bit) {
          const u64 at = kth | 1ull << bit;
          int n_at = 0;
#pragma unroll
          for (int r = 0; r < R; ++r) n_at += __popcll(__ballot(x[r] >= at));
          if (n_at >= k) kth = at;
          if (n_at == k) break;
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
          if (x[r] < kth) x[r] = 0;
      }
      u64 key[R], place = 0;
      u64 wt[R], all = 0;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        key[r] = 0;
        if (x[r] && score_of(x[r]) >= least) take(key[r], score_of(x[r]), key_token(x[r]));
        wt[r] = p < 1.0 && x[r] ? units(score_of(x[r])) : 0ull;
        all += wt[r];
      }
      const double target = p < 1.0 ? p * (k < a.V ? static_cast<double>(last_lane(wave_scan(all))) : row_mass * kUnit) : INFINITY;
      for (;;) {  // (each draw's place lies before the last one's)
        u64 mine = 0, at = 0;
#pragma unroll
        for (int r = 0; r < R; ++r)
          if (key[r] > mine && x[r] > place) {
            mine = key[r];
            at = x[r];
          }
        best = wave_top(mine);
        if (!best) break;
        const int owner = __ffsll(static_cast<long long>(__ballot(mine == best))) - 1;
        place = static_cast<u64>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(at >> 32), owner))) << 32 |
                static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(at), owner));
        int before = 0;
        u64 mass = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const bool in = x[r] > place;
          before += __popcll(__ballot(in));
          mass += in ? wt[r] : 0ull;
        }
        if (before == 0 || (before < k && (p >= 1.0 || static_cast<double>(last_lane(wave_scan(mass))) < target))) break;
      }
      if (lane == 0) s.found = best;
    }
    __syncthreads();
    return s.found;
  }

  // The choice from a list that holds every token that can be kept (and, with both a
  // top-k and a top-p, the first k tokens).
  __device__ __forceinline__ u64 from_list(int count, int k, double p, double row_mass, float least) {
    if (k == a.V && p >= 1.0) {  // the cut is `least` alone
      u64 key = 0;
      for (int i = tid; i < count; i += threads) take(key, score_of(s.list[i]), key_token(s.list[i]));
      return all_max(key);
    }
    if (count <= SRT_WAVE) return from_short<1>(count, k, p, row_mass, least);
    if (count <= 4 * SRT_WAVE) return from_short<4>(count, k, p, row_mass, least);
    if (k == a.V) return draw_from_list(count, p * row_mass, least);
    sort(count);
    const int per = (count + threads - 1) / threads, from = tid * per, to = min(from + per, min(count, k));
    double before = 0.0, target = INFINITY;
    if (p < 1.0) {
      double mine = 0.0;
      for (int i = from; i < to; ++i) mine += weight(score_of(s.list[i]));
      const double incl = wave_scan(mine);
      if (lane == SRT_WAVE - 1) s.redd[parity][wave] = incl;
      __syncthreads();
      double all = 0.0;
      before = incl - mine;
      for (int j = 0; j < waves; ++j) {
        if (j == wave) before += all;
        all += s.redd[parity][j];
      }
      parity ^= 1;
      target = p * (k < a.V ? all : row_mass);
    }
    u64 key = 0;
    for (int i = from; i < to; ++i) {
      const u64 x = s.list[i];
      const float z = score_of(x);
      if (i > 0 && (!(before < target) || z < least)) break;
      take(key, z, key_token(x));
      if (p < 1.0) before += weight(z);
    }
    return all_max(key);
  }

  // from_row's draws, in the list: the kept tokens are those before which less than
  // `target` lies, from `least` up.
  __device__ __forceinline__ u64 draw_from_list(int count, double target, float least) {
    u64 place = 0;
    for (int draw = 0; draw < kDraws; ++draw) {
      u64 best = 0, at = 0;
      for (int i = tid; i < count; i += threads) {
        const u64 x = s.list[i], held = best;
        if (x <= place || score_of(x) < least) continue;
        take(best, score_of(x), key_token(x));
        if (best != held) at = x;
      }
      const u64 all = all_max(best);
      if (!all) return 0;
      if (best == all) s.found = at;
      __syncthreads();
      place = s.found;
      u64 mass = 0;
      for (int i = tid; i < count; i += threads)
        if (s.list[i] > place) mass += units(score_of(s.list[i]));
      if (static_cast<double>(all_units(mass)) < target * kUnit) return all;  // (nothing lies before the first)
    }
    sort(count);
    u64 best = 0;
    if (tid == 0) {
      double before = 0.0;
      for (int i = 0; i < count; ++i) {
        const float z = score_of(s.list[i]);
        if (i > 0 && (!(before < target) || z < least)) break;
        take(best, z, key_token(s.list[i]));
        before += weight(z);
      }
    }
    return all_max(best);
  }

  // The workgroup's best; its place is s.found.
  __device__ __forceinline__ u64 drawn(const Draw& d) {
    const u64 all = all_max(d.best);
    if (all && d.best == all) s.found = d.at;  // (one thread's: a token is seen once)
    __syncthreads();
    return all;
  }

  // Calls f(batch number, batch, whether it is the thread's) in a wave for the batches
  // that have a score of `least` or more in one of its threads.
  template <bool kNoise, typename Fn>
  __device__ __forceinline__ void batches_from(float least, Fn f) {
    stream<kNoise>([&](int b) { return reaches(b, least); }, [&](int b, const Batch& t, bool on) {
      if (__ballot(on)) f(b, t, on);
      return false;
    });
  }

  // The best of the tokens of `least` and more before `after` in the order.
  __device__ __forceinline__ u64 candidate(u64 after, float least) {
    Draw d;
    batches_from<true>(least, [&](int b, const Batch& t, bool on) {
      float z[4 * kUnroll];
      scores(b, t, z);
#pragma unroll
      for (int q = 0; q < 4 * kUnroll; ++q) {
        const float x = add_rounded(z[q], t.g[q / 4][q % 4]);
        if (on && x > d.most && z[q] >= least && (!after || pack_key(z[q], token(b, q)) > after)) d.any(z[q], x, token(b, q));
      }
    });
    extras([&](float z, int j) {
      if (z >= least && z > -INFINITY && pack_key(z, j) > after) d.any(z, add_rounded(z, w.noise[j]), j);
    });
    return drawn(d);
  }

  // Whether the tokens before a place in the order weigh less than `target` of the
  // row's `all`.  The wave's batches are summed a few at a time; what the rest weighs
  // is known with what has been read, and most places are decided by a part of the row
  // (at a top-p of 0.9 by a third of it, on average).
  __device__ __forceinline__ bool weighs_less(u64 place, double target, double all) {
    const float edge = score_of(place);
    const int last = key_token(place), n_b = batches();
    double mass = 0.0, read = 0.0;
    extras([&](float z, int j) {
      if (!(z > -INFINITY)) return;
      const double x = exp_of(z - M);
      read += x;
      if (pack_key(z, j) > place) mass += x;
    });
    bool less = false, decided = false;
    stream<false>([](int) { return true; }, [&](int b, const Batch& t, bool) {
      float z[4 * kUnroll], in = 0.f, out = 0.f;
      scores(b, t, z);
      bool equal = false;
#pragma unroll
      for (int q = 0; q < 4 * kUnroll; ++q) {
        const float x = exp_of(z[q] - M);
        in += z[q] > edge ? x : 0.f;
        out += z[q] > edge ? 0.f : x;
        equal |= z[q] == edge;
      }
      if (equal)  // ties with the token at the place, itself among them: seldom
#pragma unroll
        for (int q = 0; q < 4 * kUnroll; ++q)
          if (z[q] == edge && token(b, q) < last) mass += exp_of(z[q] - M);
      mass += in;
      read += static_cast<double>(in) + out;
      if ((b + 1) % kStage != 0 || b + 1 == n_b) return false;
      const double before = all_sum(mass), rest = all - all_sum(read);
      less = before + rest + 1e-5 * all < target;  // (a margin for the sums' roundings)
      return decided = less || before >= target;
    });
    return decided ? less : all_sum(mass) < target;
  }

  // How many tokens lie up to a place in the order, and what they weigh.
  struct Above {
    double count, mass;
  };
  __device__ __forceinline__ Above above(u64 place, bool before, bool weigh) {
    float least = score_of(place);
    if (!(least == least)) least = -INFINITY;  // (behind every score)
    double mass = 0.0;
    int count = 0;  // of the wave
    auto counts = [&](float z, int j) {
      const u64 x = pack_key(z, j);
      return z > -INFINITY && (x > place || (x == place && !before));
    };
    batches_from<false>(least, [&](int b, const Batch& t, bool on) {
      float z[4 * kUnroll], part = 0.f;
      scores(b, t, z);
#pragma unroll
      for (int q = 0; q < 4 * kUnroll; ++q) {
        const bool in = on && counts(z[q], token(b, q));
        if (weigh) part += in ? exp_of(z[q] - M) : 0.f;
        count += __popcll(__ballot(in));
      }
      mass += part;
    });
    double c = 0.0;
    extras([&](float z, int j) {
      if (!counts(z, j)) return;
      mass += exp_of(z - M);
      c += 1.0;
    });
    return {all_sum(c + (lane == 0 ? count : 0)), weigh ? all_sum(mass) : 0.0};
  }

  // The choice among more tokens than the list holds, of which those below `lowest` and
  // `by_min` are not kept.  The best of a set that has the kept ones is the choice if it is
  // kept itself, for which what lies before it in the order is summed; if it is not,
  // the kept ones lie before it.  A draw from a set's distribution is one of the kept
  // ones' share of it, so a top-p of 0.9 takes 1.1 draws, and a kept set of a
  // millionth a dozen.  Noise that is none could be arranged to take one for every
  // token; after kDraws the last kept place is found bit by bit, as is the place of the
  // k-th token where the mass of the first k is asked for.
  // (One loop, so that each
  // pass over the row stands in the code once: what a walk runs fits the instruction
  // cache.)
  __device__ __forceinline__ u64 from_row(int k, float p, double mass, float lowest, float by_min) {
    const float least = __builtin_fmaxf(lowest, by_min);
    const bool by_k = k < a.V, by_p = p < 1.f;
    bool searching = by_k && by_p, summing = false, last = false;  // the k-th place; its mass; the last kept place is known
    double target = by_p && !by_k ? static_cast<double>(p) * mass : INFINITY;
    // The places searched for lie between the row's first and that of `lowest`, whose
    // common bits they share.
    const u64 first = pack_key(M, 0), ends = first ^ pack_key(lowest, a.V - 1);
    const int top_bit = 63 - __clzll(static_cast<long long>(ends | 1));
    const u64 common = first & ~((2ull << top_bit) - 1);
    u64 found = common, best = 0, place = 0;
    for (int bit = top_bit, draw = 0;;) {
      u64 at = place;
      if (searching) {
        at = found | 1ull << bit;
      } else if (summing) {
        at = found;
      } else {
        best = candidate(place, least);
        if (!best) return 0;
        place = at = s.found;
        if (last || !(by_k || by_p)) return best;
        if (!by_k) {
          if (score_of(place) >= least && weighs_less(place, target, mass)) return best;  // (nothing lies before the first)
          if (++draw < kDraws) continue;
          searching = true;
          continue;
        }
      }
      const Above x = above(at, !searching && !summing, searching ? target < INFINITY : by_p);
      if (searching) {
        if (x.count >= k || x.mass >= target) found = at;
        if (x.count == k && draw == 0) bit = 0;  // (the first k tokens: only their mass is asked for)
        if (--bit >= 0) continue;
        searching = false;
        if (draw == 0) {  // the k-th place
          summing = true;
        } else {          // the last kept place: its best is the choice
          last = true;
          place = max(found, 1ull) - 1;
        }
      } else if (summing) {
        summing = false;
        target = static_cast<double>(p) * x.mass;
      } else {
        if (score_of(place) >= least && x.count < k && (x.count == 0.0 || x.mass < target)) return best;
        if (++draw == kDraws) {
          searching = true;
          bit = top_bit;
          found = common;
        }
      }
    }
  }
};

// The choice at the node that the row belongs to: packed (score with noise, token), 0 if none.
template <bool kRules, bool kNoise>
__device__ __forceinline__ u64 choose(Walker<kRules>& x, int k, float p, float mp, double edge) {
  Lds& s = x.s;
  const int V = x.a.V;
  if (!(p > 0.f) || !(mp <= 1.f)) k = 1, p = 1.f, mp = 0.f;  // (a NaN too)
  if (k <= 0 || k > V) k = V;
  bool by_k = k < V, by_p = p < 1.f, by_m = mp > 0.f;
  if (!kNoise || !(by_k || by_p || by_m)) return x.template plain<kNoise>();
  for (int i = x.tid; i < kSegBins; i += x.threads) s.segbin[i] = 0;
  if (x.tid == 0) s.n = s.m = 0;
  double mass = 0.0;
  if (by_p && !by_k) mass = x.template first_pass<true>();
  else x.template first_pass<false>();
  const float M = x.M;
  if (M == -INFINITY) return 0;
  // (infinite scores: the lowest token of them, which is always kept)
  if (M == INFINITY) k = V, p = 1.f, by_k = by_p = by_m = false;
  // The scores below which nothing is kept.
  float by_min = -INFINITY;
  if (by_m) {  // the smallest float whose distance from M is no more than log(min_p), `edge`
    by_min = static_cast<float>(static_cast<double>(M) + edge);
    if (static_cast<double>(by_min) - static_cast<double>(M) < edge) by_min = nextafterf(by_min, INFINITY);
  }
  // (with both, the mass of the first k is needed, to which what weighs e^-104 adds nothing)
  float least = M == INFINITY ? M : by_k && by_p ? M - 104.f : by_min;
  if (by_p && !by_k) {
    // tokens below this weigh no more than 1 - p of the row together
    const float d = __logf(static_cast<float>(V / ((1.0 - static_cast<double>(p)) * mass)));
    least = __builtin_fmaxf(least, M - d - 0.01f);
  }
  if (by_k || by_p)
    least = __builtin_fmaxf(least, x.least_kept(by_k ? k : 0x7fffffff, by_k ? INFINITY : static_cast<double>(p) * mass));
  const int count = M == INFINITY ? kList + 1 : x.collect(least);
  if (count <= kList) return x.from_list(count, k, by_p ? static_cast<double>(p) : 1.0, mass, by_min);
  return x.from_row(k, p, mass, least, by_min);
}

template <bool kRules, bool kNoise>
__global__ __launch_bounds__(kMost) void sample_walk_kernel(SampleArgs a) {
  __shared__ Lds s;
  __shared__ uint32_t skip[kRules ? kMaxRuled / 32 : 1];
  __shared__ int32_t apart[kRules ? kApart : 1];
  __shared__ float apart_z[kRules ? kApart : 1];
  __shared__ uint16_t said_word[kRules ? kSaid : 1];
  __shared__ int32_t bias_tok[kRules ? kStaged : 1];
  __shared__ float bias_val[kRules ? kStaged : 1];
  const int b = blockIdx.x, tid = threadIdx.x, threads = blockDim.x;
  const int64_t tr = static_cast<int64_t>(b) * a.N, orow = static_cast<int64_t>(b) * (a.Dmax + 1);
  const int n = min(max(a.n_nodes[b], 1), a.N);
  for (int c = tid; c < n; c += threads) {
    s.par[c] = a.tree_parent[tr + c];
    s.tok[c] = a.tree_tokens[tr + c];
  }
  // (a division's result is the same for all lanes, and said to be: the loops over batches are to be scalar ones)
  auto scalar = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  const int lane = tid % SRT_WAVE, wave = scalar(tid / SRT_WAVE), e4 = a.V / 4;
  const int full = scalar(e4 / (kUnroll * threads)), batches = scalar((e4 + kUnroll * threads - 1) / (kUnroll * threads));
  int batch_segs = 1;
  static_assert(kSegs % kUnroll == 0 && kSegs * kMost <= 65536, "a batch's segments are of 8, 4, 2 or 1 quartets");
  while (batch_segs < kUnroll && 2 * batch_segs * batches <= kSegs) batch_segs *= 2;
  Walker<kRules> walker = {a, s, skip, apart, apart_z, said_word, 0, 0, {}, 0, tid, threads, lane, wave, threads / SRT_WAVE, e4, full,
                           max(1, scalar((batches + kSegs - 1) / kSegs)), scalar(batch_segs), 0, 0.f};
  const float p = a.top_p ? a.top_p[b] : 1.f, mp = a.min_p ? a.min_p[b] : 0.f;
  const int top_k = a.top_k ? a.top_k[b] : 0;
  const double edge = mp > 0.f ? log(static_cast<double>(mp)) : 0.0;
  int u = 0, k = 0, tok;
  for (;; ++k) {
    walker.w = rules_of(a, b, k);
    stand_on(a, walker.w, b, u);
    walker.w.invT = a.inv_temperature && a.gumbel ? a.inv_temperature[b] : 1.f;
    walker.n = k;
    // (what the thread's place decides is worked out where it is used, not kept over the walk in 100 registers)
    asm volatile("" : "+v"(walker.tid), "+v"(walker.lane));
    if constexpr (kRules) {
      // (penalties that change nothing: no counts are read)
      if (walker.w.r == 1.f && walker.w.f == 0.f && walker.w.p == 0.f) walker.w.seen = nullptr;
      const int listed = walker.w.bias1 - walker.w.bias0;
      if (k == 0) {
        if (listed <= kStaged)
          for (int i = tid; i < listed; i += threads) {
            bias_tok[i] = a.bias_tokens[walker.w.bias0 + i];
            bias_val[i] = a.bias_values[walker.w.bias0 + i];
          }
        if (walker.w.seen) walker.list_said();
        else __syncthreads();
        if (listed <= kStaged) {
          a.bias_tokens = bias_tok;
          a.bias_values = bias_val;
        }
      }
      if (listed <= kStaged) {
        walker.w.bias0 = 0;
        walker.w.bias1 = listed;
      }
      walker.mark_row();
    }
    const u64 key = choose<kRules, kNoise>(walker, top_k, p, mp, edge);
    tok = key ? key_token(key) : -1;
    __syncthreads();  // (the staged tree, at the first step; LDS is the next row's from here on)
    int child = -1;
    if (k < a.Dmax && tok >= 0) {  // children of u have larger indices
      for (int c0 = u + 1; c0 < n && child < 0; c0 += SRT_WAVE) {
        const int c = c0 + lane;
        const u64 hit = __ballot(c < n && s.par[c] == u && s.tok[c] == tok);
        if (hit) child = c0 + __ffsll(static_cast<long long>(hit)) - 1;
      }
    }
    if (tid == 0) {
      a.out_tokens[orow + k] = tok;
      a.out_nodes[orow + k] = child;  // -1 at the last step
      if (child >= 0) s.path.tok[k] = tok;
    }
    if (child < 0) break;
    u = child;
    __syncthreads();
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

}  // namespace

extern "C" int srt_accept_sample(int32_t B, int32_t N, int32_t V, int32_t Dmax, const float* logits,
                                 const float* gumbel, const srt_sampling* sampling, const srt_rules* rules,
                                 const int32_t* tree_tokens, const int32_t* tree_parent, const int32_t* n_nodes,
                                 int32_t* n_accepted, int32_t* out_tokens, int32_t* out_nodes, int32_t* n_emitted,
                                 void* stream) {
  if (!sampling || sampling->reserved != 0) return SRT_ERR_INVALID;
  if (rules && check_rules(*rules) != SRT_OK) return SRT_ERR_INVALID;
  const int st = check_args(B, N, V, Dmax, logits, 1.f, tree_tokens, tree_parent, n_nodes, n_accepted, out_tokens,
                            out_nodes);
  if (st != SRT_OK || B == 0) return st;
  if (V > (rules ? kMaxRuled : kMaxVocab)) return SRT_ERR_UNSUPPORTED;
  const unsigned threads = V <= kShortVocab ? 256 : kMost;
  if (!launchable(B, threads)) return SRT_ERR_UNSUPPORTED;

  SampleArgs a = {};
  a.logits = logits;
  a.gumbel = gumbel;
  a.tree_tokens = tree_tokens;
  a.tree_parent = tree_parent;
  a.n_nodes = n_nodes;
  a.n_accepted = n_accepted;
  a.out_tokens = out_tokens;
  a.out_nodes = out_nodes;
  a.n_emitted = n_emitted;
  a.B = B;
  a.N = N;
  a.V = V;
  a.Dmax = Dmax;
  a.inv_temperature = sampling->inv_temperature;
  a.top_k = sampling->top_k;
  a.top_p = sampling->top_p;
  a.min_p = sampling->min_p;
  hipStream_t s = as_stream(stream);
  if (rules) {
    take_rules(a, *rules);
    if (gumbel) sample_walk_kernel<true, true><<<static_cast<unsigned>(B), threads, 0, s>>>(a);
    else sample_walk_kernel<true, false><<<static_cast<unsigned>(B), threads, 0, s>>>(a);
  } else {
    if (gumbel) sample_walk_kernel<false, true><<<static_cast<unsigned>(B), threads, 0, s>>>(a);
    else sample_walk_kernel<false, false><<<static_cast<unsigned>(B), threads, 0, s>>>(a);
  }
  return launch_status();
}
