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
// GPU design.  One workgroup walks one sequence; what bounds it is reading the
// visited rows (608 KB of a 152k vocabulary).  A row is read from HBM once: its
// maximum, its sum of exp(z - max), and the maximum of every thread's every few
// entries (a segment) are taken in one pass.  A count and a lower bound of the mass
// over the segments' maxima give a score below which nothing can be kept; segments
// that reach it are read again, which a row that is sure of its tokens has few of,
// and their entries from that score up are sorted in LDS, most often a hundred.
// There the cuts are prefix sums, and noise is read at the kept tokens alone.
// Rows with more candidates than the list holds are narrowed down by histograms
// over ever smaller ranges of the score (counts, and masses in fixed point, so
// that the order of the atomics does not matter) to the one list that the last
// kept token is in.  Sequences that cut nothing, or without noise, take the plain
// arg-max in one pass.
#include "rules.h"

namespace {

constexpr int kList = 4096;       // candidates that are sorted in LDS
constexpr int kBins = 2048;       // of a histogram over a range of the score
constexpr int kSegs = 16;         // segments of a thread, at most
constexpr int kUnroll = 5;        // quartets of a thread that are under way together
constexpr int kMost = 1024;       // threads
constexpr int kSegBins = 1024;    // of the segments' maxima, 1 / 16 of the score wide
constexpr int64_t kMaxVocab = int64_t(1) << 21;
constexpr int64_t kMaxRuled = int64_t(1) << 18;  // a row's marks are held in LDS
constexpr int kShortVocab = 8192;  // rows up to which 256 threads walk
constexpr float kLog2e = 1.44269504088896341f;
constexpr uint32_t kNothing = 0x007f;  // key16 of -inf

struct SampleArgs : RulesArgs {
  const float* inv_temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
};

typedef unsigned long long u64;

__device__ inline uint32_t key16(float x) { return static_cast<uint32_t>(pack_key(x, 0) >> 48); }
// A float that is no larger than any that has this key16.
__device__ inline float floor16(uint32_t k) {
  const uint32_t u = k << 16;
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}

__device__ inline float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

__device__ inline double shfl_xor_f64(double v, int m) { return __builtin_bit_cast(double, shfl_xor_u64(__builtin_bit_cast(u64, v), m)); }

// What the workgroup shares.
struct Lds {
  union {
    u64 list[kList];               // packed candidates (score, token)
    struct {
      u64 mass[kBins];             // in units of 2^-40 of the row's largest weight
      uint32_t count[kBins];
    } hist;
  };
  uint16_t seg[kSegs * kMost];
  Path path;
  int32_t par[kMaxN], tok[kMaxN];
  u64 red[kMost / SRT_WAVE];
  double redd[kMost / SRT_WAVE];
  u64 found;
  double before;
  int32_t bin, n;
  uint32_t lo, hi;
};

template <bool kRules>
struct Walker {
  const SampleArgs& a;
  Lds& s;
  const uint32_t* skip;  // marked entries (kRules)
  Row w;
  int n;                 // tokens emitted on this walk
  int tid, threads, lane, wave, waves;
  int e4, seg_batches;   // quartets of a row; batches of a segment
  float M;               // largest score of the row

  // Score of a logit under the rules; a NaN counts as -inf.
  __device__ __forceinline__ float scored(float l, int word) const {
    if (kRules && word) l = penalised(w, l, word & kPrompt, word & kCount);
    return __builtin_fmaxf(mul_rounded(l, w.invT), -INFINITY);
  }
  __device__ __forceinline__ bool marked(int j) const { return kRules && ((skip[j >> 5] >> (j & 31)) & 1u); }

  // Scores of the batch of quartets i, i + threads, .. (-inf: none, or marked).
  __device__ __forceinline__ void batch(int i, float (&z)[4 * kUnroll], float (*g)[4 * kUnroll]) const {
    const f32x4u* r4 = reinterpret_cast<const f32x4u*>(w.logits);
    const f32x4u* g4 = reinterpret_cast<const f32x4u*>(w.noise);
    const u16x4* s4 = reinterpret_cast<const u16x4*>(w.seen);
    f32x4 x[kUnroll];
    u16x4 c[kUnroll];
    uint32_t out[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int at = i + k * threads;
      out[k] = at < e4 ? (kRules ? (skip[at >> 3] >> ((4 * at) & 31)) & 15u : 0u) : 15u;
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int at = out[k] == 15u ? i : i + k * threads;  // (the first one's line is read)
      x[k] = r4[at];
      c[k] = u16x4{0, 0, 0, 0};
      if (kRules && w.seen) c[k] = s4[at];
      if (g) {
        const f32x4 y = g4[at];
#pragma unroll
        for (int e = 0; e < 4; ++e) (*g)[4 * k + e] = y[e];
      }
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) z[4 * k + e] = (out[k] >> e) & 1u ? -INFINITY : scored(x[k][e], c[k][e]);
  }
  __device__ __forceinline__ int token(int i, int q) const { return 4 * (i + q / 4 * threads) + q % 4; }

  // f(score, token) for the entries outside the quartets: the row's last one to
  // three and, under rules, the marked ones that are allowed.
  template <typename F>
  __device__ __forceinline__ void extras(F f) const {
    const int j = 4 * e4 + tid;
    if (j < a.V && !marked(j)) f(scored(w.logits[j], w.seen ? w.seen[j] : 0), j);
    if constexpr (kRules)
      for_special(a, w, s.path, n, 0, a.V, threads, [&](int t, int from) {
        if (allowed_token(w, t))
          f(__builtin_fmaxf(mul_rounded(special_logit(a, w, s.path, n, t, from, w.logits[t]), w.invT), -INFINITY), t);
      });
  }

  // f(score, token) for every entry whose score can be `least` or more.
  template <typename F>
  __device__ __forceinline__ void visit(float least, F f) const {
    const uint32_t from = key16(least);
    int b = 0;
    for (int i = tid; i < e4; i += kUnroll * threads, ++b) {
      if (s.seg[b / seg_batches * threads + tid] < from) continue;
      float z[4 * kUnroll];
      batch(i, z, nullptr);
#pragma unroll
      for (int q = 0; q < 4 * kUnroll; ++q)
        if (z[q] >= least && z[q] > -INFINITY) f(z[q], token(i, q));
    }
    extras([&](float z, int j) {
      if (z >= least && z > -INFINITY) f(z, j);
    });
  }

  // The workgroup's largest.  Synchronises, before as well.
  __device__ __forceinline__ u64 all_max(u64 key) const {
    key = wave_max(key);
    __syncthreads();
    if (lane == 0) s.red[wave] = key;
    __syncthreads();
    return wave_max(lane < waves ? s.red[lane] : 0ull);
  }
  __device__ __forceinline__ double all_sum(double x) const {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += shfl_xor_f64(x, off);
    __syncthreads();
    if (lane == 0) s.redd[wave] = x;
    __syncthreads();
    x = lane < waves ? s.redd[lane] : 0.0;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += shfl_xor_f64(x, off);
    return x;
  }

  // arg-max of score (or of the logit, without noise) plus noise over the row.
  __device__ __forceinline__ u64 plain() const {
    Top best;
    u64 key = 0;
    for (int i = tid; i < e4; i += kUnroll * threads) {
      float z[4 * kUnroll], g[4 * kUnroll];
      batch(i, z, w.noise ? &g : nullptr);
#pragma unroll
      for (int q = 0; q < 4 * kUnroll; ++q) best.ascending(w.noise ? add_rounded(z[q], g[q]) : z[q], token(i, q));
    }
    extras([&](float z, int j) { take(key, z, j); });
    return all_max(max(key, best.key()));
  }
  __device__ __forceinline__ void take(u64& key, float z, int j) const {
    const float x = w.noise ? add_rounded(z, w.noise[j]) : z;
    if (x > -INFINITY) key = max(key, pack_key(x, j));
  }

  // The pass over the row: M, the segments' maxima, and the row's mass in units of
  // the largest weight.  M is -inf where nothing is left.
  __device__ __forceinline__ double first_pass() {
    float m = -INFINITY, sum = 0.f, seg = -INFINITY;
    int b = 0;
    auto add = [&](float top) {  // the running maximum goes up to `top`
      if (top > m) {
        sum *= exp_of(m - top);
        m = top;
      }
    };
    for (int i = tid; i < e4; i += kUnroll * threads, ++b) {
      float z[4 * kUnroll];
      batch(i, z, nullptr);
      float top = z[0];
#pragma unroll
      for (int q = 1; q < 4 * kUnroll; ++q) top = __builtin_fmaxf(top, z[q]);
      add(top);
      const float ref = m == -INFINITY ? 0.f : m;
      float part = 0.f;
#pragma unroll
      for (int q = 0; q < 4 * kUnroll; ++q) part += exp_of(z[q] - ref);
      sum += part;
      seg = __builtin_fmaxf(seg, top);
      if ((b + 1) % seg_batches == 0 || i + kUnroll * threads >= e4) {
        s.seg[b / seg_batches * threads + tid] = static_cast<uint16_t>(key16(seg));
        seg = -INFINITY;
      }
    }
    extras([&](float z, int) {
      add(z);
      if (z > -INFINITY) sum += exp_of(z - m);
    });
    const u64 top = all_max(m > -INFINITY ? pack_key(m, 0) : 0ull);
    if (!top) {
      M = -INFINITY;
      return 0.0;
    }
    const uint32_t u = static_cast<uint32_t>(top >> 32);
    M = __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
    // (m and M are finite here or M is +inf, where the sum is not used)
    return all_sum(m > -INFINITY ? static_cast<double>(sum) * exp(static_cast<double>(m) - static_cast<double>(M)) : 0.0);
  }

  // A score that no kept token is below, from the segments' maxima: `k` of them
  // are at least it, or their mass is at least `mass` of the row's.  -inf if neither is found.
  __device__ __forceinline__ float least_kept(int k, double mass) {
    uint32_t* cnt = s.hist.count;
    __syncthreads();
    for (int i = tid; i < kSegBins; i += threads) cnt[i] = 0;
    __syncthreads();
    int b = 0;
    for (int i = tid; i < e4; i += kUnroll * threads * seg_batches, ++b) {
      const uint32_t key = s.seg[b * threads + tid];
      if (key <= kNothing) continue;
      const float d = (M - floor16(key)) * 16.f;
      if (d < kSegBins - 1) atomicAdd(&cnt[static_cast<int>(d)], 1u);
    }
    __syncthreads();
    if (wave == 0) {
      constexpr int kPer = kSegBins / SRT_WAVE;
      int c = 0;
      float x = 0.f;
      for (int i = 0; i < kPer; ++i) {
        const int bin = lane * kPer + i, n = cnt[bin];
        c += n;
        x += n * exp_of(-(bin + 1) / 16.f);
      }
      int c0 = c;
      float x0 = x;
#pragma unroll
      for (int d = 1; d < SRT_WAVE; d <<= 1) {
        const int y = __shfl_up(c0, d, SRT_WAVE);
        const float v = __shfl_up(x0, d, SRT_WAVE);
        if (lane >= d) c0 += y, x0 += v;
      }
      c0 -= c;
      x0 -= x;
      int found = kSegBins;
      for (int i = 0; i < kPer && found == kSegBins; ++i) {
        const int bin = lane * kPer + i, n = cnt[bin];
        c0 += n;
        x0 += n * exp_of(-(bin + 1) / 16.f);
        // (the mass needs a margin for the roundings of its fp32 sum)
        if (n && (c0 >= k || x0 >= mass * 1.0001)) found = bin;
      }
#pragma unroll
      for (int d = SRT_WAVE / 2; d >= 1; d >>= 1) found = min(found, __shfl_xor(found, d, SRT_WAVE));
      if (lane == 0) s.bin = found;
    }
    __syncthreads();
    return s.bin < kSegBins ? M - (s.bin + 2) / 16.f : -INFINITY;
  }

  // Sorts the list's first `count` entries, largest first.
  __device__ __forceinline__ void sort(int count) const {
    int size = 64;
    while (size < count) size *= 2;
    __syncthreads();
    for (int i = count + tid; i < size; i += threads) s.list[i] = 0;
    __syncthreads();
    for (int run = 2; run <= size; run *= 2) {
      for (int d = run / 2; d >= 1; d /= 2) {
        for (int t = tid; t < size / 2; t += threads) {
          const int i = 2 * t - (t & (d - 1)), j = i + d;
          const u64 x = s.list[i], y = s.list[j];
          if ((x < y) == ((i & run) == 0)) {
            s.list[i] = y;
            s.list[j] = x;
          }
        }
        __syncthreads();
      }
    }
  }

  __device__ __forceinline__ static float score_of(u64 key) {
    const uint32_t u = static_cast<uint32_t>(key >> 32);
    return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
  }

  // Weight of a score in fixed point.
  __device__ __forceinline__ u64 fixed(float z) const { return static_cast<u64>(exp_of(z - M) * 1099511627776.f); }

  // The choice from a list that holds every token that can be kept (and, with both a
  // top-k and a top-p, the first k tokens).
  __device__ __forceinline__ u64 from_list(int count, int k, double p, double row_mass, float least) const {
    sort(count);
    const int per = (count + threads - 1) / threads;
    double mine = 0.0;
    for (int i = tid * per; i < min(tid * per + per, min(count, k)); ++i)
      mine += exp(static_cast<double>(score_of(s.list[i])) - static_cast<double>(M));
    // exclusive prefix sums over the workgroup
    double incl = mine;
#pragma unroll
    for (int d = 1; d < SRT_WAVE; d <<= 1) {
      const u64 y = __shfl_up(__builtin_bit_cast(u64, incl), d, SRT_WAVE);
      if (lane >= d) incl += __builtin_bit_cast(double, y);
    }
    if (lane == SRT_WAVE - 1) s.redd[wave] = incl;
    __syncthreads();
    double before = incl - mine, all = 0.0;
    for (int j = 0; j < waves; ++j) {
      if (j == wave) before += all;
      all += s.redd[j];
    }
    const double target = p * (k < a.V ? all : row_mass);
    u64 key = 0;
    for (int i = tid * per; i < min(tid * per + per, min(count, k)); ++i) {
      const u64 x = s.list[i];
      const float z = score_of(x);
      if (i > 0 && (!(p >= 1.0 || before < target) || z < least)) break;
      take(key, z, key_token(x));
      before += exp(static_cast<double>(z) - static_cast<double>(M));
    }
    return all_max(key);
  }

  // Packed (score, token) of the last token, from the top, at which the count of
  // tokens (kMass false) or their mass in fixed point reaches `target`; 0 if none does.
  // Only tokens of `least` and more are looked at.
  template <bool kMass>
  __device__ __forceinline__ u64 border(double target, float least) {
    float top = M, low = least;  // scores of the range
    double base = 0.0;           // measure of the tokens above it
    bool first = true;
    for (;;) {
      const float end = first ? __builtin_fmaxf(low, M - 64.f) : low;  // (what lies below falls into the last bin)
      first = false;
      if (!(end < top)) return ties<kMass>(top, target, base);
      const double scale = kBins / (static_cast<double>(top) - static_cast<double>(end));
      auto bin_of = [&](float z) { return static_cast<int>(fmin((static_cast<double>(top) - static_cast<double>(z)) * scale, kBins - 1.0)); };
      auto in = [&](float z) { return z <= top && z >= low; };
      __syncthreads();
      for (int i = tid; i < kBins; i += threads) {
        s.hist.mass[i] = 0;
        s.hist.count[i] = 0;
      }
      __syncthreads();
      visit(low, [&](float z, int) {
        if (!in(z)) return;
        const int bin = bin_of(z);
        if (kMass) atomicAdd(&s.hist.mass[bin], fixed(z));
        atomicAdd(&s.hist.count[bin], 1u);
      });
      __syncthreads();
      find<kMass>(target, base);
      const int bin = s.bin, count = s.n;
      const double above = s.before;
      if (bin < 0) return 0;
      __syncthreads();
      if (count <= kList) {
        if (tid == 0) s.n = 0;
        __syncthreads();
        visit(low, [&](float z, int j) {
          if (in(z) && bin_of(z) == bin) s.list[atomicAdd(&s.n, 1)] = pack_key(z, j);
        });
        __syncthreads();
        return in_list<kMass>(count, target - above);
      }
      // Too many: on with the range that the bin's own scores span.
      if (tid == 0) {
        s.lo = 0xFFFFFFFFu;
        s.hi = 0;
      }
      __syncthreads();
      uint32_t lo = 0xFFFFFFFFu, hi = 0;
      visit(low, [&](float z, int) {
        if (!in(z) || bin_of(z) != bin) return;
        const uint32_t u = static_cast<uint32_t>(pack_key(z, 0) >> 32);
        lo = min(lo, u);
        hi = max(hi, u);
      });
      if (hi) {
        atomicMin(&s.lo, lo);
        atomicMax(&s.hi, hi);
      }
      __syncthreads();
      top = score_of(static_cast<u64>(s.hi) << 32);
      low = score_of(static_cast<u64>(s.lo) << 32);
      base = above;
    }
  }

  // First bin at which the running measure reaches `target` (s.bin, -1: none), with
  // the measure before it (s.before) and its count (s.n).
  template <bool kMass>
  __device__ __forceinline__ void find(double target, double base) {
    if (wave == 0) {
      constexpr int kPer = kBins / SRT_WAVE;
      u64 sum = 0;
      for (int i = 0; i < kPer; ++i) sum += kMass ? s.hist.mass[lane * kPer + i] : s.hist.count[lane * kPer + i];
      u64 incl = sum;
#pragma unroll
      for (int d = 1; d < SRT_WAVE; d <<= 1) {
        const u64 y = __shfl_up(incl, d, SRT_WAVE);
        if (lane >= d) incl += y;
      }
      u64 before = incl - sum;
      int bin = kBins;
      for (int i = 0; i < kPer; ++i) {
        const u64 x = kMass ? s.hist.mass[lane * kPer + i] : s.hist.count[lane * kPer + i];
        if (x && base + static_cast<double>(before + x) >= target) {
          bin = lane * kPer + i;
          break;
        }
        before += x;
      }
      int best = bin;
#pragma unroll
      for (int d = SRT_WAVE / 2; d >= 1; d >>= 1) best = min(best, __shfl_xor(best, d, SRT_WAVE));
      if (best == kBins) {
        if (lane == 0) s.bin = -1;
      } else if (bin == best) {
        s.bin = bin;
        s.before = base + static_cast<double>(before);
        s.n = static_cast<int>(s.hist.count[bin]);
      }
    }
    __syncthreads();
  }

  // The first entry of the sorted list at which the measure reaches `target`, or the last one.
  template <bool kMass>
  __device__ __forceinline__ u64 in_list(int count, double target) {
    sort(count);
    if (tid == 0) s.found = s.list[count - 1];
    __syncthreads();
    if (wave == 0) {
      u64 run = 0;
      for (int i0 = 0; i0 < count; i0 += SRT_WAVE) {
        const int i = i0 + lane;
        const u64 x = i < count ? s.list[i] : 0ull;
        u64 incl = !x ? 0ull : kMass ? fixed(score_of(x)) : 1ull;
#pragma unroll
        for (int d = 1; d < SRT_WAVE; d <<= 1) {
          const u64 y = __shfl_up(incl, d, SRT_WAVE);
          if (lane >= d) incl += y;
        }
        const u64 hit = __ballot(x && static_cast<double>(run + incl) >= target);
        if (hit) {
          if (lane == __ffsll(static_cast<long long>(hit)) - 1) s.found = x;
          break;
        }
        run += __builtin_bit_cast(u64, __shfl(incl, SRT_WAVE - 1, SRT_WAVE));
      }
    }
    __syncthreads();
    return s.found;
  }

  // More tokens of the very score z than the list holds: the cut among them goes by
  // the token, whose range is narrowed in the same way.
  template <bool kMass>
  __device__ __forceinline__ u64 ties(float z, double target, double base) {
    const double each = kMass ? static_cast<double>(fixed(z)) : 1.0;
    const double r = each > 0.0 ? fmax(1.0, ceil((target - base) / each)) : INFINITY;  // tokens of the score that are kept
    const int width = (a.V + kBins - 1) / kBins;  // at most 1024
    __syncthreads();
    for (int i = tid; i < kBins; i += threads) s.hist.count[i] = 0;
    __syncthreads();
    visit(z, [&](float x, int j) {
      if (x == z) atomicAdd(&s.hist.count[j / width], 1u);
    });
    __syncthreads();
    find<false>(r, 0.0);
    const int bin = s.bin, count = s.n;
    const double above = s.before;
    if (bin < 0) return pack_key(z, a.V);  // all of them
    __syncthreads();
    if (tid == 0) s.n = 0;
    __syncthreads();
    visit(z, [&](float x, int j) {
      if (x != z || j / width != bin) return;
      const int at = atomicAdd(&s.n, 1);
      if (at < kList) s.list[at] = pack_key(x, j);  // (always, but for bias lists with a token's entries apart)
    });
    __syncthreads();
    return in_list<false>(min(count, kList), r - above);
  }

  // The choice at the node that the row belongs to: packed (score with noise, token), 0 if none.
  __device__ __forceinline__ u64 choose(int k, float p, float mp) {
    if (!(p > 0.f) || !(mp <= 1.f)) k = 1, p = 1.f, mp = 0.f;  // (a NaN too)
    if (k <= 0 || k > a.V) k = a.V;
    const bool by_k = k < a.V, by_p = p < 1.f, by_m = mp > 0.f;
    if (!w.noise || !(by_k || by_p || by_m)) return plain();
    const double mass = first_pass();
    if (M == -INFINITY) return 0;
    if (M == INFINITY) {  // one of the infinite scores: the lowest token, which is always kept
      u64 key = 0;
      visit(M, [&](float z, int j) { key = max(key, pack_key(z, j)); });
      return all_max(key);
    }
    // The scores below which nothing is kept.
    float least = -INFINITY;
    if (by_m) {  // the smallest float whose distance from M is no more than log(min_p)
      const double edge = static_cast<double>(M) + log(static_cast<double>(mp));
      least = static_cast<float>(edge);
      if (static_cast<double>(least) - static_cast<double>(M) < log(static_cast<double>(mp))) least = nextafterf(least, INFINITY);
    }
    const float by_min = least;
    if (by_k && by_p) least = -INFINITY;  // (the mass of the first k is needed)
    if (by_p && !by_k) {
      // tokens below this weigh no more than 1 - p of the row together
      const double d = log(static_cast<double>(a.V) / ((1.0 - static_cast<double>(p)) * mass));
      least = __builtin_fmaxf(least, M - static_cast<float>(d) - 0.01f);
    }
    if (by_k) least = __builtin_fmaxf(least, least_kept(k, INFINITY));
    else if (by_p) least = __builtin_fmaxf(least, least_kept(0x7fffffff, static_cast<double>(p) * mass));
    __syncthreads();
    if (tid == 0) s.n = 0;
    __syncthreads();
    visit(least, [&](float z, int j) {
      const int at = atomicAdd(&s.n, 1);
      if (at < kList) s.list[at] = pack_key(z, j);
    });
    __syncthreads();
    const int count = s.n;
    if (count <= kList) return from_list(count, k, by_p ? static_cast<double>(p) : 1.0, mass, by_min);
    // A long list: the last kept token first, then the choice among those from it up.
    u64 last = by_m ? pack_key(by_min, 0) & ~0xFFFFFFFFull : 0ull;
    double row_mass = mass;
    if (by_k) {
      const u64 cut = border<false>(k, least);
      last = max(last, cut);
      if (by_p) {
        double sum = 0.0;
        visit(least, [&](float z, int j) {
          if (pack_key(z, j) >= cut) sum += exp_of(z - M);
        });
        row_mass = all_sum(sum);
      }
    }
    if (by_p) last = max(last, border<true>(static_cast<double>(p) * row_mass * 1099511627776.0, least));
    u64 key = 0;
    visit(least, [&](float z, int j) {
      if (pack_key(z, j) >= last) take(key, z, j);
    });
    return all_max(key);
  }
};

template <bool kRules>
__global__ __launch_bounds__(kMost) void sample_walk_kernel(SampleArgs a) {
  __shared__ Lds s;
  __shared__ uint32_t skip[kRules ? kMaxRuled / 32 : 1];
  const int b = blockIdx.x, tid = threadIdx.x, threads = blockDim.x;
  const int64_t tr = static_cast<int64_t>(b) * a.N, orow = static_cast<int64_t>(b) * (a.Dmax + 1);
  const int n = min(max(a.n_nodes[b], 1), a.N);
  for (int c = tid; c < n; c += threads) {
    s.par[c] = a.tree_parent[tr + c];
    s.tok[c] = a.tree_tokens[tr + c];
  }
  const int lane = tid % SRT_WAVE, wave = __builtin_amdgcn_readfirstlane(tid / SRT_WAVE), e4 = a.V / 4;
  const int batches = (e4 + kUnroll * threads - 1) / (kUnroll * threads);
  Walker<kRules> walker = {a, s, skip, {}, 0, tid, threads, lane, wave, threads / SRT_WAVE, e4,
                           max(1, (batches + kSegs - 1) / kSegs), 0.f};
  const float p = a.top_p ? a.top_p[b] : 1.f, mp = a.min_p ? a.min_p[b] : 0.f;
  const int top_k = a.top_k ? a.top_k[b] : 0;
  int u = 0, k = 0, tok;
  for (;; ++k) {
    walker.w = rules_of(a, b, k);
    stand_on(a, walker.w, b, u);
    walker.w.invT = a.inv_temperature && a.gumbel ? a.inv_temperature[b] : 1.f;
    walker.n = k;
    if constexpr (kRules) mark(a, walker.w, s.path, k, 0, a.V, skip, threads);
    const u64 key = walker.choose(top_k, p, mp);
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
    sample_walk_kernel<true><<<static_cast<unsigned>(B), threads, 0, s>>>(a);
  } else {
    sample_walk_kernel<false><<<static_cast<unsigned>(B), threads, 0, s>>>(a);
  }
  return launch_status();
}
