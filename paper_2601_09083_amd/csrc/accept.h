// What the acceptance walks share: the level lists and candidates in the
// scratch, packed candidates and a step's decision.
#pragma once

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "common.h"

namespace {

using namespace srt;

typedef float f32x4 __attribute__((ext_vector_type(4)));
// Rows start at any multiple of 4 bytes (the hardware's requirement for its
// 16-byte loads too) when V is not a multiple of 4.
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kThreads = 256;
constexpr int kMaxN = 256;
constexpr int kMaxLevels = 64;   // Dmax + 1 <= 64
constexpr int kMaxChunks = 32;   // chunks per visited row, at most
constexpr int kMinChunk = 4096;  // vocabulary entries per chunk, at least
constexpr int kWalkWaves = 4;
// Entries (logits and noise) of a row that one workgroup walks faster than a
// launch per step: 64 sequences, 8-deep walks, sampled, V 1024 / 4096 / 16384 /
// 32768: 13 / 19 / 40 / 66 us against 47 / 58 / 59 / 59 with the level kernels
// (greedy 16384 / 32768 / 65536: 30 / 43 / 71 against 57 / 56 / 59; 512
// sequences alike).
constexpr int64_t kShortRow = 40960;
constexpr int kNarrowRow = 2048;  // rows up to this take 256 threads, longer ones 1024 (V 1024: 13 us against 15)

struct AcceptArgs {
  const float* logits;
  const float* gumbel;
  const int32_t* tree_tokens;
  const int32_t* tree_parent;
  const int32_t* n_nodes;
  int32_t* n_accepted;
  int32_t* out_tokens;
  int32_t* out_nodes;
  int32_t* n_emitted;
  int32_t* n_act;            // [kMaxLevels + 1] sequences walking at each level
  int32_t* act;              // [2, B] those sequences, by level parity
  int32_t* cur;              // [2, B] node each sequence stands on, by level parity
  unsigned long long* cand;  // [2, B, kMaxChunks] packed candidates of a level, by parity
  int B, N, V, Dmax, chunk, n_chunks;
  float invT;
};

// Scratch layout: level counters, two walker lists, current nodes, candidates.
struct ScratchLayout {
  size_t off_act, off_cur, off_cand, total;
};

constexpr size_t round256(size_t x) { return (x + 255) & ~size_t(255); }

constexpr ScratchLayout scratch_layout(int64_t B) {
  ScratchLayout s{};
  s.off_act = round256(sizeof(int32_t) * (kMaxLevels + 1));
  s.off_cur = s.off_act + round256(sizeof(int32_t) * 2 * static_cast<size_t>(B));
  s.off_cand = s.off_cur + round256(sizeof(int32_t) * 2 * static_cast<size_t>(B));
  s.total = s.off_cand + round256(sizeof(unsigned long long) * 2 * static_cast<size_t>(B) * kMaxChunks);
  return s;
}

__device__ inline unsigned long long pack_key(float x, int tok) {
  uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
  u = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return (static_cast<unsigned long long>(u) << 32) | static_cast<uint32_t>(~static_cast<uint32_t>(tok));
}

__device__ inline int key_token(unsigned long long k) {
  return static_cast<int>(~static_cast<uint32_t>(k & 0xFFFFFFFFull));
}

// The decision of step `level` for sequence b standing on node u, from the
// candidates of its row, in one wave: the token, and the child that carries
// it (-1 if none or if the walk is at its depth cap).
struct Step {
  int tok, child;
};

__device__ inline Step decide(const AcceptArgs& a, int b, int u, int level, int lane) {
  const unsigned long long* cand = a.cand + (static_cast<int64_t>(level & 1) * a.B + b) * kMaxChunks;
  const int64_t tr = static_cast<int64_t>(b) * a.N;
  // the node count and the tree row's first 64 nodes load together with the
  // candidates (their addresses do not depend on the step's token)
  const int n = min(max(a.n_nodes[b], 1), a.N);
  const int32_t par0 = lane < a.N ? a.tree_parent[tr + lane] : -1;
  const int32_t tok0 = lane < a.N ? a.tree_tokens[tr + lane] : -1;
  unsigned long long best = lane < a.n_chunks ? cand[lane] : 0ull;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const unsigned long long o = shfl_xor_u64(best, off);
    best = o > best ? o : best;
  }
  Step st{key_token(best), -1};
  if (level < a.Dmax) {  // children of u have larger indices
    unsigned long long m = __ballot(lane > u && lane < n && par0 == u && tok0 == st.tok);
    if (m) st.child = __ffsll(static_cast<long long>(m)) - 1;
    for (int c0 = SRT_WAVE; c0 < n && st.child < 0; c0 += SRT_WAVE) {
      const int cc = c0 + lane;
      const bool hit = cc > u && cc < n && a.tree_parent[tr + cc] == u && a.tree_tokens[tr + cc] == st.tok;
      m = __ballot(hit);
      if (m) st.child = c0 + __ffsll(static_cast<long long>(m)) - 1;
    }
  }
  return st;
}

// Host checks shared by the entry points (before any scratch is touched).
int check_args(int32_t B, int32_t N, int32_t V, int32_t Dmax, const float* logits, float inv_temperature,
               const int32_t* tree_tokens, const int32_t* tree_parent, const int32_t* n_nodes,
               const int32_t* n_accepted, const int32_t* out_tokens, const int32_t* out_nodes) {
  if (B < 0 || N < 1 || N > kMaxN || V < 1 || Dmax < 0 || Dmax >= kMaxLevels) return SRT_ERR_INVALID;
  if (!(inv_temperature == inv_temperature)) return SRT_ERR_INVALID;
  if (B == 0) return SRT_OK;
  if (!logits || !tree_tokens || !tree_parent || !n_nodes || !n_accepted || !out_tokens || !out_nodes)
    return SRT_ERR_INVALID;
  return SRT_OK;
}

// The walk's arguments on scratch memory `base` (device, 256-byte aligned, at
// least scratch_layout(B).total bytes).
AcceptArgs walk_args(int32_t B, int32_t N, int32_t V, int32_t Dmax, const float* logits, const float* gumbel,
                     float inv_temperature, const int32_t* tree_tokens, const int32_t* tree_parent,
                     const int32_t* n_nodes, int32_t* n_accepted, int32_t* out_tokens, int32_t* out_nodes,
                     int32_t* n_emitted, char* base, int unit) {
  const ScratchLayout L = scratch_layout(B);
  AcceptArgs a;
  a.logits = logits;
  a.gumbel = gumbel;
  a.tree_tokens = tree_tokens;
  a.tree_parent = tree_parent;
  a.n_nodes = n_nodes;
  a.n_accepted = n_accepted;
  a.out_tokens = out_tokens;
  a.out_nodes = out_nodes;
  a.n_emitted = n_emitted;
  a.n_act = reinterpret_cast<int32_t*>(base);
  a.act = reinterpret_cast<int32_t*>(base + L.off_act);
  a.cur = reinterpret_cast<int32_t*>(base + L.off_cur);
  a.cand = reinterpret_cast<unsigned long long*>(base + L.off_cand);
  a.B = B;
  a.N = N;
  a.V = V;
  a.Dmax = Dmax;
  // chunk: a multiple of `unit` of at least kMinChunk entries, at most kMaxChunks per row
  const int64_t per = (static_cast<int64_t>(V) + kMaxChunks - 1) / kMaxChunks;
  a.chunk = static_cast<int>(std::max<int64_t>(kMinChunk, (per + unit - 1) / unit * unit));
  a.n_chunks = static_cast<int>((static_cast<int64_t>(V) + a.chunk - 1) / a.chunk);
  a.invT = inv_temperature;
  return a;
}

}  // namespace
