// Rotary position encoding of a step's queries and keys, and the new keys and
// values written to their places in the paged cache.
//
// Method: the verification pass of Section 3 computes the queries, keys and values
// of every tree node; node i of sequence b is the token of position L + depth(i)
// and its vectors lie at slot L + i until the accepted path is moved into place.
// The pair (x0, x1) m of a head turns by the angle position * inv_freq[m]:
//   y0 = x0 cos - x1 sin,   y1 = x1 cos + x0 sin.
//
// GPU design: one read and one write of every vector, bound by HBM (16 prompts of up to
// 4096 tokens, 32 + 8 heads: 206 us a pass, 1.04 GB at 5.1 TB/s, the rate of a copy;
// 256 trees of up to 64 nodes, 28 + 4 heads: 37.2 us, 132 MB at 3.5 TB/s).  A wave
// takes a token.  Its lanes work out an angle each while the first heads' loads are
// under way, and hand them round through LDS: a lane keeps one 16-byte piece of the
// pairs for all heads that it visits, and the 8 (halves) or 4 (neighbouring dims)
// angles of it.  (Every lane working out its own: 42 us for those trees.  Two or four
// waves to a token work its angles out as often: the trees 43 and 52 us, prompts of
// 12 + 2 heads 73 against 94 and 143, and of one token per sequence no less than one.)
// Angles are formed in 64 bits and reduced to a part of a turn there -- in fp32
// position 10^6 would be off by 0.03 of a radian -- and their sine and cosine in fp32;
// products and sums are fp32 and a result is rounded to bf16 once.
#include <cmath>

#include "common.h"

using namespace srt;

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / SRT_WAVE;
constexpr int kMaxDims = 512;
constexpr int kBatch = 4;       // heads of a lane whose loads are under way together

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

struct RopeArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;        // nullptr: rows
  uint16_t* q_out;
  uint16_t* k_out;          // cache, or rows
  uint16_t* v_out;
  const float* inv_freq;
  const int32_t* depth;
  const int32_t* counts;
  const int32_t* ctx_len;
  const int32_t* bt;
  int64_t ldq, ldk, ldo, num_pages;
  int32_t B, T, Hq, Hkv, d, rot, page, max_pages;
  float factor;
};

__device__ inline float widen(uint16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }
__device__ inline uint16_t narrow(float x) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x)); }

template <bool kNeighbours, bool kCache>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
  constexpr int kPairs = kNeighbours ? 4 : 8;  // of a lane's piece
  __shared__ float2 turns_of[kWaves][kMaxDims / 2];
  const int lane = threadIdx.x % SRT_WAVE;
  // (a launch has fewer than 2^32 threads)
  const uint32_t wave = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / SRT_WAVE);
  const int b = static_cast<int>(wave / static_cast<uint32_t>(a.T));
  if (b >= a.B) return;
  const int i = static_cast<int>(wave - static_cast<uint32_t>(b) * a.T);
  const int64_t token = wave;
  if (i >= a.counts[b]) return;
  const int64_t L = a.ctx_len[b];
  const double pos = static_cast<double>(L + (a.depth ? a.depth[token] : i));

  // Where this token's keys and values go: k_at + head * k_step.
  int64_t k_at = token * a.ldo, k_step = a.d;
  bool stored = true;
  if constexpr (kCache) {
    const int64_t p = L + i;
    k_step = static_cast<int64_t>(a.page) * a.d;
    stored = p >= 0 && p < static_cast<int64_t>(a.max_pages) * a.page;
    const int pg = stored ? a.bt[static_cast<int64_t>(b) * a.max_pages + p / a.page] : -1;
    stored = pg >= 0 && pg < a.num_pages;
    k_at = static_cast<int64_t>(pg) * a.Hkv * k_step + p % a.page * a.d;
  }

  const int pieces = a.rot / (2 * kPairs);    // of a head
  const int abreast = SRT_WAVE / pieces;      // heads that a wave takes at a time
  const int c = lane % pieces, hs = lane / pieces;
  const int heads = a.Hq + a.Hkv;
  const uint16_t* q = a.q + token * a.ldq;
  const uint16_t* k = a.k + token * a.ldk;
  uint16_t* q_out = a.q_out + token * a.Hq * a.d;
  // A lane's 16 bytes are 8 first members of pairs and, half the rotated dims on,
  // their partners; or, of neighbouring dims, four whole pairs.
  const int at0 = 8 * c, at1 = kNeighbours ? 0 : at0 + a.rot / 2;
  u16x8 x0[kBatch], x1[kBatch];
  auto load = [&](int h0) {
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int h = h0 + j * abreast + hs;
      if (hs >= abreast || h >= heads) continue;
      const uint16_t* src = h < a.Hq ? q + h * a.d : k + (h - a.Hq) * a.d;
      x0[j] = *reinterpret_cast<const u16x8*>(src + at0);
      if (!kNeighbours) x1[j] = *reinterpret_cast<const u16x8*>(src + at1);
    }
  };
  load(0);
  // The angles' sines and cosines: a lane works out every 64th, and takes its own.
  // (The wave's part of LDS is its own: its writes come before its reads.)
  float2* turn = turns_of[threadIdx.x / SRT_WAVE];
  for (int m = lane; m < a.rot / 2; m += SRT_WAVE) {
    const double turns = pos * static_cast<double>(a.inv_freq[m]) * 0.15915494309189533577;  // 1 / (2 pi)
    float sine, cosine;
    sincospif(2.f * static_cast<float>(turns - rint(turns)), &sine, &cosine);
    turn[m] = make_float2(cosine * a.factor, sine * a.factor);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  float cs[kPairs], sn[kPairs];
#pragma unroll
  for (int e = 0; e < kPairs; ++e) {
    const float2 t = turn[kPairs * c + e];
    cs[e] = t.x;
    sn[e] = t.y;
  }
  for (int h0 = 0; h0 < heads; h0 += kBatch * abreast) {
    if (h0 > 0) load(h0);
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int h = h0 + j * abreast + hs;
      if (hs >= abreast || h >= heads) continue;
      u16x8 y0, y1;
#pragma unroll
      for (int e = 0; e < kPairs; ++e) {
        const float u = widen(kNeighbours ? x0[j][2 * e] : x0[j][e]);
        const float w = widen(kNeighbours ? x0[j][2 * e + 1] : x1[j][e]);
        const uint16_t r0 = narrow(u * cs[e] - w * sn[e]), r1 = narrow(w * cs[e] + u * sn[e]);
        if (kNeighbours) {
          y0[2 * e] = r0;
          y0[2 * e + 1] = r1;
        } else {
          y0[e] = r0;
          y1[e] = r1;
        }
      }
      if (h >= a.Hq && !stored) continue;
      uint16_t* dst = h < a.Hq ? q_out + h * a.d : a.k_out + k_at + (h - a.Hq) * k_step;
      *reinterpret_cast<u16x8*>(dst + at0) = y0;
      if (!kNeighbours) *reinterpret_cast<u16x8*>(dst + at1) = y1;
    }
  }

  // Dims that do not turn, and the values.
  const int rest = (a.d - a.rot) / 8;
  for (int x = lane; x < heads * rest; x += SRT_WAVE) {
    const int h = x / rest, at = a.rot + 8 * (x - h * rest);
    if (h >= a.Hq && !stored) continue;
    const uint16_t* src = h < a.Hq ? q + h * a.d : k + (h - a.Hq) * a.d;
    uint16_t* dst = h < a.Hq ? q_out + h * a.d : a.k_out + k_at + (h - a.Hq) * k_step;
    *reinterpret_cast<u16x8*>(dst + at) = *reinterpret_cast<const u16x8*>(src + at);
  }
  if constexpr (kCache) {
    const int per = a.d / 8;
    if (!stored) return;
    for (int x = lane; x < a.Hkv * per; x += SRT_WAVE) {
      const int h = x / per;
      *reinterpret_cast<u16x8*>(a.v_out + k_at + h * k_step + 8 * (x - h * per)) =
          *reinterpret_cast<const u16x8*>(a.v + token * a.ldk + 8 * x);
    }
  }
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// A token's heads side by side, `ld` elements from one token to the next.
bool rows_ok(int64_t ld, int32_t H, int32_t d) {
  return ld >= static_cast<int64_t>(H) * d && ld % 8 == 0 && ld <= (int64_t(1) << 31);
}

int check_rope(const srt_rope* rope, int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t d) {
  if (!rope || B < 0 || T < 1 || Hq < 1 || Hkv < 1 || d < 1 || rope->rot < 1 || rope->rot > d || rope->reserved != 0 ||
      (rope->interleaved & ~1) || !std::isfinite(rope->factor))
    return SRT_ERR_INVALID;
  if (d > kMaxDims || d % 8 || rope->rot % 16 || Hq > (1 << 16) || Hkv > (1 << 16)) return SRT_ERR_UNSUPPORTED;
  return SRT_OK;
}

int launch(RopeArgs& a, const srt_rope& rope, bool cache, void* stream) {
  a.inv_freq = rope.inv_freq;
  a.rot = rope.rot;
  a.factor = rope.factor;
  const int64_t tokens = static_cast<int64_t>(a.B) * a.T;
  const int64_t grid = (tokens + kWaves - 1) / kWaves;
  if (!launchable(grid, kThreads)) return SRT_ERR_UNSUPPORTED;
  hipStream_t s = as_stream(stream);
  const unsigned n = static_cast<unsigned>(grid);
  if (rope.interleaved) {
    if (cache) rope_kernel<true, true><<<n, kThreads, 0, s>>>(a);
    else rope_kernel<true, false><<<n, kThreads, 0, s>>>(a);
  } else {
    if (cache) rope_kernel<false, true><<<n, kThreads, 0, s>>>(a);
    else rope_kernel<false, false><<<n, kThreads, 0, s>>>(a);
  }
  return launch_status();
}

}  // namespace

extern "C" int srt_rope_append(const srt_rope* rope, int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t d,
                               int32_t page, int32_t max_pages, int64_t num_pages, const uint16_t* q, int64_t ldq,
                               const uint16_t* k, const uint16_t* v, int64_t ldkv, const int32_t* depth,
                               const int32_t* counts, uint16_t* q_out, uint16_t* k_cache, uint16_t* v_cache,
                               const int32_t* block_table, const int32_t* ctx_len, void* stream) {
  const int st = check_rope(rope, B, T, Hq, Hkv, d);
  if (st != SRT_OK) return st;
  if (page < 1 || max_pages < 1 || num_pages < 1 || !rows_ok(ldq, Hq, d) || !rows_ok(ldkv, Hkv, d)) return SRT_ERR_INVALID;
  if (B == 0) return SRT_OK;
  if (!rope->inv_freq || !q || !k || !v || !counts || !q_out || !k_cache || !v_cache || !block_table || !ctx_len)
    return SRT_ERR_INVALID;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(k_cache) || !aligned16(v_cache))
    return SRT_ERR_INVALID;
  RopeArgs a = {q,      k,   v,    q_out, k_cache, v_cache,   nullptr, depth, counts, ctx_len, block_table,
                ldq,    ldkv, 0,   num_pages, B,   T,         Hq,      Hkv,   d,      0,       page,
                max_pages, 0.f};
  return launch(a, *rope, true, stream);
}

extern "C" int srt_rope_rows(const srt_rope* rope, int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t d,
                             const uint16_t* q, int64_t ldq, const uint16_t* k, int64_t ldk, const int32_t* depth,
                             const int32_t* counts, const int32_t* ctx_len, uint16_t* q_out, uint16_t* k_out,
                             int64_t ldo, void* stream) {
  const int st = check_rope(rope, B, T, Hq, Hkv, d);
  if (st != SRT_OK) return st;
  if (!rows_ok(ldq, Hq, d) || !rows_ok(ldk, Hkv, d) || !rows_ok(ldo, Hkv, d)) return SRT_ERR_INVALID;
  if (B == 0) return SRT_OK;
  if (!rope->inv_freq || !q || !k || !counts || !ctx_len || !q_out || !k_out) return SRT_ERR_INVALID;
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out)) return SRT_ERR_INVALID;
  RopeArgs a = {q,   k,    nullptr, q_out, k_out, nullptr, nullptr, depth, counts, ctx_len, nullptr,
                ldq, ldk,  ldo,     0,     B,     T,       Hq,      Hkv,   d,      0,       1,
                1,   0.f};
  return launch(a, *rope, false, stream);
}
