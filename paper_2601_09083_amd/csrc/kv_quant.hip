// Writing and reading the 8-bit KV cache: new tokens, accepted paths, and
// positions back as bf16.
//
// Method: the accepted path of a verification pass becomes context (Section 3
// of the paper, classic speculative decoding; commit.hip does it for a bf16
// cache).  Here the context's open page is kept in bf16 and quantised once, when
// it is full: with amp = max(max |x|, 2^-60) over the page's values of a KV head
// and top = 448 (e4m3) or 127 (int8), scale = amp / top and the codes are
// x * (top / amp) rounded to nearest even.  (Quantising token by token would
// either fix a scale before the page's values are known or round the codes
// that are there again each time it grows.)
//
// GPU design.  The unit is a page of one KV head and tensor: a wave holds it in
// registers (a lane 8 elements of a row at a time), takes the maximum, and writes
// codes and scale.  A call with few tokens (accepted paths, single tokens) runs
// in one launch, a workgroup per sequence whose waves share out the heads and
// tensors and which advances the sequence's state at its end; long appends
// have a wave for every page and a second launch for the lengths.  In both, the
// wave that reads a sequence's tail also writes what is left over to it, after
// its reads have returned.  Bound by HBM: 2 bytes in, 1 out per value.
#include <algorithm>

#include "kv_quant.h"

using namespace srt;

namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * SRT_WAVE;
constexpr int kShort = 64;       // new tokens a sequence, up to which one workgroup writes them
constexpr float kLeastAmp = 0x1p-60f;

struct WriteArgs {
  uint8_t* pages[2];  // K, V
  float* scale[2];
  uint16_t* tail[2];
  const uint16_t* fresh[2];  // new rows [B, T, .. ld]
  const int32_t* bt;
  int32_t* ctx_len;
  const int32_t* counts;     // append: new tokens; commit: accepted nodes
  const int32_t* nodes;      // commit: [B, Dmax + 1], else nullptr
  const int32_t* emitted;    // commit: [B, Dmax + 1]
  int32_t* ctx_tail;
  int32_t* draft_len;
  int64_t ld, num_pages;
  int32_t B, T, Hkv, page, page_shift, max_pages, ctx_cap, Dmax, Qmax, e4m3;
};

// Where a sequence stands: L positions, m new rows that have room.
struct Span {
  int L, m;
};

__device__ inline Span span_of(const WriteArgs& a, int b) {
  Span s;
  s.L = min(max(a.ctx_len[b], 0), a.ctx_cap);
  s.m = a.counts[b];
  s.m = a.nodes ? min(max(s.m, 0), min(a.Dmax, a.T - 1)) + 1 : min(max(s.m, 0), a.T);
  s.m = min(s.m, a.ctx_cap - s.L);
  return s;
}

// Calls on more bf16 rows (K and V together) than the caches keep until their next
// use read and write them non-temporally: prompts of 32 sequences, 268 MB of
// rows, appended and read back 135 us with ordinary accesses, 121 so; 33 MB of
// them 27.0 and 29.5.
constexpr int64_t kStreamBytes = int64_t(128) << 20;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Code bytes of two values already scaled; e4m3's conversion and rint round to
// nearest even.
__device__ inline uint32_t codes2(float x, float y, float top, bool e4m3) {
  x = fminf(fmaxf(x, -top), top);
  y = fminf(fmaxf(y, -top), top);
  if (e4m3) return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x, y, 0, false)) & 0xffffu;
  return (static_cast<uint32_t>(static_cast<int>(rintf(x))) & 0xffu) |
         ((static_cast<uint32_t>(static_cast<int>(rintf(y))) & 0xffu) << 8);
}

__device__ inline uint2 codes8(const uint4& w, float inv, float top, bool e4m3) {
  const uint32_t c0 = codes2(bf16_lo(w.x) * inv, bf16_hi(w.x) * inv, top, e4m3);
  const uint32_t c1 = codes2(bf16_lo(w.y) * inv, bf16_hi(w.y) * inv, top, e4m3);
  const uint32_t c2 = codes2(bf16_lo(w.z) * inv, bf16_hi(w.z) * inv, top, e4m3);
  const uint32_t c3 = codes2(bf16_lo(w.w) * inv, bf16_hi(w.w) * inv, top, e4m3);
  return make_uint2(c0 | (c1 << 16), c2 | (c3 << 16));
}

// Largest magnitude of 8 values so far, as bf16 bits in both halves of m (the
// bits of magnitudes are ordered as the values are).
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ inline u16x2 amp8(const uint4& w, u16x2 m) {
  const uint32_t mag = 0x7fff7fffu;
  m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w.x & mag));
  m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w.y & mag));
  m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w.z & mag));
  return __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w.w & mag));
}

// One sequence, KV head and tensor, seen by one wave.
template <int D>
struct Head {
  static constexpr int kLanes = D / 8;               // lanes per row, 8 elements each
  static constexpr int kRows = SRT_WAVE / kLanes;    // rows per load: 4 or 8
  const WriteArgs& a;
  int b, g, t, lane;
  Span s;

  __device__ uint16_t* tail_row(int r) const {
    return a.tail[t] + ((static_cast<int64_t>(b) * a.Hkv + g) * a.page + r) * D + (lane % kLanes) * 8;
  }
  // Row of position p, L <= p < L + m: new token p - L, or the accepted node.
  __device__ const uint16_t* new_row(int p) const {
    int j = p - s.L;
    if (a.nodes) j = j == 0 ? 0 : min(max(a.nodes[static_cast<int64_t>(b) * (a.Dmax + 1) + j - 1], 0), a.T - 1);
    return a.fresh[t] + (static_cast<int64_t>(b) * a.T + j) * a.ld + static_cast<int64_t>(g) * D + (lane % kLanes) * 8;
  }
  template <bool kStream>
  __device__ uint4 row(int p) const {
    const u32x4* from = reinterpret_cast<const u32x4*>(p < s.L ? tail_row(p & (a.page - 1)) : new_row(p));
    return __builtin_bit_cast(uint4, kStream ? __builtin_nontemporal_load(from) : *from);
  }

  // Quantises the full page that starts at position p0.  Pages of 16, 32 and 64
  // tokens (kKeep = 1, 2, 4 times 16 rows) are read once and held in registers,
  // larger ones are read again for their codes.
  template <int kKeep, bool kStream>
  __device__ void page(int p0) const {
    constexpr int kPer = 16 / kRows;  // loads per 16 rows
    const int pg = a.bt[static_cast<int64_t>(b) * a.max_pages + (p0 >> a.page_shift)];
    if (pg < 0 || pg >= a.num_pages) return;
    const float top = a.e4m3 ? 448.f : 127.f;
    const int lr = lane / kLanes;
    uint4 x[kKeep][kPer];
    auto load = [&](int r0, uint4 (&y)[kPer]) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) y[i] = row<kStream>(p0 + r0 + i * kRows + lr);
    };
    u16x2 m2 = {0, 0};
#pragma unroll
    for (int k = 0; k < kKeep; ++k) load(k * 16, x[k]);
#pragma unroll
    for (int k = 0; k < kKeep; ++k)
#pragma unroll
      for (int i = 0; i < kPer; ++i) m2 = amp8(x[k][i], m2);
    if constexpr (kKeep == 4)
      for (int r0 = kKeep * 16; r0 < a.page; r0 += 16) {
        uint4 y[kPer];
        load(r0, y);
#pragma unroll
        for (int i = 0; i < kPer; ++i) m2 = amp8(y[i], m2);
      }
    float m = __uint_as_float(static_cast<uint32_t>(max(m2[0], m2[1])) << 16);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, SRT_WAVE));
    m = fmaxf(m, kLeastAmp);
    const float inv = __fdiv_rn(top, m);
    const int64_t at = static_cast<int64_t>(pg) * a.Hkv + g;
    if (lane == 0) a.scale[t][at] = __fdiv_rn(m, top);
    uint8_t* out = a.pages[t] + at * a.page * D + (lane % kLanes) * 8;
    auto store = [&](int r0, const uint4 (&y)[kPer]) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        u32x2* to = reinterpret_cast<u32x2*>(out + static_cast<int64_t>(r0 + i * kRows + lr) * D);
        const u32x2 c = __builtin_bit_cast(u32x2, codes8(y[i], inv, top, a.e4m3));
        if constexpr (kStream) __builtin_nontemporal_store(c, to);
        else *to = c;
      }
    };
#pragma unroll
    for (int k = 0; k < kKeep; ++k) store(k * 16, x[k]);
    if constexpr (kKeep == 4)
      for (int r0 = kKeep * 16; r0 < a.page; r0 += 16) {
        uint4 y[kPer];
        load(r0, y);
        store(r0, y);
      }
  }

  // The new rows of the page that stays open go to the tail.
  __device__ void rest() const {
    const int end = s.L + s.m, lr = lane / kLanes;
    const int from = max(s.L, end & ~(a.page - 1));
    // every read of the tail has returned before it is written
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    for (int p = from; p < end; p += kRows)
      if (p + lr < end)
        *reinterpret_cast<uint4*>(tail_row((p + lr) & (a.page - 1))) = *reinterpret_cast<const uint4*>(new_row(p + lr));
  }
};

// Few new tokens: a workgroup per sequence, and for a commit one wave more for
// the draft inputs.
template <int D, int kKeep>
__global__ __launch_bounds__(kThreads + SRT_WAVE) void write_short_kernel(WriteArgs a) {
  const int b = blockIdx.x, wave = threadIdx.x / SRT_WAVE;
  const Span s = span_of(a, b);
  const int first = s.L & ~(a.page - 1), end = s.L + s.m;
  if (wave < kWaves) {
    for (int i = wave; i < 2 * a.Hkv; i += kWaves) {
      const Head<D> head = {a, b, i >> 1, i & 1, static_cast<int>(threadIdx.x) % SRT_WAVE, s};
      for (int p = first; p + a.page <= end; p += a.page) head.template page<kKeep, false>(p);
      head.rest();
    }
  } else {
    const int k = min(max(a.counts[b], 0), min(a.Dmax, a.T - 1));
    advance_draft(a.ctx_tail + static_cast<int64_t>(b) * a.Qmax, a.Qmax, a.draft_len + b,
                  a.emitted + static_cast<int64_t>(b) * (a.Dmax + 1), k);
  }
  __syncthreads();  // every thread has read ctx_len[b]
  if (threadIdx.x == 0) a.ctx_len[b] = end;
}

// Many new tokens: a wave per page, KV head and tensor.  The wave of a
// sequence's first page writes the tail too.
template <int D, int kKeep, bool kStream>
__global__ __launch_bounds__(kThreads) void write_pages_kernel(WriteArgs a, int pages, int heads_at_once) {
  const int x = blockIdx.x / heads_at_once, y = blockIdx.x - x * heads_at_once;
  const int b = x / pages, i = x - b * pages;
  const int head_no = y * kWaves + threadIdx.x / SRT_WAVE;
  if (head_no >= 2 * a.Hkv) return;
  const Span s = span_of(a, b);
  const Head<D> head = {a, b, head_no >> 1, head_no & 1, static_cast<int>(threadIdx.x) % SRT_WAVE, s};
  const int p = (s.L & ~(a.page - 1)) + i * a.page;
  if (p + a.page <= s.L + s.m) head.template page<kKeep, kStream>(p);
  if (i == 0) head.rest();
}

__global__ __launch_bounds__(256) void advance_kernel(WriteArgs a) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= a.B) return;
  const Span s = span_of(a, b);
  a.ctx_len[b] = s.L + s.m;
}

// ---------------------------------------------------------------------------
// Positions back as bf16
// ---------------------------------------------------------------------------
struct ReadArgs {
  const uint8_t* pages[2];
  const float* scale[2];
  const uint16_t* tail[2];
  uint16_t* out[2];
  const int32_t* bt;
  const int32_t* ctx_len;
  const int32_t* start;
  int64_t num_pages, items;
  int32_t T, Hkv, page, page_shift, max_pages, ctx_cap, e4m3;
};

__device__ inline uint32_t pack_bf16(float lo, float hi) {
  return static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<__bf16>(lo))) |
         (static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<__bf16>(hi))) << 16);
}

// Four codes times the scale, in fp32 and rounded once.
__device__ inline uint2 values4(uint32_t w, float s, bool e4m3) {
  float f[4];
  if (e4m3) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    f[0] = lo[0];
    f[1] = lo[1];
    f[2] = hi[0];
    f[3] = hi[1];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = static_cast<int8_t>(w >> (8 * i));
  }
  return make_uint2(pack_bf16(f[0] * s, f[1] * s), pack_bf16(f[2] * s, f[3] * s));
}

// A thread takes 16 consecutive elements of a token's KV head, for K or V (y).
template <int D, bool kStream>
__global__ __launch_bounds__(256) void read_kernel(ReadArgs a) {
  constexpr int kLanes = D / 16;
  const int t = blockIdx.y;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < a.items;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int c = static_cast<int>(i % kLanes);
    const int64_t hd = i / kLanes;           // (b, token, head)
    const int g = static_cast<int>(hd % a.Hkv);
    const int64_t bt = hd / a.Hkv;
    const int64_t b = bt / a.T;
    const int64_t p = static_cast<int64_t>(a.start[b]) + (bt - b * a.T);
    const int L = min(max(a.ctx_len[b], 0), a.ctx_cap);
    if (p < 0 || p >= L) continue;
    const int slot = static_cast<int>(p) & (a.page - 1);
    uint4 lo, hi;
    if (p >= (L & ~(a.page - 1))) {
      const uint4* from = reinterpret_cast<const uint4*>(a.tail[t] + ((b * a.Hkv + g) * a.page + slot) * D + c * 16);
      lo = from[0];
      hi = from[1];
    } else {
      const int pg = a.bt[b * a.max_pages + (p >> a.page_shift)];
      uint4 w = make_uint4(0, 0, 0, 0);
      float s = 0.f;
      if (pg >= 0 && pg < a.num_pages) {
        const int64_t at = static_cast<int64_t>(pg) * a.Hkv + g;
        w = *reinterpret_cast<const uint4*>(a.pages[t] + (at * a.page + slot) * D + c * 16);
        s = a.scale[t][at];
      }
      const uint2 x0 = values4(w.x, s, a.e4m3), x1 = values4(w.y, s, a.e4m3);
      const uint2 x2 = values4(w.z, s, a.e4m3), x3 = values4(w.w, s, a.e4m3);
      lo = make_uint4(x0.x, x0.y, x1.x, x1.y);
      hi = make_uint4(x2.x, x2.y, x3.x, x3.y);
    }
    u32x4* to = reinterpret_cast<u32x4*>(a.out[t] + hd * D + c * 16);
    if constexpr (kStream) {
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, lo), to);
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, hi), to + 1);
    } else {
      to[0] = __builtin_bit_cast(u32x4, lo);
      to[1] = __builtin_bit_cast(u32x4, hi);
    }
  }
}

template <int D, int kKeep>
void launch_write(const WriteArgs& a, bool one_launch, int pages, int at_once, hipStream_t s) {
  if (one_launch) {
    write_short_kernel<D, kKeep>
        <<<static_cast<unsigned>(a.B), kThreads + (a.nodes && a.ctx_tail ? SRT_WAVE : 0), 0, s>>>(a);
    return;
  }
  const unsigned grid = static_cast<unsigned>(static_cast<int64_t>(pages) * at_once * a.B);
  if (static_cast<int64_t>(a.B) * a.T * a.Hkv * D * 4 >= kStreamBytes)
    write_pages_kernel<D, kKeep, true><<<grid, kThreads, 0, s>>>(a, pages, at_once);
  else
    write_pages_kernel<D, kKeep, false><<<grid, kThreads, 0, s>>>(a, pages, at_once);
}

int launch_write(const WriteArgs& a, int d, bool one_launch, int pages, int at_once, hipStream_t s) {
  if (d == 128) {
    if (a.page == 16) launch_write<128, 1>(a, one_launch, pages, at_once, s);
    else if (a.page == 32) launch_write<128, 2>(a, one_launch, pages, at_once, s);
    else launch_write<128, 4>(a, one_launch, pages, at_once, s);
  } else {
    if (a.page == 16) launch_write<64, 1>(a, one_launch, pages, at_once, s);
    else if (a.page == 32) launch_write<64, 2>(a, one_launch, pages, at_once, s);
    else launch_write<64, 4>(a, one_launch, pages, at_once, s);
  }
  return launch_status();
}

void fill(WriteArgs& a, const srt_kv_quant& kv, int32_t B, int32_t T, const uint16_t* k_new, const uint16_t* v_new,
          int64_t ld) {
  a.pages[0] = kv.k_pages;
  a.pages[1] = kv.v_pages;
  a.scale[0] = kv.k_scale;
  a.scale[1] = kv.v_scale;
  a.tail[0] = kv.k_tail;
  a.tail[1] = kv.v_tail;
  a.fresh[0] = k_new;
  a.fresh[1] = v_new;
  a.bt = kv.block_table;
  a.ctx_len = kv.ctx_len;
  a.nodes = a.emitted = nullptr;
  a.ctx_tail = a.draft_len = nullptr;
  a.ld = ld;
  a.num_pages = kv.num_pages;
  a.B = B;
  a.T = T;
  a.Hkv = kv.Hkv;
  a.page = kv.page;
  a.page_shift = __builtin_ctz(static_cast<unsigned>(kv.page));
  a.max_pages = kv.max_pages;
  a.ctx_cap = (kv.max_pages + 1) * kv.page - 1;
  a.Dmax = a.Qmax = 0;
  a.e4m3 = kv.kv_type == SRT_KV_E4M3;
}

}  // namespace

extern "C" int srt_kv_append(const srt_kv_quant* kv, int32_t B, int32_t T, const uint16_t* k_new,
                             const uint16_t* v_new, int64_t ld, const int32_t* counts, void* stream) {
  if (!kv || B < 0 || T < 1) return SRT_ERR_INVALID;
  int st = check_kv_sizes(*kv);
  if (st != SRT_OK) return st;
  const int64_t pages = (static_cast<int64_t>(T) + 2 * kv->page - 2) / kv->page;  // that L % page + T tokens touch
  const int64_t at_once = (2 * kv->Hkv + kWaves - 1) / kWaves;
  const int64_t per_seq = T <= kShort ? 1 : pages * at_once;  // workgroups
  if (!launchable(per_seq, kThreads) || !launchable(per_seq * B, kThreads)) return SRT_ERR_UNSUPPORTED;
  if (B == 0) return SRT_OK;
  st = check_kv_pointers(*kv);
  if (st == SRT_OK) st = check_new(*kv, k_new, v_new, ld);
  if (st != SRT_OK) return st;
  if (!counts) return SRT_ERR_INVALID;
  WriteArgs a;
  fill(a, *kv, B, T, k_new, v_new, ld);
  a.counts = counts;
  hipStream_t s = as_stream(stream);
  st = launch_write(a, kv->d, T <= kShort, static_cast<int>(pages), static_cast<int>(at_once), s);
  if (st != SRT_OK || T <= kShort) return st;
  advance_kernel<<<static_cast<unsigned>((B + 255) / 256), 256, 0, s>>>(a);
  return launch_status();
}

extern "C" int srt_commit_quant(const srt_kv_quant* kv, int32_t B, int32_t N, const uint16_t* k_new,
                                const uint16_t* v_new, int64_t ld, int32_t Dmax, const int32_t* n_accepted,
                                const int32_t* out_tokens, const int32_t* out_nodes, int32_t max_match,
                                int32_t* ctx_tail, int32_t* draft_len, void* stream) {
  if (!kv || B < 0 || N < 1 || N > 256 || Dmax < 0 || Dmax > 63) return SRT_ERR_INVALID;
  int st = check_kv_sizes(*kv);
  if (st != SRT_OK) return st;
  if ((ctx_tail == nullptr) != (draft_len == nullptr)) return SRT_ERR_INVALID;
  if (ctx_tail && (max_match < 1 || max_match > 64)) return SRT_ERR_INVALID;
  if (!launchable(B, kThreads + (ctx_tail ? SRT_WAVE : 0))) return SRT_ERR_UNSUPPORTED;
  if (B == 0) return SRT_OK;
  st = check_kv_pointers(*kv);
  if (st == SRT_OK) st = check_new(*kv, k_new, v_new, ld);
  if (st != SRT_OK) return st;
  if (!n_accepted || !out_tokens || !out_nodes) return SRT_ERR_INVALID;
  WriteArgs a;
  fill(a, *kv, B, N, k_new, v_new, ld);
  a.counts = n_accepted;
  a.nodes = out_nodes;
  a.emitted = out_tokens;
  a.ctx_tail = ctx_tail;
  a.draft_len = draft_len;
  a.Dmax = Dmax;
  a.Qmax = ctx_tail ? max_match : 0;
  return launch_write(a, kv->d, true, 0, 0, as_stream(stream));
}

extern "C" int srt_kv_read(const srt_kv_quant* kv, int32_t B, int32_t T, const int32_t* start, uint16_t* k_out,
                           uint16_t* v_out, void* stream) {
  if (!kv || B < 0 || T < 1) return SRT_ERR_INVALID;
  int st = check_kv_sizes(*kv);
  if (st != SRT_OK) return st;
  if (B == 0) return SRT_OK;
  st = check_kv_pointers(*kv);
  if (st != SRT_OK) return st;
  if (!start || !k_out || !v_out) return SRT_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out)) % 16) return SRT_ERR_INVALID;
  ReadArgs a;
  a.pages[0] = kv->k_pages;
  a.pages[1] = kv->v_pages;
  a.scale[0] = kv->k_scale;
  a.scale[1] = kv->v_scale;
  a.tail[0] = kv->k_tail;
  a.tail[1] = kv->v_tail;
  a.out[0] = k_out;
  a.out[1] = v_out;
  a.bt = kv->block_table;
  a.ctx_len = kv->ctx_len;
  a.start = start;
  a.num_pages = kv->num_pages;
  a.items = static_cast<int64_t>(B) * T * kv->Hkv * (kv->d / 16);
  a.T = T;
  a.Hkv = kv->Hkv;
  a.page = kv->page;
  a.page_shift = __builtin_ctz(static_cast<unsigned>(kv->page));
  a.max_pages = kv->max_pages;
  a.ctx_cap = (kv->max_pages + 1) * kv->page - 1;
  a.e4m3 = kv->kv_type == SRT_KV_E4M3;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>((a.items + 255) / 256, 1 << 20)), 2);
  hipStream_t s = as_stream(stream);
  const bool streams = a.items * 64 >= kStreamBytes;  // (16 elements of K and V an item)
  if (kv->d == 128) {
    if (streams) read_kernel<128, true><<<grid, 256, 0, s>>>(a);
    else read_kernel<128, false><<<grid, 256, 0, s>>>(a);
  } else {
    if (streams) read_kernel<64, true><<<grid, 256, 0, s>>>(a);
    else read_kernel<64, false><<<grid, 256, 0, s>>>(a);
  }
  return launch_status();
}
