// What the tree attention kernels share: the work list that the plan kernel
// builds, the combine of split contexts and the host's rules for both.  Each
// source that includes this has its own copy of the kernels.
#pragma once

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.h"

namespace {

using namespace srt;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * SRT_WAVE;
constexpr int kRowsPerWave = 32;
constexpr int kRowsPerBlock = kWaves * kRowsPerWave;
constexpr int kTile = 64;                  // keys per tile
constexpr int kSubRows = kTile / kWaves;   // keys of each tile one wave stages
constexpr int kMaxN = 256;                 // tree rows
constexpr int kChunk = 8192;               // keys per split, at most (the split size is chosen per call)
constexpr int kMinChunk = 1024;            // keys per split, at least
constexpr int kSmallChunk = 256;           // the same where every split has a CU of its own
constexpr int kSmallItems = 256;           // work items up to which that is so (one per CU)
constexpr int kSmallSplits = 32;           // splits of a context then, at most

// What every kernel of an attention call reads; the kernel proper adds its cache.
struct AttnBase {
  const int32_t* ctx_len;
  const int32_t* n_nodes;
  uint16_t* out;
  float* part_o;
  float* part_ml;
  int32_t* plan;  // work lists built by the plan kernel
  int64_t combine_at;  // offset (int32 elements) of the combine list in plan
  int32_t B, N, Hq, Hkv, G;
  int32_t cap;      // positions that context and tree may take together
  int32_t tree_room;  // of them, those that no context may take
  int32_t S, RB, total;
  int32_t part_rows;  // rows of a partial result
  int32_t chunk;  // keys per split: a power of two in [kSmallChunk, kChunk]
};

// Work list: plan[0] = number of items, plan[1] = next item to hand out,
// then item i at plan[kPlanHeader + 2 i] = sequence, [.. + 1] = KV head |
// split << 8 | row block << 20.  Items are ordered by decreasing cost
// (tiles, then active waves) so that the longest ones start first.
// plan[2] = number of sequences whose context spans several splits; entry e of
// them at plan[a.combine_at + 2 e] = sequence | splits << 16 (the host rejects
// B > 65535 and more than 4095 splits) and [.. + 1] = its query rows per KV
// head; plan[3] = 8-row groups of the widest of them.  (Listing every group
// here took one thread per sequence 20 to 40 us of stores; the combine kernel
// works the group out instead.)
constexpr int kPlanHeader = 64;
constexpr int kFewItems = 8;  // of a sequence, up to which its thread of the plan kernel lists them
constexpr int kCombineRows = 8;
constexpr int kPlanKeys = (kChunk / kTile) * kWaves;  // (tiles, waves) classes

__device__ inline int plan_key(int tiles, int waves) {  // 0 = most expensive
  return kPlanKeys - 1 - ((tiles - 1) * kWaves + (waves - 1));
}

template <int D>
struct Shape {
  static constexpr int KS = D / 16;            // k-steps of S^T = K Q^T
  static constexpr int DB = D / 32;            // 32-dim blocks of O^T
  static constexpr int CPR = D / 8;            // 16-byte chunks per K/V row
  static constexpr int KSTRIDE = 2 * D + 16;   // LDS bytes per K row
  static constexpr int VSTRIDE = 2 * D + 32;   // LDS bytes per V row
  static constexpr int KTILE = kTile * KSTRIDE;
  static constexpr int VTILE = kTile * VSTRIDE;
};

__device__ inline uint16_t to_bf16_bits(float x) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x)); }

struct SeqInfo {
  int n, L, total;
};

// (One limit, in scalar operations: with min(cap - n, the context's own limit) the
// compiler takes the vector unit's minimum of three, and the bf16 cache's attention of
// 256 sequences 723 us a call for 715.)
__device__ inline SeqInfo seq_info(const AttnBase& a, int b) {
  SeqInfo s;
  s.n = min(max(a.n_nodes[b], 1), min(a.N, a.cap));
  s.L = min(max(a.ctx_len[b], 0), a.cap - max(s.n, a.tree_room));
  s.total = s.L + s.n;
  return s;
}

// The two 32-lane halves of x exchanged by v_permlane32_swap: returns
// {x, x of lane ^ 32} in some order.  (Each result element is copied to a
// scalar before the bit cast: a bit cast of a vector element reads
// element 0 with this compiler.)
__device__ inline void swap_halves(float x, float& u, float& v) {
  const unsigned a = __builtin_bit_cast(unsigned, x);
  const auto s = __builtin_amdgcn_permlane32_swap(a, a, false, false);
  const unsigned s0 = s[0], s1 = s[1];
  u = __builtin_bit_cast(float, s0);
  v = __builtin_bit_cast(float, s1);
}

// Maximum / sum over the two 32-lane halves, result in every lane.
__device__ inline float max_halves(float x) {
  float u, v;
  swap_halves(x, u, v);
  return __builtin_elementwise_maximum(u, v);
}

__device__ inline float sum_halves(float x) {
  float u, v;
  swap_halves(x, u, v);
  return u + v;
}

// Builds the work list: one item per (sequence, KV head, split, row block)
// that has work, counting-sorted by decreasing (tiles, active waves of the
// first row block).  The row blocks of one (sequence, KV head, split) are
// listed next to each other, so workgroups that take them start at about
// the same time and the second stream of the same K/V tiles is served by
// the caches.  One workgroup; also resets the hand-out counter.
__global__ __launch_bounds__(1024) void tree_attn_plan_kernel(AttnBase a) {
  __shared__ int32_t cnt[kPlanKeys], off[kPlanKeys];
  __shared__ int32_t wsum[1024 / SRT_WAVE];
  __shared__ int32_t s_total[1024], s_rows[1024], s_pos[2][1024];
  __shared__ int32_t ncomb, widest;
  const int tid = threadIdx.x;
  for (int k = tid; k < kPlanKeys; k += 1024) cnt[k] = 0;
  if (tid == 0) ncomb = widest = 0;
  const int cshift = 31 - __clz(a.chunk);  // chunk is a power of two
  // Visits the item classes of a sequence: f(key, splits).
  auto classes = [&](int total, int rows, auto&& f) {
    const int full = total >> cshift;
    const int tail = total - (full << cshift);
    const int waves = min(kWaves, (rows + kRowsPerWave - 1) / kRowsPerWave);
    if (full > 0) f(0, plan_key(a.chunk / kTile, waves), full);
    if (tail > 0) f(1, plan_key((tail + kTile - 1) / kTile, waves), 1);
  };
  auto row_blocks = [&](int rows) { return (rows + kRowsPerBlock - 1) / kRowsPerBlock; };
  SeqInfo si = {0, 0, 0};  // of this thread's sequence of the current 1024
  if (tid < a.B) si = seq_info(a, tid);
  __syncthreads();
  for (int b0 = 0; b0 < a.B; b0 += 1024) {
    if (b0 > 0 && b0 + tid < a.B) si = seq_info(a, b0 + tid);
    if (b0 + tid < a.B)
      classes(si.total, si.n * a.G,
              [&](int, int key, int ns) { atomicAdd(&cnt[key], ns * a.Hkv * row_blocks(si.n * a.G)); });
  }
  __syncthreads();
  // Exclusive prefix sum of the class counts (one class per thread).
  static_assert(kPlanKeys <= 1024, "one class per thread");
  const int lane = tid % SRT_WAVE, wv = tid / SRT_WAVE;
  const int mine = tid < kPlanKeys ? cnt[tid] : 0;
  int incl = mine;
#pragma unroll
  for (int d = 1; d < SRT_WAVE; d <<= 1) {
    const int y = __shfl_up(incl, d, SRT_WAVE);
    if (lane >= d) incl += y;
  }
  if (lane == SRT_WAVE - 1) wsum[wv] = incl;
  __syncthreads();
  int before = 0;
  for (int j = 0; j < wv; ++j) before += wsum[j];
  if (tid < kPlanKeys) off[tid] = before + incl - mine;  // next free place of the class
  if (tid == 1023) {
    a.plan[0] = before + incl;  // all classes
    a.plan[1] = 0;
  }
  __syncthreads();
  // 1024 sequences at a time: a thread per sequence takes its places in the
  // class lists (and in the list of split sequences), then all threads, the
  // same number for each sequence, write the items.  (One thread per sequence
  // wrote them in up to 280 stores one after the other: 20 us for 256
  // sequences of up to 32k, 46 for 8 with 256-node trees; now 6 and 5.)  Where
  // none can have more than kFewItems the thread writes them at once, without
  // the exchange through LDS (512 sequences of one item: 19.1 us a call with it, 18.4
  // so; 256 of 4: 42.7 and 41.8).
  const bool few = a.total <= kFewItems * a.B;
  const int group = min(a.B, 1024);
  const int per_seq_log2 = group > 1 ? __clz(group - 1) - 22 : 10;  // 1024 / (group rounded up to a power of two)
  for (int b0 = 0; b0 < a.B; b0 += 1024) {
    if (a.B > 1024 && b0 + tid < a.B) si = seq_info(a, b0 + tid);
    int split_rows = 0;
    if (b0 + tid < a.B) {
      const int rows = si.n * a.G;
      s_total[tid] = si.total;
      s_rows[tid] = rows;
      classes(si.total, rows, [&](int c, int key, int ns) {
        const int rbs = row_blocks(rows);
        int at = atomicAdd(&off[key], ns * a.Hkv * rbs);
        if (!few) {
          s_pos[c][tid] = at;
          return;
        }
        const int s0 = c == 0 ? 0 : si.total >> cshift;
        for (int s = s0; s < s0 + ns; ++s)
          for (int g = 0; g < a.Hkv; ++g)
            for (int rb = 0; rb < rbs; ++rb, ++at)
              *reinterpret_cast<int2*>(a.plan + kPlanHeader + 2 * at) = make_int2(b0 + tid, g | (s << 8) | (rb << 20));
      });
      if (si.total > a.chunk) {
        *reinterpret_cast<int2*>(a.plan + a.combine_at + 2 * atomicAdd(&ncomb, 1)) =
            make_int2((b0 + tid) | ((si.total + a.chunk - 1) >> cshift) << 16, rows);
        split_rows = rows;
      }
    }
    if (a.S > 1) {  // (one atomic a wave: 64 on one word take 1.5 us)
#pragma unroll
      for (int d = SRT_WAVE / 2; d >= 1; d >>= 1) split_rows = max(split_rows, __shfl_xor(split_rows, d, SRT_WAVE));
      if (lane == 0 && split_rows > 0) atomicMax(&widest, split_rows);
    }
    if (few) continue;
    __syncthreads();
    const int i = tid >> per_seq_log2;
    if (b0 + i < a.B && i < group) {
      const int total = s_total[i], rbs = row_blocks(s_rows[i]), per = a.Hkv * rbs;
      const int full = total >> cshift, splits = (total + a.chunk - 1) >> cshift;
      for (int x = tid & ((1 << per_seq_log2) - 1); x < splits * per; x += 1 << per_seq_log2) {
        const int s = x / per, r = x - s * per, g = r / rbs;
        const int at = s < full ? s_pos[0][i] + x : s_pos[1][i] + x - full * per;
        *reinterpret_cast<int2*>(a.plan + kPlanHeader + 2 * at) = make_int2(b0 + i, g | (s << 8) | ((r - g * rbs) << 20));
      }
    }
    if (b0 + 1024 < a.B) __syncthreads();
  }
  if (few) __syncthreads();
  if (tid == 0) {
    a.plan[2] = ncomb;
    a.plan[3] = (widest + kCombineRows - 1) / kCombineRows;
  }
}

// Merges the split partials of sequences that needed more than one split:
// out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s with M = max_s m_s (m
// in log2 units).  Persistent workgroups stride over the 8-row groups of the
// plan's split sequences, one thread per row and four head dims, so partial
// reads are 16-byte coalesced.  The splits are folded with a running maximum,
// so the loads of different splits are independent.  A group is a chain of
// two round trips (entry, partials), so 16 workgroups per CU keep enough of
// them in flight: 26 -> 20 us for 256 sequences of up to 32k with trees of 1
// to 64 nodes, 44 -> 27 with full ones, 26 -> 20 for 8 of 16k-32k with
// 64-256 nodes (four workgroups per CU, and a list entry for every group).
// The groups of the widest split tree set the stride from one (sequence, KV head)
// to the next, one more where they are even, so that the first groups do not
// meet in every 2^n-th workgroup (512 one-node sequences of 8500 keys in a batch
// with room for 256 nodes: 1860 us a call with the stride of the room, 1610 so).
template <int D, bool kDirect>
__global__ __launch_bounds__(kCombineRows * D / 4) void tree_attn_combine_kernel(AttnBase a) {
  constexpr int Q = D / 4;
  const int per_head = kDirect ? (a.N * a.G + kCombineRows - 1) / kCombineRows : a.plan[3] | 1;
  const int n_units = (kDirect ? a.B : a.plan[2]) * a.Hkv * per_head;
  const int RBR = a.part_rows;
  const int q = threadIdx.x % Q;
  for (int u = blockIdx.x; u < n_units; u += gridDim.x) {
    const int e = u / (a.Hkv * per_head), rest = u - e * a.Hkv * per_head;
    const int g = rest / per_head;
    const int r = (rest - g * per_head) * kCombineRows + threadIdx.x / Q;
    int b = e, nsplit, rows;
    if constexpr (kDirect) {  // every sequence, whatever its splits
      const SeqInfo si = seq_info(a, b);
      nsplit = (si.total + a.chunk - 1) / a.chunk;
      rows = si.n * a.G;
    } else {
      const int2 entry = *reinterpret_cast<const int2*>(a.plan + a.combine_at + 2 * e);
      b = entry.x & 0xffff;
      nsplit = static_cast<int>(static_cast<uint32_t>(entry.x) >> 16);
      rows = entry.y;
    }
    if (nsplit < 2 || r >= rows) continue;
    const int64_t base = (static_cast<int64_t>(b) * a.Hkv + g) * a.S * RBR + r;
    float M = -INFINITY, den = 0.f;
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < nsplit; ++s) {
      const int64_t prow = base + static_cast<int64_t>(s) * RBR;
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * prow);
      const f32x4 os = *reinterpret_cast<const f32x4*>(a.part_o + prow * D + 4 * q);
      if (ml.x == -INFINITY) continue;
      const float mn = fmaxf(M, ml.x);
      const float c_old = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - mn);
      const float c_new = __builtin_amdgcn_exp2f(ml.x - mn);
      den = den * c_old + ml.y * c_new;
      num = num * c_old + os * c_new;
      M = mn;
    }
    const float inv = den > 0.f ? 1.f / den : 0.f;
    const int node = r / a.G, h = g * a.G + r % a.G;
    uint16_t* op = a.out + ((static_cast<int64_t>(b) * a.N + node) * a.Hq + h) * D + 4 * q;
    const uint32_t x0 = to_bf16_bits(num[0] * inv) | (uint32_t(to_bf16_bits(num[1] * inv)) << 16);
    const uint32_t x1 = to_bf16_bits(num[2] * inv) | (uint32_t(to_bf16_bits(num[3] * inv)) << 16);
    *reinterpret_cast<uint2*>(op) = make_uint2(x0, x1);
  }
}

// Whether the 8-bit cache's kernel takes a batch with half the waves a workgroup, two
// workgroups to a CU: up to 32 rows (one wave's) always, up to kNarrowRows where there are
// many (sequence, KV head) pairs, as an item takes twice as long then.  28 heads, 4 KV
// heads unless said: 512 sequences of 1000 to 8000 keys, 16 nodes: 215 -> 182 us, 256 of
// 100 to 500: 58 -> 37, of 200 to 2000: 65 -> 69; 1024 of 500 to 4000, 12 heads, 2 KV
// heads: 151 -> 112; 64 of 4k to 16k: 101 -> 138, with 8 nodes 90 -> 101.  Up to 32 rows
// it loses only where a few long contexts of many decide (32 sequences, median 1000, up
// to 8000, 4 nodes: 32 -> 35; 256 of 2 KV heads of 64: 40 -> 47), which the host cannot see.
constexpr int kNarrowRows = 128;
inline bool half_waves(int64_t pairs, int64_t rows) {
  return rows > 0 && (rows <= 32 || (rows <= kNarrowRows && pairs >= 1024));
}

// Keys per split: the largest power of two in [kMinChunk, kChunk] that still
// gives B * Hkv * RB * (capacity / chunk) >= 512 work items (two per CU of
// the 256; RB row blocks per sequence and KV head), so that small batches
// of long contexts are split over enough workgroups; large batches and wide
// trees keep 8192-key splits (fewer partial results).  A batch that leaves CUs
// idle even so is a serial chain of up to 16 tiles (about 1.3 us each); as
// long as all of its items run at once it takes 256- or 512-key splits.  28
// heads, 4 KV heads, d 128, one sequence, 8-node trees, capacity 1024 / 2048 /
// 4096: 14 / 15 / 18 us against 20 / 25 / 27 with 1024-key splits; 16
// sequences, 64-node trees, 2048: 45.7 against 45.4 (no CU left).  Contexts of
// up to 768 keys (1024 with 512-key splits) gain little over the combine's cost
// (16 sequences of 32 heads, 8 KV heads, 64 nodes, capacity 768: 34 us with
// 512-key splits, 30 with one; 4 of 4 heads, d 64, 8 nodes: 13.7 and 13.1), and
// past 32 splits the combine's own chain is the longer one (one sequence, 16k
// keys: 39 us with 63 splits, 25 with 32 or 16).  The rule goes by the block
// table's width, as the host does not know the contexts: a batch in a table as
// wide as a 32k limit takes none of these (4 sequences of 700 keys, 8 nodes:
// 18 us in a table for 8192 keys, 26 before these rules; 1 of 300: 14 us in one for
// 32768, 17 before, as only the plan kernel goes).  small = false: without
// these, for a scratch that has no room for their partials.
// rows: query rows of the widest tree for the 8-bit cache's kernel, whose items take
// half the time and less where trees are narrow, so that a few long items decide more
// often when the call ends; 0 for the bf16 cache's.  Fewer than 512 (sequence, KV head)
// pairs with trees of up to two row blocks then take 4096-key splits where they would
// take 8192: 64 sequences of 4k to 16k, 28 heads, 4 KV heads, trees of up to 8 / 16 /
// 32 / 64 nodes: 114 -> 90, 227 -> 137, 242 -> 144, 248 -> 215 us; not from 512 pairs
// (128 such sequences: 355 and 386 us), nor for wider trees, whose partial results cost
// more (8 of 256 nodes: 530 and 558).  With half the waves a workgroup they always do, as two
// of their workgroups share a CU's rate (28 heads, 4 KV heads, single tokens or 4 nodes:
// 300 sequences of 300 to 32k keys 109 -> 85 us, 256 of 2k to 8k 116 -> 114; at most 3%
// the other way, 256 of 16k to 32k: 957 -> 988; with 2048 keys 93, 120 and 1061).
int chunk_for(int32_t B, int32_t Hkv, int64_t RB, int64_t cap, bool small, int64_t rows) {
  int chunk = half_waves(static_cast<int64_t>(B) * Hkv, rows) ? kChunk / 2 : kChunk;
  auto items = [&](int c) { return static_cast<int64_t>(B) * Hkv * RB * ((cap + c - 1) / c); };
  while (chunk > kMinChunk && items(chunk) < 512) chunk /= 2;
  if (rows > 0 && chunk == kChunk && RB <= 2 && static_cast<int64_t>(B) * Hkv < 512) chunk /= 2;
  if (small && chunk == kMinChunk)
    for (int c = kSmallChunk; c < kMinChunk; c *= 2)
      if (cap > c + 512 && cap <= kSmallSplits * c && items(c) <= kSmallItems) return c;
  return chunk;
}

int splits_for(int64_t cap, int chunk) { return static_cast<int>((cap + chunk - 1) / chunk); }

// 8-row groups of all sequences and KV heads, each word pair of which the
// scratch holds room for (the list of split sequences needs less).
int64_t max_combine_units(int32_t B, int32_t N, int32_t G, int32_t Hkv) {
  return static_cast<int64_t>(B) * Hkv * ((static_cast<int64_t>(N) * G + 7) / 8);
}

// Bytes of the work lists for at most `items` items and `units` combine
// units, rounded to 256.
size_t plan_bytes(int64_t items, int64_t units) {
  return ((kPlanHeader + 2 * items + 2 * units) * sizeof(int32_t) + 255) / 256 * 256;
}

// Rows of a (sequence, KV head, split) that the partial results hold room for: whole
// row blocks for the bf16 cache's kernel, the widest tree's rows for the 8-bit one's
// (single tokens of 256 sequences of up to 32k, 28 heads, 4 KV heads: 30 MB for 1.1 GB).
int64_t part_rows(int32_t N, int32_t G, bool quant) {
  const int64_t rows = static_cast<int64_t>(N) * G;
  return quant ? rows : (rows + kRowsPerBlock - 1) / kRowsPerBlock * kRowsPerBlock;
}

size_t scratch_for(int32_t B, int32_t N, int32_t Hq, int32_t Hkv, int32_t d, int64_t cap, int chunk, bool quant) {
  const int G = Hq / Hkv;
  const int64_t RB = (N * G + kRowsPerBlock - 1) / kRowsPerBlock;
  const int S = splits_for(cap, chunk);
  const size_t plan = plan_bytes(static_cast<int64_t>(B) * Hkv * S * RB, max_combine_units(B, N, G, Hkv));
  if (S <= 1) return plan;
  return plan + static_cast<size_t>(B) * Hkv * S * part_rows(N, G, quant) * (d + 2) * sizeof(float);
}

int cu_count() {
  static int cached[64] = {0};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 0;
  if (dev < 64 && cached[dev] > 0) return cached[dev];
  int n = 0;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) return 0;
  if (dev < 64) cached[dev] = n;
  return n;
}

void launch_combine(const AttnBase& a, int d, bool direct, unsigned grid, hipStream_t s) {
  if (d == 128) {
    if (direct) tree_attn_combine_kernel<128, true><<<grid, kCombineRows * 32, 0, s>>>(a);
    else tree_attn_combine_kernel<128, false><<<grid, kCombineRows * 32, 0, s>>>(a);
  } else {
    if (direct) tree_attn_combine_kernel<64, true><<<grid, kCombineRows * 16, 0, s>>>(a);
    else tree_attn_combine_kernel<64, false><<<grid, kCombineRows * 16, 0, s>>>(a);
  }
}

int64_t combine_grid(const AttnBase& a, int cus) {
  return std::min<int64_t>(max_combine_units(a.B, a.N, a.G, a.Hkv), 16 * cus);
}

// Checks a call's sizes and scratch and fills in everything of `a` that they
// decide (B, N, Hq, Hkv and cap are set; cap beyond int32 is refused here).
int lay_out(AttnBase& a, int64_t cap, int32_t d, void* scratch, size_t scratch_bytes, bool quant) {
  const int32_t G = a.Hq / a.Hkv;
  const int64_t RB = (a.N * G + kRowsPerBlock - 1) / kRowsPerBlock;
  int chunk = chunk_for(a.B, a.Hkv, RB, cap, true, quant ? a.N * G : 0);
  if (scratch_bytes < scratch_for(a.B, a.N, a.Hq, a.Hkv, d, cap, chunk, quant))
    chunk = chunk_for(a.B, a.Hkv, RB, cap, false, 0);
  if (!scratch || scratch_bytes < scratch_for(a.B, a.N, a.Hq, a.Hkv, d, cap, chunk, quant)) return SRT_ERR_CAPACITY;
  if (reinterpret_cast<uintptr_t>(scratch) % 256) return SRT_ERR_INVALID;
  a.G = G;
  a.cap = static_cast<int32_t>(cap);
  a.chunk = chunk;
  a.S = splits_for(cap, chunk);
  a.RB = static_cast<int32_t>(RB);
  a.part_rows = static_cast<int32_t>(part_rows(a.N, G, quant));
  const int64_t total = static_cast<int64_t>(a.B) * a.Hkv * a.S * a.RB;
  if (total > (int64_t(1) << 30)) return SRT_ERR_INVALID;
  a.total = static_cast<int32_t>(total);
  const size_t pbytes = plan_bytes(total, max_combine_units(a.B, a.N, G, a.Hkv));
  a.plan = static_cast<int32_t*>(scratch);
  a.combine_at = kPlanHeader + 2 * total;
  a.part_o = a.S > 1 ? reinterpret_cast<float*>(static_cast<uint8_t*>(scratch) + pbytes) : nullptr;
  a.part_ml =
      a.S > 1 ? a.part_o + static_cast<int64_t>(a.B) * a.Hkv * a.S * a.part_rows * d : nullptr;
  return SRT_OK;
}

// Work-list packing: sequence < 65536, KV head < 256, split < 4096, row block
// < 2048, combine units < 2^31.
bool packs(int32_t B, int32_t N, int32_t Hq, int32_t Hkv, int64_t cap, bool quant) {
  if (static_cast<int64_t>(N) * (Hq / Hkv) / kRowsPerBlock > 2046) return false;
  const int64_t RB = (N * (Hq / Hkv) + kRowsPerBlock - 1) / kRowsPerBlock;
  return B <= 65535 && Hkv <= 255 && splits_for(cap, chunk_for(B, Hkv, RB, cap, true, quant ? N * (Hq / Hkv) : 0)) <= 4095 &&
         max_combine_units(B, N, Hq / Hkv, Hkv) <= (int64_t(1) << 30);
}

}  // namespace
