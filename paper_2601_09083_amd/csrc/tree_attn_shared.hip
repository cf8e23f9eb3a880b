// Tree-masked attention for batches of which groups of sequences share the pages
// of a long prefix: its keys and values are read once for a group's rows.
//
// Method: Section 3 (one decode pass verifies every drafted token) for the group
// rollouts that the paper trains on -- several answers to one prompt, whose keys
// and values lie in the cache once.  The softmax over a sequence's keys is taken
// in parts, the shared prefix and its own keys, which their running maximum m and
// sum l join exactly: out = sum_p 2^(m_p - M) o_p / sum_p 2^(m_p - M) l_p.
//
// GPU design.  The tile kernel (attn_bf16.h) takes items of two kinds: the rows of
// one sequence against a split of its own keys, and the rows of a whole group,
// 256 at a time, against a split of the prefix, where no key is masked.  Read by
// every sequence, the prefixes of a batch of single tokens are most of its bytes.
// A plan kernel (one workgroup) finds the groups' members, the keys that they can
// share -- whole pages, no further than the shortest member's context -- and the
// items, longest first; the combine kernel of attn.h joins the parts.
#include "attn_bf16.h"

namespace {

constexpr int kMaxGroups = 4096;   // groups of a batch, whose counts are held in LDS
constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / SRT_WAVE;
constexpr int kGroupsEach = kMaxGroups / kPlanThreads;
constexpr int kSeqs = 16;          // sequences or groups that a wave of the plan kernel lists at a time

struct PlanArgs {
  const int32_t* group_ids;
  const int32_t* prefix_len;
  int32_t n_groups;
};

// One workgroup: groups, item classes (as tree_attn_plan_kernel), then the lists.
__global__ __launch_bounds__(kPlanThreads) void shared_plan_kernel(SharedArgs a, PlanArgs p) {
  __shared__ int32_t cnt[kPlanKeys], off[kPlanKeys];
  __shared__ int32_t members[kMaxGroups], nodes[kMaxGroups], keys[kMaxGroups], lead[kMaxGroups];
  __shared__ int32_t wsum[2][kPlanWaves];
  __shared__ int32_t ncomb, widest;
  const int tid = threadIdx.x, lane = tid % SRT_WAVE, wv = tid / SRT_WAVE;
  const int cshift = 31 - __clz(a.chunk);
  auto group_of = [&](int b) {
    const int g = p.n_groups > 0 ? p.group_ids[b] : -1;
    return g >= 0 && g < p.n_groups ? g : -1;
  };
  auto row_blocks = [&](int rows) { return (rows + kRowsPerBlock - 1) / kRowsPerBlock; };
  // Visits the item classes of `n` nodes against `total` keys: f(class, key, splits).
  auto classes = [&](int total, int n, auto&& f) {
    const int full = total >> cshift, tail = total - (full << cshift);
    const int waves = min(kWaves, (n * a.G + kRowsPerWave - 1) / kRowsPerWave);
    if (full > 0) f(0, plan_key(a.chunk / kTile, waves), full);
    if (tail > 0) f(1, plan_key((tail + kTile - 1) / kTile, waves), 1);
  };
  auto count = [&](int total, int n) {
    const int per = a.Hkv * row_blocks(n * a.G);
    classes(total, n, [&](int, int key, int ns) { atomicAdd(&cnt[key], ns * per); });
  };

  for (int k = tid; k < kPlanKeys; k += kPlanThreads) cnt[k] = 0;
  for (int g = tid; g < p.n_groups; g += kPlanThreads) {
    members[g] = nodes[g] = 0;
    keys[g] = lead[g] = 0x7fffffff;
  }
  if (tid == 0) ncomb = widest = 0;
  __syncthreads();
  for (int b = tid; b < a.B; b += kPlanThreads) {
    const int g = group_of(b);
    if (g < 0) continue;
    const SeqInfo si = seq_info(a, b);
    atomicAdd(&members[g], 1);
    atomicAdd(&nodes[g], si.n);
    atomicMin(&keys[g], si.L);
    atomicMin(&lead[g], b);
  }
  __syncthreads();
  // Keys that each group shares, and where its nodes' list starts.
  int mine[kGroupsEach], sum = 0;
#pragma unroll
  for (int j = 0; j < kGroupsEach; ++j) {
    const int g = tid * kGroupsEach + j;
    mine[j] = 0;
    if (g >= p.n_groups) continue;
    int P = min(p.prefix_len[g], keys[g]);
    P = members[g] > 1 && P > 0 ? P & ~(a.page - 1) : 0;
    keys[g] = P;
    if (P > 0) mine[j] = nodes[g];
    sum += mine[j];
    if (P > 0) count(P, nodes[g]);
  }
  auto scan = [&](int x, int32_t* ws) {  // exclusive prefix sum over the workgroup
    int incl = x;
#pragma unroll
    for (int d = 1; d < SRT_WAVE; d <<= 1) {
      const int y = __shfl_up(incl, d, SRT_WAVE);
      if (lane >= d) incl += y;
    }
    if (lane == SRT_WAVE - 1) ws[wv] = incl;
    __syncthreads();
    int before = 0;
    for (int j = 0; j < wv; ++j) before += ws[j];
    return before + incl - x;
  };
  int at = scan(sum, wsum[0]);
#pragma unroll
  for (int j = 0; j < kGroupsEach; ++j) {
    const int g = tid * kGroupsEach + j;
    if (g >= p.n_groups) continue;
    a.group[g] = make_int4(lead[g], keys[g], at, mine[j]);
    members[g] = at;  // from here on: the next free entry of the group's list
    at += mine[j];
  }
  // Own keys of the sequences.  (The barrier of the scan ordered keys[].)
  for (int b = tid; b < a.B; b += kPlanThreads) {
    const SeqInfo si = seq_info(a, b);
    const int g = group_of(b);
    count(si.total - (g >= 0 ? keys[g] : 0), si.n);
  }
  __syncthreads();
  static_assert(kPlanKeys <= kPlanThreads, "one class per thread");
  const int n = tid < kPlanKeys ? cnt[tid] : 0;
  const int before = scan(n, wsum[1]);
  if (tid < kPlanKeys) off[tid] = before;
  if (tid == kPlanThreads - 1) {
    a.plan[0] = before + n;  // all classes
    a.plan[1] = 0;
  }
  __syncthreads();
  // The lists: a wave takes kSeqs groups, then sequences, at a time; a lane each
  // reserves its places, and all lanes write the items.
  int wide = 0;
  const int group_steps = (p.n_groups + kSeqs - 1) / kSeqs, seq_steps = (a.B + kSeqs - 1) / kSeqs;
  for (int step = wv; step < group_steps + seq_steps; step += kPlanWaves) {
    const bool prefix = step < group_steps;
    const int x = (prefix ? step : step - group_steps) * kSeqs + lane;
    int total = 0, n = 0, listed = -1, pos[2] = {0, 0};
    if (lane < kSeqs && x < (prefix ? p.n_groups : a.B)) {
      if (prefix) {
        total = keys[x];
        n = total > 0 ? nodes[x] : 0;
      } else {
        const SeqInfo si = seq_info(a, x);
        const int g = group_of(x), P = g >= 0 ? keys[g] : 0;
        total = si.total - P;
        n = si.n;
        a.seq_prefix[x] = P;
        const int parts = ((P + a.chunk - 1) >> cshift) + ((total + a.chunk - 1) >> cshift);
        if (P > 0) listed = atomicAdd(&members[g], n);
        if (parts > 1) {
          *reinterpret_cast<int2*>(a.plan + a.combine_at + 2 * atomicAdd(&ncomb, 1)) = make_int2(x | parts << 16, n * a.G);
          wide = max(wide, n * a.G);
        }
      }
      const int per = a.Hkv * row_blocks(n * a.G);
      classes(total, n, [&](int c, int key, int ns) { pos[c] = atomicAdd(&off[key], ns * per); });
    }
    for (int i = 0; i < kSeqs; ++i) {
      const int n_i = __builtin_amdgcn_readlane(n, i);
      if (n_i == 0) continue;
      const int total_i = __builtin_amdgcn_readlane(total, i), id = __builtin_amdgcn_readlane(x, i);
      const int p0 = __builtin_amdgcn_readlane(pos[0], i), p1 = __builtin_amdgcn_readlane(pos[1], i);
      const int list = __builtin_amdgcn_readlane(listed, i);
      const int rbs = row_blocks(n_i * a.G), per = a.Hkv * rbs, full = total_i >> cshift;
      const int splits = (total_i + a.chunk - 1) >> cshift;
      for (int y = lane; y < splits * per; y += SRT_WAVE) {
        const int s = y / per, r = y - s * per, g = r / rbs, rb = r - g * rbs;
        const int to = s < full ? p0 + y : p1 + y - full * per;
        *reinterpret_cast<int2*>(a.plan + kPlanHeader + 2 * to) =
            make_int2(static_cast<int>(static_cast<uint32_t>(id | rb << 16) | (prefix ? kPrefixItem : 0u)), g | s << 8);
      }
      if (list >= 0)
        for (int y = lane; y < n_i; y += SRT_WAVE) a.node_of[list + y] = id << 8 | y;
    }
  }
#pragma unroll
  for (int d = SRT_WAVE / 2; d >= 1; d >>= 1) wide = max(wide, __shfl_xor(wide, d, SRT_WAVE));
  if (lane == 0 && wide > 0) atomicMax(&widest, wide);
  __syncthreads();
  if (tid == 0) {
    a.plan[2] = ncomb;
    a.plan[3] = (widest + kCombineRows - 1) / kCombineRows;
  }
}

// What the sizes alone decide.
struct Sizes {
  int64_t rb, items, units, rows;
  int chunk, slots;      // keys per split; partial results of a row, at most
  size_t plan, groups, prefixes, nodes, part_rows, total;  // bytes
};

size_t round256(size_t x) { return (x + 255) / 256 * 256; }

Sizes sizes_for(int32_t B, int32_t N, int32_t Hq, int32_t Hkv, int32_t d, int64_t cap, int32_t n_groups) {
  Sizes z;
  const int32_t G = Hq / Hkv;
  z.rb = (static_cast<int64_t>(N) * G + kRowsPerBlock - 1) / kRowsPerBlock;
  z.chunk = chunk_for(B, Hkv, z.rb, cap, false, 0);
  // a prefix and a rest, each in splits of its own, take at most one part more than all keys together
  z.slots = splits_for(cap, z.chunk) + 1;
  z.items = static_cast<int64_t>(B) * Hkv * z.slots * z.rb;  // (a group's row blocks are no more than its members')
  z.units = max_combine_units(B, N, G, Hkv);
  z.rows = static_cast<int64_t>(B) * Hkv * z.slots * N * G;
  z.plan = plan_bytes(z.items, z.units);
  z.groups = round256(static_cast<size_t>(n_groups) * sizeof(int4));
  z.prefixes = round256(static_cast<size_t>(B) * sizeof(int32_t));
  z.nodes = round256(static_cast<size_t>(B) * N * sizeof(int32_t));
  z.total = z.plan + z.groups + z.prefixes + z.nodes + static_cast<size_t>(z.rows) * (d + 2) * sizeof(float);
  return z;
}

// Work-list packing: 16 bits of a sequence or group, 15 of a row block, 8 of a KV head, 24 of a split.
bool fits(int32_t B, int32_t N, int32_t Hq, int32_t Hkv, int64_t cap, int32_t n_groups) {
  if (B > 65535 || n_groups > kMaxGroups || Hkv > 255 || cap > (int64_t(1) << 30)) return false;
  const int64_t rows = static_cast<int64_t>(B) * N * (Hq / Hkv);
  if (rows / kRowsPerBlock > 32766) return false;
  const Sizes z = sizes_for(B, N, Hq, Hkv, 128, cap, n_groups);
  // (split counts of the combine's entries are 16 bits, and the tile kernel's offsets 31)
  return z.slots <= 32767 && z.items <= (int64_t(1) << 29) && z.units <= (int64_t(1) << 30);
}

int check_sizes(int32_t B, int32_t N, int32_t Hq, int32_t Hkv, int32_t d, int32_t page, int32_t max_pages,
                int32_t n_groups) {
  if (B < 0 || N < 1 || N > kMaxN || Hq < 1 || Hkv < 1 || Hq % Hkv || page < 1 || max_pages < 1 || n_groups < 0)
    return SRT_ERR_INVALID;
  if (d != 64 && d != 128) return SRT_ERR_UNSUPPORTED;
  if (page < 16 || (page & (page - 1))) return SRT_ERR_UNSUPPORTED;
  return fits(B, N, Hq, Hkv, static_cast<int64_t>(page) * max_pages, n_groups) ? SRT_OK : SRT_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" size_t srt_tree_attn_shared_scratch_bytes(int32_t B, int32_t N, int32_t Hq, int32_t Hkv, int32_t d,
                                                     int32_t page, int32_t max_pages, int32_t n_groups) {
  if (check_sizes(B, N, Hq, Hkv, d, page, max_pages, n_groups) != SRT_OK) return 0;
  return sizes_for(B, N, Hq, Hkv, d, static_cast<int64_t>(page) * max_pages, n_groups).total;
}

extern "C" int srt_tree_attn_shared(int32_t B, int32_t N, int32_t Hq, int32_t Hkv, int32_t d, int32_t page,
                                    int32_t max_pages, int64_t num_pages, int32_t n_groups, const uint16_t* q,
                                    const uint16_t* k_cache, const uint16_t* v_cache, const int32_t* block_table,
                                    const int32_t* ctx_len, const int32_t* tree_parent, const int32_t* n_nodes,
                                    const int32_t* group_ids, const int32_t* prefix_len, float scale, uint16_t* out,
                                    void* scratch, size_t scratch_bytes, void* stream) {
  const int st = check_sizes(B, N, Hq, Hkv, d, page, max_pages, n_groups);
  if (st == SRT_ERR_INVALID || num_pages < 1 || !std::isfinite(scale)) return SRT_ERR_INVALID;
  if (st != SRT_OK || B == 0) return st;
  if (!q || !k_cache || !v_cache || !block_table || !ctx_len || !tree_parent || !n_nodes || !out ||
      (n_groups > 0 && (!group_ids || !prefix_len)))
    return SRT_ERR_INVALID;
  const int64_t cap = static_cast<int64_t>(page) * max_pages;
  const Sizes z = sizes_for(B, N, Hq, Hkv, d, cap, n_groups);
  if (!scratch || scratch_bytes < z.total) return SRT_ERR_CAPACITY;
  if (reinterpret_cast<uintptr_t>(scratch) % 256) return SRT_ERR_INVALID;

  SharedArgs a;
  a.q = q;
  a.k = k_cache;
  a.v = v_cache;
  a.bt = block_table;
  a.ctx_len = ctx_len;
  a.parent = tree_parent;
  a.n_nodes = n_nodes;
  a.out = out;
  a.B = B;
  a.N = N;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  a.page = page;
  a.page_shift = __builtin_ctz(static_cast<unsigned>(page));
  a.max_pages = max_pages;
  a.num_pages = num_pages;
  a.scale_log2 = static_cast<float>(static_cast<double>(scale) * 1.4426950408889634);
  a.cap = static_cast<int32_t>(cap);
  a.tree_room = 0;
  a.chunk = z.chunk;
  a.S = z.slots;
  a.RB = static_cast<int32_t>(z.rb);
  a.total = static_cast<int32_t>(z.items);
  a.part_rows = N * a.G;
  uint8_t* base = static_cast<uint8_t*>(scratch);
  a.plan = reinterpret_cast<int32_t*>(base);
  a.combine_at = kPlanHeader + 2 * z.items;
  a.group = reinterpret_cast<int4*>(base + z.plan);
  a.seq_prefix = reinterpret_cast<int32_t*>(base + z.plan + z.groups);
  a.node_of = reinterpret_cast<int32_t*>(base + z.plan + z.groups + z.prefixes);
  a.part_o = reinterpret_cast<float*>(base + z.plan + z.groups + z.prefixes + z.nodes);
  a.part_ml = a.part_o + z.rows * d;

  const int cus = cu_count();
  if (cus <= 0) return SRT_ERR_HIP;
  const unsigned grid = static_cast<unsigned>(std::min<int64_t>(z.items, cus));
  hipStream_t s = as_stream(stream);
  shared_plan_kernel<<<1, kPlanThreads, 0, s>>>(a, PlanArgs{group_ids, prefix_len, n_groups});
  if (d == 128) tree_attn_kernel<128, false, SharedArgs><<<grid, kThreads, 0, s>>>(a);
  else tree_attn_kernel<64, false, SharedArgs><<<grid, kThreads, 0, s>>>(a);
  launch_combine(a, d, false, static_cast<unsigned>(combine_grid(a, cus)), s);
  return launch_status();
}
