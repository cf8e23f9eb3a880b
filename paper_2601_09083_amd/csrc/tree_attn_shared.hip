// Tree-masked attention for batches of which groups of sequences share the pages
// of a long prefix: its keys and values are read once for a group's rows.
//
// Method: Section 3 (one decode pass verifies every drafted token) for the group
// rollouts that the paper trains on -- several answers to one prompt, whose keys
// and values lie in the cache once.  The softmax over a sequence's keys is taken
// in parts, the shared prefix and its own keys, which their running maximum m and
// sum l join exactly: out = sum_p 2^(m_p - M) o_p / sum_p 2^(m_p - M) l_p.
//
// GPU design.  The tile kernel is that of tree_attn.hip, whose comments describe it;
// its items are of two kinds: the rows of one sequence against a split of its own
// keys, and the rows of a whole group, 256 at a time, against a split of the prefix,
// where no key is masked.  Single tokens are bound by the bytes of the keys that are
// left to read: 32 prompts of 2k to 8k, eight answers each, 28 + 4 heads of 128 take
// 177 us a pass, 822 MB at 4.6 TB/s (5.0 in the tile kernel's 163 us), where
// srt_tree_attn reads every prefix eight times and takes 314.  Trees are bound by the
// tile kernel's rate: 64 trees of 8 nodes over one prompt of 32k 158 to 160 us, 126 GFLOP at
// 0.8 PFLOP/s (srt_tree_attn, whose 256-row tiles are a quarter full, 608); 128 of 1 to
// 64 nodes, 12 + 2 heads, 129 to 132 us (153), 28 of them the plan and the parts' join.
// A plan kernel (one workgroup) finds the groups' members, the keys that they can
// share -- whole pages, no further than the shortest member's context -- and the
// items, longest first; the combine kernel of attn.h joins the parts.
#include "attn.h"

namespace {

struct SharedArgs : AttnBase {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* bt;
  const int32_t* parent;
  int32_t page, page_shift, max_pages;
  int64_t num_pages;
  float scale_log2;
  // what the plan kernel works out
  int4* group;           // [n_groups] first sequence, shared keys, first entry of its nodes, nodes
  int32_t* seq_prefix;   // [B] keys that the sequence's group takes for it
  int32_t* node_of;      // live nodes of the sharing sequences, group by group: sequence << 8 | node
};
constexpr int kPlanChunk = 4;  // word of the plan: keys per split
constexpr uint32_t kPrefixItem = 1u << 31;  // of an item's first word: sequence or group | row block << 16

// Buffer descriptor over `nbytes` bytes at `base` (loads past nbytes read 0).
__device__ inline __amdgpu_buffer_rsrc_t make_rsrc(const uint16_t* base, int nbytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(base), 0, nbytes, 0x00020000);
}

// kLoads 16-byte loads through one descriptor: lane byte offset voff plus
// j * step for load j.
template <int kLoads, int kStep, int kAux>
__device__ inline void buffer_load16(const uint16_t* base, int nbytes, int voff, uint4 (&r)[kLoads]) {
  const __amdgpu_buffer_rsrc_t rsrc = make_rsrc(base, nbytes);
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    const i32x4 x = __builtin_amdgcn_raw_buffer_load_b128(rsrc, voff + j * kStep, 0, kAux);
    r[j] = __builtin_bit_cast(uint4, x);
  }
}

template <int D>
__global__ __launch_bounds__(kThreads, 1) void shared_attn_kernel(SharedArgs a) {
  using Sh = Shape<D>;
  constexpr int CPR = Sh::CPR;
  __shared__ __attribute__((aligned(16))) uint8_t Ks[2 * Sh::KTILE];
  __shared__ __attribute__((aligned(16))) uint8_t Vs[2 * Sh::VTILE];
  __shared__ uint64_t anc[kMaxN][4];
  __shared__ int32_t spar[kMaxN];

  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid / SRT_WAVE);  // wave-uniform, in an SGPR
  const int lane = tid % SRT_WAVE;
  const int l32 = lane % 32;  // query row of this lane inside the wave's 32
  const int h = lane / 32;    // lane half
  const int chunk = a.plan[kPlanChunk];

  // `b`: a sequence, or a group whose rows take a split of their shared prefix.
  auto run_item = [&](const int b, const int g, const int s, const int rb, const bool prefix) {
  SeqInfo si;
  int4 group;
  int k0 = 0, part = s, nsplit, b_table = b;  // first key, partial result, partial results, block table's row
  if (prefix) {
    group = a.group[b];
    si = {group.w, group.y, group.y};  // (no key of theirs is masked)
    nsplit = 2;
    b_table = group.x;
  } else {
    si = seq_info(a, b);
    k0 = a.seq_prefix[b];
    part += (k0 + chunk - 1) / chunk;
    nsplit = part - s + (si.total - k0 + chunk - 1) / chunk;
  }
  const int rows = si.n * a.G;
  if (rb * kRowsPerBlock >= rows) return;
  // No other item reads these keys: they are loaded past the caches (single tokens as
  // above 187 us without, 177 so; where trees read most keys often no difference).
  const bool once = rows <= kRowsPerBlock;
  const int k_begin = k0 + s * chunk;
  if (k_begin >= si.total) return;
  const int k_end = min(k_begin + chunk, si.total);
  const int ntiles = (k_end - k_begin + kTile - 1) / kTile;
  const int row0 = rb * kRowsPerBlock + w * kRowsPerWave;
  const bool wave_active = row0 < rows;  // wave-uniform

  // Ancestor-or-self bitsets, needed only when this split reaches the tree.
  if (k_end > si.L) {
    for (int i = tid; i < si.n; i += kThreads) spar[i] = a.parent[static_cast<int64_t>(b) * a.N + i];
    __syncthreads();
    for (int i = tid; i < si.n; i += kThreads) {
      uint64_t bits[4] = {0, 0, 0, 0};
      int j = i;
      while (j >= 0) {
        bits[j >> 6] |= 1ull << (j & 63);
        const int pj = spar[j];
        if (pj >= j) break;  // malformed parent: stop (parents precede children)
        j = pj;
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) anc[i][x] = bits[x];
    }
  }

  // Query fragment: B operand of S^T = K Q^T; lane holds row l32 and head
  // dims 16 ks + 8 h .. +7 for k-step ks.
  const int row = row0 + l32;
  const bool row_ok = row < rows;
  int node = row_ok ? row / a.G : 0, b_row = b;  // of the sequence's tree, and the sequence
  if (prefix) {
    const int e = a.node_of[group.z + node];
    node = e & 255;
    b_row = e >> 8;
  }
  bf16x8 qf[Sh::KS];
  {
    const int hq = g * a.G + (row_ok ? row % a.G : 0);
    const bf16x8* qp =
        reinterpret_cast<const bf16x8*>(a.q + ((static_cast<int64_t>(b_row) * a.N + node) * a.Hq + hq) * D + 8 * h);
#pragma unroll
    for (int ks = 0; ks < Sh::KS; ++ks) qf[ks] = row_ok ? qp[2 * ks] : bf16x8{};
    // Q is used exactly as given: the scale is applied to the fp32 scores
    // (rounding a scaled Q back to bf16 would perturb every score by up to
    // 2^-9 of its magnitude).
  }
  const float c_log2 = a.scale_log2;  // scale * log2(e)

  f32x16 o[Sh::DB];
#pragma unroll
  for (int db = 0; db < Sh::DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[db][r] = 0.f;
  // Reference maximum (log2 units) and lane-partial sum of the row.  The
  // reference is raised only when the row maximum exceeds it by more than
  // kLazy, so most tiles need no rescale of O.
  constexpr float kLazy = 8.f;
  float m = -INFINITY;
  float l = 0.f;

  // ---- staging ----------------------------------------------------------
  // Wave w moves keys 8w .. 8w+7 of every K and V tile; they lie inside one
  // page (pages are powers of two >= 16), so one scalar buffer descriptor
  // covers exactly the valid keys and keys past the split end or on an
  // invalid page read as zero.  Loads go to registers one tile ahead and are
  // stored to LDS after the tile's compute.
  const int pshift = a.page_shift;
  const int pmask = (1 << pshift) - 1;
  const int64_t bt_row = static_cast<int64_t>(b_table) * a.max_pages;
  const int64_t head_stride = static_cast<int64_t>(a.page) * D;  // elements per (page, head)
  constexpr int kRowsPerLoad = SRT_WAVE / CPR;                    // 4 (d=128) or 8 (d=64)
  constexpr int kLoadsPerWave = kSubRows / kRowsPerLoad;          // per tile, per tensor
  static_assert(kLoadsPerWave >= 1 && kSubRows % kRowsPerLoad == 0, "staging shape");
  const int st_row = kSubRows * w + lane / CPR;  // tile row of this lane's first chunk
  const int gl_off = ((lane / CPR) * D + (lane % CPR) * 8) * 2;
  const int k_st = st_row * Sh::KSTRIDE + (lane % CPR) * 16;
  const int v_st = st_row * Sh::VSTRIDE + (lane % CPR) * 16;

  // Page ids of this wave's sub-block of every tile of the split, one tile
  // per lane and register (a split has 128 tiles), fetched once; the loop
  // reads them with v_readlane and touches no block-table memory.
  static_assert(kChunk / kTile == 2 * SRT_WAVE, "two registers of page ids per split (of at most kChunk keys)");
  int pg_lane[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int p0 = k_begin + kTile * (SRT_WAVE * j + lane) + kSubRows * w;
    pg_lane[j] = p0 < k_end ? a.bt[bt_row + (p0 >> pshift)] : -1;
  }
  auto page_of = [&](int it) {
    if (it >= ntiles) return -1;
    return it < SRT_WAVE ? __builtin_amdgcn_readlane(pg_lane[0], it)
                         : __builtin_amdgcn_readlane(pg_lane[1], it - SRT_WAVE);
  };
  uint4 kreg[kLoadsPerWave], vreg[kLoadsPerWave];
  auto load_sub = [&](const uint16_t* base, int t0, int pg, uint4 (&r)[kLoadsPerWave]) {
    const int p0 = t0 + kSubRows * w;
    const bool ok = pg >= 0 && pg < a.num_pages && p0 < k_end;
    const int nbytes = ok ? min(kSubRows, k_end - p0) * D * 2 : 0;
    const int64_t off = ok ? (static_cast<int64_t>(pg) * a.Hkv + g) * head_stride + (p0 & pmask) * D : 0;
    if (once) buffer_load16<kLoadsPerWave, kRowsPerLoad * D * 2, 2>(base + off, nbytes, gl_off, r);
    else buffer_load16<kLoadsPerWave, kRowsPerLoad * D * 2, 0>(base + off, nbytes, gl_off, r);
  };
  auto store_k = [&](uint8_t* Kb) {
#pragma unroll
    for (int j = 0; j < kLoadsPerWave; ++j) *reinterpret_cast<uint4*>(Kb + k_st + j * kRowsPerLoad * Sh::KSTRIDE) = kreg[j];
  };
  auto store_v = [&](uint8_t* Vb) {
#pragma unroll
    for (int j = 0; j < kLoadsPerWave; ++j) *reinterpret_cast<uint4*>(Vb + v_st + j * kRowsPerLoad * Sh::VSTRIDE) = vreg[j];
  };

  // ---- MFMA phases -------------------------------------------------------
  // K operand (A of S^T): lane reads key l32 (+32 kb), head dims
  // 16 ks + 8 h .. +7.
  const int k_rd = l32 * Sh::KSTRIDE + 16 * h;
  // V^T operand (A of O^T) by transposing reads: in each 16-lane group G,
  // lane x addresses key 16 ks + 4 h + x/4 (+8 for the second half of the
  // contraction) and head dims (D/2)(G%2) + 16 db + 4 (x%4) .. +3.
  const int xg = lane % 16;
  const int k_vd = (4 * h + xg / 4) * Sh::VSTRIDE + ((CPR / 2) * ((lane / 16) & 1) + (xg % 4) / 2) * 16 + 8 * (xg & 1);

  // S^T[key][row] = q . k of one tile (raw fp32 dot products): two 32-key
  // blocks.
  auto qk = [&](const uint8_t* Kb, f32x16 (&sacc)[2]) {
    // All fragment reads are issued before the first MFMA so that one LDS
    // latency, not one per k-step, is exposed.
    bf16x8 kf[Sh::KS][2];
#pragma unroll
    for (int ks = 0; ks < Sh::KS; ++ks)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        kf[ks][kb] = *reinterpret_cast<const bf16x8*>(Kb + k_rd + kb * 32 * Sh::KSTRIDE + ks * 32);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[kb][r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < Sh::KS; ++ks)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        sacc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks][kb], qf[ks], sacc[kb], 0, 0, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 2 * Sh::KS, 0);  // DS reads
    __builtin_amdgcn_sched_group_barrier(0x008, 2 * Sh::KS, 0);  // then MFMAs
  };

  // Mask, online softmax with lazy rescale; returns P in bf16.  Lane holds
  // keys 32 kb + 8 (r/4) + 4 h + r%4 of its row in sacc[kb][r].
  auto softmax = [&](int t0, f32x16 (&sacc)[2], bf16x8 (&pb)[4], float mref0) {
    // Scores in log2 units relative to the reference: q.k * scale * log2(e)
    // - mref0, one fp32 fused multiply-add per score (masked scores are set
    // to -inf afterwards, so any finite scale is safe).
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[kb][r] = __builtin_fmaf(sacc[kb][r], c_log2, -mref0);
    const bool need_mask = (t0 + kTile > si.L) || (t0 + kTile > k_end);
    if (need_mask) {
      // Visibility of keys t0 .. t0+63 for this lane's row as one 64-bit
      // window: bit x is set iff key t0 + x < k_end and it is a context key
      // or the tree position of an ancestor-or-self of the row's node.  (If
      // the split ends before the tree, bits of tree positions are cleared
      // by the k_end limit, so stale bitsets are never used.)
      const int lim = k_end - t0;
      uint64_t vis = lim >= 64 ? ~0ull : (lim <= 0 ? 0ull : (~0ull >> (64 - lim)));
      const int j0 = t0 - si.L;  // tree index of key t0
      if (j0 > -kTile) {
        uint64_t win;
        if (j0 >= 0) {
          const int wd = j0 >> 6, sh = j0 & 63;
          const uint64_t lo = wd < 4 ? anc[node][wd] : 0ull;
          const uint64_t hi = wd + 1 < 4 ? anc[node][wd + 1] : 0ull;
          win = sh ? (lo >> sh) | (hi << (64 - sh)) : lo;
        } else {
          const int sh = -j0;  // 1..63 context keys lead the window
          win = (anc[node][0] << sh) | (~0ull >> (64 - sh));
        }
        vis &= win;
      }
      // lane half h holds keys 32 kb + 8 (r/4) + 4 h + r%4
      const uint64_t vh = vis >> (4 * h);
      const uint32_t v0 = static_cast<uint32_t>(vh), v1 = static_cast<uint32_t>(vh >> 32);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const uint32_t vw = kb ? v1 : v0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int x = 8 * (r / 4) + r % 4;
          sacc[kb][r] = ((vw >> x) & 1u) ? sacc[kb][r] : -INFINITY;
        }
      }
    }
    // Probabilities exp2(score - mref0 - dm), rounded to bf16 for the second
    // product, as srt_tree_attn's (an fp32 product has a sixteenth of the matrix rate; the
    // sum l takes the rounded ones, so that they still add up to 1, and an output moves by
    // at most 2^-8 of itself and as much of the mean of |v|); sacc holds score - mref0.  Returns this lane's sum of them
    // (its 32 keys of the row, two bf16 pairs per dot2, two accumulators).
    // Contraction index 8 h + e of k-step ks <-> key 16 ks + 8 (e/4) + 4 h + e%4.
    auto probs = [&](auto dm_c, float dm) {
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      const bf16x2 one2 = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
      float ps[2] = {0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          pb[ks][e] = static_cast<__bf16>(__builtin_amdgcn_exp2f(
              decltype(dm_c)::value ? sacc[ks / 2][8 * (ks % 2) + e] - dm : sacc[ks / 2][8 * (ks % 2) + e]));
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const bf16x2 pr = {pb[ks][e], pb[ks][e + 1]};
          ps[ks & 1] = __builtin_amdgcn_fdot2_f32_bf16(pr, one2, ps[ks & 1], false);
        }
      }
      return ps[0] + ps[1];
    };
    // Fast path: exponentiate against the current reference without first
    // taking the row maximum.  If every rounded probability of the row is
    // below 2^kLazy (their sum is), no score exceeds the reference by kLazy,
    // so the reference would not be raised and these are the final values.
    // Otherwise (or while the reference is still -inf) the wave takes the
    // row maximum, raises the reference as needed and exponentiates again.
    float psum = probs(std::false_type(), 0.f);
    const bool fast = m != -INFINITY && psum < 256.f;  // 256 = 2^kLazy
    if (__ballot(!fast)) {
      // (maximum, not fmaxf: no NaN-quieting of every operand; scores are
      // finite or -inf)
      float mloc = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; r += 2)
          mloc = __builtin_elementwise_maximum(mloc, __builtin_elementwise_maximum(sacc[kb][r], sacc[kb][r + 1]));
      mloc = max_halves(mloc);
      const float ms = mloc + mref0;  // row max in log2 units
      const bool raise = ms > m + kLazy;
      if (__ballot(raise)) {
        const float mnew = raise ? ms : m;
        const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mnew);
        l *= alpha;
#pragma unroll
        for (int db = 0; db < Sh::DB; ++db) o[db] *= alpha;
        m = mnew;
      }
      psum = probs(std::true_type(), (m == -INFINITY ? 0.f : m) - mref0);
    }
    l += psum;
  };

  // O^T[d][row] += V^T P^T.
  // V^T fragments of k-steps ks0, ks0+1 (two transposing reads per MFMA).
  typedef short i16x4v __attribute__((ext_vector_type(4)));
  auto v_read = [&](const uint8_t* Vb, int ks0, i16x4v (&vf)[2][Sh::DB][2]) {
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
      for (int db = 0; db < Sh::DB; ++db)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
          vf[k2][db][hh] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) i16x4v*)(Vb + k_vd + (ks0 + k2) * 16 * Sh::VSTRIDE +
                                                          hh * 8 * Sh::VSTRIDE + db * 32));
  };
  auto pv = [&](const i16x4v (&vf)[2][Sh::DB][2], int ks0, const bf16x8 (&pb)[4]) {
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
      for (int db = 0; db < Sh::DB; ++db) {
        const bf16x8 va =
            __builtin_bit_cast(bf16x8, __builtin_shufflevector(vf[k2][db][0], vf[k2][db][1], 0, 1, 2, 3, 4, 5, 6, 7));
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pb[ks0 + k2], o[db], 0, 0, 0);
      }
  };

  // ---- tile loop ---------------------------------------------------------
  // Iteration t: global loads of tile t+1 are issued to registers; the K
  // fragments of tile t are read from LDS and S = K Q^T runs; the V^T
  // fragments are read while softmax runs on the VALU; O += V^T P^T; then
  // tile t+1 is stored into the buffers tile t-1 left.  One barrier per tile.
  {
    const int pg0 = page_of(0);
    load_sub(a.k, k_begin, pg0, kreg);
    load_sub(a.v, k_begin, pg0, vreg);
    store_k(Ks);
    store_v(Vs);
  }
  __syncthreads();

  auto step = [&](int it, auto cur_c) {
    constexpr int cur = decltype(cur_c)::value;
    const int t0 = k_begin + it * kTile;
    const bool next = it + 1 < ntiles;
    if (next) {
      const int pg = page_of(it + 1);
      load_sub(a.k, t0 + kTile, pg, kreg);
      load_sub(a.v, t0 + kTile, pg, vreg);
    }
    if (wave_active) {
      f32x16 sacc[2];
      const float mref0 = m == -INFINITY ? 0.f : m;
      qk(Ks + cur * Sh::KTILE, sacc);
      // First half of the V^T fragments is read while softmax runs, the
      // second half while the first half's MFMAs run.
      i16x4v vf0[2][Sh::DB][2], vf1[2][Sh::DB][2];
      v_read(Vs + cur * Sh::VTILE, 0, vf0);
      bf16x8 pb[4];
      softmax(t0, sacc, pb, mref0);
      v_read(Vs + cur * Sh::VTILE, 2, vf1);
      pv(vf0, 0, pb);
      pv(vf1, 2, pb);
    }
    if (next) {
      store_k(Ks + (cur ^ 1) * Sh::KTILE);
      store_v(Vs + (cur ^ 1) * Sh::VTILE);
    }
    __syncthreads();
  };
  for (int it = 0; it < ntiles; it += 2) {
    step(it, std::integral_constant<int, 0>());
    if (it + 1 < ntiles) step(it + 1, std::integral_constant<int, 1>());
  }

  // Epilogue: lane holds row l32 and, for block db and quad q = r/4, head
  // dims (D/2)(q/2) + 16 db + 8 (q%2) + 4 h + 0..3.
  const float lt = sum_halves(l);
  if (!row_ok) return;
  const int RBR = a.part_rows;
  if (nsplit == 1) {
    const int hq = g * a.G + row % a.G;
    uint16_t* op = a.out + ((static_cast<int64_t>(b_row) * a.N + node) * a.Hq + hq) * D + 4 * h;
    const float inv = lt > 0.f ? 1.f / lt : 0.f;
#pragma unroll
    for (int db = 0; db < Sh::DB; ++db) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int d0 = (D / 2) * (q / 2) + 16 * db + 8 * (q % 2);
        const uint32_t x0 =
            to_bf16_bits(o[db][4 * q] * inv) | (uint32_t(to_bf16_bits(o[db][4 * q + 1] * inv)) << 16);
        const uint32_t x1 =
            to_bf16_bits(o[db][4 * q + 2] * inv) | (uint32_t(to_bf16_bits(o[db][4 * q + 3] * inv)) << 16);
        *reinterpret_cast<uint2*>(op + d0) = make_uint2(x0, x1);
      }
    }
  } else {
    const int64_t prow = ((static_cast<int64_t>(b_row) * a.Hkv + g) * a.S + part) * RBR +
                         (prefix ? node * a.G + row % a.G : row);
    float* po = a.part_o + prow * D + 4 * h;
#pragma unroll
    for (int db = 0; db < Sh::DB; ++db) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int d0 = (D / 2) * (q / 2) + 16 * db + 8 * (q % 2);
        *reinterpret_cast<f32x4*>(po + d0) = f32x4{o[db][4 * q], o[db][4 * q + 1], o[db][4 * q + 2], o[db][4 * q + 3]};
      }
    }
    if (h == 0) {
      a.part_ml[2 * prow] = m;
      a.part_ml[2 * prow + 1] = lt;
    }
  }
  };

  // Persistent workgroups: each takes the next item of the work list until
  // the list is exhausted.
  __shared__ int32_t s_item;
  const int n_items = a.plan[0];
  for (;;) {
    if (tid == 0) s_item = atomicAdd(a.plan + 1, 1);
    __syncthreads();
    const int idx = s_item;
    if (idx >= n_items) break;
    const int b = a.plan[kPlanHeader + 2 * idx];
    const int packed = a.plan[kPlanHeader + 2 * idx + 1];
    run_item(b & 0xffff, packed & 0xff, packed >> 8, (b >> 16) & 0x7fff, static_cast<uint32_t>(b) & kPrefixItem);
    __syncthreads();  // LDS and s_item are reused by the next item
  }
}


constexpr int kMaxGroups = 4096;   // groups of a batch, whose counts are held in LDS
constexpr int kGroupsEach = 4;     // of a thread of the plan kernel
// Sequences and groups up to which the plan kernel has 256 threads: a wave to a SIMD
// runs the steps that do not depend on the batch's size in a quarter of the time (256
// single tokens 177 us a call, 180 with 1024 threads; 128 trees 129 and 131).
constexpr int kSmallPlan = 512;
constexpr int kFew = 16;           // items or nodes up to which a thread lists them by itself
// Lanes that list the items and nodes of one group or sequence otherwise (64: 13.6 us
// a plan for 128 trees of 1 to 64 nodes, 8.6 for 64 of 8 nodes with 129 splits of their
// prompt; 32: 12.4 and 9.1; 16: 11.7 and 10.1).
constexpr int kListLanes = 32;
constexpr int kMaxSplits = 32;     // of all keys of a sequence, about: a row's partial results are joined one by one

struct PlanArgs {
  const int32_t* group_ids;
  const int32_t* prefix_len;
  int32_t n_groups, slots, least_chunk;  // (slots: workgroups that run at a time)
};

// What a thread lists, or leaves to kListLanes: a group's or a sequence's items.
struct Listing {
  int id, nodes, keys, at0, at1, list;  // (a sequence's place in its group's list of nodes, or -1)
};

// Sum over the wave in its last lane, by DPP adds as wave_sum's.
__device__ inline float wave_sum_f(float x) {
  auto step = [&](auto ctrl, auto rows) {
    x += __uint_as_float(__builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(x)), decltype(ctrl)::value,
                                                     decltype(rows)::value, 0xf, false));
  };
  typedef std::integral_constant<int, 0xf> all;
  step(std::integral_constant<int, 0x111>(), all());
  step(std::integral_constant<int, 0x112>(), all());
  step(std::integral_constant<int, 0x114>(), all());
  step(std::integral_constant<int, 0x118>(), all());
  step(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());
  step(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());
  return x;
}

// What a batch takes with each number of keys per split, in tiles of a CU's time.
constexpr int kChunks = 6;  // 256 .. 8192
struct Load {
  float full = 0.f, rest = 0.f, items = 0.f, parts = 0.f;  // of a KV head: whole splits, other tiles, items, row parts
  __device__ void add(int total, int rbs, int c) {
    const int whole = total / (kSmallChunk << c), left = total - whole * (kSmallChunk << c);
    full += static_cast<float>(whole) * rbs;
    rest += static_cast<float>((left + kTile - 1) / kTile) * rbs;
    items += static_cast<float>(whole + (left > 0)) * rbs;
  }
};
constexpr float kItemTiles = 2.f;      // of an item's start and end
constexpr float kPartTiles = 1e-4f;    // of a row's part: 1 KB written and read at 5 TB/s, tiles being 2 us

// One workgroup: groups, keys per split, item classes (as tree_attn_plan_kernel),
// then the lists.  A thread of a batch has at most one group or sequence at a
// time, and lists its items if they are few (with a wave for every sequence a plan for
// 256 of them took 19 us, with 16 waves 12, and with four 10).
template <int kPlanThreads>
__global__ __launch_bounds__(kPlanThreads) void shared_plan_kernel(SharedArgs a, PlanArgs p) {
  constexpr int kPlanWaves = kPlanThreads / SRT_WAVE, kGroups = kGroupsEach * kPlanThreads;
  __shared__ int32_t cnt[kPlanKeys], off[kPlanKeys];
  __shared__ int32_t members[kGroups], nodes[kGroups], keys[kGroups], lead[kGroups], alone[kGroups];
  __shared__ int32_t wsum[2][kPlanWaves];
  __shared__ Listing left[kPlanThreads];
  __shared__ int32_t ncomb, widest, n_left, most;
  __shared__ float loads[kPlanWaves][4 * kChunks], totals[4 * kChunks];
  const int tid = threadIdx.x, lane = tid % SRT_WAVE, wv = tid / SRT_WAVE;
  auto group_of = [&](int b) {
    const int g = p.n_groups > 0 ? p.group_ids[b] : -1;
    return g >= 0 && g < p.n_groups ? g : -1;
  };
  auto row_blocks = [&](int n) { return (n * a.G + kRowsPerBlock - 1) / kRowsPerBlock; };
  // What a tile of keys costs for the rows of n nodes: a workgroup's part in it, and its waves'.
  auto tile_cost = [&](int n) { return kWaves * row_blocks(n) + (n * a.G + kRowsPerWave - 1) / kRowsPerWave; };

  for (int k = tid; k < kPlanKeys; k += kPlanThreads) cnt[k] = 0;
  for (int g = tid; g < p.n_groups; g += kPlanThreads) {
    members[g] = nodes[g] = alone[g] = 0;
    keys[g] = lead[g] = 0x7fffffff;
  }
  if (tid == 0) ncomb = widest = most = 0;
  SeqInfo si = {0, 0, 0};  // of this thread's sequence of the current kPlanThreads, and its group
  int mine = -1;
  auto take = [&](int b) {
    si = seq_info(a, b);
    mine = group_of(b);
  };
  if (tid < a.B) take(tid);
  int stated[kGroupsEach];
#pragma unroll
  for (int j = 0; j < kGroupsEach; ++j) {
    const int g = tid * kGroupsEach + j;
    stated[j] = g < p.n_groups ? p.prefix_len[g] : 0;
  }
  __syncthreads();
  for (int b = tid; b < a.B; b += kPlanThreads) {
    if (b >= kPlanThreads) take(b);
    if (mine < 0) continue;
    atomicAdd(&members[mine], 1);
    atomicAdd(&nodes[mine], si.n);
    atomicAdd(&alone[mine], tile_cost(si.n));
    atomicMin(&keys[mine], si.L);
    atomicMin(&lead[mine], b);
  }
  __syncthreads();
  // Keys that each group shares, where its nodes' list starts, and what the items take.
  int sum = 0;
  Load load[kChunks];
  int longest = 0;  // keys of a group or a sequence
#pragma unroll
  for (int j = 0; j < kGroupsEach; ++j) {
    const int g = tid * kGroupsEach + j;
    if (g >= p.n_groups) continue;
    int P = min(stated[j], keys[g]);
    P = members[g] > 1 && P > 0 ? P & ~(a.page - 1) : 0;
    // Where the rows fill the tiles by themselves, sharing saves less than the parts
    // cost that it makes of every row (32 prompts of 2k to 4k keys with eight answers,
    // 28 heads, full trees of 64 nodes: 929 us a call shared, 738 not; trees of 1 to
    // 64 nodes of 12 heads: 139 and 156).
    if (static_cast<int64_t>(alone[g] - tile_cost(nodes[g])) * (P / kTile) < static_cast<int64_t>(nodes[g]) * a.G) P = 0;
    keys[g] = P;
    if (P == 0) nodes[g] = 0;
    sum += nodes[g];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) load[c].add(P, row_blocks(nodes[g]), c);
    longest = max(longest, P);
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
#pragma unroll
    for (int j = 0; j < kPlanWaves; ++j) before += j < wv ? ws[j] : 0;
    return before + incl - x;
  };
  int at = scan(sum, wsum[0]);  // (its barrier orders keys[] and nodes[] too)
#pragma unroll
  for (int j = 0; j < kGroupsEach; ++j) {
    const int g = tid * kGroupsEach + j;
    if (g >= p.n_groups) continue;
    a.group[g] = make_int4(lead[g], keys[g], at, nodes[g]);
    members[g] = at;  // from here on: the next free entry of the group's list
    at += nodes[g];
  }
  for (int b = tid; b < a.B; b += kPlanThreads) {
    if (a.B > kPlanThreads) take(b);
    const int P = mine >= 0 ? keys[mine] : 0;
    a.seq_prefix[b] = P;
    longest = max(longest, si.total - P);
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      load[c].add(si.total - P, row_blocks(si.n), c);
      const int least = kSmallChunk << c, parts = (P + least - 1) / least + (si.total - P + least - 1) / least;
      if (parts > 1) load[c].parts += static_cast<float>(parts) * si.n * a.G;
    }
  }
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const float x[4] = {wave_sum_f(load[c].full), wave_sum_f(load[c].rest), wave_sum_f(load[c].items),
                        wave_sum_f(load[c].parts)};
    if (lane == SRT_WAVE - 1)
#pragma unroll
      for (int j = 0; j < 4; ++j) loads[wv][4 * c + j] = x[j];
  }
#pragma unroll
  for (int d = SRT_WAVE / 2; d >= 1; d >>= 1) longest = max(longest, shfl_xor(longest, d));
  if (lane == 0) atomicMax(&most, longest);
  __syncthreads();
  if (tid < 4 * kChunks) {  // (in the same order always, so that a batch's splits are the same ones)
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < kPlanWaves; ++i) x += loads[i][tid];
    totals[tid] = x;
  }
  __syncthreads();
  // Keys per split: those with which the batch is done first.
  int chunk = kChunk;
  float least_time = INFINITY;
#pragma unroll
  for (int c = kChunks - 1; c >= 0; --c) {
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = totals[4 * c + j];
    // Rounds of whole splits, then the rest of them, around which the others lie.
    const float each = (kSmallChunk << c) / kTile, whole = x[0] * a.Hkv, rounds = floorf(whole / p.slots);
    const float over = whole - rounds * p.slots, fill = (over * each + x[1] * a.Hkv) / p.slots;
    const float time = fmaxf(rounds * each + (over > 0.f ? fmaxf(each, fill) : fill),
                             fminf(each, static_cast<float>(most / kTile))) +
                       x[2] * a.Hkv / p.slots * kItemTiles + x[3] * a.Hkv * kPartTiles;
    if (time < least_time && (kSmallChunk << c) >= p.least_chunk) {
      least_time = time;
      chunk = kSmallChunk << c;
    }
  }
  const int cshift = 31 - __clz(chunk);
  auto splits_of = [&](int total) { return (total + chunk - 1) >> cshift; };
  // Visits the item classes of `n` nodes against `total` keys: f(class, key, splits).
  auto classes = [&](int total, int n, auto&& f) {
    const int full = total >> cshift, tail = total - (full << cshift);
    const int waves = min(kWaves, (n * a.G + kRowsPerWave - 1) / kRowsPerWave);
    if (full > 0) f(0, plan_key(chunk / kTile, waves), full);
    if (tail > 0) f(1, plan_key((tail + kTile - 1) / kTile, waves), 1);
  };
  auto count = [&](int total, int n) {
    const int per = a.Hkv * row_blocks(n);
    if (n > 0) classes(total, n, [&](int, int key, int ns) { atomicAdd(&cnt[key], ns * per); });
  };
  for (int g = tid; g < p.n_groups; g += kPlanThreads) count(keys[g], nodes[g]);
  for (int b = tid; b < a.B; b += kPlanThreads) {
    if (a.B > kPlanThreads) take(b);
    count(si.total - (mine >= 0 ? keys[mine] : 0), si.n);
  }
  __syncthreads();
  static_assert(kPlanKeys % kPlanThreads == 0, "classes of a thread");
  constexpr int kKeysEach = kPlanKeys / kPlanThreads;
  int n[kKeysEach], in_all = 0;
#pragma unroll
  for (int j = 0; j < kKeysEach; ++j) in_all += n[j] = cnt[tid * kKeysEach + j];
  int before = scan(in_all, wsum[1]);
#pragma unroll
  for (int j = 0; j < kKeysEach; ++j) {
    off[tid * kKeysEach + j] = before;
    before += n[j];
  }
  if (tid == kPlanThreads - 1) {
    a.plan[0] = before;  // all classes
    a.plan[1] = 0;
    a.plan[kPlanChunk] = chunk;
  }
  __syncthreads();
  // The lists, a thread to a group and then to a sequence at a time.
  int wide = 0;
  const int group_steps = (p.n_groups + kPlanThreads - 1) / kPlanThreads;
  const int seq_steps = (a.B + kPlanThreads - 1) / kPlanThreads;
  for (int step = 0; step < group_steps + seq_steps; ++step) {
    const bool prefix = step < group_steps;
    const int x = (prefix ? step : step - group_steps) * kPlanThreads + tid;
    const uint32_t kind = prefix ? kPrefixItem : 0u;
    auto write = [&](int to, int id, int g, int s, int rb) {
      *reinterpret_cast<int2*>(a.plan + kPlanHeader + 2 * to) =
          make_int2(static_cast<int>(static_cast<uint32_t>(id | rb << 16) | kind), g | s << 8);
    };
    if (tid == 0) n_left = 0;
    __syncthreads();
    Listing m = {x, 0, 0, 0, 0, -1};
    if (x < (prefix ? p.n_groups : a.B)) {
      if (prefix) {
        m.keys = keys[x];
        m.nodes = nodes[x];
      } else {
        if (a.B > kPlanThreads) take(x);
        const int P = mine >= 0 ? keys[mine] : 0;
        m.keys = si.total - P;
        m.nodes = si.n;
        if (P > 0) m.list = atomicAdd(&members[mine], si.n);
        const int parts = splits_of(P) + splits_of(m.keys);
        if (parts > 1) {
          *reinterpret_cast<int2*>(a.plan + a.combine_at + 2 * atomicAdd(&ncomb, 1)) =
              make_int2(x | parts << 16, si.n * a.G);
          wide = max(wide, si.n * a.G);
        }
      }
    }
    if (m.nodes > 0) {
      const int rbs = row_blocks(m.nodes), per = a.Hkv * rbs, splits = splits_of(m.keys);
      classes(m.keys, m.nodes, [&](int c, int key, int ns) {
        const int to = atomicAdd(&off[key], ns * per);
        (c == 0 ? m.at0 : m.at1) = to;
      });
      if (splits * per <= kFew && (m.list < 0 || m.nodes <= kFew)) {
        const int full = m.keys >> cshift;
        for (int s = 0; s < splits; ++s) {
          int to = s < full ? m.at0 + s * per : m.at1;
          for (int g = 0; g < a.Hkv; ++g)
            for (int rb = 0; rb < rbs; ++rb, ++to) write(to, x, g, s, rb);
        }
        if (m.list >= 0)
          for (int y = 0; y < m.nodes; ++y) a.node_of[m.list + y] = x << 8 | y;
      } else {
        left[atomicAdd(&n_left, 1)] = m;
      }
    }
    __syncthreads();
    for (int i = tid / kListLanes; i < n_left; i += kPlanThreads / kListLanes) {
      const Listing l = left[i];
      const int rbs = row_blocks(l.nodes), per = a.Hkv * rbs, full = l.keys >> cshift, splits = splits_of(l.keys);
      for (int y = tid % kListLanes; y < splits * per; y += kListLanes) {
        const int s = y / per, r = y - s * per, g = r / rbs;
        write(s < full ? l.at0 + y : l.at1 + y - full * per, l.id, g, s, r - g * rbs);
      }
      if (l.list >= 0)
        for (int y = tid % kListLanes; y < l.nodes; y += kListLanes) a.node_of[l.list + y] = l.id << 8 | y;
    }
    __syncthreads();
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
  int chunk, slots;      // keys per split, at least; partial results of a row, at most
  size_t plan, groups, prefixes, nodes, part_rows, total;  // bytes
};

size_t round256(size_t x) { return (x + 255) / 256 * 256; }

Sizes sizes_for(int32_t B, int32_t N, int32_t Hq, int32_t Hkv, int32_t d, int64_t cap, int32_t n_groups) {
  Sizes z;
  const int32_t G = Hq / Hkv;
  z.rb = (static_cast<int64_t>(N) * G + kRowsPerBlock - 1) / kRowsPerBlock;
  // The least keys per split that the plan kernel may choose: kMaxSplits of all keys, and
  // partial results of 1 GiB.
  const int64_t row = static_cast<int64_t>(B) * Hkv * N * G * (d + 2) * sizeof(float);
  z.chunk = kSmallChunk;
  while (z.chunk < kChunk && (splits_for(cap, z.chunk) > kMaxSplits || (splits_for(cap, z.chunk) + 1) * row > (int64_t(1) << 30)))
    z.chunk *= 2;
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
  z.total = std::max(z.total, scratch_for(B, N, Hq, Hkv, d, cap, chunk_for(B, Hkv, z.rb, cap, true, 0), false));
  return z;
}

// Whether srt_tree_attn gives every item a CU of its own: sharing has nothing to save
// there, and a plan to make and parts to join (28 heads, 4 KV heads, single tokens: 4
// answers to 2048 keys 28 us a call shared, 18 not; 16 to 2048 32 and 26; 32 to 2048, one
// item too many for the CUs, 33 and 40).
bool each_alone(int32_t B, int32_t Hkv, int64_t rb, int64_t cap, int cus) {
  const int c = chunk_for(B, Hkv, rb, cap, true, 0);
  return static_cast<int64_t>(B) * Hkv * splits_for(cap, c) * rb <= cus;
}

// Work-list packing: 16 bits of a sequence or group, 15 of a row block, 8 of a KV head, 24 of
// a split; and that of srt_tree_attn, which takes some of the calls.
bool fits(int32_t B, int32_t N, int32_t Hq, int32_t Hkv, int64_t cap, int32_t n_groups) {
  if (n_groups > kMaxGroups || cap > (int64_t(1) << 30) || !packs(B, N, Hq, Hkv, cap, false)) return false;
  const int64_t rows = static_cast<int64_t>(B) * N * (Hq / Hkv);
  if (rows / kRowsPerBlock > 32766) return false;
  const Sizes z = sizes_for(B, N, Hq, Hkv, 128, cap, n_groups);
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

  const int cus = cu_count();
  if (cus <= 0) return SRT_ERR_HIP;
  if (n_groups == 0 || each_alone(B, Hkv, z.rb, cap, cus))
    return srt_tree_attn(B, N, Hq, Hkv, d, page, max_pages, num_pages, q, k_cache, v_cache, block_table, ctx_len,
                         tree_parent, n_nodes, scale, out, scratch, scratch_bytes, stream);

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

  const unsigned grid = static_cast<unsigned>(std::min<int64_t>(z.items, cus));
  hipStream_t s = as_stream(stream);
  const PlanArgs plan = {group_ids, prefix_len, n_groups, cus, z.chunk};
  if (B <= kSmallPlan && n_groups <= kSmallPlan) shared_plan_kernel<256><<<1, 256, 0, s>>>(a, plan);
  else shared_plan_kernel<1024><<<1, 1024, 0, s>>>(a, plan);
  if (d == 128) shared_attn_kernel<128><<<grid, kThreads, 0, s>>>(a);
  else shared_attn_kernel<64><<<grid, kThreads, 0, s>>>(a);
  launch_combine(a, d, false, static_cast<unsigned>(combine_grid(a, cus)), s);
  return launch_status();
}
