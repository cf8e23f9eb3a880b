// Tree-masked attention over a paged KV cache held in 8 bits (MFMA, gfx950).
//
// Method: as tree_attn.hip -- every node of the draft tree against the
// context and its ancestors in one pass (Section 3 of the paper) -- with the
// context's full pages as e4m3 or int8 codes and a scale s for each page and
// KV head, the open page in bf16 (the tail) and the tree's own vectors in bf16
// where the projection wrote them.  With codes k, v and scales sk, sv
//   score = scale * sk * (q . k),  out = sum p * sv * v / sum p.
//
// GPU design.  The products are tree_attn.hip's: S^T = K Q^T and O^T = V^T P^T
// on v_mfma_f32_32x32x16_bf16, a query row in one lane column, P from
// registers, online softmax with a lazily raised reference.  What differs:
//   * Every code is exact in bf16, so codes are widened as they are stored to
//     LDS and enter the MFMAs unscaled; nothing is rounded before the softmax.
//     A page has at least 16 keys, so the scales are uniform over the 16 keys
//     (8 accumulator registers) of a group: sk goes into the multiplier of the
//     fused multiply-add that every score takes anyway, sv as log2 sv into
//     its addend, so the exponential is p * sv, which is what the second
//     product needs, and the sum of p is the groups' sums times 1 / sv.
//   * The pages are streamed first, then the open keys (tail and tree) in
//     tiles of their own.
//   * The bytes of a step are halved, so a batch with few query rows per KV
//     head would be bound by one wave's chain per tile (1.3 us for 64 keys in
//     tree_attn.hip, whatever the rows).  A workgroup's 8 waves are therefore
//     WR waves along the rows times 8 / WR along the keys, by the rows that the
//     item has (4 waves, two workgroups to a CU, in batches of narrow trees): up
//     to 32 rows every wave streams 32-key tiles of its own, with no barrier at
//     all, up to 64 and 128 pairs and fours of waves share a tile, and the key
//     groups' partial results are merged in LDS at the end.
#include "attn.h"
#include "kv_quant.h"

namespace {

struct QuantArgs : AttnBase {
  const uint16_t* q;
  const uint8_t* k;
  const uint8_t* v;
  const float* k_scale;
  const float* v_scale;
  const uint16_t* k_tail;
  const uint16_t* v_tail;
  const uint16_t* k_new;
  const uint16_t* v_new;
  const int32_t* bt;
  const int32_t* parent;
  int64_t ld;  // elements from one new token to the next
  int64_t num_pages;
  int32_t page, page_shift, max_pages;
  float scale_log2;
};

constexpr int kGroup = 16;  // keys that share their scales (a page has at least as many)
// Narrow trees (half_waves): workgroups of this many waves, two to a CU, so that one
// streams while the other claims, fills, drains and merges (28 heads, 4 KV heads, single
// tokens: 256 sequences of 200 to 2000 keys 52 -> 36 us, 512 of 2k to 10k 237 -> 217;
// with workgroups of two waves, four to a CU, 50 and 234).  A batch that has an item for
// every CU at most keeps 8 waves (4 sequences: 10.2 and 11.1).
constexpr int kNarrowWaves = 4;
// Bytes of a bf16 row times keys of the table, up to which a narrow batch has a
// workgroup launched for every item: no list, no claims (185 sequences of 60 keys, 8 KV
// heads of 64, 27 nodes: 37 -> 18.6 us; 28 heads, 4 KV heads of 128, 512 sequences of up
// to 1500 keys, one node: 50.7 -> 42.3; 256 of up to 2000: 35.9 -> 37.1, the longest no
// longer come first).
constexpr int64_t kUnlisted = 1536 * 2 * 128;
constexpr float kLeastScale = 0x1p-70f, kMostScale = 0x1p100f;

// Of a workgroup of W waves for trees of up to R rows (of a block, where W is 8).
template <int D, int W, int R>
struct Smem {
  using Sh = Shape<D>;
  static constexpr int kRow = Sh::KSTRIDE + Sh::VSTRIDE;
  static constexpr int kNodes = W == kWaves ? kMaxN : R;
  static constexpr int kKeys = W == kWaves || R <= 32 ? kChunk : kChunk / 2;  // of a split
  __attribute__((aligned(16))) uint8_t pool[32 * W * kRow];  // tiles, then the key groups' partial results
  uint64_t anc[kNodes][4];
  int32_t spar[kNodes];
  __attribute__((aligned(16))) float kc[kKeys / kGroup];  // scale * log2(e) * sk of the split's key groups
  __attribute__((aligned(16))) float lv[kKeys / kGroup];  // log2(sv)
  __attribute__((aligned(16))) float rv[kKeys / kGroup];  // 1 / sv
  float m[W][kRowsPerWave], l[W][kRowsPerWave];
};

// The place in a row of K or V of 16-byte chunk c of its LDS row.  A lane holds
// 16 consecutive codes of a 128-code row, two chunks when widened; the first
// chunks of a row's eight lanes are stored side by side, then the second ones,
// so that the stores are conflict-free.  Q's fragments and the epilogue follow.
template <int D>
__device__ constexpr int chunk_at(int c) {
  return D == 128 ? (c < 8 ? 2 * c : 2 * (c - 8) + 1) : c;
}

// LDS accesses of a wave's lanes before this come before those after it.
__device__ inline void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
}

// Four codes as two words of two bf16 (exact: e4m3 has 4 significant bits, int8 7).
template <int KV>
__device__ inline uint2 widen(uint32_t w) {
  if constexpr (KV == SRT_KV_E4M3) {
    const auto lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false);
    const auto hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true);
    return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
  } else {
    const float f0 = static_cast<int8_t>(w), f1 = static_cast<int8_t>(w >> 8);
    const float f2 = static_cast<int8_t>(w >> 16), f3 = static_cast<int8_t>(w >> 24);
    // the upper halves of two floats
    return make_uint2(__builtin_amdgcn_perm(__float_as_uint(f1), __float_as_uint(f0), 0x07060302u),
                      __builtin_amdgcn_perm(__float_as_uint(f3), __float_as_uint(f2), 0x07060302u));
  }
}

// One work item: rows rb * 256 .. of (sequence b, KV head g) against the keys of
// split s, with W waves, WR of them along the rows.
template <int D, int KV, int WR, int W, int R>
__device__ __forceinline__ void attend(const QuantArgs& a, Smem<D, W, R>& sm, const SeqInfo si, int b, int g, int s,
                                       int rb) {
  using Sh = Shape<D>;
  constexpr int WK = W / WR;                  // groups of waves along the keys
  constexpr int T = WR == 8 ? 64 : 32;        // keys per tile
  constexpr int KB = T / 32;                  // MFMA key blocks per tile
  constexpr int NB = WR == 1 ? 1 : 2;         // tile buffers per key group
  constexpr int KPW = T / WR;                 // keys that a wave stages of each tile
  constexpr int U = KPW < kGroup ? KPW : kGroup;  // staged through one descriptor (all in one page)
  constexpr int UPT = KPW / U;
  constexpr int LPU = U / 8;                  // loads per unit: 8 rows each, 8 lanes a row
  constexpr int EPL = D / 8;                  // codes per lane and load
  constexpr int kKeys = Smem<D, W, R>::kKeys;
  constexpr int NPG = kKeys / W / U / SRT_WAVE;  // registers of page ids
  constexpr int kTileBytes = T * (Sh::KSTRIDE + Sh::VSTRIDE);
  // Few rows: the pages are read once, by this workgroup alone, and need no
  // place in the caches (256 sequences of one node, 28 heads: 260 us with
  // ordinary loads, 225 with non-temporal ones; other row blocks read wide
  // trees' pages again: 531 and 543).
  constexpr int kAux = WR == 8 ? 0 : 2;
  static_assert(NB * WK * T <= 32 * W, "tiles fit the pool");
  static_assert(NPG * SRT_WAVE * U * W == kKeys && NPG >= 1 && NPG <= 2, "page ids of a split");

  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid / SRT_WAVE);
  const int wr = w % WR, kg = w / WR;
  const int lane = tid % SRT_WAVE, l32 = lane % 32, h = lane / 32;

  const int rows = si.n * a.G;
  const int k_begin = s * a.chunk;
  const int k_end = min(k_begin + a.chunk, si.total);
  const int nsplit = (si.total + a.chunk - 1) / a.chunk;
  const int full = si.L & ~(a.page - 1);      // keys in pages
  const int lim = min(k_end, full);           // of this split
  const int n1 = lim > k_begin ? (lim - k_begin + T - 1) / T : 0;
  const int o_begin = max(k_begin, full);     // open keys of this split: o_begin .. k_end - 1
  const int n2 = k_end > o_begin ? (k_end - o_begin + T - 1) / T : 0;
  const int row0 = rb * kRowsPerBlock + wr * kRowsPerWave;
  const bool wave_active = row0 < rows;

  // Scales of the split's key groups.
  const int64_t bt_row = static_cast<int64_t>(b) * a.max_pages;
  const int pshift = a.page_shift, pmask = a.page - 1;
  for (int i = tid; i < n1 * (T / kGroup); i += W * SRT_WAVE) {
    const int p = k_begin + i * kGroup;
    float ks = 1.f, vs = 1.f;
    if (p < lim) {
      const int pg = a.bt[bt_row + (p >> pshift)];
      if (pg >= 0 && pg < a.num_pages) {
        const int64_t at = static_cast<int64_t>(pg) * a.Hkv + g;
        ks = a.k_scale[at];
        vs = fminf(fmaxf(a.v_scale[at], kLeastScale), kMostScale);
      }
    }
    sm.kc[i] = ks * a.scale_log2;
    sm.lv[i] = __builtin_amdgcn_logf(vs);  // base 2
    sm.rv[i] = 1.f / vs;
  }
  // Ancestor-or-self bitsets, where the split reaches the tree.
  if (k_end > si.L) {
    for (int i = tid; i < si.n; i += W * SRT_WAVE) sm.spar[i] = a.parent[static_cast<int64_t>(b) * a.N + i];
    __syncthreads();
    for (int i = tid; i < si.n; i += W * SRT_WAVE) {
      uint64_t bits[4] = {0, 0, 0, 0};
      int j = i;
      while (j >= 0) {
        bits[j >> 6] |= 1ull << (j & 63);
        const int pj = sm.spar[j];
        if (pj >= j) break;  // malformed parent: stop (parents precede children)
        j = pj;
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) sm.anc[i][x] = bits[x];
    }
  }

  // Query fragment: head dims of LDS chunk 2 ks + h.
  const int row = row0 + l32;
  const bool row_ok = row < rows;
  const int node = row_ok ? row / a.G : 0;
  bf16x8 qf[Sh::KS];
  {
    const int hq = g * a.G + (row_ok ? row % a.G : 0);
    const bf16x8* qp = reinterpret_cast<const bf16x8*>(a.q + ((static_cast<int64_t>(b) * a.N + node) * a.Hq + hq) * D);
#pragma unroll
    for (int ks = 0; ks < Sh::KS; ++ks)
      qf[ks] = row_ok ? (h ? qp[chunk_at<D>(2 * ks + 1)] : qp[chunk_at<D>(2 * ks)]) : bf16x8{};
  }

  f32x16 o[Sh::DB];
#pragma unroll
  for (int db = 0; db < Sh::DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[db][r] = 0.f;
  constexpr float kLazy = 8.f;
  float m = -INFINITY;  // reference of the row (log2 units)
  float l = 0.f;        // lane-partial sum

  // ---- staging of pages ----------------------------------------------------
  // Wave wr of a key group moves keys wr * KPW .. of the group's tile, U keys
  // of one page through one descriptor (no bytes where the page is past the
  // split's pages or outside the pool: such keys read as zero).
  int pg_lane[NPG];
#pragma unroll
  for (int j = 0; j < NPG; ++j) {
    const int u = SRT_WAVE * j + lane;
    const int p0 = k_begin + ((u / UPT) * WK + kg) * T + wr * KPW + (u % UPT) * U;
    const int pg = p0 < lim ? a.bt[bt_row + (p0 >> pshift)] : -1;
    pg_lane[j] = pg >= 0 && pg < a.num_pages ? pg : -1;
  }
  typedef int ivec __attribute__((ext_vector_type(EPL / 4)));
  ivec kreg[UPT][LPU], vreg[UPT][LPU];
  const int gl_off = (lane / 8) * D + (lane % 8) * EPL;
  const int64_t head_bytes = static_cast<int64_t>(a.page) * D;
  auto load_unit = [&](const uint8_t* base, int64_t off, int nbytes, ivec (&r)[LPU]) {
    const __amdgpu_buffer_rsrc_t rsrc =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base + off), 0, nbytes, 0x00020000);
#pragma unroll
    for (int j = 0; j < LPU; ++j) {
      if constexpr (EPL == 16) r[j] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, gl_off + j * 8 * D, 0, kAux);
      else r[j] = __builtin_amdgcn_raw_buffer_load_b64(rsrc, gl_off + j * 8 * D, 0, kAux);
    }
  };
  auto load_pages = [&](int it) {
#pragma unroll
    for (int j = 0; j < UPT; ++j) {
      const int u = it * UPT + j;
      int pg = -1;
      if (u < NPG * SRT_WAVE) {
        pg = NPG == 1 || u < SRT_WAVE ? __builtin_amdgcn_readlane(pg_lane[0], u % SRT_WAVE)
                                      : __builtin_amdgcn_readlane(pg_lane[NPG - 1], u % SRT_WAVE);
      }
      const int p0 = k_begin + (it * WK + kg) * T + wr * KPW + j * U;
      const int64_t off =
          pg >= 0 ? (static_cast<int64_t>(pg) * a.Hkv + g) * head_bytes + static_cast<int64_t>(p0 & pmask) * D : 0;
      const int nbytes = pg >= 0 ? U * D : 0;
      load_unit(a.k, off, nbytes, kreg[j]);
      load_unit(a.v, off, nbytes, vreg[j]);
    }
  };
  const int st_row = wr * KPW + lane / 8;
  auto put = [&](uint8_t* to, const ivec& c) {  // one lane's codes, widened
    uint32_t x[EPL / 2];
#pragma unroll
    for (int i = 0; i < EPL / 4; ++i) {
      const uint32_t word = c[i];
      const uint2 two = widen<KV>(word);
      x[2 * i] = two.x;
      x[2 * i + 1] = two.y;
    }
#pragma unroll
    for (int i = 0; i < EPL / 8; ++i)
      *reinterpret_cast<uint4*>(to + i * D) = make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
  };
  auto store_pages = [&](uint8_t* tile) {
    uint8_t* Kb = tile + st_row * Sh::KSTRIDE + (lane % 8) * 16;
    uint8_t* Vb = tile + T * Sh::KSTRIDE + st_row * Sh::VSTRIDE + (lane % 8) * 16;
#pragma unroll
    for (int j = 0; j < UPT; ++j)
#pragma unroll
      for (int i = 0; i < LPU; ++i) {
        put(Kb + (j * U + i * 8) * Sh::KSTRIDE, kreg[j][i]);
        put(Vb + (j * U + i * 8) * Sh::VSTRIDE, vreg[j][i]);
      }
  };
  // Open keys t0 .. of a tile straight to LDS (a lane holds 16 or 8 elements of
  // a row, as for pages); keys past the split's end are zero.
  auto stage_open = [&](int t0, uint8_t* tile) {
#pragma unroll
    for (int i = 0; i < KPW / 8; ++i) {
      const int p = t0 + st_row + 8 * i;
      uint4 kx[EPL / 8], vx[EPL / 8];
#pragma unroll
      for (int e = 0; e < EPL / 8; ++e) kx[e] = vx[e] = make_uint4(0, 0, 0, 0);
      if (p < k_end) {
        const bool tail = p < si.L;
        const int64_t off = tail ? ((static_cast<int64_t>(b) * a.Hkv + g) * a.page + (p & pmask)) * D
                                 : (static_cast<int64_t>(b) * a.N + (p - si.L)) * a.ld + static_cast<int64_t>(g) * D;
        const uint4* kp = reinterpret_cast<const uint4*>((tail ? a.k_tail : a.k_new) + off + (lane % 8) * EPL);
        const uint4* vp = reinterpret_cast<const uint4*>((tail ? a.v_tail : a.v_new) + off + (lane % 8) * EPL);
#pragma unroll
        for (int e = 0; e < EPL / 8; ++e) {
          kx[e] = kp[e];
          vx[e] = vp[e];
        }
      }
      const int r = st_row + 8 * i;
#pragma unroll
      for (int e = 0; e < EPL / 8; ++e) {
        *reinterpret_cast<uint4*>(tile + r * Sh::KSTRIDE + (lane % 8) * 16 + e * D) = kx[e];
        *reinterpret_cast<uint4*>(tile + T * Sh::KSTRIDE + r * Sh::VSTRIDE + (lane % 8) * 16 + e * D) = vx[e];
      }
    }
  };

  // ---- MFMA phases (fragment layouts as in tree_attn.hip) ------------------
  const int k_rd = l32 * Sh::KSTRIDE + 16 * h;
  const int xg = lane % 16;
  const int k_vd = T * Sh::KSTRIDE + (4 * h + xg / 4) * Sh::VSTRIDE +
                   ((Sh::CPR / 2) * ((lane / 16) & 1) + (xg % 4) / 2) * 16 + 8 * (xg & 1);
  auto qk = [&](const uint8_t* tile, f32x16 (&sacc)[KB]) {
    bf16x8 kf[Sh::KS][KB];
#pragma unroll
    for (int ks = 0; ks < Sh::KS; ++ks)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
        kf[ks][kb] = *reinterpret_cast<const bf16x8*>(tile + k_rd + kb * 32 * Sh::KSTRIDE + ks * 32);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[kb][r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < Sh::KS; ++ks)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
        sacc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks][kb], qf[ks], sacc[kb], 0, 0, 0);
    // Half of the fragments are read ahead of the products, the other half as
    // those free their registers (all of them at once spill).
    __builtin_amdgcn_sched_group_barrier(0x100, KB * Sh::KS / 2, 0);
#pragma unroll
    for (int i = 0; i < Sh::KS / 2; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, KB, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, KB, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, KB * Sh::KS / 2, 0);
  };
  typedef short i16x4v __attribute__((ext_vector_type(4)));
  auto v_read = [&](const uint8_t* tile, int ks0, i16x4v (&vf)[2][Sh::DB][2]) {
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
      for (int db = 0; db < Sh::DB; ++db)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
          vf[k2][db][hh] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) i16x4v*)(tile + k_vd + (ks0 + k2) * 16 * Sh::VSTRIDE +
                                                          hh * 8 * Sh::VSTRIDE + db * 32));
  };
  auto pv = [&](const i16x4v (&vf)[2][Sh::DB][2], int ks0, const bf16x8 (&pb)[2 * KB]) {
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
      for (int db = 0; db < Sh::DB; ++db) {
        const bf16x8 va =
            __builtin_bit_cast(bf16x8, __builtin_shufflevector(vf[k2][db][0], vf[k2][db][1], 0, 1, 2, 3, 4, 5, 6, 7));
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pb[ks0 + k2], o[db], 0, 0, 0);
      }
  };

  // Scores to probabilities times sv.  Group x of a tile (keys 16 x ..) is
  // registers 8 (x % 2) .. + 7 of block x / 2 and k-step x of the second product.
  auto softmax = [&](auto open_c, int t0, f32x16 (&sacc)[KB], bf16x8 (&pb)[2 * KB]) {
    constexpr bool kOpen = decltype(open_c)::value;
    const float mref0 = m == -INFINITY ? 0.f : m;
    float lv[2 * KB], rv[2 * KB];
    if constexpr (kOpen) {
#pragma unroll
      for (int x = 0; x < 2 * KB; ++x) lv[x] = 0.f;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[kb][r] = __builtin_fmaf(sacc[kb][r], a.scale_log2, -mref0);
      // bit x of vis: key t0 + x is a tail key or an ancestor-or-self, and lies in the split
      const int lim2 = k_end - t0;
      uint64_t vis = lim2 >= 64 ? ~0ull : (~0ull >> (64 - lim2));  // lim2 >= 1
      const int j0 = t0 - si.L;  // tree index of key t0
      if (j0 > -T) {
        uint64_t win;
        if (j0 >= 0) {
          const int wd = j0 >> 6, sh = j0 & 63;
          const uint64_t lo = wd < 4 ? sm.anc[node][wd] : 0ull;
          const uint64_t hi = wd + 1 < 4 ? sm.anc[node][wd + 1] : 0ull;
          win = sh ? (lo >> sh) | (hi << (64 - sh)) : lo;
        } else {
          const int sh = -j0;  // 1..63 tail keys lead the window
          win = (sm.anc[node][0] << sh) | (~0ull >> (64 - sh));
        }
        vis &= win;
      }
      const uint64_t vh = vis >> (4 * h);
      const uint32_t v0 = static_cast<uint32_t>(vh), v1 = static_cast<uint32_t>(vh >> 32);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const uint32_t vw = kb ? v1 : v0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int x = 8 * (r / 4) + r % 4;
          sacc[kb][r] = ((vw >> x) & 1u) ? sacc[kb][r] : -INFINITY;
        }
      }
    } else {
      const int gi = (t0 - k_begin) / kGroup;
      float kc[2 * KB];
#pragma unroll
      for (int x = 0; x < 2 * KB; ++x) {
        kc[x] = sm.kc[gi + x];
        lv[x] = sm.lv[gi + x];
        rv[x] = sm.rv[gi + x];
      }
#pragma unroll
      for (int x = 0; x < 2 * KB; ++x) {
        const float c = lv[x] - mref0;
#pragma unroll
        for (int r = 0; r < 8; ++r)
          sacc[x / 2][8 * (x % 2) + r] = __builtin_fmaf(sacc[x / 2][8 * (x % 2) + r], kc[x], c);
      }
      if (t0 + T > lim) {  // groups past the split's pages
#pragma unroll
        for (int x = 0; x < 2 * KB; ++x)
          if (t0 + x * kGroup >= lim) {
#pragma unroll
            for (int r = 0; r < 8; ++r) sacc[x / 2][8 * (x % 2) + r] = -INFINITY;
          }
      }
    }
    // p * sv in bf16, the type in which the second product's MFMAs take it (as
    // tree_attn.hip's p; the same rounding of every term, at most 2^-8 of it, and
    // the largest share of the result's error), and this lane's fp32 sum of p, of
    // the rounded ones, so that the weights of a row add up to one.
    auto probs = [&](auto dm_c, float dm) {
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      const bf16x2 one2 = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
      float total = 0.f;
#pragma unroll
      for (int x = 0; x < 2 * KB; ++x) {
        float ps = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          pb[x][e] = static_cast<__bf16>(__builtin_amdgcn_exp2f(
              decltype(dm_c)::value ? sacc[x / 2][8 * (x % 2) + e] - dm : sacc[x / 2][8 * (x % 2) + e]));
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const bf16x2 pr = {pb[x][e], pb[x][e + 1]};
          ps = __builtin_amdgcn_fdot2_f32_bf16(pr, one2, ps, false);
        }
        if constexpr (kOpen) total += ps;
        else total = __builtin_fmaf(ps, rv[x], total);
      }
      return total;
    };
    // Against the current reference first; if every probability of the row is
    // below 2^kLazy (their sum is) these are the final values, else the row
    // maximum is taken, the reference raised as needed, and again.
    float psum = probs(std::false_type(), 0.f);
    const bool fast = m != -INFINITY && psum < 256.f;  // 256 = 2^kLazy
    if (__ballot(!fast)) {
      float mloc = -INFINITY;
#pragma unroll
      for (int x = 0; x < 2 * KB; ++x) {
        float mg = -INFINITY;
#pragma unroll
        for (int r = 0; r < 8; ++r) mg = __builtin_elementwise_maximum(mg, sacc[x / 2][8 * (x % 2) + r]);
        mloc = __builtin_elementwise_maximum(mloc, mg - lv[x]);
      }
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
  auto compute = [&](auto open_c, int t0, const uint8_t* tile) {
    if (!wave_active) return;
    f32x16 sacc[KB];
    qk(tile, sacc);
    i16x4v vf0[2][Sh::DB][2];
    v_read(tile, 0, vf0);
    bf16x8 pb[2 * KB];
    // Of the two waves on a SIMD the one in its softmax issues first: the other's
    // MFMAs wait little for it, its own for the softmax (8 sequences with trees of
    // 64 to 256 nodes: 530 -> 512 us; of no use where waves wait for HBM).
    if constexpr (WR >= 4) __builtin_amdgcn_s_setprio(1);
    softmax(open_c, t0, sacc, pb);
    if constexpr (WR >= 4) __builtin_amdgcn_s_setprio(0);
    if constexpr (KB == 2) {
      i16x4v vf1[2][Sh::DB][2];
      v_read(tile, 2, vf1);
      pv(vf0, 0, pb);
      pv(vf1, 2, pb);
    } else {
      pv(vf0, 0, pb);
    }
  };

  // ---- pages ----------------------------------------------------------------
  uint8_t* const mine = sm.pool + kg * kTileBytes;  // buffer 0 of the key group
  constexpr int kBuffer = WK * kTileBytes;
  if constexpr (WR == 1) {
    // A wave's tiles are its own: the LDS keeps a wave's stores and loads in
    // order, so one buffer serves and no wave waits for another.  The compiler
    // knows of one lane's addresses only: its fences keep the order of stores and
    // reads between the lanes (no instruction comes of them).
    const int iters = n1 > kg ? (n1 - kg + WK - 1) / WK : 0;
    if (iters > 0) load_pages(0);
    __syncthreads();  // the scales (and the bitsets)
    for (int it = 0; it < iters; ++it) {
      store_pages(mine);
      wave_lds_fence();
      if (it + 1 < iters) load_pages(it + 1);
      compute(std::false_type(), k_begin + (it * WK + kg) * T, mine);
      wave_lds_fence();
    }
    for (int it = kg; it < n2; it += WK) {
      stage_open(o_begin + it * T, mine);
      wave_lds_fence();
      compute(std::true_type(), o_begin + it * T, mine);
      wave_lds_fence();
    }
  } else {
    // One barrier a tile: tile t + 1 is stored into the buffers that tile t - 1 left.
    const int iters = (n1 + WK - 1) / WK;
    if (iters > 0) {
      load_pages(0);
      store_pages(mine);
    }
    __syncthreads();
    auto step = [&](int it, auto cur_c) {
      constexpr int cur = decltype(cur_c)::value;
      const bool next = it + 1 < iters;
      if (next) load_pages(it + 1);
      if (it * WK + kg < n1) compute(std::false_type(), k_begin + (it * WK + kg) * T, mine + cur * kBuffer);
      if (next) store_pages(mine + (cur ^ 1) * kBuffer);
      __syncthreads();
    };
    for (int it = 0; it < iters; it += 2) {
      step(it, std::integral_constant<int, 0>());
      if (it + 1 < iters) step(it + 1, std::integral_constant<int, 1>());
    }
    for (int it = 0; it < (n2 + WK - 1) / WK; ++it) {
      const int t = it * WK + kg, t0 = o_begin + t * T;
      if (t < n2) stage_open(t0, mine);
      __syncthreads();
      if (t < n2) compute(std::true_type(), t0, mine);
      __syncthreads();
    }
  }

  // ---- results --------------------------------------------------------------
  const float lt = sum_halves(l);
  const int64_t part0 = ((static_cast<int64_t>(b) * a.Hkv + g) * a.S + s) * a.part_rows;
  if constexpr (WK == 1) {
    if (!row_ok) return;
    const int hq = g * a.G + row % a.G;
    uint16_t* op = a.out + ((static_cast<int64_t>(b) * a.N + node) * a.Hq + hq) * D + 4 * h;
    float* po = a.part_o + (part0 + row) * D + 4 * h;
    const float inv = lt > 0.f ? 1.f / lt : 0.f;
#pragma unroll
    for (int db = 0; db < Sh::DB; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int d0 = 8 * chunk_at<D>(((D / 2) * (q / 2) + 16 * db + 8 * (q % 2)) / 8);
        if (nsplit == 1) {
          const uint32_t x0 =
              to_bf16_bits(o[db][4 * q] * inv) | (uint32_t(to_bf16_bits(o[db][4 * q + 1] * inv)) << 16);
          const uint32_t x1 =
              to_bf16_bits(o[db][4 * q + 2] * inv) | (uint32_t(to_bf16_bits(o[db][4 * q + 3] * inv)) << 16);
          *reinterpret_cast<uint2*>(op + d0) = make_uint2(x0, x1);
        } else {
          *reinterpret_cast<f32x4*>(po + d0) =
              f32x4{o[db][4 * q], o[db][4 * q + 1], o[db][4 * q + 2], o[db][4 * q + 3]};
        }
      }
    if (nsplit > 1 && h == 0) {
      a.part_ml[2 * (part0 + row)] = m;
      a.part_ml[2 * (part0 + row) + 1] = lt;
    }
  } else {
    // Merge of the key groups: out = sum 2^(m_k - M) O_k over the groups.
    constexpr int PS = D + 4;  // floats per partial row (conflict-free 16-byte stores)
    static_assert(W * kRowsPerWave * PS * 4 <= static_cast<int>(sizeof(sm.pool)), "partial results fit the pool");
    float* part = reinterpret_cast<float*>(sm.pool);
    __syncthreads();  // every wave has read its last tile
    if (wave_active) {
#pragma unroll
      for (int db = 0; db < Sh::DB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<f32x4*>(part + (w * kRowsPerWave + l32) * PS + (D / 2) * (q / 2) + 16 * db + 8 * (q % 2) +
                                    4 * h) = f32x4{o[db][4 * q], o[db][4 * q + 1], o[db][4 * q + 2], o[db][4 * q + 3]};
      if (h == 0) {
        sm.m[w][l32] = m;
        sm.l[w][l32] = lt;
      }
    }
    __syncthreads();
    constexpr int Q = D / 4;
    const int here = min(WR * kRowsPerWave, rows - rb * kRowsPerBlock);
    for (int i = tid; i < here * Q; i += W * SRT_WAVE) {
      const int r = i / Q, q = i % Q;
      const int rw = r / kRowsPerWave, rl = r % kRowsPerWave;
      float M = -INFINITY;
#pragma unroll
      for (int k = 0; k < WK; ++k) M = fmaxf(M, sm.m[k * WR + rw][rl]);
      float den = 0.f;
      f32x4 num = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        const int wv = k * WR + rw;
        const float c = sm.m[wv][rl] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm.m[wv][rl] - M);
        den = __builtin_fmaf(c, sm.l[wv][rl], den);
        num += c * *reinterpret_cast<const f32x4*>(part + (wv * kRowsPerWave + rl) * PS + 4 * q);
      }
      const int grow = rb * kRowsPerBlock + r;
      const int d0 = 8 * chunk_at<D>(q / 2) + 4 * (q % 2);
      if (nsplit == 1) {
        const float inv = den > 0.f ? 1.f / den : 0.f;
        uint16_t* op = a.out + ((static_cast<int64_t>(b) * a.N + grow / a.G) * a.Hq + g * a.G + grow % a.G) * D + d0;
        const uint32_t x0 = to_bf16_bits(num[0] * inv) | (uint32_t(to_bf16_bits(num[1] * inv)) << 16);
        const uint32_t x1 = to_bf16_bits(num[2] * inv) | (uint32_t(to_bf16_bits(num[3] * inv)) << 16);
        *reinterpret_cast<uint2*>(op) = make_uint2(x0, x1);
      } else {
        *reinterpret_cast<f32x4*>(a.part_o + (part0 + grow) * D + d0) = num;
        if (q == 0) {
          a.part_ml[2 * (part0 + grow)] = M;
          a.part_ml[2 * (part0 + grow) + 1] = den;
        }
      }
    }
  }
}

template <int D, int KV, int W, int R, bool kDirect>
__global__ __launch_bounds__(W * SRT_WAVE, 2) void tree_attn_quant_kernel(QuantArgs a) {
  __shared__ Smem<D, W, R> sm;
  auto run_item = [&](int b, int g, int s, int rb) {
    const SeqInfo si = seq_info(a, b);
    const int here = si.n * a.G - rb * kRowsPerBlock;
    if (here <= 0 || s * a.chunk >= si.total) return;
    if constexpr (R == 32) {
      attend<D, KV, 1, W>(a, sm, si, b, g, s, rb);
    } else {
      if (here <= 32) attend<D, KV, 1, W>(a, sm, si, b, g, s, rb);
      else if (here <= 64) attend<D, KV, 2, W>(a, sm, si, b, g, s, rb);
      else if (R == 128 || here <= 128) attend<D, KV, 4, W>(a, sm, si, b, g, s, rb);
      else if constexpr (R > 128) attend<D, KV, 8, W>(a, sm, si, b, g, s, rb);
    }
  };
  if constexpr (kDirect) {  // a workgroup for every item there can be
    const int x = blockIdx.x / a.RB, y = x / a.S;
    run_item(y / a.Hkv, y % a.Hkv, x - y * a.S, blockIdx.x - x * a.RB);
    return;
  }
  __shared__ int32_t s_item;
  const int n_items = a.plan[0];
  for (;;) {
    if (threadIdx.x == 0) s_item = atomicAdd(a.plan + 1, 1);
    __syncthreads();
    const int idx = __builtin_amdgcn_readfirstlane(s_item);
    if (idx >= n_items) break;
    const int b = a.plan[kPlanHeader + 2 * idx];
    const int packed = a.plan[kPlanHeader + 2 * idx + 1];
    run_item(b, packed & 0xff, (packed >> 8) & 0xfff, packed >> 20);
    __syncthreads();  // LDS and s_item are reused by the next item
  }
}

template <int D, int KV, int W, int R>
void launch_waves(const QuantArgs& a, bool direct, unsigned grid, hipStream_t s) {
  if (direct) tree_attn_quant_kernel<D, KV, W, R, true><<<grid, W * SRT_WAVE, 0, s>>>(a);
  else tree_attn_quant_kernel<D, KV, W, R, false><<<grid, W * SRT_WAVE, 0, s>>>(a);
}

template <int D, int KV>
void launch_quant(const QuantArgs& a, bool narrow, bool direct, unsigned grid, hipStream_t s) {
  if (!narrow) launch_waves<D, KV, kWaves, kRowsPerBlock>(a, direct, grid, s);
  else if (a.part_rows <= 32) launch_waves<D, KV, kNarrowWaves, 32>(a, direct, grid, s);
  else launch_waves<D, KV, kNarrowWaves, kNarrowRows>(a, direct, grid, s);
}

// Positions that the context and a tree of N nodes may take.
int64_t key_cap(const srt_kv_quant& kv, int32_t N) {
  return (static_cast<int64_t>(kv.max_pages) + 1) * kv.page - 1 + N;
}

}  // namespace

extern "C" size_t srt_tree_attn_quant_scratch_bytes(const srt_kv_quant* kv, int32_t B, int32_t N, int32_t Hq) {
  if (!kv || check_kv_sizes(*kv) != SRT_OK || B < 0 || N < 1 || N > kMaxN || Hq < 1 || Hq % kv->Hkv) return 0;
  const int64_t cap = key_cap(*kv, N);
  if (!packs(B, N, Hq, kv->Hkv, cap, true)) return 0;
  const int64_t RB = (N * (Hq / kv->Hkv) + kRowsPerBlock - 1) / kRowsPerBlock;
  return scratch_for(B, N, Hq, kv->Hkv, kv->d, cap, chunk_for(B, kv->Hkv, RB, cap, true, N * (Hq / kv->Hkv)), true);
}

extern "C" int srt_tree_attn_quant(const srt_kv_quant* kv, int32_t B, int32_t N, int32_t Hq, const uint16_t* q,
                                   const uint16_t* k_new, const uint16_t* v_new, int64_t ld,
                                   const int32_t* tree_parent, const int32_t* n_nodes, float scale, uint16_t* out,
                                   void* scratch, size_t scratch_bytes, void* stream) {
  if (!kv || B < 0 || N < 1 || N > kMaxN || Hq < 1 || !std::isfinite(scale)) return SRT_ERR_INVALID;
  int st = check_kv_sizes(*kv);
  if (st != SRT_OK) return st;
  if (Hq % kv->Hkv) return SRT_ERR_INVALID;
  const int64_t cap = key_cap(*kv, N);
  if (!packs(B, N, Hq, kv->Hkv, cap, true)) return SRT_ERR_UNSUPPORTED;
  if (B == 0) return SRT_OK;
  st = check_kv_pointers(*kv);
  if (st == SRT_OK) st = check_new(*kv, k_new, v_new, ld);
  if (st != SRT_OK) return st;
  if (!q || !tree_parent || !n_nodes || !out) return SRT_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) % 16) return SRT_ERR_INVALID;

  QuantArgs a;
  a.q = q;
  a.k = kv->k_pages;
  a.v = kv->v_pages;
  a.k_scale = kv->k_scale;
  a.v_scale = kv->v_scale;
  a.k_tail = kv->k_tail;
  a.v_tail = kv->v_tail;
  a.k_new = k_new;
  a.v_new = v_new;
  a.bt = kv->block_table;
  a.parent = tree_parent;
  a.ctx_len = kv->ctx_len;
  a.n_nodes = n_nodes;
  a.out = out;
  a.B = B;
  a.N = N;
  a.Hq = Hq;
  a.Hkv = kv->Hkv;
  a.page = kv->page;
  a.page_shift = __builtin_ctz(static_cast<unsigned>(kv->page));
  a.max_pages = kv->max_pages;
  a.num_pages = kv->num_pages;
  a.ld = ld;
  a.scale_log2 = static_cast<float>(static_cast<double>(scale) * 1.4426950408889634);
  st = lay_out(a, cap, kv->d, scratch, scratch_bytes, true);
  if (st != SRT_OK) return st;
  a.tree_room = N;

  const int cus = cu_count();
  if (cus <= 0) return SRT_ERR_HIP;
  const int64_t rows = a.part_rows;
  const bool narrow = a.total > cus && half_waves(static_cast<int64_t>(B) * kv->Hkv, rows) &&
                      (rows <= 32 || a.chunk <= kChunk / 2);
  const int places = narrow ? cus * (kWaves / kNarrowWaves) : cus;  // workgroups that run at once
  hipStream_t s = as_stream(stream);
  // Every item runs at once, or all are short: nothing to order or hand out.
  const bool direct = a.total <= places || (narrow && a.S == 1 && cap * 2 * kv->d <= kUnlisted);
  const unsigned grid = static_cast<unsigned>(direct ? a.total : std::min<int64_t>(a.total, places));
  if (!direct) tree_attn_plan_kernel<<<1, 1024, 0, s>>>(a);
  const bool e4m3 = kv->kv_type == SRT_KV_E4M3;
  if (kv->d == 128) {
    if (e4m3) launch_quant<128, SRT_KV_E4M3>(a, narrow, direct, grid, s);
    else launch_quant<128, SRT_KV_INT8>(a, narrow, direct, grid, s);
  } else {
    if (e4m3) launch_quant<64, SRT_KV_E4M3>(a, narrow, direct, grid, s);
    else launch_quant<64, SRT_KV_INT8>(a, narrow, direct, grid, s);
  }
  if (a.S > 1) launch_combine(a, kv->d, direct, static_cast<unsigned>(combine_grid(a, cus)), s);
  return launch_status();
}
