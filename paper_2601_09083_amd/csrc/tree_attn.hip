// Tree-masked attention over a paged bf16 KV cache (MFMA, gfx950).
//
// Method: Section 3 of the paper -- one decode pass of the policy verifies
// every drafted token -- and Appendix C (verification reads the KV cache
// once for all candidates).  Tree node i of sequence b attends to the whole
// committed context [0, L) and to the tree positions L + j of its
// ancestors-or-self j; query head h uses KV head h / (Hq / Hkv).
//
// GPU design.  For one (sequence, KV head) all n * G query rows (G query
// heads per KV head) share every K/V tile, so they are processed together:
// a workgroup of 8 waves owns 256 rows (32 per wave) and streams one split
// of the key range in 64-key tiles; one workgroup per CU.
//   * Products run on v_mfma_f32_32x32x16_bf16 (the full-rate bf16 shape on
//     gfx950) with fp32 accumulation: S^T = K Q^T (32 keys x 32 rows per
//     MFMA) and O^T = V^T P^T (32 head dims x 32 rows).  In this orientation
//     a query row lives in one lane column of both accumulators, so the
//     online-softmax statistics and the rescale of O are lane-local (the
//     two lane halves are merged with one permlane32 swap) and P feeds the
//     second MFMA straight from registers: the contraction index of P^T is
//     permuted to match the S^T output layout, and V^T is read with the same
//     permutation by ds_read_b64_tr_b16 transposing reads.  The head-dim
//     order inside each 32-row block of O^T is permuted too (lane halves of
//     a transposing read take head dims D/2 apart), which the epilogue undoes.
//   * K and V tiles are read from HBM with 16-byte buffer loads (one scalar
//     descriptor per 8-key sub-block of a page, so tails read as zero),
//     prefetched into registers one tile ahead and stored to double-buffered
//     LDS.  LDS rows are padded (K by 16 bytes, V by 32) so that the operand
//     reads of every MFMA are bank-conflict free and their addresses are one
//     base register plus immediate offsets.
//   * Softmax uses exp2 of fma(q.k, scale*log2(e), -reference) (Q is never
//     rescaled or re-rounded) and a lazily raised reference maximum; a tile
//     whose probabilities all stay below 2^8 of the reference (checked on
//     their sum) needs no row maximum at all.  The ancestor mask is a bitset per tree node in LDS;
//     on tiles that reach the tree positions or the end of the range each
//     row takes a 64-bit visibility window of it (two LDS words) and masks
//     its scores bit by bit.
//   * Long contexts are split into chunks of keys so the grid has enough
//     independent work (8192 keys, or a smaller power of two down to 1024
//     when the batch has few sequences and KV heads, 512 or 256 when every
//     item that the block table has room for gets a CU of its own); each
//     split writes unnormalised partial output plus (max, sum) and a small
//     combine kernel merges them.  A sequence that fits in one split writes
//     bf16 output directly.
//   * Work is scheduled by a small plan kernel that lists the (sequence, KV
//     head, split, row block) items that have work, longest first; one
//     persistent workgroup per CU takes items from an atomic counter, so no
//     CU idles on empty grid slots and long items do not form a tail.  Where
//     the block table has room for no more items than there are CUs, each
//     has a workgroup and there is no plan kernel.
#include "attn_bf16.h"

namespace {

void launch_main(const AttnArgs& a, int d, bool direct, unsigned grid, hipStream_t s) {
  if (d == 128) {
    if (direct) tree_attn_kernel<128, true, AttnArgs><<<grid, kThreads, 0, s>>>(a);
    else tree_attn_kernel<128, false, AttnArgs><<<grid, kThreads, 0, s>>>(a);
  } else {
    if (direct) tree_attn_kernel<64, true, AttnArgs><<<grid, kThreads, 0, s>>>(a);
    else tree_attn_kernel<64, false, AttnArgs><<<grid, kThreads, 0, s>>>(a);
  }
}

}  // namespace

extern "C" size_t srt_tree_attn_scratch_bytes(int32_t B, int32_t N, int32_t Hq, int32_t Hkv, int32_t d, int32_t page,
                                              int32_t max_pages) {
  if (B < 0 || N < 1 || N > kMaxN || Hq < 1 || Hkv < 1 || Hq % Hkv || page < 1 || max_pages < 1) return 0;
  const int64_t RB = (N * (Hq / Hkv) + kRowsPerBlock - 1) / kRowsPerBlock;
  const int64_t cap = static_cast<int64_t>(page) * max_pages;
  return scratch_for(B, N, Hq, Hkv, d, cap, chunk_for(B, Hkv, RB, cap, true, 0), false);
}

extern "C" int srt_tree_attn(int32_t B, int32_t N, int32_t Hq, int32_t Hkv, int32_t d, int32_t page,
                             int32_t max_pages, int64_t num_pages, const uint16_t* q, const uint16_t* k_cache,
                             const uint16_t* v_cache, const int32_t* block_table, const int32_t* ctx_len,
                             const int32_t* tree_parent, const int32_t* n_nodes, float scale, uint16_t* out,
                             void* scratch, size_t scratch_bytes, void* stream) {
  if (B < 0 || N < 1 || N > kMaxN || Hq < 1 || Hkv < 1 || Hq % Hkv || page < 1 || max_pages < 1 || num_pages < 1)
    return SRT_ERR_INVALID;
  if (!std::isfinite(scale)) return SRT_ERR_INVALID;
  if (d != 64 && d != 128) return SRT_ERR_UNSUPPORTED;
  if (page < 16 || (page & (page - 1))) return SRT_ERR_UNSUPPORTED;
  const int64_t cap = static_cast<int64_t>(page) * max_pages;
  if (!packs(B, N, Hq, Hkv, cap, false)) return SRT_ERR_UNSUPPORTED;
  if (B == 0) return SRT_OK;
  if (!q || !k_cache || !v_cache || !block_table || !ctx_len || !tree_parent || !n_nodes || !out)
    return SRT_ERR_INVALID;

  AttnArgs a;
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
  a.page = page;
  a.page_shift = __builtin_ctz(static_cast<unsigned>(page));
  a.max_pages = max_pages;
  a.num_pages = num_pages;
  a.scale_log2 = static_cast<float>(static_cast<double>(scale) * 1.4426950408889634);
  const int st = lay_out(a, cap, d, scratch, scratch_bytes, false);
  if (st != SRT_OK) return st;
  a.tree_room = 0;

  const int cus = cu_count();
  if (cus <= 0) return SRT_ERR_HIP;
  const unsigned grid = static_cast<unsigned>(std::min<int64_t>(a.total, cus));
  hipStream_t s = as_stream(stream);
  // Where every item that the batch can have gets a CU of its own there is
  // nothing to order or hand out: no plan kernel, one launch less (16
  // sequences of up to 400 keys, 8-node trees, 28 heads: 17.3 -> 13.2 us).
  const bool direct = a.total <= cus;
  if (!direct) tree_attn_plan_kernel<<<1, 1024, 0, s>>>(a);
  launch_main(a, d, direct, grid, s);
  if (a.S > 1) launch_combine(a, d, direct, static_cast<unsigned>(combine_grid(a, cus)), s);
  return launch_status();
}
