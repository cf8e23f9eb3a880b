// Host checks of the 8-bit KV cache that its entry points share.
#pragma once

#include "common.h"

namespace srt {

inline int check_kv_sizes(const srt_kv_quant& kv) {
  if (kv.kv_type != SRT_KV_E4M3 && kv.kv_type != SRT_KV_INT8) return SRT_ERR_INVALID;
  if (kv.Hkv < 1 || kv.page < 1 || kv.max_pages < 1 || kv.num_pages < 1 || kv.reserved != 0) return SRT_ERR_INVALID;
  if (kv.Hkv > 255 || (kv.d != 64 && kv.d != 128)) return SRT_ERR_UNSUPPORTED;
  if (kv.page < 16 || kv.page > 256 || (kv.page & (kv.page - 1))) return SRT_ERR_UNSUPPORTED;
  // positions stay below 2^30
  if (static_cast<int64_t>(kv.max_pages) * kv.page > (int64_t(1) << 30) - 1024) return SRT_ERR_UNSUPPORTED;
  return SRT_OK;
}

inline int check_kv_pointers(const srt_kv_quant& kv) {
  if (!kv.k_pages || !kv.v_pages || !kv.k_scale || !kv.v_scale || !kv.k_tail || !kv.v_tail || !kv.block_table ||
      !kv.ctx_len)
    return SRT_ERR_INVALID;
  const uintptr_t all = reinterpret_cast<uintptr_t>(kv.k_pages) | reinterpret_cast<uintptr_t>(kv.v_pages) |
                        reinterpret_cast<uintptr_t>(kv.k_tail) | reinterpret_cast<uintptr_t>(kv.v_tail);
  return all % 16 ? SRT_ERR_INVALID : SRT_OK;
}

// New vectors: rows of a token's KV heads, ld elements apart.
inline int check_new(const srt_kv_quant& kv, const uint16_t* k_new, const uint16_t* v_new, int64_t ld) {
  if (!k_new || !v_new || ld < static_cast<int64_t>(kv.Hkv) * kv.d || ld % 8 || ld > (int64_t(1) << 31))
    return SRT_ERR_INVALID;
  return (reinterpret_cast<uintptr_t>(k_new) | reinterpret_cast<uintptr_t>(v_new)) % 16 ? SRT_ERR_INVALID : SRT_OK;
}

}  // namespace srt
