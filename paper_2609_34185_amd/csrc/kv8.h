// What the sources of the paged 8-bit key/value cache share.
#pragma once
#include <cstdint>

#include "../../include/entropack.h"

namespace ep {

// log2 of a page's tokens, or -1 if that is no size of a page.
inline int page_shift(int page_tokens) {
  for (int s = 4; s <= 8; s++)
    if (page_tokens == 1 << s) return s;
  return -1;
}

// What is wrong with a cache description, or null.
inline const char* cache_fault(const ep_kv8_cache* c) {
  if (!c) return "null cache";
  if (page_shift(c->page_tokens) < 0) return "page_tokens must be 16, 32, 64, 128 or 256";
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return "head_dim must be 64, 128 or 256";
  if (c->dtype != EP_FP8_E4M3 && c->dtype != EP_INT8) return "the cache's dtype must be FP8_E4M3 or INT8";
  if (c->kv_heads <= 0 || c->kv_heads > 1 << 16) return "kv_heads outside 1 .. 65536";
  if (c->n_pages <= 0) return "n_pages must be positive";
  if (c->n_pages > (1 << 30) / c->kv_heads) return "n_pages * kv_heads above 2^30";
  if (!c->d_k || !c->d_v || !c->d_k_scale || !c->d_v_scale) return "null array of the cache";
  if ((reinterpret_cast<uintptr_t>(c->d_k) | reinterpret_cast<uintptr_t>(c->d_v)) & 15)
    return "codes must be 16-byte aligned";
  return nullptr;
}

}  // namespace ep
