// What the paged cache's translation units share on the host: checks of a df_paged_cache.
#pragma once

#include "df_internal.h"
#include "df_paged_walk.h"

namespace df {

inline int log2_of(int x) {
  int n = 0;
  while ((1 << n) < x) ++n;
  return n;
}

inline df_status check_paged_cache(const df_paged_cache *c) {
  if (!c) return DF_ERR_NULL;
  if (c->B <= 0 || c->H_kv <= 0 || c->n_pages <= 0 || c->max_pages <= 0 || c->page_tokens <= 0) return DF_ERR_SHAPE;
  if (c->H_kv > kMaxHeads || (c->d != 64 && c->d != 128) || (c->dtype != DF_BF16 && c->dtype != DF_FP16)) return DF_ERR_UNSUPPORTED;
  if (c->page_tokens < 16 || c->page_tokens > 1024 || (c->page_tokens & (c->page_tokens - 1))) return DF_ERR_UNSUPPORTED;
  if (c->B > (1 << 16) || c->max_pages > kMaxLen || int64_t(c->n_pages) * c->page_tokens > INT32_MAX) return DF_ERR_RANGE;
  if (!c->k_pages || !c->v_pages || !c->block_table || !c->len || !c->sink_cap || !c->win_cap) return DF_ERR_NULL;
  if (!aligned16(c->k_pages) || !aligned16(c->v_pages)) return DF_ERR_ALIGN;
  if (c->cap_stride != 0 && c->cap_stride < c->H_kv) return DF_ERR_SHAPE;
  return DF_OK;
}

}  // namespace df
