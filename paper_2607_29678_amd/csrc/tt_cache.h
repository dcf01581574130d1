// What the calls on a paged cache share: its checks, and vectors of 16 bytes.
#pragma once

#include "tt_scores.h"

namespace tt {

template <class T>
using Vec8 = T __attribute__((ext_vector_type(8)));

// TT_ERR_BAD_ARG for sizes that do not fit, TT_ERR_NULL_ARG for missing tensors.
inline int check_cache(const tt_cache& c) {
  auto in_vectors = [](int64_t n) { return n >= 0 && n % 8 == 0; };
  if ((c.type != TT_BF16 && c.type != TT_F16) || c.page_size < 1 || c.kv_heads < 1 || c.dim < 8 || c.dim > TT_MAX_HEAD_DIM ||
      c.dim % 8 || c.pages < 0 || c.pages > INT32_MAX || !in_vectors(c.page_stride) || !in_vectors(c.slot_stride) ||
      !in_vectors(c.head_stride) || (reinterpret_cast<uintptr_t>(c.keys) | reinterpret_cast<uintptr_t>(c.values)) % 16)
    return TT_ERR_BAD_ARG;
  return c.pages > 0 && (!c.keys || !c.values) ? TT_ERR_NULL_ARG : TT_OK;
}

}  // namespace tt
