// paged.cuh -- device access to the paged key-value cache: what is read from device memory as an index is
// checked before it is followed.
#pragma once

#include "../../include/ringada.h"
#include "common.cuh"

namespace ra {

// a sequence's length within [0, most]
__device__ __forceinline__ int clamp_len(int len, int most, uint32_t* err) {
  if (len < 0 || len > most) {
    set_dev_error(err, RA_DEVERR_BOUNDS);
    len = len < 0 ? 0 : most;
  }
  return len;
}
// Row of key-value head `head` at slot `slot` (within the table) of sequence b, in rows of head_dim values from the
// pools' start; -1 for a page that is none
__device__ __forceinline__ int64_t slot_row(const ra_kv_cache& c, int b, int slot, int head) {
  const int p = slot / c.page_size;
  const int page = c.block_table_dev[(int64_t)b * c.max_pages + p];
  if ((uint32_t)page >= (uint32_t)c.n_pages) {
    set_dev_error(c.err_dev, RA_DEVERR_BOUNDS);
    return -1;
  }
  return ((int64_t)page * c.n_kv_heads + head) * c.page_size + (slot - p * c.page_size);
}

}  // namespace ra
