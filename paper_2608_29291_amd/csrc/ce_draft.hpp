// Drafted decoding between its C entry points and its kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ce_router_draft.h"

namespace ce {

struct DraftMaskArgs {
  int B, rows, words;
  int staged;              // rows that LDS holds
  const int32_t* offs;
  const int32_t* parents;  // or NULL: chains
  const int32_t* base;     // or NULL
  uint32_t* mask;          // or NULL
  int32_t* positions;      // or NULL
  uint32_t* status;        // or NULL
};

struct KeepArgs {
  int B, rows, heads, row_bytes, n_pages, max_pages, page_log2;  // row_bytes: of a row of a head
  uint32_t page_bytes;                                            // between pages
  const int32_t *offs, *start, *kept, *n_kept, *table;
  char *k, *v;
};

struct TrimArgs {
  int B, max_pages, n_pages, page_log2;
  const int32_t *lens, *start, *n_kept, *table;
  int32_t* free_pages;
  const int32_t* count;
  int32_t* lens_out;
  int32_t* count_out;
  uint32_t* status;  // or NULL
};

hipError_t launch_draft_masks(DraftMaskArgs a, hipStream_t stream);
hipError_t launch_kv_keep(const KeepArgs& a, hipStream_t stream);
hipError_t launch_kv_trim(const TrimArgs& a, hipStream_t stream);

// Sizes of a step's trees.
inline int check_drafts(const ce_drafts* d) {
  if (!d || d->B < 1 || d->row_capacity < 0) return CE_ERR_INVALID_ARG;
  if (d->B > 65535 || d->row_capacity >= 1 << 24) return CE_ERR_UNSUPPORTED;
  return CE_OK;
}

}  // namespace ce
