// The paged key/value cache between its C entry points and its kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ce_router_paged.h"

namespace ce {

struct ReserveArgs {
  int B, max_pages, n_pages, page_log2, rows;
  const int32_t* lens;
  const int32_t* offs;   // or NULL
  const uint8_t* reset;  // or NULL
  int32_t* table;
  int32_t* free_pages;
  const int32_t* count;
  int32_t* lens_out;
  int32_t* count_out;
  int32_t* start;
  int32_t* slots;
  uint32_t* status;  // or NULL
  int slots_apart;   // the slots come from a launch of their own
};

struct AppendArgs {
  const char *k_new, *v_new;
  int64_t k_ld, v_ld;  // bytes between rows
  const int32_t* slots;
  int rows, Hkv, n_slots, page_log2, rows_per_block;
  char *k, *v;
  uint32_t page_bytes;  // between pages
  const float *k_scale, *v_scale;
};

// Items, partial results and cut units of the sequences before one, and its units
// that are not cut.
struct PagedPlan {
  uint32_t items, slots, cut, whole;
};

struct PagedArgs {
  const char* q;
  char* o;
  const char *k, *v;
  const float *ks, *vs;  // scales of 8-bit pages, or NULL
  const int32_t *table, *qo, *lens;
  int64_t q_ld;        // bytes between rows of q
  uint32_t page_bytes;  // bytes between pages
  int B, H, Hkv, g, q_cap, n_pages, max_pages, page_log2, causal;
  float scale_log2;  // scale * log2(e)
  int decode;        // a call of single tokens (the plan: ce_paged_tile.hpp)
  uint32_t grid;     // items that the launch has workgroups for
  float* part;       // partial results, a slot for each place
  unsigned long long* arrived;  // single tokens: counters of the chunks that meet, kPagedPlaces a level
  uint32_t* units;   // else the number of cut units and a record of each, or NULL: none is cut
  unsigned long long token;     // of this call, 48 bits
  PagedPlan* plan;   // B > kPagedScan: the sequences, then the items, (whole) the chunk length and (slots) if half of the places are filled
};

constexpr int kPagedScan = 256;    // sequences that a wave plans by itself (four a lane)
constexpr int kPagedFew = 32;     // (query, head) rows of a tile of single tokens
constexpr int kPagedTile = 128;   // and of one of many rows
constexpr int kPagedPlaces = 512; // places for workgroups: two on each CU
constexpr int kPagedRecord = 32;  // bytes of a cut unit's record
constexpr int kPagedLevels = 3;    // sixteen chunks meet at a time, 512 at most

// What the host knows of a call: the workgroups that any batch of these sizes needs.
struct PagedGrid {
  int64_t items;
  int decode;
  int cut_units;  // for the launch that adds chunks up, at most (0: no such launch)
  size_t plan_bytes, count_bytes, bytes;  // workspace: the plan, counters or records, partial results
};
PagedGrid paged_grid(int B, int H, int Hkv, int q_cap, int64_t max_keys);

hipError_t launch_kv_reserve(ReserveArgs a, hipStream_t stream);
hipError_t launch_kv_append(AppendArgs a, bool e4m3, hipStream_t stream);
hipError_t launch_paged_attention(PagedArgs a, bool e4m3, hipStream_t stream);

}  // namespace ce
