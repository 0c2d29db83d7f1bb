// C entry points of the paged key/value cache (declared in
// include/ce_router_paged.h): host validation, then the launches.
#include <hip/hip_runtime.h>
#include <math.h>

#include "ce_host.hpp"
#include "ce_paged.hpp"

using namespace ce;

namespace {

inline int hip_status(hipError_t e) { return e == hipSuccess ? CE_OK : CE_ERR_HIP; }

int log2_of_page(int page) {
  int l = 0;
  while ((1 << l) < page) ++l;
  return l;
}

// What the page table's calls read of a cache.
int check_table(const ce_kv_cache* c) {
  if (!c || c->B < 1 || c->page_size < 1 || c->n_pages < 1 || c->max_pages < 1) return CE_ERR_INVALID_ARG;
  if (c->B > 65535 || c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
    return CE_ERR_UNSUPPORTED;
  const int64_t lim = (int64_t)1 << 31;
  if ((int64_t)c->n_pages * c->page_size >= lim || (int64_t)c->max_pages * c->page_size > lim / 2)
    return CE_ERR_UNSUPPORTED;
  return CE_OK;
}

// And what the calls on its pages read.
int check_pages(const ce_kv_cache* c) {
  const int s = check_table(c);
  if (s != CE_OK) return s;
  if (c->n_kv_heads < 1) return CE_ERR_INVALID_ARG;
  if (c->head_dim != 128 || (c->dtype != CE_BF16 && c->dtype != CE_E4M3)) return CE_ERR_UNSUPPORTED;
  const int64_t page = (int64_t)c->n_kv_heads * c->page_size * 128;
  if (c->page_stride < page || c->page_stride % 16 != 0) return CE_ERR_INVALID_ARG;
  if (c->page_stride >= (int64_t)1 << 31 || c->n_kv_heads >= 1 << 16) return CE_ERR_UNSUPPORTED;
  if (!c->k_scale != !c->v_scale || (c->dtype == CE_BF16 && c->k_scale)) return CE_ERR_INVALID_ARG;
  return CE_OK;
}

// Sizes of an attention call.
int check_attn(const ce_kv_cache* c, const ce_paged_attn* at) {
  const int s = check_pages(c);
  if (s != CE_OK) return s;
  if (!at || at->n_heads < 1 || at->n_heads % c->n_kv_heads != 0 || at->q_capacity < 0) return CE_ERR_INVALID_ARG;
  if (at->n_heads / c->n_kv_heads > 4096) return CE_ERR_UNSUPPORTED;
  if (at->causal != 0 && at->causal != 1) return CE_ERR_INVALID_ARG;
  if (!(at->scale > 0.0f) || !isfinite(at->scale * 1.4426950408889634f)) return CE_ERR_INVALID_ARG;
  if ((int64_t)at->q_capacity * at->n_heads >= (int64_t)1 << 28 || (int64_t)c->B * c->n_kv_heads >= (int64_t)1 << 22)
    return CE_ERR_UNSUPPORTED;
  return CE_OK;
}

PagedGrid grid_of(const ce_kv_cache* c, const ce_paged_attn* at) {
  return paged_grid(c->B, at->n_heads, c->n_kv_heads, at->q_capacity, (int64_t)c->max_pages * c->page_size);
}

}  // namespace

extern "C" {

int ce_kv_reserve(const ce_kv_cache* cache, const int32_t* lens, const int32_t* new_offsets, int32_t row_capacity,
                  const uint8_t* reset, int32_t* free_pages, const int32_t* free_count, int32_t* lens_out,
                  int32_t* free_count_out, int32_t* start, int32_t* slots, uint32_t* status, void* stream) {
  const int s = check_table(cache);
  if (s != CE_OK) return s;
  if (row_capacity < 0 || (!new_offsets && row_capacity != 0)) return CE_ERR_INVALID_ARG;
  if (!cache->page_table || !lens || !free_pages || !free_count || !lens_out || !free_count_out || !start ||
      (row_capacity > 0 && !slots))
    return CE_ERR_INVALID_ARG;
  ReserveArgs a = {};
  a.B = cache->B;
  a.max_pages = cache->max_pages;
  a.n_pages = cache->n_pages;
  a.page_log2 = log2_of_page(cache->page_size);
  a.rows = row_capacity;
  a.lens = lens;
  a.offs = new_offsets;
  a.reset = reset;
  a.table = cache->page_table;
  a.free_pages = free_pages;
  a.count = free_count;
  a.lens_out = lens_out;
  a.count_out = free_count_out;
  a.start = start;
  a.slots = slots;
  a.status = status;
  return hip_status(launch_kv_reserve(a, static_cast<hipStream_t>(stream)));
}

int ce_kv_append(const ce_kv_cache* cache, const void* k_new, int64_t k_ld, const void* v_new, int64_t v_ld,
                 const int32_t* slots, int32_t rows, void* stream) {
  const int s = check_pages(cache);
  if (s != CE_OK) return s;
  if (rows < 0) return CE_ERR_INVALID_ARG;
  const int64_t row = (int64_t)cache->n_kv_heads * 128;
  if (k_ld < row || v_ld < row || k_ld % 8 != 0 || v_ld % 8 != 0) return CE_ERR_INVALID_ARG;
  if (k_ld >= (int64_t)1 << 31 || v_ld >= (int64_t)1 << 31) return CE_ERR_UNSUPPORTED;
  if (rows > 0 && (!k_new || !v_new || !slots || !cache->k || !cache->v)) return CE_ERR_INVALID_ARG;
  const int elem = cache->dtype == CE_E4M3 ? 1 : 2;
  AppendArgs a = {};
  a.k_new = static_cast<const char*>(k_new);
  a.v_new = static_cast<const char*>(v_new);
  a.k_ld = k_ld * 2;
  a.v_ld = v_ld * 2;
  a.slots = slots;
  a.rows = rows;
  a.Hkv = cache->n_kv_heads;
  a.n_slots = cache->n_pages * cache->page_size;
  a.page_log2 = log2_of_page(cache->page_size);
  a.k = static_cast<char*>(cache->k);
  a.v = static_cast<char*>(cache->v);
  a.page_bytes = (uint32_t)(cache->page_stride * elem);
  a.k_scale = cache->k_scale;
  a.v_scale = cache->v_scale;
  return hip_status(launch_kv_append(a, cache->dtype == CE_E4M3, static_cast<hipStream_t>(stream)));
}

size_t ce_paged_workspace_size(const ce_kv_cache* cache, const ce_paged_attn* attn) {
  return check_attn(cache, attn) == CE_OK ? grid_of(cache, attn).bytes : 0;
}

int ce_paged_attention(const ce_kv_cache* cache, const ce_paged_attn* attn, const void* q, int64_t q_ld, void* o,
                       void* ws, size_t ws_bytes, void* stream) {
  const int s = check_attn(cache, attn);
  if (s != CE_OK) return s;
  if (q_ld < (int64_t)attn->n_heads * 128 || q_ld % 8 != 0) return CE_ERR_INVALID_ARG;
  if (q_ld >= (int64_t)1 << 22) return CE_ERR_UNSUPPORTED;
  if (!attn->q_offsets || !attn->lens) return CE_ERR_INVALID_ARG;
  if (attn->q_capacity > 0 && (!q || !o || !cache->k || !cache->v || !cache->page_table)) return CE_ERR_INVALID_ARG;
  const PagedGrid p = grid_of(cache, attn);
  if (p.bytes > 0) {
    const int e = check_ws(ws, ws_bytes, p.bytes);
    if (e != CE_OK) return e;
  }
  const int elem = cache->dtype == CE_E4M3 ? 1 : 2;
  PagedArgs a = {};
  a.q = static_cast<const char*>(q);
  a.o = static_cast<char*>(o);
  a.k = static_cast<const char*>(cache->k);
  a.v = static_cast<const char*>(cache->v);
  a.ks = cache->k_scale;
  a.vs = cache->v_scale;
  a.table = cache->page_table;
  a.qo = attn->q_offsets;
  a.lens = attn->lens;
  a.q_ld = q_ld * 2;
  a.page_bytes = (uint32_t)(cache->page_stride * elem);
  a.B = cache->B;
  a.H = attn->n_heads;
  a.Hkv = cache->n_kv_heads;
  a.g = a.H / a.Hkv;
  a.q_cap = attn->q_capacity;
  a.n_pages = cache->n_pages;
  a.max_pages = cache->max_pages;
  a.page_log2 = log2_of_page(cache->page_size);
  a.causal = attn->causal;
  a.scale_log2 = attn->scale * 1.4426950408889634f;
  char* const w = static_cast<char*>(ws);
  a.plan = reinterpret_cast<PagedPlan*>(w);
  a.arrived = reinterpret_cast<unsigned long long*>(w + p.plan_bytes);
  a.units = p.cut_units ? reinterpret_cast<uint32_t*>(w + p.plan_bytes) : nullptr;
  a.part = reinterpret_cast<float*>(w + p.plan_bytes + p.count_bytes);
  return hip_status(launch_paged_attention(a, cache->dtype == CE_E4M3, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
