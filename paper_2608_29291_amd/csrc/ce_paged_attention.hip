// Attention of new tokens over a paged key/value cache (paper section 3.4: the
// packed keys and values of a routed layer are the compressed cache that
// decoding reuses), include/ce_router_paged.h:
//
//   O_b[:, h] = softmax(scale Q_b[:, h] K_b[:, kv(h)]^T + M) V_b[:, kv(h)]
//
// with the keys and values of sequence b in the pages that its row of the page
// table names. Any batch: one token a sequence, chunks of prompts, both.
//
// Rows. The g = H / H_kv query heads of a key/value head read the same keys, so
// row r of a sequence and key/value head is query r / g, head r % g, and the rows
// are cut into tiles: one of up to 32 rows for a sequence that has no more
// (paged_few: 4 waves share the keys), else tiles of 128 (paged_tile: 4 waves share
// the rows). Grouped rows waste less than one tile per query head: 551 queries of
// six heads are 26 tiles, not 30, and the tile's causal edge is g times as steep.
//
// Keys. Tiles are cut along their keys, too, where they leave places on the chip idle
// (the plan: ce_paged_tile.hpp). Every wave forms the plan by itself from the
// lengths, which only the device knows: a lane per sequence, or per four, and a few
// prefix sums; more than 256 sequences are planned by a launch of their own. The
// chunks of a cut tile meet through the workspace, where the last to arrive adds them
// up in order, so one launch does it all and no result depends on which
// workgroup came first.
//
// A key that a query does not see has no influence: its score is replaced before
// the maximum, and rows of a page behind the sequence's end read as zeros. What
// the products cannot hide, a NaN or infinity among the values under a weight of
// zero, shows as NaN in the output: a wave whose keys the causal mask cuts looks
// for it at its end and forms that output again, key by key (paged_redo).
#include <atomic>

#include "ce_device.hpp"
#include "ce_host.hpp"
#include "ce_paged.hpp"
#include "ce_paged_tile.hpp"

namespace ce {

namespace {

using namespace paged;

template <bool kF8>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_attention_kernel(PagedArgs a,
                                                                                                        int group) {
  __shared__ __attribute__((aligned(1024))) char smem[kSmem];
  // Workgroup w runs on XCD w % 8: an XCD takes `group` neighbouring items at a
  // time, whose tiles of one sequence and head find each other's keys in its L2.
  const int w = blockIdx.x;
  const int in_xcd = w / kXcdCount;
  const uint32_t at = (in_xcd / group) * (kXcdCount * group) + (w % kXcdCount) * group + in_xcd % group;
  Item it;
  if (!find_item(a, at, it)) return;
  if (it.few)
    paged_few<kF8>(a, smem, it);
  else
    paged_tile<kF8>(a, smem, it);
}

// The plan of more than kPagedScan sequences. One workgroup.
__global__ __launch_bounds__(1024) void paged_plan_kernel(PagedArgs a) {
  __shared__ int64_t scr[16];
  __shared__ float wsum[16];
  __shared__ int wmax[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = a.H / a.Hkv;
  // exclusive prefix sum over the threads, and the total
  auto scan = [&](int64_t v, int64_t& total) {
    int64_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t y = __shfl_up(x, o);
      if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) scr[wave] = x;
    __syncthreads();
    int64_t before = 0;
    total = 0;
    for (int i = 0; i < 16; ++i) {
      if (i < wave) before += scr[i];
      total += scr[i];
    }
    return before + x - v;
  };
  auto sum = [&](float v) {
    v = wave_sum(v);
    __syncthreads();
    if (lane == 0) wsum[wave] = v;
    __syncthreads();
    float s = 0.0f;
    for (int i = 0; i < 16; ++i) s += wsum[i];
    return s;
  };
  float w = 0.0f;
  int longest = 0;
  int64_t units = 0, total;
  for (int b = tid; b < a.B; b += 1024) {
    const Size s = size_of(a, b, g);
    const uint32_t n = (uint32_t)s.tiles * a.Hkv;
    w += (float)n * (float)s.nk;
    units += n;
    longest = max(longest, n ? s.nk : 0);
  }
  w = sum(w);
  longest = wave_max(longest);
  if (lane == 0) wmax[wave] = longest;
  scan(units, total);  // (its barriers stand between)
  for (int i = 0; i < 16; ++i) longest = max(longest, wmax[i]);
  uint32_t whole = whole_units((uint32_t)min(total, (int64_t)1 << 30), w, longest);
  // the units before each sequence, and the rest's keys
  float rest = 0.0f;
  int64_t base = 0;
  for (int b0 = 0; b0 < a.B; b0 += 1024) {
    const int b = b0 + tid;
    Size s = {0, 0, 0, 0};
    if (b < a.B) s = size_of(a, b, g);
    const uint32_t n = (uint32_t)s.tiles * a.Hkv;
    const int64_t first = base + scan(n, total);
    const uint32_t wh = whole_of(a, s, (uint32_t)min(first, (int64_t)1 << 30), whole);
    rest += (float)(n - wh) * (float)s.nk;
    if (b < a.B) a.plan[b].whole = wh;
    base += total;
  }
  if (whole) w = sum(rest);
  int L = chunk_length(w);
  for (;;) {
    int64_t items = 0, slots = 0;
    for (int b0 = 0; b0 < a.B; b0 += 1024) {
      const int b = b0 + tid;
      uint32_t ni = 0, ns = 0;
      if (b < a.B) counts_of(a, size_of(a, b, g), g, L, a.plan[b].whole, ni, ns);
      const int64_t i0 = items + scan(ni, total);
      items += total;
      const int64_t s0 = slots + scan(ns, total);
      slots += total;
      if (b < a.B) {
        a.plan[b].items = (uint32_t)min(i0, (int64_t)1 << 30);
        a.plan[b].slots = (uint32_t)min(s0, (int64_t)1 << 30);
      }
    }
    if (tid == 0) {
      a.plan[a.B].items = (uint32_t)min(items, (int64_t)1 << 30);
      a.plan[a.B].whole = (uint32_t)L;
    }
    // (as in find_by_scan)
    if (L == 1 << 30 || (items <= a.grid && slots <= kPagedTarget)) break;
    L = 1 << 30;
  }
}

}  // namespace

// A token that no earlier call of the process had and that memory is unlikely to
// hold by chance: a counter through a mix of its bits (a bijection), 48 bits of it, not 0.
static uint64_t paged_token() {
  static std::atomic<uint64_t> calls{0};
  uint64_t x = (calls.fetch_add(1, std::memory_order_relaxed) + 1) * 0x9e3779b97f4a7c15ull;
  x ^= x >> 31;
  x *= 0xd6e8feb86659fd93ull;
  x ^= x >> 32;
  x &= (1ull << 48) - 1;
  return x ? x : 1;
}

PagedGrid paged_grid(int B, int H, int Hkv, int q_cap, int64_t max_keys) {
  PagedGrid p = {};
  if (q_cap <= 0) return p;
  // every sequence with a query adds at most one tile that is not full
  p.items = ((int64_t)q_cap * (H / Hkv) / kPagedRows + (B < q_cap ? B : q_cap)) * Hkv;
  if (B > kPagedScan) p.plan_bytes = ((size_t)(B + 1) * sizeof(PagedPlan) + 255) / 256 * 256;
  p.bytes = p.plan_bytes;
  if (max_keys >= 2 * kMinChunk) {  // else nothing is cut
    p.items += kPagedTarget;
    p.count_bytes = (size_t)kPagedLevels * kPagedTarget * sizeof(unsigned long long);
    p.bytes += p.count_bytes + (size_t)kPagedTarget * kPagedPart * sizeof(float);
  }
  return p;
}

hipError_t launch_paged_attention(PagedArgs a, bool e4m3, hipStream_t stream) {
  if (a.q_cap <= 0) return hipSuccess;
  const PagedGrid p = paged_grid(a.B, a.H, a.Hkv, a.q_cap, (int64_t)a.max_pages << a.page_log2);
  // Items of one tile a sequence share no keys; others in groups of neighbours.
  const int group = (int64_t)a.q_cap * (a.H / a.Hkv) <= (int64_t)kFew * a.B ? 1 : 16;
  const int64_t unit = (int64_t)kXcdCount * group;
  const int64_t grid = (p.items + unit - 1) / unit * unit;
  a.grid = (uint32_t)grid;
  a.token = paged_token();
  if (a.B > kPagedScan) {
    hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(1024), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (e4m3)
    hipLaunchKernelGGL(paged_attention_kernel<true>, dim3((unsigned)grid), dim3(256), 0, stream, a, group);
  else
    hipLaunchKernelGGL(paged_attention_kernel<false>, dim3((unsigned)grid), dim3(256), 0, stream, a, group);
  return hipGetLastError();
}

}  // namespace ce
