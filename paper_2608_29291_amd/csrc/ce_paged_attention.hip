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
// A call of single tokens (no more rows than sequences, at most eight heads a key/value
// head) is a launch of its own in which all rows go 32 to a tile (paged_decode_kernel),
// with half the partial results and without the second launch.
//
// Keys. Tiles are cut along their keys, too, where they leave places on the chip idle
// (the plan: ce_paged_tile.hpp). Every wave forms the plan by itself from the
// lengths, which only the device knows: a lane per sequence, or per four, and a few
// prefix sums; more than 256 sequences are planned by a launch of their own. The
// chunks of a cut tile are added up in chunk order, so no result depends on which
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
#include "ce_paged_token.hpp"

namespace ce {

namespace {

using namespace paged;

// Workgroup w runs on XCD w % 8: an XCD takes `group` neighbouring items at a time, whose
// tiles of one sequence and head find each other's keys in its L2.
__device__ __forceinline__ uint32_t item_of(uint32_t w, uint32_t group) {
  const uint32_t in_xcd = w / kXcdCount;
  return in_xcd / group * (kXcdCount * group) + (w % kXcdCount) * group + in_xcd % group;
}

template <bool kF8, bool kTree>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_decode_kernel(PagedArgs a) {
  __shared__ __attribute__((aligned(1024))) char smem[kSmem];
  Item it;
  if (find_item<false>(a, blockIdx.x, it)) paged_few<kF8, true, kTree>(a, smem, it);
}

template <bool kF8, bool kTree>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_attention_kernel(PagedArgs a,
                                                                                                        uint32_t group) {
  __shared__ __attribute__((aligned(1024))) char smem[kSmem];
  Item it;
  if (!find_item<true>(a, item_of(blockIdx.x, group), it)) return;
  if (it.record >= 0 && it.c == 0 && threadIdx.x == 0) write_record(a, it);
  if (it.few)
    paged_few<kF8, false, kTree>(a, smem, it);
  else
    paged_tile<kF8, kTree>(a, smem, it);
}

// The plan of more than kPagedScan sequences. One workgroup.
__global__ __launch_bounds__(512) void paged_plan_kernel(PagedArgs a) {
  __shared__ int64_t scr[8];
  __shared__ float wsum[8];
  __shared__ float wmax[8];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = a.g;
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
    for (int i = 0; i < 8; ++i) {
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
    for (int i = 0; i < 8; ++i) s += wsum[i];
    return s;
  };
  float w = 0.0f, most = 0.0f;
  int64_t units = 0, total;
  for (int b = tid; b < a.B; b += 512) {
    const Size s = size_of(a, b, g);
    const uint32_t n = (uint32_t)s.tiles * a.Hkv;
    const float c = n ? cost_of(a, s, g) : 0.0f;
    w += (float)n * c;
    units += n;
    most = fmaxf(most, c);
  }
  w = sum(w);
  most = wave_max(most);
  if (lane == 0) wmax[wave] = most;
  scan(units, total);  // (its barriers stand between)
  for (int i = 0; i < 8; ++i) most = fmaxf(most, wmax[i]);
  const uint32_t whole = whole_units((uint32_t)min(total, (int64_t)1 << 30), w, most);
  // the units before each sequence, and what the rest costs
  float rest = 0.0f;
  int64_t base = 0;
  for (int b0 = 0; b0 < a.B; b0 += 512) {
    const int b = b0 + tid;
    Size s = {0, 0, 0, 0};
    if (b < a.B) s = size_of(a, b, g);
    const uint32_t n = (uint32_t)s.tiles * a.Hkv;
    const int64_t first = base + scan(n, total);
    const uint32_t wh = whole_of(a, s, (uint32_t)min(first, (int64_t)1 << 30), whole);
    rest += (float)(n - wh) * cost_of(a, s, g);
    if (b < a.B) a.plan[b].whole = wh;
    base += total;
  }
  const float w_all = w;
  const uint32_t all = (uint32_t)min(base, (int64_t)1 << 30);
  if (whole) w = sum(rest);
  int L = chunk_length(w);
  bool near = !a.decode && rounds_up(a, L);
  for (;;) {
    const bool half = a.decode && half_places(a, L, all, w_all, most);
    int64_t items = 0, slots = 0, cuts = 0;
    auto put = [](int64_t x) { return (uint32_t)min(x, (int64_t)1 << 30); };
    for (int b0 = 0; b0 < a.B; b0 += 512) {
      const int b = b0 + tid;
      Counts c = {0, 0, 0};
      if (b < a.B) c = counts_of(a, size_of(a, b, g), g, L, half, near, a.plan[b].whole);
      const int64_t i0 = items + scan(c.items, total);
      items += total;
      const int64_t s0 = slots + scan(c.slots, total);
      slots += total;
      const int64_t c0 = cuts + scan(c.cut, total);
      cuts += total;
      if (b < a.B) {
        a.plan[b].items = put(i0);
        a.plan[b].slots = put(s0);
        a.plan[b].cut = put(c0);
      }
    }
    if (tid == 0) {
      a.plan[a.B].items = put(items);
      a.plan[a.B].slots = (half ? 1 : 0) | (near ? 2 : 0);
      a.plan[a.B].whole = (uint32_t)L;
      if (a.units) *a.units = put(cuts);
    }
    // (as in find_by_scan)
    if (L == 1 << 30 || (items <= a.grid && slots <= kPagedPlaces)) break;
    if (!near) L = 1 << 30;
    near = false;
  }
}

// Partial results of the cut units, in chunk order. Bound: latency, 3 us
// for 8 x 5 rows and 6 for 512 queries over 8704 keys, whose 30 MB come from the
// caches. Workgroup (unit, y): the 32 rows y % 4 of a 128-row tile, as that wave of
// its chunks' workgroups left them (of 16 parts, a quarter of their values); of a few
// rows, eight.
template <bool kTree>
__global__ __launch_bounds__(256) void paged_combine_kernel(PagedArgs a) {
  Item it;
  read_record(a, blockIdx.x, it);  // (any content behind the last, and not used)
  if (blockIdx.x >= *a.units || it.n_chunks <= 1) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = a.g;
  const int n = it.n_chunks;
  const float c2 = score_scale(a, it.kvh);
  const float vs = a.vs ? a.vs[it.kvh] : 1.0f;
  constexpr int kPart = kSlotBytes<false> / 4;
  const float* const slot = a.part + (int64_t)it.slot * kPart;
  auto add = [&](auto n_c, auto batch_c, const float* p, int step, int r, auto out) __attribute__((always_inline)) {
    constexpr int kN = decltype(n_c)::value, kBatch = decltype(batch_c)::value;
    const float* const ps = slot + kTileRows * kDh + r;
    float m = -__builtin_inff(), l = 0.0f;
    f32x4_t x[kN];
#pragma unroll
    for (int v = 0; v < kN; ++v) x[v] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    for (int c0 = 0; c0 < n; c0 += kBatch) {
      float mc[kBatch], lc[kBatch];
      f32x4_t y[kBatch][kN];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int64_t at = (int64_t)min(c0 + i, n - 1) * kPart;
        mc[i] = ps[at];
        lc[i] = ps[at + kTileRows];
#pragma unroll
        for (int v = 0; v < kN; ++v) y[i][v] = *reinterpret_cast<const f32x4_t*>(p + at + v * step);
      }
      float m_new = m;
#pragma unroll
      for (int i = 0; i < kBatch; ++i) m_new = fmaxf(m_new, mc[i]);
      const float al = weight(m, m_new, c2);
      l *= al;
#pragma unroll
      for (int v = 0; v < kN; ++v) x[v] *= al;
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (c0 + i < n) {
          const float wi = weight(mc[i], m_new, c2);
          l = fmaf(lc[i], wi, l);
#pragma unroll
          for (int v = 0; v < kN; ++v)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[v][e] = fmaf(y[i][v][e], wi, x[v][e]);
        }
      m = m_new;
    }
    if (r >= it.rows) return;
    const int row = it.tile * tile_rows(it.few) + r;
    const int qi = row / g;
    const float inv = normalizer(l, row_sees<kTree>(a, it, qi, l));
    char* const o = a.o + ((int64_t)(it.qbase + qi) * a.H + it.kvh * g + (row - qi * g)) * kRowB;
#pragma unroll
    for (int v = 0; v < kN; ++v)
      store4<true>(o + 2 * out(v), x[v][0] * inv * vs, x[v][1] * inv * vs, x[v][2] * inv * vs, x[v][3] * inv * vs);
  };
  using One = std::integral_constant<int, 1>;
  using Four = std::integral_constant<int, 4>;
  if (it.few) {
    for (int rb = 8 * blockIdx.y; rb < it.rows; rb += 8 * gridDim.y) {
      const int r = rb + (tid >> 5), d = 4 * (tid & 31);
      const int at = min(r, it.rows - 1) * kDh + d;
      add(One{}, std::integral_constant<int, 16>{}, slot + at, 0, r, [&](int) { return d; });
    }
  } else {
    const int z = blockIdx.y & 3, r = 32 * z + (lane & 31);
    if (32 * z >= it.rows) return;
    if (gridDim.y == 4) {  // accumulators 4 wave .. +3
      add(Four{}, Four{}, slot + ((z * 16 + 4 * wave) * 64 + lane) * 4, 256, r,
          [&](int v) { return 32 * wave + 8 * v + 4 * (lane >> 5); });
    } else {
      const int acc = (int)(blockIdx.y & ~3u) + wave;
      const float* const p = slot + ((z * 16 + acc) * 64 + lane) * 4;
      auto dims = [&](int) { return 8 * acc + 4 * (lane >> 5); };
      if (n <= 4)
        add(One{}, Four{}, p, 0, r, dims);
      else
        add(One{}, std::integral_constant<int, 16>{}, p, 0, r, dims);
    }
  }
}

}  // namespace

PagedGrid paged_grid(int B, int H, int Hkv, int q_cap, int64_t max_keys, bool tree) {
  PagedGrid p = {};
  if (q_cap <= 0) return p;
  // Single tokens: no more rows than sequences, and no more than eight rows of a
  // sequence and key/value head for the chunks to meet at once. The host knows these two
  // numbers only, not what the batch holds. us, 28 / 4 heads, bf16, with this kernel and the
  // other: single tokens over 200 to 3100 keys, q of B rows and of one more, 8 9.6 / 12.7,
  // 16 14.3 / 18.3, 64 38.7 / 42.7, 200 124 / 129; one chunk in 256 places, q of fewer rows
  // than that and of more, 40 rows over 1000 keys 14.3 / 19.0, 64 over 8000 30.7 / 44.7, 200
  // over 2000 23.5 / 29.7, but 200 over 8000 62.6 / 47.4 (37.2 in a batch of one place).
  p.decode = q_cap <= B && H / Hkv <= 8;
  // every sequence with a query adds at most one tile that is not full
  auto tiles = [&](int rows) { return ((int64_t)q_cap * (H / Hkv) / rows + (B < q_cap ? B : q_cap)) * Hkv; };
  const int64_t units = tiles(p.decode ? kPagedFew : kPagedTile);
  const int64_t few = tiles(kPagedFew);
  p.short_keys = !tree || few > kPagedFewUnits ? 0 : (few > kPagedFewest ? kWholeFew : kPagedLong);
  p.items = p.short_keys ? few : units;
  if (B > kPagedScan) p.plan_bytes = ((size_t)(B + 1) * sizeof(PagedPlan) + 255) / 256 * 256;
  p.bytes = p.plan_bytes;
  if (max_keys >= 2 * kMinTile) {  // else nothing is cut
    p.items += kPagedPlaces;
    if (p.decode) {
      p.count_bytes = (size_t)kPagedLevels * kPagedPlaces * sizeof(unsigned long long);
    } else {  // a cut unit has two chunks at least
      const int64_t cut = p.short_keys > kWholeFew ? few : units;  // (shorter ones are not cut)
      p.cut_units = (int)(cut < kPagedPlaces / 2 ? cut : kPagedPlaces / 2);
      p.count_bytes = ((size_t)(kPagedPlaces / 2 + 1) * kPagedRecord + 255) / 256 * 256;
    }
    p.bytes += p.count_bytes + (size_t)kPagedPlaces * (p.decode ? kSlotBytes<true> : kSlotBytes<false>);
  }
  return p;
}

hipError_t launch_paged_attention(PagedArgs a, bool e4m3, hipStream_t stream) {
  if (a.q_cap <= 0) return hipSuccess;
  const PagedGrid p = paged_grid(a.B, a.H, a.Hkv, a.q_cap, (int64_t)a.max_pages << a.page_log2, a.mask != nullptr);
  // Groups of 1, 4, 16, 32 neighbours: 512 queries over 8704 keys 75.5, 76.2, 79.2,
  // 79.9 us, four chunks of 2048 over 7000 to 10240 888, 883, 896, 881.
  const uint32_t group = 4;
  const int64_t unit = p.decode ? 1 : (int64_t)kXcdCount * group;
  const int64_t grid = (p.items + unit - 1) / unit * unit;
  a.grid = (uint32_t)grid;
  a.decode = p.decode;
  a.short_keys = p.short_keys ? p.short_keys - kPagedShort : 0;
  static std::atomic<uint64_t> calls{0};
  a.token = paged_token(calls.fetch_add(1, std::memory_order_relaxed) + 1);
  if (a.B > kPagedScan) {
    hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(512), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const dim3 blocks((unsigned)grid), threads(256);
  auto launch = [&](auto f8, auto tree) {
    constexpr bool kF8 = decltype(f8)::value, kTree = decltype(tree)::value;
    if (p.decode) {
      hipLaunchKernelGGL((paged_decode_kernel<kF8, kTree>), blocks, threads, 0, stream, a);
      return hipGetLastError();
    }
    hipLaunchKernelGGL((paged_attention_kernel<kF8, kTree>), blocks, threads, 0, stream, a, group);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.cut_units == 0) return e;
    // Few units have many chunks: four times as many workgroups read sixteen of them at
    // a time (8 / 1 heads, five sequences of 6 to 9 tokens over 111 to 11538 keys 23.9,
    // 19.4 us; 40 of 2 to 9, 12 / 2 heads, up to 11349, 29.3, 25.7). With more units that
    // costs what it gains (two chunks of 701 beside 30 tokens 36.0, 37.2).
    const int parts = p.cut_units <= 128 ? 16 : 4;
    hipLaunchKernelGGL(paged_combine_kernel<kTree>, dim3(p.cut_units, parts), threads, 0, stream, a);
    return hipGetLastError();
  };
  using Yes = std::true_type;
  using No = std::false_type;
  if (a.mask) return e4m3 ? launch(Yes{}, Yes{}) : launch(No{}, Yes{});
  return e4m3 ? launch(Yes{}, No{}) : launch(No{}, No{});
}

}  // namespace ce
