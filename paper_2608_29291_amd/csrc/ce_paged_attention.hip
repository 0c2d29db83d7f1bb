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
// Keys. Sequences are cut along their keys, too, where the tiles alone leave the
// chip idle: with W = sum of tiles x keys and two workgroups on each of the 256
// CUs a chunk has L = W H_kv / 512 keys or more, and a sequence of n_k keys is cut
// into floor(n_k / L) chunks, so the cut ones are at most 512 workgroups together
// (a second round of a few would double the time) and as many partial results
// fit the workspace. Every wave forms the plan by itself from the lengths, which
// only the device knows: a lane per sequence, or per four, and two prefix sums; more
// than 256 sequences are planned by a launch of their own. Partial results (running
// maximum, sum, fp32 output) are combined in chunk order by a second launch, so no
// result depends on which workgroup came first.
//
// A key that a query does not see has no influence: its score is replaced before
// the maximum, and rows of a page behind the sequence's end read as zeros. What
// the products cannot hide, a NaN or infinity among the values under a weight of
// zero, shows as NaN in the output: a wave whose keys the causal mask cuts looks
// for it at its end and forms that output again, key by key (paged_redo).
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
  const int64_t j = (int64_t)(in_xcd / group) * (kXcdCount * group) + (w % kXcdCount) * group + in_xcd % group;
  Item it;
  if (!find_item(a, j, it)) return;
  if (it.few)
    paged_few<kF8>(a, smem, it);
  else
    paged_tile<kF8>(a, smem, it);
}

// The plan of more than kPagedScan sequences: prefix sums, and the chunk length
// behind them. One workgroup.
__global__ __launch_bounds__(1024) void paged_plan_kernel(PagedArgs a) {
  __shared__ int64_t scr[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = a.H / a.Hkv;
  int64_t w = 0;
  for (int b = tid; b < a.B; b += 1024) {
    const Size s = size_of(a, b, g);
    w += (int64_t)s.tiles * s.nk;
  }
  w = block_sum_i64(w, scr);
  const int L = chunk_length(a, w);
  int64_t base = 0;
  for (int b0 = 0; b0 < a.B; b0 += 1024) {
    const int b = b0 + tid;
    int64_t v = 0;
    if (b < a.B) v = counts_of(a, size_of(a, b, g), L);
    int64_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t y = __shfl_up(x, o);
      if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) scr[wave] = x;
    __syncthreads();
    int64_t before = base, total = 0;
    for (int i = 0; i < 16; ++i) {
      if (i < wave) before += scr[i];
      total += scr[i];
    }
    if (b < a.B) a.plan[b] = before + x - v;
    base += total;
  }
  if (tid == 0) {
    a.plan[a.B] = base;
    a.plan[a.B + 1] = L;
  }
}

// Partial results of the cut row tiles, in chunk order. Workgroups (tile,
// key/value head, *): up to eight chunks, eight rows at a time; more, a row at a
// time and its chunks in eight parts that meet in LDS.
__global__ __launch_bounds__(256) void paged_combine_kernel(PagedArgs a) {
  __shared__ f32x4_t acc_s[8][32];
  __shared__ float ml_s[2][8];
  Item it;
  if (!find_cut_tile(a, blockIdx.x, it)) return;
  const int kvh = blockIdx.y;
  const int tid = threadIdx.x;
  const int g = a.H / a.Hkv;
  const int n = it.tile_chunks;
  if (n <= 1) return;
  const float c2 = a.scale_log2 * (a.ks ? a.ks[kvh] : 1.0f);
  const float vs = a.vs ? a.vs[kvh] : 1.0f;
  const bool many = n > 8;
  const int at_once = many ? 1 : 8;
  const int grp = many ? tid >> 5 : 0;
  const int row_in = many ? 0 : it.few ? tid >> 5 : tid & 7;
  const int qd = many || it.few ? tid & 31 : tid >> 3;  // dims 4 qd .. +3
  const int per = many ? (n + 7) / 8 : n;
  const int c_lo = min(grp * per, n), c_hi = min(n, c_lo + per);
  const float* const slot0 = a.part + ((int64_t)(it.slot + it.tile * it.C) * a.Hkv + kvh) * kPagedPart;
  const int64_t stride = (int64_t)a.Hkv * kPagedPart;
  for (int rb = blockIdx.z * at_once; rb < it.rows; rb += gridDim.z * at_once) {
    const int r = rb + row_in;
    const int rr = min(r, it.rows - 1);
    const float* const p = slot0 + part_offset(it.few, rr, qd);
    const float* const ps = slot0 + kPagedRows * kDh + rr;
    float m = -__builtin_inff(), l = 0.0f;
    f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int c0 = c_lo; c0 < c_hi; c0 += 8) {
      float mc[8], lc[8];
      f32x4_t y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t c = (int64_t)min(c0 + i, c_hi - 1) * stride;
        mc[i] = ps[c];
        lc[i] = ps[c + kPagedRows];
        y[i] = *reinterpret_cast<const f32x4_t*>(p + c);
      }
      float m_new = m;
#pragma unroll
      for (int i = 0; i < 8; ++i) m_new = fmaxf(m_new, mc[i]);
      const float al = weight(m, m_new, c2);
      l *= al;
      x *= al;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (c0 + i < c_hi) {
          const float wi = weight(mc[i], m_new, c2);
          l = fmaf(lc[i], wi, l);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = fmaf(y[i][e], wi, x[e]);
        }
      }
      m = m_new;
    }
    if (many) {
      acc_s[grp][qd] = x;
      if (qd == 0) {
        ml_s[0][grp] = m;
        ml_s[1][grp] = l;
      }
      __syncthreads();
      m = ml_s[0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) m = fmaxf(m, ml_s[0][i]);
      l = 0.0f;
      x = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float wi = weight(ml_s[0][i], m, c2);
        l = fmaf(ml_s[1][i], wi, l);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmaf(acc_s[i][qd][e], wi, x[e]);
      }
      __syncthreads();
    }
    if (r < it.rows && grp == 0) {
      const int row = it.tile * kPagedRows + r;
      const int qi = row / g;
      const float inv = normalizer(l, vs, row_limit(a, it, qi, it.nk) > 0);
      store4<true>(a.o + ((int64_t)(it.qbase + qi) * a.H + kvh * g + (row - qi * g)) * kRowB + 8 * qd, x[0] * inv,
                   x[1] * inv, x[2] * inv, x[3] * inv);
    }
  }
}

}  // namespace

PagedGrid paged_grid(int B, int H, int Hkv, int q_cap, int64_t max_keys) {
  PagedGrid p = {};
  const int64_t rows = (int64_t)q_cap * (H / Hkv);
  // every sequence with a query adds at most one tile that is not full
  const int64_t tiles = rows / kPagedRows + (B < q_cap ? B : q_cap);
  const bool cuts = max_keys >= 2 * kMinChunk && kPagedTarget / Hkv >= 2;
  p.items = (tiles + (cuts ? kPagedTarget / Hkv : 0)) * Hkv;
  if (cuts) {
    const int64_t half = kPagedTarget / Hkv / 2;  // a cut tile has two chunks at least
    p.tiles = (int)(tiles < half ? tiles : half);
    p.rows = (int)(rows < kPagedRows ? rows : kPagedRows);
  }
  if (B > kPagedScan) p.plan_bytes = ((size_t)(B + 2) * sizeof(int64_t) + 255) / 256 * 256;
  p.bytes = q_cap > 0 ? p.plan_bytes + (cuts ? (size_t)(kPagedTarget / Hkv) * Hkv * kPagedPart * sizeof(float) : 0) : 0;
  return p;
}

hipError_t launch_paged_attention(const PagedArgs& a, bool e4m3, hipStream_t stream) {
  if (a.q_cap <= 0) return hipSuccess;
  const PagedGrid p = paged_grid(a.B, a.H, a.Hkv, a.q_cap, (int64_t)a.max_pages << a.page_log2);
  if (a.B > kPagedScan) {
    hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(1024), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  // Items of one tile a sequence share no keys; others in groups of neighbours.
  const int group = (int64_t)a.q_cap * (a.H / a.Hkv) <= (int64_t)kFew * a.B ? 1 : 16;
  const int64_t unit = (int64_t)kXcdCount * group;
  const int64_t grid = (p.items + unit - 1) / unit * unit;
  if (e4m3)
    hipLaunchKernelGGL(paged_attention_kernel<true>, dim3((unsigned)grid), dim3(256), 0, stream, a, group);
  else
    hipLaunchKernelGGL(paged_attention_kernel<false>, dim3((unsigned)grid), dim3(256), 0, stream, a, group);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.tiles == 0) return e;
  const int z = (p.rows + 7) / 8;
  hipLaunchKernelGGL(paged_combine_kernel, dim3(p.tiles, a.Hkv, z), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ce
