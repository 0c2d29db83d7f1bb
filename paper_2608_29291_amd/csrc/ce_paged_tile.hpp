// The two workgroups of paged attention (ce_paged_attention.hip): a few rows of a
// sequence against a chunk of its keys, and a tile of 128 rows.
#pragma once

#include <type_traits>

#include "ce_device.hpp"
#include "ce_paged.hpp"

namespace ce {

namespace paged {

constexpr int kDh = 128;           // head dimension
constexpr int kRowB = kDh * 2;     // bytes of a bf16 row
constexpr int kFew = 32;       // rows of a sequence that paged_few takes
constexpr int kKT = 64;            // keys per tile of paged_tile
constexpr int kBK = 32;            // keys per block: one pass of the softmax
constexpr int kKBytes = kKT * kRowB;
constexpr int kAhead = 3;          // MFMA operands read from LDS this many products ahead
constexpr float kLazy = 8.0f;      // headroom of the running maximum (exponent of 2)
constexpr int kMinChunk = 256;     // least keys of a chunk
constexpr int kOLd = kDh + 4;      // floats per row of paged_few's outputs in LDS
constexpr int kVRow = kBK * 2;     // bytes per row of paged_few's V^T
constexpr int kVTile = kDh * kVRow;
constexpr int kSmem = 4 * kFew * kOLd * 4 + 2 * 4 * kFew * 4;
static_assert(kSmem >= 4 * kKBytes && kSmem >= 4 * kVTile, "the tiles fit");

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// ------------------------------------------------------------------ the plan

struct Size {
  int qbase, nq, nk, tiles;
  bool few;
};

__device__ __forceinline__ Size size_from(const PagedArgs& a, int q0, int q1, int len, int g) {
  Size s;
  s.qbase = clampi(q0, 0, a.q_cap);
  s.nq = clampi(q1, s.qbase, a.q_cap) - s.qbase;
  s.nk = clampi(len, 0, a.max_pages << a.page_log2);
  const int rows = s.nq * g;
  s.few = rows <= kFew;
  s.tiles = s.few ? (rows > 0 ? 1 : 0) : (rows + kPagedRows - 1) / kPagedRows;
  return s;
}

__device__ __forceinline__ Size size_of(const PagedArgs& a, int b, int g) {
  return size_from(a, a.qo[b], a.qo[b + 1], a.lens[b], g);
}

// Keys per chunk for a batch of w tile-keys.
__device__ __forceinline__ int chunk_length(const PagedArgs& a, int64_t w) {
  const int64_t l = (w * a.Hkv + kPagedTarget - 1) / kPagedTarget;
  return (int)(l < kMinChunk ? kMinChunk : l > (1 << 30) ? 1 << 30 : l);
}

// A sequence's chunks (a whole number of the tiles that its waves take in turn).
__device__ __forceinline__ void cut(const PagedArgs& a, const Size& s, int L, int& C, int& chunk) {
  C = kPagedTarget / a.Hkv >= 2 ? s.nk / L : 1;
  if (C <= 1) {
    C = 1;
    chunk = s.nk;
    return;
  }
  const int unit = s.few ? 4 * kBK : kKT;
  chunk = (int)(((uint32_t)s.nk + C - 1) / (uint32_t)C + unit - 1) / unit * unit;
  C = (int)(((uint32_t)s.nk + chunk - 1) / (uint32_t)chunk);
  if (C <= 1) {
    C = 1;
    chunk = s.nk;
  }
}

// Items of a sequence and key/value head, and where it is cut its partial
// results (from bit 32) and row tiles (from bit 48).
__device__ __forceinline__ int64_t counts_of(const PagedArgs& a, const Size& s, int L) {
  int C, chunk;
  cut(a, s, L, C, chunk);
  const int64_t n = (int64_t)s.tiles * C;
  return n | (C > 1 ? (n & 0xffff) << 32 | (int64_t)(s.tiles & 0x7fff) << 48 : 0);
}

struct Item {
  int b, kvh, qbase, nq, nk;
  bool few;
  int tile, C, chunk;   // row tile, chunks of the sequence, keys of each
  int c;                // chunk of this item
  int slot;             // first partial result of the sequence (per key/value head)
  int rows;             // rows of the tile
  int vis_end;          // keys that its last row sees
  int tile_chunks;      // chunks that hold keys it sees (1: no partial results)
};

// Keys [0, row_limit) of the first `end` are seen by query qi.
__device__ __forceinline__ int row_limit(const PagedArgs& a, const Item& it, int qi, int end) {
  if (!a.causal) return end;
  return clampi(it.nk - it.nq + qi + 1, 0, end);
}


__device__ __forceinline__ int64_t readlane64(int64_t x, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)((uint64_t)x >> 32), lane);
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// Index `at` among the prefix sums' items or cut tiles.
template <bool kCutTiles>
__device__ __forceinline__ int key_of(int64_t prefix) {
  return kCutTiles ? (int)(prefix >> 48) : (int)(uint32_t)prefix;
}

// The sequence that holds item (or cut tile) number `at` of a key/value head, its
// sizes, the prefix sums before it and the chunk length; false past the last.
// Every wave finds it by itself, kPer sequences a lane.
template <bool kCutTiles, int kPer>
__device__ __forceinline__ bool find_by_scan(const PagedArgs& a, int g, int at, int& b, Size& size, int64_t& before,
                                             int& L) {
  const int lane = threadIdx.x & 63;
  Size s[kPer];
  int64_t w = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int bb = lane * kPer + i;
    s[i] = Size{0, 0, 0, 0, true};
    if (bb < a.B) s[i] = size_of(a, bb, g);
    w += (int64_t)s[i].tiles * s[i].nk;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) w += __shfl_xor(w, o);
  L = chunk_length(a, w);
  int64_t v[kPer], sum = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    v[i] = counts_of(a, s[i], L);
    sum += v[i];
  }
  int64_t x = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  const uint64_t past = __builtin_amdgcn_ballot_w64(at < key_of<kCutTiles>(x));
  if (!past) return false;
  const int ln = __builtin_ctzll(past);
  before = readlane64(x - sum, ln);
  L = __builtin_amdgcn_readfirstlane(L);
  bool found = false;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int64_t vi = readlane64(v[i], ln);
    if (!found) {
      if (i == kPer - 1 || at < key_of<kCutTiles>(before + vi)) {
        found = true;
        b = ln * kPer + i;
        size.qbase = __builtin_amdgcn_readlane(s[i].qbase, ln);
        size.nq = __builtin_amdgcn_readlane(s[i].nq, ln);
        size.nk = __builtin_amdgcn_readlane(s[i].nk, ln);
        size.tiles = __builtin_amdgcn_readlane(s[i].tiles, ln);
        size.few = size.nq * g <= kFew;
      } else {
        before += vi;
      }
    }
  }
  return true;
}

// The same from the plan in memory: three rounds of 64 samples.
template <bool kCutTiles>
__device__ __forceinline__ bool find_in_plan(const PagedArgs& a, int g, int at, int& b, Size& size, int64_t& before,
                                             int& L) {
  const int lane = threadIdx.x & 63;
  if (at >= key_of<kCutTiles>(a.plan[a.B])) return false;
  int lo = 0;  // the last sequence whose prefix is at most `at` is in [lo, lo + 64 step)
#pragma unroll
  for (int step = 4096; step > 0; step >>= 6) {
    const int i = lo + lane * step;
    const bool le = i < a.B && key_of<kCutTiles>(a.plan[i < a.B ? i : 0]) <= at;
    const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(le));
    lo += (n > 0 ? n - 1 : 0) * step;
  }
  b = __builtin_amdgcn_readfirstlane(lo);
  before = readlane64(a.plan[b], 0);
  L = __builtin_amdgcn_readfirstlane((int)a.plan[a.B + 1]);
  size = size_of(a, b, g);
  size.qbase = __builtin_amdgcn_readfirstlane(size.qbase);
  size.nq = __builtin_amdgcn_readfirstlane(size.nq);
  size.nk = __builtin_amdgcn_readfirstlane(size.nk);
  size.tiles = __builtin_amdgcn_readfirstlane(size.tiles);
  size.few = size.nq * g <= kFew;
  return true;
}

template <bool kCutTiles>
__device__ __forceinline__ bool find(const PagedArgs& a, int g, int at, int& b, Size& size, int64_t& before, int& L) {
  if (a.B <= 64) return find_by_scan<kCutTiles, 1>(a, g, at, b, size, before, L);
  if (a.B <= kPagedScan) return find_by_scan<kCutTiles, kPagedScan / 64>(a, g, at, b, size, before, L);
  return find_in_plan<kCutTiles>(a, g, at, b, size, before, L);
}

// What a row tile of the sequence sees, and where its partial results go. False
// if they would lie outside the workspace (only where offsets out of order make
// the plan's sums meaningless).
__device__ __forceinline__ bool finish_item(const PagedArgs& a, int g, const Size& s, int64_t before, Item& it) {
  it.qbase = s.qbase;
  it.nq = s.nq;
  it.nk = s.nk;
  it.few = s.few;
  const int r0 = it.tile * kPagedRows;
  it.rows = min(kPagedRows, s.nq * g - r0);
  it.vis_end = row_limit(a, it, (r0 + it.rows - 1) / g, s.nk);
  it.tile_chunks = it.C > 1 ? max(1, (it.vis_end + it.chunk - 1) / it.chunk) : 1;
  it.slot = (int)((before >> 32) & 0xffff);
  return it.C <= 1 || it.slot + s.tiles * it.C <= kPagedTarget / a.Hkv;
}

__device__ __forceinline__ bool find_item(const PagedArgs& a, int64_t j, Item& it) {
  const int g = a.H / a.Hkv;
  Size s;
  int64_t before;
  int L;
  const int64_t at = j / a.Hkv;
  if (!find<false>(a, g, (int)at, it.b, s, before, L)) return false;
  cut(a, s, L, it.C, it.chunk);
  const int n = s.tiles * it.C;
  const int rem = (int)(j - (int64_t)key_of<false>(before) * a.Hkv);
  it.kvh = rem / n;
  const int sub = rem - it.kvh * n;
  // last tiles first: under a causal mask they see the most keys
  const int back = sub / it.C;
  it.tile = s.tiles - 1 - back;
  it.c = sub - back * it.C;
  return finish_item(a, g, s, before, it) && it.c < it.tile_chunks;
}

__device__ __forceinline__ bool find_cut_tile(const PagedArgs& a, int at, Item& it) {
  const int g = a.H / a.Hkv;
  Size s;
  int64_t before;
  int L;
  if (!find<true>(a, g, at, it.b, s, before, L)) return false;
  cut(a, s, L, it.C, it.chunk);
  it.tile = at - key_of<true>(before);
  it.kvh = it.c = 0;
  return finish_item(a, g, s, before, it);
}

// ------------------------------------------------------- softmax and results

// Weight of a partial result with maximum m under the maximum m_all (raw scores;
// c2: their scale times log2 e). Without any finite maximum it counts nothing,
// except that NaN times 0 stays NaN.
__device__ __forceinline__ float weight(float m, float m_all, float c2) {
  return m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((m - m_all) * c2);
}

// Factor of the output: scale of the values / sum; a row that sees no key is zero,
// one that sees only scores of -infinity is 0 / 0.
__device__ __forceinline__ float normalizer(float l, float vs, bool sees) {
  return sees ? vs / l : 0.0f;
}

// Place of dims 4 qd .. +3 of row r in a partial result: rows of 128 floats, or
// for 128-row tiles the accumulators as the lanes hold them.
__device__ __forceinline__ int part_offset(bool few, int r, int qd) {
  if (few) return r * kDh + 4 * qd;
  return (((r >> 5) * 16 + (qd >> 1)) * 64 + (r & 31) + 32 * (qd & 1)) * 4;
}

__device__ __forceinline__ float* part_of(const PagedArgs& a, const Item& it) {
  return a.part + ((int64_t)(it.slot + it.tile * it.C + it.c) * a.Hkv + it.kvh) * kPagedPart;
}

// 8-byte LDS read that transposes 4 x 16 blocks of 16-bit values inside groups
// of 16 lanes: lane i gets value i % 4 of the 8 bytes that lanes i / 4, + 4,
// + 8, + 12 of its group point at.
__device__ __forceinline__ u32x2_t lds_read_tr(const char* __restrict__ p) {
  typedef short s16x4_t __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                         (__attribute__((address_space(3))) s16x4_t*)(p)));
}

// 4 e4m3 values (one dword) -> 4 bf16, exactly.
__device__ __forceinline__ u32x2_t e4m3_to_bf16(uint32_t x) {
  return u32x2_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, true))};
}

// x / g for 0 <= x < kPagedRows + g: off by at most 2^-22 x / g, while x + 1/2 is at
// least 1 / (2 g) from a multiple.
__device__ __forceinline__ int small_div(int x, float inv_g) { return (int)(((float)x + 0.5f) * inv_g); }

template <bool kF8>
constexpr int kPageRow = kF8 ? kDh : kRowB;  // bytes of a row of a page

// Head kvh of page number `page` of sequence b; `ok` false: not a page of the pool.
template <bool kF8>
__device__ __forceinline__ int64_t page_at(const PagedArgs& a, int kvh, int page, bool& ok) {
  ok = (uint32_t)page < (uint32_t)a.n_pages;
  return (int64_t)(ok ? page : 0) * a.page_bytes + ((int64_t)kvh << a.page_log2) * kPageRow<kF8>;
}

// Output of a wave's 32 rows again, key by key (the scores' maximum m and sum are
// right as they are): keys k0 + n kstep + 0 .. 31 below vis1, a lane's row sees those
// below vis. qf: the row, chunk s of 8 dims from kDims(s). Slow, and reached only
// where a value is NaN or infinite in a sequence's last rows.
template <bool kF8, bool kWide>
__device__ __forceinline__ void paged_redo(const PagedArgs& a, int b, int kvh, const u32x4_t (&qf)[8], f32x16_t (&oacc)[4],
                                        float m, float c2, int vis, int k0, int kstep, int vis1) {
  int lhalf = (threadIdx.x >> 5) & 1;
  asm volatile("" : "+v"(lhalf));  // no address of this path is formed before it
  const int mask = (1 << a.page_log2) - 1;
  const float mc = m == -__builtin_inff() ? 0.0f : m * c2;
#pragma unroll
  for (int i = 0; i < 4; ++i) oacc[i] = f32x16_t{};
  for (; k0 < vis1; k0 += kstep)
    for (int j = k0; j < min(k0 + 32, vis1); ++j) {
      bool ok;
      const int page = __builtin_amdgcn_readfirstlane(a.table[(int64_t)b * a.max_pages + (j >> a.page_log2)]);
      const int64_t at = page_at<kF8>(a, kvh, page, ok) + (int64_t)(j & mask) * kPageRow<kF8>;
      if (!ok) continue;  // zeros
      auto value = [&](const char* base, int d) __attribute__((always_inline)) {  // value at dim d of the row
        if constexpr (kF8) {
          const uint32_t x = *reinterpret_cast<const uint32_t*>(base + at + (d & ~3));
          const u32x2_t y = e4m3_to_bf16(x);
          const uint32_t z = (d & 2) ? y.y : y.x;
          return bf16_to_f32((d & 1) ? z >> 16 : z & 0xffffu);
        } else {
          const uint32_t x = *reinterpret_cast<const uint32_t*>(base + at + 2 * (d & ~1));
          return bf16_to_f32((d & 1) ? x >> 16 : x & 0xffffu);
        }
      };
      float sc = 0.0f;
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const int d0 = kWide ? (2 * (s >> 1) + lhalf) * 16 + 8 * (s & 1) : (2 * s + lhalf) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          sc = fmaf(bf16_to_f32((e & 1) ? qf[s][e >> 1] >> 16 : qf[s][e >> 1] & 0xffffu), value(a.k, d0 + e), sc);
        __builtin_amdgcn_sched_barrier(0);  // (few registers are left)
      }
      sc += __shfl_xor(sc, 32);
      const float p = __builtin_amdgcn_exp2f(fmaf(sc, c2, -mc));
      if (j < vis) {
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            oacc[db][v] = fmaf(p, value(a.v, 32 * db + 8 * (v >> 2) + 4 * lhalf + (v & 3)), oacc[db][v]);
            if ((v & 3) == 3) __builtin_amdgcn_sched_barrier(0);
          }
      }
    }
}

__device__ __forceinline__ bool any_nan(const f32x16_t (&oacc)[4]) {
  float t = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) t = fmaf(oacc[i][v], 0.0f, t);  // (infinities too: no harm)
  return __builtin_amdgcn_ballot_w64(t != t) != 0;
}

// ------------------------------------------------------------------ few rows

// Byte offset of unit u (4 keys) of V^T row d in a wave's tile. A write covers
// rows 8 apart and a read 32 consecutive rows; rows sit in 64-byte slots, four
// to a 256-byte bank line, and the slot and unit keys give both all 64 banks.
__device__ __forceinline__ uint32_t vt_off(int d, uint32_t u) {
  return (uint32_t)(((d & ~3) | ((d ^ (d >> 3)) & 3)) * kVRow) + ((u ^ (uint32_t)((d >> 2) & 7)) << 3);
}

// Up to 32 rows against a chunk of keys: the rows are the columns of one MFMA
// operand, the 4 waves take tiles of 32 keys in turn and share nothing until the
// end. K goes from memory to registers in operand order, V through registers
// (8-bit values converted, exactly, on the way) and a wave-private LDS tile that
// transposes it; the next tile's loads are issued as soon as the registers are
// free. Bound: memory.
template <bool kF8>
__device__ __forceinline__ void paged_few(const PagedArgs& a, char* const smem, const Item& it) {
  constexpr int kN = kF8 ? 4 : 8;  // 16-byte loads of K, and of V, per lane and tile
  float* const ml = reinterpret_cast<float*>(smem + 4 * kFew * kOLd * 4);  // [2][4][kFew]
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = a.H / a.Hkv;
  const int kvh = it.kvh;
  const int pl = a.page_log2, mask = (1 << pl) - 1;
  const float c2 = a.scale_log2 * (kF8 && a.ks ? a.ks[kvh] : 1.0f);
  const int kbeg = it.c * it.chunk;
  const int kend = min(it.nk, kbeg + it.chunk);
  const int rows = it.rows;

  // page numbers of this wave's tiles: lane 2 n + h holds that of the keys 16 h of
  // its tile n, 32 tiles (4096 keys of the chunk) at a time
  const int32_t* const table = a.table + (int64_t)it.b * a.max_pages;
  int pages = 0;
  auto load_pages = [&](int k) __attribute__((always_inline)) {  // from key k, this wave's
    const int64_t key = (int64_t)k + (lane >> 1) * 4 * kBK + 16 * (lane & 1);
    pages = key < it.nk ? table[key >> pl] : -1;
  };
  load_pages(kbeg + wave * kBK);

  // ---- the query row of this lane ----
  const int lrow = lane & 31;
  const int lhalf = lane >> 5;
  const int rr = min(lrow, rows - 1);
  const int qi = small_div(rr, 1.0f / (float)g);
  const int hq = kvh * g + (rr - qi * g);
  u32x4_t qf[8];
  {
    const char* qp = a.q + (int64_t)(it.qbase + qi) * a.q_ld + (int64_t)hq * kRowB;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const int d0 = kF8 ? (2 * (s >> 1) + lhalf) * 16 + 8 * (s & 1) : (2 * s + lhalf) * 8;
      qf[s] = *reinterpret_cast<const u32x4_t*>(qp + 2 * d0);
    }
  }
  const int vis = row_limit(a, it, qi, kend);              // keys [0, vis) are seen
  const int vis0 = row_limit(a, it, 0, kend);              // by the first row
  const int vis1 = min(it.vis_end, kend);                  // and by the last

  char* const vt = smem + wave * kVTile;
  const int vkg = lane & 7;   // keys 4 vkg .. +3 of the tile
  const int vdg = lane >> 3;  // 16 bytes vdg of a row (bf16: and vdg + 8)
  u32x4_t kf[kN], vr[kN];
  int64_t at0, at1;        // pages of the tile's two halves
  bool ok0 = true, ok1 = true;  // (of the tile in flight)
  int tile_n = 0;          // in the page numbers at hand
  // keys past the sequence's end read its last one (their scores are replaced)
  auto next_pages = [&](int k0) __attribute__((always_inline)) {
    if (tile_n == 32) {
      load_pages(k0);
      tile_n = 0;
    }
    const int p0 = __builtin_amdgcn_readlane(pages, 2 * tile_n);
    const int p1 = __builtin_amdgcn_readlane(pages, 2 * tile_n + 1);
    ++tile_n;
    at0 = page_at<kF8>(a, kvh, p0, ok0);
    at1 = at0;
    ok1 = true;
    if (k0 + 16 < it.nk) at1 = page_at<kF8>(a, kvh, p1, ok1);
  };
  auto row_at = [&](int k0, int kk) __attribute__((always_inline)) {
    const int key = min(k0 + kk, it.nk - 1);
    return (key - k0 >= 16 ? at1 : at0) + (int64_t)(key & mask) * kPageRow<kF8>;
  };
  auto load_k = [&](int k0) __attribute__((always_inline)) {
    const char* p = a.k + row_at(k0, lrow) + lhalf * 16;
#pragma unroll
    for (int s = 0; s < kN; ++s) kf[s] = *reinterpret_cast<const u32x4_t*>(p + s * 32);
  };
  auto load_v = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const char* p = a.v + row_at(k0, 4 * vkg + i) + vdg * 16;
      vr[i] = *reinterpret_cast<const u32x4_t*>(p);
      if constexpr (!kF8) vr[4 + i] = *reinterpret_cast<const u32x4_t*>(p + 128);
    }
  };

  f32x16_t oacc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) oacc[i] = f32x16_t{};
  float m_run = -__builtin_inff(), l_run = 0.0f;

  const int step = 4 * kBK;
  int k0 = kbeg + wave * kBK;
  if (k0 < vis1) {
    next_pages(k0);
    load_k(k0);
    load_v(k0);
  }
  for (; k0 < vis1; k0 += step) {
    const bool more = k0 + step < vis1;
    if (!(ok0 && ok1)) {  // a page that is none reads as zeros
      const bool kz = (lrow >= 16 && k0 + 16 < it.nk) ? !ok1 : !ok0;
      const bool vz = (vkg >= 4 && k0 + 16 < it.nk) ? !ok1 : !ok0;
#pragma unroll
      for (int s = 0; s < kN; ++s) {
        if (kz) kf[s] = u32x4_t{0, 0, 0, 0};
        if (vz) vr[s] = u32x4_t{0, 0, 0, 0};
      }
    }
    // scores: S^T = K Q^T (keys are the A operand), two chains
    f32x16_t sc = {}, s2 = {};
    if constexpr (kF8) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const u32x2_t x0 = e4m3_to_bf16(kf[s].x), x1 = e4m3_to_bf16(kf[s].y);
        const u32x2_t x2 = e4m3_to_bf16(kf[s].z), x3 = e4m3_to_bf16(kf[s].w);
        mfma_step<true>(sc, u32x4_t{x0.x, x0.y, x1.x, x1.y}, qf[2 * s]);
        mfma_step<true>(s2, u32x4_t{x2.x, x2.y, x3.x, x3.y}, qf[2 * s + 1]);
      }
    } else {
#pragma unroll
      for (int s = 0; s < 8; s += 2) {
        mfma_step<true>(sc, kf[s], qf[s]);
        mfma_step<true>(s2, kf[s + 1], qf[s + 1]);
      }
    }
    if (more) {
      next_pages(k0 + step);
      load_k(k0 + step);
    }
    sc += s2;
    if (k0 + kBK > vis0) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (k0 + 8 * (v >> 2) + 4 * lhalf + (v & 3) >= vis) sc[v] = -__builtin_inff();
    }
    // online softmax (lane = row; its keys sit in the lane and in lane ^ 32)
    float mt = sc[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) mt = fmaxf(mt, sc[v]);
    mt = fmaxf(mt, __shfl_xor(mt, 32));
    if (__builtin_amdgcn_ballot_w64((mt - m_run) * c2 > kLazy)) {
      const float m_new = fmaxf(m_run, mt);
      const float alpha = m_new == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((m_run - m_new) * c2);
#pragma unroll
      for (int i = 0; i < 4; ++i) oacc[i] *= alpha;
      l_run *= alpha;
      m_run = m_new;
    }
    const float mc = m_run == -__builtin_inff() ? 0.0f : m_run * c2;
    float rs = 0.0f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      sc[v] = __builtin_amdgcn_exp2f(fmaf(sc[v], c2, -mc));
      rs += sc[v];
    }
    l_run += rs + __shfl_xor(rs, 32);
    u32x4_t pf[2];
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int i = 0; i < 4; ++i) pf[st][i] = pack_bf16(sc[8 * st + 2 * i], sc[8 * st + 2 * i + 1]);
    // V tile to LDS, transposed (a wave's own tile: its LDS operations are in
    // order, so no barrier)
    auto put = [&](int d, uint32_t v0, uint32_t v1, uint32_t v2, uint32_t v3, bool odd) __attribute__((always_inline)) {
      const uint32_t sel = odd ? 0x07060302u : 0x05040100u;
      *reinterpret_cast<u32x2_t*>(vt + vt_off(d, (uint32_t)vkg)) =
          u32x2_t{__builtin_amdgcn_perm(v1, v0, sel), __builtin_amdgcn_perm(v3, v2, sel)};
    };
    if constexpr (kF8) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        u32x2_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = e4m3_to_bf16(vr[i][w]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          put(16 * vdg + 4 * w + e, y[0][e >> 1], y[1][e >> 1], y[2][e >> 1], y[3][e >> 1], e & 1);
      }
    } else {
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          put(64 * c + 8 * vdg + e, vr[4 * c][e >> 1], vr[4 * c + 1][e >> 1], vr[4 * c + 2][e >> 1],
              vr[4 * c + 3][e >> 1], e & 1);
    }
    if (more) load_v(k0 + step);
    // O^T += V^T P^T over 2 steps of 16 keys, in the scores' key order
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int db = 0; db < 4; ++db) {
        const u32x2_t lo = *reinterpret_cast<const u32x2_t*>(vt + vt_off(32 * db + lrow, (uint32_t)(4 * st + lhalf)));
        const u32x2_t hi =
            *reinterpret_cast<const u32x2_t*>(vt + vt_off(32 * db + lrow, (uint32_t)(4 * st + lhalf + 2)));
        mfma_step<true>(oacc[db], u32x4_t{lo.x, lo.y, hi.x, hi.y}, pf[st]);
      }
  }
  if (vis0 < vis1 && any_nan(oacc))
    paged_redo<kF8, kF8>(a, it.b, kvh, qf, oacc, m_run, c2, vis, kbeg + wave * kBK, step, vis1);

  // ---- the four waves meet: common maximum, scaled outputs through LDS ----
  int tid_e = threadIdx.x;
  asm volatile("" : "+v"(tid_e));  // (what the end needs is formed here: the loop leaves no register)
  const int erow = tid_e & 31, ehalf = (tid_e >> 5) & 1;
  if (ehalf == 0) {
    ml[wave * kFew + erow] = m_run;
    ml[(4 + wave) * kFew + erow] = l_run;
  }
  __syncthreads();  // also: every wave is done with its V tile
  float m_all = ml[erow];
#pragma unroll
  for (int w = 1; w < 4; ++w) m_all = fmaxf(m_all, ml[w * kFew + erow]);
  const float al = weight(m_run, m_all, c2);
  float* const ob = reinterpret_cast<float*>(smem);
  if (erow < rows) {
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4)
        *reinterpret_cast<f32x4_t*>(ob + (wave * kFew + erow) * kOLd + 32 * db + 8 * g4 + 4 * ehalf) =
            f32x4_t{oacc[db][4 * g4] * al, oacc[db][4 * g4 + 1] * al, oacc[db][4 * g4 + 2] * al, oacc[db][4 * g4 + 3] * al};
  }
  __syncthreads();
  const bool partial = it.tile_chunks > 1;
  const float vs = kF8 && a.vs ? a.vs[kvh] : 1.0f;
  // thread: row tid / 32 (+ 8, 16, 24), dims 4 (tid % 32) .. +3
  for (int r = tid_e >> 5; r < rows; r += 8) {
    const int qd = tid_e & 31;
    float mr = ml[r], lr = 0.0f;
#pragma unroll
    for (int w = 1; w < 4; ++w) mr = fmaxf(mr, ml[w * kFew + r]);
    f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      lr = fmaf(ml[(4 + w) * kFew + r], weight(ml[w * kFew + r], mr, c2), lr);
      x += *reinterpret_cast<const f32x4_t*>(ob + (w * kFew + r) * kOLd + 4 * qd);
    }
    if (partial) {
      float* const p = part_of(a, it);
      *reinterpret_cast<f32x4_t*>(p + part_offset(true, r, qd)) = x;
      if (qd == 0) {
        p[kPagedRows * kDh + r] = mr;
        p[kPagedRows * kDh + kPagedRows + r] = lr;
      }
    } else {
      const int q2 = small_div(r, 1.0f / (float)g);
      const float inv = normalizer(lr, vs, row_limit(a, it, q2, it.nk) > 0);
      store4<true>(a.o + ((int64_t)(it.qbase + q2) * a.H + kvh * g + (r - q2 * g)) * kRowB + 8 * qd, x[0] * inv,
                   x[1] * inv, x[2] * inv, x[3] * inv);
    }
  }
}

// ---------------------------------------------------------------- 128-row tiles

// 128 rows (32 a wave) against a chunk of keys, in tiles of 64:
//   * S^T = K Q^T on MFMA 32x32x16 (keys are the A operand, the wave's rows the B
//     operand, in registers for the whole loop), so each lane owns one row: its 16
//     scores of a block of 32 keys sit in the lane and the other 16 in lane l ^ 32;
//   * the probabilities (bf16, in operand order) times V^T, with the key index of
//     that product permuted to match the score accumulators;
//   * the 16 keys that a wave brings of a tile lie in one page (pages hold 16 rows
//     or more, from a multiple of 16): a buffer resource over them, built from the
//     page number, makes the fetch the one of a contiguous cache, with 64-bit
//     page addresses, and its range check gives zeros behind the sequence's end;
//   * bf16 pages reach LDS by whole-line DMA, chunk c of K row r at c ^ (r & 15),
//     chunk c of V row r at c ^ 4 (r & 3) (conflict-free fragment reads; V is
//     transposed by the reads). 8-bit pages come through registers, are converted
//     (exactly) once per workgroup and stored in the same layout, a tile's loads in
//     flight during the one before;
//   * a stage carries one block of 32 keys through the softmax, one probability
//     after each MFMA of two products that do not depend on it: the scores of the
//     next block and the output of the block before.
// Bound: MFMA and the softmax's VALU about alike.
template <bool kF8>
__device__ __forceinline__ void paged_tile(const PagedArgs& a, char* const smem, const Item& it) {
  // Beside other arrays in LDS the compiler ties the DMAs to the fragment reads and
  // drains them before each stage, unless their base passes through an empty asm.
  typedef __attribute__((address_space(3))) char lds_char;
  lds_char* ring = (lds_char*)smem;
  asm volatile("" : "+s"(ring));
  char* const kbuf = smem;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = a.H / a.Hkv;
  const float inv_g = 1.0f / (float)g;
  const int kvh = it.kvh;
  const int pl = a.page_log2, mask_p = (1 << pl) - 1;
  const float c2 = a.scale_log2 * (kF8 && a.ks ? a.ks[kvh] : 1.0f);
  const int kbeg = it.c * it.chunk;
  const int kend = min(it.nk, kbeg + it.chunk);
  const int ntiles = max(0, min(kend, it.vis_end) - kbeg + kKT - 1) / kKT;

  const int lrow = lane & 31;
  const int lhalf = lane >> 5;
  const int kr_sub = lane >> 4;   // row within a DMA instruction
  const int kpc = lane & 15;      // physical chunk this lane fills
  auto opaque = [](uint32_t x) __attribute__((always_inline)) {
    asm volatile("" : "+v"(x));
    return x;
  };

  // ---- rows: row r of the sequence is query r / g, head r % g of the group ----
  const int r0 = it.tile * kPagedRows;
  const int q0 = r0 / g;         // first query, and the first row's place in its group
  const int h0 = r0 - q0 * g;

  // ---- page numbers: lane l holds that of this wave's 16 keys of tile tb + l, in
  //      two windows of 64 tiles ----
  const int32_t* const table = a.table + (int64_t)it.b * a.max_pages;
  auto load_pages = [&](int tile) __attribute__((always_inline)) {
    const int64_t key = (int64_t)kbeg + ((int64_t)tile + lane) * kKT + 16 * wave;
    return key < it.nk ? table[key >> pl] : -1;
  };
  int tb = 0;
  int pages = load_pages(0), pages2 = load_pages(64);
  auto resource = [&](const char* pool, int tile) __attribute__((always_inline)) {
    const int i = tile - tb;
    const int page = i < 64 ? __builtin_amdgcn_readlane(pages, i & 63) : __builtin_amdgcn_readlane(pages2, i & 63);
    const int key = kbeg + tile * kKT + 16 * wave;
    bool ok;
    const int64_t at = page_at<kF8>(a, kvh, page, ok) + (int64_t)(key & mask_p) * kPageRow<kF8>;
    const int n = ok ? clampi(it.nk - key, 0, 16) : 0;
    return make_rsrc(pool + at, (uint32_t)(n * kPageRow<kF8>));
  };

  // ---- K and V tiles: wave w brings rows 16 w .. +15 ----
  uint32_t kvo[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 4 * i + kr_sub;
    kvo[i] = opaque((uint32_t)(r * kRowB + ((kpc ^ (r & 15)) << 4)));
  }
  const uint32_t vvo = opaque((uint32_t)(kr_sub * kRowB + ((kpc ^ (kr_sub << 2)) << 4)));
  u32x4_t kreg[2], vreg[2];  // 8-bit pages: rows 8 i + lane / 8, 16 values lane % 8
  auto fetch_k = [&](int tile, int buf) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rs = resource(a.k, tile);
    if constexpr (kF8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) kreg[i] = bload16(rs, lane * 16 + i * 1024, 0);
    } else {
      lds_char* region = ring + buf * kKBytes + 16 * wave * kRowB;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, region + 4 * i * kRowB, 16, (int)kvo[i], 0, 0, 0);
    }
  };
  auto fetch_v = [&](int tile, int buf) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rs = resource(a.v, tile);
    if constexpr (kF8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) vreg[i] = bload16(rs, lane * 16 + i * 1024, 0);
    } else {
      lds_char* region = ring + (2 + buf) * kKBytes + 16 * wave * kRowB;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, region + 4 * i * kRowB, 16, (int)vvo, 4 * i * kRowB, 0, 0);
    }
  };
  // 8-bit values to LDS: 16 of a row are its chunks 2 m and 2 m + 1, m = lane % 8
  auto put = [&](const u32x4_t (&x)[2], int base, bool is_k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = 8 * i + (lane >> 3), m = lane & 7;
      const int key = is_k ? r : (r & 3) << 2;
      char* const row = smem + base + (16 * wave + r) * kRowB;
      const u32x2_t y0 = e4m3_to_bf16(x[i].x), y1 = e4m3_to_bf16(x[i].y);
      const u32x2_t y2 = e4m3_to_bf16(x[i].z), y3 = e4m3_to_bf16(x[i].w);
      lds_write16(row, ((2 * m) ^ key) << 4, u32x4_t{y0.x, y0.y, y1.x, y1.y});
      lds_write16(row, ((2 * m + 1) ^ key) << 4, u32x4_t{y2.x, y2.y, y3.x, y3.y});
    }
  };

  u32x4_t qf[8];  // this lane's row, K steps of 16
  uint32_t koff[8];  // K fragments: row lrow, chunk (2 s + lhalf), swizzled
#pragma unroll
  for (int s2 = 0; s2 < 8; ++s2)
    koff[s2] = opaque((uint32_t)(lrow * kRowB + ((((uint32_t)(2 * s2 + lhalf)) ^ (uint32_t)(lrow & 15)) << 4)));
  // V: a transposing read gives 16 lanes the 16 dims of four keys; this lane
  // supplies 8 bytes of key 4 lhalf + (lane / 4) % 4
  uint32_t voff[4];
#pragma unroll
  for (int db = 0; db < 4; ++db) {
    const int key = (lane >> 2) & 3;
    const int c = ((db ^ key) << 2) + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    voff[db] = opaque((uint32_t)(2 * kKBytes + (4 * lhalf + key) * kRowB + (c << 4) + 8 * (lane & 1)));
  }

  f32x16_t oacc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) oacc[i] = f32x16_t{};
  float m_run = -__builtin_inff(), l_run = 0.0f;  // l_run: this lane's keys only until the epilogue
  const int qi = q0 + small_div(h0 + min(32 * wave + lrow, it.rows - 1), inv_g);  // this lane's query
  const int vis = row_limit(a, it, qi, kend);  // keys [0, vis) are seen
  const int vis0 = row_limit(a, it, __builtin_amdgcn_readfirstlane(qi), kend);  // by the wave's first row

  using Half0 = std::integral_constant<int, 0>;
  using Half1 = std::integral_constant<int, 1>;
  using Yes = std::true_type;
  using No = std::false_type;
  auto tile_max = [&](const f32x16_t& sc) __attribute__((always_inline)) {
    float m = -__builtin_inff();
#pragma unroll
    for (int v = 0; v < 16; ++v) m = fmaxf(m, sc[v]);
    return m;
  };
  // hide the keys of block `blk` this lane may not see (ragged end, causal cut)
  auto mask = [&](int blk, f32x16_t& sc, float& mt) __attribute__((always_inline)) {
    const int kbase = kbeg + blk * kBK;
    if (kbase + kBK > vis0) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (kbase + 8 * (v >> 2) + 4 * lhalf + (v & 3) >= vis) sc[v] = -__builtin_inff();
      mt = tile_max(sc);
    }
  };
  // operand of MFMA j of a stage: 0..7 the scores (32-byte K step j), 8..15
  // the output (16 keys (j - 8) / 4, 32 dims j % 4)
  auto frag = [&](int j, int khalf, int vhalf) __attribute__((always_inline)) {
    if (j < 8) return lds_read16(smem + koff[j], khalf * kBK * kRowB);
    const char* p = smem + voff[j & 3] + (vhalf * kBK + 16 * ((j - 8) >> 2)) * kRowB;
    const u32x2_t lo = lds_read_tr(p), hi = lds_read_tr(p + 8 * kRowB);
    return u32x4_t{lo.x, lo.y, hi.x, hi.y};
  };
  // One stage takes block blk (32 keys, half blk % 2 of its tile) through the
  // softmax (scores sc, lane maximum mt; probabilities to pn) while the matrix
  // cores compute the scores of block blk + 1 (into sn, lane maximum to mn) and
  // then the output of block blk - 1 (probabilities pp): one probability after
  // each MFMA, in program order. The fences keep the compiler from sorting the
  // two kinds of instructions apart again.
  auto stage = [&](auto half_c, auto first_c, auto last_c, int blk, f32x16_t& sc, f32x16_t& sn, u32x4_t (&pp)[2],
                   u32x4_t (&pn)[2], float mt, float& mn) __attribute__((always_inline)) {
    constexpr int kHalf = decltype(half_c)::value;
    constexpr bool kFirst = decltype(first_c)::value, kLast = decltype(last_c)::value;
    constexpr int kLo = kLast ? 8 : 0, kHi = kFirst ? 8 : 16;  // MFMAs of this stage
    constexpr int kPer = 16 / (kHi - kLo);                     // probabilities after each
    u32x4_t fr[16];
#pragma unroll
    for (int j = kLo; j < kLo + kAhead; ++j) fr[j] = frag(j, kHalf ^ 1, kHalf ^ 1);
    // The running maximum moves (and the output is rescaled) only when some
    // lane's block maximum exceeds it by more than kLazy in the exponent, so
    // probabilities stay below 2^kLazy; the sum l uses the same maximum, so
    // the quotient O / l does not depend on it. The output still lacks block
    // blk - 1, whose probabilities have the old maximum: it is rescaled after
    // this stage's MFMAs.
    {
      const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(mt), __float_as_uint(mt), false, false);
      mt = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
    }
    float alpha = 1.0f;
    const bool move = __builtin_amdgcn_ballot_w64((mt - m_run) * c2 > kLazy) != 0;
    if (move) {
      const float m_new = fmaxf(m_run, mt);
      if (m_new != -__builtin_inff()) alpha = __builtin_amdgcn_exp2f((m_run - m_new) * c2);
      l_run *= alpha;
      m_run = m_new;
    }
    const float mc = m_run == -__builtin_inff() ? 0.0f : m_run * c2;
    float rs = 0.0f, even = 0.0f;
    auto prob = [&](int e) __attribute__((always_inline)) {
      float p = __builtin_amdgcn_exp2f(fmaf(sc[e], c2, -mc));
      asm volatile("" : "+v"(p));  // this and the next keep the value between its fences
      if (e & 1) {
        rs += even + p;
        uint32_t w = pack_bf16(even, p);
        asm volatile("" : "+v"(w), "+v"(rs));
        pn[e >> 3][(e & 7) >> 1] = w;
      } else {
        even = p;
      }
    };
    float mx = -__builtin_inff();
    __builtin_amdgcn_s_setprio(1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = kLo; j < kHi; ++j) {
      if (j + kAhead < kHi) fr[j + kAhead] = frag(j + kAhead, kHalf ^ 1, kHalf ^ 1);
      if (j == 0) sn = f32x16_t{};
      if (j < 8)
        mfma_step<true>(sn, fr[j], qf[j]);
      else
        mfma_step<true>(oacc[j & 3], fr[j], pp[(j - 8) >> 2]);
#pragma unroll
      for (int e = (j - kLo) * kPer; e < (j - kLo + 1) * kPer; ++e) prob(e);
      if (!kLast && !kFirst && j >= 12) {
#pragma unroll
        for (int v = 4 * (j - 12); v < 4 * (j - 11); ++v) mx = fmaxf(mx, sn[v]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    l_run += rs;
    if constexpr (!kFirst) {
      if (move) {
#pragma unroll
        for (int i = 0; i < 4; ++i) oacc[i] *= alpha;
      }
    }
    if constexpr (!kLast) {
      mn = kFirst ? tile_max(sn) : mx;
      mask(blk + 1, sn, mn);
    }
  };

  // tile t: buffer t % 2 of K and of V. Scores run one block ahead and the
  // output one block behind, so between two barriers the second half of tile t
  // and the first of tile t + 1 meet K of t + 1 and V of t only, and the fetch of
  // K of t + 2 and V of t + 1 has that time to arrive (8-bit pages: it was begun
  // one iteration earlier and goes to LDS now).
  if (ntiles > 0) {
    f32x16_t sa = f32x16_t{}, sb;
    u32x4_t pa[2], pb[2];
    float ma, mb;
    // The wave's 32 rows come by whole-line DMA as well (rows past the end as
    // zeros), chunk c of row r at c ^ (r & 15), into the parts of the two V
    // buffers that this wave itself fills later.
    {
      const int last = small_div(h0 + it.rows - 1, inv_g);  // the last row's query behind q0
      const char* qp = a.q + (int64_t)(it.qbase + q0) * a.q_ld + (int64_t)kvh * g * kRowB;
      const int span = h0 + it.rows - last * g;  // heads of that query that are rows
      const __amdgpu_buffer_rsrc_t qrs =
          make_rsrc(qp, (uint32_t)((int64_t)last * a.q_ld) + (uint32_t)(span * kRowB));
      const int qb = 2 * kKBytes + 16 * wave * kRowB;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + kr_sub;
        const int x = h0 + 32 * wave + r;
        const int dq = small_div(min(x, h0 + it.rows - 1), inv_g);
        uint32_t vo = (uint32_t)(dq * (int)a.q_ld) + (uint32_t)((x - dq * g) * kRowB + ((kpc ^ (r & 15)) << 4));
        if (32 * wave + r >= it.rows) vo = 0xfffffff0u;  // zeros
        __builtin_amdgcn_raw_ptr_buffer_load_lds(qrs, ring + qb + (i >> 2) * kKBytes + 4 * (i & 3) * kRowB, 16, (int)vo, 0,
                                                 0, 0);
      }
      if constexpr (!kF8) {
        fetch_k(0, 0);
        if (ntiles > 1) {
          fetch_k(1, 1);
          wait_vmcnt<8>();
        } else {
          wait_vmcnt<4>();
        }
      } else {
        fetch_k(0, 0);
        wait_vmcnt<0>();  // (loads to registers may be issued before the DMAs)
      }
      asm volatile("" ::: "memory");
#pragma unroll
      for (int s2 = 0; s2 < 8; ++s2)
        qf[s2] = lds_read16(smem + qb + (lrow >> 4) * kKBytes + (lrow & 15) * kRowB,
                            ((2 * s2 + lhalf) ^ (lrow & 15)) << 4);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read before V takes their place
    }
    if constexpr (kF8) {
      put(kreg, 0, true);
      if (ntiles > 1) {
        fetch_k(1, 1);
        fetch_v(0, 0);
        put(kreg, kKBytes, true);
      } else {
        fetch_v(0, 0);
      }
      put(vreg, 2 * kKBytes, false);
      if (ntiles > 2) fetch_k(2, 0);
      if (ntiles > 1) fetch_v(1, 1);
    } else {
      fetch_v(0, 0);
      wait_vmcnt<4>();  // K
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) mfma_step<true>(sa, frag(j, 0, 0), qf[j]);
    ma = tile_max(sa);
    mask(0, sa, ma);
    stage(Half0{}, Yes{}, No{}, 0, sa, sb, pb, pa, ma, mb);
    if constexpr (!kF8) wait_vmcnt<0>();
    __syncthreads();  // every wave has read K of tile 0; V of tile 0 is there
    for (int t = 0; t + 1 < ntiles; ++t) {
      if (t + 1 - tb >= 64) {  // K is fetched up to two (8-bit: three) tiles ahead, V one (two)
        tb += 64;
        pages = pages2;
        pages2 = load_pages(tb + 64);
      }
      if constexpr (kF8) {
        if (t + 2 < ntiles) put(kreg, (t & 1) * kKBytes, true);
        put(vreg, (2 + ((t + 1) & 1)) * kKBytes, false);
        if (t + 3 < ntiles) fetch_k(t + 3, 0);
        if (t + 2 < ntiles) fetch_v(t + 2, 0);
      } else {
        if (t + 2 < ntiles) fetch_k(t + 2, t & 1);
      }
#pragma unroll
      for (int s2 = 0; s2 < 8; ++s2) koff[s2] ^= kKBytes;
      stage(Half1{}, No{}, No{}, 2 * t + 1, sb, sa, pa, pb, mb, ma);
      if constexpr (!kF8) fetch_v(t + 1, (t + 1) & 1);
      stage(Half0{}, No{}, No{}, 2 * t + 2, sa, sb, pb, pa, ma, mb);
#pragma unroll
      for (int db = 0; db < 4; ++db) voff[db] ^= kKBytes;
      if constexpr (!kF8) {
        wait_vmcnt<0>();
        __syncthreads();
      } else {
        lds_barrier();  // (the next tiles' loads stay in flight)
      }
    }
    stage(Half1{}, No{}, Yes{}, 2 * ntiles - 1, sb, sa, pa, pb, mb, ma);
#pragma unroll
    for (int j = 8; j < 16; ++j) mfma_step<true>(oacc[j & 3], frag(j, 0, 1), pb[(j - 8) >> 2]);
    const int last_key = min(kend, kbeg + ntiles * kKT);
    if (a.causal && vis0 < last_key && any_nan(oacc))
      paged_redo<kF8, false>(a, it.b, kvh, qf, oacc, m_run, c2, vis, kbeg, kBK, last_key);
  }

  l_run += __shfl_xor(l_run, 32);
  if (it.tile_chunks > 1) {
    // ---- partial results, as the lanes hold them ----
    float* const p = part_of(a, it);
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4)
        *reinterpret_cast<f32x4_t*>(p + ((wave * 16 + 4 * db + g4) * 64 + lane) * 4) =
            f32x4_t{oacc[db][4 * g4], oacc[db][4 * g4 + 1], oacc[db][4 * g4 + 2], oacc[db][4 * g4 + 3]};
    if (lhalf == 0) {
      p[kPagedRows * kDh + 32 * wave + lrow] = m_run;
      p[kPagedRows * kDh + kPagedRows + 32 * wave + lrow] = l_run;
    }
    return;
  }
  // ---- O = O^T / l, turned through LDS into whole rows (256 bytes by 16 lanes).
  //      The wave uses its own 8 KB of the K buffers, which no wave reads after
  //      the last barrier. ----
  const float inv = normalizer(l_run, kF8 && a.vs ? a.vs[kvh] : 1.0f, row_limit(a, it, qi, it.nk) > 0);
  char* const ob = kbuf + wave * 32 * kRowB;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4)
      store4<true>(ob + lrow * kRowB + (((4 * db + g4) ^ (lrow & 15)) << 4) + 8 * lhalf, oacc[db][4 * g4] * inv,
                   oacc[db][4 * g4 + 1] * inv, oacc[db][4 * g4 + 2] * inv, oacc[db][4 * g4 + 3] * inv);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = 4 * i + kr_sub;
    const u32x4_t w = lds_read16(ob, r * kRowB + (kpc << 4));
    if (32 * wave + r < it.rows) {
      const int x = h0 + 32 * wave + r;
      const int dq = small_div(x, inv_g);
      *reinterpret_cast<u32x4_t*>(a.o + ((int64_t)(it.qbase + q0 + dq) * a.H + kvh * g + (x - dq * g)) * kRowB +
                                  ((kpc ^ (r & 15)) << 4)) = w;
    }
  }
}

}  // namespace paged

}  // namespace ce
