// The plan and the two workgroups of paged attention (ce_paged_attention.hip): up to 32
// rows of a sequence against a chunk of its keys, and a tile of 128 rows.
#pragma once

#include <type_traits>

#include "ce_device.hpp"
#include "ce_paged.hpp"
#include "ce_softmax.hpp"

namespace ce {

namespace paged {

constexpr int kDh = 128;           // head dimension
constexpr int kRowB = kDh * 2;     // bytes of a bf16 row
constexpr int kFew = kPagedFew;
constexpr int kTileRows = kPagedTile;
constexpr int kFewLog2 = 5, kTileLog2 = 7;
static_assert(kFew == 1 << kFewLog2 && kTileRows == 1 << kTileLog2, "rows of the tiles");
constexpr int kKT = 64;            // keys per tile of paged_tile
constexpr int kBK = 32;            // keys per block: one pass of the softmax
constexpr int kKBytes = kKT * kRowB;
constexpr int kGroup = 4;          // MFMA operands read from LDS together, one group ahead
constexpr float kLazy = 8.0f;      // headroom of the running maximum (exponent of 2)
constexpr int kMinFew = 128;       // least keys of a chunk: one tile of 32 for each wave
constexpr int kWholeFew = 640;     // least keys of a sequence that is cut for a few rows
constexpr int kMaxHalf = 512;      // keys per place up to which single tokens fill half of the places,
constexpr int kMaxEven = 1024;     // and where the sequences are about equal
constexpr int kMaxMeet = 512;      // keys per chunk up to which no more than kMeet meet
constexpr int kMostOver = 24;      // chunks that are made kMeet whatever their keys
constexpr int kMinTile = 256;
constexpr int kWideMask = 4;       // words of a mask from which tiles end where their rows' bits do
constexpr int kMeet = 16;          // chunks that meet at a time in the launch itself
constexpr int kOLd = kDh + 4;      // floats per row of paged_few's outputs in LDS
constexpr int kVRow = kBK * 2;     // bytes per row of paged_few's V^T
constexpr int kVTile = kDh * kVRow;
constexpr int kSmem = 4 * kFew * kOLd * 4 + 2 * 4 * kFew * 4;
static_assert(kSmem >= 4 * 2 * kVTile && kSmem >= 4 * kKBytes && 2 * kSmem <= 160 * 1024, "the tiles fit");
static_assert(kWholeFew >= 2 * kMinTile, "the host takes 2 kMinTile keys for the least that is cut");

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// ------------------------------------------------------------------ the plan
//
// A call of single tokens (a.decode: no more rows than sequences) takes its rows 32 at
// a time (paged_few); any other takes those of a sequence that has more than 32 in
// tiles of 128 (paged_tile). Under masks of bits short sequences of small calls go 32 rows to a tile as
// well, four waves over their keys instead of one:
//   * of 96 to 639 keys, as a rule not cut, where all such tiles have a CU of their own: us, 28 / 4 heads,
//     bf16, four trees of 64 over 64, 150, 300, 500 keys 7.6, 10.2, 11.8, 16.4 / 8.3, 8.9, 10.1, 13.0; one of
//     26 7.0, 9.6, 11.3, 15.7 / 7.2, 8.4, 9.4, 11.8. With 308 tiles 12.9 / 13.2 and, 8 bits, 14.1 / 15.6 (4 x 200
//     rows, 12 / 2 heads, 300 keys);
//   * of up to 8191, in calls of at most 96 such tiles: 12 / 2 heads, bf16, a tree of 26 over 1100, 2500, 4000,
//     8000, 16000 keys 13.1, 15.0, 14.8, 17.7, 23.6 / 12.0, 12.4, 12.6, 14.3, 22.3; 42 such calls of up to 96 tiles
//     over 700 to 8000 keys on average 0.88 to 1.00 of the time, 1.11 at most; of 100 to 256 tiles 0.97 to 1.14, of
//     16000 keys 0.9 to 1.5.
//
// A unit is a row tile of a sequence for one key/value head; units are numbered
// sequence by sequence, head by head, the last tiles first (under a causal mask they
// see the most keys). A key costs a tile of 128 rows about twice what it costs a few
// rows, so keys are counted as 1 and 1/2. With S = 512 places for workgroups (two on each
// CU) and A = (sum of the units' keys) / S:
//   * a batch of many units fills S places some whole number of times and leaves
//     a rest; the units before the rest are whole, and the rest, fewer than S, are cut
//     along their keys so that they too fill the places: L = (their keys) / S;
//   * where one sequence alone has 2 A keys or more, or there are fewer units than
//     places, every unit may be cut, L = A.
// A unit of n_k keys is cut into floor(n_k / L) chunks, so the chunks of all cut units
// are at most S (a second round of a few would double the time) and as many
// partial results fit the workspace. A few rows are cut less than that where it does
// not pay (us, single tokens at 28 / 4 heads, bf16, before / after):
//   * below 640 keys not at all: 1 x 300 keys 9.7 / 7.5, 32 x 600 14.9 / 11.1;
//   * into at most 16 chunks, that meet at once, as long as these have no more than 512
//     keys: 1 x 4000 13.0 / 10.6, 8 x 5 drafted tokens over 333 to 4103 18.3 / 15.9; of
//     17 to 24 chunks 16 are made in any case: 15 sequences up to 13516 29.4 / 24.5,
//     29 up to 16281, 12 / 2 heads, 24.6 / 21.7 (of up to 32: 34 up to 16222, 8 bits,
//     8 / 1 heads, 15.8 / 17.0);
//   * single tokens into half as many where a place's share is at most 512 keys: one
//     workgroup a CU keeps the memory as busy, and fewer chunks meet: 16 sequences of
//     551 to 3100 16.4 / 15.3, 32 x 1000 18.2 / 14.8. Up to 1024 so where the sequences
//     are about equal (1 x 65537 34.5 / 32.9, 39 of one length, 4 / 4 heads, 53 / 50);
//     unequal ones need the finer cut there (half as many / this: 57, 31, 43 and 48
//     drawn sequences 38 / 29, 56 / 46, 40 / 27, 68 / 51).
//
// Under masks of bits, where L is 512 keys or more, a unit's count is rounded to the nearest, as long as
// no more than S chunks come of it. Trees of 12 to 40 sequences, lengths of 1000 to 16000 (36 drawn
// batches): between -15% and +13% of the time, -2.4% on average; 32 trees over 2100 to 16001
// keys 212 / 176 us, two prompts with images 93 / 97. With a smaller L it costs 1.3%.
//
// How the chunks meet: of single tokens, in the launch itself (a second one would
// cost 4 us of 15); of many rows, by a second launch over the whole chip, since one
// workgroup would read 64 KB a chunk.

struct Size {
  int qbase, nq, nk, tiles;
};

__device__ __forceinline__ bool is_few(const PagedArgs& a, int nq, int nk, int g) {
  return a.decode || nq * g <= kFew || (uint32_t)(nk - kPagedShort) < (uint32_t)a.short_keys;
}

__device__ __forceinline__ int tile_rows(bool few) { return few ? kFew : kTileRows; }

__device__ __forceinline__ Size size_from(const PagedArgs& a, int q0, int q1, int len, int g) {
  Size s;
  s.qbase = clampi(q0, 0, a.q_cap);
  s.nq = clampi(q1, s.qbase, a.q_cap) - s.qbase;
  s.nk = clampi(len, 0, a.max_pages << a.page_log2);
  const int few = is_few(a, s.nq, s.nk, g);
  s.tiles = (s.nq * g + tile_rows(few) - 1) >> (few ? kFewLog2 : kTileLog2);
  return s;
}

__device__ __forceinline__ Size size_of(const PagedArgs& a, int b, int g) {
  return size_from(a, a.qo[b], a.qo[b + 1], a.lens[b], g);
}

// Units before the rest, of n in all that cost w, the dearest `most`.
__device__ __forceinline__ uint32_t whole_units(uint32_t n, float w, float most) {
  return most * (0.5f * kPagedPlaces) >= w ? 0 : n / kPagedPlaces * kPagedPlaces;
}

// Keys per chunk where the units that may be cut have w keys.
__device__ __forceinline__ int chunk_length(float w) {
  const float l = w * (1.0f / kPagedPlaces);
  return l > 1e9f ? 1 << 30 : (int)l + 1;
}

// May single tokens fill half of the places? (units units, w keys, the dearest `most`)
__device__ __forceinline__ bool half_places(const PagedArgs& a, int L, uint32_t units, float w, float most) {
  return L <= kMaxHalf / 2 || (L <= kMaxEven / 2 && most * (float)units <= 1.25f * w);
}

// Are the chunks of tiles counted to the nearest?
__device__ __forceinline__ bool rounds_up(const PagedArgs& a, int L) { return a.mask && L >= 2 * kMinTile; }

// A sequence's chunks (a whole number of its waves' tiles).
__device__ __forceinline__ void cut(const PagedArgs& a, const Size& s, int g, int L, bool half, bool near, int& C,
                                    int& chunk) {
  const bool few = is_few(a, s.nq, s.nk, g);
  if (few) {
    const int l = 2 * min(L, 1 << 29);  // (2^30: nothing is cut)
    // (in calls of at most kPagedFewest tiles: where a second launch adds the chunks up 12.5 us whole, 11.8 cut, at 560
    // and 630 keys; 420 and 500 keys +1.5%, 260 and 330 +10%. Single tokens, whose chunks meet in the launch: 1 to 16
    // sequences, three layouts of heads, 540 to 639 keys, bf16 9.4 to 10.0 / 8.6 to 9.2, 8 bits 10.3 to 11.0 / 9.2 to 10.5)
    const int whole = a.short_keys > kWholeFew ? 2 * kMinTile : kWholeFew;
    C = s.nk < whole ? 1 : s.nk / max(half ? 2 * l : l, kMinFew);
    if (C > kMeet && (s.nk <= kMeet * kMaxMeet || C <= kMostOver)) C = kMeet;
  } else {
    const int l = max(L, kMinTile);
    // (shorter sequences are never cut: the host may have left the workspace out)
    C = (int)(((uint32_t)s.nk + (near && s.nk >= 2 * kMinTile ? (uint32_t)l / 2 : 0)) / (uint32_t)l);
  }
  chunk = s.nk;
  if (C > 1) {
    const int unit = few ? kBK : kKT;
    chunk = (int)(((uint32_t)s.nk + C - 1) / (uint32_t)C + unit - 1) / unit * unit;
    C = (int)(((uint32_t)s.nk + chunk - 1) / (uint32_t)chunk);
  }
  if (C <= 1) {
    C = 1;
    chunk = s.nk;
  }
}

// Of a sequence whose units begin at number `first`: those that stay whole.
__device__ __forceinline__ uint32_t whole_of(const PagedArgs& a, const Size& s, uint32_t first, uint32_t whole) {
  const uint32_t n = (uint32_t)s.tiles * a.Hkv;
  return whole <= first ? 0 : min(n, whole - first);
}

// Its keys as the plan counts them, per unit.
__device__ __forceinline__ float cost_of(const PagedArgs& a, const Size& s, int g) {
  return (float)s.nk * (is_few(a, s.nq, s.nk, g) ? 0.5f : 1.0f);
}

// Its items, its partial results, the units that have such and their chunks.
struct Counts {
  uint32_t items, slots, cut;
  int C, chunk;
};
__device__ __forceinline__ Counts counts_of(const PagedArgs& a, const Size& s, int g, int L, bool half, bool near,
                                             uint32_t whole) {
  Counts c;
  cut(a, s, g, L, half, near, c.C, c.chunk);
  const uint32_t n = (uint32_t)s.tiles * a.Hkv;
  c.cut = c.C > 1 ? n - whole : 0;
  c.slots = c.cut * c.C;
  c.items = c.C > 1 ? whole + c.slots : n;
  return c;
}

struct Item {
  int b, kvh, qbase, nq, nk;
  bool few;
  int tile, chunk;   // row tile, keys per chunk
  int c, n_chunks;   // chunk of this item, of those that hold keys its rows see (1: no partial results)
  int slot;          // partial result of its first chunk
  int record;        // its unit's number among the cut ones, or -1
  int rows;          // rows of the tile
  int vis_end;       // keys that its last row sees
};

// Keys [0, row_limit) of the first `end` are seen by query qi.
__device__ __forceinline__ int row_limit(const PagedArgs& a, const Item& it, int qi, int end) {
  if (!a.causal) return end;
  return clampi(it.nk - it.nq + qi + 1, 0, end);
}

// Under a mask of bits (kTree) a row sees the keys before the sequence's new ones, and of new key j
// bit j of its words. A block of 32 keys from offset `off` among the new ones (negative: before
// them) meets words off / 32 and the next, shifted; `left` of its keys exist.
__device__ __forceinline__ uint32_t block_bits(uint32_t lo, uint32_t hi, int off, int left) {
  const uint32_t x = __builtin_amdgcn_alignbit(hi, lo, (uint32_t)off & 31);
  return left >= 32 ? x : (left <= 0 ? 0u : x & ((1u << left) - 1));
}

// A lane's row of the mask, in vector registers (no scalar ones are left).
struct MaskRow {
  const uint32_t* row;
  int words, first;  // first: the first new key
  __device__ __forceinline__ uint32_t word(int w) const { return w < 0 ? ~0u : (w < words ? row[w] : 0u); }
  // of the 32 keys from `key` on, of which `left` exist
  __device__ __forceinline__ uint32_t block(int key, int left) const {
    const int off = key - first, w = off >> 5;
    return block_bits(word(w), word(w + 1), off, left);
  }
  __device__ __forceinline__ bool sees(int key) const {
    const int off = key - first;
    return (word(off >> 5) >> (off & 31)) & 1;
  }
};
__device__ __forceinline__ MaskRow mask_row(const PagedArgs& a, const Item& it, int qi) {
  return MaskRow{a.mask + (int64_t)(it.qbase + qi) * a.mask_words, a.mask_words, it.nk - it.nq};
}

// The row `mine` behind that which a tile holds in LDS.
__device__ __forceinline__ MaskRow held_row(const char* smem, int mine) {
  MaskRow m = *reinterpret_cast<const MaskRow*>(smem + 4 * kKBytes);
  m.row += (int64_t)mine * m.words;
  return m;
}

// Does query qi, whose weights add up to l, see any key?
template <bool kTree>
__device__ __forceinline__ bool row_sees(const PagedArgs& a, const Item& it, int qi, float l) {
  if constexpr (!kTree) return row_limit(a, it, qi, it.nk) > 0;
  if (l != 0.0f || it.nk > it.nq) return true;  // (NaN too)
  const uint32_t* const row = a.mask + (int64_t)(it.qbase + qi) * a.mask_words;
  const int lo = it.nq - it.nk;  // the first bit that stands for a key
  for (int w = lo >> 5; w < a.mask_words && 32 * w < it.nq; ++w) {
    uint32_t x = block_bits(row[w], 0, 0, it.nq - 32 * w);
    if (32 * w < lo) x &= ~0u << (lo & 31);
    if (x) return true;
  }
  return false;
}

// Inclusive prefix sum over the wave (row shifts, then the rows' last lanes).
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

// Sum over the wave, in the same order in every wave (0 is what a lane without a
// neighbour adds).
__device__ __forceinline__ float wave_sum(float v) {
#define CE_STEP(ctrl, rows) \
  v += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), ctrl, rows, 0xf, false))
  CE_STEP(0x111, 0xf);
  CE_STEP(0x112, 0xf);
  CE_STEP(0x114, 0xf);
  CE_STEP(0x118, 0xf);
  CE_STEP(0x142, 0xa);
  CE_STEP(0x143, 0xc);
#undef CE_STEP
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}

// Largest of non-negative values over the wave (their bits are in order).
__device__ __forceinline__ float wave_max(float x) {
  int v = (int)__float_as_uint(x);
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane(v, 63));
}

// The sequence that holds an item, and what was counted before it.
struct Found {
  int b;
  Size size;
  int C, chunk;                // its chunks, of keys
  uint32_t whole;              // its units that stay whole
  uint32_t before, slots, cut; // items, partial results and cut units of the sequences before
};

// The sequence of item `at`; false past the last. Every wave finds it by itself, kPer
// sequences a lane. kRecord: f.cut and, past the last item too, all cut units (n_cut).
template <int kPer, bool kRecord>
__device__ __forceinline__ bool find_by_scan(const PagedArgs& a, int g, uint32_t at, Found& f, uint32_t& n_cut) {
  const int lane = threadIdx.x & 63;
  Size s[kPer];
  float w = 0.0f, most = 0.0f;
  uint32_t units = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int b = lane * kPer + i;
    s[i] = Size{0, 0, 0, 0};
    if (b < a.B) s[i] = size_of(a, b, g);
    const uint32_t n = (uint32_t)s[i].tiles * a.Hkv;
    const float c = n ? cost_of(a, s[i], g) : 0.0f;
    w += (float)n * c;
    units += n;
    most = fmaxf(most, c);
  }
  const uint32_t units_to = wave_scan(units);
  w = wave_sum(w);
  const uint32_t all = __builtin_amdgcn_readlane(units_to, 63);
  most = wave_max(most);
  const float w_all = w;
  const uint32_t whole = whole_units(all, w, most);
  if (whole) {  // what the rest costs
    float rest = 0.0f;
    uint32_t first = units_to - units;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint32_t n = (uint32_t)s[i].tiles * a.Hkv;
      rest += (float)(n - whole_of(a, s[i], first, whole)) * cost_of(a, s[i], g);
      first += n;
    }
    w = wave_sum(rest);
  }
  int L = chunk_length(w);
  bool near = kRecord && rounds_up(a, L);
  Counts n[kPer];
  uint32_t wh[kPer], sum, sum_s, sum_c, to, slots_to;
  for (;;) {
    uint32_t first = units_to - units;
    const bool half = !kRecord && half_places(a, L, all, w_all, most);  // (a call of single tokens has no records)
    sum = sum_s = sum_c = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      wh[i] = whole_of(a, s[i], first, whole);
      n[i] = counts_of(a, s[i], g, L, half, near, wh[i]);
      first += (uint32_t)s[i].tiles * a.Hkv;
      sum += n[i].items;
      sum_s += n[i].slots;
      sum_c += n[i].cut;
    }
    slots_to = wave_scan(sum_s);
    to = wave_scan(sum);
    // More workgroups than the launch has, or slots than the workspace: too many counts were
    // rounded up, so all are rounded down; or offsets are out of order, then nothing is cut (every
    // chunk of a cut unit must run) and what lies past the grid is left.
    if (L == 1 << 30 ||
        (__builtin_amdgcn_readlane(to, 63) <= a.grid && __builtin_amdgcn_readlane(slots_to, 63) <= (uint32_t)kPagedPlaces))
      break;
    if (!near) L = 1 << 30;
    near = false;
  }
  uint32_t cut_to = 0;
  if (kRecord && a.units) {
    cut_to = wave_scan(sum_c);
    n_cut = __builtin_amdgcn_readlane(cut_to, 63);
  }
  const uint64_t past = __builtin_amdgcn_ballot_w64(at < to);
  if (!past) return false;
  const int ln = __builtin_ctzll(past);
  f.before = __builtin_amdgcn_readlane(to - sum, ln);
  f.slots = __builtin_amdgcn_readlane(slots_to - sum_s, ln);
  f.cut = __builtin_amdgcn_readlane(cut_to - sum_c, ln);
  bool found = false;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const uint32_t ni = __builtin_amdgcn_readlane(n[i].items, ln);
    if (found) continue;
    if (i == kPer - 1 || at < f.before + ni) {
      found = true;
      f.b = ln * kPer + i;
      f.size.qbase = __builtin_amdgcn_readlane(s[i].qbase, ln);
      f.size.nq = __builtin_amdgcn_readlane(s[i].nq, ln);
      f.size.nk = __builtin_amdgcn_readlane(s[i].nk, ln);
      f.size.tiles = __builtin_amdgcn_readlane(s[i].tiles, ln);
      f.whole = __builtin_amdgcn_readlane(wh[i], ln);
      f.C = __builtin_amdgcn_readlane(n[i].C, ln);
      f.chunk = __builtin_amdgcn_readlane(n[i].chunk, ln);
    } else {
      f.before += ni;
      f.slots += __builtin_amdgcn_readlane(n[i].slots, ln);
      f.cut += __builtin_amdgcn_readlane(n[i].cut, ln);
    }
  }
  return true;
}

// The same from the plan in memory: three rounds of 64 samples.
__device__ __forceinline__ bool find_in_plan(const PagedArgs& a, int g, uint32_t at, Found& f) {
  const int lane = threadIdx.x & 63;
  auto key = [&](int b) __attribute__((always_inline)) { return a.plan[b].items; };
  if (at >= key(a.B)) return false;
  int lo = 0;  // the last sequence whose count begins at or before `at` is in [lo, lo + 64 step)
#pragma unroll
  for (int step = 4096; step > 0; step >>= 6) {
    const int i = lo + lane * step;
    const bool le = i < a.B && key(i < a.B ? i : 0) <= at;
    const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(le));
    lo += (n > 0 ? n - 1 : 0) * step;
  }
  f.b = __builtin_amdgcn_readfirstlane(lo);
  f.before = __builtin_amdgcn_readfirstlane(key(f.b));
  f.slots = __builtin_amdgcn_readfirstlane(a.plan[f.b].slots);
  f.cut = __builtin_amdgcn_readfirstlane(a.plan[f.b].cut);
  f.whole = __builtin_amdgcn_readfirstlane(a.plan[f.b].whole);
  const int L = __builtin_amdgcn_readfirstlane((int)a.plan[a.B].whole);
  const uint32_t flags = __builtin_amdgcn_readfirstlane(a.plan[a.B].slots);
  const Size s = size_of(a, f.b, g);
  f.size.qbase = __builtin_amdgcn_readfirstlane(s.qbase);
  f.size.nq = __builtin_amdgcn_readfirstlane(s.nq);
  f.size.nk = __builtin_amdgcn_readfirstlane(s.nk);
  f.size.tiles = __builtin_amdgcn_readfirstlane(s.tiles);
  cut(a, f.size, g, L, flags & 1, flags & 2, f.C, f.chunk);
  f.C = __builtin_amdgcn_readfirstlane(f.C);
  f.chunk = __builtin_amdgcn_readfirstlane(f.chunk);
  return true;
}

// Item `at`; false if there is none, or its rows see no key of it. kRecord: the item's
// record number, and the first item's wave leaves the number of the records.
template <bool kRecord>
__device__ __forceinline__ bool find_item(const PagedArgs& a, uint32_t at, Item& it) {
  const int g = a.g;
  Found f;
  uint32_t n_cut = 0;
  bool found;
  if (a.B <= kPagedScan) {
    found = a.B <= 64 ? find_by_scan<1, kRecord>(a, g, at, f, n_cut)
                      : find_by_scan<kPagedScan / 64, kRecord>(a, g, at, f, n_cut);
    if (kRecord && at == 0 && threadIdx.x == 0 && a.units) *a.units = n_cut;
  } else {
    found = find_in_plan(a, g, at, f);  // (the plan's launch has left the number)
  }
  if (!found) return false;
  it.b = f.b;
  it.qbase = f.size.qbase;
  it.nq = f.size.nq;
  it.nk = f.size.nk;
  it.few = is_few(a, it.nq, it.nk, g);
  int C = f.C;
  it.chunk = f.chunk;
  uint32_t u = at - f.before;
  it.c = 0;
  it.slot = 0;
  it.record = -1;
  if (C > 1 && u >= f.whole) {
    // all units' first chunks, then their second: neighbours read the same keys
    const uint32_t v = u - f.whole, n = (uint32_t)f.size.tiles * a.Hkv - f.whole;
    it.c = (int)(v / n);
    const uint32_t back = v - it.c * n;
    it.slot = (int)(f.slots + back * C);
    if (kRecord) it.record = (int)(f.cut + back);
    u = f.whole + back;
  } else {
    C = 1;
    it.chunk = it.nk;
  }
  it.kvh = f.size.tiles == 1 ? (int)u : (int)(u / (uint32_t)f.size.tiles);
  it.tile = f.size.tiles - 1 - (int)(u - (uint32_t)it.kvh * f.size.tiles);
  const int r0 = it.tile * tile_rows(it.few);
  it.rows = min(tile_rows(it.few), it.nq * g - r0);
  it.vis_end = row_limit(a, it, (r0 + it.rows - 1) / g, it.nk);
  if (!it.few && a.mask && a.mask_words > kWideMask) {
    // the last new key that some row of the tile sees (masks of trees are too short for it to pay)
    const int q0 = r0 / g, words = a.mask_words, n = ((r0 + it.rows - 1) / g - q0 + 1) * words;
    const uint32_t* const p = a.mask + (int64_t)(it.qbase + q0) * words;
    int top = 0;  // behind it
    for (int k = threadIdx.x & 63; k < n; k += 64) {
      const uint32_t x = p[k];
      if (x) top = max(top, 32 * (k % words) + 32 - __builtin_clz(x));
    }
    top = (int)__float_as_uint(wave_max(__uint_as_float((uint32_t)top)));
    it.vis_end = clampi(it.nk - it.nq + min(top, it.nq), 0, it.nk);
  }
  it.n_chunks = C > 1 ? max(1, (int)(((uint32_t)it.vis_end + it.chunk - 1) / (uint32_t)it.chunk)) : 1;
  // (all of it is the wave's, but the divisions leave it in vector registers)
  for (int* const p : {&it.kvh, &it.tile, &it.chunk, &it.c, &it.n_chunks, &it.slot, &it.record, &it.rows, &it.vis_end})
    *p = __builtin_amdgcn_readfirstlane(*p);
  return it.c < it.n_chunks;
}

// What the launch that adds chunks up needs of a cut unit, written by its first chunk's
// workgroup: planning it once more took that launch 2 us of 5.
__device__ __forceinline__ u32x4_t* record_at(const PagedArgs& a, int n) {
  return reinterpret_cast<u32x4_t*>(a.units) + kPagedRecord / 16 * (n + 1);  // (behind their number)
}
__device__ __forceinline__ void write_record(const PagedArgs& a, const Item& it) {
  u32x4_t* const r = record_at(a, it.record);
  r[0] = u32x4_t{(uint32_t)it.qbase, (uint32_t)it.nq, (uint32_t)it.nk, (uint32_t)it.kvh};
  r[1] = u32x4_t{(uint32_t)it.tile, (uint32_t)it.slot, (uint32_t)it.n_chunks, (uint32_t)it.rows << 1 | (it.few ? 1 : 0)};
}
__device__ __forceinline__ void read_record(const PagedArgs& a, int n, Item& it) {
  const u32x4_t* const r = record_at(a, n);
  const u32x4_t x = r[0], y = r[1];
  it.qbase = __builtin_amdgcn_readfirstlane(x.x);
  it.nq = __builtin_amdgcn_readfirstlane(x.y);
  it.nk = __builtin_amdgcn_readfirstlane(x.z);
  it.kvh = __builtin_amdgcn_readfirstlane(x.w);
  it.tile = __builtin_amdgcn_readfirstlane(y.x);
  it.slot = __builtin_amdgcn_readfirstlane(y.y);
  it.n_chunks = __builtin_amdgcn_readfirstlane(y.z);
  const uint32_t w = __builtin_amdgcn_readfirstlane(y.w);
  it.rows = (int)(w >> 1);
  it.few = w & 1;
}

// ------------------------------------------------------- softmax and results

// Scale of raw scores in the exponent: softmax scale times log2 e, times that of 8-bit keys
// (ks). Both may be any positive float, their product may be none: 0 would make NaN of a masked
// score (-inf 0), and infinity one of a score of zero. The least and the largest float
// stand in for them: under the first, raw scores, below 2^128, weigh alike to within 2^-20;
// under the second, raw scores that differ at all (by 1e-36 and more, where they are normal
// floats) differ by more than the exponent holds, as they do under the product.
// (bf16: the host has seen to it, and the value stays a scalar.)
__device__ __forceinline__ float score_scale(const PagedArgs& a, int kvh) {
  if (!a.ks) return a.scale_log2;
  const float c = a.scale_log2 * a.ks[kvh];
  return c < 0x1p-149f ? 0x1p-149f : (c > 0x1.fffffep127f ? 0x1.fffffep127f : c);
}

// Weight of a partial result with maximum m under the maximum m_all (raw scores;
// c2: their scale times log2 e). Without any finite maximum it counts nothing,
// except that NaN times 0 stays NaN.
__device__ __forceinline__ float weight(float m, float m_all, float c2) {
  return m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((m - m_all) * c2);
}

// Outputs are sum * normalizer * scale of the values, in this order: scale / l could be a
// float of a few bits (a scale of 1e-38 and 600000 keys). A row that sees no key is zero, one
// that sees only scores of -infinity is 0 / 0.
__device__ __forceinline__ float normalizer(float l, bool sees) {
  return sees ? 1.0f / l : 0.0f;
}

// Partial results of the chunks of a unit meet through the workspace, in chunk order,
// so no result depends on who came first. In the launch itself: each chunk's
// workgroup writes its own and arrives; the last of a group of neighbours adds the
// group up and goes on as one chunk of the next level. Nobody waits for anybody. The
// sums move by device-coherent (sc1) stores and loads, and a workgroup arrives when
// its stores have completed, so no cache is written back or dropped.
constexpr int kSC1 = 16;            // cache-policy operand: sc1
// A slot: outputs of its rows, then their maxima, then their sums.
template <bool kDecode>
constexpr uint32_t kSlotRows = kDecode ? kFew : kTileRows;
template <bool kDecode>
constexpr uint32_t kSlotBytes = kSlotRows<kDecode> * (kDh + 2) * 4;
template <bool kDecode>
constexpr uint32_t kStats = kSlotRows<kDecode> * kDh * 4;

template <bool kDecode>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t part_rsrc(const PagedArgs& a) {
  return make_rsrc(a.part, kPagedPlaces * kSlotBytes<kDecode>);
}
__device__ __forceinline__ void part_store4(__amdgpu_buffer_rsrc_t rs, uint32_t at, float x, float y, float z, float w) {
  const u32x4_t v = {__float_as_uint(x), __float_as_uint(y), __float_as_uint(z), __float_as_uint(w)};
  __builtin_amdgcn_raw_buffer_store_b128(v, rs, (int)at, 0, kSC1);
}
__device__ __forceinline__ void part_store(__amdgpu_buffer_rsrc_t rs, uint32_t at, float x) {
  __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), rs, (int)at, 0, kSC1);
}
__device__ __forceinline__ f32x4_t part_load4(__amdgpu_buffer_rsrc_t rs, uint32_t at) {
  return __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)at, 0, kSC1));
}
__device__ __forceinline__ float part_load(__amdgpu_buffer_rsrc_t rs, uint32_t at) {
  return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, (int)at, 0, kSC1));
}

// A counter of arrivals holds the call's token above their number. Any other content,
// whatever the workspace held before, counts as none. The last to arrive leaves zero, and a
// group of one, where nobody arrives, the token with no arrivals: so a captured call may
// replay with the same token. This exchange of zero for the token, made long before the
// arrival, is all that most calls need; what it found instead of zero (the token, or
// anything) is returned.
__device__ __forceinline__ unsigned long long expect_arrivals(const PagedArgs& a, int i) {
  unsigned long long was = 0;
  if (threadIdx.x == 0)
    __hip_atomic_compare_exchange_strong(a.arrived + i, &was, a.token << 16, __ATOMIC_RELAXED, __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT);
  return was;
}

// This workgroup's stores are complete and it arrives at counter `i`, where
// expect_arrivals found `was`: is it the last of n? One addition, and where memory held
// something else one exchange before it; sixteen that exchanged until it went well
// took 8 us. `said`: a word of LDS that nobody else uses meanwhile.
__device__ __forceinline__ bool arrive_last(const PagedArgs& a, int i, int n, unsigned long long was, int* said) {
  asm volatile("" ::: "memory");
  wait_vmcnt<0>();
  __syncthreads();
  if (threadIdx.x == 0) {
    unsigned long long* const p = a.arrived + i;
    if (was != 0 && (was >> 16) != a.token)  // (if it fails, another has put the token there)
      __hip_atomic_compare_exchange_strong(p, &was, a.token << 16, __ATOMIC_RELAXED, __ATOMIC_RELAXED,
                                           __HIP_MEMORY_SCOPE_AGENT);
    was = __hip_atomic_fetch_add(p, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const bool last = (int)(was & 0xffff) == n - 1;
    if (last) __hip_atomic_store(p, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *said = last;
  }
  __syncthreads();
  const bool last = __builtin_amdgcn_readfirstlane(*said) != 0;
  __syncthreads();  // read by every wave before it is used again
  return last;
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

// x / g for 0 <= x < kTileRows + g, g <= 4096: off by at most 2^-22 x / g, while x + 1/2
// is at least 1 / (2 g) from a multiple.
__device__ __forceinline__ int small_div(int x, float inv_g) { return (int)(((float)x + 0.5f) * inv_g); }

template <bool kF8>
constexpr int kPageRow = kF8 ? kDh : kRowB;  // bytes of a row of a page

// Head kvh of page number `page` of sequence b; `ok` false: not a page of the pool.
template <bool kF8>
__device__ __forceinline__ int64_t page_at(const PagedArgs& a, int kvh, int page, bool& ok) {
  ok = (uint32_t)page < (uint32_t)a.n_pages;
  return (int64_t)((uint64_t)(uint32_t)(ok ? page : 0) * a.page_bytes) + ((uint32_t)kvh << a.page_log2) * kPageRow<kF8>;
}

// Output of a wave's 32 rows again, key by key, with maxima and sums of its own: the scores
// that it forms differ from those of the matrix instructions in their rounding, which at a score
// of 1e6 is a tenth and more of the exponent. Keys k0 + n kstep + 0 .. 31 below vis1, a
// lane's row sees those below vis. qf: the row, 8 dims a chunk, chunk s from dim
// 8 (2 s + lane / 32), or with kWide from 16 (2 (s / 2) + lane / 32) + 8 (s % 2). Slow, and
// reached only where a value is NaN or infinite in a sequence's last rows.
// kTree: and that `row` shows.
template <bool kF8, bool kWide, bool kTree>
__device__ __forceinline__ void paged_redo(const PagedArgs& a, int b, int kvh, const u32x4_t (&qf)[8], f32x16_t (&oacc)[4],
                                        float& m, float& l, float c2, int vis, int k0, int kstep, int vis1,
                                        const MaskRow& row) {
  int lhalf = (threadIdx.x >> 5) & 1;
  asm volatile("" : "+v"(lhalf));  // no address of this path is formed before it
  const int mask = (1 << a.page_log2) - 1;
  m = -__builtin_inff();
  l = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) oacc[i] = f32x16_t{};
  for (; k0 < vis1; k0 += kstep)
    for (int j = k0; j < min(k0 + 32, vis1); ++j) {
      bool ok;
      const int page = __builtin_amdgcn_readfirstlane(a.table[(int64_t)b * a.max_pages + (j >> a.page_log2)]);
      const int64_t at = page_at<kF8>(a, kvh, page, ok) + (int64_t)(j & mask) * kPageRow<kF8>;
      const char* const kp = a.k + at + lhalf * (kF8 && !kWide ? 8 : 16);
      const char* const vp = a.v + at + lhalf * (kF8 ? 4 : 8);
      auto lo = [](uint32_t x) __attribute__((always_inline)) { return __uint_as_float(x << 16); };
      auto hi = [](uint32_t x) __attribute__((always_inline)) { return __uint_as_float(x & 0xffff0000u); };
      float sc = 0.0f;
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        u32x4_t x = {0, 0, 0, 0};  // the 8 values that meet chunk s of the row
        if constexpr (kF8) {
          u32x2_t y = {0, 0};
          if (ok) y = *reinterpret_cast<const u32x2_t*>(kp + (kWide ? (s >> 1) * 32 + (s & 1) * 8 : s * 16));
          const u32x2_t e = e4m3_to_bf16(y.x), f = e4m3_to_bf16(y.y);
          x = u32x4_t{e.x, e.y, f.x, f.y};
        } else if (ok) {
          x = *reinterpret_cast<const u32x4_t*>(kp + s * 32);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) sc = fmaf(hi(qf[s][e]), hi(x[e]), fmaf(lo(qf[s][e]), lo(x[e]), sc));
        __builtin_amdgcn_sched_barrier(0);  // (few registers are left)
      }
      sc += __shfl_xor(sc, 32);
      bool sees = j < vis;
      if constexpr (kTree) sees = sees && row.sees(j);
      if (sees) {
        const float m_new = fmaxf(m, sc);
        if (m_new > m) {
          const float al = weight(m, m_new, c2);
          l *= al;
#pragma unroll
          for (int i = 0; i < 4; ++i) oacc[i] *= al;
          m = m_new;
        }
        const float p = __builtin_amdgcn_exp2f((m == -__builtin_inff() ? sc : sc - m) * c2);
        l += p;
        if (!ok) continue;  // (values of zero)
#pragma unroll
        for (int v = 0; v < 16; ++v) {  // dims 8 v + 4 lhalf .. +3
          u32x2_t x;
          if constexpr (kF8)
            x = e4m3_to_bf16(*reinterpret_cast<const uint32_t*>(vp + v * 8));
          else
            x = *reinterpret_cast<const u32x2_t*>(vp + v * 16);
          f32x16_t& o = oacc[v >> 2];
          const int r = 4 * (v & 3);
          o[r] = fmaf(p, lo(x.x), o[r]);
          o[r + 1] = fmaf(p, hi(x.x), o[r + 1]);
          o[r + 2] = fmaf(p, lo(x.y), o[r + 2]);
          o[r + 3] = fmaf(p, hi(x.y), o[r + 3]);
          __builtin_amdgcn_sched_barrier(0);
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

// Buffer over a wave's rows. A size that a vector instruction gave (a clamp has no
// scalar one) would make every load through it a loop over the lanes' buffers
// (4 x 2176 queries over 2304 keys: 148 us with such loops, 140 without).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t wave_rsrc(const void* base, uint32_t bytes) {
  return make_rsrc(base, (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes));
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
// end. Bound: memory, so a wave keeps its next tile's keys and values in flight.
//   * bf16: whole lines by DMA into LDS of the wave's own, in the layout of
//     paged_tile; a tile's fragments are read into registers at once, and the next
//     tile's DMA takes their place. (Fragments loaded straight from memory read a line
//     of 128 bytes in four instructions, and the line is gone from the cache between
//     them: one token over 65537 keys 36 us, by DMA 33, 4.1 TB/s with start and end.)
//   * 8-bit: K straight to registers in operand order (a line in four loads as well,
//     but half the bytes: 64 tokens over 2100 to 16001 keys 78 us, 4.95 TB/s), V through
//     registers, converted, exactly, and stored transposed in LDS.
template <bool kF8, bool kDecode, bool kTree>
__device__ __forceinline__ void paged_few(const PagedArgs& a, char* const smem, const Item& it) {
  float* const ml = reinterpret_cast<float*>(smem + 4 * kFew * kOLd * 4);  // [2][4][kFew]
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = a.g;
  const int kvh = it.kvh;
  const int pl = a.page_log2, mask = (1 << pl) - 1;
  const float c2 = kF8 ? score_scale(a, kvh) : a.scale_log2;
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
  const int q0 = it.tile * kFew / g, h0 = it.tile * kFew - q0 * g;  // of the tile's first row
  const int rr = h0 + min(lrow, rows - 1);
  const int dq = small_div(rr, 1.0f / (float)g);
  const int qi = q0 + dq;
  const int hq = kvh * g + (rr - dq * g);
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
  const int vis0 = kTree ? clampi(it.nk - it.nq, 0, kend) : row_limit(a, it, q0, kend);  // by the first row (or every one)
  const int vis1 = min(it.vis_end, kend);                  // and by the last
  MaskRow mrow = {nullptr, 0, 0};
  uint32_t word0 = 0;   // of the mask; as a rule the only one: 32 rows, so 32 new keys at most
  uint32_t some = ~0u;  // bit r: row r sees some key
  if constexpr (kTree) {
    mrow = mask_row(a, it, qi);
    asm volatile("" : "+v"(mrow.words), "+v"(mrow.first));
    word0 = mrow.row[0];
    some = (uint32_t)__builtin_amdgcn_ballot_w64(row_sees<true>(a, it, qi, 0.0f));
    asm volatile("" : "+v"(some));
  }

  char* const vt = smem + wave * (kF8 ? kVTile : 2 * kVTile);  // bf16: K tile, then V tile
  typedef __attribute__((address_space(3))) char lds_char;
  lds_char* ring = (lds_char*)vt;
  asm volatile("" : "+s"(ring));  // (see paged_tile)
  const int vkg = lane & 7;   // 8-bit: keys 4 vkg .. +3 of the tile
  const int vdg = lane >> 3;  // values 16 vdg .. +15 of a row
  u32x4_t kf[kF8 ? 4 : 8], vr[kF8 ? 4 : 8];
  int64_t at0, at1;             // pages of the two halves of the tile to fetch
  bool ok0 = true, ok1 = true;  // (8-bit: of the tile in flight)
  int tile_n = 0;               // in the page numbers at hand
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
  // bf16: 16 keys of one page by four DMAs; rows behind the sequence's end, and
  // all of a page that is none, come as zeros
  const int kr_sub = lane >> 4, kpc = lane & 15;
  uint32_t kvo[4], vvo = 0, koff = 0, voff[4];
  if constexpr (!kF8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) kvo[i] = (uint32_t)((4 * i + kr_sub) * kRowB + ((kpc ^ (4 * i + kr_sub)) << 4));
    vvo = (uint32_t)(kr_sub * kRowB + ((kpc ^ (kr_sub << 2)) << 4));
    koff = (uint32_t)(lrow * kRowB + ((lhalf ^ (lrow & 15)) << 4));  // K chunk 2 s + lhalf: ^ (s << 5)
#pragma unroll
    for (int db = 0; db < 4; ++db) {
      const int key = (lane >> 2) & 3;
      const int c = ((db ^ key) << 2) + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      voff[db] = (uint32_t)(kVTile + (4 * lhalf + key) * kRowB + (c << 4) + 8 * (lane & 1));
    }
  }
  auto half_rsrc = [&](const char* pool, int k0, int h) __attribute__((always_inline)) {
    const int key = k0 + 16 * h;
    const int n = (h ? ok1 : ok0) ? clampi(it.nk - key, 0, 16) : 0;
    return wave_rsrc(pool + (h ? at1 : at0) + (uint32_t)(key & mask) * kRowB, (uint32_t)(n * kRowB));
  };
  // 8-bit: keys past the sequence's end read its last one (their scores are replaced)
  auto row_at = [&](int k0, int kk) __attribute__((always_inline)) {
    const int key = min(k0 + kk, it.nk - 1);
    return (key - k0 >= 16 ? at1 : at0) + (int64_t)(key & mask) * kPageRow<kF8>;
  };
  auto load_k = [&](int k0) __attribute__((always_inline)) {
    if constexpr (kF8) {
      const char* p = a.k + row_at(k0, lrow) + lhalf * 16;
#pragma unroll
      for (int s = 0; s < 4; ++s) kf[s] = *reinterpret_cast<const u32x4_t*>(p + s * 32);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const __amdgpu_buffer_rsrc_t rs = half_rsrc(a.k, k0, h);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, ring + (16 * h + 4 * i) * kRowB, 16, (int)kvo[i], 0, 0, 0);
      }
    }
  };
  auto load_v = [&](int k0) __attribute__((always_inline)) {
    if constexpr (kF8) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        vr[i] = *reinterpret_cast<const u32x4_t*>(a.v + row_at(k0, 4 * vkg + i) + vdg * 16);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const __amdgpu_buffer_rsrc_t rs = half_rsrc(a.v, k0, h);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, ring + kVTile + (16 * h + 4 * i) * kRowB, 16, (int)vvo,
                                                   4 * i * kRowB, 0, 0);
      }
    }
  };

  unsigned long long was = 0;
  if (kDecode && it.n_chunks > 1) was = expect_arrivals(a, it.slot + it.c / kMeet * kMeet);

  f32x16_t oacc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) oacc[i] = f32x16_t{};
  float m_run = -__builtin_inff(), l_run = 0.0f;
  float mc_run = 0.0f;  // exponent of m_run
  bool far = false;     // that of some row is far

  const int step = 4 * kBK;
  int k0 = kbeg + wave * kBK;
  if (k0 < vis1) {
    next_pages(k0);
    load_k(k0);
    load_v(k0);
  }
  for (; k0 < vis1; k0 += step) {
    const bool more = k0 + step < vis1;
    if (kF8 && !(ok0 && ok1)) {  // a page that is none reads as zeros
      const bool kz = (lrow >= 16 && k0 + 16 < it.nk) ? !ok1 : !ok0;
      const bool vz = (vkg >= 4 && k0 + 16 < it.nk) ? !ok1 : !ok0;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
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
      if (more) {
        next_pages(k0 + step);
        load_k(k0 + step);
      }
    } else {
      wait_vmcnt<8>();  // K is there, V still comes
      asm volatile("" ::: "memory");
#pragma unroll
      for (int s = 0; s < 8; ++s) kf[s] = lds_read16(vt, (int)(koff ^ (s << 5)));
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read before the next tile takes its place
      if (more) {
        next_pages(k0 + step);
        load_k(k0 + step);
      }
#pragma unroll
      for (int s = 0; s < 8; s += 2) {
        mfma_step<true>(sc, kf[s], qf[s]);
        mfma_step<true>(s2, kf[s + 1], qf[s + 1]);
      }
    }
    sc += s2;
    if (k0 + kBK > vis0) {
      if constexpr (kTree) {
        const int off = k0 - mrow.first, w = off >> 5;
        const uint32_t lo = w == 0 ? word0 : mrow.word(w), hi = w == -1 ? word0 : mrow.word(w + 1);
        const uint32_t bits = block_bits(lo, hi, off, vis - k0) >> (4 * lhalf);
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (!(bits >> (8 * (v >> 2) + (v & 3)) & 1)) sc[v] = -__builtin_inff();
      } else {
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (k0 + 8 * (v >> 2) + 4 * lhalf + (v & 3) >= vis) sc[v] = -__builtin_inff();
      }
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
      mc_run = exponent_of(m_run, c2);
      far = any_far(mc_run);
    }
    float mc = mc_run, ce = c2;
    if (far) far_scores(sc, m_run, c2, mc, ce);
    float rs = 0.0f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      sc[v] = __builtin_amdgcn_exp2f(fmaf(sc[v], ce, -mc));
      rs += sc[v];
    }
    l_run += rs + __shfl_xor(rs, 32);
    // The weights become bf16 here, the type of the values (or of what 8-bit values become
    // exactly), since the matrix instructions take one type: half a step, 2^-8 of each weight.
    // Their sum keeps the unrounded ones. Error of a whole output against 64 bits, relative
    // to its size: 0.0021 to 0.0024, with weights of 32 bits 0.0017, which is the output's
    // own rounding; a second product with what is left of them would close that for half as
    // many instructions again. paged_tile does the same.
    u32x4_t pf[2];
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int i = 0; i < 4; ++i) pf[st][i] = pack_bf16(sc[8 * st + 2 * i], sc[8 * st + 2 * i + 1]);
    // O^T += V^T P^T over 2 steps of 16 keys, in the scores' key order
    if constexpr (kF8) {
      // V tile to LDS, transposed (a wave's own tile: its LDS operations are in
      // order, so no barrier)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        u32x2_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = e4m3_to_bf16(vr[i][w]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
          *reinterpret_cast<u32x2_t*>(vt + vt_off(16 * vdg + 4 * w + e, (uint32_t)vkg)) =
              u32x2_t{__builtin_amdgcn_perm(y[1][e >> 1], y[0][e >> 1], sel),
                      __builtin_amdgcn_perm(y[3][e >> 1], y[2][e >> 1], sel)};
        }
      }
      if (more) load_v(k0 + step);
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int db = 0; db < 4; ++db) {
          const u32x2_t lo = *reinterpret_cast<const u32x2_t*>(vt + vt_off(32 * db + lrow, (uint32_t)(4 * st + lhalf)));
          const u32x2_t hi =
              *reinterpret_cast<const u32x2_t*>(vt + vt_off(32 * db + lrow, (uint32_t)(4 * st + lhalf + 2)));
          mfma_step<true>(oacc[db], u32x4_t{lo.x, lo.y, hi.x, hi.y}, pf[st]);
        }
    } else {
      if (more)
        wait_vmcnt<8>();  // V is there, the next K still comes
      else
        wait_vmcnt<0>();
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const char* const p = vt + voff[i & 3] + 16 * (i >> 2) * kRowB;
        const u32x2_t lo = lds_read_tr(p), hi = lds_read_tr(p + 8 * kRowB);
        vr[i] = u32x4_t{lo.x, lo.y, hi.x, hi.y};
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) load_v(k0 + step);
#pragma unroll
      for (int i = 0; i < 8; ++i) mfma_step<true>(oacc[i & 3], vr[i], pf[i >> 2]);
    }
  }
  if (vis0 < vis1 && any_nan(oacc))
    paged_redo<kF8, kF8, kTree>(a, it.b, kvh, qf, oacc, m_run, l_run, c2, vis, kbeg + wave * kBK, step, vis1, mrow);

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
  const float vs = kF8 && a.vs ? a.vs[kvh] : 1.0f;
  // thread: rows tid / 32 (+ 8, 16, 24), dims 4 (tid % 32) .. +3
  const int qd = tid_e & 31, r_first = tid_e >> 5;
  const __amdgpu_buffer_rsrc_t prs = part_rsrc<kDecode>(a);
  auto finish = [&](int r, const f32x4_t& x, float l) __attribute__((always_inline)) {
    const int q2 = small_div(h0 + r, 1.0f / (float)g);
    const float inv = normalizer(l, kTree ? (some >> r & 1) != 0 : row_limit(a, it, q0 + q2, it.nk) > 0);
    store4<true>(a.o + ((int64_t)(it.qbase + q0 + q2) * a.H + kvh * g + (h0 + r - q2 * g)) * kRowB + 8 * qd, x[0] * inv * vs,
                 x[1] * inv * vs, x[2] * inv * vs, x[3] * inv * vs);
  };
  auto keep = [&](int slot, int r, const f32x4_t& x, float m, float l) __attribute__((always_inline)) {
    const uint32_t at = (uint32_t)slot * kSlotBytes<kDecode>;
    part_store4(prs, at + r * (kDh * 4) + qd * 16, x[0], x[1], x[2], x[3]);
    if (qd == 0) {
      part_store(prs, at + kStats<kDecode> + r * 4, m);
      part_store(prs, at + kStats<kDecode> + (kSlotRows<kDecode> + r) * 4, l);
    }
  };
  for (int r = r_first; r < rows; r += 8) {
    float mr = ml[r], lr = 0.0f;
#pragma unroll
    for (int w = 1; w < 4; ++w) mr = fmaxf(mr, ml[w * kFew + r]);
    f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      lr = fmaf(ml[(4 + w) * kFew + r], weight(ml[w * kFew + r], mr, c2), lr);
      x += *reinterpret_cast<const f32x4_t*>(ob + (w * kFew + r) * kOLd + 4 * qd);
    }
    if (it.n_chunks > 1)
      keep(it.slot + it.c, r, x, mr, lr);
    else
      finish(r, x, lr);
  }
  if constexpr (!kDecode) return;
  // ---- the chunks meet, 16 at a time, eight rows at a time; all their loads are in
  //      flight together (always sixteen, some of them twice, made 16 tokens over 551
  //      to 3100 keys 14.4 us instead of 14.0) ----
  int n = it.n_chunks, idx = it.c, stride = 1;
  for (int level = 0; n > 1; ++level) {
    const int first = idx / kMeet * kMeet, size = min(kMeet, n - first);
    const int slot = it.slot + first * stride;
    n = (n + kMeet - 1) / kMeet;
    idx /= kMeet;
    if (size > 1) {
      const int at = level * kPagedPlaces + slot;
      if (level > 0) was = expect_arrivals(a, at);
      if (!arrive_last(a, at, size, was, reinterpret_cast<int*>(ml))) return;
      int slot_v = slot;
      asm volatile("" : "+v"(slot_v));  // (sixteen offsets in scalar registers are too many)
      auto meet = [&](auto n_c, int rb) __attribute__((always_inline)) {
        constexpr int kN = decltype(n_c)::value;
        const int r = min(rb + r_first, rows - 1);
        f32x4_t y[kN];
        float mc[kN], lc[kN];
#pragma unroll
        for (int i = 0; i < kN; ++i) {
          const uint32_t at = (uint32_t)(slot_v + min(i, size - 1) * stride) * kSlotBytes<kDecode>;
          y[i] = part_load4(prs, at + r * (kDh * 4) + qd * 16);
          mc[i] = part_load(prs, at + kStats<kDecode> + r * 4);
          lc[i] = part_load(prs, at + kStats<kDecode> + (kSlotRows<kDecode> + r) * 4);
        }
        f32x4_t x = {0.0f, 0.0f, 0.0f, 0.0f};
        float m = -__builtin_inff(), l = 0.0f;
#pragma unroll
        for (int i = 0; i < kN; ++i) m = fmaxf(m, mc[i]);
#pragma unroll
        for (int i = 0; i < kN; ++i)
          if (i < size) {
            const float wi = weight(mc[i], m, c2);
            l = fmaf(lc[i], wi, l);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = fmaf(y[i][e], wi, x[e]);
          }
        if (rb + r_first < rows) {
          if (n > 1)
            keep(slot, r, x, m, l);
          else
            finish(r, x, l);
        }
      };
      for (int rb = 0; rb < rows; rb += 8)
        if (size <= kMeet / 4)
          meet(std::integral_constant<int, kMeet / 4>{}, rb);
        else if (size <= kMeet / 2)
          meet(std::integral_constant<int, kMeet / 2>{}, rb);
        else
          meet(std::integral_constant<int, kMeet>{}, rb);
    }
    stride *= kMeet;
  }
}

// ---------------------------------------------------------------- 128-row tiles

// 128 rows (32 a wave) against a chunk of keys, in tiles of 64:
//   * S^T = K Q^T on MFMA 32x32x16 (keys are the A operand, the wave's rows the B
//     operand, in registers for the whole loop), so each lane owns one row: its 16
//     scores of a block of 32 keys sit in the lane and the other 16 in lane l ^ 32;
//   * the probabilities (bf16, in operand order; the rounding: paged_few) times V^T, with
//     the key index of that product permuted to match the score accumulators;
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
// Bound: MFMA and the softmax's VALU about alike (four chunks of 2048 queries over 7000
// to 10240 keys, 28 heads, causal: 887 us, 1.07 PFLOP/s, MFMA busy 65% of the time
// and VALU 60%; 4 x 2176 queries over 2304 keys, 12 heads: 134 us, 0.92). 64 rows a
// wave, with half the LDS reads, leave one wave a SIMD: 986 and 161.
template <bool kF8, bool kTree>
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
  const int g = a.g;
  const float inv_g = 1.0f / (float)g;
  const int kvh = it.kvh;
  const int pl = a.page_log2, mask_p = (1 << pl) - 1;
  const float c2 = kF8 ? score_scale(a, kvh) : a.scale_log2;
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
  const int r0 = it.tile * kTileRows;
  const int q0 = r0 / g;         // first query, and the first row's place in its group
  const int h0 = r0 - q0 * g;

  // ---- page numbers: lane l holds that of this wave's 16 keys of the tile from tb on
  //      whose number is l modulo 64 ----
  const int32_t* const table = a.table + (int64_t)it.b * a.max_pages;
  int tb = 0, pages = 0;
  auto load_pages = [&](int tile) __attribute__((always_inline)) {
    tb = tile;
    const int64_t key = (int64_t)kbeg + (int64_t)(tile + ((lane - tile) & 63)) * kKT + 16 * wave;
    pages = key < it.nk ? table[key >> pl] : -1;
  };
  load_pages(0);
  // where a tile's 16 keys of this wave lie in the pools, and their bytes
  struct Rows {
    int64_t at;
    uint32_t bytes;
  };
  auto rows_of = [&](int tile) __attribute__((always_inline)) {
    const int key = kbeg + tile * kKT + 16 * wave;
    bool ok;
    Rows r;
    r.at = page_at<kF8>(a, kvh, __builtin_amdgcn_readlane(pages, tile & 63), ok) +
           (uint32_t)(key & mask_p) * kPageRow<kF8>;
    r.bytes = ok ? (uint32_t)clampi(it.nk - key, 0, 16) * kPageRow<kF8> : 0;
    return r;
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
  auto fetch_k = [&](const Rows& x, int buf) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rs = wave_rsrc(a.k + x.at, x.bytes);
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
  auto fetch_v = [&](const Rows& x, int buf) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rs = wave_rsrc(a.v + x.at, x.bytes);
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
  float mc_run = 0.0f;  // exponent of m_run
  bool far = false;     // that of some row is far
  const int qi = q0 + small_div(h0 + min(32 * wave + lrow, it.rows - 1), inv_g);  // this lane's query
  const int vis = row_limit(a, it, qi, kend);  // keys [0, vis) are seen
  // by the wave's first row (or every one)
  const int vis0 =
      kTree ? clampi(it.nk - it.nq, 0, kend) : row_limit(a, it, __builtin_amdgcn_readfirstlane(qi), kend);
  // Masks of the blocks of 32 keys from the first that is not all seen on, for the tile's queries, lie in
  // LDS behind the keys and values: a load from memory in the key loop would take its latency, for every
  // block of new keys. `held`: the place of the lane's block 0, far below zero where they do
  // not fit; then what such loads need is there instead. (Blocks that a wave sees whole take one
  // read and one vote: two prompts with images, 1024 and 1001 new tokens, 28 heads, 106 us, with that 97.)
  int held = 0, mine = 0;
  if constexpr (kTree) {
    constexpr int kSpare = (kSmem - 4 * kKBytes) / 4;
    uint32_t* const spare = reinterpret_cast<uint32_t*>(smem + 4 * kKBytes);
    const int b0 = max((vis0 - kbeg) >> 5, 0), per = 2 * ntiles - b0;
    const int queries = small_div(h0 + it.rows - 1, inv_g) + 1;
    mine = qi - q0;
    if (queries * max(per, 0) <= kSpare) {
      held = 4 * kKBytes + 4 * (mine * max(per, 0) - b0);
      for (int k = tid; k < queries * per; k += 256) {
        const int q = k / per, at = kbeg + 32 * (b0 + k - q * per);
        spare[k] = mask_row(a, it, q0 + q).block(at, kend - at);
      }
    } else {
      held = -(1 << 30);
      if (tid == 0) *reinterpret_cast<MaskRow*>(spare) = mask_row(a, it, q0);
    }
    asm volatile("" : "+v"(held), "+v"(mine));
  }
  int some = 1;  // does the lane's row see any key?
  if constexpr (kTree) {
    some = row_sees<true>(a, it, qi, 0.0f);
    asm volatile("" : "+v"(some));
  }

  using B0 = std::integral_constant<int, 0>;
  using B1 = std::integral_constant<int, 1>;
  using B2 = std::integral_constant<int, 2>;
  using B3 = std::integral_constant<int, 3>;
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
      if constexpr (kTree) {
        uint32_t bits;
        if (__builtin_amdgcn_readfirstlane(held) > -(1 << 29))
          bits = *reinterpret_cast<const uint32_t*>(smem + held + 4 * blk);
        else
          bits = held_row(smem, mine).block(kbase, vis - kbase);
        if (!__builtin_amdgcn_ballot_w64(bits != ~0u)) return;  // (in images most blocks are seen whole)
        bits >>= 4 * lhalf;
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (!(bits >> (8 * (v >> 2) + (v & 3)) & 1)) sc[v] = -__builtin_inff();
      } else {
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (kbase + 8 * (v >> 2) + 4 * lhalf + (v & 3) >= vis) sc[v] = -__builtin_inff();
      }
      mt = tile_max(sc);
    }
  };
  // operand of MFMA j of a stage: 0..7 the scores (32-byte K step j), 8..15
  // the output (16 keys (j - 8) / 4, 32 dims j % 4)
  // kb and vb: 32-key blocks of the two K and of the two V buffers
  auto frag = [&](int j, int kb, int vb) __attribute__((always_inline)) {
    if (j < 8) return lds_read16(smem + koff[j], kb * kBK * kRowB);
    const char* p = smem + voff[j & 3] + (vb * kBK + 16 * ((j - 8) >> 2)) * kRowB;
    const u32x2_t lo = lds_read_tr(p), hi = lds_read_tr(p + 8 * kRowB);
    return u32x4_t{lo.x, lo.y, hi.x, hi.y};
  };
  // One stage takes block blk (32 keys) through the
  // softmax (scores sc, lane maximum mt; probabilities to pn) while the matrix
  // cores compute the scores of block blk + 1 (into sn, lane maximum to mn) and
  // then the output of block blk - 1 (probabilities pp): one probability after
  // each MFMA, in program order. The fences keep the compiler from sorting the
  // two kinds of instructions apart again.
  auto stage = [&](auto kb_c, auto vb_c, auto first_c, auto last_c, int blk, f32x16_t& sc, f32x16_t& sn, u32x4_t (&pp)[2],
                   u32x4_t (&pn)[2], float mt, float& mn) __attribute__((always_inline)) {
    constexpr int kKb = decltype(kb_c)::value, kVb = decltype(vb_c)::value;
    constexpr bool kFirst = decltype(first_c)::value, kLast = decltype(last_c)::value;
    constexpr int kLo = kLast ? 8 : 0, kHi = kFirst ? 8 : 16;  // MFMAs of this stage
    constexpr int kPer = 16 / (kHi - kLo);                     // probabilities after each
    u32x4_t fr[16];
#pragma unroll
    for (int j = kLo; j < kLo + kGroup; ++j) fr[j] = frag(j, kKb, kVb);
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
      mc_run = exponent_of(m_run, c2);
      far = any_far(mc_run);
    }
    float mc = mc_run, ce = c2;
    if (far) far_scores(sc, m_run, c2, mc, ce);
    // Step k: exponential k, the exponent of k + 1, and the pair before k is added
    // and packed; nothing in a step waits for the step's own exponential.
    float rs = 0.0f, p[16], ex = fmaf(sc[0], ce, -mc);
    auto soft = [&](int k) __attribute__((always_inline)) {
      if (k < 16) {
        p[k] = __builtin_amdgcn_exp2f(ex);
        asm volatile("" : "+v"(p[k]));  // this and the others keep the values between their fences
      }
      if (k < 15) {
        ex = fmaf(sc[k + 1], ce, -mc);
        asm volatile("" : "+v"(ex));
      }
      if (k >= 2 && !(k & 1)) {
        rs += p[k - 2] + p[k - 1];
        uint32_t w = pack_bf16(p[k - 2], p[k - 1]);
        asm volatile("" : "+v"(w), "+v"(rs));
        pn[(k - 2) >> 3][((k - 2) & 7) >> 1] = w;
      }
    };
    float mx = -__builtin_inff();
    __builtin_amdgcn_s_setprio(1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = kLo; j < kHi; ++j) {
      if (j % kGroup == 0 && j + kGroup < kHi) {
#pragma unroll
        for (int i = j + kGroup; i < j + 2 * kGroup; ++i) fr[i] = frag(i, kKb, kVb);
      }
      if (j == 0) sn = f32x16_t{};
      if (j < 8)
        mfma_step<true>(sn, fr[j], qf[j]);
      else
        mfma_step<true>(oacc[j & 3], fr[j], pp[(j - 8) >> 2]);
#pragma unroll
      for (int k = (j - kLo) * kPer; k < (j - kLo + 1) * kPer; ++k) soft(k);
      if (!kLast && !kFirst && j >= 12) {
#pragma unroll
        for (int v = 4 * (j - 12); v < 4 * (j - 11); ++v) mx = fmaxf(mx, sn[v]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    soft(16);
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
    const Rows rows0 = rows_of(0);
    Rows rows1 = rows_of(1);  // of the next V (8-bit: next but one) tile to fetch
    // The wave's 32 rows come by whole-line DMA as well (rows past the end as
    // zeros), chunk c of row r at c ^ (r & 15), into the parts of the two V
    // buffers that this wave itself fills later.
    {
      const int last = small_div(h0 + it.rows - 1, inv_g);  // the last row's query behind q0
      const char* qp = a.q + (int64_t)(it.qbase + q0) * a.q_ld + (int64_t)kvh * g * kRowB;
      const int span = h0 + it.rows - last * g;  // heads of that query that are rows
      const __amdgpu_buffer_rsrc_t qrs =
          wave_rsrc(qp, (uint32_t)((int64_t)last * a.q_ld) + (uint32_t)(span * kRowB));
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
      fetch_k(rows0, 0);
      if (!kF8 && ntiles > 1) {
        fetch_k(rows1, 1);
        wait_vmcnt<8>();
      } else if (!kF8) {
        wait_vmcnt<4>();
      } else {
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
      fetch_v(rows0, 0);
      if (ntiles > 1) {
        fetch_k(rows1, 0);
        put(kreg, kKBytes, true);
      }
      put(vreg, 2 * kKBytes, false);
      if (ntiles > 1) fetch_v(rows1, 0);
      rows1 = rows_of(2);
      if (ntiles > 2) fetch_k(rows1, 0);
    } else {
      fetch_v(rows0, 0);
      wait_vmcnt<4>();  // K
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) mfma_step<true>(sa, frag(j, 0, 0), qf[j]);
    ma = tile_max(sa);
    mask(0, sa, ma);
    stage(B1{}, B0{}, Yes{}, No{}, 0, sa, sb, pb, pa, ma, mb);
    if constexpr (!kF8) wait_vmcnt<0>();
    __syncthreads();  // every wave has read K of tile 0; V of tile 0 is there
    // (two tiles a turn: the buffers are immediate offsets)
    auto turn = [&](int t, auto k0_c, auto k1_c, auto v0_c, auto v1_c) __attribute__((always_inline)) {
      constexpr int kOdd = decltype(v0_c)::value >> 1;  // t % 2
      const Rows ahead = rows_of(kF8 ? t + 3 : t + 2);
      if constexpr (kF8) {
        if (t + 2 < ntiles) put(kreg, kOdd * kKBytes, true);
        put(vreg, (2 + (kOdd ^ 1)) * kKBytes, false);
        if (t + 3 < ntiles) fetch_k(ahead, 0);
        if (t + 2 < ntiles) fetch_v(rows1, 0);
      } else {
        if (t + 2 < ntiles) fetch_k(ahead, kOdd);
      }
      stage(k0_c, v0_c, No{}, No{}, 2 * t + 1, sb, sa, pa, pb, mb, ma);
      if constexpr (!kF8) fetch_v(rows1, kOdd ^ 1);
      rows1 = ahead;
      stage(k1_c, v1_c, No{}, No{}, 2 * t + 2, sa, sb, pb, pa, ma, mb);
      if (t + 4 - tb >= 64) load_pages(t + 1);  // (the next turn looks three tiles on)
      if constexpr (!kF8) {
        wait_vmcnt<0>();
        __syncthreads();
      } else {
        lds_barrier();  // (the next tiles' loads stay in flight)
      }
    };
    int t = 0;
    for (; t + 2 < ntiles; t += 2) {
      turn(t, B2{}, B3{}, B0{}, B1{});
      turn(t + 1, B0{}, B1{}, B2{}, B3{});
    }
    if (t + 1 < ntiles) turn(t, B2{}, B3{}, B0{}, B1{});
    if ((ntiles & 1) == 0) {
#pragma unroll
      for (int db = 0; db < 4; ++db) voff[db] += kKBytes;  // V of the last tile
    }
    stage(B0{}, B0{}, No{}, Yes{}, 2 * ntiles - 1, sb, sa, pa, pb, mb, ma);
#pragma unroll
    for (int j = 8; j < 16; ++j) mfma_step<true>(oacc[j & 3], frag(j, 0, 1), pb[(j - 8) >> 2]);
    const int last_key = min(kend, kbeg + ntiles * kKT);
    if ((kTree || a.causal) && vis0 < last_key && any_nan(oacc)) {
      paged_redo<kF8, false, kTree>(a, it.b, kvh, qf, oacc, m_run, l_run, c2, vis, kbeg, kBK, last_key, kTree ? mask_row(a, it, qi) : MaskRow{});
      if (lhalf) l_run = 0.0f;  // (the whole sum, once)
    }
  }

  l_run += __shfl_xor(l_run, 32);
  if (it.n_chunks > 1) {
    // ---- partial results, as the lanes hold them, for paged_combine_kernel ----
    float* const p = a.part + (int64_t)(it.slot + it.c) * (kSlotBytes<false> / 4);
#pragma unroll
    for (int v = 0; v < 16; ++v)
      *reinterpret_cast<f32x4_t*>(p + ((wave * 16 + v) * 64 + lane) * 4) =
          f32x4_t{oacc[v >> 2][4 * (v & 3)], oacc[v >> 2][4 * (v & 3) + 1], oacc[v >> 2][4 * (v & 3) + 2],
                  oacc[v >> 2][4 * (v & 3) + 3]};
    if (lhalf == 0) {
      p[kTileRows * kDh + 32 * wave + lrow] = m_run;
      p[kTileRows * (kDh + 1) + 32 * wave + lrow] = l_run;
    }
    return;
  }
  // ---- O = O^T / l, turned through LDS into whole rows (256 bytes by 16 lanes).
  //      The wave uses its own 8 KB of the K buffers, which no wave reads after
  //      the last barrier. ----
  const float inv = normalizer(l_run, kTree ? some != 0 : row_limit(a, it, qi, it.nk) > 0);
  const float vs = kF8 && a.vs ? a.vs[kvh] : 1.0f;
  char* const ob = kbuf + wave * 32 * kRowB;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4)
      store4<true>(ob + lrow * kRowB + (((4 * db + g4) ^ (lrow & 15)) << 4) + 8 * lhalf, oacc[db][4 * g4] * inv * vs,
                   oacc[db][4 * g4 + 1] * inv * vs, oacc[db][4 * g4 + 2] * inv * vs, oacc[db][4 * g4 + 3] * inv * vs);
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
