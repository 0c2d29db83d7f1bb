// Rotary positions of packed rows (include/ce_router_rotary.h):
//   y1 = x1 cos a - x2 sin a,  y2 = x1 sin a + x2 cos a,  a = freq[i] position[axis[i]]
//
// Angles. A position times a frequency in float32 is off by 2^-24 of itself, 2e-3 rad at position
// 30000. Here a frequency is a fraction of a turn in 64-bit fixed point, so the product
// modulo 2^64 with the position (any 32 bits, negative ones too) is the turn's own
// fraction with no reduction to make; its upper 32 bits give the quadrant and the
// angle in it, within pi / 4, where Taylor polynomials of degree 9 and 10 are exact to 2^-29.
//
// Bound: memory; each value is read and written once. A thread keeps the cosines of its pairs for four
// heads, where there are rows enough; these move more than the L2 caches hold, 32 MB, and go past
// them: 17408 rows of 32 heads in bf16, 285 MB, 51 us, 5.6 TB/s (64 with ordinary loads and
// stores; one head a thread 99, two 70, eight 62).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "ce_device.hpp"
#include "ce_router_rotary.h"

namespace ce {

namespace {

constexpr int kMaxPairs = 128;
constexpr int kMaxAxes = 4;

struct RotaryArgs {
  const char* x;
  char* y;
  int64_t x_ld, y_ld;  // bytes
  const int32_t* positions;
  const int32_t* index;
  int n_positions, n_axes, inverse;
  int rows, heads, head_bytes, pairs, lanes, turning, blocks_of_heads;
  uint64_t freq[kMaxPairs];  // turns a position, modulo 1, times 2^64
  uint8_t axis[kMaxPairs];
};

// Cosine and sine of t / 2^32 turns.
__device__ __forceinline__ void turn(uint32_t t, float& c, float& s) {
  const uint32_t q = (t + (1u << 29)) >> 30;
  const float z = (float)(int32_t)(t - (q << 30)) * 1.46291807926715968105e-9f;  // 2 pi / 2^32
  const float w = z * z;
  const float sn = fmaf(z * w, fmaf(w, fmaf(w, fmaf(w, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), z);
  const float cs = fmaf(
      w, fmaf(w, fmaf(w, fmaf(w, fmaf(w, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
  c = q & 1 ? sn : cs;
  s = q & 1 ? cs : sn;
  if ((q + 1) & 2) c = -c;
  if (q & 2) s = -s;
}

template <typename E, int N>
struct alignas(N * sizeof(E)) Pack {
  E e[N];
};
// kStream: past the caches.
template <bool kStream, typename V>
__device__ __forceinline__ V load(const void* p) {
  if constexpr (!kStream)
    return *reinterpret_cast<const V*>(p);
  else if constexpr (sizeof(V) == 16)
    return __builtin_bit_cast(V, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p)));
  else if constexpr (sizeof(V) == 8)
    return __builtin_bit_cast(V, __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(p)));
  else if constexpr (sizeof(V) == 4)
    return __builtin_bit_cast(V, __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p)));
  else
    return __builtin_bit_cast(V, __builtin_nontemporal_load(reinterpret_cast<const uint16_t*>(p)));
}
template <bool kStream, typename V>
__device__ __forceinline__ void store(void* p, const V& v) {
  if constexpr (!kStream)
    *reinterpret_cast<V*>(p) = v;
  else if constexpr (sizeof(V) == 16)
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), reinterpret_cast<u32x4_t*>(p));
  else if constexpr (sizeof(V) == 8)
    __builtin_nontemporal_store(__builtin_bit_cast(u32x2_t, v), reinterpret_cast<u32x2_t*>(p));
  else if constexpr (sizeof(V) == 4)
    __builtin_nontemporal_store(__builtin_bit_cast(uint32_t, v), reinterpret_cast<uint32_t*>(p));
  else
    __builtin_nontemporal_store(__builtin_bit_cast(uint16_t, v), reinterpret_cast<uint16_t*>(p));
}

__device__ __forceinline__ float value(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ void put(uint16_t* p, float a, float b) {
  const uint32_t w = pack_bf16(a, b);
  p[0] = (uint16_t)w;
  p[1] = (uint16_t)(w >> 16);
}
__device__ __forceinline__ void put(float* p, float a, float b) {
  p[0] = a;
  p[1] = b;
}

// A thread: kN pairs of kHeads heads of a row, or kN values behind the pairs.
template <typename E, int kN, int kHeads, bool kPairs>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  using V = Pack<E, kN>;
  constexpr bool kStream = kHeads > 1;
  // Places of the thread's two vectors in a head, and pair i of its kN. (Of neighbours the vectors lie half of
  // the turned values apart, so that a wave's loads are whole lines.)
  constexpr bool kApart = !kPairs || kN > 1;
  const int per = 256 / a.lanes;  // (row, heads) items of a workgroup
  const int sub = (int)threadIdx.x / a.lanes, lane = (int)threadIdx.x - sub * a.lanes;
  const uint32_t item = blockIdx.x * (uint32_t)per + sub;
  const uint32_t row = item / (uint32_t)a.blocks_of_heads;
  if (sub >= per || row >= (uint32_t)a.rows) return;
  const int h0 = (int)(item - row * a.blocks_of_heads) * kHeads;
  const char* const xr = a.x + (int64_t)row * a.x_ld + (int64_t)h0 * a.head_bytes;
  char* const yr = a.y + (int64_t)row * a.y_ld + (int64_t)h0 * a.head_bytes;
  const int n = min(kHeads, a.heads - h0);
  const int token = a.index ? a.index[row] : (int)row;
  if (lane >= a.turning || (uint32_t)token >= (uint32_t)a.n_positions) {  // copied
    const int at0 = lane >= a.turning ? (2 * a.pairs + (lane - a.turning) * kN) : (kApart ? 1 : 2) * lane * kN;
    const int at1 = lane >= a.turning ? at0 : at0 + (kApart ? a.pairs : 1);
    if (a.x == a.y) return;
    for (int h = 0; h < n; ++h) {
      const E* const p = reinterpret_cast<const E*>(xr + (int64_t)h * a.head_bytes);
      E* const q = reinterpret_cast<E*>(yr + (int64_t)h * a.head_bytes);
      store<kStream>(q + at0, load<kStream, V>(p + at0));
      if (at1 != at0) store<kStream>(q + at1, load<kStream, V>(p + at1));
    }
    return;
  }
  const int at0 = (kApart ? 1 : 2) * lane * kN, at1 = at0 + (kApart ? a.pairs : 1);
  auto pair = [&](int i) __attribute__((always_inline)) {
    if (!kPairs || kN == 1) return lane * kN + i;
    return (i < kN / 2 ? at0 : at1 - kN) / 2 + i;
  };
  V x0[kHeads], x1[kHeads];
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    const E* const p = reinterpret_cast<const E*>(xr + (int64_t)min(h, n - 1) * a.head_bytes);
    x0[h] = load<kStream, V>(p + at0);
    x1[h] = load<kStream, V>(p + at1);
  }
  int pos[kMaxAxes];
#pragma unroll
  for (int i = 0; i < kMaxAxes; ++i) pos[i] = i < a.n_axes ? a.positions[(int64_t)i * a.n_positions + token] : 0;
  float c[kN], s[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const int k = a.axis[pair(i)];
    const int p = k == 0 ? pos[0] : (k == 1 ? pos[1] : (k == 2 ? pos[2] : pos[3]));
    uint32_t t = (uint32_t)(((uint64_t)(int64_t)p * a.freq[pair(i)]) >> 32);
    if (a.inverse) t = 0u - t;
    turn(t, c[i], s[i]);
  }
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    float y[2 * kN];  // in the order of memory
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      float u, v;
      if constexpr (kPairs) {
        u = value(2 * i < kN ? x0[h].e[(2 * i) % kN] : x1[h].e[(2 * i) % kN]);
        v = value(2 * i + 1 < kN ? x0[h].e[(2 * i + 1) % kN] : x1[h].e[(2 * i + 1) % kN]);
      } else {
        u = value(x0[h].e[i]);
        v = value(x1[h].e[i]);
      }
      const float a0 = fmaf(u, c[i], -(v * s[i])), a1 = fmaf(u, s[i], v * c[i]);
      y[kPairs ? 2 * i : i] = a0;
      y[kPairs ? 2 * i + 1 : kN + i] = a1;
    }
    if (h >= n) break;
    E w[2 * kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) put(w + 2 * i, y[2 * i], y[2 * i + 1]);
    V v0, v1;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      v0.e[i] = w[i];
      v1.e[i] = w[kN + i];
    }
    E* const q = reinterpret_cast<E*>(yr + (int64_t)h * a.head_bytes);
    store<kStream>(q + at0, v0);
    store<kStream>(q + at1, v1);
  }
}

template <typename E, int kN, bool kPairs>
hipError_t launch(RotaryArgs& a, bool many, hipStream_t stream) {
  const int per = 256 / a.lanes;
  const int heads = many ? 4 : 1;
  a.blocks_of_heads = (a.heads + heads - 1) / heads;
  const int64_t items = (int64_t)a.rows * a.blocks_of_heads;
  const dim3 grid((unsigned)((items + per - 1) / per));
  if (many)
    hipLaunchKernelGGL((rotary_kernel<E, kN, 4, kPairs>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((rotary_kernel<E, kN, 1, kPairs>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <typename E>
hipError_t launch_by_width(RotaryArgs& a, int n, bool pairs, bool many, hipStream_t stream) {
  switch (n) {
    case 8:
      if constexpr (sizeof(E) == 2) return pairs ? launch<E, 8, true>(a, many, stream) : launch<E, 8, false>(a, many, stream);
      break;
    case 4: return pairs ? launch<E, 4, true>(a, many, stream) : launch<E, 4, false>(a, many, stream);
    case 2: return pairs ? launch<E, 2, true>(a, many, stream) : launch<E, 2, false>(a, many, stream);
    default: break;
  }
  return pairs ? launch<E, 1, true>(a, many, stream) : launch<E, 1, false>(a, many, stream);
}

// freq / (2 pi) modulo 1 as a 64-bit fraction, |freq| <= 64. (64 bits of the long double's mantissa; the
// fraction's own last bit is left out, which no position makes more than 2^-32 of a turn.)
uint64_t fraction_of_turn(double freq) {
  const long double v = (long double)freq * 0.159154943091895335768883763372514362L;
  const long double part = v - (long double)(int64_t)v;  // of v's sign, below 1
  return (uint64_t)(int64_t)(part * 9223372036854775808.0L) << 1;
}

}  // namespace

}  // namespace ce

using namespace ce;

extern "C" int ce_rotary(const ce_rotary_desc* d, const void* x, int64_t x_ld, void* y, int64_t y_ld, void* stream) {
  if (!d || d->rows < 0 || d->n_heads < 1 || d->head_dim < 1 || d->n_pairs < 1 || d->n_axes < 1 || d->n_positions < 0)
    return CE_ERR_INVALID_ARG;
  if (d->layout != CE_ROTARY_HALVES && d->layout != CE_ROTARY_PAIRS) return CE_ERR_INVALID_ARG;
  if (d->inverse != 0 && d->inverse != 1) return CE_ERR_INVALID_ARG;
  if ((d->dtype != CE_BF16 && d->dtype != CE_F32) || d->head_dim % 2 != 0 || d->head_dim > 256 ||
      d->n_pairs > d->head_dim / 2 || d->n_axes > kMaxAxes || d->n_heads >= 1 << 16 ||
      (int64_t)d->rows * d->n_heads >= (int64_t)1 << 31)
    return CE_ERR_UNSUPPORTED;
  const int64_t row = (int64_t)d->n_heads * d->head_dim;
  if (x_ld < row || y_ld < row || x_ld % 8 != 0 || y_ld % 8 != 0) return CE_ERR_INVALID_ARG;
  if (x_ld >= (int64_t)1 << 40 || y_ld >= (int64_t)1 << 40) return CE_ERR_UNSUPPORTED;
  if (!d->freq) return CE_ERR_INVALID_ARG;
  RotaryArgs a = {};
  for (int i = 0; i < d->n_pairs; ++i) {
    const int k = d->axis ? d->axis[i] : 0;
    if (!(fabs(d->freq[i]) <= 64.0) || k < 0 || k >= d->n_axes) return CE_ERR_INVALID_ARG;
    a.freq[i] = fraction_of_turn(d->freq[i]);
    a.axis[i] = (uint8_t)k;
  }
  if (d->rows == 0) return CE_OK;
  if (!x || !y || (d->n_positions > 0 && !d->positions)) return CE_ERR_INVALID_ARG;
  if (x == y && x_ld != y_ld) return CE_ERR_INVALID_ARG;
  const int elem = d->dtype == CE_BF16 ? 2 : 4;
  const int rest = d->head_dim - 2 * d->n_pairs;
  // pairs of a thread: as many as two 16-byte loads hold, where the sizes allow them
  int n = 16 / elem;
  while (n > 1 && (d->n_pairs % n != 0 || rest % n != 0)) n >>= 1;
  a.x = static_cast<const char*>(x);
  a.y = static_cast<char*>(y);
  a.x_ld = x_ld * elem;
  a.y_ld = y_ld * elem;
  a.positions = d->positions;
  a.index = d->index;
  a.n_positions = d->n_positions;
  a.n_axes = d->n_axes;
  a.inverse = d->inverse;
  a.rows = d->rows;
  a.heads = d->n_heads;
  a.head_bytes = d->head_dim * elem;
  a.pairs = d->n_pairs;
  a.turning = d->n_pairs / n;
  a.lanes = a.turning + (x == y ? 0 : rest / n);
  const bool many = (int64_t)d->rows * d->n_heads * a.lanes * n * elem >= (int64_t)1 << 23;  // 32 MB, read and written
  // (a launch has fewer than 2^32 threads)
  if ((int64_t)d->rows * (many ? (d->n_heads + 3) / 4 : d->n_heads) / (256 / a.lanes) >= ((int64_t)1 << 24) - 1)
    return CE_ERR_UNSUPPORTED;
  const bool pairs = d->layout == CE_ROTARY_PAIRS;
  const hipError_t e = d->dtype == CE_BF16 ? launch_by_width<uint16_t>(a, n, pairs, many, static_cast<hipStream_t>(stream))
                                           : launch_by_width<float>(a, n, pairs, many, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? CE_OK : CE_ERR_HIP;
}
