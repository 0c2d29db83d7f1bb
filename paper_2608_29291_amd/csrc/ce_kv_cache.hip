// The paged cache's bookkeeping and writes (paper section 3.4: the packed keys
// and values of a routed layer are the compressed cache that decoding reuses).
//
// Reserve. With base_b the tokens that sequence b keeps (lens[b], or 0 where it
// is handed on), n_b its new rows and P the page size, it needs
//   need_b = ceil((base_b + n_b) / P) - ceil(base_b / P)
// pages; the pages given back are numbered by an exclusive prefix sum of
// ceil(lens_b / P) over the handed-on sequences (their places on the stack), the
// pages taken by one of need_b (their depth below its top). Both sums run in one
// workgroup, 1024 sequences at a time, saturating (a bad batch may add up to
// anything), and pages and rows are then dealt out to threads by a search in the
// sums, so there one long prompt costs no more than many short ones. Many rows get
// their slots from a second launch over the whole chip, which deals by sequence: a
// long prompt among many sequences has few of its workgroups (us of both launches: 64
// sequences of 257 rows 8.1, one of 16384 and 63 of one 12.1; 512 sequences of 33 rows
// 8.5, one of 16384 and 511 of one 17.2).
//
// Bound: latency, a few kilobytes. The chain is sizes, sums, free pages, table and
// slots: three dependent loads; 64 sequences of one row 5.0 us (7.2 with sums of 64
// bits by shuffles). Past 1024 sequences the one workgroup goes round: 5000 of one row
// 32 us, 65535 359.
//
// Append. A pure copy, or x / scale rounded to e4m3: bound by memory. A thread
// moves 16 bytes of a page; the rows of a fused projection are read where they are.
#include "ce_device.hpp"
#include "ce_host.hpp"
#include "ce_paged.hpp"
#include "ce_scan.hpp"

namespace ce {

namespace {

using namespace scan;

struct Seq {
  int base, n, held, lo;  // tokens kept, new rows, pages of base, first row
  uint32_t back, need;    // pages given back, pages to take
  bool too_long;
  uint32_t st;  // CE_DEV_* of its sizes
};

__device__ __forceinline__ Seq load_seq(const ReserveArgs& a, int b) {
  Seq s = {};
  const int most = a.max_pages << a.page_log2;
  const int len0 = a.lens[b], o0 = a.offs ? a.offs[b] : 0, o1 = a.offs ? a.offs[b + 1] : 0;
  const bool reset = a.reset && a.reset[b];
  const int len = clampi(len0, 0, most);
  s.lo = clampi(o0, 0, a.rows);
  s.n = clampi(o1, s.lo, a.rows) - s.lo;
  const uint32_t up = (1u << a.page_log2) - 1;
  const uint32_t held = ((uint32_t)len + up) >> a.page_log2;
  s.base = reset ? 0 : len;
  s.back = reset ? held : 0;
  s.held = reset ? 0 : (int)held;
  s.need = (((uint32_t)s.base + (uint32_t)s.n + up) >> a.page_log2) - (uint32_t)s.held;
  s.too_long = (uint32_t)s.held + s.need > (uint32_t)a.max_pages;
  if (s.too_long) s.need = 0;
  s.st = (len0 != len ? CE_DEV_BAD_CACHE : 0) | (s.too_long ? CE_DEV_TOO_LONG : 0) |
         (o0 < 0 || o1 < o0 || (b == 0 && o0 != 0) ? CE_DEV_BAD_OFFSETS : 0) |
         (o0 > a.rows || o1 > a.rows ? CE_DEV_OVERFLOW : 0);
  return s;
}

__global__ __launch_bounds__(1024) void kv_reserve_kernel(ReserveArgs a) {
  __shared__ uint32_t scr[32];
  __shared__ int first[1024], off[1024], cnt[1024], pos[1024], held[1024];
  __shared__ uint32_t st_s;
  __shared__ int taken_s;
  const int tid = threadIdx.x;
  if (tid == 0) st_s = 0;
  const int count0 = *a.count;
  const int end = a.offs ? clampi(a.offs[a.B], 0, a.rows) : 0;
  const bool once = a.B <= 1024;
  Seq s = {};
  if (tid < a.B) s = load_seq(a, tid);
  int count = clampi(count0, 0, a.n_pages);
  uint32_t st = count != count0 ? CE_DEV_BAD_CACHE : 0;

  // ---- the pages of handed-on sequences, on top of the stack ----
  if (a.reset) {
    for (int s0 = 0; s0 < a.B; s0 += 1024) {
      if (s0) {
        s = Seq{};
        if (s0 + tid < a.B) s = load_seq(a, s0 + tid);
      }
      uint32_t to = s.back, none = 0, total, t2;
      scan2(to, none, total, t2, scr);
      // (more than the stack has room for is pushed only if pages are held twice)
      first[tid] = (int)min(to - s.back, (uint32_t)a.n_pages);
      const uint32_t room = a.n_pages - count;
      if (total > room) st |= CE_DEV_BAD_CACHE;
      const int pushed = (int)min(total, room);
      __syncthreads();
      for (int i = tid; i < pushed; i += 1024) {
        const int k = last_at_most(first, 1024, i);
        const int page = a.table[(int64_t)(s0 + k) * a.max_pages + (i - first[k])];
        if ((uint32_t)page >= (uint32_t)a.n_pages) st |= CE_DEV_BAD_CACHE;  // (and again where it is popped)
        a.free_pages[count + i] = page;
      }
      count += pushed;
      __syncthreads();
    }
  }

  // ---- pages for the new rows ----
  uint32_t before = 0;  // needed by the chunks of sequences before
  int taken = 0;
  const bool with_slots = once && !a.slots_apart;
  for (int s0 = 0; s0 < a.B; s0 += 1024) {
    const int b = s0 + tid;
    if (!once) {
      s = Seq{};
      if (b < a.B) s = load_seq(a, b);
    }
    uint32_t to = s.need, none = 0, total, t2;
    if (tid == 0) taken_s = 0;
    scan2(to, none, total, t2, scr);
    const bool good = b < a.B && !s.too_long && (s.need == 0 || add_sat(before, to) <= (uint32_t)count);
    st |= s.st;
    if (b < a.B && !good && !s.too_long) st |= CE_DEV_NO_PAGES;
    if (b < a.B) {
      a.lens_out[b] = s.base + (good ? s.n : 0);
      a.start[b] = good ? s.base : -1;
    }
    // The sequences that are granted pages come before any that is refused some, and
    // a sum of granted pages is at most the count: `to` is what they take up to here.
    const int ex = (int)min(to - s.need, 0x7fffffffu);
    first[tid] = ex;
    off[tid] = b < a.B ? s.lo : 0x7fffffff;
    cnt[tid] = s.n;
    pos[tid] = good ? s.base : -1;
    held[tid] = s.held;
    if (good && s.need > 0) atomicMax(&taken_s, (int)to);
    __syncthreads();
    const int granted = taken_s;
    const int top = count - 1 - taken;
    for (int i = tid; i < granted; i += 1024) {
      const int k = last_at_most(first, 1024, i);
      const int page = a.free_pages[top - i];
      if ((uint32_t)page >= (uint32_t)a.n_pages) st |= CE_DEV_BAD_CACHE;
      a.table[(int64_t)(s0 + k) * a.max_pages + held[k] + (i - first[k])] = page;
    }
    if (with_slots) {
      const int mask = (1 << a.page_log2) - 1;
      for (int r = tid; r < a.rows; r += 1024) {
        int slot = -1;
        if (r < end && off[0] <= r) {
          const int k = last_at_most(off, 1024, r);
          if (pos[k] >= 0 && r - off[k] < cnt[k]) {
            const int t = pos[k] + (r - off[k]);
            const int p = t >> a.page_log2;
            const int in_new = first[k] + p - held[k];  // among the pages taken
            const int page = p < held[k] ? a.table[(int64_t)k * a.max_pages + p] : a.free_pages[top - in_new];
            if ((uint32_t)page < (uint32_t)a.n_pages) slot = (page << a.page_log2) + (t & mask);
          }
        }
        a.slots[r] = slot;
      }
    }
    before = add_sat(before, total);
    taken += granted;
    __syncthreads();
  }
  if (st) atomicOr(&st_s, st);
  __syncthreads();
  if (tid == 0) {
    *a.count_out = count - taken;
    if (a.status) *a.status = st_s;
  }
}

// Slots of many rows, after kv_reserve_kernel: the workgroups (b, *) walk the
// rows of sequence b, and all of them the rows behind the last (and before the
// first, where the offsets are wrong).
__global__ __launch_bounds__(256) void kv_slots_kernel(ReserveArgs a) {
  const int b = blockIdx.x;
  const int lo = clampi(a.offs[b], 0, a.rows);
  const int hi = clampi(a.offs[b + 1], lo, a.rows);
  const int start = a.start[b];
  const int mask = (1 << a.page_log2) - 1;
  for (int64_t r = lo + (int64_t)blockIdx.y * 256 + threadIdx.x; r < hi; r += gridDim.y * 256) {
    int slot = -1;
    if (start >= 0) {
      const int t = start + (int)(r - lo);
      const int page = a.table[(int64_t)b * a.max_pages + (t >> a.page_log2)];
      if ((uint32_t)page < (uint32_t)a.n_pages) slot = (page << a.page_log2) + (t & mask);
    }
    a.slots[r] = slot;
  }
  const int end = clampi(a.offs[a.B], 0, a.rows);
  const int64_t all = (int64_t)gridDim.x * gridDim.y * 256;
  const int64_t at = ((int64_t)blockIdx.y * gridDim.x + b) * 256 + threadIdx.x;
  for (int64_t r = end + at; r < a.rows; r += all) a.slots[r] = -1;
  const int begin = clampi(a.offs[0], 0, a.rows);
  for (int64_t r = at; r < begin; r += all) a.slots[r] = -1;
}

// 8 bf16 (a 16-byte load) / scale, limited to +-448, as 8 bytes of e4m3. The quotient
// is the correctly rounded one: with r = 1 / scale rounded to nearest, q = x r and
// q + (x - q scale) r, the remainder by one fma, is x / scale rounded to nearest
// (Markstein), in three instructions instead of the ten of a division that provides
// for every exponent. Quotients past 500, which are limited anyway, infinities,
// NaN and zeros (of either sign) keep q. kDivide: the division, for scales outside
// 1e-24 .. 1e24: the remainder of a value that is not rounded to zero reaches 2^-57 of
// the scale, which has to be a normal float.
template <bool kDivide>
__device__ __forceinline__ u32x2_t to_e4m3(const u32x4_t& x, float scale, float r) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = __uint_as_float((i & 1) ? x[i >> 1] & 0xffff0000u : x[i >> 1] << 16);
    float q;
    if constexpr (kDivide) {
      q = v / scale;
    } else {
      q = v * r;
      const float near = fmaf(fmaf(-q, scale, v), r, q);
      q = fabsf(q) < 500.0f && q != 0.0f ? near : q;
    }
    f[i] = q != q ? q : fminf(fmaxf(q, -448.0f), 448.0f);
  }
  u32x2_t w;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h], f[4 * h + 1], 0, false);
    w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h + 2], f[4 * h + 3], lo, true);
  }
  return w;
}

// A workgroup takes whole rows, a thread 16 bytes of a page at a time. 17408 rows of
// four heads into 8-bit pages, 53 MB: 11.2 us, 4.75 TB/s (a large copy runs at 4.98);
// 13.0 with a division per value, 14.6 with loads past the caches as well. Four pieces
// in flight in a thread were slower than as many threads more (20 and 17 us).
template <bool kE4m3>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
  constexpr int kPer = kE4m3 ? 8 : 16;  // 16-byte pieces of a page per row and head
  constexpr int kRow = kPer * 16;
  constexpr int kLoad = kE4m3 ? 2 : 1;  // 16-byte loads of a piece
  const uint32_t half = (uint32_t)a.Hkv * kPer;  // pieces of a row of K, and of V
  const uint32_t n = (uint32_t)a.rows_per_block * 2 * half;
  const int64_t row0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * a.rows_per_block;
  for (uint32_t i = threadIdx.x; i < n; i += 256) {
    const uint32_t rl = i / (2 * half);
    const int64_t r = row0 + rl;
    if (r >= a.rows) break;
    uint32_t c = i - rl * 2 * half;
    const int slot = a.slots[r];
    if ((uint32_t)slot >= (uint32_t)a.n_slots) continue;
    const bool is_v = c >= half;
    if (is_v) c -= half;
    const uint32_t h = c / kPer;
    const char* src = (is_v ? a.v_new + r * a.v_ld : a.k_new + r * a.k_ld) + (int64_t)c * (16 * kLoad);
    char* dst = (is_v ? a.v : a.k) + (int64_t)((uint64_t)(uint32_t)(slot >> a.page_log2) * a.page_bytes) +
                (((int64_t)h << a.page_log2) + (slot & ((1 << a.page_log2) - 1))) * kRow + (c & (kPer - 1)) * 16;
    const u32x4_t x = gload16_cached(src);
    if constexpr (kE4m3) {
      const u32x4_t y = gload16_cached(src + 16);
      const float* const sc = is_v ? a.v_scale : a.k_scale;
      const float s = sc ? sc[h] : 1.0f;
      u32x2_t p, q;
      if (__builtin_amdgcn_ballot_w64(!(s > 1e-24f && s < 1e24f))) {
        p = to_e4m3<true>(x, s, 0.0f);
        q = to_e4m3<true>(y, s, 0.0f);
      } else {
        float f = __builtin_amdgcn_rcpf(s);
        f = fmaf(fmaf(-s, f, 1.0f), f, f);
        p = to_e4m3<false>(x, s, f);
        q = to_e4m3<false>(y, s, f);
      }
      *reinterpret_cast<u32x4_t*>(dst) = u32x4_t{p.x, p.y, q.x, q.y};
    } else {
      *reinterpret_cast<u32x4_t*>(dst) = x;
    }
  }
}

}  // namespace

hipError_t launch_kv_reserve(ReserveArgs a, hipStream_t stream) {
  // Rows that one workgroup deals out itself: up to the time that a second launch
  // takes (one launch and two, 1 sequence: 1024 rows 3.5 and 5.0 us, 4096 5.4 and 5.6,
  // 8192 7.9 and 5.6; 1024 sequences: 1024 rows 4.0 and 5.6, 8192 8.1 and 5.6).
  a.slots_apart = a.offs && (a.rows > 4096 || a.B > 1024);
  hipLaunchKernelGGL(kv_reserve_kernel, dim3(1), dim3(1024), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.rows == 0) return e;
  if (a.slots_apart) {
    const int per = (int)(((int64_t)a.rows + (int64_t)a.B * 256 - 1) / ((int64_t)a.B * 256));
    hipLaunchKernelGGL(kv_slots_kernel, dim3(a.B, per < 64 ? per : 64), dim3(256), 0, stream, a);
    e = hipGetLastError();
  }
  return e;
}

hipError_t launch_kv_append(AppendArgs a, bool e4m3, hipStream_t stream) {
  if (a.rows == 0) return hipSuccess;
  // rows of a workgroup: as many as give every thread its pieces once
  const int64_t pieces = (int64_t)2 * a.Hkv * (e4m3 ? 8 : 16);
  const int64_t per = 256 / pieces;
  a.rows_per_block = per < 1 ? 1 : (int)per;
  const int64_t blocks = ((int64_t)a.rows + a.rows_per_block - 1) / a.rows_per_block;
  const int64_t x = blocks < 1 << 16 ? blocks : 1 << 16;
  const dim3 grid((unsigned)x, (unsigned)((blocks + x - 1) / x));
  if (e4m3)
    hipLaunchKernelGGL(kv_append_kernel<true>, grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(kv_append_kernel<false>, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ce
