// The paged cache's bookkeeping and writes (paper section 3.4: the packed keys
// and values of a routed layer are the compressed cache that decoding reuses).
//
// Reserve. With base_b the tokens that sequence b keeps (lens[b], or 0 where it
// is handed on), n_b its new rows and P the page size, it needs
//   need_b = ceil((base_b + n_b) / P) - ceil(base_b / P)
// pages; the pages given back are numbered by an exclusive prefix sum of
// ceil(lens_b / P) over the handed-on sequences (their places on the stack), the
// pages taken by one of need_b (their depth below its top). Both sums run in one
// workgroup, 1024 sequences at a time, in 64 bits (a bad batch may add up to
// anything), and pages and rows are then dealt out to threads by a search in the
// sums, so one long prompt costs no more than many short ones. Many rows get their
// slots from a second launch over the whole chip.
//
// Bound: latency, a few kilobytes. The chain is sizes, sums, free pages, table and
// slots: three dependent loads.
//
// Append. A pure copy, or x / scale rounded to e4m3: bound by memory. A thread
// moves 16 bytes of a page; the rows of a fused projection are read where they are.
#include "ce_device.hpp"
#include "ce_host.hpp"
#include "ce_paged.hpp"

namespace ce {

namespace {

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// Exclusive prefix sums of a and b over the 1024 threads of the workgroup, and
// their totals (scr: 32 entries of LDS). Every thread must call it.
__device__ __forceinline__ void scan2(int64_t& a, int64_t& b, int64_t& ta, int64_t& tb, int64_t* scr) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t x = a, y = b;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t u = __shfl_up(x, o), w = __shfl_up(y, o);
    if (lane >= o) {
      x += u;
      y += w;
    }
  }
  __syncthreads();
  if (lane == 63) {
    scr[wave] = x;
    scr[16 + wave] = y;
  }
  __syncthreads();
  int64_t ba = 0, bb = 0;
  ta = tb = 0;
  for (int w = 0; w < 16; ++w) {
    if (w == wave) {
      ba = ta;
      bb = tb;
    }
    ta += scr[w];
    tb += scr[16 + w];
  }
  a = ba + x - a;
  b = bb + y - b;
}

// The last i of 0 .. n - 1 with first[i] <= x (first: non-decreasing, first[0] <= x).
__device__ __forceinline__ int last_at_most(const int* first, int n, int x) {
  int lo = 0;
  for (int step = 512; step > 0; step >>= 1)
    if (lo + step < n && first[lo + step] <= x) lo += step;
  return lo;
}

struct Seq {
  int base, n, held, back, lo;  // tokens kept, new rows, pages of base, pages given back, first row
  int64_t need;                 // pages to take
  bool too_long;
  uint32_t st;  // CE_DEV_* of its sizes
};

__device__ __forceinline__ Seq load_seq(const ReserveArgs& a, int b) {
  Seq s = {};
  const int most = a.max_pages << a.page_log2;
  const int len0 = a.lens[b], o0 = a.offs ? a.offs[b] : 0, o1 = a.offs ? a.offs[b + 1] : 0;
  const int len = clampi(len0, 0, most);
  s.lo = clampi(o0, 0, a.rows);
  s.n = clampi(o1, s.lo, a.rows) - s.lo;
  const int up = (1 << a.page_log2) - 1;
  const bool reset = a.reset && a.reset[b];
  s.base = reset ? 0 : len;
  s.back = reset ? (int)(((int64_t)len + up) >> a.page_log2) : 0;
  s.held = (int)(((int64_t)s.base + up) >> a.page_log2);
  s.need = (((int64_t)s.base + s.n + up) >> a.page_log2) - s.held;
  s.too_long = s.held + s.need > a.max_pages;
  if (s.too_long) s.need = 0;
  s.st = (len0 != len ? CE_DEV_BAD_CACHE : 0) | (s.too_long ? CE_DEV_TOO_LONG : 0) |
         (o0 < 0 || o1 < o0 || (b == 0 && o0 != 0) ? CE_DEV_BAD_OFFSETS : 0) |
         (o0 > a.rows || o1 > a.rows ? CE_DEV_OVERFLOW : 0);
  return s;
}

__global__ __launch_bounds__(1024) void kv_reserve_kernel(ReserveArgs a) {
  __shared__ int64_t scr[32];
  __shared__ int first[1024], off[1024], cnt[1024], pos[1024], held[1024];
  __shared__ uint32_t st_s;
  const int tid = threadIdx.x;
  if (tid == 0) st_s = 0;
  const int count0 = *a.count;
  int64_t count = clampi(count0, 0, a.n_pages);
  uint32_t st = count != count0 ? CE_DEV_BAD_CACHE : 0;

  // ---- the pages of handed-on sequences, on top of the stack ----
  if (a.reset) {
    for (int s0 = 0; s0 < a.B; s0 += 1024) {
      Seq s = {};
      if (s0 + tid < a.B) s = load_seq(a, s0 + tid);
      int64_t ex = s.back, none = 0, total, t2;
      scan2(ex, none, total, t2, scr);
      first[tid] = (int)min(ex, (int64_t)a.n_pages);  // (past the stack: see below)
      __syncthreads();
      const int64_t room = a.n_pages - count;  // more is pushed only if pages are held twice
      if (total > room) st |= CE_DEV_BAD_CACHE;
      const int pushed = (int)min(total, room);
      for (int i = tid; i < pushed; i += 1024) {
        const int k = last_at_most(first, 1024, i);
        a.free_pages[count + i] = a.table[(int64_t)(s0 + k) * a.max_pages + (i - first[k])];
      }
      count += pushed;
      __syncthreads();
    }
  }

  // ---- pages for the new rows ----
  int64_t before = 0;  // needed by the chunks of sequences before
  int64_t taken = 0;
  const bool with_slots = a.B <= 1024 && !a.slots_apart;
  for (int s0 = 0; s0 < a.B; s0 += 1024) {
    const int b = s0 + tid;
    Seq s = {};
    if (b < a.B) s = load_seq(a, b);
    int64_t ex = s.need, got, total, granted;
    // (the second sum is of what is granted, which the first decides)
    got = 0;
    scan2(ex, got, total, granted, scr);
    const int64_t depth = before + ex;
    const bool good = b < a.B && !s.too_long && (s.need == 0 || depth + s.need <= count);
    st |= s.st;
    if (b < a.B && !good && !s.too_long) st |= CE_DEV_NO_PAGES;
    const int need = good ? (int)s.need : 0;
    if (b < a.B) {
      a.lens_out[b] = s.base + (good ? s.n : 0);
      a.start[b] = good ? s.base : -1;
    }
    // every refused sequence is deeper than the stack, so the granted ones that
    // take pages come first and their depths are without gaps
    int64_t e2 = need, none = 0, t2;
    scan2(e2, none, granted, t2, scr);
    first[tid] = (int)e2;
    off[tid] = b < a.B ? s.lo : 0x7fffffff;
    cnt[tid] = s.n;
    pos[tid] = good ? s.base : -1;
    held[tid] = s.held;
    __syncthreads();
    const int64_t top = count - 1 - taken;
    for (int i = tid; i < (int)granted; i += 1024) {
      const int k = last_at_most(first, 1024, i);
      const int page = a.free_pages[top - i];
      if ((uint32_t)page >= (uint32_t)a.n_pages) st |= CE_DEV_BAD_CACHE;
      a.table[(int64_t)(s0 + k) * a.max_pages + held[k] + (i - first[k])] = page;
    }
    if (with_slots) {
      const int mask = (1 << a.page_log2) - 1;
      const int end = a.offs ? clampi(a.offs[a.B], 0, a.rows) : 0;
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
    before += total;
    taken += granted;
    __syncthreads();
  }
  if (st) atomicOr(&st_s, st);
  __syncthreads();
  if (tid == 0) {
    *a.count_out = (int)(count - taken);
    if (a.status) *a.status = st_s;
  }
}

// Slots of many rows, after kv_reserve_kernel: the workgroups (b, *) walk the
// rows of sequence b, and all of them the rows behind the last.
__global__ __launch_bounds__(256) void kv_slots_kernel(ReserveArgs a) {
  const int b = blockIdx.x;
  const int lo = clampi(a.offs[b], 0, a.rows);
  const int hi = clampi(a.offs[b + 1], lo, a.rows);
  const int start = a.start[b];
  const int mask = (1 << a.page_log2) - 1;
  for (int r = lo + blockIdx.y * 256 + threadIdx.x; r < hi; r += gridDim.y * 256) {
    int slot = -1;
    if (start >= 0) {
      const int t = start + (r - lo);
      const int page = a.table[(int64_t)b * a.max_pages + (t >> a.page_log2)];
      if ((uint32_t)page < (uint32_t)a.n_pages) slot = (page << a.page_log2) + (t & mask);
    }
    a.slots[r] = slot;
  }
  const int end = clampi(a.offs[a.B], 0, a.rows);
  const int64_t all = (int64_t)gridDim.x * gridDim.y * 256;
  for (int64_t r = end + ((int64_t)blockIdx.y * gridDim.x + b) * 256 + threadIdx.x; r < a.rows; r += all) a.slots[r] = -1;
}

// 8 bf16 (a 16-byte load) / scale, limited to +-448, as 8 bytes of e4m3.
__device__ __forceinline__ u32x2_t to_e4m3(const u32x4_t& x, float scale) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = bf16_to_f32((i & 1) ? x[i >> 1] >> 16 : x[i >> 1] & 0xffffu) / scale;
    f[i] = v != v ? v : fminf(fmaxf(v, -448.0f), 448.0f);
  }
  u32x2_t r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h], f[4 * h + 1], 0, false);
    r[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h + 2], f[4 * h + 3], w, true);
  }
  return r;
}

template <bool kE4m3>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
  constexpr int kPer = kE4m3 ? 8 : 16;  // 16-byte chunks of a page per row and head
  constexpr int kRow = kPer * 16;
  const int per_row = 2 * a.Hkv * kPer;  // chunks of K, then of V
  const int64_t n = (int64_t)a.rows * per_row;
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
    const int r = (int)(i / per_row);
    int c = (int)(i - (int64_t)r * per_row);
    const int slot = a.slots[r];
    if ((uint32_t)slot >= (uint32_t)a.n_slots) continue;
    const bool is_v = c >= a.Hkv * kPer;
    if (is_v) c -= a.Hkv * kPer;
    const int h = c / kPer;
    const char* src = (is_v ? a.v_new + (int64_t)r * a.v_ld : a.k_new + (int64_t)r * a.k_ld) + (int64_t)c * (kE4m3 ? 32 : 16);
    char* dst = (is_v ? a.v : a.k) + (int64_t)(slot >> a.page_log2) * a.page_bytes +
                (((int64_t)h << a.page_log2) + (slot & ((1 << a.page_log2) - 1))) * kRow + (c & (kPer - 1)) * 16;
    if constexpr (kE4m3) {
      const float* sc = is_v ? a.v_scale : a.k_scale;
      const float s = sc ? sc[h] : 1.0f;
      const u32x4_t x = gload16(src), y = gload16(src + 16);
      const u32x2_t p = to_e4m3(x, s), q = to_e4m3(y, s);
      *reinterpret_cast<u32x4_t*>(dst) = u32x4_t{p.x, p.y, q.x, q.y};
    } else {
      *reinterpret_cast<u32x4_t*>(dst) = gload16(src);
    }
  }
}

}  // namespace

hipError_t launch_kv_reserve(ReserveArgs a, hipStream_t stream) {
  // Rows that one workgroup deals out itself: up to the time that a second launch takes.
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

hipError_t launch_kv_append(const AppendArgs& a, bool e4m3, hipStream_t stream) {
  if (a.rows == 0) return hipSuccess;
  const int64_t n = (int64_t)a.rows * 2 * a.Hkv * (e4m3 ? 8 : 16);
  const int64_t blocks = (n + 255) / 256;
  const int grid = (int)(blocks < 16384 ? blocks : 16384);
  if (e4m3)
    hipLaunchKernelGGL(kv_append_kernel<true>, dim3(grid), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(kv_append_kernel<false>, dim3(grid), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ce
