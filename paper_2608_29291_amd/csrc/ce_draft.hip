// Bookkeeping of drafted decoding (include/ce_router_draft.h): masks of trees, and the accepted
// rows of a step in the paged cache.
//
// Masks. Row i sees itself and its ancestors, whose numbers fall. Rows are taken 32 at a time, a word of
// the masks: five rounds of doubling (m |= m[p], p = p[p], by exchanges in the wave) give a row's
// ancestors among its 32 and the parent where they leave these, and a walk along these exits,
// through LDS, meets each word at most once: 22 steps for a chain of 700, not 700. Bound:
// latency; 16 trees of 26 rows 2.8 us, 253 of 64 and 33 with three chains of 700 and masks of 24 words
// 6.8 us (a walk parent by parent 207).
//
// Keep. Token start + j becomes token start + r_j with r_0 < r_1 < ..., so r_j >= j: what is
// written has been read before, as long as the rows are moved in order. A thread moves
// 16 bytes of a head of every row, eight rows loaded before the first is stored, and no
// other thread touches its bytes: no barrier, no copy.
//
// Trim. As ce_kv_reserve's pages of handed-on sequences: one workgroup, a prefix sum of the pages
// that come back, dealt to threads by a search in it.
#include "ce_device.hpp"
#include "ce_draft.hpp"
#include "ce_scan.hpp"

namespace ce {

namespace {

using namespace scan;

// A parent is before its row, or there is none (-1).
__device__ __forceinline__ int parent_of(int p, int i) { return p < 0 || p >= i ? -1 : p; }

constexpr int kStaged = 8192;  // rows whose words and exits LDS holds
constexpr int kTurn = 2048;    // of a longer sequence, at a time

// The word of row j, of which `up` is the parent, and the parent that it leaves its 32 rows by. Every lane
// of the 32 must call it.
__device__ __forceinline__ void link(int up, int j, uint32_t& m, int& exit) {
  const int first = j & ~31;
  int p = up >= first ? up & 31 : j & 31;  // (a row without one here points at itself)
  m = 1u << (j & 31);
#pragma unroll
  for (int r = 0; r < 5; ++r) {
    m |= (uint32_t)__shfl((int)m, p, 32);
    p = __shfl(p, p, 32);
  }
  exit = __shfl(up >= first ? -1 : up, p, 32);
}

// Masks and positions of a sequence longer than LDS holds, by one workgroup, kTurn rows at a time. Masks have bits of
// the first kTurn rows only (64 words at most), so a later row's mask is that of the row by which its walk leaves
// its kTurn, and its position follows that row's: 64 steps a row at most, however far the first ancestor is.
// One workgroup's latency bounds it: positions of a chain of 65536 rows 0.6 ms, with masks of 64 words 4.2; of
// 2^20 rows 9.5 ms (parent by parent to the root that is 2^39 steps).
__device__ __forceinline__ void long_sequence(const DraftMaskArgs& a, int lo, int n, int base, uint32_t* lds) {
  static_assert(kTurn >= 64 * 32 && kTurn % 256 == 0 && 4 * kTurn <= 3 * kStaged, "");
  uint32_t* const own = lds;
  int* const out = reinterpret_cast<int*>(lds + kTurn);
  const int tid = threadIdx.x, lane = tid & 63;
  for (int t0 = 0; t0 < n; t0 += kTurn) {
    const int here = min(kTurn, n - t0);
    for (int k0 = 0; k0 < here; k0 += 256) {
      const int j = t0 + k0 + tid;
      uint32_t m;
      int exit;
      link(j < n ? (a.parents ? parent_of(a.parents[lo + j], j) : j - 1) : -1, j, m, exit);
      own[k0 + tid] = m;
      out[k0 + tid] = exit;
    }
    __syncthreads();
    for (int k0 = 0; k0 < here; k0 += 256) {
      const int k = k0 + tid, i = t0 + k;
      int depth = 0, exit = -1;  // rows from i to the exit
      if (i < n) {
        for (exit = i; exit >= t0; exit = out[exit - t0]) depth += __builtin_popcount(own[exit - t0]);
        if (a.positions) a.positions[lo + i] = (int)((exit < 0 ? (uint32_t)base - 1 : (uint32_t)a.positions[lo + exit]) + (uint32_t)depth);
      }
      if (a.mask) {
        const int w0 = i & ~63, all = min(64, n - w0) * a.words;  // (none behind the last row)
        uint32_t* const to = a.mask + (int64_t)(lo + w0) * a.words;
        const uint32_t* const from = a.mask + (int64_t)lo * a.words;
        for (int c0 = 0; c0 < all; c0 += 64) {
          const int c = c0 + lane, r = min(c / a.words, 63);
          const int e = __shfl(exit, r);
          if (c < all) to[c] = e < 0 ? 0 : from[(int64_t)e * a.words + (c - r * a.words)];
        }
        if (t0 == 0) {  // and their words over these zeros
          asm volatile("" ::: "memory");
          wait_vmcnt<0>();
          if (i < n)
            for (int e = i; e >= 0; e = out[e])
              if (e >> 5 < a.words) a.mask[(int64_t)(lo + i) * a.words + (e >> 5)] = own[e];
        }
      }
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(256) void draft_masks_kernel(DraftMaskArgs a) {
  // words of the rows and their exits, `staged` of each
  extern __shared__ uint32_t lds[];
  uint32_t* const own = lds;
  int16_t* const out = reinterpret_cast<int16_t*>(lds + a.staged);
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int lo = clampi(a.offs[b], 0, a.rows);
  const int n = clampi(a.offs[b + 1], lo, a.rows) - lo;
  const int base = a.base ? a.base[b] : 0;
  if (n > a.staged) {
    if (blockIdx.y == 0) long_sequence(a, lo, n, base, lds);
    return;
  }
  int done = 0;  // rows that are staged
  // rows 256 y .., and on from there by as many as the workgroups of the sequence take
  for (int i0 = blockIdx.y * 256; i0 < n; i0 += gridDim.y * 256) {
    const int i = i0 + tid;
    uint32_t m = 0;
    int exit = -1;
    for (int j0 = done; j0 <= i0; j0 += 4 * 256) {
      int up[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int j = j0 + 256 * k + tid;
        up[k] = j < n && j0 + 256 * k <= i0 ? (a.parents ? parent_of(a.parents[lo + j], j) : j - 1) : -1;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (j0 + 256 * k > i0) break;
        const int j = j0 + 256 * k + tid;
        link(up[k], j, m, exit);
        own[j] = m;
        out[j] = (int16_t)exit;
      }
    }
    done = i0 + 256;
    // the wave's rows are zeros, and then their words that are none
    if (a.mask) {
      const int w0 = i0 + (tid & ~63);
      uint32_t* const to = a.mask + (int64_t)(lo + w0) * a.words;
      for (int k = lane; k < min(64, n - w0) * a.words; k += 64) to[k] = 0;
      asm volatile("" ::: "memory");
      wait_vmcnt<0>();
    }
    __syncthreads();
    if (i < n) {
      uint32_t* const row = a.mask + (int64_t)(lo + i) * a.words;
      int w = i >> 5, depth = -1;
      for (;;) {
        depth += __builtin_popcount(m);
        if (a.mask && w < a.words) row[w] = m;
        if (exit < 0) break;
        w = exit >> 5;
        m = own[exit];
        exit = out[exit];
      }
      if (a.positions) a.positions[lo + i] = (int)((uint32_t)base + (uint32_t)depth);
    }
    __syncthreads();
  }
}

// CE_DEV_* bits of the trees. One workgroup.
__global__ __launch_bounds__(1024) void draft_status_kernel(DraftMaskArgs a) {
  __shared__ uint32_t st_s;
  if (threadIdx.x == 0) st_s = 0;
  __syncthreads();
  uint32_t st = 0;
  for (int b = threadIdx.x; b < a.B; b += 1024) {
    const int o0 = a.offs[b], o1 = a.offs[b + 1];
    if (o0 < 0 || o1 < o0 || (b == 0 && o0 != 0)) st |= CE_DEV_BAD_OFFSETS;
    if (o0 > a.rows || o1 > a.rows) st |= CE_DEV_OVERFLOW;
    const int lo = clampi(o0, 0, a.rows), n = clampi(o1, lo, a.rows) - lo;
    if (a.mask && n > 32 * a.words) st |= CE_DEV_TOO_WIDE;
  }
  if (a.parents)
    for (int b = threadIdx.x >> 6; b < a.B; b += 16) {
      const int lo = clampi(a.offs[b], 0, a.rows), n = clampi(a.offs[b + 1], lo, a.rows) - lo;
      for (int i = threadIdx.x & 63; i < n; i += 64)
        if (a.parents[lo + i] >= i) st |= CE_DEV_BAD_TREE;
    }
  if (st) atomicOr(&st_s, st);
  __syncthreads();
  if (threadIdx.x == 0) *a.status = st_s;
}

constexpr int kAhead = 8;  // rows in flight in a thread

__global__ __launch_bounds__(256) void kv_keep_kernel(KeepArgs a) {
  const int b = blockIdx.x >> 1;
  const bool is_v = blockIdx.x & 1;
  const int start = a.start[b];
  const int lo = clampi(a.offs[b], 0, a.rows);
  const int n = clampi(a.offs[b + 1], lo, a.rows) - lo;
  const int kept = clampi(a.n_kept[b], 0, n);
  if (start < 0 || kept == 0) return;
  char* const pool = is_v ? a.v : a.k;
  const int32_t* const table = a.table + (int64_t)b * a.max_pages;
  const int64_t tokens = (int64_t)a.max_pages << a.page_log2;
  const int mask = (1 << a.page_log2) - 1;
  auto place = [&](int64_t token, bool& ok) {
    ok = token < tokens;
    const int page = ok ? table[token >> a.page_log2] : -1;
    ok = (uint32_t)page < (uint32_t)a.n_pages;
    return (int64_t)((uint64_t)(uint32_t)(ok ? page : 0) * a.page_bytes) + (token & mask) * a.row_bytes;
  };
  const int pieces = a.row_bytes / 16;
  for (int c = threadIdx.x; c < a.heads * pieces; c += blockDim.x) {
    const int h = c / pieces;
    char* const at = pool + ((int64_t)h << a.page_log2) * a.row_bytes + (c - h * pieces) * 16;
    int before = -1;
    for (int j0 = 0; j0 < kept; j0 += kAhead) {
      u32x4_t x[kAhead];
      int64_t to[kAhead];
      bool go[kAhead], good = true;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int j = j0 + i;
        go[i] = false;
        if (j >= kept) continue;
        const int r = a.kept[lo + j];
        good = good && r > before && r < n;
        before = r;
        if (!good || r == j) continue;
        bool ok0, ok1;
        const int64_t from = place((int64_t)start + r, ok0);
        to[i] = place((int64_t)start + j, ok1);
        go[i] = ok0 && ok1;
        if (go[i]) x[i] = *reinterpret_cast<const u32x4_t*>(at + from);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (go[i]) *reinterpret_cast<u32x4_t*>(at + to[i]) = x[i];
      if (!good) break;
    }
  }
}

__global__ __launch_bounds__(1024) void kv_trim_kernel(TrimArgs a) {
  __shared__ uint32_t scr[32];
  __shared__ int first[1024], held[1024];
  __shared__ uint32_t st_s;
  const int tid = threadIdx.x;
  if (tid == 0) st_s = 0;
  const int count0 = *a.count;
  int count = clampi(count0, 0, a.n_pages);
  uint32_t st = count != count0 ? CE_DEV_BAD_CACHE : 0;
  const int most = a.max_pages << a.page_log2;
  const uint32_t up = (1u << a.page_log2) - 1;
  for (int s0 = 0; s0 < a.B; s0 += 1024) {
    const int b = s0 + tid;
    uint32_t back = 0, none = 0, total, t2;
    held[tid] = 0;
    if (b < a.B) {
      const int len0 = a.lens[b], start = a.start[b], kept = a.n_kept[b];
      const int len = clampi(len0, 0, most);
      int now = len;
      if (start >= 0) now = (int)min((int64_t)len, (int64_t)start + max(kept, 0));
      if (len != len0 || (start >= 0 && (kept < 0 || (int64_t)start + kept > len))) st |= CE_DEV_BAD_CACHE;
      a.lens_out[b] = now;
      held[tid] = (int)(((uint32_t)now + up) >> a.page_log2);
      back = (((uint32_t)len + up) >> a.page_log2) - (uint32_t)held[tid];
    }
    uint32_t to = back;
    scan2(to, none, total, t2, scr);
    // (more than the stack has room for is pushed only if pages are held twice)
    first[tid] = (int)min(to - back, (uint32_t)a.n_pages);
    const uint32_t room = a.n_pages - count;
    if (total > room) st |= CE_DEV_BAD_CACHE;
    const int pushed = (int)min(total, room);
    __syncthreads();
    for (int i = tid; i < pushed; i += 1024) {
      const int k = last_at_most(first, 1024, i);
      const int page = a.table[(int64_t)(s0 + k) * a.max_pages + held[k] + (i - first[k])];
      if ((uint32_t)page >= (uint32_t)a.n_pages) st |= CE_DEV_BAD_CACHE;
      a.free_pages[count + i] = page;
    }
    count += pushed;
    __syncthreads();
  }
  if (st) atomicOr(&st_s, st);
  __syncthreads();
  if (tid == 0) {
    *a.count_out = count;
    if (a.status) *a.status = st_s;
  }
}

}  // namespace

hipError_t launch_draft_masks(DraftMaskArgs a, hipStream_t stream) {
  if (a.mask || a.positions) {
    // (whole passes of 256 rows)
    a.staged = a.rows < kStaged ? (a.rows + 255) / 256 * 256 : kStaged;
    const int passes = (a.rows + 255) / 256;
    const dim3 grid(a.B, passes < 4 ? (passes < 1 ? 1 : passes) : 4);
    hipLaunchKernelGGL(draft_masks_kernel, grid, dim3(256), (size_t)a.staged * 6, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.status) {
    hipLaunchKernelGGL(draft_status_kernel, dim3(1), dim3(1024), 0, stream, a);
    return hipGetLastError();
  }
  return hipSuccess;
}

hipError_t launch_kv_keep(const KeepArgs& a, hipStream_t stream) {
  if (a.rows == 0) return hipSuccess;
  const int columns = a.heads * (a.row_bytes / 16);
  const int threads = columns >= 256 ? 256 : (columns + 63) / 64 * 64;
  hipLaunchKernelGGL(kv_keep_kernel, dim3(2 * a.B), dim3(threads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_kv_trim(const TrimArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(kv_trim_kernel, dim3(1), dim3(1024), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ce
