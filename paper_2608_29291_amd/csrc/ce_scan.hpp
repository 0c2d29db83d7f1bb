// Prefix sums of one workgroup of 1024 threads, and searches in them (the paged cache's
// bookkeeping: ce_kv_cache.hip, ce_draft.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ce {

namespace scan {

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// a + b, at most 2^32 - 1: a bad batch may need any number of pages, and what is
// more than the pool holds is refused all the same.
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Inclusive prefix sum over the wave (row shifts, then the rows' last lanes).
__device__ __forceinline__ uint32_t wave_scan_sat(uint32_t v) {
  v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false));
  v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false));
  v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false));
  v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false));
  v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));
  v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));
  return v;
}

// Prefix sums of a and b up to this thread of the workgroup's 1024, itself included,
// and their totals (scr: 32 words of LDS). Every thread must call it.
__device__ __forceinline__ void scan2(uint32_t& a, uint32_t& b, uint32_t& ta, uint32_t& tb, uint32_t* scr) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  a = wave_scan_sat(a);
  b = wave_scan_sat(b);
  __syncthreads();
  if (lane == 63) {
    scr[wave] = a;
    scr[16 + wave] = b;
  }
  __syncthreads();
  // lanes 0 .. 15 hold the waves' totals of a, 16 .. 31 those of b
  uint32_t t = lane < 32 ? scr[lane] : 0;
  t = add_sat(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x111, 0xf, 0xf, false));
  t = add_sat(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x112, 0xf, 0xf, false));
  t = add_sat(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x114, 0xf, 0xf, false));
  t = add_sat(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x118, 0xf, 0xf, false));
  ta = __builtin_amdgcn_readlane(t, 15);
  tb = __builtin_amdgcn_readlane(t, 31);
  const int w = __builtin_amdgcn_readfirstlane(wave);
  if (w > 0) {
    a = add_sat(a, __builtin_amdgcn_readlane(t, w - 1));
    b = add_sat(b, __builtin_amdgcn_readlane(t, 15 + w));
  }
}

// The last i of 0 .. n - 1 with first[i] <= x (first: non-decreasing, first[0] <= x).
__device__ __forceinline__ int last_at_most(const int* first, int n, int x) {
  int lo = 0;
  for (int step = 512; step > 0; step >>= 1)
    if (lo + step < n && first[lo + step] <= x) lo += step;
  return lo;
}

}  // namespace scan

}  // namespace ce
