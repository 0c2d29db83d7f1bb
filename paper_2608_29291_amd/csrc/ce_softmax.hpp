// The weights of a softmax over scores of any size, shared by the attention kernels.
#pragma once

#include <hip/hip_runtime.h>

#include "ce_device.hpp"

namespace ce {

constexpr float kFar = 8192.0f;  // size of a maximum's exponent from which differences are taken first

// The exponent of a weight is fma(score, c2, -mc) with mc = m c2 rounded. That rounding,
// 2^-25 of mc, is common to the keys of one maximum, but not to those of another that meet
// them (2^-12 at kFar), and past 2^31 it is hundreds and more: 2 to that is no float. From
// kFar on, rows take (score - m) c2, exact up to two roundings of the difference itself;
// scores so large are rare, and a wave looks for them where its maxima move. The branch costs
// tiles of 128 rows of a paged cache 0.2 to 0.7% (a look at every block 1 to 2.2%; kept in the
// branch that moves the maxima, which such rows then always take, 0.6 to 1.5%).
__device__ __forceinline__ float exponent_of(float m, float c2) { return m == -__builtin_inff() ? 0.0f : m * c2; }
__device__ __forceinline__ bool any_far(float mc) { return __builtin_amdgcn_ballot_w64(fabsf(mc) > kFar) != 0; }
// Scores become exponents, each row's by its own rule, whatever the wave's other rows do, and
// the scale and offset still to come those of nothing.
__device__ __forceinline__ void far_scores(f32x16_t& sc, float m, float c2, float& mc, float& ce) {
  const bool far = fabsf(mc) > kFar;
#pragma unroll
  for (int v = 0; v < 16; ++v) sc[v] = far ? (sc[v] - m) * c2 : fmaf(sc[v], c2, -mc);
  mc = 0.0f;
  ce = 1.0f;
}

}  // namespace ce
