// Verification of drafted tokens against the target's probabilities (include/ce_router_draft.h).
//
// Sampling. A token is the first whose running sum of weights w_i = exp((l_i - max) / T) is above u
// times their whole. A row of 1e5 tokens has borders 1e-5 and less apart, so exponentials and
// sums in 32 bits (1e-7, with the same sign for a large weight before many small ones) would
// move one token in a hundred. Weights are formed in 64 bits: 2^(k / 256) from a table in LDS
// and a polynomial of degree 3 for the rest (error 4e-14, which moves a token of a row of 1e5 with a
// chance of 1e-8); fp64 additions and fused products issue as fast as fp32 ones here.
//
// Passes. Every row is cut into chunks of 1024 tokens. Waves work alone: the one barrier of the first two is
// behind the table's fill.
//   1. verify_stats_kernel: sum of each chunk and the maximum that it is under, two chunks at a time, the one
//      pass over the logits.
//   2. verify_rows_kernel, a wave a row: the chunks' sums give the row's whole and the chunk of its
//      token, and that chunk's weights, formed again, the token; with probabilities of the
//      drafts, whether the row's first child is accepted. Rows that the walk will not reach are
//      worked on too: all at once they cost less than one after another. The last wave of
//      a sequence to arrive makes the walk.
// With probabilities, where a first child is rejected,
//   3. verify_rest_kernel: chunk sums of what the rejection leaves of the row, and by the last
//      workgroup of a sequence the other children and the rows that the walk reaches by them, and the
//      token. Each rejection after the first is a pass over its row by these four waves alone: stars of
//      rejected children, 17 us each at 32000 tokens, 60 at 131072 (75 in 16 sequences at once), where the
//      whole call without one takes 15 and 16 (26 to 68). Chains have one rejection at most.
// What rejections leave is max(p - c q, 0) with a growing c (max(max(p - a q, 0) - b q, 0) =
// max(p - (a + b) q, 0), as q >= 0), so nothing of a row is kept between them.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "ce_device.hpp"
#include "ce_draft.hpp"
#include "ce_host.hpp"

namespace ce {

namespace {

constexpr int kPer = 16;            // tokens of a lane
constexpr int kChunk = 64 * kPer;   // tokens of a wave
constexpr int kHeld = 4;            // chunks of a row that a lane holds
constexpr int kStepsLog2 = 8, kSteps = 1 << kStepsLog2;  // of an octave, in the table
// Weights below 2^-800 of a row's largest count as none: those below 2^-812 are zeros (or stand
// for themselves in a fast sum, where 1024 of them stay below 2^-800), and sums below 2^-800 are.
constexpr double kLeast = -812.0 * kSteps;
constexpr double kNone = 0x1p-800;

constexpr int kApart = 32;  // words between counters, a cache line: arrivals at one line wait for each other

__device__ const double kExpTable[kSteps] = {  // 2^(k / kSteps)
    0x1.0000000000000p+0, 0x1.00b1afa5abcbfp+0, 0x1.0163da9fb3335p+0, 0x1.02168143b0281p+0,
    0x1.02c9a3e778061p+0, 0x1.037d42e11bbccp+0, 0x1.04315e86e7f85p+0, 0x1.04e5f72f654b1p+0,
    0x1.059b0d3158574p+0, 0x1.0650a0e3c1f89p+0, 0x1.0706b29ddf6dep+0, 0x1.07bd42b72a836p+0,
    0x1.0874518759bc8p+0, 0x1.092bdf66607e0p+0, 0x1.09e3ecac6f383p+0, 0x1.0a9c79b1f3919p+0,
    0x1.0b5586cf9890fp+0, 0x1.0c0f145e46c85p+0, 0x1.0cc922b7247f7p+0, 0x1.0d83b23395decp+0,
    0x1.0e3ec32d3d1a2p+0, 0x1.0efa55fdfa9c5p+0, 0x1.0fb66affed31bp+0, 0x1.1073028d7233ep+0,
    0x1.11301d0125b51p+0, 0x1.11edbab5e2ab6p+0, 0x1.12abdc06c31ccp+0, 0x1.136a814f204abp+0,
    0x1.1429aaea92de0p+0, 0x1.14e95934f312ep+0, 0x1.15a98c8a58e51p+0, 0x1.166a45471c3c2p+0,
    0x1.172b83c7d517bp+0, 0x1.17ed48695bbc0p+0, 0x1.18af9388c8deap+0, 0x1.1972658375d2fp+0,
    0x1.1a35beb6fcb75p+0, 0x1.1af99f8138a1cp+0, 0x1.1bbe084045cd4p+0, 0x1.1c82f95281c6bp+0,
    0x1.1d4873168b9aap+0, 0x1.1e0e75eb44027p+0, 0x1.1ed5022fcd91dp+0, 0x1.1f9c18438ce4dp+0,
    0x1.2063b88628cd6p+0, 0x1.212be3578a819p+0, 0x1.21f49917ddc96p+0, 0x1.22bdda27912d1p+0,
    0x1.2387a6e756238p+0, 0x1.2451ffb82140ap+0, 0x1.251ce4fb2a63fp+0, 0x1.25e85711ece75p+0,
    0x1.26b4565e27cddp+0, 0x1.2780e341ddf29p+0, 0x1.284dfe1f56381p+0, 0x1.291ba7591bb70p+0,
    0x1.29e9df51fdee1p+0, 0x1.2ab8a66d10f13p+0, 0x1.2b87fd0dad990p+0, 0x1.2c57e39771b2fp+0,
    0x1.2d285a6e4030bp+0, 0x1.2df961f641589p+0, 0x1.2ecafa93e2f56p+0, 0x1.2f9d24abd886bp+0,
    0x1.306fe0a31b715p+0, 0x1.31432edeeb2fdp+0, 0x1.32170fc4cd831p+0, 0x1.32eb83ba8ea32p+0,
    0x1.33c08b26416ffp+0, 0x1.3496266e3fa2dp+0, 0x1.356c55f929ff1p+0, 0x1.36431a2de883bp+0,
    0x1.371a7373aa9cbp+0, 0x1.37f26231e754ap+0, 0x1.38cae6d05d866p+0, 0x1.39a401b7140efp+0,
    0x1.3a7db34e59ff7p+0, 0x1.3b57fbfec6cf4p+0, 0x1.3c32dc313a8e5p+0, 0x1.3d0e544ede173p+0,
    0x1.3dea64c123422p+0, 0x1.3ec70df1c5175p+0, 0x1.3fa4504ac801cp+0, 0x1.40822c367a024p+0,
    0x1.4160a21f72e2ap+0, 0x1.423fb2709468ap+0, 0x1.431f5d950a897p+0, 0x1.43ffa3f84b9d4p+0,
    0x1.44e086061892dp+0, 0x1.45c2042a7d232p+0, 0x1.46a41ed1d0057p+0, 0x1.4786d668b3237p+0,
    0x1.486a2b5c13cd0p+0, 0x1.494e1e192aed2p+0, 0x1.4a32af0d7d3dep+0, 0x1.4b17dea6db7d7p+0,
    0x1.4bfdad5362a27p+0, 0x1.4ce41b817c114p+0, 0x1.4dcb299fddd0dp+0, 0x1.4eb2d81d8abffp+0,
    0x1.4f9b2769d2ca7p+0, 0x1.508417f4531eep+0, 0x1.516daa2cf6642p+0, 0x1.5257de83f4eefp+0,
    0x1.5342b569d4f82p+0, 0x1.542e2f4f6ad27p+0, 0x1.551a4ca5d920fp+0, 0x1.56070dde910d2p+0,
    0x1.56f4736b527dap+0, 0x1.57e27dbe2c4cfp+0, 0x1.58d12d497c7fdp+0, 0x1.59c0827ff07ccp+0,
    0x1.5ab07dd485429p+0, 0x1.5ba11fba87a03p+0, 0x1.5c9268a5946b7p+0, 0x1.5d84590998b93p+0,
    0x1.5e76f15ad2148p+0, 0x1.5f6a320dceb71p+0, 0x1.605e1b976dc09p+0, 0x1.6152ae6cdf6f4p+0,
    0x1.6247eb03a5585p+0, 0x1.633dd1d1929fdp+0, 0x1.6434634ccc320p+0, 0x1.652b9febc8fb7p+0,
    0x1.6623882552225p+0, 0x1.671c1c70833f6p+0, 0x1.68155d44ca973p+0, 0x1.690f4b19e9538p+0,
    0x1.6a09e667f3bcdp+0, 0x1.6b052fa75173ep+0, 0x1.6c012750bdabfp+0, 0x1.6cfdcddd47645p+0,
    0x1.6dfb23c651a2fp+0, 0x1.6ef9298593ae5p+0, 0x1.6ff7df9519484p+0, 0x1.70f7466f42e87p+0,
    0x1.71f75e8ec5f74p+0, 0x1.72f8286ead08ap+0, 0x1.73f9a48a58174p+0, 0x1.74fbd35d7cbfdp+0,
    0x1.75feb564267c9p+0, 0x1.77024b1ab6e09p+0, 0x1.780694fde5d3fp+0, 0x1.790b938ac1cf6p+0,
    0x1.7a11473eb0187p+0, 0x1.7b17b0976cfdbp+0, 0x1.7c1ed0130c132p+0, 0x1.7d26a62ff86f0p+0,
    0x1.7e2f336cf4e62p+0, 0x1.7f3878491c491p+0, 0x1.80427543e1a12p+0, 0x1.814d2add106d9p+0,
    0x1.82589994cce13p+0, 0x1.8364c1eb941f7p+0, 0x1.8471a4623c7adp+0, 0x1.857f4179f5b21p+0,
    0x1.868d99b4492edp+0, 0x1.879cad931a436p+0, 0x1.88ac7d98a6699p+0, 0x1.89bd0a478580fp+0,
    0x1.8ace5422aa0dbp+0, 0x1.8be05bad61778p+0, 0x1.8cf3216b5448cp+0, 0x1.8e06a5e0866d9p+0,
    0x1.8f1ae99157736p+0, 0x1.902fed0282c8ap+0, 0x1.9145b0b91ffc6p+0, 0x1.925c353aa2fe2p+0,
    0x1.93737b0cdc5e5p+0, 0x1.948b82b5f98e5p+0, 0x1.95a44cbc8520fp+0, 0x1.96bdd9a7670b3p+0,
    0x1.97d829fde4e50p+0, 0x1.98f33e47a22a2p+0, 0x1.9a0f170ca07bap+0, 0x1.9b2bb4d53fe0dp+0,
    0x1.9c49182a3f090p+0, 0x1.9d674194bb8d5p+0, 0x1.9e86319e32323p+0, 0x1.9fa5e8d07f29ep+0,
    0x1.a0c667b5de565p+0, 0x1.a1e7aed8eb8bbp+0, 0x1.a309bec4a2d33p+0, 0x1.a42c980460ad8p+0,
    0x1.a5503b23e255dp+0, 0x1.a674a8af46052p+0, 0x1.a799e1330b358p+0, 0x1.a8bfe53c12e59p+0,
    0x1.a9e6b5579fdbfp+0, 0x1.ab0e521356ebap+0, 0x1.ac36bbfd3f37ap+0, 0x1.ad5ff3a3c2774p+0,
    0x1.ae89f995ad3adp+0, 0x1.afb4ce622f2ffp+0, 0x1.b0e07298db666p+0, 0x1.b20ce6c9a8952p+0,
    0x1.b33a2b84f15fbp+0, 0x1.b468415b749b1p+0, 0x1.b59728de5593ap+0, 0x1.b6c6e29f1c52ap+0,
    0x1.b7f76f2fb5e47p+0, 0x1.b928cf22749e4p+0, 0x1.ba5b030a1064ap+0, 0x1.bb8e0b79a6f1fp+0,
    0x1.bcc1e904bc1d2p+0, 0x1.bdf69c3f3a207p+0, 0x1.bf2c25bd71e09p+0, 0x1.c06286141b33dp+0,
    0x1.c199bdd85529cp+0, 0x1.c2d1cd9fa652cp+0, 0x1.c40ab5fffd07ap+0, 0x1.c544778fafb22p+0,
    0x1.c67f12e57d14bp+0, 0x1.c7ba88988c933p+0, 0x1.c8f6d9406e7b5p+0, 0x1.ca3405751c4dbp+0,
    0x1.cb720dcef9069p+0, 0x1.ccb0f2e6d1675p+0, 0x1.cdf0b555dc3fap+0, 0x1.cf3155b5bab74p+0,
    0x1.d072d4a07897cp+0, 0x1.d1b532b08c968p+0, 0x1.d2f87080d89f2p+0, 0x1.d43c8eacaa1d6p+0,
    0x1.d5818dcfba487p+0, 0x1.d6c76e862e6d3p+0, 0x1.d80e316c98398p+0, 0x1.d955d71ff6075p+0,
    0x1.da9e603db3285p+0, 0x1.dbe7cd63a8315p+0, 0x1.dd321f301b460p+0, 0x1.de7d5641c0658p+0,
    0x1.dfc97337b9b5fp+0, 0x1.e11676b197d17p+0, 0x1.e264614f5a129p+0, 0x1.e3b333b16ee12p+0,
    0x1.e502ee78b3ff6p+0, 0x1.e653924676d76p+0, 0x1.e7a51fbc74c83p+0, 0x1.e8f7977cdb740p+0,
    0x1.ea4afa2a490dap+0, 0x1.eb9f4867cca6ep+0, 0x1.ecf482d8e67f1p+0, 0x1.ee4aaa2188510p+0,
    0x1.efa1bee615a27p+0, 0x1.f0f9c1cb6412ap+0, 0x1.f252b376bba97p+0, 0x1.f3ac948dd7274p+0,
    0x1.f50765b6e4540p+0, 0x1.f6632798844f8p+0, 0x1.f7bfdad9cbe14p+0, 0x1.f91d802243c89p+0,
    0x1.fa7c1819e90d8p+0, 0x1.fbdba3692d514p+0, 0x1.fd3c22b8f71f1p+0, 0x1.fe9d96b2a23d9p+0,
};

struct VerifyArgs {
  int B, rows, vocab, chunks;
  const int32_t *offs, *parents, *tokens;  // parents may be NULL
  const char* logits;
  int64_t ld;  // bytes
  const float* temps;  // or NULL
  const float* probs;  // or NULL
  int64_t probs_ld;
  const float *u_accept, *u_sample;
  int32_t *kept, *n_kept, *next;
  float* top;   // [rows x chunks]
  double* sum;  // [rows x chunks], under the chunk's own maximum
  int32_t* out;      // [rows]: the token of a row; or its first child, accepted or rejected
  uint32_t* arrived; // [B x kApart]: waves of a sequence that are done, and workgroups
  // with probabilities:
  float* most;     // [rows]: maximum and whole of a row
  double* whole;
  double* rest;    // [B x chunks]: chunk sums after the first rejection
  int32_t* at;     // [B]: the walk's row with a rejection, or -1
};

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }
__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

// What every lane has alike, in scalar registers: branches on it need no masks of lanes.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ bool uniform(bool x) { return __builtin_amdgcn_readfirstlane((int)x) != 0; }
__device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

// The lane, of which a loop's comparisons are not formed before it: they would fill the
// scalar registers.
__device__ __forceinline__ int own_lane() {
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  return lane;
}

__device__ __forceinline__ double of_lane(double x, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)u, lane), hi = __builtin_amdgcn_readlane((uint32_t)(u >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Largest over the wave; NaN is passed over.
__device__ __forceinline__ float wave_max(float v) {
#define CE_STEP(ctrl, rows) \
  v = fmaxf(v, __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp((int)0xff800000, (int)__float_as_uint(v), ctrl, rows, 0xf, false)))
  CE_STEP(0x111, 0xf);
  CE_STEP(0x112, 0xf);
  CE_STEP(0x114, 0xf);
  CE_STEP(0x118, 0xf);
  CE_STEP(0x142, 0xa);
  CE_STEP(0x143, 0xc);
#undef CE_STEP
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}

// Inclusive prefix sum over the wave (row shifts, then the rows' last lanes).
__device__ __forceinline__ double wave_scan(double v) {
  auto step = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
    const uint32_t hi =
        __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
    v += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  };
  step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});
  step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
  step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
  step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
  step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
  step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
  return v;
}

// Sums of a and b over the wave, in lane 0 of the result and in lane 32.
__device__ __forceinline__ double wave_sums(double a, double b) {
  const uint64_t ua = __builtin_bit_cast(uint64_t, a), ub = __builtin_bit_cast(uint64_t, b);
  // (the upper half of a and the lower of b change places)
  const auto lo = __builtin_amdgcn_permlane32_swap((uint32_t)ua, (uint32_t)ub, false, false);
  const auto hi = __builtin_amdgcn_permlane32_swap((uint32_t)(ua >> 32), (uint32_t)(ub >> 32), false, false);
  double v = __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
  auto step = [&](auto ctrl) __attribute__((always_inline)) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t x = __builtin_amdgcn_mov_dpp((int)(uint32_t)u, decltype(ctrl)::value, 0xf, 0xf, true);
    const uint32_t y = __builtin_amdgcn_mov_dpp((int)(uint32_t)(u >> 32), decltype(ctrl)::value, 0xf, 0xf, true);
    v += __builtin_bit_cast(double, (uint64_t)y << 32 | x);
  };
  step(std::integral_constant<int, 0xb1>{});   // lanes ^ 1
  step(std::integral_constant<int, 0x4e>{});   // ^ 2
  step(std::integral_constant<int, 0x141>{});  // mirrored in 8, and in 16
  step(std::integral_constant<int, 0x140>{});
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const auto x = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false);
  const auto y = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  return __builtin_bit_cast(double, (uint64_t)y[0] << 32 | x[0]) + __builtin_bit_cast(double, (uint64_t)y[1] << 32 | x[1]);
}

// How the logits of a row become exponents: kSteps log2 e / T, or whether only the largest counts.
struct Heat {
  double s, over_s;  // and its inverse
  bool greedy;
};
__device__ __forceinline__ Heat heat_at(const VerifyArgs& a, int b) {  // (b: a lane's own)
  const float t = a.temps ? a.temps[b] : 1.0f;
  Heat h;
  h.greedy = !(t > 0.0f);
  const double heat = h.greedy ? 1.0 : (double)t;
  h.s = 0x1.71547652b82fep+8 / heat;  // kSteps log2 e
  h.over_s = 0x1.62e42fefa39efp-9 * heat;
  return h;
}
__device__ __forceinline__ Heat heat_of(const VerifyArgs& a, int b) {
  Heat h = heat_at(a, b);
  h.greedy = uniform(h.greedy);
  return h;
}

// The table, its upper words less by k << (20 - kStepsLog2): of any number of steps the word that goes to the exponent
// is then this many bits to the left, as it is (the steps in it cancel).
constexpr int kToExponent = 20 - kStepsLog2;
__device__ __forceinline__ void load_table(double* table) {
  for (int i = threadIdx.x; i < kSteps; i += blockDim.x)
    table[i] = __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, kExpTable[i]) - ((uint64_t)i << (32 + kToExponent)));
  __syncthreads();
}
// 2^(k / kSteps) of a normal result: three instructions (the first takes the low byte, eight times).
__device__ __forceinline__ double step_power(uint32_t k, const double* table) {
  static_assert(kStepsLog2 == 8, "a byte of steps");
  uint32_t at, hi;
  asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(at) : "v"(3), "v"(k));
  const uint64_t v = __builtin_bit_cast(uint64_t, *reinterpret_cast<const double*>(reinterpret_cast<const char*>(table) + at));
  asm("v_lshl_add_u32 %0, %1, %2, %3" : "=v"(hi) : "v"(k), "n"(kToExponent), "v"((uint32_t)(v >> 32)));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | (uint32_t)v);
}

// 2^(r / kSteps), |r| <= 1/2: with x = r ln 2 / kSteps the terms 1 + x + x^2 / 2 + x^3 / 6, and of the
// next, x^4 / 24, the part d^2 x^2 / 24 (d: the largest x). Off by 4e-14 at most.
__device__ __forceinline__ double small_power(double r) {
  return fma(r, fma(r, fma(r, 0x1.c6b08d704a0c0p-29, 0x1.ebfbe4e4d734ep-19), 0x1.62e42fefa39efp-9), 1.0);
}

// exp((x - m) / T); x of NaN or -infinity: 0.
__device__ __forceinline__ double weight(float x, double m, double s, const double* table) {
  const double t = fmax(((double)x - m) * s, kLeast);
  const double k = rint(t);
  return t > kLeast ? step_power((uint32_t)(int)k, table) * small_power(t - k) : 0.0;
}

// Weights under m of many tokens. With mi = rint(m s) the exponents are counted from mi on, so
// one fused product gives the number of the table's step (by adding 2^52, in the low bits of the sum) and
// one the rest, exactly: seven 64-bit operations a token, no conversion but the logit's. Exponents
// from kLeast on stand for those below. The weights are too large by 2^((m s - mi) / kSteps), `over`.
// Scales or logits that could leave this range (usable) take weight().
struct Fast {
  double c, s;
  float floor;
  bool usable;
  double over, under;  // 2^((m s - mi) / kSteps) and its inverse
};
__device__ __forceinline__ Fast fast_of(float m, const Heat& h) {
  const double mi = rint((double)m * h.s), least = (mi + kLeast) * h.over_s;
  Fast f;
  // (the floor's rounding to float32 moves its exponent by 2^-24 of mi: less than an octave)
  f.usable = uniform(fabs(mi) < 0x1p30 && fabs(least) < 0x1p126);
  f.c = 0x1.8p52 - mi;
  f.s = h.s;
  f.floor = (float)least;
  const double r = fma((double)m, h.s, -mi);
  f.over = small_power(r);
  f.under = small_power(-r);
  return f;
}
// A weight is t p.
template <int kN>
__device__ __forceinline__ void fast_weights(const float* x, const Fast& f, const double* table, double* t, double* p) {
  double l[kN], kd[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) l[i] = (double)__builtin_amdgcn_fmed3f(x[i], f.floor, 0x1.fffffep127f);  // (NaN: the floor)
#pragma unroll
  for (int i = 0; i < kN; ++i) kd[i] = fma(l[i], f.s, f.c);
#pragma unroll
  for (int i = 0; i < kN; ++i) t[i] = step_power((uint32_t)__builtin_bit_cast(uint64_t, kd[i]), table);
#pragma unroll
  for (int i = 0; i < kN; ++i) p[i] = small_power(fma(l[i], f.s, f.c - kd[i]));
}
// Sum of a lane's weights under m; fast_of(m), of a logit that is finite.
__device__ __forceinline__ double sum_weights(const float (&x)[kPer], float m, const Fast& f, const double* table) {
  double sum = 0.0;
  if (f.usable) {
    double other = 0.0;
#pragma unroll
    for (int i = 0; i < kPer; i += 4) {
      double t[4], p[4];
      fast_weights<4>(x + i, f, table, t, p);
      sum = fma(t[0], p[0], sum);
      other = fma(t[1], p[1], other);
      sum = fma(t[2], p[2], sum);
      other = fma(t[3], p[3], other);
    }
    return (sum + other) * f.under;
  }
#pragma unroll 1
  for (int i = 0; i < kPer; ++i) {
    // (one copy of this code: the values come by a chain of selections)
    float y = x[0];
#pragma unroll
    for (int k = 1; k < kPer; ++k) y = i == k ? x[k] : y;
    sum += weight(y, (double)m, f.s, table);
  }
  return sum;
}

__device__ __forceinline__ double counted(double sum) { return sum < kNone ? 0.0 : sum; }

// Where only the largest counts, by the temperature or because it is infinite, the others
// become -infinity and it 0.
__device__ __forceinline__ void flatten(float (&x)[kPer], float& m, const Heat& h) {
  if (!h.greedy && m != __builtin_inff()) return;
#pragma unroll
  for (int i = 0; i < kPer; ++i) x[i] = x[i] == m ? 0.0f : neg_inf();
  m = 0.0f;
}

// Of fewer than 64 sequences a lane holds one's first row and heat (lane B: the last one's end).
struct Held {
  int first;
  Heat h;
};
__device__ __forceinline__ Held hold_sequences(const VerifyArgs& a) {
  Held l = {};
  if (a.B < 64) {
    const int lane = threadIdx.x & 63;
    l.first = a.offs[min(lane, a.B)];
    l.h = heat_at(a, min(lane, a.B - 1));
  }
  return l;
}

// Rows behind the last sequence's end are nobody's (a padded batch). Of their logits the first pass reads what its
// waves take first, no more: 8192 pairs of chunks from row 0 on.
__device__ __forceinline__ int end_of(const VerifyArgs& a, const Held& l) {
  return clampi(a.B < 64 ? __builtin_amdgcn_readlane(l.first, a.B) : uniform(a.offs[a.B]), 0, a.rows);
}

// The sequence of a row before the end and its heat; -1: none. Every wave by itself.
__device__ __forceinline__ int sequence_of(const VerifyArgs& a, const Held& l, int row, Heat& h) {
  const int lane = threadIdx.x & 63;
  if (a.B < 64) {
    const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < a.B && l.first <= row));
    if (n == 0) return -1;
    const int b = n - 1;
    h.s = of_lane(l.h.s, b);
    h.over_s = of_lane(l.h.over_s, b);
    h.greedy = __builtin_amdgcn_readlane(l.h.greedy, b) != 0;
    return __builtin_amdgcn_readlane(l.first, b) <= row && row < __builtin_amdgcn_readlane(l.first, n) ? b : -1;
  }
  int lo = 0;
  for (int step = a.B > 4096 ? 4096 : 64; step > 0; step >>= 6) {
    const int i = lo + lane * step;
    const bool le = i < a.B && a.offs[i < a.B ? i : 0] <= row;
    const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(le));
    lo += (n > 0 ? n - 1 : 0) * step;
  }
  lo = uniform(lo);
  if (!uniform(a.offs[lo] <= row && row < a.offs[lo + 1])) return -1;
  h = heat_of(a, lo);
  return lo;
}

template <typename E>
constexpr int kVec = 16 / sizeof(E);
__device__ __forceinline__ float value(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ float value(float x) { return x; }

// 16 of a row's values from c0 on, a wave's kChunk in order: kVec at a time (whole lines; the sum of
// a chunk), or a lane's one after another (kInOrder; running sums). Behind the row's end: the last.
template <typename E>
struct Raw {
  u32x4_t v[kPer / kVec<E>];
};
// (rows may begin anywhere: a load of 16 bytes from the element's alignment on)
typedef uint32_t u32x4_2_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_4_t __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ u32x4_t load16(const uint16_t* p) { return *reinterpret_cast<const u32x4_2_t*>(p); }
__device__ __forceinline__ u32x4_t load16(const float* p) { return *reinterpret_cast<const u32x4_4_t*>(p); }
// Word w of the 16 bytes from element i on, of a row of n: its end repeated.
__device__ __forceinline__ uint32_t word_of(const uint16_t* row, int i, int w, int n) {
  return row[min(i + 2 * w, n - 1)] | (uint32_t)row[min(i + 2 * w + 1, n - 1)] << 16;
}
__device__ __forceinline__ uint32_t word_of(const float* row, int i, int w, int n) {
  return __float_as_uint(row[min(i + w, n - 1)]);
}
template <bool kInOrder, typename E>
__device__ __forceinline__ int token_of(int c0, int lane, int j) {
  return c0 + (kInOrder ? lane * kPer + j * kVec<E> : (j * 64 + lane) * kVec<E>);
}
template <bool kInOrder, typename E>
__device__ __forceinline__ Raw<E> load_raw(const E* row, int c0, int vocab) {
  Raw<E> r;
  const int lane = own_lane();
  if (c0 + kChunk <= vocab) {
#pragma unroll
    for (int j = 0; j < kPer / kVec<E>; ++j) r.v[j] = load16(row + token_of<kInOrder, E>(c0, lane, j));
  } else {
#pragma unroll
    for (int j = 0; j < kPer / kVec<E>; ++j)
#pragma unroll
      for (int w = 0; w < 4; ++w) r.v[j][w] = word_of(row, token_of<kInOrder, E>(c0, lane, j), w, vocab);
  }
  return r;
}
template <bool kInOrder, typename E>
__device__ __forceinline__ void unpack(const Raw<E>& r, int c0, int vocab, float none, float (&x)[kPer]) {
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const uint32_t w = r.v[i / kVec<E>][i % kVec<E> / (4 / (int)sizeof(E))];
    x[i] = __uint_as_float(sizeof(E) == 4 ? w : (i & 1 ? w & 0xffff0000u : w << 16));
  }
  if (c0 + kChunk > vocab) {
    const int lane = own_lane();
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (token_of<kInOrder, E>(c0, lane, i / kVec<E>) + i % kVec<E> >= vocab) x[i] = none;
  }
}
template <bool kInOrder, typename E>
__device__ __forceinline__ void load_values(const E* row, int c0, int vocab, float none, float (&x)[kPer]) {
  unpack<kInOrder>(load_raw<kInOrder>(row, c0, vocab), c0, vocab, none, x);
}

__device__ __forceinline__ double how_many(const float (&x)[kPer], float m) {
  int n = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    n += x[k] == m;
    asm volatile("" : "+v"(n));  // (one comparison at a time: sixteen results fill the scalar registers)
  }
  return n;
}

// Maximum and sums of two chunks of a row at a time, by waves that take
// such pairs in turn, the next one's logits on their way. The sequences' rows and heats stay in the
// lanes: looking them up for each pair anew cost a tenth of the time.
// Bound: memory and some 14 instructions a token: 521 rows of 131072 in bf16, 137 MB, a third of them with
// only the largest to count, 37 us, where reading them alone takes 28 (without the table's
// reads 34); 272 of 100003 in float32, 109 MB, 24.
template <typename E>
__global__ __launch_bounds__(256) void verify_stats_kernel(VerifyArgs a) {
  __shared__ double table[kSteps];
  const int pairs = (a.chunks + 1) / 2;
  const uint32_t waves = gridDim.x * 4, all = (uint32_t)a.rows * (uint32_t)pairs;
  const uint32_t i = blockIdx.x * 4 + (uint32_t)uniform((int)(threadIdx.x >> 6));
  const int rows_on = (int)(waves / (uint32_t)pairs), pairs_on = (int)(waves - (uint32_t)rows_on * pairs);
  int row = (int)(i / (uint32_t)pairs), pair = (int)(i - (uint32_t)row * pairs);
  for (uint32_t k = blockIdx.x * 256 + threadIdx.x; k < (uint32_t)a.B; k += gridDim.x * 256) {
    a.arrived[(int64_t)k * kApart] = a.arrived[(int64_t)k * kApart + 1] = 0;
    // (offsets out of order leave sequences without a walk)
    a.n_kept[k] = 0;
    a.next[k] = -1;
    if (a.probs) a.at[k] = -1;
  }
  Raw<E> raw0, raw1;
  auto load = [&]() __attribute__((always_inline)) {
    const int c = 2 * pair;
    const E* const l = reinterpret_cast<const E*>(a.logits + (int64_t)row * a.ld);
    raw0 = load_raw<false>(l, c * kChunk, a.vocab);
    raw1 = load_raw<false>(l, (c + 1) * kChunk, a.vocab);  // (a chunk that is none: the last token)
  };
  // (Beside the offsets, which may put it behind the end: us of the call, 16, 32, 64 and 128 rows of 131072 in use of
  // 128 12.3, 13.4, 15.7, 20.6, of 1024 13.9, 13.9, 17.1, 21.0; all 1024 91.)
  if (i < all) load();
  const Held held = hold_sequences(a);
  const int end = end_of(a, held);
  load_table(table);
  while (row < end) {
    Heat h = {};
    const int b = sequence_of(a, held, row, h), c = 2 * pair;
    float x0[kPer], x1[kPer];
    unpack<false>(raw0, c * kChunk, a.vocab, neg_inf(), x0);
    unpack<false>(raw1, (c + 1) * kChunk, a.vocab, neg_inf(), x1);
    const int64_t to = (int64_t)row * a.chunks + c;
    const bool two = c + 1 < a.chunks;
    row += rows_on;
    if ((pair += pairs_on) >= pairs) {
      pair -= pairs;
      ++row;
    }
    if (row < end) load();
    if (b < 0) continue;
    float m = neg_inf();
#pragma unroll
    for (int k = 0; k < kPer; ++k) m = fmaxf(m, fmaxf(x0[k], x1[k]));  // (NaN is passed over)
    m = wave_max(m);
    double whole = 0.0;  // of the first chunk in the lower lanes, of the second in the upper
    if (m != neg_inf()) {
      double w0, w1;
      if (h.greedy || m == __builtin_inff()) {  // only the largest count
        w0 = how_many(x0, m);
        w1 = how_many(x1, m);
      } else {
        const Fast f = fast_of(m, h);
        w0 = sum_weights(x0, m, f, table);
        w1 = sum_weights(x1, m, f, table);
      }
      whole = counted(wave_sums(w0, w1));
    }
    const int second = (threadIdx.x & 63) >> 5;
    if ((threadIdx.x & 31) == 0 && (second == 0 || two)) {
      a.top[to + second] = m;
      a.sum[to + second] = whole;
    }
  }
}

// A row's chunks, kHeld a lane, one after another: maxima and sums, of which a wave holds the first 64 kHeld.
struct Parts {
  float top[kHeld];
  double part[kHeld];  // sums, then parts of the whole
};
__device__ __forceinline__ void load_parts(const VerifyArgs& a, int row, int c0, Parts& p) {
  const int64_t at = (int64_t)row * a.chunks;
  const int lane = own_lane();
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int c = c0 + lane * kHeld + k;
    p.top[k] = c < a.chunks && a.rows > 0 ? a.top[at + c] : neg_inf();
    p.part[k] = c < a.chunks && a.rows > 0 ? a.sum[at + c] : 0.0;
  }
}
// Under the row's maximum m.
__device__ __forceinline__ void scale_parts(Parts& p, float m, const Heat& h, const double* table) {
  const bool flat = h.greedy || m == __builtin_inff();
#pragma unroll
  for (int k = 0; k < kHeld; ++k)
    p.part[k] = flat ? (p.top[k] == m ? p.part[k] : 0.0) : counted(p.part[k] * weight(p.top[k], (double)m, h.s, table));
}
__device__ __forceinline__ double sum_parts(const Parts& p) {
  double s = 0.0;
#pragma unroll
  for (int k = 0; k < kHeld; ++k) s += p.part[k];
  return of_lane(wave_scan(s), 63);
}

// Maximum and whole of a row's weights, by a wave; p: the first parts, loaded.
__device__ __forceinline__ void row_whole(const VerifyArgs& a, int row, const Heat& h, float& m, double& whole, Parts& p,
                                          const double* table) {
  m = neg_inf();
#pragma unroll
  for (int k = 0; k < kHeld; ++k) m = fmaxf(m, p.top[k]);
  Parts q;
  for (int c0 = 64 * kHeld; c0 < a.chunks; c0 += 64 * kHeld) {
    load_parts(a, row, c0, q);
#pragma unroll
    for (int k = 0; k < kHeld; ++k) m = fmaxf(m, q.top[k]);
  }
  m = wave_max(m);
  whole = 0.0;
  if (m == neg_inf()) return;
  scale_parts(p, m, h, table);
  whole = sum_parts(p);
  for (int c0 = 64 * kHeld; c0 < a.chunks; c0 += 64 * kHeld) {
    load_parts(a, row, c0, q);
    scale_parts(q, m, h, table);
    whole += sum_parts(q);
  }
}

// Of a wave's values w, kN a lane and one after another, the first whose running sum from `base` on is
// above target, or -1; base grows by their sum, and last becomes the last of a value (if there is any).
template <int kN>
__device__ __forceinline__ int first_above(const double (&w)[kN], int first, double target, double& base, double& before,
                                           int& last) {
  double mine = 0.0;
  int some = -1;
#pragma unroll
  for (int k = 0; k < kN; ++k) {
    mine += w[k];
    some = w[k] > 0.0 ? k : some;
  }
  const double to = wave_scan(mine);
  const uint64_t any = __builtin_amdgcn_ballot_w64(some >= 0);
  if (any) {
    const int ln = 63 - __builtin_clzll(any);
    last = first + ln * kN + __builtin_amdgcn_readlane(some, ln);
  }
  const uint64_t past = __builtin_amdgcn_ballot_w64(some >= 0 && base + to > target);
  int found = -1;
  if (past) {
    const int ln = __builtin_ctzll(past);
    double run = base + (to - mine), under = run;
    int token = -1;
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      const double next = run + w[k];
      const bool is = token < 0 && next > target && w[k] > 0.0;
      under = is ? run : under;
      token = is ? k : token;
      run = next;
    }
    if (token < 0) {  // (the sums' last bit)
      token = some;
      under = run;
    }
    found = first + ln * kN + __builtin_amdgcn_readlane(token, ln);
    before = of_lane(under, ln);
  }
  base += of_lane(to, 63);
  return found;
}

// Logits of a row, and the probabilities that its children were drawn from.
template <typename E>
struct Row {
  const E* l;
  const float* q;
};
template <typename E>
__device__ __forceinline__ Row<E> row_of(const VerifyArgs& a, int row) {
  return Row<E>{reinterpret_cast<const E*>(a.logits + (int64_t)row * a.ld), a.probs ? a.probs + (int64_t)row * a.probs_ld : nullptr};
}

// Probabilities in the order of the logits' type.
template <bool kInOrder, typename E>
__device__ __forceinline__ void load_probs(const float* row, int c0, int vocab, float (&q)[kPer]) {
  const int lane = own_lane();
#pragma unroll
  for (int i = 0; i < kPer; i += 4) {
    const int t = token_of<kInOrder, E>(c0, lane, i / kVec<E>) + i % kVec<E>;
    u32x4_t y;
    if (c0 + kChunk <= vocab) {
      y = load16(row + t);
    } else {
#pragma unroll
      for (int w = 0; w < 4; ++w) y[w] = word_of(row, t, w, vocab);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) q[i + k] = __uint_as_float(y[k]);
  }
}

// Weights of a chunk of a row after rejections (cw: c times the row's whole).
template <bool kInOrder, typename E>
__device__ __forceinline__ void rest_weights(const Row<E>& row, int c0, int vocab, float m, const Heat& h, double cw,
                                             double (&w)[kPer], const double* table) {
  float x[kPer];
  load_values<kInOrder>(row.l, c0, vocab, neg_inf(), x);
  if (uniform(cw == 0.0)) {
    flatten(x, m, h);
#pragma unroll
    for (int i = 0; i < kPer; ++i) w[i] = weight(x[i], (double)m, h.s, table);
    return;
  }
  float q[kPer];
  load_probs<kInOrder, E>(row.q, c0, vocab, q);
  flatten(x, m, h);
#pragma unroll
  for (int i = 0; i < kPer; ++i)  // (fmaxf: NaN counts as 0)
    w[i] = fmax(weight(x[i], (double)m, h.s, table) - cw * (double)fmaxf(q[i], 0.0f), 0.0);
}

// Sum of them over a wave, the chunk's tokens in any order.
template <typename E>
__device__ __forceinline__ double rest_sum(const Row<E>& row, int c0, int vocab, float m, const Heat& h, double cw,
                                           const double* table) {
  double sum = 0.0;
  const Fast f = fast_of(m, h);
  if (uniform(cw != 0.0) && f.usable) {
    float x[kPer], q[kPer];
    load_values<false>(row.l, c0, vocab, neg_inf(), x);
    load_probs<false, E>(row.q, c0, vocab, q);
    const double co = cw * f.over;
#pragma unroll
    for (int i = 0; i < kPer; i += 4) {
      double t[4], p[4];
      fast_weights<4>(x + i, f, table, t, p);
#pragma unroll
      for (int k = 0; k < 4; ++k) sum += fmax(t[k] * p[k] - co * (double)fmaxf(q[i + k], 0.0f), 0.0);
    }
    sum *= f.under;
  } else {
    double w[kPer];
    rest_weights<false>(row, c0, vocab, m, h, cw, w, table);
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum += w[i];
  }
  return counted(of_lane(wave_scan(sum), 63));
}

// The token of a row in the chunk where a running sum passes the target, `before` up to it.
template <typename E>
__device__ __forceinline__ int token_in(const VerifyArgs& a, const Row<E>& row, int chunk, float m, const Heat& h, double cw,
                                        double target, double before, const double* table) {
  double w[kPer], under;
  rest_weights<true>(row, chunk * kChunk, a.vocab, m, h, cw, w, table);
  int last = -1;
  const int token = first_above(w, chunk * kChunk, target, before, under, last);
  return token < 0 ? last : token;
}

// A token sampled from p itself.
template <typename E>
__device__ __forceinline__ int pick(const VerifyArgs& a, int row, float m, const Heat& h, double whole, const Parts& p,
                                    const double* table) {
  const double target = h.greedy ? 0.0 : (double)a.u_sample[row] * whole;
  double base = 0.0, before = 0.0;
  int last = 0, chunk = first_above(p.part, 0, target, base, before, last);
  for (int c0 = 64 * kHeld; c0 < a.chunks && chunk < 0; c0 += 64 * kHeld) {
    Parts q;
    load_parts(a, row, c0, q);
    scale_parts(q, m, h, table);
    chunk = first_above(q.part, c0, target, base, before, last);
  }
  if (chunk < 0) {
    chunk = last;
    before = (double)neg_inf();  // (its last token)
  }
  return token_in<E>(a, row_of<E>(a, row), chunk, m, h, 0.0, target, before, table);
}

// Is the child's token accepted? (sw: S times the row's whole)
template <typename E>
__device__ __forceinline__ bool accepted(const VerifyArgs& a, const Row<E>& row, int child_row, int x, float m, const Heat& h,
                                         double cw, double sw, const double* table) {
  const float l = value(row.l[x]);
  const double q = (double)fmaxf(row.q[x], 0.0f);
  const double p = m == __builtin_inff() ? (l == m ? 1.0 : 0.0) : weight(l, (double)m, h.s, table);
  return uniform((double)a.u_accept[child_row] * q * sw < fmax(p - cw * q, 0.0));
}

// Child of row `cur` after row `from` of a sequence's n rows, by a wave: the first (with the token
// `want`, unless it is negative), or -1.
__device__ __forceinline__ int next_child(const VerifyArgs& a, int lo, int n, int cur, int from, int want) {
  if (!a.parents) {
    const int i = cur + 1;
    return i > from && i < n && (want < 0 || uniform(a.tokens[lo + i] == want)) ? i : -1;
  }
  for (int i0 = from + 1; i0 < n; i0 += 64) {
    const int i = i0 + own_lane();
    bool is = i < n && a.parents[lo + i] == cur;
    if (is && want >= 0) is = a.tokens[lo + i] == want;
    const uint64_t m = __builtin_amdgcn_ballot_w64(is);
    if (m) return i0 + __builtin_ctzll(m);
  }
  return -1;
}
// And the first with a token of the vocabulary (x).
__device__ __forceinline__ int next_asked(const VerifyArgs& a, int lo, int n, int cur, int from, int& x) {
  do {
    from = next_child(a, lo, n, cur, from, -1);
    x = from >= 0 ? uniform(a.tokens[lo + from]) : 0;
  } while (from >= 0 && (uint32_t)x >= (uint32_t)a.vocab);
  return from;
}

// What a row tells the walk: its token (or -1: it has no distribution), or with probabilities its first
// child, if that is accepted (below kRejected), if it is not (from kRejected on), or its token
// if it has no child (from kToken on).
constexpr int kRejected = 1 << 24, kToken = 1 << 25;

// The walk of a sequence, by a wave: rows 0 .. 63 are in its lanes.
template <bool kProbs>
__device__ __forceinline__ void walk(const VerifyArgs& a, int b, int lo, int n, bool drawn) {
  const int lane = threadIdx.x & 63;
  auto out_of = [&](int i) __attribute__((always_inline)) {
    return __hip_atomic_load(a.out + lo + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  int out = -1, parent = -1, tok = -1;
  if (lane < n) {
    out = out_of(lane);
    parent = a.parents ? a.parents[lo + lane] : lane - 1;
    if (!drawn) tok = a.tokens[lo + lane];
  }
  int cur = 0, kept = 0, token = -1, mine = -1;
  bool rejected = false;
  while (kept < n) {
    if (kept < 64)
      mine = lane == kept ? cur : mine;
    else if (lane == 0)
      a.kept[lo + kept] = cur;
    ++kept;
    const int f = uniform(cur < 64 ? __builtin_amdgcn_readlane(out, cur & 63) : out_of(cur));
    int child = -1;
    if (!drawn) {
      token = f;
      if (token >= 0) {
        const uint64_t m = __builtin_amdgcn_ballot_w64(lane > cur && lane < n && parent == cur && tok == token);
        child = m ? (int)__builtin_ctzll(m) : (n > 64 ? next_child(a, lo, n, cur, max(cur, 63), token) : -1);
      }
    } else if (f >= kToken) {
      token = f - kToken;
    } else if (f >= kRejected) {
      rejected = true;
    } else {
      child = f;  // (-1: no distribution)
    }
    if (child <= cur || child >= n) break;
    cur = child;
  }
  if (lane < min(kept, n)) a.kept[lo + lane] = mine;
  for (int i = kept + lane; i < n; i += 64) a.kept[lo + i] = -1;
  if (lane == 0) {
    if (kProbs) a.at[b] = rejected ? cur : -1;
    a.n_kept[b] = kept;
    a.next[b] = token;
  }
}

template <typename E, bool kProbs>
__global__ __launch_bounds__(64) void verify_rows_kernel(VerifyArgs args) {
  __shared__ double table[kSteps];
  __shared__ VerifyArgs held;  // (in LDS: twenty pointers leave no scalar registers)
  if (kProbs && threadIdx.x == 0) held = args;
  // waves of the rows, then one of each sequence
  const int row = (int)blockIdx.x < args.rows ? (int)blockIdx.x : -1;
  Parts p;
  load_parts(args, max(row, 0), 0, p);
  const Held sequences = hold_sequences(args);
  load_table(table);  // (the loads before it come at the same time)
  Heat h = {};
  const int b = row < 0 ? (int)blockIdx.x - args.rows : row < end_of(args, sequences) ? sequence_of(args, sequences, row, h) : -1;
  const VerifyArgs& a = kProbs ? held : args;
  if (b < 0) return;
  const int lo = uniform(clampi(a.offs[b], 0, a.rows)), n = uniform(clampi(a.offs[b + 1], lo, a.rows) - lo);
  if (row < 0) h = heat_of(a, b);
  const bool drawn = kProbs && !h.greedy;
  const int lane = threadIdx.x;
  if (row >= 0) {
    float m;
    double whole;
    row_whole(a, row, h, m, whole, p, table);
    int out = -1;
    bool need = m != neg_inf();
    if (drawn && need) {
      int x;
      const int child = next_asked(a, lo, n, row - lo, row - lo, x);
      if (child >= 0) {
        need = false;  // (a token is needed only where no child is left)
        const bool yes = accepted<E>(a, row_of<E>(a, row), lo + child, x, m, h, 0.0, whole, table);
        out = yes ? child : kRejected + child;
        if (lane == 0) {
          a.most[row] = m;
          a.whole[row] = whole;
        }
      }
    }
    if (need) out = pick<E>(a, row, m, h, whole, p, table) + (drawn ? kToken : 0);
    if (lane == 0) __hip_atomic_store(a.out + row, out, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  // The stores reach the device's memory before the wave arrives (nobody waits for it), and the last of
  // the sequence's n + 1 waves reads them there.
  asm volatile("" ::: "memory");
  wait_vmcnt<0>();
  uint32_t before = 0;  // (of a call without rows, without a workspace: none)
  if (lane == 0 && args.rows > 0) before = __hip_atomic_fetch_add(a.arrived + (int64_t)b * kApart, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (uniform((int)before) != n) return;
  walk<kProbs>(a, b, lo, n, drawn);
}

// A row of a sequence's walk with a rejection, -1 if there is none.
__device__ __forceinline__ int row_at(const VerifyArgs& a, int b, int n) {
  const int cur = uniform(a.at[b]);
  return cur < n ? cur : -1;
}

// A chunk's sum, for and by workgroups on any XCD.
__device__ __forceinline__ void put_rest(double* p, double x) {
  __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ double get_rest(const double* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Workgroup (b, g): chunks 4 g .. +3 of the row of sequence b where a first child is rejected; the
// last of the sequence's goes on from there.
template <typename E>
__global__ __launch_bounds__(256) void verify_rest_kernel(VerifyArgs args) {
  __shared__ double table[kSteps];
  __shared__ VerifyArgs a;  // (as above)
  __shared__ int last_s;
  const int groups = (args.chunks + 3) / 4;
  const int b = (int)(blockIdx.x / (uint32_t)groups);
  if (uniform(args.at[b]) < 0) return;
  if (threadIdx.x == 0) a = args;
  load_table(table);
  const int wave = uniform((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
  const int lo = uniform(clampi(a.offs[b], 0, a.rows)), n = uniform(clampi(a.offs[b + 1], lo, a.rows) - lo);
  int cur = row_at(a, b, n);
  if (cur < 0) return;
  Heat h = heat_of(a, b);
  h.greedy = false;
  double* const rest = a.rest + (int64_t)b * a.chunks;
  // the row cur, whose first child is rejected, and the child to ask next with its token (loaded before
  // the sums, which take as long)
  Row<E> r;
  float m, u;
  double cw;
  int child, x;
  auto enter = [&]() __attribute__((always_inline)) {
    const int row = lo + cur;
    r = row_of<E>(a, row);
    m = uniform(a.most[row]);
    cw = a.whole[row];
    u = a.u_sample[row];
    child = next_asked(a, lo, n, cur, clampi(uniform(a.out[row]) - kRejected, cur, n), x);
  };
  enter();
  int kept = uniform(clampi(a.n_kept[b], 0, n)), token = -1;
  {
    const int c = ((int)blockIdx.x - b * groups) * 4 + wave;
    if (c < a.chunks) {
      const double sum = rest_sum(r, c * kChunk, a.vocab, m, h, cw, table);
      if (lane == 0) put_rest(rest + c, sum);
    }
    asm volatile("" ::: "memory");
    wait_vmcnt<0>();
    __syncthreads();
    if (threadIdx.x == 0)
      last_s = __hip_atomic_fetch_add(a.arrived + (int64_t)b * kApart + 1, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
               (uint32_t)groups - 1;
    __syncthreads();
    if (!uniform(last_s != 0)) return;
  }
  bool have_rest = true;
  for (;;) {
    double sw;
    bool yes = false, last = false;
    for (;;) {
      if (!have_rest) {
        __syncthreads();  // every wave has read the sums before
        for (int c = wave; c < a.chunks; c += 4) {
          double w[kPer], sum = 0.0;
          rest_weights<false>(r, c * kChunk, a.vocab, m, h, cw, w, table);
#pragma unroll
          for (int i = 0; i < kPer; ++i) sum += w[i];
          sum = counted(of_lane(wave_scan(sum), 63));
          if (lane == 0) put_rest(rest + c, sum);
        }
        wait_vmcnt<0>();
        __syncthreads();
      }
      have_rest = false;
      sw = 0.0;
      for (int c0 = 0; c0 < a.chunks; c0 += 64) sw += of_lane(wave_scan(c0 + lane < a.chunks ? get_rest(rest + c0 + lane) : 0.0), 63);
      if (child >= 0 && !last) {
        yes = accepted<E>(a, r, lo + child, x, m, h, cw, sw, table);
        if (yes) break;
        cw += sw;
        child = next_asked(a, lo, n, cur, child, x);
        continue;
      }
      // no child is left: a token of what is left of the row
      if (uniform(sw > 0.0)) {
        const double target = (double)u * sw;
        double base = 0.0, before = 0.0;
        int some = 0, chunk = -1;
        for (int c0 = 0; c0 < a.chunks && chunk < 0; c0 += 64) {
          const double part[1] = {c0 + lane < a.chunks ? get_rest(rest + c0 + lane) : 0.0};
          chunk = first_above(part, c0, target, base, before, some);
        }
        if (chunk < 0) {
          chunk = some;
          before = (double)neg_inf();
        }
        token = token_in<E>(a, r, chunk, m, h, cw, target, before, table);
      }
      if (token >= 0 || last) break;
      cw = 0.0;  // p = q: nothing is left of it (but roundings), p itself counts
      last = true;
    }
    int f = -1;
    if (yes) {  // and on to the next row with a rejection
      f = child;
      while (f > cur && f < n) {  // (as all are but where the offsets are out of order)
        cur = f;
        if (threadIdx.x == 0 && kept < n) a.kept[lo + kept] = cur;
        ++kept;
        f = uniform(a.out[lo + cur]);
      }
    }
    if (f >= kRejected && f < kToken) {
      enter();
      continue;
    }
    if (f >= kToken) token = f - kToken;  // a row without a child
    break;
  }
  if (threadIdx.x == 0) {
    a.n_kept[b] = min(kept, n);
    a.next[b] = token;
  }
}

size_t aligned(size_t x) { return (x + 255) / 256 * 256; }

int chunks_of(int vocab) { return (vocab + kChunk - 1) / kChunk; }

int check_sizes(const ce_drafts* d, int32_t vocab) {
  const int s = check_drafts(d);
  if (s != CE_OK) return s;
  if (vocab < 1) return CE_ERR_INVALID_ARG;
  if (vocab >= 1 << 24 || (int64_t)d->row_capacity * vocab >= (int64_t)1 << 40 ||
      (int64_t)d->B * ((chunks_of(vocab) + 3) / 4) >= (int64_t)1 << 24)  // (workgroups of 256 in one launch)
    return CE_ERR_UNSUPPORTED;
  return CE_OK;
}

template <typename E>
hipError_t launch(const VerifyArgs& a, hipStream_t stream) {
  auto blocks = [](int64_t waves) { return dim3((unsigned)((waves + 3) / 4)); };
  const int64_t pairs = (int64_t)a.rows * ((a.chunks + 1) / 2);
  // Twice the waves that the chip holds at once (four a SIMD): 521 rows of 131072, 272 of 100003 in float32, the whole call,
  // with 4, 6, 8, 16 a SIMD 45.4, 45.0, 43.9, 44.7 and 46.3, 46.9, 45.7, 45.8 us.
  const int64_t most = 4 * 256 * 8;
  hipError_t e = hipSuccess;
  if (a.rows > 0) {
    hipLaunchKernelGGL(verify_stats_kernel<E>, blocks(pairs < most ? pairs : most), dim3(256), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const dim3 waves(a.rows + a.B);
  if (!a.probs) {
    hipLaunchKernelGGL((verify_rows_kernel<E, false>), waves, dim3(64), 0, stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((verify_rows_kernel<E, true>), waves, dim3(64), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(verify_rest_kernel<E>, dim3((unsigned)((int64_t)a.B * ((a.chunks + 3) / 4))), dim3(256), 0, stream, a);
  return hipGetLastError();
}

// Places of a workspace.
struct Places {
  size_t top, out, arrived, most, whole, rest, at, bytes;
};
Places places_of(const ce_drafts* d, int32_t vocab, bool probs) {
  const size_t rows = d->row_capacity, chunks = chunks_of(vocab), with = probs ? 1 : 0;
  Places p;
  p.top = aligned(rows * chunks * sizeof(double));
  p.out = p.top + aligned(rows * chunks * sizeof(float));
  p.arrived = p.out + aligned(rows * sizeof(int32_t));
  p.most = p.arrived + aligned((size_t)d->B * kApart * sizeof(uint32_t));
  p.whole = p.most + aligned(with * rows * sizeof(float));
  p.rest = p.whole + aligned(with * rows * sizeof(double));
  p.at = p.rest + aligned(with * d->B * chunks * sizeof(double));
  p.bytes = p.at + aligned(with * d->B * sizeof(int32_t));
  return p;
}

}  // namespace

}  // namespace ce

using namespace ce;

extern "C" {

size_t ce_verify_workspace_size(const ce_drafts* drafts, int32_t vocab, int with_probs) {
  if (check_sizes(drafts, vocab) != CE_OK || drafts->row_capacity == 0) return 0;
  return places_of(drafts, vocab, with_probs != 0).bytes;
}

int ce_verify_drafts(const ce_drafts* drafts, int32_t vocab, const void* logits, int64_t logits_ld, int dtype,
                     const float* temperature, const float* draft_probs, int64_t probs_ld, const float* u_accept,
                     const float* u_sample, int32_t* kept_rows, int32_t* n_kept, int32_t* next_token, void* ws,
                     size_t ws_bytes, void* stream) {
  const int s = check_sizes(drafts, vocab);
  if (s != CE_OK) return s;
  if (dtype != CE_BF16 && dtype != CE_F32) return CE_ERR_UNSUPPORTED;
  if (logits_ld < vocab || (draft_probs && probs_ld < vocab) || !draft_probs != !u_accept) return CE_ERR_INVALID_ARG;
  if (logits_ld >= (int64_t)1 << 32 || (draft_probs && probs_ld >= (int64_t)1 << 32)) return CE_ERR_UNSUPPORTED;
  const int rows = drafts->row_capacity;
  if (!drafts->offsets || !n_kept || !next_token) return CE_ERR_INVALID_ARG;
  if (rows > 0 && (!drafts->tokens || !logits || !u_sample || !kept_rows)) return CE_ERR_INVALID_ARG;
  const Places p = places_of(drafts, vocab, draft_probs != nullptr);
  if (rows > 0) {
    const int e = check_ws(ws, ws_bytes, p.bytes);
    if (e != CE_OK) return e;
  }
  VerifyArgs a = {};
  a.B = drafts->B;
  a.rows = rows;
  a.vocab = vocab;
  a.chunks = chunks_of(vocab);
  a.offs = drafts->offsets;
  a.parents = drafts->parents;
  a.tokens = drafts->tokens;
  a.logits = static_cast<const char*>(logits);
  a.ld = logits_ld * (dtype == CE_BF16 ? 2 : 4);
  a.temps = temperature;
  a.probs = rows > 0 ? draft_probs : nullptr;
  a.probs_ld = probs_ld;
  a.u_accept = u_accept;
  a.u_sample = u_sample;
  a.kept = kept_rows;
  a.n_kept = n_kept;
  a.next = next_token;
  char* const w = static_cast<char*>(ws);
  a.sum = reinterpret_cast<double*>(w);
  a.top = reinterpret_cast<float*>(w + p.top);
  a.out = reinterpret_cast<int32_t*>(w + p.out);
  a.arrived = reinterpret_cast<uint32_t*>(w + p.arrived);
  a.most = reinterpret_cast<float*>(w + p.most);
  a.whole = reinterpret_cast<double*>(w + p.whole);
  a.rest = reinterpret_cast<double*>(w + p.rest);
  a.at = reinterpret_cast<int32_t*>(w + p.at);
  const hipError_t e = dtype == CE_BF16 ? launch<uint16_t>(a, static_cast<hipStream_t>(stream))
                                        : launch<float>(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? CE_OK : CE_ERR_HIP;
}

}  // extern "C"
