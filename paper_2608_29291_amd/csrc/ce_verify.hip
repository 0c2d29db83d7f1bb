// Verification of drafted tokens against the target's probabilities (include/ce_router_draft.h).
//
// Sampling. A token is the first whose running sum of weights w_i = exp((l_i - max) / T) is above u
// times their whole. A row of 1e5 tokens has borders 1e-5 and less apart, so exponentials and
// sums in 32 bits (1e-7, with the same sign for a large weight before many small ones) would
// move one token in a hundred. Weights are formed in 64 bits: 2^(k / 32) from a table of 32 in
// LDS, each in banks of its own, and a polynomial of degree 5 for the rest, |r| <= 1 / 64 octave
// (error 2e-15); fp64 instructions issue as fast as fp32 ones here.
//
// Passes. Every row is cut into chunks of kChunk tokens.
//   1. verify_stats_kernel: maximum and sum of each chunk, the one pass over the logits.
//   2. verify_rows_kernel: the chunks' sums give the row's whole and the chunk of its token, and
//      that chunk's weights, formed again, the token; with probabilities of the drafts, whether the
//      row's first child is accepted. Each row by a workgroup of its own, also rows that the
//      walk will not reach, since rows in parallel cost less than a walk row by row.
//   3. verify_rest_kernel, with probabilities only: chunk sums of what a first rejection leaves of
//      the row where it happens.
//   4. verify_walk_kernel: follows the tree; a second rejection at a row is a pass over that row.
// What rejections leave is max(p - c q, 0) with a growing c (max(max(p - a q, 0) - b q, 0) =
// max(p - (a + b) q, 0), as q >= 0), so nothing of a row is kept between them.
#include <hip/hip_runtime.h>

#include "ce_device.hpp"
#include "ce_draft.hpp"
#include "ce_host.hpp"

namespace ce {

namespace {

constexpr int kPer = 16;               // tokens of a thread
constexpr int kThreads = 256;
constexpr int kChunk = kThreads * kPer;  // tokens of a chunk
constexpr double kLeast = -40960.0;    // exponents of 2^(1/32) below it are zeros

__device__ const double kTable[32] = {  // 2^(k / 32)
    0x1.0000000000000p+0, 0x1.059b0d3158574p+0, 0x1.0b5586cf9890fp+0, 0x1.11301d0125b51p+0,
    0x1.172b83c7d517bp+0, 0x1.1d4873168b9aap+0, 0x1.2387a6e756238p+0, 0x1.29e9df51fdee1p+0,
    0x1.306fe0a31b715p+0, 0x1.371a7373aa9cbp+0, 0x1.3dea64c123422p+0, 0x1.44e086061892dp+0,
    0x1.4bfdad5362a27p+0, 0x1.5342b569d4f82p+0, 0x1.5ab07dd485429p+0, 0x1.6247eb03a5585p+0,
    0x1.6a09e667f3bcdp+0, 0x1.71f75e8ec5f74p+0, 0x1.7a11473eb0187p+0, 0x1.82589994cce13p+0,
    0x1.8ace5422aa0dbp+0, 0x1.93737b0cdc5e5p+0, 0x1.9c49182a3f090p+0, 0x1.a5503b23e255dp+0,
    0x1.ae89f995ad3adp+0, 0x1.b7f76f2fb5e47p+0, 0x1.c199bdd85529cp+0, 0x1.cb720dcef9069p+0,
    0x1.d5818dcfba487p+0, 0x1.dfc97337b9b5fp+0, 0x1.ea4afa2a490dap+0, 0x1.f50765b6e4540p+0,
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
  float* top;      // [rows x chunks]
  double* sum;     // [rows x chunks], under the chunk's own maximum
  int32_t* picked; // [rows]: the token of a row
  // with probabilities:
  int32_t* first;  // [rows]: the first child, accepted (>= 0) or not (-2 - it), or none (-1)
  double* whole;   // [rows]: maximum and whole of a row
  float* most;
  double* rest;    // [B x chunks]: chunk sums after the first rejection
};

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }
// What every lane has alike, in scalar registers: branches on it need no masks of lanes.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ bool uniform(bool x) { return __builtin_amdgcn_readfirstlane((int)x) != 0; }
__device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

// The thread's number, of which a loop's comparisons are not formed before it: they would fill the
// scalar registers.
__device__ __forceinline__ int own_thread() {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  return tid;
}

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

// How the logits of a row become exponents: 32 log2 e / T, or whether only the largest counts.
struct Heat {
  double s;
  bool greedy;
};
__device__ __forceinline__ Heat heat_of(const VerifyArgs& a, int b) {
  const float t = a.temps ? a.temps[b] : 1.0f;
  Heat h;
  h.greedy = !(t > 0.0f);
  h.s = 46.166241308446828384 / (h.greedy ? 1.0 : (double)t);  // 32 log2 e
  return h;
}

// The table, and the polynomial's coefficients ln(2)^i / 32^i / i!. A kernel that is short of scalar
// registers keeps these in vector registers (kVector).
struct Exp {
  const double* table;
  double c5, c4, c3, c2, c1;
};
template <bool kVector = false>
__device__ __forceinline__ Exp exp_of(const double* table) {
  Exp e = {table, 0x1.5d87fe78a6731p-35, 0x1.3b2ab6fba4e77p-27, 0x1.c6b08d704a0c0p-20, 0x1.ebfbdff82c58fp-13, 0x1.62e42fefa39efp-6};
  if constexpr (kVector) asm volatile("" : "+v"(e.c5), "+v"(e.c4), "+v"(e.c3), "+v"(e.c2), "+v"(e.c1));
  return e;
}

// exp((x - m) / T); x of NaN or -infinity: 0.
__device__ __forceinline__ double weight(float x, double m, double s, const Exp& e) {
  const double t = fmax(((double)x - m) * s, kLeast);
  const double k = rint(t);
  const double r = t - k;
  const int n = (int)k;
  double p = fma(r, e.c5, e.c4);
  p = fma(r, p, e.c3);
  p = fma(r, p, e.c2);
  p = fma(r, p, e.c1);
  p = fma(r, p, 1.0);
  return ldexp(e.table[n & 31] * p, n >> 5);
}

// Where only the largest counts, by the temperature or because it is infinite, the others
// become -infinity and it 0.
__device__ __forceinline__ void flatten(float (&x)[kPer], float& m, const Heat& h) {
  if (!h.greedy && m != __builtin_inff()) return;
#pragma unroll
  for (int i = 0; i < kPer; ++i) x[i] = x[i] == m ? 0.0f : neg_inf();
  m = 0.0f;
}

// The sequence of a row, or -1. Every wave by itself.
__device__ __forceinline__ int sequence_of(const VerifyArgs& a, int row) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  for (int step = a.B > 4096 ? 4096 : (a.B > 64 ? 64 : 1); step > 0; step >>= 6) {
    const int i = lo + lane * step;
    const bool le = i < a.B && a.offs[i < a.B ? i : 0] <= row;
    const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(le));
    lo += (n > 0 ? n - 1 : 0) * step;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  return a.offs[lo] <= row && row < a.offs[lo + 1] ? lo : -1;
}

// Token (j, e) of a thread of a chunk from token c0 on is c0 + (j kThreads + thread) kVec + e: 16 bytes
// of logits at a time.
template <typename E>
constexpr int kVec = 16 / sizeof(E);

__device__ __forceinline__ float logit(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ float logit(float x) { return x; }

template <typename E>
__device__ __forceinline__ void load_logits(const E* row, int c0, int vocab, float (&x)[kPer]) {
  const int tid = own_thread();
#pragma unroll
  for (int j = 0; j < kPer / kVec<E>; ++j) {
    const int i = c0 + (j * kThreads + tid) * kVec<E>;
    if (i + kVec<E> <= vocab) {
      E v[kVec<E>];
      __builtin_memcpy(v, row + i, 16);  // (rows may begin anywhere)
#pragma unroll
      for (int e = 0; e < kVec<E>; ++e) x[j * kVec<E> + e] = logit(v[e]);
    } else {
#pragma unroll
      for (int e = 0; e < kVec<E>; ++e) {
        const float y = logit(row[min(i + e, vocab - 1)]);
        x[j * kVec<E> + e] = i + e < vocab ? y : neg_inf();
      }
    }
  }
}

struct Scratch {
  double table[32];
  double waves[kThreads / 64];
  float tops[kThreads / 64];
  int first[kThreads / 64];
};

__device__ __forceinline__ void load_table(Scratch& s) {
  if (threadIdx.x < 32) s.table[threadIdx.x] = kTable[threadIdx.x];
}

__device__ __forceinline__ float block_max(float v, Scratch& s) {
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  __syncthreads();
  const int tid = own_thread();
  if ((tid & 63) == 0) s.tops[tid >> 6] = v;
  __syncthreads();
  v = s.tops[0];
  for (int i = 1; i < kThreads / 64; ++i) v = fmaxf(v, s.tops[i]);
  return uniform(v);
}

// Inclusive prefix sum over the block, and the whole.
__device__ __forceinline__ double block_scan(double v, double& whole, Scratch& s) {
  const int tid = own_thread(), lane = tid & 63, wave = tid >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_up(v, o);
    if (lane >= o) v += y;
  }
  __syncthreads();
  if (lane == 63) s.waves[wave] = v;
  __syncthreads();
  double before = 0.0;
  whole = 0.0;
  for (int i = 0; i < kThreads / 64; ++i) {
    if (i == wave) before = whole;
    whole += s.waves[i];
  }
  return before + v;
}

// The first thread of the block for which `is` holds, or -1.
__device__ __forceinline__ int block_first(bool is, Scratch& s) {
  const uint64_t m = __builtin_amdgcn_ballot_w64(is);
  __syncthreads();
  const int tid = own_thread();
  if ((tid & 63) == 0) s.first[tid >> 6] = m ? tid + __builtin_ctzll(m) : 1 << 30;
  __syncthreads();
  int f = s.first[0];
  for (int i = 1; i < kThreads / 64; ++i) f = min(f, s.first[i]);
  return uniform(f == 1 << 30 ? -1 : f);
}

// The largest x of the block.
__device__ __forceinline__ int block_most(int x, Scratch& s) {
  for (int o = 32; o > 0; o >>= 1) x = max(x, __shfl_xor(x, o));
  __syncthreads();
  const int tid = own_thread();
  if ((tid & 63) == 0) s.first[tid >> 6] = x;
  __syncthreads();
  for (int i = 0; i < kThreads / 64; ++i) x = max(x, s.first[i]);
  return uniform(x);
}

// Maximum and sum of a chunk of a row.
template <typename E>
__global__ __launch_bounds__(256) void verify_stats_kernel(VerifyArgs a) {
  __shared__ Scratch scr;
  const int row = (int)(blockIdx.x / (uint32_t)a.chunks), c = (int)(blockIdx.x - (uint32_t)row * a.chunks);
  const int b = sequence_of(a, row);
  if (b < 0) return;
  load_table(scr);
  const Exp ex = exp_of(scr.table);
  const Heat h = heat_of(a, b);
  float x[kPer];
  load_logits<E>(reinterpret_cast<const E*>(a.logits + (int64_t)row * a.ld), c * kChunk, a.vocab, x);
  float m = neg_inf();
#pragma unroll
  for (int i = 0; i < kPer; ++i) m = fmaxf(m, x[i]);  // (NaN is passed over)
  m = block_max(m, scr);
  double sum = 0.0, whole = 0.0;
  if (m != neg_inf()) {
    float under = m;
    flatten(x, under, h);
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum += weight(x[i], (double)under, h.s, ex);
    block_scan(sum, whole, scr);
  }
  if (threadIdx.x == 0) {
    a.top[blockIdx.x] = m;
    a.sum[blockIdx.x] = whole;
  }
}

// A chunk's sum under the row's maximum.
__device__ __forceinline__ double chunk_part(const VerifyArgs& a, int64_t at, float m, const Heat& h, const Exp& ex) {
  const float mc = a.top[at];
  if (h.greedy || m == __builtin_inff()) return mc == m ? a.sum[at] : 0.0;
  return a.sum[at] * weight(mc, (double)m, h.s, ex);
}

// Maximum and whole of a row's weights from its chunks.
__device__ __forceinline__ void row_whole(const VerifyArgs& a, int row, const Heat& h, float& m, double& whole,
                                          const Exp& ex, Scratch& scr) {
  const int64_t at = (int64_t)row * a.chunks;
  m = neg_inf();
  for (int c = threadIdx.x; c < a.chunks; c += kThreads) m = fmaxf(m, a.top[at + c]);
  m = block_max(m, scr);
  whole = 0.0;
  if (m == neg_inf()) return;
  for (int c0 = 0; c0 < a.chunks; c0 += kThreads) {
    const int c = c0 + threadIdx.x;
    double tile;
    block_scan(c < a.chunks ? chunk_part(a, at + c, m, h, ex) : 0.0, tile, scr);
    whole += tile;
  }
}

// The first of a thread's weights w (in the order of tokens: block, thread, place) whose running sum
// from `base` on is above `target`, or -1; base grows by their whole, last becomes the last token of
// a positive weight.
template <typename E>
__device__ __forceinline__ int first_above(const double (&w)[kPer], int c0, double target, double& base, int& last,
                                           Scratch& scr) {
  int found = -1;
#pragma unroll
  for (int j = 0; j < kPer / kVec<E>; ++j) {
    const int i0 = c0 + (j * kThreads + (int)threadIdx.x) * kVec<E>;
    double mine = 0.0;
    int some = -1;
#pragma unroll
    for (int e = 0; e < kVec<E>; ++e) {
      mine += w[j * kVec<E> + e];
      if (w[j * kVec<E> + e] > 0.0) some = i0 + e;
    }
    double whole;
    const double to = block_scan(mine, whole, scr);
    const int thread = found < 0 ? block_first(base + to > target, scr) : -1;
    if (thread >= 0) {
      int token = -1;
      if ((int)threadIdx.x == thread) {
        double run = base + (to - mine);
#pragma unroll
        for (int e = 0; e < kVec<E>; ++e) {
          run += w[j * kVec<E> + e];
          token = token < 0 && run > target && w[j * kVec<E> + e] > 0.0 ? i0 + e : token;
        }
        if (token < 0) token = some;  // (the sums' last bit)
      }
      found = block_most(token, scr);
    }
    last = max(last, block_most(some, scr));
    base += whole;
  }
  return found;
}

template <typename E>
__device__ __forceinline__ void load_weights(const E* row, int c0, int vocab, float m, const Heat& h, double (&w)[kPer],
                                             const Exp& ex) {
  float x[kPer];
  load_logits<E>(row, c0, vocab, x);
  flatten(x, m, h);
#pragma unroll
  for (int i = 0; i < kPer; ++i) w[i] = weight(x[i], (double)m, h.s, ex);
}

// q of the tokens of load_logits<E>.
template <typename E>
__device__ __forceinline__ void load_probs(const float* row, int c0, int vocab, float (&q)[kPer]) {
  const int tid = own_thread();
#pragma unroll
  for (int j = 0; j < kPer / kVec<E>; ++j) {
    const int i = c0 + (j * kThreads + tid) * kVec<E>;
    if (i + kVec<E> <= vocab) {
#pragma unroll
      for (int e = 0; e < kVec<E>; e += 4) __builtin_memcpy(&q[j * kVec<E> + e], row + i + e, 16);
    } else {
#pragma unroll
      for (int e = 0; e < kVec<E>; ++e) {
        const float y = row[min(i + e, vocab - 1)];
        q[j * kVec<E> + e] = i + e < vocab ? y : 0.0f;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) q[i] = fmaxf(q[i], 0.0f);  // (NaN: 0)
}

// Child of row `cur` after row `from` of a sequence's n rows, by one wave: the first (with the token
// `want`, unless it is negative), or -1.
__device__ __forceinline__ int next_child(const VerifyArgs& a, int lo, int n, int cur, int from, int want) {
  const int lane = threadIdx.x & 63;
  if (!a.parents) {
    const int i = cur + 1;
    return i > from && i < n && (want < 0 || a.tokens[lo + i] == want) ? i : -1;
  }
  for (int i0 = from + 1; i0 < n; i0 += 64) {
    const int i = i0 + lane;
    bool is = i < n && a.parents[lo + i] == cur;
    if (is && want >= 0) is = a.tokens[lo + i] == want;
    const uint64_t m = __builtin_amdgcn_ballot_w64(is);
    if (m) return i0 + __builtin_ctzll(m);
  }
  return -1;
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

// Weights of a chunk of a row after rejections (cw: c times the row's whole).
template <typename E>
__device__ __forceinline__ void rest_weights(const Row<E>& row, int c0, int vocab, float m, const Heat& h, double cw,
                                             double (&w)[kPer], const Exp& ex) {
  load_weights<E>(row.l, c0, vocab, m, h, w, ex);
  if (uniform(cw == 0.0)) return;
  float q[kPer];
  load_probs<E>(row.q, c0, vocab, q);
#pragma unroll
  for (int i = 0; i < kPer; ++i) w[i] = fmax(w[i] - cw * (double)q[i], 0.0);
}

// The chunk where the running sum of parts (part(c), of the chunks in order) is above target, the sum
// before it, and the last chunk with a part if there is none.
template <typename F>
__device__ __forceinline__ int find_chunk(int chunks, double target, double& before, Scratch& scr, const F& part) {
  int last = 0;
  double base = 0.0;
  before = 0.0;
  for (int c0 = 0; c0 < chunks; c0 += kThreads) {
    const int c = c0 + threadIdx.x;
    const double x = c < chunks ? part(c) : 0.0;
    double tile;
    const double to = block_scan(x, tile, scr);
    const int t = block_first(x > 0.0 && base + to > target, scr);
    if (t >= 0) {
      __syncthreads();
      if ((int)threadIdx.x == t) scr.waves[0] = base + (to - x);
      __syncthreads();
      before = scr.waves[0];
      return c0 + t;
    }
    last = max(last, block_most(x > 0.0 ? c : -1, scr));
    base += tile;
  }
  return last;
}

// A row's token, from the parts of its chunks.
template <typename E, typename F>
__device__ __forceinline__ int pick(const VerifyArgs& a, const Row<E>& row, float m, const Heat& h, double cw, double target, const Exp& ex, Scratch& scr,
                                    const F& part) {
  double before;
  const int c0 = find_chunk(a.chunks, target, before, scr, part) * kChunk;
  double w[kPer];
  rest_weights<E>(row, c0, a.vocab, m, h, cw, w, ex);
  int some = -1;
  const int token = first_above<E>(w, c0, target, before, some, scr);
  return token < 0 ? some : token;
}

// Is the child's token accepted? (sw: S times the row's whole)
template <typename E>
__device__ __forceinline__ bool accepted(const VerifyArgs& a, const Row<E>& row, int child_row, int x, float m, const Heat& h, double cw,
                                         double sw, const Exp& ex) {
  const float l = logit(row.l[x]);
  const double q = (double)fmaxf(row.q[x], 0.0f);
  const double p = m == __builtin_inff() ? (l == m ? 1.0 : 0.0) : weight(l, (double)m, h.s, ex);
  return uniform((double)a.u_accept[child_row] * q * sw < fmax(p - cw * q, 0.0));
}

template <typename E>
__global__ __launch_bounds__(256) void verify_rows_kernel(VerifyArgs a) {
  __shared__ Scratch scr;
  const int row = blockIdx.x;
  const int b = sequence_of(a, row);
  if (b < 0) return;
  const Heat h = heat_of(a, b);
  load_table(scr);
  const Exp ex = exp_of(scr.table);
  float m;
  double whole;
  row_whole(a, row, h, m, whole, ex, scr);
  const bool drawn = a.probs && !h.greedy;
  int child = -1, x = 0;
  if (drawn) {  // the first child with a token of the vocabulary
    const int lo = clampi(a.offs[b], 0, a.rows), n = clampi(a.offs[b + 1], lo, a.rows) - lo;
    child = row - lo;
    do {
      child = next_child(a, lo, n, row - lo, child, -1);
      if (child >= 0) x = uniform(a.tokens[lo + child]);
    } while (child >= 0 && (uint32_t)x >= (uint32_t)a.vocab);
    if (child >= 0 && m != neg_inf()) {
      const bool yes = accepted<E>(a, row_of<E>(a, row), lo + child, x, m, h, 0.0, whole, ex);
      if (threadIdx.x == 0) {
        a.first[row] = yes ? child : -2 - child;
        a.whole[row] = whole;
        a.most[row] = m;
      }
      return;  // (a token is needed only where no child is left)
    }
  }
  int token = -1;
  if (m != neg_inf()) {
    const int64_t at = (int64_t)row * a.chunks;
    token = pick<E>(a, row_of<E>(a, row), m, h, 0.0, h.greedy ? 0.0 : (double)a.u_sample[row] * whole, ex, scr,
                    [&](int c) { return chunk_part(a, at + c, m, h, ex); });
  }
  if (threadIdx.x == 0) {
    a.picked[row] = token;
    if (drawn) a.first[row] = -1;
  }
}

// Row cur's first child as verify_rows_kernel left it. (Rows that lie in no sequence, or in two, where
// the offsets are out of order, may have any; only rows behind cur are children.)
__device__ __forceinline__ int first_child(const VerifyArgs& a, int lo, int n, int cur) {
  const int f = __builtin_amdgcn_readfirstlane(a.first[lo + cur]);
  const int child = f >= 0 ? f : -2 - f;
  return child > cur && child < n ? f : -1;
}

template <typename E>
__global__ __launch_bounds__(256) void verify_rest_kernel(VerifyArgs a) {
  __shared__ Scratch scr;
  const int b = (int)(blockIdx.x / (uint32_t)a.chunks), c = (int)(blockIdx.x - (uint32_t)b * a.chunks);
  const int lo = clampi(a.offs[b], 0, a.rows), n = clampi(a.offs[b + 1], lo, a.rows) - lo;
  const Heat h = heat_of(a, b);
  if (n == 0 || h.greedy) return;
  int cur = 0, f;
  while ((f = first_child(a, lo, n, cur)) >= 0) cur = f;
  if (f == -1) return;
  load_table(scr);
  const Exp ex = exp_of(scr.table);
  __syncthreads();
  const int row = lo + cur;
  double whole, w[kPer], sum = 0.0;
  rest_weights<E>(row_of<E>(a, row), c * kChunk, a.vocab, a.most[row], h, a.whole[row], w, ex);
#pragma unroll
  for (int i = 0; i < kPer; ++i) sum += w[i];
  block_scan(sum, whole, scr);
  if (threadIdx.x == 0) a.rest[blockIdx.x] = whole;
}

template <typename E, bool kProbs>
__global__ __launch_bounds__(256) void verify_walk_kernel(VerifyArgs args) {
  __shared__ Scratch scr;
  __shared__ VerifyArgs held;  // (the arguments in LDS: twenty pointers leave no scalar registers)
  if constexpr (kProbs) {
    if (threadIdx.x == 0) held = args;
    __syncthreads();
  }
  const VerifyArgs& a = kProbs ? held : args;
  const int b = blockIdx.x;
  const int lo = clampi(a.offs[b], 0, a.rows), n = clampi(a.offs[b + 1], lo, a.rows) - lo;
  const Heat h = heat_of(a, b);
  const bool drawn = kProbs && !h.greedy;
  const Exp ex = exp_of<true>(scr.table);
  int cur = 0, kept = 0, token = -1;
  bool have_rest = true;  // of the first row with a rejection
  if (drawn) {
    load_table(scr);
    __syncthreads();
  }
  while (kept < n) {
    if (threadIdx.x == 0) a.kept[lo + kept] = cur;
    ++kept;
    int child;
    if (!drawn) {
      token = uniform(a.picked[lo + cur]);
      child = token < 0 ? -1 : next_child(a, lo, n, cur, cur, token);
      if (child < 0) break;
      cur = child;
      continue;
    }
    const int f = first_child(a, lo, n, cur);
    if (f == -1) {
      token = a.picked[lo + cur];
      break;
    }
    if (f >= 0) {
      cur = f;
      continue;
    }
    // its first child is rejected
    double* const rest = a.rest + (int64_t)b * a.chunks;
    const int row = lo + cur;
    const Row<E> r = row_of<E>(a, row);
    const float m = uniform(a.most[row]);
    const Heat warm = {h.s, false};
    double cw = a.whole[row], sw;
    bool yes = false, last = false;
    child = -2 - f;
    for (;;) {
      if (!have_rest) {
        for (int c = 0; c < a.chunks; ++c) {
          double w[kPer], sum = 0.0, part;
          rest_weights<E>(r, c * kChunk, a.vocab, m, warm, cw, w, ex);
#pragma unroll
          for (int i = 0; i < kPer; ++i) sum += w[i];
          block_scan(sum, part, scr);
          if (threadIdx.x == 0) rest[c] = part;
        }
        __syncthreads();
      }
      have_rest = false;
      sw = 0.0;
      for (int c0 = 0; c0 < a.chunks; c0 += kThreads) {
        double part;
        block_scan(c0 + (int)threadIdx.x < a.chunks ? rest[c0 + threadIdx.x] : 0.0, part, scr);
        sw += part;
      }
      if (last) break;
      int x = 0;
      do {
        child = next_child(a, lo, n, cur, child, -1);
        if (child >= 0) x = uniform(a.tokens[lo + child]);
      } while (child >= 0 && (uint32_t)x >= (uint32_t)a.vocab);
      if (child >= 0) {
        yes = accepted<E>(a, r, lo + child, x, m, warm, cw, sw, ex);
        if (yes) break;
        cw += sw;
      } else {
        if (uniform(sw > 0.0)) break;
        cw = 0.0;  // p = q: nothing is left of it, p itself counts
        last = true;
      }
    }
    if (yes) {
      cur = child;
      continue;
    }
    token = pick<E>(a, r, m, warm, cw, (double)a.u_sample[row] * sw, ex, scr, [&](int c) { return rest[c]; });
    break;
  }
  for (int i = kept + threadIdx.x; i < n; i += kThreads) a.kept[lo + i] = -1;
  if (threadIdx.x == 0) {
    a.n_kept[b] = kept;
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
      (int64_t)d->B * chunks_of(vocab) >= (int64_t)1 << 28)
    return CE_ERR_UNSUPPORTED;
  return CE_OK;
}

template <typename E>
hipError_t launch(const VerifyArgs& a, hipStream_t stream) {
  if (a.rows > 0) {
    hipLaunchKernelGGL(verify_stats_kernel<E>, dim3((unsigned)((int64_t)a.rows * a.chunks)), dim3(256), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(verify_rows_kernel<E>, dim3(a.rows), dim3(kThreads), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.probs) {
      hipLaunchKernelGGL(verify_rest_kernel<E>, dim3((unsigned)((int64_t)a.B * a.chunks)), dim3(kThreads), 0, stream, a);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  if (a.probs)
    hipLaunchKernelGGL((verify_walk_kernel<E, true>), dim3(a.B), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((verify_walk_kernel<E, false>), dim3(a.B), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

// Places of a workspace.
struct Places {
  size_t top, picked, first, whole, most, rest, bytes;
};
Places places_of(const ce_drafts* d, int32_t vocab, bool probs) {
  const size_t rows = d->row_capacity, chunks = chunks_of(vocab);
  Places p;
  p.top = aligned(rows * chunks * sizeof(double));
  p.picked = p.top + aligned(rows * chunks * sizeof(float));
  p.first = p.picked + aligned(rows * sizeof(int32_t));
  p.whole = p.first + (probs ? aligned(rows * sizeof(int32_t)) : 0);
  p.most = p.whole + (probs ? aligned(rows * sizeof(double)) : 0);
  p.rest = p.most + (probs ? aligned(rows * sizeof(float)) : 0);
  p.bytes = p.rest + (probs ? aligned(d->B * chunks * sizeof(double)) : 0);
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
  if (rows > 0) {
    const int e = check_ws(ws, ws_bytes, places_of(drafts, vocab, draft_probs != nullptr).bytes);
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
  a.probs = draft_probs;
  a.probs_ld = probs_ld;
  a.u_accept = u_accept;
  a.u_sample = u_sample;
  a.kept = kept_rows;
  a.n_kept = n_kept;
  a.next = next_token;
  const Places p = places_of(drafts, vocab, draft_probs != nullptr);
  char* const w = static_cast<char*>(ws);
  a.sum = reinterpret_cast<double*>(w);
  a.top = reinterpret_cast<float*>(w + p.top);
  a.picked = reinterpret_cast<int32_t*>(w + p.picked);
  a.first = reinterpret_cast<int32_t*>(w + p.first);
  a.whole = reinterpret_cast<double*>(w + p.whole);
  a.most = reinterpret_cast<float*>(w + p.most);
  a.rest = reinterpret_cast<double*>(w + p.rest);
  const hipError_t e = dtype == CE_BF16 ? launch<uint16_t>(a, static_cast<hipStream_t>(stream))
                                        : launch<float>(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? CE_OK : CE_ERR_HIP;
}

}  // extern "C"
