// The token of a call of paged attention (no HIP: tests build it for the host).
#pragma once

#include <stdint.h>

namespace ce {

constexpr uint64_t kTokenMask = (1ull << 48) - 1;  // a counter of arrivals holds 16 bits below it

// Token of call number `call` (from 1): no other of 2^48 - 1 calls has it, and memory is
// unlikely to hold it by chance. Each step maps the numbers of 48 bits one to one: an odd
// factor modulo 2^48, and a xor with the number's own upper part, shifted down.
constexpr uint64_t paged_token(uint64_t call) {
  uint64_t x = (call * 0x9e3779b97f4bull) & kTokenMask;
  x ^= x >> 24;
  x = (x * 0xd6e8feb86659ull) & kTokenMask;
  return x ^ (x >> 25);
}

}  // namespace ce
