"""The tokens by which the chunks of paged attention meet, built for the host: no two calls of
a process have the same."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_tokens_of_many_calls_differ(tmp_path):
    src = tmp_path / "token.cpp"
    src.write_text(r'''
#include <stdio.h>
#include <algorithm>
#include <vector>
#include "ce_paged_token.hpp"
using namespace ce;
// x from its token, step by step: shown here to be one to one
static uint64_t inverse(uint64_t odd) {  // modulo 2^48, Newton
  uint64_t y = odd;
  for (int i = 0; i < 6; ++i) y *= 2 - odd * y;
  return y & kTokenMask;
}
static uint64_t call_of(uint64_t x) {
  x ^= x >> 25;  // 25 + 25 bits are more than 48: one step undoes it
  x = (x * inverse(0xd6e8feb86659ull)) & kTokenMask;
  x ^= x >> 24;  // (24 + 24 = 48)
  return (x * inverse(0x9e3779b97f4bull)) & kTokenMask;
}
int main() {
  const uint64_t n = 1 << 25;
  std::vector<uint64_t> t(n);
  for (uint64_t i = 0; i < n; ++i) t[i] = paged_token(i + 1);
  for (uint64_t i = 0; i < n; ++i)
    if (t[i] == 0 || t[i] > kTokenMask || call_of(t[i]) != i + 1) return printf("call %llu\n", (unsigned long long)i + 1), 1;
  for (uint64_t k = 1; k < 48; ++k)
    for (uint64_t d = 0; d < 3; ++d) {
      const uint64_t c = (1ull << k) + d - (k > 1);
      if (call_of(paged_token(c)) != c) return printf("call 2^%llu + %llu\n", (unsigned long long)k, (unsigned long long)d), 1;
    }
  std::sort(t.begin(), t.end());
  if (std::adjacent_find(t.begin(), t.end()) != t.end()) return printf("the same twice\n"), 1;
  printf("OK\n");
  return 0;
}
''')
    exe = tmp_path / "token"
    r = subprocess.run(["g++", "-std=c++17", "-O2", f"-I{os.path.join(ROOT, 'paper_2608_29291_amd', 'csrc')}", str(src), "-o",
                        str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "OK\n", r.stdout + r.stderr
