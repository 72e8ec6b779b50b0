"""The rows that a write or a read of the 8-bit cache takes, and the blocks that a write gives to its workgroups (dam_span.h): the
header, plain C++, runs here on the CPU under sanitizers, over small sizes against a count of the rows and at the ends of the 32 bits,
where a block that a call does not have starts beyond them, against 64-bit arithmetic."""
import os
import subprocess

from paper_2506_11104_amd import build as hip_build

PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include "dam_span.h"
using namespace dam;
static int fail(const char *what, int64_t a, int64_t b, int64_t c, int64_t d) {
  return std::printf("%s: %lld %lld %lld %lld\n", what, (long long)a, (long long)b, (long long)c, (long long)d), 1;
}
int main() {
  for (int cap = 1; cap <= 40; ++cap)  // every span of a small cache
    for (int start = -2; start <= cap + 2; ++start)
      for (int n = 1; n <= 45; ++n)
        for (int count : {-3, 0, 1, 2, n - 1, n, n + 7}) {
          const Span s = span_of(start, count, n, cap);
          int rows = 0;
          for (int r = 0; r < std::min(std::max(count, 0), n); ++r) rows += start >= 0 && start + r < cap;
          if (start >= cap) rows = 0;
          if (s.count != rows || (rows && s.start != start)) return fail("span", cap, start, n, count);
          for (int block : {16, 32}) {
            int found = 0;
            for (int nth = 0; nth < most_blocks(n, cap, block); ++nth) {
              const int b = nth_block(s, block, nth);
              int held = 0;
              for (int r = 0; r < s.count; ++r) held += b >= 0 && (s.start + r) / block == b;
              if (b >= 0 && !held) return fail("a block without a row", cap, start, n, count);
              found += held;
            }
            if (found != s.count) return fail("rows in no block", cap, start, n, count);
          }
        }
  const int most = INT32_MAX - 1024;
  for (int cap : {most, most - 1, (1 << 30) + 70, 1 << 30})
    for (int back : {1, 2, 5, 127, 128, 1000, 1 << 20, cap - 1, cap})
      for (int n : {1, 130, (1 << 30) - 1, 1 << 30, most})
        for (int count : {1, n / 2, n, INT32_MAX})
          for (int block : {16, 32, 64, 128}) {
            const Span s = span_of(cap - back, count, n, cap);
            if (s.count != std::min<int64_t>(std::min(count, n), back)) return fail("count", cap, back, n, count);
            const int64_t many = most_blocks(n, cap, block), last = s.count ? (s.start + (int64_t)s.count - 1) / block : -1;
            for (int64_t nth : {(int64_t)0, (int64_t)1, last - s.start / block, last - s.start / block + 1, many / 2, many - 1}) {
              if (nth < 0 || nth >= many) continue;
              const int64_t b = s.start / block + nth;
              if (nth_block(s, block, (int)nth) != (s.count && b <= last ? b : -1)) return fail("block", cap, s.start, n, nth);
            }
            if (s.count && last - s.start / block >= many) return fail("blocks of a call", cap, back, n, block);
          }
  return std::puts("all"), 0;
}
"""


def test_spans_and_their_blocks(tmp_path):
    src, exe = tmp_path / "span.cpp", tmp_path / "span"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I" + hip_build.CSRC, str(src),
                    "-o", str(exe)], check=True, timeout=120)
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=0")
    r = subprocess.run([str(exe)], env=env, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "all", r.stdout + r.stderr[-2000:]
