"""The arithmetic of the attention's spans and steps (csrc/attn_span.hpp), compiled into a plain C++ program that walks over
every step that a workgroup of the kernel for single tokens would take: no look-up outside a sequence's row of the table,
whatever the lengths, and no token left out that some row sees; windows of any size."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdint>
#include <cstdio>
#include <initializer_list>
#include <set>
#include "attn_span.hpp"
using namespace mpq;
int main() {
  int bad = 0;
  // lengths that a device array may name: nothing, within the table, beyond it by little and by much
  for (int64_t room : {16, 32, 128, 1024})
    for (int64_t kv_len : {(int64_t)0, (int64_t)1, (int64_t)15, (int64_t)130, (int64_t)999, (int64_t)1000, (int64_t)1024, (int64_t)1093,
                           (int64_t)5000, (int64_t)0x7FFFFFFF})
      for (int64_t window : {0, 1, 10, 33, 64, 256, 5000})
        for (int causal : {0, 1}) {
          if (window && !causal) continue;
          for (int64_t n : {1, 5, 40, 300})
            for (int group : {1, 3}) {
              const int64_t len = kv_len < room ? kv_len : room;
              for (int64_t tile = 0; tile * 16 < n * group; ++tile) {
                const int64_t first = tile * 16 / group, end = tile * 16 + 15 < n * group ? tile * 16 + 15 : n * group - 1;
                const Span span = {seen(kv_len - n + first, len, causal, window).lo, seen(kv_len - n + end / group, len, causal, window).hi};
                for (int tokens : {32, 64})
                  for (int splits : {1, 3, 256}) {
                    std::set<int64_t> taken;
                    for (int split = 0; split < splits; ++split) {
                      const Steps s = steps_of(span, tokens, splits, split);
                      for (int64_t t = s.t0; t < s.t1; ++t) {
                        if (t - s.t0 > room) { bad = 1; break; }
                        for (int64_t tok = t * tokens; tok < (t + 1) * tokens; tok += 16)
                          if (tok < span.hi && (tok < 0 || tok >= room)) {
                            std::printf("token %lld of a table of %lld: length %lld window %lld rows %lld\n", (long long)tok,
                                        (long long)room, (long long)kv_len, (long long)window, (long long)n);
                            bad = 1;
                          }
                        if (!taken.insert(t).second) { std::printf("step %lld twice\n", (long long)t); bad = 1; }
                      }
                    }
                    for (int64_t row = first; row <= end / group; ++row) {
                      const Span own = seen(kv_len - n + row, len, causal, window);
                      for (int64_t tok = own.lo; tok < own.hi; ++tok)
                        if (!taken.count(tok / tokens)) { std::printf("token %lld left out\n", (long long)tok); bad = 1; break; }
                    }
                    if (bad) return 1;
                  }
              }
            }
        }
  // windows up to the type's end mean what the widest that reaches any token means, also for rows in front of the first token
  for (int64_t window : {(int64_t)1 << 31, ((int64_t)1 << 32) - 1, (int64_t)1 << 32, INT64_MAX - 100, INT64_MAX})
    for (int64_t p : {-((int64_t)1 << 31), (int64_t)-1000, (int64_t)-70, (int64_t)-3, (int64_t)-1, (int64_t)0, (int64_t)5, ((int64_t)1 << 31) - 2}) {
      const Span s = seen(p, 1000, true, cut_window(window));
      const int64_t hi = p + 1 < 1000 ? p + 1 : 1000;
      if (s.lo != 0 || s.hi != hi) { std::printf("window %lld at %lld: %lld .. %lld\n", (long long)window, (long long)p, (long long)s.lo, (long long)s.hi); bad = 1; }
    }
  for (int64_t window : {0, 1, 75, 0x7FFFFFFF})
    if (cut_window(window) != window) bad = 1;
  if (bad) return 1;
  std::puts("spans ok");
  return 0;
}
"""


def test_spans_and_steps(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "spans.cpp", tmp_path / "spans"
    src.write_text(PROGRAM)
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-I",
                    os.path.join(ROOT, "paper_2302_01382_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and "spans ok" in r.stdout, r.stdout + r.stderr
