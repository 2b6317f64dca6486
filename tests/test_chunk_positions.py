"""Positions at the ends of int32 in the plan of a chunk's attention: no sum of them may overflow (checked by the
compiler's own sanitizer, on the CPU)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SRC = r"""
#include "chunk_items.h"
#include <climits>
#include <cstdio>
using namespace fpk;
int main() {
  for (int p : {INT_MAX, INT_MAX - 3, 1 << 30, 5001, 5000, 4999, -1, -700, INT_MIN})
    for (int G : {1, 8, 128})
      for (int n : {1, 5, 700}) {
        const int tt = ck_tile_tokens(G), T = 2 * tt, max_len = 5000;
        CkSeq s;
        const bool fine = p >= 0 && (long long)p + n <= max_len;
        if (s.set(0, n, p, tt, 700, max_len) != fine || s.bad == fine) return printf("%d %d: bounds\n", p, n), 1;
        for (int u = 0; u < s.units; ++u)
          for (int t = 0; t < T && u * T + t < s.n; ++t) {  // keys that row u T + t sees
            const int lim = std::min(s.end, s.pos + u * T + t + 1);
            const long long want = std::min<long long>(max_len, (long long)p + u * T + t + 1);
            if ((lim > 0 ? lim : 0) != (want > 0 ? want : 0)) return printf("%d %d %d: %d\n", p, n, u * T + t, lim), 1;
            if (lim > s.tiles(u, T) * kCkKeys) return printf("%d %d: tiles\n", p, n), 1;
          }
        if (s.cost(T) <= 0 || s.unit_at(s.cost(T) - 1, T) != s.units - 1) return printf("%d %d: line\n", p, n), 1;
      }
  puts("ok");
}
"""


def test_positions_at_the_ends_of_int32(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "pos.cpp", tmp_path / "pos"
    src.write_text(SRC)
    subprocess.run([cxx, "-O1", "-std=c++17", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error", "-I",
                    os.path.join(ROOT, "paper_2501_13111_gb300", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.stdout.strip() == "ok", r.stdout + r.stderr
