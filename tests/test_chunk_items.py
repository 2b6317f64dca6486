"""The line of units that the attention of a chunk cuts into equal stretches (chunk_items.h): closed forms against
plain sums, and every key tile of every unit taken exactly once whatever the lengths, groups and CTAs."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SRC = r"""
#include "chunk_items.h"
#include <cstdio>
#include <cstdlib>
#include <vector>
using namespace fpk;
static int bad(const char* what, int it) { printf("%s at %d\n", what, it); return 1; }
int main() {
  srand(1);
  for (int it = 0; it < 20000; ++it) {
    const int G = 1 + rand() % 128, tt = ck_tile_tokens(G), T = 2 * tt;
    if (tt < 1 || tt * G > 128 || (tt < 128 && 2 * tt * G <= 128)) return bad("tile tokens", it);
    const int n = rand() % (rand() % 4 == 0 ? 3000 : 200), top = rand() % 10 == 0 ? rand() % 4000 + 1 : 10000;
    const int pos = rand() % 30 == 0 ? -(rand() % 100) : rand() % 3 == 0 ? rand() % 10 : rand() % 5000;
    const int most = rand() % 20 == 0 ? rand() % 100 + 1 : 5000;
    CkSeq s;
    const bool fine = s.set(0, n, pos, tt, most, top);
    if (fine != (n <= most && (n == 0 || (pos >= 0 && pos + n <= top)))) return bad("bounds", it);
    int x = 0;
    for (int u = 0; u < s.units; ++u) {
      const int nt = s.tiles(u, T);
      if (s.before(u, T) != x) return bad("before", it);
      int e = std::min(pos + (u + 1) * T, pos + s.n);
      if (s.bad) e = std::max(0, std::min(pos + s.n, top));
      if (nt != (e + 127) / 128) return bad("tiles", it);
      const int places = kCkStart + (s.n - u * T > tt ? 2 : 1) * nt;
      if (s.places(u, T) != places) return bad("places", it);
      if (s.unit_at(x, T) != u || s.unit_at(x + places - 1, T) != u) return bad("unit_at", it);
      x += places;
    }
    if (s.cost(T) != x) return bad("cost", it);
  }
  for (int it = 0; it < 3000; ++it) {  // the stretches
    const int G = 1 + rand() % 16, tt = ck_tile_tokens(G), T = 2 * tt, B = 1 + rand() % 12, Hkv = 1 + rand() % 5;
    const int grid = 1 + rand() % 152;
    struct Unit { int x; int nt, w; std::vector<int> seen; int own = -1, parts = 0; int all() const { return kCkStart + w * nt; } };
    std::vector<Unit> units;
    int W = 0;
    for (int b = 0; b < B; ++b) {
      CkSeq s;
      s.set(0, rand() % 3 ? rand() % 9 : rand() % 700, rand() % 2 ? rand() % 50 : rand() % 4000, tt, 1000, 5000);
      for (int h = 0; h < Hkv; ++h)
        for (int u = 0; u < s.units; ++u) {
          units.push_back({W, s.tiles(u, T), s.weight(u, T), std::vector<int>(s.tiles(u, T))});
          W += units.back().all();
        }
    }
    const int g = ck_ctas(W, grid);
    if (g < 1 || g > grid) return bad("ctas", it);
    auto begin = [&](int c) -> int {
      if (c >= g) return W;
      const int x = ck_begin(c, W, g);
      if (x != (long long)W * c / g) return -1;
      for (auto& u : units)
        if (x >= u.x && x < u.x + u.all()) return u.x + ck_snap(x - u.x, u.nt, u.w);
      return W;
    };
    for (int c = 0; c < grid; ++c) {
      const int lo = begin(c), hi = begin(c + 1);
      if (hi < lo) return bad("order", it);
      for (auto& u : units) {
        const int p = std::max(lo, u.x), q = std::min(hi, u.x + u.all());
        if (p >= q) continue;
        if (p > u.x && (p - u.x - kCkStart) % u.w) return bad("a border inside a key tile", it);
        const int t0 = std::max(0, p - u.x - kCkStart) / u.w, t1 = std::max(0, q - u.x - kCkStart) / u.w;
        if (p > u.x && t0 < kCkSnap) return bad("a border inside a unit's start", it);
        if (t1 <= t0) return bad("a part without keys", it);
        for (int t = t0; t < t1; ++t) ++u.seen[t];
        if (u.own < 0) u.own = c;
        if (c != u.own + u.parts++) return bad("the parts of a unit are not neighbours", it);
      }
    }
    for (auto& u : units) {
      int own, parts;
      ck_parts(u.x, u.nt, u.w, W, g, &own, &parts);
      if (u.nt > 0 && u.parts > 1 && (own != u.own || parts != u.parts)) return bad("ck_parts", it);
    }
    for (auto& u : units)
      for (int k : u.seen)
        if (k != 1) return bad("a key tile is not taken once", it);
  }
  puts("ok");
}
"""


def test_units_and_stretches(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "items.cpp", tmp_path / "items"
    src.write_text(SRC)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2501_13111_gb300", "csrc"), str(src), "-o",
                    str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.stdout.strip() == "ok", r.stdout
