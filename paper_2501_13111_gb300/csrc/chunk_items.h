// How the attention of a chunk is cut up (attn_chunk.cuh).  Host and device.
//
// The G query heads of a KV head read the same keys, so their rows are packed:
// row r of a query tile is token r / G, head r % G; a tile holds the largest power of
// two of tokens with at most 128 rows, a unit up to two tiles of one (sequence, KV
// head).  (Groups that are no power of two leave rows idle, up to 63 of 128: 40 heads
// on 8 take 112 us where 32 on 8 take 61, the same chunks.)  The units, sequence by
// sequence, KV head by KV head, lie on a line, each with kCkStart places, what
// starting it costs, and for each of its key tiles as many as it has query tiles, one
// or two.  CTA c of g takes an equal stretch of that line, so every SM has as much to
// do whatever the lengths are; a unit that a border cuts leaves a partial result with
// every CTA, and the last of them to finish adds them (attn_chunk.cuh).
#pragma once

#include <algorithm>
#include <cstdint>

#ifdef __CUDACC__
#define FP_CK __host__ __device__ __forceinline__
#else
#define FP_CK inline
#endif

namespace fpk {

constexpr int kCkKeys = 128;  // keys a tile, and rows a query tile
constexpr int kCkStart = 3;
constexpr int kCkSnap = 2;      // key tiles at a unit's ends that a border does not cut off
constexpr int kCkLeast = 4;     // places a CTA takes at least (a power of two)

// Tokens of a query tile.
FP_CK int ck_tile_tokens(int G) {
  int t = 128;
  while (t * G > 128) t >>= 1;
  return t;
}

// One sequence's chunk, after its lengths have been looked over.
struct CkSeq {
  int row0, n;  // first row, rows
  int pos;      // position of the first row
  int end;      // cached positions that it reads (its last row's, at most max_len)
  int units;
  bool bad;     // lengths beyond the bounds: every unit is given all key tiles

  // first and count as in cu, position p; false: a bound is broken
  FP_CK bool set(int first, int count, int p, int tile_tokens, int max_new, int max_len) {
    row0 = first;
    n = count < max_new ? count : max_new;
    pos = p < max_len ? p : max_len;  // (behind the bound every row sees the same keys)
    const long long e = (long long)p + n;
    end = (int)(e < 0 ? 0 : e > max_len ? max_len : e);
    bad = n > 0 && (p < 0 || e > max_len);
    units = (n + 2 * tile_tokens - 1) / (2 * tile_tokens);
    return !bad && count <= max_new;
  }
  FP_CK int all_tiles() const { return (end + kCkKeys - 1) / kCkKeys; }
  // key tiles of unit u (T: tokens a unit, a power of two)
  FP_CK int tiles(int u, int T) const {
    return bad || u == units - 1 ? all_tiles() : (pos + (u + 1) * T + kCkKeys - 1) / kCkKeys;
  }
  // key tiles of units 0 .. u-1, u < units
  FP_CK int tiles_before(int u, int T) const {
    if (bad) return u * all_tiles();
    const int a0 = (pos + kCkKeys - 1) / kCkKeys;
    if (T > kCkKeys) return u * a0 + u * (u + 1);  // 256
    // ceil((pos + i T) / 128): the first unit ends in tile a0 or the next, and every
    // 128 / T = 2^lg units move on by one tile
    int lg = 0;
    while ((T << lg) < kCkKeys) ++lg;
    const int k = (a0 * kCkKeys - pos) >> (7 - lg);  // units that end within tile a0's keys
    if (u <= k) return u * a0;
    const int v = u - k, q = v >> lg, rem = v & ((1 << lg) - 1);
    return u * a0 + (((q * (q + 1)) >> 1) << lg) + rem * (q + 1);
  }
  // places a key tile of unit u takes
  FP_CK int weight(int u, int T) const { return n - u * T > T / 2 ? 2 : 1; }
  FP_CK int before(int u, int T) const { return u * kCkStart + 2 * tiles_before(u, T); }  // (all but the last: two tiles)
  FP_CK int places(int u, int T) const { return kCkStart + weight(u, T) * tiles(u, T); }
  // places of one KV head's units (ck_fits: below 2^31)
  FP_CK int cost(int T) const { return units == 0 ? 0 : before(units - 1, T) + places(units - 1, T); }
  // the unit that holds place x < cost
  FP_CK int unit_at(int x, int T) const {
    int lo = 0, hi = units;  // before(lo) <= x
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (before(mid, T) <= x) lo = mid;
      else hi = mid;
    }
    return lo;
  }
};

// Whether the line of any batch within these bounds is shorter than 2^31 places.
inline bool ck_fits(int n_tokens, int B, int max_len, int Hkv, int tile_tokens) {
  const long long units = n_tokens / (2 * tile_tokens) + (long long)B;
  return units * Hkv < (1LL << 31) && units * Hkv * (kCkStart + 2 * ((max_len + kCkKeys - 1LL) / kCkKeys)) < (1LL << 31);
}

// A border at place `off` of a unit of nt key tiles of `weight` places, moved back to the
// beginning of a key tile and off the unit's ends: the place to cut at, 0 (before the
// unit) or all its places (behind it).
FP_CK int ck_snap(int off, int nt, int weight) {
  const int t = off < kCkStart ? 0 : (off - kCkStart) / weight;
  return t < kCkSnap ? 0 : t > nt - kCkSnap ? kCkStart + weight * nt : kCkStart + weight * t;
}

// Where the stretch of CTA c of g begins, before its border is moved: floor(W c / g).
FP_CK int ck_begin(int c, int W, int g) {
  const unsigned q = (unsigned)W / (unsigned)g, r = (unsigned)W - q * g;
  return (int)(q * c + r * c / (unsigned)g);
}

// The first of g CTAs with ck_begin(c) >= t (1 <= t).
FP_CK int ck_first_from(int t, int W, int g) {
  return (int)(((unsigned long long)t * g + (unsigned)W - 1) / (unsigned)W);
}

// The CTAs that share the unit of nt key tiles at place x: *own begins it, *parts in all.
FP_CK void ck_parts(int x, int nt, int weight, int W, int g, int* own, int* parts) {
  *own = ck_first_from(x + kCkStart + weight * kCkSnap, W, g) - 1;
  *parts = ck_first_from(x + kCkStart + weight * (nt - kCkSnap + 1), W, g) - *own;
}

// CTAs that take part of W places.
FP_CK int ck_ctas(int W, int grid) {
  const int most = W / kCkLeast > 1 ? W / kCkLeast : 1;
  return most < grid ? most : grid;
}

}  // namespace fpk
