// Beam search over the LM head's logits: the best continuations of each group of beams,
// page tables that follow the chosen beams, and the copies of part-filled pages.
#include <algorithm>

#include "chunk.cuh"
#include "kernels.cuh"
#include "pair.cuh"

namespace fpk {

// ------------------------------------------------------------------ selection
// The W best of score_w + x_wt - lse(x_w) over the W beams and V tokens of a group, ties to
// the lowest (w, t).  A beam's order is its logits' order, so one pass finds both its
// normaliser and its W candidates: a CTA takes a piece of a row, holds it in registers and
// leaves the piece's sum of exponentials and its W largest logits, in order; the last CTA
// of the group to finish merges each beam's pieces, then the beams.
// Two candidates of different beams must fall as 64 bits would have them, so scores are
// pairs of fp32.  The normaliser: with an integer reference k (the maximum's log2,
// rounded up), sum_i 2^(x_i log2 e - k) in fp32, one rounding an exponent; sets with
// other references are scaled exactly; lse = (k + exponent of s) ln 2 + log(significand of s).
// Every warp has the reference of its own values, so that a set of banned tokens (any finite
// value, down to the least) must not disturb the others: where the maximum m is beyond 2^30, k
// would be too coarse, or infinite.  There fp32's neighbours are 128 apart, so that only the
// values equal to m count: s is their number, and m itself the reference.
// Sorting is by counting: a value's place is the number of larger ones, found by comparisons
// that wait for nothing.  (One maximum after the other took 12 us where this takes 10.)  A
// piece's candidates are the few values that reach the W-th largest of 32 groups' maxima; of
// sorted lists, ordered by their heads, entry e of the r-th counts only if r + e < W.
// Measured: 32 groups of 4 beams, 32000 tokens 10.5 us (1.6 TB/s), 1 of 8, 128001 tokens
// 10.2 (10.3 and 10.1 with one form of reference, wrong beside such bans).  Bound by latency:
// loads 2.5 us, exponentials 0.7, candidates 1.5, the group's ticket 1.2, lists 1.5, beams 1.
constexpr int kBsThreads = 512, kBsWarps = kBsThreads / 32, kBsItems = 8;
constexpr int kBsPiece = kBsThreads * kBsItems * 4;  // values held at once
constexpr int kBsSplits = 32;                        // pieces of a row, at most
constexpr size_t kBsHead = FP_BEAM_MAX_GROUPS * 4;   // tickets, whatever the call's B

// A logit and its token as one number: larger logits first, then lower tokens.  0: none
// (-inf too: a banned token).
FP_DEV uint32_t bs_ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
FP_DEV float bs_value(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
FP_DEV unsigned long long bs_key(float x, int t) {
  return x > -INFINITY ? (unsigned long long)bs_ordered(x + 0.f) << 32 | (uint32_t)~t : 0ull;
}
FP_DEV unsigned long long bs_warp_max(unsigned long long k) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32));
  const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
  return (unsigned long long)hi << 32 | lo;
}
FP_DEV float bs_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2^d, d <= 0; an integer from -126 on
FP_DEV float bs_pow2(float d) { return d < -126.f ? 0.f : __uint_as_float((uint32_t)(127 + (int)d) << 23); }

// A set's reference r and its sum against it (-inf: nothing in it).  r is k / 2, or m where that is
// beyond kBsFar: half of k = m log2 e stays below, so one order serves both, and of two sets that
// are not both near the lower one's factor is 2^-126 or less: 0.
constexpr float kBsFar = 0x1p30f;
struct BsSum {
  float r, s;
};
FP_DEV BsSum bs_add(BsSum a, BsSum b) {
  const float r = fmaxf(a.r, b.r);
  if (r == -INFINITY) return {r, a.s + b.s};
  return {r, a.s * bs_pow2(2.f * (a.r - r)) + b.s * bs_pow2(2.f * (b.r - r))};
}

struct BsArgs {
  const float* x;
  int V, B, W, S, per;  // pieces a row, values a piece (a multiple of 4)
  const float* score;
  const int32_t* done;
  int end;
  int32_t *parent, *token;
  float* new_score;
  int32_t* new_done;
  int32_t* tickets;           // [B]
  float2* sums;               // [B W S]
  unsigned long long* best;   // [B W S][W]
  int32_t* err;
};

constexpr int kBsCands = 512;   // candidates of a piece that are sorted out at once
constexpr int kBsLists = 128;   // entries of a row's lists: pieces times W, at most

// W sorted lists, ordered by their heads: entry e of the list with the r-th largest head has
// r + e larger ones, so the W largest of all are among the W (W + 1) / 2 with r + e < W.
// The first of list r's among those:
constexpr int kBsTriangle = FP_BEAM_MAX * (FP_BEAM_MAX + 1) / 2;
FP_DEV int bs_first(int r, int W) { return r * W - r * (r - 1) / 2; }

template <int ITEMS>
__global__ void __launch_bounds__(kBsThreads, 2) beam_select_kernel(const BsArgs a) {
  __shared__ unsigned long long s_best[2][kBsWarps], s_list[2][FP_BEAM_MAX];
  __shared__ BsSum s_sum[kBsWarps];
  __shared__ int s_last, s_n;
  __shared__ uint32_t s_bar;
  __shared__ __align__(16) uint32_t s_top[32];
  __shared__ int s_done[FP_BEAM_MAX];
  __shared__ union {
    unsigned long long cand[kBsCands];
    struct {
      unsigned long long list[kBsLists], some[kBsLists];
    } row[kBsWarps];
    struct {
      unsigned long long score[FP_BEAM_MAX][FP_BEAM_MAX], some[kBsTriangle];
      int place[kBsTriangle];
    } beam;
  } s_u;
  __shared__ Pair s_off[FP_BEAM_MAX];                             // score - lse of a beam
  __shared__ float s_ref[FP_BEAM_MAX];                            // (both against this)
  __shared__ unsigned long long s_row[FP_BEAM_MAX][FP_BEAM_MAX];  // its candidates
  constexpr int PIECE = kBsThreads * ITEMS * 4;
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, W = a.W, S = a.S;
  const int row = blockIdx.x / S, piece = blockIdx.x - row * S, b = row / W;
  const float* x = a.x + (long long)row * a.V;
  const long long lo = (long long)piece * a.per;
  const int end = (int)min((long long)a.V, lo + a.per);
  const bool vec = ((uintptr_t)(x + lo) & 15) == 0;
  const float score = __ldg(a.score + row);
  const bool ended = a.done && __ldg(a.done + row) != 0;
  if (!ended && score > -INFINITY) {
    BsSum sum = {-INFINITY, 0.f};
    int list = 0;  // which of the two holds the best so far
    if (threadIdx.x < FP_BEAM_MAX) s_list[0][threadIdx.x] = 0;
    for (long long c0 = lo; c0 < end; c0 += PIECE) {
      // this thread's values: four tokens from c0 + 4 (i kBsThreads + thread) on
      float v[ITEMS][4];
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const long long t = c0 + 4 * (i * kBsThreads + (int)threadIdx.x);
        if (vec && t + 3 < end) {
          const float4 f = __ldg(reinterpret_cast<const float4*>(x + t));
          v[i][0] = f.x, v[i][1] = f.y, v[i][2] = f.z, v[i][3] = f.w;
        } else {
#pragma unroll
          for (int y = 0; y < 4; ++y) v[i][y] = t + y < end ? __ldg(x + t + y) : -INFINITY;
        }
      }
      float mt = -INFINITY;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) mt = fmaxf(mt, fmaxf(fmaxf(v[i][0], v[i][1]), fmaxf(v[i][2], v[i][3])));
      // the maxima of 32 groups of threads: the W-th largest of them is no larger than the
      // W-th largest value, and little smaller
      float m = mt;
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      if ((lane & 15) == 0) s_top[threadIdx.x >> 4] = m > -INFINITY ? bs_ordered(m + 0.f) : 0u;
      if (threadIdx.x == 0) s_n = 0;
      __syncthreads();
      if (warp == 0) {  // (by one warp: all of them took the issue slots of the exponentials)
        const uint32_t mine = s_top[lane];
        int rank = 0;
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          const uint4 q = *reinterpret_cast<const uint4*>(s_top + i);
          const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
          for (int y = 0; y < 4; ++y) rank += u[y] > mine || (u[y] == mine && i + y < lane);
        }
        if (rank == W - 1) s_bar = max(mine, 1u);  // (0: nothing)
      }
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
      {
        // x log2 e in two parts (1.4426950408889634).  Far away the exponent is x/2 + (x/2 - m): 0
        // for m, -64 or less for others (a factor of 0 would turn -inf into a NaN)
        constexpr float kHi = 1.44269502162933349609375f, kLo = 1.92596299e-8f;
        const bool far = !(m > -kBsFar && m <= kBsFar);
        const float hi = far ? 0.5f : kHi, lo = far ? 0.5f : kLo;
        const float k = m == -INFINITY ? 0.f : far ? m : ceilf(m * kHi);
        const float2 hi2 = make_float2(hi, hi), lo2 = make_float2(lo, lo), k2 = make_float2(-k, -k);
        float2 s[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
          for (int y = 0; y < 4; y += 2) {
            const float2 x2 = make_float2(v[i][y], v[i][y + 1]), e = fp_fma2(x2, lo2, fp_fma2(x2, hi2, k2));
            s[y / 2] = fp_add2(s[y / 2], make_float2(bs_ex2(e.x), bs_ex2(e.y)));
          }
        const float t = warp_sum((s[0].x + s[0].y) + (s[1].x + s[1].y));
        sum = bs_add(sum, {m == -INFINITY && t == 0.f ? -INFINITY : far ? k : 0.5f * k, t});
      }
      __syncthreads();
      const uint32_t bar = s_bar;
      // what is no smaller, and the best so far
      auto put = [&](unsigned long long k) {
        const int at = atomicAdd(&s_n, 1);
        if (at < kBsCands) s_u.cand[at] = k;
      };
      if (mt > -INFINITY && bs_ordered(mt + 0.f) >= bar) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
          for (int y = 0; y < 4; ++y)
            if (v[i][y] > -INFINITY && bs_ordered(v[i][y] + 0.f) >= bar) put(bs_key(v[i][y], (int)(c0 + 4 * (i * kBsThreads + (int)threadIdx.x)) + y));
      }
      unsigned long long mine = threadIdx.x < W ? s_list[list][threadIdx.x] : 0ull;
      if (mine != 0) put(mine);
      __syncthreads();
      const int n = s_n;
      if (n <= kBsCands) {
        // each one's place in the order is the number of larger ones
        if (threadIdx.x < n) {
          const unsigned long long k = s_u.cand[threadIdx.x];
          int rank = 0;
#pragma unroll 4
          for (int i = 0; i < n; ++i) rank += s_u.cand[i] > k;
          if (rank < W) s_list[list ^ 1][rank] = k;
        } else if (threadIdx.x < W) {
          s_list[list ^ 1][threadIdx.x] = 0;
        }
      } else {
        // Too many are as large (equal logits by the hundred): the W largest of all, one after the
        // other.
        unsigned long long best = mine, won = ~0ull;
        auto look = [&]() {
          best = mine < won ? mine : 0ull;
#pragma unroll
          for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const unsigned long long k = bs_key(v[i][y], (int)(c0 + 4 * (i * kBsThreads + (int)threadIdx.x)) + y);
              if (k < won && k > best) best = k;
            }
        };
        look();
        for (int r = 0; r < W; ++r) {
          const unsigned long long wm = bs_warp_max(best);
          if (lane == 0) s_best[r & 1][warp] = wm;
          __syncthreads();
          won = bs_warp_max(lane < kBsWarps ? s_best[r & 1][lane] : 0ull);
          if (threadIdx.x == 0) s_list[list ^ 1][r] = won;
          if (best == won && won != 0) look();
        }
      }
      list ^= 1;
      __syncthreads();
    }
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    if (warp == 0) {
      BsSum p = lane < kBsWarps ? s_sum[lane] : BsSum{-INFINITY, 0.f};
#pragma unroll
      for (int o = kBsWarps / 2; o > 0; o >>= 1)
        p = bs_add(p, {__shfl_xor_sync(0xffffffffu, p.r, o), __shfl_xor_sync(0xffffffffu, p.s, o)});
      if (lane == 0) a.sums[blockIdx.x] = make_float2(p.r, p.s);
      if (lane < W) a.best[(long long)blockIdx.x * W + lane] = s_list[list][lane];
    }
  }
  // the last CTA of the group goes on
  if (warp == 0) {
    __threadfence();
    __syncwarp();
    if (lane == 0) {
      const bool last = atomicAdd(a.tickets + b, 1) == W * S - 1;
      if (last) a.tickets[b] = 0;
      s_last = last;
      __threadfence();
    }
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  // each beam: its normaliser, and the W best of its pieces
  for (int w = warp; w < W; w += kBsWarps) {
    const int r = b * W + w;
    const float sc = __ldcg(a.score + r);
    const bool kept = a.done && __ldcg(a.done + r) != 0, real = sc > -INFINITY && sc < INFINITY;
    // (all that is needed at once, of beams that left nothing too)
    BsSum p = {-INFINITY, 0.f};
    if (lane < S) {
      const float2 f = __ldcg(a.sums + (long long)r * S + lane);
      p = {f.x, f.y};
    }
    const unsigned long long* lists = a.best + (long long)r * S * W;
#pragma unroll
    for (int i = 0; i < kBsLists; i += 32)
      if (i + lane < S * W) s_u.row[warp].list[i + lane] = __ldcg(lists + i + lane);
    if (lane == 0) s_done[w] = kept;
    if (lane < W) s_row[w][lane] = 0;
    __syncwarp();
    if (!real || kept) {  // no candidates, or the one that keeps it as it is
      if (!real && sc != -INFINITY && lane == 0 && a.err) atomicExch(a.err, 1);
      if (lane == 0) {
        if (real) s_row[w][0] = 1ull << 32 | (uint32_t)~a.end;
        s_off[w] = {sc, 0.f};
        s_ref[w] = 0.f;
      }
      continue;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      p = bs_add(p, {__shfl_xor_sync(0xffffffffu, p.r, o), __shfl_xor_sync(0xffffffffu, p.s, o)});
    const bool fine = p.s > 0.f && p.s < INFINITY;  // (a NaN or +inf among the logits: neither)
    if (!fine && p.r != -INFINITY && lane == 0 && a.err) atomicExch(a.err, 1);
    if (lane == 0) {
      const int e = (int)(__float_as_uint(p.s) >> 23) - 127 + 1;  // s = 2^e f, 1/2 <= f < 1
      const float f = __uint_as_float((__float_as_uint(p.s) & 0x7fffffu) | 0x3f000000u);
      // n = k + e: a pair, as k may be of 2^30, where fp32 holds multiples of 128 (rows of such
      // logits).  n ln 2 as a pair (0.693147180559945309), its error carried along
      constexpr float kHi = 0.693147182464599609375f, kLo = -1.904654299957767e-9f;
      const bool far = fabsf(p.r) >= kBsFar;
      const Pair n = sum2(far ? 0.f : 2.f * p.r, (float)e);
      const float h = __fmul_rn(n.hi, kHi);
      const Pair lse = add(tidy(h, __fmaf_rn(n.hi, kLo, __fmaf_rn(n.hi, kHi, -h))), Pair{__fmaf_rn(n.lo, kHi, logf(f)), 0.f});
      s_off[w] = add(Pair{sc, 0.f}, Pair{-lse.hi, -lse.lo});
      s_ref[w] = far ? p.r : 0.f;
    }
    // the pieces' lists, those that count side by side; each one's place is the number of
    // larger ones
    const unsigned long long* list = s_u.row[warp].list;
    unsigned long long* some = s_u.row[warp].some;
    const unsigned long long head = fine && lane < S ? list[lane * W] : 0ull;
    const int alive = __popc(__ballot_sync(0xffffffffu, head != 0));
    int r2 = 0;
#pragma unroll 8
    for (int i = 0; i < S; ++i) r2 += list[i * W] > head;
    if (head != 0)
      for (int i = 0; i < W - r2; ++i) some[bs_first(r2, W) + i] = list[lane * W + i];
    __syncwarp();
    const int n = bs_first(min(alive, W), W);
    for (int i0 = 0; i0 < n; i0 += 64) {
      const unsigned long long k = i0 + lane < n ? some[i0 + lane] : 0ull, k1 = i0 + 32 + lane < n ? some[i0 + 32 + lane] : 0ull;
      int rank = 0, rank1 = 0;
#pragma unroll 8
      for (int i = 0; i < n; ++i) {
        const unsigned long long u = some[i];
        rank += u > k, rank1 += u > k1;
      }
      if (k != 0 && rank < W) s_row[w][rank] = k;
      if (k1 != 0 && rank1 < W) s_row[w][rank1] = k1;
    }
    __syncwarp();
  }
  __syncthreads();
  // the beams' lists in the same way: scores as pairs (0: none, as where a sum falls below the least
  // fp32), ties to the lowest beam and, in a beam, the order of its list
  int valid = 0;
  for (int i = threadIdx.x; i < W * W; i += kBsThreads) {
    const int w = i / W;
    const unsigned long long k = s_row[w][i - w * W];
    unsigned long long score = 0;
    if (k != 0) {
      Pair v = s_off[w];
      if (k >> 32 != 1) {
        const Pair x = sum2(bs_value((uint32_t)(k >> 32)), -s_ref[w]);
        v = add(sum2(x.hi, v.hi), Pair{v.lo, x.lo});
      }
      if (v.hi > -INFINITY) {
        score = (unsigned long long)bs_ordered(v.hi + 0.f) << 32 | bs_ordered(v.lo + 0.f);
        ++valid;
      }
    }
    s_u.beam.score[w][i - w * W] = score;
  }
  if (threadIdx.x == 0) s_n = 0;
  __syncthreads();
  if (valid) atomicAdd(&s_n, valid);
  for (int i = threadIdx.x; i < W * W; i += kBsThreads) {
    const int w = i / W, e = i - w * W;
    const unsigned long long head = s_u.beam.score[w][0];
    int r = 0;
#pragma unroll 4
    for (int o = 0; o < W; ++o) {
      const unsigned long long v = s_u.beam.score[o][0];
      r += v > head || (v == head && o < w);
    }
    if (r + e < W) {
      s_u.beam.some[bs_first(r, W) + e] = s_u.beam.score[w][e];
      s_u.beam.place[bs_first(r, W) + e] = i;
    }
  }
  const int n = bs_first(W, W);
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kBsThreads) {
    const unsigned long long v = s_u.beam.some[i];
    const int at = s_u.beam.place[i];
    int rank = 0, same = 0;
#pragma unroll 8
    for (int o = 0; o < n; ++o) {
      const unsigned long long u = s_u.beam.some[o];
      rank += u > v, same += u == v;
    }
    if (v == 0) continue;
    if (same > 1)
      for (int o = 0; o < n; ++o) rank += s_u.beam.some[o] == v && s_u.beam.place[o] < at;
    if (rank < W) {
      const int w = at / W, c = b * W + rank, t = (int)~(uint32_t)s_row[w][at - w * W];
      a.parent[c] = w;
      a.token[c] = t;
      a.new_score[c] = bs_value((uint32_t)(v >> 32));
      if (a.new_done) a.new_done[c] = s_done[w] || t == a.end;
    }
  }
  __syncthreads();
  for (int i = s_n + threadIdx.x; i < W; i += kBsThreads) {  // fewer candidates than places
    const int c = b * W + i;
    a.parent[c] = -1;
    a.token[c] = -1;
    a.new_score[c] = -INFINITY;
    if (a.new_done) a.new_done[c] = 0;
  }
}

// Pieces of a row: as many as it needs to be held in registers, more where the rows do not
// fill the GPU, and no more than the lists' room (us: 8 rows of 128001 as 8 | 16 pieces 12.4 |
// 11.3, 128 rows of 32000 as 1 | 2 | 4 pieces 17 | 11.6 | 14).
static int bs_splits(int rows, int W, int V) {
  const int most = std::min(kBsSplits, kBsLists / W);
  int S = std::min(most, (V + kBsPiece - 1) / kBsPiece);
  while (2 * S <= most && (long long)rows * S < 152 && V / S >= 4096) S *= 2;
  return S;
}

static size_t bs_align(size_t n) { return (n + 255) / 256 * 256; }

size_t beam_select_ws_bytes(int B, int W, int V) {
  const size_t rows = (size_t)B * W, S = bs_splits((int)rows, W, V);
  return kBsHead + bs_align(rows * S * 8) + rows * S * W * 8;
}

cudaError_t launch_beam_select(const float* logits, int V, int B, int W, const float* score, const int32_t* done, int end,
                               int32_t* parent, int32_t* token, float* new_score, int32_t* new_done, void* ws, int32_t* err,
                               cudaStream_t s) {
  if (B <= 0) return cudaSuccess;
  const int S = bs_splits(B * W, W, V);
  uint8_t* p = (uint8_t*)ws;
  uint8_t* sums = p + kBsHead;
  uint8_t* best = sums + bs_align((size_t)B * W * S * 8);
  const BsArgs a = {logits, V, B, W, S, ((V + S - 1) / S + 3) / 4 * 4, score, done, end, parent, token, new_score, new_done,
                    (int32_t*)p, (float2*)sums, (unsigned long long*)best, err};
  auto go = [&](auto kern) { return launch_early(kern, dim3((unsigned)(B * W * S)), dim3(kBsThreads), 0, s, a); };
  const int items = (a.per + 4 * kBsThreads - 1) / (4 * kBsThreads);
  return items <= 2 ? go(beam_select_kernel<2>) : items <= 4 ? go(beam_select_kernel<4>) : go(beam_select_kernel<kBsItems>);
}

// ------------------------------------------------------------------ reordering
// Beam w's new row of the page table is its parent's: the pages of full blocks shared, the
// blocks not begun its own.  The block that is part-filled has a page of its own for every
// beam: the first of a beam's children takes its page as it is, the others, in order, the
// pages of the beams without children (there are as many as are needed), into which the
// parent's rows then have to be copied.  So nothing that is copied from is written to,
// and no page is taken or given back.  One CTA a beam, its group's parents in a warp's
// lanes.  Bound by latency: 128 beams of 135 pages 2.0 us.
__global__ void __launch_bounds__(128)
    beam_reorder_kernel(int W, int pps, int page_size, const int32_t* __restrict__ len, const int32_t* __restrict__ parent,
                        const int32_t* __restrict__ in, int32_t* __restrict__ out, int32_t* __restrict__ from,
                        int32_t* __restrict__ to, int32_t* __restrict__ rows, int32_t* err) {
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.x / W, w = blockIdx.x - b * W, lane = threadIdx.x & 31;
  const int32_t* group = in + (long long)b * W * pps;
  const int n = __ldg(len + b);
  const bool bad_len = n < 0 || n > (long long)pps * page_size;
  int p = lane < W ? __ldg(parent + b * W + lane) : -1;
  const bool bad = p < -1 || p >= W;
  if (bad) p = -1;
  if (__any_sync(0xffffffffu, bad || bad_len) && threadIdx.x == 0 && err) atomicExch(err, 1);
  if (bad_len) p = lane < W ? lane : -1;  // the group stays as it is
  const unsigned same = __match_any_sync(0xffffffffu, p);
  const bool keeps = p >= 0 && __ffs(same) - 1 == lane;
  const unsigned born = __reduce_or_sync(0xffffffffu, p >= 0 ? 1u << p : 0u);
  unsigned spare = ~born & (W == 32 ? ~0u : (1u << W) - 1);
  const unsigned others = __ballot_sync(0xffffffffu, lane < W && !keeps);
  const int mine = __shfl_sync(0xffffffffu, p, w);
  const bool kept = __shfl_sync(0xffffffffu, (int)keeps, w);
  for (int i = __popc(others & ((1u << w) - 1)); i > 0; --i) spare &= spare - 1;
  const int page_of = kept ? mine : __ffs(spare) - 1;  // whose page of the part-filled block this beam takes
  const int tail = bad_len ? pps : n / page_size, rem = bad_len ? 0 : n % page_size;
  const int32_t* own = group + (long long)w * pps;
  const int32_t* came = mine >= 0 ? group + (long long)mine * pps : own;
  int32_t* o = out + (long long)blockIdx.x * pps;
  for (int i = threadIdx.x; i < pps; i += 128)
    o[i] = i < tail ? __ldg(came + i) : i == tail && rem > 0 ? __ldg(group + (long long)page_of * pps + i) : __ldg(own + i);
  if (threadIdx.x == 0) {
    const bool copy = rem > 0 && mine >= 0 && !kept;
    from[blockIdx.x] = copy ? __ldg(came + tail) : -1;
    to[blockIdx.x] = copy ? __ldg(group + (long long)page_of * pps + tail) : -1;
    rows[blockIdx.x] = copy ? rem : 0;
  }
}

cudaError_t launch_beam_reorder(int B, int W, int pps, int page_size, const int32_t* len, const int32_t* parent,
                                const int32_t* in, int32_t* out, int32_t* from, int32_t* to, int32_t* rows, int32_t* err,
                                cudaStream_t s) {
  if (B <= 0) return cudaSuccess;
  return launch_early(beam_reorder_kernel, dim3(B * W), dim3(128), 0, s, W, pps, page_size, len, parent, in, out, from, to, rows,
                err);
}

// ------------------------------------------------------------------ copies of pages
// The first rows of one page to another, all KV heads, K, V and scales.  A head's rows
// stand together, so a copy is 2 Hkv runs; a warp takes a run, 16 bytes a lane, all of it
// on its way before the first is written.  Bound by latency, then bytes: 128 beams, 8 int8
// heads 2.0 us, 40 beams, 40 bf16 heads 2.1 us.
constexpr int kKcWarps = 8;

template <int RB>  // bytes of a head's row
__global__ void __launch_bounds__(kKcWarps * 32)
    kv_copy_kernel(fp_kv_view kv, const int32_t* __restrict__ from, const int32_t* __restrict__ to,
                   const int32_t* __restrict__ rows, int32_t* err) {
  pdl_trigger();
  pdl_wait();
  const int i = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int src = __ldg(from + i), dst = __ldg(to + i), n = __ldg(rows + i);
  if (src == -1 || n == 0) return;
  if (src < 0 || src >= kv.n_pages || dst < 0 || dst >= kv.n_pages || n < 0 || n > kv.page_size) {
    if (threadIdx.x == 0 && err) atomicExch(err, 1);
    return;
  }
  for (int item = blockIdx.y * kKcWarps + warp; item < 2 * kv.n_kv_heads; item += gridDim.y * kKcWarps) {
    const bool is_v = item >= kv.n_kv_heads;
    const int h = is_v ? item - kv.n_kv_heads : item;
    const long long r0 = ((long long)src * kv.n_kv_heads + h) * kv.page_size, r1 = ((long long)dst * kv.n_kv_heads + h) * kv.page_size;
    uint8_t* pool = (uint8_t*)(is_v ? kv.v_pool : kv.k_pool);
    constexpr int N = RB / 32;  // 16-byte pieces a lane has of sixteen rows
    uint4 v[N];
#pragma unroll
    for (int k = 0; k < N; ++k)
      if ((k * 32 + lane) * 16 < n * RB) v[k] = *reinterpret_cast<const uint4*>(pool + r0 * RB + (k * 32 + lane) * 16);
    float* scale = kv.kvquant == FP_KV_INT8 ? (is_v ? kv.v_scale : kv.k_scale) : nullptr;
    if (scale && lane < n) scale[r1 + lane] = scale[r0 + lane];
#pragma unroll
    for (int k = 0; k < N; ++k)
      if ((k * 32 + lane) * 16 < n * RB) *reinterpret_cast<uint4*>(pool + r1 * RB + (k * 32 + lane) * 16) = v[k];
  }
}

cudaError_t launch_kv_copy(const fp_kv_view& kv, int n, const int32_t* from, const int32_t* to, const int32_t* rows,
                           int32_t* err, cudaStream_t s) {
  if (n <= 0) return cudaSuccess;
  const dim3 grid(n, std::min((2 * kv.n_kv_heads + kKcWarps - 1) / kKcWarps, 1024));
  auto go = [&](auto kern) { return launch_early(kern, grid, dim3(kKcWarps * 32), 0, s, kv, from, to, rows, err); };
  const int rb = kv.head_dim * (kv.kvquant == FP_KV_INT8 ? 1 : 2);
  return rb == 64 ? go(kv_copy_kernel<64>) : rb == 128 ? go(kv_copy_kernel<128>) : go(kv_copy_kernel<256>);
}

}  // namespace fpk
