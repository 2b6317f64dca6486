// Probabilities of the LM head's logits, and the verification of drafted tokens
// against them with given random numbers (speculative decoding).  Both stand
// beside the greedy choice of fp_rows.cu: one cluster of CTAs a row.
#include <cooperative_groups.h>

#include <utility>

#include "chunk.cuh"
#include "kernels.cuh"
#include "pair.cuh"

namespace cg = cooperative_groups;

namespace fpk {

// ------------------------------------------------------------------ softmax
// y_i = exp((x_i - max x) / T) / sum_j exp((x_j - max x) / T), T the row's
// temperature; T = 0: 1 at the lowest index of the maximum, else 0.
//
// A cluster of 1 to 8 CTAs a row, so that few long rows have as many SMs as many
// short ones.  Each warp keeps its part of the row in registers (ITEMS 16-byte groups
// a thread) as exponentials against its own maximum; the warps' maxima and sums meet
// once through shared and distributed shared memory, and each value is written as
// e 2^((m_warp - m) c) / sum: one read, one write, one meeting.  Rows of more than
// 262144 values (512 threads x 16 groups x 8 CTAs) are read a second time instead.
// Groups are aligned in memory: the row's first and last may be part of a neighbour's.
// Bound by latency and bytes one after the other (CTAs read, meet and write in step) and
// by the waves: two CTAs an SM are 304 places, so 152 rows of 32000, in clusters of two,
// take 11.1 us (3.5 TB/s) and 160 rows, whose last eight start when others have ended,
// 15.4 (2.7 TB/s).  3 rows of 128001 6.3.
constexpr int kSmThreads = 512, kSmWarps = kSmThreads / 32, kSmItems = 16, kSmMaxCTAs = 8;

FP_DEV float sm_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A set's maximum and its sum of exponentials against it, or (T = 0) the lowest index
// of the maximum.
struct SmPart {
  float m, s;
  int at;
};
FP_DEV void sm_add(SmPart& a, float m, float s, int at, float c) {
  const float m2 = fmaxf(a.m, m);
  // (a set without values has s = 0: its -inf - -inf stays out)
  const float fa = a.m == -INFINITY ? 0.f : sm_ex2((a.m - m2) * c), fb = m == -INFINITY ? 0.f : sm_ex2((m - m2) * c);
  a.s = a.s * fa + s * fb;
  if (m == a.m) a.at = min(a.at, at);
  else if (m > a.m) a.at = at;
  a.m = m2;
}

// ITEMS 0: any length, read twice.
template <int ITEMS>
__global__ void __launch_bounds__(kSmThreads)
    softmax_kernel(const float* x, int V, const float* __restrict__ temp, float* y, int32_t* err) {
  __shared__ SmPart s_part[kSmWarps], s_cta;
  pdl_trigger();
  pdl_wait();
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long row = blockIdx.x / C;
  const float* xr = x + row * V;
  float* yr = y + row * V;
  // groups of four: group g holds values 4 g - skew .. 4 g - skew + 3
  const int skew = (int)(((uintptr_t)xr & 15) >> 2), groups = (V + skew + 3) >> 2;
  const int per = ((groups + C - 1) / C + 31) & ~31;  // of a CTA, by whole warps
  const int g0 = min(groups, rank * per), g1 = min(groups, g0 + per);
  const float t = temp ? __ldg(temp + row) : 1.f;
  const bool bad = !(t >= 0.f) || isinf(t), greedy = t == 0.f;
  if (bad && rank == 0 && threadIdx.x == 0 && err) atomicExch(err, 1);
  const float c = greedy ? 1.f : fminf(1.4426950408889634f / t, 3.4e38f);
  auto load = [&](int g) -> float4 {
    const int i = 4 * g - skew;
    if (g >= g1) return make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    if (i >= 0 && i + 3 < V) return *reinterpret_cast<const float4*>(xr + i);
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = i + k >= 0 && i + k < V ? xr[i + k] : -INFINITY;
    return make_float4(v[0], v[1], v[2], v[3]);
  };
  auto top = [](float4 v) { return fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)); };
  auto lowest = [&](float4 v, int g, float m, int at) {  // the lowest index of m so far
    const int i = 4 * g - skew;
    return min(at, v.x == m ? i : v.y == m ? i + 1 : v.z == m ? i + 2 : v.w == m ? i + 3 : 0x7fffffff);
  };
  auto expo = [&](float4 v, float m) {  // against m (-inf: a set that is masked throughout)
    const float r = m == -INFINITY ? 0.f : m;
    return make_float4(sm_ex2((v.x - r) * c), sm_ex2((v.y - r) * c), sm_ex2((v.z - r) * c), sm_ex2((v.w - r) * c));
  };

  // this warp's part, ITEMS groups a lane in registers
  float4 v[ITEMS ? ITEMS : 1];
  SmPart p = {-INFINITY, 0.f, 0x7fffffff};
  if constexpr (ITEMS > 0) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) v[k] = load(g0 + k * kSmThreads + (int)threadIdx.x);
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) p.m = fmaxf(p.m, top(v[k]));
    p.m = warp_max(p.m);
    if (greedy) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) p.at = lowest(v[k], g0 + k * kSmThreads + (int)threadIdx.x, p.m, p.at);
      p.at = __reduce_min_sync(0xffffffffu, p.at);
    } else {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        v[k] = expo(v[k], p.m);
        p.s += (v[k].x + v[k].y) + (v[k].z + v[k].w);
      }
      p.s = warp_sum(p.s);
    }
  } else {
#pragma unroll 1
    for (int g = g0 + (int)threadIdx.x; g < g1; g += 4 * kSmThreads) {
      float4 w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = load(g + k * kSmThreads);
      float m = -INFINITY, s = 0.f;
      int at = 0x7fffffff;
#pragma unroll
      for (int k = 0; k < 4; ++k) m = fmaxf(m, top(w[k]));
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (greedy) at = lowest(w[k], g + k * kSmThreads, m, at);
        const float4 e = expo(w[k], m);
        s += (e.x + e.y) + (e.z + e.w);
      }
      sm_add(p, m, s, at, c);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      sm_add(p, __shfl_xor_sync(0xffffffffu, p.m, o), __shfl_xor_sync(0xffffffffu, p.s, o),
             __shfl_xor_sync(0xffffffffu, p.at, o), c);
  }
  const float mine = p.m;  // what this warp's exponentials are against
  if (lane == 0) s_part[warp] = p;
  __syncthreads();
  p = s_part[lane & (kSmWarps - 1)];
#pragma unroll
  for (int o = kSmWarps / 2; o > 0; o >>= 1)
    sm_add(p, __shfl_xor_sync(0xffffffffu, p.m, o), __shfl_xor_sync(0xffffffffu, p.s, o),
           __shfl_xor_sync(0xffffffffu, p.at, o), c);
  if (C > 1) {
    if (threadIdx.x == 0) s_cta = p;
    cluster.sync();
    p = *cluster.map_shared_rank(&s_cta, lane & (C - 1));
    for (int o = C / 2; o > 0; o >>= 1)
      sm_add(p, __shfl_xor_sync(0xffffffffu, p.m, o), __shfl_xor_sync(0xffffffffu, p.s, o),
             __shfl_xor_sync(0xffffffffu, p.at, o), c);
  }

  const bool nothing = bad || (p.m == -INFINITY && (greedy || p.s == 0.f));  // (a NaN: p.s is one)
  const bool same = ((uintptr_t)xr & 15) == ((uintptr_t)yr & 15);
  auto store = [&](int g, float4 o) {
    const int i = 4 * g - skew;
    if (g >= g1) return;
    if (same && i >= 0 && i + 3 < V) {
      *reinterpret_cast<float4*>(yr + i) = o;
      return;
    }
    const float f[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k >= 0 && i + k < V) yr[i + k] = f[k];
  };
  float f = 1.f / p.s;
  if (ITEMS > 0 && p.s == p.s) f = mine == -INFINITY ? 0.f : sm_ex2((mine - p.m) * c) / p.s;
  auto emit = [&](int g, float4 e) {
    float4 o;
    if (nothing) {
      o = make_float4(0.f, 0.f, 0.f, 0.f);
    } else if (greedy) {
      const int i = 4 * g - skew;
      o = make_float4(i == p.at ? 1.f : 0.f, i + 1 == p.at ? 1.f : 0.f, i + 2 == p.at ? 1.f : 0.f, i + 3 == p.at ? 1.f : 0.f);
    } else {
      o = make_float4(e.x * f, e.y * f, e.z * f, e.w * f);
    }
    store(g, o);
  };
  if constexpr (ITEMS > 0) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) emit(g0 + k * kSmThreads + (int)threadIdx.x, v[k]);
  } else {
#pragma unroll 4
    for (int g = g0 + (int)threadIdx.x; g < g1; g += kSmThreads) emit(g, expo(load(g), p.m));
  }
  if (C > 1) cluster.sync();  // the others have read this CTA's part
}

// CTAs a row, a power of two: few, so that a thread holds up to eight groups, but enough
// for few rows to reach most SMs.  Larger clusters cost more to start than their
// parallel loads give (us with up to 8 | 4 | 2 groups a thread: 400 rows of 50000 44.8 |
// 66 | 66, 160 x 32000 15.0 | 15.2 | 23).
cudaError_t launch_softmax(const float* logits, int M, int V, const float* temp, float* probs, int32_t* err,
                           cudaStream_t s) {
  if (M <= 0) return cudaSuccess;
  const int groups = V / 4 + 2;
  int C = 1;
  while (C < kSmMaxCTAs && (groups > 8 * kSmThreads * C || (long long)M * C < 128)) C *= 2;
  while (C > 1 && groups <= kSmThreads / 2 * C) C /= 2;  // no CTA without work
  const int items = (groups + C * kSmThreads - 1) / (C * kSmThreads);
  auto go = [&](auto kern) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)M * C);
    cfg.blockDim = dim3(kSmThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = C;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = g_pdl ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, logits, V, temp, probs, err);
  };
  return items <= 2 ? go(softmax_kernel<2>) : items <= 4 ? go(softmax_kernel<4>) : items <= 8 ? go(softmax_kernel<8>) : items <= kSmItems ? go(softmax_kernel<kSmItems>) : go(softmax_kernel<0>);
}

// ------------------------------------------------------------------ verification
// Sequence b's rows are its last accepted token and the k drafted after it.  Row
// i's draft t (the token of row i + 1) is accepted while u_i q_i(t) < p_i(t); a is the
// first refused row, or k.  The token after it is drawn from w = max(0, p_a - q_a)
// (a < k), or p_k: the lowest t with sum_{s <= t} w_s > r sum w.
// A border is a sum of up to V fp32 values and has to fall where fp64 puts it, but
// fp64 is slow here (an addition takes about 300 cycles, and there were forty one
// after another: 21 us for 32 sequences of 32000 tokens).  So sums are pairs of fp32,
// hi + lo, the error of every addition carried along: good to 2^-46 or better.
// Differences p - q and products u q are exact as pairs (the error-free sum of Knuth, TAOCP
// vol. 2, 4.2.2, and Dekker's renormalisation, Numer. Math. 18, 1971).
// A cluster of 8 CTAs a sequence: every warp sums a run of consecutive weights, the
// CTAs' totals meet through distributed shared memory, and the warp whose run holds
// the border looks through it again (from L2): 32 pieces, then the piece's tokens.
// Bound by latency: cu, the drafts, their probabilities, the row, the meeting and the
// second look follow one another.
constexpr int kVfCTAs = 8, kVfThreads = 512, kVfWarps = kVfThreads / 32, kVfRuns = kVfCTAs * kVfWarps;

// Of the lanes whose weight counts, the first whose sum is past the border; rounding at
// the very end, an r of 1 or more or a NaN leaves none: the last then.  -1: no weight at all.
FP_DEV int holder(Pair upto, float w, Border border) {
  const unsigned has = __ballot_sync(0xffffffffu, w > 0.f), over = __ballot_sync(0xffffffffu, w > 0.f && past(upto, border));
  return over ? __ffs(over) - 1 : 31 - __clz(has);
}

// The weight of token t: p, less q where there is one, without token `gone`; none below zero.
FP_DEV Pair weight(const float* p, const float* q, int t, int gone) {
  Pair w = sum2(__ldg(p + t), q ? -__ldg(q + t) : 0.f);
  if (!(w.hi > 0.f) || t == gone) w = {0.f, 0.f};
  return w;
}

__global__ void __cluster_dims__(kVfCTAs, 1, 1) __launch_bounds__(kVfThreads)
    verify_kernel(const float* __restrict__ p, const float* __restrict__ q, int V, int n_tokens, int B,
                  const int32_t* __restrict__ cu, const int32_t* __restrict__ tokens, const float* __restrict__ u,
                  const float* __restrict__ r, int32_t* __restrict__ out, int32_t* __restrict__ n_out, int32_t* err) {
  __shared__ Pair s_sum[kVfWarps], s_cta;
  __shared__ int s_a;
  pdl_trigger();
  pdl_wait();
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), b = blockIdx.x / kVfCTAs;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (blockIdx.x == 0) chunk_check(cu, B, n_tokens, err);
  int row0, n;
  chunk_rows(cu, b, n_tokens, &row0, &n);
  if (n == 0) {  // no rows: nothing to verify (the whole cluster leaves)
    if (rank == 0 && threadIdx.x == 0) n_out[b] = 0;
    return;
  }
  // the first refused draft
  if (warp == 0) {
    int a = n - 1;
#pragma unroll 1
    for (int i0 = 0; i0 < n - 1; i0 += 32) {
      const int i = i0 + lane;
      bool refused = false, ok = true;
      if (i < n - 1) {
        const int t = __ldg(tokens + row0 + i + 1);
        ok = t >= 0 && t < V;
        const long long at = (long long)(row0 + i) * V + (ok ? t : 0);
        // u q < p exactly: the rounded product, and where that is p its error.  Both sides
        // times 2^80 where the error of a product near p could underflow.
        float qt = q ? __ldg(q + at) : 1.f, pt = __ldg(p + at);
        const float ui = __ldg(u + row0 + i);
        if (pt < 1e-15f && qt < 0x1p40f) qt *= 0x1p80f, pt *= 0x1p80f;
        const float x = __fmul_rn(ui, qt), e = __fmaf_rn(ui, qt, -x);
        refused = !ok || !(x < pt || (x == pt && e < 0.f));
      }
      const unsigned any = __ballot_sync(0xffffffffu, refused);
      if (any) {
        a = i0 + __ffs(any) - 1;
        if (i == a && !ok && rank == 0 && err) atomicExch(err, 1);  // (what is behind it may be padding)
        break;
      }
    }
    if (lane == 0) s_a = a;
  }
  __syncthreads();
  const int a = s_a;
  const float* pr = p + (long long)(row0 + a) * V;
  const float* qr = a < n - 1 && q ? q + (long long)(row0 + a) * V : nullptr;
  int gone = a < n - 1 && !q ? __ldg(tokens + row0 + a + 1) : -1;
  const int run = (V + kVfRuns - 1) / kVfRuns;
  const int lo = (int)min((long long)V, (long long)(rank * kVfWarps + warp) * run), hi = min(V, lo + run);
  const float rb = __ldg(r + b);
  for (int turn = 0; turn < 2; ++turn) {
    Pair s = {0.f, 0.f};
#pragma unroll 1
    for (int t0 = lo + lane; t0 < hi; t0 += 16 * 32) {  // sixteen loads in flight
      float x[16], y[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const int t = t0 + 32 * k;
        x[k] = t < hi ? __ldg(pr + t) : 0.f;
        y[k] = t < hi && qr ? __ldg(qr + t) : 0.f;
      }
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        Pair w = sum2(x[k], -y[k]);
        if (!(w.hi > 0.f) || t0 + 32 * k == gone) w = {0.f, 0.f};
        const Pair f = sum2(s.hi, w.hi);
        s = {f.hi, __fadd_rn(s.lo, __fadd_rn(f.lo, w.lo))};
      }
    }
    s = shfl(scan<32>(tidy(s.hi, s.lo), lane), 31);
    if (lane == 0) s_sum[warp] = s;
    __syncthreads();
    const Pair mine = s_sum[lane & (kVfWarps - 1)], upto = scan<kVfWarps>(mine, lane);  // within this CTA
    if (threadIdx.x == kVfWarps - 1) s_cta = upto;
    cluster.sync();
    const Pair theirs = *cluster.map_shared_rank(&s_cta, lane & (kVfCTAs - 1)), all = scan<kVfCTAs>(theirs, lane);
    const Pair total = shfl(all, kVfCTAs - 1);
    auto leave = cluster.barrier_arrive();  // (a CTA stays until the others have read its total)
    const bool drawable = total.hi > 0.f && total.hi < INFINITY;
    if (drawable) {
      const Border border = border_at(total, rb);
      if (holder(all, lane < kVfCTAs ? theirs.hi : 0.f, border) == rank) {
        const Pair before = rank ? shfl(all, rank - 1) : Pair{0.f, 0.f};
        const Pair to = add(before, upto);
        if (holder(to, lane < kVfWarps ? mine.hi : 0.f, border) == warp) {
          const Pair from = warp ? shfl(to, warp - 1) : before;
          // within the run: 32 pieces, then the tokens of the piece
          const int seg = (hi - lo + 31) / 32;
          Pair ps = {0.f, 0.f};
#pragma unroll 4
          for (int t = lo + lane * seg; t < min(hi, lo + (lane + 1) * seg); ++t) ps = add(ps, weight(pr, qr, t, gone));
          const Pair pu = add(from, scan<32>(ps, lane));
          const int piece = holder(pu, ps.hi, border);
          Pair at = piece ? shfl(pu, piece - 1) : from;
          int token = -1;
          const int t1 = min(hi, lo + (piece + 1) * seg);
#pragma unroll 1
          for (int t0 = lo + piece * seg; t0 < t1; t0 += 32) {
            const Pair w = t0 + lane < t1 ? weight(pr, qr, t0 + lane, gone) : Pair{0.f, 0.f};
            const Pair wu = add(at, scan<32>(w, lane));
            const int l = holder(wu, w.hi, border);
            if (l >= 0) token = t0 + l;
            if (__any_sync(0xffffffffu, w.hi > 0.f && past(wu, border))) break;
            at = shfl(wu, 31);
          }
          if (lane == 0) {
            out[row0 + a] = token;
            n_out[b] = a + 1;
          }
        }
      }
    }
    cluster.barrier_wait(std::move(leave));
    if (drawable) break;
    if (turn == 0 && (qr || gone >= 0)) {  // the draft leaves nothing (p <= q throughout): the target's own
      qr = nullptr;
      gone = -1;
      continue;
    }
    if (rank == 0 && threadIdx.x == 0) {
      if (err) atomicExch(err, 1);
      out[row0 + a] = -1;
      n_out[b] = a;
    }
    break;
  }
  // the accepted drafts, and nothing behind the token drawn after them
  if (rank == 0)
    for (int i = threadIdx.x; i < n; i += kVfThreads)
      if (i != a) out[row0 + i] = i < a ? __ldg(tokens + row0 + i + 1) : -1;
}

cudaError_t launch_verify_draft(const float* p, const float* q, int V, int n_tokens, int B, const int32_t* cu,
                                const int32_t* tokens, const float* u, const float* r, int32_t* out, int32_t* n_out,
                                int32_t* err, cudaStream_t s) {
  if (B <= 0) return cudaSuccess;
  return launch(verify_kernel, dim3(B * kVfCTAs), dim3(kVfThreads), 0, s, p, q, V, n_tokens, B, cu, tokens, u, r, out,
                n_out, err);
}

// ------------------------------------------------------------------ verification of a tree
// From row 0 of a sequence's tree down: a token is drawn from the row's distribution, the
// lowest t with sum_{s <= t} p_s > u sum p; the row's child with that token is the next
// row, and where it has none the token is the one after the accepted ones.  What comes
// out is distributed as p, whatever was drafted.  Each step as in the verification above,
// the sums in pairs; the warp that finds the token finds the child, and tells the cluster.
__global__ void __cluster_dims__(kVfCTAs, 1, 1) __launch_bounds__(kVfThreads)
    verify_tree_kernel(const float* __restrict__ p, int V, int n_tokens, int B, const int32_t* __restrict__ cu,
                       const int32_t* __restrict__ parent, const int32_t* __restrict__ tokens,
                       const float* __restrict__ u, int32_t* __restrict__ path, int32_t* __restrict__ out,
                       int32_t* __restrict__ n_out, int32_t* err) {
  __shared__ Pair s_sum[kVfWarps], s_cta;
  __shared__ int s_next;
  pdl_trigger();
  pdl_wait();
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), b = blockIdx.x / kVfCTAs;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (blockIdx.x == 0) chunk_check(cu, B, n_tokens, err);
  int row0, n;
  chunk_rows(cu, b, n_tokens, &row0, &n);
  if (n == 0) {  // (the whole cluster leaves)
    if (rank == 0 && threadIdx.x == 0) n_out[b] = 0;
    return;
  }
  const int run = (V + kVfRuns - 1) / kVfRuns;
  const int lo = (int)min((long long)V, (long long)(rank * kVfWarps + warp) * run), hi = min(V, lo + run);
  int cur = 0, a = 0;
  for (;; ++a) {
    const float* pr = p + (long long)(row0 + cur) * V;
    const float r = __ldg(u + row0 + cur);
    Pair s = {0.f, 0.f};
#pragma unroll 1
    for (int t0 = lo + lane; t0 < hi; t0 += 16 * 32) {  // sixteen loads in flight
      float x[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) x[k] = t0 + 32 * k < hi ? __ldg(pr + t0 + 32 * k) : 0.f;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const Pair f = sum2(s.hi, x[k] > 0.f ? x[k] : 0.f);
        s = {f.hi, __fadd_rn(s.lo, f.lo)};
      }
    }
    s = shfl(scan<32>(tidy(s.hi, s.lo), lane), 31);
    if (lane == 0) s_sum[warp] = s;
    __syncthreads();
    const Pair mine = s_sum[lane & (kVfWarps - 1)], upto = scan<kVfWarps>(mine, lane);  // within this CTA
    if (threadIdx.x == kVfWarps - 1) s_cta = upto;
    cluster.sync();
    const Pair theirs = *cluster.map_shared_rank(&s_cta, lane & (kVfCTAs - 1)), all = scan<kVfCTAs>(theirs, lane);
    const Pair total = shfl(all, kVfCTAs - 1);
    const bool drawable = total.hi > 0.f && total.hi < INFINITY;
    if (drawable) {
      const Border border = border_at(total, r);
      if (holder(all, lane < kVfCTAs ? theirs.hi : 0.f, border) == rank) {
        const Pair before = rank ? shfl(all, rank - 1) : Pair{0.f, 0.f};
        const Pair to = add(before, upto);
        if (holder(to, lane < kVfWarps ? mine.hi : 0.f, border) == warp) {
          const Pair from = warp ? shfl(to, warp - 1) : before;
          // within the run: 32 pieces, then the tokens of the piece
          const int seg = (hi - lo + 31) / 32;
          Pair ps = {0.f, 0.f};
#pragma unroll 4
          for (int t = lo + lane * seg; t < min(hi, lo + (lane + 1) * seg); ++t) ps = add(ps, weight(pr, nullptr, t, -1));
          const Pair pu = add(from, scan<32>(ps, lane));
          const int piece = holder(pu, ps.hi, border);
          Pair at = piece ? shfl(pu, piece - 1) : from;
          int token = -1;
          const int t1 = min(hi, lo + (piece + 1) * seg);
#pragma unroll 1
          for (int t0 = lo + piece * seg; t0 < t1; t0 += 32) {
            const Pair w = t0 + lane < t1 ? weight(pr, nullptr, t0 + lane, -1) : Pair{0.f, 0.f};
            const Pair wu = add(at, scan<32>(w, lane));
            const int l = holder(wu, w.hi, border);
            if (l >= 0) token = t0 + l;
            if (__any_sync(0xffffffffu, w.hi > 0.f && past(wu, border))) break;
            at = shfl(wu, 31);
          }
          int child = -1;
#pragma unroll 1
          for (int i0 = cur + 1; i0 < n && child < 0; i0 += 32) {
            const int i = i0 + lane;
            const bool it = i < n && __ldg(parent + row0 + i) == cur && __ldg(tokens + row0 + i) == token;
            const unsigned any = __ballot_sync(0xffffffffu, it);
            if (any) child = i0 + __ffs(any) - 1;
          }
          if (lane == 0) out[row0 + a] = token, path[row0 + a] = cur;
          if (lane < kVfCTAs) *cluster.map_shared_rank(&s_next, lane) = child;
        }
      }
    }
    cluster.sync();
    if (!drawable) {
      if (rank == 0 && threadIdx.x == 0) {
        if (err) atomicExch(err, 1);
        out[row0 + a] = -1, path[row0 + a] = cur;
        n_out[b] = a;
      }
      break;
    }
    if (s_next < 0) {
      if (rank == 0 && threadIdx.x == 0) n_out[b] = a + 1;
      break;
    }
    cur = s_next;
  }
  if (rank == 0)
    for (int i = a + 1 + (int)threadIdx.x; i < n; i += kVfThreads) out[row0 + i] = -1, path[row0 + i] = -1;
}

// The same in two kernels: a token drawn for every row at once, then the way down.  More
// is read, but nothing waits for a step before it.  Bound by bytes and issue slots for
// many rows (32 trees of 16 rows of 32000 tokens: 49 MB in 11 us), else by latency.
//
// A warp, a CTA or a cluster of up to 8 CTAs a row (launch_verify_tree): a warp takes a run
// of consecutive weights, in 16-byte groups aligned in memory, as 32 chunks of 32 k groups,
// and sums each of them; its lanes then hold a chunk's sum each.  The runs' sums meet, and
// the warp whose run holds the border has the chunk by a scan, and reads that one again.
// The token (-1: no weight, or an infinite one) stands in out until the second kernel has
// read it.
// Every weight costs issue slots, so a group is summed exactly by packed additions, x + z
// beside y + w, and the lanes' sums of eight chunks change places through shared memory, not
// by shuffles; four groups a lane are on their way while four are summed.
constexpr int kTdThreads = 256, kTdWarps = kTdThreads / 32, kTdMaxCTAs = 8;
constexpr int kTdRow = 33;  // a chunk's lane sums in shared memory, padded

// T: warps a row, 1 or all.  ONE: k is 1 (runs of up to 4096 weights).
template <int T, bool ONE>
__global__ void __launch_bounds__(kTdThreads, 3)
    tree_draw_kernel(const float* __restrict__ p, int V, int n_tokens, int B, const int32_t* __restrict__ cu,
                     const float* __restrict__ u, int32_t* __restrict__ out, int32_t* err) {
  __shared__ Pair s_sum[kTdWarps], s_cta, s_chunk[kTdWarps][32];
  __shared__ float2 s_lane[kTdWarps][8 * kTdRow];
  pdl_wait();
  pdl_trigger();  // (what came before is over once the second kernel starts)
  cg::cluster_group cluster = cg::this_cluster();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int C = T == 1 ? 1 : (int)cluster.num_blocks(), rank = T == 1 ? 0 : (int)cluster.block_rank();
  const int row = T == 1 ? blockIdx.x * kTdWarps + warp : blockIdx.x / C;
  if (blockIdx.x == 0) chunk_check(cu, B, n_tokens, err);
  if (T == 1 && row >= n_tokens) return;
  const float* pr = p + (long long)row * V;
  // group g holds weights 4 g - skew .. 4 g - skew + 3
  const int skew = (int)(((uintptr_t)pr & 15) >> 2), groups = (V + skew + 3) >> 2, runs = C * T;
  const int k = ONE ? 1 : (groups + runs * 1024 - 1) / (runs * 1024);
  const int run = (groups + runs - 1) / runs;
  const int g0 = min(groups, (T == 1 ? 0 : rank * T + warp) * run), g1 = min(groups, g0 + run);
  auto load = [&](int g) -> float4 {
    const int i = 4 * g - skew;
    if (g < g1 && i >= 0 && i + 3 < V) return __ldg(reinterpret_cast<const float4*>(pr + i));
    float v[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) v[y] = g < g1 && i + y >= 0 && i + y < V ? __ldg(pr + i + y) : 0.f;
    return make_float4(v[0], v[1], v[2], v[3]);
  };
  float4 x[4];
  // groups j of chunks c .. c + 3
  auto fetch = [&](int c, int j) {
    const int at = g0 + c * 32 * k;
    if (4 * at >= skew && at + 128 * k <= g1 && 4 * (at + 128 * k) - skew <= V) {
      const float4* q = reinterpret_cast<const float4*>(pr - skew) + at + j * 32 + lane;
#pragma unroll
      for (int y = 0; y < 4; ++y) x[y] = __ldg(q + y * k * 32);
    } else {
#pragma unroll
      for (int y = 0; y < 4; ++y) x[y] = load(at + (y * k + j) * 32 + lane);
    }
  };
  fetch(0, 0);
  const float r = __ldg(u + row);
  // a group's sum, exact but for the last addition (an error of 2^-48 of it)
  auto sum4 = [](float4 x) -> Pair {
    const float2 a = make_float2(fmaxf(x.x, 0.f), fmaxf(x.y, 0.f)), b = make_float2(fmaxf(x.z, 0.f), fmaxf(x.w, 0.f));
    const float2 n1 = make_float2(-1.f, -1.f), s = fp_add2(a, b), t = fp_fma2(a, n1, s);  // t = s - a
    const float2 e = fp_add2(fp_fma2(fp_fma2(t, n1, s), n1, a), fp_fma2(t, n1, b));      // (a - (s - t)) + (b - t)
    const Pair c = sum2(s.x, s.y);
    return {c.hi, __fadd_rn(c.lo, __fadd_rn(e.x, e.y))};
  };
  auto take = [](Pair& s, Pair w) {
    const Pair f = sum2(s.hi, w.hi);
    s = {f.hi, __fadd_rn(s.lo, __fadd_rn(f.lo, w.lo))};
  };
  if (chunk_owner(cu, B, row) < 0) return;  // (the whole cluster leaves)
  s_chunk[warp][lane] = {0.f, 0.f};
  __syncwarp();
#pragma unroll 1
  for (int c0 = 0; c0 < 32 && g0 + c0 * 32 * k < g1; c0 += 8) {
    Pair s[8];
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
#pragma unroll
      for (int c = 0; c < 4; ++c) s[h + c] = {0.f, 0.f};
#pragma unroll 1
      for (int j = 0; j < k; ++j) {
        float4 y[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] = x[c];
        if (j + 1 < k) fetch(c0 + h, j + 1);
        else if (c0 + h + 4 < 32) fetch(c0 + h + 4, 0);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (ONE) s[h + c] = sum4(y[c]);
          else take(s[h + c], sum4(y[c]));
        if (ONE) break;
      }
    }
    // four lanes a chunk: eight lanes' sums each, then those of the four
#pragma unroll
    for (int c = 0; c < 8; ++c) s_lane[warp][c * kTdRow + lane] = make_float2(s[c].hi, s[c].lo);
    __syncwarp();
    Pair w = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 f = s_lane[warp][(lane >> 2) * kTdRow + (lane & 3) * 8 + i];
      take(w, Pair{f.x, f.y});
    }
    w = tidy(w.hi, w.lo);
#pragma unroll
    for (int o = 1; o < 4; o <<= 1)
      w = add(w, Pair{__shfl_xor_sync(0xffffffffu, w.hi, o), __shfl_xor_sync(0xffffffffu, w.lo, o)});
    if ((lane & 3) == 0) s_chunk[warp][c0 + (lane >> 2)] = w;
    __syncwarp();
  }
  const Pair chunk = s_chunk[warp][lane], chunks = scan<32>(chunk, lane);
  Pair total = shfl(chunks, 31), before = {0.f, 0.f};
  bool here = true;
  if constexpr (T > 1) {
    if (lane == 31) s_sum[warp] = chunks;
    __syncthreads();
    const Pair mine = s_sum[lane & (kTdWarps - 1)], upto = scan<kTdWarps>(mine, lane);  // within this CTA
    total = shfl(upto, kTdWarps - 1);
    if (C > 1) {
      if (threadIdx.x == 0) s_cta = total;
      cluster.sync();
      const Pair theirs = lane < C ? *cluster.map_shared_rank(&s_cta, lane) : Pair{0.f, 0.f}, all = scan<kTdMaxCTAs>(theirs, lane);
      total = shfl(all, kTdMaxCTAs - 1);
      cluster.barrier_arrive();
      here = holder(all, lane < C ? theirs.hi : 0.f, border_at(total, r)) == rank;
      if (rank) before = shfl(all, rank - 1);
    }
    const Pair to = add(before, upto);
    here = here && holder(to, lane < kTdWarps ? mine.hi : 0.f, border_at(total, r)) == warp;
    if (warp) before = shfl(to, warp - 1);
  }
  const bool drawable = total.hi > 0.f && total.hi < INFINITY;
  if (!drawable && rank == 0 && (T == 1 ? lane : threadIdx.x) == 0) out[row] = -1;
  if (drawable && here) {
    const Border border = border_at(total, r);
    const Pair pu = add(before, chunks);
    const int c = holder(pu, chunk.hi, border);
    Pair at = c ? shfl(pu, c - 1) : before;
    int token = -1;
#pragma unroll 1
    for (int j = 0; j < k; ++j) {  // 32 groups at a time
      const int g = g0 + (c * k + j) * 32 + lane;
      const float4 f4 = load(g);
      Pair w = sum4(f4);
      w = tidy(w.hi, w.lo);
      const Pair wu = add(at, scan<32>(w, lane));
      const int l = holder(wu, w.hi, border);
      if (l >= 0) {  // within a group, by its lane: the first past the border, or the last that counts
        const Pair from = l ? shfl(wu, l - 1) : at;
        if (lane == l) {
          const float v[4] = {f4.x, f4.y, f4.z, f4.w};
          Pair f = from;
          int t = -1;
          bool over = false;
#pragma unroll
          for (int y = 0; y < 4; ++y)
            if (v[y] > 0.f && !over) {
              f = add(f, Pair{v[y], 0.f});
              t = y;
              over = past(f, border);
            }
          token = 4 * g - skew + t;
        }
        token = __shfl_sync(0xffffffffu, token, l);
      }
      if (__any_sync(0xffffffffu, w.hi > 0.f && past(wu, border))) break;
      at = shfl(wu, 31);
    }
    if (lane == 0) out[row] = token;
  }
  if (C > 1) cluster.barrier_wait();  // (a CTA stays until the others have read its sum)
}

// One CTA a sequence, the tree's first rows in shared memory.  A step reads the token drawn
// behind a row, then writes it at the step's own place, which no later step reads: the way
// ascends.
constexpr int kTwThreads = 128, kTwRows = 1024;

__global__ void __launch_bounds__(kTwThreads)
    tree_walk_kernel(bool early, int n_tokens, int B, const int32_t* __restrict__ cu, const int32_t* __restrict__ parent,
                     const int32_t* __restrict__ tokens, int32_t* __restrict__ path, int32_t* out,
                     int32_t* __restrict__ n_out, int32_t* err) {
  __shared__ int s_parent[kTwRows], s_token[kTwRows], s_drawn[kTwRows];
  const int b = blockIdx.x, lane = threadIdx.x & 31;
  int row0, n;
  // the tree, while tokens are drawn: what came before that is over (the drawing kernel lets
  // this one start behind its own wait)
  if (early) {
    chunk_rows(cu, b, n_tokens, &row0, &n);
    for (int i = threadIdx.x; i < min(n, kTwRows); i += kTwThreads)
      s_parent[i] = __ldg(parent + row0 + i), s_token[i] = __ldg(tokens + row0 + i);
  }
  pdl_trigger();
  pdl_wait();
  if (!early) {
    if (b == 0) chunk_check(cu, B, n_tokens, err);
    chunk_rows(cu, b, n_tokens, &row0, &n);
  }
  if (n == 0) {
    if (threadIdx.x == 0) n_out[b] = 0;
    return;
  }
  for (int i = threadIdx.x; i < min(n, kTwRows); i += kTwThreads) s_drawn[i] = out[row0 + i];
  __syncthreads();
  if (threadIdx.x >= 32) return;
  int cur = 0, a = 0;
  for (;; ++a) {
    const int token = cur < kTwRows ? s_drawn[cur] : out[row0 + cur];
    __syncwarp();
    if (lane == 0) path[row0 + a] = cur, out[row0 + a] = token;
    int child = -1;
#pragma unroll 1
    for (int i0 = cur + 1; i0 < n && child < 0 && token >= 0; i0 += 32) {
      const int i = i0 + lane;
      const int up = i >= n ? -1 : i < kTwRows ? s_parent[i] : __ldg(parent + row0 + i);
      const int t = i >= n ? -1 : i < kTwRows ? s_token[i] : __ldg(tokens + row0 + i);
      const unsigned any = __ballot_sync(0xffffffffu, up == cur && t == token);
      if (any) child = i0 + __ffs(any) - 1;
    }
    if (token < 0 && lane == 0 && err) atomicExch(err, 1);
    if (child < 0) {
      if (lane == 0) n_out[b] = token < 0 ? a : a + 1;
      break;
    }
    cur = child;
  }
  for (int i = a + 1 + lane; i < n; i += 32) out[row0 + i] = -1, path[row0 + i] = -1;
}

// Every row's token at once, or one after the other (us): 32 trees of up to 16 rows, 32000
// tokens 14 | 30, 1 of 60, 100003 tokens 13 | 23, 64 of up to 100, 2500 tokens 19 | 54; 32 of up
// to 40, 32000 tokens (30 M weights) 30 | 33, of up to 80 (61 M) 53 | 37.  So up to 2^25 weights.
constexpr long long kTdMost = 1LL << 25;
constexpr int kTdPlaces = 152 * 3;  // CTAs that the GPU holds
// Rows from which a warp takes each (us, a CTA a row | a warp): 4900 rows of 2500 tokens
// 53 | 19, 1400 of 10000 27 | 35, 960 of 32000 30 | 56, 580 of 10000 13 | 18.
constexpr int kTdMany = 2048;

cudaError_t launch_verify_tree(const float* p, int V, int n_tokens, int B, const int32_t* cu, const int32_t* parent,
                               const int32_t* tokens, const float* u, int32_t* path, int32_t* out, int32_t* n_out,
                               int32_t* err, cudaStream_t s) {
  if (B <= 0) return cudaSuccess;
  if ((long long)n_tokens * V > kTdMost)
    return launch_early(verify_tree_kernel, dim3(B * kVfCTAs), dim3(kVfThreads), 0, s, p, V, n_tokens, B, cu, parent, tokens,
                        u, path, out, n_out, err);
  if (n_tokens > 0) {
    const int groups = V / 4 + 2;
    const bool many = n_tokens >= kTdMany;
    int C = 1;
    while (!many && C < kTdMaxCTAs && n_tokens * 2LL * C <= kTdPlaces && V / C >= 8192) C *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(many ? (n_tokens + kTdWarps - 1) / kTdWarps : (unsigned)n_tokens * C);
    cfg.blockDim = dim3(kTdThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = C;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    auto go = [&](auto kern) { return cudaLaunchKernelEx(&cfg, kern, p, V, n_tokens, B, cu, u, out, err); };
    const bool one = groups <= 1024 * (many ? 1 : kTdWarps * C);
    FP_CUDA_TRY(many ? (one ? go(tree_draw_kernel<1, true>) : go(tree_draw_kernel<1, false>))
                     : (one ? go(tree_draw_kernel<kTdWarps, true>) : go(tree_draw_kernel<kTdWarps, false>)));
  }
  return launch_early(tree_walk_kernel, dim3(B), dim3(kTwThreads), 0, s, n_tokens > 0, n_tokens, B, cu, parent, tokens, path, out, n_out,
                      err);
}

}  // namespace fpk
