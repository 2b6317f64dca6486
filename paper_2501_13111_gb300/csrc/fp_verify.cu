// Probabilities of the LM head's logits, and the verification of drafted tokens
// against them with given random numbers (speculative decoding).  Both stand
// beside the greedy choice of fp_rows.cu: one cluster of CTAs a row.
#include <cooperative_groups.h>

#include <utility>

#include "chunk.cuh"
#include "kernels.cuh"

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

struct Pair {
  float hi, lo;
};
// a + b, exactly
FP_DEV Pair sum2(float a, float b) {
  const float s = __fadd_rn(a, b), v = __fsub_rn(s, a);
  return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, v)), __fsub_rn(b, v))};
}
// hi + lo with hi the nearer fp32 (|hi| >= |lo|)
FP_DEV Pair tidy(float hi, float lo) {
  const float s = __fadd_rn(hi, lo);
  return {s, __fsub_rn(lo, __fsub_rn(s, hi))};
}
FP_DEV Pair add(Pair a, Pair b) {
  const Pair s = sum2(a.hi, b.hi);
  return tidy(s.hi, __fadd_rn(s.lo, __fadd_rn(a.lo, b.lo)));
}
FP_DEV Pair times(Pair a, float r) {
  const float h = __fmul_rn(a.hi, r);
  return tidy(h, __fmaf_rn(a.lo, r, __fmaf_rn(a.hi, r, -h)));
}
FP_DEV bool greater(Pair a, Pair b) {
  const Pair d = sum2(a.hi, -b.hi);
  return __fadd_rn(d.hi, __fadd_rn(d.lo, __fsub_rn(a.lo, b.lo))) > 0.f;
}
FP_DEV Pair shfl(Pair v, int l) { return {__shfl_sync(0xffffffffu, v.hi, l), __shfl_sync(0xffffffffu, v.lo, l)}; }

// Inclusive sums over groups of N lanes, lower lanes first.
template <int N>
FP_DEV Pair scan(Pair v, int lane) {
#pragma unroll
  for (int o = 1; o < N; o <<= 1) {
    const Pair f = {__shfl_up_sync(0xffffffffu, v.hi, o, N), __shfl_up_sync(0xffffffffu, v.lo, o, N)};
    if ((lane & (N - 1)) >= o) v = add(f, v);
  }
  return v;
}

// Of the lanes whose weight counts, the first whose sum is past the border; rounding at
// the very end, an r of 1 or more or a NaN leaves none: the last then.  -1: no weight at all.
FP_DEV int holder(Pair upto, float w, Pair border) {
  const unsigned has = __ballot_sync(0xffffffffu, w > 0.f), past = __ballot_sync(0xffffffffu, w > 0.f && greater(upto, border));
  return past ? __ffs(past) - 1 : 31 - __clz(has);
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
      const Pair border = times(total, rb);
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
            if (__any_sync(0xffffffffu, w.hi > 0.f && greater(wu, border))) break;
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

}  // namespace fpk
