// Probabilities of the LM head's logits, and the verification of drafted tokens
// against them with given random numbers (speculative decoding).  Both stand
// beside the greedy choice of fp_rows.cu: one cluster of CTAs a row.
#include <cooperative_groups.h>

#include "chunk.cuh"
#include "kernels.cuh"

namespace cg = cooperative_groups;

namespace fpk {

// ------------------------------------------------------------------ softmax
// y_i = exp((x_i - max x) / T) / sum_j exp((x_j - max x) / T), T the row's
// temperature; T = 0: 1 at the lowest index of the maximum, else 0.
constexpr int kSmThreads = 512;

FP_DEV float sm_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The block's sum, maximum or minimum of v (every thread gets it); red: 16 words.
template <typename T, typename F>
FP_DEV T block_all(T v, T* red, F f) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[threadIdx.x & 15];
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// The plain form: one CTA a row, three passes over it.
__global__ void __launch_bounds__(kSmThreads)
    softmax_kernel(const float* __restrict__ x, int V, const float* __restrict__ temp, float* __restrict__ y,
                   int32_t* err) {
  __shared__ float red[16];
  __shared__ int redi[16];
  pdl_trigger();
  pdl_wait();
  const long long base = (long long)blockIdx.x * V;
  const float t = temp ? temp[blockIdx.x] : 1.f;
  const bool bad = !(t >= 0.f) || isinf(t);
  if (bad && threadIdx.x == 0 && err) atomicExch(err, 1);
  float mx = -INFINITY;
  for (int i = threadIdx.x; i < V; i += kSmThreads) mx = fmaxf(mx, x[base + i]);
  mx = block_all(mx, red, [](float a, float b) { return fmaxf(a, b); });
  if (bad || mx == -INFINITY) {
    for (int i = threadIdx.x; i < V; i += kSmThreads) y[base + i] = 0.f;
    return;
  }
  if (t == 0.f) {
    int at = 0x7fffffff;
    for (int i = threadIdx.x; i < V; i += kSmThreads)
      if (x[base + i] == mx) at = min(at, i);
    at = block_all(at, redi, [](int a, int b) { return min(a, b); });
    for (int i = threadIdx.x; i < V; i += kSmThreads) y[base + i] = i == at ? 1.f : 0.f;
    return;
  }
  const float c = fminf(1.4426950408889634f / t, 3.4e38f);
  float s = 0.f;
  for (int i = threadIdx.x; i < V; i += kSmThreads) s += sm_ex2((x[base + i] - mx) * c);
  s = block_all(s, red, [](float a, float b) { return a + b; });
  for (int i = threadIdx.x; i < V; i += kSmThreads) y[base + i] = sm_ex2((x[base + i] - mx) * c) / s;
}

cudaError_t launch_softmax(const float* logits, int M, int V, const float* temp, float* probs, int32_t* err,
                           cudaStream_t s) {
  if (M <= 0) return cudaSuccess;
  return launch(softmax_kernel, dim3(M), dim3(kSmThreads), 0, s, logits, V, temp, probs, err);
}

// ------------------------------------------------------------------ verification
// Sequence b's rows are its last accepted token and the k drafted after it.  Row
// i's draft t (the token of row i + 1) is accepted while u_i q_i(t) < p_i(t)
// (products of two fp32 in fp64: exact); a is the first refused row, or k.  The
// token after it is drawn from w = max(0, p_a - q_a) (a < k), or p_k: the lowest t
// with sum_{s <= t} w_s > r sum w.
// A border is a sum of up to V fp32 values and has to fall where fp64 puts it, but
// fp64 adds are rare here (2 lanes a cycle and SM against 128): each weight is kept
// as d + e (the exact difference, two fp32), each lane's sum as s + c with the
// error of every addition carried along, good to about 2^-46; only the lanes' sums
// are joined in fp64.  A cluster of 8 CTAs a sequence: every warp sums a run of
// consecutive weights, the 128 sums meet through distributed shared memory, and
// the warp whose run holds the border looks through it again (from L2).
constexpr int kVfCTAs = 8, kVfThreads = 512, kVfWarps = kVfThreads / 32, kVfRuns = kVfCTAs * kVfWarps;

struct Pair {  // hi + lo
  float hi, lo;
};
// a - b, exactly
FP_DEV Pair diff2(float a, float b) {
  const float d = __fsub_rn(a, b), v = __fsub_rn(d, a);
  return {d, __fsub_rn(__fsub_rn(a, __fsub_rn(d, v)), __fadd_rn(b, v))};
}
// s += w, the addition's error to s.lo
FP_DEV void add2(Pair& s, Pair w) {
  const float t = __fadd_rn(s.hi, w.hi), v = __fsub_rn(t, s.hi);
  const float e = __fadd_rn(__fsub_rn(s.hi, __fsub_rn(t, v)), __fsub_rn(w.hi, v));
  s.hi = t;
  s.lo = __fadd_rn(s.lo, __fadd_rn(e, w.lo));
}
FP_DEV double value(Pair p) { return (double)p.hi + (double)p.lo; }

FP_DEV double warp_sum_d(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Inclusive sums over the lanes.
FP_DEV double scan_d(double v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double f = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += f;
  }
  return v;
}

// The weight of token t: p, less q where there is one, without token `gone`; none below zero.
FP_DEV Pair weight(const float* p, const float* q, int t, int gone) {
  Pair w = q ? diff2(__ldg(p + t), __ldg(q + t)) : Pair{__ldg(p + t), 0.f};
  if (!(w.hi > 0.f) || t == gone) w = {0.f, 0.f};
  return w;
}

__global__ void __cluster_dims__(kVfCTAs, 1, 1) __launch_bounds__(kVfThreads)
    verify_kernel(const float* __restrict__ p, const float* __restrict__ q, int V, int n_tokens, int B,
                  const int32_t* __restrict__ cu, const int32_t* __restrict__ tokens, const float* __restrict__ u,
                  const float* __restrict__ r, int32_t* __restrict__ out, int32_t* __restrict__ n_out, int32_t* err) {
  __shared__ double s_sum[kVfWarps];
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
    for (int i0 = 0; i0 < n - 1; i0 += 32) {
      const int i = i0 + lane;
      bool refused = false;
      if (i < n - 1) {
        const int t = __ldg(tokens + row0 + i + 1);
        const bool ok = t >= 0 && t < V;
        if (!ok && rank == 0 && err) atomicExch(err, 1);
        const long long at = (long long)(row0 + i) * V + (ok ? t : 0);
        refused = !ok || !((double)__ldg(u + row0 + i) * (q ? (double)__ldg(q + at) : 1.0) < (double)__ldg(p + at));
      }
      const unsigned any = __ballot_sync(0xffffffffu, refused);
      if (any) {
        a = i0 + __ffs(any) - 1;
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
  const int lo = min((long long)V, (long long)(rank * kVfWarps + warp) * run), hi = min(V, lo + run);
  for (int turn = 0; turn < 2; ++turn) {
    Pair s = {0.f, 0.f};
#pragma unroll 8
    for (int t = lo + lane; t < hi; t += 32) add2(s, weight(pr, qr, t, gone));
    const double mine = warp_sum_d(value(s));
    if (lane == 0) s_sum[warp] = mine;
    cluster.sync();
    // Every warp, in one order: the runs' sums and what is before each of them.
    constexpr int R = kVfRuns / 32;
    double v[R], upto[R], all = 0.;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int k = lane * R + j;
      v[j] = cluster.map_shared_rank(s_sum, k / kVfWarps)[k % kVfWarps];
      all += v[j];
    }
    all = scan_d(all, lane);
    const double total = __shfl_sync(0xffffffffu, all, 31);
    double before = __shfl_up_sync(0xffffffffu, all, 1);
    if (lane == 0) before = 0.;
    cluster.sync();  // the sums have been read
    if (!(total > 0.) || !(total < (double)INFINITY)) {
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
    // the run that holds the border: the first that reaches past it (r >= 1 or
    // NaN: none; then the last that holds a weight)
    const double border = (double)__ldg(r + b) * total;
    int first = kVfRuns, last = -1;
    double from = 0.;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      upto[j] = before + v[j];
      if (v[j] > 0.) {
        last = lane * R + j;
        if (first == kVfRuns && upto[j] > border) first = lane * R + j;
      }
      if (lane * R + j == rank * kVfWarps + warp) from = before;
      before = upto[j];
    }
    first = __reduce_min_sync(0xffffffffu, first);
    last = __reduce_max_sync(0xffffffffu, last);
    if (first == kVfRuns) first = last;
    from = __shfl_sync(0xffffffffu, from, (rank * kVfWarps + warp) / R);
    if (first != rank * kVfWarps + warp) break;
    // within the run: 32 pieces, then the tokens of the piece
    const int seg = (hi - lo + 31) / 32;
    Pair ps = {0.f, 0.f};
    for (int t = lo + lane * seg; t < min(hi, lo + (lane + 1) * seg); ++t) add2(ps, weight(pr, qr, t, gone));
    const double pv = value(ps), pu = from + scan_d(pv, lane);
    unsigned has = __ballot_sync(0xffffffffu, pv > 0.), past = __ballot_sync(0xffffffffu, pv > 0. && pu > border);
    const int piece = past ? __ffs(past) - 1 : 31 - __clz(has);
    double at = __shfl_sync(0xffffffffu, pu - pv, piece);
    int token = -1;
    const int t1 = min(hi, lo + (piece + 1) * seg);
    for (int t0 = lo + piece * seg; t0 < t1; t0 += 32) {
      const double w = t0 + lane < t1 ? value(weight(pr, qr, t0 + lane, gone)) : 0.;
      const double wu = at + scan_d(w, lane);
      has = __ballot_sync(0xffffffffu, w > 0.);
      past = __ballot_sync(0xffffffffu, w > 0. && wu > border);
      if (past || has) token = t0 + (past ? __ffs(past) - 1 : 31 - __clz(has));
      if (past) break;
      at = __shfl_sync(0xffffffffu, wu, 31);
    }
    if (lane == 0) {
      out[row0 + a] = token;
      n_out[b] = a + 1;
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
