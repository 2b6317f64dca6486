// Trees of drafted tokens: their plan (depths and ancestor masks), and the rows of an
// accepted path moved together in the cache.
#include <algorithm>

#include "chunk.cuh"
#include "kernels.cuh"

namespace fpk {

// ------------------------------------------------------------------ plan
// depth_i = number of ancestors of row i; mask_i = row i and its ancestors, bit j of word
// w for row 32 w + j.  Parents stand before their children, so a way up only descends: a
// thread follows it for one row and one word, from the row to the first ancestor below the
// word's rows.  One CTA a sequence, its parents in shared memory.  Bound by latency: cu,
// parents, the longest way; 32 trees of 16 rows, and 8 of 64, 2.0 to 2.3 us.  Every (row, word)
// goes its whole way, so deep trees cost up to the cube of their rows: a chain of 64 5.2 us, of
// 256 64, of 1024 3460 (a tree of 1024 rows at random 94, a star 48).
constexpr int kTpThreads = 256;

__global__ void __launch_bounds__(kTpThreads)
    tree_plan_kernel(const int32_t* __restrict__ parent, int n_tokens, int B, const int32_t* __restrict__ cu, int max_new,
                     int32_t* __restrict__ depth, uint32_t* __restrict__ mask, int stride, int32_t* err) {
  __shared__ int16_t s_up[FP_TREE_MAX_ROWS];
  pdl_trigger();
  pdl_wait();
  if (blockIdx.x == 0) chunk_check(cu, B, n_tokens, err);
  int row0, n;
  chunk_rows(cu, blockIdx.x, n_tokens, &row0, &n);
  bool bad = n > max_new;
  n = min(n, max_new);
  for (int i = threadIdx.x; i < n; i += kTpThreads) {
    int p = __ldg(parent + row0 + i);
    if (p < -1 || p >= i) p = -1, bad = true;
    s_up[i] = (int16_t)p;
  }
  if (bad && err) atomicExch(err, 1);
  __syncthreads();
  for (int x = threadIdx.x; x < n * stride; x += kTpThreads) {
    const int i = x / stride, w = x - i * stride;
    int j = i, d = 0;
    while (j >= 32 * w + 32) j = s_up[j];
    uint32_t m = 0;
    for (; j >= 32 * w; j = s_up[j]) m |= 1u << (j & 31);
    mask[(long long)row0 * stride + x] = m;
    if (w > 0) continue;
    for (j = s_up[i]; j >= 0; j = s_up[j]) ++d;
    depth[row0 + i] = d;
  }
}

cudaError_t launch_tree_plan(const int32_t* parent, int n_tokens, int B, const int32_t* cu, int max_new, int32_t* depth,
                             uint32_t* mask, int mask_stride, int32_t* err, cudaStream_t s) {
  if (n_tokens <= 0 || B <= 0 || max_new <= 0) return cudaSuccess;
  return launch_early(tree_plan_kernel, dim3(B), dim3(kTpThreads), 0, s, parent, n_tokens, B, cu, max_new, depth, mask,
                mask_stride, err);
}

// ------------------------------------------------------------------ commit
// Position pos + j takes what position pos + path_j holds, in place.  The path ascends
// (path_j >= j), so a row that is written is one that no later step reads: a warp takes a
// (sequence, K or V, head), looks up to 32 rows of the path up, one a lane, and goes down
// them in order, a batch of rows read before it is written.  No other warp touches its
// rows.  Bound by latency: cu, path, pages, rows; 32 paths, 8 int8 heads 3.1 us, 8 paths, 40
// bf16 heads 3.0 us.
constexpr int kCmWarps = 8;

template <int RB>  // bytes of a head's row
__global__ void __launch_bounds__(kCmWarps * 32)
    kv_commit_kernel(fp_kv_view kv, int n_tokens, int B, const int32_t* __restrict__ cu, const int32_t* __restrict__ pos,
                     const int32_t* __restrict__ path, int32_t* err) {
  constexpr int C = RB / 16, R = 32 / C;  // 16-byte pieces a row; rows a warp moves side by side
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (b == 0 && blockIdx.y == 0) chunk_check(cu, B, n_tokens, err);
  for (int item = blockIdx.y * kCmWarps + warp; item < 2 * kv.n_kv_heads; item += gridDim.y * kCmWarps) {
    const bool is_v = item >= kv.n_kv_heads;
    const int h = is_v ? item - kv.n_kv_heads : item;
    int row0, n;
    chunk_rows(cu, b, n_tokens, &row0, &n);
    uint8_t* pool = (uint8_t*)(is_v ? kv.v_pool : kv.k_pool);
    float* scale = kv.kvquant == FP_KV_INT8 ? (is_v ? kv.v_scale : kv.k_scale) : nullptr;
    const long long p0 = __ldg(pos + b);
    int last = -1;  // the path's row before
    for (int j0 = 0; j0 < n; j0 += 32) {
      const int j = j0 + lane;
      const int from = j < n ? __ldg(path + row0 + j) : -1;
      int before = __shfl_up_sync(0xffffffffu, from, 1);
      if (lane == 0) before = last;
      last = __shfl_sync(0xffffffffu, from, 31);
      const unsigned ends = __ballot_sync(0xffffffffu, from == -1),
                     wrong = __ballot_sync(0xffffffffu, from != -1 && (from < 0 || from <= before || from >= n));
      const int count = min(32, min(ends ? __ffs(ends) - 1 : 32, wrong ? __ffs(wrong) - 1 : 32));
      if (wrong && (!ends || __ffs(wrong) < __ffs(ends)) && lane == 0 && err) atomicExch(err, 1);
      // pool rows of head h (-1: no such place)
      long long src = -1, dst = -1;
      if (lane < count && from != j) {
        src = cache_row(kv, b, p0 + from), dst = cache_row(kv, b, p0 + j);
        if (src < 0 || dst < 0) {
          if (err) atomicExch(err, 1);
          src = dst = -1;
        }
      }
      src += (long long)h * kv.page_size, dst += (long long)h * kv.page_size;
      const bool on = lane < count && from != j && dst >= (long long)h * kv.page_size;
      const unsigned move = __ballot_sync(0xffffffffu, on);
      // scales: all 32 read, then written
      if (scale) {
        const float s = on ? scale[src] : 0.f;
        __syncwarp();
        if (on) scale[dst] = s;
      }
      // rows r, r + R, .. of the path a lane: eight in flight
      for (int r0 = 0; r0 < count; r0 += 8 * R) {
        uint4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int r = r0 + k * R + lane / C;
          const long long at = __shfl_sync(0xffffffffu, src, r & 31);
          if (r < count && (move >> (r & 31) & 1)) v[k] = *reinterpret_cast<const uint4*>(pool + at * RB + (lane % C) * 16);
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int r = r0 + k * R + lane / C;
          const long long at = __shfl_sync(0xffffffffu, dst, r & 31);
          if (r < count && (move >> (r & 31) & 1)) *reinterpret_cast<uint4*>(pool + at * RB + (lane % C) * 16) = v[k];
        }
        __syncwarp();
      }
      if (count < 32) break;
    }
  }
}

cudaError_t launch_kv_commit(const fp_kv_view& kv, int n_tokens, int B, const int32_t* cu, const int32_t* pos,
                             const int32_t* path, int32_t* err, cudaStream_t s) {
  if (n_tokens <= 0 || B <= 0) return cudaSuccess;
  const dim3 grid(B, std::min((2 * kv.n_kv_heads + kCmWarps - 1) / kCmWarps, 1024));
  auto go = [&](auto kern) { return launch_early(kern, grid, dim3(kCmWarps * 32), 0, s, kv, n_tokens, B, cu, pos, path, err); };
  const int rb = kv.head_dim * (kv.kvquant == FP_KV_INT8 ? 1 : 2);
  return rb == 64 ? go(kv_commit_kernel<64>) : rb == 128 ? go(kv_commit_kernel<128>) : go(kv_commit_kernel<256>);
}

}  // namespace fpk
