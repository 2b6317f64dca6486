// Ragged batches of new tokens, shared by the chunk kernels (fp_chunk.cu,
// attn_chunk.cuh, fp_tree.cu, fp_verify.cu): sequence b's rows are cu[b] .. cu[b+1]-1 of
// the packed buffers, at positions pos[b] on.  cu and pos live on the device,
// so nothing on the host has seen them: every index taken from them is checked
// here before it is used.
#pragma once

#include "common.cuh"
#include "../../include/fp_ops.h"

namespace fpk {

// Rows of sequence b that lie in the buffers: first and count (0: none).
FP_DEV void chunk_rows(const int32_t* cu, int b, int n_tokens, int* first, int* count) {
  const int lo = __ldg(cu + b), hi = __ldg(cu + b + 1);
  *first = max(lo, 0);
  *count = max(0, min(hi, n_tokens) - *first);
}

// The sequence that owns `row`, or -1: the last b with cu[b] <= row, if its rows
// reach that far (a row behind the last sequence, or between two, has none).  For a
// whole warp, 32 places probed at a time: a search one by one waits for memory five
// times for 32 sequences, this one once.
FP_DEV int chunk_owner(const int32_t* cu, int B, int row) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = B;  // cu[lo - 1] <= row < cu[hi]
#pragma unroll 1
  while (lo < hi) {
    const int step = (hi - lo + 31) >> 5, at = lo + (lane + 1) * step - 1;  // the last of each of 32 pieces
    const int n = __popc(__ballot_sync(0xffffffffu, at < hi && __ldg(cu + min(at, B)) <= row));
    hi = min(hi, lo + (n + 1) * step - 1);
    lo += n * step;
  }
  return lo > 0 && row < __ldg(cu + lo) ? lo - 1 : -1;
}

// Where position p of sequence b lives: the row of head 0 in the pools (heads are
// page_size rows apart), or -1 for a position outside the cache or a bad page.
FP_DEV long long cache_row(const fp_kv_view& kv, int b, long long p) {
  if (p < 0 || p >= (long long)kv.pages_per_seq * kv.page_size) return -1;
  const int page = __ldg(kv.page_table + (long long)b * kv.pages_per_seq + (int)p / kv.page_size);
  if (page < 0 || page >= kv.n_pages) return -1;
  return (long long)page * kv.n_kv_heads * kv.page_size + (int)p % kv.page_size;
}

// A whole block looks cu over: *err = 1 where it decreases or leaves [0, n_tokens].
FP_DEV void chunk_check(const int32_t* cu, int B, int n_tokens, int32_t* err) {
  if (!err) return;
  for (int b = threadIdx.x; b <= B; b += blockDim.x) {
    const int v = __ldg(cu + b);
    if (v < 0 || v > n_tokens || (b > 0 && v < __ldg(cu + b - 1))) atomicExch(err, 1);
  }
}

}  // namespace fpk
