// Attention of a tree of drafted tokens over the paged cache (attn_chunk.cuh): a row sees
// the cached prefix and, of the rows beside it, those that its mask words name.
#include "attn_chunk.cuh"

namespace fpk {

cudaError_t launch_attention_tree(const uint16_t* q, int q_stride, int n_tokens, int B, int n_heads, const fp_kv_view& kv,
                                  const int32_t* cu, const int32_t* pos, const uint32_t* mask, int mask_stride, int max_new,
                                  int max_len, uint16_t* out, void* ws, int32_t* err, cudaStream_t s) {
  if (n_tokens <= 0 || B <= 0) return cudaSuccess;
  const int G = n_heads / kv.n_kv_heads;
  const CkArgs a = {cu, pos, n_tokens, B, n_heads, kv.n_kv_heads, G, max_new, max_len, ck_tile_tokens(G), mask, mask_stride,
                    kv.page_table, kv.pages_per_seq, kv.n_pages, (const int8_t*)kv.k_pool, (const int8_t*)kv.v_pool,
                    kv.k_scale, kv.v_scale, out, (uint8_t*)ws, err, attention_chunk_wait_limit()};
  return kv.head_dim == 64 ? launch_ck<64, true>(q, q_stride, kv, a, s) : launch_ck<128, true>(q, q_stride, kv, a, s);
}

}  // namespace fpk
