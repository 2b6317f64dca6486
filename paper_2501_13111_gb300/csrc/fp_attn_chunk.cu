// Attention of a chunk of new tokens over the paged cache (attn_chunk.cuh): every row sees
// the keys up to its own position.
#include "attn_chunk.cuh"

namespace fpk {

// The plan's places and a unit's places in the output are 32-bit.
bool attention_chunk_fits(int n_tokens, int B, int n_heads, int n_kv_heads, int head_dim, int max_len) {
  const int T = ck_tile_tokens(n_heads / n_kv_heads);
  return ck_fits(n_tokens, B, max_len, n_kv_heads, T) && 2LL * T * n_heads * head_dim < (1LL << 31);
}

size_t attention_chunk_ws_bytes(int B, int n_heads, int n_kv_heads, int head_dim, int max_new) {
  return kCkHead + (size_t)2 * kCkMaxCtas * (head_dim == 64 ? ck_slot<64>() : ck_slot<128>());
}

// Of the launches that follow (lowered by tests of the failure path; other waits keep
// kTcSpinLimit, so that copies and MMAs in flight are drained).
static std::atomic<long long> g_ck_wait_limit{kTcSpinLimit};
void attention_chunk_wait_limit(long long rounds) { g_ck_wait_limit.store(rounds, std::memory_order_relaxed); }
long long attention_chunk_wait_limit() { return g_ck_wait_limit.load(std::memory_order_relaxed); }

cudaError_t launch_attention_chunk(const uint16_t* q, int q_stride, int n_tokens, int B, int n_heads,
                                   const fp_kv_view& kv, const int32_t* cu, const int32_t* pos, int max_new, int max_len,
                                   uint16_t* out, void* ws, int32_t* err, cudaStream_t s) {
  if (n_tokens <= 0 || B <= 0) return cudaSuccess;
  const int G = n_heads / kv.n_kv_heads;
  const CkArgs a = {cu, pos, n_tokens, B, n_heads, kv.n_kv_heads, G, max_new, max_len, ck_tile_tokens(G), nullptr, 0, kv.page_table,
                    kv.pages_per_seq, kv.n_pages, (const int8_t*)kv.k_pool, (const int8_t*)kv.v_pool, kv.k_scale, kv.v_scale,
                    out, (uint8_t*)ws, err, g_ck_wait_limit.load(std::memory_order_relaxed)};
  return kv.head_dim == 64 ? launch_ck<64, false>(q, q_stride, kv, a, s) : launch_ck<128, false>(q, q_stride, kv, a, s);
}

}  // namespace fpk
