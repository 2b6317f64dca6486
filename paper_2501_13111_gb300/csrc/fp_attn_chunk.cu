// Attention of a chunk of new tokens over the paged cache: row i of sequence b
// (position pos[b] + i) attends over positions 0 .. pos[b] + i,
// o = softmax(q K^T / sqrt(hd)) V.
//
// One warp a (token, query head), one key at a time with a running maximum and
// sum: the plain sum, right for every shape, each cached key read by every row.
#include "chunk.cuh"
#include "kernels.cuh"

namespace fpk {

template <int HD, bool KV8>
__global__ void __launch_bounds__(256)
    attn_chunk_rows_kernel(const uint16_t* __restrict__ q, int q_stride, int n_tokens, int B, int H, fp_kv_view kv,
                           const int32_t* __restrict__ cu, const int32_t* __restrict__ pos, int max_new, int max_len,
                           uint16_t* __restrict__ out, int32_t* err) {
  pdl_trigger();
  pdl_wait();
  constexpr int E = HD / 32;
  if (blockIdx.x == 0) chunk_check(cu, B, n_tokens, err);
  const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (w >= (long long)n_tokens * H) return;
  const int m = (int)(w / H), h = (int)(w % H);
  const int b = chunk_owner(cu, B, m);
  if (b < 0) return;
  if (m - __ldg(cu + b) >= max_new) {
    if (lane == 0 && err) atomicExch(err, 1);
    return;
  }
  long long n = (long long)__ldg(pos + b) + (m - __ldg(cu + b)) + 1;  // keys of this row
  if ((n < 1 || n > max_len) && lane == 0 && err) atomicExch(err, 1);
  n = n > max_len ? max_len : n;
  const int Hkv = kv.n_kv_heads, kvh = h / (H / Hkv);
  float x[E], o[E];
#pragma unroll
  for (int j = 0; j < E; ++j) {
    x[j] = bf2f(q[(long long)m * q_stride + h * HD + lane + 32 * j]) * rsqrtf((float)HD);
    o[j] = 0.f;
  }
  float mx = -INFINITY, l = 0.f;
  for (int key = 0; key < (int)n; ++key) {
    const int page = __ldg(kv.page_table + (long long)b * kv.pages_per_seq + key / kv.page_size);
    const bool ok = page >= 0 && page < kv.n_pages;
    if (!ok && lane == 0 && err) atomicExch(err, 1);
    const long long r = ((long long)(ok ? page : 0) * Hkv + kvh) * kv.page_size + key % kv.page_size;
    float kf[E], vf[E];
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const long long a = r * HD + lane + 32 * j;
      if constexpr (KV8) {  // as fp_op_kv_read returns them
        kf[j] = bf2f(f2bf((float)((const int8_t*)kv.k_pool)[a] * kv.k_scale[r]));
        vf[j] = bf2f(f2bf((float)((const int8_t*)kv.v_pool)[a] * kv.v_scale[r]));
      } else {
        kf[j] = bf2f(((const uint16_t*)kv.k_pool)[a]);
        vf[j] = bf2f(((const uint16_t*)kv.v_pool)[a]);
      }
      if (!ok) kf[j] = vf[j] = 0.f;
    }
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < E; ++j) s += x[j] * kf[j];
    s = warp_sum(s);
    const float m2 = fmaxf(mx, s), a = expf(mx - m2), pr = expf(s - m2);
    mx = m2;
    l = l * a + pr;
#pragma unroll
    for (int j = 0; j < E; ++j) o[j] = o[j] * a + pr * vf[j];
  }
  const float inv = n > 0 ? 1.f / l : 0.f;
#pragma unroll
  for (int j = 0; j < E; ++j) out[((long long)m * H + h) * HD + lane + 32 * j] = f2bf(o[j] * inv);
}

size_t attention_chunk_ws_bytes(int B, int n_heads, int n_kv_heads, int head_dim, int max_new) { return 256; }

cudaError_t launch_attention_chunk(const uint16_t* q, int q_stride, int n_tokens, int B, int n_heads,
                                   const fp_kv_view& kv, const int32_t* cu, const int32_t* pos, int max_new, int max_len,
                                   uint16_t* out, void* ws, int32_t* err, cudaStream_t s) {
  if (n_tokens <= 0 || B <= 0) return cudaSuccess;
  const unsigned blocks = (unsigned)(((long long)n_tokens * n_heads + 7) / 8);
  auto go = [&](auto kern) {
    return launch(kern, dim3(blocks), dim3(256), 0, s, q, q_stride, n_tokens, B, n_heads, kv, cu, pos, max_new, max_len,
                  out, err);
  };
  if (kv.head_dim == 64)
    return kv.kvquant == FP_KV_INT8 ? go(attn_chunk_rows_kernel<64, true>) : go(attn_chunk_rows_kernel<64, false>);
  return kv.kvquant == FP_KV_INT8 ? go(attn_chunk_rows_kernel<128, true>) : go(attn_chunk_rows_kernel<128, false>);
}

}  // namespace fpk
