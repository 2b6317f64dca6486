// Chunks of new tokens and the paged cache: RoPE + append of a ragged batch
// (the next piece of each prompt, or drafted tokens), and cached positions read
// back as bf16.  The KV cache and its INT8 variant are a deployment
// configuration (Sec. 2, Sec. 3.2, table "Models and configurations").
#include "chunk.cuh"
#include "kernels.cuh"

namespace fpk {

FP_DEV void unpack8(uint4 v, float* f) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = bf2x2f(w[i]);
    f[2 * i] = p.x;
    f[2 * i + 1] = p.y;
  }
}
FP_DEV uint4 pack8(const float* f) {
  return make_uint4(pack_bf2(f[0], f[1]), pack_bf2(f[2], f[3]), pack_bf2(f[4], f[5]), pack_bf2(f[6], f[7]));
}
// Eight codes q = clamp(rint(x / s)), as fp_op_rope_kv writes them.
FP_DEV uint2 codes8(const float* x, float s) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float r = s > 0.f ? rintf(__fdiv_rn(x[i], s)) : 0.f;
    w[i >> 2] |= ((uint32_t)(int)fminf(fmaxf(r, -127.f), 127.f) & 0xFFu) << (8 * (i & 3));
  }
  return make_uint2(w[0], w[1]);
}

// ------------------------------------------------------------------ RoPE + append
// (a, b) -> (a cos - b sin, b cos + a sin) for the pairs (i, i + hd/2) of the
// query and key heads, in fp32 with one rounding to bf16; keys and values then go
// to their page, an int8 row as q = rint(x / s) with s = max|x| / 127.  One CTA a
// token: HD / 16 lanes hold a head, 16 bytes of each half, so that a rotated pair
// and (by shuffles among those lanes) a row's maximum stay in the warp, and each
// lane reads its cosines once for all heads.  Bound by bytes (qkv in, queries and
// cache rows out) for many rows, by latency for few: with the read back below, chunks of
// 4 x up to 1000 rows of 40 heads take 63 us (5.5 TB/s), 160 rows of 64 heads on 8, int8, 6.6.
// Four CTAs an SM, for the loads in flight: 64 registers, a few of 74 spilled (three: 68 us,
// five: 71).
// TREE: a row's place in the cache is pos[b] + i, what it is rotated by pos[b] + depth[row].
// 32 trees of up to 16 rows (391), 64 heads on 8, int8, 7.3 us; 8 of up to 64 (380), 40 heads, bf16
// 6.7, where their bytes take about 3: three chains of loads (sequence, position and depth, page and
// cosines) one behind the other, then three or four turns over the heads, each of which waits
// for loads that went out a turn before.
template <int HD, bool KV8, bool TREE>
__global__ void __launch_bounds__(256, 4)
    rope_kv_chunk_kernel(const uint16_t* qkv, int row_stride, int n_tokens, int B, int H, fp_kv_view kv,
                         const int32_t* __restrict__ cu, const int32_t* __restrict__ pos,
                         const int32_t* __restrict__ depth, const float* __restrict__ cs, uint16_t* q_out, int q_out_stride, int32_t* err) {
  pdl_trigger();
  pdl_wait();
  constexpr int L = HD / 16;  // lanes a head
  const int m = blockIdx.x, c = threadIdx.x % L, Hkv = kv.n_kv_heads, slots = H + 2 * Hkv;
  // the first heads are on their way while the sequence is looked for
  const uint16_t* src = qkv + (long long)m * row_stride + 8 * c;
  const uint16_t* first = src + min((int)threadIdx.x / L, slots - 1) * HD;
  uint4 lo = *reinterpret_cast<const uint4*>(first), hi = *reinterpret_cast<const uint4*>(first + HD / 2);
  if (m == 0) chunk_check(cu, B, n_tokens, err);
  const int b = chunk_owner(cu, B, m);
  if (b < 0) return;
  const long long p = (long long)__ldg(pos + b) + (m - __ldg(cu + b));
  const long long most = (long long)kv.pages_per_seq * kv.page_size;
  const long long at = TREE ? (long long)__ldg(pos + b) + __ldg(depth + m) : p;  // the position it is rotated by
  if (p < 0 || p >= most || (TREE && (at < 0 || at >= most))) {
    if (threadIdx.x == 0 && err) atomicExch(err, 1);
    return;
  }
  const long long row = cache_row(kv, b, p);
  if (row < 0 && threadIdx.x == 0 && err) atomicExch(err, 1);
  float co[8], si[8];
  const float4* t = reinterpret_cast<const float4*>(cs + at * HD + 16 * c);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 f = __ldg(t + i);
    co[2 * i] = f.x, si[2 * i] = f.y, co[2 * i + 1] = f.z, si[2 * i + 1] = f.w;
  }
  // every lane of a warp takes every turn: the shuffles need them all
  for (int s0 = 0; s0 < slots; s0 += 256 / L) {
    const int slot = s0 + threadIdx.x / L;
    const bool on = slot < slots;
    float x[16];
    unpack8(lo, x);
    unpack8(hi, x + 8);
    const uint16_t* sp = src + min(slot + 256 / L, slots - 1) * HD;  // the next turn's
    if (s0 + 256 / L < slots) lo = *reinterpret_cast<const uint4*>(sp), hi = *reinterpret_cast<const uint4*>(sp + HD / 2);
    if (slot < H + Hkv) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float a = x[i], bb = x[i + 8];
        x[i] = bf2f(f2bf(a * co[i] - bb * si[i]));
        x[i + 8] = bf2f(f2bf(bb * co[i] + a * si[i]));
      }
    }
    float amax = 0.f;
    if constexpr (KV8) {
#pragma unroll
      for (int i = 0; i < 16; ++i) amax = fmaxf(amax, fabsf(x[i]));
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    }
    if (!on) continue;
    if (slot < H) {
      uint16_t* d = q_out + (long long)m * q_out_stride + slot * HD + 8 * c;
      *reinterpret_cast<uint4*>(d) = pack8(x);
      *reinterpret_cast<uint4*>(d + HD / 2) = pack8(x + 8);
      continue;
    }
    if (row < 0) continue;
    const bool is_v = slot >= H + Hkv;
    const long long r = row + (long long)(slot - H - (is_v ? Hkv : 0)) * kv.page_size;
    if constexpr (KV8) {
      const float s = __fdiv_rn(amax, 127.f);
      int8_t* d = (int8_t*)(is_v ? kv.v_pool : kv.k_pool) + r * HD + 8 * c;
      *reinterpret_cast<uint2*>(d) = codes8(x, s);
      *reinterpret_cast<uint2*>(d + HD / 2) = codes8(x + 8, s);
      if (c == 0) (is_v ? kv.v_scale : kv.k_scale)[r] = s;
    } else {
      uint16_t* d = (uint16_t*)(is_v ? kv.v_pool : kv.k_pool) + r * HD + 8 * c;
      *reinterpret_cast<uint4*>(d) = pack8(x);
      *reinterpret_cast<uint4*>(d + HD / 2) = pack8(x + 8);
    }
  }
}

template <bool TREE>
static cudaError_t launch_append(const uint16_t* qkv, int row_stride, int n_tokens, int B, int n_heads, const fp_kv_view& kv,
                                 const int32_t* cu, const int32_t* pos, const int32_t* depth, const float* rope_cs,
                                 uint16_t* q_out, int q_out_stride, int32_t* err, cudaStream_t s) {
  if (n_tokens <= 0 || B <= 0) return cudaSuccess;
  auto go = [&](auto kern) {
    return launch_early(kern, dim3(n_tokens), dim3(256), 0, s, qkv, row_stride, n_tokens, B, n_heads, kv, cu, pos, depth,
                        rope_cs, q_out, q_out_stride, err);
  };
  const bool i8 = kv.kvquant == FP_KV_INT8;
  if (kv.head_dim == 64) return i8 ? go(rope_kv_chunk_kernel<64, true, TREE>) : go(rope_kv_chunk_kernel<64, false, TREE>);
  return i8 ? go(rope_kv_chunk_kernel<128, true, TREE>) : go(rope_kv_chunk_kernel<128, false, TREE>);
}

cudaError_t launch_rope_kv_chunk(const uint16_t* qkv, int row_stride, int n_tokens, int B, int n_heads,
                                 const fp_kv_view& kv, const int32_t* cu, const int32_t* pos, const float* rope_cs,
                                 uint16_t* q_out, int q_out_stride, int32_t* err, cudaStream_t s) {
  return launch_append<false>(qkv, row_stride, n_tokens, B, n_heads, kv, cu, pos, nullptr, rope_cs, q_out, q_out_stride,
                              err, s);
}

cudaError_t launch_rope_kv_tree(const uint16_t* qkv, int row_stride, int n_tokens, int B, int n_heads,
                                const fp_kv_view& kv, const int32_t* cu, const int32_t* pos, const int32_t* depth,
                                const float* rope_cs, uint16_t* q_out, int q_out_stride, int32_t* err, cudaStream_t s) {
  return launch_append<true>(qkv, row_stride, n_tokens, B, n_heads, kv, cu, pos, depth, rope_cs, q_out, q_out_stride, err,
                             s);
}

// ------------------------------------------------------------------ read back
// bf16(q s) (bf16 cache: the values) of positions pos[b] + i into row cu[b] + i.
// One CTA a token, 8 elements a thread and turn.  Bound by bytes.
template <int HD, bool KV8>
__global__ void __launch_bounds__(256)
    kv_read_kernel(fp_kv_view kv, int n_tokens, int B, const int32_t* __restrict__ cu, const int32_t* __restrict__ pos,
                   uint16_t* __restrict__ k_out, uint16_t* __restrict__ v_out, int out_stride, int32_t* err) {
  pdl_trigger();
  pdl_wait();
  constexpr int C = HD / 8;  // pieces a head
  const int m = blockIdx.x;
  if (m == 0) chunk_check(cu, B, n_tokens, err);
  const int b = chunk_owner(cu, B, m);
  if (b < 0) return;
  const long long row = cache_row(kv, b, (long long)__ldg(pos + b) + (m - __ldg(cu + b)));
  if (row < 0 && threadIdx.x == 0 && err) atomicExch(err, 1);
  const int half = kv.n_kv_heads * C;
  for (int i = threadIdx.x; i < 2 * half; i += 256) {
    const bool is_v = i >= half;
    const int h = (is_v ? i - half : i) / C, c = i % C;
    uint16_t* d = (is_v ? v_out : k_out) + (long long)m * out_stride + h * HD + 8 * c;
    uint4 o = make_uint4(0, 0, 0, 0);
    if (row >= 0) {
      const long long r = row + (long long)h * kv.page_size;
      if constexpr (KV8) {
        const uint2 w = *reinterpret_cast<const uint2*>((const int8_t*)(is_v ? kv.v_pool : kv.k_pool) + r * HD + 8 * c);
        const float s = (is_v ? kv.v_scale : kv.k_scale)[r];
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)(int8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3))) * s;
        o = pack8(x);
      } else {
        o = *reinterpret_cast<const uint4*>((const uint16_t*)(is_v ? kv.v_pool : kv.k_pool) + r * HD + 8 * c);
      }
    }
    *reinterpret_cast<uint4*>(d) = o;
  }
}

cudaError_t launch_kv_read(const fp_kv_view& kv, int n_tokens, int B, const int32_t* cu, const int32_t* pos,
                           uint16_t* k_out, uint16_t* v_out, int out_stride, int32_t* err, cudaStream_t s) {
  if (n_tokens <= 0 || B <= 0) return cudaSuccess;
  auto go = [&](auto kern) {
    return launch_early(kern, dim3(n_tokens), dim3(256), 0, s, kv, n_tokens, B, cu, pos, k_out, v_out, out_stride, err);
  };
  if (kv.head_dim == 64) return kv.kvquant == FP_KV_INT8 ? go(kv_read_kernel<64, true>) : go(kv_read_kernel<64, false>);
  return kv.kvquant == FP_KV_INT8 ? go(kv_read_kernel<128, true>) : go(kv_read_kernel<128, false>);
}

}  // namespace fpk
