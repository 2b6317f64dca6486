// Attention of a chunk of new tokens over the paged cache, on the tcgen05 tensor
// cores: row i of sequence b (position pos[b] + i) attends over positions
// 0 .. pos[b] + i, o = softmax(q K^T / sqrt(hd)) V, for ragged chunks of one token to
// thousands (chunked prefill, drafted tokens, decoding, mixed).
//
// One persistent CTA per SM takes an equal stretch of the line of units that
// chunk_items.h lays out: tiles of 128 packed rows (the heads of a KV head's group
// side by side) against tiles of 128 keys.  A unit of two tiles shares every key
// tile between them; a unit of one has its key tiles taken in turn by the two
// softmax groups, each with its own maximum, sum and accumulator, added at the end.
// Tensor memory: the scores of each group (128 columns, P over them as bf16 pairs)
// and its output accumulator.
//   warps 0-15  softmax, two groups of 8: a thread has one query row (TMEM lane) and
//               half of the tile's keys; the two halves of a row meet over their
//               maximum in shared memory.  P = 2^(s - m) is rounded to bf16 for the
//               second product (2^-8 of each p, the sums in fp32); the reference m
//               moves only when a tile passes it by 2^8 (O and the row sum are
//               rescaled then).  At the end of a unit they write its rows;
//   warp 16     TMA: the unit's Q tiles (one box per 64 columns: tokens x heads) and,
//               page by page, the keys; warp 18 the values.  One box a page, in the
//               order [8 rows][64 columns] the descriptors step through;
//   warp 17     owns the TMEM and issues the MMAs: O += P(t) V(t), then the group's
//               next scores over the columns that P(t) has left;
//   warps 20-23 (int8 cache) K and V tiles from the codes: bf16(q s), the values that
//               fp_op_kv_read returns (a byte permute gives fp32 2^15 + 128 + q, an exact
//               subtraction q; 2^-8 of a value, as a bf16 cache's own rounding).
// Slots behind the sequence's last position may hold anything: their scores are
// masked, their V rows are zeroed before the product.
// Every wait on an mbarrier is bounded (error 2 past the limit).
#include <algorithm>

#include "attn_tc.cuh"
#include "chunk.cuh"
#include "chunk_items.h"
#include "kernels.cuh"

namespace fpk {

constexpr int kCkSoft = 16;                       // softmax warps
constexpr int kCkWarpQ = 16, kCkWarpMma = 17, kCkWarpV = 18, kCkWarpWiden = 20;
template <bool KV8>
constexpr int ck_threads() { return KV8 ? 768 : 640; }
// Registers, moved to the softmax: 640 threads launch with 96, 512 x 104 + 128 x 64 =
// 640 x 96; 768 (int8 cache) with 80, 512 x 88 + 256 x 64 = 768 x 80
constexpr int kCkRing = 2;                        // K tiles in shared memory, and V tiles
constexpr uint32_t kCkTmemCols = 512, kCkO = 256; // O of group j at kCkO + 128 j, its scores at 128 j
constexpr int kCkStage = 32 * 32;                 // a warp's 32 output rows, 16 columns at a time
constexpr float kCkSlack = 8.f;                   // log2 of the largest P before the reference moves
constexpr int kCkRows = 256;                      // rows of a unit
template <int HD>
constexpr int ck_tile_bytes() { return kCkKeys * HD * 2; }
template <int HD>
constexpr int ck_smem() { return (2 + 2 * kCkRing) * ck_tile_bytes<HD>() + kCkSoft * kCkStage + 1024; }

// Workspace: per CTA where its stretch begins, which unit it began and left
// unfinished, and two partial results (slot 0: of a unit begun by an earlier CTA,
// slot 1: of the one it left): fp32 O as [HD / 4][256 rows][4], then (m, l) [256 rows].
struct CkLeft {
  long long end;  // the unit's end on the line; 0: none was left
  int row0, i0, n, kvh, pair;
};
constexpr size_t kCkHead = 64 * 1024;  // begins and CkLeft of up to 1024 CTAs
template <int HD>
constexpr size_t ck_slot() { return (size_t)kCkRows * (HD * 4 + 8); }

// [8 rows][64 columns] atoms: 8-row groups `sbo` bytes apart, K-major.
FP_DEV uint64_t ck_sdesc_k(uint32_t saddr, uint32_t sbo) {
  return (uint64_t)((saddr & 0x3FFFF) >> 4) | (uint64_t)1 << 16 | (uint64_t)(sbo >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;
}
// The same atoms MN-major: 64 columns on `lbo` bytes, 8-row groups along K `sbo`.
FP_DEV uint64_t ck_sdesc_mn(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
  return (uint64_t)((saddr & 0x3FFFF) >> 4) | (uint64_t)(lbo >> 4) << 16 | (uint64_t)(sbo >> 4) << 32 |
         (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
FP_DEV void ck_tma_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
      : "memory");
}
FP_DEV float2 ck_fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n .reg .b64 a, b, c, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n"
      " fma.rn.f32x2 d, a, b, c;\n mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
FP_DEV float2 ck_add2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n"
      " add.rn.f32x2 d, a, b;\n mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

FP_DEV float2 ck_mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n"
      " mul.rn.f32x2 d, a, b;\n mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

struct CkArgs {
  const int32_t *cu, *pos;
  int n_tokens, B, H, Hkv, G, max_new, max_len;
  int tile_tokens;
  const int32_t* page_table;
  int pages_per_seq, n_pages;
  const int8_t *k8, *v8;
  const float *k_scale, *v_scale;
  uint16_t* out;
  uint8_t* ws;
  int32_t* err;
};

// A place on the line: unit u of KV head kvh of sequence b, `off` places into it.
struct CkAt {
  int b, kvh, u, off;
  long long x;  // its place on the line
};

// The pieces of units that a stretch of `len` places from `at` takes.
struct CkWalk {
  const CkArgs& a;
  CkSeq s;
  int b, kvh, u, off;
  long long x, rem;
  // the present piece: unit u of (b, kvh), key tiles t0 .. t1-1 of nt (0: no keys)
  int t0, t1, nt, nt0, i0;
  bool pair, first, last;  // two tiles; the unit's first / last part
  FP_DEV CkWalk(const CkArgs& a, const CkAt& at, long long len)
      : a(a), b(at.b), kvh(at.kvh), u(at.u), off(at.off), x(at.x), rem(at.b < a.B ? len : 0) {
    if (rem > 0) {
      load();
      skip();
    }
  }
  // on to a sequence that has rows (there is one while places are left)
  FP_DEV void skip() {
    while (s.units == 0 && rem > 0)
      if (b + 1 < a.B) ++b, load();
      else rem = 0;
  }
  FP_DEV void load() {
    int first, count;
    chunk_rows(a.cu, b, a.n_tokens, &first, &count);
    s.set(first, count, __ldg(a.pos + b), a.tile_tokens, a.max_new, a.max_len);
  }
  FP_DEV bool next() {
    if (rem <= 0) return false;
    const int T = 2 * a.tile_tokens;
    nt = s.tiles(u, T);
    i0 = u * T;
    pair = s.n - i0 > a.tile_tokens;
    // the first tile's own last key tile
    nt0 = s.bad || !pair ? nt : (s.pos + i0 + a.tile_tokens + kCkKeys - 1) / kCkKeys;
    const long long left = kCkStart + nt - off;
    const int take = (int)(left < rem ? left : rem);
    t0 = max(0, off - kCkStart);
    t1 = min(nt, max(0, off + take - kCkStart));
    first = off == 0;
    last = take == left;
    ub = b, ukvh = kvh, us = s, ux = x - off;
    rem -= take;
    x += take;
    off = 0;
    if (rem > 0 && ++u == s.units) {
      u = 0;
      if (++kvh == a.Hkv) {
        kvh = 0;
        s.units = 0;
        skip();
      }
    }
    return true;
  }
  // of the present piece (b, kvh, u, s are the next one's)
  int ub, ukvh;
  CkSeq us;
  long long ux;  // where its unit begins
  FP_DEV bool uses(int j) const { return pair ? (j ? true : t0 < nt0) && t1 > t0 : t1 - t0 > j; }
  FP_DEV int end_of(int j) const { return pair && j == 0 ? min(t1, nt0) : t1; }
};

template <int HD, bool KV8>
__global__ void __launch_bounds__(ck_threads<KV8>(), 1)
    attn_chunk_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CkArgs a) {
  constexpr int TILE = ck_tile_bytes<HD>(), NH = HD / 64, SBO = NH * 1024, PAGE = 2 * SBO, R = kCkRing;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ uint64_t qfull, qempty, kfull[R], kempty[R], vfull[R], vempty[R], sfull[2], pfull[2], ofull[2], oempty[2],
      xch[2][4], met[4], mma_done;
  __shared__ float s_x[2][2][2][kCkKeys];        // [group][parity][half][row]: what the halves of a row exchange
  __shared__ float2 s_ml[2][2][2][kCkKeys];      // [parity][group][half][row]: maximum and sum, units of one tile
  __shared__ uint32_t tmem_base;
  __shared__ int abort_word;
  __shared__ CkAt s_at[2];                       // where this CTA's stretch begins, and the next one's
  __shared__ long long s_scan[32];
  volatile int* abort_flag = &abort_word;
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* sQ = smem;
  uint8_t* sK = smem + 2 * TILE;
  uint8_t* sV = sK + R * TILE;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int NT = ck_threads<KV8>(), NW = NT / 32;
  auto fail = [&]() {
    *abort_flag = 1;
    if (a.err) atomicExch(a.err, 2);
  };

  pdl_trigger();
  if (threadIdx.x == 0) {
    mbar_init(&qfull, 1);
    mbar_init(&qempty, 1);
    for (int i = 0; i < R; ++i) {
      mbar_init(&kfull[i], KV8 ? 4 : 1);
      mbar_init(&kempty[i], 1);
      mbar_init(&vfull[i], KV8 ? 4 : 1);
      mbar_init(&vempty[i], 1);
    }
    for (int j = 0; j < 2; ++j) {
      mbar_init(&sfull[j], 1);
      mbar_init(&pfull[j], 8);
      mbar_init(&ofull[j], 1);
      mbar_init(&oempty[j], 16);
      for (int i = 0; i < 4; ++i) mbar_init(&xch[j][i], 2);
    }
    for (int i = 0; i < 4; ++i) mbar_init(&met[i], 4);
    mbar_init(&mma_done, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kCkWarpMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)),
                 "r"(kCkTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();

  // ---------------- the line: its length, and where this CTA's stretch begins and ends.
  // Two passes over the sequences, the first for the sum (a batch of up to NT
  // sequences has its costs in registers by then).
  {
    if (blockIdx.x == 0) chunk_check(a.cu, a.B, a.n_tokens, a.err);
    const int T = 2 * a.tile_tokens;
    auto cost = [&](int b, CkSeq& s) -> long long {
      int first, count;
      chunk_rows(a.cu, b, a.n_tokens, &first, &count);
      const bool fine = s.set(first, count, __ldg(a.pos + b), a.tile_tokens, a.max_new, a.max_len);
      if (!fine && a.err && blockIdx.x == 0) atomicExch(a.err, 1);
      return s.cost(T) * a.Hkv;
    };
    // inclusive sum over the block of one value a thread, and the block's total
    auto scan = [&](long long v, long long* total) {
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long f = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += f;
      }
      __syncthreads();  // s_scan of the last call has been read
      if (lane == 31) s_scan[warp] = v;
      __syncthreads();
      long long before = 0, all = 0;
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        const long long w = s_scan[i];
        before += i < warp ? w : 0;
        all += w;
      }
      *total = all;
      return v + before;
    };
    CkSeq s;
    long long W = 0, mine = 0, incl = 0;
    for (int b0 = 0; b0 < a.B; b0 += NT) {
      const int b = b0 + (int)threadIdx.x;
      mine = b < a.B ? cost(b, s) : 0;
      long long all;
      incl = scan(mine, &all);
      W += all;
    }
    const int g = ck_ctas(W, gridDim.x);
    const int c = blockIdx.x;
    if (threadIdx.x < 2) {  // nothing here, or the line's end
      s_at[threadIdx.x] = {a.B, 0, 0, 0, W};
    }
    __syncthreads();
    long long base = 0;
    for (int b0 = 0; b0 < a.B; b0 += NT) {
      const int b = b0 + (int)threadIdx.x;
      if (a.B > NT) {
        mine = b < a.B ? cost(b, s) : 0;
        long long all;
        incl = base + scan(mine, &all);
        base += all;
      }
      const long long before = incl - mine;
#pragma unroll 1
      for (int e = 0; e < 2; ++e) {
        const int k = c + e;
        if (k >= g) continue;  // the end
        const long long x = W * k / g;
        if (mine == 0 || x < before || x >= incl) continue;
        const long long per = mine / a.Hkv, in = (x - before) % per;
        const int kvh = (int)((x - before) / per), u = s.unit_at(in, T), nt = s.tiles(u, T);
        const long long start = s.before(u, T);
        const int off = ck_snap((int)(in - start), nt);
        CkAt at = {b, kvh, u, off, before + kvh * per + start + off};
        if (off == kCkStart + nt) {  // behind the unit: the next one's beginning
          at.off = 0;
          if (++at.u == s.units) {
            at.u = 0;
            if (++at.kvh == a.Hkv) at.kvh = 0, ++at.b;
          }
        }
        s_at[e] = at;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;
  const CkAt at = s_at[0];
  const long long len = s_at[1].x - at.x;
  if (threadIdx.x == 0) {
    reinterpret_cast<long long*>(a.ws)[blockIdx.x] = at.x;
    reinterpret_cast<CkLeft*>(a.ws + kCkHead / 4)[blockIdx.x].end = 0;
  }

  if (warp >= kCkSoft) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(64));
  }
  if (warp == kCkWarpQ || (warp == kCkWarpV && !KV8)) {
    // ---------------- TMA: warp 16 the Q tiles (and K), warp 18 V.  Lanes 0-7 copy a
    // page of a key tile each; the next tile's page ids are read while this one is in
    // flight.  A page behind the sequence's end, or a bad one, reads zeros.
    const bool is_v = warp == kCkWarpV;
    const CUtensorMap* map = is_v ? &map_v : &map_k;
    uint64_t *full = is_v ? vfull : kfull, *empty = is_v ? vempty : kempty;
    uint8_t* dst = is_v ? sV : sK;
    if (lane == 0) {
      if (!is_v) asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
      if (!KV8) asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
    }
    int n = 0, kn = 0;
    bool ok = true;
    CkWalk w(a, at, len);
    while (ok && w.next()) {
      if (w.t1 <= w.t0) continue;
      if (!is_v) {
        if (n > 0) ok = __all_sync(0xffffffffu, mbar_wait(&qempty, (n - 1) & 1)) && !*abort_flag;
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          break;
        }
        if (lane == 0) {
          const int tiles = w.pair ? 2 : 1;
          mbar_expect_tx(&qfull, tiles * NH * a.tile_tokens * a.G * 128);
          for (int j = 0; j < tiles; ++j)
#pragma unroll
            for (int h = 0; h < NH; ++h)
              ck_tma_4d(sQ + j * TILE + h * (TILE / NH), &map_q, 0, h, w.ukvh * a.G,
                        w.us.row0 + w.i0 + j * a.tile_tokens, &qfull);
        }
        ++n;
        if (KV8) continue;
      }
      const int32_t* pt = a.page_table + (long long)w.ub * a.pages_per_seq;
      auto page_row = [&](int t) {  // 8-row group of this lane's page; -2 reads zeros
        const int key0 = t * kCkKeys + lane * 16;
        if (lane >= 8 || key0 >= w.us.end) return -2;
        const int id = __ldg(pt + key0 / 16);
        if (id >= 0 && id < a.n_pages) return (id * a.Hkv + w.ukvh) * 2;
        if (a.err && !is_v) atomicExch(a.err, 1);
        return -2;
      };
      int row = page_row(w.t0);
      for (int t = w.t0; t < w.t1; ++t, ++kn) {
        const int s = kn % R;
        if (kn >= R) ok = mbar_wait(&empty[s], ((kn / R) & 1) ^ 1);
        ok = __all_sync(0xffffffffu, ok && !*abort_flag);
        if (!ok) break;
        if (lane == 0) mbar_expect_tx(&full[s], TILE);
        __syncwarp();
        if (lane < 8) ck_tma_4d(dst + s * TILE + lane * PAGE, map, 0, 0, 0, row, &full[s]);
        if (t + 1 < w.t1) row = page_row(t + 1);
      }
    }
    if (!ok && lane == 0) fail();
    if (lane == 0) {  // copies still in flight land before the CTA leaves
      if (!is_v && n > 0) mbar_wait(&qfull, (n - 1) & 1);
      if (!KV8)
        for (int t = max(0, kn - R); t < kn; ++t) mbar_wait(&full[t % R], (t / R) & 1);
    }
  } else if (warp == kCkWarpMma) {
    // ---------------- MMA issuer: every lane runs the loop, one issues.
    constexpr uint32_t idesc_s = tc_idesc(kCkKeys, kCkKeys), idesc_o = tc_idesc(kCkKeys, HD) | (1u << 16);
    const uint64_t qd = sdesc(smem_u32(sQ)), kd = ck_sdesc_k(smem_u32(sK), SBO),
                   vd = ck_sdesc_mn(smem_u32(sV), 1024, SBO);
    int n = 0, kn = 0, pn[2] = {0, 0}, on[2] = {0, 0};
    bool ok = true;
    // descriptor start addresses count 16-byte units
    auto scores = [&](int j, int q, int s) {  // S_j = Q_q K^T of ring tile s (issuing lane only)
      const uint64_t qj = qd + q * (TILE >> 4), ks = kd + s * (TILE >> 4);
#pragma unroll
      for (int kk = 0; kk < HD / 16; ++kk)
        tc_mma(tmem + j * kCkKeys, qj + ((((kk >> 2) * (TILE / NH)) + (kk & 3) * 32) >> 4),
               ks + (((kk >> 2) * 1024 + (kk & 3) * 32) >> 4), idesc_s, kk > 0 ? 1u : 0u);
      tc_commit(&sfull[j]);
    };
    auto values = [&](int j, int s, bool first) {  // O_j (+)= P_j V of ring tile s (issuing lane only)
      const uint64_t vs = vd + s * (TILE >> 4);
#pragma unroll
      for (int kk = 0; kk < kCkKeys / 16; ++kk)  // a page a step; P in two halves of 64 keys
        tc_mma_ts(tmem + kCkO + j * 128, tmem + j * kCkKeys + (kk >> 2) * 64 + (kk & 3) * 8, vs + kk * (PAGE >> 4), idesc_o,
                  (!first || kk > 0) ? 1u : 0u);
    };
    CkWalk w(a, at, len);
    while (ok && w.next()) {
      const int steps = w.t1 - w.t0;
      if (steps <= 0) continue;
      // V rows behind the sequence's last position, zeroed before they are multiplied
      auto clean = [&](int t, int s) {
        const int lo = w.us.end - t * kCkKeys;
        if (KV8 || lo >= kCkKeys || (lo & 15) == 0) return;
        const int page = lo >> 4;
        for (int x = (lo & 15) * (HD / 8) + lane; x < 16 * (HD / 8); x += 32) {
          const int r = x / (HD / 8), c = x % (HD / 8);  // whole rows: the swizzle stays inside them
          *reinterpret_cast<uint4*>(sV + s * TILE + page * PAGE + (r >> 3) * SBO + (c >> 3) * 1024 + (r & 7) * 128 +
                                    (c & 7) * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async();
        __syncwarp();
      };
      ok = mbar_wait(&qfull, n & 1) && mbar_wait(&kfull[kn % R], (kn / R) & 1) && !*abort_flag;
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      ++n;
      tc_fence_after();
      if (!w.pair) {
        // one query tile: key tile t0 + i is group i % 2's, scores two tiles ahead
        if (elect_one()) {
          scores(0, 0, kn % R);
          tc_commit(&kempty[kn % R]);
          if (steps == 1) tc_commit(&qempty);
        }
        __syncwarp();
        if (steps > 1) {
          ok = __all_sync(0xffffffffu, mbar_wait(&kfull[(kn + 1) % R], ((kn + 1) / R) & 1));
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            scores(1, 0, (kn + 1) % R);
            tc_commit(&kempty[(kn + 1) % R]);
            if (steps == 2) tc_commit(&qempty);
          }
          __syncwarp();
        }
        for (int i = 0; i < steps && ok; ++i, ++kn) {
          const int s = kn % R, j = i & 1;
          const int p = j ? pn[1] : pn[0], o = j ? on[1] : on[0];
          ok = mbar_wait(&vfull[s], (kn / R) & 1) &&
               (i + 2 >= steps || mbar_wait(&kfull[s], ((kn + R) / R) & 1)) && mbar_wait(&pfull[j], p & 1) &&
               (i > 1 || o == 0 || mbar_wait(&oempty[j], (o - 1) & 1)) && !*abort_flag;
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          clean(w.t0 + i, s);
          tc_fence_after();
          if (elect_one()) {
            values(j, s, i < 2);
            tc_commit(&vempty[s]);
            if (i + 2 < steps) {
              scores(j, 0, s);
              tc_commit(&kempty[s]);
            } else {
              tc_commit(&ofull[j]);
            }
            if (i + 3 == steps) tc_commit(&qempty);
          }
          __syncwarp();
          if (j) ++pn[1], on[1] += i + 2 >= steps;
          else ++pn[0], on[0] += i + 2 >= steps;
        }
        continue;
      }
      const int e0 = w.end_of(0), e1 = w.t1;  // e0 <= e1: where each tile's keys end
      if (elect_one()) {
        if (w.t0 < e0) scores(0, 0, kn % R);
        scores(1, 1, kn % R);
        tc_commit(&kempty[kn % R]);
        if (steps == 1) tc_commit(&qempty);
      }
      __syncwarp();
      for (int t = w.t0; t < e1 && ok; ++t, ++kn) {
        const int s = kn % R, s1 = (kn + 1) % R;
        ok = mbar_wait(&vfull[s], (kn / R) & 1);
        if (t + 1 < e1) ok = ok && mbar_wait(&kfull[s1], ((kn + 1) / R) & 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        clean(t, s);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int e = j ? e1 : e0;
          if (t >= e || !ok) continue;
          // P_j(t) is written, and (first tile) the last unit's output has been read
          ok = mbar_wait(&pfull[j], pn[j] & 1) && (t > w.t0 || on[j] == 0 || mbar_wait(&oempty[j], (on[j] - 1) & 1)) &&
               !*abort_flag;
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) continue;
          ++pn[j];
          tc_fence_after();
          if (elect_one()) {
            values(j, s, t == w.t0);
            if (t + 1 < e) scores(j, j, s1);
            else tc_commit(&ofull[j]);
          }
          __syncwarp();
          if (t + 1 >= e) ++on[j];
        }
        if (!ok) break;
        if (elect_one()) {
          tc_commit(&vempty[s]);
          if (t + 1 < e1) tc_commit(&kempty[s1]);
          if (t + 2 == e1) tc_commit(&qempty);  // the unit's last scores: Q may be overwritten
        }
        __syncwarp();
      }
    }
    if (!ok && lane == 0) fail();
    if (elect_one()) tc_commit(&mma_done);
    __syncwarp();
    mbar_wait(&mma_done, 0);
  } else if (KV8 && warp >= kCkWarpWiden) {
    // ---------------- int8 cache: bf16(q s) of the key tiles' rows.  Thread: 16 codes
    // (chunk c) of row rr of every 16 / IN pages; its codes of the next half tile (V
    // after K, then the next tile's K) are in flight while it writes this one's.
    constexpr int C = HD / 16;                // chunks a row
    constexpr int PER = 128 / C, N = kCkKeys / PER;  // rows at a time, turns a tile
    const int wi = threadIdx.x - kCkWarpWiden * 32, c = wi % C, rr = wi / C;
    int kn = 0;
    bool ok = true;
    CkWalk w(a, at, len);
    while (ok && w.next()) {
      const int32_t* pt = a.page_table + (long long)w.ub * a.pages_per_seq;
      for (int t = w.t0; t < w.t1 && ok; ++t, ++kn) {
        int rowi[N];  // pool rows (fewer than 2^31); -1 reads zeros
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int key = t * kCkKeys + i * PER + rr;
          rowi[i] = -1;
          if (key < w.us.end) {
            const int id = __ldg(pt + key / 16);
            if (id >= 0 && id < a.n_pages) rowi[i] = (id * a.Hkv + w.ukvh) * 16 + key % 16;
            else if (a.err && c == 0) atomicExch(a.err, 1);
          }
        }
#pragma unroll 1
        for (int which = 0; which < 2; ++which) {
          const int8_t* pool = which ? a.v8 : a.k8;
          const float* scale = which ? a.v_scale : a.k_scale;
          uint4 cw[N];
          float sc[N];
#pragma unroll
          for (int i = 0; i < N; ++i) {
            cw[i] = rowi[i] >= 0 ? ld_nc16(pool + (long long)rowi[i] * HD + c * 16) : make_uint4(0, 0, 0, 0);
            sc[i] = rowi[i] >= 0 ? __ldg(scale + rowi[i]) : 0.f;
          }
          const int s = kn % R;
          if (kn >= R) ok = mbar_wait(which ? &vempty[s] : &kempty[s], ((kn / R) & 1) ^ 1);
          if (!__all_sync(0xffffffffu, ok) || __any_sync(0xffffffffu, *abort_flag != 0)) {
            ok = false;
            break;
          }
          uint8_t* dst = (which ? sV : sK) + s * TILE + (c >> 2) * 1024;
          const int cb = 2 * (c & 3);
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const int row = i * PER + rr, sw = row & 7;
            const uint32_t ww[4] = {cw[i].x ^ 0x80808080u, cw[i].y ^ 0x80808080u, cw[i].z ^ 0x80808080u,
                                    cw[i].w ^ 0x80808080u};
            const float2 s2 = make_float2(sc[i], sc[i]), z2 = make_float2(-32896.f, -32896.f);
            uint32_t o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {  // codes 2j, 2j + 1: fp32 2^15 + 128 + q
              const uint32_t u = ww[j >> 1];
              const float lo = __uint_as_float(__byte_perm(u, 0x47000000u, (j & 1) ? 0x7424 : 0x7404));
              const float hi = __uint_as_float(__byte_perm(u, 0x47000000u, (j & 1) ? 0x7434 : 0x7414));
              const float2 f = ck_mul2(ck_add2(make_float2(lo, hi), z2), s2);
              o[j] = pa_pack(f.x, f.y);
            }
            const uint4 e = make_uint4(o[0], o[1], o[2], o[3]), f = make_uint4(o[4], o[5], o[6], o[7]);
            uint8_t* rp = dst + (row >> 3) * SBO + sw * 128;
            // the lanes of a row's upper half write their odd chunk first: eight lanes, eight banks of 16 bytes
            if (c < 4) {
              *reinterpret_cast<uint4*>(rp + ((cb ^ sw) << 4)) = e;
              *reinterpret_cast<uint4*>(rp + (((cb + 1) ^ sw) << 4)) = f;
            } else {
              *reinterpret_cast<uint4*>(rp + (((cb + 1) ^ sw) << 4)) = f;
              *reinterpret_cast<uint4*>(rp + ((cb ^ sw) << 4)) = e;
            }
          }
          fence_proxy_async();  // the MMAs read the tile through the async proxy
          __syncwarp();
          if (lane == 0) mbar_arrive(which ? &vfull[s] : &kfull[s]);
        }
      }
    }
    if (!ok && lane == 0) fail();
  } else if (warp < kCkSoft) {
    // ---------------- softmax: group j, half `half` of the keys, row 32 quad + lane
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(KV8 ? 88 : 104));
    const int j = warp >> 3, half = (warp >> 2) & 1, quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)(quad * 32) << 16);
    const uint32_t ts = lane_base + j * kCkKeys + half * 64, to = lane_base + kCkO + j * 128;
    const float scale = kPaLog2e * rsqrtf((float)HD);
    const int tok = row / a.G;  // of a tile's packed rows
    const bool packed = row < a.tile_tokens * a.G;
    int sn = 0, on[2] = {0, 0}, xn = 0, mn = 0;
    bool ok = true;
    uint8_t* stage = sV + R * TILE + warp * kCkStage;
    CkWalk w(a, at, len);
    while (ok && w.next()) {
      const int jq = w.pair ? j : 0;  // this group's query tile
      const int tile_i0 = w.i0 + jq * a.tile_tokens, tile_n = min(a.tile_tokens, w.us.n - tile_i0);
      const bool on_row = packed && tok < tile_n;
      const bool on_warp = __any_sync(0xffffffffu, on_row);
      // keys of this row, and of the tile's first
      const int lim = on_row ? min(w.us.end, w.us.pos + tile_i0 + tok + 1) : 0;
      const int lim0 = min(w.us.end, w.us.pos + tile_i0 + 1);
      const int t_end = w.end_of(j), t_first = w.pair ? w.t0 : w.t0 + j, stride = w.pair ? 1 : 2;
      float m = -INFINITY;  // reference maximum (log2 domain)
      float2 l2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
      for (int t = t_first; t < t_end; t += stride, ++sn) {
        ok = __all_sync(0xffffffffu, mbar_wait(&sfull[j], sn & 1));
        if (!ok) break;
        if (on_warp) {
          tc_fence_after();
          // the scores stay in registers from their maximum to P, or (int8 cache: fewer
          // registers a thread) are read again 32 at a time
          float v[KV8 ? 32 : 64];
          const int key0 = t * kCkKeys + half * 64;
          const bool masked = (t + 1) * kCkKeys > lim0;
          auto load = [&](int x0, float* d) {
            tc_ld<32>(ts + x0, reinterpret_cast<uint32_t*>(d));
            if (masked) {
#pragma unroll
              for (int x = 0; x < 32; ++x)
                if (key0 + x0 + x >= lim) d[x] = -INFINITY;
            }
          };
          float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int x0 = 0; x0 < 64; x0 += 32) {
            float* d = KV8 ? v : v + x0;
            load(x0, d);
#pragma unroll
            for (int x = 0; x < 32; x += 8)
#pragma unroll
              for (int y = 0; y < 4; ++y) m4[y] = fmaxf(m4[y], fmaxf(d[x + 2 * y], d[x + 2 * y + 1]));
          }
          float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * scale;
          // the other half's maximum
          s_x[j][xn & 1][half][row] = mx;
          __syncwarp();
          if (lane == 0) mbar_arrive(&xch[j][quad]);
          ok = __all_sync(0xffffffffu, mbar_wait(&xch[j][quad], xn & 1));
          if (!ok) break;
          mx = fmaxf(mx, s_x[j][xn & 1][half ^ 1][row]);
          ++xn;
          // move the reference when the tile would exceed it by more than 2^kCkSlack
          float corr = 1.f;
          if (mx > m + kCkSlack) {
            corr = exp2f(m - mx);  // 0 on the first tile
            m = mx;
            l2[0].x *= corr, l2[0].y *= corr, l2[1].x *= corr, l2[1].y *= corr;
          }
          if (t > t_first && __any_sync(0xffffffffu, corr != 1.f)) {
            // O holds P V of the earlier tiles (complete: S(t) was issued after it)
#pragma unroll 1
            for (int x = half * (HD / 2); x < (half + 1) * (HD / 2); x += 16) {
              uint32_t o[16];
              tc_ld<16>(to + x, o);
#pragma unroll
              for (int y = 0; y < 16; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * corr);
              tc_st16(to + x, o);
            }
          }
          const float mref = m == -INFINITY ? 0.f : m;
          const float2 sc2 = make_float2(scale, scale), nm2 = make_float2(-mref, -mref);
#pragma unroll
          for (int x0 = 0; x0 < 64; x0 += 32) {
            uint32_t pw[16];
            float* d = KV8 ? v : v + x0;
            if (KV8) load(x0, d);
#pragma unroll
            for (int x = 0; x < 32; x += 2) {
              const float2 e = ck_fma2(make_float2(d[x], d[x + 1]), sc2, nm2);
              const float2 p = make_float2(pa_ex2(e.x), pa_ex2(e.y));
              l2[(x >> 1) & 1] = ck_add2(l2[(x >> 1) & 1], p);
              pw[x / 2] = pa_pack(p.x, p.y);
            }
            tc_st16(ts + x0 / 2, pw);
          }
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
        }
        if (lane == 0) mbar_arrive(&pfull[j]);
      }
      if (!ok) break;
      float l = (l2[0].x + l2[0].y) + (l2[1].x + l2[1].y);
      // ---- the piece's output
      const bool whole = w.first && w.last, empty = w.t1 <= w.t0;
      const bool use0 = w.uses(0), use1 = w.uses(1);
      float a0 = 1.f, a1 = 0.f;  // factors of O_0 and O_1 (units of one tile), or of O_j
      if (w.pair) {
        if (j ? use1 : use0) {
          if (on_warp) {
            s_x[j][xn & 1][half][row] = l;
            __syncwarp();
            if (lane == 0) mbar_arrive(&xch[j][quad]);
            ok = __all_sync(0xffffffffu, mbar_wait(&xch[j][quad], xn & 1));
            if (!ok) break;
            l += s_x[j][xn & 1][half ^ 1][row];
            ++xn;
          }
          ok = __all_sync(0xffffffffu, mbar_wait(&ofull[j], (j ? on[1] : on[0]) & 1));
          if (!ok) break;
        }
        on[0] += use0, on[1] += use1;
      } else if (!empty) {
        // every warp meets here, those without rows too: past this point both groups
        // have seen the accumulators of the pieces before
        s_ml[mn & 1][j][half][row] = make_float2(m, l);
        __syncwarp();
        if (lane == 0) mbar_arrive(&met[quad]);
        ok = __all_sync(0xffffffffu, mbar_wait(&met[quad], mn & 1));
        if (!ok) break;
        const float2 p0 = s_ml[mn & 1][0][0][row], p1 = s_ml[mn & 1][1][0][row];
        const float l0 = p0.y + s_ml[mn & 1][0][1][row].y, l1 = p1.y + s_ml[mn & 1][1][1][row].y;
        ++mn;
        m = fmaxf(p0.x, p1.x);
        a0 = p0.x == -INFINITY ? 0.f : exp2f(p0.x - m);
        a1 = p1.x == -INFINITY ? 0.f : exp2f(p1.x - m);
        l = a0 * l0 + a1 * l1;
        ok = __all_sync(0xffffffffu, mbar_wait(&ofull[0], on[0] & 1) && (!use1 || mbar_wait(&ofull[1], on[1] & 1)));
        if (!ok) break;
        ++on[0];
        on[1] += use1;
      }
      tc_fence_after();
      const bool have = w.pair ? (j ? use1 : use0) : !empty;  // an accumulator to read
      const float inv = l > 0.f ? 1.f / l : 0.f;
      const int q4 = w.pair ? half : 2 * j + half;
      const int cols = w.pair ? HD / 2 : HD / 4, x0 = q4 * cols;
      if (on_warp) {
        const uint32_t src = w.pair ? to : lane_base + kCkO;
        auto load = [&](int x, float* r) {  // 16 columns of the sums
#pragma unroll
          for (int y = 0; y < 16; ++y) r[y] = 0.f;
          if (!have) return;
          tc_ld<16>(src + x, reinterpret_cast<uint32_t*>(r));
          if (w.pair) return;
          if (use1) {
            uint32_t u[16];
            tc_ld<16>(src + 128 + x, u);
#pragma unroll
            for (int y = 0; y < 16; ++y) r[y] = a0 * r[y] + a1 * __uint_as_float(u[y]);
          }
        };
        if (whole) {
          // through shared memory, two lanes to a row's 32 bytes
          uint16_t* o = a.out + (long long)(w.us.row0 + tile_i0) * a.H * HD + (long long)w.ukvh * a.G * HD;
          for (int x = x0; x < x0 + cols; x += 16) {
            float r[16];
            load(x, r);
            uint4 p[2];
            uint32_t* pw = reinterpret_cast<uint32_t*>(p);
#pragma unroll
            for (int y = 0; y < 8; ++y) pw[y] = pa_pack(r[2 * y] * inv, r[2 * y + 1] * inv);
            const int sw = (lane >> 2) & 1;
            *reinterpret_cast<uint4*>(stage + lane * 32 + (sw << 4)) = p[0];
            *reinterpret_cast<uint4*>(stage + lane * 32 + ((sw ^ 1) << 4)) = p[1];
            __syncwarp();
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const int lr = y * 16 + (lane >> 1), r2 = quad * 32 + lr, t2 = r2 / a.G;
              const uint4 v = *reinterpret_cast<const uint4*>(stage + lr * 32 + (((lane & 1) ^ ((lr >> 2) & 1)) << 4));
              if (r2 < a.tile_tokens * a.G && t2 < tile_n)
                *reinterpret_cast<uint4*>(o + (long long)t2 * a.H * HD + (r2 - t2 * a.G) * HD + x + (lane & 1) * 8) = v;
            }
            __syncwarp();
          }
        } else {
          uint8_t* slot = a.ws + kCkHead + ((size_t)blockIdx.x * 2 + (w.first ? 1 : 0)) * ck_slot<HD>();
          const int r = jq * kCkKeys + row;
          if (have)
            for (int x = x0; x < x0 + cols; x += 16) {
              float f[16];
              load(x, f);
#pragma unroll
              for (int y = 0; y < 4; ++y)
                reinterpret_cast<float4*>(slot)[(size_t)(x / 4 + y) * kCkRows + r] =
                    make_float4(f[4 * y], f[4 * y + 1], f[4 * y + 2], f[4 * y + 3]);
            }
          if (q4 == 0)
            reinterpret_cast<float2*>(slot + (size_t)kCkRows * HD * 4)[r] =
                make_float2(have && l > 0.f ? m : -INFINITY, have ? l : 0.f);
        }
      }
      if (have) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (w.pair) {  // the 16 arrivals of an accumulator: two from each of its own group's warps
            mbar_arrive(&oempty[j]);
            mbar_arrive(&oempty[j]);
          } else {
            mbar_arrive(&oempty[0]);
            if (use1) mbar_arrive(&oempty[1]);
          }
        }
      }
      if (threadIdx.x == 0 && w.first && !w.last) {
        const CkLeft left = {w.ux + kCkStart + w.nt, w.us.row0, w.i0, w.us.n, w.ukvh, w.pair};
        reinterpret_cast<CkLeft*>(a.ws + kCkHead / 4)[blockIdx.x] = left;
      }
    }
    if (!ok && lane == 0) fail();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kCkWarpMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCkTmemCols) : "memory");
  }
}

// ------------------------------------------------------------------ joining the parts
// Block (c, s): rows 32 (s / HC) .. + 31 and columns 32 (s % HC) .. + 31 of the unit
// that CTA c began and left unfinished: o = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i
// over the CTAs whose stretches begin before the unit's end, in their order.
constexpr int kCkJoinParts = 4;  // shares of a unit's parts, added in order at the end
template <int HD>
__global__ void __launch_bounds__(256 * kCkJoinParts)
    attn_chunk_join_kernel(const uint8_t* __restrict__ ws, int ctas, int H, int G, int tile_tokens,
                           uint16_t* __restrict__ out) {
  constexpr int HC = HD / 32;
  __shared__ float4 s_o[kCkJoinParts - 1][256];
  __shared__ float2 s_ml[kCkJoinParts][32];
  pdl_trigger();
  pdl_wait();
  const int c = blockIdx.x;
  const CkLeft u = reinterpret_cast<const CkLeft*>(ws + kCkHead / 4)[c];
  if (u.end == 0) return;
  const int rows0 = 32 * (blockIdx.y / HC);
  const int tile = rows0 / kCkKeys, i0 = u.i0 + tile * tile_tokens, n = min(tile_tokens, u.n - i0);
  if ((tile && !u.pair) || (rows0 % kCkKeys) >= n * G) return;
  // rows in the lanes' low bits where the parts are read, columns where the result is written
  const int tid = threadIdx.x & 255, part = threadIdx.x >> 8;
  const int lr = (tid & 7) + 8 * (tid >> 6), c4 = 8 * (blockIdx.y % HC) + ((tid >> 3) & 7);
  const long long* begins = reinterpret_cast<const long long*>(ws);
  auto slot = [&](int k) { return ws + kCkHead + ((size_t)k * 2 + (k == c ? 1 : 0)) * ck_slot<HD>(); };
  auto begun = [&](int k) { return k < ctas ? begins[k] : 0x7fffffffffffffffLL; };
  // the unit's parts: CTA c and the ones after it that begin before its end
  int last = c;
  while (last + 1 < ctas && begins[last + 1] < u.end) ++last;
  const int per = (last - c + kCkJoinParts) / kCkJoinParts, k0 = c + part * per, k1 = min(last + 1, k0 + per);
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k = k0; k < k1; ++k) {
    if (k > c && begun(k + 1) == begins[k]) continue;  // no stretch
    const uint8_t* p = slot(k);
    const float2 ml = reinterpret_cast<const float2*>(p + (size_t)kCkRows * HD * 4)[rows0 + lr];
    if (ml.x == -INFINITY) continue;
    const float4 f = reinterpret_cast<const float4*>(p)[(size_t)c4 * kCkRows + rows0 + lr];
    const float m2 = fmaxf(m, ml.x), x = exp2f(m - m2), y = exp2f(ml.x - m2);
    m = m2;
    l = l * x + ml.y * y;
    o = make_float4(o.x * x + f.x * y, o.y * x + f.y * y, o.z * x + f.z * y, o.w * x + f.w * y);
  }
  if (part) s_o[part - 1][tid] = o;
  if (((tid >> 3) & 7) == 0) s_ml[part][lr] = make_float2(m, l);
  __syncthreads();
  if (part) return;
#pragma unroll
  for (int k = 1; k < kCkJoinParts; ++k) {
    const float2 ml = s_ml[k][lr];
    if (ml.x == -INFINITY) continue;
    const float4 f = s_o[k - 1][tid];
    const float m2 = fmaxf(m, ml.x), x = exp2f(m - m2), y = exp2f(ml.x - m2);
    m = m2;
    l = l * x + ml.y * y;
    o = make_float4(o.x * x + f.x * y, o.y * x + f.y * y, o.z * x + f.z * y, o.w * x + f.w * y);
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  const int r = rows0 % kCkKeys + lr, tok = r / G;
  if (r >= tile_tokens * G || tok >= n) return;
  *reinterpret_cast<uint2*>(out + ((long long)(u.row0 + i0 + tok) * H + (long long)u.kvh * G + r % G) * HD + c4 * 4) =
      make_uint2(pa_pack(o.x * inv, o.y * inv), pa_pack(o.z * inv, o.w * inv));
}

// Row-major [d3][d2][d1][d0] of bf16 (strides in bytes), 128-byte swizzle.
static bool make_tensor_map_4d(CUtensorMap* map, const void* base, const long long (&dim)[4], const long long (&stride)[3],
                               const int (&box)[4]) {
  typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
                   q == cudaDriverEntryPointSuccess
               ? (Encode)p
               : (Encode)nullptr;
  }();
  if (!fn) return false;
  cuuint64_t d[4], st[3];
  cuuint32_t b[4], one[4] = {1, 1, 1, 1};
  for (int i = 0; i < 4; ++i) d[i] = (cuuint64_t)dim[i], b[i] = (cuuint32_t)box[i];
  for (int i = 0; i < 3; ++i) st[i] = (cuuint64_t)stride[i];
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), d, st, b, one,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static int ck_sms() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
      sms <= 0)
    sms = 152;
  return std::min(sms, 1024);
}

size_t attention_chunk_ws_bytes(int B, int n_heads, int n_kv_heads, int head_dim, int max_new) {
  return kCkHead + (size_t)2 * 152 * (head_dim == 64 ? ck_slot<64>() : ck_slot<128>());
}

template <int HD, bool KV8>
static cudaError_t launch_ck(const uint16_t* q, int q_stride, const fp_kv_view& kv, const CkArgs& a, cudaStream_t s) {
  CUtensorMap mq, mk, mv;
  // q [tokens][heads][halves][64], box [tile tokens][G][1][64]
  if (!make_tensor_map_4d(&mq, q, {64, HD / 64, a.H, a.n_tokens}, {128, HD * 2, 2LL * q_stride},
                          {64, 1, a.G, a.tile_tokens}))
    return cudaErrorInvalidValue;
  mk = mv = mq;
  if (!KV8) {
    // pools [row / 8][halves][8 rows][64] of rows of HD, box: a page's 16 rows of a head
    const long long groups = (long long)kv.n_pages * kv.n_kv_heads * 2;
    for (int i = 0; i < 2; ++i)
      if (!make_tensor_map_4d(i ? &mv : &mk, i ? kv.v_pool : kv.k_pool, {64, 8, HD / 64, groups}, {HD * 2, 128, 8 * HD * 2},
                              {64, 8, HD / 64, 2}))
        return cudaErrorInvalidValue;
  }
  static std::atomic<unsigned long long> attr{0};
  FP_CUDA_TRY(smem_limit_once(attn_chunk_kernel<HD, KV8>, ck_smem<HD>(), &attr));
  const int grid = std::min(ck_sms(), 152);
  FP_CUDA_TRY(launch(attn_chunk_kernel<HD, KV8>, dim3(grid), dim3(ck_threads<KV8>()), (size_t)ck_smem<HD>(), s, mq, mk, mv, a));
  // the parts of units that several CTAs took: blocks of 32 rows and 32 columns
  const int rows = std::min(kCkRows, (std::min(a.max_new, 2 * a.tile_tokens) + a.tile_tokens - 1) / a.tile_tokens * kCkKeys);
  return launch_early(attn_chunk_join_kernel<HD>, dim3(grid, rows / 32 * (HD / 32)), dim3(256 * kCkJoinParts), 0, s,
                      (const uint8_t*)a.ws, grid, a.H, a.G, a.tile_tokens, a.out);
}

cudaError_t launch_attention_chunk(const uint16_t* q, int q_stride, int n_tokens, int B, int n_heads,
                                   const fp_kv_view& kv, const int32_t* cu, const int32_t* pos, int max_new, int max_len,
                                   uint16_t* out, void* ws, int32_t* err, cudaStream_t s) {
  if (n_tokens <= 0 || B <= 0) return cudaSuccess;
  const int G = n_heads / kv.n_kv_heads;
  const CkArgs a = {cu, pos, n_tokens, B, n_heads, kv.n_kv_heads, G, max_new, max_len, ck_tile_tokens(G), kv.page_table,
                    kv.pages_per_seq, kv.n_pages, (const int8_t*)kv.k_pool, (const int8_t*)kv.v_pool, kv.k_scale, kv.v_scale,
                    out, (uint8_t*)ws, err};
  if (kv.head_dim == 64)
    return kv.kvquant == FP_KV_INT8 ? launch_ck<64, true>(q, q_stride, kv, a, s) : launch_ck<64, false>(q, q_stride, kv, a, s);
  return kv.kvquant == FP_KV_INT8 ? launch_ck<128, true>(q, q_stride, kv, a, s) : launch_ck<128, false>(q, q_stride, kv, a, s);
}

}  // namespace fpk
