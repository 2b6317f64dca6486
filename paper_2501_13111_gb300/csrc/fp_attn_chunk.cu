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
//   warps 0-7   softmax, two groups of 4: one query row (TMEM lane) a thread.
//               P = 2^(s - m) is rounded to bf16 for the second product (2^-8 of each
//               p, the sums in fp32), 64 keys at a time from registers, so that the first
//               half's products run while the second half is computed; the reference m
//               moves only when a half passes it by 2^8 (O and the row sum are rescaled
//               then).  At the end of a piece they write its rows, or the part
//               that this CTA has of them: the last CTA to finish a unit adds its parts up;
//   warp 8      TMA: the unit's Q tiles (one box per 64 columns: tokens x heads) and,
//               page by page, the keys.  One box a page, in the order [8 rows][64
//               columns] the descriptors step through.  (int8 cache: it finds the pages
//               of each tile instead, sends their codes on to L2, and stages the scales);
//   warps 9, 10 issue the MMAs of a group each: O += P(t) V(t), then the group's next
//               scores over the columns that P(t) has left.  (One warp for both groups
//               left the tensor pipe idle for half of each step: a wait costs 100-200
//               cycles while the operands' reads fill shared memory's bandwidth, and
//               there were five in a row.)  Warp 9 owns the TMEM;
//   warp 11     plans the CTA's stretch, describes its pieces of units to the others,
//               and (bf16 cache) copies the values;
//   warps 12-19 (int8 cache) K and V tiles of the codes as bf16, exact (a byte permute
//               gives fp32 2^15 + 128 + q, a subtraction q).  A key's K scale multiplies
//               its score column, its V scale its column of P, both in fp32.  (Tiles of
//               bf16(q s) took 54 us where this takes 63, 420 where 496, see below, but
//               were further from the sums in 64 bits: 0.0040 against 0.0024, relative.)
// Measured (launches in a graph, heads of 128): 8 sequences of 5 rows to position 612, 32
// heads, bf16 cache 23.1 us (2.7 TB/s); 32 of 5 rows to 2148, 64 heads on 8, int8 63 us
// (1.8 TB/s); 4 chunks of 512 rows to 2048, 40 heads, bf16 77 us (747 TFLOP/s); 2 of 1024
// rows to 8000, 64 heads on 8, int8 496 us (815 TFLOP/s).  A step of two query tiles takes
// about 3800 cycles where its MMAs need 2080: a group's scores wait for its P, P for the
// scores, and what is in between is as long as the other group's products; with an int8
// cache the scales' way from shared memory, which the MMAs keep busy, comes on top (chunk
// int8 406 us with constants instead).  Small batches: about 7000 cycles
// pass before the first scores and 8000 behind the last.
// Slots behind the sequence's last position may hold anything: their scores are
// masked, their V rows are zeroed before the product (int8 cache: read as zeros).
// Every wait on an mbarrier is bounded (error 2 past the limit).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "attn_tc.cuh"
#include "chunk.cuh"
#include "chunk_items.h"
#include "kernels.cuh"

namespace fpk {

constexpr int kCkSoft = 8;                        // softmax warps
constexpr int kCkWarpQ = 8, kCkWarpMma = 9, kCkWarpPlan = 11, kCkWarpWiden = 12, kCkWiden = 8;
template <bool KV8>
constexpr int ck_threads() { return KV8 ? (kCkWarpWiden + kCkWiden) * 32 : 384; }
// Registers a thread: 384 threads may have 168, and take 163 or 167 (heads of 128, 64);
// 640 (int8 cache) launch with 96, moved to the softmax: 256 x 128 + 384 x 72 < 640 x 96 (with 120 and 80 its row
// spills more: chunk int8 504 us against 496)
constexpr int kCkReaders = kCkSoft + 3;           // warps that read each piece's description: softmax, Q, MMA
constexpr int kCkPieces = 4;                      // pieces described ahead
constexpr int kCkAhead = 4;                       // int8 cache: key tiles whose pages are known ahead
constexpr int kCkScales = 8;                      // tiles of scales: a tile is described once the widening of
                                                  // the one kCkAhead before it is over, which P V of the second
                                                  // tile before that preceded: the eighth before it is done with
constexpr int kCkRing = 2;                        // K tiles in shared memory, and V tiles
constexpr uint32_t kCkTmemCols = 512, kCkO = 256; // O of group j at kCkO + 128 j, its scores at 128 j
constexpr int kCkStage = 32 * 64;                 // a warp's 32 output rows, 32 columns at a time
constexpr float kCkSlack = 8.f;                   // log2 of the largest P before the reference moves
constexpr int kCkRows = 256;                      // rows of a unit
template <int HD>
constexpr int ck_tile_bytes() { return kCkKeys * HD * 2; }
template <int HD>
constexpr int ck_smem() { return (2 + 2 * kCkRing) * ck_tile_bytes<HD>() + kCkSoft * kCkStage + 1024; }

// Workspace: tickets (zero between calls), then for every CTA two partial results (slot
// 0: of a unit begun by an earlier CTA, slot 1: of the one it began and left): fp32 O as
// [HD / 4][256 rows][4], (m, l) [256 rows], and (m, l) of a group of parts added up.
// The parts of a unit are added in groups of kCkGroup CTAs, then the groups' sums:
// tickets [owner][group], the last for the groups.
constexpr int kCkGroup = 13, kCkMaxCtas = 152;  // 12 groups at most
constexpr size_t kCkTickets = 16;
constexpr size_t kCkHead = 64 * 1024;
static_assert(kCkMaxCtas * kCkTickets * 4 <= kCkHead, "tickets");
template <int HD>
constexpr size_t ck_slot() { return (size_t)kCkRows * (HD * 4 + 16); }

// [8 rows][64 columns] atoms: 8-row groups `sbo` bytes apart, K-major.
FP_DEV uint64_t ck_sdesc_k(uint32_t saddr, uint32_t sbo) {
  return (uint64_t)((saddr & 0x3FFFF) >> 4) | (uint64_t)1 << 16 | (uint64_t)(sbo >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;
}
FP_DEV void ck_tma_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
      : "memory");
}
FP_DEV float ck_max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
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
  long long wait_limit;  // rounds of the issuers' wait for a V tile
};

// A piece of a unit, as the planning warp describes it.
struct __align__(16) CkPiece {
  int t0, t1, e0;   // key tiles t0 .. t1-1; where the first of two tiles' end
  int flags;
  int row0, n, pos; // the unit's first row, its rows (tokens), the first one's position
  int end;          // cached positions of the sequence that may be read
  int b, kvh;
  int own, parts;   // the CTA that begins the unit, and how many take part of it
  FP_DEV bool pair() const { return flags & 1; }    // two query tiles
  FP_DEV bool first() const { return flags & 2; }   // the unit's first part
  FP_DEV bool last() const { return flags & 4; }
  FP_DEV bool done() const { return flags & 8; }    // no piece: the stretch is walked
  FP_DEV bool empty() const { return t1 <= t0; }
  FP_DEV bool uses(int j) const { return pair() ? (j ? t1 > t0 : e0 > t0) : t1 - t0 > j; }  // accumulator j
};

// The plan of this CTA's stretch, by one whole warp, and its pieces one by one.  One
// warp's instructions follow each other at 4-6 cycles and every kernel starts with cold
// instruction caches, so it is kept short: 32-bit places (ck_fits), both ends of the
// stretch in two lanes at once.
struct CkWalk {
  const CkArgs& a;
  CkSeq s;
  int b, kvh, u, off;  // the next place: `off` into unit u of (b, kvh)
  int x, rem;          // its place on the line, and places left
  int W, g;            // the line's length, shared among g CTAs
  FP_DEV int load(int bb, bool* fine) {  // sequence bb, and its places; false: a bound is broken
    const int lo = __ldg(a.cu + bb), hi = __ldg(a.cu + bb + 1), p = __ldg(a.pos + bb);
    *fine = s.set(lo, hi - lo, p, a.tile_tokens, a.max_new, a.max_len);
    return lo < 0 || hi < lo || hi > a.n_tokens ? -1 : s.cost(2 * a.tile_tokens) * a.Hkv;
  }
  FP_DEV CkWalk(const CkArgs& a) : a(a) {
    const int lane = threadIdx.x & 31, T = 2 * a.tile_tokens;
    // the line's length (up to 32 sequences: their places stay in the lanes)
    int c = 0;
    bool fine = true, good = true;
    W = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < a.B; b0 += 32) {
      c = 0;
      bool f = true;
      if (b0 + lane < a.B) c = load(b0 + lane, &f);
      fine = fine && f && c >= 0, good = good && c >= 0;
      W += c;
    }
    if (!__all_sync(0xffffffffu, fine) && blockIdx.x == 0 && lane == 0 && a.err) atomicExch(a.err, 1);
    // (a cu that decreases or leaves the buffers: nothing is done)
    W = __all_sync(0xffffffffu, good) ? __reduce_add_sync(0xffffffffu, W) : 0;
    b = a.B, kvh = u = off = 0, x = W, rem = 0;
    if (W == 0) return;
    g = ck_ctas(W, gridDim.x);
    // lane 0: where the stretch begins, lane 1 where the next one does
    const int cta = min((int)blockIdx.x + (lane & 1), g), at = cta < g ? ck_begin(cta, W, g) : W;
    const int at0 = __shfl_sync(0xffffffffu, at, 0), at1 = __shfl_sync(0xffffffffu, at, 1);
    if (at0 >= W) return;
    int base = 0;
    CkSeq mine;
    int from = 0, per = 1;
    bool found0 = false, found1 = at1 >= W;
#pragma unroll 1
    for (int b0 = 0; b0 < a.B && !(found0 && found1); b0 += 32) {
      bool f;
      if (a.B > 32) c = b0 + lane < a.B ? load(b0 + lane, &f) : 0;
      int incl = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      incl += base;
      base = __shfl_sync(0xffffffffu, incl, 31);
      const unsigned m0 = __ballot_sync(0xffffffffu, at0 < incl), m1 = __ballot_sync(0xffffffffu, at1 < incl);
      const bool new0 = m0 && !found0, new1 = m1 && !found1;
      found0 |= new0, found1 |= new1;
      const int l = lane == 1 ? __ffs(m1) - 1 : __ffs(m0) - 1;  // whose sequence this lane looks into
      const int sb = b0 + l, first = __shfl_sync(0xffffffffu, incl - c, l & 31), cost = __shfl_sync(0xffffffffu, c, l & 31);
      CkSeq t;
      t.row0 = __shfl_sync(0xffffffffu, s.row0, l & 31), t.n = __shfl_sync(0xffffffffu, s.n, l & 31);
      t.pos = __shfl_sync(0xffffffffu, s.pos, l & 31), t.end = __shfl_sync(0xffffffffu, s.end, l & 31);
      t.units = __shfl_sync(0xffffffffu, s.units, l & 31), t.bad = __shfl_sync(0xffffffffu, s.bad, l & 31);
      if (lane == 1 ? new1 : new0) mine = t, b = sb, from = first, per = cost / a.Hkv;
    }
    if (b < a.B) {  // the unit at this place, and the border off the unit's ends
      kvh = (unsigned)(at - from) / (unsigned)per;
      const int in = at - from - kvh * per;
      u = mine.unit_at(in, T);
      const int start = mine.before(u, T);
      off = ck_snap(in - start, mine.tiles(u, T), mine.weight(u, T));
      x = from + kvh * per + start + off;
      if (off == mine.places(u, T)) {  // behind the unit: the next one's beginning
        off = 0;
        if (++u == mine.units) u = 0, ++kvh;
      }
    }
    rem = __shfl_sync(0xffffffffu, x, 1);  // (x = W where no CTA follows)
    b = __shfl_sync(0xffffffffu, b, 0), kvh = __shfl_sync(0xffffffffu, kvh, 0), u = __shfl_sync(0xffffffffu, u, 0);
    off = __shfl_sync(0xffffffffu, off, 0), x = __shfl_sync(0xffffffffu, x, 0);
    s.row0 = __shfl_sync(0xffffffffu, mine.row0, 0), s.n = __shfl_sync(0xffffffffu, mine.n, 0);
    s.pos = __shfl_sync(0xffffffffu, mine.pos, 0), s.end = __shfl_sync(0xffffffffu, mine.end, 0);
    s.units = __shfl_sync(0xffffffffu, mine.units, 0), s.bad = __shfl_sync(0xffffffffu, mine.bad, 0);
    rem -= x;
    if (kvh == a.Hkv) turn();
  }
  // on to the next sequence that has rows (there is one while places are left)
  FP_DEV void turn() {
    kvh = 0;
    s.units = 0;
    bool f;
    while (s.units == 0 && rem > 0)
      if (b + 1 < a.B) load(++b, &f);
      else rem = 0;
  }
  FP_DEV void next(CkPiece* p) {
    if (rem <= 0) {
      p->flags = 8;
      return;
    }
    const int T = 2 * a.tile_tokens, nt = s.tiles(u, T), i0 = u * T;
    const bool pair = s.n - i0 > a.tile_tokens;
    const int lg = pair ? 1 : 0, left = kCkStart + (nt << lg) - off, take = min(left, rem);
    p->t0 = max(0, off - kCkStart) >> lg;
    p->t1 = min(nt, max(0, off + take - kCkStart) >> lg);
    // the first tile's own last key tile
    p->e0 = min(p->t1, s.bad || !pair ? nt : (s.pos + i0 + a.tile_tokens + kCkKeys - 1) / kCkKeys);
    p->flags = (pair ? 1 : 0) | (off == 0 ? 2 : 0) | (take == left ? 4 : 0);
    p->row0 = s.row0 + i0, p->n = min(T, s.n - i0), p->pos = s.pos + i0, p->end = s.end;
    p->b = b, p->kvh = kvh, p->own = blockIdx.x, p->parts = 1;
    if (off != 0 || take != left) ck_parts(x - off, nt, 1 + lg, W, g, &p->own, &p->parts);
    rem -= take;
    x += take;
    off = 0;
    if (rem > 0 && ++u == s.units) {
      u = 0;
      if (++kvh == a.Hkv) turn();
    }
  }
};

template <int HD, bool KV8>
__global__ void __launch_bounds__(ck_threads<KV8>(), 1)
    attn_chunk_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CkArgs a) {
  constexpr int TILE = ck_tile_bytes<HD>(), NH = HD / 64, SBO = NH * 1024, PAGE = 2 * SBO, R = kCkRing;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  struct Bars {
    uint64_t kfull[R], vfull[R], kempty[R], vempty[R], qfull, qempty, sfull[2], hdone[2], pfull[2][2], ofull[2], oempty[2], part[2], join, met[4],
        mma, dfull[kCkPieces], dempty[kCkPieces], done[2], ifull[kCkAhead], iempty[kCkAhead];
  };
  __shared__ Bars bar;
  __shared__ CkPiece s_piece[kCkPieces];
  __shared__ float2 s_ml[2][2][kCkKeys];         // [parity][group][row]: maximum and sum, units of one tile
  __shared__ uint32_t tmem_base;
  __shared__ CkPiece s_left[2];                  // units that other CTAs have a part of
  __shared__ int abort_word, s_last[2];
  __shared__ int2 s_page[KV8 ? kCkAhead : 1][8];  // int8: pool row of a tile's pages, and how many of their rows count
  __shared__ __align__(16) float s_scale[KV8 ? kCkScales : 1][2][kCkKeys];  // int8: K's (by hd^-1/2 log2 e) and V's
  volatile int* abort_flag = &abort_word;
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* sQ = smem;
  uint8_t* sK = smem + 2 * TILE;
  uint8_t* sV = sK + R * TILE;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto fail = [&]() {
    *abort_flag = 1;
    if (a.err) atomicExch(a.err, 2);
  };

  pdl_trigger();
  {
    // arrivals of each barrier, in their order
    constexpr int NB = sizeof(Bars) / 8;
    uint64_t* p = reinterpret_cast<uint64_t*>(&bar);
    for (int i = threadIdx.x; i < NB; i += ck_threads<KV8>()) {
      const uint64_t* q = p + i;
      int n = 1;
      if (q < bar.kempty) n = KV8 ? kCkWiden / 2 : 1;
      else if (q < &bar.qfull) n = 2;
      else if (q == &bar.qempty || q == &bar.mma) n = 2;
      else if (q >= &bar.pfull[0][0] && q < bar.ofull) n = 4;
      else if (q >= bar.oempty && q < bar.met) n = 8;  // oempty, part, join
      else if (q >= bar.met && q < &bar.mma) n = 2;
      else if (q >= bar.dempty && q < bar.done) n = kCkReaders;
      else if (q >= bar.iempty) n = kCkWiden;
      mbar_init(p + i, n);
    }
    if (threadIdx.x == 0) *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_wait();
  __syncthreads();

  // The next piece, for a whole warp; false: the stretch is done, or (ok false) a wait ran out.
  int pc = 0;
  auto next = [&](CkPiece& w, bool& ok) {
    const int i = pc % kCkPieces;
    ok = __all_sync(0xffffffffu, mbar_wait(&bar.dfull[i], (pc / kCkPieces) & 1)) && !*abort_flag;
    if (!__all_sync(0xffffffffu, ok)) return ok = false;
    w = s_piece[i];
    __syncwarp();
    if (lane == 0) mbar_arrive(&bar.dempty[i]);
    ++pc;
    return !w.done();
  };

  if (KV8 && warp >= kCkSoft) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
  if (warp == kCkWarpPlan || warp == kCkWarpQ) {
    // ---------------- warp 11: the plan, the pieces, V.  Warp 8: Q tiles and K.  Lanes
    // 0-7 copy a page of a key tile each; the next tile's page ids are read while this
    // one is in flight.  A page behind the sequence's end, or a bad one, reads zeros.
    const bool is_v = warp == kCkWarpPlan;
    const CUtensorMap* map = is_v ? &map_v : &map_k;
    uint64_t *full = is_v ? bar.vfull : bar.kfull, *empty = is_v ? bar.vempty : bar.kempty;
    uint8_t* dst = is_v ? sV : sK;
    int n = 0, kn = 0;
    bool ok = true;
    auto copy = [&](const CkPiece& w) {
      const int32_t* pt = a.page_table + (long long)w.b * a.pages_per_seq;
      // The Q tiles, behind the first key tile: that one goes out (and the widening of the
      // last unit's last tile, which looks a tile ahead, goes on) while Q is still in use.
      auto queries = [&]() {
        if (n > 0) ok = mbar_wait(&bar.qempty, (n - 1) & 1) && !*abort_flag;
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) return;
        if (lane == 0) {
          const int tiles = w.pair() ? 2 : 1;
          mbar_expect_tx(&bar.qfull, tiles * NH * a.tile_tokens * a.G * 128);
#pragma unroll 1
          for (int j = 0; j < tiles; ++j)
#pragma unroll
            for (int h = 0; h < NH; ++h)
              ck_tma_4d(sQ + j * TILE + h * (TILE / NH), &map_q, 0, h, w.kvh * a.G, w.row0 + j * a.tile_tokens, &bar.qfull);
        }
        ++n;
      };
      if constexpr (KV8) {
        // the tile's pages to the widening warps, its codes and scales to L2
        auto page = [&](int t) {
          const int key0 = t * kCkKeys + lane * 16;
          if (lane >= 8 || t >= w.t1 || key0 >= w.end) return -1;
          return __ldg(pt + key0 / 16);
        };
        int id = page(w.t0), at, rows;
        float ks[4], vs[4];
        // a tile's pages to L2, and its scales on their way: four keys' a lane, 0 for rows
        // that do not count
        auto fetch = [&](int t) {
          const int count = w.end - t * kCkKeys - lane * 16;
          at = -1;
          if (id >= 0 && id < a.n_pages) {
            at = (id * a.Hkv + w.kvh) * 16;
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(a.k8 + (long long)at * HD), "n"(16 * HD) : "memory");
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(a.v8 + (long long)at * HD), "n"(16 * HD) : "memory");
          } else if (lane < 8 && count > 0 && a.err) {
            atomicExch(a.err, 1);
          }
          rows = at < 0 ? 0 : min(16, max(0, count));
          const int first = __shfl_sync(0xffffffffu, at, lane >> 2) + (lane & 3) * 4;
          const int on = __shfl_sync(0xffffffffu, rows, lane >> 2) - (lane & 3) * 4;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            ks[i] = i < on ? __ldg(a.k_scale + first + i) : 0.f;
            vs[i] = i < on ? __ldg(a.v_scale + first + i) : 0.f;
          }
        };
        fetch(w.t0);
        id = page(w.t0 + 1);
        for (int t = w.t0; t < w.t1; ++t, ++kn) {
          const int s = kn % kCkAhead;
          const float c = kPaLog2e * rsqrtf((float)HD);
          const float4 kf = make_float4(ks[0] * c, ks[1] * c, ks[2] * c, ks[3] * c), vf = make_float4(vs[0], vs[1], vs[2], vs[3]);
          const int2 page_rows = make_int2(at, rows);
          if (t + 1 < w.t1) fetch(t + 1), id = page(t + 2);
          if (kn >= kCkAhead) ok = mbar_wait(&bar.iempty[s], ((kn / kCkAhead) & 1) ^ 1);
          ok = __all_sync(0xffffffffu, ok && !*abort_flag);
          if (!ok) return;
          *reinterpret_cast<float4*>(&s_scale[kn % kCkScales][0][lane * 4]) = kf;
          *reinterpret_cast<float4*>(&s_scale[kn % kCkScales][1][lane * 4]) = vf;
          if (lane < 8) s_page[s][lane] = page_rows;
          __syncwarp();
          if (lane == 0) mbar_arrive(&bar.ifull[s]);
          if (t == w.t0) queries();
          if (!ok) return;
        }
      } else {
        auto page = [&](int t) {
          const int key0 = t * kCkKeys + lane * 16;
          if (lane >= 8 || t >= w.t1 || key0 >= w.end) return -1;
          return __ldg(pt + key0 / 16);
        };
        int id = page(w.t0);
        for (int t = w.t0; t < w.t1; ++t) {
          const int s = kn % R, next_id = page(t + 1);
          const bool there = id >= 0 && id < a.n_pages;
          if (!there && !is_v && lane < 8 && t * kCkKeys + lane * 16 < w.end && a.err) atomicExch(a.err, 1);
          const int group = there ? (id * a.Hkv + w.kvh) * 2 : -2;  // of 8 pool rows; -2 reads zeros
          if (kn >= R) ok = mbar_wait(&empty[s], ((kn / R) & 1) ^ 1);
          ok = __all_sync(0xffffffffu, ok && !*abort_flag);
          if (!ok) return;
          if (lane == 0) mbar_expect_tx(&full[s], TILE);
          __syncwarp();
          if (lane < 8) ck_tma_4d(dst + s * TILE + lane * PAGE, map, 0, 0, 0, group, &full[s]);
          ++kn;  // in flight from here on, wherever this ends: the drain below waits for it
          id = next_id;
          if (!is_v && t == w.t0) queries();
          if (!ok) return;
        }
      }
    };
    if (is_v) {
      CkWalk walk(a);
      // piece m + 1 is described before the values of piece m are copied
      CkPiece w, w1;
      auto tell = [&](int m, CkPiece* p) {
        walk.next(p);
        const int i = m % kCkPieces;
        if (m >= kCkPieces) ok = __all_sync(0xffffffffu, mbar_wait(&bar.dempty[i], ((m / kCkPieces) & 1) ^ 1)) && !*abort_flag;
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          return;
        }
        if (lane == 0) {
          s_piece[i] = *p;
          mbar_arrive(&bar.dfull[i]);
        }
        __syncwarp();
      };
      tell(0, &w);
      for (int m = 0; ok && !w.done(); ++m) {
        tell(m + 1, &w1);
        if (ok && !w.empty() && !KV8) copy(w);
        w = w1;
      }
    } else {
      CkPiece w;
      while (next(w, ok)) {
        if (!w.empty()) copy(w);
        if (!ok) break;
      }
      if (KV8 && ok) {  // no more tiles
        const int s = kn % kCkAhead;
        if (kn >= kCkAhead) ok = __all_sync(0xffffffffu, mbar_wait(&bar.iempty[s], ((kn / kCkAhead) & 1) ^ 1));
        if (lane == 0) {
          s_page[s][0] = make_int2(-2, 0);
          mbar_arrive(&bar.ifull[s]);
        }
      }
    }
    if (!ok && lane == 0) fail();
    if (lane == 0) {  // copies still in flight land before the CTA leaves
      if (!is_v && n > 0) mbar_wait(&bar.qfull, (n - 1) & 1);
      if (!KV8)
        for (int t = max(0, kn - R); t < kn; ++t) mbar_wait(&full[t % R], (t / R) & 1);
    }
  } else if (warp == kCkWarpMma || warp == kCkWarpMma + 1) {
    // ---------------- MMA issuers, a group each: every lane runs the loop, one issues.
    // The group is a constant of the code that issues, the ring slot comes from a vote, and
    // an allocation of all 512 columns begins at column 0, so no operand has to be moved
    // to a uniform register MMA by MMA.
    if (warp == kCkWarpMma) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)),
                   "r"(kCkTmemCols)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
      tc_fence_before();
    }
    auto role = [&](auto cj) {
      constexpr int j = decltype(cj)::value;
      constexpr uint32_t idesc_s = tc_idesc(kCkKeys, kCkKeys), idesc_o = tc_idesc(kCkKeys, HD) | (1u << 16);
      const uint64_t qd = sdesc(smem_u32(sQ)), kd = ck_sdesc_k(smem_u32(sK), SBO),
                     vd = sdesc_mn(smem_u32(sV), 1024, SBO);
      int n = 0, kn = 0, pn = 0, on = 0;
      bool ok = true;
      // A vote's result is in a uniform register, and so is all that follows from it.
      auto uniform = [](bool b) { return __any_sync(0xffffffffu, b) ? 1 : 0; };
      // S_j = Q K^T of ring slot s (descriptor start addresses count 16-byte units)
      auto scores = [&](int q, int s) {
        const uint64_t qs = qd + q * (TILE >> 4), ks = kd + s * (TILE >> 4);
#pragma unroll 1
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            tc_mma(j * kCkKeys, qs + h * (TILE / NH >> 4) + kk * 2, ks + h * (1024 >> 4) + kk * 2, idesc_s, h + kk > 0 ? 1u : 0u);
        tc_commit(&bar.sfull[j]);
      };
      // O_j (+)= P_j V of ring slot s, half h of the keys: a page a step
      auto values = [&](int s, int h, bool first) {
        const uint64_t vs = vd + s * (TILE >> 4) + h * (4 * PAGE >> 4);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          tc_mma_ts(kCkO + j * 128, j * kCkKeys + h * 64 + kk * 8, vs + kk * (PAGE >> 4), idesc_o, kk > 0 || !first ? 1u : 0u);
      };
      CkPiece w;
      while (next(w, ok)) {
        const int steps = w.t1 - w.t0;
        if (steps <= 0) continue;
        const bool pair = w.pair();
        // this group's key tiles: piece tiles i0, i0 + di, .. below i1
        const int i0 = pair ? 0 : j, di = pair ? 1 : 2, i1 = pair && j == 0 ? w.e0 - w.t0 : steps;
        // the other group leaves tile i to this one: then both arrivals are this one's
        auto alone = [&](int i) { return !pair || (j == 1 && i >= w.e0 - w.t0); };
        auto release = [&](uint64_t* b, bool twice) {
          tc_commit(b);
          if (twice) tc_commit(b);
        };
        // both issuers have seen every tile of the pieces before (their phases are over)
        if (lane == 0) mbar_arrive(&bar.mma);
        ok = mbar_wait(&bar.mma, n & 1) && mbar_wait(&bar.qfull, n & 1) && !*abort_flag;
        if (i0 < i1) ok = ok && mbar_wait(&bar.kfull[(kn + i0) % R], ((kn + i0) / R) & 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        ++n;
        tc_fence_after();
        const bool q_alone = pair ? j == 1 && w.e0 <= w.t0 : steps == 1;  // the other group has no scores here
        const int q = uniform(j && pair);
        if (i0 < i1) {
          const int u = uniform((kn + i0) & 1);
          if (elect_one()) {
            scores(q, u);
            release(&bar.kempty[(kn + i0) % R], alone(i0));
            if (i0 + di >= i1) release(&bar.qempty, q_alone);
          }
          __syncwarp();
        }
        for (int i = i0; i < i1; i += di) {
          const int s = (kn + i) % R, s1 = (kn + i + di) % R;
          const bool more = i + di < i1;
          // V is there; (first tile) the last unit's output has been read
          ok = mbar_wait_n(&bar.vfull[s], ((kn + i) / R) & 1, a.wait_limit) &&
               (i > i0 || on == 0 || mbar_wait(&bar.oempty[j], (on - 1) & 1));
          // V rows behind the sequence's last position, zeroed before they are multiplied
          // (by both issuers where both read them)
          const int lo = w.end - (w.t0 + i) * kCkKeys;
          if (!KV8 && lo < kCkKeys && (lo & 15)) {
            for (int x = (lo & 15) * (HD / 8) + lane; x < 16 * (HD / 8); x += 32) {
              const int r = x / (HD / 8), c = x % (HD / 8);  // whole rows: the swizzle stays inside them
              *reinterpret_cast<uint4*>(sV + s * TILE + (lo >> 4) * PAGE + (r >> 3) * SBO + (c >> 3) * 1024 + (r & 7) * 128 +
                                        (c & 7) * 16) = make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async();
          }
          if (more) ok = ok && mbar_wait(&bar.kfull[s1], ((kn + i + di) / R) & 1);
          const int u = uniform(s), u1 = uniform(s1), first = uniform(i == i0);
          // a half of the keys: P V, then the next tile's scores over the columns that P leaves
          auto half = [&](auto ch) {
            constexpr int h = decltype(ch)::value;
            ok = __all_sync(0xffffffffu, ok && mbar_wait(&bar.pfull[j][h], pn & 1)) && !*abort_flag;
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) return;
            tc_fence_after();
            if (elect_one()) {
              values(u, h, h == 0 && first);
              if (h == 0) {
                tc_commit(&bar.hdone[j]);
              } else {
                release(&bar.vempty[s], alone(i));
                if (more) {
                  scores(q, u1);
                  release(&bar.kempty[s1], alone(i + di));
                  if (i + 2 * di >= i1) release(&bar.qempty, q_alone);
                } else {
                  tc_commit(&bar.ofull[j]);
                }
              }
            }
            __syncwarp();
          };
          half(std::integral_constant<int, 0>());
          half(std::integral_constant<int, 1>());
          if (!ok) break;
          ++pn;
        }
        if (!ok) break;
        on += i0 < i1;
        kn += steps;
      }
      if (!ok && lane == 0) fail();
      if (elect_one()) tc_commit(&bar.done[j]);
      __syncwarp();
      mbar_wait(&bar.done[j], 0);
    };
    if (warp == kCkWarpMma) role(std::integral_constant<int, 0>());
    else role(std::integral_constant<int, 1>());
  } else if (KV8 && warp >= kCkWarpWiden) {
    // ---------------- int8 cache: the codes of the key tiles' rows as bf16, four warps for K
    // and four for V.  Thread: 16 codes (chunk c) of every PER-th row.  Each register of codes
    // is filled again, for the next tile, as soon as it has been written out: a whole
    // tile's codes, 32 KB an SM, are in flight throughout, across pieces too.
    constexpr int C = HD / 16;                                      // chunks a row
    constexpr int PER = 16 * kCkWiden / C, N = kCkKeys / PER;       // rows at a time, turns a tile
    const bool is_v = warp >= kCkWarpWiden + kCkWiden / 2;
    // four chunks of two rows go out at a time, whose swizzles differ: eight banks of 16 bytes
    const int wi = threadIdx.x % (16 * kCkWiden), c = C == 4 ? wi & 3 : (wi & 3) | (wi >> 1 & 4);
    const int rr = C == 4 ? wi >> 2 : (wi >> 4) * 2 + (wi >> 2 & 1);
    const int8_t* pool = (is_v ? a.v8 : a.k8) + c * 16;
    uint64_t *full = is_v ? bar.vfull : bar.kfull, *empty = is_v ? bar.vempty : bar.kempty;
    uint8_t* tiles = (is_v ? sV : sK) + (rr >> 3) * SBO + (c >> 2) * 1024 + (rr & 7) * 128;
    const int o0 = ((2 * (c & 3)) ^ (rr & 7)) << 4, o1 = ((2 * (c & 3) + 1) ^ (rr & 7)) << 4;
    uint4 cw[N];
    int row[N];  // pool rows (fewer than 2^31) of the tile to be read; -1 reads zeros
    bool ok = true;
    // this thread's rows of tile k; false: there is none (or a wait ran out)
    auto rows = [&](int k) {
      const int s = k % kCkAhead;
      ok = __all_sync(0xffffffffu, mbar_wait(&bar.ifull[s], (k / kCkAhead) & 1));
      const bool there = ok && s_page[s][0].x != -2;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = i * PER + rr;
        const int2 p = s_page[s][r >> 4];
        row[i] = there && (r & 15) < p.y ? p.x + (r & 15) : -1;
      }
      return there;
    };
    auto fetch = [&](int i) {
      cw[i] = row[i] >= 0 ? ld_nc16(pool + (long long)row[i] * HD) : make_uint4(0, 0, 0, 0);
    };
    bool more = rows(0);
#pragma unroll
    for (int i = 0; i < N; ++i) fetch(i);
    for (int kn = 0; more; ++kn) {
      const int s = kn % R;
      more = rows(kn + 1);
      if (kn >= R) ok = __all_sync(0xffffffffu, ok && mbar_wait(&empty[s], ((kn / R) & 1) ^ 1));
      if (!ok) break;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint32_t ww[4] = {cw[i].x ^ 0x80808080u, cw[i].y ^ 0x80808080u, cw[i].z ^ 0x80808080u, cw[i].w ^ 0x80808080u};
        const float2 z2 = make_float2(-32896.f, -32896.f);
        uint32_t o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {  // codes 2j, 2j + 1: fp32 2^15 + 128 + q
          const uint32_t u = ww[j >> 1];
          const float lo = __uint_as_float(__byte_perm(u, 0x47000000u, (j & 1) ? 0x7424 : 0x7404));
          const float hi = __uint_as_float(__byte_perm(u, 0x47000000u, (j & 1) ? 0x7434 : 0x7414));
          const float2 f = pa_add2(make_float2(lo, hi), z2);
          o[j] = pa_pack(f.x, f.y);
        }
        uint8_t* rp = tiles + s * TILE + i * (PER / 8 * SBO);
        *reinterpret_cast<uint4*>(rp + o0) = make_uint4(o[0], o[1], o[2], o[3]);
        *reinterpret_cast<uint4*>(rp + o1) = make_uint4(o[4], o[5], o[6], o[7]);
        fetch(i);
      }
      fence_proxy_async();  // the MMAs read the tile through the async proxy
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&full[s]);
        mbar_arrive(&bar.iempty[kn % kCkAhead]);
      }
    }
    if (!ok && lane == 0) fail();
  } else if (warp < kCkSoft) {
    // ---------------- softmax: group j, row 32 quad + lane (TMEM begins at column 0)
    if (KV8) asm volatile("setmaxnreg.inc.sync.aligned.u32 128;");
    const int j = warp >> 2, quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
    const uint32_t ts = lane_base + j * kCkKeys, to = lane_base + kCkO + j * 128;
    const float scale = kPaLog2e * rsqrtf((float)HD);
    const int tok = row / a.G;  // of a tile's packed rows
    const bool packed = row < a.tile_tokens * a.G;
    int sn = 0, on[2] = {0, 0}, mn = 0, left = 0, kb = 0;
    bool ok = true;
    uint8_t* stage = sV + R * TILE + warp * kCkStage;
    constexpr size_t ML = (size_t)kCkRows * HD * 4;
    auto slot = [&](const CkPiece& w, int i) {  // part i of a unit
      return a.ws + kCkHead + ((size_t)(w.own + i) * 2 + (i == 0 ? 1 : 0)) * ck_slot<HD>();
    };
    // row block rb (32 of a unit's packed rows, one a lane), columns x .. x + 31, to a slot
    auto keep = [&](uint8_t* p, int rb, int x, const float* r) {
#pragma unroll
      for (int y = 0; y < 8; ++y)
        reinterpret_cast<float4*>(p)[(size_t)(x / 4 + y) * kCkRows + rb * 32 + lane] =
            make_float4(r[4 * y], r[4 * y + 1], r[4 * y + 2], r[4 * y + 3]);
    };
    // where rows 8 y + lane / 4 of a row block begin in the unit's output, or -1
    auto begins = [&](const CkPiece& w, int rb, int* at) {
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int r2 = (rb & 3) * 32 + y * 8 + (lane >> 2), t2 = r2 / a.G, t = t2 + (rb >> 2) * a.tile_tokens;
        at[y] = t2 < a.tile_tokens && t < w.n ? (t * a.H + r2 - t2 * a.G) * HD : -1;
      }
    };
    // ... to out, times inv, through shared memory: four lanes to a row's 64 bytes; chunk c
    // of row r at c ^ (r / 2 % 4)
    auto write = [&](const CkPiece& w, const int* at, int x, const float* r, float inv) {
      uint16_t* o = a.out + ((long long)w.row0 * a.H + (long long)w.kvh * a.G) * HD;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t p[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) p[y] = pa_pack(r[8 * c + 2 * y] * inv, r[8 * c + 2 * y + 1] * inv);
        *reinterpret_cast<uint4*>(stage + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4)) = make_uint4(p[0], p[1], p[2], p[3]);
      }
      __syncwarp();
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int lr = y * 8 + (lane >> 2);
        const uint4 p = *reinterpret_cast<const uint4*>(stage + lr * 64 + (((lane & 3) ^ ((lr >> 1) & 3)) << 4));
        if (at[y] >= 0) *reinterpret_cast<uint4*>(o + at[y] + x + (lane & 3) * 8) = p;
      }
      __syncwarp();
    };
    // This CTA's part of s_left[left - 1] is written: by the last of its group of parts?
    // (One thread asks; the answer is read behind a meeting of the warps.)
    int jn = 0;
    bool behind = false;
    auto ticket = [&]() {
      if (warp == 0) {
        ok = __all_sync(0xffffffffu, mbar_wait(&bar.part[left - 1], 0));
        if (lane == 0 && ok) {
          const CkPiece& p = s_left[left - 1];
          const int mine = (blockIdx.x - p.own) / kCkGroup;
          int* t = reinterpret_cast<int*>(a.ws) + p.own * kCkTickets + mine;
          const bool last = atomicAdd(t, 1) == min(kCkGroup, p.parts - mine * kCkGroup) - 1;
          if (last) *t = 0;
          s_last[left - 1] = last;
        }
        __syncwarp();
      }
      behind = false;
    };
    CkPiece w;
    while (next(w, ok)) {
      const bool pair = w.pair();
      const int jq = pair ? j : 0;  // this group's query tile
      const int tile_n = min(a.tile_tokens, w.n - jq * a.tile_tokens), tile_pos = w.pos + jq * a.tile_tokens;
      const bool on_row = packed && tok < tile_n;
      const bool on_warp = __any_sync(0xffffffffu, on_row);
      // keys of this row, and of the tile's first
      const int lim = on_row ? min(w.end, tile_pos + tok + 1) : 0, lim0 = min(w.end, tile_pos + 1);
      const int t_end = jq == 0 && pair ? w.e0 : w.t1, t_first = pair ? w.t0 : w.t0 + j, stride = pair ? 1 : 2;
      float m = -INFINITY;  // reference maximum (log2 domain)
      float2 l2[4];         // row sum
#pragma unroll
      for (int y = 0; y < 4; ++y) l2[y] = make_float2(0.f, 0.f);
      // Half a tile of keys at a time: while one half's scores are here, the products of
      // the other run.
#pragma unroll 1
      for (int t = t_first; t < t_end && ok; t += stride, ++sn) {
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          if (h == 0) {
            ok = __all_sync(0xffffffffu, mbar_wait(&bar.sfull[j], sn & 1));
            if (!ok) break;
            if (behind && t > t_first) ticket();
          }
          if (!on_warp) {
            if (lane == 0) mbar_arrive(&bar.pfull[j][h]);
            continue;
          }
          tc_fence_after();
          // The 64 scores stay in registers, the loop over the halves is rolled: the maximum
          // of all 128 first, and the scores read again, took 80 us where this takes 77
          // (chunk bf16); all 128 in registers, this loop, the issuers' and the widening ones
          // were more than the instruction caches hold.
          const int key0 = t * kCkKeys + h * 64, seen = lim - key0;  // keys of this half that are the row's
          const bool masked = key0 + 64 > lim0;
          const uint32_t tsh = ts + h * 64;
          const float* sc = KV8 ? &s_scale[(kb + t - w.t0) % kCkScales][0][h * 64] : nullptr;  // (V's kCkKeys on)
          float v[64];  // scores (int8 cache: times their keys' K scales)
          tc_ld<64>(tsh, reinterpret_cast<uint32_t*>(v));
          if constexpr (KV8) {
#pragma unroll
            for (int x = 0; x < 64; x += 4) {
              const float4 f = *reinterpret_cast<const float4*>(sc + x);
              const float2 p = pa_mul2(make_float2(v[x], v[x + 1]), make_float2(f.x, f.y));
              const float2 q = pa_mul2(make_float2(v[x + 2], v[x + 3]), make_float2(f.z, f.w));
              v[x] = p.x, v[x + 1] = p.y, v[x + 2] = q.x, v[x + 3] = q.y;
            }
          }
          if (masked) {
#pragma unroll
            for (int x = 0; x < 64; ++x)
              if (x >= seen) v[x] = -INFINITY;
          }
          float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int x = 0; x < 64; x += 8)
#pragma unroll
            for (int y = 0; y < 4; ++y) m4[y] = ck_max3(m4[y], v[x + 2 * y], v[x + 2 * y + 1]);
          const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * (KV8 ? 1.f : scale);
          // move the reference when the tile would exceed it by more than 2^kCkSlack
          float corr = 1.f;
          if (mx > m + kCkSlack) {
            corr = exp2f(m - mx);  // 0 on the first tile
            m = mx;
#pragma unroll
            for (int y = 0; y < 4; ++y) l2[y] = pa_mul2(l2[y], make_float2(corr, corr));
          }
          if ((h || t > t_first) && __any_sync(0xffffffffu, corr != 1.f)) {
            // O holds P V of the halves before: those of earlier tiles are complete (this one's
            // scores were issued after them)
            if (h) ok = __all_sync(0xffffffffu, mbar_wait(&bar.hdone[j], sn & 1));
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int x = 0; x < HD; x += 16) {
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
          for (int x0 = 0; x0 < 64; x0 += 32) {  // P (int8 cache: times the V scales)
            uint32_t pw[16];
#pragma unroll
            for (int x = x0; x < x0 + 32; x += 4) {
              float4 f;
              if constexpr (KV8) f = *reinterpret_cast<const float4*>(sc + kCkKeys + x);
#pragma unroll
              for (int y = 0; y < 4; y += 2) {
                const float2 s2 = make_float2(v[x + y], v[x + y + 1]), e = KV8 ? pa_add2(s2, nm2) : pa_fma2(s2, sc2, nm2);
                float2 p = make_float2(pa_ex2(e.x), pa_ex2(e.y));
                l2[(x + y) / 2 % 4] = pa_add2(l2[(x + y) / 2 % 4], p);
                if constexpr (KV8) p = pa_mul2(p, y ? make_float2(f.z, f.w) : make_float2(f.x, f.y));
                pw[(x - x0 + y) / 2] = pa_pack(p.x, p.y);
              }
            }
            tc_st16(tsh + x0 / 2, pw);
          }
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bar.pfull[j][h]);
        }
      }
      if (!ok) break;
      float l = ((l2[0].x + l2[0].y) + (l2[1].x + l2[1].y)) + ((l2[2].x + l2[2].y) + (l2[3].x + l2[3].y));
      kb += max(0, w.t1 - w.t0);
      // ---- the piece's output
      const bool whole = w.first() && w.last(), empty = w.empty();
      const bool use0 = w.uses(0), use1 = w.uses(1);
      float a0 = 1.f, a1 = 0.f;  // factors of O_0 and O_1 (units of one tile)
      if (pair) {
        if (j ? use1 : use0) {
          ok = __all_sync(0xffffffffu, mbar_wait(&bar.ofull[j], (j ? on[1] : on[0]) & 1));
          if (!ok) break;
        }
        on[0] += use0, on[1] += use1;
      } else if (!empty) {
        // every warp meets here, those without rows too: past this point both groups
        // have seen the accumulators of the pieces before
        s_ml[mn & 1][j][row] = make_float2(m, l);
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar.met[quad]);
        ok = mbar_wait(&bar.met[quad], mn & 1);
        ok = __all_sync(0xffffffffu, ok && mbar_wait(&bar.ofull[0], on[0] & 1) && (!use1 || mbar_wait(&bar.ofull[1], on[1] & 1)));
        if (!ok) break;
        ++on[0];
        on[1] += use1;
        const float2 p0 = s_ml[mn & 1][0][row], p1 = s_ml[mn & 1][1][row];
        ++mn;
        m = fmaxf(p0.x, p1.x);
        a0 = p0.x == -INFINITY ? 0.f : exp2f(p0.x - m);
        a1 = p1.x == -INFINITY ? 0.f : exp2f(p1.x - m);
        l = a0 * p0.y + a1 * p1.y;
      }
      tc_fence_after();
      const bool have = pair ? (j ? use1 : use0) : !empty;  // an accumulator to read
      const float inv = l == 0.f ? 0.f : 1.f / l;  // (a row without keys: zeros)
      // pair: this group's tile, all columns; else half of the sum's columns a group
      const int x0 = pair ? 0 : j * (HD / 2), x1 = pair ? HD : x0 + HD / 2;
      const uint32_t src = pair ? to : lane_base + kCkO;
      auto load = [&](int x, float* r) {  // 32 columns of the sums
        if (!have) {
#pragma unroll
          for (int y = 0; y < 32; ++y) r[y] = 0.f;
          return;
        }
        tc_ld<32>(src + x, reinterpret_cast<uint32_t*>(r));
        if (pair) return;
#pragma unroll
        for (int y = 0; y < 32; ++y) r[y] *= a0;
        if (!use1) return;
#pragma unroll
        for (int y0 = 0; y0 < 32; y0 += 16) {
          uint32_t u[16];
          tc_ld<16>(src + 128 + x + y0, u);
#pragma unroll
          for (int y = 0; y < 16; ++y) r[y0 + y] = fmaf(a1, __uint_as_float(u[y]), r[y0 + y]);
        }
      };
      if (on_warp) {
        const int rb = jq * 4 + quad;
        if (whole) {
          int at[4];
          begins(w, rb, at);
#pragma unroll 1
          for (int x = x0; x < x1; x += 32) {
            float r[32];
            load(x, r);
            write(w, at, x, r, inv);
          }
        } else {
          uint8_t* p = slot(w, blockIdx.x - w.own);
          if (have)
#pragma unroll 1
            for (int x = x0; x < x1; x += 32) {
              float r[32];
              load(x, r);
              keep(p, rb, x, r);
            }
          // A part without keys of the row has l = 0 and is marked by -inf: the join leaves it
          // out.  One with a NaN score has a NaN l, and no reference where there was no other:
          // any finite one hands the NaN on.
          if (x0 == 0) {
            const float ls = have ? l : 0.f;
            reinterpret_cast<float2*>(p + ML)[rb * 32 + lane] =
                make_float2(ls == 0.f ? -INFINITY : m == -INFINITY ? 0.f : m, ls);
          }
        }
      }
      if (have) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (pair) {  // the 8 arrivals of an accumulator: two from each of its own group's warps
            mbar_arrive(&bar.oempty[j]);
            mbar_arrive(&bar.oempty[j]);
          } else {
            mbar_arrive(&bar.oempty[0]);
            if (use1) mbar_arrive(&bar.oempty[1]);
          }
        }
      }
      if (!whole) {
        if (behind) ticket();
        if (threadIdx.x == 0) s_left[left] = w;
        ++left;
        // (the ticket waits for a tile of the next piece, by when every warp is here)
        __threadfence();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar.part[left - 1]);
        behind = true;
      }
    }
    // ---- units that other CTAs have a part of (at most two: the stretch's first and
    // last): o = sum 2^(m_i - m) O_i / sum 2^(m_i - m) l_i over the unit's parts, in their
    // order, by the last CTA to bring its part: first among kCkGroup neighbours, then (a
    // unit that more CTAs share) the last group among the groups.
    auto meet = [&]() {
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar.join);
      ok = ok && __all_sync(0xffffffffu, mbar_wait(&bar.join, jn++ & 1));
    };
    if (left > 0 && ok) {
      if (behind) ticket();
      meet();
      __threadfence();
    }
    for (int k = 0; k < left && ok; ++k) {
      if (!s_last[k]) continue;
      w = s_left[k];
      const int groups = (w.parts + kCkGroup - 1) / kCkGroup;
      int i0 = (blockIdx.x - w.own) / kCkGroup * kCkGroup, step = 1, n = min(kCkGroup, w.parts - i0);
      size_t ml_at = ML;
      // the unit's rows by 32, 32 columns at a time, over the warps
      const int rows = w.pair() ? kCkKeys + (w.n - a.tile_tokens) * a.G : w.n * a.G;
      for (int turn = groups > 1 ? 0 : 1; turn < 2 && ok; ++turn) {
#pragma unroll 1
        for (int item = warp; item < (rows + 31) / 32 * (HD / 32); item += kCkSoft) {
          const int rb = item / (HD / 32), x = item % (HD / 32) * 32;
          float mm = -INFINITY, ll = 0.f, r[32];
#pragma unroll
          for (int y = 0; y < 32; ++y) r[y] = 0.f;
#pragma unroll 2
          for (int i = 0; i < n; ++i) {
            const uint8_t* p = slot(w, i0 + i * step);
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(p + ml_at) + rb * 32 + lane);
            float4 f[8];
#pragma unroll
            for (int y = 0; y < 8; ++y) f[y] = __ldcg(reinterpret_cast<const float4*>(p) + (size_t)(x / 4 + y) * kCkRows + rb * 32 + lane);
            if (ml.x == -INFINITY) continue;  // (its O may not have been written)
            const float m2 = fmaxf(mm, ml.x), c0 = exp2f(mm - m2), c1 = exp2f(ml.x - m2);
            mm = m2;
            ll = ll * c0 + ml.y * c1;
#pragma unroll
            for (int y = 0; y < 8; ++y) {
              r[4 * y] = r[4 * y] * c0 + f[y].x * c1, r[4 * y + 1] = r[4 * y + 1] * c0 + f[y].y * c1;
              r[4 * y + 2] = r[4 * y + 2] * c0 + f[y].z * c1, r[4 * y + 3] = r[4 * y + 3] * c0 + f[y].w * c1;
            }
          }
          if (turn == 0) {
            keep(slot(w, i0), rb, x, r);
            if (x == 0) reinterpret_cast<float2*>(slot(w, i0) + ML + kCkRows * 8)[rb * 32 + lane] = make_float2(mm, ll);
          } else {
            int at[4];
            begins(w, rb, at);
            write(w, at, x, r, ll == 0.f ? 0.f : 1.f / ll);
          }
        }
        if (turn == 0) {
          __threadfence();
          meet();
          if (threadIdx.x == 0) {
            int* t = reinterpret_cast<int*>(a.ws) + w.own * kCkTickets + kCkTickets - 1;
            const bool last = atomicAdd(t, 1) == groups - 1;
            if (last) *t = 0;
            s_last[k] = last;
          }
          meet();
          __threadfence();
          if (!s_last[k]) break;
          i0 = 0, step = kCkGroup, n = groups, ml_at = ML + kCkRows * 8;
        }
      }
    }
    if (!ok && lane == 0) fail();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kCkWarpMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kCkTmemCols) : "memory");
  }
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
    sms = kCkMaxCtas;
  return sms;
}

// The plan's places and a unit's places in the output are 32-bit.
bool attention_chunk_fits(int n_tokens, int B, int n_heads, int n_kv_heads, int head_dim, int max_len) {
  const int T = ck_tile_tokens(n_heads / n_kv_heads);
  return ck_fits(n_tokens, B, max_len, n_kv_heads, T) && 2LL * T * n_heads * head_dim < (1LL << 31);
}

size_t attention_chunk_ws_bytes(int B, int n_heads, int n_kv_heads, int head_dim, int max_new) {
  return kCkHead + (size_t)2 * kCkMaxCtas * (head_dim == 64 ? ck_slot<64>() : ck_slot<128>());
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
  return launch(attn_chunk_kernel<HD, KV8>, dim3(std::min(ck_sms(), kCkMaxCtas)), dim3(ck_threads<KV8>()),
                (size_t)ck_smem<HD>(), s, mq, mk, mv, a);
}

// Of the launches that follow (lowered by tests of the failure path; other waits keep
// kTcSpinLimit, so that copies and MMAs in flight are drained).
static std::atomic<long long> g_ck_wait_limit{kTcSpinLimit};
void attention_chunk_wait_limit(long long rounds) { g_ck_wait_limit.store(rounds, std::memory_order_relaxed); }

cudaError_t launch_attention_chunk(const uint16_t* q, int q_stride, int n_tokens, int B, int n_heads,
                                   const fp_kv_view& kv, const int32_t* cu, const int32_t* pos, int max_new, int max_len,
                                   uint16_t* out, void* ws, int32_t* err, cudaStream_t s) {
  if (n_tokens <= 0 || B <= 0) return cudaSuccess;
  const int G = n_heads / kv.n_kv_heads;
  const CkArgs a = {cu, pos, n_tokens, B, n_heads, kv.n_kv_heads, G, max_new, max_len, ck_tile_tokens(G), kv.page_table,
                    kv.pages_per_seq, kv.n_pages, (const int8_t*)kv.k_pool, (const int8_t*)kv.v_pool, kv.k_scale, kv.v_scale,
                    out, (uint8_t*)ws, err, g_ck_wait_limit.load(std::memory_order_relaxed)};
  if (kv.head_dim == 64)
    return kv.kvquant == FP_KV_INT8 ? launch_ck<64, true>(q, q_stride, kv, a, s) : launch_ck<64, false>(q, q_stride, kv, a, s);
  return kv.kvquant == FP_KV_INT8 ? launch_ck<128, true>(q, q_stride, kv, a, s) : launch_ck<128, false>(q, q_stride, kv, a, s);
}

}  // namespace fpk
