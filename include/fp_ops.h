/*
 * fp_ops.h -- one C entry point per step of the fingerprint forward pass.
 *
 * These are the kernels the fingerprint runtime (fp.h) strings together,
 * exposed one by one on caller-owned DEVICE buffers so each step can be
 * checked against the oracle and timed alone.  Steps follow the decoder
 * block the fingerprint keeps from its LLM (arXiv 2501.13111, Sec. 1 "Our
 * work", Sec. 5.1) under the deployment configurations of Sec. 3.2 (weight
 * and KV-cache quantisation).
 *
 * Conventions:
 *   - Every pointer argument is a device pointer unless its name starts
 *     with host_.  Buffers are row-major; bf16 is passed as its uint16 bits.
 *   - The launch is asynchronous on `stream` (cudaStream_t, NULL = legacy
 *     default stream).  Arguments are checked on the host before any launch:
 *     FP_ERR_INVALID_ARG / FP_ERR_UNSUPPORTED and nothing is launched.
 *     FP_ERR_CUDA if the launch itself fails.  Nothing is allocated.
 *   - Output buffers must not overlap inputs unless a function says so.
 *   - Return codes are the FP_* codes of fp.h.
 */
#ifndef FP_OPS_H
#define FP_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "fp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Quantise a bf16 weight matrix w [N][K] into the wquant format of fp.h
 * (Sec. 3.2; formats in fp.h).  int8: codes int8 [N][K], scales bf16 [N].
 * int4: codes uint8 [N][K/2], scales and zeros bf16 [N][K/128]; K % 128 == 0.
 * bf16: codes receives a copy of w.  Codes are bit-exact with the reading
 * (fp32 IEEE division, round half to even). */
int fp_op_quantize(int wquant, const uint16_t* w, int N, int K, void* codes, uint16_t* scales,
                   uint16_t* zeros, void* stream);

/* Quantise w [N][K] (bf16) into the FP_W_GPTQ4 format of fp.h: int4 over
 * the act-order groups of perm (int32 [K], a permutation of 0..K-1; group g
 * holds the channels perm[128g .. 128g+127]), codes stored in act order
 * ([N][K/2], the int4 packing), scales and zeros bf16 [N][K/128]
 * (GPTQ4, Sec. 3.2 and the table "Models and configurations").  K % 128 ==
 * 0.  An entry of perm outside [0, K) reads as a zero weight. */
int fp_op_quantize_gptq4(const uint16_t* w, int N, int K, const int32_t* perm, void* codes, uint16_t* scales,
                         uint16_t* zeros, void* stream);

/* Fill w [n] with the seeded bf16 weights of stream `stream_id` (SplitMix64
 * counter-based draws, Irwin-Hall(4), sigma 0.02; elements start..start+n-1). */
int fp_op_init_weights(uint16_t* w, long long n, unsigned long long seed, long long stream_id,
                       long long start, void* stream);

/* Epilogues of fp_op_linear. */
enum {
  FP_EPI_STORE = 0,  /* y bf16 [M][N]                                          */
  FP_EPI_RESID = 1,  /* y bf16 [M][N] = residual + x W^T; residual may equal y  */
  FP_EPI_SWIGLU = 2, /* W rows = [gate (N/2 rows); up (N/2 rows)];
                        y bf16 [M][N/2] = silu(x Wg^T) * (x Wu^T)             */
  FP_EPI_F32 = 3     /* y fp32 [M][N]                                          */
};

/* Weight-only linear y = x W^T (the "linear layers" of the block) with the
 * dequantisation fused: x bf16 [M][K]; W in the wquant format of fp.h
 * (codes / scales / zeros as fp_op_quantize writes them); fp32 accumulation.
 * Kernel choice depends on M, N, K and the pointers' alignment.  M <= 64, decode: by
 * default the GEMV on mma.sync with the codes dequantised in registers (the work is
 * cut into equal ranges of (128-row block, K step), one per resident CTA, and shared
 * blocks are reduced from fp32 partials in a fixed order; smaller matrices give each
 * block a cluster of CTAs that add in rank order; gemv_cluster).  It stages x for int8 and
 * int4 codes as fp16.  With 16-byte aligned x and codes instead, on tcgen05:
 *   int4, M <= 16 and, with SwiGLU, M <= 32, a bf16 result, larger matrices (f8_pays;
 *     scales and zeros 16-byte aligned too): 8-bit operands, the codes as they are; x split by a first kernel
 *     into two e4m3 pieces an element, which carry it exactly down to 2^-13 of the
 *     largest value of its row and group of 128 channels and to 2^-22 of that value
 *     below; scales and zero points applied in fp32; a row of x that holds an infinity
 *     or a NaN gives NaN; where that would lose more than 2^-10 of a row, or a row holds
 *     an infinity or a NaN, M >= 17 runs again on the next kernel;
 *   int4, M >= 17 (scales and zeros 16-byte aligned too): each weight expanded in TMEM
 *     to bf16((q - z) s) as the prefill GEMM does;
 *   int8, M >= 33, and from 17 long rows and larger matrices (q4tc_preferred): codes
 *     expanded in TMEM, the row scale applied to the fp32 sums;
 *   bf16, M >= 17, larger matrices (btc_preferred): fed by TMA.
 * A K that is not a multiple of the
 * GEMV's K step falls back to one warp per output row on the CUDA cores.
 * M > 64, prefill: the tcgen05 GEMM.  For M > 64 with int8
 * or int4 weights the GEMM either reads a bf16 expansion of W that it writes
 * into the workspace band by band (at most 128 MB; the faster path), or, when
 * the workspace is NULL or smaller than that, dequantises the codes inside
 * the GEMM (bf16 weight tiles built in shared memory for every 256-token
 * tile; no workspace; about two thirds of the speed; x and codes 16-byte
 * aligned).  workspace: 16-byte aligned, at least
 * fp_op_linear_workspace_bytes(wquant, M, N, K) bytes (may be NULL when that
 * is 0, or for the in-kernel dequantisation above), else FP_ERR_INVALID_ARG.
 * Its leading bytes are ticket counters
 * that must be zero before the first call (e.g. a zeroed buffer); every call
 * leaves them zero again, so one workspace serves any sequence of calls on
 * one stream (calls that overlap on the GPU need separate workspaces). */
int fp_op_linear(int wquant, int epilogue, const uint16_t* x, int M, int N, int K, const void* codes,
                 const uint16_t* scales, const uint16_t* zeros, const uint16_t* residual, void* y,
                 void* workspace, size_t workspace_bytes, void* stream);
size_t fp_op_linear_workspace_bytes(int wquant, int M, int N, int K);

/* The weight-only linear of fp_op_linear for FP_W_GPTQ4 weights (codes,
 * scales, zeros as fp_op_quantize_gptq4 writes them; perm the act order).
 * y = x W^T with W in channel order.  M <= 64: x is gathered into the act
 * order in the workspace (one kernel, which also splits it where the linear
 * takes 8-bit operands) and the int4 decode linear runs on it;
 * M > 64: the weights are expanded back into channel order (the inverse act
 * order is computed into the workspace) and the prefill GEMM multiplies x as
 * it is.  workspace: 256-byte aligned, at least
 * fp_op_linear_gptq4_workspace_bytes(M, N, K) bytes, its leading ticket
 * counters zero before the first call (every call leaves them zero).  An
 * entry of perm outside [0, K) reads as zero and sets *err = 1 (err may be
 * NULL).  K % 128 == 0 (FP_ERR_UNSUPPORTED). */
int fp_op_linear_gptq4(int epilogue, const uint16_t* x, int M, int N, int K, const int32_t* perm, const void* codes,
                       const uint16_t* scales, const uint16_t* zeros, const uint16_t* residual, void* y,
                       void* workspace, size_t workspace_bytes, int32_t* err, void* stream);
size_t fp_op_linear_gptq4_workspace_bytes(int M, int N, int K);

/* RMSNorm of selected rows: y[r] = x[r*row_stride + row_offset] /
 * sqrt(mean(x^2) + eps) * g, r < M; x, y, g bf16; fp32 arithmetic. */
int fp_op_rmsnorm(const uint16_t* x, int M, int d, int row_stride, int row_offset, const uint16_t* g,
                  float eps, uint16_t* y, void* stream);

/* Embedding gather h[m] = E[tok[m]]; tok int32 [M], E bf16 [V][d].  An id
 * outside [0, V) writes a zero row and sets *err = 1 (err may be NULL). */
int fp_op_embed(const int32_t* tok, int M, const uint16_t* E, int V, int d, uint16_t* h, int32_t* err,
                void* stream);

/* Paged KV cache view.  Pools are [n_pages][n_kv_heads][page_size][head_dim]
 * (bf16 or int8 codes); scales (int8 only) fp32 [n_pages][n_kv_heads][page_size];
 * page_table int32 [batch][pages_per_seq]: position p of sequence b lives in
 * page page_table[b][p / page_size], slot p % page_size. */
typedef struct fp_kv_view {
  int kvquant, n_kv_heads, head_dim, page_size, pages_per_seq, n_pages;
  void* k_pool;
  void* v_pool;
  float* k_scale;
  float* v_scale;
  const int32_t* page_table;
} fp_kv_view;

/* RoPE table for positions 0..max_pos-1: cs fp32 [max_pos][head_dim/2][2] =
 * (cos, sin) of p * base^(-2i/hd), computed on the host in fp64 and rounded
 * to fp32, then copied to the device (synchronous). */
int fp_op_rope_table(int max_pos, int head_dim, float base, float* cs, void* stream);

/* RoPE + KV-cache append.  qkv bf16 [B*S][row_stride]: per token, H query
 * heads, then Hkv key heads, then Hkv value heads, head_dim each.  Token s
 * of sequence b sits at position pos[b] + s.  Query and key heads are
 * rotated (rotate-half); queries are written back in place; keys (rotated,
 * rounded to bf16) and values go to the cache, quantised per (token, KV
 * head) when kvquant is int8.  rope_cs (fp_op_rope_table) must cover
 * pages_per_seq * page_size positions.  A position outside
 * [0, pages_per_seq * page_size) or a page id outside the pool sets
 * *err = 1 (err may be NULL) and skips that head. */
int fp_op_rope_kv(uint16_t* qkv, int B, int S, int row_stride, int n_heads, const fp_kv_view* kv,
                  const int32_t* pos, const float* rope_cs, int32_t* err, void* stream);

/* Decode attention: one query row per sequence, q bf16 [B][q_stride] (head h
 * at h*head_dim), attends over positions 0 .. len[b]-1 of the cache
 * (softmax(q K^T / sqrt(hd)) V, query head j reads KV head j / (H/Hkv));
 * out bf16 [B][n_heads*head_dim].  Split over the context in chunks; the
 * partial results stay in the shared memory of a cluster of CTAs where one takes
 * the splits' place (dec_cluster), else go to `workspace`
 * (fp_op_attention_decode_workspace_bytes for at most max_len cached positions;
 * to be there whatever the splits) and a second kernel combines them.
 * len[b] in [1, max_len]; a larger len[b] is clipped to max_len and sets
 * *err = 1 (err may be NULL). */
int fp_op_attention_decode(const uint16_t* q, int q_stride, int B, int n_heads, const fp_kv_view* kv,
                           const int32_t* len, int max_len, uint16_t* out, void* workspace,
                           size_t workspace_bytes, int32_t* err, void* stream);
size_t fp_op_attention_decode_workspace_bytes(int B, int n_heads, int head_dim, int max_len);

/* Context splits fp_op_attention_decode uses for B sequences, n_kv_heads KV
 * heads of head_dim, a kvquant cache of 16-token pages with 16-byte aligned
 * pools, and max_len cached positions (0 for a non-positive argument).  With
 * 1 split the kernel normalises in place and never touches the workspace;
 * with more, the CTAs of a cluster merge their partials or the partials go to
 * the workspace and a second kernel merges them. */
int fp_op_attention_decode_splits(int B, int n_kv_heads, int head_dim, int kvquant, int max_len);

/* Decode attention without a caller workspace, for callers that cannot
 * allocate device memory (a host whose device memory is all reserved by
 * another framework's pool, a plugin that must not call the allocator, a
 * latency-critical loop that cannot risk the synchronisation of cudaMalloc).
 * The paper has no counterpart: this is a deployment convenience of this
 * library only.
 *
 * Same arguments, kernels and results as fp_op_attention_decode, but the
 * split partials go to a scratch array of FP_NOALLOC_SCRATCH_BYTES (32 MiB)
 * compiled into the library.  Every GPU that loads the library holds that
 * array until the process exits.  The call allocates nothing.
 *   - A request whose fp_op_attention_decode_workspace_bytes(B, n_heads,
 *     head_dim, max_len) exceeds FP_NOALLOC_SCRATCH_BYTES returns
 *     FP_ERR_UNSUPPORTED before anything is launched.
 *   - The first call on a device looks up the array's device address on that
 *     device (cudaGetSymbolAddress, with the device current) and caches it
 *     with the id of the device's current context; make that first call
 *     before any stream capture.  After a device reset the context differs,
 *     and the next call looks the address up again (make it, too, outside a
 *     capture).
 *   - All calls share the one array, which keeps the last call's contents;
 *     each call writes every partial it reads back, so nothing needs
 *     clearing.  Calls that overlap on the GPU (other streams, other host
 *     threads) race on the array: serialise them. */
#define FP_NOALLOC_SCRATCH_BYTES (32u << 20)
int fp_op_attention_decode_noalloc(const uint16_t* q, int q_stride, int B, int n_heads, const fp_kv_view* kv,
                                   const int32_t* len, int max_len, uint16_t* out, int32_t* err, void* stream);

/* Prefill attention: causal, S query rows per sequence at positions 0..S-1,
 * q bf16 [B*S][q_stride]; keys/values read from the cache positions 0..S-1;
 * out bf16 [B*S][n_heads*head_dim].  head_dim 128 with 16-token pages,
 * 16-byte aligned q (q_stride a multiple of 8) and pools runs on tcgen05
 * (scores and output accumulated in TMEM); other shapes on mma.sync.  An
 * int8 cache enters as its codes, with each key's K scale multiplying its
 * score column and its V scale its probability column in fp32; on tcgen05
 * the int8-cache products run in fp16 (codes exact, q converted, P carrying
 * the V scales times a power of two that keeps it in the fp16 normal
 * range), and a q element beyond the fp16 range sets *err = 3 (the output
 * is then invalid).  A page id outside [0, n_pages) reads zeros and sets
 * *err = 1. */
int fp_op_attention_prefill(const uint16_t* q, int q_stride, int B, int S, int n_heads,
                            const fp_kv_view* kv, uint16_t* out, int32_t* err, void* stream);

/* ---- Chunks of new tokens over a cache that already holds something: the next
 * piece of each prompt (chunked prefill), drafted tokens to be verified, or one
 * token a sequence, mixed as they come.  The batch is ragged: cu int32 [B + 1]
 * does not decrease, sequence b's rows are cu[b] .. cu[b+1]-1 of the packed
 * buffers (none is allowed), and its row i sits at position pos[b] + i (pos
 * int32 [B]: what the cache held before the chunk).  n_tokens rows are in the
 * buffers; rows that no sequence owns (behind cu[B], before cu[0]) are left as
 * they were.  cu and pos are read on the device, so one captured launch serves
 * other lengths within the same bounds.  A cu that decreases or leaves
 * [0, n_tokens] sets *err = 1 (err may be NULL) and no row outside the buffers is
 * touched (fp_op_attention_chunk: nothing is written).  All buffers are 16-byte
 * aligned and strides multiples of 8 elements, else FP_ERR_UNSUPPORTED; pools hold
 * fewer than 2^31 rows. */

/* RoPE + KV-cache append of a chunk: as fp_op_rope_kv, for a ragged batch and
 * with the rotated queries to q_out bf16 [n_tokens][q_out_stride] (head h at
 * h*head_dim; q_out == qkv rotates in place and takes the same stride, else
 * FP_ERR_INVALID_ARG; no other overlap).  qkv bf16
 * [n_tokens][row_stride]: H query heads, Hkv key heads, Hkv value heads.
 * Positions outside the cache set *err = 1 and skip the row, a page id outside
 * the pool sets *err = 1 and skips the row's cache writes.  Two rows must not
 * write the same cache position. */
int fp_op_rope_kv_chunk(const uint16_t* qkv, int row_stride, int n_tokens, int B, int n_heads, const fp_kv_view* kv,
                        const int32_t* cu, const int32_t* pos, const float* rope_cs, uint16_t* q_out, int q_out_stride,
                        int32_t* err, void* stream);

/* Cached positions read back: row cu[b] + i of k_out and v_out (bf16
 * [n_tokens][out_stride], KV head h at h*head_dim) is position pos[b] + i of
 * sequence b, an int8 cache as bf16(code * scale).  A position outside the cache
 * or a page id outside the pool gives a row of zeros and sets *err = 1. */
int fp_op_kv_read(const fp_kv_view* kv, int n_tokens, int B, const int32_t* cu, const int32_t* pos, uint16_t* k_out,
                  uint16_t* v_out, int out_stride, int32_t* err, void* stream);

/* Attention of a chunk: row i of sequence b attends over cache positions
 * 0 .. pos[b] + i (the chunk's own keys included: append them first);
 * softmax(q K^T / sqrt(hd)) V, query head j reads KV head j / (H/Hkv), H/Hkv <=
 * 128.  q bf16 [n_tokens][q_stride] (head h at h*head_dim), out bf16
 * [n_tokens][n_heads*head_dim].
 * max_new: at least every sequence's number of rows; max_len: at least every
 * pos[b] + rows.  A sequence beyond either sets *err = 1: its rows behind the
 * first max_new are left as they were, keys behind max_len are not read (either 0:
 * nothing is done).  A row at
 * a negative position has no keys: zeros, and *err = 1.  A page id outside the
 * pool reads as zero keys and values and sets *err = 1.
 * An int8 cache enters as its codes, exact in bf16, the scales multiplied in fp32;
 * P is rounded to bf16.  A score that is NaN or +inf (a query or a key that is not
 * finite) makes the rows that see it NaN, and no others; a row whose scores are all
 * -inf is zeros.  Cache slots behind a sequence's last position may hold
 * anything; its cached V, and an int8 cache's V scales, must be finite (a NaN
 * or an infinity there may reach rows before its position, in the same 128).
 * Batches that could make more than 2^31 tiles of work, by n_tokens, B, the heads
 * and max_len, are FP_ERR_UNSUPPORTED, as are heads so many that T output rows, T
 * twice the largest power of two up to 128 / (H/Hkv), have 2^31 elements.
 * workspace: 256-byte aligned, at least
 * fp_op_attention_chunk_workspace_bytes(B, n_heads, n_kv_heads, head_dim, max_new)
 * bytes (0: a shape that is refused; else by head_dim alone: 21 MB for 64, 41 MB
 * for 128).  Its leading 64 KB hold ticket counters that
 * must be zero before the first call; every call leaves them zero again, so one
 * workspace serves any sequence of calls of its shape or smaller ones on one
 * stream (calls that overlap on the GPU need separate workspaces; zero it again
 * after a call that set *err = 2, a wait that ran out). */
int fp_op_attention_chunk(const uint16_t* q, int q_stride, int n_tokens, int B, int n_heads, const fp_kv_view* kv,
                          const int32_t* cu, const int32_t* pos, int max_new, int max_len, uint16_t* out,
                          void* workspace, size_t workspace_bytes, int32_t* err, void* stream);
size_t fp_op_attention_chunk_workspace_bytes(int B, int n_heads, int n_kv_heads, int head_dim, int max_new);

/* Probabilities of logits fp32 [M][V]: probs[m] = softmax(logits[m] / T),
 * T = temperature[m] (fp32 [M]; NULL: 1).  T = 0 is the greedy choice: 1 at the
 * lowest index of the largest logit, else 0.  -inf masks a token; a row that
 * masks all of them gives zeros.  A NaN or +inf in a row with T > 0 gives NaN
 * throughout (at T = 0 a NaN is passed over; a row of nothing else gives zeros).
 * A T that is negative, infinite or NaN gives a row of zeros and
 * sets *err = 1 (err may be NULL).  probs may be logits.  M to 2^27 and V to 2^30,
 * else FP_ERR_UNSUPPORTED. */
int fp_op_softmax(const float* logits, int M, int V, const float* temperature, float* probs, int32_t* err,
                  void* stream);

/* Verification of drafted tokens against the target's probabilities, from given
 * random numbers.  Sequence b's rows cu[b] .. cu[b+1]-1 are its last accepted
 * token and the k drafted after it (tokens int32 [n_tokens]; the first one's id is
 * not read); row i of p fp32 [n_tokens][V] is the target's distribution of the
 * token after row i, row i < k of q that which draft i + 1 was drawn from (q NULL:
 * drafts without one, taken as certain).  In order, the draft t after row i is
 * accepted if u_accept[cu[b] + i] * q_i(t) < p_i(t); a is the number accepted.
 * Then one token is drawn: a < k from max(0, p_a - q_a) (q NULL: from p_a without
 * the refused token), a = k from p_k; it is the lowest t whose running sum exceeds
 * u_draw[b] times the whole sum (u in [0, 1); the weights need not add up to 1).
 * If that distribution is all zero, p_a itself is drawn from; a NaN weighs nothing.
 * out_tokens int32 [n_tokens]: rows 0 .. a-1 of the sequence the accepted drafts,
 * row a the drawn token, -1 behind it; n_out int32 [B]: a + 1 (0: a sequence
 * without rows).  A sum that is zero or not finite draws nothing: row a is -1,
 * n_out a, *err = 1 (err may be NULL).  A draft outside [0, V) is refused and sets
 * *err = 1; drafts behind the first refused one are not looked at (padding of any
 * value will do).  Sums are held in pairs of fp32 (48 bits).  V to 2^30 and B to
 * 2^27, else FP_ERR_UNSUPPORTED. */
int fp_op_verify_draft(const float* p, const float* q, int V, int n_tokens, int B, const int32_t* cu,
                       const int32_t* tokens, const float* u_accept, const float* u_draw, int32_t* out_tokens,
                       int32_t* n_out, int32_t* err, void* stream);

/* ---- Trees of drafted tokens: several continuations of each sequence verified in
 * one pass.  The batch is ragged as above.  A sequence's rows are its tree: row 0 its
 * last accepted token, every other row a drafted token whose parent, an earlier row,
 * is the token before it.  Row i stands in the cache at position pos[b] + i until the
 * accepted path is known, but is rotated by pos[b] + its depth.  A step: plan the tree
 * once; in every layer append, then attend; draw and accept; in every layer commit the
 * path.  For a chain (each row's parent the row before) all of this is the chunk's. */

/* Rows of a tree that fp_op_tree_plan takes. */
#define FP_TREE_MAX_ROWS 1024

/* The plan of a batch of trees.  parent int32 [n_tokens]: the row, within its own
 * sequence, of the token before, less than the row's own, or -1 for none (the cached
 * prefix is before it; rows other than 0 may have none).  depth int32 [n_tokens]:
 * each row's number of ancestors.  mask uint32 [n_tokens][mask_stride]: bit j % 32 of
 * word j / 32 is set where row j of the sequence is the row itself or an ancestor; the
 * words' other bits are clear.  (Quick for trees as they are drafted; a chain of 1024
 * rows takes 3.5 ms.)  mask_stride at least ceil(max_new / 32), at most 65536;
 * max_new: at least every sequence's rows, at most FP_TREE_MAX_ROWS (0: nothing is
 * done).  Another parent is taken for -1 and sets *err = 1 (err may be NULL); so does a
 * sequence of more than max_new rows, whose rows behind those are left as they were. */
int fp_op_tree_plan(const int32_t* parent, int n_tokens, int B, const int32_t* cu, int max_new, int32_t* depth,
                    uint32_t* mask, int mask_stride, int32_t* err, void* stream);

/* RoPE + KV-cache append of a batch of trees: as fp_op_rope_kv_chunk (row i goes to
 * position pos[b] + i), with row i rotated by position pos[b] + depth[row] (depth
 * int32 [n_tokens]).  A rotated position outside the cache's positions sets *err = 1
 * and skips the row too. */
int fp_op_rope_kv_tree(const uint16_t* qkv, int row_stride, int n_tokens, int B, int n_heads, const fp_kv_view* kv,
                       const int32_t* cu, const int32_t* pos, const int32_t* depth, const float* rope_cs,
                       uint16_t* q_out, int q_out_stride, int32_t* err, void* stream);

/* Attention of a batch of trees: as fp_op_attention_chunk, but row i of sequence b
 * sees positions 0 .. pos[b] - 1 and, of the sequence's own rows, those whose bit its
 * mask words have set (mask uint32 [n_tokens][mask_stride], as fp_op_tree_plan writes
 * them; any mask will do, rows may see later rows).  Bits behind the sequence's last
 * row do not count, nor do those of rows behind the first max_new.  mask_stride at least
 * ceil(max_new / 32).  A row that sees
 * nothing (pos[b] = 0 and no bit) is zeros.  A sequence at a negative position has
 * no keys at all: zeros, and *err = 1.  Cached V that are not finite may reach rows
 * that do not see them, in the same 128 positions.  All else, bounds, errors,
 * accuracy and workspace, as there (a workspace may serve both). */
int fp_op_attention_tree(const uint16_t* q, int q_stride, int n_tokens, int B, int n_heads, const fp_kv_view* kv,
                         const int32_t* cu, const int32_t* pos, const uint32_t* mask, int mask_stride, int max_new,
                         int max_len, uint16_t* out, void* workspace, size_t workspace_bytes, int32_t* err,
                         void* stream);
size_t fp_op_attention_tree_workspace_bytes(int B, int n_heads, int n_kv_heads, int head_dim, int max_new);

/* Verification of a batch of trees against the target's probabilities, from given
 * random numbers.  Row i of p fp32 [n_tokens][V] is the target's distribution of the
 * token after row i; tokens int32 [n_tokens] the drafted tokens (row 0's is not read);
 * parent as for fp_op_tree_plan.  From row 0 on: a token is drawn from the row's
 * distribution, the lowest t whose running sum exceeds u[row] times the whole sum (u
 * fp32 [n_tokens], in [0, 1); the weights need not add up to 1, a NaN or a negative
 * one weighs nothing).  If a child of the row (the lowest that is behind it and names
 * it as its parent) has that token, it is accepted and the next row; else the token is
 * the last.  So what comes out is distributed as the target says, whatever was drafted.
 * path int32 [n_tokens]: the accepted rows, row 0 first, within the sequence;
 * out_tokens int32 [n_tokens]: the tokens drawn after each, the accepted ones and the
 * last; both -1 behind; n_out int32 [B]: their number (0: a sequence without rows).
 * A sum that is zero or not finite draws nothing: the row is in path, its token -1 and
 * not counted, *err = 1 (err may be NULL).  Sums are held in pairs of fp32 (48 bits).
 * V to 2^30 and B to 2^27, else FP_ERR_UNSUPPORTED. */
int fp_op_verify_tree(const float* p, int V, int n_tokens, int B, const int32_t* cu, const int32_t* parent,
                      const int32_t* tokens, const float* u, int32_t* path, int32_t* out_tokens, int32_t* n_out,
                      int32_t* err, void* stream);

/* The accepted path's rows of the cache moved together: position pos[b] + j of
 * sequence b takes what position pos[b] + path[cu[b] + j] holds (K, V and an int8
 * cache's scales, bit for bit), for j = 0, 1, .. up to the first -1 or the sequence's
 * last row.  A path ascends (path as fp_op_verify_tree writes it); an entry that does
 * not, or is no row of the sequence, sets *err = 1 (err may be NULL) and ends the
 * sequence's path there.  A position outside the cache or a page id outside the pool
 * sets *err = 1 and skips the row.  No two sequences may hold these positions in the
 * same pages. */
int fp_op_kv_commit(const fp_kv_view* kv, int n_tokens, int B, const int32_t* cu, const int32_t* pos,
                    const int32_t* path, int32_t* err, void* stream);

/* ---- Beams: B groups of W hypotheses each, W up to FP_BEAM_MAX (else
 * FP_ERR_UNSUPPORTED), B up to FP_BEAM_MAX_GROUPS (the same).  Beam w of group b is row b * W + w of all buffers,
 * and a sequence of its own in the paged cache (a row of the page table). */
#define FP_BEAM_MAX 32
#define FP_BEAM_MAX_GROUPS 16384

/* The best continuations.  logits fp32 [B*W][V], score fp32 [B*W] (a hypothesis' sum of
 * log-probabilities; -inf: there is none).  A group's candidates are (w, t) with the
 * value score[w] + logits[w][t] - log sum_s exp(logits[w][s]); the W largest, in falling
 * order, ties to the lowest w, then t: parent int32 [B*W] their w, token int32 [B*W]
 * their t, new_score fp32 [B*W] their values.  A logit of -inf bans its token (a low
 * finite one, down to the least, all but does: it is a candidate with its value, none
 * where that is below the least fp32).  done
 * int32 [B*W] (NULL: none): where it is not 0 the hypothesis has ended; its logits are
 * not read, its one candidate is end_token with its score as it is.  new_done int32
 * [B*W] (may be NULL): 1 where the parent had ended or the token is end_token, else 0.
 * end_token in [-1, V); -1: none (done must be NULL then).  With fewer than W candidates
 * the places left are parent -1, token -1, score -inf, done 0.  A logit that is NaN or
 * +inf in a row that is read, or a score that is NaN or +inf leaves the hypothesis
 * without candidates and sets *err = 1 (err may be NULL).  Values are ordered by sums in
 * pairs of fp32, the normaliser good to 2^-19, or to 2^-44 of the row's largest logit
 * where that is up to 2^30 and 2^-44 of it is more.  new_score may be score, new_done done; no other
 * overlap.  V to 2^30.  workspace: 256-byte aligned, at least
 * fp_op_beam_select_workspace_bytes(B, W, V) bytes (0: a shape that is refused); its
 * leading 64 KB are ticket counters that must be zero before the first call; every call
 * leaves them zero again, so one workspace serves any sequence of calls on one stream
 * that it is large enough for (calls that overlap on the GPU need separate workspaces). */
int fp_op_beam_select(const float* logits, int V, int B, int W, const float* score, const int32_t* done, int end_token,
                      int32_t* parent, int32_t* token, float* new_score, int32_t* new_done, void* workspace,
                      size_t workspace_bytes, int32_t* err, void* stream);
size_t fp_op_beam_select_workspace_bytes(int B, int W, int V);

/* Page tables that follow the chosen beams.  table_in int32 [B*W][pages_per_seq] is
 * what the beams had, len int32 [B] their cached positions, parent as
 * fp_op_beam_select writes it (-1: no hypothesis; the beam keeps its own full blocks, its
 * part-filled one may be any that is left, and nothing is copied).  In table_out (another
 * buffer) a beam has its parent's pages for the full blocks of page_size positions, shared,
 * and its own for the blocks not begun.  The part-filled block (len[b] % page_size > 0)
 * needs a page of its own for every beam, as table_in must have it: the first of a beam's children
 * keeps its page, the others take, in order, the pages of the beams without children, in
 * order, and for those copy_from and copy_to int32 [B*W] are the pages and copy_rows
 * int32 [B*W] the rows that fp_op_kv_copy has to copy in every layer; all other places
 * -1, -1, 0.  So pages are neither taken nor given back.  (A prompt's beams start from
 * one: parent 0 throughout.)  A length outside
 * [0, pages_per_seq * page_size] leaves the group's rows as they are, a parent outside
 * [-1, W) is taken for -1; both set *err = 1 (err may be NULL).  page_size 16. */
int fp_op_beam_reorder(int B, int W, int pages_per_seq, int page_size, const int32_t* len, const int32_t* parent,
                       const int32_t* table_in, int32_t* table_out, int32_t* copy_from, int32_t* copy_to,
                       int32_t* copy_rows, int32_t* err, void* stream);

/* Pages copied within the pools: the first rows[i] positions of page from[i] to page
 * to[i], all KV heads, K, V and an int8 cache's scales, for i < n (int32 [n] each);
 * from[i] = -1 or rows[i] = 0: nothing.  No page may be written twice or both read and
 * written in a call.  A page id outside the pool or rows[i] outside [0, page_size] sets
 * *err = 1 (err may be NULL) and skips the copy.  Pools 16-byte aligned, else
 * FP_ERR_UNSUPPORTED.  (The view's page table is to be there, but is not read.) */
int fp_op_kv_copy(const fp_kv_view* kv, int n, const int32_t* from, const int32_t* to, const int32_t* rows,
                  int32_t* err, void* stream);

/* Test hook for the failure path of the pipelined tensor-core kernels (the
 * paper has no counterpart).  Every wait of those kernels is bounded; a role
 * whose wait runs out stops, the CTA drains its copies and MMAs in flight,
 * frees its tensor memory and records status 2 in the error word, which the
 * runtime reports as FP_ERR_DEVICE_ASSERT.  This sets how many polling rounds
 * the prefill GEMM's MMA thread waits for a stage of operands on the current
 * device, and the MMA warps of fp_op_attention_chunk and fp_op_attention_tree for a tile of values in the
 * launches that follow: rounds >= 0 (0 gives up at once) or < 0 to restore the
 * default; all other waits keep the default.  Synchronous; not for use while
 * kernels of the library are running. */
int fp_debug_set_wait_limit(long long rounds);

/* Greedy choice out[m] = argmax logits[m][:V] (fp32); ties to the lowest id. */
int fp_op_argmax(const float* logits, int M, int V, int32_t* out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FP_OPS_H */
