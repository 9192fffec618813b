/* lp_ops.h -- single-kernel entry points of the serving step, for parity
 * checks and kernel timing.  They launch exactly the kernels the engine runs
 * (those of the last two sections, a batch that shares a prefix and a cache
 * held in 4 bits, are for callers that plan their own steps), on
 * caller-provided device buffers, asynchronously on `hip_stream` (a
 * hipStream_t, NULL for the null stream).
 * All pointers are device pointers unless stated otherwise; the caller owns
 * every buffer.  Each returns LP_OK or
 * LP_EINVAL (bad sizes; checked before any launch) or LP_EHIP (launch error);
 * lp_last_error(NULL) then holds a message.  A call with no rows (M, rows or
 * n_seq equal to 0) checks its sizes, then returns LP_OK without a launch or
 * any memory access; its pointers may be null.
 *
 * `dtype` is LP_F32, LP_BF16 or LP_F16: the element type of weights and
 * activations (bf16 as raw 16-bit patterns).  Accumulation is fp32 in all.
 */
#ifndef LP_OPS_H
#define LP_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "lp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Y[M x N] (fp32, row stride N) = X[M x K] (row stride ldx) times W[N x K]^T:
 * the weight-GEMM contraction of every projection of the decoder (Q/K/V,
 * output, gate/up, down, LM head) that both phases of Sec. II-A run every
 * token through (the paper fixes no layer math; the Llama-style decoder is
 * a reading).  For LP_BF16 / LP_F16, W is in the tiled
 * weight layout that lp_op_pack_weight writes; for LP_F32 it is row-major
 * [N x K].  16-bit types with M <= 64 take the decode kernel, larger M the
 * prefill kernel; `k_splits` > 1 splits K across workgroups (prefill: only
 * when K is a multiple of 128; the count is rounded to whole K chunks) and
 * needs `ws` of at least k_splits * M * N * 4 bytes (fp32 partials).  K must
 * be a multiple of 8, N even; 16-byte aligned rows. */
int lp_op_gemm(int32_t dtype, const void *X, int64_t ldx, const void *W, float *Y, int32_t M, int32_t N,
               int32_t K, int32_t k_splits, void *ws, size_t ws_bytes, void *hip_stream);

/* Which kernel lp_op_gemm (16-bit types) runs for this shape and split
 * request, for the same contraction as above: `kind` 0 = decode kernel
 * (M <= 64), 1 = prefill kernel with one workgroup per CU, 2 = prefill
 * kernel with two 128-row workgroups per CU, 3 = LDS-tiled kernel (K not a
 * multiple of 128); `tile_rows` = rows per output tile; `splits` = the K
 * splits it uses; `xcd_group` = row tiles per group of the prefill kernel's
 * XCD-aware tile order, 0 for the plain order.  The plan is for row strides
 * below 2^27 elements: from there on lp_op_gemm runs the LDS-tiled kernel
 * where this call names a prefill kernel, with the whole sum in the first
 * partial when K is split.  `k_splits` as for lp_op_gemm, except that 0 asks
 * for the split count a prefill step of the engine chooses by itself for
 * M > 64.  Host-only, no device call.  Returns LP_EINVAL for non-positive sizes or
 * null outputs. */
int lp_op_gemm_plan(int32_t M, int32_t N, int32_t K, int32_t k_splits, int32_t *kind, int32_t *tile_rows,
                    int32_t *splits, int32_t *xcd_group);

/* The tiled weight layout of the 16-bit GEMMs (weights of Sec. II-A's
 * decoder, stored for the decode phase's weight stream).  A row-major [N x K]
 * matrix W (row n = output feature n, stride K, K % 8 == 0) becomes
 * ceil(N/16) * ceil(K/32) tiles of 16 rows x 32 columns, 512 elements (1 KB) each;
 * tile (i, j) has index j * ceil(N/16) + i (the tiles of one 32-column step
 * side by side) and holds rows 16i..16i+15, columns 32j..32j+31, its element
 * (r, c) at position
 * 8 * (r + 16 * (c / 8)) + c % 8.  Rows >= N and columns >= K are zero.
 * lp_op_packed_weight_bytes gives the size (0 for other dtypes or
 * non-positive sizes); lp_op_pack_weight writes W_packed (device, that many
 * bytes, caller-owned, 16-byte aligned like W) on `hip_stream`.  LP_EINVAL for
 * null pointers, bad sizes or a dtype other than LP_BF16 / LP_F16. */
size_t lp_op_packed_weight_bytes(int32_t dtype, int32_t N, int32_t K);
int lp_op_pack_weight(int32_t dtype, const void *W, void *W_packed, int32_t N, int32_t K, void *hip_stream);

/* RMSNorm of the decoder layer (run by both phases of Sec. II-A; the norm is
 * a reading of the architecture, which the paper leaves open):
 * y[r] = x[r] / sqrt(mean(x[r]^2) + eps) * g for r < rows; x fp32
 * [rows x d] (first incremented in place by the n_part fp32 partial arrays
 * part[s][rows][d] when n_part > 0), g fp32 [d], y [rows x d] in dtype.
 * d <= 8192. */
int lp_op_rmsnorm(int32_t dtype, float *x, const float *part, int32_t n_part, const float *g, void *y,
                  int32_t rows, int32_t d, float eps, void *hip_stream);

/* Decode attention of one layer (Sec. II-A's decode phase reads the KV cache
 * of every earlier position).  q, out: [M x Hq x hd] in dtype.  KV cache of
 * one layer in blocks of 64 tokens: k_cache [n_blocks][Hkv][64][hd],
 * v_cache [n_blocks][Hkv][hd][64] (transposed per block); block_table
 * [*][max_blocks] int32 lists each slot's blocks.  Row m reads slot
 * row_slot[m] over positions 0..row_pos[m] (ctx = row_pos[m] + 1 <= max_ctx;
 * a larger ctx is clamped to max_ctx, so the kernels stay inside ws and the
 * first max_ctx positions of the block table).
 * ws: at least lp_op_decode_attention_ws_bytes(M, Hq, hd, max_ctx) bytes. */
size_t lp_op_decode_attention_ws_bytes(int32_t M, int32_t n_heads, int32_t head_dim, int32_t max_ctx);
int lp_op_decode_attention(int32_t dtype, const void *q, void *out, const void *k_cache, const void *v_cache,
                           const int32_t *block_table, int32_t max_blocks, int64_t n_blocks,
                           const int32_t *row_slot, const int32_t *row_pos, int32_t M, int32_t n_heads,
                           int32_t n_kv_heads, int32_t head_dim, int32_t max_ctx, void *ws, size_t ws_bytes,
                           void *hip_stream);

/* lp_op_decode_attention without a workspace argument, for callers that
 * cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc).  Arguments, layouts and results
 * are those of lp_op_decode_attention; the chunk partials go to a static
 * device array of LP_NOALLOC_SCRATCH_BYTES (32 MiB) that the library holds on
 * every GPU it runs on until the process ends.  The call allocates and frees
 * nothing.  LP_EINVAL when lp_op_decode_attention_ws_bytes(M, n_heads,
 * head_dim, max_ctx) exceeds the array (64 rows of 32 heads of head_dim 128
 * fit contexts up to 7,936 positions), checked before any device call.  Every
 * call on one GPU shares that GPU's array: calls that overlap in time on one
 * GPU (other streams, other threads) race and must be serialised by the
 * caller. */
#define LP_NOALLOC_SCRATCH_BYTES (32u << 20)
int lp_op_decode_attention_noalloc(int32_t dtype, const void *q, void *out, const void *k_cache,
                                   const void *v_cache, const int32_t *block_table, int32_t max_blocks,
                                   int64_t n_blocks, const int32_t *row_slot, const int32_t *row_pos, int32_t M,
                                   int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_ctx,
                                   void *hip_stream);

/* Causal prefill attention of one layer over packed prompts (Sec. II-A's
 * prompt processing): sequence j owns rows [seq_start[j], seq_start[j+1]) of
 * q/out ([rows x Hq x hd]) at positions 0.., and its keys/values are already
 * in the cache of slot seq_slot[j] (layout as above).  max_len bounds every
 * sequence length: of a longer one, rows from max_len on may be left out, and
 * none past the max_blocks * 64 positions of its block table row is computed.
 * 16-bit caches that are not on 16 bytes take a slower kernel. */
int lp_op_prefill_attention(int32_t dtype, const void *q, void *out, const void *k_cache, const void *v_cache,
                            const int32_t *block_table, int32_t max_blocks, int64_t n_blocks,
                            const int32_t *seq_start, const int32_t *seq_slot, int32_t n_seq, int32_t max_len,
                            int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, void *hip_stream);

/* Greedy decoding, the token choice of each prefill and decode step of Sec.
 * II-A under greedy requests: tokens[m] = argmax of logits row m (fp32, row
 * stride ld), lowest index on ties; a NaN is never chosen, and a row of
 * nothing but NaN gives 0x7fffffff (which the engine embeds as NaN).
 * tokens [M] int32 (device). */
int lp_op_argmax(const float *logits, int64_t ld, int32_t M, int32_t V, int32_t *tokens, void *hip_stream);

/* The device weight generator (see lp_init_weights_random): dst[rows x cols]
 * in dtype gets element (r, c) of canonical tensor `tensor_id`, unpermuted;
 * LP_F16 stores the bf16-rounded value (as a bf16 model held in fp16). */
int lp_op_init_weight(int32_t dtype, void *dst, uint64_t seed, int32_t tensor_id, int64_t rows, int64_t cols,
                      float std, void *hip_stream);

/* Sampling parameters of one row (requests carry them, Sec. III-A):
 * temperature <= 0 or top_p <= 0 mean greedy; top_k 0 means no top-k limit;
 * top_p >= 1 means no nucleus limit; key / counter: the Philox4x32-10 key
 * and the first three counter words of the row's random draw (the fourth is
 * the constant 0x53414D50). */
typedef struct {
  float temperature;
  int32_t top_k;
  float top_p;
  uint32_t key[2];
  uint32_t counter[3];
} lp_sample_params;

/* Next token of each of M rows of fp32 logits (row stride ld >= V) under its
 * sampling parameters; tokens [M] int32 (device).  Greedy rows take the
 * lowest index among the maxima.  Otherwise, with m the row maximum:
 * candidates are all tokens, or for 0 < top_k < V the tokens whose logit is
 * at least the top_k-th largest (ties kept); a candidate's weight is
 * q = floor(exp((logit - m) / temperature) * 2^40); for top_p < 1 the kept
 * candidates are those with q >= t, t the largest value whose heavier-or-
 * equal candidates weigh at least ceil(Z * floor(top_p * 2^24) / 2^24) (Z the
 * candidates' total); the draw r = floor(Z_kept * u24 / 2^24), u24 the first
 * Philox output word >> 8, picks the kept candidate, in vocabulary order,
 * whose cumulative weight interval holds r.  V <= 2^21 (LP_EINVAL beyond). */
int lp_op_sample(const float *logits, int64_t ld, int32_t M, int32_t V, const lp_sample_params *params,
                 int32_t *tokens, void *hip_stream);

/* ---- a batch whose sequences begin with the same prefix ----
 *
 * Requests of one service often start with the same tokens (an instruction, a
 * document they ask about).  The K and V of those P = prefix_len positions are
 * kept once, in the cache blocks prefix_blocks[0 .. ceil(P / 64)); a
 * sequence's own positions, P and up, are in the blocks of its row of the
 * block table, position p in entry p / 64 at place p % 64, as everywhere in
 * this header.  The entries below floor(P / 64) of a table row name the
 * prefix's whole blocks; with P a multiple of 64 the table is therefore one
 * that lp_op_decode_attention and lp_op_prefill_attention read too.  A prefix
 * that ends inside a block leaves the first P % 64 places of a sequence's
 * first own block unused.  P = 0 is no prefix (prefix_blocks may be null).
 *
 * The four calls below make a step: tables and cache entries from lengths,
 * the projection's K and V into the cache, attention over it.  They share
 * these rules.  Positions, slots, entries and block ids are data on the
 * device, which no call can check before it launches; what does not fit is
 * left out, never read or written through: a slot outside 0 .. n_slots - 1, a
 * block id outside 0 .. n_blocks - 1 (-1 marks one that is missing), a
 * negative position.  q, out, the caches and ws start on 16 bytes (LP_EINVAL
 * otherwise).  A call keeps nothing from one call to the next, in ws neither,
 * so ws needs no clearing; calls that overlap in time need one each. */

/* Block tables, packed row offsets and cache entries of one step, from
 * lengths that are on the device.  Sequence j (slot seq_slot[j], no slot
 * twice) holds cached[j] positions before the step and lengths[j] after it:
 * its n_j = max(0, lengths[j] - max(0, cached[j])) new positions are packed
 * rows.
 *   seq_start[0 .. n_seq]   exclusive sums of n_j (at most 2^31 - 1)
 *   free_start[0 .. n_seq]  *free_head plus exclusive sums of the blocks each
 *                           sequence takes: its new ones are
 *                           free_blocks[free_start[j] ..].  free_start[n_seq]
 *                           is the next free_head; past n_free, blocks are
 *                           lacking.  free_head may point at it.
 *   block_table             [n_slots][max_blocks], updated: entries below
 *                           floor(P / 64) that the length reaches become the
 *                           prefix's blocks; where lengths[j] > P, entries
 *                           from have_j up to ceil(lengths[j] / 64) the
 *                           blocks taken, -1 if they are lacking; have_j =
 *                           ceil(cached[j] / 64) if cached[j] > P, else
 *                           floor(P / 64).  Others stay.
 *   row_slot, row_pos,      [max_rows]: slot, position and cache entry (64 *
 *   row_entry               block + place) of each row; the entry is -1 where
 *                           there is no block: past the table's width, or
 *                           lacking.  Rows from seq_start[n_seq] on get -1 in
 *                           all three, rows from max_rows on are left out.
 * Rows at positions below P (a request that computes the prefix itself) have
 * their entry in prefix_blocks.  All pointers but prefix_blocks (P < 1) and
 * free_blocks (n_free = 0) are required when n_seq > 0; with n_seq = 0 nothing
 * is written. */
int lp_op_block_tables(const int32_t *seq_slot, const int32_t *cached, const int32_t *lengths, int32_t n_seq,
                       const int32_t *prefix_blocks, int32_t prefix_len, const int32_t *free_blocks, int32_t n_free,
                       const int32_t *free_head, int32_t *block_table, int32_t n_slots, int32_t max_blocks,
                       int32_t *seq_start, int32_t *free_start, int32_t *row_slot, int32_t *row_pos,
                       int64_t *row_entry, int32_t max_rows, void *hip_stream);

/* The QKV projection of `rows` rows as lp_op_gemm writes it (fp32, row stride
 * ld >= (Hq + 2 Hkv) hd elements: query heads, key heads, value heads), made
 * ready for attention: q and k heads get the rotary embedding of their row's
 * position (dimensions i and i + hd / 2 form a pair, rotated by the angle
 * whose cosine and sine are rope_cos[pos][i], rope_sin[pos][i], tables of
 * n_pos positions), q goes to q [rows][Hq][hd] and k, v to the cache at
 * row_entry, all rounded to dtype once.  K and V of a row with an entry
 * outside 0 .. 64 n_blocks - 1 are left out; of a row with a position outside
 * 0 .. n_pos - 1, everything.  No two rows may have the same entry.  qkv and
 * the tables start on 8 bytes, ld is even; head_dim 64 or 128; rows (Hq + 2
 * Hkv) at most 2^23. */
int lp_op_qkv_append(int32_t dtype, const float *qkv, int64_t ld, const float *rope_cos, const float *rope_sin,
                     int32_t n_pos, const int32_t *row_pos, const int64_t *row_entry, int32_t rows, void *q,
                     void *k_cache, void *v_cache, int64_t n_blocks, int32_t n_heads, int32_t n_kv_heads,
                     int32_t head_dim, void *hip_stream);

/* Decode attention with a shared prefix: row m of q, out [M][Hq][hd] reads
 * positions 0 .. row_pos[m] of slot row_slot[m], those below P from the
 * prefix's blocks.  Contexts longer than max_ctx are clamped to it.  A row that
 * reads nothing (position -1, no such slot, all its blocks missing), or whose
 * every score is minus infinity, gets zeros.  Any group Hq / Hkv; head_dim 64
 * or 128 in every dtype; 64 * max_blocks >= max_ctx where max_ctx > P.
 * max_ctx, prefix_len and M Hq are at most 2^30.  A call that would launch 2^23
 * workgroups or more is refused as well: none is with M Hq (16 + max_ctx / 4096)
 * up to 2^22, all are from M Hq = 2^25 on.
 * ws: at least lp_op_prefix_decode_attention_ws_bytes of the same sizes, which is
 * 0 for sizes out of the limits above.  It does not look at the workgroups,
 * which depend on dtype and sequences too: those show at the call. */
size_t lp_op_prefix_decode_attention_ws_bytes(int32_t M, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                              int32_t prefix_len, int32_t max_ctx);
int lp_op_prefix_decode_attention(int32_t dtype, const void *q, void *out, const void *k_cache, const void *v_cache,
                                  int64_t n_blocks, const int32_t *prefix_blocks, int32_t prefix_len,
                                  const int32_t *block_table, int32_t n_slots, int32_t max_blocks,
                                  const int32_t *row_slot, const int32_t *row_pos, int32_t M, int32_t n_heads,
                                  int32_t n_kv_heads, int32_t head_dim, int32_t max_ctx, void *ws, size_t ws_bytes,
                                  void *hip_stream);

/* Causal attention of packed new tokens with a shared prefix: sequence j owns
 * rows [seq_start[j], seq_start[j + 1]) of q, out [rows][Hq][hd], at positions
 * seq_pos[j], seq_pos[j] + 1, ... of slot seq_slot[j]; each row reads
 * positions 0 up to its own.  K and V of the new positions are in the cache
 * already, as are those before them (a sequence may go on from any context:
 * the prefix, one longer than it, or none of it).  Contexts and rows that read
 * nothing as for decode; all rows of a sequence whose seq_pos is negative are
 * such.  max_new bounds the rows of every sequence (rows of a longer one from
 * max_new on hold no result); rows of no sequence stay as they are.  seq_start
 * ascends; entries below 0 count as 0, those above `rows` as `rows`.  Sequences
 * without rows take no workgroups.  Limits and ws as for decode, with `rows`
 * for M. */
size_t lp_op_prefix_prefill_attention_ws_bytes(int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                               int32_t prefix_len, int32_t max_ctx);
int lp_op_prefix_prefill_attention(int32_t dtype, const void *q, void *out, const void *k_cache, const void *v_cache,
                                   int64_t n_blocks, const int32_t *prefix_blocks, int32_t prefix_len,
                                   const int32_t *block_table, int32_t n_slots, int32_t max_blocks,
                                   const int32_t *seq_start, const int32_t *seq_slot, const int32_t *seq_pos,
                                   int32_t n_seq, int32_t rows, int32_t max_new, int32_t n_heads, int32_t n_kv_heads,
                                   int32_t head_dim, int32_t max_ctx, void *ws, size_t ws_bytes, void *hip_stream);

/* ---- a K/V cache held in 4 bits ----
 *
 * The contexts of decode are read at the rate of the memory, and they fill it: a
 * cache of 4.5 bits a value holds 3.6 times the positions of a 16-bit one and is
 * read 3.6 times as fast.  The calls below write it, attend over it and bring
 * entries back; block ids, entries (64 * block + place), slots and positions are
 * those of the calls above (lp_op_block_tables makes them, with prefix_len 0 or
 * a multiple of 64), and so are the rules for what does not fit: it is left out,
 * never read or written through.  q, out, the caches and ws start on 16 bytes
 * (LP_EINVAL otherwise); ws needs no clearing, and calls that overlap in time
 * need one each.
 *
 * 32 consecutive dims of a head at one position are a group, with one scale s:
 * the least number that is not below a sixth of the group's largest magnitude
 * and is a multiple of 2^-23 of at most 6 significant bits; at most 10,752; NaN
 * if the group holds an infinity or NaN (all its values are then NaN).  A value
 * is held as its sign and the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (codes 0 ..
 * 7) times s, of two equally near ones the even code; past 6 s, 6.  The values
 * held have 8 significant bits and are exact in every dtype.
 *
 * cache: for each block and KV head 72 head_dim bytes, [n_blocks][Hkv][72 hd],
 * that do not depend on dtype.  With J = hd / 32, a byte two codes (sign above
 * the three bits), the lower dim in the low half:
 *   K codes   [64][hd / 2]       byte 4 J i + 4 j + b: dims 32 j + 8 i + 2 b and
 *                                the next (i, b < 4, j < J)
 *   K scales  [64][J] fp16
 *   V codes   [16][hd / 8][4][4] word w of positions 4 n .. 4 n + 3 side by side;
 *                                byte J r + j of a position's hd / 2 bytes: dims
 *                                32 j + 2 r and the next (r < 16)
 *   V scales  [J][64] fp16
 * Any bytes are a cache: places that no row may read need not be cleared; those
 * that rows read hold what lp_op_kv4_append wrote, or scales and codes of the kind.
 *
 * Attention of 16-bit types rounds each weight once, to fp16.  bf16 rows of q of
 * longer prompts are taken to fp16 by their largest element: elements below 2^-14
 * of it are then off by up to 2^-25 of it, which only keys far larger in their dims
 * than in the largest's would show. */

/* Bytes of a cache; 0 for sizes that no call takes. */
size_t lp_op_kv4_cache_bytes(int64_t n_blocks, int32_t n_kv_heads, int32_t head_dim);

/* lp_op_qkv_append into a cache held in 4 bits: the same arguments, rotation,
 * rules and limits, with K (rotated) and V quantised from fp32 at row_entry;
 * dtype is q's. */
int lp_op_kv4_append(int32_t dtype, const float *qkv, int64_t ld, const float *rope_cos, const float *rope_sin,
                     int32_t n_pos, const int32_t *row_pos, const int64_t *row_entry, int32_t rows, void *q,
                     void *cache, int64_t n_blocks, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                     void *hip_stream);

/* Entries of a 4-bit cache back into an ordinary cache of dtype (k_cache
 * [n_dst_blocks][Hkv][64][hd], v_cache [n_dst_blocks][Hkv][hd][64]): K and V of
 * src_entry[i] go to dst_entry[i], i < rows, exactly.  Rows with either entry
 * outside its cache are left out.  No two rows may have the same dst_entry.
 * rows Hkv at most 2^26, ceil(rows / 64) Hkv below 2^24. */
int lp_op_kv4_read(int32_t dtype, const void *cache, int64_t n_blocks, const int64_t *src_entry,
                   const int64_t *dst_entry, int32_t rows, void *k_cache, void *v_cache, int64_t n_dst_blocks,
                   int32_t n_kv_heads, int32_t head_dim, void *hip_stream);

/* Decode attention over a 4-bit cache: row m of q, out [M][Hq][hd] reads
 * positions 0 .. row_pos[m] of slot row_slot[m].  Contexts longer than max_ctx
 * are clamped to it; 64 * max_blocks >= max_ctx.  A row that reads nothing
 * (position -1, no such slot, all its blocks missing), or whose every score is
 * minus infinity, gets zeros.  Scores q k, before the scale 1 / sqrt(hd), are
 * fp32 numbers: q of any size may be given as long as they are below 2^128.  Any
 * group Hq / Hkv; head_dim 64 or 128.  max_ctx and M Hq are at most 2^30.  A
 * call that would launch 2^23 workgroups or more is refused as well: none is
 * with M Hq below 2^22 and max_ctx up to 2^20, all are from M Hq = 2^25 on.
 * ws: at least lp_op_kv4_decode_attention_ws_bytes of the same sizes, which is 0
 * for sizes out of the limits above and ascends in M and max_ctx: the workspace
 * of a batch's limits serves its smaller steps. */
size_t lp_op_kv4_decode_attention_ws_bytes(int32_t M, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                           int32_t max_ctx);
int lp_op_kv4_decode_attention(int32_t dtype, const void *q, void *out, const void *cache, int64_t n_blocks,
                               const int32_t *block_table, int32_t n_slots, int32_t max_blocks,
                               const int32_t *row_slot, const int32_t *row_pos, int32_t M, int32_t n_heads,
                               int32_t n_kv_heads, int32_t head_dim, int32_t max_ctx, void *ws, size_t ws_bytes,
                               void *hip_stream);

/* Causal attention of packed new tokens over a 4-bit cache: sequence j owns rows
 * [seq_start[j], seq_start[j + 1]) of q, out [rows][Hq][hd], at positions
 * seq_pos[j], seq_pos[j] + 1, ... of slot seq_slot[j]; each row reads positions
 * 0 up to its own, the new ones among them as the cache holds them.  Rows,
 * offsets, max_new and rows of no sequence as for
 * lp_op_prefix_prefill_attention; limits and ws as for decode, with `rows` for
 * M. */
size_t lp_op_kv4_prefill_attention_ws_bytes(int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                            int32_t max_ctx);
int lp_op_kv4_prefill_attention(int32_t dtype, const void *q, void *out, const void *cache, int64_t n_blocks,
                                const int32_t *block_table, int32_t n_slots, int32_t max_blocks,
                                const int32_t *seq_start, const int32_t *seq_slot, const int32_t *seq_pos,
                                int32_t n_seq, int32_t rows, int32_t max_new, int32_t n_heads, int32_t n_kv_heads,
                                int32_t head_dim, int32_t max_ctx, void *ws, size_t ws_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* LP_OPS_H */
