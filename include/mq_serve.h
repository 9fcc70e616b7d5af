/*
 * mq_serve.h -- C boundary of the library's operators for serving and search over the paged 8-bit cache.
 *
 * mq_seq.h has the cache, single new tokens against it, and whole prompts.  The calls here are what a decoder with
 * self-attention needs around them:
 *   mq_chunk_attention      several new tokens per sequence over the cache (proposed tokens that are checked, prompts taken in by
 *                           pieces, ends of translations that are scored again);
 *   mq_kv_fork              the tables of continued sequences: beams reordered, answers begun from one prompt, ended sequences
 *                           dropped, blocks copied before two sequences write to one, new blocks for the tokens to come;
 *   mq_kv_compact           the used blocks of a cache moved to its front;
 *   mq_add_rms_norm*        residual addition and root-mean-square norm, its result in the type, as 8-bit rows, or as a packed operand;
 *   mq_w4_*                 parameters in 4 bits with scales and zeros of groups, and products of a few rows with them.
 *
 * The general rules of mq.h and the rules at the top of mq_seq.h (types, rows, heads, packed sequences, sizes) hold: device
 * pointers on the current device, caller-owned buffers, calls that only enqueue on `stream` and return an mq_status, arguments
 * checked before anything is enqueued.  No call here waits inside a kernel for other workgroups, none needs a prepared workspace,
 * none keeps anything from one call to the next; calls that may overlap in time need a workspace each.  Results depend neither on
 * what else runs nor on an order of atomics.
 */
#ifndef MQ_SERVE_H_
#define MQ_SERVE_H_

#include "mq_seq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- attention of new tokens over the cache -----------------------------------
 * Sequence b has lens[b] tokens in the cache, of which the last n are new (mq_kv_append has brought them in) and have a query
 * each: token rows first[b] .. first[b + 1] - 1 of q, n = first[b + 1] - first[b].  Query i attends to the tokens
 * t <= lens[b] - n + i, itself and what is ahead of it, or to all lens[b] if causal == 0:
 *   out[i] = sum_t p_t V[t],  p = softmax over the tokens seen of scale (q[i] . K[t]),  per head;
 * zeros where a query sees nothing, else NaN where it holds a NaN or an infinity.
 *   lens: device int32 [B]; values above max_len count as max_len, negative ones as 0.  max_len <= 64 table_width.
 *   first: device int32 [B + 1] over T token rows.  q: T token rows of `heads` heads, out likewise (it may be q itself, with
 *     ldo = ldq); rows that belong to no sequence are left as they are.
 * Queries enter the products exactly: one, two or three bfloat16 parts (bfloat16, binary16, binary32; elements below 2^-100 of
 * their row's largest may be lost).  The cache's integers are bfloat16 values as they are.  Probabilities times the scale of the
 * values' block enter as two parts (16-bit types, 16 bits) or three (binary32, 24 bits).  16-bit types: values of a block whose
 * largest is below 2^-119 count as zeros, and bits of values below 2^-100 may be lost; the weights of such tokens count in the
 * denominator all the same.  Sums and softmax statistics are binary32.
 * ws: device, 16-byte aligned, mq_chunk_attention_ws_bytes (0 for invalid arguments).  One launch where max_len <= 1152 (up to
 * 2048 if there is work for all of the chip) and rows are few, else two or three: shares are planned from the lengths, computed, and
 * joined.  Refused with MQ_ERR_SHAPE are calls that would take a launch of 2^32 threads (2^24 tiles of 32 rows x kv heads in one launch,
 * 2^22 where parts are joined), and calls of which that plan cannot count the blocks in 31 bits (some 2^31 / (max_len / 64) tiles of 32
 * rows). */
size_t mq_chunk_attention_ws_bytes(size_t B, size_t T, size_t max_len, int heads, int kv_heads, size_t head_dim);
int mq_chunk_attention(const mq_kv_cache* cache, const int32_t* table, size_t table_width, const int32_t* first,
                       const int32_t* lens, size_t B, size_t T, size_t max_len, int causal, const void* q, size_t ldq, int heads,
                       int dtype, float scale, void* out, size_t ldo, void* ws, size_t ws_bytes, void* stream);

/* ---- tables of continued sequences ---------------------------------------------
 * Row b of the new table, of B_new, continues sequence p = parent[b] of the old one, of B; parent values outside [0, B) begin an
 * empty sequence.  Any number of rows may continue one sequence; a sequence that no row continues is dropped, and its blocks are
 * free again as soon as no row of the new table has them.  There is no count of references to keep: who uses a block says the
 * table alone.
 *   lens: device int32 [B], tokens the cache holds of each sequence (values outside [0, 64 table_width] count as the nearest bound).
 *   keep: device int32 [blocks] or NULL; a block with keep != 0 is held by somebody else (a prompt kept for later): it is read
 *     by any number of rows, never written to, moved or handed out.
 *   grow: device int32 [B_new], tokens that the next append brings to row b (negative ones count as 0).
 * Row b takes over the first ceil(len / 64) entries of its parent (entries that are no block become -1).  If its last block is
 * part full and grow[b] > 0, row b will write to it: if it is kept, if any row has it without writing to it, or if a lower row
 * writes to it, row b gets a new block with a copy of it.  Further entries up to ceil((len + grow[b]) / 64), table_width at most,
 * are new blocks.  New blocks are those that are not kept and that no row takes over, handed out in ascending order to the entries
 * in order of (row, column).  Entries for which none is left, and all others, are -1.
 *   table_new: device int32 [B_new][table_width]; lens_new: device int32 [B_new], the parent's len (what mq_kv_append takes
 *     as `held`); neither may overlap table or lens.  missing: device int32 [1], entries for which no block was left (a part full
 *     block among them is lost to its row: where missing is not 0, continue fewer rows from the old table; no block that the old
 *     table's rows hold and that some row continues has been written to).
 * The old table's other rows are not valid any more: their free blocks may have been handed out.
 * ws: device, 16-byte aligned, mq_kv_fork_ws_bytes (0 for invalid arguments).  blocks < 2^30, B_new table_width < 2^32.  Two
 * launches for small tables (up to 8192 blocks, 4096 rows, 16384 entries), else four. */
size_t mq_kv_fork_ws_bytes(size_t blocks, size_t B_new, size_t table_width);
int mq_kv_fork(const mq_kv_cache* cache, const int32_t* keep, const int32_t* table, size_t table_width, const int32_t* lens,
               size_t B, const int32_t* parent, const int32_t* grow, size_t B_new, int32_t* table_new, int32_t* lens_new,
               int32_t* missing, void* ws, size_t ws_bytes, void* stream);

/* Moves blocks so that the used ones are the first: with U blocks used (kept, or among the first ceil(lens[b] / 64) entries of
 * a row), used blocks U, U + 1, .. go, in ascending order, to the unused ones below U, in ascending order; the others stay.
 *   table_new: device int32 [B][table_width]: the table after that (it may be `table` itself); entries past a sequence's tokens
 *     and entries that are no block are -1.
 *   moved: device int32 [blocks], required: where each block is now, -1 for unused ones (for holders of kept blocks).
 *   used: device int32 [1], U.
 * keep as above (and to be renumbered by the caller, from moved).  ws: mq_kv_compact_ws_bytes.  blocks < 2^30.  Two launches for
 * small tables, as above, else four. */
size_t mq_kv_compact_ws_bytes(size_t blocks);
int mq_kv_compact(const mq_kv_cache* cache, const int32_t* keep, const int32_t* table, size_t table_width, const int32_t* lens,
                  size_t B, int32_t* table_new, int32_t* moved, int32_t* used, void* ws, size_t ws_bytes, void* stream);

/* ---- residual addition and root-mean-square norm -----------------------------------
 * For M rows of d <= 16384 elements of a type:
 *   h = x + r, rounded to the type (h = x where r is NULL);   y = h / sqrt(mean(h^2) + eps) gamma
 * in binary32 (h^2 is summed in binary32: below 2^56 nothing overflows; squares of elements below 2^-63 lose bits, which shows where
 * eps is smaller still).  gamma: device float [d].  h: rows that receive h, or NULL; h may be x or r itself, and y may be, with its
 * ld, but h and y must not overlap.  One launch each.
 *   mq_add_rms_norm:        y rounded to the type, rows ldy apart.
 *   mq_add_rms_norm_rows8:  q[m][i] = clamp(rne(y s), +-127) as int8 rows ldq apart, with a multiplier for each row,
 *     s = scale[m] = 127 / max |y|, the largest binary32 number at most (1 for a row of zeros; NaN, and zeros in q, for a row that
 *     holds a NaN or an infinity).
 *   mq_add_rms_norm_pack8:  q = quant_int(y, s[0]), device float [1] given, as the packed 8-bit operand of mq.h's products
 *     (mq_packed_bytes(8, M, d) bytes, padding included, 16-byte aligned). */
int mq_add_rms_norm(const void* x, size_t ldx, const void* r, size_t ldr, int dtype, const float* gamma, size_t M, size_t d,
                    float eps, void* h, size_t ldh, void* y, size_t ldy, void* stream);
int mq_add_rms_norm_rows8(const void* x, size_t ldx, const void* r, size_t ldr, int dtype, const float* gamma, size_t M, size_t d,
                          float eps, void* h, size_t ldh, int8_t* q, size_t ldq, float* scale, void* stream);
int mq_add_rms_norm_pack8(const void* x, size_t ldx, const void* r, size_t ldr, int dtype, const float* gamma, size_t M, size_t d,
                          float eps, void* h, size_t ldh, const float* s, void* packed, void* stream);

/* ---- parameters in 4 bits ------------------------------------------------------
 * Element k of row n of an [N x K] parameter is (c - z) s with a code c and, for every group of `group` (32, 64 or 128) neighbours
 * along k, a zero z, both in 0 .. 15, and a scale s.  The last group of a row may be shorter.  groups = ceil(K / group).
 * Scales are held with 20 bits of mantissa (rounded to nearest: all of a binary16 or bfloat16 value; scales below 2^-126 are
 * rounded to multiples of 2^-145).  N, K <= 2^24.
 *   mq_w4_bytes: size of the packed parameter (0 for invalid arguments), opaque and position independent.
 *   mq_w4_pack: codes device uint8 [N x K] (the low four bits count), scales device float [N x groups], zeros device uint8
 *     [N x groups] or NULL (8 everywhere).
 *   mq_w4_prepare: codes and scales of a device float [N x K]: z = 8, s = max |w| of the group / 7 (rounded to what is held),
 *     c = 8 + clamp(rne(w / s), -8, 7).  NaNs become 0; a group that holds an infinity comes out as NaN altogether.
 *   mq_w4_unpack: w device float [N x K] receives (c - z) s. */
size_t mq_w4_bytes(size_t N, size_t K, int group);
int mq_w4_pack(const uint8_t* codes, const float* scales, const uint8_t* zeros, size_t N, size_t K, int group, void* packed,
               void* stream);
int mq_w4_prepare(const float* w, size_t N, size_t K, int group, void* packed, void* stream);
int mq_w4_unpack(const void* packed, size_t N, size_t K, int group, float* w, void* stream);

/* y[m][n] = sum_k x[m][k] (c[n][k] - z) s + bias[n] for a few rows (about 1 to 200; any number is served but for launches of 2^32
 * threads: some rows / 32 x N / 64 >= 2^24).
 *   x: M rows of K elements, ldx apart, of type xtype: an mq_dtype, or MQ_ROWS8: int8 with the multipliers row_scale, device
 *     float [M] (an element q stands for q / row_scale[m], as mq_add_rms_norm_rows8 leaves them); row_scale is NULL for the others.
 *   y: M rows of N elements, ldy apart, of type ytype (an mq_dtype).  bias: device float [N] or NULL.
 * x enters the products exactly (1, 1, 2, 3 bfloat16 parts for int8, bfloat16, binary16, binary32; of magnitudes below 2^-100 the
 * last bits of the latter may be lost), codes and zeros exactly (of binary32 rows c - z, of the others c and z in sums of their own),
 * scales after the sums over a group; sums are binary32, and up to 31 sum |x| over a group must be one of its numbers.  A row of x
 * with a NaN or an infinity gives no finite number.  y must not overlap x.  packed: 16-byte aligned.  ws: device, 16-byte aligned,
 * mq_w4_product_ws_bytes(M, N, K) bytes (0 for invalid arguments).  One launch for up to 32, 16 or 8 rows (8-bit and bfloat16,
 * binary16, binary32) if they are whole 16-byte pieces, else two, or three where a contraction is split over workgroups. */
#define MQ_ROWS8 3
size_t mq_w4_product_ws_bytes(size_t M, size_t N, size_t K);
int mq_w4_product(const void* x, size_t ldx, int xtype, const float* row_scale, const void* packed, size_t M, size_t N, size_t K,
                  int group, const float* bias, void* y, size_t ldy, int ytype, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MQ_SERVE_H_ */
