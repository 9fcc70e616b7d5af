/*
 * mq_seq.h -- C boundary of the library's operators on token sequences.
 *
 * mq.h serves a decoder whose self-attention is a running average.  The calls here serve models that attend to their own
 * tokens (the Transformer rows of the paper's tables), next to the same 8-bit products:
 *   mq_kv_append                    new keys and values into a paged cache held in 8 bits, rotated by position on the way;
 *   mq_cached_attention             one query per sequence over such a cache (a decode step);
 *   mq_prompt_attention             packed sequences of different lengths (an encoder, a prompt, forced decoding);
 *   mq_gemm_token_logprob_packed    log probabilities of given words, entropy, best alternatives (scoring).
 *
 * The general rules of mq.h hold: device pointers on the current device, caller-owned buffers, calls that only enqueue on
 * `stream` and return an mq_status, arguments checked before anything is enqueued.  No call here waits inside a kernel for
 * other workgroups, none needs a prepared workspace, and none keeps anything from one call to the next; a workspace's
 * contents are irrelevant on entry and undefined on return, so calls that may overlap in time (two streams, two captured
 * graphs) need one each.  Results depend neither on what else runs nor on an order of atomics.
 *
 * Types.  Queries, keys, values and outputs are of one type, an mq_dtype.  Sums, softmax statistics and angles are binary32 or
 * better whatever the type, and a result is rounded to the type once; what enters a product with fewer bits (probabilities, and
 * queries of the cache) stands with each call.  Softmax sums of values are formed before they are divided, so values within a
 * factor of 256 times the number of keys of the largest binary32 value may overflow.
 * Rows.  A "token row" holds heads x head_dim neighbouring elements, head after head; rows are `ld` elements apart
 * (ld >= heads head_dim), so that queries, keys and values may be columns of one product's result.  Base pointers and ld need
 * the alignment of one element only (rows and heads that start on 16 bytes load faster).
 * Heads.  Queries have `heads` heads, keys and values kv_heads; heads is a multiple of kv_heads and query head h reads
 * kv head h / (heads / kv_heads).  1 <= head_dim <= 256, heads <= 1024.
 * Packed sequences.  `first` is a device int32 [B + 1], ascending, first[0] >= 0: sequence b has token rows first[b] ..
 * first[b + 1] - 1.  Empty sequences are allowed; rows in front of first[0] and from first[B] on belong to nobody: nothing of
 * theirs is read or written.  Values outside [0, rows] are taken as the nearest bound, and a sequence whose end lies before
 * its start is empty: a bad list gives wrong results, never a read or write outside the buffers.
 * Sizes.  Rows, sequences and table columns are 1 .. 2^30 each; a call that would take a launch of 2^32 threads or more (some
 * 2^23 sequences x 8 heads, some 2^26 rows to score) is refused with MQ_ERR_SHAPE.
 */
#ifndef MQ_SEQ_H_
#define MQ_SEQ_H_

#include "mq.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum mq_dtype {
  MQ_F32 = 0,   /* binary32 */
  MQ_F16 = 1,   /* binary16 */
  MQ_BF16 = 2   /* bfloat16 */
} mq_dtype;

/* ---- the cache ------------------------------------------------------------
 * Keys and values of `blocks` blocks of MQ_KV_BLOCK tokens, 8 bit, with one scale for each block, head, and keys or values:
 *   keys    int8  [blocks][kv_heads][64][dk]   dk = head_dim rounded up to a multiple of 64
 *   values  int8  [blocks][kv_heads][dv][64]   dv = head_dim rounded up to a multiple of 16; token t of the block lies at
 *                                              place 16 ((t / 4) % 4) + 4 (t / 16) + t % 4 of its row
 *   amax    float [blocks][kv_heads][2]        largest |key|, largest |value| of the block
 * An element q stands for q amax / 127.  mq_kv_key_bytes / mq_kv_value_bytes are the sizes (0 for invalid arguments); amax has
 * 2 blocks kv_heads floats.  Nothing has to be initialised: a block is written whole when its first token arrives.
 * Which blocks a sequence owns says its row of a table, device int32 [B][table_width]: token t of the sequence lies in block
 * table[b][t / 64].  Blocks may be shared by sequences that only read them.  An entry outside [0, blocks) stands for no block:
 * nothing is written there, and attention leaves its tokens out. */
#define MQ_KV_BLOCK 64
typedef struct mq_kv_cache {   /* host struct, device pointers inside */
  int8_t* keys;                /* 16-byte aligned */
  int8_t* values;              /* 16-byte aligned */
  float* amax;                 /* 8-byte aligned */
  size_t blocks;
  int kv_heads;
  size_t head_dim;
} mq_kv_cache;
size_t mq_kv_key_bytes(size_t blocks, int kv_heads, size_t head_dim);
size_t mq_kv_value_bytes(size_t blocks, int kv_heads, size_t head_dim);

/* Appends the tokens of B packed sequences to the cache, and rotates queries and keys by position if asked to.
 *   first: as above over the T token rows of k, v (and q), or NULL if every sequence has one token (T = B).
 *   held: device int32 [B], tokens of the sequence that the cache holds already: its i-th new token takes position
 *     held[b] + i.  Tokens at negative positions or past table_width blocks are left out of the cache.
 *   k, v: token rows of kv_heads heads.  q: token rows of `heads` heads, or NULL.
 *   freq: device float [rot / 2], or NULL with rot = 0.  rot (even, <= head_dim) elements of every head are rotated: pair i
 *     by the angle position freq[i], formed and applied in binary64 and rounded once to binary32.  Pair i is elements
 *     (2 i, 2 i + 1) if interleaved != 0, else (i, i + rot / 2).  Any scaling for long contexts is in freq.
 *   k_out, q_out: NULL, or dense token rows [T x kv_heads head_dim], [T x heads head_dim] that receive the rotated keys and
 *     queries in their type; q_out needs q and the other way round.  They must not overlap the inputs.
 * In the cache, for every block and head and for keys and values each: with a' = the largest finite magnitude among the new
 * tokens and a = max(a', amax), or a = a' if the block's first place is among the new ones (the block then starts anew, its
 * other places zero), elements held become clamp(rne(q (amax / a)), +-127) where a > amax, new ones
 * clamp(rne(x (127 / a)), +-127), each quotient and product rounded to binary32 (127 / 0 counts as 1); NaN becomes 0, amax a.
 * A block that this call writes to must belong to one sequence of it. One launch. */
int mq_kv_append(const mq_kv_cache* cache, const int32_t* table, size_t table_width, const int32_t* first, const int32_t* held,
                 size_t B, size_t T, const void* k, size_t ldk, const void* v, size_t ldv, const void* q, size_t ldq,
                 int heads, int dtype, const float* freq, size_t rot, int interleaved, void* k_out, void* q_out, void* stream);

/* Attention of one query per sequence over the first lens[b] tokens of its cache:
 *   out[b] = sum_t p_t V[t],  p = softmax over t < lens[b] of scale (q[b] . K[t]),  per head;
 * zeros where nothing is there to attend to, else NaN where the query holds a NaN or an infinity.
 *   lens: device int32 [B]; values above max_len count as max_len, negative ones as 0.  max_len <= 64 table_width.
 *   q: token rows [B] of `heads` heads, out likewise (it may be q itself, with ldo = ldq).
 * Queries and probabilities enter the integer products with a scale of their own for each row, binary32 ones as 24-bit
 * values, 16-bit types as 16-bit values; sums are exact, the softmax statistics binary32.
 * ws: device, 16-byte aligned, mq_cached_attention_ws_bytes (0 for invalid arguments).  One launch, two where a sequence is
 * split over workgroups. */
size_t mq_cached_attention_ws_bytes(size_t B, size_t max_len, int heads, int kv_heads, size_t head_dim);
int mq_cached_attention(const mq_kv_cache* cache, const int32_t* table, size_t table_width, const int32_t* lens, size_t B,
                        size_t max_len, const void* q, size_t ldq, int heads, int dtype, float scale, void* out, size_t ldo,
                        void* ws, size_t ws_bytes, void* stream);

/* Attention of packed sequences: sequence b has queries q_first[b] .. and keys k_first[b] .. (both as described at the top,
 * over Tq and Tk token rows).  With n queries and m keys, query i attends to all m keys, or, if causal != 0, to the keys
 * j <= i + m - n (the last query sees all; queries that see none give zeros).
 *   out[i] = sum_j p_j v[j],  p = softmax over the keys seen of scale (q[i] . k[j]),  per head.
 * What lies at places a query does not see never counts, whatever it holds.  A key position with a NaN or an infinity in its
 * key or its value turns the whole output (of that head) of every query that sees it into NaN; a query with a NaN or an
 * infinity that sees any key gives NaN.
 * Binary32 operands are multiplied as binary32, or as three bfloat16 parts that hold all of their 24 bits (of magnitudes below
 * 2^-100 the last ones may be lost); probabilities of 16-bit types are rounded to the type.  Sums and softmax statistics are
 * binary32.
 * ws: device, 256-byte aligned, mq_prompt_attention_ws_bytes (0 for invalid arguments): keys and values in the order the
 * products read them.  Two launches; one where the sequences have up to 192 queries and keys on average, 16-bit
 * types 128 (128 and 48 where head_dim > 128).
 * out must not overlap k or v; it may be q itself, with ldo = ldq. */
size_t mq_prompt_attention_ws_bytes(int dtype, size_t B, size_t Tk, int kv_heads, size_t head_dim);
int mq_prompt_attention(const void* q, size_t ldq, const void* k, size_t ldk, const void* v, size_t ldv, int dtype,
                        const int32_t* q_first, const int32_t* k_first, size_t B, size_t Tq, size_t Tk, int heads,
                        int kv_heads, size_t head_dim, int causal, float scale, void* out, size_t ldo, void* ws,
                        size_t ws_bytes, void* stream);

/* Scores given words under the output layer, with y[n] = (float) acc[n] / (sA sW) over all N words as in
 * mq_gemm_topk_packed, logits never stored:
 *   logprob[m] = y[target[m]] - log sum_n exp(y[n]);  0 where target[m] lies outside [0, N) (a padded place)
 *   entropy[m] = - sum_n p[n] log p[n]                                  (entropy may be NULL)
 *   tok[m][j], alt_logprob[m][j], j < k: the k words with the largest sums, best first, ties towards the lower word, and
 *     their log probabilities                                           (k = 0: both NULL)
 * packedA: [M x K], packedW: [N x K], both 8 bit.  0 <= k <= 8, k <= N.  K <= 1024, N <= 2^24 (MQ_ERR_UNSUPPORTED beyond).
 * The words are exact (chosen on the integer sums); sums of the softmax are binary32.
 * ws: device, 16-byte aligned, mq_token_logprob_ws_bytes(M, N, k) (0 for invalid arguments).  Two launches. */
size_t mq_token_logprob_ws_bytes(size_t M, size_t N, int k);
int mq_gemm_token_logprob_packed(const void* packedA, const void* packedW, size_t M, size_t N, size_t K, const float* sA,
                                 const float* sW, const int32_t* target, int k, float* logprob, float* entropy,
                                 int32_t* tok, float* alt_logprob, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MQ_SEQ_H_ */
