// C boundary of the sequence operators (include/mq_seq.h): argument checks, then launches.  Nothing here computes.
#include "mq_seq_common.h"

namespace mq {
namespace {

constexpr size_t kMaxRows = (size_t)1 << 30;        // token rows, sequences, table columns
constexpr size_t kMaxElems = (size_t)1 << 40;
constexpr size_t kMaxDim = 256, kMaxHeads = 1024;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
bool dtype_ok(int dtype) { return dtype == MQ_F32 || dtype == MQ_F16 || dtype == MQ_BF16; }
bool heads_ok(int heads, int kv_heads, size_t d) {
  return heads > 0 && kv_heads > 0 && (size_t)heads <= kMaxHeads && heads % kv_heads == 0 && d >= 1 && d <= kMaxDim;
}
bool count_ok(size_t n) { return n >= 1 && n <= kMaxRows; }
// rows of `heads` heads, `ld` elements apart
bool rows_ok(size_t rows, size_t ld, int heads, size_t d) {
  return count_ok(rows) && ld >= (size_t)heads * d && ld <= kMaxElems / rows;
}

int cache_checks(const mq_kv_cache* c, const int32_t* table, size_t table_width) {
  if (c == nullptr || table == nullptr || c->keys == nullptr || c->values == nullptr || c->amax == nullptr) return MQ_ERR_NULL;
  if (!heads_ok(c->kv_heads, c->kv_heads, c->head_dim) || c->blocks == 0 || c->blocks >= (size_t)1 << 31 ||
      mq_kv_key_bytes(c->blocks, c->kv_heads, c->head_dim) == 0 || !count_ok(table_width))
    return MQ_ERR_SHAPE;
  if (!aligned(c->keys, 16) || !aligned(c->values, 16) || !aligned(c->amax, 8) || !aligned(table, 4)) return MQ_ERR_ALIGN;
  return MQ_OK;
}

}  // namespace
}  // namespace mq

using namespace mq;

extern "C" {

size_t mq_kv_key_bytes(size_t blocks, int kv_heads, size_t head_dim) {
  if (!heads_ok(kv_heads, kv_heads, head_dim) || blocks == 0 || blocks >= (size_t)1 << 31) return 0;
  return blocks * (size_t)kv_heads * kKvBlock * kv_dk((unsigned)head_dim);
}

size_t mq_kv_value_bytes(size_t blocks, int kv_heads, size_t head_dim) {
  if (!heads_ok(kv_heads, kv_heads, head_dim) || blocks == 0 || blocks >= (size_t)1 << 31) return 0;
  return blocks * (size_t)kv_heads * kKvBlock * kv_dv((unsigned)head_dim);
}

int mq_kv_append(const mq_kv_cache* cache, const int32_t* table, size_t table_width, const int32_t* first, const int32_t* held,
                 size_t B, size_t T, const void* k, size_t ldk, const void* v, size_t ldv, const void* q, size_t ldq,
                 int heads, int dtype, const float* freq, size_t rot, int interleaved, void* k_out, void* q_out, void* stream) {
  if (!dtype_ok(dtype)) return MQ_ERR_DTYPE;
  const int rc = cache_checks(cache, table, table_width);
  if (rc != MQ_OK) return rc;
  if (held == nullptr || k == nullptr || v == nullptr || (q == nullptr) != (q_out == nullptr) || (rot > 0 && freq == nullptr))
    return MQ_ERR_NULL;
  const int hk = cache->kv_heads;
  const size_t d = cache->head_dim, es = elem_bytes(dtype);
  if (!count_ok(B) || !count_ok(T) || (first == nullptr && T != B) || !rows_ok(T, ldk, hk, d) || !rows_ok(T, ldv, hk, d))
    return MQ_ERR_SHAPE;
  if (rot % 2 != 0 || rot > d) return MQ_ERR_SHAPE;
  if (q != nullptr && (!heads_ok(heads, hk, d) || !rows_ok(T, ldq, heads, d))) return MQ_ERR_SHAPE;
  if (!aligned(held, 4) || (first != nullptr && !aligned(first, 4)) || !aligned(k, es) || !aligned(v, es) ||
      (q != nullptr && (!aligned(q, es) || !aligned(q_out, es))) || (k_out != nullptr && !aligned(k_out, es)) ||
      (freq != nullptr && !aligned(freq, 4)))
    return MQ_ERR_ALIGN;
  return launch_kv_append(*cache, table, table_width, first, held, B, T, k, ldk, v, ldv, q, ldq, heads, dtype, freq, rot,
                          interleaved, k_out, q_out, static_cast<hipStream_t>(stream));
}

size_t mq_cached_attention_ws_bytes(size_t B, size_t max_len, int heads, int kv_heads, size_t head_dim) {
  if (!heads_ok(heads, kv_heads, head_dim) || !count_ok(B) || !count_ok(max_len)) return 0;
  return cached_attention_ws_bytes(B, max_len, heads, kv_heads, head_dim);
}

int mq_cached_attention(const mq_kv_cache* cache, const int32_t* table, size_t table_width, const int32_t* lens, size_t B,
                        size_t max_len, const void* q, size_t ldq, int heads, int dtype, float scale, void* out, size_t ldo,
                        void* ws, size_t ws_bytes, void* stream) {
  if (!dtype_ok(dtype)) return MQ_ERR_DTYPE;
  const int rc = cache_checks(cache, table, table_width);
  if (rc != MQ_OK) return rc;
  if (lens == nullptr || q == nullptr || out == nullptr || ws == nullptr) return MQ_ERR_NULL;
  const size_t d = cache->head_dim, es = elem_bytes(dtype);
  if (!heads_ok(heads, cache->kv_heads, d) || !count_ok(max_len) || max_len > table_width * kKvBlock ||
      !rows_ok(B, ldq, heads, d) || !rows_ok(B, ldo, heads, d))
    return MQ_ERR_SHAPE;
  if (!aligned(lens, 4) || !aligned(q, es) || !aligned(out, es) || !aligned(ws, 16)) return MQ_ERR_ALIGN;
  if (ws_bytes < mq_cached_attention_ws_bytes(B, max_len, heads, cache->kv_heads, d)) return MQ_ERR_WORKSPACE;
  return launch_cached_attention(*cache, table, table_width, lens, B, max_len, q, ldq, heads, dtype, scale, out, ldo, ws,
                                 static_cast<hipStream_t>(stream));
}

size_t mq_prompt_attention_ws_bytes(int dtype, size_t B, size_t Tk, int kv_heads, size_t head_dim) {
  if (!dtype_ok(dtype) || !heads_ok(kv_heads, kv_heads, head_dim) || !count_ok(B) || !count_ok(Tk)) return 0;
  return prompt_attention_ws_bytes(dtype, B, Tk, kv_heads, head_dim);
}

int mq_prompt_attention(const void* q, size_t ldq, const void* k, size_t ldk, const void* v, size_t ldv, int dtype,
                        const int32_t* q_first, const int32_t* k_first, size_t B, size_t Tq, size_t Tk, int heads,
                        int kv_heads, size_t head_dim, int causal, float scale, void* out, size_t ldo, void* ws,
                        size_t ws_bytes, void* stream) {
  if (!dtype_ok(dtype)) return MQ_ERR_DTYPE;
  if (q == nullptr || k == nullptr || v == nullptr || q_first == nullptr || k_first == nullptr || out == nullptr || ws == nullptr)
    return MQ_ERR_NULL;
  if (!heads_ok(heads, kv_heads, head_dim) || !count_ok(B) || !rows_ok(Tq, ldq, heads, head_dim) ||
      !rows_ok(Tk, ldk, kv_heads, head_dim) || !rows_ok(Tk, ldv, kv_heads, head_dim) || !rows_ok(Tq, ldo, heads, head_dim))
    return MQ_ERR_SHAPE;
  const size_t es = elem_bytes(dtype);
  if (!aligned(q, es) || !aligned(k, es) || !aligned(v, es) || !aligned(out, es) || !aligned(q_first, 4) ||
      !aligned(k_first, 4) || !aligned(ws, 256))
    return MQ_ERR_ALIGN;
  if (ws_bytes < mq_prompt_attention_ws_bytes(dtype, B, Tk, kv_heads, head_dim)) return MQ_ERR_WORKSPACE;
  return launch_prompt_attention(q, ldq, k, ldk, v, ldv, dtype, q_first, k_first, B, Tq, Tk, heads, kv_heads, head_dim, causal,
                                 scale, out, ldo, ws, static_cast<hipStream_t>(stream));
}

size_t mq_token_logprob_ws_bytes(size_t M, size_t N, int k) {
  if (!count_ok(M) || !count_ok(N) || k < 0 || k > 8) return 0;
  return token_logprob_ws_bytes(M, N, k);
}

int mq_gemm_token_logprob_packed(const void* packedA, const void* packedW, size_t M, size_t N, size_t K, const float* sA,
                                 const float* sW, const int32_t* target, int k, float* logprob, float* entropy,
                                 int32_t* tok, float* alt_logprob, void* ws, size_t ws_bytes, void* stream) {
  if (packedA == nullptr || packedW == nullptr || sA == nullptr || sW == nullptr || target == nullptr || logprob == nullptr ||
      ws == nullptr || (k > 0 && (tok == nullptr || alt_logprob == nullptr)))
    return MQ_ERR_NULL;
  if (!count_ok(M) || !count_ok(N) || !count_ok(K) || k < 0 || k > 8 || (size_t)k > N || M > kMaxElems / N) return MQ_ERR_SHAPE;
  if (!aligned(packedA, 16) || !aligned(packedW, 16) || !aligned(sA, 4) || !aligned(sW, 4) || !aligned(target, 4) ||
      !aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(tok, 4) || !aligned(alt_logprob, 4) || !aligned(ws, 16))
    return MQ_ERR_ALIGN;
  if (K > 1024 || N > (size_t)1 << 24) return MQ_ERR_UNSUPPORTED;
  if (ws_bytes < mq_token_logprob_ws_bytes(M, N, k)) return MQ_ERR_WORKSPACE;
  return launch_token_logprob(packedA, packedW, M, N, K, sA, sW, target, k, logprob, entropy, tok, alt_logprob, ws,
                              static_cast<hipStream_t>(stream));
}

}  // extern "C"
