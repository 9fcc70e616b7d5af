// C boundary of the serving operators (include/mq_serve.h): argument checks, then launches.  Nothing here computes.
#include <cmath>

#include "mq_seq_checks.h"
#include "mq_serve_common.h"

using namespace mq;

namespace {

constexpr size_t kMaxTableBlocks = (size_t)1 << 30, kMaxNormDim = 16384, kMaxW4 = (size_t)1 << 24;

bool plain_rows_ok(size_t rows, size_t ld, size_t d) { return count_ok(rows) && ld >= d && ld <= kMaxElems / rows; }
bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }
bool w4_ok(size_t N, size_t K) { return N >= 1 && N <= kMaxW4 && K >= 1 && K <= kMaxW4 && N <= kMaxElems / K; }

// what the three forms of the norm share; out: of y's or q's rows
int norm_checks(const void* x, size_t ldx, const void* r, size_t ldr, int dtype, const float* gamma, size_t M, size_t d, float eps,
                const void* h, size_t ldh) {
  if (!dtype_ok(dtype)) return MQ_ERR_DTYPE;
  if (x == nullptr || gamma == nullptr) return MQ_ERR_NULL;
  if (d == 0 || d > kMaxNormDim || !plain_rows_ok(M, ldx, d) || (r != nullptr && !plain_rows_ok(M, ldr, d)) ||
      (h != nullptr && !plain_rows_ok(M, ldh, d)) || !(eps >= 0.f) || std::isinf(eps))
    return MQ_ERR_SHAPE;
  const size_t es = elem_bytes(dtype);
  if (!aligned(x, es) || !aligned(r, es) || !aligned(h, es) || !aligned(gamma, 4)) return MQ_ERR_ALIGN;
  return MQ_OK;
}

int w4_checks(const void* packed, const void* other, size_t N, size_t K, int group) {
  if (packed == nullptr || other == nullptr) return MQ_ERR_NULL;
  if (!w4_ok(N, K) || !group_ok(group)) return MQ_ERR_SHAPE;
  if (!aligned(packed, 16)) return MQ_ERR_ALIGN;
  return MQ_OK;
}

}  // namespace

extern "C" {

size_t mq_chunk_attention_ws_bytes(size_t B, size_t T, size_t max_len, int heads, int kv_heads, size_t head_dim) {
  if (!heads_ok(heads, kv_heads, head_dim) || !count_ok(B) || !count_ok(T) || !count_ok(max_len)) return 0;
  return chunk_attention_ws_bytes(B, T, max_len, heads, kv_heads, head_dim);
}

int mq_chunk_attention(const mq_kv_cache* cache, const int32_t* table, size_t table_width, const int32_t* first,
                       const int32_t* lens, size_t B, size_t T, size_t max_len, int causal, const void* q, size_t ldq, int heads,
                       int dtype, float scale, void* out, size_t ldo, void* ws, size_t ws_bytes, void* stream) {
  if (!dtype_ok(dtype)) return MQ_ERR_DTYPE;
  const int rc = cache_checks(cache, table, table_width);
  if (rc != MQ_OK) return rc;
  if (first == nullptr || lens == nullptr || q == nullptr || out == nullptr || ws == nullptr) return MQ_ERR_NULL;
  const size_t d = cache->head_dim, es = elem_bytes(dtype);
  if (!heads_ok(heads, cache->kv_heads, d) || !count_ok(B) || !count_ok(max_len) || max_len > table_width * kKvBlock ||
      !rows_ok(T, ldq, heads, d) || !rows_ok(T, ldo, heads, d))
    return MQ_ERR_SHAPE;
  if (!aligned(first, 4) || !aligned(lens, 4) || !aligned(q, es) || !aligned(out, es) || !aligned(ws, 16)) return MQ_ERR_ALIGN;
  if (ws_bytes < mq_chunk_attention_ws_bytes(B, T, max_len, heads, cache->kv_heads, d)) return MQ_ERR_WORKSPACE;
  return launch_chunk_attention(*cache, table, table_width, first, lens, B, T, max_len, causal, q, ldq, heads, dtype, scale, out,
                                ldo, ws, static_cast<hipStream_t>(stream));
}

size_t mq_kv_fork_ws_bytes(size_t blocks, size_t B_new, size_t table_width) {
  if (blocks == 0 || blocks >= kMaxTableBlocks || !count_ok(B_new) || !count_ok(table_width)) return 0;
  return kv_fork_ws_bytes(blocks, B_new, table_width);
}

int mq_kv_fork(const mq_kv_cache* cache, const int32_t* keep, const int32_t* table, size_t table_width, const int32_t* lens,
               size_t B, const int32_t* parent, const int32_t* grow, size_t B_new, int32_t* table_new, int32_t* lens_new,
               int32_t* missing, void* ws, size_t ws_bytes, void* stream) {
  const int rc = cache_checks(cache, table, table_width);
  if (rc != MQ_OK) return rc;
  if (lens == nullptr || parent == nullptr || grow == nullptr || table_new == nullptr || lens_new == nullptr || missing == nullptr ||
      ws == nullptr)
    return MQ_ERR_NULL;
  if (!count_ok(B) || !count_ok(B_new) || cache->blocks >= kMaxTableBlocks || table_width > kMaxTableBlocks / 64 ||
      B > kMaxElems / table_width || B_new > 0xffffffffu / table_width)        // (new entries are counted in 32 bits)
    return MQ_ERR_SHAPE;
  if (!aligned(keep, 4) || !aligned(lens, 4) || !aligned(parent, 4) || !aligned(grow, 4) || !aligned(table_new, 4) ||
      !aligned(lens_new, 4) || !aligned(missing, 4) || !aligned(ws, 16))
    return MQ_ERR_ALIGN;
  if (ws_bytes < mq_kv_fork_ws_bytes(cache->blocks, B_new, table_width)) return MQ_ERR_WORKSPACE;
  return launch_kv_fork(*cache, keep, table, table_width, lens, B, parent, grow, B_new, table_new, lens_new, missing, ws,
                        static_cast<hipStream_t>(stream));
}

size_t mq_kv_compact_ws_bytes(size_t blocks) {
  if (blocks == 0 || blocks >= kMaxTableBlocks) return 0;
  return kv_compact_ws_bytes(blocks);
}

int mq_kv_compact(const mq_kv_cache* cache, const int32_t* keep, const int32_t* table, size_t table_width, const int32_t* lens,
                  size_t B, int32_t* table_new, int32_t* moved, int32_t* used, void* ws, size_t ws_bytes, void* stream) {
  const int rc = cache_checks(cache, table, table_width);
  if (rc != MQ_OK) return rc;
  if (lens == nullptr || table_new == nullptr || moved == nullptr || used == nullptr || ws == nullptr) return MQ_ERR_NULL;
  if (!count_ok(B) || cache->blocks >= kMaxTableBlocks || table_width > kMaxTableBlocks / 64 || B > kMaxElems / table_width)
    return MQ_ERR_SHAPE;
  if (!aligned(keep, 4) || !aligned(lens, 4) || !aligned(table_new, 4) || !aligned(moved, 4) || !aligned(used, 4) || !aligned(ws, 16))
    return MQ_ERR_ALIGN;
  if (ws_bytes < mq_kv_compact_ws_bytes(cache->blocks)) return MQ_ERR_WORKSPACE;
  return launch_kv_compact(*cache, keep, table, table_width, lens, B, table_new, moved, used, ws, static_cast<hipStream_t>(stream));
}

int mq_add_rms_norm(const void* x, size_t ldx, const void* r, size_t ldr, int dtype, const float* gamma, size_t M, size_t d,
                    float eps, void* h, size_t ldh, void* y, size_t ldy, void* stream) {
  const int rc = norm_checks(x, ldx, r, ldr, dtype, gamma, M, d, eps, h, ldh);
  if (rc != MQ_OK) return rc;
  if (y == nullptr) return MQ_ERR_NULL;
  if (!plain_rows_ok(M, ldy, d)) return MQ_ERR_SHAPE;
  if (!aligned(y, elem_bytes(dtype))) return MQ_ERR_ALIGN;
  return launch_rms_norm({x, r, ldx, ldr, ldh, ldy, gamma, h, y, nullptr, nullptr, (unsigned)M, (unsigned)d, eps}, dtype, kNormType,
                         static_cast<hipStream_t>(stream));
}

int mq_add_rms_norm_rows8(const void* x, size_t ldx, const void* r, size_t ldr, int dtype, const float* gamma, size_t M, size_t d,
                          float eps, void* h, size_t ldh, int8_t* q, size_t ldq, float* scale, void* stream) {
  const int rc = norm_checks(x, ldx, r, ldr, dtype, gamma, M, d, eps, h, ldh);
  if (rc != MQ_OK) return rc;
  if (q == nullptr || scale == nullptr) return MQ_ERR_NULL;
  if (!plain_rows_ok(M, ldq, d)) return MQ_ERR_SHAPE;
  if (!aligned(scale, 4)) return MQ_ERR_ALIGN;
  return launch_rms_norm({x, r, ldx, ldr, ldh, ldq, gamma, h, q, scale, nullptr, (unsigned)M, (unsigned)d, eps}, dtype, kNormRows8,
                         static_cast<hipStream_t>(stream));
}

int mq_add_rms_norm_pack8(const void* x, size_t ldx, const void* r, size_t ldr, int dtype, const float* gamma, size_t M, size_t d,
                          float eps, void* h, size_t ldh, const float* s, void* packed, void* stream) {
  const int rc = norm_checks(x, ldx, r, ldr, dtype, gamma, M, d, eps, h, ldh);
  if (rc != MQ_OK) return rc;
  if (s == nullptr || packed == nullptr) return MQ_ERR_NULL;
  if (!aligned(s, 4) || !aligned(packed, 16)) return MQ_ERR_ALIGN;
  return launch_rms_norm({x, r, ldx, ldr, ldh, 0, gamma, h, packed, nullptr, s, (unsigned)M, (unsigned)d, eps}, dtype, kNormPack8,
                         static_cast<hipStream_t>(stream));
}

size_t mq_w4_bytes(size_t N, size_t K, int group) { return w4_ok(N, K) && group_ok(group) ? w4_bytes(N, K, group) : 0; }

int mq_w4_pack(const uint8_t* codes, const float* scales, const uint8_t* zeros, size_t N, size_t K, int group, void* packed,
               void* stream) {
  const int rc = w4_checks(packed, codes, N, K, group);
  if (rc != MQ_OK) return rc;
  if (scales == nullptr) return MQ_ERR_NULL;
  if (!aligned(scales, 4)) return MQ_ERR_ALIGN;
  return launch_w4_pack(codes, scales, zeros, N, K, group, packed, static_cast<hipStream_t>(stream));
}

int mq_w4_prepare(const float* w, size_t N, size_t K, int group, void* packed, void* stream) {
  const int rc = w4_checks(packed, w, N, K, group);
  if (rc != MQ_OK) return rc;
  if (!aligned(w, 4)) return MQ_ERR_ALIGN;
  return launch_w4_prepare(w, N, K, group, packed, static_cast<hipStream_t>(stream));
}

int mq_w4_unpack(const void* packed, size_t N, size_t K, int group, float* w, void* stream) {
  const int rc = w4_checks(packed, w, N, K, group);
  if (rc != MQ_OK) return rc;
  if (!aligned(w, 4)) return MQ_ERR_ALIGN;
  return launch_w4_unpack(packed, N, K, group, w, static_cast<hipStream_t>(stream));
}

size_t mq_w4_product_ws_bytes(size_t M, size_t N, size_t K) {
  if (!count_ok(M) || !w4_ok(N, K) || M > kMaxElems / N || M > kMaxElems / K) return 0;
  return w4_product_ws_bytes(M, N, K);
}

int mq_w4_product(const void* x, size_t ldx, int xtype, const float* row_scale, const void* packed, size_t M, size_t N, size_t K,
                  int group, const float* bias, void* y, size_t ldy, int ytype, void* ws, size_t ws_bytes, void* stream) {
  if ((!dtype_ok(xtype) && xtype != MQ_ROWS8) || !dtype_ok(ytype)) return MQ_ERR_DTYPE;
  if (x == nullptr || packed == nullptr || y == nullptr || ws == nullptr || (xtype == MQ_ROWS8) != (row_scale != nullptr))
    return MQ_ERR_NULL;
  if (!w4_ok(N, K) || !group_ok(group) || !plain_rows_ok(M, ldx, K) || !plain_rows_ok(M, ldy, N)) return MQ_ERR_SHAPE;
  if (!aligned(x, xtype == MQ_ROWS8 ? 1 : elem_bytes(xtype)) || !aligned(row_scale, 4) || !aligned(packed, 16) || !aligned(bias, 4) ||
      !aligned(y, elem_bytes(ytype)) || !aligned(ws, 16))
    return MQ_ERR_ALIGN;
  if (ws_bytes < mq_w4_product_ws_bytes(M, N, K)) return MQ_ERR_WORKSPACE;
  return launch_w4_product(x, ldx, xtype, row_scale, packed, M, N, K, group, bias, y, ldy, ytype, ws,
                           static_cast<hipStream_t>(stream));
}

}  // extern "C"
