// Argument checks that the boundaries of the sequence and serving operators share.  Nothing here computes.
#pragma once

#include "mq_seq_common.h"

namespace mq {

constexpr size_t kMaxRows = (size_t)1 << 30;        // token rows, sequences, table columns
constexpr size_t kMaxElems = (size_t)1 << 40;
constexpr size_t kMaxDim = 256, kMaxHeads = 1024;

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline bool dtype_ok(int dtype) { return dtype == MQ_F32 || dtype == MQ_F16 || dtype == MQ_BF16; }
inline bool heads_ok(int heads, int kv_heads, size_t d) {
  return heads > 0 && kv_heads > 0 && (size_t)heads <= kMaxHeads && heads % kv_heads == 0 && d >= 1 && d <= kMaxDim;
}
inline bool count_ok(size_t n) { return n >= 1 && n <= kMaxRows; }
// rows of `heads` heads, `ld` elements apart
inline bool rows_ok(size_t rows, size_t ld, int heads, size_t d) {
  return count_ok(rows) && ld >= (size_t)heads * d && ld <= kMaxElems / rows;
}

inline int cache_checks(const mq_kv_cache* c, const int32_t* table, size_t table_width) {
  if (c == nullptr || table == nullptr || c->keys == nullptr || c->values == nullptr || c->amax == nullptr) return MQ_ERR_NULL;
  if (!heads_ok(c->kv_heads, c->kv_heads, c->head_dim) || c->blocks == 0 || c->blocks >= (size_t)1 << 31 ||
      mq_kv_key_bytes(c->blocks, c->kv_heads, c->head_dim) == 0 || !count_ok(table_width))
    return MQ_ERR_SHAPE;
  if (!aligned(c->keys, 16) || !aligned(c->values, 16) || !aligned(c->amax, 8) || !aligned(table, 4)) return MQ_ERR_ALIGN;
  return MQ_OK;
}

}  // namespace mq
