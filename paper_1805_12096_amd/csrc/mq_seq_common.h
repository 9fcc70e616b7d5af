// Pieces shared by the kernels of the sequence operators (include/mq_seq.h).
#pragma once

#include <hip/hip_runtime.h>

#include "mq_internal.h"
#include "mq_seq.h"

namespace mq {

// ---- element types ----------------------------------------------------------------------------------------------------

template <int DT>
struct Elem;
template <>
struct Elem<MQ_F32> {
  using T = float;
};
template <>
struct Elem<MQ_F16> {
  using T = _Float16;
};
template <>
struct Elem<MQ_BF16> {
  using T = __bf16;
};
inline size_t elem_bytes(int dtype) { return dtype == MQ_F32 ? 4 : 2; }

// Calls f with the element type as a compile-time constant.
template <typename F>
inline int with_dtype(int dtype, F f) {
  switch (dtype) {
    case MQ_F32: return f(std::integral_constant<int, MQ_F32>{});
    case MQ_F16: return f(std::integral_constant<int, MQ_F16>{});
    default: return f(std::integral_constant<int, MQ_BF16>{});
  }
}

// ---- cache layout -----------------------------------------------------------------------------------------------------

constexpr int kKvBlock = MQ_KV_BLOCK;
__host__ __device__ inline unsigned kv_dk(unsigned d) { return (d + 63) / 64 * 64; }
__host__ __device__ inline unsigned kv_dv(unsigned d) { return (d + 15) / 16 * 16; }
// place of a block's token t in a row of values: the score product leaves lane group g with tokens 16 i + 4 g + r, and these
// are the 16 neighbours that the group's lanes contract in the next product
__host__ __device__ inline unsigned kv_place(unsigned t) { return 16 * ((t / 4) % 4) + 4 * (t / 16) + t % 4; }

// ---- packed sequences -------------------------------------------------------------------------------------------------

// entry b of a list of first rows, as the nearest bound of [0, rows]
__device__ __forceinline__ unsigned first_at(const int32_t* __restrict__ first, unsigned b, unsigned rows) {
  const int f = first[b];
  return f < 0 ? 0u : (unsigned)f > rows ? rows : (unsigned)f;
}

// Last i in [0, n) with key(i) <= x for keys that ascend, -1 if there is none.  The 64 lanes look at 64 entries at a time, so
// that up to 64 entries are one trip to memory and up to 4096 two; every lane gets the answer.  Ends for any keys.
template <typename Key>
__device__ __forceinline__ int wave_search(unsigned n, unsigned x, Key key) {
  const unsigned lane = threadIdx.x % kWave;
  unsigned lo = 0, hi = n;
  while (hi - lo > kWave) {
    const unsigned step = (hi - lo + kWave - 1) / kWave, i = lo + lane * step;
    const unsigned c = __popcll(__ballot(i < hi && key(i < hi ? i : lo) <= x));
    if (c == 0) return -1;
    lo += (c - 1) * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  const unsigned i = lo + lane;
  const unsigned c = __popcll(__ballot(i < hi && key(i < hi ? i : lo) <= x));
  return (int)(lo + c) - 1;
}

// Whether a launch of that many workgroups is one: a grid has fewer than 2^32 threads.
inline bool launchable(size_t workgroups, size_t threads) { return workgroups < ((size_t)1 << 32) / threads; }

int launch_kv_append(const mq_kv_cache& cache, const int32_t* table, size_t table_width, const int32_t* first,
                     const int32_t* held, size_t B, size_t T, const void* k, size_t ldk, const void* v, size_t ldv,
                     const void* q, size_t ldq, int heads, int dtype, const float* freq, size_t rot, int interleaved,
                     void* k_out, void* q_out, hipStream_t s);
size_t cached_attention_ws_bytes(size_t B, size_t max_len, int heads, int kv_heads, size_t d);
int launch_cached_attention(const mq_kv_cache& cache, const int32_t* table, size_t table_width, const int32_t* lens, size_t B,
                            size_t max_len, const void* q, size_t ldq, int heads, int dtype, float scale, void* out,
                            size_t ldo, void* ws, hipStream_t s);
size_t prompt_attention_ws_bytes(int dtype, size_t B, size_t Tk, int kv_heads, size_t d);
int launch_prompt_attention(const void* q, size_t ldq, const void* k, size_t ldk, const void* v, size_t ldv, int dtype,
                            const int32_t* q_first, const int32_t* k_first, size_t B, size_t Tq, size_t Tk, int heads,
                            int kv_heads, size_t d, int causal, float scale, void* out, size_t ldo, void* ws, hipStream_t s);
size_t token_logprob_ws_bytes(size_t M, size_t N, int k);
int launch_token_logprob(const void* packedA, const void* packedW, size_t M, size_t N, size_t K, const float* sA,
                         const float* sW, const int32_t* target, int k, float* logprob, float* entropy, int32_t* tok,
                         float* alt, void* ws, hipStream_t s);

}  // namespace mq
