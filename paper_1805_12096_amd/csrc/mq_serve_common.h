// Pieces shared by the kernels of the serving operators (include/mq_serve.h).
#pragma once

#include "mq_gemm_common.h"
#include "mq_seq_common.h"
#include "mq_serve.h"

namespace mq {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

// How many bfloat16 parts hold every bit of an element.
template <int DT>
constexpr int kParts = DT == MQ_F32 ? 3 : DT == MQ_F16 ? 2 : 1;

// x as a sum of NP bfloat16 values, each the nearest to what the ones before leave over.
template <int NP>
__device__ __forceinline__ void split_bf16(float x, __bf16 (&part)[NP]) {
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    part[i] = (__bf16)x;
    if (i + 1 < NP) x -= (float)part[i];
  }
}

// Byte I of a word, signed, as binary32: one instruction (the compiler takes up to three).
template <int I>
__device__ __forceinline__ float f32_of_byte(unsigned x) {
  float y;
  if constexpr (I == 0) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(y) : "v"(x));
  else if constexpr (I == 1) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(y) : "v"(x));
  else if constexpr (I == 2) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(y) : "v"(x));
  else asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(y) : "v"(x));
  return y;
}
// Eight signed bytes as bfloat16 values (8 bits: exact): the upper halves of their binary32 values.
__device__ __forceinline__ bf8 bf16_of_bytes(unsigned lo, unsigned hi) {
  auto upper = [](float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); };
  const u4 w = {upper(f32_of_byte<0>(lo), f32_of_byte<1>(lo)), upper(f32_of_byte<2>(lo), f32_of_byte<3>(lo)),
                upper(f32_of_byte<0>(hi), f32_of_byte<1>(hi)), upper(f32_of_byte<2>(hi), f32_of_byte<3>(hi))};
  return __builtin_bit_cast(bf8, w);
}
// Sums of matrix instructions that inline assembly reads next: it keeps the wait states (12 of a 32 x 32 x 16 product) that the
// compiler keeps only in front of instructions of its own.
__device__ __forceinline__ void settle(v16f& a, v16f& b) { asm volatile("s_nop 15" : "+v"(a), "+v"(b)); }
__device__ __forceinline__ void settle(v16f& a) { asm volatile("s_nop 15" : "+v"(a)); }
// The largest of three, NaNs left out (fmaxf would quiet each operand in an instruction of its own).  settle() goes in front of
// it where a matrix instruction wrote an operand.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(y) : "v"(a), "v"(b), "v"(c));
  return y;
}

__device__ __forceinline__ void store_as(void* y, int type, size_t at, float v) {
  if (type == MQ_F32) static_cast<float*>(y)[at] = v;
  else if (type == MQ_F16) static_cast<_Float16*>(y)[at] = (_Float16)v;
  else static_cast<__bf16*>(y)[at] = (__bf16)v;
}

size_t chunk_attention_ws_bytes(size_t B, size_t T, size_t max_len, int heads, int kv_heads, size_t d);
int launch_chunk_attention(const mq_kv_cache& cache, const int32_t* table, size_t table_width, const int32_t* first,
                           const int32_t* lens, size_t B, size_t T, size_t max_len, int causal, const void* q, size_t ldq,
                           int heads, int dtype, float scale, void* out, size_t ldo, void* ws, hipStream_t s);
size_t kv_fork_ws_bytes(size_t blocks, size_t B_new, size_t table_width);
int launch_kv_fork(const mq_kv_cache& cache, const int32_t* keep, const int32_t* table, size_t table_width, const int32_t* lens,
                   size_t B, const int32_t* parent, const int32_t* grow, size_t B_new, int32_t* table_new, int32_t* lens_new,
                   int32_t* missing, void* ws, hipStream_t s);
size_t kv_compact_ws_bytes(size_t blocks);
int launch_kv_compact(const mq_kv_cache& cache, const int32_t* keep, const int32_t* table, size_t table_width, const int32_t* lens,
                      size_t B, int32_t* table_new, int32_t* moved, int32_t* used, void* ws, hipStream_t s);

enum NormForm { kNormType, kNormRows8, kNormPack8 };
struct NormArgs {
  const void *x, *r;
  size_t ldx, ldr, ldh, ldy;            // ldy: of y or q
  const float* gamma;
  void *h, *y;                          // y: rows of the type, int8 rows, or the packed operand
  float* scale;                         // rows8: multipliers out
  const float* s;                       // pack8: the multiplier
  unsigned M, d;
  float eps;
};
int launch_rms_norm(const NormArgs& a, int dtype, NormForm form, hipStream_t s);

size_t w4_bytes(size_t N, size_t K, int group);
int launch_w4_pack(const uint8_t* codes, const float* scales, const uint8_t* zeros, size_t N, size_t K, int group, void* packed,
                   hipStream_t s);
int launch_w4_prepare(const float* w, size_t N, size_t K, int group, void* packed, hipStream_t s);
int launch_w4_unpack(const void* packed, size_t N, size_t K, int group, float* w, hipStream_t s);
size_t w4_product_ws_bytes(size_t M, size_t N, size_t K);
int launch_w4_product(const void* x, size_t ldx, int xtype, const float* row_scale, const void* packed, size_t M, size_t N,
                      size_t K, int group, const float* bias, void* y, size_t ldy, int ytype, void* ws, hipStream_t s);

}  // namespace mq
