// Residual addition and root-mean-square norm (include/mq_serve.h): h = x + r, y = h / sqrt(mean(h^2) + eps) gamma.
//
// One pass: a row stays in registers between its sum of squares and its store, a wave for a row of up to 512 elements, a workgroup
// of 256 threads for a longer one, in pieces of 8 elements a thread.  Bound by bytes where rows are many (8192 rows of 4096 bfloat16,
// x, r, h and y: 268 MB in 55 us, 4.85 TB/s; a copy of that size reaches 4.7), else by the way of one row (64 rows of 4096: 5.6 us).
#include <type_traits>

#include "mq_glue.h"
#include "mq_serve_common.h"

namespace mq {

namespace {

constexpr int kV = 8;                 // elements of a thread's piece

template <typename T>
__device__ __forceinline__ void load8(const T* src, unsigned left, bool wide, float (&v)[kV]) {
  if (wide) {
    constexpr int W = 16 / sizeof(T);
    typedef T tw __attribute__((ext_vector_type(W)));
#pragma unroll
    for (int j = 0; j < kV; j += W) {
      const tw w = *reinterpret_cast<const tw*>(src + j);
#pragma unroll
      for (int k = 0; k < W; ++k) v[j + k] = (float)w[k];
    }
  } else {
#pragma unroll
    for (int j = 0; j < kV; ++j) v[j] = j < (int)left ? (float)src[j] : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* dst, unsigned left, bool wide, const float (&v)[kV]) {
  if (wide) {
    constexpr int W = 16 / sizeof(T);
    typedef T tw __attribute__((ext_vector_type(W)));
#pragma unroll
    for (int j = 0; j < kV; j += W) {
      tw w;
#pragma unroll
      for (int k = 0; k < W; ++k) w[k] = (T)v[j + k];
      *reinterpret_cast<tw*>(dst + j) = w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < kV; ++j)
      if (j < (int)left) dst[j] = (T)v[j];
  }
}

// quant_int of one value, as a byte
__device__ __forceinline__ unsigned quant8(float x, float s) {
  const float y = rintf(x * s);
  return (unsigned)(int)(y != y ? 0.f : fminf(fmaxf(y, -127.f), 127.f)) & 255u;
}

// op over the threads of a row: a wave, or all of the workgroup through `box`
template <bool WIDE_ROW, typename Op>
__device__ __forceinline__ float row_reduce(float v, float* box, Op op) {
  v = wave_reduce_f(v, op);
  if constexpr (WIDE_ROW) {
    const unsigned wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
    if (threadIdx.x % kWave == 0) box[wave] = v;
    __syncthreads();
    v = box[0];
    for (unsigned w = 1; w < waves; ++w) v = op(v, box[w]);
  }
  return v;
}

// WIDE_ROW: a workgroup for a row, else a wave; CH: pieces of a thread.  wide: whole 16-byte pieces everywhere (bits: x, r, h, y).
template <int DT, int FORM, bool WIDE_ROW, int CH>
__global__ __launch_bounds__(256) void k_rms_norm(const NormArgs p, unsigned wide) {
  using T = typename Elem<DT>::T;
  __shared__ float box[2][4];
  const unsigned threads = WIDE_ROW ? blockDim.x : kWave, t = WIDE_ROW ? threadIdx.x : threadIdx.x % kWave;
  const size_t m = WIDE_ROW ? blockIdx.x : (size_t)blockIdx.x * (blockDim.x / kWave) + threadIdx.x / kWave;
  const unsigned padded = FORM == kNormPack8 ? (p.M + kFragRows - 1) / kFragRows * kFragRows : p.M;
  if (m >= padded) return;
  const bool real = m < p.M;            // (rows behind the last are zeros of a packed operand)
  float v[CH][kV], sum = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const unsigned i = (c * threads + t) * kV, left = real && i < p.d ? p.d - i : 0;
#pragma unroll
    for (int j = 0; j < kV; ++j) v[c][j] = 0.f;
    if (left > 0) {
      load8(static_cast<const T*>(p.x) + m * p.ldx + i, left, left >= kV && (wide & 1), v[c]);
      if (p.r != nullptr) {
        float r[kV];
        load8(static_cast<const T*>(p.r) + m * p.ldr + i, left, left >= kV && (wide & 2), r);
#pragma unroll
        for (int j = 0; j < kV; ++j) v[c][j] = (float)(T)(v[c][j] + r[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < kV; ++j) sum = fmaf(v[c][j], v[c][j], sum);
  }
  sum = row_reduce<WIDE_ROW>(sum, box[0], [](float a, float b) { return a + b; });
  const float rms = __fdiv_rn(1.f, __fsqrt_rn(__fdiv_rn(sum, (float)p.d) + p.eps));
  float most = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const unsigned i = (c * threads + t) * kV, left = real && i < p.d ? p.d - i : 0;
    if (left == 0) continue;
    float g[kV];
    load8(p.gamma + i, left, left >= kV && (wide & 16), g);
    if (p.h != nullptr) store8(static_cast<T*>(p.h) + m * p.ldh + i, left, left >= kV && (wide & 4), v[c]);
#pragma unroll
    for (int j = 0; j < kV; ++j) {
      v[c][j] = v[c][j] * rms * g[j];
      if (j < (int)left) most = fmaxf(most, fabsf(v[c][j]));
    }
    if constexpr (FORM == kNormType) store8(static_cast<T*>(p.y) + m * p.ldy + i, left, left >= kV && (wide & 8), v[c]);
  }
  if constexpr (FORM == kNormType) return;
  float s;
  if constexpr (FORM == kNormRows8) {
    most = row_reduce<WIDE_ROW>(most, box[1], [](float a, float b) { return fmaxf(a, b); });
    // a NaN or an infinity in h shows in the sum of squares, one that gamma makes in the maximum or not at all
    // (an infinite multiplier, of a row below 127 / the largest number, would make 127 of all that is not zero)
    s = !(sum <= 3.402823466e38f) || most == INFINITY ? NAN : most > 0.f ? fminf(__fdiv_rn(127.f, most), 3.402823466e38f) : 1.f;
    if (t == 0) p.scale[m] = s;
  } else {
    s = *p.s;
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const unsigned i = (c * threads + t) * kV;
    unsigned b[kV];
#pragma unroll
    for (int j = 0; j < kV; ++j) b[j] = real && i + j < p.d ? quant8(v[c][j], s) : 0;
    const uint2 w = make_uint2(b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24, b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24);
    if constexpr (FORM == kNormRows8) {
      int8_t* dst = static_cast<int8_t*>(p.y) + m * p.ldy + i;
      if (i + kV <= p.d && (wide & 8)) {
        *reinterpret_cast<uint2*>(dst) = w;
      } else {
#pragma unroll
        for (int j = 0; j < kV; ++j)
          if (i + j < p.d) dst[j] = (int8_t)b[j];
      }
    } else {
      const PackedDims pd(8, p.M, p.d);
      if (i < pd.Kp)
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y) + pd.frag_offset(m / kFragRows, i / kFragK) +
                                  (m % kFragRows + 32 * (i % kFragK / 16)) * 16 + i % 16) = w;
    }
  }
}

}  // namespace

int launch_rms_norm(const NormArgs& a, int dtype, NormForm form, hipStream_t s) {
  const size_t es = elem_bytes(dtype), piece = 16 / es;
  auto whole = [&](const void* p, size_t ld, size_t n, size_t align) {
    return ld % n == 0 && reinterpret_cast<uintptr_t>(p) % align == 0;
  };
  unsigned wide = 0;
  if (whole(a.x, a.ldx, piece, 16)) wide |= 1;
  if (whole(a.r, a.ldr, piece, 16)) wide |= 2;
  if (whole(a.h, a.ldh, piece, 16)) wide |= 4;
  if (form == kNormType ? whole(a.y, a.ldy, piece, 16) : whole(a.y, a.ldy, 8, 8)) wide |= 8;
  if (whole(a.gamma, 0, 4, 16)) wide |= 16;
  const size_t rows = form == kNormPack8 ? round_up(a.M, kFragRows) : a.M;
  // a packed row reaches to the next multiple of 64 elements
  const size_t d = form == kNormPack8 ? round_up(a.d, kKPad) : a.d;
  const bool wide_row = d > (size_t)kWave * kV;
  const size_t wgs = wide_row ? rows : (rows + 3) / 4;
  if (!launchable(wgs, 256)) return MQ_ERR_SHAPE;
  return with_dtype(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    auto go = [&](auto kern) {
      hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(256), 0, s, a, wide);
      return check_hip(hipGetLastError());
    };
    auto sized = [&](auto f) {
      constexpr int F = decltype(f)::value;
      if (!wide_row) return go(k_rms_norm<DT, F, false, 1>);
      if (d <= 2048) return go(k_rms_norm<DT, F, true, 1>);
      if (d <= 4096) return go(k_rms_norm<DT, F, true, 2>);
      if (d <= 8192) return go(k_rms_norm<DT, F, true, 4>);
      return go(k_rms_norm<DT, F, true, 8>);
    };
    switch (form) {
      case kNormType: return sized(std::integral_constant<int, kNormType>{});
      case kNormRows8: return sized(std::integral_constant<int, kNormRows8>{});
      default: return sized(std::integral_constant<int, kNormPack8>{});
    }
  });
}

}  // namespace mq
