// Parameters in 4 bits and products of a few rows with them (include/mq_serve.h): y = x w^T, w = (c - z) s.
//
// Packed: fragments of 16 rows x 128 elements, 1 KB, lane l of a wave 16 bytes: word w has the codes of row l % 16, elements
// 32 w + 8 (l / 16) .., what lane l feeds to v_mfma_f32_16x16x32_bf16 as operand a.  Code 2 p lies in nibble p of the word's
// lower half, code 2 p + 1 in nibble p of the upper, so a pair shifted and masked once is two bfloat16 mantissas: 16 + c, exactly.
// y = sum_g s (sum_k (16 + c) x - (16 + z) sum_k x): a product with ones gives sum_k x where the other product leaves its results.
// Scales follow the fragments: a word for each (16 rows, group, row), 20 bits of mantissa of the scale and the zero below them.
#include <type_traits>

#include "mq_glue.h"
#include "mq_serve_common.h"

namespace mq {

namespace {

constexpr unsigned kNT = 16, kKT = 128;          // rows and elements of a fragment
constexpr unsigned kTopScale = 0xfffffff0u;

struct W4Dims {
  size_t tiles, frags, groups;                   // row tiles, fragments and groups (whole fragments') of a row tile
  __host__ __device__ W4Dims(size_t N, size_t K, int group)
      : tiles((N + kNT - 1) / kNT), frags((K + kKT - 1) / kKT), groups(frags * (kKT / group)) {}
  __host__ __device__ size_t scales_at() const { return tiles * frags * 1024; }
  __host__ __device__ size_t bytes() const { return scales_at() + tiles * groups * kNT * sizeof(uint32_t); }
};

__device__ __forceinline__ unsigned held_scale(float s) {        // rounded to 20 bits of mantissa
  const unsigned b = __float_as_uint(s);
  if ((b & 0x7f800000u) == 0x7f800000u) return b & kTopScale;
  return (b + 7u + ((b >> 4) & 1u)) & kTopScale;
}
// where code k of row n lies: its word, and its nibble
__device__ __forceinline__ size_t word_of(const W4Dims& d, size_t n, size_t k) {
  const unsigned kk = k % kKT, lane = n % kNT + 16 * (kk % 32 / 8);
  return ((n / kNT * d.frags + k / kKT) * 1024 + lane * 16) / 4 + kk / 32;
}
__device__ __forceinline__ unsigned nibble_of(size_t k) { return 16 * (k % 2) + 4 * (k % 8 / 2); }

// a thread for each word of codes, then for each scale
template <typename Code, typename Scale>
__device__ __forceinline__ void fill(size_t N, size_t K, int group, void* packed, Code code, Scale scale) {
  const W4Dims d(N, K, group);
  const size_t words = d.tiles * d.frags * 256, scales = d.tiles * d.groups * kNT;
  for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < words + scales; i += (size_t)gridDim.x * blockDim.x) {
    unsigned v = 0;
    if (i < words) {
      const size_t frag = i / 256, tile = frag / d.frags;
      const unsigned lane = i % 256 / 4, w = i % 4;
      const size_t n = tile * kNT + lane % 16, k0 = frag % d.frags * kKT + 32 * w + 8 * (lane / 16);
      for (unsigned j = 0; j < 8; ++j)
        if (n < N && k0 + j < K) v |= (code(n, k0 + j) & 15u) << nibble_of(j);
    } else {
      const size_t at = i - words, n = at / (d.groups * kNT) * kNT + at % kNT, g = at / kNT % d.groups;
      if (n < N && g * group < K) v = scale(n, g);
    }
    static_cast<uint32_t*>(packed)[i] = v;
  }
}

__global__ __launch_bounds__(256) void k_w4_pack(const uint8_t* codes, const float* scales, const uint8_t* zeros, size_t N, size_t K,
                                                 int group, void* packed) {
  const size_t groups = (K + group - 1) / group;
  fill(N, K, group, packed, [&](size_t n, size_t k) { return (unsigned)codes[n * K + k]; },
       [&](size_t n, size_t g) {
         return held_scale(scales[n * groups + g]) | (zeros == nullptr ? 8u : zeros[n * groups + g] & 15u);
       });
}

__device__ float group_scale(const float* w, size_t K, size_t n, size_t g, int group) {
  float most = 0.f;
  for (size_t k = g * group; k < K && k < (g + 1) * group; ++k) most = fmaxf(most, fabsf(w[n * K + k]));
  return __uint_as_float(held_scale(__fdiv_rn(most, 7.f)));
}
__global__ __launch_bounds__(256) void k_w4_prepare(const float* w, size_t N, size_t K, int group, void* packed) {
  const W4Dims d(N, K, group);
  // scales first (a thread for each), codes from them: both by this workgroup, so row tiles are its units
  for (size_t tile = blockIdx.x; tile < d.tiles; tile += gridDim.x) {
    uint32_t* scales = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(packed) + d.scales_at()) + tile * d.groups * kNT;
    for (size_t i = threadIdx.x; i < d.groups * kNT; i += blockDim.x) {
      const size_t n = tile * kNT + i % kNT, g = i / kNT;
      scales[i] = n < N && g * group < K ? __float_as_uint(group_scale(w, K, n, g, group)) | 8u : 0u;
    }
    __syncthreads();
    for (size_t i = threadIdx.x; i < d.frags * 256; i += blockDim.x) {
      const unsigned lane = i % 256 / 4, wd = i % 4;
      const size_t n = tile * kNT + lane % 16, k0 = i / 256 * kKT + 32 * wd + 8 * (lane / 16);
      unsigned v = 0;
      for (unsigned j = 0; j < 8; ++j) {
        if (n >= N || k0 + j >= K) continue;
        const float s = __uint_as_float(scales[(k0 + j) / group * kNT + lane % 16] & kTopScale), x = w[n * K + k0 + j];
        const float q = s > 0.f ? rintf(__fdiv_rn(x, s)) : 0.f;
        v |= (unsigned)(8 + (int)(q != q ? 0.f : fminf(fmaxf(q, -8.f), 7.f))) << nibble_of(j);
      }
      static_cast<uint32_t*>(packed)[tile * d.frags * 256 + i] = v;
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(256) void k_w4_unpack(const void* packed, size_t N, size_t K, int group, float* w) {
  const W4Dims d(N, K, group);
  const uint32_t *words = static_cast<const uint32_t*>(packed),
                 *scales = reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(packed) + d.scales_at());
  for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < N * K; i += (size_t)gridDim.x * blockDim.x) {
    const size_t n = i / K, k = i % K;
    const unsigned c = words[word_of(d, n, k)] >> nibble_of(k) & 15u;
    const unsigned s = scales[(n / kNT * d.groups + k / group) * kNT + n % kNT];
    w[i] = (float)((int)c - (int)(s & 15u)) * __uint_as_float(s & kTopScale);
  }
}

// ---- the product ------------------------------------------------------------------------------------------------------

struct W4Params {
  const void* x;
  const float *row_scale, *bias;
  const uint8_t* packed;
  void* y;
  float* part;
  size_t ldx, ldy;
  unsigned M, N, K, frags;
  int ytype, vec;
};

template <int XT>
struct XElem { using T = typename Elem<XT>::T; };
template <>
struct XElem<MQ_ROWS8> { using T = int8_t; };
template <int XT>
constexpr int kXParts = XT == MQ_ROWS8 ? 1 : kParts<XT == MQ_ROWS8 ? MQ_BF16 : XT>;

// 16 + c of eight codes
__device__ __forceinline__ bf8 codes16(unsigned w) {
  constexpr unsigned mask = 0x00780078u, top = 0x41804180u;
  const u4 v = {(w << 3 & mask) | top, (w >> 1 & mask) | top, (w >> 5 & mask) | top, (w >> 9 & mask) | top};
  return __builtin_bit_cast(bf8, v);
}

// elements k .. k + 7 of a row as parts; left: how many there are
template <int XT, int NP>
__device__ __forceinline__ void x_parts(const typename XElem<XT>::T* src, int left, bool vec, bf8 (&part)[NP]) {
  using T = typename XElem<XT>::T;
  if constexpr (XT == MQ_ROWS8) {
    uint2 b = make_uint2(0, 0);
    if (vec) {
      if (left >= 8) b = *reinterpret_cast<const uint2*>(src);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const unsigned v = j < left ? (unsigned)(uint8_t)src[j] : 0u;
        if (j < 4) b.x |= v << 8 * j;
        else b.y |= v << 8 * (j - 4);
      }
    }
    part[0] = bf16_of_bytes(b.x, b.y);
  } else {
    T v[8];
    if (vec) {                          // (rows are whole pieces then)
      constexpr int W = 16 / sizeof(T);
      typedef T tw __attribute__((ext_vector_type(W)));
#pragma unroll
      for (int j = 0; j < 8; j += W) {
        tw w = {};
        if (j < left) w = *reinterpret_cast<const tw*>(src + j);
#pragma unroll
        for (int i = 0; i < W; ++i) v[j + i] = w[i];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = j < left ? src[j] : (T)0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      __bf16 p[NP];
      if constexpr (NP == 1) p[0] = v[j];
      else split_bf16<NP>((float)v[j], p);
#pragma unroll
      for (int i = 0; i < NP; ++i) part[i][j] = p[i];
    }
  }
}

// A workgroup has a row tile of the parameter and 16 MT rows of x; its waves take the fragments in turn and join in LDS.
template <int XT, int GROUP, int MT>
__global__ __launch_bounds__(512) void k_w4_product(const W4Params p) {
  using T = typename XElem<XT>::T;
  constexpr int NP = kXParts<XT>, GF = kKT / GROUP, SG = GROUP / 32;      // groups of a fragment, steps of a group
  extern __shared__ float lds[];                 // [waves][MT 16][17]
  const unsigned lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  const unsigned tile = blockIdx.x, m0 = blockIdx.y * 16 * MT, col = lane % 16, grp = lane / 16;
  const W4Dims d(p.N, p.K, GROUP);
  const uint8_t* frag = p.packed + (size_t)tile * d.frags * 1024 + lane * 16;
  const uint32_t* scales = reinterpret_cast<const uint32_t*>(p.packed + d.scales_at()) + (size_t)tile * d.groups * kNT + 4 * grp;
  const T* row[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) row[t] = static_cast<const T*>(p.x) + (size_t)min(m0 + 16 * t + col, p.M - 1) * p.ldx;
  const u4 one = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
  const bf8 ones = __builtin_bit_cast(bf8, one);
  float y[MT][4] = {};
  for (unsigned f = wave; f < p.frags; f += waves) {
    const u4 w = *reinterpret_cast<const u4*>(frag + (size_t)f * 1024);
    u4 sc[GF];
#pragma unroll
    for (int g = 0; g < GF; ++g) sc[g] = *reinterpret_cast<const u4*>(scales + ((size_t)f * GF + g) * kNT);
#pragma unroll
    for (int g = 0; g < GF; ++g) {
      v4f acc[MT] = {}, sum[MT] = {};
#pragma unroll
      for (int i = 0; i < SG; ++i) {
        const int step = g * SG + i, k = (int)(f * kKT + step * 32 + 8 * grp), left = (int)p.K - k;
        const bf8 a = codes16(w[step]);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          bf8 x[NP];
          x_parts<XT, NP>(row[t] + k, left, p.vec, x);
#pragma unroll
          for (int j = NP - 1; j >= 0; --j) {
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, x[j], acc[t], 0, 0, 0);
            sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, x[j], sum[t], 0, 0, 0);
          }
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float s = __uint_as_float(sc[g][r] & kTopScale), z = (float)(16u + (sc[g][r] & 15u));
#pragma unroll
        for (int t = 0; t < MT; ++t) y[t][r] = fmaf(s, fmaf(-z, sum[t][r], acc[t][r]), y[t][r]);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) lds[(wave * MT * 16 + t * 16 + col) * 17 + 4 * grp + r] = y[t][r];
  __syncthreads();
  for (unsigned i = threadIdx.x; i < MT * 256; i += blockDim.x) {
    const unsigned m = m0 + i / 16, n = tile * kNT + i % 16;
    float v = 0.f;
    for (unsigned w = 0; w < waves; ++w) v += lds[(w * MT * 16 + i / 16) * 17 + i % 16];
    if (m >= p.M || n >= p.N) continue;
    if (XT == MQ_ROWS8) v = __fdiv_rn(v, p.row_scale[m]);
    store_as(p.y, p.ytype, (size_t)m * p.ldy + n, p.bias != nullptr ? v + p.bias[n] : v);
  }
}

unsigned fill_wgs(size_t items) {
  const size_t n = (items + 255) / 256;
  return (unsigned)(n < 65536 ? n : 65536);
}

}  // namespace

size_t w4_bytes(size_t N, size_t K, int group) { return W4Dims(N, K, group).bytes(); }

int launch_w4_pack(const uint8_t* codes, const float* scales, const uint8_t* zeros, size_t N, size_t K, int group, void* packed,
                   hipStream_t s) {
  hipLaunchKernelGGL(k_w4_pack, dim3(fill_wgs(W4Dims(N, K, group).bytes() / 4)), dim3(256), 0, s, codes, scales, zeros, N, K, group,
                     packed);
  return check_hip(hipGetLastError());
}
int launch_w4_prepare(const float* w, size_t N, size_t K, int group, void* packed, hipStream_t s) {
  const size_t tiles = W4Dims(N, K, group).tiles;
  hipLaunchKernelGGL(k_w4_prepare, dim3((unsigned)(tiles < 65536 ? tiles : 65536)), dim3(256), 0, s, w, N, K, group, packed);
  return check_hip(hipGetLastError());
}
int launch_w4_unpack(const void* packed, size_t N, size_t K, int group, float* w, hipStream_t s) {
  hipLaunchKernelGGL(k_w4_unpack, dim3(fill_wgs(N * K)), dim3(256), 0, s, packed, N, K, group, w);
  return check_hip(hipGetLastError());
}

size_t w4_product_ws_bytes(size_t, size_t, size_t) { return 16; }

int launch_w4_product(const void* x, size_t ldx, int xtype, const float* row_scale, const void* packed, size_t M, size_t N,
                      size_t K, int group, const float* bias, void* y, size_t ldy, int ytype, void*, hipStream_t s) {
  const W4Dims d(N, K, group);
  const size_t es = xtype == MQ_ROWS8 ? 1 : elem_bytes(xtype), piece = es == 1 ? 8 : 16 / es;
  const W4Params p{x, row_scale, bias, static_cast<const uint8_t*>(packed), y, nullptr, ldx, ldy, (unsigned)M, (unsigned)N,
                   (unsigned)K, (unsigned)d.frags, ytype,
                   K % piece == 0 && ldx % piece == 0 && reinterpret_cast<uintptr_t>(x) % (piece * es) == 0};
  const unsigned waves = d.frags < 8 ? (unsigned)d.frags : 8u;
  auto go = [&](auto xt, auto gr) {
    auto sized = [&](auto mt) {
      constexpr int MT = decltype(mt)::value;
      const size_t chunks = (M + 16 * MT - 1) / (16 * MT);
      if (!launchable(d.tiles * chunks, waves * kWave) || chunks > 65535) return (int)MQ_ERR_SHAPE;
      hipLaunchKernelGGL((k_w4_product<decltype(xt)::value, decltype(gr)::value, MT>), dim3((unsigned)d.tiles, (unsigned)chunks),
                         dim3(waves * kWave), waves * MT * 16 * 17 * sizeof(float), s, p);
      return check_hip(hipGetLastError());
    };
    if (M <= 16) return sized(std::integral_constant<int, 1>{});
    if (M <= 32) return sized(std::integral_constant<int, 2>{});
    return sized(std::integral_constant<int, 4>{});
  };
  auto grouped = [&](auto xt) {
    if (group == 32) return go(xt, std::integral_constant<int, 32>{});
    if (group == 64) return go(xt, std::integral_constant<int, 64>{});
    return go(xt, std::integral_constant<int, 128>{});
  };
  if (xtype == MQ_ROWS8) return grouped(std::integral_constant<int, MQ_ROWS8>{});
  return with_dtype(xtype, grouped);
}

}  // namespace mq
