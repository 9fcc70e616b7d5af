// Parameters in 4 bits and products of a few rows with them (include/mq_serve.h): y = x w^T, w = (c - z) s.
//
// Packed: fragments of 16 rows x 128 elements, 1 KB, lane l of a wave 16 bytes: word w has the codes of row l % 16, elements
// 32 w + 8 (l / 16) .., what lane l feeds to v_mfma_f32_16x16x32_bf16 as operand b (x is a, so
// that a lane has results of one row of the parameter, and needs one scale).  Code 2 p lies in nibble p of the word's
// lower half, code 2 p + 1 in nibble p of the upper, so a pair shifted and masked once is two bfloat16 mantissas: 16 + c, exactly.
// y = sum_g s (sum_k (16 + c) x - (16 + z) sum_k x): a product with ones gives sum_k x where the other product leaves its results.
// That difference is off by roundings of up to 31 sum |x|.  Of binary32 rows they would show (one element, its zero next to its code: 16
// times the rounding of the result), so there c - z is formed in bytes and y = sum_g s sum_k (c - z) x.
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

// What a product takes of x and of codes.  8-bit rows: signed bytes and the codes as bytes, sums whole numbers (below 2^24, so
// exact in binary32).  Others: bfloat16 parts and 16 + c, of binary32 c - z, sums binary32.
template <int XT>
struct Operand {
  static constexpr bool kBytes = XT == MQ_ROWS8, kNoZeros = XT == MQ_F32;       // (kNoZeros: nothing is left to take off)
  static constexpr int NP = kXParts<XT>, kOffset = kBytes ? 0 : 16;
  using Piece = typename std::conditional<kBytes, long, bf8>::type;
  using Acc = typename std::conditional<kBytes, v4i, v4f>::type;
  static __device__ __forceinline__ Acc mfma(Piece a, Piece b, Acc c) {
    if constexpr (kBytes) return __builtin_amdgcn_mfma_i32_16x16x32_i8(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  // scale: the word that holds the group's zero
  static __device__ __forceinline__ Piece codes(unsigned w, unsigned scale) {
    if constexpr (kBytes) {             // codes 0 4 1 5 2 6 3 7
      return __builtin_bit_cast(long, make_uint2(w & 0x0f0f0f0fu, w >> 4 & 0x0f0f0f0fu));
    } else if constexpr (kNoZeros) {
      const unsigned z = (scale & 15u) * 0x01010101u;
      auto less = [&](unsigned c) { return (((c & 0x0f0f0f0fu) | 0x80808080u) - z) ^ 0x80808080u; };         // (no byte borrows)
      const unsigned a = less(w), b = less(w >> 4);
      auto pair = [](float x, float y) { return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u); };
      const u4 v = {pair(f32_of_byte<0>(a), f32_of_byte<2>(a)), pair(f32_of_byte<0>(b), f32_of_byte<2>(b)),
                    pair(f32_of_byte<1>(a), f32_of_byte<3>(a)), pair(f32_of_byte<1>(b), f32_of_byte<3>(b))};
      return __builtin_bit_cast(bf8, v);
    } else {
      constexpr unsigned mask = 0x00780078u, top = 0x41804180u;
      const u4 v = {(w << 3 & mask) | top, (w >> 1 & mask) | top, (w >> 5 & mask) | top, (w >> 9 & mask) | top};
      return __builtin_bit_cast(bf8, v);
    }
  }
  static __device__ __forceinline__ Piece ones() {
    if constexpr (kBytes) return 0x0101010101010101l;
    else return __builtin_bit_cast(bf8, u4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
  }
};

__device__ __forceinline__ float scale_of(unsigned w) { return __uint_as_float(w & kTopScale); }
template <int XT>
__device__ __forceinline__ float offset_of(unsigned w) {
  return (float)(Operand<XT>::kOffset + (w & 15u));
}

// Elements k .. k + 7 of a row of x as they lie, zeros from K on.
template <int XT>
struct Raw {
  typename XElem<XT>::T v[8];
};
template <int XT>
__device__ __forceinline__ Raw<XT> raw8(const typename XElem<XT>::T* row, int k, int K) {
  Raw<XT> r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r.v[j] = k + j < K ? row[k + j] : (typename XElem<XT>::T)0;
  return r;
}
// Eight signed bytes in the order in which eight codes come out of a word.
__device__ __forceinline__ long in_code_order(uint2 b) {
  return __builtin_bit_cast(long, make_uint2(__builtin_amdgcn_perm(b.y, b.x, 0x05010400u), __builtin_amdgcn_perm(b.y, b.x, 0x07030602u)));
}
// The same as operand parts.
template <int XT>
__device__ __forceinline__ void x_parts(const Raw<XT>& r, typename Operand<XT>::Piece (&part)[Operand<XT>::NP]) {
  constexpr int NP = Operand<XT>::NP;
  if constexpr (XT == MQ_ROWS8) {
    part[0] = in_code_order(__builtin_bit_cast(uint2, r));
  } else if constexpr (NP == 1) {
    part[0] = __builtin_bit_cast(bf8, r);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      __bf16 p[NP];
      split_bf16<NP>((float)r.v[j], p);
#pragma unroll
      for (int i = 0; i < NP; ++i) part[i][j] = p[i];
    }
  }
}

// Steps of 32 elements of a group, after which its zero is taken off a sum and its scale put to it.
template <int GROUP>
constexpr int kEvery = GROUP / 32;

constexpr unsigned kFewWaves = 4;      // of a workgroup, at most

// Few rows, of whole 16-byte pieces.  A workgroup has 16 rows of the parameter and 16 MT rows of x; its waves take the
// fragments in turn, the next ones' loads ahead of this one's products, and join in LDS.  Bound by the start and the way to memory of
// one round of workgroups more than by bytes: 11000 x 4096, groups of 64, 24 rows of 8 bits 25 MB in 11.6 us (2.2 TB/s).  A lane of an
// operand has a row of x of its own; loaded like that, every lane would be an access to the nearest cache of its own (64 a load
// instead of 8 .. 16, which bound this form).  So x comes in lines, and each wave turns its lines, as operand parts, in a part of LDS;
// of rows that are not there nothing is turned.
// (Two workgroups to a compute unit: the compiler then keeps sums in vector registers, with no copies; 12.6 -> 11.8 us.)
template <int XT, int GROUP, int MT>
__global__ __launch_bounds__(kFewWaves * kWave, 2) void k_w4_few(const W4Params p) {
  using T = typename XElem<XT>::T;
  constexpr int NP = kXParts<XT>, GF = kKT / GROUP, SG = GROUP / 32;      // groups of a fragment, steps of a group
  constexpr int EVERY = kEvery<GROUP>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float* const lds = reinterpret_cast<float*>(smem);       // [waves][MT 16][17], afterwards
  const unsigned lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  const unsigned tile = blockIdx.x, col = lane % 16, grp = lane / 16;
  const W4Dims d(p.N, p.K, GROUP);
  const uint8_t* const frag = p.packed + tile * d.frags * 1024;
  const uint32_t* const scales = reinterpret_cast<const uint32_t*>(p.packed + d.scales_at()) + tile * d.groups * kNT;
  // a row's elements of a fragment are SLOTS pieces of 16 bytes, LINES rows to a load; of its parts PSLOTS pieces each, piece j of
  // row r at place j ^ (r & 7)
  constexpr unsigned SLOTS = 8 * sizeof(T), LINES = kWave / SLOTS, XI = 16 / LINES, PER = 16 / sizeof(T);
  constexpr unsigned PSLOTS = XT == MQ_ROWS8 ? 8 : 16;
  u4* const turn = reinterpret_cast<u4*>(smem) + (size_t)wave * MT * NP * 16 * PSLOTS;
  using Op = Operand<XT>;
  using Piece = typename Op::Piece;
  const Piece ones = Op::ones();
  float y[MT][4] = {};
  // codes and scales of AHEAD fragments are on their way: enough that memory is busy; x, out of the nearest cache, of the next
  constexpr int AHEAD = 4;
  u4 w[AHEAD];
  unsigned sc[AHEAD][GF];
  u4 x[MT][XI];
  auto load = [&](int at, unsigned f) __attribute__((always_inline)) {
    f = min(f, p.frags - 1);
    w[at] = *reinterpret_cast<const u4*>(frag + (size_t)f * 1024 + lane * 16);
#pragma unroll
    for (int g = 0; g < GF; ++g) sc[at][g] = (scales + ((size_t)f * GF + g) * kNT)[col];
  };
  auto load_x = [&](unsigned f) __attribute__((always_inline)) {
    f = min(f, p.frags - 1);
    const unsigned e = f * kKT + lane % SLOTS * PER;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (unsigned i = 0; i < XI; ++i) {
        const size_t m = min(16 * t + i * LINES + lane / SLOTS, p.M - 1);
        x[t][i] = *reinterpret_cast<const u4*>(static_cast<const T*>(p.x) + m * p.ldx + min(e, p.K - PER));
        if (e >= p.K) x[t][i] = u4{};
      }
  };
  auto turn_x = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (unsigned i = 0; i < XI; ++i) {
        if (16 * t + i * LINES >= p.M) continue;
        const unsigned r = i * LINES + lane / SLOTS, j = lane % SLOTS;
        if constexpr (NP == 1) {
          turn[(16 * t + r) * PSLOTS + (j ^ (r & 7))] = x[t][i];
        } else {
          typedef T tw __attribute__((ext_vector_type(PER)));
          typedef __bf16 bw __attribute__((ext_vector_type(PER)));
          const tw v = __builtin_bit_cast(tw, x[t][i]);
          bw part[NP];
#pragma unroll
          for (unsigned e = 0; e < PER; ++e) {
            __bf16 b[NP];
            split_bf16<NP>((float)v[e], b);
#pragma unroll
            for (int k = 0; k < NP; ++k) part[k][e] = b[k];
          }
#pragma unroll
          for (int k = 0; k < NP; ++k) {           // (binary32: half a place)
            u4* const to = turn + ((t * NP + k) * 16 + r) * PSLOTS + ((j * PER / 8) ^ (r & 7));
            reinterpret_cast<bw*>(to)[PER == 8 ? 0 : j % 2] = part[k];
          }
        }
      }
  };
  // part k of elements 32 step + 8 grp .. of row 16 t + col
  auto read_x = [&](int t, int k, int step) __attribute__((always_inline)) {
    const u4* const at = turn + ((t * NP + k) * 16 + col) * PSLOTS;
    if constexpr (XT == MQ_ROWS8) {
      const uint2 b = reinterpret_cast<const uint2*>(at + ((2 * step + grp / 2) ^ (col & 7)))[grp % 2];
      return in_code_order(b);
    } else {
      return __builtin_bit_cast(bf8, at[(4 * step + grp) ^ (col & 7)]);
    }
  };
  auto multiply = [&](int at) __attribute__((always_inline)) {
    typename Op::Acc acc[MT], sum[MT];
#pragma unroll
    for (int step = 0; step < 4; ++step) {
      const Piece c = Op::codes(w[at][step], sc[at][step / SG]);
#pragma unroll
      for (int t = 0; t < MT; ++t) {
#pragma unroll
        for (int j = NP - 1; j >= 0; --j) {
          const bool begins = step % EVERY == 0 && j == NP - 1;
          const Piece xp = read_x(t, j, step);
          acc[t] = Op::mfma(xp, c, begins ? typename Op::Acc{} : acc[t]);
          if constexpr (!Op::kNoZeros) sum[t] = Op::mfma(xp, ones, begins ? typename Op::Acc{} : sum[t]);
        }
      }
      if (step % EVERY != EVERY - 1) continue;
      const float s = scale_of(sc[at][step / SG]), z = offset_of<XT>(sc[at][step / SG]);
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          y[t][r] = fmaf(s, Op::kNoZeros ? (float)acc[t][r] : fmaf(-z, (float)sum[t][r], (float)acc[t][r]), y[t][r]);
    }
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) load(i, wave + i * waves);
  load_x(wave);
  for (unsigned f = wave; f < p.frags; f += AHEAD * waves)
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const unsigned now = f + i * waves;
      if (now >= p.frags) break;
      turn_x();                                  // (a wave's accesses to LDS are in order)
      load_x(now + waves);
      multiply(i);
      load(i, now + AHEAD * waves);
    }
  __syncthreads();
  constexpr int PITCH = 17;
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) lds[(wave * MT * 16 + t * 16 + 4 * grp + r) * PITCH + col] = y[t][r];
  __syncthreads();
  for (unsigned i = threadIdx.x; i < MT * 256; i += blockDim.x) {
    const unsigned mm = i / 16, nn = i % 16, m = mm, n = tile * kNT + nn;
    float v = 0.f;
    for (unsigned w = 0; w < waves; ++w) v += lds[(w * MT * 16 + mm) * PITCH + nn];
    if (m >= p.M || n >= p.N) continue;
    if (XT == MQ_ROWS8) v = __fdiv_rn(v, p.row_scale[m]);
    store_as(p.y, p.ytype, (size_t)m * p.ldy + n, p.bias != nullptr ? v + p.bias[n] : v);
  }
}

// Many rows.  150 rows of binary32, 2048 x 8000, groups of 32: 29 us, of which x 4.5, the product 20 and the join 4; the product is
// bound by vector instructions (codes less zeros, scales: 57 % of the clocks, matrix ones 34 %).  x comes as operand parts, and (but for
// binary32) sums of groups, from a launch of its own: each is used by every row tile of the parameter.  A workgroup has
// 16 NT x 16 MT results and a run of fragments, its waves take the run's fragments in turn and join in LDS, runs through the
// workspace.
// (of several parts of x only half as many rows fit the registers beside those of the next step)
constexpr int many_mt(int parts) { return parts == 1 ? 4 : 2; }
constexpr int kManyNT = 4, kManyWaves = 4;

// operand parts [row tile][fragment][step][part][lane], 16 bytes each (8 of 8-bit rows), then sums of kEvery steps [row tile][..][16 rows]
struct XDims {
  size_t tiles, frags;
  int parts;
  __host__ __device__ XDims(size_t M, size_t K, int np) : tiles((M + 15) / 16), frags((K + kKT - 1) / kKT), parts(np) {}
  __host__ __device__ size_t sums_at() const { return tiles * frags * 4 * parts * 1024; }
  __host__ __device__ size_t bytes() const { return sums_at() + tiles * frags * 4 * 16 * sizeof(float); }
};

// a wave for each row tile and fragment
template <int XT, int GROUP>
__global__ __launch_bounds__(256) void k_w4_x(const W4Params p, uint8_t* to) {
  using T = typename XElem<XT>::T;
  using Piece = typename Operand<XT>::Piece;
  constexpr int NP = kXParts<XT>, EVERY = kEvery<GROUP>;
  const XDims x(p.M, p.K, NP);
  const unsigned lane = threadIdx.x % kWave, col = lane % 16, grp = lane / 16;
  const size_t all = x.tiles * x.frags;
  for (size_t s = (size_t)blockIdx.x * 4 + threadIdx.x / kWave; s < all; s += (size_t)gridDim.x * 4) {
    const size_t m = s / x.frags * 16 + col;
    const T* row = static_cast<const T*>(p.x) + (m < p.M ? m : p.M - 1) * p.ldx;
    Raw<XT> r[4] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = (int)(s % x.frags * kKT + 32 * i + 8 * grp);
      if (p.vec && k + 8 <= (int)p.K) {              // (rows are whole 16-byte pieces)
        typedef T t8 __attribute__((ext_vector_type(8), aligned(sizeof(T) == 1 ? 8 : 16)));
        r[i] = __builtin_bit_cast(Raw<XT>, *reinterpret_cast<const t8*>(row + k));
      } else {
        r[i] = raw8<XT>(row, k, (int)p.K);
      }
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      Piece part[NP];
      x_parts<XT>(r[i], part);
      Piece* dst = reinterpret_cast<Piece*>(to) + (s * 4 + i) * NP * kWave + lane;
#pragma unroll
      for (int k = 0; k < NP; ++k) dst[k * kWave] = part[k];
      if (Operand<XT>::kNoZeros) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += (float)r[i].v[j];
      if (i % EVERY != EVERY - 1) continue;
      auto add = [](float a, float b) { return a + b; };
      sum = across16_f(across32_f(sum, add), add);
      if (grp == 0) reinterpret_cast<float*>(to + x.sums_at())[(s * (4 / EVERY) + i / EVERY) * 16 + col] = sum;
      sum = 0.f;
    }
  }
}

template <int XT, int GROUP>
__global__ __launch_bounds__(kManyWaves * kWave, 2) void k_w4_many(const W4Params p, const uint8_t* xs, unsigned ntiles, unsigned runs, unsigned run) {
  constexpr int NP = kXParts<XT>, GF = kKT / GROUP, SG = GROUP / 32, MT = many_mt(NP), NT = kManyNT, EVERY = kEvery<GROUP>;
  extern __shared__ float lds[];                 // [waves][MT 16][NT 16 + 1]
  const unsigned lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), col = lane % 16, grp = lane / 16;
  // neighbouring workgroups share rows of x: those of one XCD its parts
  // (all in one axis: the others have no more than 65535 workgroups)
  const unsigned m0 = blockIdx.x / (ntiles * runs) * MT, at = blockIdx.x % (ntiles * runs);
  const unsigned nt = at % ntiles, k0 = at / ntiles * run, k1 = min(k0 + run, p.frags);
  const W4Dims d(p.N, p.K, GROUP);
  const XDims xd(p.M, p.K, NP);
  const uint8_t* frag[NT];
  const uint32_t* scales[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const size_t t = min(nt * NT + n, (unsigned)d.tiles - 1);
    frag[n] = p.packed + t * d.frags * 1024;
    scales[n] = reinterpret_cast<const uint32_t*>(p.packed + d.scales_at()) + t * d.groups * kNT;
  }
  using Op = Operand<XT>;
  using Piece = typename Op::Piece;
  const Piece* xp[MT];
  const float* xsum[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const size_t tile = min(m0 + t, (unsigned)xd.tiles - 1);
    xp[t] = reinterpret_cast<const Piece*>(xs) + tile * xd.frags * 4 * NP * kWave;
    xsum[t] = reinterpret_cast<const float*>(xs + xd.sums_at()) + tile * xd.frags * (4 / EVERY) * 16;
  }
  float y[NT][MT][4] = {};
  // codes and scales of the next fragment and x of the next step are on their way
  u4 w[2][NT];
  unsigned sc[2][NT][GF];
  Piece x[2][MT][NP];
  auto load = [&](int at, unsigned f) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      w[at][n] = *reinterpret_cast<const u4*>(frag[n] + (size_t)f * 1024 + lane * 16);
#pragma unroll
      for (int g = 0; g < GF; ++g) sc[at][n][g] = (scales[n] + ((size_t)f * GF + g) * kNT)[col];
    }
  };
  auto load_x = [&](int at, unsigned f, int step) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int j = 0; j < NP; ++j) x[at][t][j] = (xp[t] + (((size_t)f * 4 + step) * NP + j) * kWave)[lane];
  };
  auto multiply = [&](int at, unsigned f, unsigned next) __attribute__((always_inline)) {
    typename Op::Acc acc[NT][MT];
    v4f sum[MT];
#pragma unroll
    for (int step = 0; step < 4; ++step) {
      load_x((step + 1) % 2, step < 3 ? f : next, (step + 1) % 4);
      // (the compiler would ask for them where they are used: 11000 x 4096, groups of 128, 64 rows 48 us instead of 31)
      if (Op::kNoZeros) __builtin_amdgcn_sched_barrier(0);
      if (!Op::kNoZeros && step % EVERY == 0)
#pragma unroll
        for (int t = 0; t < MT; ++t) sum[t] = reinterpret_cast<const v4f*>(xsum[t] + ((size_t)f * (4 / EVERY) + step / EVERY) * 16)[grp];
      Piece c[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) c[n] = Op::codes(w[at][n][step], sc[at][n][step / SG]);
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int j = NP - 1; j >= 0; --j)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            acc[n][t] = Op::mfma(x[step % 2][t][j], c[n], step % EVERY == 0 && j == NP - 1 ? typename Op::Acc{} : acc[n][t]);
      if (step % EVERY != EVERY - 1) continue;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float s = scale_of(sc[at][n][step / SG]), z = offset_of<XT>(sc[at][n][step / SG]);
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            y[n][t][r] = fmaf(s, Op::kNoZeros ? (float)acc[n][t][r] : fmaf(-z, sum[t][r], (float)acc[n][t][r]), y[n][t][r]);
      }
    }
  };
  unsigned f = k0 + wave;
  if (f < k1) {
    load(0, f);
    load_x(0, f, 0);
  }
  while (f < k1) {
    unsigned next = min(f + kManyWaves, k1 - 1);      // (past the run's end: something that is there)
    load(1, next);
    multiply(0, f, next);
    f += kManyWaves;
    if (f >= k1) break;
    next = min(f + kManyWaves, k1 - 1);
    load(0, next);
    multiply(1, f, next);
    f += kManyWaves;
  }
  constexpr int PITCH = NT * 16 + 1;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) lds[((wave * MT + t) * 16 + 4 * grp + r) * PITCH + n * 16 + col] = y[n][t][r];
  __syncthreads();
  for (unsigned i = threadIdx.x; i < MT * 16 * NT * 16; i += kManyWaves * kWave) {
    const unsigned mm = i / (NT * 16), nn = i % (NT * 16), m = m0 * 16 + mm, n = nt * NT * 16 + nn;
    if (m >= p.M || n >= p.N) continue;
    float v = 0.f;
    for (unsigned u = 0; u < kManyWaves; ++u) v += lds[(u * MT * 16 + mm) * PITCH + nn];
    if (runs > 1) {
      p.part[((size_t)(k0 / run) * p.M + m) * p.N + n] = v;
      continue;
    }
    if (XT == MQ_ROWS8) v = __fdiv_rn(v, p.row_scale[m]);
    store_as(p.y, p.ytype, (size_t)m * p.ldy + n, p.bias != nullptr ? v + p.bias[n] : v);
  }
}

// The runs of a contraction, in order.
__global__ __launch_bounds__(256) void k_w4_join(const W4Params p, unsigned runs) {
  const size_t all = (size_t)p.M * p.N;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (size_t)gridDim.x * 256) {
    const size_t m = i / p.N, n = i % p.N;
    float v = 0.f;
    for (unsigned s = 0; s < runs; ++s) v += p.part[s * all + i];
    if (p.row_scale != nullptr) v = __fdiv_rn(v, p.row_scale[m]);
    store_as(p.y, p.ytype, m * p.ldy + n, p.bias != nullptr ? v + p.bias[n] : v);
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

namespace {

// rows of x up to which the form for few rows is taken, if they are whole pieces (more parts fill LDS)
constexpr size_t few_rows(int parts) { return parts == 1 ? 32 : parts == 2 ? 16 : 8; }
struct ManyForm {
  unsigned ntiles, chunks, runs, run;
};
ManyForm many_form(size_t M, size_t N, size_t K, int parts) {
  const size_t rows = 16 * (size_t)many_mt(parts), nt = (N + 16 * kManyNT - 1) / (16 * kManyNT), mt = (M + rows - 1) / rows, frags = (K + kKT - 1) / kKT;
  size_t want = nt * mt < 512 ? 512 / (nt * mt) : 1;      // two workgroups to a compute unit
  const size_t most = (frags + kManyWaves - 1) / kManyWaves;
  if (want > most) want = most;
  if (want > 16) want = 16;
  const size_t run = (frags + want - 1) / want;
  return {(unsigned)nt, (unsigned)mt, (unsigned)((frags + run - 1) / run), (unsigned)run};
}

}  // namespace

size_t w4_product_ws_bytes(size_t M, size_t N, size_t K) {
  unsigned runs = 1;                   // (whatever the type)
  for (int parts = 1; parts <= 3; ++parts) {
    const unsigned n = many_form(M, N, K, parts).runs;
    runs = n > runs ? n : runs;
  }
  return round_up(XDims(M, K, 3).bytes(), 256) + (runs > 1 ? (size_t)runs * M * N * sizeof(float) : 0);
}

int launch_w4_product(const void* x, size_t ldx, int xtype, const float* row_scale, const void* packed, size_t M, size_t N,
                      size_t K, int group, const float* bias, void* y, size_t ldy, int ytype, void* ws, hipStream_t s) {
  const W4Dims d(N, K, group);
  const size_t es = xtype == MQ_ROWS8 ? 1 : elem_bytes(xtype), piece = 16 / es;
  uint8_t* xs = static_cast<uint8_t*>(ws);
  const W4Params p{x, row_scale, bias, static_cast<const uint8_t*>(packed), y,
                   reinterpret_cast<float*>(xs + round_up(XDims(M, K, 3).bytes(), 256)), ldx, ldy, (unsigned)M,
                   (unsigned)N, (unsigned)K, (unsigned)d.frags, ytype,
                   K % piece == 0 && ldx % piece == 0 && reinterpret_cast<uintptr_t>(x) % (piece * es) == 0};
  auto go = [&](auto xt, auto gr) {
    constexpr int XT = decltype(xt)::value, GROUP = decltype(gr)::value;
    if (M <= few_rows(kXParts<XT>) && p.vec) {
      auto sized = [&](auto mt) {
        constexpr int MT = decltype(mt)::value;
        constexpr size_t turned = XT == MQ_ROWS8 ? kKT : 2 * kKT * kXParts<XT>;         // bytes of a row in LDS
        const size_t waves = d.frags < kFewWaves ? d.frags : kFewWaves;
        if (!launchable(d.tiles, waves * kWave)) return (int)MQ_ERR_SHAPE;
        hipLaunchKernelGGL((k_w4_few<XT, GROUP, MT>), dim3((unsigned)d.tiles), dim3((unsigned)(waves * kWave)),
                           waves * MT * 16 * (turned > 68 ? turned : 68), s, p);
        return check_hip(hipGetLastError());
      };
      if constexpr (kXParts<XT> == 1) {
        if (M > 16) return sized(std::integral_constant<int, 2>{});
      }
      return sized(std::integral_constant<int, 1>{});
    }
    const ManyForm f = many_form(M, N, K, kXParts<XT>);
    const size_t wgs = (size_t)f.ntiles * f.runs * f.chunks;
    if (!launchable(wgs, kManyWaves * kWave)) return (int)MQ_ERR_SHAPE;
    const size_t waves = XDims(M, K, 1).tiles * d.frags;
    hipLaunchKernelGGL((k_w4_x<XT, GROUP>), dim3((unsigned)(waves < 16384 ? (waves + 3) / 4 : 4096)), dim3(256), 0, s, p, xs);
    constexpr size_t lds = kManyWaves * many_mt(kXParts<XT>) * 16 * (kManyNT * 16 + 1) * sizeof(float);
    auto kern = k_w4_many<XT, GROUP>;
    if (lds > 65536) {
      const int rc = check_hip(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
      if (rc != MQ_OK) return rc;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(kManyWaves * kWave), lds, s, p, xs, f.ntiles, f.runs, f.run);
    if (f.runs > 1) hipLaunchKernelGGL(k_w4_join, dim3((unsigned)(M * N < 1048576 ? (M * N + 255) / 256 : 4096)), dim3(256), 0, s, p, f.runs);
    return check_hip(hipGetLastError());
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
