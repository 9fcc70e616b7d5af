// Attention of packed sequences (include/mq_seq.h), one pass over the keys with the running maximum and sum of the softmax.
//
// A first kernel brings keys and values into the order in which the matrix instructions take them, in units of 32 keys of one
// kv head, every piece of 1 KB the operand of one v_mfma_f32_32x32x16 (lane l its 16 bytes at 16 l):
//   K: operand a of S^T = K Q^T: lane l key l % 32, 8 columns from 16 f + 8 (l / 32);
//   V: operand a of O^T = V^T P^T: lane l column 32 t + l % 32, the 8 keys 16 s + 8 (j / 4) + 4 (l / 32) + j % 4.
// That is the order in which S^T leaves the scores of query l % 32 in lane l, so the probabilities become operand b without
// leaving their lane.  Odd widths and lengths are padded with zeros here, strides and alignment are dealt with here, and what is
// not finite becomes zero and is noted (a bit for each key), so that it cannot reach queries that do not see it.
// The second kernel streams the units through LDS, two tiles of keys in turn where they fit, for 32 queries of one head per wave.
// 16-bit types are multiplied as they are.  Binary32 becomes three bfloat16 parts (8 + 8 + 8 bits: all of it, at any
// magnitude), and a product the six of part i with part j, i + j <= 2; what is left out is below 2^-24 of the factors' product.
#include <type_traits>

#include "mq_gemm_common.h"
#include "mq_glue.h"
#include "mq_seq_common.h"

namespace mq {

namespace {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

constexpr int kUnit = 32;                  // keys of a unit
constexpr int kQ = 32;                     // queries of a wave
constexpr int kW = 4;
constexpr int kLds = 160 * 1024;

// parts of an element, and what a part is
template <int DT>
constexpr int kParts = DT == MQ_F32 ? 3 : 1;
template <int DT>
using Part = std::conditional_t<DT == MQ_F16, _Float16, __bf16>;
template <int DT>
using Part8 = std::conditional_t<DT == MQ_F16, h8, b8>;

constexpr unsigned padded(unsigned d) { return (d + 31) / 32 * 32; }
// bytes of a unit: keys, then values
__host__ __device__ inline unsigned unit_bytes(unsigned d, int parts) { return 2 * kUnit * ((d + 31) / 32 * 32) * 2 * parts; }

struct PromptParams {
  const void *q, *k, *v;
  void* out;
  const int32_t *q_first, *k_first;
  uint8_t* units;                          // [slots][kv_heads][unit]
  unsigned* bad;                           // [slots][kv_heads]: keys that are not finite
  size_t ldq, ldk, ldv, ldo;
  unsigned B, Tq, Tk, heads, kv_heads, d, q_slots;
  int causal;
  float scale2;
};

// (the largest binary32 values would round to a bfloat16 infinity: they leave their last bits to the next part)
template <int DT, bool ANY = true>
__device__ __forceinline__ void split_parts(const float (&x)[8], Part8<DT> (&part)[kParts<DT>]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float rest = x[j];
    if constexpr (ANY && DT == MQ_F32) {
      const float most = fabsf(rest) <= 3.402823466e38f ? __uint_as_float(0x7F7F0000u) : INFINITY;
      part[0][j] = (Part<DT>)fminf(fmaxf(rest, -most), most);
      rest -= (float)part[0][j];
#pragma unroll
      for (int i = 1; i < kParts<DT>; ++i) {
        part[i][j] = (Part<DT>)rest;
        rest -= (float)part[i][j];
      }
      continue;
    }
#pragma unroll
    for (int i = 0; i < kParts<DT>; ++i) {
      part[i][j] = (Part<DT>)rest;
      rest -= (float)part[i][j];
    }
  }
}

// keys of sequence b start at unit first[b] / 32 + b: room for every sequence's last, partly filled one
template <int DT>
__global__ __launch_bounds__(256) void k_prompt_pack(const PromptParams p) {
  using T = typename Elem<DT>::T;
  constexpr int NP = kParts<DT>;
  __shared__ unsigned bad;
  const unsigned slot = blockIdx.x / p.kv_heads, h = blockIdx.x % p.kv_heads, tid = threadIdx.x, d = p.d;
  const int b = wave_search(p.B, slot, [&](unsigned i) { return first_at(p.k_first, i, p.Tk) / kUnit + i; });
  if (b < 0) return;
  const unsigned f0 = first_at(p.k_first, b, p.Tk), f1 = first_at(p.k_first, b + 1, p.Tk), n = f1 > f0 ? f1 - f0 : 0;
  const unsigned j0 = (slot - (f0 / kUnit + (unsigned)b)) * kUnit;
  if (j0 >= n) return;
  const unsigned keys = n - j0 < (unsigned)kUnit ? n - j0 : (unsigned)kUnit;
  if (tid == 0) bad = 0;
  __syncthreads();
  const T* k = static_cast<const T*>(p.k) + (size_t)(f0 + j0) * p.ldk + (size_t)h * d;
  const T* v = static_cast<const T*>(p.v) + (size_t)(f0 + j0) * p.ldv + (size_t)h * d;
  const unsigned dp = (d + 31) / 32 * 32;
  uint8_t* unit = p.units + ((size_t)slot * p.kv_heads + h) * unit_bytes(d, NP);
  auto value = [&](const T* row, unsigned key, unsigned i, size_t ld) -> float {
    if (key >= keys || i >= d) return 0.f;
    const float x = (float)row[key * ld + i];
    if (fabsf(x) <= 3.402823466e38f) return x;
    atomicOr(&bad, 1u << key);
    return 0.f;
  };
  auto put = [&](const float (&x)[8], uint8_t* to) {
    Part8<DT> part[NP];
    split_parts<DT>(x, part);
#pragma unroll
    for (int i = 0; i < NP; ++i) *reinterpret_cast<Part8<DT>*>(to + i * 1024) = part[i];
  };
  for (unsigned i = tid; i < dp / 16 * 64; i += 256) {
    const unsigned f = i / 64, lane = i % 64;
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = value(k, lane % 32, f * 16 + lane / 32 * 8 + j, p.ldk);
    put(x, unit + (size_t)f * NP * 1024 + lane * 16);
  }
  for (unsigned i = tid; i < dp / 16 * 64; i += 256) {
    const unsigned f = i / 64, lane = i % 64;                // f = 2 t + s
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = value(v, f % 2 * 16 + j / 4 * 8 + lane / 32 * 4 + j % 4, f / 2 * 32 + lane % 32, p.ldv);
    put(x, unit + (size_t)(dp / 16 + f) * NP * 1024 + lane * 16);
  }
  __syncthreads();
  if (tid == 0) p.bad[(size_t)slot * p.kv_heads + h] = bad;
}

__device__ __forceinline__ v16f mfma(b8 a, b8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ v16f mfma(h8 a, h8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
// a . b of the parts whose weights are above 2^-24
template <int NP, typename P8>
__device__ __forceinline__ v16f mfma_parts(const P8 (&a)[NP], const P8 (&b)[NP], v16f c) {
#pragma unroll
  for (int sum = NP - 1; sum >= 0; --sum)
#pragma unroll
    for (int i = 0; i <= sum; ++i) c = mfma(a[i], b[sum - i], c);
  return c;
}

// ND: 32-column pieces of a head.  NU: units of a tile.  BUF: tiles in LDS.
template <int DT, int ND, int NU, int BUF>
__global__ __launch_bounds__(kW * kWave) void k_prompt_attention(const PromptParams p) {
  using T = typename Elem<DT>::T;
  using P8 = Part8<DT>;
  constexpr int NP = kParts<DT>;
  constexpr unsigned UNIT = 2 * kUnit * 32 * ND * 2 * NP, TILE = NU * UNIT;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const unsigned lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const unsigned col = lane % 32, half = lane / 32, d = p.d;
  const unsigned per = p.heads / p.kv_heads;
  // one kv head's workgroups next to each other on an XCD, whose L2 then holds its units; the last queries, which see most, first
  const unsigned id = xcd_remap(blockIdx.x, gridDim.x);
  const unsigned kvh = id / (p.q_slots * per), in = id % (p.q_slots * per);
  const unsigned slot = p.q_slots - 1 - in / per, head = kvh * per + in % per;
  constexpr unsigned BM = kW * kQ;
  const int b = wave_search(p.B, slot, [&](unsigned i) { return first_at(p.q_first, i, p.Tq) / BM + i; });
  if (b < 0) return;
  const unsigned q0 = first_at(p.q_first, b, p.Tq), q1 = first_at(p.q_first, b + 1, p.Tq), nq = q1 > q0 ? q1 - q0 : 0;
  const unsigned k0 = first_at(p.k_first, b, p.Tk), k1 = first_at(p.k_first, b + 1, p.Tk), nk = k1 > k0 ? k1 - k0 : 0;
  const unsigned i0 = (slot - (q0 / BM + (unsigned)b)) * BM;
  if (i0 >= nq) return;
  const unsigned unit0 = __builtin_amdgcn_readfirstlane(k0 / kUnit + (unsigned)b);
  // keys [0, seen) are seen by query i
  auto seen_by = [&](unsigned i) -> unsigned {
    if (!p.causal) return nk;
    const long long s = (long long)i + 1 + (long long)nk - (long long)nq;
    return s < 0 ? 0u : s > (long long)nk ? nk : (unsigned)s;
  };
  const unsigned iw = i0 + wave * kQ, i = iw + col;
  const bool mine = i < nq;
  const unsigned seen = mine ? seen_by(i) : 0u;
  const unsigned last = nq - i0 < BM ? nq - 1 : i0 + BM - 1;
  const unsigned tiles = __builtin_amdgcn_readfirstlane((seen_by(last) + kUnit * NU - 1) / (kUnit * NU));
  const unsigned wave_last = iw < nq ? seen_by(nq - iw < (unsigned)kQ ? nq - 1 : iw + kQ - 1) : 0u;   // most keys of this wave
  const unsigned wave_least = iw + kQ <= nq ? seen_by(iw) : 0u;                                        // fewest

  P8 qf[2 * ND][NP];
  {
    const T* src = static_cast<const T*>(p.q) + (size_t)(q0 + (mine ? i : i0)) * p.ldq + (size_t)head * d;
#pragma unroll
    for (int f = 0; f < 2 * ND; ++f) {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const unsigned c = f * 16 + half * 8 + j;
        x[j] = mine && c < d ? (float)src[c] : 0.f;
      }
      split_parts<DT>(x, qf[f]);
    }
  }
  const unsigned units = (nk + kUnit - 1) / kUnit;          // that the sequence has
  const uint8_t* base = p.units + ((size_t)unit0 * p.kv_heads + kvh) * UNIT;
  const size_t pitch = (size_t)p.kv_heads * UNIT;
  auto fetch = [&](unsigned tile, unsigned buf) {
#pragma unroll
    for (unsigned u = 0; u < NU; ++u) {
      const unsigned n = tile * NU + u < units ? tile * NU + u : units - 1;      // past the end: the last one, masked
      const uint8_t* src = base + n * pitch + lane * 16;
      uint8_t* dst = smem + buf * TILE + u * UNIT;
#pragma unroll
      for (unsigned c = 0; c < UNIT / 1024 / kW; ++c) {
        const unsigned piece = c * kW + wave;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + piece * 1024),
                                         (__attribute__((address_space(3))) void*)(dst + piece * 1024), 16, 0, 0);
      }
    }
  };
  static_assert(UNIT % (1024 * kW) == 0, "pieces of a unit");

  v16f o[ND];
#pragma unroll
  for (int t = 0; t < ND; ++t) o[t] = v16f{};
  float top = -INFINITY, total = 0.f;
  bool poison = false;
  if (tiles > 0 && BUF == 2) fetch(0, 0);
  for (unsigned tile = 0; tile < tiles; ++tile) {
    const unsigned buf = BUF == 2 ? tile & 1 : 0;
    if (BUF == 1) {
      __syncthreads();                       // everybody is done with the tile before
      fetch(tile, 0);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);      // this wave's pieces are in LDS
    __syncthreads();
    if (BUF == 2 && tile + 1 < tiles) fetch(tile + 1, buf ^ 1);
    const unsigned j0 = tile * NU * kUnit;
    if (j0 >= wave_last) continue;
    const uint8_t* at = smem + buf * TILE + lane * 16;
    v16f s[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      s[u] = v16f{};
#pragma unroll
      for (int f = 0; f < 2 * ND; ++f) {
        P8 kf[NP];
#pragma unroll
        for (int n = 0; n < NP; ++n) kf[n] = *reinterpret_cast<const P8*>(at + u * UNIT + (f * NP + n) * 1024);
        s[u] = mfma_parts<NP>(kf, qf[f], s[u]);
      }
    }
    const bool whole = j0 + NU * kUnit <= wave_least;        // every query of the wave sees every key of the tile
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const unsigned j = j0 + u * kUnit + 8 * (r / 4) + 4 * half + r % 4;
        s[u][r] = whole || j < seen ? s[u][r] * p.scale2 : -INFINITY;
        m = fmaxf(m, s[u][r]);
      }
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const unsigned n = tile * NU + u;
      if (n < units) {
        const unsigned w = p.bad[(size_t)(unit0 + n) * p.kv_heads + kvh];
        const unsigned first = n * kUnit;
        if (w != 0 && seen > first) poison |= (seen - first >= 32 ? w : w & ((1u << (seen - first)) - 1)) != 0;
      }
    }
    m = fmaxf(top, across32_f(m, [](float a, float b) { return fmaxf(a, b); }));
    const float ref = m == -INFINITY ? 0.f : m, keep = __builtin_amdgcn_exp2f(top - ref);
    top = m;
    total *= keep;
#pragma unroll
    for (int t = 0; t < ND; ++t) o[t] *= keep;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int step = 0; step < 2; ++step) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          e[j] = __builtin_amdgcn_exp2f(s[u][8 * step + j] - ref);
          total += e[j];
        }
        P8 pf[NP];
        split_parts<DT, false>(e, pf);
#pragma unroll
        for (int t = 0; t < ND; ++t) {
          P8 vf[NP];
#pragma unroll
          for (int n = 0; n < NP; ++n)
            vf[n] = *reinterpret_cast<const P8*>(at + u * UNIT + ((2 * ND + 2 * t + step) * NP + n) * 1024);
          o[t] = mfma_parts<NP>(vf, pf, o[t]);
        }
      }
  }
  total = across32_f(total, [](float a, float b) { return a + b; });
  if (!mine) return;
  const float inv = poison ? NAN : total == 0.f ? 0.f : __fdiv_rn(1.f, total);
  T* dst = static_cast<T*>(p.out) + (size_t)(q0 + i) * p.ldo + (size_t)head * d;
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const unsigned c = 32 * t + 8 * (r / 4) + 4 * half + r % 4;
      if (c < d) dst[c] = (T)(o[t][r] * inv);
    }
}

}  // namespace

static size_t k_slots(size_t B, size_t Tk) { return Tk / kUnit + B; }

size_t prompt_attention_ws_bytes(int dtype, size_t B, size_t Tk, int kv_heads, size_t d) {
  const size_t n = k_slots(B, Tk) * (size_t)kv_heads;
  return n * unit_bytes((unsigned)d, dtype == MQ_F32 ? 3 : 1) + round_up(n * sizeof(unsigned), 256);
}

int launch_prompt_attention(const void* q, size_t ldq, const void* k, size_t ldk, const void* v, size_t ldv, int dtype,
                            const int32_t* q_first, const int32_t* k_first, size_t B, size_t Tq, size_t Tk, int heads,
                            int kv_heads, size_t d, int causal, float scale, void* out, size_t ldo, void* ws, hipStream_t s) {
  const size_t n = k_slots(B, Tk) * (size_t)kv_heads, q_slots = Tq / (kW * kQ) + B, wgs = q_slots * (size_t)heads;
  if (n >= (size_t)1 << 31 || wgs >= (size_t)1 << 31) return MQ_ERR_SHAPE;
  uint8_t* units = static_cast<uint8_t*>(ws);
  PromptParams p{q, k, v, out, q_first, k_first, units,
                 reinterpret_cast<unsigned*>(units + n * unit_bytes((unsigned)d, dtype == MQ_F32 ? 3 : 1)),
                 ldq, ldk, ldv, ldo, (unsigned)B, (unsigned)Tq, (unsigned)Tk, (unsigned)heads, (unsigned)kv_heads, (unsigned)d,
                 (unsigned)q_slots, causal, scale * 1.44269504088896340736f};
  return with_dtype(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    hipLaunchKernelGGL((k_prompt_pack<DT>), dim3((unsigned)n), dim3(256), 0, s, p);
    int rc = check_hip(hipGetLastError());
    if (rc != MQ_OK) return rc;
    auto go = [&](auto nd) {
      constexpr int ND = decltype(nd)::value;
      // two units to a tile and two tiles in LDS where they fit, else one of both
      constexpr unsigned UNIT = 2 * kUnit * 32 * ND * 2 * kParts<DT>;
      constexpr int NU = 4 * UNIT <= kLds ? 2 : 1, BUF = 2 * NU * UNIT <= kLds ? 2 : 1;
      auto kern = k_prompt_attention<DT, ND, NU, BUF>;
      constexpr unsigned lds = NU * BUF * UNIT;
      if (lds > 65536) {
        const int e = check_hip(hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                    hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        if (e != MQ_OK) return e;
      }
      hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(kW * kWave), lds, s, p);
      return check_hip(hipGetLastError());
    };
    switch (padded((unsigned)d) / 32) {
      case 1: return go(std::integral_constant<int, 1>{});
      case 2: return go(std::integral_constant<int, 2>{});
      case 3: return go(std::integral_constant<int, 3>{});
      case 4: return go(std::integral_constant<int, 4>{});
      case 5: return go(std::integral_constant<int, 5>{});
      case 6: return go(std::integral_constant<int, 6>{});
      case 7: return go(std::integral_constant<int, 7>{});
      default: return go(std::integral_constant<int, 8>{});
    }
  });
}

}  // namespace mq
