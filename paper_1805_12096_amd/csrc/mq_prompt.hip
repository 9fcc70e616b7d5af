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
// 16-bit types are multiplied as they are, and probabilities are rounded to the type, because the matrix instructions take both
// operands of one type and two parts of each probability would double the second product.  3 sequences of
// 4500 .. 8190 in bfloat16 are 2.0e-3 off the result in 64 bits, with binary32 probabilities 1.5e-3 (the result's own rounding).
// Binary32 becomes three bfloat16 parts (8 + 8 + 8 bits: all of it, from 2^-100 up, where the third is above bfloat16's
// subnormals), and a product the six of part i with part j, i + j <= 2; what is left out is below 2^-24 of the factors' product.
// (Six bfloat16 products take 0.75 of the time of one on the binary32 matrix instruction, 1236 / 6 against 154 TFLOP/s, and
// leave it its lanes' layout.)
// Bound by matrix and vector instructions, which overlap in part only: 10 documents of 333 .. 1900 tokens, 16 heads of 64,
// binary32, causal, take 188 us, about 40 of them the first kernel (43 us with an attention of no queries behind it); while the
// second's compute units are busy, 40 % of the clocks have a matrix instruction and 40 % a vector one, and a wave waits a third
// of its time.
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
  uint8_t* units;                          // [kv_heads][k_slots][unit]
  unsigned* bad;                           // [kv_heads][k_slots]: keys that are not finite
  size_t ldq, ldk, ldv, ldo;
  unsigned B, Tq, Tk, heads, kv_heads, d, q_slots, k_slots;
  int causal;
  int negative;                            // scale2 is the scale's magnitude
  int vec;                                 // every row and head starts on 16 bytes
  float scale2;
};

// Binary32: the first part is the upper half of the word (no rounding, which could carry the largest values to infinity), the
// second the rest rounded, the third what is left, 8 bits at most.  NaN and infinities end up as NaN in the second.
template <int DT>
__device__ __forceinline__ void split_parts(const float (&x)[8], Part8<DT> (&part)[kParts<DT>]) {
  if constexpr (DT == MQ_F32) {
    u4 w;
    float r[8], r2[8];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = __builtin_amdgcn_perm(__float_as_uint(x[2 * j + 1]), __float_as_uint(x[2 * j]), 0x07060302u);
    part[0] = __builtin_bit_cast(b8, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = x[j] - __uint_as_float(__float_as_uint(x[j]) & 0xFFFF0000u);
#pragma unroll
    for (int j = 0; j < 8; ++j) part[1][j] = (__bf16)r[j];
    w = __builtin_bit_cast(u4, part[1]);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      r2[j] = r[j] - __uint_as_float(j % 2 == 0 ? w[j / 2] << 16 : w[j / 2] & 0xFFFF0000u);
#pragma unroll
    for (int j = 0; j < 8; ++j) part[2][j] = (__bf16)r2[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) part[0][j] = (Part<DT>)x[j];
  }
}

// 8 neighbouring columns from c on of a row, zeros past d.  Loads in front of every choice: a load behind a condition is waited
// for on its own.  vec: rows are whole 16-byte pieces.
template <int DT>
__device__ __forceinline__ void row8(const typename Elem<DT>::T* row, unsigned c, unsigned d, bool vec, float (&x)[8]) {
  using T = typename Elem<DT>::T;
  if (vec) {
    constexpr int W = 16 / sizeof(T);
    typedef T tw __attribute__((ext_vector_type(W)));
#pragma unroll
    for (int i = 0; i < 8; i += W) {
      const tw v = *reinterpret_cast<const tw*>(row + (c < d ? c + i : 0));
#pragma unroll
      for (int j = 0; j < W; ++j) x[i + j] = (float)v[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)row[c + j < d ? c + j : 0];
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = c + j < d ? x[j] : 0.f;
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
  uint8_t* unit = p.units + ((size_t)h * p.k_slots + slot) * unit_bytes(d, NP);
  auto put = [&](float (&x)[8], auto key_of, uint8_t* to) {
    float check = 0.f;                       // NaN as soon as one of them is not finite
#pragma unroll
    for (int j = 0; j < 8; ++j) check = fmaf(x[j], 0.f, check);
    if (__builtin_expect(check != check, 0))
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (!(fabsf(x[j]) <= 3.402823466e38f)) {
          atomicOr(&bad, 1u << key_of(j));
          x[j] = 0.f;
        }
    Part8<DT> part[NP];
    split_parts<DT>(x, part);
#pragma unroll
    for (int i = 0; i < NP; ++i) *reinterpret_cast<Part8<DT>*>(to + i * 1024) = part[i];
  };
  // (keys past the end repeat the last one: masked where they are used)
  for (unsigned i = tid; i < dp / 16 * 64; i += 256) {
    const unsigned f = i / 64, lane = i % 64, key = min(lane % 32, keys - 1);
    float x[8];
    row8<DT>(k + (size_t)key * p.ldk, f * 16 + lane / 32 * 8, d, p.vec, x);
    put(x, [&](int) { return key; }, unit + (size_t)f * NP * 1024 + lane * 16);
  }
  for (unsigned i = tid; i < dp / 16 * 64; i += 256) {
    const unsigned f = i / 64, lane = i % 64, c = f / 2 * 32 + lane % 32;                // f = 2 t + s
    auto key_of = [&](int j) { return min(f % 2 * 16 + j / 4 * 8 + lane / 32 * 4 + j % 4, keys - 1); };
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)v[key_of(j) * p.ldv + (c < d ? c : 0)];
    put(x, key_of, unit + (size_t)(dp / 16 + f) * NP * 1024 + lane * 16);
  }
  __syncthreads();
  if (tid == 0) p.bad[(size_t)h * p.k_slots + slot] = bad;
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

// Keys [0, this) are seen by query i of a sequence.
__device__ __forceinline__ unsigned keys_seen(const PromptParams& p, unsigned i, unsigned nq, unsigned nk) {
  if (!p.causal) return nk;
  const long long s = (long long)i + 1 + (long long)nk - (long long)nq;
  return s < 0 ? 0u : s > (long long)nk ? nk : (unsigned)s;
}

// Slot of queries and head of a workgroup: the last queries of a sequence, which see most, first, and neighbouring heads, which
// share keys and values, on one XCD (exactly where the heads are a multiple of eight), whose L2 then holds their units.
__device__ __forceinline__ void which(const PromptParams& p, unsigned& slot, unsigned& head) {
  slot = p.q_slots - 1 - blockIdx.x / p.heads;
  head = xcd_remap(blockIdx.x % p.heads, p.heads);
}

// What a query's sums are multiplied by.  Where keys are seen but nothing was summed, all scores were minus infinity (an infinite
// element of the query): there is no softmax, and the row is NaN, as with any other infinite score.
__device__ __forceinline__ float inverse_of(float total, bool poison, unsigned seen) {
  if (total == 0.f) return poison || seen > 0 ? NAN : 0.f;
  return poison ? NAN : __fdiv_rn(1.f, total);
}

// Four neighbouring columns of an output row, times inv.  vec: rows are whole 16-byte pieces.
template <int DT>
__device__ __forceinline__ void store4(typename Elem<DT>::T* row, float a, float b, float c, float e, float inv, unsigned at,
                                       unsigned d, bool vec) {
  using T = typename Elem<DT>::T;
  typedef T t4 __attribute__((ext_vector_type(4)));
  const t4 v = {(T)(a * inv), (T)(b * inv), (T)(c * inv), (T)(e * inv)};
  if (vec) {
    if (at < d) *reinterpret_cast<t4*>(row + at) = v;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (at + j < d) row[at + j] = v[j];
  }
}

// ND: 32-column pieces of a head.  NU: units of a tile.  BUF: tiles in LDS.  KS: groups of waves that take the tiles in turn and
// join at the end (a workgroup's way through a long sequence is what a call of few sequences waits for).
template <int DT, int ND, int NU, int BUF, int KS>
__global__ __launch_bounds__(KS * kW * kWave) void k_prompt_attention(const PromptParams p) {
  using T = typename Elem<DT>::T;
  using P8 = Part8<DT>;
  constexpr int NP = kParts<DT>;
  constexpr unsigned UNIT = 2 * kUnit * 32 * ND * 2 * NP, TILE = NU * UNIT;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const unsigned lane = threadIdx.x % kWave, any_wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const unsigned wave = any_wave % kW, group = any_wave / kW;
  const unsigned col = lane % 32, half = lane / 32, d = p.d;
  const unsigned per = p.heads / p.kv_heads;
  unsigned slot, head;
  which(p, slot, head);
  const unsigned kvh = head / per;
  constexpr unsigned BM = kW * kQ;
  const int b = wave_search(p.B, slot, [&](unsigned i) { return first_at(p.q_first, i, p.Tq) / BM + i; });
  if (b < 0) return;
  const unsigned q0 = first_at(p.q_first, b, p.Tq), q1 = first_at(p.q_first, b + 1, p.Tq), nq = q1 > q0 ? q1 - q0 : 0;
  const unsigned k0 = first_at(p.k_first, b, p.Tk), k1 = first_at(p.k_first, b + 1, p.Tk), nk = k1 > k0 ? k1 - k0 : 0;
  const unsigned i0 = (slot - (q0 / BM + (unsigned)b)) * BM;
  if (i0 >= nq) return;
  const unsigned unit0 = __builtin_amdgcn_readfirstlane(k0 / kUnit + (unsigned)b);
  auto seen_by = [&](unsigned i) { return keys_seen(p, i, nq, nk); };
  const unsigned iw = i0 + wave * kQ, i = iw + col;
  const bool mine = i < nq;
  const unsigned seen = mine ? seen_by(i) : 0u;
  const unsigned last = nq - i0 < BM ? nq - 1 : i0 + BM - 1;
  const unsigned tiles = __builtin_amdgcn_readfirstlane((seen_by(last) + kUnit * NU - 1) / (kUnit * NU));
  const unsigned wave_last = iw < nq ? seen_by(nq - iw < (unsigned)kQ ? nq - 1 : iw + kQ - 1) : 0u;   // most keys of this wave
  const unsigned wave_least = iw + kQ <= nq ? seen_by(iw) : 0u;                                        // fewest

  const unsigned units = (nk + kUnit - 1) / kUnit;          // that the sequence has
  const uint8_t* base = p.units + ((size_t)kvh * p.k_slots + unit0) * UNIT;
  auto fetch = [&](unsigned tile, unsigned buf) {
#pragma unroll
    for (unsigned u = 0; u < NU; ++u) {
      const unsigned n = tile * NU + u < units ? tile * NU + u : units - 1;      // past the end: the last one, masked
      const uint8_t* src = base + (size_t)n * UNIT + lane * 16;
      uint8_t* dst = smem + (buf * KS + group) * TILE + u * UNIT;
#pragma unroll
      for (unsigned c = 0; c < UNIT / 1024 / kW; ++c) {
        const unsigned piece = c * kW + wave;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + piece * 1024),
                                         (__attribute__((address_space(3))) void*)(dst + piece * 1024), 16, 0, 0);
      }
    }
  };
  static_assert(UNIT % (1024 * kW) == 0, "pieces of a unit");

  if (tiles > 0 && BUF == 2) fetch(group, 0);              // (on its way while the queries come)
  P8 qf[2 * ND][NP];
  {
    const T* src = static_cast<const T*>(p.q) + (size_t)(q0 + (mine ? i : i0)) * p.ldq + (size_t)head * d;
#pragma unroll
    for (int f = 0; f < 2 * ND; ++f) {
      float x[8];
      row8<DT>(src, f * 16 + half * 8, d, p.vec, x);
      split_parts<DT>(x, qf[f]);
    }
  }
  v16f o[ND];
#pragma unroll
  for (int t = 0; t < ND; ++t) o[t] = v16f{};
  float top = -INFINITY, total = 0.f;
  bool poison = false;
  // (looked at in front of the loop: in it, this load would be waited for behind the next tile's)
  unsigned any = 0;
  for (unsigned n = lane; n < units; n += kWave) any |= p.bad[(size_t)kvh * p.k_slots + unit0 + n];
  const bool some_bad = __any(any != 0);
  const unsigned steps = (tiles + KS - 1) / KS;            // (past the end: keys that nobody sees)
  for (unsigned step = 0; step < steps; ++step) {
    const unsigned buf = BUF == 2 ? step & 1 : 0, tile = step * KS + group;
    if (BUF == 1) {
      __syncthreads();                       // everybody is done with the tile before
      fetch(tile, 0);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);      // this wave's pieces are in LDS
    __syncthreads();
    if (BUF == 2 && step + 1 < steps) fetch(tile + KS, buf ^ 1);
    const unsigned j0 = tile * NU * kUnit;
    if (j0 >= wave_last) continue;
    const uint8_t* at = smem + (buf * KS + group) * TILE + lane * 16;
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
    if (__builtin_expect(some_bad, 0))
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const unsigned n = tile * NU + u;
      if (n < units) {
        const unsigned w = p.bad[(size_t)kvh * p.k_slots + unit0 + n];
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
      for (int part = 0; part < 2; ++part) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          e[j] = __builtin_amdgcn_exp2f(s[u][8 * part + j] - ref);
          total += e[j];
        }
        P8 pf[NP];
        split_parts<DT>(e, pf);
#pragma unroll
        for (int t = 0; t < ND; ++t) {
          P8 vf[NP];
#pragma unroll
          for (int n = 0; n < NP; ++n)
            vf[n] = *reinterpret_cast<const P8*>(at + u * UNIT + ((2 * ND + 2 * t + part) * NP + n) * 1024);
          o[t] = mfma_parts<NP>(vf, pf, o[t]);
        }
      }
  }
  if constexpr (KS == 2) {
    // the second group's sums to the first, wave by wave; a lane's piece next to its neighbours'
    constexpr int ROWS = 16 * ND + 3;
    static_assert(kW * ROWS * kWave * 4 <= KS * BUF * TILE, "the sums of a group");
    float* box = reinterpret_cast<float*>(smem) + wave * ROWS * kWave + lane;
    __syncthreads();
    if (group == 1) {
#pragma unroll
      for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) box[(16 * t + r) * kWave] = o[t][r];
      box[16 * ND * kWave] = top;
      box[(16 * ND + 1) * kWave] = total;
      box[(16 * ND + 2) * kWave] = poison ? 1.f : 0.f;
    }
    __syncthreads();
    if (group == 1) return;
    const float other = box[16 * ND * kWave], m = fmaxf(top, other), ref = m == -INFINITY ? 0.f : m;
    const float a = __builtin_amdgcn_exp2f(top - ref), b = __builtin_amdgcn_exp2f(other - ref);
    total = total * a + box[(16 * ND + 1) * kWave] * b;
    poison |= box[(16 * ND + 2) * kWave] != 0.f;
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] = o[t][r] * a + box[(16 * t + r) * kWave] * b;
  }
  total = across32_f(total, [](float a, float b) { return a + b; });
  if (!mine) return;
  const float inv = inverse_of(total, poison, seen);
  T* dst = static_cast<T*>(p.out) + (size_t)(q0 + i) * p.ldo + (size_t)head * d;
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      store4<DT>(dst, o[t][r], o[t][r + 1], o[t][r + 2], o[t][r + 3], inv, 32 * t + 2 * r + 4 * half, d, p.vec);
}

// ---- long sequences, 16-bit types ------------------------------------------------------------------------------------------
// With 32 queries per wave every piece of K or V that a wave takes from LDS feeds one matrix instruction, and the four SIMDs'
// 4 KB in 32 clocks are all that LDS gives; the softmax's vector instructions take as long as the matrix ones besides.  So
// here a wave has two tiles of 32 queries, which halves what it reads, alone on its SIMD with twice the registers, and works
// on three units at a time, so that nothing in a step waits for anything else in it:
//   S = K Q^T of unit n + 2 and O += V P of unit n (matrix)   beside   P = exp2(S - m) of unit n + 1 (vector),
// K and V pieces on their way from LDS a few instructions ahead.
// The reference m of a query's softmax moves only when a score exceeds it by more than kSlack, in powers of two (a branch that
// is hardly ever taken), so that O is hardly ever rescaled.  A ring of units in LDS, one barrier for two units.
// 3 sequences of 4500 .. 8190 bfloat16 tokens, 32 heads of 128 over 8, causal: 1.28 .. 1.32 ms with the packing kernel from card
// to card, 880 .. 910 TFLOP/s (the first form, one tile a wave, one step after the other: 1.86).  Matrix instructions take 43 % of
// the busy clocks, vector ones 44 %; a wave, alone on its SIMD, waits for a quarter of them.
#define MQ_INLINE __attribute__((always_inline))
constexpr int kRing = 8;
constexpr float kSlack = 8.f;

// One result of a matrix instruction, out of its accumulation register at this place.  (The compiler would copy all sixteen as
// soon as they are there, and wait for that.)  The compiler does not see what is read here, so whoever reads the first result
// lets the twelve wait states go by that an 8-pass instruction needs on gfx950: FIRST.  (It may belong to the product issued
// last: the compiler puts two tiles' last products in either order.  The other tile's first read is sixteen behind it.)
template <bool FIRST>
__device__ __forceinline__ float accumulated(float x) {
  float y;
  if constexpr (FIRST) asm volatile("s_nop 11\n\tv_accvgpr_read_b32 %0, %1" : "=v"(y) : "a"(x));
  else asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(y) : "a"(x));
  return y;
}
template <int DT>
__device__ __forceinline__ unsigned pack2(float a, float b) {
  typedef Part<DT> p2 __attribute__((ext_vector_type(2)));
  const p2 x = {(Part<DT>)a, (Part<DT>)b};
  unsigned w = __builtin_bit_cast(unsigned, x);
  asm("" : "+v"(w));                       // here, not where the last of eight is known
  return w;
}
// sum + both elements of w (as rounded: what is divided by then is the sum of what is multiplied)
template <int DT>
__device__ __forceinline__ float add2(unsigned w, float sum) {
  if constexpr (DT == MQ_F16) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const h2 one = {(_Float16)1.f, (_Float16)1.f};
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, w), one, sum, false);
  } else {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    const b2 one = {(__bf16)1.f, (__bf16)1.f};
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, w), one, sum, false);
  }
}
// Sums of matrix instructions times a factor, from accumulation registers and back.  (The compiler would otherwise take the
// copies that the vector unit needs out of the branch, into every step.)
__device__ __forceinline__ void scale_sums(v16f& o, float factor) {
  asm volatile("" : "+a"(o));
  o *= factor;
  asm volatile("" : "+a"(o));
}

template <int DT, int ND>
__global__ __launch_bounds__(kW * kWave, 1) void k_prompt_wide(const PromptParams p) {
  using T = typename Elem<DT>::T;
  using P8 = Part8<DT>;
  constexpr unsigned UNIT = 2 * kUnit * 32 * ND * 2, PW = UNIT / 1024 / kW, BM = 2 * kW * kQ;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const unsigned lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const unsigned col = lane % 32, half = lane / 32, d = p.d;
  const unsigned per = p.heads / p.kv_heads;
  unsigned slot, head;
  which(p, slot, head);
  const unsigned kvh = head / per;
  const int b = __builtin_amdgcn_readfirstlane(wave_search(p.B, slot, [&](unsigned i) { return first_at(p.q_first, i, p.Tq) / BM + i; }));
  if (b < 0) return;
  const unsigned q0 = first_at(p.q_first, b, p.Tq), q1 = first_at(p.q_first, b + 1, p.Tq), nq = q1 > q0 ? q1 - q0 : 0;
  const unsigned k0 = first_at(p.k_first, b, p.Tk), k1 = first_at(p.k_first, b + 1, p.Tk), nk = k1 > k0 ? k1 - k0 : 0;
  const unsigned i0 = (slot - (q0 / BM + (unsigned)b)) * BM;
  if (i0 >= nq) return;
  const unsigned unit0 = k0 / kUnit + (unsigned)b, units = (nk + kUnit - 1) / kUnit;
  auto seen_by = [&](unsigned i) { return keys_seen(p, i, nq, nk); };
  const unsigned iw = i0 + wave * 2 * kQ;
  const unsigned last = min(i0 + BM, nq) - 1, wave_last = min(iw + 2 * kQ, nq) - 1;
  const unsigned n_wg = __builtin_amdgcn_readfirstlane((seen_by(last) + kUnit - 1) / kUnit);
  const unsigned n_wave = iw < nq ? __builtin_amdgcn_readfirstlane((seen_by(wave_last) + kUnit - 1) / kUnit) : 0u;
  // units before this one are seen whole by every query of the workgroup
  const unsigned n_full = __builtin_amdgcn_readfirstlane(seen_by(i0) / kUnit);

  const uint8_t* base = p.units + ((size_t)kvh * p.k_slots + unit0) * UNIT + wave * 1024 + lane * 16;
  auto fetch = [&](unsigned n) {
    const uint8_t* src = base + (size_t)(n < units ? n : units - 1) * UNIT;       // past the end: the last one, masked
    uint8_t* dst = smem + n % kRing * UNIT + wave * 1024;
#pragma unroll
    for (unsigned c = 0; c < PW; ++c)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + c * (kW * 1024)),
                                       (__attribute__((address_space(3))) void*)(dst + c * (kW * 1024)), 16, 0, 0);
  };

  // (the first units are on their way while the queries come)
  if (n_wg > 0)
#pragma unroll
    for (unsigned n = 0; n + 2 < (unsigned)kRing; ++n) fetch(n);
  unsigned seen[2];
  P8 qf[2][2 * ND];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const unsigned i = iw + c * kQ + col;
    const bool mine = i < nq;
    seen[c] = mine ? seen_by(i) : 0u;
    const T* src = static_cast<const T*>(p.q) + (size_t)(q0 + (mine ? i : i0)) * p.ldq + (size_t)head * d;
#pragma unroll
    for (int f = 0; f < 2 * ND; ++f)
    {
      float x[8];
      row8<DT>(src, f * 16 + half * 8, d, p.vec, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) qf[c][f][j] = (Part<DT>)(p.negative ? -x[j] : x[j]);   // (the scale's sign: what is masked stays at minus infinity)
    }
  }
  v16f o[2][ND];
  float sa[2][16], sb[2][16], high_a[2], high_b[2];       // scores of two units, and the largest of a lane's 16
  u4 pa[2][2] = {}, pb[2][2] = {};                        // probabilities, eight of the type each
  float last_e[2];
  float top[2] = {-INFINITY, -INFINITY}, total[2] = {0.f, 0.f};
  bool poison[2] = {false, false};
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int t = 0; t < ND; ++t) o[c][t] = v16f{};

  // what has to be known before the exponentials of unit n: masks, and whether a reference moves.  `held`: probabilities whose
  // product with V is still to come
  auto settle = [&](auto masked, float (&s)[2][16], float (&high)[2], u4 (&held)[2][2], unsigned n) MQ_INLINE {
    float m[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      if constexpr (decltype(masked)::value) {
        high[c] = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          if (n * kUnit + 8 * (r / 4) + 4 * half + r % 4 >= seen[c]) s[c][r] = -INFINITY;
          high[c] = fmaxf(high[c], s[c][r]);
        }
      }
      m[c] = across32_f(high[c], [](float a, float b) { return fmaxf(a, b); }) * p.scale2;
    }
    if (__builtin_expect(__any(m[0] > top[0] + kSlack || m[1] > top[1] + kSlack), 0)) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        // (only for the queries concerned: no other query's result depends on theirs)
        const float now = m[c] > top[c] + kSlack ? m[c] : top[c], keep = now == top[c] ? 1.f : __builtin_amdgcn_exp2f(top[c] - now);
        top[c] = now;
        total[c] *= keep;
#pragma unroll
        for (int t = 0; t < ND; ++t) scale_sums(o[c][t], keep);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          P8 x = __builtin_bit_cast(P8, held[c][i]);
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = (Part<DT>)((float)x[j] * keep);
          held[c][i] = __builtin_bit_cast(u4, x);
        }
      }
    }
  };
  // exponentials [from, end) of the 32 that a lane has of a unit; two neighbours become a word of the operand
  auto exponentials = [&](const float (&s)[2][16], u4 (&to)[2][2], int from, int end) MQ_INLINE {
#pragma unroll
    for (int i = from; i < end; ++i) {
      const int c = i / 16, r = i % 16;
      last_e[i % 2] = __builtin_amdgcn_exp2f(fmaf(s[c][r], p.scale2, -(top[c] == -INFINITY ? 0.f : top[c])));
      if (i % 2 == 1) {
        const unsigned w = pack2<DT>(last_e[0], last_e[1]);
        to[c][r / 8][r % 8 / 2] = w;
        total[c] = add2<DT>(w, total[c]);
      }
    }
  };
  // scores [from, end) of the 32, out of the matrix instructions' registers
  auto take = [&](const v16f (&x)[2], float (&s)[2][16], float (&high)[2], int from, int end) MQ_INLINE {
#pragma unroll
    for (int i = from; i < end; ++i) {
      const int c = i / 16, r = i % 16;
      s[c][r] = i == 0 ? accumulated<true>(x[c][r]) : accumulated<false>(x[c][r]);
      if (r % 2 == 1) high[c] = r == 1 ? fmaxf(s[c][0], s[c][1]) : fmaxf(fmaxf(high[c], s[c][r - 1]), s[c][r]);
    }
  };
  auto scores = [&](unsigned n, float (&s)[2][16], float (&high)[2]) MQ_INLINE {
    const uint8_t* at = smem + n % kRing * UNIT + lane * 16;
    v16f x[2] = {};
#pragma unroll
    for (int f = 0; f < 2 * ND; ++f) {
      const P8 kf = *reinterpret_cast<const P8*>(at + f * 1024);
      x[0] = mfma(kf, qf[0][f], x[0]);
      x[1] = mfma(kf, qf[1][f], x[1]);
    }
    __builtin_amdgcn_sched_barrier(0);                     // (take counts on all of them being issued)
    take(x, s, high, 0, 32);
  };
  // step n, with the scores of unit n + 1 in s and its probabilities to go to `to`, unit n's in `held`, unit n + 2's scores to go
  // to `next`: 8 ND matrix instructions, each with its share of the vector ones behind it, in this order.  The exponentials lie
  // mostly beside K's half, the way of the new scores beside V's.  V's pieces are asked for while K's are multiplied, those of
  // unit n + 3's K while V's are.  (Left to itself, the compiler waits for each as it asks.)
  P8 kf[2 * ND];
  auto step = [&](auto masked, unsigned n, float (&s)[2][16], float (&high)[2], float (&next)[2][16], float (&next_high)[2], u4 (&held)[2][2],
                  u4 (&to)[2][2]) MQ_INLINE {
    constexpr int N = 4 * ND, EARLY = 22;                  // exponentials of the first half
    const uint8_t *kat = smem + (n + 3) % kRing * UNIT + lane * 16, *vat = smem + n % kRing * UNIT + 2 * ND * 1024 + lane * 16;
    P8 vf[2 * ND];
    settle(masked, s, high, held, n + 1);
    v16f x[2] = {};
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) {
      const int c = i % 2, f = i / 2 % (2 * ND), t = f % ND, h = f / ND, j = i - N;
      if (i < 2 * ND) vf[i] = *reinterpret_cast<const P8*>(vat + (2 * (i % ND) + i / ND) * 1024);
      if (i >= N && i < N + 2 * ND) kf[j] = *reinterpret_cast<const P8*>(kat + j * 1024);
      if (i < N) {
        x[c] = mfma(kf[f], qf[c][f], x[c]);
        exponentials(s, to, i * EARLY / N, (i + 1) * EARLY / N);
      } else {
        o[c][t] = mfma(vf[f], __builtin_bit_cast(P8, held[c][h]), o[c][t]);
        exponentials(s, to, EARLY + j * (32 - EARLY) / N, EARLY + (j + 1) * (32 - EARLY) / N);
        if (j >= 2) take(x, next, next_high, (j - 2) * 32 / (N - 2), (j - 1) * 32 / (N - 2));
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // before steps n and n + 1: units up to n + 4 are there, and nobody reads units n - 2 and n - 1 any more
  auto arrive = [&](unsigned n) {
    constexpr unsigned ahead = (kRing - 7) * PW;
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (ahead & 15) | (ahead >> 4) << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    fetch(n + kRing - 2);
    fetch(n + kRing - 1);
  };
  // keys that are not finite, 64 units at a time
  auto look = [&](unsigned n) {
    const unsigned at = n + lane < units ? n + lane : units - 1;
    const unsigned w = p.bad[(size_t)kvh * p.k_slots + unit0 + at];
    unsigned long long some = __ballot(w != 0 && n + lane < units);
    while (some != 0) {
      const int l = __ffsll((long long)some) - 1;
      some &= some - 1;
      const unsigned bits = __builtin_amdgcn_readlane((int)w, l), from = (n + l) * kUnit;
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (seen[c] > from) poison[c] |= (seen[c] - from >= 32 ? bits : bits & ((1u << (seen[c] - from)) - 1)) != 0;
    }
  };

  if (n_wg > 0) {
    unsigned any = 0;
    for (unsigned n = lane; n < min(n_wg, units); n += kWave) any |= p.bad[(size_t)kvh * p.k_slots + unit0 + n];
    if (__builtin_expect(__any(any != 0), 0))
      for (unsigned n = 0; n < n_wg; n += kWave) look(n);
    __builtin_amdgcn_s_waitcnt(0x0F70);
    __syncthreads();
    scores(0, sa, high_a);
    scores(1, sb, high_b);
#pragma unroll
    for (int f = 0; f < 2 * ND; ++f) kf[f] = *reinterpret_cast<const P8*>(smem + 2 * UNIT + f * 1024 + lane * 16);
    settle(std::true_type{}, sa, high_a, pb, 0);
    exponentials(sa, pa, 0, 32);
    unsigned n = 0;
    auto two = [&](auto masked) MQ_INLINE {
      step(masked, n, sb, high_b, sa, high_a, pa, pb);
      step(masked, n + 1, sa, high_a, sb, high_b, pb, pa);
    };
    for (; n + 2 < n_full; n += 2) {
      arrive(n);
      two(std::false_type{});
    }
    for (; n < n_wg; n += 2) {
      arrive(n);
      if (n < n_wave) two(std::true_type{});     // (a wave whose queries see fewer units keeps the others company)
    }
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const unsigned i = iw + c * kQ + col;
    const float sum = across32_f(total[c], [](float a, float b) { return a + b; });
    if (i >= nq) continue;
    const float inv = inverse_of(sum, poison[c], seen[c]);
    T* dst = static_cast<T*>(p.out) + (size_t)(q0 + i) * p.ldo + (size_t)head * d;
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        store4<DT>(dst, o[c][t][r], o[c][t][r + 1], o[c][t][r + 2], o[c][t][r + 3], inv, 32 * t + 2 * r + 4 * half, d, p.vec);
  }
}

// ---- short sequences ---------------------------------------------------------------------------------------------------
// Sentences of a few dozen words: nothing is reused often enough to be worth an order of its own, and a second launch and a walk
// through LDS cost more than the product.  A wave takes 16 queries of one head and reads keys and values as they are; waves
// wait for nobody.  The tiles are 16 x 16 (sentences leave half of a 32 x 32 one empty), and binary32 runs on the binary32
// matrix instruction: splitting operands that are used once costs more vector instructions than it saves matrix ones.
// Lane l: query (or key) l % 16, place group g = l / 16.  An operand's 8 elements are, for a 16-bit type, the 8 neighbouring
// contracted places 8 g .. of 32, for binary32 two times four, 4 g .. of 16.
// 300 sentences of 2 .. 60 binary32 words, 8 heads of 64: 19 us, 9.6 of them bytes.  What bounds it is the longest sentences' chain
// of loads and products, and the load units (a key is read by every 16 queries of every head that it serves).  Operands are kept
// as binary32 also for 16-bit types: heads of more than 128 leave one wave a SIMD, and rows that are not whole 16-byte pieces
// spill at 97 .. 128 and above 192.
constexpr int kQShort = 16;

// The column that element j of a lane's n-th 8 stands for.
template <int DT>
__device__ __forceinline__ constexpr unsigned column_of(unsigned n, unsigned g, unsigned j) {
  return DT == MQ_F32 ? 32 * n + 16 * (j / 4) + 4 * g + j % 4 : 32 * n + 8 * g + j;
}

// A lane's 8 elements of the row at base + row as floats; columns past d repeat the row's first.  VEC: whole 16-byte pieces
template <int DT, bool VEC>
__device__ __forceinline__ void load8(const typename Elem<DT>::T* base, unsigned row, unsigned n, unsigned g, unsigned d, float (&x)[8]) {
  using T = typename Elem<DT>::T;
  if constexpr (VEC) {
    constexpr int W = DT == MQ_F32 ? 4 : 8;
    typedef T tw __attribute__((ext_vector_type(W)));
#pragma unroll
    for (int i = 0; i < 8; i += W) {
      const unsigned c = column_of<DT>(n, g, i);
      const tw v = *reinterpret_cast<const tw*>(base + (row + (c < d ? c : 0)));
#pragma unroll
      for (int j = 0; j < W; ++j) x[i + j] = (float)v[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const unsigned c = column_of<DT>(n, g, j);
      x[j] = (float)base[row + (c < d ? c : 0)];
    }
  }
}

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
// contracts 32 columns
template <int DT>
__device__ __forceinline__ v4f mfma_columns(const float (&a)[8], const float (&b)[8], v4f c) {
  if constexpr (DT == MQ_F32) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
  } else {
    Part8<DT> x, y;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = (Part<DT>)a[j];
      y[j] = (Part<DT>)b[j];
    }
    if constexpr (DT == MQ_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
  }
}
// contracts 16 keys, of which a lane holds 4 g .. 4 g + 3
template <int DT>
__device__ __forceinline__ v4f mfma_keys(const float (&a)[4], const float (&b)[4], v4f c) {
  if constexpr (DT == MQ_F32) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
  } else if constexpr (DT == MQ_F16) {
    const h4 x = {(_Float16)a[0], (_Float16)a[1], (_Float16)a[2], (_Float16)a[3]},
             y = {(_Float16)b[0], (_Float16)b[1], (_Float16)b[2], (_Float16)b[3]};
    return __builtin_amdgcn_mfma_f32_16x16x16f16(x, y, c, 0, 0, 0);
  } else {
    typedef short s4 __attribute__((ext_vector_type(4)));
    const b4 x = {(__bf16)a[0], (__bf16)a[1], (__bf16)a[2], (__bf16)a[3]},
             y = {(__bf16)b[0], (__bf16)b[1], (__bf16)b[2], (__bf16)b[3]};
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s4, x), __builtin_bit_cast(s4, y), c, 0, 0, 0);
  }
}

template <int DT, int ND, bool VEC>
__global__ __launch_bounds__(256, ND <= 2 ? 3 : ND <= 4 ? 2 : 1) void k_prompt_short(const PromptParams p) {
  using T = typename Elem<DT>::T;
  const unsigned lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const unsigned col = lane % 16, g = lane / 16, d = p.d;
  const unsigned id = xcd_remap(blockIdx.x, gridDim.x) * 4 + wave, slot = id / p.heads, head = id % p.heads;
  const unsigned kvh = head / (p.heads / p.kv_heads);
  const int b = __builtin_amdgcn_readfirstlane(
      slot < p.q_slots ? wave_search(p.B, slot, [&](unsigned i) { return first_at(p.q_first, i, p.Tq) / kQShort + i; }) : -1);
  if (b < 0) return;
  const unsigned q0 = first_at(p.q_first, b, p.Tq), q1 = first_at(p.q_first, b + 1, p.Tq), nq = q1 > q0 ? q1 - q0 : 0;
  const unsigned k0 = first_at(p.k_first, b, p.Tk), k1 = first_at(p.k_first, b + 1, p.Tk), nk = k1 > k0 ? k1 - k0 : 0;
  const unsigned i0 = (slot - (q0 / kQShort + (unsigned)b)) * kQShort, i = i0 + col;
  if (i0 >= nq) return;
  auto seen_by = [&](unsigned i) { return keys_seen(p, i, nq, nk); };
  const bool mine = i < nq;
  const unsigned seen = mine ? seen_by(i) : 0u;
  const unsigned most = __builtin_amdgcn_readfirstlane(seen_by(nq - i0 < (unsigned)kQShort ? nq - 1 : i0 + kQShort - 1));
  const T* src = static_cast<const T*>(p.q) + (size_t)(q0 + i0) * p.ldq + (size_t)head * d;
  const T* kp = static_cast<const T*>(p.k) + (size_t)k0 * p.ldk + (size_t)kvh * d;
  const T* vp = static_cast<const T*>(p.v) + (size_t)k0 * p.ldv + (size_t)kvh * d;
  const unsigned ldk = (unsigned)p.ldk, ldv = (unsigned)p.ldv;       // 32 rows are below 2^31 bytes
  float qx[ND][8];
#pragma unroll
  for (int n = 0; n < ND; ++n) {
    load8<DT, VEC>(src, (mine ? col : 0) * (unsigned)p.ldq, n, g, d, qx[n]);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (column_of<DT>(n, g, j) >= d) qx[n][j] = 0.f;               // what keys have there then does not count
  }
  // keys [j0, j0 + 16) and their values.  Keys past the end repeat the last one: masked below.  Columns past d repeat one that
  // is there: not stored
  auto fetch = [&](unsigned j0, float (&kx)[ND][8], float (&vx)[2 * ND][4]) {
    const T *kj = kp + (size_t)j0 * p.ldk, *vj = vp + (size_t)j0 * p.ldv;
    const unsigned last = nk - j0 - 1, krow = min(col, last) * ldk;
#pragma unroll
    for (int n = 0; n < ND; ++n) load8<DT, VEC>(kj, krow, n, g, d, kx[n]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned vrow = min(4 * g + j, last) * ldv;
#pragma unroll
      for (int t = 0; t < 2 * ND; ++t) vx[t][j] = (float)vj[vrow + (16 * t + col < d ? 16 * t + col : 0)];
    }
  };
  v4f o[2 * ND];
#pragma unroll
  for (int t = 0; t < 2 * ND; ++t) o[t] = v4f{};
  float top = -INFINITY, total = 0.f;
  bool poison = false;
  float kn[ND][8], vn[2 * ND][4];
  if (most > 0) fetch(0, kn, vn);
  for (unsigned j0 = 0; j0 < most; j0 += 16) {
    float kx[ND][8], vx[2 * ND][4];
    float check = 0.f;                                 // NaN as soon as one of them is not finite
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        kx[n][j] = kn[n][j];
        vx[2 * n + j / 4][j % 4] = vn[2 * n + j / 4][j % 4];
        check = fmaf(kx[n][j], 0.f, fmaf(vx[2 * n + j / 4][j % 4], 0.f, check));
      }
    if (j0 + 16 < most) fetch(j0 + 16, kn, vn);
    if (__any(check != check)) {
      unsigned bad = 0;                                // keys that are not finite; their elements become zero
      auto clean = [&](float& x, unsigned key) {
        const bool fine = fabsf(x) <= 3.402823466e38f;
        x = fine ? x : 0.f;
        bad |= fine ? 0u : 1u << key;
        asm volatile("" : "+v"(bad));                  // one after the other: so many conditions at once do not fit
      };
#pragma unroll
      for (int n = 0; n < ND; ++n)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          clean(kx[n][j], col);
          clean(vx[2 * n + j / 4][j % 4], 4 * g + j % 4);
        }
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) bad |= __shfl_xor(bad, off, 64);
      if (seen > j0) poison |= (seen - j0 >= 16 ? bad : bad & ((1u << (seen - j0)) - 1)) != 0;
    }
    v4f s = {};
#pragma unroll
    for (int n = 0; n < ND; ++n) s = mfma_columns<DT>(kx[n], qx[n], s);
    float e[4], m = -INFINITY;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      e[j] = j0 + 4 * g + j < seen ? s[j] * p.scale2 : -INFINITY;
      m = fmaxf(m, e[j]);
    }
    auto larger = [](float a, float b) { return fmaxf(a, b); };
    m = fmaxf(top, across16_f(across32_f(m, larger), larger));
    const float ref = m == -INFINITY ? 0.f : m, keep = __builtin_amdgcn_exp2f(top - ref);
    top = m;
    total *= keep;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      e[j] = __builtin_amdgcn_exp2f(e[j] - ref);
      total += e[j];
    }
#pragma unroll
    for (int t = 0; t < 2 * ND; ++t) o[t] = mfma_keys<DT>(vx[t], e, o[t] * keep);
  }
  auto sum = [](float a, float b) { return a + b; };
  total = across16_f(across32_f(total, sum), sum);
  if (!mine) return;
  const float inv = inverse_of(total, poison, seen);
  T* dst = static_cast<T*>(p.out) + (size_t)(q0 + i) * p.ldo + (size_t)head * d;
#pragma unroll
  for (int t = 0; t < 2 * ND; ++t) store4<DT>(dst, o[t][0], o[t][1], o[t][2], o[t][3], inv, 16 * t + 4 * g, d, VEC);
}

}  // namespace

// Which kernel: by the mean length, the only one known without reading the lists.  (Where one sequence is far longer than
// the mean that is the wrong one: one of 8000 among 63 of 1, 32 heads of 128 over 8, bfloat16, takes 6.6 ms in the short form;
// and 512 queries on 8000 keys, which are not many queries, 263 us in the form between.)  Measured (us, causal, sequences x length,
// d = 64 with 8 heads | d = 128 with 16 heads over 4):
//   binary32, pack + attention / short: 64 x 96 41 / 19 | 75 / 62, 32 x 192 37 / 32 | 98 / 99, 32 x 256 52 / 51 | 120 / 155,
//     8 x 800 72 / 96
//   bfloat16, pack + attention / short: 64 x 96 18 / 13 | 39 / 39, 64 x 128 25 / 17 | 58 / 55, 32 x 192 19 / 20 | 39 / 57,
//     16 x 400 25 / 34 | 54 / 98
//   bfloat16, pack + attention / pack + wide: 8 x 1100 52 / 60 | 100 / 116, 16 x 1500 110 / 104 | 277 / 286,
//     4 x 2000 72 / 64 | 142 / 131, 3 x 3000 90 / 89 | 199 / 184, 2 x 8000 296 / 289 | 701 / 566
// d = 256 with 4 heads | d = 192 with 16 heads over 4, pack + attention / short:
//   binary32: 256 x 2 84 / 11 | 182 / 26, 64 x 64 59 / 34 | 83 / 67, 32 x 128 59 / 55 | 119 / 99, 32 x 192 97 / 111 | 147 / 188
//   bfloat16: 256 x 2 61 / 11 | 156 / 30, 100 x 32 37 / 23 | 78 / 53, 64 x 64 36 / 28 | 50 / 66, 64 x 96 46 / 51 | 71 / 105
constexpr size_t kShortMean32 = 192, kShortMean16 = 128, kShortMeanWide32 = 128, kShortMeanWide16 = 48, kLongMean = 1536;

static size_t k_slots(size_t B, size_t Tk) { return Tk / kUnit + B; }

size_t prompt_attention_ws_bytes(int dtype, size_t B, size_t Tk, int kv_heads, size_t d) {
  const size_t n = k_slots(B, Tk) * (size_t)kv_heads;
  return n * unit_bytes((unsigned)d, dtype == MQ_F32 ? 3 : 1) + round_up(n * sizeof(unsigned), 256);
}

int launch_prompt_attention(const void* q, size_t ldq, const void* k, size_t ldk, const void* v, size_t ldv, int dtype,
                            const int32_t* q_first, const int32_t* k_first, size_t B, size_t Tq, size_t Tk, int heads,
                            int kv_heads, size_t d, int causal, float scale, void* out, size_t ldo, void* ws, hipStream_t s) {
  const size_t n = k_slots(B, Tk) * (size_t)kv_heads, q_slots = Tq / (kW * kQ) + B;
  const size_t few = (dtype == MQ_F32 ? d <= 128 ? kShortMean32 : kShortMeanWide32 : d <= 128 ? kShortMean16 : kShortMeanWide16) * B;
  const bool is_short = ldq < (size_t)1 << 24 && ldk < (size_t)1 << 24 && ldv < (size_t)1 << 24 && Tq <= few && Tk <= few;
  const bool is_long = d <= 128 && scale != 0.f && Tq >= kLongMean * B;
  // every launch of the call, before the first
  const size_t h = (size_t)heads;
  if (is_short ? !launchable(((Tq / kQShort + B) * h + 3) / 4, 256)
               : !launchable(n, 256) || !launchable(q_slots * h, dtype == MQ_F32 ? 2 * kW * kWave : kW * kWave))
    return MQ_ERR_SHAPE;
  const size_t per16 = 16 / elem_bytes(dtype);
  auto whole = [&](const void* x, size_t ld) { return reinterpret_cast<uintptr_t>(x) % 16 == 0 && ld % per16 == 0; };
  const bool vec = d % 8 == 0 && whole(q, ldq) && whole(k, ldk) && whole(v, ldv) && whole(out, ldo);
  uint8_t* units = static_cast<uint8_t*>(ws);
  PromptParams p{q, k, v, out, q_first, k_first, units,
                 reinterpret_cast<unsigned*>(units + n * unit_bytes((unsigned)d, dtype == MQ_F32 ? 3 : 1)),
                 ldq, ldk, ldv, ldo, (unsigned)B, (unsigned)Tq, (unsigned)Tk, (unsigned)heads, (unsigned)kv_heads, (unsigned)d,
                 (unsigned)q_slots, (unsigned)k_slots(B, Tk), causal, 0, vec, scale * 1.44269504088896340736f};
  return with_dtype(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    if (is_short) {
      p.q_slots = (unsigned)(Tq / kQShort + B);
      auto go = [&](auto nd) {
        constexpr int ND = decltype(nd)::value;
        const unsigned n = (unsigned)(((size_t)p.q_slots * p.heads + 3) / 4);
        if (vec) hipLaunchKernelGGL((k_prompt_short<DT, ND, true>), dim3(n), dim3(256), 0, s, p);
        else hipLaunchKernelGGL((k_prompt_short<DT, ND, false>), dim3(n), dim3(256), 0, s, p);
        return check_hip(hipGetLastError());
      };
      switch (padded(p.d) / 32) {
        case 1: return go(std::integral_constant<int, 1>{});
        case 2: return go(std::integral_constant<int, 2>{});
        case 3: return go(std::integral_constant<int, 3>{});
        case 4: return go(std::integral_constant<int, 4>{});
        case 5:
        case 6: return go(std::integral_constant<int, 6>{});
        default: return go(std::integral_constant<int, 8>{});
      }
    }
    hipLaunchKernelGGL((k_prompt_pack<DT>), dim3((unsigned)n), dim3(256), 0, s, p);
    int rc = check_hip(hipGetLastError());
    if (rc != MQ_OK) return rc;
    if constexpr (DT != MQ_F32) {
      if (is_long) {
        p.q_slots = (unsigned)(Tq / (2 * kW * kQ) + B);
        p.negative = scale < 0.f;
        p.scale2 = fabsf(p.scale2);
        auto go = [&](auto nd) {
          constexpr int ND = decltype(nd)::value;
          constexpr unsigned lds = kRing * 2 * kUnit * 32 * ND * 2;
          auto kern = k_prompt_wide<DT, ND>;
          if (lds > 65536) {
            const int e = check_hip(hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                        hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
            if (e != MQ_OK) return e;
          }
          hipLaunchKernelGGL(kern, dim3((unsigned)(p.q_slots * (size_t)p.heads)), dim3(kW * kWave), lds, s, p);
          return check_hip(hipGetLastError());
        };
        switch (padded(p.d) / 32) {
          case 1: return go(std::integral_constant<int, 1>{});
          case 2: return go(std::integral_constant<int, 2>{});
          case 3: return go(std::integral_constant<int, 3>{});
          default: return go(std::integral_constant<int, 4>{});
        }
      }
    }
    auto go = [&](auto nd) {
      constexpr int ND = decltype(nd)::value;
      // two units to a tile and two tiles in LDS where they fit, else one of both
      constexpr unsigned UNIT = 2 * kUnit * 32 * ND * 2 * kParts<DT>;
      constexpr int NU = DT != MQ_F32 && 4 * UNIT <= kLds ? 2 : 1, BUF = 2 * NU * UNIT <= kLds ? 2 : 1;
      // and two groups of waves, where LDS holds as much for each
      constexpr int KS = DT == MQ_F32 && 2 * NU * BUF * UNIT <= kLds ? 2 : 1;
      auto kern = k_prompt_attention<DT, ND, NU, BUF, KS>;
      constexpr unsigned lds = NU * BUF * KS * UNIT;
      if (lds > 65536) {
        const int e = check_hip(hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                    hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        if (e != MQ_OK) return e;
      }
      hipLaunchKernelGGL(kern, dim3((unsigned)(p.q_slots * (size_t)heads)), dim3(KS * kW * kWave), lds, s, p);
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
