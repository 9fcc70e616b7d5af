// Log probabilities of given words, entropy and best alternatives under the 8-bit output layer (include/mq_seq.h).
//
// y[m][n] = acc[m][n] / (sA sW) over tens of thousands of words is never stored.  The product runs on v_mfma_i32_32x32x32_i8 with
// 32 words as operand a and 32 rows of hidden states as operand b: lane l then holds 16 words for ONE row (l % 32), so the
// softmax statistics and the list of best words are plain registers of the lane.  The hidden states stay in registers for the
// whole launch, the embedding streams through LDS once per workgroup column; both are packed in operand order already.
//   * statistics in base 2 relative to c = -(largest sum so far) u2, u2 = log2(e) / (sA sW):  z = fma(acc, u2, c),
//     l = sum 2^z, t = sum 2^z z; moving c by -D turns (l, t) into 2^-D (l, t - D l).  log2 sum 2^(y log2 e) = log2(l) - c
//     for the very c that was used, whatever it was rounded to, and the entropy is ln 2 (log2 l - t / l).
//   * best words: sums are below 2^24, so sum << 7 | 127 - place is a 32-bit key that orders by sum, then by earlier place, for
//     128 places of a lane (8 units of 32 words); a sorted list takes a key with one maximum and medians of three.  After 8
//     units the list is decoded and merged into one of 64-bit keys (sum, word).
// Every (row, workgroup column) leaves its statistics and list in the workspace; a second kernel joins them, a wave per row,
// and forms the given word's sum itself (one dot product of K bytes).
#include <type_traits>

#include "mq_gemm_common.h"
#include "mq_glue.h"
#include "mq_seq_common.h"

namespace mq {

namespace {

constexpr int kWaves = 8;
constexpr int kTagBits = 7, kUnitsPerList = 8;
constexpr int kNone = -2147483647 - 1;          // below every key: sums are above -2^24

struct LogprobParams {
  const uint8_t *packedA, *packedW;
  unsigned M, N, K, kfrags;
  unsigned columns, row_waves;          // workgroups that share the words; waves of a workgroup that share the rows
  float4* stat;                         // [M][columns words groups]: c, l, t
  unsigned long long* list;             // the same, NB keys each
  const float *sA, *sW;
  const int32_t* target;
  int k;
  float *logprob, *entropy, *alt;
  int32_t* tok;
};

typedef unsigned long long u64;
// (sum, word) as a key: larger sum first, then lower word; 0 = none
__device__ __forceinline__ u64 key_of(int sum, unsigned word) {
  return ((u64)((unsigned)sum ^ 0x80000000u) << 32) | (0xFFFFFFFFu - word);
}
__device__ __forceinline__ int sum_of(u64 key) { return (int)((unsigned)(key >> 32) ^ 0x80000000u); }
__device__ __forceinline__ unsigned word_of(u64 key) { return 0xFFFFFFFFu - (unsigned)key; }

__device__ __forceinline__ int median3(int a, int b, int c) { return max(min(a, b), min(max(a, b), c)); }

// top = the NB largest of two descending lists, descending (NB a power of two)
template <int NB>
__device__ __forceinline__ void merge_lists(u64 (&top)[NB], const u64 (&other)[NB]) {
#pragma unroll
  for (int j = 0; j < NB; ++j) top[j] = top[j] > other[NB - 1 - j] ? top[j] : other[NB - 1 - j];
#pragma unroll
  for (int half = NB / 2; half >= 1; half /= 2)
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if ((j & half) == 0) {
        const u64 a = top[j], b = top[j + half];
        top[j] = a > b ? a : b;
        top[j + half] = a > b ? b : a;
      }
}

// (c, l, t) of the union of two sets of words
__device__ __forceinline__ void join_stats(float& c, float& l, float& t, float c2, float l2, float t2) {
  const float low = fminf(c, c2), a = c - low, b = c2 - low;       // the lower c belongs to the larger maximum
  const float ea = __builtin_amdgcn_exp2f(-a), eb = __builtin_amdgcn_exp2f(-b);
  t = ea * (t - (l > 0.f ? a * l : 0.f)) + eb * (t2 - (l2 > 0.f ? b * l2 : 0.f));
  l = ea * l + eb * l2;
  c = low;
}

// KF: 32-element pieces of K held, CT: 32-row tiles of a wave, NB: length of the list of best words (0: none)
template <int KF, int CT, int NB>
__global__ __launch_bounds__(kWaves * kWave) void k_logprob_stream(const LogprobParams p) {
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const unsigned lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const unsigned wr = wave % p.row_waves, wn = wave / p.row_waves, word_waves = kWaves / p.row_waves;
  const unsigned column = blockIdx.x % p.columns, chunk = blockIdx.x / p.columns;
  const unsigned tile0 = (chunk * p.row_waves + wr) * CT, tiles = (p.M + 31) / 32;
  const unsigned units = (p.N + 31) / 32, stages = (units + word_waves - 1) / word_waves;
  const unsigned kf = p.kfrags, unit_bytes = kf * kFragBytes, stage_bytes = word_waves * unit_bytes;
  const float u2 = __fmul_rn(__fdiv_rn(1.0f, __fmul_rn(*p.sA, *p.sW)), 1.44269504088896340736f);

  v4i h[CT][KF];
#pragma unroll
  for (int i = 0; i < CT; ++i) {
    const unsigned t = tile0 + i < tiles ? tile0 + i : tiles - 1;
#pragma unroll
    for (int f = 0; f < KF; ++f)
      h[i][f] = f < (int)kf ? *reinterpret_cast<const v4i*>(p.packedA + ((size_t)t * kf + f) * kFragBytes + lane * 16) : v4i{};
  }
  float c[CT], l[CT], t[CT];
  int ref[CT];
  int best[CT][NB > 0 ? NB : 1];
  u64 top[CT][NB > 0 ? NB : 1];
#pragma unroll
  for (int i = 0; i < CT; ++i) {
    ref[i] = kNone;
    c[i] = 0.f;
    l[i] = t[i] = 0.f;
#pragma unroll
    for (int j = 0; j < (NB > 0 ? NB : 1); ++j) {
      best[i][j] = kNone;
      top[i][j] = 0;
    }
  }
  auto fetch = [&](unsigned stage, unsigned buf) {
    const unsigned u0 = stage * word_waves;
    for (unsigned piece = wave; piece < word_waves * kf; piece += kWaves) {
      const unsigned u = u0 + piece / kf < units ? u0 + piece / kf : units - 1;
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(p.packedW + ((size_t)u * kf + piece % kf) * kFragBytes + lane * 16),
          (__attribute__((address_space(3))) void*)(smem + buf * stage_bytes + piece * kFragBytes), 16, 0, 0);
    }
  };
  unsigned held = 0, list_unit = 0;              // units in the 32-bit lists, and the first of them
  const unsigned unit_step = p.columns * word_waves;
  auto flush = [&]() {
    if constexpr (NB > 0) {
#pragma unroll
      for (int i = 0; i < CT; ++i) {
        u64 keys[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          const unsigned place = 127u - ((unsigned)best[i][j] & 127u), r = place % 16;
          const unsigned word = (list_unit + place / 16 * unit_step) * 32 + 8 * (r / 4) + 4 * (lane / 32) + r % 4;
          keys[j] = best[i][j] == kNone ? 0 : key_of(best[i][j] >> kTagBits, word);
          best[i][j] = kNone;
        }
        merge_lists<NB>(top[i], keys);
      }
    }
    held = 0;
  };
  unsigned buf = 0;
  if (column < stages) fetch(column, 0);
  for (unsigned stage = column; stage < stages; stage += p.columns) {
    __builtin_amdgcn_s_waitcnt(0x0F70);
    __syncthreads();
    if (stage + p.columns < stages) fetch(stage + p.columns, buf ^ 1);
    const unsigned unit = stage * word_waves + wn;
    const uint8_t* at = smem + buf * stage_bytes + wn * unit_bytes + lane * 16;
    buf ^= 1;
    if (unit >= units || tile0 >= tiles) continue;
    v16i acc[CT];
#pragma unroll
    for (int i = 0; i < CT; ++i) acc[i] = v16i{};
#pragma unroll
    for (int f = 0; f < KF; ++f)
      if (f < (int)kf) {
        const v4i w = *reinterpret_cast<const v4i*>(at + f * kFragBytes);
#pragma unroll
        for (int i = 0; i < CT; ++i) acc[i] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w, h[i][f], acc[i], 0, 0, 0);
      }
    if (held == 0) list_unit = unit;
    const unsigned n0 = unit * 32 + 4 * (lane / 32);
    const bool whole = unit * 32 + 32 <= p.N;
#pragma unroll
    for (int i = 0; i < CT; ++i) {
      auto there = [&](int r) { return whole || n0 + 8 * (r / 4) + r % 4 < p.N; };
      int most = kNone;
#pragma unroll
      for (int r = 0; r < 16; ++r) most = max(most, there(r) ? acc[i][r] : kNone);
      if (__any(most > ref[i])) {
        const int now = max(most, ref[i]);
        const float cn = now == kNone ? 0.f : -(float)now * u2, D = l[i] > 0.f ? c[i] - cn : 0.f, e = __builtin_amdgcn_exp2f(-D);
        t[i] = e * (t[i] - D * l[i]);
        l[i] *= e;
        c[i] = cn;
        ref[i] = now;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float z = fmaf((float)acc[i][r], u2, c[i]), e = there(r) ? __builtin_amdgcn_exp2f(z) : 0.f;
        l[i] += e;
        t[i] = fmaf(e, z, t[i]);
        if constexpr (NB > 0) {
          const int key = there(r) ? (acc[i][r] << kTagBits) | (127 - (int)(held * 16 + r)) : kNone;
#pragma unroll
          for (int j = NB - 1; j > 0; --j) best[i][j] = median3(best[i][j - 1], best[i][j], key);
          best[i][0] = max(best[i][0], key);
        }
      }
    }
    if (++held == kUnitsPerList) flush();
  }
  if (tile0 >= tiles) return;
  flush();
  const unsigned groups = p.columns * word_waves, group = column * word_waves + wn;
#pragma unroll
  for (int i = 0; i < CT; ++i) {
    const unsigned m = (tile0 + i) * 32 + lane % 32;
    // the two lanes of a row.  A lane without words has l = 0 and must not set the reference
    const float c2 = __shfl_xor(c[i], 32, 64), l2 = __shfl_xor(l[i], 32, 64), t2 = __shfl_xor(t[i], 32, 64);
    const int ref2 = __shfl_xor(ref[i], 32, 64);
    if (ref[i] == kNone) {
      c[i] = c2;
      l[i] = l2;
      t[i] = t2;
    } else if (ref2 != kNone) {
      join_stats(c[i], l[i], t[i], c2, l2, t2);
    }
    const bool any = ref[i] != kNone || ref2 != kNone;
    if constexpr (NB > 0) {
      u64 other[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) other[j] = __shfl_xor(top[i][j], 32, 64);
      merge_lists<NB>(top[i], other);
    }
    if (lane < 32 && tile0 + i < tiles && m < p.M) {
      p.stat[(size_t)m * groups + group] = make_float4(c[i], l[i], t[i], any ? 1.f : 0.f);
      if constexpr (NB > 0)
#pragma unroll
        for (int j = 0; j < NB; ++j) p.list[((size_t)m * groups + group) * NB + j] = top[i][j];
    }
  }
}

// A wave per row.
template <int NB>
__global__ __launch_bounds__(256) void k_logprob_join(const LogprobParams p, unsigned groups) {
  const unsigned lane = threadIdx.x % kWave, m = blockIdx.x * (256 / kWave) + threadIdx.x / kWave;
  if (m >= p.M) return;
  const float u2 = __fmul_rn(__fdiv_rn(1.0f, __fmul_rn(*p.sA, *p.sW)), 1.44269504088896340736f);
  float c = 0.f, l = 0.f, t = 0.f;
  bool any = false;
  u64 top[NB > 0 ? NB : 1] = {};
  for (unsigned g = lane; g < groups; g += kWave) {
    const float4 s = p.stat[(size_t)m * groups + g];
    if (s.w != 0.f) {
      if (any) join_stats(c, l, t, s.x, s.y, s.z);
      else { c = s.x; l = s.y; t = s.z; }
      any = true;
    }
    if constexpr (NB > 0) {
      u64 other[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) other[j] = p.list[((size_t)m * groups + g) * NB + j];
      merge_lists<NB>(top, other);
    }
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const float c2 = __shfl_xor(c, off, 64), l2 = __shfl_xor(l, off, 64), t2 = __shfl_xor(t, off, 64);
    const bool any2 = __shfl_xor((int)any, off, 64) != 0;
    if (any && any2) join_stats(c, l, t, c2, l2, t2);
    else if (any2) { c = c2; l = l2; t = t2; }
    any |= any2;
    if constexpr (NB > 0) {
      u64 other[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) other[j] = __shfl_xor(top[j], off, 64);
      merge_lists<NB>(top, other);
    }
  }
  // the given word's sum: 16 elements of K per lane, element k of row n in piece k / 32, half (k / 16) % 2
  const int word = p.target[m];
  const bool given = word >= 0 && (unsigned)word < p.N;
  int sum = 0;
  if (given)
    for (unsigned i = lane; i < p.kfrags * 2; i += kWave) {
      const size_t in = (size_t)(i / 2) * kFragBytes + (i % 2) * 512;
      const v4i a = *reinterpret_cast<const v4i*>(p.packedA + (size_t)(m / 32) * p.kfrags * kFragBytes + in + m % 32 * 16);
      const v4i w = *reinterpret_cast<const v4i*>(p.packedW + (size_t)(word / 32) * p.kfrags * kFragBytes + in + word % 32 * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) sum = __builtin_amdgcn_sdot4(a[j], w[j], sum, false);
    }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
  const float norm = log2f(l), ln2 = 0.69314718055994530942f;
  if (lane == 0) {
    p.logprob[m] = given ? (fmaf((float)sum, u2, c) - norm) * ln2 : 0.f;
    if (p.entropy != nullptr) {
      const float H = (norm - __fdiv_rn(t, l)) * ln2;
      p.entropy[m] = H < 0.f ? 0.f : H;            // (rounding)
    }
  }
  if constexpr (NB > 0)
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (lane == (unsigned)j && j < p.k) {
        p.tok[(size_t)m * p.k + j] = (int32_t)word_of(top[j]);
        p.alt[(size_t)m * p.k + j] = (fmaf((float)sum_of(top[j]), u2, c) - norm) * ln2;
      }
}

struct Shape {
  unsigned row_waves, ct, chunks, columns, groups;
};
Shape shape_of(size_t M, size_t N, bool wide) {
  Shape s;
  const size_t tiles = (M + 31) / 32, units = (N + 31) / 32;
  s.ct = !wide && tiles > 8 ? 2 : 1;
  const size_t waves = (tiles + s.ct - 1) / s.ct;
  s.row_waves = wide ? 4 : 2;           // (so that two stages fit LDS)
  while (s.row_waves < 8 && s.row_waves < waves) s.row_waves *= 2;
  s.chunks = (unsigned)((waves + s.row_waves - 1) / s.row_waves);
  const size_t stages = (units + kWaves / s.row_waves - 1) / (kWaves / s.row_waves);
  const size_t want = s.chunks >= 256 ? 1 : 256 / s.chunks;
  s.columns = (unsigned)(want < stages ? want : stages);
  s.groups = s.columns * (kWaves / s.row_waves);
  return s;
}
int list_length(int k) { return k == 0 ? 0 : k <= 4 ? 4 : 8; }

}  // namespace

size_t token_logprob_ws_bytes(size_t M, size_t N, int k) {
  size_t most = 0;
  for (int wide = 0; wide < 2; ++wide) {
    const size_t n = M * shape_of(M, N, wide != 0).groups * (sizeof(float4) + list_length(k) * sizeof(u64));
    if (n > most) most = n;
  }
  return most;
}

int launch_token_logprob(const void* packedA, const void* packedW, size_t M, size_t N, size_t K, const float* sA,
                         const float* sW, const int32_t* target, int k, float* logprob, float* entropy, int32_t* tok,
                         float* alt, void* ws, hipStream_t s) {
  const unsigned kf = (unsigned)PackedDims(8, N, K).kfrags;
  const Shape sh = shape_of(M, N, kf > 16);
  LogprobParams p{static_cast<const uint8_t*>(packedA), static_cast<const uint8_t*>(packedW), (unsigned)M, (unsigned)N,
                  (unsigned)K, kf, sh.columns, sh.row_waves, static_cast<float4*>(ws),
                  reinterpret_cast<u64*>(static_cast<float4*>(ws) + M * sh.groups), sA, sW, target, k, logprob, entropy, alt, tok};
  auto go = [&](auto kfc, auto ctc, auto nbc) {
    constexpr int NB = decltype(nbc)::value;
    auto kern = k_logprob_stream<decltype(kfc)::value, decltype(ctc)::value, NB>;
    const unsigned lds = 2 * kWaves / sh.row_waves * kf * kFragBytes;
    if (lds > 65536) {
      const int e = check_hip(hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                  hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
      if (e != MQ_OK) return e;
    }
    hipLaunchKernelGGL(kern, dim3(sh.columns * sh.chunks), dim3(kWaves * kWave), lds, s, p);
    const int rc = check_hip(hipGetLastError());
    if (rc != MQ_OK) return rc;
    hipLaunchKernelGGL((k_logprob_join<NB>), dim3((unsigned)((M + 3) / 4)), dim3(256), 0, s, p, sh.groups);
    return check_hip(hipGetLastError());
  };
  auto with_list = [&](auto kfc, auto ctc) {
    switch (list_length(k)) {
      case 0: return go(kfc, ctc, std::integral_constant<int, 0>{});
      case 4: return go(kfc, ctc, std::integral_constant<int, 4>{});
      default: return go(kfc, ctc, std::integral_constant<int, 8>{});
    }
  };
  if (kf > 16) return with_list(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
  if (sh.ct == 2) return with_list(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
  return with_list(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
}

}  // namespace mq
