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
// Bound by the matrix instructions where there are many rows (8192 x 36000 x 1024: 292 .. 300 us with the join, 2.0 POP/s; they
// take 53 % of the clocks in which the compute units are busy, vector ones 36 %).  With 384 rows (36000 x 512, 4 best words,
// 24.5 us with the join) a compute unit is busy for 37 000 clocks, about 16 us, of which vector instructions, twelve for a word with a
// list, take half and matrix instructions 18 %; a wave waits a third of its time, for the start, where every workgroup fetches its
// rows' hidden states, and for the end, after four or five stages.
// u2 is rounded once more than 1 / (sA sW) and a lane adds up its words one after the other: 2.2e-7 off the result in 64 bits
// (8192 rows; 6.8e-8 with a sum over the whole row at once).
// Every (row, workgroup column) leaves its statistics and list in the workspace; a second kernel joins them, a wave per row,
// and forms the given word's sum itself (one dot product of K bytes).
#include <type_traits>

#include "mq_gemm_common.h"
#include "mq_glue.h"
#include "mq_seq_common.h"

namespace mq {

namespace {

// waves of a workgroup at most, by what a wave's registers leave room for (KF: pieces of K held, CT: tiles of 32 rows)
constexpr int most_waves(int KF, int CT) { return KF == 16 && CT == 1 ? 12 : 8; }
constexpr unsigned kMostColumns = 256;
constexpr size_t kLdsBytes = 160 * 1024;
#define MQ_INLINE __attribute__((always_inline))
constexpr int kTagBits = 7, kUnitsPerList = 8;
constexpr int kNone = -2147483647 - 1;          // below every key: sums are above -2^24

struct LogprobParams {
  const uint8_t *packedA, *packedW;
  unsigned M, N, kfrags;
  unsigned columns, row_waves, ring;    // workgroups that share the words; waves of one that share the rows; stages in LDS
  float4* stat;                         // [M][columns]: c, l, t, whether there are words
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

// Waits until at most n loads of this wave are on their way (fewer where n is none of the steps).
__device__ __forceinline__ void wait_loads(unsigned n) {
  asm volatile("" ::: "memory");
#define MQ_WAIT(N) __builtin_amdgcn_s_waitcnt(((N) & 15) | ((N) >> 4) << 14 | 0x0F70)
  if (n >= 32) MQ_WAIT(32);
  else if (n >= 24) MQ_WAIT(24);
  else if (n >= 16) MQ_WAIT(16);
  else if (n >= 12) MQ_WAIT(12);
  else if (n >= 8) MQ_WAIT(8);
  else if (n >= 6) MQ_WAIT(6);
  else if (n >= 4) MQ_WAIT(4);
  else if (n >= 2) MQ_WAIT(2);
  else MQ_WAIT(0);
#undef MQ_WAIT
}

// A wave's statistics and list of a tile, joined over the two lanes of a row and over the waves that shared its words, to the
// workspace.
template <int NB, int CT>
__device__ __forceinline__ void finish(const LogprobParams& p, uint8_t* smem, int x, unsigned tile, unsigned tiles, unsigned column,
                                       unsigned wave, unsigned wr, unsigned wn, unsigned word_waves, unsigned waves, unsigned lane,
                                       int ref, float c, float l, float t, u64 (&top)[NB > 0 ? NB : 1]) {
  // the two lanes of a row.  A lane without words has l = 0 and must not set the reference
  const float c2 = __shfl_xor(c, 32, 64), l2 = __shfl_xor(l, 32, 64), t2 = __shfl_xor(t, 32, 64);
  const int ref2 = __shfl_xor(ref, 32, 64);
  if (ref == kNone) {
    c = c2;
    l = l2;
    t = t2;
  } else if (ref2 != kNone) {
    join_stats(c, l, t, c2, l2, t2);
  }
  bool any = ref != kNone || ref2 != kNone;
  if constexpr (NB > 0) {
    u64 other[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) other[j] = __shfl_xor(top[j], 32, 64);
    merge_lists<NB>(top, other);
  }
  // the waves that shared the words of a row, through LDS
  if (word_waves > 1) {
    __builtin_amdgcn_s_waitcnt(0x0F70);          // (loads for stages that are not there land in LDS too)
    __syncthreads();
    float4* stat = reinterpret_cast<float4*>(smem);
    u64* list = reinterpret_cast<u64*>(smem + waves * 32 * sizeof(float4));
    if (wn > 0 && lane < 32) {
      stat[wave * 32 + lane] = make_float4(c, l, t, any ? 1.f : 0.f);
      if constexpr (NB > 0)
#pragma unroll
        for (int j = 0; j < NB; ++j) list[(wave * 32 + lane) * NB + j] = top[j];
    }
    __syncthreads();
    for (unsigned w = 1; w < word_waves && wn == 0; ++w) {
      const unsigned at = (w * p.row_waves + wr) * 32 + lane % 32;
      const float4 s = stat[at];
      if (s.w != 0.f) {
        if (any) join_stats(c, l, t, s.x, s.y, s.z);
        else { c = s.x; l = s.y; t = s.z; }
        any = true;
      }
      if constexpr (NB > 0) {
        u64 other[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) other[j] = list[at * NB + j];
        merge_lists<NB>(top, other);
      }
    }
  }
  const unsigned m = tile * 32 + lane;
  if (wn == 0 && lane < 32 && tile < tiles && m < p.M) {
    p.stat[(size_t)m * p.columns + column] = make_float4(c, l, t, any ? 1.f : 0.f);
    if constexpr (NB > 0)
#pragma unroll
      for (int j = 0; j < NB; ++j) p.list[((size_t)m * p.columns + column) * NB + j] = top[j];
  }
}

// KF: 32-element pieces of K held, CT: tiles of 32 rows, NB: length of the list of best words (0: none)
// A unit's matrix instructions stand beside the vector ones of the unit before (all of K held: K of 512 or 1024 elements; other
// widths one after the other).  Pieces are asked of LDS three ahead.
template <int KF, int CT, int NB>
__global__ __launch_bounds__(most_waves(KF, CT) * kWave, 1) void k_logprob_stream(const LogprobParams p) {
  constexpr int NL = NB > 0 ? NB : 1;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const unsigned lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  const unsigned wr = wave % p.row_waves, wn = wave / p.row_waves, word_waves = waves / p.row_waves;
  const unsigned column = blockIdx.x % p.columns, chunk = blockIdx.x / p.columns;
  const unsigned tile = (chunk * p.row_waves + wr) * CT, tiles = (p.M + 31) / 32;
  const unsigned units = (p.N + 31) / 32, stages = (units + word_waves - 1) / word_waves;
  const unsigned kf = p.kfrags, unit_bytes = kf * kFragBytes, stage_bytes = word_waves * unit_bytes;
  const unsigned pieces = word_waves * kf, each = (pieces + waves - 1) / waves;      // 1 KB pieces of a stage, loads of a wave
  const unsigned mine = column < stages ? (stages - column + p.columns - 1) / p.columns : 0u;      // this workgroup's stages

  // every wave issues the same number of loads for a stage (a piece may come twice), past the last stage as well: how many are
  // on their way at a given point does not depend on anything
  // (a stage's units lie next to each other; slots and places by addition, a division would stand in front of every stage)
  const size_t step = (size_t)p.columns * pieces, all = (size_t)units * kf;
  size_t next = (size_t)column * pieces;         // first piece of the stage that is fetched next
  unsigned next_left = mine, next_slot = 0, slot = 0;
  const unsigned ring_bytes = p.ring * stage_bytes;
  auto fetch = [&]() MQ_INLINE {
    for (unsigned j = 0; j < each; ++j) {
      const unsigned piece = min(wave + j * waves, pieces - 1);
      const size_t at = next + piece < all ? next + piece : all - 1;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(p.packedW + at * kFragBytes + lane * 16),
                                       (__attribute__((address_space(3))) void*)(smem + next_slot + piece * kFragBytes), 16, 0, 0);
    }
    if (next_left > 1) {
      --next_left;
      next += step;
    }
    next_slot = next_slot + stage_bytes == ring_bytes ? 0 : next_slot + stage_bytes;
  };
  if (mine > 0)
    for (unsigned i = 0; i + 1 < p.ring; ++i) fetch();
  const float u2 = __fmul_rn(__fdiv_rn(1.0f, __fmul_rn(*p.sA, *p.sW)), 1.44269504088896340736f);
  v4i h[CT][KF];
#pragma unroll
  for (int x = 0; x < CT; ++x) {
    const uint8_t* rows = p.packedA + (size_t)min(tile + x, tiles - 1) * kf * kFragBytes + lane * 16;
#pragma unroll
    for (int f = 0; f < KF; ++f) h[x][f] = *reinterpret_cast<const v4i*>(rows + (f < (int)kf ? f : 0) * kFragBytes);
  }
  float c[CT], l[CT], t[CT];
  int ref[CT], best[CT][NL];
  u64 top[CT][NL];
#pragma unroll
  for (int x = 0; x < CT; ++x) {
    c[x] = l[x] = t[x] = 0.f;
    ref[x] = kNone;
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      best[x][j] = kNone;
      top[x][j] = 0;
    }
  }
  unsigned held = 0, list_unit = 0;              // units in the 32-bit lists, and the first of them
  const unsigned unit_step = p.columns * word_waves;
  auto flush = [&]() MQ_INLINE {
    if constexpr (NB > 0)
#pragma unroll
      for (int x = 0; x < CT; ++x) {
        u64 keys[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          const unsigned place = 127u - ((unsigned)best[x][j] & 127u), r = place % 16;
          const unsigned word = (list_unit + place / 16 * unit_step) * 32 + 8 * (r / 4) + 4 * (lane / 32) + r % 4;
          keys[j] = best[x][j] == kNone ? 0 : key_of(best[x][j] >> kTagBits, word);
          best[x][j] = kNone;
        }
        merge_lists<NB>(top[x], keys);
      }
    held = 0;
  };
  int sums[CT][16];                              // of unit `unit`, whose turn with the vector unit is next
  unsigned unit = 0;
  // the vocabulary's last unit may have fewer than 32 words; a wave has it last
  auto there = [&](auto whole, int r) MQ_INLINE {
    return decltype(whole)::value || unit * 32 + 4 * (lane / 32) + 8 * (r / 4) + r % 4 < p.N;
  };
  auto settle = [&](auto whole) MQ_INLINE {
    if (held == 0) list_unit = unit;
#pragma unroll
    for (int x = 0; x < CT; ++x) {
      int most = kNone;
#pragma unroll
      for (int r = 0; r < 16; r += 2)
        most = max(max(most, there(whole, r) ? sums[x][r] : kNone), there(whole, r + 1) ? sums[x][r + 1] : kNone);
      if (__builtin_expect(__any(most > ref[x]), 0)) {
        const int now = max(most, ref[x]);
        const float cn = now == kNone ? 0.f : -(float)now * u2, D = l[x] > 0.f ? c[x] - cn : 0.f, e = __builtin_amdgcn_exp2f(-D);
        t[x] = e * (t[x] - D * l[x]);
        l[x] *= e;
        c[x] = cn;
        ref[x] = now;
      }
    }
  };
  // words [from, end) of the CT 16
  auto take = [&](auto whole, int tag, int from, int end) MQ_INLINE {
#pragma unroll
    for (int i = from; i < end; ++i) {
      const int x = i / 16, r = i % 16;
      const float z = fmaf((float)sums[x][r], u2, c[x]), e = there(whole, r) ? __builtin_amdgcn_exp2f(z) : 0.f;
      l[x] += e;
      t[x] = fmaf(e, z, t[x]);
      if constexpr (NB > 0) {
        const int key = there(whole, r) ? (sums[x][r] << kTagBits) + (tag - r) : kNone;
#pragma unroll
        for (int j = NB - 1; j > 0; --j) best[x][j] = median3(best[x][j - 1], best[x][j], key);
        best[x][0] = max(best[x][0], key);
      }
    }
  };
  auto tag = [&]() MQ_INLINE { return __builtin_amdgcn_readfirstlane(127 - (int)(held * 16)); };
  auto counted = [&]() MQ_INLINE { if (++held == kUnitsPerList) flush(); };
  const uint8_t* here = nullptr;                 // this wave's unit of the stage
  auto arrive = [&]() MQ_INLINE {
    wait_loads((p.ring - 2) * each);
    __builtin_amdgcn_s_barrier();                // the next stage is there, and nobody reads the one before
    asm volatile("" ::: "memory");
    fetch();
    here = smem + slot + wn * unit_bytes + lane * 16;
    slot = slot + stage_bytes == ring_bytes ? 0 : slot + stage_bytes;
  };
  // unit's sums; `beside`: the words of the unit before, settled already
  auto multiply = [&](const uint8_t* at, auto beside) MQ_INLINE {
    constexpr int AHEAD = 3;
    v4i piece[AHEAD + 1];
    auto read = [&](int f) MQ_INLINE { piece[f % (AHEAD + 1)] = *reinterpret_cast<const v4i*>(at + f * kFragBytes); };
#pragma unroll
    for (int f = 0; f < AHEAD; ++f) read(f);
    if constexpr (decltype(beside)::value) settle(std::true_type{});
    const int from = tag();
    v16i acc[CT] = {};
#pragma unroll
    for (int f = 0; f < KF; ++f) {
      if (f + AHEAD < KF) read(f + AHEAD);
#pragma unroll
      for (int x = 0; x < CT; ++x) acc[x] = __builtin_amdgcn_mfma_i32_32x32x32_i8(piece[f % (AHEAD + 1)], h[x][f], acc[x], 0, 0, 0);
      if constexpr (decltype(beside)::value) take(std::true_type{}, from, f * 16 * CT / KF, (f + 1) * 16 * CT / KF);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int x = 0; x < CT; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) sums[x][r] = acc[x][r];
  };
  const unsigned first = column * word_waves + wn;
  // this wave's units: stages [0, count)
  const unsigned count = tile < tiles && first < units ? (units - first + unit_step - 1) / unit_step : 0u;
  auto last = [&]() MQ_INLINE {
    if (unit * 32 + 32 <= p.N) {
      settle(std::true_type{});
      take(std::true_type{}, tag(), 0, 16 * CT);
    } else {
      settle(std::false_type{});
      take(std::false_type{}, tag(), 0, 16 * CT);
    }
    counted();
  };
  // Overlapped only where all of K held is there (449 .. 512 and 961 .. 1024 elements): with a check for each piece the order
  // cannot be kept.  8192 rows x 36000, overlapped / not, us: K = 512 156 / 260, with 4 best words 216 / 249; K = 1024 292 / 335,
  // 326 / 399.  384 rows with 4 best words: 24.7 / 26.3, 32.3 / 38.6.  Widths in between take the other loop, and longer than the
  // next whole one: 448 240, 640 282, 768 303, 960 331 (8192 rows).
  if (kf == KF) {
    if (mine > 0) {
      arrive();
      if (count > 0) {
        unit = first;
        multiply(here, std::false_type{});
      }
    }
    for (unsigned i = 1; i < mine; ++i) {
      arrive();
      if (i >= count) continue;
      multiply(here, std::true_type{});
      counted();
      unit += unit_step;
    }
    if (count > 0) last();
  } else {
    for (unsigned i = 0; i < mine; ++i) {
      arrive();
      if (i >= count) continue;
      unit = first + i * unit_step;
      v16i acc[CT] = {};
#pragma unroll
      for (int f = 0; f < KF; ++f)
        if (f < (int)kf) {
          const v4i w = *reinterpret_cast<const v4i*>(here + f * kFragBytes);
#pragma unroll
          for (int x = 0; x < CT; ++x) acc[x] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w, h[x][f], acc[x], 0, 0, 0);
        }
#pragma unroll
      for (int x = 0; x < CT; ++x)
#pragma unroll
        for (int r = 0; r < 16; ++r) sums[x][r] = acc[x][r];
      last();
    }
  }
  flush();
#pragma unroll
  for (int x = 0; x < CT; ++x)
    finish<NB, CT>(p, smem, x, tile + x, tiles, column, wave, wr, wn, word_waves, waves, lane, ref[x], c[x], l[x], t[x], top[x]);
}

// A wave per row.
template <int NB>
__global__ __launch_bounds__(256) void k_logprob_join(const LogprobParams p) {
  const unsigned lane = threadIdx.x % kWave, m = blockIdx.x * (256 / kWave) + threadIdx.x / kWave;
  if (m >= p.M) return;
  const int word = p.target[m];
  const float u2 = __fmul_rn(__fdiv_rn(1.0f, __fmul_rn(*p.sA, *p.sW)), 1.44269504088896340736f);
  float c = 0.f, l = 0.f, t = 0.f;
  bool any = false;
  u64 top[NB > 0 ? NB : 1] = {};
  // up to four parts a lane, all asked for at once
  float4 stat[kMostColumns / kWave];
  u64 list[kMostColumns / kWave][NB > 0 ? NB : 1];
#pragma unroll
  for (int i = 0; i < kMostColumns / kWave; ++i) {
    const size_t at = (size_t)m * p.columns + min(lane + i * kWave, p.columns - 1);
    stat[i] = p.stat[at];
    if constexpr (NB > 0)
#pragma unroll
      for (int j = 0; j < NB; ++j) list[i][j] = p.list[at * NB + j];
  }
  // the given word's: 16 elements of K per lane, element k of row n in piece k / 32, half (k / 16) % 2 (2 kfrags <= 64)
  const bool given = word >= 0 && (unsigned)word < p.N;
  const unsigned i0 = min(lane, p.kfrags * 2 - 1), n0 = given ? (unsigned)word : 0u;
  const size_t in = (size_t)(i0 / 2) * kFragBytes + (i0 % 2) * 512;
  const v4i pa = *reinterpret_cast<const v4i*>(p.packedA + (size_t)(m / 32) * p.kfrags * kFragBytes + in + m % 32 * 16);
  const v4i pw = *reinterpret_cast<const v4i*>(p.packedW + (size_t)(n0 / 32) * p.kfrags * kFragBytes + in + n0 % 32 * 16);
#pragma unroll
  for (int i = 0; i < kMostColumns / kWave; ++i) {
    if (lane + i * kWave >= p.columns) break;
    if (stat[i].w != 0.f) {
      if (any) join_stats(c, l, t, stat[i].x, stat[i].y, stat[i].z);
      else { c = stat[i].x; l = stat[i].y; t = stat[i].z; }
      any = true;
    }
    if constexpr (NB > 0) merge_lists<NB>(top, list[i]);
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
  int sum = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) sum = __builtin_amdgcn_sdot4(pa[j], pw[j], sum, false);
  if (lane >= p.kfrags * 2) sum = 0;
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

// How the product is dealt.  A workgroup's waves share its rows, 32 each, and, where there are few of them, the words of a stage;
// as many columns of workgroups as fill the chip once.
// Two tiles of rows a wave halve what it reads from LDS, and take twice its registers, so half the waves.  Measured over 36000
// words, one tile / two (us): K = 512 without a list 768 rows 27 / 30, 1024 rows 36 / 31, 4096 rows 91 / 84, 8192 rows 170 / 156;
// with 4 best words 1024 rows 42 / 43, 8192 rows 217 / 246; K = 1024 8192 rows 292 / 290 without a list, 326 / 349 with.
inline bool two_tiles(size_t M, unsigned kf, int nb) { return kf <= 16 && nb == 0 && M > 896; }
struct Shape {
  unsigned ct, row_waves, word_waves, chunks, columns, ring, most_columns;     // (columns whatever K is)
};
Shape shape_of(size_t M, size_t N, unsigned kf, int nb) {
  Shape s;
  s.ct = two_tiles(M, kf, nb) ? 2 : 1;
  const size_t tiles = ((M + 31) / 32 + s.ct - 1) / s.ct, units = (N + 31) / 32, most = most_waves(kf > 16 ? 32 : 16, (int)s.ct);
  s.chunks = (unsigned)((tiles + most - 1) / most);
  s.row_waves = (unsigned)((tiles + s.chunks - 1) / s.chunks);
  const size_t want = s.chunks >= kMostColumns ? 1 : kMostColumns / s.chunks;
  s.most_columns = (unsigned)want;
  // units of a stage: as many waves as there are, as one round of the columns needs, and as LDS holds twice
  size_t words = most / s.row_waves;
  const size_t needed = (units + want - 1) / want, fit = kLdsBytes / 2 / (kf * kFragBytes);
  words = words < needed ? words : needed;
  words = words < fit ? words : fit;
  s.word_waves = (unsigned)(words > 1 ? words : 1);
  const size_t stages = (units + s.word_waves - 1) / s.word_waves;
  s.columns = (unsigned)(want < stages ? want : stages);
  const size_t ring = kLdsBytes / (s.word_waves * kf * kFragBytes), each = (stages + s.columns - 1) / s.columns + 1;
  s.ring = (unsigned)(ring < 2 ? 2 : ring < each ? ring : each < 2 ? 2 : each);
  if (s.ring > 8) s.ring = 8;
  return s;
}
int list_length(int k) { return k == 0 ? 0 : k <= 4 ? 4 : 8; }

}  // namespace

size_t token_logprob_ws_bytes(size_t M, size_t N, int k) {
  // (K is not known here: the wider layout has more chunks of rows, but may hold one tile a wave where the other has two)
  const int nb = list_length(k);
  const size_t a = shape_of(M, N, 16, nb).most_columns, b = shape_of(M, N, 32, nb).most_columns;
  return M * (a > b ? a : b) * (sizeof(float4) + nb * sizeof(u64));
}

int launch_token_logprob(const void* packedA, const void* packedW, size_t M, size_t N, size_t K, const float* sA,
                         const float* sW, const int32_t* target, int k, float* logprob, float* entropy, int32_t* tok,
                         float* alt, void* ws, hipStream_t s) {
  const unsigned kf = (unsigned)PackedDims(8, N, K).kfrags;
  const Shape sh = shape_of(M, N, kf, list_length(k));
  LogprobParams p{static_cast<const uint8_t*>(packedA), static_cast<const uint8_t*>(packedW), (unsigned)M, (unsigned)N,
                  kf, sh.columns, sh.row_waves, sh.ring, static_cast<float4*>(ws),
                  reinterpret_cast<u64*>(static_cast<float4*>(ws) + M * sh.columns), sA, sW, target, k, logprob, entropy, alt, tok};
  if (!launchable((size_t)sh.columns * sh.chunks, sh.row_waves * sh.word_waves * kWave) || !launchable((M + 3) / 4, 256))
    return MQ_ERR_SHAPE;
  auto go = [&](auto kfc, auto ctc, auto nbc) {
    constexpr int NB = decltype(nbc)::value;
    auto kern = k_logprob_stream<decltype(kfc)::value, decltype(ctc)::value, NB>;
    const unsigned waves = sh.row_waves * sh.word_waves;
    const size_t ring = (size_t)sh.ring * sh.word_waves * kf * kFragBytes, join = waves * 32 * (sizeof(float4) + NB * sizeof(u64));
    const size_t lds = sh.word_waves > 1 && join > ring ? join : ring;
    if (lds > 65536) {
      const int e = check_hip(hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                  hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
      if (e != MQ_OK) return e;
    }
    hipLaunchKernelGGL(kern, dim3(sh.columns * sh.chunks), dim3(waves * kWave), lds, s, p);
    const int rc = check_hip(hipGetLastError());
    if (rc != MQ_OK) return rc;
    hipLaunchKernelGGL((k_logprob_join<NB>), dim3((unsigned)((M + 3) / 4)), dim3(256), 0, s, p);
    return check_hip(hipGetLastError());
  };
  constexpr std::integral_constant<int, 1> one;
  constexpr std::integral_constant<int, 2> two;
  auto with_list = [&](auto kfc) {
    switch (list_length(k)) {
      case 0: return go(kfc, one, std::integral_constant<int, 0>{});
      case 4: return go(kfc, one, std::integral_constant<int, 4>{});
      default: return go(kfc, one, std::integral_constant<int, 8>{});
    }
  };
  if (kf > 16) return with_list(std::integral_constant<int, 32>{});
  if (sh.ct == 2) return go(std::integral_constant<int, 16>{}, two, std::integral_constant<int, 0>{});
  return with_list(std::integral_constant<int, 16>{});
}

}  // namespace mq
