// Attention of one query per sequence over a paged 8-bit cache (include/mq_seq.h): out = sum_t p_t V[t] with
// p = softmax_t(scale q . K[t]).
//
// The cache streams through once and everything else is small, so the bound is its bytes; the arithmetic must not get in their
// way.  Both products run on v_mfma_i32_16x16x64_i8 and take the cache's bytes from global memory as they are:
//   * S^T = K q^T: 16 tokens x 64 columns of K are operand a (lane l: token l % 16, 16 neighbouring bytes), the queries
//     of one kv head (up to 16 rows, the heads that share it) operand b.  A query row enters as NP signed bytes per element
//     (digits in base 256 of rint(q scale), scale from the row's largest magnitude): two for 16-bit types, three for binary32.
//   * lane l then holds, for query l % 16, the scores of tokens 16 i + 4 (l / 16) + r -- 16 of the block's 64.  The values of
//     the cache lie in that order (kv_place), so the probabilities are operand b of out^T = V^T p^T without leaving their
//     lane: again NP bytes each, relative to the block's largest probability.  (Relative to the block, not to the running
//     maximum: a long run of small probabilities keeps its bits.)
//   * the sums of a block are exact integers; block scales, the rescaling of the softmax and the digits' weights are one
//     multiply-add per element of the 16 x dv result.
// No LDS and no exchange between lanes inside the loop but the maximum over four lane groups.  The next block's keys are asked for
// as soon as this one's are multiplied, its values likewise; which blocks they are a wave reads 64 at a time.  A workgroup takes
// `run` neighbouring blocks of a sequence, its waves in turn; they join in LDS, the workgroups of a sequence through the
// workspace.  Runs are equally long whatever the sequences' lengths, so that long and short ones keep the chip busy to the end --
// where the longest has several: from 512 workgroups on every sequence is one run, and one far longer than the others is
// waited for (one of 32000 tokens among 63 of 500, 8 kv heads of 128: 214 us for 28 us of bytes; 64 of 2000: 45 us).
// Digits are what 8-bit products take.  Three of a binary32 query are 24 bits of its row's largest element, and of a
// probability 24 of its block's largest; two are 16 bits, more than a 16-bit type has.  Against 64 bits the outputs are as
// far off as with binary32 products: 3.9e-7 (1 sequence of 777, binary32), 1.7e-3 (32 of 4000 .. 32000, bfloat16).
#include <type_traits>

#include "mq_gemm_common.h"
#include "mq_glue.h"
#include "mq_seq_common.h"

namespace mq {

namespace {

constexpr int kW = 4;                 // waves of a workgroup of a split sequence
// waves of a workgroup at most, by what a wave's registers leave room for (DC: 64-column pieces of a key)
constexpr int most_waves(int dc) { return dc == 1 ? 16 : dc == 2 ? 8 : 4; }
constexpr int kRows = 16;             // query rows of a wave

struct CachedParams {
  const int8_t *keys, *values;
  const float* amax;
  const int32_t *table, *lens;
  const void* q;
  void* out;
  float* part;                        // [B][heads][splits][dv + 2]: sums, maximum, total; splits runs of `run` blocks
  size_t ldq, ldo, table_width, blocks;
  unsigned max_len, kv_heads, heads, d, splits, run;
  float scale2;                       // scale log2(e)
  int vec;                            // rows of queries are whole 16-byte pieces
};

// the largest sum of digits 256^i that NP signed bytes hold whatever the lower ones are
template <int NP>
constexpr float kDigits = NP == 2 ? 127.f * 256.f : 127.f * 65536.f;

// Byte i of four words, for i < NP, as the four bytes of w[i].
template <int NP>
__device__ __forceinline__ void gather_bytes(const unsigned (&x)[4], unsigned (&w)[NP]) {
  const unsigned a = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u), b = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u);
  w[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
  w[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  if constexpr (NP == 3)
    w[2] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(x[3], x[2], 0x0C0C0602u), __builtin_amdgcn_perm(x[1], x[0], 0x0C0C0602u), 0x05040100u);
}
// Signed digits of four integers: adding 128 at every place makes the bytes the digits plus 128.
template <int NP>
__device__ __forceinline__ void digits_of(const int (&n)[4], unsigned (&w)[NP]) {
  unsigned x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = (unsigned)n[j] + (NP == 3 ? 0x808080u : 0x8080u);
  gather_bytes<NP>(x, w);
#pragma unroll
  for (int i = 0; i < NP; ++i) w[i] ^= 0x80808080u;
}
// The same of e kDigits, 0 <= e <= 1, rounded: the sum with 2^23 and the 128s has units as its last place, so the multiply-add
// rounds and the bytes of its result are the digits plus 128 (the third, whose 128 is 2^23 itself, is the digit).
template <int NP>
__device__ __forceinline__ void digits_of_share(const float (&e)[4], unsigned (&w)[NP]) {
  unsigned x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = __float_as_uint(fmaf(e[j], kDigits<NP>, NP == 3 ? 8421504.f : 8388608.f + 32896.f));
  gather_bytes<NP>(x, w);
  w[0] ^= 0x80808080u;
  w[1] ^= 0x80808080u;
}
template <int NP>
__device__ __forceinline__ float join_digits(const v4i (&a)[NP], int r) {
  if constexpr (NP == 2) return (float)((a[1][r] << 8) + a[0][r]);
  return fmaf((float)((a[2][r] << 8) + a[1][r]), 256.f, (float)a[0][r]);
}

// over the four groups of 16 lanes
template <typename Op>
__device__ __forceinline__ float groups_f(float v, Op op) {
  return across16_f(across32_f(v, op), op);
}
__device__ __forceinline__ float fmax2(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float fadd2(float a, float b) { return a + b; }
__device__ __forceinline__ float finite_or_0(float m) { return m == -INFINITY ? 0.f : m; }

template <int DT, int DC>             // DC: 64-column pieces of a key
__global__ __launch_bounds__(most_waves(DC) * kWave) void k_cached_attention(const CachedParams p) {
  using T = typename Elem<DT>::T;
  constexpr int NP = DT == MQ_F32 ? 3 : 2;
  constexpr int ND = 4 * DC;          // 16-column pieces of a value row, at most
  extern __shared__ float lds[];      // [waves][rows][ND 16 + 1] sums, [waves][2][rows] maxima and totals
  const unsigned lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  const unsigned col = lane % 16, grp = lane / 16;
  const unsigned split = blockIdx.x % p.splits, kvh = blockIdx.x / p.splits % p.kv_heads;
  const unsigned per = p.heads / p.kv_heads, tiles = (per + kRows - 1) / kRows;
  const unsigned tile = blockIdx.x / (p.splits * p.kv_heads) % tiles, b = blockIdx.x / (p.splits * p.kv_heads * tiles);
  const unsigned rows = min(per - tile * kRows, (unsigned)kRows), head0 = kvh * per + tile * kRows, d = p.d;
  auto sums = [&](unsigned w, unsigned row, unsigned c) -> float& { return lds[(w * rows + row) * (ND * 16 + 1) + c]; };
  auto stat = [&](unsigned w, unsigned i, unsigned row) -> float& { return lds[waves * rows * (ND * 16 + 1) + (w * 2 + i) * rows + row]; };
  const int len_any = p.lens[b];
  const unsigned len = len_any < 0 ? 0u : min((unsigned)len_any, p.max_len), nblocks = (len + kKvBlock - 1) / kKvBlock;
  const unsigned dk = kv_dk(d), dv = kv_dv(d), nd = dv / 16;
  const int32_t* table = p.table + (size_t)b * p.table_width;
  // this workgroup's blocks [start, end), this wave's every waves-th of them
  const unsigned start = split * p.run, end = min(start + p.run, nblocks);
  if (split > 0 && start >= nblocks) return;           // (the first run answers for an empty sequence)
  const unsigned mine = end > start + wave ? __builtin_amdgcn_readfirstlane((end - start - wave + waves - 1) / waves) : 0u;
  auto look = [&](unsigned i) {                        // 64 of the wave's blocks, from its i-th on
    const size_t pg = start + wave + (size_t)(i + lane) * waves;
    return table[pg < p.table_width ? pg : p.table_width - 1];
  };
  int ids = look(0);                                   // (does not wait for the length)

  float acc[ND][4];
  float top = -INFINITY, total = 0.f;
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[t][r] = 0.f;
  u4 kf[4][DC], vf[ND];
  float2 am, am_next;
  bool there, there_next;                              // whether the block is one
  size_t at_next;
  auto find = [&](unsigned i) {                        // the wave's i-th block
    if (i % kWave == 0 && i > 0) ids = look(i);
    const int block = __builtin_amdgcn_readlane(ids, i % kWave);
    there_next = block >= 0 && (size_t)block < p.blocks;
    at_next = (size_t)(there_next ? block : 0) * p.kv_heads + kvh;
  };
  auto bring_keys = [&] {
    const int8_t* kp = p.keys + at_next * kKvBlock * dk + col * dk + grp * 16;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int c = 0; c < DC; ++c) kf[t][c] = *reinterpret_cast<const u4*>(kp + (size_t)t * 16 * dk + c * 64);
    am_next = reinterpret_cast<const float2*>(p.amax)[at_next];
  };
  auto bring_values = [&] {                            // lane l of piece t: row 16 t + l % 16, bytes 16 (l / 16) ..
    const int8_t* vp = p.values + at_next * dv * kKvBlock + col * kKvBlock + grp * 16;
#pragma unroll
    for (int t = 0; t < ND; ++t)
      if (t < (int)nd) vf[t] = *reinterpret_cast<const u4*>(vp + t * 16 * kKvBlock);
  };
  if (mine > 0) {
    find(0);
    bring_keys();
    bring_values();
  }
  // the query row of this lane's column, in digits
  v4i qd[DC][NP];
  float qscale;
  {
    const T* src = static_cast<const T*>(p.q) + (size_t)b * p.ldq + (size_t)(head0 + (col < rows ? col : 0)) * d;
    float x[DC][16], m = 0.f;
    bool bad = false;
    // (loads in front of every choice: a load behind a condition is waited for on its own)
    if (p.vec) {
      constexpr int W = 16 / sizeof(T);
      typedef T tw __attribute__((ext_vector_type(W)));
#pragma unroll
      for (int c = 0; c < DC; ++c)
#pragma unroll
        for (int j = 0; j < 16; j += W) {
          const unsigned i = c * 64 + grp * 16 + j;
          const tw v = *reinterpret_cast<const tw*>(src + (i < d ? i : 0));
#pragma unroll
          for (int k = 0; k < W; ++k) x[c][j + k] = (float)v[k];
        }
    } else {
#pragma unroll
      for (int c = 0; c < DC; ++c)
#pragma unroll
        for (int j = 0; j < 16; ++j) x[c][j] = (float)src[c * 64 + grp * 16 + j < d ? c * 64 + grp * 16 + j : 0];
    }
#pragma unroll
    for (int c = 0; c < DC; ++c)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        if (col >= rows || c * 64 + grp * 16 + j >= d) x[c][j] = 0.f;
        bad |= !(fabsf(x[c][j]) <= 3.402823466e38f);
        m = fmaxf(m, fabsf(x[c][j]));
      }
    m = groups_f(bad ? INFINITY : m, fmax2);
    const float s = m > 0.f ? __fdiv_rn(kDigits<NP>, m) : 0.f;
    const bool fits = s <= 3.402823466e38f;        // (a row below 2^-104: its digits are left 0)
    // a row with a NaN or an infinity gives NaN
    qscale = m == INFINITY ? NAN : fits ? m * (p.scale2 / kDigits<NP>) : 0.f;
#pragma unroll
    for (int c = 0; c < DC; ++c)
#pragma unroll
      for (int w4 = 0; w4 < 4; ++w4) {
        unsigned w[NP];
        int n[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) n[j] = m < INFINITY && fits ? (int)rintf(x[c][4 * w4 + j] * s) : 0;
        digits_of<NP>(n, w);
#pragma unroll
        for (int i = 0; i < NP; ++i) qd[c][i][w4] = (int)w[i];
      }
  }

  for (unsigned i = 0; i < mine; ++i) {
    const unsigned pg = start + wave + i * waves;
    am = am_next;
    there = there_next;
    if (i + 1 < mine) find(i + 1);
    float sc[4][4];
    float mt = -INFINITY;
    const float f = qscale * (am.x * (1.f / 127.f));
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      v4i a[NP] = {};
#pragma unroll
      for (int c = 0; c < DC; ++c) {
#pragma unroll
        for (int j = 0; j < NP; ++j) a[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(as_v4i(kf[t][c]), qd[c][j], a[j], 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        sc[t][r] = join_digits<NP>(a, r) * f;
      }
    }
    if (!there || (pg + 1) * kKvBlock > len)
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (!there || pg * kKvBlock + t * 16 + grp * 4 + r >= len) sc[t][r] = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) mt = fmaxf(mt, sc[t][r]);
    if (i + 1 < mine) bring_keys();
    mt = groups_f(mt, fmax2);
    const float base = finite_or_0(mt);
    float lt = 0.f;
    v4i pd[NP];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      unsigned w[NP];
      float e[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        e[r] = __builtin_amdgcn_exp2f(sc[t][r] - base);
        lt += e[r];
      }
      digits_of_share<NP>(e, w);
#pragma unroll
      for (int j = 0; j < NP; ++j) pd[j][t] = (int)w[j];
    }
    const float now = fmaxf(top, mt), keep = __builtin_amdgcn_exp2f(top - finite_or_0(now)),
                in = __builtin_amdgcn_exp2f(mt - finite_or_0(now));
    total = fmaf(total, keep, lt * in);
    top = now;
    // (where there is no block, block 0 was read, whose maximum may be anything: 0 times that must not get in)
    const float fv = there ? in * (am.y * (1.f / (127.f * kDigits<NP>))) : 0.f;
#pragma unroll
    for (int t = 0; t < ND; ++t)
      if (t < (int)nd) {
        v4i a[NP] = {};
#pragma unroll
        for (int j = 0; j < NP; ++j) a[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(as_v4i(vf[t]), pd[j], a[j], 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[t][r] = fmaf(acc[t][r], keep, join_digits<NP>(a, r) * fv);
      }
    if (i + 1 < mine) bring_values();
  }
  total = groups_f(total, fadd2);

  // the waves
  if (col < rows)
#pragma unroll
    for (int t = 0; t < ND; ++t)
      if (t < (int)nd)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums(wave, col, 16 * t + 4 * grp + r) = acc[t][r];
  if (grp == 0 && col < rows) {
    stat(wave, 0, col) = top;
    stat(wave, 1, col) = total;
  }
  __syncthreads();
  for (unsigned i = threadIdx.x; i < rows * dv; i += blockDim.x) {
    const unsigned r = i / dv, c = i % dv;
    float m = -INFINITY, l = 0.f, x = 0.f;
    for (unsigned w = 0; w < waves; ++w) m = fmaxf(m, stat(w, 0, r));
    const float base = finite_or_0(m);
    for (unsigned w = 0; w < waves; ++w) {
      const float e = __builtin_amdgcn_exp2f(stat(w, 0, r) - base);
      l = fmaf(e, stat(w, 1, r), l);
      x = fmaf(e, sums(w, r, c), x);
    }
    if (p.splits == 1) {
      if (c < d) static_cast<T*>(p.out)[(size_t)b * p.ldo + (size_t)(head0 + r) * d + c] = (T)(l == 0.f ? 0.f : __fdiv_rn(x, l));
    } else {
      float* to = p.part + (((size_t)b * p.heads + head0 + r) * p.splits + split) * (dv + 2);
      to[c] = x;
      if (c == 0) {
        to[dv] = m;
        to[dv + 1] = l;
      }
    }
  }
}

// The parts of a split sequence: a workgroup per (sequence, head).  Few runs: a thread per column.  Many (kMany): every run's
// weight once, then threads per column that take the runs in turn.  Whole calls, few / many, us: 2 runs 38.5 / 39.6 (32 sequences of
// 5000, 8 heads of 64, binary32), 4 runs 29.4 / 28.8 (21), 8 runs 18.8 / 16.0 (8), 82 runs 48.6 / 14.4 (3 of 20753, 2 heads).
constexpr unsigned kMany = 3;
constexpr unsigned kJoin = 512;                // threads, and runs of a sequence, at most
unsigned join_columns(unsigned d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }
template <int DT, bool MANY>
__global__ __launch_bounds__(kJoin) void k_cached_join(const CachedParams p, unsigned columns) {
  using T = typename Elem<DT>::T;
  __shared__ float weight[kJoin], box[kJoin], red[2][kJoin / kWave];
  const unsigned dv = kv_dv(p.d), tid = threadIdx.x, b = blockIdx.x / p.heads, h = blockIdx.x % p.heads, pitch = dv + 2;
  const unsigned threads = blockDim.x, groups = threads / columns, c = tid % columns, g = tid / columns;
  const float* part = p.part + (size_t)blockIdx.x * p.splits * pitch;
  // the runs that the sequence has
  const int len_any = p.lens[b];
  const unsigned len = len_any < 0 ? 0u : min((unsigned)len_any, p.max_len), tokens = p.run * kKvBlock;
  const unsigned runs = max(1u, (len + tokens - 1) / tokens);
  float m = -INFINITY, l = 0.f, x = 0.f;
  const float* mine = part + min(c, p.d - 1);
  T* dst = static_cast<T*>(p.out) + (size_t)b * p.ldo + (size_t)h * p.d + c;
  if constexpr (!MANY) {
    for (unsigned s = 0; s < runs; ++s) m = fmaxf(m, part[s * pitch + dv]);
    const float base = finite_or_0(m);
    for (unsigned s = 0; s < runs; ++s) {
      const float e = __builtin_amdgcn_exp2f(part[s * pitch + dv] - base);
      l = fmaf(e, part[s * pitch + dv + 1], l);
      x = fmaf(e, mine[s * pitch], x);
    }
    if (c < p.d) *dst = (T)(l == 0.f ? 0.f : __fdiv_rn(x, l));
    return;
  }
  for (unsigned s = tid; s < runs; s += threads) m = fmaxf(m, part[s * pitch + dv]);
  m = wave_max_f(m);
  if (tid % kWave == 0) red[0][tid / kWave] = m;
  __syncthreads();
  for (unsigned w = 0; w < threads / kWave; ++w) m = fmaxf(m, red[0][w]);
  const float base = finite_or_0(m);
  for (unsigned s = tid; s < runs; s += threads) {
    const float e = __builtin_amdgcn_exp2f(part[s * pitch + dv] - base);
    weight[s] = e;
    l = fmaf(e, part[s * pitch + dv + 1], l);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) l += __shfl_xor(l, off, 64);
  if (tid % kWave == 0) red[1][tid / kWave] = l;
  __syncthreads();
  l = 0.f;
  for (unsigned w = 0; w < threads / kWave; ++w) l += red[1][w];
#pragma unroll 8
  for (unsigned s = g; s < runs; s += groups) x = fmaf(weight[s], mine[s * pitch], x);
  box[tid] = x;
  __syncthreads();
  if (g > 0) return;
  for (unsigned i = 1; i < groups; ++i) x += box[i * columns + c];
  if (c < p.d) *dst = (T)(l == 0.f ? 0.f : __fdiv_rn(x, l));
}

// Blocks to a run, runs of the longest sequence, waves of a workgroup.  As many runs as fill the chip's 512 places for
// workgroups once where all sequences are as long as they may be, while a wave still has a block: 32 sequences of 4000 .. 32000
// tokens, 8 kv heads of 128, take 209 us with that many, 224 with twice as many and 247 with four times (a workgroup's start and
// end), 311 with half.  One wave where two blocks are all there is.
constexpr size_t kFull = 1024;
struct Split {
  unsigned run, splits, waves;
};
Split split_of(size_t B, size_t max_len, int heads, int kv_heads, size_t d) {
  const size_t per = (size_t)(heads / kv_heads), wgs = B * (size_t)kv_heads * ((per + kRows - 1) / kRows);
  const size_t blocks = (max_len + kKvBlock - 1) / kKvBlock, want = (512 + wgs - 1) / wgs;
  // one workgroup for a sequence of few blocks: no second launch.  As many waves as there are blocks while the chip has room
  const size_t rows = per < (size_t)kRows ? per : kRows, dc = kv_dk((unsigned)d) / 64;
  size_t waves = most_waves((int)dc);
  while (waves > 1 && waves * rows * (dc * 64 + 3) * sizeof(float) > 65536) waves /= 2;
  if (blocks <= 2 * waves) {
    const size_t room = wgs >= kFull ? (blocks + 1) / 2 : blocks;
    return {(unsigned)blocks, 1u, (unsigned)(room < waves ? room : waves)};
  }
  size_t run = (blocks + want - 1) / want;
  if (run < (size_t)kW) run = kW;
  waves = waves < (size_t)kW ? waves : kW;
  return {(unsigned)run, (unsigned)((blocks + run - 1) / run), (unsigned)waves};
}

}  // namespace

size_t cached_attention_ws_bytes(size_t B, size_t max_len, int heads, int kv_heads, size_t d) {
  const unsigned splits = split_of(B, max_len, heads, kv_heads, d).splits;
  return splits == 1 ? 16 : B * (size_t)heads * splits * (kv_dv((unsigned)d) + 2) * sizeof(float);
}

int launch_cached_attention(const mq_kv_cache& cache, const int32_t* table, size_t table_width, const int32_t* lens, size_t B,
                            size_t max_len, const void* q, size_t ldq, int heads, int dtype, float scale, void* out,
                            size_t ldo, void* ws, hipStream_t s) {
  const Split split = split_of(B, max_len, heads, cache.kv_heads, cache.head_dim);
  const unsigned splits = split.splits;
  const size_t per = (size_t)(heads / cache.kv_heads);
  const size_t wgs = B * (size_t)cache.kv_heads * ((per + kRows - 1) / kRows) * splits;
  if (!launchable(wgs, split.waves * kWave) || (splits > 1 && !launchable(B * (size_t)heads, kJoin))) return MQ_ERR_SHAPE;
  const size_t piece = 16 / elem_bytes(dtype);
  const int vec = cache.head_dim % piece == 0 && ldq % piece == 0 && reinterpret_cast<uintptr_t>(q) % 16 == 0;
  const CachedParams p{cache.keys, cache.values, cache.amax, table, lens, q, out, static_cast<float*>(ws), ldq, ldo,
                       table_width, cache.blocks, (unsigned)max_len, (unsigned)cache.kv_heads, (unsigned)heads,
                       (unsigned)cache.head_dim, splits, split.run, scale * 1.44269504088896340736f, vec};
  return with_dtype(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    const unsigned pieces = kv_dk(p.d) / 64;
    const size_t lds = split.waves * (per < (size_t)kRows ? per : kRows) * (pieces * 64 + 1 + 2) * sizeof(float);
    int rc = MQ_OK;
    auto go = [&](auto kern) {
      if (lds > 65536)
        rc = check_hip(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
      if (rc == MQ_OK) hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(split.waves * kWave), lds, s, p);
    };
    switch (pieces) {
      case 1: go(k_cached_attention<DT, 1>); break;
      case 2: go(k_cached_attention<DT, 2>); break;
      case 3: go(k_cached_attention<DT, 3>); break;
      default: go(k_cached_attention<DT, 4>); break;
    }
    if (rc == MQ_OK) rc = check_hip(hipGetLastError());
    if (rc != MQ_OK || splits == 1) return rc;
    const unsigned columns = join_columns(p.d);
    if (splits >= kMany)
      hipLaunchKernelGGL((k_cached_join<DT, true>), dim3((unsigned)(B * (size_t)heads)), dim3(kJoin), 0, s, p, columns);
    else
      hipLaunchKernelGGL((k_cached_join<DT, false>), dim3((unsigned)(B * (size_t)heads)), dim3(columns), 0, s, p, columns);
    return check_hip(hipGetLastError());
  });
}

}  // namespace mq
