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
// No LDS and no exchange between lanes inside the loop but the maximum over four lane groups.  A wave takes every W-th block of
// a sequence; the four waves of a workgroup join in LDS, the workgroups of a split sequence through the workspace.
#include <type_traits>

#include "mq_gemm_common.h"
#include "mq_glue.h"
#include "mq_seq_common.h"

namespace mq {

namespace {

constexpr int kW = 4;                 // waves of a workgroup
constexpr int kRows = 16;             // query rows of a wave

struct CachedParams {
  const int8_t *keys, *values;
  const float* amax;
  const int32_t *table, *lens;
  const void* q;
  void* out;
  float* part;                        // [B][heads][splits][dv + 2]: sums, maximum, total
  size_t ldq, ldo, table_width, blocks;
  unsigned max_len, kv_heads, heads, d, splits;
  float scale2;                       // scale log2(e)
};

// the largest sum of digits 256^i that NP signed bytes hold whatever the lower ones are
template <int NP>
constexpr float kDigits = NP == 2 ? 127.f * 256.f : 127.f * 65536.f;

// digits of n, least significant first, one byte each into byte `at` of w[0 .. NP)
template <int NP>
__device__ __forceinline__ void put_digits(int n, int at, unsigned (&w)[NP]) {
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int low = i + 1 < NP ? (int)(int8_t)n : n;
    w[i] |= ((unsigned)low & 255u) << (8 * at);
    n = (n - low) >> 8;
  }
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
__global__ __launch_bounds__(kW * kWave) void k_cached_attention(const CachedParams p) {
  using T = typename Elem<DT>::T;
  constexpr int NP = DT == MQ_F32 ? 3 : 2;
  constexpr int ND = 4 * DC;          // 16-column pieces of a value row, at most
  __shared__ float sums[kW][kRows][ND * 16 + 1];
  __shared__ float stat[kW][2][kRows];
  const unsigned lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const unsigned col = lane % 16, grp = lane / 16;
  const unsigned split = blockIdx.x % p.splits, kvh = blockIdx.x / p.splits % p.kv_heads;
  const unsigned per = p.heads / p.kv_heads, tiles = (per + kRows - 1) / kRows;
  const unsigned tile = blockIdx.x / (p.splits * p.kv_heads) % tiles, b = blockIdx.x / (p.splits * p.kv_heads * tiles);
  const unsigned rows = min(per - tile * kRows, (unsigned)kRows), head0 = kvh * per + tile * kRows, d = p.d;
  const int len_any = p.lens[b];
  const unsigned len = len_any < 0 ? 0u : min((unsigned)len_any, p.max_len), nblocks = (len + kKvBlock - 1) / kKvBlock;
  const unsigned dk = kv_dk(d), dv = kv_dv(d), nd = dv / 16;
  const int32_t* table = p.table + (size_t)b * p.table_width;

  // the query row of this lane's column, in digits
  v4i qd[DC][NP];
  float qscale;
  {
    const T* src = static_cast<const T*>(p.q) + (size_t)b * p.ldq + (size_t)(head0 + col) * d;
    float x[DC][16], m = 0.f;
    bool bad = false;
#pragma unroll
    for (int c = 0; c < DC; ++c)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const unsigned i = c * 64 + grp * 16 + j;
        x[c][j] = col < rows && i < d ? (float)src[i] : 0.f;
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
        unsigned w[NP] = {};
#pragma unroll
        for (int j = 0; j < 4; ++j) put_digits<NP>(m < INFINITY && fits ? (int)rintf(x[c][4 * w4 + j] * s) : 0, j, w);
#pragma unroll
        for (int i = 0; i < NP; ++i) qd[c][i][w4] = (int)w[i];
      }
  }

  float acc[ND][4];
  float top = -INFINITY, total = 0.f;
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[t][r] = 0.f;
  for (unsigned pg = split * kW + wave; pg < nblocks; pg += p.splits * kW) {
    const int block = table[pg];
    if (block < 0 || (size_t)block >= p.blocks) continue;
    const size_t at = (size_t)block * p.kv_heads + kvh;
    const int8_t* kp = p.keys + at * kKvBlock * dk + col * dk + grp * 16;
    const int8_t* vp = p.values + at * dv * kKvBlock + lane * 16;
    const float2 am = reinterpret_cast<const float2*>(p.amax)[at];
    u4 vf[ND];
#pragma unroll
    for (int t = 0; t < ND; ++t)
      if (t < (int)nd) {
        // lane l of piece t: row 16 t + l % 16, bytes 16 (l / 16) ..
        vf[t] = *reinterpret_cast<const u4*>(p.values + at * dv * kKvBlock + (size_t)(16 * t + col) * kKvBlock + grp * 16);
      }
    (void)vp;
    float sc[4][4];
    float mt = -INFINITY;
    const float f = qscale * (am.x * (1.f / 127.f));
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      v4i a[NP] = {};
#pragma unroll
      for (int c = 0; c < DC; ++c) {
        const u4 kf = *reinterpret_cast<const u4*>(kp + (size_t)t * 16 * dk + c * 64);
#pragma unroll
        for (int i = 0; i < NP; ++i) a[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(as_v4i(kf), qd[c][i], a[i], 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = join_digits<NP>(a, r) * f;
        sc[t][r] = pg * kKvBlock + t * 16 + grp * 4 + r < len ? x : -INFINITY;
        mt = fmaxf(mt, sc[t][r]);
      }
    }
    mt = groups_f(mt, fmax2);
    const float base = finite_or_0(mt);
    float lt = 0.f;
    v4i pd[NP];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      unsigned w[NP] = {};
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float e = __builtin_amdgcn_exp2f(sc[t][r] - base);
        lt += e;
        put_digits<NP>((int)rintf(e * kDigits<NP>), r, w);
      }
#pragma unroll
      for (int i = 0; i < NP; ++i) pd[i][t] = (int)w[i];
    }
    const float now = fmaxf(top, mt), keep = __builtin_amdgcn_exp2f(top - finite_or_0(now)),
                in = __builtin_amdgcn_exp2f(mt - finite_or_0(now));
    total = fmaf(total, keep, lt * in);
    top = now;
    const float fv = in * (am.y * (1.f / (127.f * kDigits<NP>)));
#pragma unroll
    for (int t = 0; t < ND; ++t)
      if (t < (int)nd) {
        v4i a[NP] = {};
#pragma unroll
        for (int i = 0; i < NP; ++i) a[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(as_v4i(vf[t]), pd[i], a[i], 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[t][r] = fmaf(acc[t][r], keep, join_digits<NP>(a, r) * fv);
      }
  }
  total = groups_f(total, fadd2);

  // the four waves
#pragma unroll
  for (int t = 0; t < ND; ++t)
    if (t < (int)nd)
#pragma unroll
      for (int r = 0; r < 4; ++r) sums[wave][col][16 * t + 4 * grp + r] = acc[t][r];
  if (grp == 0) {
    stat[wave][0][col] = top;
    stat[wave][1][col] = total;
  }
  __syncthreads();
  for (unsigned i = threadIdx.x; i < rows * dv; i += kW * kWave) {
    const unsigned r = i / dv, c = i % dv;
    float m = -INFINITY, l = 0.f, x = 0.f;
#pragma unroll
    for (int w = 0; w < kW; ++w) m = fmaxf(m, stat[w][0][r]);
    const float base = finite_or_0(m);
#pragma unroll
    for (int w = 0; w < kW; ++w) {
      const float e = __builtin_amdgcn_exp2f(stat[w][0][r] - base);
      l = fmaf(e, stat[w][1][r], l);
      x = fmaf(e, sums[w][r][c], x);
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

// The parts of a split sequence: a workgroup per (sequence, head), a thread per column.
template <int DT>
__global__ __launch_bounds__(256) void k_cached_join(const CachedParams p) {
  using T = typename Elem<DT>::T;
  const unsigned dv = kv_dv(p.d), c = threadIdx.x, b = blockIdx.x / p.heads, h = blockIdx.x % p.heads;
  if (c >= p.d) return;
  const float* part = p.part + (size_t)blockIdx.x * p.splits * (dv + 2);
  float m = -INFINITY, l = 0.f, x = 0.f;
  for (unsigned s = 0; s < p.splits; ++s) m = fmaxf(m, part[s * (dv + 2) + dv]);
  const float base = finite_or_0(m);
  for (unsigned s = 0; s < p.splits; ++s) {
    const float e = __builtin_amdgcn_exp2f(part[s * (dv + 2) + dv] - base);
    l = fmaf(e, part[s * (dv + 2) + dv + 1], l);
    x = fmaf(e, part[s * (dv + 2) + c], x);
  }
  static_cast<T*>(p.out)[(size_t)b * p.ldo + (size_t)h * p.d + c] = (T)(l == 0.f ? 0.f : __fdiv_rn(x, l));
}

// Workgroups that share a sequence: as many as it takes to give every compute unit two, while each wave still has a block.
unsigned splits_of(size_t B, size_t max_len, int heads, int kv_heads) {
  const size_t per = (size_t)(heads / kv_heads), wgs = B * (size_t)kv_heads * ((per + kRows - 1) / kRows);
  const size_t want = (512 + wgs - 1) / wgs, most = (max_len + kW * kKvBlock - 1) / (kW * kKvBlock);
  return (unsigned)(want < most ? want : most);
}

}  // namespace

size_t cached_attention_ws_bytes(size_t B, size_t max_len, int heads, int kv_heads, size_t d) {
  const unsigned splits = splits_of(B, max_len, heads, kv_heads);
  return splits == 1 ? 16 : B * (size_t)heads * splits * (kv_dv((unsigned)d) + 2) * sizeof(float);
}

int launch_cached_attention(const mq_kv_cache& cache, const int32_t* table, size_t table_width, const int32_t* lens, size_t B,
                            size_t max_len, const void* q, size_t ldq, int heads, int dtype, float scale, void* out,
                            size_t ldo, void* ws, hipStream_t s) {
  const unsigned splits = splits_of(B, max_len, heads, cache.kv_heads);
  const size_t per = (size_t)(heads / cache.kv_heads);
  const size_t wgs = B * (size_t)cache.kv_heads * ((per + kRows - 1) / kRows) * splits;
  if (wgs >= (size_t)1 << 31 || B * (size_t)heads >= (size_t)1 << 31) return MQ_ERR_SHAPE;
  const CachedParams p{cache.keys, cache.values, cache.amax, table, lens, q, out, static_cast<float*>(ws), ldq, ldo,
                       table_width, cache.blocks, (unsigned)max_len, (unsigned)cache.kv_heads, (unsigned)heads,
                       (unsigned)cache.head_dim, splits, scale * 1.44269504088896340736f};
  return with_dtype(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(kW * kWave), 0, s, p); };
    switch (kv_dk(p.d) / 64) {
      case 1: go(k_cached_attention<DT, 1>); break;
      case 2: go(k_cached_attention<DT, 2>); break;
      case 3: go(k_cached_attention<DT, 3>); break;
      default: go(k_cached_attention<DT, 4>); break;
    }
    int rc = check_hip(hipGetLastError());
    if (rc != MQ_OK || splits == 1) return rc;
    hipLaunchKernelGGL((k_cached_join<DT>), dim3((unsigned)(B * (size_t)heads)), dim3(256), 0, s, p);
    return check_hip(hipGetLastError());
  });
}

}  // namespace mq
