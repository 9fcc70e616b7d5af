// Attention of several new tokens per sequence over a paged 8-bit cache (include/mq_serve.h): out_i = sum_t p_t V[t] with
// p = softmax_{t <= len - n + i}(scale q_i . K[t]).
//
// One pass over the cache with the running maximum and sum of each query.  The queries of a sequence that share a kv head, n
// tokens x the heads of the group, are rows of one product: S^T = K q^T on v_mfma_f32_32x32x16_bf16, 32 tokens of K as operand
// a, 32 query rows as operand b.  Lane l then has, for row l % 32, the scores of tokens 8 (r / 4) + 4 (l / 32) + r % 4 of 32, and
// the cache keeps the values of a block in an order (kv_place) in which these lanes' probabilities are operand b of out^T = V^T p^T
// as they are.  The cache's integers are bfloat16 values exactly (8 bits); queries and probabilities enter as one, two or three
// bfloat16 parts.  Scales: a block's for the keys goes into the scores' factor, a block's for the values into the probabilities,
// so sums stay in the accumulators from block to block.
#include <type_traits>

#include "mq_glue.h"
#include "mq_serve_common.h"

namespace mq {

namespace {

constexpr int kRows = 32;             // query rows of a tile
constexpr int kWaves = 4;             // of a workgroup, at most

struct ChunkParams {
  const int8_t *keys, *values;
  const float* amax;
  const int32_t *table, *first, *lens;
  const void* q;
  void* out;
  float* part;                        // [T][heads][splits][dv + 2]: sums, maximum, total; splits runs of `run` blocks
  size_t ldq, ldo, table_width, blocks;
  unsigned B, T, max_len, kv_heads, heads, d, splits, run;
  float scale2;                       // scale log2(e)
  int causal;
};

__device__ __forceinline__ float finite_or_0(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float fmax2(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float fadd2(float a, float b) { return a + b; }

// A tile of query rows: row i of its sequence's n x per is token i / per, head i % per of the group.
struct Tile {
  int b;                              // sequence, -1: no such tile
  unsigned first, n, row0, rows, len; // its first token row and new tokens, the tile's first row and rows, tokens in the cache
};
// Tiles of sequence b lie from tile number first[b] per / 32 + b on: enough for each, whatever the lengths.
__device__ __forceinline__ Tile find_tile(const ChunkParams& p, unsigned slot, unsigned per) {
  auto start = [&](unsigned i) { return first_at(p.first, i, p.T) * per / kRows + i; };
  const int b = __builtin_amdgcn_readfirstlane(wave_search(p.B, slot, start));
  if (b < 0) return {-1, 0, 0, 0, 0, 0};
  const unsigned f = first_at(p.first, b, p.T), e = first_at(p.first, b + 1, p.T), n = e > f ? e - f : 0;
  const unsigned row0 = (slot - start(b)) * kRows;
  if (row0 >= n * per) return {-1, 0, 0, 0, 0, 0};
  const int len = p.lens[b];
  return {b, f, n, row0, min(n * per - row0, (unsigned)kRows), len < 0 ? 0u : min((unsigned)len, p.max_len)};
}
// Tokens that query i of n sees.
__device__ __forceinline__ unsigned seen_by(const ChunkParams& p, const Tile& t, unsigned i) {
  if (!p.causal) return t.len;
  const long long s = (long long)t.len - t.n + i + 1;
  return s < 0 ? 0u : (unsigned)s;
}

template <int DT, int DC>             // DC: 64-column pieces of a key
__global__ __launch_bounds__(kWaves * kWave) void k_chunk_attention(const ChunkParams p) {
  using T = typename Elem<DT>::T;
  constexpr int NP = kParts<DT>;
  constexpr int NK = 2 * DC, ND = 2 * DC;      // 32-column pieces of a key, 32-column pieces of a value at most
  extern __shared__ __attribute__((aligned(16))) char smem[];
  bf8* const ql = reinterpret_cast<bf8*>(smem);                                  // [NP][NK][2][64 lanes]
  float* const sums = reinterpret_cast<float*>(smem);                            // [32][ND 32 + 1], afterwards
  __shared__ float fac[kRows], stat[2][kWaves][kRows];
  const unsigned lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  const unsigned col = lane % 32, grp = lane / 32;
  const unsigned split = blockIdx.x % p.splits, kvh = blockIdx.x / p.splits % p.kv_heads, slot = blockIdx.x / (p.splits * p.kv_heads);
  const unsigned per = p.heads / p.kv_heads, d = p.d, dk = kv_dk(d), dv = kv_dv(d);
  const Tile tile = find_tile(p, slot, per);
  if (tile.b < 0) return;
  auto row_at = [&](unsigned r) {              // element offset of row r's queries in q, without the row pitch: token, head
    const unsigned i = tile.row0 + r;
    return make_uint2(tile.first + i / per, kvh * per + i % per);
  };
  const unsigned last = tile.row0 + tile.rows - 1;
  const unsigned most = seen_by(p, tile, last / per), least = seen_by(p, tile, tile.row0 / per);
  const unsigned mine_sees = seen_by(p, tile, min(tile.row0 + col, last) / per);
  const unsigned nblocks = (most + kKvBlock - 1) / kKvBlock;
  const unsigned start = split * p.run, end = min(start + p.run, nblocks);
  if (split > 0 && start >= nblocks) return;   // (the first run answers for rows that see nothing)

  // queries: a power of two off each row, so that its largest element is 1 .. 2, then parts in operand order
  {
    const unsigned r = threadIdx.x / 8 % kRows, j0 = threadIdx.x % 8, step = blockDim.x / 8;
    for (unsigned rr = threadIdx.x / 8; rr < kRows; rr += step) {
      float m = 0.f;
      if (rr < tile.rows) {
        const uint2 at = row_at(rr);
        const T* src = static_cast<const T*>(p.q) + (size_t)at.x * p.ldq + (size_t)at.y * d;
        for (unsigned j = j0; j < d; j += 8) {
          const float x = fabsf((float)src[j]);
          m = x <= 3.402823466e38f ? fmaxf(m, x) : INFINITY;
          if (m == INFINITY) break;
        }
      }
#pragma unroll
      for (int off = 4; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 8));
      if (j0 == 0) fac[rr] = m;
    }
    (void)r;
    __syncthreads();
    for (unsigned u = threadIdx.x; u < NK * 2 * kWave; u += blockDim.x) {
      const unsigned l = u % kWave, c = u / (2 * kWave), s = u / kWave % 2, rr = l % 32, k = 32 * c + 16 * (l / 32) + 8 * s;
      const float m = fac[rr];
      const int e = m > 0.f && m < INFINITY ? max((int)(__float_as_uint(m) >> 23) - 127, -126) : 0;
      const float mul = __uint_as_float((unsigned)(127 - e) << 23);          // 2^-e
      bf8 part[NP];
      const uint2 at = row_at(rr < tile.rows ? rr : 0);
      const T* src = static_cast<const T*>(p.q) + (size_t)at.x * p.ldq + (size_t)at.y * d;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float x = rr < tile.rows && k + j < d ? (float)src[k + j] : 0.f;
        x = m == INFINITY ? NAN : x * mul;                                    // a row with a NaN or an infinity gives NaN
        __bf16 v[NP];
        split_bf16<NP>(x, v);
#pragma unroll
        for (int i = 0; i < NP; ++i) part[i][j] = v[i];
      }
#pragma unroll
      for (int i = 0; i < NP; ++i) ql[(i * NK * 2 + c * 2 + s) * kWave + l] = part[i];
    }
    __syncthreads();
  }
  float qscale;
  {
    const float m = fac[col];
    const int e = m > 0.f && m < INFINITY ? max((int)(__float_as_uint(m) >> 23) - 127, -126) : 0;
    qscale = ldexpf(p.scale2, e);
  }

  float acc_top = -INFINITY, total = 0.f;      // of row l % 32; the total of this lane's tokens
  v16f acc[ND] = {};
  const int32_t* table = p.table + (size_t)tile.b * p.table_width;
  for (unsigned pg = start + wave; pg < end; pg += waves) {
    const int id = pg < p.table_width ? table[pg] : -1;
    const int block = __builtin_amdgcn_readfirstlane(id);
    const bool there = block >= 0 && (size_t)block < p.blocks;
    if (!there) continue;
    const size_t at = (size_t)block * p.kv_heads + kvh;
    const float2 am = reinterpret_cast<const float2*>(p.amax)[at];
    const int8_t* kp = p.keys + at * kKvBlock * dk + (size_t)col * dk + grp * 16;
    const int8_t* vp = p.values + at * dv * kKvBlock + grp * 16;
    u4 kf[2][NK], vf[ND][2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < NK; ++c) kf[t][c] = *reinterpret_cast<const u4*>(kp + (size_t)t * 32 * dk + c * 32);
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) vf[t][h] = *reinterpret_cast<const u4*>(vp + (size_t)min(32 * t + col, dv - 1) * kKvBlock + 32 * h);
    v16f sc[2] = {};
#pragma unroll
    for (int c = 0; c < NK; ++c)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        bf8 a[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) a[t] = bf16_of_bytes(kf[t][c][2 * s], kf[t][c][2 * s + 1]);
#pragma unroll
        for (int i = NP - 1; i >= 0; --i) {
          const bf8 b = ql[(i * NK * 2 + c * 2 + s) * kWave + lane];
#pragma unroll
          for (int t = 0; t < 2; ++t) sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[t], b, sc[t], 0, 0, 0);
        }
      }
    const float f = qscale * (am.x * (1.f / 127.f));
    float mt = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[t][r] *= f;
    if ((pg + 1) * kKvBlock > least)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (pg * kKvBlock + 32 * t + 8 * (r / 4) + 4 * grp + r % 4 >= mine_sees) sc[t][r] = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) mt = fmaxf(mt, sc[t][r]);
    mt = across32_f(mt, fmax2);
    const float now = fmaxf(acc_top, mt), base = finite_or_0(now), keep = __builtin_amdgcn_exp2f(acc_top - base);
    acc_top = now;
    total *= keep;
    if (__any(keep != 1.f))
#pragma unroll
      for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[t][r] *= keep;
    const float fv = am.y * (1.f / 127.f);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bf8 pr[NP];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float e = __builtin_amdgcn_exp2f(sc[j / 2][8 * (j % 2) + k] - base);
        total += e;
        __bf16 v[NP];
        split_bf16<NP>(e * fv, v);
#pragma unroll
        for (int i = 0; i < NP; ++i) pr[i][k] = v[i];
      }
#pragma unroll
      for (int t = 0; t < ND; ++t) {
        const bf8 a = bf16_of_bytes(vf[t][0][j], vf[t][1][j]);
#pragma unroll
        for (int i = NP - 1; i >= 0; --i) acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pr[i], acc[t], 0, 0, 0);
      }
    }
  }
  total = across32_f(total, fadd2);

  // the waves, one after the other
  if (grp == 0) {
    stat[0][wave][col] = acc_top;
    stat[1][wave][col] = total;
  }
  __syncthreads();                             // (and nobody reads queries any more)
  float m = -INFINITY;
  for (unsigned w = 0; w < waves; ++w) m = fmaxf(m, stat[0][w][col]);
  const float weight = __builtin_amdgcn_exp2f(acc_top - finite_or_0(m));
  const unsigned pitch = ND * 32 + 1;
  for (unsigned w = 0; w < waves; ++w) {
    if (w == wave)
#pragma unroll
      for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float& to = sums[col * pitch + 32 * t + 8 * (r / 4) + 4 * grp + r % 4];
          const float x = acc[t][r] * weight;
          to = w == 0 ? x : to + x;
        }
    __syncthreads();
  }
  for (unsigned i = threadIdx.x; i < tile.rows * dv; i += blockDim.x) {
    const unsigned r = i / dv, c = i % dv;
    float mm = -INFINITY, l = 0.f;
    for (unsigned w = 0; w < waves; ++w) mm = fmaxf(mm, stat[0][w][r]);
    for (unsigned w = 0; w < waves; ++w) l = fmaf(__builtin_amdgcn_exp2f(stat[0][w][r] - finite_or_0(mm)), stat[1][w][r], l);
    const float x = sums[r * pitch + c];
    const uint2 at = row_at(r);
    if (p.splits == 1) {
      if (c < d) static_cast<T*>(p.out)[(size_t)at.x * p.ldo + (size_t)at.y * d + c] = (T)(l == 0.f ? 0.f : __fdiv_rn(x, l));
    } else {
      float* to = p.part + (((size_t)at.x * p.heads + at.y) * p.splits + split) * (dv + 2);
      to[c] = x;
      if (c == 0) {
        to[dv] = mm;
        to[dv + 1] = l;
      }
    }
  }
}

// The parts of split sequences: a wave per (token, head).
template <int DT>
__global__ __launch_bounds__(256) void k_chunk_join(const ChunkParams p) {
  using T = typename Elem<DT>::T;
  const unsigned lane = threadIdx.x % kWave, dv = kv_dv(p.d), pitch = dv + 2, per = p.heads / p.kv_heads;
  const unsigned rows = (unsigned)(blockIdx.x * (256 / kWave) + threadIdx.x / kWave), t = rows / p.heads, h = rows % p.heads;
  if (t >= p.T) return;
  const int b = __builtin_amdgcn_readfirstlane(wave_search(p.B, t, [&](unsigned i) { return first_at(p.first, i, p.T); }));
  if (b < 0) return;
  const unsigned f = first_at(p.first, b, p.T), e = first_at(p.first, b + 1, p.T);
  if (t >= e) return;
  // runs of the tile that the row is in
  Tile tile{b, f, e - f, 0, 0, 0};
  const int len = p.lens[b];
  tile.len = len < 0 ? 0u : min((unsigned)len, p.max_len);
  const unsigned row = (t - f) * per + h % per, last = min(row / kRows * kRows + kRows, tile.n * per) - 1;
  const unsigned tokens = p.run * kKvBlock, runs = max(1u, (seen_by(p, tile, last / per) + tokens - 1) / tokens);
  const float* part = p.part + ((size_t)t * p.heads + h) * p.splits * pitch;
  float m = -INFINITY;
  for (unsigned s = 0; s < runs; ++s) m = fmaxf(m, part[s * pitch + dv]);
  const float base = finite_or_0(m);
  float l = 0.f, x[4] = {};
  for (unsigned s = 0; s < runs; ++s) {
    const float w = __builtin_amdgcn_exp2f(part[s * pitch + dv] - base);
    l = fmaf(w, part[s * pitch + dv + 1], l);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (lane + 64 * j < p.d) x[j] = fmaf(w, part[s * pitch + lane + 64 * j], x[j]);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (lane + 64 * j < p.d)
      static_cast<T*>(p.out)[(size_t)t * p.ldo + (size_t)h * p.d + lane + 64 * j] = (T)(l == 0.f ? 0.f : __fdiv_rn(x[j], l));
}

struct Split {
  unsigned run, splits, waves;
  size_t slots;
};
Split split_of(size_t B, size_t T, size_t max_len, int heads, int kv_heads) {
  const size_t per = (size_t)(heads / kv_heads), slots = T * per / kRows + B, wgs = slots * (size_t)kv_heads;
  const size_t blocks = (max_len + kKvBlock - 1) / kKvBlock, want = (512 + wgs - 1) / wgs;
  if (blocks <= 2 * kWaves) return {(unsigned)blocks, 1u, (unsigned)(blocks < kWaves ? blocks : kWaves), slots};
  size_t run = (blocks + want - 1) / want;
  if (run < (size_t)kWaves) run = kWaves;
  return {(unsigned)run, (unsigned)((blocks + run - 1) / run), kWaves, slots};
}

}  // namespace

size_t chunk_attention_ws_bytes(size_t B, size_t T, size_t max_len, int heads, int kv_heads, size_t d) {
  const unsigned splits = split_of(B, T, max_len, heads, kv_heads).splits;
  return splits == 1 ? 16 : T * (size_t)heads * splits * (kv_dv((unsigned)d) + 2) * sizeof(float);
}

int launch_chunk_attention(const mq_kv_cache& cache, const int32_t* table, size_t table_width, const int32_t* first,
                           const int32_t* lens, size_t B, size_t T, size_t max_len, int causal, const void* q, size_t ldq,
                           int heads, int dtype, float scale, void* out, size_t ldo, void* ws, hipStream_t s) {
  const Split split = split_of(B, T, max_len, heads, cache.kv_heads);
  const size_t wgs = split.slots * (size_t)cache.kv_heads * split.splits;
  const size_t joins = (T * (size_t)heads + 3) / 4;
  if (!launchable(wgs, kWaves * kWave) || (split.splits > 1 && !launchable(joins, 256))) return MQ_ERR_SHAPE;
  const ChunkParams p{cache.keys, cache.values, cache.amax, table, first, lens, q, out, static_cast<float*>(ws), ldq, ldo,
                      table_width, cache.blocks, (unsigned)B, (unsigned)T, (unsigned)max_len, (unsigned)cache.kv_heads,
                      (unsigned)heads, (unsigned)cache.head_dim, split.splits, split.run, scale * 1.44269504088896340736f, causal};
  return with_dtype(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    const size_t pieces = kv_dk(p.d) / 64;
    const size_t ql = kParts<DT> * pieces * 4 * kWave * 16, sums = kRows * (pieces * 64 + 1) * sizeof(float);
    const size_t lds = ql > sums ? ql : sums;
    auto go = [&](auto kern) {
      hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(split.waves * kWave), lds, s, p);
      return check_hip(hipGetLastError());
    };
    int rc;
    switch (pieces) {
      case 1: rc = go(k_chunk_attention<DT, 1>); break;
      case 2: rc = go(k_chunk_attention<DT, 2>); break;
      case 3: rc = go(k_chunk_attention<DT, 3>); break;
      default: rc = go(k_chunk_attention<DT, 4>); break;
    }
    if (rc != MQ_OK || split.splits == 1) return rc;
    hipLaunchKernelGGL(k_chunk_join<DT>, dim3((unsigned)joins), dim3(256), 0, s, p);
    return check_hip(hipGetLastError());
  });
}

}  // namespace mq
