// New keys and values into the paged 8-bit cache of include/mq_seq.h, with the position rotation on the way.
//
// A block of 64 tokens has one scale per head, so whoever writes to it has to see every new token of it first: one workgroup per
// (block touched, kv head).  It forms the rotated keys and the values in LDS, agrees on the two maxima, and writes -- the
// whole block where it starts anew or a maximum grew (what it holds is then requantized), else only the places of the new
// tokens.  Nobody else writes to the block, so there is nothing to wait for and no atomic.  Queries are rotated by workgroups
// behind those, a wave per token.
// Bound by bytes for prompts and by the chain of dependent loads (sequence, table, amax) for single tokens.
#include <type_traits>

#include "mq_glue.h"
#include "mq_seq_common.h"

namespace mq {

namespace {

constexpr int kT = 256;
constexpr int kTokensPerWg = kT / kWave;      // of the query rotation

struct AppendParams {
  const void *k, *v, *q;
  const int32_t *table, *first, *held;
  const float* freq;
  size_t ldk, ldv, ldq, table_width, blocks;
  int8_t *keys, *values;
  float* amax;
  void *k_out, *q_out;
  unsigned B, T, kv_heads, heads, d, rot, page_wgs;
  int interleaved;
};

// sin and cos in binary64 of an angle up to 2^31: the nearest multiple of pi/2 is taken off in two pieces (Cody and Waite),
// the rest, at most pi/4, goes into the Taylor series, whose first terms left out are below 1e-16.
struct SinCos {
  double sin, cos;
};
__device__ __forceinline__ SinCos sincos_f64(double a) {
  const double n = rint(a * 0.63661977236758134308);
  const double r = fma(-n, 6.123233995736766036e-17, fma(-n, 1.57079632679489661923, a)), z = r * r;
  double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;       // 1 / 15!, 1 / 16!
  s = fma(s, z, 1.0 / 6227020800.0);
  s = fma(s, z, -1.0 / 39916800.0);
  s = fma(s, z, 1.0 / 362880.0);
  s = fma(s, z, -1.0 / 5040.0);
  s = fma(s, z, 1.0 / 120.0);
  s = fma(s, z, -1.0 / 6.0);
  s = fma(s * z, r, r);
  c = fma(c, z, -1.0 / 87178291200.0);
  c = fma(c, z, 1.0 / 479001600.0);
  c = fma(c, z, -1.0 / 3628800.0);
  c = fma(c, z, 1.0 / 40320.0);
  c = fma(c, z, -1.0 / 720.0);
  c = fma(c, z, 1.0 / 24.0);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const int quarter = (int)((long long)n & 3);
  const double x = quarter & 1 ? c : s, y = quarter & 1 ? s : c;
  return {quarter & 2 ? -x : x, quarter == 1 || quarter == 2 ? -y : y};
}
__device__ __forceinline__ void rotate(float& x, float& y, const SinCos& w) {
  const double u = x, v = y;
  x = (float)(u * w.cos - v * w.sin);
  y = (float)(v * w.cos + u * w.sin);
}

__device__ __forceinline__ float finite_abs(float x) {
  const float m = fabsf(x);
  return m <= 3.402823466e38f ? m : 0.f;         // NaN and infinities do not count
}
// quant_int of one value, as a byte
__device__ __forceinline__ unsigned quant8(float x, float s) {
  const float y = rintf(x * s);
  return (unsigned)(int)(y != y ? 0.f : fminf(fmaxf(y, -127.f), 127.f)) & 255u;
}
__device__ __forceinline__ unsigned requant8(unsigned byte, float ratio) { return quant8((float)(int8_t)byte, ratio); }

static_assert(kKvBlock == 64, "positions are shifted by 6");

template <int DT>
__device__ void rotate_queries(const AppendParams& p, unsigned wg) {
  using T = typename Elem<DT>::T;
  const unsigned lane = threadIdx.x % kWave, t = wg * kTokensPerWg + threadIdx.x / kWave;
  if (t >= p.T) return;
  int b = (int)t;
  unsigned f0 = t;
  if (p.first != nullptr) {
    b = wave_search(p.B + 1, t, [&](unsigned i) { return first_at(p.first, i, p.T); });
    if (b < 0 || b >= (int)p.B) return;            // a row that belongs to no sequence
    f0 = first_at(p.first, b, p.T);
  }
  const double pos = (double)((long long)p.held[b] + (long long)(t - f0));
  const unsigned half = p.rot / 2;
  constexpr int kMaxPairs = 256 / 2 / kWave;
  SinCos w[kMaxPairs];
#pragma unroll
  for (int j = 0; j < kMaxPairs; ++j)
    if (lane + j * kWave < half) w[j] = sincos_f64(pos * (double)p.freq[lane + j * kWave]);
  const T* src = static_cast<const T*>(p.q) + (size_t)t * p.ldq;
  T* dst = static_cast<T*>(p.q_out) + (size_t)t * p.heads * p.d;
  for (unsigned h = 0; h < p.heads; ++h) {
    const unsigned at = h * p.d;
#pragma unroll
    for (int j = 0; j < kMaxPairs; ++j) {
      const unsigned i = lane + j * kWave;
      if (i < half) {
        const unsigned one = at + (p.interleaved ? 2 * i : i), two = at + (p.interleaved ? 2 * i + 1 : i + half);
        float x = (float)src[one], y = (float)src[two];
        rotate(x, y, w[j]);
        dst[one] = (T)x;
        dst[two] = (T)y;
      }
    }
    for (unsigned i = p.rot + lane; i < p.d; i += kWave) dst[at + i] = src[at + i];
  }
}

template <int DT>
__global__ __launch_bounds__(kT) void k_kv_append(const AppendParams p) {
  using T = typename Elem<DT>::T;
  extern __shared__ float lds[];
  __shared__ float red[2][kT / kWave];
  if (blockIdx.x >= p.page_wgs) return rotate_queries<DT>(p, blockIdx.x - p.page_wgs);
  const unsigned slot = blockIdx.x / p.kv_heads, h = blockIdx.x % p.kv_heads, tid = threadIdx.x;
  int b = (int)slot;
  unsigned f0 = slot, n = 1, local = 0;
  if (p.first != nullptr) {
    // sequence b touches at most n / 64 + 2 blocks; its slots start at first[b] / 64 + 2 b
    auto base = [&](unsigned i) { return first_at(p.first, i, p.T) / kKvBlock + 2 * i; };
    b = wave_search(p.B, slot, base);
    if (b < 0) return;
    f0 = first_at(p.first, b, p.T);
    const unsigned f1 = first_at(p.first, b + 1, p.T);
    n = f1 > f0 ? f1 - f0 : 0;
    local = slot - (f0 / kKvBlock + 2 * (unsigned)b);
  }
  const long long held = p.held[b];
  // positions [t0, t1) of this block that are new; blocks count from the one the first new token falls into
  const long long page = (held >> 6) + local;
  const long long p0 = page * kKvBlock;
  const long long t0 = held > p0 ? held : p0, t1 = held + n < p0 + kKvBlock ? held + n : p0 + kKvBlock;
  if (t0 >= t1) return;
  const unsigned nt = (unsigned)(t1 - t0), row0 = f0 + (unsigned)(t0 - held), d = p.d, pitch = d + 1;
  int block = -1;
  if (page >= 0 && page < (long long)p.table_width) block = p.table[(size_t)b * p.table_width + page];
  const bool cached = block >= 0 && (size_t)block < p.blocks;
  const size_t at = (size_t)(cached ? block : 0) * p.kv_heads + h;
  const float2 had = reinterpret_cast<const float2*>(p.amax)[at];

  float* sk = lds;
  float* sv = lds + (size_t)nt * pitch;
  const T* kin = static_cast<const T*>(p.k) + (size_t)row0 * p.ldk + (size_t)h * d;
  const T* vin = static_cast<const T*>(p.v) + (size_t)row0 * p.ldv + (size_t)h * d;
  T* kout = p.k_out == nullptr ? nullptr : static_cast<T*>(p.k_out) + ((size_t)row0 * p.kv_heads + h) * d;
  const size_t ko = (size_t)p.kv_heads * d;
  float mk = 0.f, mv = 0.f;
  auto key = [&](unsigned t, unsigned i, float x) {
    sk[t * pitch + i] = x;
    mk = fmaxf(mk, finite_abs(x));
    if (kout != nullptr) kout[t * ko + i] = (T)x;
  };
  const unsigned half = p.rot / 2;
  for (unsigned i = tid; i < nt * half; i += kT) {
    const unsigned t = i / half, j = i % half;
    const unsigned one = p.interleaved ? 2 * j : j, two = p.interleaved ? 2 * j + 1 : j + half;
    float x = (float)kin[t * p.ldk + one], y = (float)kin[t * p.ldk + two];
    rotate(x, y, sincos_f64((double)(t0 + t) * (double)p.freq[j]));
    key(t, one, x);
    key(t, two, y);
  }
  const unsigned rest = d - p.rot;
  for (unsigned i = tid; i < nt * rest; i += kT) key(i / rest, p.rot + i % rest, (float)kin[i / rest * p.ldk + p.rot + i % rest]);
  for (unsigned i = tid; i < nt * d; i += kT) {
    const float x = (float)vin[i / d * p.ldv + i % d];
    sv[i / d * pitch + i % d] = x;
    mv = fmaxf(mv, finite_abs(x));
  }
  mk = wave_max_f(mk);
  mv = wave_max_f(mv);
  if (tid % kWave == 0) {
    red[0][tid / kWave] = mk;
    red[1][tid / kWave] = mv;
  }
  __syncthreads();
  if (!cached) return;
#pragma unroll
  for (int w = 0; w < kT / kWave; ++w) {
    mk = fmaxf(mk, red[0][w]);
    mv = fmaxf(mv, red[1][w]);
  }
  const unsigned lo = (unsigned)(t0 - p0), hi = lo + nt;
  const bool fresh = lo == 0;
  if (!fresh) {
    mk = fmaxf(mk, had.x);
    mv = fmaxf(mv, had.y);
  }
  if (tid == 0) reinterpret_cast<float2*>(p.amax)[at] = make_float2(mk, mv);
  auto mult = [](float a) { return a > 0.f ? __fdiv_rn(127.f, a) : 1.f; };
  const float ck = mult(mk), cv = mult(mv);
  const bool all_k = fresh || mk > had.x, all_v = fresh || mv > had.y;
  const float rk = mk > had.x ? __fdiv_rn(had.x, mk) : 1.f, rv = mv > had.y ? __fdiv_rn(had.y, mv) : 1.f;
  // four neighbouring bytes: new ones from LDS, others as they were (0 in a block that starts anew)
  auto merge = [&](unsigned* word, bool any_old, float ratio, auto is_new, auto fresh_byte) {
    const unsigned was = any_old && !fresh ? *word : 0u;
    unsigned w = 0;
#pragma unroll
    for (unsigned c = 0; c < 4; ++c)
      w |= (is_new(c) ? fresh_byte(c) : requant8(was >> (8 * c), ratio)) << (8 * c);
    *word = w;
  };
  const unsigned dk4 = kv_dk(d) / 4, dv = kv_dv(d);
  unsigned* kw = reinterpret_cast<unsigned*>(p.keys) + at * kKvBlock * dk4;
  unsigned* vw = reinterpret_cast<unsigned*>(p.values) + at * dv * (kKvBlock / 4);
  const unsigned ka = all_k ? 0 : lo, kb = all_k ? (unsigned)kKvBlock : hi;
  for (unsigned i = tid; i < (kb - ka) * dk4; i += kT) {
    const unsigned t = ka + i / dk4, c0 = i % dk4 * 4;
    const bool is_new = t >= lo && t < hi;
    merge(kw + t * dk4 + i % dk4, !is_new, rk, [&](unsigned) { return is_new; },
          [&](unsigned c) { return c0 + c < d ? quant8(sk[(t - lo) * pitch + c0 + c], ck) : 0u; });
  }
  const unsigned va = all_v ? 0 : lo / 4, vb = all_v ? 16 : (hi + 3) / 4;      // groups of four tokens
  for (unsigned i = tid; i < (vb - va) * dv; i += kT) {
    const unsigned row = i / (vb - va), g = va + i % (vb - va);
    merge(vw + row * (kKvBlock / 4) + kv_place(4 * g) / 4, 4 * g < lo || 4 * g + 4 > hi, rv,
          [&](unsigned c) { return 4 * g + c >= lo && 4 * g + c < hi; },
          [&](unsigned c) { return row < d ? quant8(sv[(4 * g + c - lo) * pitch + row], cv) : 0u; });
  }
}

}  // namespace

int launch_kv_append(const mq_kv_cache& cache, const int32_t* table, size_t table_width, const int32_t* first,
                     const int32_t* held, size_t B, size_t T, const void* k, size_t ldk, const void* v, size_t ldv,
                     const void* q, size_t ldq, int heads, int dtype, const float* freq, size_t rot, int interleaved,
                     void* k_out, void* q_out, hipStream_t s) {
  const size_t slots = first == nullptr ? B : T / kKvBlock + 2 * B;
  const size_t page_wgs = slots * (size_t)cache.kv_heads;
  const size_t q_wgs = q == nullptr ? 0 : (T + kTokensPerWg - 1) / kTokensPerWg;
  if (page_wgs + q_wgs >= (size_t)1 << 31) return MQ_ERR_SHAPE;
  AppendParams p{k, v, q, table, first, held, freq, ldk, ldv, ldq, table_width, cache.blocks, cache.keys, cache.values,
                 cache.amax, k_out, q_out, (unsigned)B, (unsigned)T, (unsigned)cache.kv_heads, (unsigned)heads,
                 (unsigned)cache.head_dim, (unsigned)rot, (unsigned)page_wgs, interleaved};
  const size_t tokens = first == nullptr ? 1 : T < (size_t)kKvBlock ? T : (size_t)kKvBlock;      // of one block, at most
  const size_t lds = 2 * tokens * (cache.head_dim + 1) * sizeof(float);
  return with_dtype(dtype, [&](auto dt) {
    auto kern = k_kv_append<decltype(dt)::value>;
    if (lds > 65536) {
      const int rc = check_hip(hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
      if (rc != MQ_OK) return rc;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)(page_wgs + q_wgs)), dim3(kT), lds, s, p);
    return check_hip(hipGetLastError());
  });
}

}  // namespace mq
