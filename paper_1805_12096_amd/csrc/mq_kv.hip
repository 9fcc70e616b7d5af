// New keys and values into the paged 8-bit cache of include/mq_seq.h, with the position rotation on the way.
//
// A block of 64 tokens has one scale per head, so whoever writes to it has to see every new token of it first: one workgroup per
// (block touched, kv head).  It forms the rotated keys and the values in LDS, agrees on the two maxima, and writes -- the
// whole block where it starts anew or a maximum grew (what it holds is then requantized), else only the places of the new
// tokens.  Nobody else writes to the block, so there is nothing to wait for and no atomic.  Queries are rotated by workgroups
// behind those, a wave per token.
// Bound by bytes for prompts (449 MB in 128 us, 3.5 TB/s; element by element 508) and by the chain of dependent loads (sequence,
// table, amax) for single tokens (64 sequences, 32 heads of 128 over 8: 7 us; element by element 16).  Where the maximum of every
// block grows and all of it is requantized, single tokens take 13 us instead of 6 (the same) and 15 instead of 7 (300 sequences,
// 8 heads of 64, binary32).
//
// Rows of whole 16-byte pieces (k_kv_append_rows): what a workgroup rotates and quantizes stays in registers between the two
// maxima and the stores.  A thread has 16 elements of a key, the two groups of 8 that are rotated together, and for the values
// 4 tokens x 2 columns, whose bytes are one word of a row of the cache each.  256 threads take a block at once; where a call
// brings few tokens to a block, 64 threads take 8 (4 for wide heads) at a time, sines and cosines formed by all of them in LDS.
// Vector instructions take half of the clocks in which a prompt's compute units are busy, and 184 registers leave two waves a SIMD.
// Other rows, and rotations that are not a multiple of 16 elements: k_kv_append, element by element (12 prompts of 2000, 32 heads
// of 80 over 8, bfloat16: 380 us with 40 elements rotated, 150 with 80).
#include <type_traits>

#include "mq_glue.h"
#include "mq_seq_common.h"

namespace mq {

namespace {

constexpr int kT = 256;
constexpr int kTokensPerWg = kT / kWave;      // of the query rotation
// pieces of 16 elements of a token's queries, a wave at a time (about 250 tokens of 128 heads of 256: 27 us, a wave per token 124)
constexpr int kQPieces = 256;

struct AppendParams {
  const void *k, *v, *q;
  const int32_t *table, *first, *held;
  const float* freq;
  size_t ldk, ldv, ldq, table_width, blocks;
  int8_t *keys, *values;
  float* amax;
  void *k_out, *q_out;
  unsigned B, T, kv_heads, heads, d, rot, page_wgs;
  unsigned slot_tokens, slot_more;      // sequence b's slots start at first[b] / slot_tokens + slot_more b
  unsigned q_parts;                     // waves of a token of queries
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
    auto base = [&](unsigned i) { return first_at(p.first, i, p.T) / p.slot_tokens + p.slot_more * i; };
    b = wave_search(p.B, slot, base);
    if (b < 0) return;
    f0 = first_at(p.first, b, p.T);
    const unsigned f1 = first_at(p.first, b + 1, p.T);
    n = f1 > f0 ? f1 - f0 : 0;
    local = slot - (f0 / p.slot_tokens + p.slot_more * (unsigned)b);
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

// ---- rows of whole 16-byte pieces --------------------------------------------------------------------------------------

// 8 elements as floats
template <int DT>
__device__ __forceinline__ void load8(const typename Elem<DT>::T* at, float* x) {
  using T = typename Elem<DT>::T;
  constexpr int W = 16 / sizeof(T);
  typedef T tw __attribute__((ext_vector_type(W)));
#pragma unroll
  for (int i = 0; i < 8; i += W) {
    const tw v = *reinterpret_cast<const tw*>(at + i);
#pragma unroll
    for (int j = 0; j < W; ++j) x[i + j] = (float)v[j];
  }
}
template <int DT>
__device__ __forceinline__ void store8(typename Elem<DT>::T* at, const float* x) {
  using T = typename Elem<DT>::T;
  constexpr int W = 16 / sizeof(T);
  typedef T tw __attribute__((ext_vector_type(W)));
#pragma unroll
  for (int i = 0; i < 8; i += W) {
    tw v;
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = (T)x[i + j];
    *reinterpret_cast<tw*>(at + i) = v;
  }
}
// Of the u-th 16 elements of a head: where its two groups of 8 start.  Rotated halves take a group of each half.
__device__ __forceinline__ void groups_of(unsigned u, unsigned rot, int interleaved, unsigned& one, unsigned& two) {
  const bool halves = !interleaved && u < rot / 16;
  one = halves ? 8 * u : 16 * u;
  two = halves ? 8 * u + rot / 2 : 16 * u + 8;
}
// Rotates them; angle(i) is pair i's.
template <typename Angle>
__device__ __forceinline__ void rotate16(float (&x)[16], unsigned u, unsigned rot, int interleaved, Angle angle) {
  if (u >= rot / 16) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const SinCos w = angle(8 * u + j);
    if (interleaved) rotate(x[2 * j], x[2 * j + 1], w);
    else rotate(x[j], x[8 + j], w);
  }
}
__device__ __forceinline__ unsigned pack4(float a, float b, float c, float d, float s) {
  return quant8(a, s) | quant8(b, s) << 8 | quant8(c, s) << 16 | quant8(d, s) << 24;
}
__device__ __forceinline__ unsigned requant4(unsigned w, float ratio) {
  return requant8(w, ratio) | requant8(w >> 8, ratio) << 8 | requant8(w >> 16, ratio) << 16 | requant8(w >> 24, ratio) << 24;
}
typedef uint32_t w4 __attribute__((ext_vector_type(4)));
typedef uint32_t w2 __attribute__((ext_vector_type(2)));

// TH threads; KI, VI: a thread's 16 elements of keys and 4 x 2 of values, of a chunk of CG groups of four tokens
template <int DT, int TH, int KI, int VI>
__global__ __launch_bounds__(TH) void k_kv_append_rows(const AppendParams p) {
  using T = typename Elem<DT>::T;
  constexpr bool kTable = TH == kWave;                // (one wave: no table or maximum crosses waves)
  // sines and cosines: of a chunk's tokens, or of every eighth position of the block and of 0 .. 7, whose products are all
  // (angles are exact: 24 bits of frequency times 29 of position)
  extern __shared__ SinCos table[];
  __shared__ float red[2][TH / kWave];
  __shared__ unsigned image[kTable ? 1 : 256 * 17];   // a block of values, rows of 16 words and one of padding
  const unsigned tid = threadIdx.x, d = p.d, half = p.rot / 2, d16 = d / 16;

  if (blockIdx.x >= p.page_wgs) {
    // queries: a wave per token and F kWave pieces of 16 elements
    const unsigned lane = tid % kWave, wg = blockIdx.x - p.page_wgs, t = wg / p.q_parts * (TH / kWave) + tid / kWave;
    __shared__ SinCos turn[TH / kWave][128];
    int b = -1;
    unsigned f0 = t;
    if (t < p.T) {
      b = (int)t;
      if (p.first != nullptr) {
        b = wave_search(p.B + 1, t, [&](unsigned i) { return first_at(p.first, i, p.T); });
        if (b >= (int)p.B) b = -1;                    // a row that belongs to no sequence
        if (b >= 0) f0 = first_at(p.first, b, p.T);
      }
    }
    if (b >= 0) {
      const double pos = (double)((long long)p.held[b] + (long long)(t - f0));
      for (unsigned i = lane; i < half; i += kWave) turn[tid / kWave][i] = sincos_f64(pos * (double)p.freq[i]);
    }
    __syncthreads();
    if (b < 0) return;
    const T* src = static_cast<const T*>(p.q) + (size_t)t * p.ldq;
    T* dst = static_cast<T*>(p.q_out) + (size_t)t * p.heads * d;
    constexpr int F = kQPieces / kWave;               // in flight
    const unsigned items = p.heads * d16, i0 = wg % p.q_parts * kQPieces + lane;
    float x[F][16];
    unsigned one[F], two[F], u[F];
#pragma unroll
    for (int f = 0; f < F; ++f) {
      const unsigned i = min(i0 + f * kWave, items - 1);
      u[f] = i % d16;
      groups_of(u[f], p.rot, p.interleaved, one[f], two[f]);
      one[f] += i / d16 * d;
      two[f] += i / d16 * d;
      load8<DT>(src + one[f], x[f]);
      load8<DT>(src + two[f], x[f] + 8);
    }
#pragma unroll
    for (int f = 0; f < F; ++f) {
      if (i0 + f * kWave >= items) break;
      rotate16(x[f], u[f], p.rot, p.interleaved, [&](unsigned j) { return turn[tid / kWave][j]; });
      store8<DT>(dst + one[f], x[f]);
      store8<DT>(dst + two[f], x[f] + 8);
    }
    return;
  }

  const unsigned slot = blockIdx.x / p.kv_heads, h = blockIdx.x % p.kv_heads;
  int b = (int)slot;
  unsigned f0 = slot, n = 1, local = 0;
  long long held = p.held[min(slot, p.B - 1)];        // (right where every sequence in front has one token: no search then)
  const bool alone = kTable && p.slot_more == 0 && slot < p.B && p.first != nullptr && first_at(p.first, slot, p.T) == slot &&
                     first_at(p.first, slot + 1, p.T) == slot + 1;
  if (p.first != nullptr && !alone) {
    auto base = [&](unsigned i) { return first_at(p.first, i, p.T) / p.slot_tokens + p.slot_more * i; };
    b = wave_search(p.B, slot, base);
    if (b < 0) return;
    f0 = first_at(p.first, b, p.T);
    const unsigned f1 = first_at(p.first, b + 1, p.T);
    n = f1 > f0 ? f1 - f0 : 0;
    local = slot - (f0 / p.slot_tokens + p.slot_more * (unsigned)b);
    held = p.held[b];
  }
  const long long page = (held >> 6) + local, p0 = page * kKvBlock;
  const long long t0 = held > p0 ? held : p0, t1 = held + n < p0 + kKvBlock ? held + n : p0 + kKvBlock;
  if (t0 >= t1) return;
  const unsigned lo = (unsigned)(t0 - p0), hi = (unsigned)(t1 - p0), row0 = f0 + (unsigned)(t0 - held);
  int block = -1;
  if (page >= 0 && page < (long long)p.table_width) block = p.table[(size_t)b * p.table_width + page];
  const T* kin = static_cast<const T*>(p.k) + (size_t)row0 * p.ldk + (size_t)h * d;
  const T* vin = static_cast<const T*>(p.v) + (size_t)row0 * p.ldv + (size_t)h * d;
  T* kout = p.k_out == nullptr ? nullptr : static_cast<T*>(p.k_out) + ((size_t)row0 * p.kv_heads + h) * d;
  const size_t ko = (size_t)p.kv_heads * d;
  // chunks of CG groups of four tokens, from the first group with a new token
  const unsigned CG = kTable ? (d > 128 ? 1 : 2) : 16, g_first = lo / 4, g_end = (hi + 3) / 4, d2 = d / 2;
  const unsigned chunks = (g_end - g_first + CG - 1) / CG;
  float kx[KI][16], vx[VI][2][4];
  // keys [t, end) and value groups of chunk c; `out`: rotated keys leave as well
  auto bring = [&](unsigned c, bool out) {
    const unsigned ga = g_first + c * CG, ta = max(lo, 4 * ga), tb = min(hi, 4 * (ga + CG));
    if constexpr (kTable) {
      __syncthreads();
      for (unsigned i = tid; i < (tb - ta) * half; i += TH)
        table[i] = sincos_f64((double)(p0 + ta + i / half) * (double)p.freq[i % half]);
      __syncthreads();
    } else {
      const double eighth = (double)p0;
      for (unsigned i = tid; i < 16 * half; i += TH) {
        const unsigned k = i / half;
        table[i] = sincos_f64((k < 8 ? eighth + 8 * k : (double)(k - 8)) * (double)p.freq[i % half]);
      }
    }
#pragma unroll
    for (int i = 0; i < KI; ++i) {
      const unsigned item = tid + i * TH, t = ta + item / d16, u = item % d16;
      if (t < tb) {
        unsigned one, two;
        groups_of(u, p.rot, p.interleaved, one, two);
        load8<DT>(kin + (size_t)(t - lo) * p.ldk + one, kx[i]);
        load8<DT>(kin + (size_t)(t - lo) * p.ldk + two, kx[i] + 8);
      }
    }
#pragma unroll
    for (int i = 0; i < VI; ++i) {
      const unsigned item = tid + i * TH, g = ga + item / d2, col = item % d2 * 2;
      if (g < ga + CG && g < g_end)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const unsigned t = min(max(4 * g + j, lo), hi - 1);        // (others' places are not used)
          typedef T t2 __attribute__((ext_vector_type(2)));
          const t2 v = *reinterpret_cast<const t2*>(vin + (size_t)(t - lo) * p.ldv + col);
          vx[i][0][j] = (float)v[0];
          vx[i][1][j] = (float)v[1];
        }
    }
    if constexpr (!kTable) __syncthreads();
#pragma unroll
    for (int i = 0; i < KI; ++i) {
      const unsigned item = tid + i * TH, t = ta + item / d16, u = item % d16;
      if (t < tb) {
        rotate16(kx[i], u, p.rot, p.interleaved, [&](unsigned j) -> SinCos {
          if constexpr (kTable) return table[(t - ta) * half + j];
          const SinCos a = table[t / 8 * half + j], b = table[(8 + t % 8) * half + j];
          return {a.sin * b.cos + a.cos * b.sin, a.cos * b.cos - a.sin * b.sin};
        });
        if (out && kout != nullptr) {
          unsigned one, two;
          groups_of(u, p.rot, p.interleaved, one, two);
          store8<DT>(kout + (size_t)(t - lo) * ko + one, kx[i]);
          store8<DT>(kout + (size_t)(t - lo) * ko + two, kx[i] + 8);
        }
      }
    }
  };
  float mk = 0.f, mv = 0.f;
  bring(0, true);
  // (the block's number is on its way meanwhile)
  const bool cached = block >= 0 && (size_t)block < p.blocks, fresh = lo == 0;
  const size_t at = (size_t)(cached ? block : 0) * p.kv_heads + h;
  const float2 had = reinterpret_cast<const float2*>(p.amax)[at];
  const unsigned dk = kv_dk(d), kwords4 = kKvBlock * dk / 16, vwords4 = d * kKvBlock / 16;      // (kv_dv(d) is d)
  int8_t* keys = p.keys + at * kKvBlock * dk;
  unsigned* values = reinterpret_cast<unsigned*>(p.values) + at * d * (kKvBlock / 4);
  // the words of values that the first chunk's tokens share with others
  unsigned old[VI][2] = {};
  if (!fresh)
#pragma unroll
    for (int i = 0; i < VI; ++i) {
      if (kTable) {
        const unsigned g = g_first + (tid + i * TH) / d2, col = (tid + i * TH) % d2 * 2;
        const bool some = g < g_first + CG && g < g_end;
#pragma unroll
        for (int j = 0; j < 2; ++j) old[i][j] = values[((some ? col : 0) + j) * (kKvBlock / 4) + (some ? kv_place(4 * g) / 4 : 0)];
      }
    }
  for (unsigned c = 0; c < chunks; ++c) {
    if (c > 0) bring(c, true);
    const unsigned ga = g_first + c * CG, ta = max(lo, 4 * ga), tb = min(hi, 4 * (ga + CG));
#pragma unroll
    for (int i = 0; i < KI; ++i)
      if (ta + (tid + i * TH) / d16 < tb)
#pragma unroll
        for (int j = 0; j < 16; ++j) mk = fmaxf(mk, finite_abs(kx[i][j]));
#pragma unroll
    for (int i = 0; i < VI; ++i) {
      const unsigned g = ga + (tid + i * TH) / d2;
      if (g < ga + CG && g < g_end)
#pragma unroll
        for (int j = 0; j < 4; ++j) mv = fmaxf(mv, fmaxf(finite_abs(vx[i][0][j]), finite_abs(vx[i][1][j])));
    }
  }
  mk = wave_max_f(mk);
  mv = wave_max_f(mv);
  if constexpr (TH > kWave) {
    if (tid % kWave == 0) {
      red[0][tid / kWave] = mk;
      red[1][tid / kWave] = mv;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < TH / kWave; ++w) {
      mk = fmaxf(mk, red[0][w]);
      mv = fmaxf(mv, red[1][w]);
    }
  }
  if (!cached) return;
  if (!fresh) {
    mk = fmaxf(mk, had.x);
    mv = fmaxf(mv, had.y);
  }
  if (tid == 0) reinterpret_cast<float2*>(p.amax)[at] = make_float2(mk, mv);
  auto mult = [](float a) { return a > 0.f ? __fdiv_rn(127.f, a) : 1.f; };
  const float ck = mult(mk), cv = mult(mv);
  // a block that starts anew is zero but for the new tokens; one whose maximum grew is requantized
  const bool whole = hi - lo == (unsigned)kKvBlock, by_image = !kTable && fresh;
  if (fresh) {
    if (!whole || dk != d)
      for (unsigned i = tid; i < kwords4; i += TH) reinterpret_cast<w4*>(keys)[i] = w4{};
    if (by_image) {
      if (!whole)
        for (unsigned i = tid; i < d * 17; i += TH) image[i] = 0;
    } else {
      for (unsigned i = tid; i < vwords4; i += TH) reinterpret_cast<w4*>(values)[i] = w4{};
    }
  } else {
    auto again = [&](w4* at, unsigned count, float ratio) {
      for (unsigned i = tid; i < count; i += TH) {
        w4 w = at[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = requant4(w[j], ratio);
        at[i] = w;
      }
    };
    if (mk > had.x) again(reinterpret_cast<w4*>(keys), kwords4, __fdiv_rn(had.x, mk));
    if (mv > had.y) again(reinterpret_cast<w4*>(values), vwords4, __fdiv_rn(had.y, mv));
  }
  __syncthreads();                                    // before the new tokens' places are written
  for (unsigned c = 0; c < chunks; ++c) {
    if (chunks > 1) bring(c, false);
    const unsigned ga = g_first + c * CG, ta = max(lo, 4 * ga), tb = min(hi, 4 * (ga + CG));
#pragma unroll
    for (int i = 0; i < KI; ++i) {
      const unsigned item = tid + i * TH, t = ta + item / d16;
      if (t < tb) {
        unsigned one, two;
        groups_of(item % d16, p.rot, p.interleaved, one, two);
        const float (&x)[16] = kx[i];
        const w2 a = {pack4(x[0], x[1], x[2], x[3], ck), pack4(x[4], x[5], x[6], x[7], ck)},
                 b2 = {pack4(x[8], x[9], x[10], x[11], ck), pack4(x[12], x[13], x[14], x[15], ck)};
        *reinterpret_cast<w2*>(keys + t * dk + one) = a;
        *reinterpret_cast<w2*>(keys + t * dk + two) = b2;
      }
    }
#pragma unroll
    for (int i = 0; i < VI; ++i) {
      const unsigned item = tid + i * TH, g = ga + item / d2, col = item % d2 * 2, word = kv_place(4 * g) / 4;
      if (g < ga + CG && g < g_end) {
        // bytes of the word that are new
        const unsigned from = 4 * g < lo ? lo - 4 * g : 0, end = 4 * g + 4 > hi ? hi - 4 * g : 4;
        const unsigned mask = (end == 4 ? 0xFFFFFFFFu : (1u << (8 * end)) - 1) & ~((1u << (8 * from)) - 1);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const unsigned w = pack4(vx[i][j][0], vx[i][j][1], vx[i][j][2], vx[i][j][3], cv) & mask;
          if (by_image) {
            image[(col + j) * 17 + word] = w;
          } else {
            unsigned* to = values + (col + j) * (kKvBlock / 4) + word;
            const bool kept = kTable && chunks == 1 && !(mv > had.y);        // (what was read early still holds)
            *to = mask == 0xFFFFFFFFu || fresh ? w : ((kept ? old[i][j] : *to) & ~mask) | w;
          }
        }
      }
    }
  }
  if (by_image) {
    __syncthreads();
    for (unsigned i = tid; i < vwords4; i += TH) {
      const unsigned* from = image + i / 4 * 17 + i % 4 * 4;
      reinterpret_cast<w4*>(values)[i] = w4{from[0], from[1], from[2], from[3]};
    }
  }
}

}  // namespace

int launch_kv_append(const mq_kv_cache& cache, const int32_t* table, size_t table_width, const int32_t* first,
                     const int32_t* held, size_t B, size_t T, const void* k, size_t ldk, const void* v, size_t ldv,
                     const void* q, size_t ldq, int heads, int dtype, const float* freq, size_t rot, int interleaved,
                     void* k_out, void* q_out, hipStream_t s) {
  // A sequence of n tokens touches at most n / 64 + 2 blocks, and no more than n: slots by whichever is fewer in all.  The
  // latter means few tokens to a block.
  const bool few = first == nullptr || T < T / kKvBlock + 2 * B;
  const size_t slots = first == nullptr ? B : few ? T : T / kKvBlock + 2 * B;
  const size_t page_wgs = slots * (size_t)cache.kv_heads, d = cache.head_dim;
  const size_t piece = 16 / elem_bytes(dtype);
  auto whole = [&](const void* x, size_t ld) { return reinterpret_cast<uintptr_t>(x) % 16 == 0 && ld % piece == 0; };
  const bool rows = d % 16 == 0 && rot % 16 == 0 && whole(k, ldk) && whole(v, ldv) && whole(k_out, 0) &&
                    (q == nullptr || (whole(q, ldq) && whole(q_out, 0)));
  // One wave to a block where a sequence's tokens are one chunk of its: 200 sequences, 8 heads of 64, binary32, 3 tokens each
  // 16 us with four waves and 9 with one, 8 tokens 16 and 10 (13 behind others); 100 sequences, 8 heads of 128 and 32 of queries,
  // bfloat16, 3 tokens 20 and 10, 8 tokens 23 and 15 (22 behind others).  With four, 64 sequences of the latter heads take 18 us
  // for 9 tokens each, 20 for 16, 27 for 32.
  const bool narrow = T <= 8 * B;
  const size_t q_tokens = rows && narrow ? 1 : kTokensPerWg;
  const size_t q_parts = rows && q != nullptr ? ((size_t)heads * (d / 16) + kQPieces - 1) / kQPieces : 1;
  const size_t q_wgs = q == nullptr ? 0 : (T + q_tokens - 1) / q_tokens * q_parts;
  if (!launchable(page_wgs + q_wgs, rows && narrow ? kWave : kT)) return MQ_ERR_SHAPE;
  const AppendParams p{k, v, q, table, first, held, freq, ldk, ldv, ldq, table_width, cache.blocks, cache.keys, cache.values,
                       cache.amax, k_out, q_out, (unsigned)B, (unsigned)T, (unsigned)cache.kv_heads, (unsigned)heads,
                       (unsigned)d, (unsigned)rot, (unsigned)page_wgs, few ? 1u : (unsigned)kKvBlock, few ? 0u : 2u,
                       (unsigned)q_parts, interleaved};
  const unsigned wgs = (unsigned)(page_wgs + q_wgs);
  return with_dtype(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    if (rows) {
      const size_t table = narrow ? 512 * sizeof(SinCos) : 16 * (rot / 2) * sizeof(SinCos);
      auto go = [&](auto kern, int threads) { hipLaunchKernelGGL(kern, dim3(wgs), dim3(threads), table, s, p); };
      if (narrow) go(k_kv_append_rows<DT, 64, 1, 2>, 64);
      else if (d <= 64) go(k_kv_append_rows<DT, 256, 1, 2>, 256);
      else if (d <= 128) go(k_kv_append_rows<DT, 256, 2, 4>, 256);
      else go(k_kv_append_rows<DT, 256, 4, 8>, 256);
      return check_hip(hipGetLastError());
    }
    const size_t tokens = first == nullptr ? 1 : T < (size_t)kKvBlock ? T : (size_t)kKvBlock;      // of one block, at most
    const size_t lds = 2 * tokens * (d + 1) * sizeof(float);
    auto kern = k_kv_append<DT>;
    if (lds > 65536) {
      const int rc = check_hip(hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
      if (rc != MQ_OK) return rc;
    }
    hipLaunchKernelGGL(kern, dim3(wgs), dim3(kT), lds, s, p);
    return check_hip(hipGetLastError());
  });
}

}  // namespace mq
