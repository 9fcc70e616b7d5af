// Attention of several new tokens per sequence over a paged 8-bit cache (include/mq_serve.h): out_i = sum_t p_t V[t] with
// p = softmax_{t <= len - n + i}(scale q_i . K[t]).
//
// One pass over the cache with the running maximum and sum of each query.  The queries of a sequence that share a kv head, n
// tokens x the heads of the group, are rows of one product: S^T = K q^T on v_mfma_f32_32x32x16_bf16, 32 tokens of K as operand
// a, 32 query rows as operand b.  Lane l then has, for row l % 32, the scores of tokens 8 (r / 4) + 4 (l / 32) + r % 4 of 32, and
// the cache keeps the values of a block in an order (kv_place) in which these lanes' probabilities are operand b of out^T = V^T p^T
// as they are.  The cache's integers are bfloat16 values exactly (8 bits); queries enter as one, two or three bfloat16 parts,
// probabilities as two or three.  Scales: a block's for the keys goes into the scores' factor, a block's for the values into the
// probabilities, so sums stay in the accumulators from block to block.
#include <type_traits>

#include "mq_glue.h"
#include "mq_serve_common.h"

namespace mq {

namespace {

constexpr unsigned kRows = 32;        // query rows of a tile where there are few
constexpr unsigned kWaves = 4;        // of a workgroup of that form, at most
// How far (as a power of two) a row's scores may rise over the reference that its sums are relative to before they are
// rescaled: exponentials up to 2^8 lose nothing in a binary format, and a maximum that rises a little does not cost anything.
constexpr float kSlack = 8.f;

struct ChunkParams {
  const int8_t *keys, *values;
  const float* amax;
  const int32_t *table, *first, *lens;
  const void* q;
  void* out;
  float* part;                        // [workgroups][2][rows of a tile][dv + 4]: sums, reference, total
  size_t ldq, ldo, table_width, blocks;
  unsigned B, T, max_len, kv_heads, heads, d;
  float scale2;                       // scale log2(e)
  int causal;
  unsigned* plan;                     // [slots + 1] blocks of the tiles in front of each tile, the share, then at 16 bytes [slots] tiles
  unsigned slots, least;              // tiles at most; blocks that a workgroup takes at least
  int here;                           // whether the workgroups plan for themselves
};

// Exponent of the power of two taken off a row whose largest magnitude is m.  (126 at most: the multiplier 2^-127 is no normal number,
// and its bits would be those of zero; a row of 2^127 and more keeps magnitudes of 2 .. 4.)
__device__ __forceinline__ int row_exponent(float m) {
  return m > 0.f && m < INFINITY ? min(max((int)(__float_as_uint(m) >> 23) - 127, -126), 126) : 0;
}
// The same number, and nothing that the compiler keeps comparisons with: dozens of kept masks do not fit the scalar registers.
__device__ __forceinline__ unsigned again(unsigned x) {
  asm volatile("" : "+s"(x));
  return x;
}
// How many bfloat16 parts hold a probability: 16 bits for 16-bit types.  (One part, 8 bits, is as coarse as a bfloat16 result: four
// pieces of 300 .. 1100 tokens on 2000 .. 16000 in 412 us instead of 542, but off by 2.3e-3 from 64 bits instead of 1.7e-3.)
template <int DT>
constexpr int kWeightParts = DT == MQ_F32 ? 3 : 2;
__device__ __forceinline__ float finite_or_0(float m) { return m == -INFINITY ? 0.f : m; }

// A block's value is integer x unit x m.  m goes into the exponent of its tokens' weights, which the exponential flushes below
// 2^-126: an m below 2^-60 would take weights with it that count in the denominator.  There m is 1 .. 2 and the power of two, unit,
// is put to the integers (which stay bfloat16 values).  Values below any normal number are zeros.
struct ValueScale {
  float m, unit;
};
__device__ __forceinline__ ValueScale value_scale(float amax) {
  const float s = amax * (1.f / 127.f);
  const unsigned b = __float_as_uint(s);
  if (s < 0x1p-126f) return {1.f, 0.f};
  if (s < 0x1p-60f) return {__uint_as_float((b & 0x007fffffu) | 0x3f800000u), __uint_as_float(b & 0x7f800000u)};
  return {s, 1.f};
}
__device__ __forceinline__ unsigned uniform_bits(float x) { return (unsigned)__builtin_amdgcn_readfirstlane((int)__float_as_uint(x)); }
// Integers as bfloat16 values times a unit (its bits), the same for the wave; it is 1 but for very small values.
__device__ __forceinline__ bf8 in_units(bf8 v, unsigned unit) {
  if (unit != 0x3f800000u) {
    const float f = __uint_as_float(unit);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (__bf16)((float)v[i] * f);
  }
  return v;
}
__device__ __forceinline__ float fmax2(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float fadd2(float a, float b) { return a + b; }

// sum + a + b, as rounded: what is divided by then is the sum of what is multiplied.
__device__ __forceinline__ float add2(__bf16 a, __bf16 b, float sum) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_fdot2_f32_bf16(b2{a, b}, b2{(__bf16)1.f, (__bf16)1.f}, sum, false);
}

// A tile of query rows: row i of its sequence's n x per is token i / per, head i % per of the group.
struct alignas(8) Tile {
  int b;                              // sequence, -1: no such tile
  unsigned first, n, row0, rows, len; // its first token row and new tokens, the tile's first row and rows, tokens in the cache
};
// Tiles of sequence b lie from tile number first[b] per / ROWS + b on: enough for each, whatever the lengths.
template <unsigned ROWS>
__device__ __forceinline__ Tile tile_of(const ChunkParams& p, int b, unsigned f, unsigned e, int len, unsigned slot, unsigned per) {
  const unsigned n = e > f ? e - f : 0, row0 = (slot - (f * per / ROWS + b)) * ROWS;
  if (row0 >= n * per) return {-1, 0, 0, 0, 0, 0};
  return {b, f, n, row0, min(n * per - row0, ROWS), len < 0 ? 0u : min((unsigned)len, p.max_len)};
}
template <unsigned ROWS>
__device__ __forceinline__ Tile tile_of(const ChunkParams& p, int b, unsigned slot, unsigned per) {
  if (b < 0) return {-1, 0, 0, 0, 0, 0};
  return tile_of<ROWS>(p, b, first_at(p.first, b, p.T), first_at(p.first, b + 1, p.T), p.lens[b], slot, per);
}
template <unsigned ROWS>
__device__ __forceinline__ Tile find_tile(const ChunkParams& p, unsigned slot, unsigned per) {
  auto start = [&](unsigned i) { return first_at(p.first, i, p.T) * per / ROWS + i; };
  return tile_of<ROWS>(p, __builtin_amdgcn_readfirstlane(wave_search(p.B, slot, start)), slot, per);
}
// Tokens that query i of n sees.
__device__ __forceinline__ unsigned seen_by(const ChunkParams& p, const Tile& t, unsigned i) {
  if (!p.causal) return t.len;
  const long long s = (long long)t.len - t.n + i + 1;
  return s < 0 ? 0u : (unsigned)s;
}

// ---- equal shares ---------------------------------------------------------------------------------------------------------
//
// Lengths are known on the device only, so a first small launch sums up the blocks that each tile of rows sees.  The workgroups,
// as many as have room at once, share the blocks of all tiles and kv heads in one line equally: each has some tiles whole, and parts of
// the tiles at its two ends, which go to the workspace and are joined.  (Instead of runs of equal length, a workgroup each, as many
// of every tile as the longest needs: four pieces of 300 .. 1100 tokens on 2000 .. 16000, 526 us when equal shares were new, at 453.)

constexpr int kPlan = 1024;           // threads of the workgroup that plans

// Blocks that a tile's last row sees, one at least: every tile belongs to somebody.
__device__ __forceinline__ unsigned tile_blocks(const ChunkParams& p, const Tile& t, unsigned per) {
  return t.b < 0 ? 0u : max(1u, (seen_by(p, t, (t.row0 + t.rows - 1) / per) + kKvBlock - 1) / kKvBlock);
}

__device__ __forceinline__ Tile* planned(const ChunkParams& p) {
  return reinterpret_cast<Tile*>(p.plan + (p.slots + 5) / 4 * 4);
}

// Blocks that a workgroup has, where there are `each` >= 4 workgroups to a kv head and `line` blocks.
__device__ __forceinline__ unsigned share_of_head(const ChunkParams& p, unsigned line, unsigned each) {
  return max(p.least, (line + each - 1) / each);
}
// Blocks of the line that a workgroup has, and where the next kv head's begin: at another workgroup, if there are enough of them (one
// that had the ends of two would take its way to memory twice).
struct Share {
  unsigned long long blocks, pitch;
};
__device__ __forceinline__ Share share_of(const ChunkParams& p, unsigned line, unsigned planned, unsigned groups) {
  if (groups / p.kv_heads >= 4) return {planned, (unsigned long long)((line + planned - 1) / planned) * planned};
  return {max((unsigned long long)p.least, ((unsigned long long)line * p.kv_heads + groups - 1) / groups), line};
}

// sum over the threads in front of this one of the workgroup, and over all
template <int WAVES>
__device__ __forceinline__ unsigned sum_ahead(unsigned n, unsigned* box, unsigned& all) {
  const unsigned lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  unsigned x = n;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const unsigned y = __shfl_up(x, off, kWave);
    if (lane >= (unsigned)off) x += y;
  }
  __syncthreads();
  if (lane == kWave - 1) box[wave] = x;
  __syncthreads();
  unsigned before = x - n;
  all = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w < (int)wave) before += box[w];
    all += box[w];
  }
  return before;
}
// The sequence in [0, B) whose tiles a slot is among: those of sequence b start at first(b) per / ROWS + b.
template <unsigned ROWS, typename F>
__device__ __forceinline__ unsigned sequence_of(unsigned B, unsigned slot, unsigned per, F first) {
  unsigned lo = 0, hi = B;
  while (hi - lo > 1) {
    const unsigned mid = (lo + hi) / 2;
    if (first(mid) * per / ROWS + mid <= slot) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <unsigned ROWS>
__global__ __launch_bounds__(kPlan) void k_chunk_plan(const ChunkParams p, unsigned groups) {
  __shared__ unsigned box[kPlan / kWave];
  const unsigned per = p.heads / p.kv_heads;
  unsigned ahead = 0;
  for (unsigned at = 0; at < p.slots; at += kPlan) {
    const unsigned slot = at + threadIdx.x;
    const unsigned b = sequence_of<ROWS>(p.B, slot, per, [&](unsigned i) { return first_at(p.first, i, p.T); });
    unsigned n = 0, all;
    if (slot < p.slots) {
      const Tile t = tile_of<ROWS>(p, (int)b, slot, per);
      n = tile_blocks(p, t, per);
      planned(p)[slot] = t;
    }
    const unsigned before = sum_ahead<kPlan / kWave>(n, box, all);
    if (slot < p.slots) p.plan[slot] = ahead + before;
    ahead += all;
  }
  if (threadIdx.x == 0) {
    p.plan[p.slots] = ahead;
    p.plan[p.slots + 1] = share_of_head(p, ahead, max(groups / p.kv_heads, 1u));
  }
}

// The same by every workgroup of few rows for itself, in LDS: a launch less, for the way of two loads.  The first one leaves the plan
// for the join.  (Two workgroups of 78 KB to a compute unit have room for as many tiles.)
// Where there are at least four workgroups to a tile and shares are short each has blocks of one only, for the same reason: tiles begin
// at a share of their own, whose last may have less (8 sequences of 4 new tokens on 4000, 32 heads over 8 of 128: 33.5 -> 26.9 us;
// 16 on 12000, shares of 63: 85 -> 94, so not there).
constexpr unsigned kHere = 192, kAlone = 16;
struct PlanHere {
  unsigned starts[kHere + 2], box[kWaves];
  Tile tiles[kHere];
};
template <unsigned WAVES>
__device__ __forceinline__ void plan_here(const ChunkParams& p, PlanHere& to) {
  static_assert(WAVES * kWave >= kHere, "a thread for each tile");
  const unsigned slot = threadIdx.x, per = p.heads / p.kv_heads;
  for (unsigned b = threadIdx.x; b <= p.B; b += WAVES * kWave) {                      // (B <= slots)
    to.starts[b] = first_at(p.first, b, p.T);
    if (b < p.B) to.tiles[b].len = (unsigned)p.lens[b];
  }
  __syncthreads();
  Tile t{-1, 0, 0, 0, 0, 0};
  if (slot < p.slots) {
    const unsigned b = sequence_of<kRows>(p.B, slot, per, [&](unsigned i) { return to.starts[i]; });
    t = tile_of<kRows>(p, (int)b, to.starts[b], to.starts[b + 1], (int)to.tiles[b].len, slot, per);
  }
  const unsigned n = tile_blocks(p, t, per), each = max(gridDim.x / p.kv_heads, 1u);
  unsigned all, tiles;
  sum_ahead<WAVES>(n > 0 ? 1u : 0u, to.box, tiles);         // (nobody reads what they held any more)
  unsigned before = sum_ahead<WAVES>(n, to.box, all), share = share_of_head(p, all, each);
  const unsigned line = all;
  auto alone = [&](unsigned blocks) {                       // (whole turns of the waves)
    share = (blocks + kWaves - 1) / kWaves * kWaves;
    before = sum_ahead<WAVES>((n + share - 1) / share * share, to.box, all);
  };
  if (tiles <= each / 4 && share <= kAlone) {
    alone(share);
    if (all > each * share) alone(share_of_head(p, line, each - tiles));       // (enough whatever the lengths)
  }
  if (slot < p.slots) {
    to.starts[slot] = before;
    to.tiles[slot] = t;
  }
  if (slot == 0) {
    to.starts[p.slots] = all;
    to.starts[p.slots + 1] = share;
  }
  if (blockIdx.x == 0) {
    if (slot < p.slots) {
      p.plan[slot] = before;
      planned(p)[slot] = t;
    }
    if (slot == 0) {
      p.plan[p.slots] = all;
      p.plan[p.slots + 1] = share;
    }
  }
  __syncthreads();
}

// A workgroup's next part of the line: blocks [start, end) of a tile and a kv head; whole: all that the tile has.
struct LinePart {
  unsigned kvh, start, end, next;     // next: where the next tile begins in the line
  bool whole;
  Tile tile;
};
__device__ __forceinline__ LinePart part_at(const ChunkParams& p, const unsigned* starts, const Tile* tiles, unsigned kvh,
                                            unsigned place, unsigned long long most) {
  const unsigned slot = (unsigned)__builtin_amdgcn_readfirstlane(wave_search(p.slots, place, [&](unsigned i) { return starts[i]; }));
  const Tile t = tiles[slot];
  const unsigned blocks = tile_blocks(p, t, p.heads / p.kv_heads), start = place - starts[slot];
  const unsigned end = (unsigned)min((unsigned long long)blocks, start + most);
  auto uniform = [](unsigned x) { return (unsigned)__builtin_amdgcn_readfirstlane((int)x); };
  return {kvh, uniform(start), uniform(end), uniform(starts[slot + 1]), start == 0 && end == blocks,
          Tile{(int)uniform((unsigned)t.b), uniform(t.first), uniform(t.n), uniform(t.row0), uniform(t.rows), uniform(t.len)}};
}
// Calls f(part, where a part that is not whole goes) for all parts of this workgroup.  An eighth of the line to each XCD, whose
// workgroups then read the same heads' blocks.
template <typename F>
__device__ __forceinline__ void each_part(const ChunkParams& p, const unsigned* starts, const Tile* tiles, F f) {
  const unsigned me = blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;
  const unsigned line = (unsigned)__builtin_amdgcn_readfirstlane((int)starts[p.slots]);
  const Share share = share_of(p, line, (unsigned)__builtin_amdgcn_readfirstlane((int)starts[p.slots + 1]), gridDim.x);
  const unsigned long long to = min((me + 1) * share.blocks, share.pitch * p.kv_heads);
  unsigned kvh = 0;                   // (no division: there are few heads, and a workgroup has one or two)
  unsigned long long at = me * share.blocks, place = at;
  for (unsigned n = 0; at < to; ++n) {
    while (place >= share.pitch) {
      place -= share.pitch;
      ++kvh;
    }
    if (place >= line) break;         // (a kv head's last share may be shorter)
    const LinePart part = part_at(p, starts, tiles, kvh, (unsigned)place, to - at);
    const unsigned next = part.next - (unsigned)place;
    at += next;
    place += next;
    f(part, me * 2 + (n > 0 ? 1 : 0));
  }
}

// ---- few rows -------------------------------------------------------------------------------------------------------------
//
// A workgroup has 32 rows; its waves take the blocks in turn, each through its own part of LDS with no barrier, and join there.
// Bound by the bytes of the cache where sequences are long: 32 sequences of 4 new tokens, 32 heads over 8 of 128, 16000 tokens
// held, 1.05 GB in 211 us, 5.0 TB/s (a copy, half of it writes, reaches 4.7); 1000 .. 9000 held, 243 MB in 74 us (3.3 TB/s), of
// which plan, start and join take 15.  Few tokens are bound by the way of one block, some 1.5 us: 64 sequences of up to 512 8.4 us.
// Blocks come by the loads that go to LDS directly, 1 KB each in whole lines (a lane that loads its own row is an access of its own
// to the nearest cache, 64 a load: 117 us), keys of the next block as soon as this one's are in registers, values likewise.

// LDS of a wave's block of keys and values, loads of 1 KB of either, and waves of a workgroup at most: 160 KB hold its blocks and
// the queries.
template <int DC>
constexpr unsigned kWaveBytes = 2 * kKvBlock * 64 * DC;
template <int DC>
constexpr int kLoads = 4 * DC;
constexpr unsigned few_waves(int parts, int dc) { return dc == 4 && parts > 1 ? 3 : kWaves; }
// s_waitcnt's operand for at most n loads on their way, nothing else waited for but LDS
constexpr int waitcnt_loads(int n) { return (n & 15) | (n >> 4) << 14 | 0x0070; }

template <int DT, int DC>             // DC: 64-column pieces of a key
__device__ __forceinline__ void few_rows(const ChunkParams& p, int vec, const LinePart& part, unsigned to_part) {
  using T = typename Elem<DT>::T;
  constexpr int NP = kParts<DT>, PP = kWeightParts<DT>;
  constexpr int NK = 2 * DC, ND = 2 * DC;      // 32-column pieces of a key, 32-column pieces of a value at most
  constexpr int U = NK * 2;                    // units of 8 elements of a query
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  bf8* const ql = reinterpret_cast<bf8*>(smem);                                  // [NP][U][64 lanes], then each wave's blocks
  __shared__ unsigned fac[kRows];               // largest magnitudes, as bits
  __shared__ float stat[2][kWaves][kRows];
  // (unknown to the compiler to be the same each time: it would keep dozens of places and masks from one part to the next)
  unsigned lane = threadIdx.x % kWave, d = p.d;
  asm volatile("" : "+v"(lane), "+s"(d));
  constexpr unsigned W = few_waves(NP, DC);
  const unsigned wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), col = lane % 32, grp = lane / 32;
  const unsigned per = p.heads / p.kv_heads, dk = kv_dk(d), dv = kv_dv(d), kvh = part.kvh;
  const Tile tile = part.tile;
  auto row_at = [&](unsigned r) {              // element offset of row r's queries in q, without the row pitch: token, head
    const unsigned i = tile.row0 + r;
    return make_uint2(tile.first + i / per, kvh * per + i % per);
  };
  const unsigned last = tile.row0 + tile.rows - 1;
  const unsigned most = seen_by(p, tile, last / per), least = seen_by(p, tile, tile.row0 / per);
  const unsigned mine_sees = seen_by(p, tile, min(tile.row0 + col, last) / per);
  const unsigned start = part.start, end = min(part.end, (most + kKvBlock - 1) / kKvBlock);

  // this wave's blocks, every W-th of the part: which ones is looked up 64 at a time, keys and values are asked for as soon as
  // the registers of those of the block before are free
  const int32_t* table = p.table + (size_t)tile.b * p.table_width;
  const unsigned mine = end > start + wave ? __builtin_amdgcn_readfirstlane((end - start - wave + W - 1) / W) : 0u;
  auto look = [&](unsigned i) {
    const size_t pg = start + wave + (size_t)(i + lane) * W;
    return table[pg < p.table_width ? pg : p.table_width - 1];
  };
  int ids = look(0);
  bool there = true, there_next = true;
  size_t at_next = 0;
  float2 am_next;
  // this wave's part of LDS: keys as they lie, rows of dk bytes, then values, rows of 64; piece j of 16 bytes of row r lies at place
  // j ^ turned(r), so that eight rows' pieces are on different banks
  char* const mine_lds = smem + NP * U * 1024 + wave * kWaveBytes<DC>;
  auto turned = [](unsigned r) { return DC % 2 == 0 ? r & 7 : r >> 1 & 3; };
  auto find = [&](unsigned i) {
    if (i % kWave == 0 && i > 0) ids = look(i);
    const int block = __builtin_amdgcn_readlane(ids, i % kWave);
    there_next = block >= 0 && (size_t)block < p.blocks;
    at_next = (size_t)(there_next ? block : 0) * p.kv_heads + kvh;
  };
  auto bring = [&](const int8_t* from, unsigned to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                     (__attribute__((address_space(3))) void*)(mine_lds + to), 16, 0, 0);
  };
  // kLoads loads each, whatever the width
  auto bring_keys = [&] {
    const int8_t* kp = p.keys + at_next * kKvBlock * dk;
    am_next = reinterpret_cast<const float2*>(p.amax)[at_next];
#pragma unroll
    for (int i = 0; i < kLoads<DC>; ++i) {
      const unsigned piece = i * kWave + lane, r = piece / (4 * DC), j = piece % (4 * DC);
      bring(kp + (size_t)r * dk + (j ^ turned(r)) * 16, i * 1024);
    }
  };
  auto bring_values = [&] {
    const int8_t* vp = p.values + at_next * dv * kKvBlock;
#pragma unroll
    for (int i = 0; i < kLoads<DC>; ++i) {                 // (16 rows each; those that are not there repeat the last)
      const unsigned at = min((unsigned)i, dv / 16 - 1), r = at * 16 + lane / 4;
      bring(vp + r * kKvBlock + ((lane % 4) ^ (r >> 1 & 3)) * 16, kKvBlock * 64 * DC + at * 1024);
    }
  };
  auto key_piece = [&](int t, int c) {                     // row 32 t + col, bytes 32 c + 16 grp ..
    const unsigned r = 32 * t + col;
    return *reinterpret_cast<const u4*>(mine_lds + r * (64 * DC) + ((2 * c + grp) ^ turned(r)) * 16);
  };
  auto value_piece = [&](int t, int h) {                   // row 32 t + col, bytes 16 grp + 32 h ..
    const unsigned r = 32 * t + col;
    return *reinterpret_cast<const u4*>(mine_lds + kKvBlock * 64 * DC + r * kKvBlock + ((grp + 2 * h) ^ (r >> 1 & 3)) * 16);
  };
  // until at most N of this wave's loads are on their way, and all that it read from LDS is there
  auto arrived = [&](auto n) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(waitcnt_loads(decltype(n)::value));
    asm volatile("" ::: "memory");
  };

  if (mine > 0) {
    find(0);
    bring_keys();
    bring_values();
  }
  // queries: a power of two off each row, so that its largest element is 1 .. 2 (4 from 2^127 on), then parts in operand order.  Unit u
  // of lane l is elements 32 (u / 2) + 16 (l / 32) + 8 (u % 2) .. of row l % 32
  {
    const unsigned rr = min(col, tile.rows - 1);
    const uint2 at = row_at(rr);
    const T* src = static_cast<const T*>(p.q) + (size_t)at.x * p.ldq + (size_t)at.y * d;
    if (threadIdx.x < kRows) fac[threadIdx.x] = 0;
    constexpr unsigned EACH = (U + W - 1) / W;             // units of a wave
    float x[EACH][8], m = 0.f;
#pragma unroll
    for (unsigned n = 0; n < EACH; ++n) {
      const unsigned u = wave + W * n, k = 32 * (u / 2) + 16 * grp + 8 * (u % 2);
      if (vec & 1) {
        constexpr int E = 16 / sizeof(T);
        typedef T tw __attribute__((ext_vector_type(E)));
#pragma unroll
        for (int j = 0; j < 8; j += E) {
          const tw w = *reinterpret_cast<const tw*>(src + min(k + j, d - E));
#pragma unroll
          for (int i = 0; i < E; ++i) x[n][j + i] = k + j < d ? (float)w[i] : 0.f;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[n][j] = k + j < d ? (float)src[k + j] : 0.f;
      }
    }
#pragma unroll
    for (unsigned n = 0; n < EACH; ++n)
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(x[n][j]) <= 3.402823466e38f ? fabsf(x[n][j]) : INFINITY);
    __syncthreads();
    // (magnitudes are in the order of their bits; a maximum does not depend on the order)
    atomicMax(&fac[col], __float_as_uint(across32_f(m, fmax2)));
    __syncthreads();
    const float most_of_row = __uint_as_float(fac[col]);
    const float mul = __uint_as_float((unsigned)(127 - row_exponent(most_of_row)) << 23) * (p.scale2 < 0.f ? -1.f : 1.f);
#pragma unroll
    for (unsigned n = 0; n < EACH; ++n) {
      const unsigned u = wave + W * n;
      bf8 part[NP];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        __bf16 b[NP];
        split_bf16<NP>(most_of_row == INFINITY ? NAN : x[n][j] * mul, b);     // a row with a NaN or an infinity gives NaN
#pragma unroll
        for (int i = 0; i < NP; ++i) part[i][j] = b[i];
      }
      if (u < U)
#pragma unroll
        for (int i = 0; i < NP; ++i) ql[(i * U + u) * kWave + lane] = part[i];
    }
  }
  __syncthreads();
  const float qscale = ldexpf(fabsf(p.scale2), row_exponent(__uint_as_float(fac[col]))) * (1.f / 127.f);

  float acc_top = -INFINITY, total = 0.f;      // of row l % 32; the total of this lane's tokens
  v16f acc[ND] = {};
  constexpr bool FOLD = PP < 3;
  for (unsigned i = 0; i < mine; ++i) {
    const unsigned pg = start + wave + i * W;
    const float2 am = am_next;
    there = there_next;
    if (i + 1 < mine) find(i + 1);
    arrived(std::integral_constant<int, kLoads<DC>>{});    // (all but this block's values)
    v16f sc[2] = {};
    u4 kf[2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      bf8 a[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (u % 2 == 0) kf[t] = key_piece(t, u / 2);
        a[t] = bf16_of_bytes(kf[t][2 * (u % 2)], kf[t][2 * (u % 2) + 1]);
      }
#pragma unroll
      for (int k = NP - 1; k >= 0; --k) {
        const bf8 b = ql[(k * U + u) * kWave + lane];
#pragma unroll
        for (int t = 0; t < 2; ++t) sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[t], b, sc[t], 0, 0, 0);
      }
    }
    arrived(std::integral_constant<int, kLoads<DC>>{});    // (nothing is read from the keys' place any more)
    if (i + 1 < mine) bring_keys();
    if (!there || (pg + 1) * kKvBlock > least) {
      const long long room = (long long)mine_sees - (long long)pg * kKvBlock - 4 * (int)grp;
      const int limit = !there || room < 0 ? 0 : room > kKvBlock ? kKvBlock : (int)room;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (limit <= 32 * t + 8 * (r / 4) + r % 4) sc[t][r] = -INFINITY;
    }
    float f = there ? qscale * am.x : 0.f, mt = -INFINITY;
    f = f == 0.f ? 1e-30f : f;                 // (0 times a masked score would be NaN; others are below 2^24)
    settle(sc[0], sc[1]);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; r += 2) mt = max3(mt, sc[t][r], sc[t][r + 1]);
    mt = across32_f(mt, fmax2) * f;
    if (__any(mt > acc_top + kSlack)) {
      // (only for the rows concerned: no other row's result depends on theirs)
      const float now = mt > acc_top + kSlack ? mt : acc_top, keep = now == acc_top ? 1.f : __builtin_amdgcn_exp2f(acc_top - now);
      acc_top = now;
      total *= keep;
#pragma unroll
      for (int t = 0; t < ND; ++t) acc[t] *= keep;
    }
    // (where there is no block, block 0 was read, whose maxima may be anything)
    const float fv = there ? am.y * (1.f / 127.f) : 0.f;
    const ValueScale vs = FOLD ? value_scale(there ? am.y : 0.f) : ValueScale{1.f, 1.f};
    const unsigned unit = uniform_bits(vs.unit);
    const float base = (FOLD ? __builtin_amdgcn_logf(vs.m) : 0.f) - finite_or_0(acc_top);
    float sum = 0.f;
    u4 vf[ND][2];
    if (i + 1 < mine) arrived(std::integral_constant<int, kLoads<DC>>{});      // (all but the next block's keys)
    else arrived(std::integral_constant<int, 0>{});
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bf8 pr[PP];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float e = __builtin_amdgcn_exp2f(fmaf(sc[j / 2][8 * (j % 2) + k], f, base));
        if (!FOLD) sum += e;
        __bf16 v[PP];
        split_bf16<PP>(FOLD ? e : e * fv, v);
#pragma unroll
        for (int n = 0; n < PP; ++n) {
          pr[n][k] = v[n];
          if (FOLD && k % 2 == 1) sum = add2(pr[n][k - 1], v[n], sum);
        }
      }
#pragma unroll
      for (int t = 0; t < ND; ++t) {
        if (j == 0) {
          vf[t][0] = value_piece(t, 0);
          vf[t][1] = value_piece(t, 1);
        }
        const bf8 a = in_units(bf16_of_bytes(vf[t][0][j], vf[t][1][j]), unit);
#pragma unroll
        for (int k = PP - 1; k >= 0; --k) acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pr[k], acc[t], 0, 0, 0);
      }
    }
    total = FOLD ? fmaf(sum, __fdiv_rn(1.f, vs.m), total) : total + sum;
    if (i + 1 < mine) {
      arrived(std::integral_constant<int, kLoads<DC>>{});
      bring_values();
    }
  }
  total = across32_f(total, fadd2);

  // every wave leaves its sums where its blocks were, rows of 64 DC numbers, four at place j ^ (row & 7); eight threads join a row
  if (grp == 0) {
    stat[0][wave][col] = acc_top;
    stat[1][wave][col] = total;
  }
  {
    v4f* const mine_sums = reinterpret_cast<v4f*>(mine_lds) + col * (16 * DC);
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        mine_sums[(8 * t + r / 2 + grp) ^ (col & 7)] = v4f{acc[t][r], acc[t][r + 1], acc[t][r + 2], acc[t][r + 3]};
  }
  __syncthreads();
  for (unsigned r = threadIdx.x / 8; r < tile.rows; r += W * kWave / 8) {
    const unsigned j0 = threadIdx.x % 8;
    float m = -INFINITY, l = 0.f, weight[W];
#pragma unroll
    for (unsigned w = 0; w < W; ++w) m = fmaxf(m, stat[0][w][r]);
#pragma unroll
    for (unsigned w = 0; w < W; ++w) {
      weight[w] = __builtin_amdgcn_exp2f(stat[0][w][r] - finite_or_0(m));
      l = fmaf(weight[w], stat[1][w][r], l);
    }
    const uint2 at = row_at(r);
    T* const out = static_cast<T*>(p.out) + (size_t)at.x * p.ldo + (size_t)at.y * d;
    float* const parts = p.part + ((size_t)to_part * kRows + r) * (dv + 4);
    const char* const first = smem + NP * U * 1024 + r * (256 * DC);
#pragma unroll
    for (int j = 0; j < 2 * DC; ++j) {
      const unsigned c4 = j0 + 8 * j, c = 4 * c4;
      if (c >= dv) continue;
      v4f x = {};
#pragma unroll
      for (unsigned w = 0; w < W; ++w) x += weight[w] * *reinterpret_cast<const v4f*>(first + w * kWaveBytes<DC> + (c4 ^ (r & 7)) * 16);
      if (!part.whole) {
        *reinterpret_cast<v4f*>(parts + c) = x;
        continue;
      }
      typedef T t4 __attribute__((ext_vector_type(4)));
      t4 v;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = (T)(l == 0.f ? 0.f : __fdiv_rn(x[k], l));
      if ((vec & 2) && c < d) {
        *reinterpret_cast<t4*>(out + c) = v;
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (c + k < d) out[c + k] = v[k];
      }
    }
    if (!part.whole && j0 == 0) *reinterpret_cast<float2*>(parts + dv) = make_float2(m, l);
  }
}

// One workgroup for each tile and kv head, or equal shares (SHARES).  (Two waves a SIMD where 256 registers do: the compiler then
// leaves accumulation registers alone, and copies to and from them.)
template <int DT, int DC, bool SHARES>
__global__ __launch_bounds__(kWaves * kWave, DC > 2 ? 1 : 2) void k_chunk_few(const ChunkParams p, int vec) {
  if constexpr (SHARES) {
    __shared__ PlanHere mine;
    if (p.here) plan_here<few_waves(kParts<DT>, DC)>(p, mine);
    each_part(p, p.here ? mine.starts : p.plan, p.here ? mine.tiles : planned(p), [&](const LinePart& part, unsigned to) {
      few_rows<DT, DC>(p, vec, part, to);
      __syncthreads();
    });
  } else {
    // (heads next to each other: on a chip whose workgroups go to its eight XCDs by turns, eight heads have one each)
    const Tile tile = find_tile<kRows>(p, blockIdx.x / p.kv_heads, p.heads / p.kv_heads);
    if (tile.b >= 0) few_rows<DT, DC>(p, vec, LinePart{blockIdx.x % p.kv_heads, 0, 0xffffffffu, 0, true, tile}, 0);
  }
}

// ---- many rows ----------------------------------------------------------------------------------------------------------
//
// A workgroup's waves have 32 rows each and go through the same blocks, which they bring into LDS together, converted to
// bfloat16 once, in operand order.  Scores are 32 tokens ahead: their products stand beside the exponentials of the 32 tokens
// before, and the conversions of blocks to come beside the products of the values.  One barrier a block; three places in
// LDS for keys, since this block's and the next one's are read while those of the one after come, two for values.
// The scale of a block's values goes into the exponent (for binary32, whose 24 bits the logarithm would cost some, into a product).
// Bound by what a SIMD can issue: 32 heads of 128 over 8, four pieces of 300 .. 1100 tokens on 2000 .. 16000, bfloat16, 328 GFLOP
// in 535 us (613 TFLOP/s of 1236 that a large library product reaches; 492 GFLOP of products, since probabilities are two parts).  Of the
// 1043 thousand clocks of a SIMD the matrix unit has 494 and the vector unit 597, which hardly overlap: exponentials, their parts,
// conversions, masks and sums cost more than the products.  One workgroup of eight waves shares each block where registers let two waves
// stay on a SIMD (four of 64 rows each, with probabilities of one part: 714 us, eight of 32 then 526).

// Sums of matrix instructions times a factor, from accumulation registers and back.  (The compiler would otherwise take the
// copies that the vector unit needs out of the branch, into every step.)
template <bool VECTOR>
__device__ __forceinline__ void scale_sums(v16f& o, float factor) {
  if constexpr (VECTOR) {
    o *= factor;
    return;
  }
  asm volatile("" : "+a"(o));
  o *= factor;
  asm volatile("" : "+a"(o));
}

template <int DT, int DC>
struct TileForm {
  // two waves a SIMD where their registers fit
  static constexpr int NP = kParts<DT>, PP = kWeightParts<DT>, W = NP * DC <= 2 ? 8 : 4, kRowsOfWg = W * 32;
  static constexpr int kUnits = 8 * DC;                    // 1 KB pieces of a block's keys, and of its values
  static constexpr size_t kLds = 5 * (size_t)kUnits * 1024;       // three blocks of keys, two of values
  static constexpr bool kFold = PP < 3;
};

template <int DT, int DC>
__device__ __forceinline__ void many_rows(const ChunkParams& p, int vec, const LinePart& part, unsigned to_part) {
  using T = typename Elem<DT>::T;
  using Form = TileForm<DT, DC>;
  constexpr int NP = Form::NP, PP = Form::PP, W = Form::W, NK = 2 * DC, ND = 2 * DC, KU = Form::kUnits;
  extern __shared__ __attribute__((aligned(16))) bf8 tile_lds[];                 // keys [3][KU][64], values [2][KU][64]
  bf8 *const kl = tile_lds, *const vl = tile_lds + 3 * KU * kWave;
  // (unknown to the compiler to be the same each time: it would keep dozens of places and masks from one part to the next)
  unsigned lane = threadIdx.x % kWave, d = p.d;
  asm volatile("" : "+v"(lane), "+s"(d));
  const unsigned wave = __builtin_amdgcn_readfirstlane((threadIdx.x - threadIdx.x % kWave + lane) / kWave), col = lane % 32, grp = lane / 32;
  const unsigned per = p.heads / p.kv_heads, dk = kv_dk(d), dv = kv_dv(d), kvh = part.kvh, start = part.start;
  const Tile tile = part.tile;
  const unsigned nblocks = (seen_by(p, tile, (tile.row0 + tile.rows - 1) / per) + kKvBlock - 1) / kKvBlock;
  const unsigned count = min(part.end, nblocks) > start ? min(part.end, nblocks) - start : 0;
  // this wave's rows; past the tile's end they repeat its last and are not stored
  const unsigned row = wave * 32 + col, in_seq = tile.row0 + min(row, tile.rows - 1);
  const bool stored = row < tile.rows;
  const uint2 at = make_uint2(tile.first + in_seq / per, kvh * per + in_seq % per);
  const unsigned mine_sees = seen_by(p, tile, in_seq / per);
  const unsigned least = __builtin_amdgcn_readfirstlane(mine_sees);        // (ascends along the rows)

  // what a wave brings: keys piece n: units 2 i, 2 i + 1 with i = wave + W n = t NK + c: token 32 t + col, bytes 32 c + 16 grp ..
  // values piece n: units 2 i, 2 i + 1 with i = wave + W n = 2 tile + half: row 32 tile + col, 8 bytes of either 16 that hold lane
  // group grp's tokens
  constexpr int KP = (2 * NK + W - 1) / W, VP = (2 * ND + W - 1) / W;
  const int32_t* table = p.table + (size_t)tile.b * p.table_width;
  auto look = [&](unsigned i) {
    const size_t pg = start + (size_t)i + lane;
    return table[pg < p.table_width ? pg : p.table_width - 1];
  };
  u4 rk[KP];
  uint2 rv[VP][2];
  float ak = 0.f, av = 0.f;                                // scales of the blocks that rk and rv hold
  int ids_k = look(0), ids_v = ids_k;
  auto block_of = [&](int& ids, unsigned i, bool& there) {
    if (i % kWave == 0 && i > 0) ids = look(i);
    const int block = __builtin_amdgcn_readlane(ids, i % kWave);
    there = block >= 0 && (size_t)block < p.blocks;
    return (size_t)(there ? block : 0) * p.kv_heads + kvh;
  };
  bool there_k = true, there_v = true;
  auto fetch_keys = [&](unsigned i) {
    if (i >= count) return;
    const size_t b = block_of(ids_k, i, there_k);
    const int8_t* kp = p.keys + b * kKvBlock * dk + (size_t)col * dk + grp * 16;
#pragma unroll
    for (int n = 0; n < KP; ++n) {
      const unsigned u = wave + W * n;
      if (W * n + W <= 2 * NK || u < 2 * NK) rk[n] = *reinterpret_cast<const u4*>(kp + (size_t)(u / NK) * 32 * dk + u % NK * 32);
    }
    ak = p.amax[2 * b];
  };
  auto fetch_values = [&](unsigned i) {
    if (i >= count) return;
    const size_t b = block_of(ids_v, i, there_v);
    const int8_t* vp = p.values + b * dv * kKvBlock + grp * 16;
#pragma unroll
    for (int n = 0; n < VP; ++n)
      if (W * n + W <= 2 * ND || wave + W * n < 2 * ND) {
        const unsigned u = wave + W * n;
        const int8_t* row = vp + (size_t)min(32 * (u / 2) + col, dv - 1) * kKvBlock + u % 2 * 8;
        rv[n][0] = *reinterpret_cast<const uint2*>(row);
        rv[n][1] = *reinterpret_cast<const uint2*>(row + 32);
      }
    av = p.amax[2 * b + 1];
  };
  auto put_key = [&](unsigned buf, int n, int s) {
    if (W * n + W <= 2 * NK || wave + W * n < 2 * NK)
      kl[(buf * KU + 2 * (wave + W * n) + s) * kWave + lane] = bf16_of_bytes(rk[n][2 * s], rk[n][2 * s + 1]);
  };
  auto put_value = [&](unsigned buf, int n, int j) {
    if (W * n + W <= 2 * ND || wave + W * n < 2 * ND)
      vl[(buf * KU + 2 * (wave + W * n) + j) * kWave + lane] = bf16_of_bytes(j ? rv[n][0].y : rv[n][0].x, j ? rv[n][1].y : rv[n][1].x);
  };
  // (very small values are put in their unit afterwards, each wave its own: the steps that put them stay in one piece)
  auto put_units = [&](unsigned buf) {
    if (!Form::kFold) return;
    const unsigned unit = uniform_bits(value_scale(av).unit);
    if (unit == 0x3f800000u) return;
#pragma unroll
    for (int n = 0; n < VP; ++n)
      if (W * n + W <= 2 * ND || wave + W * n < 2 * ND)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          bf8& v = vl[(buf * KU + 2 * (wave + W * n) + j) * kWave + lane];
          v = in_units(v, unit);
        }
  };
  auto put_keys = [&](unsigned buf) {
#pragma unroll
    for (int n = 0; n < KP; ++n)
#pragma unroll
      for (int s = 0; s < 2; ++s) put_key(buf, n, s);
  };
  auto put_values = [&](unsigned buf) {
#pragma unroll
    for (int n = 0; n < VP; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) put_value(buf, n, j);
    put_units(buf);
  };
  fetch_keys(0);

  // queries in operand order, a power of two off each row
  bf8 qf[NP][NK * 2];
  const T* src = static_cast<const T*>(p.q) + (size_t)at.x * p.ldq + (size_t)at.y * d;
  float m = 0.f;
  auto query = [&](int u, float (&v)[8]) {
    const unsigned k = 32 * (u / 2) + 16 * grp + 8 * (u % 2), d = again(p.d);
    if (vec & 1) {
      constexpr int W = 16 / sizeof(T);
      typedef T tw __attribute__((ext_vector_type(W)));
#pragma unroll
      for (int j = 0; j < 8; j += W) {
        tw w = {};
        if (k + j < d) w = *reinterpret_cast<const tw*>(src + k + j);
#pragma unroll
        for (int i = 0; i < W; ++i) v[j + i] = (float)w[i];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = k + j < d ? (float)src[k + j] : 0.f;
    }
  };
#pragma unroll
  for (int u = 0; u < NK * 2; ++u) {
    float v[8];
    query(u, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(v[j]) <= 3.402823466e38f ? fabsf(v[j]) : INFINITY);
  }
  m = across32_f(m, fmax2);
  const int e = row_exponent(m);
  const float mul = __uint_as_float((unsigned)(127 - e) << 23) * (p.scale2 < 0.f ? -1.f : 1.f);
  const float qscale = ldexpf(fabsf(p.scale2), e) * (1.f / 127.f);
#pragma unroll
  for (int u = 0; u < NK * 2; ++u) {
    float v[8];
    query(u, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      __bf16 b[NP];
      split_bf16<NP>(m == INFINITY ? NAN : v[j] * mul, b);
#pragma unroll
      for (int i = 0; i < NP; ++i) qf[i][u][j] = b[i];
    }
  }

  float ref = -INFINITY, total = 0.f;
  v16f acc[ND] = {}, sc[2];                    // sums; scores of a block's two halves
  // a half block's scores take STEPS products a row tile and part, its sums of values as many: their pieces are asked for from
  // LDS four products ahead
  constexpr int STEPS = NK * 2, AHEAD = 4;
  static_assert(STEPS == 2 * ND && STEPS % AHEAD == 0, "");
  bf8 piece[AHEAD];
  auto read_key = [&](const bf8* ku, auto half, int u) __attribute__((always_inline)) {
    constexpr int t = decltype(half)::value;
    piece[u % AHEAD] = ku[(2 * (t * NK + u / 2) + u % 2) * kWave];
  };
  auto score_step = [&](auto half, int u) __attribute__((always_inline)) {
    constexpr int t = decltype(half)::value;
#pragma unroll
    for (int k = NP - 1; k >= 0; --k)
      sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(piece[u % AHEAD], qf[k][u], u == 0 && k == NP - 1 ? v16f{} : sc[t], 0, 0, 0);
  };
  // scales and presence of the block in turn and the next
  float ak_at[2] = {}, av_now = 0.f;
  bool th_at[2] = {true, true};
  if (count > 0) {
    put_keys(0);
    ak_at[0] = ak;
    th_at[0] = there_k;
    fetch_keys(1);
    fetch_values(0);
    put_keys(1);
    ak_at[1] = ak;
    th_at[1] = there_k;
    fetch_keys(2);
    put_values(0);
    av_now = av;
    fetch_values(1);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) read_key(kl + lane, std::integral_constant<int, 0>{}, u);
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
      score_step(std::integral_constant<int, 0>{}, u);
      if (u + AHEAD < STEPS) read_key(kl + lane, std::integral_constant<int, 0>{}, u + AHEAD);
      else read_key(kl + lane, std::integral_constant<int, 1>{}, u + AHEAD - STEPS);
    }
    settle(sc[0]);                             // (later scores have half a block's sums of values behind them)
  }
  unsigned now = 0, next = 1, after = 2;       // places of the keys of blocks i, i + 1, i + 2
  constexpr bool FOLD = Form::kFold;
  float sum = 0.f;                             // of a half block's probabilities times the values' scale, of this lane's tokens
  float inverse = 0.f;                         // of that scale
  for (unsigned i = 0; i < count; ++i) {
    const unsigned pg = start + i, odd = i % 2;
    const bool there = th_at[0];
    float f = there ? qscale * ak_at[0] : 0.f;
    f = f == 0.f ? 1e-30f : f;                 // (0 times a masked score would be NaN; others are below 2^24)
    // (where there is no block, block 0 was read, whose maxima may be anything)
    const float fv = there ? av_now * (1.f / 127.f) : 0.f;
    const ValueScale vs = FOLD ? value_scale(there ? av_now : 0.f) : ValueScale{1.f, 1.f};
    const float lift = __builtin_amdgcn_logf(vs.m), inverse_now = __fdiv_rn(1.f, vs.m);
    const bool masks = !there || (pg + 1) * kKvBlock > least;
    const bf8* vu = vl + (size_t)odd * KU * kWave + lane;
    // half t's exponentials and values, beside them the other half's scores, of this block (t = 0) or the next; keys_then: those
    // of the scores after
    auto half = [&](auto which, const bf8* keys_now, const bf8* keys_then) __attribute__((always_inline)) {
      constexpr int t = decltype(which)::value;
      auto read_value = [&](int u) __attribute__((always_inline)) { piece[u % AHEAD] = vu[(4 * (u % ND) + 2 * t + u / ND) * kWave]; };
      if (masks) {
        const long long room = (long long)mine_sees - (long long)pg * kKvBlock - 4 * (int)grp;
        const int limit = !there || room < 0 ? 0 : room > kKvBlock ? kKvBlock : (int)room;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (limit <= 32 * t + 8 * (r / 4) + r % 4) sc[t][r] = -INFINITY;
      }
      if constexpr (FOLD) {
        total = fmaf(sum, inverse, total);
        sum = 0.f;
        inverse = inverse_now;
      }
      float m = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; r += 2) m = max3(m, sc[t][r], sc[t][r + 1]);
      const float mt = across32_f(m, fmax2) * f;
      if (__builtin_expect(__any(mt > ref + kSlack), 0)) {
        // (only for the rows concerned: no other row's result depends on theirs)
        const float top = mt > ref + kSlack ? mt : ref;
        const float keep = top == ref ? 1.f : __builtin_amdgcn_exp2f(ref - top);
        ref = top;
        total *= keep;
#pragma unroll
        for (int c = 0; c < ND; ++c) scale_sums<Form::W == 8>(acc[c], keep);
      }
      const float base = FOLD ? lift - finite_or_0(ref) : -finite_or_0(ref);
      bf8 pr[PP][2];
      // exponentials [from, end) of the 16 that a lane has of each row
      auto exponentials = [&](int from, int end) __attribute__((always_inline)) {
#pragma unroll
        for (int n = from; n < end; ++n) {
          const float e = __builtin_amdgcn_exp2f(fmaf(sc[t][n], f, base));
          if (!FOLD) total += e;
          __bf16 b[PP];
          split_bf16<PP>(FOLD ? e : e * fv, b);
#pragma unroll
          for (int k = 0; k < PP; ++k) {
            pr[k][n / 8][n % 8] = b[k];
            if (FOLD && n % 2 == 1) sum = add2(pr[k][n / 8][n % 8 - 1], b[k], sum);
          }
        }
      };
      constexpr int EARLY = 12;                // (the others beside the first half of the sums of values)
#pragma unroll
      for (int u = 0; u < STEPS; ++u) {
        score_step(std::integral_constant<int, 1 - t>{}, u);
        if (u + AHEAD < STEPS) read_key(keys_now, std::integral_constant<int, 1 - t>{}, u + AHEAD);
        else read_value(u + AHEAD - STEPS);
        exponentials(u * EARLY / STEPS, (u + 1) * EARLY / STEPS);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int u = 0; u < STEPS; ++u) {
        const int j = u / ND, c = u % ND;
#pragma unroll
        for (int k = PP - 1; k >= 0; --k)
          acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(piece[u % AHEAD], pr[k][j], acc[c], 0, 0, 0);
        if (u + AHEAD < STEPS) read_value(u + AHEAD);
        else read_key(keys_then, std::integral_constant<int, t>{}, u + AHEAD - STEPS);
        if (j == 0) exponentials(EARLY + c * (16 - EARLY) / ND, EARLY + (c + 1) * (16 - EARLY) / ND);
        if constexpr (t == 0) {
#pragma unroll
          for (int n = 0; n < 2 * KP; ++n)
            if (n * STEPS / (2 * KP) == u) put_key(after, n / 2, n % 2);
        } else {
#pragma unroll
          for (int n = 0; n < 2 * VP; ++n)
            if (n * STEPS / (2 * VP) == u) put_value(1 - odd, n / 2, n % 2);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    const bf8 *keys_now = kl + now * KU * kWave + lane, *keys_next = kl + next * KU * kWave + lane;
    half(std::integral_constant<int, 0>{}, keys_now, keys_next);
    ak_at[0] = ak_at[1];
    th_at[0] = th_at[1];
    ak_at[1] = ak;
    th_at[1] = there_k;
    fetch_keys(i + 3);
    half(std::integral_constant<int, 1>{}, keys_next, keys_next);
    put_units(1 - odd);
    av_now = av;
    fetch_values(i + 2);
    const unsigned free = now;
    now = next;
    next = after;
    after = free;
    __syncthreads();
  }

  // every lane has four neighbouring columns of its row at a time
  const float l = across32_f(FOLD ? fmaf(sum, inverse, total) : total, fadd2);
  if (!stored) return;
  if (part.whole) {
    const bool whole = vec & 2;
    T* to = static_cast<T*>(p.out) + (size_t)at.x * p.ldo + (size_t)at.y * d;
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const unsigned c = 32 * t + 2 * r + 4 * grp, end = again(p.d);
        T v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (T)(l == 0.f ? 0.f : __fdiv_rn(acc[t][r + j], l));
        if (whole && c < end) {
          typedef T t4 __attribute__((ext_vector_type(4)));
          *reinterpret_cast<t4*>(to + c) = t4{v[0], v[1], v[2], v[3]};
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (c + j < end) to[c + j] = v[j];
        }
      }
  } else {
    float* to = p.part + ((size_t)to_part * Form::kRowsOfWg + wave * 32 + col) * (dv + 4);
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const unsigned c = 32 * t + 8 * r + 4 * grp;
        if (c < dv) *reinterpret_cast<v4f*>(to + c) = v4f{acc[t][4 * r], acc[t][4 * r + 1], acc[t][4 * r + 2], acc[t][4 * r + 3]};
      }
    if (grp == 0) {
      to[dv] = ref;
      to[dv + 1] = l;
    }
  }
}

template <int DT, int DC>
__global__ __launch_bounds__((TileForm<DT, DC>::W) * kWave, 1) void k_chunk_tiles(const ChunkParams p, int vec) {
  each_part(p, p.plan, planned(p), [&](const LinePart& part, unsigned to) { many_rows<DT, DC>(p, vec, part, to); });
}

// The parts of tiles that more than one workgroup had.  A workgroup for eight rows of a tile and a kv head, 32 threads a row, where
// rows are few and parts may be many; for 32 rows, eight threads a row, where there are many rows of few parts.
constexpr unsigned join_rows(unsigned tile_rows) { return tile_rows > kRows ? 32 : 8; }
template <int DT, unsigned ROWS>
__global__ __launch_bounds__(256) void k_chunk_join(const ChunkParams p, unsigned groups) {
  using T = typename Elem<DT>::T;
  constexpr unsigned JR = join_rows(ROWS), TH = 256 / JR, NX = 64 / TH, AHEAD = TH / 4;      // threads of a row, fours of columns each
  const unsigned chunk = blockIdx.x % (ROWS / JR), kvh = blockIdx.x / (ROWS / JR) % p.kv_heads, slot = blockIdx.x / (ROWS / JR * p.kv_heads);
  const unsigned dv = kv_dv(p.d), pitch = dv + 4, per = p.heads / p.kv_heads;
  const Tile tile = planned(p)[slot];
  const unsigned first = p.plan[slot], last = p.plan[slot + 1];
  const unsigned line = p.plan[p.slots];
  const Share split = share_of(p, line, p.plan[p.slots + 1], groups);
  const unsigned long long share = split.blocks, base = split.pitch * kvh;
  const unsigned r = chunk * JR + threadIdx.x / TH, j0 = threadIdx.x % TH;
  if (tile.b < 0 || r >= tile.rows) return;
  const unsigned g0 = (unsigned)((base + first) / share), g1 = (unsigned)((base + last - 1) / share), runs = g1 - g0 + 1;
  if (runs == 1) return;                                   // (one workgroup had all of it)
  const bool inside = base + first != g0 * share;
  // a workgroup's first part; of the first workgroup its last, if it had other tiles before
  auto run = [&](unsigned i) { return p.part + (((size_t)(g0 + i) * 2 + (i == 0 && inside ? 1 : 0)) * ROWS + r) * pitch; };
  auto over = [](float v, auto op) {                       // the threads of a row
#pragma unroll
    for (int off = TH / 2; off >= 1; off >>= 1) v = op(v, __shfl_xor(v, off, TH));
    return v;
  };
  // references of TH parts at a time, one for each thread
  float m = -INFINITY, l = 0.f;
  for (unsigned i = j0; i < runs; i += TH) m = fmaxf(m, run(i)[dv]);
  const float top = finite_or_0(over(m, fmax2));
  v4f x[NX] = {};
  for (unsigned at = 0; at < runs; at += TH) {
    const float2 stat = *reinterpret_cast<const float2*>(run(min(at + j0, runs - 1)) + dv);
    const bool mine = at + j0 < runs;
    const float w = mine ? __builtin_amdgcn_exp2f(stat.x - top) : 0.f;
    l += over(mine ? w * stat.y : 0.f, fadd2);             // (a row of NaNs has weights of 0 and totals of NaN)
    for (unsigned k = 0; k < min(runs - at, TH); k += AHEAD) {
      v4f v[AHEAD][NX];
#pragma unroll
      for (unsigned i = 0; i < AHEAD; ++i)
#pragma unroll
        for (unsigned j = 0; j < NX; ++j)
          v[i][j] = *reinterpret_cast<const v4f*>(run(min(at + k + i, runs - 1)) + min(4 * (j0 + TH * j), dv - 4));
#pragma unroll
      for (unsigned i = 0; i < AHEAD; ++i) {
        const float wi = __shfl(w, (int)(k + i), TH);
        if (at + k + i >= runs) continue;
#pragma unroll
        for (unsigned j = 0; j < NX; ++j) x[j] += wi * v[i][j];
      }
    }
  }
  const unsigned i = tile.row0 + r;
  T* dst = static_cast<T*>(p.out) + (size_t)(tile.first + i / per) * p.ldo + (size_t)(kvh * per + i % per) * p.d;
#pragma unroll
  for (unsigned j = 0; j < NX; ++j)
#pragma unroll
    for (unsigned k = 0; k < 4; ++k)
      if (4 * (j0 + TH * j) + k < p.d) dst[4 * (j0 + TH * j) + k] = (T)(l == 0.f ? 0.f : __fdiv_rn(x[j][k], l));
}

struct Form {
  bool many, shares;
  unsigned tile_rows, groups, least;  // rows of a tile; workgroups that share the line, blocks that one takes at least
  size_t slots;
};
// The form for many rows is for calls whose rows of a sequence and kv head, on average, fill its tiles (256 or 128 rows; past their rows it
// works for nothing), and that are long enough for its plan, its longer start and its parts, some 30 us.  Few rows / many, us of a call
// (rows, then rows x longest sequence x width of all heads in 10^9):
// heads of 128, 32 over 8, 8 sequences on 4000: bfloat16 (tiles of 256) 160 (5.3) 73 / 77, 192 (6.4) 82 / 79, 256 (8.5) 96 / 85, 288 (9.6) 127 /
//   135, 384 (13) 144 / 128; binary16 (128) 128 (4.2) 66 / 78, 192 (6.4) 106 / 109, 256 127 / 109, 288 146 / 144; binary32 (128) 192 120 / 118,
//   256 149 / 124; 16 over 16, 16 on 2000, binary16, 128 (8.9) 155 / 107, 160 (11) 187 / 192, 192 (14) 223 / 196; 8 over 8, 64 on 1000, 96 (6.9)
//   180 / 128;
// of 64, 16 over 4, 16 on 8000: bfloat16 (256) 256 (8.5) 101 / 103, 384 (13) 148 / 166, 512 (17) 189 / 169; binary32 (128) 256 128 / 131, 384
//   204 / 185; 8 over 8, 64 on 1000: bfloat16 256 (11) 112 / 122, 384 (17) 171 / 230, binary32 256 149 / 156, 512 (25) 326 / 326;
// of 256, 8 over 4, 4 on 4000: bfloat16 (128) 256 (4.3) 77 / 79, 384 (6.6) 101 / 92, 1024 (19) 220 / 163; 8 over 8, 16 on 4000, 64 (8.5) 132 / 143,
//   96 196 / 149; of 192, 16 over 4, 16 on 4000, 128 (6.3) 85 / 92, 192 (9.6) 141 / 133.
constexpr size_t many_work(size_t d) { return d <= 64 ? (size_t)3 << 32 : (size_t)3 << 31; }
constexpr bool many_rows(size_t rows, size_t tile, size_t d) { return rows * 8 >= round_up(rows, tile) * (d <= 64 ? 7 : 6); }
// Blocks of the longest sequence up to which a workgroup takes all of a tile's: where equal shares would be one turn of the waves at
// most (three blocks a workgroup), and else.  One workgroup / shares, us: bfloat16, 32 heads over 8 of 128, 4 new tokens, 1 sequence
// on 1000 tokens 15.2 / 17.5, 1300 18.9 / 15.5, 2000 23.0 / 15.8, 4 on 2000 25.2 / 20.8, 8 on 1300 21.0 / 21.7, 16 on 1700 24.2 / 28.7,
// on 2000 26.3 / 30.2, 32 on 2000 40 / 42; binary32, 8 heads of 64, 16 on 1300 20.1 / 30.7.
constexpr size_t kShort = 18, kLong = 32;
Form form_of(int dtype, size_t B, size_t T, size_t max_len, int heads, int kv_heads, size_t d) {
  const size_t per = (size_t)(heads / kv_heads), blocks = (max_len + kKvBlock - 1) / kKvBlock;
  Form f{};
  const bool wide = (dtype == MQ_BF16 && d <= 128) || (d <= 64 && dtype == MQ_F16);
  const size_t rows = T * per / B, tile = wide ? 256 : 128;
  // (binary32 queries of wide heads do not fit beside the sums)
  f.many = rows > 0 && many_rows(rows, tile, d) && T * (size_t)heads * d >= many_work(d) / max_len && !(dtype == MQ_F32 && d > 128);
  f.shares = f.many || blocks > kLong;
  f.tile_rows = kRows;
  f.least = f.many ? 8 : 4;
  // as many as there is room for at once: registers and LDS hold three (binary32: two), two (of bfloat16) or one; of the form for many rows
  // one of eight waves, and two of four waves (their registers) up to 64 columns only.  (More, in rounds, begin and join again: 32 heads over
  // 8 of 128, binary16, 4 new tokens of 32 sequences on 4000 109 us instead of 79, 32 of 8 90 instead of 65, 256 of 8 364 instead of 336; 8
  // over 4 of 256, bfloat16, 800 of 4 on 4000 275 instead of 236; 8 of 64, binary32, 1 of 64 on 2500 74 instead of 53.)
  f.groups = d <= 64 ? (dtype == MQ_F32 ? 512 : 768) : d <= 128 && dtype == MQ_BF16 ? 512 : 256;
  if (f.many) {
    f.tile_rows = (unsigned)tile;
    f.groups = wide || d > 64 ? 256 : 512;
  }
  f.slots = T * per / f.tile_rows + B;
  if (blocks > kShort && f.slots <= kHere && f.slots * blocks * kv_heads <= (size_t)3 * f.groups) f.shares = true;
  // no more workgroups than there may be shares of the least length
  const size_t least = f.least, line = blocks < ((size_t)1 << 40) / f.slots ? f.slots * blocks * kv_heads : (size_t)1 << 40;
  const size_t most = (line + 8 * least - 1) / (8 * least) * 8;
  if (f.groups > most) f.groups = (unsigned)most;
  return f;
}
// Floats of the parts, in front of the plan.
size_t part_floats(const Form& f, size_t d) { return f.shares ? (size_t)f.groups * 2 * f.tile_rows * (kv_dv((unsigned)d) + 4) : 4; }

}  // namespace

size_t chunk_attention_ws_bytes(size_t B, size_t T, size_t max_len, int heads, int kv_heads, size_t d) {
  size_t most = 0;                    // (whatever the type)
  for (int dtype : {MQ_F32, MQ_F16, MQ_BF16}) {
    const Form f = form_of(dtype, B, T, max_len, heads, kv_heads, d);
    const size_t n = part_floats(f, d) + (f.shares ? (f.slots + 5) / 4 * 4 + f.slots * sizeof(Tile) / sizeof(float) : 0);
    most = n > most ? n : most;
  }
  return most * sizeof(float);
}

int launch_chunk_attention(const mq_kv_cache& cache, const int32_t* table, size_t table_width, const int32_t* first,
                           const int32_t* lens, size_t B, size_t T, size_t max_len, int causal, const void* q, size_t ldq,
                           int heads, int dtype, float scale, void* out, size_t ldo, void* ws, hipStream_t s) {
  const Form form = form_of(dtype, B, T, max_len, heads, cache.kv_heads, cache.head_dim);
  const size_t tiles = form.slots * (size_t)cache.kv_heads, joins = tiles * (form.tile_rows / join_rows(form.tile_rows));
  const size_t blocks = (max_len + kKvBlock - 1) / kKvBlock;
  // (parts are joined where shares are equal only, and there blocks of all tiles are counted in 32 bits, with room for sums)
  if (!launchable(form.shares ? joins : tiles, kWaves * kWave) || form.slots > (((size_t)1 << 31) - 1) / blocks) return MQ_ERR_SHAPE;
  float* part = static_cast<float*>(ws);
  const ChunkParams p{cache.keys, cache.values, cache.amax, table, first, lens, q, out, part, ldq, ldo,
                      table_width, cache.blocks, (unsigned)B, (unsigned)T, (unsigned)max_len, (unsigned)cache.kv_heads,
                      (unsigned)heads, (unsigned)cache.head_dim, scale * 1.44269504088896340736f, causal,
                      reinterpret_cast<unsigned*>(part + part_floats(form, cache.head_dim)), (unsigned)form.slots, form.least,
                      !form.many && form.slots <= kHere};
  const size_t piece = 16 / elem_bytes(dtype);
  // whole 16-byte pieces of queries, four neighbouring results at once
  const int vec = (cache.head_dim % piece == 0 && ldq % piece == 0 && reinterpret_cast<uintptr_t>(q) % 16 == 0 ? 1 : 0) |
                  (cache.head_dim % 4 == 0 && ldo % 4 == 0 && reinterpret_cast<uintptr_t>(out) % (4 * elem_bytes(dtype)) == 0 ? 2 : 0);
  return with_dtype(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    auto sized = [&](auto dc) {
      constexpr int DC = decltype(dc)::value;
      if (form.many) {
        if constexpr (!(DT == MQ_F32 && DC > 2)) {
          using Tiles = TileForm<DT, DC>;
          constexpr unsigned ROWS = Tiles::kRowsOfWg;
          auto kern = k_chunk_tiles<DT, DC>;
          if (Tiles::kLds > 65536) {
            const int rc = check_hip(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)Tiles::kLds));
            if (rc != MQ_OK) return rc;
          }
          hipLaunchKernelGGL(k_chunk_plan<ROWS>, dim3(1), dim3(kPlan), 0, s, p, form.groups);
          hipLaunchKernelGGL(kern, dim3(form.groups), dim3(Tiles::W * kWave), Tiles::kLds, s, p, vec);
          hipLaunchKernelGGL((k_chunk_join<DT, ROWS>), dim3((unsigned)joins), dim3(256), 0, s, p, form.groups);
        }
        return check_hip(hipGetLastError());
      }
      constexpr unsigned waves = few_waves(kParts<DT>, DC);
      constexpr size_t lds = (size_t)kParts<DT> * DC * 4096 + waves * kWaveBytes<DC>;
      auto go = [&](auto kern, unsigned grid) {
        if (lds > 65536) {
          const int rc = check_hip(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
          if (rc != MQ_OK) return rc;
        }
        hipLaunchKernelGGL(kern, dim3(grid), dim3(waves * kWave), lds, s, p, vec);
        return check_hip(hipGetLastError());
      };
      if (!form.shares) {
        return go(k_chunk_few<DT, DC, false>, (unsigned)tiles);
      }
      if (!p.here) hipLaunchKernelGGL(k_chunk_plan<kRows>, dim3(1), dim3(kPlan), 0, s, p, form.groups);
      if (const int rc = go(k_chunk_few<DT, DC, true>, form.groups); rc != MQ_OK) return rc;
      hipLaunchKernelGGL((k_chunk_join<DT, kRows>), dim3((unsigned)joins), dim3(256), 0, s, p, form.groups);
      return check_hip(hipGetLastError());
    };
    switch (kv_dk(p.d) / 64) {
      case 1: return sized(std::integral_constant<int, 1>{});
      case 2: return sized(std::integral_constant<int, 2>{});
      case 3: return sized(std::integral_constant<int, 3>{});
      default: return sized(std::integral_constant<int, 4>{});
    }
  });
}

}  // namespace mq
