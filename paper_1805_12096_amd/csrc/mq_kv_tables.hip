// Tables of continued sequences and compaction of the paged cache (include/mq_serve.h).
//
// Who uses a block says the new table alone, so there is no count of references that could go wrong: a word for each block
// takes the minimum of what its users want of it, 0 for reading (or keeping), b + 1 for row b that will write to it.  Minima of
// integers do not depend on their order.  A row keeps a block that it writes to iff the word is its own; blocks whose word was
// never touched are free.
// Two forms: where tables and cache are small, one workgroup does all but the copies with the words in LDS; else the words lie in
// the workspace and clearing, counting, handing out and writing are launches of their own.  Bound by launches and by chains of
// dependent loads (parent, length, entry) where little is copied, by the copies' bytes where much is: 300 rows of 5 columns 14 us
// (in four launches 20), of which the tables are 5; 90 rows compacted 13 (19); 226 MB of moved blocks in 47 of 58 us, 4.8 TB/s.
#include "mq_serve_common.h"

namespace mq {

namespace {

constexpr int kT = 256;
constexpr int kScan = 1024;           // threads of the workgroup that counts
constexpr int kFree = 0x7fffffff;

struct Tables {
  const int32_t *keep, *table, *lens, *parent, *grow;
  int32_t *table_new, *lens_new, *missing, *moved, *used;
  int32_t *state, *list, *offset;     // a word for each block; blocks handed out in order, or moves; rows' first needs
  size_t width;
  unsigned B, B_new, blocks;
};

struct RowOf {
  const int32_t* entries;
  unsigned len, held, end;
  bool open;                          // whether the last block held will be written to
};
__device__ __forceinline__ RowOf row_of(const Tables& p, size_t b) {
  const int parent = p.parent == nullptr ? (int)b : p.parent[b];
  const bool known = parent >= 0 && (unsigned)parent < p.B;
  const int n = known ? p.lens[parent] : 0, more = p.grow == nullptr ? 0 : p.grow[b];
  const unsigned long long room = (unsigned long long)p.width * kKvBlock;
  const unsigned len = n < 0 ? 0u : (unsigned long long)n < room ? (unsigned)n : (unsigned)room;
  const unsigned held = (len + kKvBlock - 1) / kKvBlock;
  const unsigned long long end = ((unsigned long long)len + (more > 0 ? (unsigned)more : 0u) + kKvBlock - 1) / kKvBlock;
  return {p.table + (size_t)(known ? parent : 0) * p.width, len, held, (unsigned)(end < p.width ? end : p.width),
          more > 0 && len % kKvBlock != 0};
}
__device__ __forceinline__ bool is_block(const Tables& p, int e) { return e >= 0 && (unsigned)e < p.blocks; }

__global__ __launch_bounds__(kT) void k_tables_clear(const Tables p) {
  for (size_t i = (size_t)blockIdx.x * kT + threadIdx.x; i < p.blocks; i += (size_t)gridDim.x * kT)
    p.state[i] = p.keep != nullptr && p.keep[i] != 0 ? 0 : kFree;
}

// a wave for each row
__global__ __launch_bounds__(kT) void k_tables_count(const Tables p) {
  const size_t b = (size_t)blockIdx.x * (kT / kWave) + threadIdx.x / kWave;
  if (b >= p.B_new) return;
  const RowOf r = row_of(p, b);
  for (unsigned j = threadIdx.x % kWave; j < r.held; j += 4 * kWave) {
    int e[4];                                              // (four loads at a time)
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = r.entries[min(j + i * kWave, r.held - 1)];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned at = j + i * kWave;
      if (at < r.held && is_block(p, e[i])) atomicMin(p.state + e[i], r.open && at + 1 == r.held ? (int)b + 1 : 0);      // (nobody waits)
    }
  }
}

// sum over the threads in front of this one of the workgroup's kScan, and over all
__device__ __forceinline__ unsigned scan(unsigned v, unsigned* box, unsigned& all) {
  const unsigned lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  unsigned x = v;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const unsigned y = __shfl_up(x, off, kWave);
    if (lane >= (unsigned)off) x += y;
  }
  __syncthreads();
  if (lane == kWave - 1) box[wave] = x;
  __syncthreads();
  unsigned ahead = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < kScan / kWave; ++w) {
    if (w < (int)wave) ahead += box[w];
    all += box[w];
  }
  return ahead + x - v;
}

// Whether row b, which writes to its last block, needs a copy of it.
__device__ __forceinline__ bool copies(const Tables& p, const RowOf& r, size_t b) {
  if (!r.open) return false;
  const int e = r.entries[r.held - 1];
  return is_block(p, e) && p.state[e] != (int)b + 1;
}

__global__ __launch_bounds__(kScan) void k_fork_assign(const Tables p) {
  __shared__ unsigned box[kScan / kWave];
  unsigned needs = 0;
  for (size_t at = 0; at < p.B_new; at += kScan) {
    const size_t b = at + threadIdx.x;
    unsigned mine = 0, all;
    if (b < p.B_new) {
      const RowOf r = row_of(p, b);
      mine = r.end - r.held + (copies(p, r, b) ? 1 : 0);
    }
    const unsigned before = scan(mine, box, all);
    if (b < p.B_new) p.offset[b] = (int)min(needs + before, p.blocks);
    needs = needs + all < needs ? 0xffffffffu : needs + all;
  }
  // free blocks, as many as are needed
  unsigned found = 0;
  for (size_t at = 0; at < p.blocks && found < needs; at += kScan) {
    const size_t i = at + threadIdx.x;
    const bool free = i < p.blocks && p.state[i] == kFree;
    unsigned all;
    const unsigned before = scan(free, box, all);
    if (free) p.list[found + before] = (int)i;
    found += all;
  }
  if (threadIdx.x == 0) {
    p.offset[p.B_new] = (int)min(found, needs);
    *p.missing = needs > found ? (int)min(needs - found, 0x7fffffffu) : 0;
  }
}

// Copies a block of the cache by all threads of `groups` workgroups, of which this is the g-th.
__device__ __forceinline__ void copy_block(const mq_kv_cache& c, size_t from, size_t to, unsigned g, unsigned groups) {
  const size_t kb = (size_t)c.kv_heads * kKvBlock * kv_dk((unsigned)c.head_dim), vb = (size_t)c.kv_heads * kKvBlock * kv_dv((unsigned)c.head_dim);
  const u4 *ks = reinterpret_cast<const u4*>(c.keys + from * kb), *vs = reinterpret_cast<const u4*>(c.values + from * vb);
  u4 *kd = reinterpret_cast<u4*>(c.keys + to * kb), *vd = reinterpret_cast<u4*>(c.values + to * vb);
  for (size_t i = (size_t)g * kT + threadIdx.x; i < kb / 16; i += (size_t)groups * kT) kd[i] = ks[i];
  for (size_t i = (size_t)g * kT + threadIdx.x; i < vb / 16; i += (size_t)groups * kT) vd[i] = vs[i];
  if (g == 0)
    for (unsigned i = threadIdx.x; i < 2u * c.kv_heads; i += kT) c.amax[to * 2 * c.kv_heads + i] = c.amax[from * 2 * c.kv_heads + i];
}

// `groups` workgroups for each row: the row's entries by the first, its copy by all
__global__ __launch_bounds__(kT) void k_fork_write(const Tables p, const mq_kv_cache c, unsigned groups) {
  const size_t b = blockIdx.x / groups;
  const unsigned g = blockIdx.x % groups;
  const RowOf r = row_of(p, b);
  const bool copy = copies(p, r, b);
  const unsigned given = (unsigned)p.offset[p.B_new], first = (unsigned)p.offset[b];
  auto handed = [&](unsigned long long i) { return i < given ? p.list[i] : -1; };
  if (g == 0) {
    int32_t* to = p.table_new + b * p.width;
    for (size_t j = threadIdx.x; j < p.width; j += kT) {
      int e = -1;
      if (j < r.held && !(copy && j + 1 == r.held)) {
        e = r.entries[j];
        if (!is_block(p, e)) e = -1;
      } else if (j < r.end) {
        e = handed((unsigned long long)first + (copy ? 1 : 0) + j - r.held);
      }
      to[j] = e;
    }
    if (threadIdx.x == 0) p.lens_new[b] = (int)r.len;
  }
  if (copy) {
    const int to = handed(first);
    if (to >= 0) copy_block(c, r.entries[r.held - 1], to, g, groups);
  }
}

// Used blocks are counted, then the holes below their number and the used blocks from there on are listed.
__global__ __launch_bounds__(kScan) void k_compact_plan(const Tables p) {
  __shared__ unsigned box[kScan / kWave];
  unsigned mine = 0, used;
  for (size_t i = threadIdx.x; i < p.blocks; i += kScan) mine += p.state[i] != kFree;
  scan(mine, box, used);
  unsigned holes = 0, moves = 0;
  int32_t* from = p.list;
  int32_t* to = p.list + p.blocks / 2 + 1;                 // (at most half of the blocks move)
  for (size_t at = 0; at < p.blocks; at += kScan) {
    const size_t i = at + threadIdx.x;
    const bool is = i < p.blocks && p.state[i] != kFree, hole = i < used && !is, move = i >= used && is;
    unsigned all;
    const unsigned before = scan((hole ? 1u : 0u) | (move ? 1u << 16 : 0u), box, all);
    if (hole) to[holes + (before & 0xffffu)] = (int)i;
    if (move) from[moves + (before >> 16)] = (int)i;
    if (i < p.blocks) p.moved[i] = is ? (int)i : -1;
    holes += all & 0xffffu;
    moves += all >> 16;
  }
  __syncthreads();                                         // (the lists are this workgroup's own)
  for (unsigned i = threadIdx.x; i < moves; i += kScan) p.moved[from[i]] = to[i];
  if (threadIdx.x == 0) {
    *p.used = (int)used;
    p.offset[0] = (int)moves;
  }
}

// workgroups [0, rows) write the table, the others copy
__global__ __launch_bounds__(kT) void k_compact_apply(const Tables p, const mq_kv_cache c, unsigned table_wgs, unsigned groups) {
  if (blockIdx.x < table_wgs) {
    for (size_t b = blockIdx.x; b < p.B; b += table_wgs) {
      const RowOf r = row_of(p, b);
      for (size_t j = threadIdx.x; j < p.width; j += kT) {
        const int e = j < r.held ? r.entries[j] : -1;
        p.table_new[b * p.width + j] = is_block(p, e) ? p.moved[e] : -1;
      }
    }
    return;
  }
  const unsigned wg = blockIdx.x - table_wgs, movers = (gridDim.x - table_wgs) / groups, moves = (unsigned)p.offset[0];
  const int32_t *from = p.list, *to = p.list + p.blocks / 2 + 1;
  for (unsigned i = wg / groups; i < moves; i += movers) copy_block(c, from[i], to[i], wg % groups, groups);
}

// ---- small tables ---------------------------------------------------------------------------------------------------------

constexpr size_t kSmallBlocks = 8192, kSmallRows = 4096, kSmallEntries = 16384;
// words and a list of the blocks, then the rows
constexpr size_t small_lds(size_t blocks, size_t rows) { return 2 * round_up(blocks, 2) * sizeof(int32_t) + rows * sizeof(int4); }

// A row in LDS: its parent (-1: none), tokens, end of its blocks (below 0: its last one held will be written to), first new block.
__device__ __forceinline__ unsigned held_of(const int4& r) { return ((unsigned)r.y + kKvBlock - 1) / kKvBlock; }
__device__ __forceinline__ unsigned end_of(const int4& r) { return (unsigned)r.z & 0x7fffffffu; }

// The rows and the words of the blocks, in LDS.  A thread for each row, then for each entry: loads that depend on each other are
// few, and all rows' at once.
__device__ __forceinline__ void count_small(const Tables& p, int32_t* state, int4* rows) {
  for (unsigned b = threadIdx.x; b < p.B_new; b += kScan) {
    const RowOf r = row_of(p, b);
    rows[b] = make_int4((int)((r.entries - p.table) / p.width), (int)r.len, (int)(r.end | (r.open ? 0x80000000u : 0u)), 0);
  }
  for (unsigned i = threadIdx.x; i < p.blocks; i += kScan) state[i] = p.keep != nullptr && p.keep[i] != 0 ? 0 : kFree;
  __syncthreads();
  const unsigned width = (unsigned)p.width, entries = p.B_new * width;
  for (unsigned at = threadIdx.x; at < entries; at += 4 * kScan) {
    int e[4];                                              // (four loads at a time)
#pragma unroll
    for (unsigned k = 0; k < 4; ++k) {
      const unsigned i = min(at + k * kScan, entries - 1);
      e[k] = p.table[(size_t)rows[i / width].x * width + i % width];
    }
#pragma unroll
    for (unsigned k = 0; k < 4; ++k) {
      const unsigned i = at + k * kScan, b = i / width, j = i % width;
      if (i >= entries) break;
      const unsigned held = held_of(rows[b]);
      if (j < held && is_block(p, e[k])) atomicMin(state + e[k], rows[b].z < 0 && j + 1 == held ? (int)b + 1 : 0);
    }
  }
  __syncthreads();
}

// Everything of a fork but the copies, which row b's pair (from, to) at p.list + 2 b says; to < 0: none.
__global__ __launch_bounds__(kScan) void k_fork_small(const Tables p) {
  extern __shared__ __attribute__((aligned(16))) int32_t words[];
  __shared__ unsigned box[kScan / kWave];
  const unsigned half = (p.blocks + 1) / 2 * 2;
  int32_t *state = words, *list = words + half;
  int4* rows = reinterpret_cast<int4*>(words + 2 * half);
  count_small(p, state, rows);
  unsigned found = 0;
  for (unsigned at = 0; at < p.blocks; at += kScan) {
    const unsigned i = at + threadIdx.x;
    const bool free = i < p.blocks && state[i] == kFree;
    unsigned all;
    const unsigned before = scan(free, box, all);
    if (free) list[found + before] = (int)i;
    found += all;
  }
  __syncthreads();
  const unsigned width = (unsigned)p.width;
  unsigned needs = 0;
  for (unsigned at = 0; at < p.B_new; at += kScan) {
    const unsigned b = at + threadIdx.x;
    unsigned mine = 0, all;
    int from = -1;
    int4 r{};
    if (b < p.B_new) {
      r = rows[b];
      const unsigned held = held_of(r);
      if (r.z < 0) {
        const int e = p.table[(size_t)r.x * width + held - 1];
        if (is_block(p, e) && state[e] != (int)b + 1) from = e;
      }
      mine = end_of(r) - held + (from >= 0 ? 1 : 0);
    }
    const unsigned first = needs + scan(mine, box, all);
    needs += all;
    if (b < p.B_new) {
      const int to = from >= 0 && first < found ? list[first] : -1;
      reinterpret_cast<int2*>(p.list)[b] = make_int2(from, to);
      p.lens_new[b] = r.y;
      // (what the last pass needs: whether the last block held is a copy, and which)
      rows[b].w = (int)(first + (from >= 0 ? 1 : 0));
      rows[b].z = (int)(end_of(r) | (from >= 0 ? 0x80000000u : 0u));
    }
  }
  __syncthreads();
  for (unsigned i = threadIdx.x; i < p.B_new * width; i += kScan) {
    const unsigned b = i / width, j = i % width;
    const int4 r = rows[b];
    const unsigned held = held_of(r);
    int e = -1;
    if (j < held && !(r.z < 0 && j + 1 == held)) {
      e = p.table[(size_t)r.x * width + j];
      if (!is_block(p, e)) e = -1;
    } else if (j < end_of(r)) {
      const unsigned at = (unsigned)r.w + j - held;        // (a copy: one in front of the first)
      e = at < found ? list[at] : -1;
    }
    p.table_new[i] = e;
  }
  if (threadIdx.x == 0) *p.missing = needs > found ? (int)(needs - found) : 0;
}

__global__ __launch_bounds__(kT) void k_fork_copy(const int32_t* pairs, const mq_kv_cache c, unsigned groups) {
  const int2 pair = reinterpret_cast<const int2*>(pairs)[blockIdx.x / groups];
  if (pair.y >= 0) copy_block(c, pair.x, pair.y, blockIdx.x % groups, groups);
}

// Everything of a compaction but the copies: pairs (from, to) at p.list, their number at p.offset.
__global__ __launch_bounds__(kScan) void k_compact_small(const Tables p) {
  extern __shared__ __attribute__((aligned(16))) int32_t words[];
  __shared__ unsigned box[kScan / kWave];
  const unsigned half = (p.blocks + 1) / 2 * 2;
  int32_t *state = words, *holes = words + half;           // a block's word becomes where it is afterwards
  int4* rows = reinterpret_cast<int4*>(words + 2 * half);
  count_small(p, state, rows);
  unsigned mine = 0, used;
  for (unsigned i = threadIdx.x; i < p.blocks; i += kScan) mine += state[i] != kFree;
  scan(mine, box, used);
  unsigned n_holes = 0, moves = 0;
  for (unsigned at = 0; at < p.blocks; at += kScan) {
    const unsigned i = at + threadIdx.x;
    const bool is = i < p.blocks && state[i] != kFree, hole = i < used && !is, move = i >= used && is;
    unsigned all;
    const unsigned before = scan((hole ? 1u : 0u) | (move ? 1u << 16 : 0u), box, all);
    // holes lie below `used`, so that all are listed before the first block that moves is met -- but for those of the same round
    if (hole) holes[n_holes + (before & 0xffffu)] = (int)i;
    __syncthreads();
    int to = is ? (int)i : -1;
    if (move) {
      to = holes[moves + (before >> 16)];
      reinterpret_cast<int2*>(p.list)[moves + (before >> 16)] = make_int2((int)i, to);
    }
    if (i < p.blocks) {
      p.moved[i] = to;
      state[i] = to;
    }
    n_holes += all & 0xffffu;
    moves += all >> 16;
  }
  __syncthreads();
  const unsigned width = (unsigned)p.width;
  const unsigned entries = p.B * width;
  for (unsigned at = threadIdx.x; at < entries; at += 4 * kScan) {
    int e[4];
#pragma unroll
    for (unsigned k = 0; k < 4; ++k) e[k] = p.table[min(at + k * kScan, entries - 1)];
#pragma unroll
    for (unsigned k = 0; k < 4; ++k) {
      const unsigned i = at + k * kScan;
      if (i < entries) p.table_new[i] = i % width < held_of(rows[i / width]) && is_block(p, e[k]) ? state[e[k]] : -1;
    }
  }
  if (threadIdx.x == 0) {
    *p.used = (int)used;
    p.offset[0] = (int)moves;
  }
}

__global__ __launch_bounds__(kT) void k_compact_copy(const int32_t* pairs, const int32_t* moves, const mq_kv_cache c, unsigned groups) {
  const unsigned movers = gridDim.x / groups, n = (unsigned)moves[0];
  for (unsigned i = blockIdx.x / groups; i < n; i += movers) {
    const int2 pair = reinterpret_cast<const int2*>(pairs)[i];
    copy_block(c, pair.x, pair.y, blockIdx.x % groups, groups);
  }
}

// workgroups that share a copy: 16 KB each
unsigned copy_groups(const mq_kv_cache& c) {
  const size_t bytes = (size_t)c.kv_heads * kKvBlock * (kv_dk((unsigned)c.head_dim) + kv_dv((unsigned)c.head_dim));
  return (unsigned)((bytes + 16383) / 16384);
}
int allow_lds(const void* kernel, size_t bytes) {
  return bytes <= 65536 ? (int)MQ_OK : check_hip(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
}
unsigned clear_wgs(size_t blocks) { return (unsigned)((blocks + kT - 1) / kT < 1024 ? (blocks + kT - 1) / kT : 1024); }

}  // namespace

size_t kv_fork_ws_bytes(size_t blocks, size_t B_new, size_t) {
  const size_t words = 2 * blocks > 2 * B_new ? 2 * blocks : 2 * B_new;        // words and list, or pairs
  return (words + B_new + 1) * sizeof(int32_t);
}
size_t kv_compact_ws_bytes(size_t blocks) { return (2 * blocks + 4) * sizeof(int32_t); }

int launch_kv_fork(const mq_kv_cache& cache, const int32_t* keep, const int32_t* table, size_t table_width, const int32_t* lens,
                   size_t B, const int32_t* parent, const int32_t* grow, size_t B_new, int32_t* table_new, int32_t* lens_new,
                   int32_t* missing, void* ws, hipStream_t s) {
  const unsigned groups = copy_groups(cache);
  if (!launchable(B_new * groups, kT)) return MQ_ERR_SHAPE;
  int32_t* w = static_cast<int32_t*>(ws);
  if (cache.blocks <= kSmallBlocks && B_new <= kSmallRows && B_new <= kSmallEntries / table_width) {
    const size_t lds = small_lds(cache.blocks, B_new);
    if (const int rc = allow_lds(reinterpret_cast<const void*>(k_fork_small), lds); rc != MQ_OK) return rc;
    const Tables p{keep, table, lens, parent, grow, table_new, lens_new, missing, nullptr, nullptr, nullptr, w, w + 2 * B_new,
                   table_width, (unsigned)B, (unsigned)B_new, (unsigned)cache.blocks};
    hipLaunchKernelGGL(k_fork_small, dim3(1), dim3(kScan), lds, s, p);
    hipLaunchKernelGGL(k_fork_copy, dim3((unsigned)(B_new * groups)), dim3(kT), 0, s, w, cache, groups);
    return check_hip(hipGetLastError());
  }
  const Tables p{keep, table, lens, parent, grow, table_new, lens_new, missing, nullptr, nullptr, w, w + cache.blocks,
                 w + 2 * cache.blocks, table_width, (unsigned)B, (unsigned)B_new, (unsigned)cache.blocks};
  hipLaunchKernelGGL(k_tables_clear, dim3(clear_wgs(cache.blocks)), dim3(kT), 0, s, p);
  hipLaunchKernelGGL(k_tables_count, dim3((unsigned)((B_new + 3) / 4)), dim3(kT), 0, s, p);
  hipLaunchKernelGGL(k_fork_assign, dim3(1), dim3(kScan), 0, s, p);
  hipLaunchKernelGGL(k_fork_write, dim3((unsigned)(B_new * groups)), dim3(kT), 0, s, p, cache, groups);
  return check_hip(hipGetLastError());
}

int launch_kv_compact(const mq_kv_cache& cache, const int32_t* keep, const int32_t* table, size_t table_width, const int32_t* lens,
                      size_t B, int32_t* table_new, int32_t* moved, int32_t* used, void* ws, hipStream_t s) {
  if (!launchable((B + 3) / 4, kT)) return MQ_ERR_SHAPE;
  const unsigned groups = copy_groups(cache);
  int32_t* w = static_cast<int32_t*>(ws);
  const size_t most = cache.blocks / 2 + 1;
  const unsigned movers = (unsigned)(most < 512 ? most : 512);
  if (cache.blocks <= kSmallBlocks && B <= kSmallRows && B <= kSmallEntries / table_width) {
    const size_t lds = small_lds(cache.blocks, B);
    if (const int rc = allow_lds(reinterpret_cast<const void*>(k_compact_small), lds); rc != MQ_OK) return rc;
    const Tables p{keep, table, lens, nullptr, nullptr, table_new, nullptr, nullptr, moved, used, nullptr, w, w + 2 * cache.blocks + 2,
                   table_width, (unsigned)B, (unsigned)B, (unsigned)cache.blocks};
    hipLaunchKernelGGL(k_compact_small, dim3(1), dim3(kScan), lds, s, p);
    hipLaunchKernelGGL(k_compact_copy, dim3(movers * groups), dim3(kT), 0, s, w, w + 2 * cache.blocks + 2, cache, groups);
    return check_hip(hipGetLastError());
  }
  const Tables p{keep, table, lens, nullptr, nullptr, table_new, nullptr, nullptr, moved, used, w, w + cache.blocks,
                 w + 2 * cache.blocks + 2, table_width, (unsigned)B, (unsigned)B, (unsigned)cache.blocks};
  hipLaunchKernelGGL(k_tables_clear, dim3(clear_wgs(cache.blocks)), dim3(kT), 0, s, p);
  hipLaunchKernelGGL(k_tables_count, dim3((unsigned)((B + 3) / 4)), dim3(kT), 0, s, p);
  hipLaunchKernelGGL(k_compact_plan, dim3(1), dim3(kScan), 0, s, p);
  const unsigned table_wgs = (unsigned)(B < 1024 ? B : 1024);
  hipLaunchKernelGGL(k_compact_apply, dim3(table_wgs + movers * groups), dim3(kT), 0, s, p, cache, table_wgs, groups);
  return check_hip(hipGetLastError());
}

}  // namespace mq
