// tokens.hip -- new tokens' keys and values into the paged cache, and kept tokens moved together (gfx950).
//
// Copies, bit for bit, between the caller's rows or the cache's own slots and the tiles of the cache: a
// token of one kv head is 16 chunks of 16 bytes in its K tile (256 bytes apart) and 128 elements of 2
// bytes in its V tile (32 bytes apart).  HBM-bound.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "packed_rows.h"
#include "paged_addr.h"
#include "tokens.h"

namespace bana {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

constexpr int kChunks = kHeadDim / 8;  // 16-byte pieces of a token's key or value

// Block of token t of sequence b, or -1 where the table or the pool has none.
__device__ __forceinline__ int block_of(const int32_t* __restrict__ table, const CacheShape& s, int b, int64_t t) {
  if (t < 0 || t >= (int64_t)s.max_blocks * kBlockSize) return -1;
  const int blk = table[(int64_t)b * s.max_blocks + (t >> 4)];
  return blk >= 0 && blk <= s.last_block ? blk : -1;
}

// The same without a branch, so that several lookups are under way at once.
__device__ __forceinline__ int block_of_flat(const int32_t* __restrict__ row, const CacheShape& s, int64_t t) {
  const int64_t end = (int64_t)s.max_blocks * kBlockSize;
  const int blk = row[min(max(t, (int64_t)0), end - 1) >> 4];
  return (t >= 0) & (t < end) & (blk >= 0) & (blk <= s.last_block) ? blk : -1;
}

// One workgroup per (block that new tokens of a sequence fall into, kv head).  The block's K chunk goes straight
// from the rows to the tile (16 bytes per thread, neighbouring threads on neighbouring slots, so the tile's
// writes are contiguous and a row is read in 64-byte pieces); the V rows pass through LDS, from where a thread
// writes 8 tokens of one dim with one store.  Blocks that the new tokens cover in part are written element by
// element.  The x-th block of sequence b is workgroup floor(row_begin[b] / 16) + 2 b + x of its head: n rows
// touch at most floor(n / 16) + 2 blocks.
// HBM-bound.  Measured on MI355X: 48 single tokens 4.4 us, prompts of 8,000 tokens together (8 kv heads, 88 MB)
// 18 us, 4.9 TB/s (a copy reaches 4.75); V element by element 25, a workgroup per row, two bytes of V a store, 88.
__global__ __launch_bounds__(256) void append_kernel(const uint16_t* __restrict__ k_rows,
                                                     const uint16_t* __restrict__ v_rows, int rows,
                                                     const int32_t* __restrict__ row_begin,
                                                     const int32_t* __restrict__ first,
                                                     const int32_t* __restrict__ table, uint16_t* __restrict__ k,
                                                     uint16_t* __restrict__ v, CacheShape s, FastDiv by_hkv,
                                                     float seqs_per_place) {
  constexpr int kPad = kHeadDim + 8;  // LDS row of a token: 16-byte pieces, rows 4 banks apart
  __shared__ __attribute__((aligned(16))) uint16_t sm_v[kBlockSize * kPad];
  const unsigned place = by_hkv.quotient(blockIdx.x);
  const int g = (int)(blockIdx.x - place * s.Hkv);
  auto first_place = [](int i, int row) { return row / kBlockSize + 2 * i; };
  const SeqRows x = find_rows(row_begin, first, rows, s.B, (int)place, seqs_per_place, threadIdx.x & 63,
                              first_place);
  const int b = x.b, r0 = x.begin, n = x.end - x.begin;
  const int64_t t0 = x.value;  // may be negative: those rows are skipped
  const int64_t from = max(t0, (int64_t)0), j = (from >> 4) + ((int)place - first_place(b, r0));
  if (j < (from >> 4) || j * kBlockSize >= t0 + n) return;
  const int blk = block_of(table, s, b, j * kBlockSize);
  if (blk < 0) return;
  const int64_t tile = kv_tile(blk, g, s.Hkv) * kTileElems;
  // Slots [lo, hi) of the block are new; slot x is row r0 + j 16 + x - t0.
  const int lo = (int)max(from - j * kBlockSize, (int64_t)0);
  const int hi = (int)min(t0 + n - j * kBlockSize, (int64_t)kBlockSize);
  const int64_t row0 = r0 + j * kBlockSize - t0;
  {
    const int x = threadIdx.x >> 4, ch = threadIdx.x & 15;
    if (x >= lo && x < hi)
      *reinterpret_cast<u32x4*>(sm_v + x * kPad + 8 * ch) =
          *reinterpret_cast<const u32x4*>(v_rows + ((row0 + x) * s.Hkv + g) * kHeadDim + 8 * ch);
  }
  {
    const int x = threadIdx.x & 15, ch = threadIdx.x >> 4;
    if (x >= lo && x < hi)
      *reinterpret_cast<u32x4*>(k + tile + (ch * kBlockSize + x) * 8) =
          *reinterpret_cast<const u32x4*>(k_rows + ((row0 + x) * s.Hkv + g) * kHeadDim + 8 * ch);
  }
  race_check_delay(threadIdx.x >> 6);
  __syncthreads();
  race_check_barrier();
  const int d = threadIdx.x >> 1, x0 = (threadIdx.x & 1) * 8;
  u16x8 val;
#pragma unroll
  for (int e = 0; e < 8; ++e) val[e] = sm_v[(x0 + e) * kPad + d];  // rows outside [lo, hi) are not used
  uint16_t* to = v + tile + d * kBlockSize + x0;
  if (lo <= x0 && x0 + 8 <= hi) {
    *reinterpret_cast<u16x8*>(to) = val;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (x0 + e >= lo && x0 + e < hi) to[e] = val[e];
  }
}

// Tokens move along their own axis only, so the 8 dims of a K chunk, and any 8 dims of V, of one sequence and kv
// head are moved without regard to any other: 32 workgroups of W wavefronts for each (sequence, kv head).  In
// a step the wavefronts take consecutive places of the list, and all have read before any writes; as
// kept[i] >= i, a later step reads nothing that this one writes.  The next step's kept tokens and their blocks
// are looked up meanwhile, without branches, so that many lookups are under way at once.
//  * K: a lane moves the 16 bytes of one token, kKeyUnroll tokens in flight.
//  * V: kPlaces places for a wavefront, counted from a multiple of 8 tokens.  The blocks they come from (256 bytes
//    each for 8 dims, each read once) pass through LDS, kParts at a time; a lane then gathers 8 places of one dim
//    and writes them with one store.
// HBM-bound where every place moves.  Measured on MI355X: 6 sequences of 9000 tokens, every second one kept, 8 kv
// heads: 80 us for 331 MB (blocks are read whole; 221 MB are kept tokens read and written), 4.2 TB/s.  A workgroup
// for each (sequence, kv head), as below, took 490.
//
// Few kept tokens leave most of these lanes idle, and their 32 workgroups per pair start for nothing.  The kernel below
// has one, which walks 16 tokens at a time and reads V element by element: faster up to a length that grows with the
// number of pairs.  us, below / here: 384 pairs 7 kept 4.4 / 35, 126 kept 20 / 41, 252 kept 37 / 44, 504 kept 91 / 59;
// 48 pairs 63 kept 6.1 / 6.8, 126 kept 10 / 7.0; 8 pairs 63 kept 5.8 / 4.7.
inline int few_kept(unsigned pairs) { return (int)std::min(32 + pairs / 4 * 3, 256u); }

// Wavefronts of a workgroup: 8 where that leaves at most one workgroup to a CU (1 sequence of 30000 tokens, half
// kept: 73 us, with 4 78), else 4, three of which fit on a CU (6 of 9000: 80, with 8 94; four on a CU 95).
constexpr unsigned kFewGroups = 256;
constexpr int kKeyUnroll = 4;
constexpr int kPlaces = 128;  // of a wavefront's V step
constexpr int kParts = 32;    // source blocks of a wavefront in LDS

template <int W>
__device__ __forceinline__ void compact_keys(uint16_t* __restrict__ k, const int32_t* __restrict__ table,
                                             const int32_t* __restrict__ kept, int n, int64_t t0, int b, int g, int ch,
                                             const CacheShape& s) {
  constexpr int kOwn = 64 * kKeyUnroll, kStep = kOwn * W;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t* row = table + (int64_t)b * s.max_blocks;
  int64_t to[kKeyUnroll], of[kKeyUnroll];
  auto look_up = [&](int base) {
    int x[kKeyUnroll], blk[kKeyUnroll], blk_of[kKeyUnroll];
#pragma unroll
    for (int u = 0; u < kKeyUnroll; ++u) x[u] = kept[min(base + 64 * u + lane, n - 1)];
#pragma unroll
    for (int u = 0; u < kKeyUnroll; ++u) {
      blk[u] = block_of_flat(row, s, t0 + base + 64 * u + lane);
      blk_of[u] = block_of_flat(row, s, t0 + x[u]);
    }
#pragma unroll
    for (int u = 0; u < kKeyUnroll; ++u) {
      const int i = base + 64 * u + lane;
      const bool moves = (i < n) & (x[u] > i) & (blk[u] >= 0) & (blk_of[u] >= 0);  // else in its place already
      to[u] = moves ? kv_tile(blk[u], g, s.Hkv) * kTileElems + (ch * kBlockSize + ((t0 + i) & 15)) * 8 : -1;
      of[u] = moves ? kv_tile(blk_of[u], g, s.Hkv) * kTileElems + (ch * kBlockSize + ((t0 + x[u]) & 15)) * 8 : -1;
    }
  };
  if (n <= 0) return;
  look_up(wave * kOwn);
  for (int base = 0; base < n; base += kStep) {
    u32x4 key[kKeyUnroll];
    int64_t at[kKeyUnroll];
    race_check_delay(wave);
#pragma unroll
    for (int u = 0; u < kKeyUnroll; ++u) {
      at[u] = to[u];
      if (of[u] >= 0) key[u] = *reinterpret_cast<const u32x4*>(k + of[u]);
    }
    look_up(base + kStep + wave * kOwn);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // what this wavefront reads has arrived
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kKeyUnroll; ++u)
      if (at[u] >= 0) *reinterpret_cast<u32x4*>(k + at[u]) = key[u];
  }
}

__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <int W>
__device__ __forceinline__ void compact_values(uint16_t* __restrict__ v, const int32_t* __restrict__ table,
                                               const int32_t* __restrict__ kept, int n, int64_t t0, int b, int g,
                                               int dims, const CacheShape& s) {
  constexpr int U = kPlaces / 64;
  constexpr int kStep = kPlaces * W;
  __shared__ __attribute__((aligned(16))) uint16_t sm_parts[W][kParts * 128];  // [block][8 dims][16 tokens]
  __shared__ __attribute__((aligned(16))) uint16_t sm_froms[W][kPlaces];  // 256 x block's number + 2 x slot
  __shared__ int32_t sm_blocks[W][kPlaces];                               // pool block of each number
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = lane >> 3, h = lane & 7;
  uint16_t* sm_part = sm_parts[wave];
  uint16_t* sm_from = sm_froms[wave];
  int32_t* sm_block = sm_blocks[wave];
  const int shift = (int)(t0 & 7);  // place p is token t0 - shift + p, kept entry p - shift
  const int places = shift + n;
  int x[U], from_blk[U], to_blk[U];  // of places 64 u + lane; the block of places 64 u + 8 h on
  const int32_t* row = table + (int64_t)b * s.max_blocks;
  auto look_up = [&](int base) {
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = kept[min(max(base + 64 * u + lane - shift, 0), n - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      to_blk[u] = block_of_flat(row, s, t0 - shift + base + 64 * u + 8 * h);
      from_blk[u] = block_of_flat(row, s, t0 + x[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = base + 64 * u + lane - shift;
      if (base + 64 * u + 8 * h >= places) to_blk[u] = -1;
      if ((i < 0) | (i >= n) | (x[u] < i)) from_blk[u] = -1;
    }
  };
  if (n <= 0) return;
  look_up(wave * kPlaces);
  for (int step = 0; step < places; step += kStep) {
    const int base = step + wave * kPlaces;
    // Number the source blocks: a place opens a new one where its block is not that of the place with a source before.
    int count = 0, last = -1;
    bool moves = false;
    unsigned have[U];  // which of this lane's 8 places have a source
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int own = from_blk[u] >= 0 ? x[u] : -1;
      moves |= own > base + 64 * u + lane - shift;
      const uint64_t valid = __ballot(own >= 0), below = valid & ((uint64_t{1} << lane) - 1);
      const int y = __shfl(own, below != 0 ? 63 - __clzll(below) : 0);
      const int prev = below != 0 ? y : last;  // of the place before that has a source
      const bool opens = own >= 0 && (prev < 0 || (t0 + own) >> 4 != (t0 + prev) >> 4);
      const uint64_t mask = __ballot(opens);
      const int number = count + __popcll(mask & ((2ull << lane) - 1)) - 1;
      sm_from[64 * u + lane] = own >= 0 ? (uint16_t)(number * 256 + 2 * (int)((t0 + own) & 15)) : (uint16_t)0;
      have[u] = (unsigned)(valid >> (8 * h)) & 0xFFu;
      if (opens) sm_block[number] = from_blk[u];
      count += (int)__popcll(mask);
      if (valid != 0) last = __builtin_amdgcn_readlane(own, 63 - __clzll(valid));
    }
    const bool any = __any(moves);
    race_check_delay(wave);
    u16x8 val[U] = {}, from[U];
    int64_t to[U];
    wave_lds_fence();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      from[u] = *reinterpret_cast<const u16x8*>(sm_from + 64 * u + 8 * h);
      to[u] = -1;
      if (to_blk[u] >= 0)
        to[u] = kv_tile(to_blk[u], g, s.Hkv) * kTileElems + (dims * 8 + e) * kBlockSize +
                ((t0 - shift + base + 64 * u + 8 * h) & 15);
    }
    for (int part = 0; any && part < count; part += kParts) {
      const int m = min(kParts, count - part);
      u32x4 y[kParts / 4];
#pragma unroll
      for (int q = 0; q < kParts / 4; ++q) {
        const int d = 4 * q + (lane >> 4);
        if (4 * q < m && d < m)
          y[q] = *reinterpret_cast<const u32x4*>(v + kv_tile(sm_block[part + d], g, s.Hkv) * kTileElems +
                                                 dims * 8 * kBlockSize + (lane & 15) * 8);
      }
#pragma unroll
      for (int q = 0; q < kParts / 4; ++q) {
        const int d = 4 * q + (lane >> 4);
        if (4 * q < m && d < m) *reinterpret_cast<u32x4*>(sm_part + d * 128 + (lane & 15) * 8) = y[q];
      }
      wave_lds_fence();
      const char* mine = reinterpret_cast<const char*>(sm_part) + e * kBlockSize * 2;
      if (count <= kParts) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int j = 0; j < 8; ++j) val[u][j] = *reinterpret_cast<const uint16_t*>(mine + from[u][j]);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const unsigned at = (unsigned)from[u][j] - 256u * part;
            const bool here = at < 256u * m;
            const uint16_t x = *reinterpret_cast<const uint16_t*>(mine + (here ? at : 0u));
            val[u][j] = here ? x : val[u][j];
          }
      }
      wave_lds_fence();
    }
    look_up(base + kStep);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // what this wavefront reads has arrived
    __syncthreads();
    if (any) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (to[u] < 0) continue;
        if (have[u] == 0xFFu) {
          *reinterpret_cast<u16x8*>(v + to[u]) = val[u];
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (have[u] >> j & 1) v[to[u] + j] = val[u][j];
        }
      }
    }
  }
}

template <int W>
__global__ __launch_bounds__(64 * W) void compact_kernel(uint16_t* __restrict__ k, uint16_t* __restrict__ v,
                                                         const int32_t* __restrict__ table,
                                                         const int32_t* __restrict__ first,
                                                         const int32_t* __restrict__ kept, int max_kept,
                                                         const int32_t* __restrict__ n_kept, CacheShape s) {
  // The K chunks of all pairs, then the groups of V dims: mixed, they take 87 us where this takes 80.
  const int pairs = (int)(gridDim.x >> 5), x = (int)(blockIdx.x >> 4), part = (int)(blockIdx.x & 15);
  const bool values = x >= pairs;
  const int pair = values ? x - pairs : x;
  const int b = pair / s.Hkv, g = pair - b * s.Hkv;
  const int n = min(max(n_kept[b], 0), max_kept);
  const int32_t* list = kept + (int64_t)b * max_kept;
  if (values) compact_values<W>(v, table, list, n, first[b], b, g, part, s);
  else compact_keys<W>(k, table, list, n, first[b], b, g, part, s);
}

// Few tokens: one workgroup per (sequence, kv head), 16 kept tokens at a time, a thread for each token and 8 dims.
__global__ __launch_bounds__(256) void compact_few_kernel(uint16_t* __restrict__ k, uint16_t* __restrict__ v,
                                                          const int32_t* __restrict__ table,
                                                          const int32_t* __restrict__ first,
                                                          const int32_t* __restrict__ kept, int max_kept,
                                                          const int32_t* __restrict__ n_kept, CacheShape s) {
  const int b = blockIdx.x / s.Hkv, g = blockIdx.x % s.Hkv;
  const int n = min(max(n_kept[b], 0), max_kept);
  const int64_t t0 = first[b];
  const int i = threadIdx.x & 15, ch = threadIdx.x >> 4;  // token of the step, chunk of 8 dims
  for (int base = 0; base < n; base += 16) {
    int to = -1, of = -1;
    int64_t t_of = 0;
    if (base + i < n) {
      const int x = kept[(int64_t)b * max_kept + base + i];
      t_of = t0 + x;
      if (x > base + i) {  // else in its place already
        to = block_of(table, s, b, t0 + base + i);
        of = block_of(table, s, b, t_of);
      }
    }
    const bool move = to >= 0 && of >= 0;
    race_check_delay(threadIdx.x >> 6);
    u32x4 key;
    u16x8 val;
    if (move) {
      const int64_t tile = kv_tile(of, g, s.Hkv) * kTileElems;
      const int slot = (int)(t_of & 15);
      key = *reinterpret_cast<const u32x4*>(k + tile + (ch * kBlockSize + slot) * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) val[e] = v[tile + (8 * ch + e) * kBlockSize + slot];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // what this wavefront reads has arrived
    __syncthreads();
    if (move) {
      const int64_t tile = kv_tile(to, g, s.Hkv) * kTileElems;
      const int slot = (int)((t0 + base + i) & 15);
      *reinterpret_cast<u32x4*>(k + tile + (ch * kBlockSize + slot) * 8) = key;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[tile + (8 * ch + e) * kBlockSize + slot] = val[e];
    }
  }
}

}  // namespace

hipError_t launch_append(const void* k_rows, const void* v_rows, int rows, const int32_t* row_begin,
                         const int32_t* first, const int32_t* table, void* k, void* v, CacheShape s,
                         hipStream_t stream) {
  const unsigned places = (unsigned)(rows / kBlockSize) + 2 * (unsigned)s.B;
  FastDiv by_hkv;
  by_hkv.set((uint32_t)s.Hkv);
  hipLaunchKernelGGL(append_kernel, dim3(places * (unsigned)s.Hkv), dim3(256), 0, stream,
                     static_cast<const uint16_t*>(k_rows), static_cast<const uint16_t*>(v_rows), rows, row_begin, first,
                     table, static_cast<uint16_t*>(k), static_cast<uint16_t*>(v), s, by_hkv,
                     (float)s.B / (float)places);
  return hipGetLastError();
}

hipError_t launch_compact(void* k, void* v, const int32_t* table, const int32_t* first, const int32_t* kept,
                          int max_kept, const int32_t* n_kept, CacheShape s, hipStream_t stream) {
  const unsigned pairs = (unsigned)s.B * (unsigned)s.Hkv;
  if (max_kept <= few_kept(pairs))
    hipLaunchKernelGGL(compact_few_kernel, dim3(pairs), dim3(256), 0, stream, static_cast<uint16_t*>(k),
                       static_cast<uint16_t*>(v), table, first, kept, max_kept, n_kept, s);
  else if (pairs * 32u <= kFewGroups)
    hipLaunchKernelGGL((compact_kernel<8>), dim3(pairs * 32u), dim3(64 * 8), 0, stream, static_cast<uint16_t*>(k),
                       static_cast<uint16_t*>(v), table, first, kept, max_kept, n_kept, s);
  else
    hipLaunchKernelGGL((compact_kernel<4>), dim3(pairs * 32u), dim3(64 * 4), 0, stream, static_cast<uint16_t*>(k),
                       static_cast<uint16_t*>(v), table, first, kept, max_kept, n_kept, s);
  return hipGetLastError();
}

}  // namespace bana
