// tokens.hip -- new tokens' keys and values into the paged cache, and kept tokens moved together (gfx950).
//
// Copies, bit for bit, between the caller's rows or the cache's own slots and the tiles of the cache: a
// token of one kv head is 16 chunks of 16 bytes in its K tile (256 bytes apart) and 128 elements of 2
// bytes in its V tile (32 bytes apart).  HBM-bound.
#include <hip/hip_runtime.h>
#include <stdint.h>

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

// One workgroup per row: thread (g, chunk) moves 16 bytes of the row's key and of its value.
__global__ __launch_bounds__(256) void append_kernel(const uint16_t* __restrict__ k_rows,
                                                     const uint16_t* __restrict__ v_rows, int rows,
                                                     const int32_t* __restrict__ row_begin,
                                                     const int32_t* __restrict__ first,
                                                     const int32_t* __restrict__ table, uint16_t* __restrict__ k,
                                                     uint16_t* __restrict__ v, CacheShape s) {
  const int r = blockIdx.x;
  const int b = last_at_most(s.B, r, threadIdx.x & 63, [&](int i) { return row_start(row_begin, i, rows); });
  const int r0 = row_start(row_begin, b, rows);
  if (r < r0 || r >= row_start(row_begin, b + 1, rows)) return;
  const int64_t t = (int64_t)first[b] + (r - r0);
  const int blk = block_of(table, s, b, t);
  if (blk < 0) return;
  const int slot = (int)(t & 15);
  for (int x = threadIdx.x; x < s.Hkv * kChunks; x += 256) {
    const int g = x / kChunks, ch = x % kChunks;
    const int64_t row = ((int64_t)r * s.Hkv + g) * kHeadDim + 8 * ch;
    const int64_t tile = kv_tile(blk, g, s.Hkv) * kTileElems;
    *reinterpret_cast<u32x4*>(k + tile + (ch * kBlockSize + slot) * 8) = *reinterpret_cast<const u32x4*>(k_rows + row);
    const u16x8 val = *reinterpret_cast<const u16x8*>(v_rows + row);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[tile + (8 * ch + e) * kBlockSize + slot] = val[e];
  }
}

// One workgroup per (sequence, kv head), 16 kept tokens at a time.  kept[i] >= i, so a step reads nothing
// that an earlier step has written; within a step everything is read before anything is written.
__global__ __launch_bounds__(256) void compact_kernel(uint16_t* __restrict__ k, uint16_t* __restrict__ v,
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
    int64_t from = 0;
    if (base + i < n) {
      const int x = kept[(int64_t)b * max_kept + base + i];
      from = t0 + x;
      if (x > base + i) {
        to = block_of(table, s, b, t0 + base + i);
        of = block_of(table, s, b, from);
      }
    }
    const bool move = to >= 0 && of >= 0;
    u32x4 key;
    u16x8 val;
    if (move) {
      const int64_t tile = kv_tile(of, g, s.Hkv) * kTileElems;
      const int slot = (int)(from & 15);
      key = *reinterpret_cast<const u32x4*>(k + tile + (ch * kBlockSize + slot) * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) val[e] = v[tile + (8 * ch + e) * kBlockSize + slot];
    }
    __syncthreads();
    if (move) {
      const int64_t tile = kv_tile(to, g, s.Hkv) * kTileElems;
      const int slot = (int)((t0 + base + i) & 15);
      *reinterpret_cast<u32x4*>(k + tile + (ch * kBlockSize + slot) * 8) = key;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[tile + (8 * ch + e) * kBlockSize + slot] = val[e];
    }
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_append(const void* k_rows, const void* v_rows, int rows, const int32_t* row_begin,
                         const int32_t* first, const int32_t* table, void* k, void* v, CacheShape s,
                         hipStream_t stream) {
  hipLaunchKernelGGL(append_kernel, dim3((unsigned)rows), dim3(256), 0, stream, static_cast<const uint16_t*>(k_rows),
                     static_cast<const uint16_t*>(v_rows), rows, row_begin, first, table, static_cast<uint16_t*>(k),
                     static_cast<uint16_t*>(v), s);
  return hipGetLastError();
}

hipError_t launch_compact(void* k, void* v, const int32_t* table, const int32_t* first, const int32_t* kept,
                          int max_kept, const int32_t* n_kept, CacheShape s, hipStream_t stream) {
  hipLaunchKernelGGL(compact_kernel, dim3((unsigned)(s.B * s.Hkv)), dim3(256), 0, stream, static_cast<uint16_t*>(k),
                     static_cast<uint16_t*>(v), table, first, kept, max_kept, n_kept, s);
  return hipGetLastError();
}

}  // namespace bana
