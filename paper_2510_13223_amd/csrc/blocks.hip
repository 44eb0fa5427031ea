// blocks.hip -- blocks of the cache handed out, shared and taken back on the device (gfx950).
//
// The state is the block table and one count per block; a block with the count 0 is free, and the lowest
// free numbers are taken first, so there is no free list whose order could depend on timing.  A call
// that takes blocks first makes its plan in one workgroup (what is asked for, whether it can be had, which
// blocks), then carries it out; a plan that cannot be carried out changes nothing but *status.
//
// Bound by the latency of dependent reads, not by their bytes: lengths, table entries, counts, list, each a round trip
// of some 0.7 us, and two launches for a fork.  Measured on MI355X: blocks for 128 drafts of 64 tokens, pool of
// 116,000, 8.6 us; 96 forks of 1500 tokens, 8 kv heads, 12.4 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged_addr.h"
#include "tokens.h"

namespace bana {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;

__device__ __forceinline__ int blocks_of(int64_t tokens) {
  return tokens <= 0 ? 0 : (int)((tokens + kBlockSize - 1) / kBlockSize);
}

// Exclusive prefix sum of x over the workgroup, and the sum of all; every thread calls it.
__device__ __forceinline__ int block_scan(int x, int* sm, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int y = __shfl_up(incl, off);
    if (lane >= off) incl += y;
  }
  __syncthreads();  // sm may still be read from the scan before
  race_check_delay(wave);
  if (lane == 63) sm[wave] = incl;
  __syncthreads();
  race_check_barrier();
  int before = incl - x, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    if (w < wave) before += sm[w];
    all += sm[w];
  }
  *total = all;
  return before;
}

// The free blocks among the counts [base, base + 1024 N), N to a thread, the first `need` of them into
// list[found..]; how many there are.
template <int N>
__device__ __forceinline__ int free_among(const int32_t* __restrict__ refs, int64_t num_blocks, int64_t base,
                                          int64_t need, int64_t found, int32_t* __restrict__ list, int* sm) {
  typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
  const int64_t first = base + (int64_t)threadIdx.x * N;
  unsigned bits = 0;
  if (first + N <= num_blocks) {
    i32x4 x[N / 4];
#pragma unroll
    for (int q = 0; q < N / 4; ++q) x[q] = *reinterpret_cast<const i32x4*>(refs + first + 4 * q);
#pragma unroll
    for (int e = 0; e < N; ++e) bits |= (unsigned)(x[e >> 2][e & 3] == 0) << e;
  } else {
    for (int e = 0; e < N; ++e)
      if (first + e < num_blocks) bits |= (unsigned)(refs[first + e] == 0) << e;
  }
  int total;
  int64_t at = found + block_scan((int)__popc(bits), sm, &total);
  for (; bits != 0 && at < need; bits &= bits - 1, ++at) list[at] = (int32_t)(first + __ffs(bits) - 1);
  return total;
}

// The numbers of the `need` lowest free blocks into list[0..need); the number found (>= need unless there
// are fewer).  Most calls end in the first round, of 4 counts to a thread (draft steps in a pool of 116,000
// blocks: 9 us with 4, 10.3 with 16); in a full pool the rounds of 16 need a quarter of the memory latencies.
__device__ __forceinline__ int64_t find_free(const int32_t* __restrict__ refs, int64_t num_blocks, int64_t need,
                                             int32_t* __restrict__ list, int* sm) {
  if (need == 0) return 0;
  int64_t found = free_among<4>(refs, num_blocks, 0, need, 0, list, sm);
  for (int64_t base = kPlanThreads * 4; base < num_blocks && found < need; base += kPlanThreads * 16)
    found += free_among<16>(refs, num_blocks, base, need, found, list, sm);
  return found;
}

// Workspace: [0] 1 if the plan holds, [2..] 64-bit need; [64, 64 + B) counts or marks, [64 + B, 64 + 2 B) prefix
// sums, then the list of blocks.
__global__ __launch_bounds__(kPlanThreads) void reserve_kernel(int32_t* __restrict__ table,
                                                               const int32_t* __restrict__ lens,
                                                               const int32_t* __restrict__ need,
                                                               int32_t* __restrict__ refs, int64_t num_blocks,
                                                               int32_t* __restrict__ status,
                                                               int32_t* __restrict__ ws, CacheShape s) {
  __shared__ int sm[kPlanWaves];
  int32_t* before = ws + 64;
  int32_t* list = ws + 64 + 2 * (int64_t)s.B;
  int64_t total = 0;
  bool wide = false;
  for (int b0 = 0; b0 < s.B; b0 += kPlanThreads) {
    const int b = b0 + threadIdx.x;
    int count = 0;
    if (b < s.B) {
      const int j1 = blocks_of(need[b]), end = min(j1, s.max_blocks);
      wide |= j1 > s.max_blocks;
      for (int j = blocks_of(lens[b]); j < end; j += 4) {
        int32_t x[4];  // four entries under way at once
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = table[(int64_t)b * s.max_blocks + min(j + u, end - 1)];
#pragma unroll
        for (int u = 0; u < 4; ++u) count += (j + u < end) & (x[u] < 0);
      }
    }
    int sum;
    const int at = block_scan(count, sm, &sum);
    if (b < s.B) before[b] = (int32_t)(total + at);
    total += sum;
  }
  const bool too_wide = __syncthreads_or(wide);
  if (total == 0 && !too_wide) return;
  const int64_t found = too_wide || total > num_blocks ? 0 : find_free(refs, num_blocks, total, list, sm);
  if (too_wide || found < total) {
    if (threadIdx.x == 0) atomicMax(status, too_wide ? 3 : 1);
    return;
  }
  __syncthreads();
  for (int b = threadIdx.x; b < s.B; b += kPlanThreads) {
    const int end = blocks_of(need[b]);
    int at = before[b];
    for (int j = blocks_of(lens[b]); j < end; j += 4) {
      int32_t* entry = table + (int64_t)b * s.max_blocks + j;
      int32_t x[4], fresh[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] = entry[min(u, end - 1 - j)];
#pragma unroll
      for (int u = 0; u < 4; ++u) fresh[u] = list[max(min((int64_t)at + u, total - 1), (int64_t)0)];
#pragma unroll
      for (int u = 0, k = 0; u < 4; ++u) {
        if (j + u >= end || x[u] >= 0) continue;
        const int32_t blk = k == 0 ? fresh[0] : k == 1 ? fresh[1] : k == 2 ? fresh[2] : fresh[3];
        entry[u] = blk;
        refs[blk] = 1;
        ++k, ++at;
      }
    }
  }
}

__device__ __forceinline__ int64_t length_of(const int32_t* __restrict__ lens, int b, const CacheShape& s) {
  return min((int64_t)max(lens[b], 0), (int64_t)s.max_blocks * kBlockSize);
}

__global__ __launch_bounds__(kPlanThreads) void fork_plan_kernel(const int32_t* __restrict__ src,
                                                                 const int32_t* __restrict__ dst, int n,
                                                                 const int32_t* __restrict__ table,
                                                                 const int32_t* __restrict__ lens,
                                                                 int32_t* __restrict__ refs, int64_t num_blocks,
                                                                 int32_t* __restrict__ status,
                                                                 int32_t* __restrict__ ws, CacheShape s) {
  __shared__ int sm[kPlanWaves];
  int32_t* mark = ws + 64;            // [B]: 1 + the fork that writes the sequence, 0: none
  int32_t* list = ws + 64 + s.B;      // [min(n, B)] block of each fork that takes one, in order
  for (int b = threadIdx.x; b < s.B; b += kPlanThreads) mark[b] = 0;
  __syncthreads();
  bool bad = n > s.B;
  for (int i = threadIdx.x; i < n && !bad; i += kPlanThreads) {
    const int d = dst[i], c = src[i];
    bad = d < 0 || d >= s.B || c < 0 || c >= s.B || table[(int64_t)d * s.max_blocks] != -1 ||
          atomicExch(mark + d, 1) != 0;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n && !bad; i += kPlanThreads)
    bad = __hip_atomic_load(mark + src[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != 0;
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) {
      atomicMax(status, 2);
      ws[0] = 0;
    }
    return;
  }
  int64_t total = 0;
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    int sum;
    const int at = block_scan(i < n && length_of(lens, src[i], s) % kBlockSize != 0, sm, &sum);
    if (i < n) mark[i] = (int32_t)(total + at);  // place in the list (the marks are done with)
    total += sum;
  }
  const int64_t found = total > num_blocks ? 0 : find_free(refs, num_blocks, total, list, sm);
  if (found < total) {
    if (threadIdx.x == 0) {
      atomicMax(status, 1);
      ws[0] = 0;
    }
    return;
  }
  __syncthreads();
  for (int64_t i = threadIdx.x; i < total; i += kPlanThreads) refs[list[i]] = 1;
  if (threadIdx.x == 0) ws[0] = 1;
}

// kForkParts workgroups per fork: the shared entries (the first), and the copy of the last block if it is partly
// filled, each a share of its bytes.
constexpr int kForkParts = 8;

__global__ __launch_bounds__(256) void fork_kernel(const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                   u32x4* __restrict__ k, u32x4* __restrict__ v,
                                                   int32_t* __restrict__ table, int32_t* __restrict__ lens,
                                                   int32_t* __restrict__ refs, int32_t* __restrict__ status,
                                                   const int32_t* __restrict__ ws, CacheShape s) {
  if (ws[0] == 0) return;
  const int i = blockIdx.x / kForkParts, part = blockIdx.x % kForkParts;
  const int from = src[i], to = dst[i];
  const int64_t len = length_of(lens, from, s);
  const int whole = (int)(len / kBlockSize);
  const int32_t* of = table + (int64_t)from * s.max_blocks;
  int32_t* entry = table + (int64_t)to * s.max_blocks;
  bool bad = false;
  if (part == 0) {
    for (int j = threadIdx.x; j < whole; j += 256) {
      const int32_t blk = of[j];
      entry[j] = blk;
      if (blk >= 0 && blk <= s.last_block) atomicAdd(refs + blk, 1);
      else bad = true;
    }
    if (threadIdx.x == 0) lens[to] = (int32_t)len;
  }
  if (len % kBlockSize != 0) {
    const int32_t fresh = ws[64 + s.B + ws[64 + i]];
    const int32_t blk = of[whole];
    if (part == 0 && threadIdx.x == 0) entry[whole] = fresh;
    if (blk >= 0 && blk <= s.last_block) {
      const int64_t n16 = (int64_t)s.Hkv * kTileElems / 8;
      for (int64_t x = part * 256 + threadIdx.x; x < n16; x += 256 * kForkParts) {
        const u32x4 key = k[blk * n16 + x], val = v[blk * n16 + x];
        k[fresh * n16 + x] = key;
        v[fresh * n16 + x] = val;
      }
    } else {
      bad = true;
    }
  }
  if (bad) atomicMax(status, 4);
}

__global__ __launch_bounds__(256) void release_kernel(int32_t* __restrict__ table, const int32_t* __restrict__ keep,
                                                      int32_t* __restrict__ refs, int32_t* __restrict__ status,
                                                      CacheShape s) {
  for (int b = blockIdx.x; b < s.B; b += gridDim.x) {
    for (int64_t j = (int64_t)blocks_of(keep[b]) + threadIdx.x; j < s.max_blocks; j += 256) {
      int32_t* entry = table + (int64_t)b * s.max_blocks + j;
      const int32_t blk = *entry;
      if (blk == -1) continue;
      *entry = -1;
      if (blk < 0 || blk > s.last_block) {
        atomicMax(status, 4);
      } else if (atomicSub(refs + blk, 1) <= 0) {
        atomicAdd(refs + blk, 1);
        atomicMax(status, 4);
      }
    }
  }
}

}  // namespace

hipError_t launch_reserve(int32_t* table, const int32_t* lens, const int32_t* need, int32_t* refs, int64_t num_blocks,
                          int32_t* status, int32_t* workspace, CacheShape s, hipStream_t stream) {
  hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(kPlanThreads), 0, stream, table, lens, need, refs, num_blocks,
                     status, workspace, s);
  return hipGetLastError();
}

hipError_t launch_fork(const int32_t* src, const int32_t* dst, int n, void* k, void* v, int32_t* table, int32_t* lens,
                       int32_t* refs, int64_t num_blocks, int32_t* status, int32_t* workspace, CacheShape s,
                       hipStream_t stream) {
  hipLaunchKernelGGL(fork_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, src, dst, n, table, lens, refs,
                     num_blocks, status, workspace, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(fork_kernel, dim3((unsigned)n * kForkParts), dim3(256), 0, stream, src, dst,
                     static_cast<u32x4*>(k), static_cast<u32x4*>(v), table, lens, refs, status, workspace, s);
  return hipGetLastError();
}

hipError_t launch_release(int32_t* table, const int32_t* keep, int32_t* refs, int32_t* status, CacheShape s,
                          hipStream_t stream) {
  const unsigned groups = s.B < 65536 ? s.B : 65536;
  hipLaunchKernelGGL(release_kernel, dim3(groups), dim3(256), 0, stream, table, keep, refs, status, s);
  return hipGetLastError();
}

}  // namespace bana
