// blocks.hip -- blocks of the cache handed out, shared and taken back on the device (gfx950).
//
// The state is the block table and one count per block; a block with the count 0 is free, and the lowest
// free numbers are taken first, so there is no free list whose order could depend on timing.  A call
// that takes blocks first makes its plan in one workgroup (what is asked for, whether it can be had, which
// blocks), then carries it out; a plan that cannot be carried out changes nothing but *status.
//
// Bound by the latency of dependent reads, not by their bytes: lengths, table entries, counts, list, each a round trip
// of some 0.7 us, and two launches for a fork.  Measured on MI355X: blocks for 128 drafts of 64 tokens, pool of
// 116,000, 8.6 us; 96 forks of 1500 tokens, 8 kv heads, and their release, 15.4 us.
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

// Workspace: reserve has prefix sums in [64, 64 + B) and the list of blocks from 64 + 2 B on.  Fork: [0] 1 if the plan
// holds, [1] 1 if a source names a block without references, [64, 64 + B) marks, then places in the list, [64 + B,
// 64 + 2 B) the list, then the blocks kept from the search.
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
        for (int u = 0; u < 4; ++u) count += (j + u < end) & (x[u] == -1);
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
        if (j + u >= end || x[u] != -1) continue;
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

// One fork of a call, its indices in order (else valid is false).
struct Fork {
  int src, dst;
  int64_t len;  // of the source
  bool valid;
};

__device__ __forceinline__ Fork fork_at(const int32_t* __restrict__ src, const int32_t* __restrict__ dst, int i,
                                        const int32_t* __restrict__ table, const int32_t* __restrict__ lens,
                                        const CacheShape& s) {
  const int a = src[i], d = dst[i];
  const bool inside = a >= 0 && a < s.B && d >= 0 && d < s.B;
  const int64_t len = length_of(lens, inside ? a : 0, s);
  return {a, d, len, inside && table[(int64_t)(inside ? d : 0) * s.max_blocks] == -1};
}

// f(block, named) for every entry of the sources of the forks i that are chosen(i, fork): whether it names a block of the
// pool, and which (else some block of it).  fork(i) is fork i.  A thread takes a piece of a source's entries, so that
// those of 1024 forks are under way together.  Every thread calls it.
constexpr int kPiece = 4;

template <typename G, typename C, typename F>
__device__ __forceinline__ void for_source_blocks(int n, G fork, const int32_t* __restrict__ table,
                                                  const CacheShape& s, int* sm, C chosen, F f) {
  typedef int32_t i32x4 __attribute__((ext_vector_type(4), aligned(4)));
  __shared__ int sm_seq[kPlanThreads], sm_entries[kPlanThreads], sm_first[kPlanThreads];
  int half = 1;  // of the forks looked at together, a power of two
  while (2 * half < min(n, kPlanThreads)) half *= 2;
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    int seq = 0, entries = 0;
    if (i < n) {
      const Fork x = fork(i);
      seq = x.src;
      if (chosen(i, x)) entries = blocks_of(x.len);
    }
    int pieces;
    const int first = block_scan((entries + kPiece - 1) / kPiece, sm, &pieces);
    race_check_delay(threadIdx.x >> 6);
    sm_seq[threadIdx.x] = seq, sm_entries[threadIdx.x] = entries, sm_first[threadIdx.x] = first;
    __syncthreads();
    race_check_barrier();
    for (int x = threadIdx.x; x < pieces; x += kPlanThreads) {
      int k = 0;  // the last fork whose pieces start at x or before
      for (int step = half; step >= 1; step /= 2)
        if (sm_first[k + step] <= x) k += step;
      const int32_t* row = table + (int64_t)sm_seq[k] * s.max_blocks;
      const int j = (x - sm_first[k]) * kPiece, end = sm_entries[k];
      i32x4 blk[kPiece / 4];
      if (j + kPiece <= s.max_blocks) {
#pragma unroll
        for (int q = 0; q < kPiece / 4; ++q) blk[q] = *reinterpret_cast<const i32x4*>(row + j + 4 * q);
      } else {
#pragma unroll
        for (int e = 0; e < kPiece; ++e) blk[e >> 2][e & 3] = row[min(j + e, end - 1)];
      }
#pragma unroll
      for (int e = 0; e < kPiece; ++e) {
        const int y = blk[e >> 2][e & 3];
        f(min(max(y, 0), s.last_block), (j + e < end) & (y >= 0) & (y <= s.last_block));
      }
    }
  }
}

// The counts of the blocks that the sources name are judged before any changes: one without references is left alone by
// the forks (ws[1] tells them to look; looking always would cost the next kernel 9 us, as loads of the counts then meet
// the atomics on them) and is no free block of this call, whatever its count.  96 forks of 32 sequences of 1500 tokens:
// 8.6 us, without the walk over the sources' entries 5.4; with 16 entries to a thread 9.4, most of that more code to fetch.
__global__ __launch_bounds__(kPlanThreads) void fork_plan_kernel(const int32_t* __restrict__ src,
                                                                 const int32_t* __restrict__ dst, int n,
                                                                 const int32_t* __restrict__ table,
                                                                 const int32_t* __restrict__ lens, int32_t* refs,
                                                                 int64_t num_blocks, int32_t* __restrict__ status,
                                                                 int32_t* __restrict__ ws, CacheShape s) {
  __shared__ int sm[kPlanWaves], sm_held;
  int32_t* mark = ws + 64;        // [B]: 0 none, 1 a destination, 2 + i the source of fork i (the last of them)
  int32_t* list = ws + 64 + s.B;  // [min(n, B)] block of each fork that takes one, in order
  int32_t* held = list + s.B;     // [min(entries, num_blocks)] blocks kept from the search
  const int own_i = threadIdx.x;
  Fork own = {};
  if (own_i < n) own = fork_at(src, dst, own_i, table, lens, s);
  auto fork = [&](int i) { return i == own_i ? own : fork_at(src, dst, i, table, lens, s); };
  for (int b = threadIdx.x; b < s.B; b += kPlanThreads) mark[b] = 0;
  if (threadIdx.x == 0) sm_held = 0;
  __syncthreads();
  bool bad = n > s.B;
  for (int i = own_i; i < n && !bad; i += kPlanThreads) {
    const Fork x = fork(i);
    bad = !x.valid || atomicExch(mark + x.dst, 1) != 0;
  }
  const bool valid = !bad;
  __syncthreads();
  bool odd = false;
  for_source_blocks(
      n, fork, table, s, sm,
      [&](int i, const Fork& x) {
        const int before = valid ? atomicMax(mark + x.src, 2 + i) : 1;
        bad |= before == 1;
        return before == 0;
      },
      [&](int blk, bool named) { odd |= named & (refs[blk] <= 0); });
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) {
      atomicMax(status, 2);
      ws[0] = 0;
    }
    return;
  }
  odd = __syncthreads_or(odd);
  if (odd) {  // rare, and wrong of the caller: counts of 0 are marked until the search is over
    for_source_blocks(
        n, fork, table, s, sm,
        [&](int i, const Fork& x) {
          return __hip_atomic_load(mark + x.src, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 2 + i;
        },
        [&](int blk, bool named) {
          if (named && atomicCAS(refs + blk, 0, INT32_MIN) == 0) held[atomicAdd(&sm_held, 1)] = blk;
        });
    __syncthreads();
    __threadfence();  // the search reads around the atomics
  }
  int64_t total = 0;
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    int sum;
    const int at = block_scan(i < n && fork(i).len % kBlockSize != 0, sm, &sum);
    if (i < n) mark[i] = (int32_t)(total + at);  // place in the list (the marks are done with)
    total += sum;
  }
  const int64_t found = total > num_blocks ? 0 : find_free(refs, num_blocks, total, list, sm);
  __syncthreads();
  for (int x = threadIdx.x; x < sm_held; x += kPlanThreads) refs[held[x]] = 0;
  if (found < total) {
    if (threadIdx.x == 0) {
      atomicMax(status, 1);
      ws[0] = 0;
    }
    return;
  }
  for (int64_t i = threadIdx.x; i < total; i += kPlanThreads) refs[list[i]] = 1;
  if (threadIdx.x == 0) ws[0] = 1, ws[1] = odd;
}

// kForkParts workgroups per fork: the shared entries (the first), and the copy of the last block if it is partly
// filled, each a share of its bytes.
constexpr int kForkParts = 8;

__global__ __launch_bounds__(256) void fork_kernel(const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                   u32x4* __restrict__ k, u32x4* __restrict__ v,
                                                   int32_t* __restrict__ table, int32_t* __restrict__ lens,
                                                   int32_t* __restrict__ refs, int32_t* __restrict__ status,
                                                   const int32_t* __restrict__ ws, CacheShape s) {
  const int holds = ws[0], odd = ws[1];
  if (holds == 0) return;
  const int i = blockIdx.x / kForkParts, part = blockIdx.x % kForkParts;
  const int from = src[i], to = dst[i];
  const int64_t len = length_of(lens, from, s);
  const int whole = (int)(len / kBlockSize);
  const int32_t* of = table + (int64_t)from * s.max_blocks;
  int32_t* entry = table + (int64_t)to * s.max_blocks;
  bool bad = false;
  // Forks raise only counts above 0, and the plan took no block that a source names: a count keeps its sign.
  auto counted = [&](int32_t blk) {
    return odd == 0 || __hip_atomic_load(refs + blk, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) > 0;
  };
  if (part == 0) {
    for (int j = threadIdx.x; j < whole; j += 256) {
      const int32_t blk = of[j];
      entry[j] = blk;
      if (blk >= 0 && blk <= s.last_block && counted(blk)) atomicAdd(refs + blk, 1);
      else bad = true;
    }
    if (threadIdx.x == 0) lens[to] = (int32_t)len;
  }
  if (len % kBlockSize != 0) {
    const int32_t fresh = ws[64 + s.B + ws[64 + i]];
    const int32_t blk = of[whole];
    if (part == 0 && threadIdx.x == 0) entry[whole] = fresh;
    if (blk >= 0 && blk <= s.last_block) {
      bad |= part == 0 && !counted(blk);
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
