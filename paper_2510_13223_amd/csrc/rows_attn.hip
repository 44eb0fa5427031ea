// rows_attn.hip -- attention of several new tokens per sequence over the paged cache (gfx950).
//
// Row r of sequence b, query head h, over the tokens that the row sees:
//   s_t = scale q[r][h].k_t,  out = sum_t exp(s_t - lse) v_t,  lse = ln sum_t exp(s_t)
// Two kinds of sight share one kernel:
//  * tree: some ranges of the context, whole, and the nodes whose bit is set in the row's mask;
//  * window: tokens t <= pos with pos - t < window or t < sinks.
//
// The columns of the score product are the (row, head of the group) pairs of one sequence and kv head,
// c = i G + h, 16 to a tile; one wavefront takes one tile and walks the blocks that any of its rows sees
// with the products, layouts and one-pass softmax of the decode kernel (attn_partial.hip).  A tile's
// number among all tiles of a kv head is floor(row_begin[b] G / 16) + b plus its place in the sequence:
// unique, as a sequence of n rows has at most floor(end G / 16) - floor(begin G / 16) + 1 tiles, so the
// grid follows from the number of rows and sequences alone and a wavefront finds its sequence by search.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "packed_rows.h"
#include "paged_addr.h"
#include "tokens.h"

namespace bana {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kCols = 16;
constexpr int kDimTiles = kHeadDim / 16;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ uint32_t bf16_bits(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return (u >> 16) | 0x40u;  // NaN stays NaN
  return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}
__device__ __forceinline__ float bf16_value(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }

// The token ranges that the rows of a tile see, one per lane, as a list of blocks (as in the decode kernel).
struct Ranges {
  int t0, t1, nblk, vend;

  __device__ __forceinline__ void scan(int lane) {
    nblk = t1 > t0 ? ((t1 - 1) >> 4) - (t0 >> 4) + 1 : 0;
    vend = nblk;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int y = __shfl_up(vend, off);
      if (lane >= off) vend += y;
    }
  }
};

// Element of a row that a token is seen by.
template <RowsMode MODE>
struct Sight {
  int pos, window, sinks;  // window: position of the row (-1: sees nothing)
  uint64_t nodes;          // tree: the nodes it sees

  __device__ __forceinline__ bool token(int t) const { return t <= pos && (t > pos - window || t < sinks); }
  __device__ __forceinline__ bool node(int j) const { return (nodes >> (j & 63)) & 1; }
};

template <RowsMode MODE, bool BF16>
__global__ __launch_bounds__(64) void rows_attn_kernel(RowsAttnArgs a) {
  const int lane = threadIdx.x, col = lane & 15, quad = lane >> 4;
  const int G = a.G, B = a.s.B;
  const unsigned slot = a.by_hkv.quotient(blockIdx.x);
  const int g = (int)(blockIdx.x - slot * a.s.Hkv);
  auto first_slot = [&](int b) { return row_start(a.row_begin, b, a.rows) * G / kCols + b; };
  const int b = last_at_most(B, (int)slot, lane, first_slot);
  const int r0 = row_start(a.row_begin, b, a.rows);
  const int n = row_start(a.row_begin, b + 1, a.rows) - r0;
  const int c0 = ((int)slot - (r0 * G / kCols + b)) * kCols;
  if (c0 < 0 || c0 >= n * G) return;

  const int c = c0 + col;
  const bool live = c < n * G;
  const int i = live ? (int)a.by_g.quotient(c) : n - 1;
  const int h = live ? c - i * G : 0;
  const int64_t qrow = (int64_t)(r0 + i) * a.Hq + g * G + h;
  const int span = a.s.max_blocks * kBlockSize;

  // What the rows see, together and each.
  Sight<MODE> sight;
  Ranges rg;
  rg.t0 = rg.t1 = 0;
  int n_ranges;
  int tree0 = -1;
  if (MODE == RowsMode::kTree) {
    n_ranges = a.n_parts + 1;
    tree0 = min(a.tree_begin[b], span);
    const int nodes = min(n, 64);
    sight.nodes = a.mask[r0 + i];
    if (nodes < 64) sight.nodes &= (uint64_t{1} << nodes) - 1;
    if (lane < a.n_parts) {
      rg.t0 = max(a.begin[(int64_t)lane * B + b], 0);
      rg.t1 = min(a.end[(int64_t)lane * B + b], span);
    } else if (lane == a.n_parts && tree0 >= 0) {
      rg.t0 = tree0;
      rg.t1 = tree0 + min(nodes, span - tree0);
    }
  } else {
    n_ranges = 2;
    const int len = min(max(a.seq_lens[b], 0), span);
    sight.window = a.window;
    sight.sinks = a.sinks;
    sight.pos = max(len - n + i, -1);
    const int i0 = (int)a.by_g.quotient(c0), i1 = (int)a.by_g.quotient(min(c0 + kCols, n * G) - 1);
    const int p0 = max(len - n + i0, 0), p1 = max(len - n + i1, -1);
    const int lo = a.begin != nullptr ? max(a.begin[b], 0) : 0;
    const int hi = min(a.end != nullptr ? min(a.end[b], span) : span, p1 + 1);
    int w0 = max(p0 - a.window + 1, lo);
    const int s1 = min(a.sinks, hi);
    if (w0 <= s1) w0 = lo;  // sinks and window touch: one range
    else if (lane == 0) {
      rg.t0 = lo;
      rg.t1 = s1;
    }
    if (lane == 1) {
      rg.t0 = w0;
      rg.t1 = hi;
    }
  }
  rg.scan(lane);

  bf16x8 qop[4];
  const uint16_t* qsrc = a.q + qrow * kHeadDim + 8 * quad;
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    u32x4 x = *reinterpret_cast<const u32x4*>(qsrc + 32 * kk);
    if (!live) x = u32x4{0u, 0u, 0u, 0u};
    qop[kk] = __builtin_bit_cast(bf16x8, x);
  }
  f32x4 acc[kDimTiles];
#pragma unroll
  for (int dt = 0; dt < kDimTiles; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, lsum = 0.f;  // m: running max of the scores in powers of two

  for (int p = 0; p < n_ranges; ++p) {
    const int t0 = __builtin_amdgcn_readlane(rg.t0, p), t1 = __builtin_amdgcn_readlane(rg.t1, p);
    const bool tree = MODE == RowsMode::kTree && p == a.n_parts;
    for (int j = t0 >> 4; t0 < t1 && j * kBlockSize < t1; ++j) {
      const int32_t blk = min(max(table_lookup(a.table, a.s.max_blocks, b, j), 0), a.s.last_block);
      const int64_t tile = kv_tile(blk, g, a.s.Hkv) * kTileElems;
      const u32x4* ksrc = reinterpret_cast<const u32x4*>(a.k + tile) + (quad * kBlockSize + col);
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ksrc[4 * kBlockSize * kk]), qop[kk], s,
                                                    0, 0, 0);
      const u32x2* vsrc = reinterpret_cast<const u32x2*>(a.v + tile + col * kBlockSize + 4 * quad);
      u32x2 vr[kDimTiles];
#pragma unroll
      for (int dt = 0; dt < kDimTiles; ++dt) vr[dt] = vsrc[4 * 16 * dt];
      bool ok[4];
      uint32_t keep[2] = {0, 0};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = j * kBlockSize + 4 * quad + e;
        const bool in = t >= t0 && t < t1;
        ok[e] = in && (MODE == RowsMode::kTree ? !tree || sight.node(t - tree0) : sight.token(t));
        if (in) keep[e >> 1] |= 0xFFFFu << (16 * (e & 1));
        s[e] = ok[e] ? s[e] * a.scale : -INFINITY;
      }
      bool odd = false;  // a value that is not finite: only the rows that see it may meet it
#pragma unroll
      for (int dt = 0; dt < kDimTiles; ++dt) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          vr[dt][w] &= keep[w];
          odd |= (vr[dt][w] & 0x7F80u) == 0x7F80u || (vr[dt][w] & 0x7F800000u) == 0x7F800000u;
        }
      }
      float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_new = fmaxf(m, mx);
      const float base = m_new == -INFINITY ? 0.f : m_new;  // nothing seen yet
      const float alpha = __builtin_amdgcn_exp2f(m - base);
      m = m_new;
      float w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_exp2f(s[e] - base);
      lsum = lsum * alpha + ((w[0] + w[1]) + (w[2] + w[3]));
#pragma unroll
      for (int dt = 0; dt < kDimTiles; ++dt) acc[dt] *= alpha;
      if (__any(odd)) {
        for (int t = 0; t < kBlockSize; ++t) {
          const int from = (t >> 2) * 16 + col;
          const int e = t & 3;
          const float mine = e == 0 ? w[0] : e == 1 ? w[1] : e == 2 ? w[2] : w[3];
          const bool seen = __shfl((int)(e == 0 ? ok[0] : e == 1 ? ok[1] : e == 2 ? ok[2] : ok[3]), from);
          const float weight = __shfl(mine, from);
#pragma unroll
          for (int dt = 0; dt < kDimTiles; ++dt)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const float val = bf16_value(a.v[tile + (16 * dt + 4 * quad + x) * kBlockSize + t]);
              if (seen) acc[dt][x] += weight * val;
            }
        }
        continue;
      }
      float rest[4] = {w[0], w[1], w[2], w[3]};
#pragma unroll
      for (int term = 0; term < (BF16 ? 1 : 3); ++term) {
        uint32_t bits[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          bits[e] = bf16_bits(rest[e]);
          rest[e] -= bf16_value(bits[e]);
        }
        const i16x4 pop = __builtin_bit_cast(i16x4, u32x2{bits[0] | bits[1] << 16, bits[2] | bits[3] << 16});
#pragma unroll
        for (int dt = 0; dt < kDimTiles; ++dt)
          acc[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(i16x4, vr[dt]), pop, acc[dt], 0, 0, 0);
      }
    }
  }

  lsum += __shfl_xor(lsum, 16);
  lsum += __shfl_xor(lsum, 32);
  if (!live) return;
  const bool empty = lsum == 0.f;
  const float inv = empty ? 0.f : 1.0f / lsum;
#pragma unroll
  for (int dt = 0; dt < kDimTiles; ++dt) {
    const f32x4 o = acc[dt] * inv;
    const int64_t at = qrow * kHeadDim + 16 * dt + 4 * quad;
    if (BF16)
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + at) =
          u32x2{bf16_bits(o[0]) | bf16_bits(o[1]) << 16, bf16_bits(o[2]) | bf16_bits(o[3]) << 16};
    else
      *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = o;
  }
  if (a.lse != nullptr && quad == 0) a.lse[qrow] = empty ? -INFINITY : (m + log2f(lsum)) * kLn2;
}

}  // namespace

hipError_t launch_rows_attn(const RowsAttnArgs& a, RowsMode mode, bool bf16, hipStream_t stream) {
  const unsigned slots = (unsigned)((int64_t)a.rows * a.G / kCols + a.s.B);
  const dim3 grid(slots * (unsigned)a.s.Hkv), block(64);
  if (mode == RowsMode::kTree) {
    if (bf16) hipLaunchKernelGGL((rows_attn_kernel<RowsMode::kTree, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((rows_attn_kernel<RowsMode::kTree, false>), grid, block, 0, stream, a);
  } else {
    if (bf16) hipLaunchKernelGGL((rows_attn_kernel<RowsMode::kWindow, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((rows_attn_kernel<RowsMode::kWindow, false>), grid, block, 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace bana
