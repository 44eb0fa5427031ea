// rows_attn.hip -- attention of several new tokens per sequence over the paged cache (gfx950).
//
// Row r of sequence b, query head h, over the tokens that the row sees:
//   s_t = scale q[r][h].k_t,  out = sum_t exp(s_t - lse) v_t,  lse = ln sum_t exp(s_t)
// Two kinds of sight share the kernels:
//  * tree: some ranges of the context, whole, and the nodes whose bit is set in the row's mask;
//  * window: tokens t <= pos with pos - t < window or t < sinks.
//
// The columns of the score product are the (row, head of the group) pairs of one sequence and kv head,
// c = i G + h.  A workgroup takes a tile of CT neighbouring columns of one sequence and kv head and walks
// the blocks that any of its rows sees.  A tile's number among all tiles of a kv head is
// floor(row_begin[b] G / CT) + b plus its place in the sequence: unique, as a sequence's columns [x, y)
// make at most floor(y / CT) - floor(x / CT) + 1 tiles, so the grid follows from the number of rows and sequences
// alone and a workgroup finds its sequence by search.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "packed_rows.h"
#include "paged_addr.h"
#include "tokens.h"

namespace bana {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// Two floats rounded to bf16 (nearest, ties to even), the first in the low half.
__device__ __forceinline__ uint32_t bf16_pair(float x, float y) {
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
}
__device__ __forceinline__ float low_value(uint32_t pair) { return __builtin_bit_cast(float, pair << 16); }
__device__ __forceinline__ float high_value(uint32_t pair) { return __builtin_bit_cast(float, pair & 0xFFFF0000u); }

// The columns [c0, c0 + CT) of sequence b and kv head g that a workgroup computes.
struct Tile {
  int b, g, r0, n, c0;  // first row and number of rows of the sequence
  int tokens;           // window: its tokens, in the table; tree: where its nodes begin
  bool any;             // some column exists
};

// Where sequences have a few tiles or less and one load sees them all, their tiles are counted, so that those that
// exist are numbered without gaps.  (The numbering by floor(row_begin[b] G / CT) + b leaves one behind every sequence
// whose columns fill its tiles, and workgroups that end at once every so often leave some CUs without work.)
// 24 trees of 32 nodes, groups of 4, by that numbering / counted: fp32 165 / 124 us, bf16 119 / 102; a count costs
// up to 0.8 us.
template <RowsMode MODE, int CT>
__device__ __forceinline__ Tile find_tile(const RowsAttnArgs& a, unsigned wg, int lane) {
  const unsigned slot = a.by_hkv.quotient(wg);
  const int B = a.s.B;
  const int32_t* values = MODE == RowsMode::kTree ? a.tree_begin : a.seq_lens;
  Tile t;
  t.g = (int)(wg - slot * a.s.Hkv);
  int value;
  if (a.count_tiles) {  // B <= 64: a sequence per lane
    const int start = row_start(a.row_begin, min(lane, B), a.rows), its = values[min(lane, B - 1)];
    const int n = row_start(a.row_begin, min(lane + 1, B), a.rows) - start;
    const int tiles = (max(n, 0) * a.G + CT - 1) / CT;
    int past = tiles;  // tiles of the sequences up to this one
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int y = __shfl_up(past, off);
      if (lane >= off) past += y;
    }
    const uint64_t behind = __ballot(past > (int)slot);
    t.b = behind != 0 ? __ffsll((unsigned long long)behind) - 1 : 0;  // past the last tile: c0 is outside
    t.r0 = __builtin_amdgcn_readlane(start, t.b);
    t.n = __builtin_amdgcn_readlane(n, t.b);
    value = __builtin_amdgcn_readlane(its, t.b);
    t.c0 = behind != 0 ? ((int)slot - __builtin_amdgcn_readlane(past - tiles, t.b)) * CT : -1;
  } else {
    auto first_slot = [&](int b, int row) { return row * a.G / CT + b; };
    const SeqRows x = find_rows(a.row_begin, values, a.rows, B, (int)slot, a.seqs_per_slot, lane, first_slot);
    t.b = x.b;
    t.r0 = x.begin;
    t.n = x.end - x.begin;
    value = x.value;
    t.c0 = ((int)slot - first_slot(x.b, x.begin)) * CT;
  }
  t.any = t.c0 >= 0 && t.c0 < t.n * a.G;
  const int span = a.s.max_blocks * kBlockSize;
  t.tokens = MODE == RowsMode::kTree ? min(value, span) : min(max(value, 0), span);
  return t;
}

// What one column's row sees, beside the ranges.
template <RowsMode MODE>
struct Sight;
template <>
struct Sight<RowsMode::kTree> {
  uint64_t nodes;
};
template <>
struct Sight<RowsMode::kWindow> {
  int pos;  // -1: before the first token, sees nothing
};

// The token ranges that the rows of a tile see, one per lane, their blocks one after the other making one
// list (a tile's rows may see parts of a range only).
struct Ranges {
  int t0, t1, nblk, vend;  // this lane's: tokens, blocks, end of its blocks in the list
  int count, total;        // ranges, blocks of all
  int tree;                // tree: the range of the nodes
  int tree0;               // and its first token

  __device__ __forceinline__ void scan(int lane) {
    nblk = t1 > t0 ? ((t1 - 1) >> 4) - (t0 >> 4) + 1 : 0;
    vend = nblk;
    if (count > 2) {
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(vend, off);
        if (lane >= off) vend += y;
      }
    } else {
      const int first = __builtin_amdgcn_readlane(nblk, 0);
      if (lane == 1) vend += first;
    }
    total = __builtin_amdgcn_readlane(vend, count - 1);
  }
};

// Ranges seen by the columns [ca, cb) of a tile (rows i = c / G).
template <RowsMode MODE>
__device__ __forceinline__ Ranges find_ranges(const RowsAttnArgs& a, const Tile& t, int ca, int cb, int lane) {
  Ranges r;
  const int span = a.s.max_blocks * kBlockSize, B = a.s.B;
  r.t0 = r.t1 = 0;
  if (MODE == RowsMode::kTree) {
    r.count = a.n_parts + 1;
    r.tree = a.n_parts;
    r.tree0 = t.tokens;
    if (lane < a.n_parts) {
      r.t0 = max(a.begin[(int64_t)lane * B + t.b], 0);
      r.t1 = min(a.end[(int64_t)lane * B + t.b], span);
    } else if (lane == a.n_parts && r.tree0 >= 0) {
      r.t0 = r.tree0;
      r.t1 = r.tree0 + min(min(t.n, 64), span - r.tree0);
    }
  } else {
    r.count = 2;
    r.tree = r.tree0 = -1;
    const int len = t.tokens;
    const int p0 = max(len - t.n + (int)a.by_g.quotient(ca), 0), p1 = max(len - t.n + (int)a.by_g.quotient(cb - 1), -1);
    const int lo = a.begin != nullptr ? max(a.begin[t.b], 0) : 0;
    const int hi = min(a.end != nullptr ? min(a.end[t.b], span) : span, p1 + 1);
    const int w0 = max(p0 - a.window + 1, lo), s1 = min(a.sinks, hi);
    const bool apart = w0 > s1;  // sinks and window do not touch: two ranges
    if (lane == 0 && apart) {
      r.t0 = lo;
      r.t1 = s1;
    }
    if (lane == 1) {
      r.t0 = apart ? w0 : lo;
      r.t1 = hi;
    }
  }
  r.scan(lane);
  return r;
}

// The range that holds block v of the list (wave-uniform; v does not decrease from call to call), and which
// of its blocks are seen whole by all rows at positions [p0, p1].
struct Cursor {
  int p = -1, vend = 0;    // range, end of its blocks in the list
  int offset = 0;          // logical block of list entry v: v + offset
  int t0 = 0, t1 = 0;      // tokens of the range
  int wbegin = 0, wend = 0;  // list entries seen whole

  template <RowsMode MODE>
  __device__ __forceinline__ void seek(const RowsAttnArgs& a, const Ranges& r, int v, int p0, int p1) {
    while (v >= vend && p + 1 < r.count) {
      ++p;
      vend = __builtin_amdgcn_readlane(r.vend, p);
      t0 = __builtin_amdgcn_readlane(r.t0, p);
      t1 = __builtin_amdgcn_readlane(r.t1, p);
      offset = (t0 >> 4) - (vend - __builtin_amdgcn_readlane(r.nblk, p));
      int from = t0, end = t1;
      if (MODE == RowsMode::kTree) {
        if (p == r.tree) end = from;
      } else {
        end = min(t1, p0 + 1);
        if (p == 1) from = max(t0, p1 - a.window + 1);
      }
      wbegin = ((from + kBlockSize - 1) >> 4) - offset;
      wend = (end >> 4) - offset;
    }
  }
};

// A block of a step: its first token and the tokens of its range.  Past the list's end: the last block, with
// nothing of it seen.
struct Block {
  int first, t0, t1;
  bool tree;
};

template <RowsMode MODE>
__device__ __forceinline__ Block block_at(const RowsAttnArgs& a, const Ranges& r, Cursor& c, int v, int p0, int p1) {
  c.seek<MODE>(a, r, v, p0, p1);
  const bool past = v >= r.total;
  return {((past ? r.total - 1 : v) + c.offset) * kBlockSize, past ? 0 : c.t0, past ? 0 : c.t1, c.p == r.tree};
}

// Blocks of the pool for list entries v, one per lane (any order); past the end those of the last entry.
__device__ __forceinline__ int pool_blocks(const RowsAttnArgs& a, const Ranges& r, int b, int v) {
  v = min(v, r.total - 1);
  int offset = 0;
  for (int p = 0; p < r.count; ++p) {
    const int vend = __builtin_amdgcn_readlane(r.vend, p), nblk = __builtin_amdgcn_readlane(r.nblk, p);
    if (v >= vend - nblk) offset = (__builtin_amdgcn_readlane(r.t0, p) >> 4) - (vend - nblk);
  }
  return min(max(a.table[(int64_t)b * a.s.max_blocks + v + offset], 0), a.s.last_block);
}

// Whether token t of a block is seen by a row.  (Without branches: hipcc 7.2 dropped one of the conditional
// stores that a form with && and || led to.)
template <RowsMode MODE>
__device__ __forceinline__ bool seen(const RowsAttnArgs& a, const Ranges& r, const Block& c, const Sight<MODE>& s,
                                     int t) {
  const bool in = (t >= c.t0) & (t < c.t1);
  if constexpr (MODE == RowsMode::kTree) {
    return in & (!c.tree | (((uint32_t)(s.nodes >> ((t - r.tree0) & 63)) & 1u) != 0));
  } else {
    return in & (t <= s.pos) & ((t > s.pos - a.window) | (t < a.sinks));
  }
}

template <RowsMode MODE>
__device__ __forceinline__ Sight<MODE> sight_of(const RowsAttnArgs& a, const Tile& t, int i) {
  Sight<MODE> s;
  if constexpr (MODE == RowsMode::kTree) {
    s.nodes = a.mask[t.r0 + i];
    if (t.n < 64) s.nodes &= (uint64_t{1} << t.n) - 1;
  } else {
    s.pos = max(t.tokens - t.n + i, -1);
  }
  return s;
}

// One row: this lane has the dims STRIDE j + first + [0, 4) in acc[j].  m in powers of two.
template <bool BF16, int STRIDE>
__device__ __forceinline__ void store_row(void* __restrict__ out, float* __restrict__ lse, int64_t row,
                                          const f32x4 (&acc)[kHeadDim / STRIDE], float l, float m, int first) {
  const bool empty = l == 0.f;
  const float inv = 1.0f / l;
#pragma unroll
  for (int j = 0; j < kHeadDim / STRIDE; ++j) {
    // A row whose scores are all -inf has sums of NaN where values are infinite: 0 by choice, not by the product.
    const f32x4 o = empty ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[j] * inv;
    const int64_t at = row * kHeadDim + STRIDE * j + first;
    if (BF16)
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(out) + at) = u32x2{bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3])};
    else
      *reinterpret_cast<f32x4*>(static_cast<float*>(out) + at) = o;
  }
  if (lse != nullptr && first == 0) lse[row] = empty ? -INFINITY : (m + log2f(l)) * kLn2;
}

// ---- the kernel: K and V shared through LDS ---------------------------------------------------------
//
// Four wavefronts of COLS columns each walk the same list of blocks, two blocks (32 tokens) a step.  The
// step's four 4 KiB tiles come from memory straight into LDS (each wavefront requests one, one or two steps ahead)
// and feed the operands of all four.  A wavefront's products, for 32 columns (16: in brackets):
//   scores  S^T[32 tok x 32 col]: 8 x v_mfma_f32_32x32x16_bf16 over the 128 dims
//           [two of 16 tok x 16 col: 4 x v_mfma_f32_16x16x32_bf16 each]
//   values  O^T[128 dim x 32 col] += V^T P^T: 4 tiles of 32 dims, one product of 16 tokens per block
//           [8 tiles of 16 dims, one product of the 32 tokens]
// A value product takes 8 consecutive tokens from each lane: slots 8 (hi & 1) + [0, 8) of a block, hi = lane / COLS.
// The rows of the score products are assigned to tokens so that they leave exactly these in that lane, and P
// never leaves it.  Every fragment is one 16-byte LDS read per lane, no two lanes of a phase (0-3, 12-15, 20-23, 24-27
// and so on) on the same bank: with 16 columns the second block's K tile lies 64 bytes off, with 32 it must not (it
// cost a third of the LDS cycles); of V, each 16 dims hold the first 8 tokens of all dims, then the last 8.
//
// The running maximum is raised only where a score exceeds it by 2^8 (the weights are then at most 2^8, which
// changes no relative rounding), which spares most steps the rescaling of the sums.  A bf16 result takes its weights
// rounded to bf16, half a step of the result's own type; an fp32 result takes them as three bf16 terms, 24 bits.
// Their sum is of the unrounded ones in both.
//
// What bounds it, 32 columns: the matrix and vector units, at the clock that the card's power leaves them (1.8 GHz; the
// matrix units are busy half of its cycles).  A step of
// a wavefront is 16 matrix instructions of 32 cycles, some 80 vector instructions and 16 exponentials, and 16 KiB of
// LDS reads; three workgroups on a CU overlap them in part.  2 x 4096 new tokens, 32 heads, window 4096, bf16: 537 to
// 560 us, 1.0 PFLOP/s, where a library product of 8192^3 reaches 1.47; the same call on zeros takes 425.  Without the
// weights' computation 444, with one LDS fragment for all 498, without both 401.  32 trees of 64 nodes over 8000
// tokens, 64 heads: 597 to 620 us.  Instructions of 16 x 16 x 32 for 32 columns: 2 % more; 64 columns a wavefront, one
// per SIMD, with the next step's scores before this step's values, were slower (the registers of two steps spill).
// At three workgroups on a CU the bf16 kernels spill 5 registers (window) or 9 (tree); a masked step reads one back, and
// its wait takes in the requests under way.
// 16 columns: HBM.  64 single tokens, window 4096: 169 us, 6.4 TB/s.
constexpr int kTileBytes = kTileElems * 2;
constexpr int kKStep = 2 * kTileBytes + 128;    // K tiles of a step, the second 64 bytes off
constexpr int kVStep = 2 * kTileBytes;
constexpr int kStep = kKStep + kVStep;          // K, then V
constexpr float kSlack = 8.f;
constexpr int W = 4;  // wavefronts of a workgroup
static_assert(32 * W == kRowsTile, "the planner's tile");

// 4 KiB from memory into LDS: lane l's 16 bytes at base + offset[x] go to lds + 1024 x + 16 l.  STREAM: past the caches.
// base may have been read from a lane just before, and a memory instruction must not read a scalar register within 5
// wait states of the vector instruction that wrote it; nobody counts them into inline assembly, so it has them itself:
// one of the move, four of the s_nop.  (Setting m0 takes one more only before a load that uses it.)
#pragma clang diagnostic ignored "-Winline-asm"  // m0 as a clobber: nothing else here uses it
#define FETCH_4K(hint)                                                                                        \
  asm volatile(                                                                                               \
      "s_mov_b32 m0, %4\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %5" hint                                   \
      "\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5" hint                      \
      "\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %5" hint                      \
      "\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %5" hint ::"v"(offset[0]),    \
      "v"(offset[1]), "v"(offset[2]), "v"(offset[3]), "s"(lds), "s"(base)                                     \
      : "memory", "m0", "scc")
template <bool STREAM>
__device__ __forceinline__ void fetch_4k(uint64_t base, const uint32_t (&offset)[4], uint32_t lds) {
  if (STREAM) FETCH_4K(" nt");
  else FETCH_4K("");
}
#undef FETCH_4K

struct Yes {
  static constexpr bool value = true;
};
struct No {
  static constexpr bool value = false;
};

// Steps in LDS, one in use, the others on their way, and the workgroups whose rings fill a CU's LDS.  With 16 columns,
// where the start of many short lists counts, four workgroups of a ring of 2 (2048 single tokens, window 64: 173 us,
// three of 3: 203; 24 ragged drafts 71, 76); with 32, three of 3, but the three terms of an fp32 result's weights take
// the registers of one.
template <int COLS>
constexpr int kRingSteps = COLS == 16 ? 2 : 3;
template <bool BF16, int COLS>
constexpr int kWavesPerSimd = COLS == 16 ? 4 : BF16 ? 3 : 2;

template <RowsMode MODE, bool BF16, int COLS>
__global__ __launch_bounds__(64 * W)
__attribute__((amdgpu_waves_per_eu(kWavesPerSimd<BF16, COLS>, kWavesPerSimd<BF16, COLS>)))
void rows_attn_kernel(RowsAttnArgs a) {
  constexpr bool kWide = COLS == 32;
  constexpr int kRing = kRingSteps<COLS>;
  constexpr int CT = COLS * W;          // columns of a workgroup
  constexpr int kLoads = 4;             // requests of a wavefront and step, 1 KiB each
  constexpr int kTerms = BF16 ? 1 : 3;  // bf16 parts of a weight
  constexpr int kTok = COLS / 2;        // tokens of a lane and step
  constexpr int kGroups = kTok / 8;     // of 8, an operand of the value product each
  constexpr int kStride = kWide ? 8 : 16;  // this lane's sums: dims kStride j + 4 hi + [0, 4)
  constexpr int kAcc = kHeadDim / kStride;
  constexpr int kQ = kWide ? 8 : 4;
  constexpr int kApart = kWide ? 0 : 64;  // bytes between a step's K tiles
  __shared__ __attribute__((aligned(16))) char ring[kRing * kStep];
  __shared__ int odd_tile[2];  // a V tile had values that are not finite
  const int lane = threadIdx.x & 63, col = lane & (COLS - 1), hi = lane / COLS;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned chunk = a.by_tiles.quotient(blockIdx.x);
  // The last tiles of a prompt see the most tokens: they start first, so that short ones fill the end (a prompt of
  // 8000 tokens 568 -> 516 us, six of 750, window 512, 55 -> 46).
  const Tile t = find_tile<MODE, CT>(a, a.tiles - 1 - (blockIdx.x - chunk * a.tiles), lane);
  if (!t.any) return;
  const int C = t.n * a.G;
  const Ranges rg = find_ranges<MODE>(a, t, t.c0, min(t.c0 + CT, C), lane);
  // This chunk's steps [s0, s0 + np) of the list's.
  const int steps = (rg.total + 1) >> 1;
  const int per = max((int)(((unsigned)steps + a.nc - 1) / (unsigned)a.nc), a.least);
  const int s0 = min((int)chunk * per, steps), np = min(per, steps - s0);

  // This lane's column.
  const int c_own = t.c0 + wave * COLS + col;
  const bool active = t.c0 + wave * COLS < C, live = c_own < C;
  const int i_own = live ? (int)a.by_g.quotient(c_own) : t.n - 1, h_own = live ? c_own - i_own * a.G : 0;
  const int64_t row = (int64_t)(t.r0 + i_own) * a.Hq + t.g * a.G + h_own;
  const Sight<MODE> sight = sight_of<MODE>(a, t, i_own);
  bf16x8 qop[kQ];
#pragma unroll
  for (int kk = 0; kk < kQ; ++kk) {
    u32x4 x = *reinterpret_cast<const u32x4*>(a.q + row * kHeadDim + (kHeadDim / kQ) * kk + 8 * hi);
    if (!live) x = u32x4{0u, 0u, 0u, 0u};
    qop[kk] = __builtin_bit_cast(bf16x8, x);
  }
  int p0 = 0, p1 = 0;  // positions of the tile's first and last row
  if (MODE == RowsMode::kWindow) {
    const int base = t.tokens - t.n;
    p0 = max(base + (int)a.by_g.quotient(t.c0), -1);
    p1 = max(base + (int)a.by_g.quotient(min(t.c0 + CT, C) - 1), 0);
  }

  f32x4 acc[kAcc];
#pragma unroll
  for (int j = 0; j < kAcc; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;                // running maximum (in powers of two) and this lane's share of the sum
  float minus_base = 0.f, limit = -INFINITY;   // -m (0 while nothing is seen); scores above this raise the maximum

  if (np > 0) {
    // Requests: wavefronts 0 and 1 bring the K tiles of a step's blocks, 2 and 3 the V tiles.
    const bool is_v = wave >= 2;
    const int x_of = wave & 1;  // block of the step
    uint32_t lane_off[4];
#pragma unroll
    for (int x = 0; x < 4; ++x)
      lane_off[x] = 1024 * x + (is_v ? (lane >> 5) * 512 + (lane & 15) * 32 + ((lane >> 4) & 1) * 16 : lane * 16);
    const uint32_t ring_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)ring +
                             (is_v ? kKStep : kApart * x_of) + x_of * kTileBytes;
    const uint64_t pool = reinterpret_cast<uint64_t>(is_v ? a.v : a.k);
    uint32_t tile_lo = 0, tile_hi = 0;  // addresses of the wavefront's tiles, 64 steps at a time, one per lane
    auto request = [&](int step, int at) __attribute__((always_inline)) {  // into the ring at byte `at`
      if ((step & 63) == 0) {
        const int blk = pool_blocks(a, rg, t.b, 2 * (s0 + step + lane) + x_of);
        const uint64_t tile = pool + kv_tile(blk, t.g, a.s.Hkv) * kTileBytes;
        tile_lo = (uint32_t)tile, tile_hi = (uint32_t)(tile >> 32);
      }
      const uint64_t base = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(tile_hi, step & 63) << 32 |
                            (uint32_t)__builtin_amdgcn_readlane(tile_lo, step & 63);
      fetch_4k<!kWide>(base, lane_off, __builtin_amdgcn_readfirstlane(ring_at + at));
    };
    float s[kTok];
    u32x4 pw[kGroups][kTerms];  // weights of the step as operands
    int cur = 0;                // the step's place in the ring
    // Where this lane's fragments start: row `col` of a score product is block col / 16 [col / 8], slot
    // 8 (col >> 2 & 1) + 4 (col >> 3 & 1) [+ 0, 4 for the second product] + (col & 3).
    const char* k_frag = ring + (kWide ? col >> 4 : col >> 3) * (kTileBytes + kApart) + hi * 256 +
                         (8 * ((col >> 2) & 1) + (kWide ? 4 * ((col >> 3) & 1) : 0) + (col & 3)) * 16;
    const char* v_frag = ring + kKStep + (col & 15) * 16 +
                         (kWide ? (col >> 4) * 512 + hi * 256 : (hi >> 1) * kTileBytes + (hi & 1) * 256);

    auto scores = [&]() __attribute__((always_inline)) {
      const char* kt = k_frag + cur;
      if constexpr (kWide) {
        f32x16 x = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kt + 512 * kk), qop[kk], x,
                                                      0, 0, 0);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = x[e];
      } else {
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8*>(kt + 64 * y + 1024 * kk),
                                                        qop[kk], x, 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[4 * y + e] = x[e];
        }
      }
    };
    // The step's weights as operands; this lane's sum of them.
    auto weights = [&]() __attribute__((always_inline)) -> float {
      float sum[kTok / 2];
#pragma unroll
      for (int e = 0; e < kTok / 2; ++e) {
        const int g = e >> 2, at = e & 3;
        float x = exp2_of(fmaf(s[2 * e], a.scale, minus_base));
        float y = exp2_of(fmaf(s[2 * e + 1], a.scale, minus_base));
        sum[e] = x + y;
        pw[g][0][at] = bf16_pair(x, y);
        if constexpr (kTerms == 3) {
          x -= low_value(pw[g][0][at]), y -= high_value(pw[g][0][at]);
          pw[g][1][at] = bf16_pair(x, y);
          x -= low_value(pw[g][1][at]), y -= high_value(pw[g][1][at]);
          pw[g][2][at] = bf16_pair(x, y);
        }
      }
#pragma unroll
      for (int n = kTok / 4; n >= 1; n /= 2)
#pragma unroll
        for (int e = 0; e < n; ++e) sum[e] += sum[e + n];
      return sum[0];
    };
    auto values = [&]() __attribute__((always_inline)) {
      const char* vt = v_frag + cur;
      if constexpr (kWide) {
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
          f32x16 x;
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = acc[4 * dt + (r >> 2)][r & 3];
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            const bf16x8 vf = *reinterpret_cast<const bf16x8*>(vt + g * kTileBytes + 1024 * dt);
#pragma unroll
            for (int term = 0; term < kTerms; ++term)
              x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, pw[g][term]), x, 0, 0, 0);
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[4 * dt + (r >> 2)][r & 3] = x[r];
        }
      } else {
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
          const bf16x8 vf = *reinterpret_cast<const bf16x8*>(vt + 512 * dt);
#pragma unroll
          for (int term = 0; term < kTerms; ++term)
            acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, pw[0][term]), acc[dt],
                                                              0, 0, 0);
        }
      }
    };
    // A V tile that not every row sees whole, before the products read it: tokens outside the range are cleared
    // (their slots may hold anything), and values that are not finite too, as a weight of 0 would not keep them
    // from the rows that do not see them.  Whether there were any: the rows that do see them take them one by one.
    auto clean = [&](int first, int from, int end) __attribute__((always_inline)) {
      char* vt = ring + cur + kKStep + x_of * kTileBytes;
      bool odd = false;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        u32x4* at = reinterpret_cast<u32x4*>(vt + 1024 * x + 16 * lane);  // 8 tokens of one dim
        u32x4 val = *at;
        const int tok = first + ((lane >> 4) & 1) * 8;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int u = tok + 2 * e;
          val[e] &= (u >= from && u < end ? 0x0000FFFFu : 0u) | (u + 1 >= from && u + 1 < end ? 0xFFFF0000u : 0u);
          if ((val[e] & 0x7F80u) == 0x7F80u) val[e] &= 0xFFFF0000u, odd = true;
          if ((val[e] & 0x7F800000u) == 0x7F800000u) val[e] &= 0x0000FFFFu, odd = true;
        }
        *at = val;
      }
      const bool any = __any(odd);
      if (lane == 0) odd_tile[x_of] = any;
    };
    auto odd_values = [&](Block c, int x) __attribute__((always_inline)) {
      const int blk_of = min(max(table_lookup(a.table, a.s.max_blocks, t.b, c.first >> 4), 0), a.s.last_block);
      const uint16_t* vt = a.v + kv_tile(blk_of, t.g, a.s.Hkv) * kTileElems;
#pragma unroll 1
      for (int slot = 0; slot < kBlockSize; ++slot) {
        const int tok = c.first + slot;
        if (tok < c.t0 || tok >= c.t1) continue;
        const int from = ((kWide ? 0 : 2 * x) + (slot >> 3)) * COLS + col;  // the lane with this token's weight
        float w = 0.f;
#pragma unroll
        for (int term = 0; term < kTerms; ++term) {
          uint32_t w4[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t lower = pw[0][term][e], upper = pw[kGroups - 1][term][e];
            w4[e] = x ? upper : lower;
          }
          const uint32_t lo = slot & 4 ? w4[2] : w4[0], up = slot & 4 ? w4[3] : w4[1];
          const uint32_t pair = (uint32_t)__shfl((int)(slot & 2 ? up : lo), from);
          w += slot & 1 ? high_value(pair) : low_value(pair);
        }
        if (!seen<MODE>(a, rg, c, sight, tok)) w = -1.f;
#pragma unroll
        for (int j = 0; j < kAcc; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t bits = vt[(kStride * j + 4 * hi + e) * kBlockSize + slot];
            const bool take = ((bits & 0x7F80u) == 0x7F80u) & !(w < 0.f);
            acc[j][e] += take ? w * low_value(bits) : 0.f;
          }
      }
    };

    // The sums follow the maximum where a score exceeds it by more than the slack.
    auto raise_maximum = [&]() __attribute__((always_inline)) {
      float top = s[0];
#pragma unroll
      for (int e = 1; e < kTok; ++e) top = fmaxf(top, s[e]);
      if (__any(top > limit)) {
        float x = top * a.scale;
        if (!kWide) x = fmaxf(x, __shfl_xor(x, 16));
        x = fmaxf(x, __shfl_xor(x, 32));
        const float m_new = fmaxf(m, x);
        minus_base = m_new == -INFINITY ? 0.f : -m_new;
        const float alpha = exp2_of(m + minus_base);
        m = m_new;
        limit = (m + kSlack) / a.scale;
        l *= alpha;
#pragma unroll
        for (int j = 0; j < kAcc; ++j) acc[j] *= alpha;
      }
    };
    auto next = [&](int i) __attribute__((always_inline)) {
      // Everybody's tiles of this step are there, and nobody reads those of the step before.
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kRing - 2) * kLoads) : "memory");
      race_check_delay(wave);
      request(i + kRing - 1, cur == 0 ? (kRing - 1) * kStep : cur - kStep);
    };
    bool slow = false;  // take every step as one that not every row sees whole
    auto walk = [&](auto computes) __attribute__((always_inline)) {
      constexpr bool kComputes = decltype(computes)::value;
      Cursor c;
      Block now0, now1;
      int whole = 0;  // steps from here on that all rows see whole
#pragma unroll 1
      for (int i = 0; i < np; ++i) {
        next(i);
        bool part = false;
        if (whole == 0) {
          const int v = 2 * (s0 + i);
          c.seek<MODE>(a, rg, v, p0, p1);
          if (v >= c.wbegin && !slow) whole = max((c.wend - v) >> 1, 0);
          part = whole == 0;
          if (part) {
            now0 = block_at<MODE>(a, rg, c, v, p0, p1);
            now1 = block_at<MODE>(a, rg, c, v + 1, p0, p1);
            race_check_delay(wave);
            if (is_v) clean(x_of ? now1.first : now0.first, x_of ? now1.t0 : now0.t0, x_of ? now1.t1 : now0.t1);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
          }
        }
        if (!part) --whole;
        if constexpr (kComputes) {
          scores();
          if (part) {
#pragma unroll
            for (int e = 0; e < kTok; ++e) {
              const bool second = kWide ? e >= 8 : hi >= 2;  // the token's block
              const Block mine = {second ? now1.first : now0.first, second ? now1.t0 : now0.t0,
                                  second ? now1.t1 : now0.t1, second ? now1.tree : now0.tree};
              const bool ok = seen<MODE>(a, rg, mine, sight, mine.first + 8 * (hi & 1) + (e & 7));
              s[e] = ok ? s[e] : -INFINITY;
            }
          }
          raise_maximum();
          l += weights();
          if (part) {
#pragma unroll 1
            for (int x = odd_tile[0] ? 0 : 1; x < (odd_tile[1] ? 2 : 1); ++x) odd_values(x ? now1 : now0, x);
          }
          values();
        }
        cur = cur == (kRing - 1) * kStep ? 0 : cur + kStep;
      }
    };
    for (;;) {
#pragma unroll
      for (int x = 0; x < kRing - 1; ++x) request(x, x * kStep);
      if (active) walk(Yes{});
      else walk(No{});
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no request outlives the workgroup's LDS
      if constexpr (kTerms == 1) break;
      // An infinite value that all rows see met the later terms of its weight, which may be 0 or negative: NaN where
      // the definition has the infinity.  Where sums are not finite though the weights are, once more, the slow way.
      // The look at the sums costs 0.1 to 1 % (2 x 4096 rows, window 4096, 979 us; 24 x 12 rows over 2000 tokens, 56).
      if (slow) break;
      float lost = 0.f, all = l;  // NaN if any of the sums is not finite
#pragma unroll
      for (int j = 0; j < kAcc; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) lost = fmaf(acc[j][e], 0.f, lost);
      if (!kWide) all += __shfl_xor(all, 16);
      all += __shfl_xor(all, 32);
      if (!__syncthreads_or(live & (all > 0.f) & (lost != lost))) break;
      slow = true;
      cur = 0, l = 0.f, m = limit = -INFINITY, minus_base = 0.f;
#pragma unroll
      for (int j = 0; j < kAcc; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  if (!active) return;
  if (!kWide) l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (!live) return;
  if (a.nc == 1) {
    store_row<BF16, kStride>(a.out, a.lse, row, acc, l, m, 4 * hi);
  } else if (np > 0) {  // a chunk's partial row
    const int64_t base = (int64_t)chunk * a.rows * a.Hq;
    store_row<false, kStride>(a.part_out + base * kHeadDim, a.part_lse + base, row, acc, l, m, 4 * hi);
  } else if (hi == 0) {
    a.part_lse[(int64_t)chunk * a.rows * a.Hq + row] = -INFINITY;
  }
}

// Merge of the chunks' partial rows (as merge.hip's, on packed rows): out = sum_c w_c out_c / sum_c w_c with
// w_c = exp(lse_c - max).  32 lanes read a row, KP groups of them share its chunks.
template <bool BF16, int KP>
__global__ __launch_bounds__(32 * (KP < 8 ? 8 : KP)) void rows_merge_kernel(RowsAttnArgs a) {
  constexpr int kRows = KP < 8 ? 8 / KP : 1;  // rows of a workgroup
  __shared__ float sm_m[kRows * KP], sm_l[kRows * KP];
  __shared__ f32x4 sm_o[kRows * KP][32];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, k = group % KP;
  const int64_t first = (int64_t)row_start(a.row_begin, 0, a.rows) * a.Hq;
  const int64_t r = first + (int64_t)blockIdx.x * kRows + group / KP, n = (int64_t)a.rows * a.Hq;
  const bool live = r < (int64_t)row_start(a.row_begin, a.s.B, a.rows) * a.Hq;
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if (live) {
    for (int c0 = k; c0 < a.nc; c0 += 4 * KP) {
      float x[4];
      f32x4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int c = min(c0 + u * KP, a.nc - 1);
        x[u] = a.part_lse[c * n + r];
        if (KP > 1) v[u] = reinterpret_cast<const f32x4*>(a.part_out + (c * n + r) * kHeadDim)[lane];
      }
      if (KP == 1) {  // many rows: only the parts that are not empty (24 ragged drafts 78.6 -> 76.8 us)
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (x[u] != -INFINITY)
            v[u] = reinterpret_cast<const f32x4*>(a.part_out + (min(c0 + u, a.nc - 1) * n + r) * kHeadDim)[lane];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (c0 + u * KP >= a.nc || x[u] == -INFINITY) continue;  // an empty part's row may hold anything
        const float m_new = fmaxf(m, x[u]);
        const float w = expf(x[u] - m_new), old = m == -INFINITY ? 0.f : expf(m - m_new);
        l = l * old + w;
        o = o * old + w * v[u];
        m = m_new;
      }
    }
  }
  if (KP > 1) {
    race_check_delay(threadIdx.x >> 6);
    if (lane == 0) sm_m[group] = m, sm_l[group] = l;
    sm_o[group][lane] = o;
    __syncthreads();
    race_check_barrier();
    if (!live || k != 0) return;
    float M = -INFINITY;
#pragma unroll
    for (int i = 0; i < KP; ++i) M = fmaxf(M, sm_m[group + i]);
    l = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < KP; ++i) {
      // A group without a live part adds nothing; one whose only parts are NaN has no maximum but NaN sums.
      const float mi = sm_m[group + i], li = sm_l[group + i];
      if (li == 0.f) continue;
      const float w = mi == M ? 1.f : expf(mi - M);
      l += w * li;
      o += w * sm_o[group + i][lane];
    }
    m = M;
  }
  if (!live) return;
  const bool empty = l == 0.f;
  o *= empty ? 0.f : 1.0f / l;
  if (BF16)
    reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + r * kHeadDim)[lane] =
        u32x2{bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3])};
  else
    reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + r * kHeadDim)[lane] = o;
  if (a.lse != nullptr && lane == 0) a.lse[r] = empty ? -INFINITY : m + logf(l);
}

template <RowsMode MODE, bool BF16>
void launch_tiles(const RowsAttnArgs& a, hipStream_t stream) {
  const dim3 grid(a.tiles * (unsigned)a.nc), block(64 * W);
  if (a.tile == kRowsTile) hipLaunchKernelGGL((rows_attn_kernel<MODE, BF16, 32>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((rows_attn_kernel<MODE, BF16, 16>), grid, block, 0, stream, a);
}

template <bool BF16>
void launch_merge_rows(const RowsAttnArgs& a, hipStream_t stream) {
  const int64_t n = (int64_t)a.rows * a.Hq;
  if (a.merge_groups == 1)
    hipLaunchKernelGGL((rows_merge_kernel<BF16, 1>), dim3((unsigned)((n + 7) / 8)), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((rows_merge_kernel<BF16, 8>), dim3((unsigned)n), dim3(256), 0, stream, a);
}

}  // namespace

hipError_t launch_rows_attn(const RowsAttnArgs& args, RowsMode mode, bool bf16, hipStream_t stream) {
  RowsAttnArgs a = args;
  const int64_t slots = (int64_t)a.rows * a.G / a.tile + a.s.B;
  a.tiles = (unsigned)slots * (unsigned)a.s.Hkv;
  a.seqs_per_slot = (float)a.s.B / (float)slots;
  a.count_tiles = a.s.B > 1 && a.s.B <= 64 && (int64_t)a.rows * a.G * 4 >= (int64_t)a.tile * a.s.B &&
                  (int64_t)a.rows * a.G < (int64_t)a.tile * a.s.B * 8;
  a.by_tiles.set(a.tiles);
  if (mode == RowsMode::kTree) {
    if (bf16) launch_tiles<RowsMode::kTree, true>(a, stream);
    else launch_tiles<RowsMode::kTree, false>(a, stream);
  } else {
    if (bf16) launch_tiles<RowsMode::kWindow, true>(a, stream);
    else launch_tiles<RowsMode::kWindow, false>(a, stream);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.nc == 1) return e;
  if (bf16) launch_merge_rows<true>(a, stream);
  else launch_merge_rows<false>(a, stream);
  return hipGetLastError();
}

}  // namespace bana
