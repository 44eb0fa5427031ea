// tokens_api.cpp -- C ABI of bana_tokens.h: argument checks, launch planning, launches.
//
// As in bana_api.cpp, everything that the host can see is checked before HIP is touched, and plans are a pure
// function of the dims and sizes of the call.
#include "bana_tokens.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "api_checks.h"
#include "tokens.h"

namespace {

using bana::aligned16;
using bana::check_dims;
using bana::device_status;

constexpr int kHeadDim = 128;
constexpr int kBlockSize = 16;
constexpr int64_t kMaxRows = int64_t{1} << 24;           // rows: a workgroup of 256 threads each in 32 bits
constexpr int64_t kMaxHeadRows = int64_t{1} << 26;       // rows x heads
constexpr int64_t kMaxPairs = int64_t{1} << 23;          // batch x kv heads of an attention: its workgroups likewise
constexpr int64_t kMaxTokenPairs = int64_t{1} << 18;     // of append and compact: 32 workgroups each in 32 bits
constexpr int kMaxForks = 1 << 20;                       // 8 workgroups each in 32 bits
constexpr int kMaxKept = 1 << 30;                        // places of a step past the list's end in 32 bits
constexpr int kMaxTreeParts = 63;                        // ranges of a tree call: with the nodes, one per lane
constexpr int64_t kMaxLaunchItems = UINT32_MAX;          // work-items of one launch
constexpr int kMaxChunks = 128;
constexpr int kMinChunkSteps = 2;
constexpr double kStepLatencyUs = 0.7;                   // of the planner's estimate (plan_rows)
constexpr double kStartSteps = 1.5;                      // a workgroup's start, in steps
constexpr double kRoundUs = 3;                           // a round of workgroups behind the first
constexpr double kMergeUs = 4;
constexpr double kPartBytesPerUs = 4e6;
constexpr int kRowsTileRows = 128;                       // rows of a tile at most (a group of 1)
constexpr int64_t kMaxListBlocks = int64_t{1} << 30;     // blocks of all ranges of a sequence

bana::CacheShape shape_of(const bana_dims* d) {
  return {d->batch, d->num_kv_heads, d->max_blocks_per_seq,
          (int)std::min<int64_t>(d->num_blocks - 1, INT32_MAX)};
}

bana_status check_rows(const bana_dims* d, int64_t rows, int heads) {
  if (rows < 0) return BANA_ERR_INVALID;
  return rows >= kMaxRows || rows * heads >= kMaxHeadRows ? BANA_ERR_UNSUPPORTED : BANA_OK;
}

// What both attention calls check.
bana_status check_attention(const bana_dims* d, int64_t rows, const int32_t* row_begin, const void* q,
                            const void* k_cache, const void* v_cache, const int32_t* block_table, float scale,
                            const void* out, int32_t out_type, const void* workspace) {
  bana_status st = check_dims(d);
  if (st == BANA_OK) st = check_rows(d, rows, d->num_q_heads);
  if (st == BANA_OK && (int64_t)d->batch * d->num_kv_heads > kMaxPairs) st = BANA_ERR_UNSUPPORTED;
  if (st != BANA_OK) return st;
  if (!row_begin || !q || !k_cache || !v_cache || !block_table || !out) return BANA_ERR_INVALID;
  if (out_type != BANA_OUT_F32 && out_type != BANA_OUT_BF16) return BANA_ERR_INVALID;
  if (!(scale > 0.f) || !std::isfinite(scale * 1.5f)) return BANA_ERR_INVALID;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out) ||
      (workspace != nullptr && !aligned16(workspace)))
    return BANA_ERR_INVALID;
  return BANA_OK;
}

bana::RowsAttnArgs attention_args(const bana_dims* d, int64_t rows, const int32_t* row_begin, const void* q,
                                  const void* k_cache, const void* v_cache, const int32_t* block_table, float scale,
                                  void* out, float* lse) {
  bana::RowsAttnArgs a{};
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k_cache);
  a.v = static_cast<const uint16_t*>(v_cache);
  a.table = block_table;
  a.row_begin = row_begin;
  a.scale = (float)((double)scale * 1.4426950408889634);
  a.rows = (int)rows;
  a.Hq = d->num_q_heads;
  a.G = d->num_q_heads / d->num_kv_heads;
  a.s = shape_of(d);
  a.by_hkv.set((uint32_t)d->num_kv_heads);
  a.by_g.set((uint32_t)a.G);
  a.out = out;
  a.lse = lse;
  return a;
}

// How a call's tiles are cut.  A tile is 128 columns (rows x heads of a group), or 64 where sequences have no more
// on the mean: four wavefronts of 16 columns then share what two of 32 would do one after the other (24 drafts of
// 13 nodes, groups of 4, fp32: 106 -> 71 us), and the loads go past the caches, as most sequences then have one tile (of
// those drafts some have two that read the same context, and it is 76 us so, 78 otherwise).
//
// A tile's list of steps (32 tokens) is cut into chunks where that is estimated to be faster.  With n
// workgroups at work, of at most `slots`, a step takes max(latency, n x step_us): alone it is bound by the chain of
// its products, all together by HBM or the matrix and vector units.  Each workgroup's start costs it
// kStartSteps more, a round of them behind the first kRoundUs; the last chunks run on while the GPU empties, a
// quarter of a chunk's latency on the mean; each chunk's partial rows are written and read once more, after a launch.
// Times in us, measured on MI355X (step_us is the whole call's time per step, here in ns):
//   64 columns, bf16 / fp32:  2.5 / 2.7     128 columns, bf16 / fp32:  2.2 / 4.4     latency of a step 0.7
// Calls that fixed the rule, one chunk -> as planned: 8 rows over 700 tokens 34 -> 11.8; 64 rows, window 4096, 178
// -> 168; 1 row over 16000 tokens 211 -> 18.5; 2048 rows x 64 heads, 3200 to 12800 tokens, 646 -> 618; prompts of 750
// rows, window 512, stay whole (46, in two chunks 83).
//
// A chunk is never shorter than planned for the longest list, so that short lists do not make many.  Without the
// hint max_range_tokens that is the table's span, and a list far below it stays in one chunk.
struct RowsPlan {
  int nc = 1;
  int least = 1;  // steps of a chunk at least
  int merge_groups = 1;
  int tile = bana::kRowsTile;
};

// The call's longest row sees at most `tokens` tokens.
RowsPlan plan_rows(const bana_dims* d, int64_t rows, int64_t tokens, bool bf16) {
  RowsPlan p;
  const int G = d->num_q_heads / d->num_kv_heads;
  const bool thin = rows * G <= (int64_t)d->batch * (bana::kRowsTile / 2);
  p.tile = thin ? bana::kRowsTile / 2 : bana::kRowsTile;
  const int64_t tiles = std::max<int64_t>(rows * G / p.tile, std::min<int64_t>(d->batch, rows));
  const double groups = (double)tiles * d->num_kv_heads;
  const int64_t steps = std::max<int64_t>(1, (tokens + bana::kRowsStep - 1) / bana::kRowsStep);
  const int64_t mean = d->total_range_tokens > 0
                           ? std::min<int64_t>(steps, d->total_range_tokens / d->batch / bana::kRowsStep + 1)
                           : steps;
  const double slots = thin ? 1024 : bf16 ? 768 : 512;
  const double step_us = (thin ? (bf16 ? 2.5 : 2.7) : bf16 ? 2.2 : 4.4) * 1e-3;
  const double part_us = (double)rows * d->num_q_heads * 2 * (kHeadDim + 1) * sizeof(float) / kPartBytesPerUs;
  double best = 0;
  for (int nc = 1; nc <= kMaxChunks; ++nc) {
    const int64_t chunk = (steps + nc - 1) / nc;
    if (nc > 1 && chunk < kMinChunkSteps) break;
    const double used = mean < steps ? std::min<double>(nc, (double)mean / chunk + 0.5) : nc;  // chunks of a tile
    const double busy = std::min(slots, std::max(groups * used, 1.0));
    const double one = (chunk + kStartSteps) * std::max(kStepLatencyUs, step_us * busy);
    const double all = groups * (mean + used * kStartSteps) * step_us + 0.25 * chunk * kStepLatencyUs +
                       kRoundUs * std::max(groups * used / slots - 1, 0.0);
    const double time = std::max(one, all) + (nc > 1 ? kMergeUs + used * part_us : 0);
    if (nc == 1 || time < best) {
      best = time;
      p.nc = nc;
      p.least = (int)std::min<int64_t>(chunk, INT32_MAX);
    }
  }
  const int64_t launched = (rows * G / p.tile + d->batch) * d->num_kv_heads;
  if (launched * p.nc * 256 > kMaxLaunchItems) p.nc = 1;
  p.merge_groups = rows * d->num_q_heads < 4096 && p.nc > 4 ? 8 : 1;
  return p;
}

// Workspace: partial rows [nc][rows][Hq][128] fp32, then their lse.
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
size_t part_bytes(const bana_dims* d, int64_t rows, const RowsPlan& p) {
  return align256((size_t)p.nc * rows * d->num_q_heads * kHeadDim * sizeof(float));
}
size_t workspace_for(const bana_dims* d, int64_t rows, const RowsPlan& p) {
  if (p.nc == 1) return 0;
  return part_bytes(d, rows, p) + align256((size_t)p.nc * rows * d->num_q_heads * sizeof(float));
}

// The most tokens that a sequence has in the cache.
int64_t longest(const bana_dims* d) {
  const int64_t span = (int64_t)d->max_blocks_per_seq * kBlockSize;
  return d->max_range_tokens > 0 ? std::min<int64_t>(span, d->max_range_tokens) : span;
}
int64_t window_tokens(const bana_dims* d, int32_t window, int32_t sinks) {
  return std::min<int64_t>(longest(d), (int64_t)window + sinks + kRowsTileRows);
}

void set_plan(bana::RowsAttnArgs& a, const bana_dims* d, RowsPlan p, void* workspace, size_t workspace_bytes) {
  if (p.nc > 1 && (workspace == nullptr || workspace_bytes < workspace_for(d, a.rows, p))) p.nc = p.least = 1;
  a.tile = p.tile;
  a.nc = p.nc;
  a.least = p.least;
  a.merge_groups = p.merge_groups;
  if (p.nc > 1) {
    a.part_out = static_cast<float*>(workspace);
    a.part_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) + part_bytes(d, a.rows, p));
  }
}

// The workspace of a call with either type of result.
size_t most_workspace(const bana_dims* d, int64_t rows, int64_t tokens) {
  return std::max(workspace_for(d, rows, plan_rows(d, rows, tokens, true)),
                  workspace_for(d, rows, plan_rows(d, rows, tokens, false)));
}

bool plannable(const bana_dims* d, int64_t rows) {
  return check_dims(d) == BANA_OK && rows > 0 && check_rows(d, rows, d->num_q_heads) == BANA_OK &&
         (int64_t)d->batch * d->num_kv_heads <= kMaxPairs;
}

}  // namespace

extern "C" {

size_t bana_tree_attn_workspace_bytes(const bana_dims* d, int64_t rows, int32_t n_parts) {
  if (!plannable(d, rows) || n_parts < 1 || n_parts > kMaxTreeParts) return 0;
  return most_workspace(d, rows, longest(d));
}

size_t bana_window_attn_workspace_bytes(const bana_dims* d, int64_t rows, int32_t window, int32_t sinks) {
  if (!plannable(d, rows) || window < 1 || sinks < 0) return 0;
  return most_workspace(d, rows, window_tokens(d, window, sinks));
}

bana_status bana_tree_attn(const bana_dims* d, int64_t rows, const int32_t* row_begin, const void* q,
                           const void* k_cache, const void* v_cache, const int32_t* block_table,
                           const int32_t* kv_range_begin, const int32_t* kv_range_end, int32_t n_parts,
                           const int32_t* tree_begin, const uint64_t* tree_mask, float scale, void* out,
                           int32_t out_type, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  const bana_status st =
      check_attention(d, rows, row_begin, q, k_cache, v_cache, block_table, scale, out, out_type, workspace);
  if (st != BANA_OK) return st;
  if (!kv_range_begin || !kv_range_end || !tree_begin || !tree_mask || n_parts < 1) return BANA_ERR_INVALID;
  if (n_parts > kMaxTreeParts || (int64_t)n_parts * d->max_blocks_per_seq > kMaxListBlocks)
    return BANA_ERR_UNSUPPORTED;
  if (rows == 0) return BANA_OK;
  bana::RowsAttnArgs a = attention_args(d, rows, row_begin, q, k_cache, v_cache, block_table, scale, out, lse);
  a.begin = kv_range_begin;
  a.end = kv_range_end;
  a.n_parts = n_parts;
  a.tree_begin = tree_begin;
  a.mask = tree_mask;
  set_plan(a, d, plan_rows(d, rows, longest(d), out_type == BANA_OUT_BF16), workspace, workspace_bytes);
  return device_status(bana::launch_rows_attn(a, bana::RowsMode::kTree, out_type == BANA_OUT_BF16,
                                              static_cast<hipStream_t>(stream)));
}

bana_status bana_window_attn(const bana_dims* d, int64_t rows, const int32_t* row_begin, const void* q,
                             const void* k_cache, const void* v_cache, const int32_t* block_table,
                             const int32_t* seq_lens, const int32_t* kv_range_begin, const int32_t* kv_range_end,
                             int32_t window, int32_t sinks, float scale, void* out, int32_t out_type, float* lse,
                             void* workspace, size_t workspace_bytes, void* stream) {
  const bana_status st =
      check_attention(d, rows, row_begin, q, k_cache, v_cache, block_table, scale, out, out_type, workspace);
  if (st != BANA_OK) return st;
  if (!seq_lens || (kv_range_begin == nullptr) != (kv_range_end == nullptr) || window < 1 || sinks < 0)
    return BANA_ERR_INVALID;
  if (rows == 0) return BANA_OK;
  bana::RowsAttnArgs a = attention_args(d, rows, row_begin, q, k_cache, v_cache, block_table, scale, out, lse);
  a.begin = kv_range_begin;
  a.end = kv_range_end;
  a.seq_lens = seq_lens;
  a.window = window;
  a.sinks = sinks;
  const RowsPlan p = plan_rows(d, rows, window_tokens(d, window, sinks), out_type == BANA_OUT_BF16);
  set_plan(a, d, p, workspace, workspace_bytes);
  return device_status(bana::launch_rows_attn(a, bana::RowsMode::kWindow, out_type == BANA_OUT_BF16,
                                              static_cast<hipStream_t>(stream)));
}

bana_status bana_append_kv(const bana_dims* d, int64_t rows, const int32_t* row_begin, const int32_t* first_token,
                           const void* k_rows, const void* v_rows, const int32_t* block_table, void* k_cache,
                           void* v_cache, void* stream) {
  bana_status st = check_dims(d);
  if (st == BANA_OK) st = check_rows(d, rows, d->num_kv_heads);
  if (st == BANA_OK && (int64_t)d->batch * d->num_kv_heads > kMaxTokenPairs) st = BANA_ERR_UNSUPPORTED;
  if (st != BANA_OK) return st;
  if (!row_begin || !first_token || !k_rows || !v_rows || !block_table || !k_cache || !v_cache)
    return BANA_ERR_INVALID;
  if (!aligned16(k_rows) || !aligned16(v_rows) || !aligned16(k_cache) || !aligned16(v_cache)) return BANA_ERR_INVALID;
  if (rows == 0) return BANA_OK;
  return device_status(bana::launch_append(k_rows, v_rows, (int)rows, row_begin, first_token, block_table, k_cache,
                                           v_cache, shape_of(d), static_cast<hipStream_t>(stream)));
}

bana_status bana_compact_kv_tokens(const bana_dims* d, void* k_cache, void* v_cache, const int32_t* block_table,
                                   const int32_t* first_token, const int32_t* kept, int32_t max_kept,
                                   const int32_t* n_kept, void* stream) {
  const bana_status st = check_dims(d);
  if (st != BANA_OK) return st;
  if (!k_cache || !v_cache || !block_table || !first_token || !kept || !n_kept || max_kept < 0)
    return BANA_ERR_INVALID;
  if (!aligned16(k_cache) || !aligned16(v_cache)) return BANA_ERR_INVALID;
  if ((int64_t)d->batch * d->num_kv_heads > kMaxTokenPairs || max_kept >= kMaxKept) return BANA_ERR_UNSUPPORTED;
  if (max_kept == 0) return BANA_OK;
  return device_status(bana::launch_compact(k_cache, v_cache, block_table, first_token, kept, max_kept, n_kept,
                                            shape_of(d), static_cast<hipStream_t>(stream)));
}

size_t bana_kv_blocks_workspace_bytes(const bana_dims* d) {
  if (check_dims(d) != BANA_OK) return 0;
  return bana::kv_blocks_workspace_ints(d->batch, d->max_blocks_per_seq, d->num_blocks) * sizeof(int32_t);
}

bana_status bana_reserve_kv_blocks(const bana_dims* d, int32_t* block_table, const int32_t* seq_lens,
                                   const int32_t* need_lens, int32_t* block_refs, int32_t* status, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  const bana_status st = check_dims(d);
  if (st != BANA_OK) return st;
  if (!block_table || !seq_lens || !need_lens || !block_refs || !status || !workspace || !aligned16(workspace) ||
      !aligned16(block_refs) || workspace_bytes < bana_kv_blocks_workspace_bytes(d))
    return BANA_ERR_INVALID;
  if (d->num_blocks > INT32_MAX) return BANA_ERR_UNSUPPORTED;  // table entries are 32-bit
  if ((int64_t)d->batch * d->max_blocks_per_seq > INT32_MAX) return BANA_ERR_UNSUPPORTED;  // 32-bit sums of entries
  return device_status(bana::launch_reserve(block_table, seq_lens, need_lens, block_refs, d->num_blocks, status,
                                            static_cast<int32_t*>(workspace), shape_of(d),
                                            static_cast<hipStream_t>(stream)));
}

bana_status bana_fork_kv_seqs(const bana_dims* d, const int32_t* src_seq, const int32_t* dst_seq, int32_t n,
                              void* k_cache, void* v_cache, int32_t* block_table, int32_t* seq_lens,
                              int32_t* block_refs, int32_t* status, void* workspace, size_t workspace_bytes,
                              void* stream) {
  const bana_status st = check_dims(d);
  if (st != BANA_OK) return st;
  if (!src_seq || !dst_seq || n < 0 || n > d->batch || !k_cache || !v_cache || !block_table || !seq_lens ||
      !block_refs || !status || !workspace || !aligned16(workspace) || !aligned16(k_cache) || !aligned16(v_cache) ||
      !aligned16(block_refs) || workspace_bytes < bana_kv_blocks_workspace_bytes(d))
    return BANA_ERR_INVALID;
  if (d->num_blocks > INT32_MAX || n >= kMaxForks) return BANA_ERR_UNSUPPORTED;
  if (n == 0) return BANA_OK;
  return device_status(bana::launch_fork(src_seq, dst_seq, n, k_cache, v_cache, block_table, seq_lens, block_refs,
                                         d->num_blocks, status, static_cast<int32_t*>(workspace), shape_of(d),
                                         static_cast<hipStream_t>(stream)));
}

bana_status bana_release_kv_blocks(const bana_dims* d, int32_t* block_table, const int32_t* keep_lens,
                                   int32_t* block_refs, int32_t* status, void* stream) {
  const bana_status st = check_dims(d);
  if (st != BANA_OK) return st;
  if (!block_table || !keep_lens || !block_refs || !status) return BANA_ERR_INVALID;
  if (d->num_blocks > INT32_MAX) return BANA_ERR_UNSUPPORTED;
  return device_status(bana::launch_release(block_table, keep_lens, block_refs, status, shape_of(d),
                                            static_cast<hipStream_t>(stream)));
}

}  // extern "C"
