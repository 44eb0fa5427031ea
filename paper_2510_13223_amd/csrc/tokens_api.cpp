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
constexpr int kMaxTreeParts = 63;                        // ranges of a tree call: with the nodes, one per lane
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

}  // namespace

extern "C" {

size_t bana_tree_attn_workspace_bytes(const bana_dims* d, int64_t rows, int32_t n_parts) {
  (void)d, (void)rows, (void)n_parts;
  return 0;
}

size_t bana_window_attn_workspace_bytes(const bana_dims* d, int64_t rows, int32_t window, int32_t sinks) {
  (void)d, (void)rows, (void)window, (void)sinks;
  return 0;
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
  (void)workspace_bytes;
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
  (void)workspace_bytes;
  return device_status(bana::launch_rows_attn(a, bana::RowsMode::kWindow, out_type == BANA_OUT_BF16,
                                              static_cast<hipStream_t>(stream)));
}

bana_status bana_append_kv(const bana_dims* d, int64_t rows, const int32_t* row_begin, const int32_t* first_token,
                           const void* k_rows, const void* v_rows, const int32_t* block_table, void* k_cache,
                           void* v_cache, void* stream) {
  bana_status st = check_dims(d);
  if (st == BANA_OK) st = check_rows(d, rows, d->num_kv_heads);
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
  // A workgroup of 256 threads per (sequence, kv head) in 32 bits.
  if ((int64_t)d->batch * d->num_kv_heads >= kMaxRows) return BANA_ERR_UNSUPPORTED;
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
      workspace_bytes < bana_kv_blocks_workspace_bytes(d))
    return BANA_ERR_INVALID;
  if (d->num_blocks > INT32_MAX) return BANA_ERR_UNSUPPORTED;  // table entries are 32-bit
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
      workspace_bytes < bana_kv_blocks_workspace_bytes(d))
    return BANA_ERR_INVALID;
  if (d->num_blocks > INT32_MAX || n >= kMaxRows) return BANA_ERR_UNSUPPORTED;
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
