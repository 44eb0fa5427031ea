// tokens.h -- host-side launchers of the kernels behind bana_tokens.h (internal to libbana.so).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "bana_tokens.h"
#include "kernels.h"

namespace bana {

// The shapes of a call that the kernels index by.
struct CacheShape {
  int B, Hkv, max_blocks;
  int last_block;  // highest block number of the pool that a table entry can name
};

// Attention of packed rows (rows_attn.hip).
struct RowsAttnArgs {
  const uint16_t* q;         // bf16 [rows][Hq][128]
  const uint16_t* k;         // pools and table as in kernels.h
  const uint16_t* v;
  const int32_t* table;
  const int32_t* row_begin;  // [B + 1]
  const int32_t* begin;      // tree: [n_parts][B]; window: [B] or NULL
  const int32_t* end;
  const int32_t* tree_begin; // tree: [B]
  const uint64_t* mask;      // tree: [rows]
  const int32_t* seq_lens;   // window: [B]
  int n_parts, window, sinks;
  float scale;               // of the scores, times log2 e: weights are powers of two
  int rows, Hq, G;
  CacheShape s;
  FastDiv by_hkv, by_g;
  void* out;                 // [rows][Hq][128], fp32 or bf16
  float* lse;                // [rows][Hq] or NULL
  // A tile's steps (32 tokens each) are cut into nc chunks of at least `least` steps, whose partial rows
  // [nc][rows][Hq] the merge joins (nc 1: none); merge_groups (1 or 8) groups of lanes share a row's chunks.
  int tile;  // columns (rows x heads of a group) of a workgroup: kRowsTile or half of it
  int nc, least, merge_groups;
  float* part_out;
  float* part_lse;
  // Set by the launcher:
  unsigned tiles;       // workgroups of a chunk
  float seqs_per_slot;  // sequences per tile of a kv head
  bool count_tiles;     // number the tiles by counting them, not by their sequence's first row
  FastDiv by_tiles;
};

constexpr int kRowsTile = 128;  // columns of a workgroup, half as many where sequences have few
constexpr int kRowsStep = 32;   // tokens of a step

enum class RowsMode { kTree, kWindow };

hipError_t launch_rows_attn(const RowsAttnArgs& a, RowsMode mode, bool bf16, hipStream_t stream);

// New tokens' keys and values into the cache, and kept tokens moved together (tokens.hip).
hipError_t launch_append(const void* k_rows, const void* v_rows, int rows, const int32_t* row_begin,
                         const int32_t* first, const int32_t* table, void* k, void* v, CacheShape s,
                         hipStream_t stream);
hipError_t launch_compact(void* k, void* v, const int32_t* table, const int32_t* first, const int32_t* kept,
                          int max_kept, const int32_t* n_kept, CacheShape s, hipStream_t stream);

// Blocks handed out, shared and taken back (blocks.hip).  workspace: kv_blocks_workspace(B, width, blocks) ints.
inline size_t kv_blocks_workspace_ints(int64_t B, int64_t max_blocks, int64_t num_blocks) {
  const int64_t entries = B * max_blocks;
  return 64 + 2 * (size_t)B + (size_t)(entries < num_blocks ? entries : num_blocks);
}
hipError_t launch_reserve(int32_t* table, const int32_t* lens, const int32_t* need, int32_t* refs, int64_t num_blocks,
                          int32_t* status, int32_t* workspace, CacheShape s, hipStream_t stream);
hipError_t launch_fork(const int32_t* src, const int32_t* dst, int n, void* k, void* v, int32_t* table, int32_t* lens,
                       int32_t* refs, int64_t num_blocks, int32_t* status, int32_t* workspace, CacheShape s,
                       hipStream_t stream);
hipError_t launch_release(int32_t* table, const int32_t* keep, int32_t* refs, int32_t* status, CacheShape s,
                          hipStream_t stream);

}  // namespace bana
