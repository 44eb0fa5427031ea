// sanitize_tokens.cpp -- the entry points of bana_tokens.h built for the CPU with AddressSanitizer and
// UndefinedBehaviorSanitizer, driven by a seeded sweep of ordinary and extreme sizes.  The launchers are
// stubs that check the planned launches against the call's buffers (fake addresses, never dereferenced)
// and the 32-bit launch limits.  Linked with sanitize_host.cpp's stubs for the calls of bana.h.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <cmath>
#include <random>
#include <vector>

#include "tokens.h"

namespace {

long g_case = 0, g_launches = 0;
struct Region {
  uintptr_t lo, hi;
};
std::vector<Region> g_regions;

#define REQUIRE(c)                                                                       \
  do {                                                                                   \
    if (!(c)) {                                                                          \
      fprintf(stderr, "check failed: %s (line %d, case %ld)\n", #c, __LINE__, g_case); \
      abort();                                                                           \
    }                                                                                    \
  } while (0)

bool inside(const void* p, unsigned __int128 bytes) {  // fake buffers are cut at 2^44 bytes, where the next begins
  if (bytes > (uint64_t{1} << 44)) bytes = uint64_t{1} << 44;
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  for (const Region& r : g_regions)
    if (a >= r.lo && (unsigned __int128)a + bytes <= r.hi) return true;
  return false;
}

void check_shape(const bana::CacheShape& s, const int32_t* table) {
  REQUIRE(s.B >= 1 && s.Hkv >= 1 && s.max_blocks >= 1 && s.last_block >= 0);
  REQUIRE(inside(table, (unsigned __int128)s.B * s.max_blocks * 4));
}

}  // namespace

namespace bana {

hipError_t launch_rows_attn(const RowsAttnArgs& a, RowsMode mode, bool bf16, hipStream_t) {
  ++g_launches;
  check_shape(a.s, a.table);
  REQUIRE(a.rows >= 1 && a.G >= 1 && a.G <= 16 && a.G * a.s.Hkv == a.Hq && a.scale > 0 && std::isfinite(a.scale));
  const unsigned __int128 head_rows = (unsigned __int128)a.rows * a.Hq;
  REQUIRE(inside(a.q, head_rows * 256) && inside(a.row_begin, ((unsigned __int128)a.s.B + 1) * 4));
  REQUIRE(inside(a.out, head_rows * 128 * (bf16 ? 2 : 4)) && (a.lse == nullptr || inside(a.lse, head_rows * 4)));
  REQUIRE(a.tile == kRowsTile || a.tile == kRowsTile / 2);
  const uint64_t groups = ((uint64_t)a.rows * a.G / a.tile + a.s.B) * a.s.Hkv;
  REQUIRE(a.nc >= 1 && a.least >= 1 && groups * a.nc * 256 <= UINT32_MAX);
  REQUIRE(a.merge_groups == 1 || a.merge_groups == 8);
  if (a.nc > 1) {
    REQUIRE(inside(a.part_out, head_rows * a.nc * 512) && inside(a.part_lse, head_rows * a.nc * 4));
    REQUIRE((uint64_t)a.rows * a.Hq * (a.merge_groups == 8 ? 256 : 32) <= UINT32_MAX);
  }
  const unsigned __int128 per_seq = (unsigned __int128)a.s.B * 4;
  if (mode == RowsMode::kTree) {
    REQUIRE(a.n_parts >= 1 && a.n_parts <= 63 && inside(a.begin, per_seq * a.n_parts) &&
            inside(a.end, per_seq * a.n_parts));
    REQUIRE(inside(a.tree_begin, per_seq) && inside(a.mask, (unsigned __int128)a.rows * 8));
  } else {
    REQUIRE(inside(a.seq_lens, per_seq) && a.window >= 1 && a.sinks >= 0);
    REQUIRE((a.begin == nullptr) == (a.end == nullptr));
    REQUIRE(a.begin == nullptr || (inside(a.begin, per_seq) && inside(a.end, per_seq)));
  }
  return hipSuccess;
}

hipError_t launch_append(const void* k_rows, const void* v_rows, int rows, const int32_t* row_begin,
                         const int32_t* first, const int32_t* table, void* k, void* v, CacheShape s, hipStream_t) {
  ++g_launches;
  check_shape(s, table);
  REQUIRE(rows >= 1 && ((uint64_t)rows / 16 + 2 * (uint64_t)s.B) * s.Hkv * 256 <= UINT32_MAX);
  const unsigned __int128 bytes = (unsigned __int128)rows * s.Hkv * 256;
  REQUIRE(inside(k_rows, bytes) && inside(v_rows, bytes) && inside(k, 1) && inside(v, 1));
  REQUIRE(inside(row_begin, ((unsigned __int128)s.B + 1) * 4) && inside(first, (unsigned __int128)s.B * 4));
  return hipSuccess;
}

hipError_t launch_compact(void* k, void* v, const int32_t* table, const int32_t* first, const int32_t* kept,
                          int max_kept, const int32_t* n_kept, CacheShape s, hipStream_t) {
  ++g_launches;
  check_shape(s, table);
  REQUIRE(max_kept >= 1 && (uint64_t)s.B * s.Hkv * 32 * 256 <= UINT32_MAX && inside(k, 1) && inside(v, 1));
  REQUIRE(inside(first, (unsigned __int128)s.B * 4) && inside(n_kept, (unsigned __int128)s.B * 4));
  REQUIRE(inside(kept, (unsigned __int128)s.B * max_kept * 4));
  return hipSuccess;
}

void check_blocks(const int32_t* table, const int32_t* refs, int64_t num_blocks, const int32_t* status,
                  const int32_t* ws, const CacheShape& s) {
  ++g_launches;
  check_shape(s, table);
  REQUIRE(num_blocks >= 1 && num_blocks <= INT32_MAX && s.last_block == num_blocks - 1);
  REQUIRE(inside(refs, (unsigned __int128)num_blocks * 4) && inside(status, 4));
  if (ws) REQUIRE(inside(ws, (unsigned __int128)kv_blocks_workspace_ints(s.B, s.max_blocks, num_blocks) * 4));
}

hipError_t launch_reserve(int32_t* table, const int32_t* lens, const int32_t* need, int32_t* refs, int64_t num_blocks,
                          int32_t* status, int32_t* ws, CacheShape s, hipStream_t) {
  check_blocks(table, refs, num_blocks, status, ws, s);
  REQUIRE((int64_t)s.B * s.max_blocks <= INT32_MAX);
  REQUIRE(ws && inside(lens, (unsigned __int128)s.B * 4) && inside(need, (unsigned __int128)s.B * 4));
  return hipSuccess;
}

hipError_t launch_fork(const int32_t* src, const int32_t* dst, int n, void* k, void* v, int32_t* table, int32_t* lens,
                       int32_t* refs, int64_t num_blocks, int32_t* status, int32_t* ws, CacheShape s, hipStream_t) {
  check_blocks(table, refs, num_blocks, status, ws, s);
  REQUIRE(ws && n >= 1 && n <= s.B && (uint64_t)n * 8 * 256 <= UINT32_MAX && inside(k, 1) && inside(v, 1));
  REQUIRE(inside(src, (uint64_t)n * 4) && inside(dst, (uint64_t)n * 4) && inside(lens, (unsigned __int128)s.B * 4));
  return hipSuccess;
}

hipError_t launch_release(int32_t* table, const int32_t* keep, int32_t* refs, int32_t* status, CacheShape s,
                          hipStream_t) {
  check_blocks(table, refs, (int64_t)s.last_block + 1, status, nullptr, s);
  REQUIRE(inside(keep, (unsigned __int128)s.B * 4));
  return hipSuccess;
}

}  // namespace bana

namespace {

std::mt19937_64 g_rng(20260311);

template <typename T>
T pick(std::initializer_list<T> xs) {
  return *(xs.begin() + std::uniform_int_distribution<size_t>(0, xs.size() - 1)(g_rng));
}

void* fake(int i) { return reinterpret_cast<void*>((uintptr_t)(i + 1) << 44); }

}  // namespace

int main(int argc, char** argv) {
  const long n_cases = argc > 1 ? atol(argv[1]) : 20000;
  long ok_calls = 0;
  for (g_case = 0; g_case < n_cases; ++g_case) {
    bana_dims d{};
    d.batch = (int32_t)pick<int64_t>({1, 1, 2, 7, 64, 300, 5000, 65536, 1 << 20, (1 << 26) - 1, 0});
    d.num_kv_heads = (int32_t)pick<int64_t>({1, 2, 8, 40, 128});
    d.num_q_heads = d.num_kv_heads * pick<int>({1, 4, 7, 8, 16, 17});
    d.head_dim = 128, d.block_size = 16;
    d.max_blocks_per_seq = (int32_t)pick<int64_t>({1, 16, 256, 8192, 1 << 20, INT32_MAX / 16, 0});
    d.num_blocks = pick<int64_t>({1, 1000, 100000, INT32_MAX, int64_t{1} << 40});
    d.max_range_tokens = (int32_t)pick<int64_t>({0, 1, 300, 4096, 131072, INT32_MAX, -1});
    d.total_range_tokens = pick<int64_t>({0, 1, (int64_t)d.batch * 1000, int64_t{1} << 50, INT64_MAX});
    const int64_t rows = pick<int64_t>({0, 1, 5, 64, 1000, 8192, 100000, (1 << 24) - 1, 1 << 24, INT64_MAX, -1});
    const int32_t parts = (int32_t)pick<int64_t>({1, 2, 63, 64, 0});
    const int32_t window = (int32_t)pick<int64_t>({1, 100, 4096, INT32_MAX, 0});
    const int32_t sinks = (int32_t)pick<int64_t>({0, 4, 1000, INT32_MAX, -1});
    const float scale = pick<float>({1.0f, 0.0884f, 1e-30f, 3e38f, 0.f});
    const int32_t type = pick<int32_t>({BANA_OUT_F32, BANA_OUT_BF16});
    const int32_t max_kept = (int32_t)pick<int64_t>({0, 1, 64, 100000, INT32_MAX});
    const int32_t n = (int32_t)pick<int64_t>({0, 1, d.batch, (int64_t)d.batch + 1});

    g_regions.clear();
    auto add = [](int i, unsigned __int128 bytes) {
      const uintptr_t lo = reinterpret_cast<uintptr_t>(fake(i));
      const uint64_t size = bytes > (uint64_t{1} << 44) ? uint64_t{1} << 44 : (uint64_t)bytes;
      g_regions.push_back({lo, lo + size});
    };
    const unsigned __int128 B = d.batch > 0 ? d.batch : 1, R = rows > 0 && rows < (1 << 26) ? rows : 1;
    add(0, R * d.num_q_heads * 256);                              // q
    add(1, 1), add(2, 1);                                         // pools
    add(3, B * (d.max_blocks_per_seq > 0 ? d.max_blocks_per_seq : 1) * 4);  // table
    add(4, (B + 1) * 4);                                          // row_begin
    add(5, B * 4 * 63), add(6, B * 4 * 63);                       // ranges
    add(7, B * 4), add(8, R * 8);                                 // tree_begin or lengths, masks
    add(9, R * d.num_q_heads * 128 * (type == BANA_OUT_BF16 ? 2 : 4));
    add(10, R * d.num_q_heads * 4);
    add(11, R * d.num_kv_heads * 256), add(12, R * d.num_kv_heads * 256);
    add(13, B * (max_kept > 0 ? max_kept : 1) * 4);
    add(14, (unsigned __int128)d.num_blocks * 4), add(15, 4);     // counts, status
    const size_t blocks_ws = bana_kv_blocks_workspace_bytes(&d);
    add(16, blocks_ws);
    const size_t tree_ws = bana_tree_attn_workspace_bytes(&d, rows, parts);
    const size_t window_ws = bana_window_attn_workspace_bytes(&d, rows, window, sinks);
    const bool have = pick<int>({0, 1, 1});
    add(17, have ? tree_ws : 0), add(18, have ? window_ws : 0);

    auto I = [&](int i) { return static_cast<int32_t*>(fake(i)); };
    float* lse = pick<int>({0, 1}) ? static_cast<float*>(fake(10)) : nullptr;
    const bool cut = pick<int>({0, 1});
    bana_status st[7];
    st[0] = bana_tree_attn(&d, rows, I(4), fake(0), fake(1), fake(2), I(3), I(5), I(6), parts, I(7),
                           static_cast<uint64_t*>(fake(8)), scale, fake(9), type, lse,
                           have && tree_ws ? fake(17) : nullptr, have ? tree_ws : 0, nullptr);
    st[1] = bana_window_attn(&d, rows, I(4), fake(0), fake(1), fake(2), I(3), I(7), cut ? I(5) : nullptr,
                             cut ? I(6) : nullptr, window, sinks, scale, fake(9), type, lse,
                             have && window_ws ? fake(18) : nullptr, have ? window_ws : 0, nullptr);
    st[2] = bana_append_kv(&d, rows, I(4), I(7), fake(11), fake(12), I(3), fake(1), fake(2), nullptr);
    st[3] = bana_compact_kv_tokens(&d, fake(1), fake(2), I(3), I(7), I(13), max_kept, I(5), nullptr);
    st[4] = bana_reserve_kv_blocks(&d, I(3), I(7), I(5), I(14), I(15), fake(16), blocks_ws, nullptr);
    st[5] = bana_fork_kv_seqs(&d, I(5), I(6), n, fake(1), fake(2), I(3), I(7), I(14), I(15), fake(16), blocks_ws,
                              nullptr);
    st[6] = bana_release_kv_blocks(&d, I(3), I(7), I(14), I(15), nullptr);
    for (bana_status s : st) {
      REQUIRE(s == BANA_OK || s == BANA_ERR_INVALID || s == BANA_ERR_UNSUPPORTED);
      ok_calls += s == BANA_OK;
    }
  }
  printf("sanitized host sweep: %ld cases, %ld calls accepted, %ld launches checked\n", n_cases, ok_calls, g_launches);
  return 0;
}
