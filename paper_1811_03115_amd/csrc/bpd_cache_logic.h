// Sizes and launch shapes of the cache operators.  No HIP dependency: bpd_cache.hip includes it, and the host check compiles it with the
// system compiler.
#pragma once

#include <cstddef>
#include <cstdint>

#include "../../include/bpd.h"

namespace {

// bf16 heads of 64 and 128 dimensions lie in operand order, groups of 32 keys; all others as rows
inline bool cache_grouped(const bpd_cache& c) { return c.dtype == BPD_BF16 && c.head_dim != 16; }
inline size_t cache_element(const bpd_cache& c) { return c.dtype == BPD_BF16 ? 2 : 4; }
inline size_t cache_layer_elements(const bpd_cache& c) { return (size_t)c.max_batch * c.n_kv_heads * c.capacity * c.head_dim; }
// What is wrong with a cache's sizes (null: nothing)
inline const char* cache_sizes_wrong(const bpd_cache* c) {
  if (!c) return "cache: null";
  if (c->dtype != BPD_F32 && c->dtype != BPD_BF16) return "cache: dtype is BPD_F32 or BPD_BF16";
  if (c->head_dim != 16 && c->head_dim != 64 && c->head_dim != 128) return "cache: head_dim is 16, 64 or 128";
  if (c->n_layers < 1 || c->max_batch < 1 || c->max_batch > 65535 || c->n_kv_heads < 1 || c->n_kv_heads > 1024) return "cache: n_layers >= 1, max_batch 1..65535, n_kv_heads 1..1024";
  if (c->capacity < 1 || c->capacity > (1 << 24)) return "cache: capacity 1..2^24";
  if (cache_grouped(*c) && c->capacity % 32) return "cache: capacity of a cache in operand order is a multiple of 32";
  return nullptr;
}
inline const char* cache_wrong(const bpd_cache* c) {
  if (const char* w = cache_sizes_wrong(c)) return w;
  if (!c->k || !c->v || ((uintptr_t)c->k & 15) || ((uintptr_t)c->v & 15)) return "cache: k or v null, or not aligned to 16 bytes";
  return nullptr;
}
inline const char* attention_sizes_wrong(const bpd_cache& c, int B, int T, int heads) {
  if (B < 0 || B > c.max_batch) return "attention: B outside 0..max_batch";
  if (T < 0 || T > BPD_TREE_MAX) return "attention: T outside 0..BPD_TREE_MAX";
  if (heads < 1 || heads % c.n_kv_heads || heads / c.n_kv_heads > 64) return "attention: heads are 1 to 64 times the cache's";
  return nullptr;
}
inline const char* block_wrong(const bpd_cache&, int block) {
  return block == 32 || block == 64 || block == 128 ? nullptr : "blocks: 32, 64 or 128 rows";
}
inline size_t summaries_elements(const bpd_cache& c, int block) {
  const size_t tiles = ((size_t)c.capacity / block + 63) / 64;
  return (size_t)c.max_batch * c.n_kv_heads * tiles * 2 * c.head_dim * 64;
}

struct TreePlan { bool rows; int mt, wide, blocks, nsplit; size_t chosen_at, score_at, bytes; };
// Parts that `groups` of 32 keys are split into, for as many (sequence, key head, row block)s as there are: the fewest rounds of as many workgroups as the chip has room for (a CU's
// registers: four of fp32 rows, three of 64 rows that share 128-wide keys, otherwise two) times what a workgroup takes, in units of an item: its items (one in four where the
// waves split them) and five for its beginning and end; and for joining parts four more, or, of rows that share keys, 4 us and what writing and reading them takes, by an
// item's 0.24 us for each 16 rows of a wave and as much for each 64 dimensions.  (52 x 4 row blocks over 46 groups: three parts, 624 workgroups, 74 us; two 51.  32 pairs of 512 rows, 10 groups:
// 128-wide one part 25.5 us, three 33.9; 64-wide 20.1, 29.6.)
// Where every wave takes items of its own, one workgroup of eight waves for all of them is the other way, without the second launch.  Its time in us: an item is 8 KiB of
// 64-wide keys and values, 5.2 TB/s for all and some 100 GB/s for one CU's (tiles of 16 rows: that many times as much); of the two the longer one and a tenth of the other, and
// 5.5 for the launch.  In parts: the first, the waves' own items at 0.5, the launch, and 3 for joining; and never less than the 14.6 that the host takes for two launches (one: 11.6).
// Not if it takes longer than that and the cache is one whose parts go by length (attend()): one sequence alone may be long.
// (64-wide, 64 pairs, 94 groups: one part 14.3 us a call, eight 16.2; 8 pairs, 94 groups 12.4, 14.5; 188 groups 17.5, 14.8.  128-wide, 128 pairs, 31 groups: 15.5, 19.2; 32 pairs, 94 groups:
// 22, 16.5.)
inline int split_of(const TreePlan& p, long pairs, long groups, bool grouped, int cus) {
  const long room = (long)(!grouped ? 4 : (p.rows && p.mt == 1 ? 3 : 2)) * cus, step = p.rows ? 1 : 4;
  long best = 1;
  double least = 0;
  for (long n = 1; n <= 64 && (n == 1 || n * 4 <= groups); ++n) {
    const double join = n == 1 ? 0 : (p.rows ? (4 + 0.0063 * pairs * n * p.mt * p.wide) / (0.24 * (p.mt + p.wide)) : 4);
    const double cost = (double)((pairs * n + room - 1) / room * ((groups + n * step - 1) / (n * step) + 5)) + join;
    if (n == 1 || cost < least) { best = n; least = cost; }
  }
  if (best > 1 && grouped && !p.rows) {
    const double hbm = 0.0016 * p.wide * pairs * groups, cu = 0.08 * p.wide * p.mt * ((pairs + cus - 1) / cus) * groups;
    const double one = 5.5 + (hbm > cu ? hbm + 0.1 * cu : cu + 0.1 * hbm), parts = 5.5 + hbm + 0.5 * ((groups + 4 * best - 1) / (4 * best)) + 3;
    if (one <= 14.6 || (one <= parts && groups < 128)) best = 1;
  }
  return (int)best;
}
// Kernel (rows: the waves share the keys), row tiles of 16 (per wave), row blocks, parts that the keys are split into, and what the workspace holds: partial
// results, then (block > 0) bits of the chosen blocks and their bounds.
inline TreePlan plan_attention(const bpd_cache& c, int B, int T, int heads, int block, int cus) {
  TreePlan p{};
  const int R = T * (heads / c.n_kv_heads);
  const bool grouped = cache_grouped(c);
  p.rows = grouped && R > (c.head_dim == 64 ? 48 : 16);        // (more tiles than that in one wave's registers: spills)
  p.mt = p.rows ? (R > 64 ? 2 : 1) : (grouped ? (R + 15) / 16 : 1);
  p.wide = c.head_dim / 64;
  const int per = p.rows ? 64 * p.mt : (grouped ? 48 : 16);
  p.blocks = (R + per - 1) / per;
  p.nsplit = split_of(p, (long)B * c.n_kv_heads * p.blocks, (c.capacity + 31) / 32, grouped, cus);
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  p.bytes = p.nsplit > 1 ? up((size_t)B * c.n_kv_heads * p.nsplit * R * (c.head_dim + 2) * 4) : 0;
  if (block && c.capacity / block > 0) {
    const size_t nb = c.capacity / block, rows = (size_t)B * c.n_kv_heads * T;
    p.chosen_at = p.bytes; p.bytes += up(rows * ((nb + 31) / 32) * 4);
    p.score_at = p.bytes; p.bytes += up(rows * ((nb + 63) / 64) * 64 * 8);
  }
  return p;
}

}  // namespace
