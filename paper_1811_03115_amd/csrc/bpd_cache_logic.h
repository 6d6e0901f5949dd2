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
inline const char* block_wrong(const bpd_cache&, int block) {
  return block == 32 || block == 64 || block == 128 ? nullptr : "blocks: 32, 64 or 128 rows";
}
inline size_t summaries_elements(const bpd_cache& c, int block) {
  const size_t tiles = ((size_t)c.capacity / block + 63) / 64;
  return (size_t)c.max_batch * c.n_kv_heads * tiles * 2 * c.head_dim * 64;
}

struct TreePlan { bool rows; int mt, blocks, nsplit; size_t chosen_at, score_at, bytes; };
// Parts that `groups` of 32 keys are split into, for as many (sequence, key head, row block)s as there are: the fewest rounds of as many workgroups as the chip has room for (a CU's
// registers: four of fp32 rows, three of 64 rows that share 128-wide keys, otherwise two) times what a workgroup takes, in units of an item: its items (one in four where the
// waves split them) and five for its beginning and end; four more for joining parts.  (52 x 4 row blocks over 46 groups: three parts, 624 workgroups, 74 us; two 51.
// 64 pairs, 95 groups: one part 29 us, four 21, eight 17.)
inline int split_of(const TreePlan& p, long pairs, long groups, bool grouped, int cus) {
  const long room = (long)(!grouped ? 4 : (p.rows && p.mt == 1 ? 3 : 2)) * cus, step = p.rows ? 1 : 4;
  long best = 1, least = 0;
  for (long n = 1; n <= 64 && (n == 1 || n * 4 <= groups); ++n) {
    const long cost = (pairs * n + room - 1) / room * ((groups + n * step - 1) / (n * step) + 5) + (n > 1 ? 4 : 0);
    if (n == 1 || cost < least) { best = n; least = cost; }
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
