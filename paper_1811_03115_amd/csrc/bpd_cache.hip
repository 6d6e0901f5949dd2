// Host side of the cache operators of include/bpd.h: checks of their arguments, sizes, launches.  They take no context: what they need is in
// their arguments, and they run on the current device and the stream that they are given.
#include "../../include/bpd.h"
#include "bpd_cache_ops.h"
#include "bpd_cache_launch.h"
#include "bpd_cache_logic.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <string>

namespace {

thread_local std::string op_error;

int refuse(int code, const char* what) {
  try { op_error = what; } catch (...) {}
  return code;
}
int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return BPD_OK;
  try { op_error = std::string(what) + ": " + hipGetErrorString(e); } catch (...) {}
  return BPD_E_HIP;
}
// Compute units of the current device
int compute_units() {
  static std::atomic<int> known[64];
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 256;
  if (dev >= 0 && dev < 64 && (cus = known[dev].load(std::memory_order_relaxed)) > 0) return cus;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus < 1) return 256;
  if (dev >= 0 && dev < 64) known[dev].store(cus, std::memory_order_relaxed);
  return cus;
}
bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
// Can four elements (of 2 or 4 bytes) of rows be moved at once, eight of bf16?
bool rows_aligned(const bpd_rows& r) {
  const int64_t m = r.dtype == BPD_F32 ? 3 : 7;
  return aligned16(r.data) && ((r.layer | r.seq | r.row | r.head) & m) == 0;
}
const char* rows_wrong(const bpd_rows* r) {
  if (!r || !r->data) return "rows: null";
  if (r->dtype != BPD_F32 && r->dtype != BPD_BF16) return "rows: dtype is BPD_F32 or BPD_BF16";
  if ((uintptr_t)r->data & (r->dtype == BPD_F32 ? 3 : 1)) return "rows: not aligned to an element";
  return nullptr;
}
RowsP rows_of(const bpd_rows& r) { return RowsP{r.data, r.dtype == BPD_F32, rows_aligned(r) ? 1 : 0, (long)r.layer, (long)r.seq, (long)r.row, (long)r.head}; }

template <int D, int MT, int NW, bool SPARSE>
void attend_waves(const TreeP& p, hipStream_t s) {
  const dim3 grid(p.parts, p.kv);
  if constexpr (MT == 1 || (MT == 2 && D == 64)) {      // (more rows of fp32 queries: attend_groups)
    if (p.q_f32) { hipLaunchKernelGGL((tree_attention_kernel<D, MT, NW, true, SPARSE>), grid, dim3(64 * NW), 0, s, p); return; }
  }
  hipLaunchKernelGGL((tree_attention_kernel<D, MT, NW, false, SPARSE>), grid, dim3(64 * NW), 0, s, p);
}
template <int D, int MT, bool SPARSE>
void attend_few(const TreeP& p, hipStream_t s) {
  // Eight waves where one workgroup has all of the keys (split_of()), they are more than four waves' first items, and a CU would have no second workgroup.  (64-wide, 32 rows, 128 pairs, 94 groups
  // 22.6 us a call, four waves 26.1; 1024 pairs, 5 groups: a step of six layers 709 us, 678.)
  if (p.nsplit == 1 && p.cap > 128 && (long)p.parts * p.kv <= compute_units()) attend_waves<D, MT, 8, SPARSE>(p, s); else attend_waves<D, MT, 4, SPARSE>(p, s);
}
template <int D, bool SPARSE>
void attend_groups(const TreeP& p, const TreePlan& plan, hipStream_t s) {
  const int R = p.T * p.G;
  if (plan.rows || (p.q_f32 && R > (D == 64 ? 32 : 16))) {
    if (p.q_f32) hipLaunchKernelGGL((tree_attention_rows_kernel<D, 1, 4, true, SPARSE>), dim3(p.parts * ((R + 63) / 64), p.kv), dim3(256), 0, s, p);
    else if (plan.mt == 1) hipLaunchKernelGGL((tree_attention_rows_kernel<D, 1, 4, false, SPARSE>), dim3(p.parts * plan.blocks, p.kv), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((tree_attention_rows_kernel<D, 2, 4, false, SPARSE>), dim3(p.parts * plan.blocks, p.kv), dim3(256), 0, s, p);
  } else if constexpr (D == 64) {
    if (plan.mt == 1) attend_few<D, 1, SPARSE>(p, s);
    else if (plan.mt == 2) attend_few<D, 2, SPARSE>(p, s);
    else attend_few<D, 3, SPARSE>(p, s);
  } else attend_few<D, 1, SPARSE>(p, s);
}
template <int D>
void join(const TreeP& p, hipStream_t s) {
  const long rows = (long)p.B * p.kv * p.T * p.G;
  // a wave has D / 4 lanes per part: more than eight rounds of that, and few rows, are for four waves
  if (p.nsplit > 8 * 256 / D && rows < 4096) hipLaunchKernelGGL((tree_join_kernel<D, 4>), dim3((unsigned)rows), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((tree_join_kernel<D, 1>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, p);
}
template <bool SPARSE>
void attend(const bpd_cache& c, const TreeP& args, TreePlan plan, hipStream_t s, const BoundP* blocks = nullptr) {
  const int D = c.head_dim;
  TreeP p = args;
  if (SPARSE) {                                  // at most so many groups are seen: fewer parts than the workspace has room for
    const BoundP& bp = *blocks;
    const long most = std::min((long)(c.capacity + 31) / 32, (long)std::min<long>(p.T, 1 + p.T / 4) * ((long)bp.first + bp.recent + bp.top) * p.bg + p.bg + 4);
    plan.nsplit = std::min(plan.nsplit, split_of(plan, (long)p.B * p.kv * plan.blocks, most, cache_grouped(c), compute_units()));
  }
  // (by length: a lane knows one sequence's; its sums cost some 1 us, which short caches do not have; chosen blocks are about as many in every sequence)
  p.nsplit = plan.nsplit; p.parts = p.B * plan.nsplit; p.by_length = !SPARSE && plan.nsplit > 1 && p.B > 1 && p.B <= 64 && c.capacity >= 4096;
  if (cache_grouped(c)) {
    if (D == 64) attend_groups<64, SPARSE>(p, plan, s); else attend_groups<128, SPARSE>(p, plan, s);
  } else {
    const dim3 grid(p.parts * plan.blocks, p.kv);
    if (c.dtype == BPD_BF16) hipLaunchKernelGGL((tree_rows_kernel<bf16_t, 16, SPARSE>), grid, dim3(256), 0, s, p);
    else if (D == 16) hipLaunchKernelGGL((tree_rows_kernel<float, 16, SPARSE>), grid, dim3(256), 0, s, p);
    else if (D == 64) hipLaunchKernelGGL((tree_rows_kernel<float, 64, SPARSE>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((tree_rows_kernel<float, 128, SPARSE>), grid, dim3(256), 0, s, p);
  }
  if (p.parts > p.B) { if (D == 16) join<16>(p, s); else if (D == 64) join<64>(p, s); else join<128>(p, s); }
}

// Bounds of the blocks, with fresh summaries (no nodes: those alone), and the blocks that each node sees
void choose_blocks(const bpd_cache& c, const BoundP& bp, hipStream_t s) {
  const dim3 grid(bp.tiles * (bp.t.T > 16 ? (bp.t.T + 15) / 16 : 1), bp.t.kv, bp.t.B);
  const int D = c.head_dim;
  if (cache_grouped(c)) {
    if (D == 64) hipLaunchKernelGGL((block_bounds_kernel<bf16_t, 64, true>), grid, dim3(256), 0, s, bp);
    else hipLaunchKernelGGL((block_bounds_kernel<bf16_t, 128, true>), grid, dim3(256), 0, s, bp);
  } else if (c.dtype == BPD_BF16) hipLaunchKernelGGL((block_bounds_kernel<bf16_t, 16, false>), grid, dim3(256), 0, s, bp);
  else if (D == 16) hipLaunchKernelGGL((block_bounds_kernel<float, 16, false>), grid, dim3(256), 0, s, bp);
  else if (D == 64) hipLaunchKernelGGL((block_bounds_kernel<float, 64, false>), grid, dim3(256), 0, s, bp);
  else hipLaunchKernelGGL((block_bounds_kernel<float, 128, false>), grid, dim3(256), 0, s, bp);
  if (bp.t.T == 0) return;
  const dim3 nodes(bp.t.T, bp.t.kv, bp.t.B);
  if (bp.tiles <= 2) hipLaunchKernelGGL((block_pick_kernel<128, 1>), nodes, dim3(128), 0, s, bp);
  else if (bp.tiles <= 8) hipLaunchKernelGGL((block_pick_kernel<512, 1>), nodes, dim3(512), 0, s, bp);
  else hipLaunchKernelGGL((block_pick_kernel<512, TREE_BLOCKS_MAX / 512>), nodes, dim3(512), 0, s, bp);
}
// What the blocks of a call are, and where their bounds and bits go
BoundP bound_args(TreeP& p, const bpd_cache& c, const bpd_blocks& blocks, unsigned* chosen, double* score) {
  BoundP bp{};
  const int nb = c.capacity / blocks.block;
  p.words = (nb + 31) / 32; p.bg = blocks.block / 32; p.chosen = chosen;
  bp.t = p;
  bp.summaries = blocks.summaries; bp.tiles = (nb + 63) / 64;
  bp.block = blocks.block; bp.first = blocks.first; bp.recent = blocks.recent; bp.top = blocks.top;
  bp.added = blocks.added; bp.added_all = -1; bp.score = score; bp.chosen = chosen;
  return bp;
}

constexpr float LOG2_E = 1.44269504088896340736f;
// What bpd_tree_attention and bpd_sparse_attention check alike; null: nothing is wrong
const char* attention_wrong(const bpd_cache* c, const bpd_rows* q, const bpd_rows* out, const int32_t* length, int B, int T, int heads, float scale) {
  if (const char* w = cache_wrong(c)) return w;
  if (const char* w = attention_sizes_wrong(*c, B, T, heads)) return w;
  if (!std::isfinite(scale * LOG2_E)) return "attention: scale is not finite, or not times log2(e)";
  if (B == 0 || T == 0) return nullptr;          // (nothing is read)
  if (const char* w = rows_wrong(q)) return w;
  if (const char* w = rows_wrong(out)) return w;
  return length ? nullptr : "attention: null length";
}
TreeP attention_args(const bpd_cache& c, const bpd_rows& q, const bpd_rows& out, const int32_t* length, const int32_t* parent, int B, int T, int heads, float scale) {
  TreeP p{};
  p.q = q.data; p.q_seq = (long)q.seq; p.q_row = (long)q.row; p.q_head = (long)q.head;
  p.out = const_cast<void*>(out.data); p.o_seq = (long)out.seq; p.o_row = (long)out.row; p.o_head = (long)out.head;
  p.K = c.k; p.V = c.v;
  p.B = B; p.T = T; p.H = heads; p.kv = c.n_kv_heads; p.G = heads / c.n_kv_heads; p.cap = c.capacity;
  p.length = length; p.parent = parent;
  p.scale = scale == 0.f ? 1.f : fabsf(scale) * LOG2_E;
  p.sign = scale > 0.f ? 1.f : (scale < 0.f ? -1.f : 0.f);
  p.q_f32 = q.dtype == BPD_F32; p.o_f32 = out.dtype == BPD_F32;
  p.vec = rows_aligned(q) && rows_aligned(out);
  return p;
}

}  // namespace

void launch_block_attention(const BlockAttention& a, hipStream_t stream) {
  const bpd_cache& c = a.cache;
  const int dh = c.head_dim, d = a.heads * dh, block = a.blocks ? a.blocks->block : 0;
  const bpd_rows q{a.q, BPD_F32, 0, (int64_t)a.T * d, d, dh}, out{a.out, c.dtype, 0, (int64_t)a.T * d, d, dh};
  TreeP p = attention_args(c, q, out, a.length, nullptr, a.B, a.T, a.heads, a.scale);
  p.seq = a.seq; p.tree = a.tree; p.packed = a.packed ? d : 0;
  TreePlan plan = plan_attention(c, a.B, a.T, a.heads, block, a.cus);
  p.part = (float*)a.scratch;
  const size_t one = (size_t)a.B * c.n_kv_heads * a.T * (dh + 2) * 4;           // bytes of one part of the keys
  if (!block && plan.nsplit > 1 && plan.nsplit * one > a.scratch_bytes) plan.nsplit = (int)(a.scratch_bytes / one) > 1 ? (int)(a.scratch_bytes / one) : 1;
  if (!block || c.capacity < block) { attend<false>(c, p, plan, stream); return; }
  BoundP bp = bound_args(p, c, *a.blocks, (unsigned*)((char*)a.scratch + plan.chosen_at), (double*)((char*)a.scratch + plan.score_at));
  bp.added_all = a.added;
  choose_blocks(c, bp, stream);
  attend<true>(c, p, plan, stream, &bp);
}
void launch_summaries(const bpd_cache& c, const int* length, int B, int block, void* summaries, hipStream_t stream) {
  if (c.capacity < block) return;
  const bpd_rows none{};
  TreeP p = attention_args(c, none, none, length, nullptr, B, 0, c.n_kv_heads, 1.f);
  const bpd_blocks blocks{block, 0, 0, 0, summaries, nullptr, nullptr};
  choose_blocks(c, bound_args(p, c, blocks, nullptr, nullptr), stream);
}
void launch_tree_move(const bpd_cache& c, const int* path, int ld, const int* accepted, const int* length, int B, hipStream_t s) {
  const MoveP p{path, accepted, length, ld, c.k, c.v, (long)cache_layer_elements(c), c.n_kv_heads, c.capacity};
  const dim3 grid(c.n_kv_heads, c.n_layers, B);
  // (the decoder's heads have 64 dimensions, or 16)
  if (cache_grouped(c)) hipLaunchKernelGGL((tree_move_kernel<bf16_t, 64, true>), grid, dim3(256), 0, s, p);
  else if (c.dtype == BPD_BF16) hipLaunchKernelGGL((tree_move_kernel<bf16_t, 16, false>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((tree_move_kernel<float, 16, false>), grid, dim3(256), 0, s, p);
}

extern "C" {

const char* bpd_op_error(void) { return op_error.c_str(); }

size_t bpd_cache_bytes(const bpd_cache* c) {
  if (cache_sizes_wrong(c)) return 0;
  return cache_layer_elements(*c) * c->n_layers * cache_element(*c);
}

size_t bpd_summaries_bytes(const bpd_cache* c, int block) {
  if (cache_sizes_wrong(c) || block_wrong(*c, block) || c->capacity / block > BPD_BLOCKS_MAX) return 0;
  return summaries_elements(*c, block) * cache_element(*c);
}

size_t bpd_attention_workspace_bytes(const bpd_cache* c, int B, int T, int heads, int block) {
  if (cache_sizes_wrong(c) || B < 1 || attention_sizes_wrong(*c, B, T, heads) || T < 1) return 0;
  if (block && (block_wrong(*c, block) || c->capacity / block > BPD_BLOCKS_MAX)) return 0;
  return plan_attention(*c, B, T, heads, block, compute_units()).bytes;
}

int bpd_cache_store(const bpd_cache* c, const bpd_rows* k, const bpd_rows* v, const int32_t* start, const int32_t* count, int B, int T, void* hip_stream) {
  if (const char* w = cache_wrong(c)) return refuse(BPD_E_ARG, w);
  if (B < 0 || B > c->max_batch || T < 0) return refuse(BPD_E_ARG, "bpd_cache_store: B outside 0..max_batch, or T < 0");
  if (T > c->capacity) return refuse(BPD_E_CAPACITY, "bpd_cache_store: more rows than the cache has");
  if ((int64_t)B * c->n_layers > 65535) return refuse(BPD_E_CAPACITY, "bpd_cache_store: more than 65535 sequences times layers");
  if (B == 0 || T == 0) return BPD_OK;
  if (const char* w = rows_wrong(k)) return refuse(BPD_E_ARG, w);
  if (const char* w = rows_wrong(v)) return refuse(BPD_E_ARG, w);
  if (!start) return refuse(BPD_E_ARG, "bpd_cache_store: null start");
  StoreP p{rows_of(*k), rows_of(*v), c->k, c->v, (long)cache_layer_elements(*c), B, T, c->n_kv_heads, c->capacity, start, count};
  const hipStream_t s = (hipStream_t)hip_stream;
  if (cache_grouped(*c)) {
    const dim3 grid((T + 30) / 32 + 1, c->n_kv_heads, B * c->n_layers);
    if (c->head_dim == 64) hipLaunchKernelGGL(store_groups_kernel<64>, grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(store_groups_kernel<128>, grid, dim3(256), 0, s, p);
  } else {
    const dim3 grid(std::min(T, 1 << 16), 1, B * c->n_layers);           // (2^24 rows would be 2^32 threads, one more than a launch has)
    if (c->dtype == BPD_F32) hipLaunchKernelGGL(store_rows_kernel<float>, grid, dim3(256), 0, s, p, c->head_dim);
    else hipLaunchKernelGGL(store_rows_kernel<bf16_t>, grid, dim3(256), 0, s, p, c->head_dim);
  }
  return launched("bpd_cache_store");
}

int bpd_tree_attention(const bpd_cache* c, const bpd_rows* q, const bpd_rows* out, const int32_t* length, const int32_t* parent, int B, int T, int heads,
                       float scale, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (const char* w = attention_wrong(c, q, out, length, B, T, heads, scale)) return refuse(BPD_E_ARG, w);
  if (B == 0 || T == 0) return BPD_OK;
  const TreePlan plan = plan_attention(*c, B, T, heads, 0, compute_units());
  if (plan.bytes > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < plan.bytes)) return refuse(BPD_E_CAPACITY, "bpd_tree_attention: workspace too small or not aligned to 16 bytes");
  TreeP p = attention_args(*c, *q, *out, length, parent, B, T, heads, scale);
  p.part = (float*)workspace;
  attend<false>(*c, p, plan, (hipStream_t)hip_stream);
  return launched("bpd_tree_attention");
}

int bpd_sparse_attention(const bpd_cache* c, const bpd_rows* q, const bpd_rows* out, const int32_t* length, const int32_t* parent, int B, int T, int heads,
                         float scale, const bpd_blocks* blocks, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (const char* w = attention_wrong(c, q, out, length, B, T, heads, scale)) return refuse(BPD_E_ARG, w);
  if (!blocks) return refuse(BPD_E_ARG, "bpd_sparse_attention: null blocks");
  if (const char* w = block_wrong(*c, blocks->block)) return refuse(BPD_E_ARG, w);
  if (blocks->first < 0 || blocks->recent < 0 || blocks->top < 0) return refuse(BPD_E_ARG, "bpd_sparse_attention: first, recent and top are not negative");
  const int nb = c->capacity / blocks->block;
  if (nb > BPD_BLOCKS_MAX) return refuse(BPD_E_CAPACITY, "bpd_sparse_attention: more than BPD_BLOCKS_MAX blocks");
  if (nb > 0 && (!blocks->summaries || !aligned16(blocks->summaries))) return refuse(BPD_E_ARG, "bpd_sparse_attention: summaries null or not aligned to 16 bytes");
  if (B == 0 || T == 0) return BPD_OK;
  const TreePlan plan = plan_attention(*c, B, T, heads, blocks->block, compute_units());
  if (plan.bytes > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < plan.bytes)) return refuse(BPD_E_CAPACITY, "bpd_sparse_attention: workspace too small or not aligned to 16 bytes");
  const hipStream_t s = (hipStream_t)hip_stream;
  TreeP p = attention_args(*c, *q, *out, length, parent, B, T, heads, scale);
  p.part = (float*)workspace;
  if (nb == 0) {                                 // nothing to choose from
    attend<false>(*c, p, plan, s);
    return launched("bpd_sparse_attention");
  }
  unsigned* chosen = blocks->chosen ? blocks->chosen : (unsigned*)((char*)workspace + plan.chosen_at);
  const BoundP bp = bound_args(p, *c, *blocks, chosen, (double*)((char*)workspace + plan.score_at));
  choose_blocks(*c, bp, s);
  attend<true>(*c, p, plan, s, &bp);
  return launched("bpd_sparse_attention");
}

int bpd_tree_accept(const int32_t* parent, const int32_t* token, const int32_t* expect, const int32_t* best, const int32_t* length, const int32_t* room, int eos_id,
                    int B, int T, int32_t* path, int32_t* accepted, int32_t* next, int32_t* new_length, const bpd_cache* c, void* hip_stream) {
  if (B < 0 || B > 65535 || T < 0 || T > BPD_TREE_MAX) return refuse(BPD_E_ARG, "bpd_tree_accept: B outside 0..65535, or T outside 0..BPD_TREE_MAX");
  if (c) {
    if (const char* w = cache_wrong(c)) return refuse(BPD_E_ARG, w);
    if (B > c->max_batch) return refuse(BPD_E_ARG, "bpd_tree_accept: B over max_batch");
    if (c->n_layers > 65535) return refuse(BPD_E_CAPACITY, "bpd_tree_accept: more than 65535 layers");
  }
  if (B == 0) return BPD_OK;
  if (!expect || !length || !accepted || !next || !new_length || (T > 0 && (!parent || !token || !best || !path))) return refuse(BPD_E_ARG, "bpd_tree_accept: null argument");
  // (every workgroup reads the inputs, one writes the results)
  struct Ints { const void* p; size_t n; };
  const Ints in[] = {{parent, (size_t)B * T}, {token, (size_t)B * T}, {best, (size_t)B * T}, {expect, (size_t)B}, {length, (size_t)B}, {room, room ? (size_t)B : 0}};
  const Ints res[] = {{path, (size_t)B * T}, {accepted, (size_t)B}, {next, (size_t)B}, {new_length, (size_t)B}};
  auto meet = [](const Ints& a, const Ints& b) { return a.n && b.n && (const char*)a.p < (const char*)b.p + 4 * b.n && (const char*)b.p < (const char*)a.p + 4 * a.n; };
  for (const Ints& r : res) {
    for (const Ints& i : in) if (meet(r, i)) return refuse(BPD_E_ARG, "bpd_tree_accept: results overlap what is read");
    for (const Ints* o = res; o < &r; ++o) if (meet(r, *o)) return refuse(BPD_E_ARG, "bpd_tree_accept: results overlap each other");
  }
  AcceptP p{parent, token, expect, best, length, room, path, accepted, next, new_length, eos_id, T, B, nullptr, nullptr, 0, 1, 0};
  const hipStream_t s = (hipStream_t)hip_stream;
  dim3 grid(1, 1, B);
  int D = 64;
  bool f32 = false, grouped = true;
  if (c) {
    p.K = c->k; p.V = c->v; p.layer = (long)cache_layer_elements(*c); p.kv = c->n_kv_heads; p.cap = c->capacity;
    grid = dim3(c->n_kv_heads, c->n_layers, B);
    D = c->head_dim; f32 = c->dtype == BPD_F32; grouped = cache_grouped(*c);
  }
  if (grouped) {
    if (D == 64) hipLaunchKernelGGL((tree_accept_kernel<bf16_t, 64, true>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((tree_accept_kernel<bf16_t, 128, true>), grid, dim3(256), 0, s, p);
  } else if (!f32) hipLaunchKernelGGL((tree_accept_kernel<bf16_t, 16, false>), grid, dim3(256), 0, s, p);
  else if (D == 16) hipLaunchKernelGGL((tree_accept_kernel<float, 16, false>), grid, dim3(256), 0, s, p);
  else if (D == 64) hipLaunchKernelGGL((tree_accept_kernel<float, 64, false>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((tree_accept_kernel<float, 128, false>), grid, dim3(256), 0, s, p);
  return launched("bpd_tree_accept");
}

}  // extern "C"
