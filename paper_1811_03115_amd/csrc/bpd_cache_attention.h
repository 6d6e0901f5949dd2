// Attention of a block of drafted tokens that form a tree, over a cache of keys and values, whole or by chosen blocks.
//
// Sequence b has len committed rows in the cache, and behind them the T rows of its drafts: node i at row len + i.  Node i's
// ancestors are  anc(i) = {i} + anc(parent_i),  parent -1 standing for the prefix itself.  Its query sees the prefix (all of it, or
// chosen blocks and what is behind the last complete one) and the rows of anc(i):
//     out[i] = sum_j p_j V_j,   p = softmax_j(scale q_i . K_j)
// in one pass over the keys with a running maximum and sum per row (fp32, base 2).  Query heads that share a key head are rows of
// the same product: row r of a (sequence, key head) pair is node r / G, head r % G of the group's G.
//
// A node is absent if its parent is neither -1 nor an earlier node, if its row is past the cache's end, or if an ancestor is absent; a
// sequence of negative length has none.  Absent nodes are seen by nobody and their results are zero.
#pragma once
#include "bpd_device.h"

constexpr int TREE_MAX = 64;                     // nodes of a tree: one wave, one 64-bit word of ancestors
constexpr int TREE_GROUP = 32;                   // keys per group of a cache in operand order

struct TreeP {
  const void* q; long q_seq, q_row, q_head;      // elements from sequence to sequence, row to row, head to head; bf16 or fp32
  void* out; long o_seq, o_row, o_head;
  const void *K, *V;                             // one layer's cache
  int B, T, H, kv, G, cap;                       // cap: rows per sequence
  const int* length; const int* parent;          // parent null: a chain
  float scale;                                   // times log2(e)
  int nsplit; float* part;                       // partial results [b][kv head][row block][split][rows x (D + 2)]
  int q_f32, o_f32, vec;                         // vec: rows of q and out are 16-byte aligned
  // chosen blocks (null: the whole prefix): bits [b][kv head][node][words], blocks of `bg` groups of 32 keys
  const unsigned* chosen; int words, bg;
};

typedef unsigned long long mask64;

// Ancestors of node `lane` (bits), and whether it is there, by all 64 lanes of a wave: after round n a node knows 2^n of its ancestors.
__device__ __forceinline__ void tree_ancestors(const int* parent, int T, int there, int lane, mask64& anc, bool& ok) {
  if (!parent) {                                 // a chain
    ok = lane < there;
    anc = ok ? (~0ull >> (63 - lane)) : 0ull;
    return;
  }
  int p = lane < T ? parent[lane] : -2;
  int good = lane < there && p >= -1 && p < lane;
  if (!good) p = -1;
  unsigned lo = lane < 32 ? 1u << lane : 0u, hi = lane < 32 ? 0u : 1u << (lane - 32);
#pragma unroll
  for (int n = 0; n < 6; ++n) {
    const int from = p < 0 ? lane : p;           // (its own: nothing new)
    lo |= (unsigned)__shfl((int)lo, from, 64);
    hi |= (unsigned)__shfl((int)hi, from, 64);
    good &= __shfl(good, from, 64);
    const int up = __shfl(p, from, 64);
    p = p < 0 ? -1 : up;
  }
  ok = good;
  anc = good ? ((mask64)hi << 32 | lo) : 0ull;
}

// Rows committed and drafted that the cache holds
__device__ __forceinline__ void tree_extent(const TreeP& p, int b, int& len, int& there) {
  len = p.length[b];
  there = len < 0 ? 0 : (len >= p.cap ? 0 : (p.T < p.cap - len ? p.T : p.cap - len));
  len = len < 0 ? 0 : (len > p.cap ? p.cap : len);
}

// Four results of a row
__device__ __forceinline__ void tree_store4(const TreeP& p, int b, int node, int h, int c, const f32x4& v) {
  const long at = (long)b * p.o_seq + (long)node * p.o_row + (long)h * p.o_head + c;
  if (p.o_f32) {
    float* o = (float*)p.out + at;
    if (p.vec) *(f32x4*)o = v; else { o[0] = v[0]; o[1] = v[1]; o[2] = v[2]; o[3] = v[3]; }
  } else {
    bf16_t* o = (bf16_t*)p.out + at;
    const u32x2 w = u32x2{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
    if (p.vec) *(u32x2*)o = w;
    else { o[0] = (bf16_t)w[0]; o[1] = (bf16_t)(w[0] >> 16); o[2] = (bf16_t)w[1]; o[3] = (bf16_t)(w[1] >> 16); }
  }
}
// Eight elements of a query (c % 8 == 0) in fp32
__device__ __forceinline__ void tree_q8(const TreeP& p, int b, int node, int h, int c, float (&v)[8]) {
  const long at = (long)b * p.q_seq + (long)node * p.q_row + (long)h * p.q_head + c;
  if (p.q_f32) {
    const float* q = (const float*)p.q + at;
    if (p.vec) {
      const f32x4 x = *(const f32x4*)q, y = *(const f32x4*)(q + 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) { v[j] = x[j]; v[4 + j] = y[j]; }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = q[j];
    }
  } else {
    const bf16_t* q = (const bf16_t*)p.q + at;
    u32x4 w;
    if (p.vec) w = *(const u32x4*)q;
    else {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = (unsigned)q[2 * j] | (unsigned)q[2 * j + 1] << 16;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) { v[2 * j] = __uint_as_float(w[j] << 16); v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u); }
  }
}
// fp32 operands as a bf16 pair hi + lo, which keeps them to 2^-17
__device__ __forceinline__ void tree_pair(const float (&v)[8], bf16x8& hi, bf16x8& lo) {
  unsigned h[4], l[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    h[j] = cvt_pk_bf16(v[2 * j], v[2 * j + 1]);
    l[j] = cvt_pk_bf16(v[2 * j] - __uint_as_float(h[j] << 16), v[2 * j + 1] - __uint_as_float(h[j] & 0xFFFF0000u));
  }
  hi = __builtin_bit_cast(bf16x8, (u32x4{h[0], h[1], h[2], h[3]}));
  lo = __builtin_bit_cast(bf16x8, (u32x4{l[0], l[1], l[2], l[3]}));
}

// The keys that a workgroup walks, as items of one group of 32: the chosen blocks' groups, then those behind the last complete block.
// Dense: every group of 0 .. ngr - 1.
struct TreeItems {
  int listed, tail0, n;                          // items that come from the list, first group of the rest, items in all
  const unsigned short* list; int bg;
  __device__ __forceinline__ int group(int i) const {
    if (!list) return i;
    if (i >= listed) return tail0 + i - listed;
    const int at = i / bg;
    return list[at] * bg + i - at * bg;
  }
};
constexpr int TREE_BLOCKS_MAX = 4096;            // blocks of rows that can be chosen from
// List of the blocks that any node n0 .. n1 - 1 has chosen, in order; bits: [TREE_BLOCKS_MAX / 32] words of scratch.  All threads; blocks of threads >= words.
__device__ __forceinline__ int tree_list(const unsigned* chosen, int words, int n0, int n1, int done, unsigned short* list, int* sums) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  unsigned bits = 0;
  if (tid < words) {
    for (int n = n0; n < n1; ++n) bits |= chosen[(long)n * words + tid];
    const int left = done - 32 * tid;            // (bits past the last complete block: none are set)
    if (left < 32) bits = left <= 0 ? 0u : bits & ((1u << left) - 1u);
  }
  const int cnt = __popc(bits);
  int upto = cnt;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) { const int v = __shfl_up(upto, o, 64); if (lane >= o) upto += v; }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int base = 0, all = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) { if (w < wave) base += sums[w]; all += sums[w]; }
  int at = base + upto - cnt;
  while (bits) { const int j = __ffs(bits) - 1; bits &= bits - 1; list[at++] = (unsigned short)(32 * tid + j); }
  __syncthreads();
  return all;
}

// bf16 heads of D = 64 or 128 in operand order (groups of 32 keys, D x 32 elements of K and as many of V, bpd_attention.h for D = 64; the same with
// D / 32 steps of K and D / 16 tiles of V otherwise): every operand is one 1 KiB load, nothing of K and V goes through LDS.
// A workgroup has 16 MT rows of one (sequence, key head) and every nsplit-th part of its items; its four waves split those by single items, each with its own
// maximum, sum and results, and meet once in LDS.
//   scores^T = K Q^T       32 keys x 16 rows per item and row tile
//   softmax                in the lane, then across the four lanes of a row
//   out^T += V^T P^T       the probabilities as they lie are the second operand
// Queries of bf16 are exact, those of fp32 a pair; the scale is applied to the fp32 scores.  Probabilities go in as a pair hi + lo: as single bf16 numbers their rounding
// adds as much error as that of the bf16 results (sum over keys of p (1 +- 2^-9) v), which the pair's second product takes to 2^-17.
template <int D, int MT, bool QF32, bool SPARSE>
__global__ __launch_bounds__(256) void tree_attention_kernel(TreeP p) {
  constexpr int KS = D / 32, VT = D / 16, GRP = TREE_GROUP * D;
  __shared__ __attribute__((aligned(16))) f32x4 o_s[4][VT][64];
  __shared__ float m_s[4][MT * 16], l_s[4][MT * 16];
  __shared__ unsigned short list_s[SPARSE ? TREE_BLOCKS_MAX : 1];
  __shared__ int sums_s[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lq = lane >> 4;
  const int split = blockIdx.x % p.nsplit, hk = blockIdx.x / p.nsplit, rb = blockIdx.y, b = blockIdx.z;
  const int R = p.T * p.G, r0 = rb * 16 * MT;
  int len, there;
  tree_extent(p, b, len, there);
  const int* parent = p.parent ? p.parent + (long)b * p.T : nullptr;
  mask64 anc; bool ok;
  tree_ancestors(parent, p.T, there, lane, anc, ok);
  const mask64 present = __ballot(ok);
  // this lane's rows
  mask64 seen[MT]; int node[MT]; bool row_ok[MT];
  bf16x8 qh[MT][KS], ql[QF32 ? MT : 1][KS];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int r = r0 + 16 * t + lr, n = r < R ? r / p.G : 0;
    node[t] = n;
    seen[t] = (mask64)(unsigned)__shfl((int)(anc >> 32), n, 64) << 32 | (unsigned)__shfl((int)anc, n, 64);
    row_ok[t] = r < R && seen[t] != 0;
    if (r >= R) seen[t] = 0;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      float v[8] = {};
      if (row_ok[t]) tree_q8(p, b, n, hk * p.G + r - n * p.G, 32 * s + 8 * lq, v);
      bf16x8 lo;
      tree_pair(v, qh[t][s], lo);
      if constexpr (QF32) ql[t][s] = lo;
    }
  }
  const int ngr = (len + there + 31) >> 5;
  TreeItems it{0, 0, ngr, nullptr, 1};
  const unsigned* picks = nullptr;
  if constexpr (SPARSE) {
    picks = p.chosen + ((long)b * p.kv + hk) * p.T * p.words;
    const int done = len / (32 * p.bg), n0 = r0 / p.G, n1 = min(p.T, (min(R, r0 + 16 * MT) + p.G - 1) / p.G);
    it.list = list_s; it.bg = p.bg; it.tail0 = done * p.bg;
    it.listed = tree_list(picks, p.words, n0, n1, done, list_s, sums_s) * p.bg;
    it.n = it.listed + ngr - it.tail0;
  }
  const int i0 = (int)((long)it.n * split / p.nsplit), i1 = (int)((long)it.n * (split + 1) / p.nsplit);
  const bf16_t* Kb = (const bf16_t*)p.K + ((size_t)b * p.kv + hk) * p.cap * D;
  const bf16_t* Vb = (const bf16_t*)p.V + ((size_t)b * p.kv + hk) * p.cap * D;
  float m_run[MT], l_run[MT];
  f32x4 acc[MT][VT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    m_run[t] = -INFINITY; l_run[t] = 0.f;
#pragma unroll
    for (int x = 0; x < VT; ++x) acc[t][x] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  for (int i = i0 + wave; i < i1; i += 4) {
    const int g = __builtin_amdgcn_readfirstlane(it.group(i));
    const u32x4* kp = (const u32x4*)(Kb + (size_t)g * GRP) + lane;
    const u32x4* vp = (const u32x4*)(Vb + (size_t)g * GRP) + lane;
    u32x4 kf[2 * KS], vf[VT];
#pragma unroll
    for (int x = 0; x < 2 * KS; ++x) kf[x] = kp[x * 64];
#pragma unroll
    for (int x = 0; x < VT; ++x) vf[x] = vp[x * 64];
    const int at = 32 * g + 8 * lq - len;        // this lane's first key among the drafts
    const bool edge = 32 * g + 32 > len;         // (the same for the whole wave)
    if (edge) {                                  // values of rows that nobody sees: their probabilities are zero, their bits unknown
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        unsigned known = 0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int n = at + 2 * w + e;
          if (n < 0 || (n < 64 && (present >> n & 1))) known |= 0xFFFFu << (16 * e);
        }
#pragma unroll
        for (int x = 0; x < VT; ++x) vf[x][w] &= known;
      }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      bool vis = row_ok[t];
      if constexpr (SPARSE) {
        if (i < it.listed) { const int blk = g / p.bg; vis = vis && (picks[(long)node[t] * p.words + (blk >> 5)] >> (blk & 31) & 1); }
      }
      f32x4 s[2];
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x4 a = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < KS; ++x) {
          const bf16x8 ka = __builtin_bit_cast(bf16x8, kf[u * KS + x]);
          a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qh[t][x], a, 0, 0, 0);
          if constexpr (QF32) a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, ql[t][x], a, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int n = at + 4 * u + r;
          const bool in = !edge || n < 0 ? vis : (n < 64 && (seen[t] >> n & 1));
          a[r] = in ? a[r] * p.scale : -INFINITY;
          mx = fmaxf(mx, a[r]);
        }
        s[u] = a;
      }
      mx = max_rows(mx);
      const float m_new = fmaxf(m_run[t], mx), m_use = m_new == -INFINITY ? 0.f : m_new;
      float sum = 0.f, pv[8];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) { const float e = __builtin_amdgcn_exp2f(s[u][r] - m_use); pv[4 * u + r] = e; sum += e; }
      sum = sum_rows(sum);
      const float alpha = __builtin_amdgcn_exp2f(m_run[t] - m_use);
      l_run[t] = l_run[t] * alpha + sum;
      m_run[t] = m_new;
#pragma unroll
      for (int x = 0; x < VT; ++x) acc[t][x] *= alpha;
      bf16x8 ph, pl;
      tree_pair(pv, ph, pl);
#pragma unroll
      for (int x = 0; x < VT; ++x) {
        const bf16x8 va = __builtin_bit_cast(bf16x8, vf[x]);
        acc[t][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, ph, acc[t][x], 0, 0, 0);
        acc[t][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pl, acc[t][x], 0, 0, 0);
      }
    }
  }
  // the waves meet
#pragma unroll
  for (int t = 0; t < MT; ++t)
    if (lq == 0) { m_s[wave][16 * t + lr] = m_run[t]; l_s[wave][16 * t + lr] = l_run[t]; }
  const long tile0 = (((long)b * p.kv + hk) * gridDim.y + rb) * p.nsplit + split;
  float* part = p.part + tile0 * (16 * MT) * (D + 2);
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    if (t > 0) __syncthreads();
#pragma unroll
    for (int x = 0; x < VT; ++x) o_s[wave][x][lane] = acc[t][x];
    __syncthreads();
    for (int x = wave; x < VT; x += 4) {
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) M = fmaxf(M, m_s[w][16 * t + lr]);
      f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
      const float M0 = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float a = __builtin_amdgcn_exp2f(m_s[w][16 * t + lr] - M0);
        L = fmaf(l_s[w][16 * t + lr], a, L);
        o += o_s[w][x][lane] * a;
      }
      const int r = r0 + 16 * t + lr;
      if (p.nsplit > 1) {
        *(f32x4*)(part + (16 * t + lr) * D + 16 * x + 4 * lq) = o;
        if (x == wave && wave == 0 && lq == 0) { part[16 * MT * D + 16 * t + lr] = M; part[16 * MT * (D + 1) + 16 * t + lr] = L; }
      } else if (r < R) {
        const float inv = 1.f / L;
        tree_store4(p, b, node[t], hk * p.G + r - node[t] * p.G, 16 * x + 4 * lq, row_ok[t] && L > 0.f ? o * inv : (row_ok[t] && L != L ? f32x4{L, L, L, L} : f32x4{0.f, 0.f, 0.f, 0.f}));
      }
    }
  }
}

// fp32 caches, and bf16 ones of 16-wide heads, whose rows lie as they are ([rows][kv heads][D]): the same walk in fp32 on
// v_mfma_f32_16x16x4_f32 (keys in tiles of 16).  One element per lane and operand: K's dimensions go in by fours as they lie, of V a lane takes the
// dimension of its own from each of its four keys, and nothing is transposed.
template <typename S, int D, bool SPARSE>
__global__ __launch_bounds__(256) void tree_rows_kernel(TreeP p) {
  constexpr int VT = D / 16;
  __shared__ __attribute__((aligned(16))) f32x4 o_s[4][VT][64];
  __shared__ float m_s[4][16], l_s[4][16];
  __shared__ unsigned short list_s[SPARSE ? TREE_BLOCKS_MAX : 1];
  __shared__ int sums_s[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lq = lane >> 4;
  const int split = blockIdx.x % p.nsplit, hk = blockIdx.x / p.nsplit, rb = blockIdx.y, b = blockIdx.z;
  const int R = p.T * p.G, r0 = rb * 16;
  int len, there;
  tree_extent(p, b, len, there);
  const int* parent = p.parent ? p.parent + (long)b * p.T : nullptr;
  mask64 anc; bool ok;
  tree_ancestors(parent, p.T, there, lane, anc, ok);
  const mask64 present = __ballot(ok);
  const int row = r0 + lr, node = row < R ? row / p.G : 0;
  mask64 seen = (mask64)(unsigned)__shfl((int)(anc >> 32), node, 64) << 32 | (unsigned)__shfl((int)anc, node, 64);
  const bool row_ok = row < R && seen != 0;
  if (row >= R) seen = 0;
  float q[VT][4];                                // dimensions 16 x + 4 lq + j
#pragma unroll
  for (int x = 0; x < VT; ++x)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const long at = (long)b * p.q_seq + (long)node * p.q_row + (long)(hk * p.G + row - node * p.G) * p.q_head + 16 * x + 4 * lq + j;
      q[x][j] = !row_ok ? 0.f : (p.q_f32 ? ((const float*)p.q)[at] : bf2f(((const bf16_t*)p.q)[at]));
    }
  const int ngr = (len + there + 31) >> 5;
  TreeItems it{0, 0, ngr, nullptr, 1};
  const unsigned* picks = nullptr;
  if constexpr (SPARSE) {
    picks = p.chosen + ((long)b * p.kv + hk) * p.T * p.words;
    const int done = len / (32 * p.bg), n0 = r0 / p.G, n1 = min(p.T, (min(R, r0 + 16) + p.G - 1) / p.G);
    it.list = list_s; it.bg = p.bg; it.tail0 = done * p.bg;
    it.listed = tree_list(picks, p.words, n0, n1, done, list_s, sums_s) * p.bg;
    it.n = it.listed + ngr - it.tail0;
  }
  const int i0 = (int)((long)it.n * split / p.nsplit), i1 = (int)((long)it.n * (split + 1) / p.nsplit);
  const long stride = (long)p.kv * D;
  const S* Kb = (const S*)p.K + (long)b * p.cap * stride + hk * D;
  const S* Vb = (const S*)p.V + (long)b * p.cap * stride + hk * D;
  float m_run = -INFINITY, l_run = 0.f;
  f32x4 acc[VT];
#pragma unroll
  for (int x = 0; x < VT; ++x) acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int i = i0 + wave; i < i1; i += 4) {
    const int g = __builtin_amdgcn_readfirstlane(it.group(i));
    bool vis = row_ok;
    if constexpr (SPARSE) {
      if (i < it.listed) { const int blk = g / p.bg; vis = vis && (picks[(long)node * p.words + (blk >> 5)] >> (blk & 31) & 1); }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int k0 = 32 * g + 16 * u, end = len + there;
      if (k0 >= end) break;                      // (the same for the whole wave)
      const int key = min(k0 + lr, end - 1);     // K: this lane's key; past the last one nothing is read
      f32x4 a = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < VT; ++x) {
        const S* kp = Kb + key * stride + 16 * x + 4 * lq;
        float kv[4];
        if constexpr (sizeof(S) == 4) { const f32x4 w = *(const f32x4*)kp; kv[0] = w[0]; kv[1] = w[1]; kv[2] = w[2]; kv[3] = w[3]; }
        else { const u32x2 w = *(const u32x2*)kp; kv[0] = __uint_as_float(w[0] << 16); kv[1] = __uint_as_float(w[0] & 0xFFFF0000u); kv[2] = __uint_as_float(w[1] << 16); kv[3] = __uint_as_float(w[1] & 0xFFFF0000u); }
#pragma unroll
        for (int j = 0; j < 4; ++j) a = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[j], q[x][j], a, 0, 0, 0);
      }
      float vv[VT][4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int kk = k0 + 4 * lq + r, n = kk - len;
        const bool known = kk < len || (n < 64 && kk < end && (present >> n & 1));
#pragma unroll
        for (int x = 0; x < VT; ++x) { const float v = to_f<S>(Vb[min(kk, end - 1) * stride + 16 * x + lr]); vv[x][r] = known ? v : 0.f; }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int n = k0 + 4 * lq + r - len;
        const bool in = n < 0 ? vis : (n < 64 && (seen >> n & 1));
        a[r] = in ? a[r] * p.scale : -INFINITY;
        mx = fmaxf(mx, a[r]);
      }
      mx = max_rows(mx);
      const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < 4; ++r) { a[r] = exp2f(a[r] - m_use); sum += a[r]; }
      sum = sum_rows(sum);
      const float alpha = exp2f(m_run - m_use);
      l_run = l_run * alpha + sum;
      m_run = m_new;
#pragma unroll
      for (int x = 0; x < VT; ++x) {
        acc[x] *= alpha;
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(vv[x][r], a[r], acc[x], 0, 0, 0);
      }
    }
  }
  if (lq == 0) { m_s[wave][lr] = m_run; l_s[wave][lr] = l_run; }
#pragma unroll
  for (int x = 0; x < VT; ++x) o_s[wave][x][lane] = acc[x];
  __syncthreads();
  float* part = p.part + ((((long)b * p.kv + hk) * gridDim.y + rb) * p.nsplit + split) * 16 * (D + 2);
  for (int x = wave; x < VT; x += 4) {
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, m_s[w][lr]);
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    const float M0 = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float a = exp2f(m_s[w][lr] - M0);
      L = fmaf(l_s[w][lr], a, L);
      o += o_s[w][x][lane] * a;
    }
    if (p.nsplit > 1) {
      *(f32x4*)(part + lr * D + 16 * x + 4 * lq) = o;
      if (x == 0 && lq == 0) { part[16 * D + lr] = M; part[16 * (D + 1) + lr] = L; }
    } else if (row < R) {
      tree_store4(p, b, node, hk * p.G + row - node * p.G, 16 * x + 4 * lq, row_ok && L > 0.f ? o / L : (row_ok && L != L ? f32x4{L, L, L, L} : f32x4{0.f, 0.f, 0.f, 0.f}));
    }
  }
}

// Partial results of the splits joined:  out = sum_s o_s 2^(m_s - M) / sum_s l_s 2^(m_s - M).  A row per D / 4 lanes, RB rows per row block.
template <int D>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeP p, int RB) {
  constexpr int Q = D / 4;                       // lanes of a row
  const int R = p.T * p.G, blocks = (R + RB - 1) / RB;
  const long id = (long)blockIdx.x * (256 / Q) + threadIdx.x / Q;      // (row, key head, sequence)
  if (id >= (long)p.B * p.kv * R) return;
  const int c = threadIdx.x % Q * 4, r = (int)(id % R), rb = r / RB, rr = r - rb * RB;
  const long pair = id / R;
  const int hk = (int)(pair % p.kv), b = (int)(pair / p.kv), node = r / p.G;
  const long step = (long)RB * (D + 2);
  const float* part = p.part + (pair * blocks + rb) * p.nsplit * step;
  float M = -INFINITY, L = 0.f;
  for (int s = 0; s < p.nsplit; ++s) M = fmaxf(M, part[s * step + RB * D + rr]);
  const float M0 = M == -INFINITY ? 0.f : M;
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < p.nsplit; ++s) {
    const float a = exp2f(part[s * step + RB * D + rr] - M0);
    L = fmaf(part[s * step + RB * (D + 1) + rr], a, L);
    o += *(const f32x4*)(part + s * step + rr * D + c) * a;
  }
  // (an absent node has seen nothing anywhere: L = 0)
  tree_store4(p, b, node, hk * p.G + r - node * p.G, c, L > 0.f ? o / L : (L != L ? f32x4{L, L, L, L} : f32x4{0.f, 0.f, 0.f, 0.f}));
}
