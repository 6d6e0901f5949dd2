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

#include <type_traits>

constexpr int TREE_MAX = 64;                     // nodes of a tree: one wave, one 64-bit word of ancestors
constexpr int TREE_GROUP = 32;                   // keys per group of a cache in operand order

struct TreeP {
  const void* q; long q_seq, q_row, q_head;      // elements from sequence to sequence, row to row, head to head; bf16 or fp32
  void* out; long o_seq, o_row, o_head;
  const void *K, *V;                             // one layer's cache
  int B, T, H, kv, G, cap;                       // cap: rows per sequence
  const int* length; const int* parent;          // parent null: a chain
  float scale, sign;                             // |scale| log2(e) (1 for a scale of 0), and the scale's sign (0)
  // the decoder's own steps: slots of sequences (cache and summaries of sequence seq[b], -1: none), a tree in a word for all, results as packed_at() of so many columns
  const int* seq; unsigned long long tree; int packed;
  // parts of the keys: `parts` in all of each key head's sequences, nsplit of each sequence, or (by_length) as many as its share of the keys; their results
  int nsplit, parts, by_length; float* part;
  int q_f32, o_f32, vec;                         // vec: rows of q and out are 16-byte aligned
  // chosen blocks (null: the whole prefix): bits [b][kv head][node][words], blocks of `bg` groups of 32 keys
  const unsigned* chosen; int words, bg;
};

typedef unsigned long long mask64;

// Where the element (key, dimension c) lies in a sequence's and head's part of a cache in operand order (c % 8 == 0: eight dimensions of K side by side)
template <int D> __device__ __forceinline__ size_t k_at(int key, int c) {
  return (size_t)(key >> 5) * (TREE_GROUP * D) + ((key >> 2) & 1) * (16 * D) + (c >> 5) * 512 + (((c >> 3) & 3) * 16 + ((key >> 3) & 3) * 4 + (key & 3)) * 8 + (c & 7);
}
template <int D> __device__ __forceinline__ size_t v_at(int key, int c) {
  return (size_t)(key >> 5) * (TREE_GROUP * D) + (c >> 4) * 512 + (((key >> 3) & 3) * 16 + (c & 15)) * 8 + (key & 7);
}

// Ancestors of node `lane` (bits), and whether it is there, by all 64 lanes of a wave: after round n a node knows 2^n of its ancestors.
__device__ __forceinline__ void tree_ancestors(const TreeP& tp, int b, int there, int lane, mask64& anc, bool& ok) {
  if (!tp.parent && !tp.tree) {                  // a chain
    ok = lane < there;
    anc = ok ? (~0ull >> (63 - lane)) : 0ull;
    return;
  }
  int p = -2;
  if (lane < tp.T) p = tp.parent ? tp.parent[(long)b * tp.T + lane] : (lane ? tree_parent(tp.tree, lane) : -1);
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

// Whose cache a sequence (or slot) has, and rows committed and drafted that it holds
__device__ __forceinline__ int tree_cache(const TreeP& p, int b) { const int s = p.seq ? p.seq[b] : b; return s < 0 ? 0 : s; }
__device__ __forceinline__ void tree_extent(const TreeP& p, int b, int& len, int& there) {
  len = p.length[b];
  if (p.seq && p.seq[b] < 0) len = -1;
  there = len < 0 ? 0 : (len >= p.cap ? 0 : (p.T < p.cap - len ? p.T : p.cap - len));
  len = len < 0 ? 0 : (len > p.cap ? p.cap : len);
}

// The sequence that a part belongs to, its number among that sequence's parts, how many those are and where they begin.  By length (up to 64 sequences, a lane each): one part each,
// and the others as the keys are spread.  (Eight documents of 8000 .. 32000 keys in equal numbers of parts: the longest one's decide.)
struct TreePart { int b, split, n, first; };
__device__ __forceinline__ void tree_shares(const TreeP& p, int lane, int& n, int& end) {
  const int len = lane < p.B ? p.length[lane] : -1;
  long items = len < 0 ? 0 : (min(len, p.cap) + p.T + 31) >> 5, all = items;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) all += __shfl_xor(all, o, 64);
  n = lane < p.B ? 1 + (all ? (int)((long)(p.parts - p.B) * items / all) : 0) : 0;
  end = n;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) { const int v = __shfl_up(end, o, 64); if (lane >= o) end += v; }
}
__device__ __forceinline__ TreePart tree_part(const TreeP& p, int at, int lane) {      // (b < 0: nobody's)
  if (!p.by_length) return TreePart{at / p.nsplit, at % p.nsplit, p.nsplit, at - at % p.nsplit};
  int n, end;
  tree_shares(p, lane, n, end);
  const mask64 mine = __ballot(at >= end - n && at < end);
  const int b = mine ? __ffsll((long long)mine) - 1 : -1, q = b < 0 ? 0 : b;
  const int nb = __builtin_amdgcn_readfirstlane(__shfl(n, q, 64)), first = __builtin_amdgcn_readfirstlane(__shfl(end, q, 64)) - nb;
  return TreePart{__builtin_amdgcn_readfirstlane(b), at - first, nb, first};
}
// ... of sequence b, by a wave whose lanes ask for sequences of their own
__device__ __forceinline__ void tree_parts_of(const TreeP& p, int b, int lane, int& n, int& first) {
  n = p.nsplit; first = b * p.nsplit;
  if (!p.by_length) return;
  int m, end;
  tree_shares(p, lane, m, end);
  n = __shfl(m, b, 64); first = __shfl(end, b, 64) - n;
}

// Four results of a row
__device__ __forceinline__ void tree_store4(const TreeP& p, int b, int node, int h, int c, const f32x4& v) {
  const long at = p.packed ? (long)packed_at((long)b * p.T + node, h * (int)p.o_head + c, p.packed) : (long)b * p.o_seq + (long)node * p.o_row + (long)h * p.o_head + c;
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
__device__ __forceinline__ float tree_q1(const TreeP& p, int b, int node, int h, int c) {
  const long at = (long)b * p.q_seq + (long)node * p.q_row + (long)h * p.q_head + c;
  return p.q_f32 ? ((const float*)p.q)[at] : bf2f(((const bf16_t*)p.q)[at]);
}
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
// List of the blocks that any node n0 .. n1 - 1 has chosen, in order, by all threads (at least as many as there are words).  The nodes' words are dealt to the threads: one trip to
// memory for up to 256 of them.  (A thread per word that walks the nodes: 0.5 us each.)
__device__ __forceinline__ int tree_list(const unsigned* chosen, int words, int n0, int n1, int done, unsigned short* list, int* sums, unsigned* bits_s) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, parts = (int)blockDim.x / words;
  if (tid < words) bits_s[tid] = 0;
  __syncthreads();
  if (tid < parts * words) {
    const int part = tid / words, w = tid - part * words;
    unsigned any = 0;
#pragma unroll 4
    for (int n = n0 + part; n < n1; n += parts) any |= chosen[(long)n * words + w];
    if (any) atomicOr(&bits_s[w], any);
  }
  __syncthreads();
  unsigned bits = 0;
  if (tid < words) {
    bits = bits_s[tid];
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

// What a wave does with one item (32 keys) for its MT row tiles, keys and values being operands in registers.
//   scores^T = K Q^T       32 keys x 16 rows per tile
//   softmax                p = 2^(s scale - m); m is raised, and sums and results with it, only when a score passes it by 2^8 (fp32 has room for that; nothing is rounded by
//                          it): maxima over the four lanes of a row, and multiplications of all results, are then rare.  Sums stay in their lanes until the end.
//   out^T += V^T P^T       the probabilities as they lie are the second operand
// Queries of bf16 are exact, those of fp32 a pair.  Probabilities go in as a pair hi + lo: as single bf16 numbers their rounding adds as much error as that of the bf16
// results (sum over keys of p (1 +- 2^-9) v), which the pair's second product takes to 2^-17.  (Against 64 bits, 40 and 2999 keys: fp32 results 2.1e-6 and 2.3e-6 of their size, fp32 weights
// 0.3e-6 and 0.8e-6; bf16 results 0.0017 either way, 0.2% of them the second nearest number instead of 0 to 0.09%.)
constexpr float TREE_SLACK = 8.f;
template <int D, int MT, bool QF32>
struct TreeTiles {
  static constexpr int KS = D / 32, VT = D / 16;
  float m[MT], l[MT];                            // per row what is subtracted (base 2; -inf: nothing seen), and this lane's part of the sum
  f32x4 acc[MT][VT];                             // dimensions 16 x + 4 lq + r of row lr
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      m[t] = -INFINITY; l[t] = 0.f;
#pragma unroll
      for (int x = 0; x < VT; ++x) acc[t][x] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  // kf, vf: the item's operands; at: this lane's first key among the drafts; edge: whether any key of the item is a draft (the same for the whole wave); vis: whether
  // row t sees the item's committed keys; seen: the drafts that it sees; q(t, x): its operand
  // SAFE: values one by one (value(key, dimension)), for the keys that a row sees and no others: a product's zero times what is not finite is not zero.  Nor are zeros that a pair of an
  // fp32 query adds: scores that are no number come once more, of the query as it is (score(t, key of this lane)).
  template <bool SAFE, typename Q, typename QL, typename V, typename S>
  __device__ __forceinline__ void item(const u32x4 (&kf)[2 * KS], const u32x4 (&vf)[VT], int at, bool edge, const bool (&vis)[MT], const mask64 (&seen)[MT], float scale, const Q& q, const QL& ql, const V& value, const S& score) {
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      f32x4 s[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x4 a = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < KS; ++x) {
          const bf16x8 ka = __builtin_bit_cast(bf16x8, kf[u * KS + x]);
          a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, q(t, x), a, 0, 0, 0);
          if constexpr (QF32) a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, ql(t, x), a, 0, 0, 0);
        }
        s[u] = a;
      }
      if constexpr (SAFE && QF32) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) if (s[u][r] != s[u][r]) s[u][r] = score(t, 4 * u + r);
      }
      if (edge) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int n = at + 4 * u + r;
            const bool in = n < 0 ? vis[t] : (n < 64 && (seen[t] >> n & 1));
            s[u][r] = in ? s[u][r] : -INFINITY;
          }
      } else {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[u][r] = vis[t] ? s[u][r] : -INFINITY;
      }
      float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))) * scale;
      if (__any(mx > m[t] + TREE_SLACK)) {
        mx = max_rows(mx);
        const float up = fmaxf(m[t], mx), alpha = up == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[t] - up);
        m[t] = up;
        l[t] *= alpha;
#pragma unroll
        for (int x = 0; x < VT; ++x) acc[t][x] *= alpha;
      }
      const float sub = m[t] == -INFINITY ? 0.f : m[t];
      float pv[8];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) { const float e = __builtin_amdgcn_exp2f(fmaf(s[u][r], scale, -sub)); pv[4 * u + r] = e; l[t] += e; }
      if constexpr (SAFE) {
        const int lane = threadIdx.x & 63, lr = lane & 15, lq = lane >> 4;
#pragma unroll 1
        for (int jq = 0; jq < 4; ++jq)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float pj = __shfl(pv[j], 16 * jq + lr, 64);
            const int n = at + 8 * (jq - lq) + j;
            if (n < 0 ? vis[t] : (n < 64 && (seen[t] >> n & 1))) {
#pragma unroll
              for (int x = 0; x < VT; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[t][x][r] = fmaf(pj, value(8 * jq + j, 16 * x + 4 * lq + r), acc[t][x][r]);
            }
          }
      } else {
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
  }
  // Is any of this lane's results not finite?
  __device__ __forceinline__ bool unclean() const {
    float z = 0.f;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int x = 0; x < VT; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) z = fmaf(acc[t][x][r], 0.f, z);
    return z != 0.f;                             // (0 times any of them)
  }
};
// Values of rows that nobody sees (behind the drafts, absent nodes): their probabilities are zero, their bits unknown.  at: as above
template <int VT>
__device__ __forceinline__ void tree_blank(u32x4 (&vf)[VT], int at, mask64 present) {
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
// Row r of a (sequence, key head) pair: its node, what it sees of the drafts, whether it is there
__device__ __forceinline__ void tree_row(const TreeP& p, int r, int R, mask64 anc, int& node, mask64& seen, bool& ok) {
  node = r < R ? r / p.G : 0;
  seen = (mask64)(unsigned)__shfl((int)(anc >> 32), node, 64) << 32 | (unsigned)__shfl((int)anc, node, 64);
  if (r >= R) seen = 0;
  ok = seen != 0;
}
// Its query's operand for the dimensions 32 x + 8 lq ..; hi and what that leaves
__device__ __forceinline__ void tree_q_operand(const TreeP& p, int b, int hk, int r, int node, bool ok, int c, bf16x8& hi, bf16x8& lo) {
  float v[8] = {};
  if (ok) tree_q8(p, b, node, hk * p.G + r - node * p.G, c, v);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] *= p.sign;    // (of the scale: the maximum is that of the products)
  tree_pair(v, hi, lo);
}
// q . K_key of a row that is there, term by term; K: the sequence's and head's keys in operand order
template <int D>
__device__ __forceinline__ float tree_score(const TreeP& p, int b, int hk, int r, int node, const bf16_t* K, int key) {
  float sum = 0.f;
#pragma unroll 1
  for (int c = 0; c < D; ++c) sum = fmaf(p.sign * tree_q1(p, b, node, hk * p.G + r - node * p.G, c), bf2f(K[k_at<D>(key, c)]), sum);
  return sum;
}
// What a row's sums make of it.  No weights at all: an absent node's zeros, or (there: all of its scores are -inf) no number, 0 / 0
__device__ __forceinline__ f32x4 tree_quotient(const f32x4& o, float L, bool there) {
  const float none = L != L || there ? NAN : 0.f;
  return L > 0.f ? o * (1.f / L) : f32x4{none, none, none, none};
}
// A row's result or partial result: dimensions c .. c + 3; there: its node is not absent.  Partial results: [key head][part][row][D], then [key head][part][row] maxima and as many sums
// (of a row that is there and has no weights in the part: 1, which the maximum of -inf takes away where another part has some)
__device__ __forceinline__ void tree_finish4(const TreeP& p, int D, int b, int hk, int part, int r, int R, int node, bool there, int c, float M, float L, const f32x4& o) {
  if (r >= R) return;
  if (p.parts > p.B) {
    const long at = ((long)hk * p.parts + part) * R + r, rows = (long)p.kv * p.parts * R;
    *(f32x4*)(p.part + at * D + c) = o;
    if (c == 0) { p.part[rows * D + at] = M; p.part[rows * (D + 1) + at] = L == 0.f && there ? 1.f : L; }
  } else {
    tree_store4(p, b, node, hk * p.G + r - node * p.G, c, tree_quotient(o, L, there));
  }
}

// bf16 heads of D = 64 or 128 in operand order (groups of 32 keys, D x 32 elements of K and as many of V, bpd_attention.h for D = 64; the same with
// D / 32 steps of K and D / 16 tiles of V otherwise): every operand is one 1 KiB load, nothing of K and V goes through LDS.
// Up to 48 rows (16 of 128-wide heads): a workgroup has all of a (sequence, key head) pair's, and one part of its items; its NW waves take single items in turn, each with its own
// maximum, sum and results, and meet once in LDS.  What bounds it is the stream of K and V; the next item's keys are asked for while this one's values are multiplied.
template <int D, int MT, int NW, bool QF32, bool SPARSE>
__global__ __launch_bounds__(64 * NW, 2) void tree_attention_kernel(TreeP p) {
  constexpr int KS = D / 32, VT = D / 16, GRP = TREE_GROUP * D, SLOTS = NW / 2 > 4 ? NW / 2 : 4;
  __shared__ __attribute__((aligned(16))) f32x4 o_s[SLOTS][VT][64];
  __shared__ float m_s[NW][MT * 16], l_s[NW][MT * 16];
  __shared__ unsigned short list_s[SPARSE ? TREE_BLOCKS_MAX : 1];
  __shared__ int sums_s[NW];
  __shared__ unsigned bits_s[SPARSE ? TREE_BLOCKS_MAX / 32 : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lq = lane >> 4;
  const int at_part = blockIdx.x, hk = blockIdx.y, R = p.T * p.G;
  const TreePart part = tree_part(p, at_part, lane);
  if (part.b < 0) return;
  const int b = part.b;
  const long pair = (long)b * p.kv + hk;
  const size_t own = ((size_t)tree_cache(p, b) * p.kv + hk) * p.cap * D;
  const u32x4* Kb = (const u32x4*)((const bf16_t*)p.K + own) + lane;
  const u32x4* Vb = (const u32x4*)((const bf16_t*)p.V + own) + lane;
  u32x4 kf[2 * KS], kn[2 * KS], vf[VT];
  auto load_k = [&](u32x4 (&k)[2 * KS], int g) {
#pragma unroll
    for (int x = 0; x < 2 * KS; ++x) k[x] = Kb[(size_t)g * (GRP / 8) + x * 64];
  };
  // with all keys here the first item's keys do not wait for the length
  if (!SPARSE && part.n == 1) load_k(kf, min(wave, p.cap / 32 - 1));
  int len, there;
  tree_extent(p, b, len, there);
  mask64 anc; bool ok;
  tree_ancestors(p, b, there, lane, anc, ok);
  const mask64 present = __ballot(ok);
  mask64 seen[MT]; int node[MT]; bool row_ok[MT];
  bf16x8 qh[MT][KS], ql[QF32 ? MT : 1][KS];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int r = 16 * t + lr;
    tree_row(p, r, R, anc, node[t], seen[t], row_ok[t]);
    bf16x8 lo;
#pragma unroll
    for (int x = 0; x < KS; ++x) { tree_q_operand(p, b, hk, r, node[t], row_ok[t], 32 * x + 8 * lq, qh[t][x], lo); if constexpr (QF32) ql[t][x] = lo; }
  }
  const int ngr = (len + there + 31) >> 5;
  TreeItems it{0, 0, ngr, nullptr, 1};
  const unsigned* picks = nullptr;
  if constexpr (SPARSE) {
    picks = p.chosen + pair * p.T * p.words;
    const int done = len / (32 * p.bg);
    it.list = list_s; it.bg = p.bg; it.tail0 = done * p.bg;
    it.listed = tree_list(picks, p.words, 0, p.T, done, list_s, sums_s, bits_s) * p.bg;
    it.n = it.listed + ngr - it.tail0;
  }
  const int i0 = (int)((long)it.n * part.split / part.n), i1 = (int)((long)it.n * (part.split + 1) / part.n);
  TreeTiles<D, MT, QF32> tiles;
  tiles.clear();
  unsigned word[SPARSE ? MT : 1];                // has the row chosen the item's block?
  auto load_words = [&](int ii, int gg) {
    if constexpr (SPARSE) {
      const int blk = gg / p.bg;
#pragma unroll
      for (int t = 0; t < MT; ++t) word[t] = ii < it.listed ? picks[(long)node[t] * p.words + (blk >> 5)] >> (blk & 31) & 1 : 1u;
    }
  };
  // one item, whose keys are here; ahead(): asks for what comes next
  auto one = [&](auto safe, u32x4 (&k)[2 * KS], int g, const auto& ahead) {
    constexpr bool SAFE = decltype(safe)::value;
    if constexpr (!SAFE) {
#pragma unroll
      for (int x = 0; x < VT; ++x) vf[x] = Vb[(size_t)g * (GRP / 8) + x * 64];
    }
    bool vis[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) { vis[t] = row_ok[t]; if constexpr (SPARSE) vis[t] = vis[t] && word[t]; }
    ahead();
    const int at = 32 * g + 8 * lq - len;
    const bool edge = 32 * g + 32 > len;
    if (!SAFE && edge) tree_blank<VT>(vf, at, present);
    tiles.template item<SAFE>(k, vf, at, edge, vis, seen, p.scale, [&](int t, int x) { return qh[t][x]; },
                              [&](int t, int x) { return ql[QF32 ? t : 0][x]; }, [&](int j, int c) { return bf2f(((const bf16_t*)p.V)[own + v_at<D>(32 * g + j, c)]); },
                              [&](int t, int j) { return row_ok[t] ? tree_score<D>(p, b, hk, 16 * t + lr, node[t], (const bf16_t*)p.K + own, 32 * g + 8 * lq + j) : 0.f; });
  };
  {
    int i = i0 + wave, g = i < i1 ? __builtin_amdgcn_readfirstlane(it.group(i)) : 0;
    if (i < i1) {
      load_words(i, g);
      if (SPARSE || part.n > 1) load_k(kf, g);
    }
    auto step = [&](u32x4 (&k)[2 * KS], u32x4 (&k_next)[2 * KS]) {
      const int next = i + NW, gn = next < i1 ? __builtin_amdgcn_readfirstlane(it.group(next)) : g;
      one(std::false_type{}, k, g, [&]() { if (next < i1) { load_words(next, gn); load_k(k_next, gn); } });
      i = next; g = gn;
    };
    while (i < i1) {                             // (two sets of keys in turn)
      step(kf, kn);
      if (i >= i1) break;
      step(kn, kf);
    }
  }
  if (__any(tiles.unclean())) {                  // again, value by value
    tiles.clear();
#pragma unroll 1
    for (int i = i0 + wave; i < i1; i += NW) {
      const int g = __builtin_amdgcn_readfirstlane(it.group(i));
      load_words(i, g);
      load_k(kf, g);
      one(std::true_type{}, kf, g, [&]() {});
    }
  }
  // the waves meet: maxima and sums first, then the upper half's results into the lower half's until four are left
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    tiles.l[t] = sum_rows(tiles.l[t]);
    if (lq == 0) { m_s[wave][16 * t + lr] = tiles.m[t]; l_s[wave][16 * t + lr] = tiles.l[t]; }
  }
  __syncthreads();
  float M[MT], L[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    M[t] = -INFINITY; L[t] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) M[t] = fmaxf(M[t], m_s[w][16 * t + lr]);
    const float M0 = M[t] == -INFINITY ? 0.f : M[t];
#pragma unroll
    for (int w = 0; w < NW; ++w) L[t] = fmaf(l_s[w][16 * t + lr], __builtin_amdgcn_exp2f(m_s[w][16 * t + lr] - M0), L[t]);
    const float a = __builtin_amdgcn_exp2f(tiles.m[t] - M0);
#pragma unroll
    for (int x = 0; x < VT; ++x) tiles.acc[t][x] *= a;
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) {
#pragma unroll
    for (int h = NW / 2; h >= 4; h /= 2) {
      if (wave >= h && wave < 2 * h) {
#pragma unroll
        for (int x = 0; x < VT; ++x) o_s[wave - h][x][lane] = tiles.acc[t][x];
      }
      __syncthreads();
      if (wave < h) {
#pragma unroll
        for (int x = 0; x < VT; ++x) tiles.acc[t][x] += o_s[wave][x][lane];
      }
      __syncthreads();
    }
    if (wave < 4) {
#pragma unroll
      for (int x = 0; x < VT; ++x) o_s[wave][x][lane] = tiles.acc[t][x];
    }
    __syncthreads();
    for (int x = wave; x < VT; x += NW) {
      const f32x4 o = (o_s[0][x][lane] + o_s[1][x][lane]) + (o_s[2][x][lane] + o_s[3][x][lane]);
      tree_finish4(p, D, b, hk, at_part, 16 * t + lr, R, node[t], row_ok[t], 16 * x + 4 * lq, M[t], L[t], o);
    }
    if (t + 1 < MT) __syncthreads();
  }
}

// More rows: the waves have rows of their own, 16 MT each, and walk the same items, which come through LDS, two buffers in turn: an operand is loaded once for 16 MT NW
// rows.  What bounds it is the matrix cores (6 D products per row and 64 keys, with the pairs) and, beside them, the exponentials.
template <int D, int MT, int NW, bool QF32, bool SPARSE>
__global__ __launch_bounds__(64 * NW, 2) void tree_attention_rows_kernel(TreeP p) {
  constexpr int KS = D / 32, VT = D / 16, GRP = TREE_GROUP * D, PIECES = 4 * D, PER = 2 * PIECES / (64 * NW);   // 16-byte pieces of K (and of V) in an item; of both per thread
  static_assert(PER >= 1, "");
  __shared__ __attribute__((aligned(16))) u32x4 kv_s[2][2 * PIECES];
  __shared__ unsigned short list_s[SPARSE ? TREE_BLOCKS_MAX : 1];
  __shared__ int sums_s[NW];
  __shared__ unsigned bits_s[SPARSE ? TREE_BLOCKS_MAX / 32 : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lq = lane >> 4;
  const int at_part = blockIdx.x % p.parts, rb = blockIdx.x / p.parts, hk = blockIdx.y, R = p.T * p.G, r0 = (rb * NW + wave) * 16 * MT;
  const TreePart part = tree_part(p, at_part, lane);
  if (part.b < 0) return;
  const int b = part.b;
  const long pair = (long)b * p.kv + hk;
  int len, there;
  tree_extent(p, b, len, there);
  mask64 anc; bool ok;
  tree_ancestors(p, b, there, lane, anc, ok);
  const mask64 present = __ballot(ok);
  mask64 seen[MT]; int node[MT]; bool row_ok[MT];
  bf16x8 qh[MT][KS], ql[QF32 ? MT : 1][KS];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int r = r0 + 16 * t + lr;
    tree_row(p, r, R, anc, node[t], seen[t], row_ok[t]);
    bf16x8 lo;
#pragma unroll
    for (int x = 0; x < KS; ++x) { tree_q_operand(p, b, hk, r, node[t], row_ok[t], 32 * x + 8 * lq, qh[t][x], lo); if constexpr (QF32) ql[t][x] = lo; }
  }
  const int ngr = (len + there + 31) >> 5;
  TreeItems it{0, 0, ngr, nullptr, 1};
  const unsigned* picks = nullptr;
  if constexpr (SPARSE) {
    picks = p.chosen + pair * p.T * p.words;
    const int done = len / (32 * p.bg), w0 = rb * NW * 16 * MT, w1 = min(R, w0 + NW * 16 * MT);
    it.list = list_s; it.bg = p.bg; it.tail0 = done * p.bg;
    it.listed = tree_list(picks, p.words, w0 / p.G, (w1 + p.G - 1) / p.G, done, list_s, sums_s, bits_s) * p.bg;
    it.n = it.listed + ngr - it.tail0;
  }
  const int i0 = (int)((long)it.n * part.split / part.n), i1 = (int)((long)it.n * (part.split + 1) / part.n);
  const size_t own = ((size_t)tree_cache(p, b) * p.kv + hk) * p.cap * D;
  const u32x4* Kb = (const u32x4*)((const bf16_t*)p.K + own);
  const u32x4* Vb = (const u32x4*)((const bf16_t*)p.V + own);
  TreeTiles<D, MT, QF32> tiles;
  tiles.clear();
  u32x4 kvn[PER];                                // (a wave's pieces are all of K or all of V)
  auto ask = [&](int g) {
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      const int z = (wave + x * NW) * 64;
      kvn[x] = (z < PIECES ? Kb + (size_t)g * (GRP / 8) + z : Vb + (size_t)g * (GRP / 8) + z - PIECES)[lane];
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int x = 0; x < PER; ++x) kv_s[buf][tid + x * 64 * NW] = kvn[x];
  };
  unsigned word[SPARSE ? MT : 1];                // has the row chosen the item's block?
  auto load_words = [&](int ii, int gg) {
    if constexpr (SPARSE) {
      const int blk = gg / p.bg;
#pragma unroll
      for (int t = 0; t < MT; ++t) word[t] = ii < it.listed ? picks[(long)node[t] * p.words + (blk >> 5)] >> (blk & 31) & 1 : 1u;
    }
  };
  auto walk = [&](auto safe) {
    constexpr bool SAFE = decltype(safe)::value;
    int g = 0;
    if (i0 < i1) { g = __builtin_amdgcn_readfirstlane(it.group(i0)); load_words(i0, g); ask(g); put(0); }
    __syncthreads();
    for (int i = i0; i < i1; ++i) {
      const int buf = (i - i0) & 1;
      const int gn = i + 1 < i1 ? __builtin_amdgcn_readfirstlane(it.group(i + 1)) : g;
      unsigned now[SPARSE ? MT : 1];
#pragma unroll
      for (int t = 0; t < (SPARSE ? MT : 0); ++t) now[t] = word[t];
      if (i + 1 < i1) { load_words(i + 1, gn); ask(gn); }
      u32x4 kf[2 * KS], vf[VT];
#pragma unroll
      for (int x = 0; x < 2 * KS; ++x) kf[x] = kv_s[buf][x * 64 + lane];
      if constexpr (!SAFE) {
#pragma unroll
        for (int x = 0; x < VT; ++x) vf[x] = kv_s[buf][PIECES + x * 64 + lane];
      }
      bool vis[MT];
#pragma unroll
      for (int t = 0; t < MT; ++t) { vis[t] = row_ok[t]; if constexpr (SPARSE) vis[t] = vis[t] && now[t]; }
      const int at = 32 * g + 8 * lq - len;
      const bool edge = 32 * g + 32 > len;
      if (!SAFE && edge) tree_blank<VT>(vf, at, present);
      tiles.template item<SAFE>(kf, vf, at, edge, vis, seen, p.scale, [&](int t, int x) { return qh[t][x]; }, [&](int t, int x) { return ql[QF32 ? t : 0][x]; },
                                [&](int j, int c) { return bf2f(((const bf16_t*)p.V)[own + v_at<D>(32 * g + j, c)]); },
                                [&](int t, int j) { return row_ok[t] ? tree_score<D>(p, b, hk, r0 + 16 * t + lr, node[t], (const bf16_t*)p.K + own, 32 * g + 8 * lq + j) : 0.f; });
      if (i + 1 < i1) put(buf ^ 1);
      __syncthreads();
      g = gn;
    }
  };
  walk(std::false_type{});
  if (__syncthreads_or(tiles.unclean())) { tiles.clear(); walk(std::true_type{}); }
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const float L = sum_rows(tiles.l[t]);
#pragma unroll
    for (int x = 0; x < VT; ++x) tree_finish4(p, D, b, hk, at_part, r0 + 16 * t + lr, R, node[t], row_ok[t], 16 * x + 4 * lq, tiles.m[t], L, tiles.acc[t][x]);
  }
}

// fp32 caches, and bf16 ones of 16-wide heads, whose rows lie as they are ([rows][kv heads][D]): the same walk in fp32 on
// v_mfma_f32_16x16x4_f32 (keys in tiles of 16).  One element per lane and operand: K's dimensions go in by fours as they lie, of V a lane takes the
// dimension of its own from each of its four keys, and nothing is transposed.
template <typename S, int D, bool SPARSE>
__global__ __launch_bounds__(256) void tree_rows_kernel(TreeP p) {
  constexpr int VT = D / 16, CH = VT;
  __shared__ __attribute__((aligned(16))) f32x4 o_s[4][VT][64];
  __shared__ float m_s[4][16], l_s[4][16];
  __shared__ unsigned short list_s[SPARSE ? TREE_BLOCKS_MAX : 1];
  __shared__ int sums_s[4];
  __shared__ unsigned bits_s[SPARSE ? TREE_BLOCKS_MAX / 32 : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lq = lane >> 4;
  const int at_part = blockIdx.x % p.parts, rb = blockIdx.x / p.parts, hk = blockIdx.y, R = p.T * p.G, r0 = rb * 16;
  const TreePart part = tree_part(p, at_part, lane);
  if (part.b < 0) return;
  const int b = part.b;
  int len, there;
  tree_extent(p, b, len, there);
  mask64 anc; bool ok;
  tree_ancestors(p, b, there, lane, anc, ok);
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
      q[x][j] = !row_ok ? 0.f : p.sign * (p.q_f32 ? ((const float*)p.q)[at] : bf2f(((const bf16_t*)p.q)[at]));
    }
  const int ngr = (len + there + 31) >> 5;
  TreeItems it{0, 0, ngr, nullptr, 1};
  const unsigned* picks = nullptr;
  if constexpr (SPARSE) {
    picks = p.chosen + ((long)b * p.kv + hk) * p.T * p.words;
    const int done = len / (32 * p.bg), n0 = r0 / p.G, n1 = min(p.T, (min(R, r0 + 16) + p.G - 1) / p.G);
    it.list = list_s; it.bg = p.bg; it.tail0 = done * p.bg;
    it.listed = tree_list(picks, p.words, n0, n1, done, list_s, sums_s, bits_s) * p.bg;
    it.n = it.listed + ngr - it.tail0;
  }
  const int i0 = (int)((long)it.n * part.split / part.n), i1 = (int)((long)it.n * (part.split + 1) / part.n);
  const long stride = (long)p.kv * D;
  const long own = (long)tree_cache(p, b) * p.cap * stride + hk * D;
  const S* Kb = (const S*)p.K + own;
  const S* Vb = (const S*)p.V + own;
  float m_run, l_run;
  f32x4 acc[VT];
  auto walk = [&](auto safe) {
    constexpr bool SAFE = decltype(safe)::value;
    m_run = -INFINITY; l_run = 0.f;
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
        f32x4 part_a[CH];                          // (sums of an eighth of the dimensions, then of those: a chain over 128 of them is off by three times as much)
#pragma unroll
        for (int x = 0; x < CH; ++x) part_a[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < VT; ++x) {
          const S* kp = Kb + key * stride + 16 * x + 4 * lq;
          float kv[4];
          if constexpr (sizeof(S) == 4) { const f32x4 w = *(const f32x4*)kp; kv[0] = w[0]; kv[1] = w[1]; kv[2] = w[2]; kv[3] = w[3]; }
          else { const u32x2 w = *(const u32x2*)kp; kv[0] = __uint_as_float(w[0] << 16); kv[1] = __uint_as_float(w[0] & 0xFFFF0000u); kv[2] = __uint_as_float(w[1] << 16); kv[3] = __uint_as_float(w[1] & 0xFFFF0000u); }
#pragma unroll
          for (int j = 0; j < 4; ++j) part_a[x % CH] = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[j], q[x][j], part_a[x % CH], 0, 0, 0);
        }
        f32x4 a = part_a[0];
        if constexpr (CH == 4) a = (part_a[0] + part_a[1]) + (part_a[2] + part_a[3]);
        if constexpr (CH == 8) a = ((part_a[0] + part_a[1]) + (part_a[2] + part_a[3])) + ((part_a[4] + part_a[5]) + (part_a[6] + part_a[7]));
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
          a[r] = in ? a[r] : -INFINITY;
          mx = fmaxf(mx, a[r]);
        }
        // (scaled in the difference: the rounding of m is the same factor in every weight, and no other is made)
        mx = max_rows(mx) * p.scale;
        const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) { a[r] = exp2f(fmaf(a[r], p.scale, -m_use)); sum += a[r]; }
        sum = sum_rows(sum);
        const float alpha = exp2f(m_run - m_use);
        l_run = l_run * alpha + sum;
        m_run = m_new;
#pragma unroll
        for (int x = 0; x < VT; ++x) acc[x] *= alpha;
        if constexpr (SAFE) {                    // (as TreeTiles::item)
#pragma unroll 1
          for (int jq = 0; jq < 4; ++jq)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float pj = __shfl(a[j], 16 * jq + lr, 64);
              const int kk = k0 + 4 * jq + j, n = kk - len;
              if (n < 0 ? vis : (n < 64 && (seen >> n & 1))) {
#pragma unroll
                for (int x = 0; x < VT; ++x)
#pragma unroll
                  for (int r = 0; r < 4; ++r) acc[x][r] = fmaf(pj, to_f<S>(Vb[kk * stride + 16 * x + 4 * lq + r]), acc[x][r]);
              }
            }
        } else {
#pragma unroll
          for (int x = 0; x < VT; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(vv[x][r], a[r], acc[x], 0, 0, 0);
        }
      }
    }
  };
  walk(std::false_type{});
  float z = 0.f;
#pragma unroll
  for (int x = 0; x < VT; ++x)
#pragma unroll
    for (int r = 0; r < 4; ++r) z = fmaf(acc[x][r], 0.f, z);
  if (__any(z != 0.f)) walk(std::true_type{});
  if (lq == 0) { m_s[wave][lr] = m_run; l_s[wave][lr] = l_run; }
#pragma unroll
  for (int x = 0; x < VT; ++x) o_s[wave][x][lane] = acc[x];
  __syncthreads();
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
    tree_finish4(p, D, b, hk, at_part, row, R, node, row_ok, 16 * x + 4 * lq, M, L, o);
  }
}

// Partial results of a row's parts joined:  out = sum_s o_s 2^(m_s - M) / sum_s l_s 2^(m_s - M).  NW waves per row: their lanes find the maximum, then D / 4 of them at a time
// take a part each, all of a thread's under way together, and meet in LDS: three trips to memory whatever the number of parts (64 of them, one thread after the other: 33 us;
// so 5).
template <int D, int NW>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeP p) {
  constexpr int Q = D / 4, NG = 64 * NW / Q;
  __shared__ __attribute__((aligned(16))) f32x4 o_s[256];
  __shared__ float l_s[256];
  const int R = p.T * p.G, tid = threadIdx.x, lane = tid & 63, own = tid % (64 * NW), c = own % Q, ng = own / Q;
  const long id = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (4 / NW) + tid / (64 * NW)));
  const bool live = id < (long)p.B * p.kv * R;
  const int pair = live ? (int)(id / R) : 0, r = live ? (int)(id - (long)pair * R) : 0, b = pair / p.kv, hk = pair - b * p.kv;
  int n, first;
  tree_parts_of(p, b, lane, n, first);
  n = __builtin_amdgcn_readfirstlane(n); first = __builtin_amdgcn_readfirstlane(first);
  const long at = ((long)hk * p.parts + first) * R + r, rows = (long)p.kv * p.parts * R;
  const float *ms = p.part + rows * D + at, *ls = ms + rows;
  float M = -INFINITY;
  for (int s = lane; s < n; s += 64) M = fmaxf(M, ms[(long)s * R]);
  M = wave_max(M);
  const float M0 = M == -INFINITY ? 0.f : M;
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  float L = 0.f;
#pragma unroll 4
  for (int s = ng; s < n; s += NG) {
    const float a = exp2f(ms[(long)s * R] - M0);
    L = fmaf(ls[(long)s * R], a, L);
    o += *(const f32x4*)(p.part + (at + (long)s * R) * D + 4 * c) * a;
  }
  o_s[tid] = o; l_s[tid] = L;
  __syncthreads();
  if (ng || !live) return;
  const int used = min(NG, n);
  for (int x = 1; x < used; ++x) { o += o_s[tid + x * Q]; L += l_s[tid + x * Q]; }
  const int node = r / p.G;
  const float none = L != L || (L == 0.f && ls[0] != 0.f) ? NAN : 0.f;           // (as tree_quotient; without weights in all parts, and there: 1 in each)
  tree_store4(p, b, node, hk * p.G + r - node * p.G, 4 * c, L > 0.f ? o / L : f32x4{none, none, none, none});
}
