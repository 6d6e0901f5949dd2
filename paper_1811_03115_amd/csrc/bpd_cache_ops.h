// Rows stored into a cache, blocks of it chosen by a bound of their scores, and trees of drafts verified.  Included by bpd_cache.hip after
// bpd_cache_attention.h.
#pragma once
#include "bpd_cache_attention.h"

// ------------------------------------------------------------------------------------------------ rows into a cache

struct RowsP { const void* data; int f32, vec; long layer, seq, row, head; };      // vec: eight elements can be loaded at once
struct StoreP {
  RowsP k, v;
  void *K, *V; long layer;                       // elements of a layer's cache
  int B, T, kv, cap;
  const int* start; const int* count;            // count null: T
};
__device__ __forceinline__ u32x4 rows_bf16x8(const RowsP& p, long at) {
  if (!p.f32) {
    const bf16_t* s = (const bf16_t*)p.data + at;
    if (p.vec) return *(const u32x4*)s;
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (unsigned)s[2 * j] | (unsigned)s[2 * j + 1] << 16;
    return w;
  }
  const float* s = (const float*)p.data + at;
  u32x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = cvt_pk_bf16(s[2 * j], s[2 * j + 1]);
  return w;
}
// Which rows of sequence b's part go where: row i to key first + i, for lo <= i < hi
__device__ __forceinline__ void store_extent(const StoreP& p, int b, int& first, int& lo, int& hi) {
  first = p.start[b];
  int n = p.count ? p.count[b] : p.T;
  n = n < 0 ? 0 : (n > p.T ? p.T : n);
  lo = 0;
  hi = first < 0 || first >= p.cap ? 0 : (n < p.cap - first ? n : p.cap - first);
}
// One group of 32 keys of one (layer, sequence, head) per workgroup.  A stream in and a stream out: K goes by 16-byte pieces straight to its place; V, of which eight
// keys of a dimension lie side by side, is turned in LDS.  Pieces that only some of the new rows are in keep the others.
template <int D>
__global__ __launch_bounds__(256) void store_groups_kernel(StoreP p) {
  constexpr int PIECES = 4 * D;                  // of 8 elements, in a group of K, and in one of V
  __shared__ __attribute__((aligned(16))) bf16_t v_s[32][D + 8];
  const int tid = threadIdx.x, h = blockIdx.y, layer = blockIdx.z / p.B, b = blockIdx.z - layer * p.B;
  int first, lo, hi;
  store_extent(p, b, first, lo, hi);
  if (hi <= lo) return;
  const int key0 = ((first >> 5) + (int)blockIdx.x) * 32;
  if (key0 >= first + hi) return;
  const long ks = (long)layer * p.k.layer + (long)b * p.k.seq + (long)h * p.k.head, vs = (long)layer * p.v.layer + (long)b * p.v.seq + (long)h * p.v.head;
  const size_t part = (size_t)layer * p.layer + ((size_t)b * p.kv + h) * p.cap * D + (size_t)key0 * D;
  bf16_t *K = (bf16_t*)p.K + part, *V = (bf16_t*)p.V + part;
  constexpr int N = PIECES / 256;
  u32x4 v[N], k[N];
  bool there[N];                                 // (all loads first: four sequences of up to 8100 rows, 8 heads of 128 32.8 us instead of 34.3)
#pragma unroll
  for (int j = 0; j < N; ++j) {                  // V's rows: D / 8 pieces each
    const int x = j * 256 + tid, key = x / (D / 8), i = key0 + key - first;
    v[j] = u32x4{0, 0, 0, 0};
    if (i >= lo && i < hi) v[j] = rows_bf16x8(p.v, vs + (long)i * p.v.row + x % (D / 8) * 8);
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {                  // [t][s][q][a][r]
    const int x = j * 256 + tid, r = x & 3, a = (x >> 2) & 3, q = (x >> 4) & 3, s = (x >> 6) % (D / 32), t = (x >> 6) / (D / 32), i = key0 + 8 * a + 4 * t + r - first;
    there[j] = i >= lo && i < hi;
    if (there[j]) k[j] = rows_bf16x8(p.k, ks + (long)i * p.k.row + 32 * s + 8 * q);
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int x = j * 256 + tid;
    *(u32x4*)&v_s[x / (D / 8)][x % (D / 8) * 8] = v[j];
  }
#pragma unroll
  for (int j = 0; j < N; ++j) if (there[j]) *(u32x4*)(K + (j * 256 + tid) * 8) = k[j];
  __syncthreads();
  for (int x = tid; x < PIECES; x += 256) {      // [tile][q][c]
    const int c = x & 15, q = (x >> 4) & 3, t = x >> 6, i = key0 + 8 * q - first;
    bf16_t e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = v_s[8 * q + j][16 * t + c];
    if (i >= lo && i + 7 < hi) {
      u32x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = (unsigned)e[2 * j] | (unsigned)e[2 * j + 1] << 16;
      *(u32x4*)(V + x * 8) = w;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) if (i + j >= lo && i + j < hi) V[x * 8 + j] = e[j];
    }
  }
}
// Caches whose rows lie as they are: an element per thread
template <typename S>
__global__ __launch_bounds__(256) void store_rows_kernel(StoreP p, int D) {
  const int layer = blockIdx.z / p.B, b = blockIdx.z - layer * p.B;
  int first, lo, hi;
  store_extent(p, b, first, lo, hi);
  for (int i = lo + blockIdx.x; i < hi; i += gridDim.x) for (int x = threadIdx.x; x < p.kv * D; x += 256) {
    const int h = x / D, c = x - h * D;
    const size_t to = (size_t)layer * p.layer + ((size_t)b * p.cap + first + i) * p.kv * D + x;
    const long ka = (long)layer * p.k.layer + (long)b * p.k.seq + (long)i * p.k.row + (long)h * p.k.head + c, va = (long)layer * p.v.layer + (long)b * p.v.seq + (long)i * p.v.row + (long)h * p.v.head + c;
    ((S*)p.K)[to] = from_f<S>(p.k.f32 ? ((const float*)p.k.data)[ka] : bf2f(((const bf16_t*)p.k.data)[ka]));
    ((S*)p.V)[to] = from_f<S>(p.v.f32 ? ((const float*)p.v.data)[va] : bf2f(((const bf16_t*)p.v.data)[va]));
  }
}

// ------------------------------------------------------------------------------------------------ blocks chosen by a bound

// Summaries: per (sequence, key head) tiles of 64 blocks, [2: smallest, largest][D / 8][64 blocks][8], so that a wave with a block per lane reads 1 KiB at a time.
struct BoundP {
  TreeP t;
  void* summaries; int tiles;                    // 64 blocks each
  int block, first, recent, top;
  const int* added; int added_all;               // rows behind which the summaries are still those of the last call; null: added_all for each (< 0: all are made anew)
  double* score;                                 // [b][kv head][node][64 tiles]
  unsigned* chosen;                              // [b][kv head][node][words]
};
// Eight of a cache's elements as they come
template <typename S> struct Eight;
template <> struct Eight<bf16_t> {
  u32x4 w;
  __device__ __forceinline__ void load(const bf16_t* k) { w = *(const u32x4*)k; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) { v[2 * j] = __uint_as_float(w[j] << 16); v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u); }
  }
};
template <> struct Eight<float> {
  f32x4 x, y;
  __device__ __forceinline__ void load(const float* k) { x = *(const f32x4*)k; y = *(const f32x4*)(k + 4); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) { v[j] = x[j]; v[4 + j] = y[j]; }
  }
};
typedef double f64x4 __attribute__((ext_vector_type(4)));
// The bound of one (node, block), term by term: sum is where the block's summary begins.  (No key but NaN in a dimension: no number.)
template <typename S, int D>
__device__ double block_bound(const TreeP& t, int b, int n, int hk, const S* sum) {
  double bound = 0.0;
  for (int c = 0; c < D; ++c) {
    const S* at = sum + (size_t)(c / 8) * 512 + c % 8;
    const double mn = to_f<S>(at[0]), mx = to_f<S>(at[(size_t)(D / 8) * 512]);
    for (int g = 0; g < t.G; ++g) {
      const double v = t.sign * tree_q1(t, b, n, hk * t.G + g, c), x = v * mn, y = v * mx;
      bound += mn > mx ? (double)NAN : (x != x ? x : (y != y || y > x ? y : x));
    }
  }
  return bound;
}
// Upper bound of a group's scores in a block, summed over its G heads (q: with the scale's sign):  sum_g sum_c max(q_gc min_c, q_gc max_c) = sum_c max_c sum_g q+_gc + min_c sum_g q-_gc, so that
// the heads are added first and cost nothing, and what is left is a product of 16 nodes with 64 blocks over 2 D.  In 64 bits, on v_mfma_f64_16x16x4_f64: products of bf16 numbers and
// their sums are then as good as exact, and which blocks are chosen does not depend on an order of summation.  (On the vector units the nodes' sums, the same for all lanes, come out
// of LDS once per block and wave, which bounds it: 7 nodes, 1000 blocks of 128 dimensions in 32 pairs 13.6 us.)
// One tile of 64 blocks of one (sequence, key head), and 16 nodes, per workgroup: a wave has 16 blocks, and of 32 dimensions at a time lane 16 q + c eight of block c.
// Blocks that the last rows have touched are summarised first, by each of a tile's workgroups (the same values; one block in most calls).
template <typename S, int D, bool GROUPED>
__global__ __launch_bounds__(256) void block_bounds_kernel(BoundP p) {
  constexpr int C8 = D / 8, W = C8, PER = 256 / W;
  __shared__ double q_s[2 * C8][8][17];          // [eight dimensions: negative parts, then positive][dimension][node]
  __shared__ float part_s[4][2][D];              // [wave][smallest, largest]
  const TreeP& t = p.t;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hk = blockIdx.y, b = blockIdx.z;
  const int tile = blockIdx.x % p.tiles, n0 = blockIdx.x / p.tiles * 16, nn = min(16, t.T - n0);
  // (nothing of this waits for the length: summaries, as far as they stay, and queries)
  const size_t own = tree_cache(t, b);
  S* sum = (S*)p.summaries + ((own * t.kv + hk) * p.tiles + tile) * (2 * D * 64);
  const int c = lane & 15, q = lane >> 4;
  Eight<S> v[C8 / 2];
  auto load = [&]() {
#pragma unroll
    for (int x = 0; x < C8 / 2; ++x) v[x].load(sum + ((size_t)(4 * x + q) * 64 + 16 * wave + c) * 8);
  };
  if (nn > 0) load();
  for (int x = tid; x < 16 * C8; x += 256) {
    const int n = x & 15, c8 = x >> 4;
    double pos[8] = {}, neg[8] = {};
    if (n < nn) {
#pragma unroll 4
      for (int g = 0; g < t.G; ++g) {
        float v[8];
        tree_q8(t, b, n0 + n, hk * t.G + g, 8 * c8, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {            // (the scale's size changes no order, its sign does; one that is no number goes to both)
          const float x = v[j] * t.sign;
          pos[j] += (double)(x < 0.f ? 0.f : x); neg[j] += (double)(x > 0.f ? 0.f : x);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) { q_s[c8][j][n] = neg[j]; q_s[C8 + c8][j][n] = pos[j]; }
  }
  int len, there;
  tree_extent(t, b, len, there);
  const int done = len / p.block, blk0 = 64 * tile;
  if (blk0 >= done) return;
  int from = p.added_all < 0 ? 0 : max(0, len - p.added_all) / p.block;
  if (p.added) { const int n = p.added[b]; from = n < 0 ? done : (n >= len ? 0 : (len - n) / p.block); }
  const int f0 = max(from, blk0), f1 = min(done, blk0 + 64);
  for (int blk = f0; blk < f1; ++blk) {          // a thread has eight dimensions of every PER-th row; lanes of the same dimensions meet by moves, waves in LDS
    const int w = tid % W;
    float mn[8], mx[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) { mn[j] = INFINITY; mx[j] = -INFINITY; }
#pragma unroll 4
    for (int r = tid / W; r < p.block; r += PER) {
      const int key = blk * p.block + r;
      const S* k;
      if constexpr (GROUPED) k = (const S*)t.K + (own * t.kv + hk) * t.cap * D + k_at<D>(key, 8 * w);
      else k = (const S*)t.K + (own * t.cap + key) * t.kv * D + (size_t)hk * D + 8 * w;
      Eight<S> e;
      float f[8];
      e.load(k);
      e.get(f);
#pragma unroll
      for (int j = 0; j < 8; ++j) { mn[j] = fminf(mn[j], f[j]); mx[j] = fmaxf(mx[j], f[j]); }
    }
#pragma unroll
    for (int x = W; x < 64; x <<= 1)
#pragma unroll
      for (int j = 0; j < 8; ++j) { mn[j] = fminf(mn[j], __shfl_xor(mn[j], x, 64)); mx[j] = fmaxf(mx[j], __shfl_xor(mx[j], x, 64)); }
    if (lane < W) {
#pragma unroll
      for (int j = 0; j < 8; ++j) { part_s[wave][0][8 * w + j] = mn[j]; part_s[wave][1][8 * w + j] = mx[j]; }
    }
    __syncthreads();
    if (tid < 2 * D) {
      const int big = tid / D, c = tid - big * D;
      float v = part_s[0][big][c];
#pragma unroll
      for (int x = 1; x < 4; ++x) { const float u = part_s[x][big][c]; v = big ? fmaxf(v, u) : fminf(v, u); }
      sum[((size_t)(big * W + c / 8) * 64 + blk - blk0) * 8 + c % 8] = from_f<S>(v);
    }
    __syncthreads();                             // (and what has been written is there for all of the workgroup)
  }
  if (nn <= 0) return;                           // (summaries alone)
  if (f1 > f0) load();
  __syncthreads();
  const bool known = blk0 + 16 * wave + c < done;
  // (Not finite: the sum as it is defined.  A part that is zero times an infinite key is no number, and heads that have been added first hide such a part of one of them, or make -inf
  // of a dimension without a key.)
  auto finish = [&](int n, double bound) {
    if (!(fabs(bound) < (double)INFINITY) && known) bound = block_bound<S, D>(t, b, n0 + n, hk, sum + (16 * wave + c) * 8);
    p.score[((((size_t)b * t.kv + hk) * t.T + n0 + n) * p.tiles + tile) * 64 + 16 * wave + c] = bound;
  };
  if (nn <= 2) {                                 // (most of the product would be of nodes that are not there: one node, 1875 blocks of 128 dimensions 7.5 us instead of 8.9)
    for (int n = 0; n < nn; ++n) {
      double even = 0.0, odd = 0.0;
#pragma unroll
      for (int x = 0; x < C8 / 2; ++x) {
        float f[8];
        v[x].get(f);
#pragma unroll
        for (int j = 0; j < 8; j += 2) { even = fma(q_s[4 * x + q][j][n], (double)f[j], even); odd = fma(q_s[4 * x + q][j + 1][n], (double)f[j + 1], odd); }
      }
      even += odd;
      even += __shfl_xor(even, 16, 64);
      even += __shfl_xor(even, 32, 64);
      if (q == n) finish(n, even);
    }
    return;
  }
  f64x4 acc = f64x4{0, 0, 0, 0}, odd = acc;      // (two chains)
#pragma unroll
  for (int x = 0; x < C8 / 2; ++x) {
    float f[8];
    v[x].get(f);
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      acc = __builtin_amdgcn_mfma_f64_16x16x4f64(q_s[4 * x + q][j][c], (double)f[j], acc, 0, 0, 0);
      odd = __builtin_amdgcn_mfma_f64_16x16x4f64(q_s[4 * x + q][j + 1][c], (double)f[j + 1], odd, 0, 0, 0);
    }
  }
  acc += odd;
#pragma unroll
  for (int i = 0; i < 4; ++i) if (4 * i + q < nn) finish(4 * i + q, acc[i]);         // node 4 i + q, block c of the wave's
}

// Order-preserving key of a bound: a larger one has a larger key, one that is no number the smallest
__device__ __forceinline__ unsigned long long bound_key(double score) {
  const double s = score + 0.0;                  // (no negative zero)
  const unsigned long long u = (unsigned long long)__double_as_longlong(s);
  return s != s ? 1ull : (u >> 63 ? ~u : u | 1ull << 63);
}
// A workgroup of T threads for the up to T N blocks of one (node, key head, sequence): the first and the last ones, and of the others the `top` with the largest bounds, ties to the
// lower block; a bound that is no number comes last.  Order-preserving 64-bit keys, in registers; a digit of eight bits at a time from the first bit in which they differ (most keys share
// sign and exponent, and a histogram of those would be one counter), until the digit that the last chosen one is in holds no more than are wanted.  A histogram per digit,
// all cleared at the start, which every wave adds up by itself: one barrier a digit.  (Two or three digits mostly: 94 blocks 5.0 us, 1875 5.8, of which a launch is 2.  Bit by bit with ballots, one wave: 94
// blocks 5.1; eight waves, a barrier a bit: 1875 blocks 9.2.)
template <int T, int N>
__global__ __launch_bounds__(T) void block_pick_kernel(BoundP p) {
  __shared__ __attribute__((aligned(16))) unsigned hist[8][256];
  __shared__ unsigned long long and_s[T / 64], or_s[T / 64];
  __shared__ int cnt_s[N][T / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
  const TreeP& t = p.t;
  const size_t row = ((size_t)b * t.kv + hk) * t.T + n;
  const double* score = p.score + row * p.tiles * 64;
  double s[N];                              // (before the length is there; what is behind the complete blocks is not looked at)
#pragma unroll
  for (int j = 0; j < N; ++j) { const int blk = j * T + tid; s[j] = blk < p.tiles * 64 ? score[blk] : 0.0; }
  for (int x = tid; x < 8 * 256 / 4; x += T) ((u32x4*)hist)[x] = u32x4{0, 0, 0, 0};
  int len, there;
  tree_extent(t, b, len, there);
  mask64 anc; bool ok;
  tree_ancestors(t, b, there, lane, anc, ok);
  const bool there_n = __ballot(ok) >> n & 1;
  const int done = len / p.block, lo = min(p.first, done), hi = max(lo, done - p.recent), words = t.words;
  const int cand = hi - lo, take = there_n ? min(p.top, cand) : 0;
  unsigned* out = p.chosen + row * words;
  unsigned chosen = take == cand ? ~0u : 0u;     // bit j: block j T + tid, if it is a candidate
  if (take > 0 && take < cand) {
    unsigned long long key[N], a = ~0ull, o = 0ull;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int blk = j * T + tid;
      const bool in = blk >= lo && blk < hi;
      key[j] = in ? bound_key(s[j]) : 0ull;      // (0: no candidate's)
      if (in) { a &= key[j]; o |= key[j]; }
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) { a &= __shfl_xor(a, x, 64); o |= __shfl_xor(o, x, 64); }
    if (lane == 0) { and_s[wave] = a; or_s[wave] = o; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < T / 64; ++w) { a &= and_s[w]; o |= or_s[w]; }
    const unsigned long long differ = a ^ o;
    int need = take;                             // of the keys whose upper bits are thr's, so many are chosen
    int top_bit = differ ? 64 - __clzll((long long)differ) : 0;        // bits from here on up are the same in all
    unsigned long long thr = top_bit < 64 ? a >> top_bit << top_bit : 0ull;
    bool whole = false;                          // all of those
    for (int level = 0; top_bit > 0 && !whole; ++level) {
      const int bits = min(8, top_bit), sh = top_bit - bits;
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (key[j] && (top_bit >= 64 || key[j] >> top_bit == thr >> top_bit)) atomicAdd(&hist[level][(key[j] >> sh) & ((1u << bits) - 1)], 1u);
      __syncthreads();
      const u32x4 c = *(const u32x4*)&hist[level][252 - 4 * lane];     // from the largest digit down: the first at which `need` are reached
      const unsigned mine = c[0] + c[1] + c[2] + c[3];
      unsigned upto = mine;
#pragma unroll
      for (int x = 1; x < 64; x <<= 1) { const unsigned v = __shfl_up(upto, x, 64); if (lane >= x) upto += v; }
      unsigned before = upto - mine;
      const int src = __ffsll((long long)__ballot(upto >= (unsigned)need)) - 1;
      int digit = 255 - 4 * lane;
      unsigned left = c[3];
      if (before + left < (unsigned)need) { before += left; left = c[2]; --digit; }
      if (before + left < (unsigned)need) { before += left; left = c[1]; --digit; }
      if (before + left < (unsigned)need) { before += left; left = c[0]; --digit; }
      thr |= (unsigned long long)__builtin_amdgcn_readlane(digit, src) << sh;
      need -= __builtin_amdgcn_readlane((int)before, src);
      top_bit = sh;
      whole = __builtin_amdgcn_readlane((int)left, src) == need;
    }
    if (whole) {                                 // (thr's lower bits are zero)
#pragma unroll
      for (int j = 0; j < N; ++j) chosen |= (unsigned)(key[j] >= thr) << j;
    } else {                                     // ties, of all bits: the lowest blocks
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const mask64 m = __ballot(key[j] == thr);
        if (lane == 0) cnt_s[j][wave] = __popcll(m);
      }
      __syncthreads();
      int before = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const mask64 m = __ballot(key[j] == thr);
        int at = before + __popcll(m & ((1ull << lane) - 1));
        for (int w = 0; w < T / 64; ++w) { const int c = cnt_s[j][w]; if (w < wave) at += c; before += c; }
        chosen |= (unsigned)(key[j] > thr || (key[j] == thr && at < need)) << j;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int blk = j * T + tid;
    const bool pick = there_n && blk < done && (blk < lo || blk >= hi || (chosen >> j & 1));
    const mask64 m = __ballot(pick);
    const int w = (j * T + wave * 64) / 32;
    if (lane < 2 && w + lane < words) out[w + lane] = (unsigned)(m >> (32 * lane));
  }
}

// ------------------------------------------------------------------------------------------------ trees verified

struct AcceptP {
  const int *parent, *token, *expect, *best, *length, *room;
  int *path, *accepted, *next, *new_length;
  int eos, T, B;
  void *K, *V; long layer; int kv, cap;          // K null: no rows to move
};
// The longest path of nodes that p_1 agrees with: from the prefix down, each time the first child of the last accepted node whose token is the one that is wanted there.
// Cut behind the first EOS and at `room`; nodes whose rows are past the cache's end are absent.  By one wave, a node per lane; every workgroup finds it again (some 100 cycles per accepted node, less than a
// second launch), and moves the rows of one layer's (sequence, head) that the path skipped to: read as a whole, then written.
__device__ __forceinline__ int accept_walk(const AcceptP& p, int b, int lane, int& node, int& next) {
  const int T = p.T, par = lane < T ? p.parent[(long)b * T + lane] : -2, tok = lane < T ? p.token[(long)b * T + lane] : 0, bst = lane < T ? p.best[(long)b * T + lane] : 0;
  int want = p.expect[b], cur = -1, n = 0, most = T;
  const int len = p.length[b], there = p.K ? min(T, p.cap - len) : T;
  if (p.room) most = min(most, p.room[b]);
  if (len < 0) most = 0;
  node = -1;
  while (n < most) {
    const mask64 m = __ballot(lane > cur && lane < there && par == cur && tok == want);
    if (!m) break;
    cur = __ffsll((long long)m) - 1;
    if (lane == n) node = cur;
    ++n;
    want = __shfl(bst, cur, 64);
    if (p.eos >= 0 && __shfl(tok, cur, 64) == p.eos) break;
  }
  next = want;
  return n;
}
// Rows len + path_s[m] of one layer's (sequence, head) to len + m, for m < n, sixteen at a time: read, then written.  (Nodes come in order, path_s[m] >= m: what a batch
// writes is read by none that follows, and its barrier stands between its writes and the reads before.)
template <typename S, int D, bool GROUPED>
__device__ __forceinline__ void accept_move(S* K, S* V, int b, int h, int kv, int cap, int len, int n, const int* path_s, int tid) {
  constexpr int M = 16, KP = (M * D / 8 + 255) / 256, VP = M * D / 256;
  if constexpr (GROUPED) { K += ((size_t)b * kv + h) * cap * D; V += ((size_t)b * kv + h) * cap * D; }
  else { const size_t at = ((size_t)b * cap + len) * kv * D + (size_t)h * D; K += at; V += at; }
  for (int m0 = 0; m0 < n; m0 += M) {
    u32x4 k[GROUPED ? KP : 1]; S ke[GROUPED ? 1 : VP], v[VP];
    if constexpr (GROUPED) {
#pragma unroll
      for (int x = 0; x < KP; ++x) {
        const int e = x * 256 + tid, m = m0 + e / (D / 8), c = e % (D / 8) * 8;
        if (e < M * D / 8 && m < n && path_s[m] != m) k[x] = *(const u32x4*)(K + k_at<D>(len + path_s[m], c));
      }
    }
#pragma unroll
    for (int x = 0; x < VP; ++x) {
      const int e = x * 256 + tid, m = m0 + e / D, c = e % D;
      if (m < n && path_s[m] != m) {
        if constexpr (GROUPED) v[x] = V[v_at<D>(len + path_s[m], c)];
        else { const size_t s = (size_t)path_s[m] * kv * D + c; ke[x] = K[s]; v[x] = V[s]; }
      }
    }
    __syncthreads();
    if constexpr (GROUPED) {
#pragma unroll
      for (int x = 0; x < KP; ++x) {
        const int e = x * 256 + tid, m = m0 + e / (D / 8), c = e % (D / 8) * 8;
        if (e < M * D / 8 && m < n && path_s[m] != m) *(u32x4*)(K + k_at<D>(len + m, c)) = k[x];
      }
    }
#pragma unroll
    for (int x = 0; x < VP; ++x) {
      const int e = x * 256 + tid, m = m0 + e / D, c = e % D;
      if (m < n && path_s[m] != m) {
        if constexpr (GROUPED) V[v_at<D>(len + m, c)] = v[x];
        else { const size_t s = (size_t)m * kv * D + c; K[s] = ke[x]; V[s] = v[x]; }
      }
    }
  }
}
template <typename S, int D, bool GROUPED>
__global__ __launch_bounds__(256) void tree_accept_kernel(AcceptP p) {
  __shared__ int path_s[TREE_MAX];
  __shared__ int n_s;
  const int tid = threadIdx.x, lane = tid & 63, h = blockIdx.x, layer = blockIdx.y, b = blockIdx.z;
  const int len = p.length[b];
  if (tid < 64) {
    int node, next;
    const int n = accept_walk(p, b, lane, node, next);
    path_s[lane] = node;
    if (lane == 0) n_s = n;
    if (h == 0 && layer == 0) {
      if (lane < p.T) p.path[(long)b * p.T + lane] = node;
      if (lane == 0) { p.accepted[b] = n; p.next[b] = next; p.new_length[b] = len + n; }
    }
  }
  __syncthreads();
  const int n = n_s;
  if (!p.K || n == 0 || path_s[n - 1] == n - 1) return;          // (nodes come in order: then none has moved)
  accept_move<S, D, GROUPED>((S*)p.K + (size_t)layer * p.layer, (S*)p.V + (size_t)layer * p.layer, b, h, p.kv, p.cap, len, n, path_s, tid);
}
// The same for a path that has been found already: accepted[b] nodes path[b * ld ..], length[b] with them
struct MoveP { const int *path, *accepted, *length; int ld; void *K, *V; long layer; int kv, cap; };
template <typename S, int D, bool GROUPED>
__global__ __launch_bounds__(256) void tree_move_kernel(MoveP p) {
  __shared__ int path_s[TREE_MAX];
  const int tid = threadIdx.x, h = blockIdx.x, layer = blockIdx.y, b = blockIdx.z, n = min(p.accepted[b], p.ld);
  if (tid < n) path_s[tid] = p.path[(long)b * p.ld + tid];
  __syncthreads();
  if (n <= 0 || path_s[n - 1] == n - 1) return;
  accept_move<S, D, GROUPED>((S*)p.K + (size_t)layer * p.layer, (S*)p.V + (size_t)layer * p.layer, b, h, p.kv, p.cap, p.length[b] - n, n, path_s, tid);
}
