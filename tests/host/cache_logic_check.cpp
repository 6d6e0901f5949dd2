// Launch plans of the cache operators (csrc/bpd_cache_logic.h) on random sizes: parts, row blocks and workspace regions cover what the kernels write, and nothing overflows.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "../../paper_1811_03115_amd/csrc/bpd_cache_logic.h"

#define CHECK(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); return 1; } } while (0)

int main() {
  std::mt19937_64 rng(1811);
  auto log_to = [&](double most) { return (int)std::exp(std::uniform_real_distribution<>(0, std::log(most + 0.99))(rng)); };
  for (int n = 0; n < 20000; ++n) {
    bpd_cache c{(void*)64, (void*)64, (int)(rng() % 2), log_to(40), log_to(300), log_to(64), (int[]){16, 64, 128}[rng() % 3], log_to(200000)};
    if (cache_grouped(c)) c.capacity = (c.capacity + 31) / 32 * 32;
    CHECK(!cache_wrong(&c));
    const int B = 1 + (int)(rng() % c.max_batch), T = log_to(64), G = log_to(64), heads = G * c.n_kv_heads, R = T * G, block = (int[]){0, 32, 64, 128}[rng() % 4];
    if (block && c.capacity / block > BPD_BLOCKS_MAX) continue;
    const int cus = rng() % 8 ? 256 : log_to(304);
    const TreePlan p = plan_attention(c, B, T, heads, block, cus);
    const int per = p.rows ? 64 * p.mt : (cache_grouped(c) ? 16 * p.mt : 16);
    CHECK(p.nsplit >= 1 && p.nsplit <= 64 && (p.nsplit == 1 || p.nsplit * 4 <= (c.capacity + 31) / 32));
    CHECK((long)p.blocks * per >= R && (long)(p.blocks - 1) * per < R);
    CHECK(p.rows || !cache_grouped(c) || p.blocks == 1);          // (the kernel that has all of a pair's rows)
    CHECK(!p.rows || p.mt == 1 || p.mt == 2);
    CHECK(p.rows || !cache_grouped(c) || p.mt <= (c.head_dim == 64 ? 3 : 1));
    size_t parts = p.nsplit > 1 ? (size_t)B * c.n_kv_heads * p.nsplit * R * (c.head_dim + 2) * 4 : 0, end = parts;
    if (block && c.capacity / block) {
      const size_t nb = c.capacity / block, rows = (size_t)B * c.n_kv_heads * T;
      CHECK(p.chosen_at >= parts && p.chosen_at % 256 == 0 && p.score_at % 256 == 0);
      CHECK(p.score_at >= p.chosen_at + rows * ((nb + 31) / 32) * 4);
      end = p.score_at + rows * ((nb + 63) / 64) * 64 * 8;
      CHECK((nb + 31) / 32 <= 128);                               // (a thread of the list per word)
    }
    CHECK(p.bytes >= end);
    // chosen blocks: as many parts as the fewer keys want, and no more than there is room for
    if (block) CHECK(split_of(p, (long)B * c.n_kv_heads * p.blocks, 1 + (long)(rng() % 64), cache_grouped(c), cus) <= 16);
  }
  std::printf("ok\n");
  return 0;
}
