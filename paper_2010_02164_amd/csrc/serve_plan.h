// Which kernels a call of the serving operators gets: rules on sizes alone, so
// that they can be asked without a GPU.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "../../include/streambeam.h"

namespace sb {

// -- products in 8-bit integers ---------------------------------------------------

constexpr int FEW_WAVES = 8, FEW_STEP = 64;   // of k_linear_few: waves, and values of the depth in a piece
constexpr int TILE_K = 128;                   // of k_linear_tiles: values of the depth in a step

// How a product is cut up: by few rows, or by tiles, whose depth is split where they
// leave units without work. Times in microseconds, as measured: what a step of 128
// of the depth takes (a tile of 256 x 256: 2; of 128 x 128: 0.75, two in a unit 1.3),
// a launch and its ends 4, a join 4 and its bytes at 4 TB/s; few rows: 4 pieces of a
// wave 3.3 (up to 32 rows) or 5.2.
struct LinearPlan {
  int tile;   // 0: few rows
  int m, n, splits;
};
inline LinearPlan linear_plan(const sb_linear_args &a, int n_cu) {
  if (a.rows <= 16) return {0, 0, 0, 1};
  const auto up = [](long long x, long long y) { return (int)((x + y - 1) / y); };
  const int steps = up(a.depth, TILE_K), m = up(a.rows, 128), n = up(a.channels, 128);
  const double tiles = (double)m * n;
  LinearPlan best = {128, m, n, 1};
  double least = 1e30;
  for (int s = 1; s <= 16 && (s == 1 || steps >= 4 * s); ++s) {
    const double groups = tiles * s, step = groups <= n_cu ? 0.75 : 1.3 * std::ceil(groups / (2 * n_cu));
    const double time = 4 + up(steps, s) * step + (s > 1 ? 4 + groups * 128 * 128 * 8 / 4e6 : 0);
    if (time < least) {
      least = time;
      best.splits = up(steps, up(steps, s));   // (none without a step)
    }
  }
  const int m2 = up(a.rows, 256), n2 = up(a.channels, 256);
  if (4 + steps * 2.0 * std::ceil((double)m2 * n2 / n_cu) < least) best = {256, m2, n2, 1};
  if (a.rows <= 64) {
    const double batches = up(up(a.depth, FEW_STEP), 4 * FEW_WAVES), rounds = std::ceil((double)up(a.channels, 32) / n_cu);
    if (3.5 + rounds * batches * (a.rows <= 32 ? 3.3 : 5.2) < least) best = {0, 0, 0, 1};
  }
  return best;
}

// -- attention over a shared prefix --------------------------------------------------

// Kinds of a pass: 1 and 2, 16 and 32 rows by waves that take 32 keys each; MANY,
// 128 rows by workgroups that take 64. They go by the rows that read the same keys.
constexpr int MANY = 8;
struct SharedKinds {
  int prefix, own;
};
inline SharedKinds shared_kinds(const sb_shared_args &x) {
  constexpr int FEW = 16;
  const sb_attention_args &a = x.own;
  const long long G = a.q_heads / a.kv_heads, group_rows = (a.n_tokens * G + x.n_groups - 1) / x.n_groups, request_rows = std::max(a.max_q, 1) * G;
  const int own = request_rows <= FEW ? 1 : request_rows <= 4 * FEW ? 2 : MANY;
  const int prefix = group_rows <= FEW ? 1 : group_rows <= 2 * FEW ? 2 : MANY;
  return {own == MANY ? MANY : std::max(prefix, own), own};
}

// -- selection of pages -------------------------------------------------------------

// Whether scores are made 16 tokens at a time by the matrix unit, by how many tokens a
// request has on average. Scores and lists in us, a token at a time and 16, at 1, 4, 8
// and 16 tokens a request: 12 requests of 5000 to 50000 tokens, pages of 16, 8 heads of
// 128: 35 and 91, 64 and 85, 98 and 78, 172 and 92; 12 of 20000 to 120000, pages of 64,
// 4 of 64: 28 and 51, 38 and 38, 46 and 38, 67 and 50; 48 of 2000 to 20000, pages of 32,
// 8 of 128: 35 and 84, 65 and 71, 127 and 75, 234 and 91; one of 20000, pages of 16, 4
// of 128: 17 and 22, 19 and 23, 21 and 24, 24 and 25. (One prompt of 300 among 15
// single tokens, 20 on average: 154 and 332.)
inline bool many_scores(const sb_select_args &a) { return a.n_tokens >= 8LL * a.n_requests; }

// Pages that are ranked, as max_kv lets expect.
inline long long pages_between(const sb_select_args &a) {
  return std::max(1LL, (std::max(a.max_kv, 1) + a.page_size - 1LL) / a.page_size - a.first - a.last);
}

// k_pick's threads a list, and the pages that each of them keeps in registers. (Of
// 1250 pages, 4 lists: 256 threads 9.9 us, 1024 8.5; of up to 3125, 384 lists: 15.0
// and 16.9.)
struct PickPlan {
  int threads, per;
};
inline PickPlan pick_plan(long long between, long long lists, int n_cu) {
  if (between <= 1024) return {256, 4};
  if (between <= 4096 && lists >= n_cu) return {256, 16};
  return {1024, between <= 4096 ? 4 : 16};
}

}  // namespace sb
