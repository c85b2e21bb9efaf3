// Causal attention of new tokens over a paged cache, grouped heads, with an
// optional sliding window and first tokens that stay visible.
//
// attn_pass.h has the passes over the keys; here is who makes them.
//
// k_attn_few: 16 rows at a time (single tokens); bound by reading the cache. A
// wave takes 32 keys at a time by itself, the four waves of a workgroup take
// turns. Caches differ in length, so the workgroups share the tiles of all
// requests evenly, wherever requests begin and end; k_attn_join adds the parts
// of those that more than one had a share in. 64 requests of 200 to 9000
// tokens, 8 heads of 128 in bf16: 238 us, 5.07 TB/s (278 us where each request
// was cut into the same number of parts; reading the same rows alone: 220 us).
// k_attn_many: 128 rows a workgroup (prompts), 64 keys at a time in LDS, the keys
// of few prompts split over workgroups (k_attn_many_join); bound
// by the matrix products and the exponentials between them: three prompts of 1500
// to 4100 tokens over up to 8200, window 2048, 32 heads of 128: 391 us, 722
// TFLOP/s (a library product of 8192^3: 1250), the matrix unit busy 35, the vector
// unit 45, LDS 38 percent of a compute unit's busy cycles.
#include <algorithm>
#include <cmath>

#include "attn_pass.h"

namespace sb {
namespace {

// What the workgroups of k_attn_few leave for k_attn_join. A unit is up to 16
// rows of a request; units are numbered through all requests. Workgroup j's part
// of unit u is number j + u: each step in either is a part of its own.
struct Shares {
  int groups;   // workgroups per key/value head that share the tiles; 0: one per request
  int units;    // most units that there can be if max_q holds; those beyond are not shared
  int parts() const { return groups + units; }
  size_t bytes(const sb_attention_args &a) const {
    return groups == 0 ? 0 : ((size_t)units + 1) * 16 + (size_t)a.kv_heads * parts() * FEW_ROWS * (a.head_dim + 2) * 4;
  }
};
struct UnitInfo {
  int first, count;   // its parts; 1: there is none, its result is there
  int request, r0;
};
// In the workspace: the number of units (in a place of 16 bytes), their infos,
// the parts' sums [kv_heads][parts][16][D], their (maximum, sum) [..][16].
__device__ __forceinline__ UnitInfo *unit_infos(void *work) { return static_cast<UnitInfo *>(work) + 1; }
template <int D>
__device__ __forceinline__ float *part_sums(const sb_attention_args &a, void *work, int groups, int units, int hk, int part) {
  float *p = reinterpret_cast<float *>(static_cast<UnitInfo *>(work) + 1 + units);
  return p + ((size_t)hk * (groups + units) + part) * (FEW_ROWS * D);
}
template <int D>
__device__ __forceinline__ float2 *part_stats(const sb_attention_args &a, void *work, int groups, int units, int hk, int part) {
  return reinterpret_cast<float2 *>(part_sums<D>(a, work, groups, units, a.kv_heads, 0)) + ((size_t)hk * (groups + units) + part) * FEW_ROWS;
}

// Tiles t_begin .. t_end of the span's rows: their result, or, as a share, part
// `part` of it (below 0: the result).
template <int DT, int D>
__device__ __forceinline__ void few_share(const sb_attention_args &a, const Span &s, int b, int hk, int t_begin, int t_end, int part, int groups,
                                          int units, void *work, FewShared<D> &sh) {
  const int G = a.q_heads / a.kv_heads;
  few_unit<DT, D>(a, s, hk, a.table + b * a.table_stride, t_begin, t_end, sh, [&](int rw, int col, float top, float sum, const f4 &acc) {
    if (part < 0) {
      const int qi = rw / G;
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      uint16_t *dst = static_cast<uint16_t *>(a.out) + (s.q0 + qi) * a.out_token + (hk * G + rw - qi * G) * a.out_head + col;
      *reinterpret_cast<u2 *>(dst) = u2{Half<DT>::pack(acc[0] * inv, acc[1] * inv), Half<DT>::pack(acc[2] * inv, acc[3] * inv)};
    } else {
      *reinterpret_cast<f4 *>(part_sums<D>(a, work, groups, units, hk, part) + (rw - s.r0) * D + col) = acc;
      if (col == 0) part_stats<D>(a, work, groups, units, hk, part)[rw - s.r0] = make_float2(top, sum);
    }
  });
}

template <int DT, int D>
__global__ __launch_bounds__(AT_THREADS, few_groups(D)) void k_attn_few(sb_attention_args a, int groups, int units, void *work) {
  __shared__ FewShared<D> sh;
  const int hk = blockIdx.y, j = blockIdx.x;
  Span s;
  if (groups == 0) {   // a request each
    span_request(a, j, s);
    for (int r0 = 0; r0 < s.rows; r0 += FEW_ROWS) {
      span_rows(a, r0, FEW_ROWS, s);
      few_share<DT, D>(a, s, j, hk, 0, few_tiles(s), -1, 0, 0, nullptr, sh);
    }
    return;
  }
  // Units and tiles before each request: every workgroup adds them up, a few
  // neighbouring requests a thread.
  __shared__ long long wave_tiles[AT_WAVES];
  __shared__ int wave_units[AT_WAVES];
  __shared__ long long start_tile;   // of the request that this workgroup's share begins in
  __shared__ int start_request, start_unit;
  if (threadIdx.x == 0) start_request = a.n_requests;
  const int per_thread = (a.n_requests + AT_THREADS - 1) / AT_THREADS, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int b0 = threadIdx.x * per_thread, b1 = min(b0 + per_thread, a.n_requests);
  auto count = [&](int b, int &n, long long &t) {
    span_request(a, b, s);
    n = 0;
    t = 0;
    for (int r0 = 0; r0 < s.rows; r0 += FEW_ROWS) {
      span_rows(a, r0, FEW_ROWS, s);
      t += few_tiles(s);
      ++n;
    }
  };
  int n = 0;
  long long t = 0;
  for (int b = b0; b < b1; ++b) {
    int bn;
    long long bt;
    count(b, bn, bt);
    n += bn;
    t += bt;
  }
  int n_upto = n;
  long long t_upto = t;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(n_upto, o, 64);
    const long long y = __shfl_up(t_upto, o, 64);
    if (lane >= o) {
      n_upto += x;
      t_upto += y;
    }
  }
  if (lane == 63) {
    wave_units[w] = n_upto;
    wave_tiles[w] = t_upto;
  }
  __syncthreads();
  long long all = 0;
  int all_units = 0;
#pragma unroll
  for (int x = 0; x < AT_WAVES; ++x) {
    if (x < w) {
      n_upto += wave_units[x];
      t_upto += wave_tiles[x];
    }
    all += wave_tiles[x];
    all_units += wave_units[x];
  }
  // Shares of a whole number of tiles for each wave.
  auto divide = [&](long long x, long long y) { return all < (1LL << 30) ? (long long)((int)x / (int)y) : x / y; };   // x <= all + groups
  const long long per = (divide(all + groups - 1, groups) + AT_WAVES - 1) & -AT_WAVES;
  const long long begin = j * per, end = min(begin + per, all);
  if (j == 0 && hk == 0 && threadIdx.x == 0) *static_cast<int *>(work) = min(all_units, units);
  if (begin >= end) return;
  if (t_upto - t <= begin && begin < t_upto) {   // (one thread)
    int u = n_upto - n;
    long long at = t_upto - t;
    for (int b = b0; b < b1; ++b) {
      int bn;
      long long bt;
      count(b, bn, bt);
      if (begin < at + bt) {
        start_request = b;
        start_unit = u;
        start_tile = at;
        break;
      }
      u += bn;
      at += bt;
    }
  }
  __syncthreads();
  int u = start_unit;
  long long at = start_tile;   // of the unit's first tile
  for (int b = start_request; b < a.n_requests && at < end; ++b) {
    span_request(a, b, s);
    for (int r0 = 0; r0 < s.rows && at < end; r0 += FEW_ROWS, ++u) {
      span_rows(a, r0, FEW_ROWS, s);
      const int tiles = few_tiles(s);
      const long long next = at + tiles;
      if (next > begin) {
        const int t0 = (int)max(begin - at, 0LL), t1 = u < units ? (int)min(end - at, (long long)tiles) : tiles;
        const bool whole = t0 == 0 && t1 == tiles;
        if (u < units && t0 == 0 && hk == 0 && threadIdx.x == 0)
          unit_infos(work)[u] = UnitInfo{j + u, whole ? 1 : (int)min(divide(next - 1, per), groups - 1LL) - j + 1, b, r0};
        if (u < units || t0 == 0) few_share<DT, D>(a, s, b, hk, t0, t1, whole ? -1 : j + u, groups, units, work, sh);
      }
      at = next;
    }
  }
}

// A wave a row of the unit: every fourth part in each 16 lanes, in order, then the
// four sums. (4 to 5 us, a launch and three reads one after the other; with all
// parts in turn the 128 of one request of 16000 tokens took 15.)
template <int DT, int D>
__global__ __launch_bounds__(AT_THREADS) void k_attn_join(sb_attention_args a, int groups, int units, void *work) {
  constexpr int E = D / 16;
  const int u = blockIdx.x, hk = blockIdx.y, lane = threadIdx.x & 63;
  const int rr = blockIdx.z * AT_WAVES + (threadIdx.x >> 6), col = (lane & 15) * E, turn = lane >> 4;
  if (u >= *static_cast<const int *>(work)) return;
  const UnitInfo info = unit_infos(work)[u];
  if (info.count <= 1) return;
  Span s;
  span_request(a, info.request, s);
  const int G = a.q_heads / a.kv_heads, row = info.r0 + rr, qi = row / G;
  if (row >= s.rows) return;
  const float2 *stats = part_stats<D>(a, work, groups, units, hk, info.first) + rr;
  const float *sums = part_sums<D>(a, work, groups, units, hk, info.first) + rr * D + col;
  float mx = -INFINITY;
#pragma unroll 4
  for (int x = turn; x < info.count; x += 4) mx = fmaxf(mx, stats[x * FEW_ROWS].x);
  mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
  mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
  const float base = mx == -INFINITY ? 0.0f : mx;
  float acc[E], sum = 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.0f;
#pragma unroll 4
  for (int x = turn; x < info.count; x += 4) {
    const float2 st = stats[x * FEW_ROWS];
    const float f = __builtin_amdgcn_exp2f(st.x - base);
    sum += f * st.y;
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const f4 v = *reinterpret_cast<const f4 *>(sums + (size_t)x * (FEW_ROWS * D) + e);
#pragma unroll
      for (int y = 0; y < 4; ++y) acc[e + y] += f * v[y];
    }
  }
#pragma unroll
  for (int o = 16; o < 64; o <<= 1) {
    sum += __shfl_xor(sum, o, 64);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] += __shfl_xor(acc[e], o, 64);
  }
  if (turn != 0) return;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint16_t *dst = static_cast<uint16_t *>(a.out) + (s.q0 + qi) * a.out_token + (hk * G + row - qi * G) * a.out_head + col;
#pragma unroll
  for (int e = 0; e < E; e += 4)
    *reinterpret_cast<u2 *>(dst + e) = u2{Half<DT>::pack(acc[e] * inv, acc[e + 1] * inv), Half<DT>::pack(acc[e + 2] * inv, acc[e + 3] * inv)};
}

// Few long prompts leave units without work: their keys are then split, too, and
// the parts [grid place][key/value head][128][D] added up by k_attn_many_join.
template <int DT, int D>
__global__ __launch_bounds__(AT_THREADS, D == 256 ? 1 : 2) void k_attn_many(sb_attention_args a, int splits, void *work) {
  constexpr int KS = D / 16, DB = D / 32;
  __shared__ ManyShared<D> sh;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l32 = lane & 31, h2 = lane >> 5;
  // Heads side by side: workgroups go to the 8 XCDs in turn, so that tiles of
  // one head, which read the same keys, share an L2.
  const int G = a.q_heads / a.kv_heads, hk = (int)(blockIdx.x % a.kv_heads);
  const int part = (int)((gridDim.x - 1 - blockIdx.x) / a.kv_heads);   // (long prompts' last tiles first)
  Span s;
  const int b = span_tile(a, part / splits, s), r0 = s.r0;
  if (b < 0) return;
  const int *table = a.table + b * a.table_stride;
  const uint16_t *kc = static_cast<const uint16_t *>(a.k_cache) + hk * a.kc_head;
  const uint16_t *vc = static_cast<const uint16_t *>(a.v_cache) + hk * a.vc_head;
  const int row = r0 + 32 * w + l32, i = row / G, p = s.position(i);
  const bool real = row < s.rows;
  // Scores stay as the products give them and are scaled where they go into
  // the exponential, so the scale has to be positive: a negative one turns q's
  // signs, and with 0 all scores are those of q = 0.
  const uint32_t q_sign = a.scale < 0.0f ? 0x80008000u : 0u;
  u4 q[KS];
#pragma unroll
  for (int x = 0; x < KS; ++x) {
    const uint16_t *src = static_cast<const uint16_t *>(a.q) + (s.q0 + i) * a.q_token + (hk * G + row - i * G) * a.q_head;
    q[x] = real && a.scale != 0.0f ? *reinterpret_cast<const u4 *>(src + 16 * x + 8 * h2) ^ q_sign : u4{0, 0, 0, 0};
  }
  f16v o[DB];
  float ref, sum;
  const int tiles = (s.n_vis + MANY_KEYS - 1) / MANY_KEYS, each = (tiles + splits - 1) / splits;
  const int t0 = min(part % splits * each, tiles), count = min(each, tiles - t0);
  if (!many_keys<DT, D, false, false>(a, s, table, kc, vc, q, p, real, t0, count, sh, o, ref, sum))
    many_keys<DT, D, true, false>(a, s, table, kc, vc, q, p, real, t0, count, sh, o, ref, sum);
  sum += __shfl_xor(sum, 32, 64);
  if (!real) return;
  if (splits > 1) {
    const long long at = (long long)part * a.kv_heads + hk;
    float *sums = static_cast<float *>(work) + (at * MANY_ROWS + 32 * w + l32) * D;
    float2 *stats = reinterpret_cast<float2 *>(static_cast<float *>(work) + (long long)gridDim.x * MANY_ROWS * D);
    const float c = a.scale == 0.0f ? 1.0f : (float)(fabs((double)a.scale) * LOG2E);
    if (h2 == 0) stats[at * MANY_ROWS + 32 * w + l32] = make_float2(ref == -INFINITY ? -INFINITY : ref * c, sum);
#pragma unroll
    for (int x = 0; x < DB; ++x)
#pragma unroll
      for (int e = 0; e < 16; e += 4) *reinterpret_cast<f4 *>(sums + 32 * x + 2 * e + 4 * h2) = f4{o[x][e], o[x][e + 1], o[x][e + 2], o[x][e + 3]};
    return;
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint16_t *dst = static_cast<uint16_t *>(a.out) + (s.q0 + i) * a.out_token + (hk * G + row - i * G) * a.out_head;
#pragma unroll
  for (int x = 0; x < DB; ++x)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *reinterpret_cast<u2 *>(dst + 32 * x + 2 * e + 4 * h2) =
          u2{Half<DT>::pack(o[x][e] * inv, o[x][e + 1] * inv), Half<DT>::pack(o[x][e + 2] * inv, o[x][e + 3] * inv)};
}

// 16 rows of a tile, 16 threads each: the parts in order.
template <int DT, int D>
__global__ __launch_bounds__(AT_THREADS) void k_attn_many_join(sb_attention_args a, int splits, const void *work) {
  constexpr int E = D / 16;
  const int tile = blockIdx.x, hk = blockIdx.y, rr = blockIdx.z * 16 + (threadIdx.x >> 4), col = (threadIdx.x & 15) * E;
  Span s;
  const int b = span_tile(a, tile, s);
  if (b < 0) return;
  const int G = a.q_heads / a.kv_heads, row = s.r0 + rr, qi = row / G;
  if (row >= s.rows) return;
  const long long parts = (long long)gridDim.x * splits * a.kv_heads, at = (long long)tile * splits * a.kv_heads + hk;
  const float *sums = static_cast<const float *>(work) + (at * MANY_ROWS + rr) * D + col;
  const float2 *stats = reinterpret_cast<const float2 *>(static_cast<const float *>(work) + parts * MANY_ROWS * D) + at * MANY_ROWS + rr;
  const long long step = (long long)a.kv_heads * MANY_ROWS;
  float mx = -INFINITY;
  for (int x = 0; x < splits; ++x) mx = fmaxf(mx, stats[x * step].x);
  const float base = mx == -INFINITY ? 0.0f : mx;
  float acc[E], sum = 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.0f;
#pragma unroll 4
  for (int x = 0; x < splits; ++x) {
    const float2 st = stats[x * step];
    const float f = __builtin_amdgcn_exp2f(st.x - base);
    sum += f * st.y;
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const f4 v = *reinterpret_cast<const f4 *>(sums + x * step * D + e);
#pragma unroll
      for (int y = 0; y < 4; ++y) acc[e + y] += f * v[y];
    }
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint16_t *dst = static_cast<uint16_t *>(a.out) + (s.q0 + qi) * a.out_token + (hk * G + row - qi * G) * a.out_head + col;
#pragma unroll
  for (int e = 0; e < E; e += 4)
    *reinterpret_cast<u2 *>(dst + e) = u2{Half<DT>::pack(acc[e] * inv, acc[e + 1] * inv), Half<DT>::pack(acc[e + 2] * inv, acc[e + 3] * inv)};
}

// The work that the bounds allow. Keys: that a query sees. Units of 16 rows; tiles
// of 128 rows, and places for them in the grid, for each key/value head.
// k_attn_many splits keys into as many parts as fill the units, of SPLIT_TILES
// tiles at least (8 heads of 128, 4 query heads each; one prompt of 512 tokens
// over 8000: 109 us, in one piece 250; over 1000: 37 and 38; 2048 over 8000, which
// fill the units: 301 and 301).
constexpr int SPLIT_TILES = 8;
struct Load {
  long long G, keys, units, tiles, grid;
  int splits;
  Load(const sb_attention_args &a, int n_cu) : G(a.q_heads / a.kv_heads) {
    const long long rows = std::max(a.max_q, 1) * G, all = a.n_tokens * G;
    keys = std::max(a.max_kv, 1);
    if (a.window > 0) keys = std::min(keys, (long long)a.window + a.sinks + a.max_q);
    units = std::min(all / FEW_ROWS + a.n_requests, (rows + FEW_ROWS - 1) / FEW_ROWS * a.n_requests);
    tiles = std::min(all / MANY_ROWS + a.n_requests, (rows + MANY_ROWS - 1) / MANY_ROWS * a.n_requests);
    grid = all / MANY_ROWS + a.n_requests;
    const long long room = (a.head_dim == 256 ? 1 : 2) * (long long)n_cu;   // workgroups that the units hold at once
    splits = (int)std::max(1LL, std::min({room / (tiles * a.kv_heads), 2 * room / (grid * a.kv_heads), keys / (SPLIT_TILES * MANY_KEYS)}));
  }
  size_t parts_bytes(const sb_attention_args &a) const {
    return splits == 1 ? 0 : (size_t)grid * a.kv_heads * splits * MANY_ROWS * (a.head_dim + 2) * 4;
  }
};

// More than 16 rows of a request read its keys once in k_attn_many, in k_attn_few
// every 16 of them again (16 requests over 3000 keys, 32 rows: 49 and 75 us, 64
// rows: 53 and 133; one request over 8000 keys, 32 rows: 32 and 36).
bool many(const sb_attention_args &a) { return std::max(a.max_q, 1) * (long long)(a.q_heads / a.kv_heads) > FEW_ROWS; }

// How k_attn_few's workgroups share the work: as many per head as the units
// hold at once, fewer where the keys that a query may be expected to see give no
// wave a tile. Requests enough to fill the units SHARE_BELOW times over balance
// themselves, a workgroup each (8 heads of 128; 128 requests of 200 to 6000
// tokens: shared 203 us, not shared 252; 260 of 200 to 4000: 274 and 280; 300 of
// 100 to 1000: 123 and 103; 2000 of 20 to 300: 309 and 266).
// So do short caches: 500 tokens, 1 request of 4 heads: 12.9 and 12.0 us, 100 of
// 8: 45 and 38; 1000 tokens, 1 of 4: 12.6 and 18.8, 8 of 8: 16 and 21.
constexpr int SHARE_BELOW = 4, SHARE_KEYS = 512;
Shares shares(const sb_attention_args &a, const Load &l, int n_cu) {
  const long long places = (long long)few_groups(a.head_dim) * n_cu;
  if ((long long)a.n_requests * a.kv_heads >= SHARE_BELOW * places) return {0, 0};
  if (l.keys <= SHARE_KEYS) return {0, 0};
  const long long tiles = ((l.keys + FEW_KEYS - 1) / FEW_KEYS + 1) * l.units;
  return {(int)std::max(1LL, std::min((places + a.kv_heads - 1) / a.kv_heads, (tiles + AT_WAVES - 1) / AT_WAVES)), (int)l.units};
}

template <int DT, int D>
hipError_t launch(const sb_attention_args &a, int n_cu, void *work, hipStream_t s) {
  const Load l(a, n_cu);
  if (many(a)) {
    hipLaunchKernelGGL((k_attn_many<DT, D>), dim3((unsigned)(l.grid * a.kv_heads * l.splits)), dim3(AT_THREADS), 0, s, a, l.splits, work);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || l.splits == 1) return e;
    hipLaunchKernelGGL((k_attn_many_join<DT, D>), dim3((unsigned)l.grid, a.kv_heads, MANY_ROWS / 16), dim3(AT_THREADS), 0, s, a, l.splits, work);
    return hipGetLastError();
  }
  const Shares sh = shares(a, l, n_cu);
  hipLaunchKernelGGL((k_attn_few<DT, D>), dim3(sh.groups ? sh.groups : a.n_requests, a.kv_heads), dim3(AT_THREADS), 0, s, a, sh.groups, sh.units,
                     work);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || sh.groups <= 1) return e;
  hipLaunchKernelGGL((k_attn_join<DT, D>), dim3(sh.units, a.kv_heads, FEW_ROWS / AT_WAVES), dim3(AT_THREADS), 0, s, a, sh.groups, sh.units, work);
  return hipGetLastError();
}

}  // namespace

int64_t attention_workspace(const sb_attention_args &a, int n_cu) {
  const Load l(a, n_cu);
  return (int64_t)(many(a) ? l.parts_bytes(a) : shares(a, l, n_cu).bytes(a));
}

hipError_t launch_paged_attention(const sb_attention_args &a, int n_cu, void *work, hipStream_t s) {
  if (a.dtype == SB_BF16) {
    if (a.head_dim == 64) return launch<SB_BF16, 64>(a, n_cu, work, s);
    if (a.head_dim == 128) return launch<SB_BF16, 128>(a, n_cu, work, s);
    return launch<SB_BF16, 256>(a, n_cu, work, s);
  }
  if (a.head_dim == 64) return launch<SB_F16, 64>(a, n_cu, work, s);
  if (a.head_dim == 128) return launch<SB_F16, 128>(a, n_cu, work, s);
  return launch<SB_F16, 256>(a, n_cu, work, s);
}

}  // namespace sb
