// Attention over a prefix that the requests of a group share, and over each
// request's own tokens behind it, in the paged cache.
//
// The queries of a group's requests are neighbours, so they are the rows of one
// pass over the prefix, as a request's are over its own keys (attn_pass.h), but
// that every row sees every key. k_shared makes both passes. Each unit of rows is
// cut into pieces of its keys, a piece a workgroup (a workgroup that takes the end
// of one unit and the start of the next waits for the memory twice: 10 to 20 us more
// in small calls); a piece leaves a part: the rows' sums, and the reference and sum
// of their weights. k_shared_join adds a row's parts up.
#include <algorithm>

#include "attn_pass.h"
#include "serve_plan.h"

namespace sb {
namespace {

struct Prefix {
  const int *table, *lens, *group_start;
  long long stride;
  int n_groups, pages;
};

// A unit is up to `rows` rows of an item (a group, a request). Units have places:
// those of an item start at (its first token) G / rows + the item's number, which
// leaves at least one place each.
//
// The prefixes are few and long: every workgroup adds up their tiles, so that the
// pieces fill the card evenly; workgroup j's is part j, and a unit's first part and
// their count are its info. The requests' own tokens are many and short: a unit
// has `splits` workgroups, for `tiles` of its tiles each, or for more where they are
// too few; part u splits + x is that of piece x of the unit at place u.
struct Pass {
  int places, rows;
  int fill;             // prefixes: workgroups per key/value head that the card holds
  int splits, tiles;    // own
  // Pieces there can be, per head: of the prefixes at most one a unit more than the
  // tiles fill (see run_prefix).
  __host__ __device__ int groups() const { return fill > 0 ? max(fill, places + (fill + 1) / 2) + 1 : places * splits; }
  // Tiles of a piece of an own unit, and the number of its pieces.
  __device__ __forceinline__ int piece(int n, int round) const { return (max(tiles, (n + splits - 1) / splits) + round - 1) & -round; }
};
struct Cut {
  Pass prefix, own;
  bool own_first;   // in the grid
};

struct Info {
  int first, count;   // a unit's parts
};
struct Ahead {
  int group, token;   // a request's group (-1: none) and its first token
};

// In the workspace: both passes' parts, sums [kv_heads][groups][rows][D] and
// (reference, sum) [kv_heads][groups][rows], the prefixes' units' infos, and what
// is ahead of each request.
struct Parts {
  float *sums[2];
  float2 *stats[2];
  Info *infos;
  Ahead *ahead;
  __host__ __device__ Parts(const sb_attention_args &a, const Cut &c, void *work) {
    const long long n0 = a.kv_heads * (long long)c.prefix.groups() * c.prefix.rows, n1 = a.kv_heads * (long long)c.own.groups() * c.own.rows;
    sums[0] = static_cast<float *>(work);
    sums[1] = sums[0] + n0 * a.head_dim;
    stats[0] = reinterpret_cast<float2 *>(sums[1] + n1 * a.head_dim);
    stats[1] = stats[0] + n0;
    infos = reinterpret_cast<Info *>(stats[1] + n1);
    ahead = reinterpret_cast<Ahead *>(infos + c.prefix.places);
  }
};

__device__ __forceinline__ int group_token(const sb_attention_args &a, const Prefix &p, int g) {
  return min(max(a.q_start[min(max(p.group_start[g], 0), a.n_requests)], 0), a.n_tokens);
}

// Group g's queries as rows over its prefix.
__device__ __forceinline__ void span_group(const sb_attention_args &a, const Prefix &p, int g, Span &s) {
  s.q0 = group_token(a, p, g);
  s.m = max(group_token(a, p, g + 1) - s.q0, 0);
  s.n = s.n_vis = (int)min((long long)max(p.lens[g], 0), (long long)p.pages * a.page_size);
  s.rows = s.m * (a.q_heads / a.kv_heads);
  s.all = true;
  s.ns = s.lo = 0;
  s.p_first = s.p_last = s.n - 1;
}

__host__ __device__ constexpr int rows_of(int kind) { return kind == MANY ? MANY_ROWS : FEW_ROWS * kind; }

template <int D, int KIND>
struct PassShared {
  FewShared<D, KIND> x;
};
template <int D>
struct PassShared<D, MANY> {
  ManyShared<D> x;
};
template <int D, int P, int O>
union SharedLds {
  PassShared<D, P> prefix;
  PassShared<D, O> own;
};

// What a workgroup looks its piece up with.
struct Scan {
  unsigned long long tiles[AT_WAVES];
  unsigned units[AT_WAVES], pieces[AT_WAVES], at;
  int item;
};

// 128 rows by a workgroup. (Each weight in two parts, as by waves, so that what a
// request gets does not go by how many others there are: 64 requests behind 8000
// tokens take 79 to 82 us for 76, 120 behind two of 24000 and 33000 484 to 500 for 444.)
template <int DT, int D>
__device__ __forceinline__ void part_many(const sb_attention_args &a, const Span &s, int hk, const int *table, int t0, int count, float *sums,
                                          float2 *stats, ManyShared<D> &sh) {
  constexpr int KS = D / 16, DB = D / 32;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l32 = lane & 31, h2 = lane >> 5, G = a.q_heads / a.kv_heads;
  const uint16_t *kc = static_cast<const uint16_t *>(a.k_cache) + hk * a.kc_head;
  const uint16_t *vc = static_cast<const uint16_t *>(a.v_cache) + hk * a.vc_head;
  const int row = s.r0 + 32 * w + l32, i = row / G, p = s.position(i);
  const bool real = row < s.rows;
  // (A negative scale turns q's signs, with 0 all scores are those of q = 0.)
  const uint32_t q_sign = a.scale < 0.0f ? 0x80008000u : 0u;
  u4 q[KS];
#pragma unroll
  for (int x = 0; x < KS; ++x) {
    const uint16_t *src = static_cast<const uint16_t *>(a.q) + (s.q0 + i) * a.q_token + (hk * G + row - i * G) * a.q_head;
    q[x] = real && a.scale != 0.0f ? *reinterpret_cast<const u4 *>(src + 16 * x + 8 * h2) ^ q_sign : u4{0, 0, 0, 0};
  }
  f16v o[DB];
  float ref, sum;
  if (!many_keys<DT, D, false, true>(a, s, table, kc, vc, q, p, real, t0, count, sh, o, ref, sum))
    many_keys<DT, D, true, true>(a, s, table, kc, vc, q, p, real, t0, count, sh, o, ref, sum);
  sum += __shfl_xor(sum, 32, 64);
  if (!real) return;
  const int at = 32 * w + l32;
  if (h2 == 0) stats[at] = make_float2(many_reference<DT>(a, ref), sum);
  sums += at * D;
#pragma unroll
  for (int x = 0; x < DB; ++x)
#pragma unroll
    for (int e = 0; e < 16; e += 4) *reinterpret_cast<f4 *>(sums + 32 * x + 2 * e + 4 * h2) = f4{o[x][e], o[x][e + 1], o[x][e + 2], o[x][e + 3]};
}

__device__ __forceinline__ unsigned scan_up(unsigned v) {   // of the lanes up to this one
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned y = __shfl_up(v, o, 64);
    if ((int)(threadIdx.x & 63) >= o) v += y;
  }
  return v;
}

// A unit's tiles (one where it sees nothing: somebody has to say so).
constexpr int keys_of(int kind) { return kind == MANY ? MANY_KEYS : FEW_KEYS; }
constexpr int round_of(int kind) { return kind == MANY ? 1 : AT_WAVES; }   // tiles that a workgroup takes at once
constexpr int least_of(int kind) { return kind == MANY ? 8 : AT_WAVES; }   // of a piece
template <int KIND>
__device__ __forceinline__ int tiles_of(const Span &s) { return max((s.n_vis + keys_of(KIND) - 1) / keys_of(KIND), 1); }

// Tiles t0 .. t1 of the span's rows, as part `part` of a pass.
template <int DT, int D, int KIND>
__device__ __forceinline__ void run_piece(const sb_attention_args &a, const Span &s, const Pass &pass, float *sums, float2 *stats, int hk,
                                          const int *table, int t0, int t1, int part, PassShared<D, KIND> &sh) {
  const long long base = ((long long)hk * pass.groups() + part) * rows_of(KIND);
  sums += base * D;
  stats += base;
  if constexpr (KIND == MANY) {
    part_many<DT, D>(a, s, hk, table, t0, max(min(t1, (s.n_vis + MANY_KEYS - 1) / MANY_KEYS) - t0, 0), sums, stats, sh.x);
  } else {
    few_unit<DT, D, KIND>(a, s, hk, table, t0, t1, sh.x, [&](int rw, int col, float top, float sum, const f4 &acc) {
      *reinterpret_cast<f4 *>(sums + (rw - s.r0) * D + col) = acc;
      if (col == 0) stats[rw - s.r0] = make_float2(top - raise<DT>(0), sum);
    });
  }
}

// Workgroup j's piece of the prefixes.
template <int DT, int D, int KIND>
__device__ __forceinline__ void run_prefix(const sb_attention_args &a, const Prefix &p, const Pass &pass, const Parts &out, int hk, int j,
                                           PassShared<D, KIND> &sh, Scan &scan) {
  constexpr int ROWS = rows_of(KIND), ROUND = round_of(KIND), LEAST = least_of(KIND);
  const int G = a.q_heads / a.kv_heads, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  Span s;
  // A group's units, which are alike, and the tiles of one, whole rounds.
  const auto units_of = [&](int g, int &n, int &t) {
    span_group(a, p, g, s);
    n = (s.rows + ROWS - 1) / ROWS;
    t = (tiles_of<KIND>(s) + ROUND - 1) & -ROUND;
  };
  const int per_thread = (p.n_groups + AT_THREADS - 1) / AT_THREADS, g0 = threadIdx.x * per_thread, g1 = min(g0 + per_thread, p.n_groups);
  // (Groups that lie over each other have any number of units, and counts may pass
  // 2^32: a unit that its group does not have is left out at the end.)
  unsigned long long tiles = 0;
  unsigned units = 0;
  int n = 0, t = 0;   // (of the last group looked at: the only one, nearly always)
  for (int g = g0; g < g1; ++g) {
    units_of(g, n, t);
    tiles += (unsigned long long)t * n;
    units += n;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    tiles += __shfl_xor(tiles, o, 64);
    units += __shfl_xor(units, o, 64);
  }
  if (lane == 0) {
    scan.tiles[w] = tiles;
    scan.units[w] = units;
  }
  if (threadIdx.x == 0) scan.item = -1;
  __syncthreads();
  tiles = 0;
  units = 0;
#pragma unroll
  for (int x = 0; x < AT_WAVES; ++x) {
    tiles += scan.tiles[x];
    units += scan.units[x];
  }
  // Tiles of a piece: every unit may leave one that is not full, so that there are at
  // most `room` and the units pieces. (fp32's rounding makes less than the one
  // workgroup more that there is.)
  const int half = (pass.fill + 1) / 2, room = units < (unsigned)pass.fill ? max(pass.fill - (int)units, half) : half;
  const float want = (float)tiles / (float)room;
  const int per = ((want < 1e9f ? max((int)ceilf(want), LEAST) : 1 << 30) + ROUND - 1) & -ROUND;
  const auto pieces_of = [&](int t) { return (t + per - 1) / per; };
  unsigned mine = 0;
  for (int g = g0; g < g1; ++g) {
    if (per_thread > 1) units_of(g, n, t);
    mine += (unsigned)pieces_of(t) * n;
  }
  unsigned upto = scan_up(mine);
  if (lane == 63) scan.pieces[w] = upto;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < AT_WAVES; ++x)
    if (x < w) upto += scan.pieces[x];
  unsigned rest = j - (upto - mine);
  if (rest < mine) {   // (one thread)
    for (int g = g0; g < g1; ++g) {
      if (per_thread > 1) units_of(g, n, t);
      const unsigned here = (unsigned)pieces_of(t) * n;
      if (rest < here) {
        scan.item = g;
        scan.at = rest;
        break;
      }
      rest -= here;
    }
  }
  __syncthreads();
  const int g = scan.item;
  if (g < 0) return;
  units_of(g, n, t);
  const int pieces = pieces_of(t), unit = (int)(scan.at / (unsigned)pieces), x = (int)(scan.at - (unsigned)(unit * pieces));
  if (unit >= n) return;
  s.r0 = unit * ROWS;
  if (x == 0 && hk == 0 && threadIdx.x == 0) out.infos[(int)((long long)s.q0 * G / ROWS) + g + unit] = Info{j, pieces};
  run_piece<DT, D, KIND>(a, s, pass, out.sums[0], out.stats[0], hk, p.table + g * p.stride, x * per, min(x * per + per, t), j, sh);
}

// Piece x of the own units at place `place` (by waves: of a request, whose units take
// turns).
template <int DT, int D, int KIND>
__device__ __forceinline__ void run_own(const sb_attention_args &a, const Prefix &p, const Pass &pass, const Parts &out, int hk, int place, int x,
                                        PassShared<D, KIND> &sh) {
  constexpr int ROWS = rows_of(KIND), ROUND = round_of(KIND);
  const int G = a.q_heads / a.kv_heads;
  Span s;
  int b = place;
  if constexpr (KIND == MANY) b = span_tile(a, place, s);
  else span_request(a, b, s);
  if (b < 0) return;
  const int *table = a.table + b * a.table_stride;
  const int r_first = KIND == MANY ? s.r0 : 0, r_end = KIND == MANY ? min(s.r0 + 1, s.rows) : s.rows;
  for (int r0 = r_first; r0 < r_end; r0 += ROWS) {
    span_rows(a, r0, ROWS, s);
    const int tiles = tiles_of<KIND>(s), per = pass.piece(tiles, ROUND), u = (int)((long long)s.q0 * G / ROWS) + b + r0 / ROWS;
    if (x * per < tiles)
      run_piece<DT, D, KIND>(a, s, pass, out.sums[1], out.stats[1], hk, table, x * per, min(x * per + per, tiles), u * pass.splits + x, sh);
  }
  if (x == 0 && r_first == 0 && hk == 0) {   // what is ahead of the request?
    int found = 0;
    for (int g = threadIdx.x; g < p.n_groups; g += AT_THREADS) {
      if (min(max(p.group_start[g], 0), a.n_requests) <= b && b < min(max(p.group_start[g + 1], 0), a.n_requests)) {
        out.ahead[b] = Ahead{g, group_token(a, p, g)};
        found = 1;
      }
    }
    if (!__syncthreads_or(found) && threadIdx.x == 0) out.ahead[b] = Ahead{-1, 0};
  }
}

// Workgroups of one pass, then those of the other; of each the key/value heads side
// by side, so that those of one head, which read the same keys, share an XCD's L2. Both
// passes in one kernel take the registers and the LDS of the larger one: at heads of 128
// a pass of 128 rows lets two workgroups into a compute unit, and 61 (with 16 own rows),
// 100 (32) and 173 (128) registers are spilled, 40 with two passes of 32.
template <int DT, int D, int P, int O>
__global__ __launch_bounds__(AT_THREADS, D == 256 ? 1 : 2) void k_shared(sb_attention_args a, Prefix p, Cut c, void *work) {
  __shared__ SharedLds<D, P, O> sh;
  __shared__ Scan scan;
  const Parts out(a, c, work);
  const int hk = (int)(blockIdx.x % a.kv_heads), j = (int)(blockIdx.x / a.kv_heads);
  const int prefixes = c.prefix.groups(), own = (int)(gridDim.x / a.kv_heads) - prefixes;
  const bool is_own = c.own_first ? j < own : j >= prefixes;
  if (is_own) {
    const int y = c.own_first ? j : j - prefixes;
    run_own<DT, D, O>(a, p, c.own, out, hk, y / c.own.splits, y % c.own.splits, sh.own);
  } else {
    run_prefix<DT, D, P>(a, p, c.prefix, out, hk, c.own_first ? j - own : j, sh.prefix, scan);
  }
}

// A wave a row.
template <int DT, int D, int O>
__global__ __launch_bounds__(AT_THREADS) void k_shared_join(sb_attention_args a, Prefix p, Cut c, void *work) {
  const Parts in(a, c, work);
  const int b = blockIdx.x, G = a.q_heads / a.kv_heads;
  Span s;
  span_request(a, b, s);
  if (s.m == 0) return;
  const Ahead ahead = in.ahead[b];
  const int pr = c.prefix.rows;
  constexpr int ROWS = rows_of(O);
  const long long rows = (long long)s.m * a.q_heads, step = (long long)gridDim.y * AT_WAVES;
  const long long gap = (long long)a.kv_heads * c.prefix.groups() * pr;   // the own parts' rows stand behind the prefixes'
  for (long long r = (long long)blockIdx.y * AT_WAVES + (threadIdx.x >> 6); r < rows; r += step) {
    const int i = (int)(r / a.q_heads), h = (int)(r - (long long)i * a.q_heads), hk = h / G, g = h - hk * G, orow = i * G + g;
    span_rows(a, orow & -ROWS, ROWS, s);
    const int tiles = tiles_of<O>(s), per = c.own.piece(tiles, round_of(O)), own = (tiles + per - 1) / per;
    const long long u = (long long)s.q0 * G / ROWS + b + orow / ROWS;
    // (Wrong state may have left anything: no part outside those there are.)
    const long long prow = ((long long)s.q0 + i - ahead.token) * G + g;
    const bool follows = (unsigned)ahead.group < (unsigned)p.n_groups && ahead.token >= 0 && prow >= 0;
    const long long pu = follows ? (long long)ahead.token * G / pr + ahead.group + prow / pr : 0;
    Info f = follows && pu < c.prefix.places ? in.infos[pu] : Info{0, 0};
    f.first = min(max(f.first, 0), c.prefix.groups());
    f.count = min(max(f.count, 0), c.prefix.groups() - f.first);
    const long long at0 = ((long long)hk * c.prefix.groups() + f.first) * pr + (follows ? prow % pr : 0);
    const long long at1 = gap + ((long long)hk * c.own.groups() + u * c.own.splits) * ROWS + orow % ROWS;
    join_row<DT, D>(in.sums[0], in.stats[0], f.count + own, [&](int x) { return x < f.count ? at0 + (long long)x * pr : at1 + (long long)(x - f.count) * ROWS; },
                    static_cast<uint16_t *>(a.out) + (s.q0 + i) * a.out_token + h * a.out_head);
  }
}

Cut cut(const sb_shared_args &x, int n_cu) {
  const sb_attention_args &a = x.own;
  const SharedKinds k = shared_kinds(x);
  const long long G = a.q_heads / a.kv_heads, all = a.n_tokens * G, room = (a.head_dim == 256 ? 1 : 2) * (long long)n_cu;
  Cut c = {};
  {   // workgroups: as many as the units hold at once, fewer where the bounds let expect no more tiles
    const int rows = rows_of(k.prefix);
    const long long item_rows = (all + x.n_groups - 1) / x.n_groups, places = all / rows + x.n_groups;
    const long long units = std::min(places, (item_rows + rows - 1) / rows * x.n_groups);
    const long long tiles = units * std::max((x.max_prefix + keys_of(k.prefix) - 1LL) / keys_of(k.prefix), 1LL);
    c.prefix.places = (int)places;
    c.prefix.rows = rows;
    c.prefix.fill = (int)std::max(1LL, std::min((room + a.kv_heads - 1) / a.kv_heads, tiles));
    // Prefixes that do not fill the card come behind the own tokens and fill up what
    // those leave (64 requests of 20 to 1500 tokens behind one of 8000: 87 to 80 us);
    // long ones come first (120 behind two of 24000 and 33000: 420, else 508).
    c.own_first = tiles <= c.prefix.fill * (long long)least_of(k.prefix);
  }
  {   // pieces of one round at least; few requests are cut up until they fill the units (every workgroup more costs: 12 us for 1000)
    const int rows = rows_of(k.own), round = round_of(k.own), least = k.own == MANY ? 6 : round;
    const long long places = k.own == MANY ? all / rows + a.n_requests : a.n_requests;
    const long long tiles = std::max((a.max_kv + keys_of(k.own) - 1LL) / keys_of(k.own), 1LL);
    const long long piece = std::max((long long)least, places * a.kv_heads * tiles / room);
    c.own.places = (int)(all / rows + a.n_requests);
    c.own.rows = rows;
    c.own.tiles = (int)std::min((piece + round - 1) / round * round, 1LL << 24);
    c.own.splits = (int)((tiles + c.own.tiles - 1) / c.own.tiles);
  }
  return c;
}

template <int DT, int D>
hipError_t launch(const sb_shared_args &x, int n_cu, void *work, hipStream_t s) {
  const sb_attention_args &a = x.own;
  const Cut c = cut(x, n_cu);
  const SharedKinds k = shared_kinds(x);
  const Prefix p = {x.prefix_table, x.prefix_lens, x.group_start, x.prefix_stride, x.n_groups, x.prefix_pages};
  const long long own = (k.own == MANY ? c.own.places : a.n_requests) * (long long)c.own.splits;
  const dim3 grid((unsigned)((c.prefix.groups() + own) * a.kv_heads));
  const dim3 rows((unsigned)a.n_requests, (unsigned)std::min(((long long)std::max(a.max_q, 1) * a.q_heads + AT_WAVES - 1) / AT_WAVES, 1024LL));
  const auto run = [&](auto kernel, auto join) {
    hipLaunchKernelGGL(kernel, grid, dim3(AT_THREADS), 0, s, a, p, c, work);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(join, rows, dim3(AT_THREADS), 0, s, a, p, c, work);
    return hipGetLastError();
  };
  if (k.own == MANY) return run(k_shared<DT, D, MANY, MANY>, k_shared_join<DT, D, MANY>);
  if (k.own == 2) return k.prefix == 2 ? run(k_shared<DT, D, 2, 2>, k_shared_join<DT, D, 2>) : run(k_shared<DT, D, MANY, 2>, k_shared_join<DT, D, 2>);
  return k.prefix == 1 ? run(k_shared<DT, D, 1, 1>, k_shared_join<DT, D, 1>)
                       : k.prefix == 2 ? run(k_shared<DT, D, 2, 1>, k_shared_join<DT, D, 1>) : run(k_shared<DT, D, MANY, 1>, k_shared_join<DT, D, 1>);
}

}  // namespace

int64_t shared_workspace(const sb_shared_args &x, int n_cu) {
  const Parts end(x.own, cut(x, n_cu), nullptr);
  return (int64_t)(reinterpret_cast<uintptr_t>(end.ahead) + sizeof(Ahead) * (uintptr_t)x.own.n_requests);
}

hipError_t launch_shared_attention(const sb_shared_args &x, int n_cu, void *work, hipStream_t s) {
  if (x.own.dtype == SB_BF16) {
    if (x.own.head_dim == 64) return launch<SB_BF16, 64>(x, n_cu, work, s);
    if (x.own.head_dim == 128) return launch<SB_BF16, 128>(x, n_cu, work, s);
    return launch<SB_BF16, 256>(x, n_cu, work, s);
  }
  if (x.own.head_dim == 64) return launch<SB_F16, 64>(x, n_cu, work, s);
  if (x.own.head_dim == 128) return launch<SB_F16, 128>(x, n_cu, work, s);
  return launch<SB_F16, 256>(x, n_cu, work, s);
}

}  // namespace sb
