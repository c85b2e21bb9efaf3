// Attention over a prefix that the requests of a group share, and over each
// request's own tokens behind it, in the paged cache.
//
// The queries of a group's requests are neighbours, so they are the rows of one
// pass over the prefix, as a request's are over its own keys (attn_pass.h), but
// that every row sees every key. k_shared makes both kinds of pass, over splits of
// the keys where the units would be left without work; each leaves a part: the
// rows' sums, and the reference and sum of their weights. k_shared_join adds a
// row's parts up.
#include <algorithm>

#include "attn_pass.h"

namespace sb {
namespace {

struct Prefix {
  const int *table, *lens, *group_start;
  long long stride;
  int n_groups, pages;
};

// How the passes are cut up. Places: of a tile of rows in the grid.
struct Cut {
  bool prefix_many, own_many;   // 128 rows a workgroup, not 16
  int prefix_places, own_places;
  int prefix_splits, own_splits;
};

// In the workspace: the parts' sums [splits][n_tokens][q_heads][D], their
// (reference, sum) [splits][n_tokens][q_heads], those of the prefix first, and
// how many parts of the prefix each request's rows have.
struct Parts {
  float *sums;
  float2 *stats;
  int *ahead;
  long long rows;   // n_tokens q_heads
  __device__ __forceinline__ Parts(const sb_attention_args &a, const Cut &c, void *work) : rows((long long)a.n_tokens * a.q_heads) {
    const long long all = rows * (c.prefix_splits + c.own_splits);
    sums = static_cast<float *>(work);
    stats = reinterpret_cast<float2 *>(sums + all * a.head_dim);
    ahead = reinterpret_cast<int *>(stats + all);
  }
};

__device__ __forceinline__ int group_token(const sb_attention_args &a, const Prefix &p, int g) {
  return min(max(a.q_start[min(max(p.group_start[g], 0), a.n_requests)], 0), a.n_tokens);
}

// The rows of place `place` of the grid, ROWS a tile, as those of a group over its
// prefix: tiles of group g start at (its first token) G / ROWS + g. Returns the
// group, -1 where the place is empty.
template <int ROWS>
__device__ __forceinline__ int span_prefix(const sb_attention_args &a, const Prefix &p, int place, Span &s) {
  const int G = a.q_heads / a.kv_heads;
  int g = 0, gh = p.n_groups;
  while (gh - g > 1) {
    const int mid = (g + gh) >> 1;
    if ((long long)group_token(a, p, mid) * G / ROWS + mid <= place) g = mid;
    else gh = mid;
  }
  s.q0 = group_token(a, p, g);
  s.m = max(group_token(a, p, g + 1) - s.q0, 0);
  s.n = (int)min((long long)max(p.lens[g], 0), (long long)p.pages * a.page_size);
  s.rows = s.m * G;
  s.all = true;
  const long long r0 = (place - ((long long)s.q0 * G / ROWS + g)) * ROWS;
  if (r0 < 0 || r0 >= s.rows) return -1;
  s.r0 = (int)r0;
  s.ns = s.lo = 0;
  s.n_vis = s.n;
  s.p_first = s.p_last = s.n - 1;
  return g;
}

template <int D>
union SharedLds {
  FewShared<D> few;
  ManyShared<D> many;
};

// 16 rows of s over split `split` of their keys, as part `part`.
template <int DT, int D>
__device__ __forceinline__ void part_few(const sb_attention_args &a, const Span &s, int hk, const int *table, int split, int splits, int part,
                                         const Parts &out, FewShared<D> &sh) {
  const int G = a.q_heads / a.kv_heads, tiles = few_tiles(s), each = (tiles + splits - 1) / splits;
  const int t0 = min(split * each, tiles), t1 = min(t0 + each, tiles);
  few_unit<DT, D>(a, s, hk, table, t0, t1, sh, [&](int rw, int col, float top, float sum, const f4 &acc) {
    const int i = rw / G;
    const long long at = part * out.rows + (long long)(s.q0 + i) * a.q_heads + hk * G + rw - i * G;
    *reinterpret_cast<f4 *>(out.sums + at * D + col) = acc;
    if (col == 0) out.stats[at] = make_float2(top - raise<DT>(0), sum);
  });
}

template <int DT, int D>
__device__ __forceinline__ void part_many(const sb_attention_args &a, const Span &s, int hk, const int *table, int split, int splits, int part,
                                          const Parts &out, ManyShared<D> &sh) {
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
  const int tiles = (s.n_vis + MANY_KEYS - 1) / MANY_KEYS, each = (tiles + splits - 1) / splits;
  const int t0 = min(split * each, tiles), count = min(each, tiles - t0);
  if (!many_keys<DT, D, false>(a, s, table, kc, vc, q, p, real, t0, count, sh, o, ref, sum))
    many_keys<DT, D, true>(a, s, table, kc, vc, q, p, real, t0, count, sh, o, ref, sum);
  sum += __shfl_xor(sum, 32, 64);
  if (!real) return;
  const long long at = part * out.rows + (long long)(s.q0 + i) * a.q_heads + hk * G + row - i * G;
  if (h2 == 0) out.stats[at] = make_float2(many_reference<DT>(a, ref), sum);
  float *sums = out.sums + at * D;
#pragma unroll
  for (int x = 0; x < DB; ++x)
#pragma unroll
    for (int e = 0; e < 16; e += 4) *reinterpret_cast<f4 *>(sums + 32 * x + 2 * e + 4 * h2) = f4{o[x][e], o[x][e + 1], o[x][e + 2], o[x][e + 3]};
}

// Workgroups of the prefixes' passes first, then the requests' own; of each the
// key/value heads side by side, so that those of one head, which read the same
// keys, share an XCD's L2.
template <int DT, int D>
__global__ __launch_bounds__(AT_THREADS, D == 256 ? 1 : 2) void k_shared(sb_attention_args a, Prefix p, Cut c, void *work) {
  __shared__ SharedLds<D> sh;
  const Parts out(a, c, work);
  const int hk = (int)(blockIdx.x % a.kv_heads), j = (int)(blockIdx.x / a.kv_heads), prefixes = c.prefix_places * c.prefix_splits;
  Span s;
  if (j < prefixes) {
    const int split = j % c.prefix_splits, place = j / c.prefix_splits;
    if (c.prefix_many) {
      const int g = span_prefix<MANY_ROWS>(a, p, place, s);
      if (g >= 0) part_many<DT, D>(a, s, hk, p.table + g * p.stride, split, c.prefix_splits, split, out, sh.many);
    } else {
      const int g = span_prefix<FEW_ROWS>(a, p, place, s);
      if (g >= 0) part_few<DT, D>(a, s, hk, p.table + g * p.stride, split, c.prefix_splits, split, out, sh.few);
    }
    return;
  }
  const int split = (j - prefixes) % c.own_splits, place = (j - prefixes) / c.own_splits;
  int b = place;
  if (c.own_many) b = span_tile(a, place, s);
  else span_request(a, b, s);
  if (b < 0) return;
  if (hk == 0 && split == 0 && (!c.own_many || s.r0 == 0)) {   // has the request a prefix?
    int found = 0;
    for (int g = threadIdx.x; g < p.n_groups; g += AT_THREADS)
      found |= min(max(p.group_start[g], 0), a.n_requests) <= b && b < min(max(p.group_start[g + 1], 0), a.n_requests);
    found = __syncthreads_or(found);
    if (threadIdx.x == 0) out.ahead[b] = found ? c.prefix_splits : 0;
  }
  const int part = c.prefix_splits + split;
  if (c.own_many) {
    part_many<DT, D>(a, s, hk, a.table + b * a.table_stride, split, c.own_splits, part, out, sh.many);
  } else {
    for (int r0 = 0; r0 < s.rows; r0 += FEW_ROWS) {
      span_rows(a, r0, FEW_ROWS, s);
      part_few<DT, D>(a, s, hk, a.table + b * a.table_stride, split, c.own_splits, part, out, sh.few);
    }
  }
}

// A wave a row.
template <int DT, int D>
__global__ __launch_bounds__(AT_THREADS) void k_shared_join(sb_attention_args a, Cut c, void *work) {
  const Parts in(a, c, work);
  const int b = blockIdx.x;
  Span s;
  span_request(a, b, s);
  if (s.m == 0) return;
  const int ahead = min(max(in.ahead[b], 0), c.prefix_splits), gap = c.prefix_splits - ahead;
  const long long rows = (long long)s.m * a.q_heads, step = (long long)gridDim.y * AT_WAVES;
  for (long long r = (long long)blockIdx.y * AT_WAVES + (threadIdx.x >> 6); r < rows; r += step) {
    const long long at = (long long)s.q0 * a.q_heads + r;
    join_row<DT, D>(in.sums, in.stats, ahead + c.own_splits, [&](int x) { return (x < ahead ? x : x + gap) * in.rows + at; },
                    static_cast<uint16_t *>(a.out) + (s.q0 + r / a.q_heads) * a.out_token + (r % a.q_heads) * a.out_head);
  }
}

// Splits: as many as fill the units, of SPLIT_KEYS keys at least.
constexpr int SPLIT_KEYS = 512;
Cut cut(const sb_shared_args &x, int n_cu) {
  const sb_attention_args &a = x.own;
  const long long G = a.q_heads / a.kv_heads, all = a.n_tokens * G, room = (a.head_dim == 256 ? 1 : 2) * (long long)n_cu;
  const auto splits = [&](long long tiles, long long places, int keys) {
    return (int)std::max(1LL, std::min({room / (tiles * a.kv_heads), 2 * room / (places * a.kv_heads), (long long)keys / SPLIT_KEYS}));
  };
  Cut c;
  const long long group_rows = (all + x.n_groups - 1) / x.n_groups, request_rows = std::max(a.max_q, 1) * G;
  c.prefix_many = group_rows > FEW_ROWS;
  c.own_many = request_rows > FEW_ROWS;
  const long long ptile = c.prefix_many ? MANY_ROWS : FEW_ROWS;
  c.prefix_places = (int)(all / ptile + x.n_groups);
  c.prefix_splits = splits(std::min((long long)c.prefix_places, (group_rows + ptile - 1) / ptile * x.n_groups), c.prefix_places, x.max_prefix);
  c.own_places = c.own_many ? (int)(all / MANY_ROWS + a.n_requests) : a.n_requests;
  c.own_splits = splits(c.own_places, c.own_places, a.max_kv);
  return c;
}

template <int DT, int D>
hipError_t launch(const sb_shared_args &x, int n_cu, void *work, hipStream_t s) {
  const sb_attention_args &a = x.own;
  const Cut c = cut(x, n_cu);
  const Prefix p = {x.prefix_table, x.prefix_lens, x.group_start, x.prefix_stride, x.n_groups, x.prefix_pages};
  const long long grid = ((long long)c.prefix_places * c.prefix_splits + (long long)c.own_places * c.own_splits) * a.kv_heads;
  hipLaunchKernelGGL((k_shared<DT, D>), dim3((unsigned)grid), dim3(AT_THREADS), 0, s, a, p, c, work);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long long join = std::min(((long long)std::max(a.max_q, 1) * a.q_heads + AT_WAVES - 1) / AT_WAVES, 1024LL);
  hipLaunchKernelGGL((k_shared_join<DT, D>), dim3((unsigned)a.n_requests, (unsigned)join), dim3(AT_THREADS), 0, s, a, c, work);
  return hipGetLastError();
}

}  // namespace

int64_t shared_workspace(const sb_shared_args &x, int n_cu) {
  const sb_attention_args &a = x.own;
  const Cut c = cut(x, n_cu);
  return (int64_t)(c.prefix_splits + c.own_splits) * a.n_tokens * a.q_heads * (a.head_dim * 4 + 8) + 4LL * a.n_requests;
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
