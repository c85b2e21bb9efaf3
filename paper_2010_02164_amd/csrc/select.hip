// Selected pages of a paged cache: the bounds of their keys, the pages that each
// query attends to by them, and the attention over those.
//
// With the smallest and largest of each value over a page's keys, the largest score
// that one of its keys can have with a query is sum max(q_i lo_i, q_i hi_i) =
// sum max(q_i, 0) hi_i + min(q_i, 0) lo_i: linear in the bounds, so that a group's
// heads are added up before, and one product of 2 D values ranks a page for all
// of them. Sums are fp64, where products of 16-bit values are exact and their sums
// nearly always: the order of the pages does not depend on that of the sums.
#include <algorithm>

#include "attn_pass.h"
#include "serve_plan.h"
#include "wave.h"

namespace sb {
namespace {

typedef unsigned long long u64;

// -- bounds ------------------------------------------------------------------------

constexpr int BD_THREADS = 256;

// A wave takes 128 values of a page (a lane 8 of them, of every fourth key). Bound by
// its chain of waits (lengths, table, keys): 4 us for one request, 7 for 48.
template <int DT>
__global__ __launch_bounds__(BD_THREADS) void k_bounds(sb_bounds_args a) {
  const int b = blockIdx.x, lane = threadIdx.x & 63, turn = lane >> 4;
  const int n = (int)min((long long)max(a.lens[b], 0), (long long)a.max_pages * a.page_size);
  const int m = (int)min(max((long long)a.q_start[b + 1] - a.q_start[b], 0LL), (long long)n);
  if (m == 0) return;
  const int first = (n - m) / a.page_size, values = a.kv_heads * a.head_dim, blocks = (values + 127) / 128;
  const long long units = (long long)((n - 1) / a.page_size - first + 1) * blocks;
  for (long long u = blockIdx.y * (BD_THREADS / 64) + (threadIdx.x >> 6); u < units; u += gridDim.y * (BD_THREADS / 64)) {
    const int c = first + (int)(u / blocks), at = (int)(u % blocks) * 128 + (lane & 15) * 8;
    const int page = a.table[b * a.table_stride + c];
    if ((unsigned)page >= (unsigned)a.n_pages) continue;
    const bool real = at < values;
    const int keys = min(a.page_size, n - c * a.page_size), head = real ? at / a.head_dim : 0;
    const uint16_t *src = static_cast<const uint16_t *>(a.k_cache) + page * a.kc_page + head * a.kc_head + (real ? at - head * a.head_dim : 0);
    float lo[8], hi[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      lo[x] = INFINITY;
      hi[x] = -INFINITY;
    }
    // (A NaN stays: nothing is smaller or larger.)
    auto take = [&](int x, float l, float h) {
      lo[x] = l < lo[x] || l != l ? l : lo[x];
      hi[x] = h > hi[x] || h != h ? h : hi[x];
    };
#pragma unroll 4
    for (int k = turn; k < keys; k += 4) {
      const u4 v = *reinterpret_cast<const u4 *>(src + k * a.kc_slot);
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const float f = Half<DT>::to_float(x & 1 ? v[x >> 1] >> 16 : v[x >> 1] & 0xFFFFu);
        take(x, f, f);
      }
    }
#pragma unroll
    for (int o = 16; o < 64; o <<= 1)
#pragma unroll
      for (int x = 0; x < 8; ++x) take(x, __shfl_xor(lo[x], o, 64), __shfl_xor(hi[x], o, 64));
    if (turn < 2 && real) {
      u4 out;
#pragma unroll
      for (int x = 0; x < 4; ++x) out[x] = turn ? Half<DT>::pack(hi[2 * x], hi[2 * x + 1]) : Half<DT>::pack(lo[2 * x], lo[2 * x + 1]);
      *reinterpret_cast<u4 *>(static_cast<uint16_t *>(a.bounds) + ((long long)page * 2 + turn) * values + at) = out;
    }
  }
}

// -- selection -----------------------------------------------------------------------

constexpr int SL_THREADS = 256, SL_WAVES = 4;

// Of token t: its request, its position (-1: before the request's first token) and
// how many pages there are up to it. False where it is of no request. (Called by all
// threads; `found` in LDS, 0 before. Starts and lengths are loaded together: each
// wait for memory is a microsecond of a small call's.)
struct Query {
  int b, p, n;
};
__device__ __forceinline__ bool query_of(const sb_select_args &a, int t, u64 *found, Query &q) {
  for (int b = threadIdx.x; b < a.n_requests; b += blockDim.x) {
    const int from = a.q_start[b], to = min(a.q_start[b + 1], a.n_tokens), len = a.lens[b];
    if (from <= t && t < to) {
      const long long p = max(min((long long)max(len, 0), (long long)a.max_pages * a.page_size) - to + t, -1LL);
      atomicMax(found, (u64)b << 32 | (u64)(p + 2));
    }
  }
  __syncthreads();
  const u64 at = *found;
  if (at == 0) return false;
  q.b = (int)(at >> 32);
  q.p = (int)(uint32_t)at - 2;
  q.n = q.p < 0 ? 0 : q.p / a.page_size + 1;
  return true;
}

// Sums over neighbouring lanes (wave.h's stages).
template <int S>
__device__ __forceinline__ double add_stage(double v) {
  u64 x, y;
  stage64<S>((u64)__double_as_longlong(v), x, y);
  return __longlong_as_double((long long)x) + __longlong_as_double((long long)y);
}

// The place a grid's step behind `at`, or `end`: with rows of nearly 2^31 pages the sum
// would pass an int.
__device__ __forceinline__ int step_on(int at, int step, int end) { return end - at > step ? at + step : end; }

// A score as a number whose order is the scores': NaN last, and all of them above
// NOT_THERE, which pages outside the cache have.
constexpr u64 NOT_THERE = 0;
__device__ __forceinline__ u64 order_of(double score) {
  const u64 bits = (u64)__double_as_longlong(score + 0.0);   // (of -0 and 0 one)
  return score != score ? ~0ULL : bits ^ (bits >> 63 ? ~0ULL : 1ULL << 63);
}

// Scores of the pages first .. n - last - 1 of token t0 + blockIdx.z, head
// blockIdx.y, those of `chunk` pages a workgroup, to keys [tokens][kv_heads][max_pages].
// Bound by reading the bounds: 48 requests of 5000 to 50000 tokens, pages of 16, 8
// heads of 128: 84 us, 4.0 TB/s (heads side by side in the grid: 89; 2 or 8 loads of
// each bound in flight: 90, 87; a load at a time: 96).
template <int DT, int D>
__global__ __launch_bounds__(SL_THREADS) void k_scores(sb_select_args a, int t0, int chunk, u64 *keys) {
  constexpr int L = D / 8, P = 64 / L;   // lanes of a page, pages a wave takes at once
  __shared__ u64 found;
  const int t = t0 + blockIdx.z, hk = blockIdx.y, G = a.q_heads / a.kv_heads, lane = threadIdx.x & 63, col = lane % L;
  if (threadIdx.x == 0) found = 0;
  double up[8], down[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) up[x] = down[x] = 0.0;
  for (int g = 0; g < G; ++g) {
    const u4 v = *reinterpret_cast<const u4 *>(static_cast<const uint16_t *>(a.q) + t * a.q_token + (hk * G + g) * a.q_head + 8 * col);
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const float f = Half<DT>::to_float(x & 1 ? v[x >> 1] >> 16 : v[x >> 1] & 0xFFFFu);
      if (f != f) up[x] = f;   // (NaN: neither above nor below 0)
      up[x] += f > 0.0f ? f : 0.0f;
      down[x] += f < 0.0f ? f : 0.0f;
    }
  }
  __syncthreads();
  Query q;
  if (!query_of(a, t, &found, q) || q.n <= (long long)a.first + a.top + a.last) return;
  const int *table = a.table + q.b * a.table_stride;
  const long long row = (long long)a.kv_heads * D;
  const uint16_t *bounds = static_cast<const uint16_t *>(a.bounds) + (long long)hk * D + 8 * col;
  u64 *out = keys + ((long long)blockIdx.z * a.kv_heads + hk) * a.max_pages;
  const int end = q.n - a.last;
  for (int at = blockIdx.x * chunk + a.first; at < end; at = step_on(at, gridDim.x * chunk, end)) {
    const int stop = min(at + chunk, end);
    // A wave's pages are looked up together, then taken a few at a time, with their
    // loads in flight together.
    constexpr int BATCH = 4;
    const int each = chunk / SL_WAVES, wave_stop = min(at + ((int)(threadIdx.x >> 6) + 1) * each, stop);   // (each: 16 to 128)
    for (int c0 = at + (int)(threadIdx.x >> 6) * each; c0 < wave_stop; c0 += 64) {
      const int page = c0 + lane < wave_stop ? table[c0 + lane] : -1;
      for (int s0 = 0; s0 < 64 && c0 + s0 < wave_stop; s0 += BATCH * P) {
        u4 lo[BATCH], hi[BATCH];
        bool there[BATCH];
#pragma unroll
        for (int x = 0; x < BATCH; ++x) {
          const int mine = __shfl(page, s0 + x * P + lane / L, 64);
          there[x] = (unsigned)mine < (unsigned)a.n_pages;
          const uint16_t *src = bounds + (there[x] ? 2LL * mine * row : 0);
          lo[x] = *reinterpret_cast<const u4 *>(src);
          hi[x] = *reinterpret_cast<const u4 *>(src + row);
        }
#pragma unroll
        for (int x = 0; x < BATCH; ++x) {
          double s = 0.0;
#pragma unroll
          for (int y = 0; y < 8; ++y) {
            s = fma((double)Half<DT>::to_float(y & 1 ? hi[x][y >> 1] >> 16 : hi[x][y >> 1] & 0xFFFFu), up[y], s);
            s = fma((double)Half<DT>::to_float(y & 1 ? lo[x][y >> 1] >> 16 : lo[x][y >> 1] & 0xFFFFu), down[y], s);
          }
          s = add_stage<2>(add_stage<1>(add_stage<0>(s)));
          if constexpr (L >= 16) s = add_stage<3>(s);
          if constexpr (L >= 32) s = add_stage<4>(s);
          const int c = c0 + s0 + x * P + lane / L;
          if (col == 0 && c < wave_stop) out[c] = there[x] ? order_of(s) : NOT_THERE;
        }
      }
    }
  }
}

// The same for prompts, 16 tokens a workgroup, by the matrix unit in fp64: its rows are
// the tokens' sums, in LDS as its lanes take them, its columns 16 pages a wave. Lane l
// has values l / 16 D / 4 .. of a bound (which value stands for which k of a product
// does not matter, as long as both operands have the same). Tokens of several requests
// take a turn each. 900 tokens over 24000 to 30000, pages of 32, 4 heads of 128: 66 us,
// by k_scores 157, most of it conversions and sums (four tokens a workgroup there: 156).
constexpr int SP_TOKENS = 16;
typedef double d4 __attribute__((ext_vector_type(4)));
template <int DT, int D>
__global__ __launch_bounds__(SL_THREADS) void k_scores_many(sb_select_args a, int t0, int t_end, int chunk, u64 *keys) {
  constexpr int Q = D / 4, PIECES = Q / 8;   // values and 16-byte pieces of a lane
  __shared__ double sums[2 * Q][64];          // [product][lane]: the first Q with the larger bounds, the others with the smaller
  __shared__ u64 found[SP_TOKENS];
  const int z = blockIdx.z * SP_TOKENS, t = t0 + z, hk = blockIdx.y, G = a.q_heads / a.kv_heads;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4;
  if (threadIdx.x < SP_TOKENS) found[threadIdx.x] = 0;
  for (int x = threadIdx.x; x < SP_TOKENS * (D / 8); x += SL_THREADS) {
    const int token = x & (SP_TOKENS - 1), d = x / SP_TOKENS * 8;
    const uint16_t *src = static_cast<const uint16_t *>(a.q) + min(t + token, t_end - 1) * a.q_token + hk * G * a.q_head + d;
    double up[8], down[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) up[y] = down[y] = 0.0;
    for (int g = 0; g < G; ++g) {
      const u4 v = *reinterpret_cast<const u4 *>(src + g * a.q_head);
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const float f = Half<DT>::to_float(y & 1 ? v[y >> 1] >> 16 : v[y >> 1] & 0xFFFFu);
        if (f != f) up[y] = f;
        up[y] += f > 0.0f ? f : 0.0f;
        down[y] += f < 0.0f ? f : 0.0f;
      }
    }
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      sums[(d + y) % Q][(d + y) / Q * 16 + token] = up[y];
      sums[Q + (d + y) % Q][(d + y) / Q * 16 + token] = down[y];
    }
  }
  __syncthreads();
  for (int b = threadIdx.x; b < a.n_requests; b += SL_THREADS) {
    const int next = min(a.q_start[b + 1], a.n_tokens), from = max(a.q_start[b], t), to = min(next, min(t + SP_TOKENS, t_end));
    const long long len = min((long long)max(a.lens[b], 0), (long long)a.max_pages * a.page_size);
    for (int x = from; x < to; ++x) {
      const long long p = max(len - next + x, -1LL);
      atomicMax(&found[x - t], (u64)b << 32 | (u64)(p + 2));
    }
  }
  __syncthreads();
  // The lane's four tokens (rows g4 + 4 i of a product's result) and the ends of their pages.
  const auto request_of = [&](int token, int &end) {
    const u64 at = found[token];
    const int p = (int)(uint32_t)at - 2, n = at == 0 || p < 0 ? 0 : p / a.page_size + 1;
    end = n - a.last;
    return n > (long long)a.first + a.top + a.last ? (int)(at >> 32) : -1;
  };
  const long long row = (long long)a.kv_heads * D, next = (long long)a.kv_heads * a.max_pages;
  const uint16_t *bounds = static_cast<const uint16_t *>(a.bounds) + (long long)hk * D + g4 * Q;
  u64 *out = keys + ((long long)z * a.kv_heads + hk) * a.max_pages;
  int before = -1;
  for (int turn = 0; turn < SP_TOKENS; ++turn) {   // a request a turn (those that follow each other are one)
    int end;
    const int b = request_of(turn, end);
    if (b < 0 || b == before) continue;
    before = b;
    end = 0;
    int ends[4];
    for (int x = 0; x < SP_TOKENS; ++x) {
      int e;
      if (request_of(x, e) == b) end = max(end, e);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int e;
      ends[i] = request_of(g4 + 4 * i, e) == b ? e : 0;
    }
    const int *table = a.table + b * a.table_stride;
    for (int at = blockIdx.x * chunk + a.first; at < end; at = step_on(at, gridDim.x * chunk, end)) {
      const int stop = min(at + chunk, end);
      for (int c0 = at + (int)(threadIdx.x >> 6) * 16; c0 < stop; c0 += SL_WAVES * 16) {
        const int c = c0 + l16, page = c < stop ? table[c] : -1;
        const bool there = (unsigned)page < (unsigned)a.n_pages;
        const uint16_t *src = bounds + (there ? 2LL * page * row : 0);
        u4 hi[PIECES], lo[PIECES];
#pragma unroll
        for (int x = 0; x < PIECES; ++x) {
          hi[x] = *reinterpret_cast<const u4 *>(src + row + 8 * x);
          lo[x] = *reinterpret_cast<const u4 *>(src + 8 * x);
        }
        d4 s[2] = {d4{0, 0, 0, 0}, d4{0, 0, 0, 0}};
#pragma unroll
        for (int x = 0; x < PIECES; ++x)
#pragma unroll
          for (int y = 0; y < 8; ++y) {
            const double h = Half<DT>::to_float(y & 1 ? hi[x][y >> 1] >> 16 : hi[x][y >> 1] & 0xFFFFu);
            const double l = Half<DT>::to_float(y & 1 ? lo[x][y >> 1] >> 16 : lo[x][y >> 1] & 0xFFFFu);
            s[0] = __builtin_amdgcn_mfma_f64_16x16x4f64(sums[8 * x + y][lane], h, s[0], 0, 0, 0);
            s[1] = __builtin_amdgcn_mfma_f64_16x16x4f64(sums[Q + 8 * x + y][lane], l, s[1], 0, 0, 0);
          }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c < min(stop, ends[i])) out[(g4 + 4 * i) * next + c] = there ? order_of(s[0][i] + s[1][i]) : NOT_THERE;
      }
    }
  }
}

constexpr int BINS = 2048, LIST = 256;

// The list of token t0 + blockIdx.x, head blockIdx.y: the key of the last page
// taken is found by counting keys in bins, ever finer, until those of its bin fit
// a list; then the pages above it are written in order. A thread has PER keys that
// follow each other in registers; where there are more pages than that, the passes
// read them from memory again (48 requests of 5000 to 50000 tokens in pages of 16:
// 20 us where all did).
template <int THREADS, int PER>
__global__ __launch_bounds__(THREADS) void k_pick(sb_select_args a, int t0, const u64 *all_keys) {
  constexpr int WAVES = THREADS / 64;
  __shared__ int bins[BINS], wave_sums[2][WAVES][2], listed, bin_at, bin_before;
  __shared__ u64 found, list[LIST], ends[WAVES][2], cut_key;
  __shared__ int cut_equal;
  const int t = t0 + blockIdx.x, hk = blockIdx.y, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int width = a.first + a.top + a.last;
  int *out = a.pages + ((long long)t * a.kv_heads + hk) * width;
  Query q;
  if (threadIdx.x == 0) found = 0;
  __syncthreads();
  const bool real = query_of(a, t, &found, q);
  if (hk == 0 && threadIdx.x == 0)
    a.kept[t] = !real ? -1 : q.n <= width ? q.p + 1 : (width - 1) * a.page_size + q.p % a.page_size + 1;
  if (!real || q.n <= width) {
    for (int x = threadIdx.x; x < width; x += THREADS) out[x] = real && x < q.n ? a.table[q.b * a.table_stride + x] : -1;
    return;
  }
  const int *table = a.table + q.b * a.table_stride;
  const u64 *keys = all_keys + ((long long)blockIdx.x * a.kv_heads + hk) * a.max_pages;
  const int begin = a.first, end = q.n - a.last, mine = begin + min((int)threadIdx.x * PER, end - begin);
  const bool held = end - begin <= THREADS * PER;   // all keys in registers
  u64 k[PER];
  if (held && a.top > 0) {
#pragma unroll
    for (int x = 0; x < PER; ++x) k[x] = mine + x < end ? keys[mine + x] : 0;
  }
  for (int x = threadIdx.x; x < a.first; x += THREADS) out[x] = table[x];
  for (int x = threadIdx.x; x < a.last; x += THREADS) out[a.first + a.top + x] = table[q.n - a.last + x];
  if (a.top == 0) return;
  const auto each = [&](const auto &f) {
    if (held) {
#pragma unroll
      for (int x = 0; x < PER; ++x)
        if (mine + x < end) f(k[x]);
    } else {
      for (int c = begin + threadIdx.x; c < end; c += THREADS) f(keys[c]);
    }
  };
  u64 lo = ~0ULL, hi = 0;
  each([&](u64 key) {
    lo = min(lo, key);
    hi = max(hi, key);
  });
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    lo = min(lo, (u64)__shfl_xor((long long)lo, o, 64));
    hi = max(hi, (u64)__shfl_xor((long long)hi, o, 64));
  }
  if (lane == 0) {
    ends[w][0] = lo;
    ends[w][1] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < WAVES; ++x) {
    lo = min(lo, ends[x][0]);
    hi = max(hi, ends[x][1]);
  }
  int want = a.top;   // the want'th largest of the keys from lo to hi is the last one taken
  for (;;) {
    if (lo == hi) {
      if (threadIdx.x == 0) {
        cut_key = lo;
        cut_equal = want;
      }
      break;
    }
    const int shift = max(64 - __clzll((long long)(hi - lo)) - 11, 0);   // bins of 2^shift keys
    for (int x = threadIdx.x; x < BINS; x += THREADS) bins[x] = 0;
    if (threadIdx.x == 0) listed = 0;
    __syncthreads();
    each([&](u64 key) {
      if (key >= lo && key <= hi) atomicAdd(&bins[(hi - key) >> shift], 1);   // (bin 0: the largest)
    });
    __syncthreads();
    // Some bins a thread: where their sum passes want.
    constexpr int OWN = BINS / THREADS;
    int sum = 0;
#pragma unroll
    for (int x = 0; x < OWN; ++x) sum += bins[threadIdx.x * OWN + x];
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(upto, o, 64);
      if (lane >= o) upto += y;
    }
    if (lane == 63) wave_sums[0][w][0] = upto;
    __syncthreads();
    for (int x = 0; x < w; ++x) upto += wave_sums[0][x][0];
    if (upto - sum < want && want <= upto) {   // (one thread)
      int before = upto - sum, x = threadIdx.x * OWN;
      while (before + bins[x] < want) before += bins[x++];
      bin_at = x;
      bin_before = before;
    }
    __syncthreads();
    const int bin = bin_at, count = bins[bin];
    want -= bin_before;
    const u64 top = hi - ((u64)bin << shift), width_of = (1ULL << shift) - 1;
    hi = top;
    lo = top - lo > width_of ? top - width_of : lo;
    if (count <= LIST) {
      each([&](u64 key) {
        if (key >= lo && key <= hi) list[atomicAdd(&listed, 1)] = key;
      });
      __syncthreads();
      if (threadIdx.x < count) {
        const u64 key = list[threadIdx.x];
        int above = 0, equal = 0;
        for (int x = 0; x < count; ++x) {
          above += list[x] > key;
          equal += list[x] == key;
        }
        if (above < want && want <= above + equal) {   // (equal keys write the same)
          cut_key = key;
          cut_equal = want - above;
        }
      }
      break;
    }
    __syncthreads();
  }
  __syncthreads();
  const u64 cut = cut_key;
  const int equal_taken = cut_equal;
  // Pages above the cut, and the first of those on it, in the cache's order.
  if (held) {
    int above = 0, equal = 0;
    each([&](u64 key) {
      above += key > cut;
      equal += key == cut;
    });
    int na = above, ne = equal;   // up to this thread
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(na, o, 64), y = __shfl_up(ne, o, 64);
      if (lane >= o) {
        na += x;
        ne += y;
      }
    }
    if (lane == 63) {
      wave_sums[1][w][0] = na;
      wave_sums[1][w][1] = ne;
    }
    __syncthreads();
    na -= above;
    ne -= equal;
    for (int x = 0; x < w; ++x) {
      na += wave_sums[1][x][0];
      ne += wave_sums[1][x][1];
    }
    if (above + equal == 0) return;
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      const bool there = mine + x < end, over = there && k[x] > cut, on = there && k[x] == cut;
      if (over || (on && ne < equal_taken)) out[a.first + na + min(ne, equal_taken)] = table[mine + x];
      na += over;
      ne += on;
    }
    return;
  }
  int above_before = 0, equal_before = 0;
  for (int c0 = begin, turn = 0; c0 < end; c0 += THREADS, turn ^= 1) {
    const int c = c0 + threadIdx.x;
    const u64 key = c < end ? keys[c] : 0;
    const bool above = c < end && key > cut, equal = c < end && key == cut;
    const u64 ma = __ballot(above), me = __ballot(equal), below = (1ULL << lane) - 1;
    if (lane == 0) {
      wave_sums[turn][w][0] = __popcll(ma);
      wave_sums[turn][w][1] = __popcll(me);
    }
    __syncthreads();
    int na = above_before + __popcll(ma & below), ne = equal_before + __popcll(me & below);
#pragma unroll
    for (int x = 0; x < WAVES; ++x) {
      if (x < w) {
        na += wave_sums[turn][x][0];
        ne += wave_sums[turn][x][1];
      }
      above_before += wave_sums[turn][x][0];
      equal_before += wave_sums[turn][x][1];
    }
    if (above || (equal && ne < equal_taken)) out[a.first + na + min(ne, equal_taken)] = table[c];
  }
}

// -- attention over the selected pages -----------------------------------------------

// A token's heads of a group are up to 16 rows of one pass over its selected keys
// (attn_pass.h), which all of them see. Bound by reading the keys: 48 tokens, 8 heads of
// 128, 2048 keys each: 86 us, 4.7 TB/s; a prompt's, where pages come from the caches,
// by the waits for them: 900 tokens, 4 heads, 2080 keys: 297 to 304 us in a series of
// them, 322 between a step's other kernels, 12.6 TB/s (two workgroups a compute unit,
// not three: 340, and the 48 tokens 86 to 89; values asked for together with the keys:
// 323 and 99, out of registers, by two workgroups 348 and 93).
// In the workspace: the parts' sums [splits][n_tokens][q_heads][D] and their
// (reference, sum).
template <int DT, int D>
__global__ __launch_bounds__(AT_THREADS, D <= 128 ? 3 : 1) void k_selected(sb_attention_args a, const int *kept, int splits, void *work) {
  __shared__ FewShared<D> sh;
  const int G = a.q_heads / a.kv_heads, hk = (int)(blockIdx.x % a.kv_heads), j = (int)(blockIdx.x / a.kv_heads);
  const int t = j / splits, split = j % splits, n = kept[t];
  if (n < 0) return;
  const long long rows = (long long)a.n_tokens * a.q_heads;
  float *sums = static_cast<float *>(work);
  float2 *stats = reinterpret_cast<float2 *>(sums + rows * splits * D);
  Span s;
  s.q0 = t;
  s.m = 1;
  s.n = s.n_vis = (int)min((long long)n, (long long)a.max_pages * a.page_size);
  s.rows = G;
  s.ns = s.lo = 0;
  s.p_first = s.p_last = s.n - 1;
  s.all = true;
  const int *table = a.table + ((long long)t * a.kv_heads + hk) * a.table_stride;
  const int tiles = few_tiles(s), each = (tiles + splits - 1) / splits, t0 = min(split * each, tiles), t1 = min(t0 + each, tiles);
  for (int r0 = 0; r0 < G; r0 += FEW_ROWS) {
    s.r0 = r0;
    few_unit<DT, D>(a, s, hk, table, t0, t1, sh, [&](int rw, int col, float top, float sum, const f4 &acc) {
      if (splits == 1) {
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        uint16_t *dst = static_cast<uint16_t *>(a.out) + t * a.out_token + (hk * G + rw) * a.out_head + col;
        *reinterpret_cast<u2 *>(dst) = u2{Half<DT>::pack(acc[0] * inv, acc[1] * inv), Half<DT>::pack(acc[2] * inv, acc[3] * inv)};
        return;
      }
      const long long at = split * rows + (long long)t * a.q_heads + hk * G + rw;
      *reinterpret_cast<f4 *>(sums + at * D + col) = acc;
      if (col == 0) stats[at] = make_float2(top, sum);
    });
  }
}

template <int DT, int D>
__global__ __launch_bounds__(AT_THREADS) void k_selected_join(sb_attention_args a, const int *kept, int splits, const void *work) {
  const long long rows = (long long)a.n_tokens * a.q_heads, at = (long long)blockIdx.x * AT_WAVES + (threadIdx.x >> 6);
  if (at >= rows || kept[at / a.q_heads] < 0) return;
  const float *sums = static_cast<const float *>(work);
  join_row<DT, D>(sums, reinterpret_cast<const float2 *>(sums + rows * splits * D), splits, [&](int x) { return x * rows + at; },
                  static_cast<uint16_t *>(a.out) + at / a.q_heads * a.out_token + at % a.q_heads * a.out_head);
}

// Splits where tokens and heads are too few for the units, of SPLIT_KEYS keys at
// least.
constexpr int SPLIT_KEYS = 128;
int splits_of(const sb_selected_args &x, int n_cu) {
  const long long room = (x.head_dim <= 128 ? 3 : 1) * (long long)n_cu;
  return (int)std::max(1LL, std::min(room / ((long long)x.n_tokens * x.kv_heads), (long long)x.width * x.page_size / SPLIT_KEYS));
}

template <int DT, int D>
hipError_t attend(const sb_selected_args &x, int n_cu, void *work, hipStream_t s) {
  sb_attention_args a = {};
  a.q = x.q, a.k_cache = x.k_cache, a.v_cache = x.v_cache, a.table = x.pages, a.out = x.out;
  a.q_token = x.q_token, a.q_head = x.q_head, a.out_token = x.out_token, a.out_head = x.out_head;
  a.kc_page = x.kc_page, a.kc_slot = x.kc_slot, a.kc_head = x.kc_head, a.vc_page = x.vc_page, a.vc_slot = x.vc_slot, a.vc_head = x.vc_head;
  a.table_stride = a.max_pages = x.width;
  a.n_tokens = x.n_tokens, a.q_heads = x.q_heads, a.kv_heads = x.kv_heads, a.head_dim = D, a.n_pages = x.n_pages, a.page_size = x.page_size;
  a.scale = x.scale;
  const int splits = splits_of(x, n_cu);
  hipLaunchKernelGGL((k_selected<DT, D>), dim3((unsigned)((long long)x.n_tokens * splits * x.kv_heads)), dim3(AT_THREADS), 0, s, a, x.kept,
                     splits, work);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  const long long rows = (long long)x.n_tokens * x.q_heads;
  hipLaunchKernelGGL((k_selected_join<DT, D>), dim3((unsigned)((rows + AT_WAVES - 1) / AT_WAVES)), dim3(AT_THREADS), 0, s, a, x.kept, splits, work);
  return hipGetLastError();
}

// Tokens whose scores are kept at a time.
constexpr long long SCORE_BYTES = 256 << 20;
long long tokens_at_once(const sb_select_args &a) {
  return std::max(1LL, std::min({(long long)a.n_tokens, SCORE_BYTES / ((long long)a.kv_heads * a.max_pages * 8), 65535LL}));
}

template <int DT, int D>
hipError_t select(const sb_select_args &a, int n_cu, void *work, hipStream_t s) {
  const long long step = tokens_at_once(a);
  const long long between = pages_between(a);
  const bool many = many_scores(a);
  for (long long t0 = 0; t0 < a.n_tokens; t0 += step) {
    const unsigned tokens = (unsigned)std::min(step, a.n_tokens - t0);
    if (a.top > 0) {
      // Pages enough for a workgroup that reading the queries is a small part.
      constexpr long long LEAST = 64, MOST = 512;
      const long long rows = (many ? (tokens + SP_TOKENS - 1) / SP_TOKENS : tokens) * (long long)a.kv_heads;
      const long long chunk = std::min(MOST, std::max(LEAST, between * rows / ((many ? 3 : 8) * n_cu) / LEAST * LEAST));
      const unsigned chunks = (unsigned)std::min(65535LL, (between + chunk - 1) / chunk);
      if (many) {
        hipLaunchKernelGGL((k_scores_many<DT, D>), dim3(chunks, a.kv_heads, (tokens + SP_TOKENS - 1) / SP_TOKENS), dim3(SL_THREADS), 0, s, a,
                           (int)t0, (int)(t0 + tokens), (int)chunk, static_cast<u64 *>(work));
      } else {
        hipLaunchKernelGGL((k_scores<DT, D>), dim3(chunks, a.kv_heads, tokens), dim3(SL_THREADS), 0, s, a, (int)t0, (int)chunk,
                           static_cast<u64 *>(work));
      }
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    const auto pick = [&](auto kernel, int threads) {
      hipLaunchKernelGGL(kernel, dim3(tokens, a.kv_heads), dim3(threads), 0, s, a, (int)t0, static_cast<const u64 *>(work));
    };
    const PickPlan p = pick_plan(between, (long long)tokens * a.kv_heads, n_cu);
    if (p.threads == 256) {
      if (p.per == 4) pick(k_pick<256, 4>, 256);
      else pick(k_pick<256, 16>, 256);
    } else {
      if (p.per == 4) pick(k_pick<1024, 4>, 1024);
      else pick(k_pick<1024, 16>, 1024);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_bounds(const sb_bounds_args &a, hipStream_t s) {
  const long long pages = std::max(a.max_q, 1) / a.page_size + 2LL, units = pages * ((a.kv_heads * a.head_dim + 127) / 128);
  const dim3 grid((unsigned)a.n_requests, (unsigned)std::min((units + BD_THREADS / 64 - 1) / (BD_THREADS / 64), 1024LL));
  if (a.dtype == SB_BF16) hipLaunchKernelGGL((k_bounds<SB_BF16>), grid, dim3(BD_THREADS), 0, s, a);
  else hipLaunchKernelGGL((k_bounds<SB_F16>), grid, dim3(BD_THREADS), 0, s, a);
  return hipGetLastError();
}

int64_t select_workspace(const sb_select_args &a) { return tokens_at_once(a) * a.kv_heads * a.max_pages * 8; }

int64_t selected_workspace(const sb_selected_args &a, int n_cu) {
  if (a.n_tokens == 0) return 0;
  const int splits = splits_of(a, n_cu);
  return splits == 1 ? 0 : (int64_t)splits * a.n_tokens * a.q_heads * (a.head_dim + 2) * 4;
}

#define BY_TYPE_AND_SIZE(fn, a, ...)                                              \
  if (a.dtype == SB_BF16) {                                                       \
    if (a.head_dim == 64) return fn<SB_BF16, 64>(a, __VA_ARGS__);                 \
    if (a.head_dim == 128) return fn<SB_BF16, 128>(a, __VA_ARGS__);               \
    return fn<SB_BF16, 256>(a, __VA_ARGS__);                                      \
  }                                                                               \
  if (a.head_dim == 64) return fn<SB_F16, 64>(a, __VA_ARGS__);                    \
  if (a.head_dim == 128) return fn<SB_F16, 128>(a, __VA_ARGS__);                  \
  return fn<SB_F16, 256>(a, __VA_ARGS__)

hipError_t launch_select(const sb_select_args &a, int n_cu, void *work, hipStream_t s) { BY_TYPE_AND_SIZE(select, a, n_cu, work, s); }
hipError_t launch_selected_attention(const sb_selected_args &a, int n_cu, void *work, hipStream_t s) {
  BY_TYPE_AND_SIZE(attend, a, n_cu, work, s);
}

}  // namespace sb
