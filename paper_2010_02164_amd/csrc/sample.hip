// One token per row of logits under temperature, top-k, top-p and min-p,
// drawn with a given number. One workgroup per row.
//
// Every filter keeps a prefix of the tokens ranked by (-z, index), so the kept
// tokens are those above one cut (a logit and, among its equals, an index),
// and no row is sorted: a radix search over the ordered bits of the logits
// finds where a sum of counts (top-k) or of weights (top-p) passes its limit,
// and the draw is the same search over the kept tokens' indexes.
//
// Rows with top-k, or min-p alone, are read once where their likely tokens are spread
// over the vocabulary: a sample of the row (four runs of 512 neighbouring 16-byte
// pieces) gives a bound that the k-th largest logit then hardly ever is below, and
// the pass over the row lists the tokens from that bound on. A list of fewer than k
// sends the row the other way. So do likely tokens that gather in one of the runs
// (top-k 50 of 128000 in fp32: 30 us; with logits that fall as ln(1 + i / 100)
// with the index i 96). min-p alone bounds the tokens by the sample's largest.
// A short list is sorted, where every filter keeps a prefix; a longer one
// (up to 4096) is searched in registers and LDS. A row of 32000 logits in fp32
// takes 10.5 us, of which launching and reading it takes 6 (17.6 us where short
// lists were searched, too). 512 threads: two rows share a unit, and 320 rows
// run at once (1024 threads: 38 instead of 34 us; 29 since tokens are listed
// behind the pass instead of within it).
//
// Rows without top-k but with top-p need every weight. A pass adds them up into
// bins of equal ratio, which names the bin that the cut is in, a second lists
// that bin, a third draws; they read caches, and are bound by the 22 fp64 and
// integer operations of a weight. One workgroup took such a row 2 to 4 times as
// long as the others; with a workspace the passes run as kernels of their own,
// in chunks over all compute units: 512 rows of 128000 in fp32, part of them
// with top-k, 57 us in k_sample, 32, 8, 19 and 18 in the others. (A row's last
// chunk taking the next step in the same launch made 188 us into 1021: fences
// between the XCDs' caches cost more than launches.)
//
// Weights are whole multiples of 2^-44 in 64-bit integers: up to 2^18 of them
// add up without rounding or overflow, in any order, so that partial sums of
// waves and LDS atomics give one result. 44 bits below the largest weight
// keep the sum of 2^18 roundings under 2^-27 of it in the worst case and near
// 2^-36 in practice, below what u (24 bits) tells apart.
#include <algorithm>

#include "serve.h"
#include "wave.h"

namespace sb {
namespace {

typedef unsigned long long u64;
typedef unsigned int u4 __attribute__((ext_vector_type(4)));

constexpr int SM_THREADS = 512;
constexpr int SM_WAVES = SM_THREADS / 64;
constexpr double ONE = 0x1p44;        // the weight of the largest logit
constexpr int LIST_PER = 8, LIST_MAX = LIST_PER * SM_THREADS;
// Lists up to RANKED are sorted for top-p, up to half of it else (a row of 32000;
// top-k 20, a list of about 80: 12.6 us, searched 14.0, with top-p 12.8 and 17.2; 100,
// about 250: 16.1 and 15.5, with top-p 16.3 and 18.6; 200, 430: 19.5 and 16.3, 19.6
// and 19.4). From up to DIRECT kept tokens the draw compares indexes (5 kept: 10.3
// us, searched 11.2; 20: 12.6 and 12.6; 60: 16.6 and 14.3).
constexpr int RANKED = SM_THREADS, DIRECT = 24;
constexpr int BIN_BITS = 9, BINS = 1 << BIN_BITS;
constexpr int TAB_BITS = 9;           // 2^x by a table of 2^(i / 512) and a cubic
constexpr int TAB = 1 << TAB_BITS;
constexpr int CHUNK = 16384;          // tokens of a row that a workgroup of the wide kernels takes
constexpr int CHUNKS_MAX = SB_SAMPLE_MAX_VOCAB / CHUNK;
// The largest top-k that is read off the sample.
constexpr int SAMPLED_K = 1536;
// 16-byte pieces a thread loads at once: of the sample, and of a pass (4 there
// made the code of the passes larger than the instruction cache).
constexpr int SAMPLE = 4, PASS = 2, LOOK = 4;
constexpr int QUEUE = SAMPLE;   // pieces of a thread that its list takes after the pass
static_assert(SM_THREADS * QUEUE * 2 <= BINS * 8 && SB_SAMPLE_MAX_VOCAB / 4 <= 1 << 16, "the pieces' numbers fit the bins' place");

// The bits of z in an order that ascends with it; NaN counts as -inf.
__device__ __forceinline__ uint32_t order_bits(float z) {
  if (!(z >= -INFINITY)) z = -INFINITY;
  const uint32_t b = __float_as_uint(z + 0.0f);   // -0 is 0
  return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float from_order(uint32_t b) { return __uint_as_float(b ^ (b >> 31 ? 0x80000000u : 0xFFFFFFFFu)); }
constexpr uint32_t LOWEST = 0x007FFFFFu;   // order_bits(-inf)

// A row: elements before the first 16-byte address, whole pieces, the rest.
template <int DT>
struct Row {
  static constexpr int VEC = DT == SB_F32 ? 4 : 8, ES = DT == SB_F32 ? 4 : 2;
  const unsigned char *at;
  int V, head, pieces;
  __device__ __forceinline__ Row(const void *row, int n) : at(static_cast<const unsigned char *>(row)), V(n) {
    head = min((int)((16 - (reinterpret_cast<uintptr_t>(at) & 15)) & 15) / ES, V);
    pieces = (V - head) / VEC;
  }
  __device__ __forceinline__ float one(int i) const {
    if constexpr (DT == SB_F32) return reinterpret_cast<const float *>(at)[i];
    else return Half<DT>::to_float(reinterpret_cast<const uint16_t *>(at)[i]);
  }
  __device__ __forceinline__ u4 piece(int j) const { return *reinterpret_cast<const u4 *>(at + head * ES + (size_t)j * 16); }
  static __device__ __forceinline__ void unpack(const u4 &x, float (&z)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      if constexpr (DT == SB_F32) z[i] = __uint_as_float(x[i]);
      else z[i] = Half<DT>::to_float(i & 1 ? x[i >> 1] >> 16 : x[i >> 1] & 0xFFFFu);
    }
  }
  // f(z, i0) for pieces first, first + step, ... of [first, end): values i0 .. i0 + VEC - 1.
  template <int BATCH, typename F>
  __device__ __forceinline__ void each_piece(int first, int end, int step, F f) const {
#pragma unroll 1
    for (int j0 = first; j0 < end; j0 += BATCH * step) {
      u4 x[BATCH];
#pragma unroll
      for (int b = 0; b < BATCH; ++b)
        if (j0 + b * step < end) x[b] = piece(j0 + b * step);
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        if (j0 + b * step >= end) break;
        float z[VEC];
        unpack(x[b], z);
        f(z, head + (j0 + b * step) * VEC);
      }
    }
  }
  // The elements outside the pieces, one a thread, -inf in the other places.
  template <typename F>
  __device__ __forceinline__ void each_end(F f) const {
    const int rest = V - pieces * VEC;
    if ((int)threadIdx.x < rest) {
      const int i = (int)threadIdx.x < head ? (int)threadIdx.x : pieces * VEC + (int)threadIdx.x;
      float z[VEC];
      z[0] = one(i);
#pragma unroll
      for (int e = 1; e < VEC; ++e) z[e] = -INFINITY;
      f(z, i);
    }
  }
  template <int BATCH = PASS, typename F>
  __device__ __forceinline__ void each(F f) const {
    each_piece<BATCH>(threadIdx.x, pieces, SM_THREADS, f);
    each_end(f);
  }
};

struct Shared {
  double tab[TAB];             // 2^(44 + i / 512)
  u64 hist[BINS];
  u64 part[SM_WAVES], ends[2][8];
  alignas(16) uint32_t key[LIST_MAX];   // listed tokens: order bits
  int idx[LIST_MAX];                    // and indexes
  u64 rest, at_cut;
  uint32_t digit;
  int n, token;
};

// A row's weights: 2^44 exp((z - top) / T), rounded.
struct Weigher {
  const double *tab;
  double top, c;   // c = 512 log2(e) / T. With a largest logit of +inf: 2^128 and 512, far from all others
  __device__ __forceinline__ Weigher(const double *t, float largest, float T)
      : tab(t), top(largest == INFINITY ? 0x1p128 : (double)largest),
        c(largest == INFINITY ? TAB : TAB * 1.4426950408889634074 / (double)T) {}
  // 512 log2 of the weight (of the largest: 0). NaN, and -inf with T = inf: the lowest.
  static constexpr double LOW = -64.0 * TAB;
  __device__ __forceinline__ double log2w(float z) const { return fmin(fmax(((double)z - top) * c, LOW), 0.0); }
  // x = n + r with |r| <= 1/2: 2^(x / 512) = 2^(n / 512) (1 + r ln 2 / 512 + ...);
  // the cubic leaves out (2^-10 ln 2)^4 / 24 = 2^-46.7. The result as the bits of
  // 2^52 + weight, whose last bits are the weight rounded to a whole number.
  static constexpr u64 RAW = 0x4330000000000000ull;   // those of 2^52
  __device__ __forceinline__ u64 raw(double x) const {
    constexpr double MAGIC = 0x1.8p52, A = 0.69314718055994531 / TAB;
    const double t = x + MAGIC;
    const int n = __double2loint(t);
    const double r = x - (t - MAGIC);
    const double y = fma(fma(fma(r, A * A * A / 6.0, A * A / 2.0), r, A), r, 1.0);
    return (u64)__double_as_longlong(ldexp(tab[n & (TAB - 1)] * y, n >> TAB_BITS) + 0x1p52);
  }
  __device__ __forceinline__ u64 of(double x) const { return raw(x) - RAW; }
  __device__ __forceinline__ u64 operator()(float z) const { return of(log2w(z)); }
};
template <typename S>
__device__ __forceinline__ void fill_table(S &sh) {
  if (threadIdx.x < TAB) sh.tab[threadIdx.x] = exp2(44.0 + threadIdx.x * (1.0 / TAB));
}

// Sums and maxima over a wave through the lanes' own paths (a shuffle through
// LDS takes about 130 cycles, and a search has dozens of steps).
template <int S>
__device__ __forceinline__ u64 sum_stage(u64 v) {
  u64 a, b;
  stage64<S>(v, a, b);
  return a + b;
}
__device__ __forceinline__ u64 wave_sum(u64 v) {
  return sum_stage<5>(sum_stage<4>(sum_stage<3>(sum_stage<2>(sum_stage<1>(sum_stage<0>(v))))));
}
template <int S>
__device__ __forceinline__ uint32_t max_stage(uint32_t v) {
  uint32_t a, b;
  stage32<S>(v, a, b);
  return max(a, b);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  return max_stage<5>(max_stage<4>(max_stage<3>(max_stage<2>(max_stage<1>(max_stage<0>(v))))));
}
template <typename S>
__device__ __forceinline__ u64 block_sum(u64 v, S &sh) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = v;
  __syncthreads();
  u64 s = 0;
#pragma unroll
  for (int i = 0; i < SM_WAVES; ++i) s += sh.part[i];
  return s;
}
__device__ __forceinline__ uint32_t block_max(uint32_t v, Shared &sh) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < SM_WAVES; ++i) v = max(v, (uint32_t)sh.part[i]);
  return v;
}

__device__ __forceinline__ void clear_bins(Shared &sh) {
  __syncthreads();
  if (threadIdx.x < BINS) sh.hist[threadIdx.x] = 0;
  __syncthreads();
}
// The bin at which the bins' sum, from bin 0 up, first passes `limit`; the last
// one where it never does. rest: limit less what lies before the bin; at: what
// is in it.
__device__ __forceinline__ uint32_t find_bin(u64 limit, u64 &rest, u64 &at, Shared &sh) {
  constexpr int PER = BINS / 64;
  __syncthreads();
  if (threadIdx.x < 64) {
    u64 h[PER], s = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) s += h[j] = sh.hist[threadIdx.x * PER + j];
    u64 before = wave_scan(s) - s;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const bool last = threadIdx.x == 63 && j == PER - 1;
      if (before <= limit && (limit < before + h[j] || last)) {
        sh.digit = threadIdx.x * PER + j;
        sh.rest = limit - before;
        sh.at_cut = h[j];
      }
      before += h[j];
    }
  }
  __syncthreads();
  rest = sh.rest;
  at = sh.at_cut;
  return sh.digit;
}

// Each thread's share of a list, in registers.
struct Items {
  uint32_t key[LIST_PER];
  int idx[LIST_PER];
  u64 w[LIST_PER];   // 0: not there, or not kept
};

// The key at which the items' weights, in ascending order of their keys, first
// total more than `limit`, which they do. keys < 2^bits.
template <typename K>
__device__ __forceinline__ uint32_t list_search(const Items &it, K key, int bits, u64 limit, u64 &rest, u64 &at, Shared &sh) {
  uint32_t prefix = 0;
  int shift = bits;
  do {
    const int take = min(BIN_BITS, shift);
    shift -= take;
    clear_bins(sh);
#pragma unroll
    for (int j = 0; j < LIST_PER; ++j) {
      const uint32_t k = key(j);
      if (it.w[j] && (shift + take >= 32 || (k >> (shift + take)) == prefix)) atomicAdd(&sh.hist[(k >> shift) & ((1u << take) - 1)], it.w[j]);
    }
    prefix = (prefix << take) | find_bin(limit, rest, at, sh);
    limit = rest;
  } while (shift > 0);
  return prefix;
}

// Likewise over the row's tokens, from the largest logit down, 8 bits a pass;
// weight(z) is a token's weight. For rows whose cut lies among more equal
// or nearly equal logits than the list holds.
template <int DT, typename F>
__device__ __forceinline__ uint32_t row_search(const Row<DT> &row, u64 limit, F weight, u64 &rest, u64 &at, Shared &sh) {
  uint32_t prefix = 0;
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    clear_bins(sh);
    row.each([&](const float (&z)[Row<DT>::VEC], int) {
#pragma unroll
      for (int e = 0; e < Row<DT>::VEC; ++e) {
        const uint32_t b = order_bits(z[e]), d = ~b;
        if (shift == 24 || (d >> (shift + 8)) == prefix) {
          const u64 w = weight(z[e]);
          if (w) atomicAdd(&sh.hist[(d >> shift) & 255u], w);
        }
      }
    });
    prefix = (prefix << 8) | find_bin(limit, rest, at, sh);
    limit = rest;
  }
  return ~prefix;
}

// The smallest index up to which the weights total more than limit(total),
// which they do; weights(z, i0, w) gives those of a piece, each + RAW. Each wave adds up a
// stretch of pieces (the row's ends are stretches of their own), then all
// threads share the stretch that passes the limit.
template <int DT, typename F, typename L>
__device__ __forceinline__ int locate(const Row<DT> &row, F weights, L limit_of, u64 &total, Shared &sh) {
  constexpr int VEC = Row<DT>::VEC;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int len = (row.pieces + SM_WAVES - 1) / SM_WAVES;   // pieces a wave
  u64 s = 0;
  row.template each_piece<PASS>(min(w * len, row.pieces) + lane, min((w + 1) * len, row.pieces), 64, [&](const float (&z)[VEC], int i0) {
    u64 x[VEC];
    weights(z, i0, x);
#pragma unroll
    for (int e = 0; e < VEC; ++e) s += x[e];
    s -= VEC * Weigher::RAW;
  });
  s = wave_sum(s);
  __syncthreads();
  if (lane == 0) sh.part[w] = s;
  // Ends: a wave each, one token a lane.
  if (w < 2) {
    const int i0 = w == 0 ? 0 : row.head + row.pieces * VEC, count = w == 0 ? row.head : row.V - i0;
    u64 x[VEC];
    float z[VEC];
    z[0] = lane < count ? row.one(i0 + lane) : -INFINITY;
#pragma unroll
    for (int e = 1; e < VEC; ++e) z[e] = -INFINITY;
    weights(z, i0 + lane, x);
    x[0] = wave_scan(x[0] - Weigher::RAW);
    if (lane < 8) sh.ends[w][lane] = x[0];   // (up to 7 tokens)
  }
  __syncthreads();
  const u64 first = sh.ends[0][7], last = sh.ends[1][7];
  total = first + last;
#pragma unroll
  for (int i = 0; i < SM_WAVES; ++i) total += sh.part[i];
  u64 limit = limit_of(total), before = first;
  if (limit < first || limit >= total - last) {
    const int e = limit < first ? 0 : 1;
    if (e == 1) limit -= total - last;
    int i = 0;
    while (i < 7 && sh.ends[e][i] <= limit) ++i;
    return (e == 0 ? 0 : row.head + row.pieces * VEC) + i;
  }
  int x = 0;
  while (x < SM_WAVES - 1 && before + sh.part[x] <= limit) before += sh.part[x++];
  limit -= before;
  // The stretch in threads' shares of neighbouring pieces, walked twice: for
  // their sums, then by the thread that passes the limit.
  const int lo = min(x * len, row.pieces), hi = min(lo + len, row.pieces), per = (hi - lo + SM_THREADS - 1) / SM_THREADS;
  const int a0 = min(lo + (int)threadIdx.x * per, hi);
  int a1 = min(a0 + per, hi);
  u64 run = 0, mine = 0;
#pragma unroll 1
  for (int turn = 0; turn < 2; ++turn) {
#pragma unroll 1
    for (int j = a0; j < a1; ++j) {
      float z[VEC];
      u64 y[VEC];
      Row<DT>::unpack(row.piece(j), z);
      weights(z, row.head + j * VEC, y);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const u64 x = y[e] - Weigher::RAW;
        if (turn == 1 && run <= limit && limit < run + x) sh.token = row.head + j * VEC + e;
        run += x;
      }
    }
    if (turn == 1) break;
    mine = run;
    u64 upto = wave_scan(mine);
    __syncthreads();
    if (lane == 63) sh.part[w] = upto;
    __syncthreads();
    for (int i = 0; i < w; ++i) upto += sh.part[i];
    run = upto - mine;
    if (run > limit || limit >= upto) a1 = a0;
  }
  __syncthreads();
  return sh.token;
}

// Takes this thread's share of the list; weight(bits).
template <typename F>
__device__ __forceinline__ void take_list(Items &it, int n, F weight, const Shared &sh) {
#pragma unroll
  for (int j = 0; j < LIST_PER; ++j) {
    const int at = j * SM_THREADS + threadIdx.x;
    const bool on = at < n;
    it.key[j] = on ? sh.key[at] : 0;
    it.idx[j] = on ? sh.idx[at] : 0;
    it.w[j] = on ? weight(it.key[j]) : 0;
  }
}

__device__ __forceinline__ void list_token(uint32_t bits, int i, Shared &sh) {
  const int at = atomicAdd(&sh.n, 1);
  if (at < LIST_MAX) {
    sh.key[at] = bits;
    sh.idx[at] = i;
  }
}

// A short list sorted by (-z, index): each token counts those before it (a search
// would pass four barriers for each of its digits).
struct Ranked {   // the token of rank threadIdx.x
  uint32_t key;
  int idx;
  u64 w, before;   // its weight (0: not there), and what those before it total
};
template <typename F>
__device__ __forceinline__ Ranked rank_list(int n, F weight, Shared &sh) {
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  // Behind the list: keys by rank, equals in any order and then by their indexes.
  uint32_t *keys = sh.key + 2 * RANKED, *sharing = sh.key + 3 * RANKED;
  int *any_order = sh.idx + 2 * RANKED, *sorted = sh.idx + 3 * RANKED;
  if (tid < 4) sh.key[n + tid] = 0;   // before none
  sharing[tid] = 0;
  if (tid == 0) sh.at_cut = 0, sh.digit = 0;
  __syncthreads();
  int rank = 0;
  const uint32_t key = sh.key[tid];
  const int idx = sh.idx[tid];
  if (tid < n) {
#pragma unroll 4
    for (int x = 0; x < n; x += 4) {
      const u4 k = *reinterpret_cast<const u4 *>(&sh.key[x]);
#pragma unroll
      for (int e = 0; e < 4; ++e) rank += k[e] > key;
    }
    const int at = rank + (int)atomicAdd(&sharing[rank], 1u);
    keys[at] = key;
    any_order[at] = idx;
  }
  __syncthreads();
  if (tid < n) {
    const int equals = (int)sharing[rank];
    int at = rank;
    if (equals > 1)
#pragma unroll 4
      for (int x = 0; x < equals; ++x) at += any_order[rank + x] < idx;
    sorted[at] = idx;
  }
  __syncthreads();
  Ranked me = {0, 0, 0, 0};
  if (tid < n) {
    me.key = keys[tid];
    me.idx = sorted[tid];
    me.w = weight(me.key);
  }
  const u64 upto = wave_scan(me.w);
  if (lane == 63) sh.part[wv] = upto;
  __syncthreads();
  me.before = upto - me.w;
#pragma unroll
  for (int i = 0; i < SM_WAVES; ++i) me.before += i < wv ? sh.part[i] : 0;
  return me;
}

__device__ __forceinline__ int bits_of(uint32_t x) { return 32 - __clz((int)x); }   // x < 2^bits; 0 for 0

// Leaves the listed tokens up to the cut at best - d, of its equals the first
// before / each + 1 (`at`: what they total). Returns the last index of those
// that stay, V if all do.
__device__ __forceinline__ int cut_list(Items &it, uint32_t best, uint32_t d, u64 before, u64 each, u64 at, int V, Shared &sh) {
  int last = V;
  if (at > before + each) {   // not all of its equals stay
    Items eq = it;
#pragma unroll
    for (int j = 0; j < LIST_PER; ++j) eq.w[j] = it.w[j] && best - it.key[j] == d;
    u64 rest, a2;
    last = (int)list_search(eq, [&](int j) { return (uint32_t)eq.idx[j]; }, bits_of(V - 1), before / each, rest, a2, sh);
  }
#pragma unroll
  for (int j = 0; j < LIST_PER; ++j) {
    const uint32_t dj = best - it.key[j];
    if (dj > d || (dj == d && it.idx[j] > last)) it.w[j] = 0;
  }
  return last;
}

struct Params {
  float T, p, mp, u;   // p: 1 where it keeps all; mp: 0 likewise, at most 1
  int k;               // 0 where it keeps all
  bool greedy;
  __device__ __forceinline__ Params(const sb_sample_args &a, int r) {
    T = a.temperature ? a.temperature[r] : 1.0f;
    k = a.top_k && a.top_k[r] > 0 && a.top_k[r] < a.vocab ? a.top_k[r] : 0;
    p = a.top_p && a.top_p[r] < 1.0f ? a.top_p[r] : 1.0f;
    mp = a.min_p && a.min_p[r] > 0.0f ? fminf(a.min_p[r], 1.0f) : 0.0f;
    u = a.u[r] > 0.0f ? fminf(a.u[r], 1.0f) : 0.0f;
    greedy = !(T > 0.0f);
  }
  __device__ __forceinline__ u64 draw_limit(u64 total) const { return min((u64)((double)u * (double)total), total - 1); }
  // Kept where the weights ranked before total less than p z_k, so at most
  // this: the cut is where they first total more.
  __device__ __forceinline__ u64 top_p_limit(u64 z_k) const { return (u64)fmax(ceil((double)p * (double)z_k), 1.0) - 1; }
  // Weights below (1 - p) / V of the largest total less than 1 - p of all: the
  // cut is not among those further below it than this (two octaves to spare
  // for rounding).
  __device__ __forceinline__ double top_p_reach(int V) const {
    return fmin(TAB * (2.0 + log2((double)V / fmax(1.0 - (double)p, 1e-9))), -Weigher::LOW);
  }
};

// The draw from a short list that holds every token that may be kept.
__device__ __forceinline__ int draw_ranked(int n, const Params &pr, const Weigher &weigh, int V, u64 &total, Shared &sh) {
  const Ranked me = rank_list(n, [&](uint32_t b) { return weigh(from_order(b)); }, sh);
  if (pr.greedy) {
    total = (u64)ONE;
    if (threadIdx.x == 0) sh.token = me.idx;
    __syncthreads();
    return sh.token;
  }
  const int keep = pr.k > 0 ? min(pr.k, n) : n;
  u64 limit = ~0ull;
  if (pr.p < 1.0f) {
    if ((int)threadIdx.x == keep - 1) sh.rest = me.before + me.w;
    __syncthreads();
    limit = pr.top_p_limit(sh.rest);
  }
  // Every filter leaves the first so many.
  const bool kept = (int)threadIdx.x < keep && me.before <= limit && me.w >= (u64)ceil((double)pr.mp * ONE) && me.w > 0;
  const u64 on = __ballot(kept);
  if (on && (int)(threadIdx.x & 63) == 63 - __builtin_clzll(on)) {   // the wave's last
    atomicAdd(&sh.digit, (uint32_t)__popcll(on));
    atomicMax(&sh.at_cut, me.before + me.w);
  }
  sh.hist[threadIdx.x] = kept ? me.w : 0;
  __syncthreads();
  const int m = (int)sh.digit;
  total = sh.at_cut;
  limit = pr.draw_limit(total);
  if (m > DIRECT) {
    Items it;
#pragma unroll
    for (int j = 1; j < LIST_PER; ++j) it.w[j] = 0, it.idx[j] = 0;
    it.idx[0] = me.idx;
    it.w[0] = kept ? me.w : 0;
    u64 rest, at;
    return (int)list_search(it, [&](int j) { return (uint32_t)it.idx[j]; }, bits_of(V - 1), limit, rest, at, sh);
  }
  if (kept) {   // what the kept tokens of lower indexes total
    const int *sorted = sh.idx + 3 * RANKED;
    u64 before = 0;
#pragma unroll 4
    for (int x = 0; x < m; ++x) before += sorted[x] < me.idx ? sh.hist[x] : 0;
    if (before <= limit && limit < before + me.w) sh.token = me.idx;
  }
  __syncthreads();
  return sh.token;
}

// What is kept of a row: logits above `lo`, and those equal to it with an
// index up to `last`. (Never NaN or -inf.)
struct Cut {
  static constexpr int ALL = 0x7FFFFFFF;
  float lo = -3.4028234663852886e38f;
  int last = ALL;
  __device__ __forceinline__ float masked(float z, int i) const {
    float y = z >= lo ? z : -INFINITY;
    if (last != ALL) y = ((z == lo) & (i > last)) ? -INFINITY : y;
    return y;
  }
  __device__ __forceinline__ void raise(float z) {
    if (z > lo) {
      lo = z;
      last = ALL;
    }
  }
};

// The lowest order bits in [lo, hi] that pred holds for; from there on it
// holds, at hi it does. The lanes of a wave try 64 at once.
template <typename P>
__device__ __forceinline__ uint32_t first_bits(uint32_t lo, uint32_t hi, P pred) {
  while (lo < hi) {
    const uint32_t step = (hi - lo) / 64 + 1, mid = lo + (threadIdx.x & 63) * step;
    const u64 m = __ballot(pred(min(mid, hi)));
    const int f = m ? __builtin_ctzll(m) : 64;
    if (f < 64) hi = min(lo + f * step, hi);
    if (f > 0) lo = min(lo + (f - 1) * step + 1, hi);
    else hi = lo;
  }
  return lo;
}

// The lowest logit that min-p keeps.
__device__ __forceinline__ float min_p_logit(const Params &pr, const Weigher &weigh, uint32_t best) {
  const u64 floor_w = (u64)ceil((double)pr.mp * ONE);
  return from_order(first_bits(LOWEST, best, [&](uint32_t b) { return weigh(from_order(b)) >= floor_w; }));
}

// Bins of equal ratio, from the largest weight down to the smallest one there
// is, or that can matter; what is below in the last.
struct Bins {
  double scale;
  __device__ __forceinline__ Bins(const Weigher &weigh, float low, double reach)
      : scale((BINS - 2) / fmin(fmax(-weigh.log2w(low), 0.05), reach)) {}
  __device__ __forceinline__ int of(double x) const { return min(__double2loint(fma(x, -scale, 0x1.8p52)), BINS - 1); }   // to the nearest
  // The bin's logits lie in [first, last]: bins fall as logits rise.
  __device__ __forceinline__ void range(const Weigher &weigh, int bin, uint32_t best, uint32_t &first, uint32_t &last) const {
    auto from = [&](int most) { return first_bits(LOWEST, best, [&](uint32_t b) { return of(weigh.log2w(from_order(b))) <= most; }); };
    first = max(from(bin), LOWEST + 1);
    last = bin > 0 ? from(bin - 1) - 1 : best;
  }
};

// A pass that adds a row's (or a chunk's) kept weights, or counts, into sh.hist;
// all: their sum. i_off: the index of the row's first token.
template <int DT>
__device__ __forceinline__ void add_bins(const Row<DT> &row, int i_off, const Weigher &weigh, const Bins &bins, const Cut &cut, bool count,
                                         u64 &all, Shared &sh) {
  constexpr int VEC = Row<DT>::VEC;
  clear_bins(sh);
  u64 below = 0;
  all = 0;
  row.each([&](const float (&z)[VEC], int i0) {
    u64 w[VEC];
    int at[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {   // no branches here: the tokens' chains of operations run side by side
      const float y = cut.masked(z[e], i_off + i0 + e);
      const double x = weigh.log2w(y);
      w[e] = count ? (u64)(y > -INFINITY) : weigh.of(x);
      at[e] = bins.of(x);
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      all += w[e];
      if (at[e] < BINS - 1) {
        if (w[e]) atomicAdd(&sh.hist[at[e]], w[e]);
      } else {
        below += w[e];
      }
    }
  });
  below = block_sum(below, sh);
  all = block_sum(all, sh);
  if (threadIdx.x == 0) sh.hist[BINS - 1] = below;
}

// A pass that lists the kept tokens with logits from z_lo to z_hi in LDS;
// returns how many there are.
template <int DT>
__device__ __forceinline__ int list_range(const Row<DT> &row, int i_off, float z_lo, float z_hi, const Cut &cut, Shared &sh) {
  constexpr int VEC = Row<DT>::VEC;
  if (threadIdx.x == 0) sh.n = 0;
  __syncthreads();
  row.each([&](const float (&z)[VEC], int i0) {
    float m = z[0];
#pragma unroll
    for (int e = 1; e < VEC; ++e) m = fmaxf(m, z[e]);
    if (!(m >= z_lo)) return;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float y = cut.masked(z[e], i_off + i0 + e);
      if (y >= z_lo && y <= z_hi) list_token(order_bits(y), i_off + i0 + e, sh);
    }
  });
  __syncthreads();
  return sh.n;
}

// A piece's kept weights, + RAW. A wave without kept tokens takes none.
template <int VEC>
__device__ __forceinline__ void kept_weights(const float (&z)[VEC], int i, const Weigher &weigh, const Cut &cut, u64 (&w)[VEC]) {
  float m = z[0];
#pragma unroll
  for (int e = 1; e < VEC; ++e) m = fmaxf(m, z[e]);
#pragma unroll
  for (int e = 0; e < VEC; ++e) w[e] = Weigher::RAW;
  if (!(m >= cut.lo)) return;
#pragma unroll
  for (int e = 0; e < VEC; ++e) w[e] = weigh.raw(weigh.log2w(cut.masked(z[e], i + e)));
}

// A whole row by one workgroup, any filters: top-k by counts, top-p by weights,
// then the draw; one code for all, its passes being much of the kernels'.
template <int DT>
__device__ __forceinline__ int wide_row(const Row<DT> &row, const Params &pr, const Weigher &weigh, uint32_t best, float low, u64 &total, Shared &sh) {
  constexpr int VEC = Row<DT>::VEC;
  Cut cut;
  int token = 0;
#pragma unroll 1
  for (int stage = pr.greedy ? 2 : 0; stage < 3; ++stage) {
    const bool count = stage == 0;
    uint32_t bits = 0;
    u64 limit = 0;
    if (stage < 2) {
      if (count ? pr.k == 0 : pr.p == 1.0f) continue;
      const Bins bins(weigh, low, count ? -Weigher::LOW : pr.top_p_reach(row.V));
      u64 all, rest, at;
      add_bins<DT>(row, 0, weigh, bins, cut, count, all, sh);
      limit = count ? (u64)(pr.k - 1) : pr.top_p_limit(all);
      if (limit >= all) continue;
      uint32_t first, last;
      bins.range(weigh, (int)find_bin(limit, rest, at, sh), best, first, last);
      const int m = list_range<DT>(row, 0, from_order(first), from_order(last), cut, sh);
      if (m <= LIST_MAX) {
        Items it;
        take_list(it, m, [&](uint32_t b) { return count ? (u64)1 : weigh(from_order(b)); }, sh);
        bits = best - list_search(it, [&](int j) { return best - it.key[j]; }, 32, rest, rest, at, sh);
      } else {   // (all equals of the cut: kept ones and others weigh the same, and the limit is among the kept)
        bits = row_search<DT>(row, limit, [&](float z) { return z >= cut.lo ? count ? (u64)1 : weigh(z) : 0; }, rest, at, sh);
      }
      const u64 each = count ? 1 : weigh(from_order(bits));
      const float z = from_order(bits);
      if (at <= rest + each) {   // all of the cut's equals stay
        cut.raise(z);
        continue;
      }
      limit = rest / each;   // the first so many of them, and one
    } else if (pr.greedy) {
      bits = best;
    } else if (pr.mp > 0.0f) {
      cut.raise(min_p_logit(pr, weigh, best));
    }
    const int found = locate<DT>(
        row,
        [&](const float (&z)[VEC], int i0, u64 (&w)[VEC]) {
          if (!bits) return kept_weights<VEC>(z, i0, weigh, cut, w);
#pragma unroll
          for (int e = 0; e < VEC; ++e) w[e] = Weigher::RAW + (order_bits(z[e]) == bits);
        },
        [&](u64 t) { return bits ? limit : pr.draw_limit(t); }, total, sh);
    if (stage == 2) {
      token = found;
    } else {
      const float z = from_order(bits);
      cut.last = z > cut.lo ? found : min(cut.last, found);
      cut.lo = z;
    }
  }
  if (pr.greedy) total = (u64)ONE;
  return token;
}

__device__ __forceinline__ void put_token(const sb_sample_args &a, int r, int token, float z, float top, const Params &pr, u64 total) {
  if (threadIdx.x != 0) return;
  a.tokens[r] = token;
  const double x = pr.greedy || top == INFINITY ? 0.0 : ((double)z - (double)top) / (double)pr.T;
  if (a.logprobs) a.logprobs[r] = (float)(x - log((double)total / ONE));
}

// A row that the wide kernels take: in the workspace, one a row.
struct WideRow {
  int kind;                 // 0: not such a row, 1: top-p, 2: no cut but min-p's
  int n;                    // listed tokens (more than LIST_MAX: not all of them are)
  int pad[2];
  uint32_t best;            // order bits of the largest logit
  float low;                // the smallest finite one
  // Top-p, from k_wide_cut on: whether the cut leaves tokens out, the order bits
  // of the bin that it is in, and what of its limit is left there.
  int cut;
  uint32_t first, last;
  float z_mp;               // the lowest logit that min-p keeps
  u64 rest;
  u64 totals[CHUNKS_MAX];   // kept weights of a chunk, without the listed ones
  uint32_t key[LIST_MAX];
  int idx[LIST_MAX];
};
static_assert(RANKED <= BINS && LIST_MAX >= 4 * RANKED, "room for what is sorted behind the list, and for its weights");
static_assert(sizeof(WideRow) % 16 == 0, "rows of the workspace stay aligned");
__host__ __device__ __forceinline__ int chunks_of(int V) { return (V + CHUNK - 1) / CHUNK; }
// Behind them: a chunk's bins. (Atomics on one set of a row's took as long as
// the weights.)
__device__ __forceinline__ u64 *bins_at(const sb_sample_args &a, WideRow *wide, int r, int c) {
  return reinterpret_cast<u64 *>(wide + a.rows) + ((size_t)r * chunks_of(a.vocab) + c) * BINS;
}

template <int DT>
__device__ __forceinline__ const unsigned char *row_at(const sb_sample_args &a, int r) {
  return static_cast<const unsigned char *>(a.logits) + (size_t)r * a.row_stride * Row<DT>::ES;
}

template <int DT>
__global__ __launch_bounds__(SM_THREADS, 4) void k_sample(sb_sample_args a, WideRow *wide) {
  constexpr int VEC = Row<DT>::VEC;
  __shared__ Shared sh;
  const int r = blockIdx.x, V = a.vocab, tid = threadIdx.x;
  const Row<DT> row(row_at<DT>(a, r), V);
  const Params pr(a, r);
  const int k = pr.k;
  const float p = pr.p, mp = pr.mp;
  const bool greedy = pr.greedy;

  // The sample: SAMPLE pieces a thread, from as many places of the row.
  const int apart = max((row.pieces + SAMPLE - 1) / SAMPLE, SM_THREADS);
  u4 x[SAMPLE];
  float zs[2] = {-INFINITY, -INFINITY};   // the largest of each half of this thread's
#pragma unroll
  for (int b = 0; b < SAMPLE; ++b) {
    const int j = b * apart + tid;
    if (j < row.pieces) x[b] = row.piece(j);
  }
  fill_table(sh);   // while they are on their way
#pragma unroll
  for (int b = 0; b < SAMPLE; ++b) {
    const int j = b * apart + tid;
    if (j < row.pieces) {
      float z[VEC];
      Row<DT>::unpack(x[b], z);
#pragma unroll
      for (int e = 0; e < VEC; ++e) zs[b & 1] = fmaxf(zs[b & 1], z[e]);
    }
  }
  if (tid == 0) {
    sh.n = 0;
    if (wide) wide[r].kind = 0;
  }
  const uint32_t seen = block_max(order_bits(fmaxf(zs[0], zs[1])), sh);   // (its barriers also publish the table and n)
  // Whether the tokens that matter are read off the sample, and from which on.
  const bool sampled = greedy || (k > 0 && k <= SAMPLED_K) || (k == 0 && p == 1.0f && mp > 0.0f);
  float bound = -INFINITY;
  bool sure = true;   // nothing that matters lies below the bound
  if (greedy) {
    bound = from_order(seen);
  } else if (sampled) {
    if (k > 0) {
      // Read off the sample as the k-th largest is off the row, or a lower
      // one (of k tokens, the sample's share and five times its spread, and 6)
      // where that lists fewer: no bound in itself, so the list is counted.
      const float share = (float)(min(SAMPLE * SM_THREADS, row.pieces) * VEC) / (float)V, kf = (float)k * share;
      const int want = min(k, (int)(kf + 5.0f * sqrtf(kf)) + 6);
      sure = want == k;
      // To a sixteenth of its distance (in order bits) from the largest, away
      // from that, which keeps it a bound: bins of four bits and an exponent.
      clear_bins(sh);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t d = seen - order_bits(zs[j]), e = 31 - __clz((int)(d | 16));   // e >= 4
        atomicAdd(&sh.hist[(e - 4) * 16 + (d >> (e - 4))], 1ull);
      }
      u64 rest, at;
      const uint32_t bin = find_bin((u64)(want - 1), rest, at, sh), e4 = bin < 32 ? 0 : bin / 16 - 1;
      const u64 d = ((u64)(bin - e4 * 16) + 1 << e4) - 1;   // the furthest of the bin
      bound = from_order(seen - (uint32_t)min(d, (u64)(seen - LOWEST)));
    }
    // min-p keeps the weights that round to min_p or more, half a step of theirs
    // below it (at least half a step): z >= top + T ln(min_p - 2^-45), top at least
    // the sample's (less a little for the rounding here).
    if (p == 1.0f && mp > 0.0f && from_order(seen) < INFINITY) {
      const double m = from_order(seen), t = (double)pr.T * log(fmax((double)mp - 0x1p-45, 0x1p-45));
      const float bf = (float)(m + t - 1e-6 * (fabs(m) + fabs(t)) - 1e-30);
      sure |= bf >= bound;
      bound = fmaxf(bound, bf);
    }
  }

  // The pass over the row: its largest logit, its smallest finite one, and
  // the tokens from the bound on.
  float zm = -INFINITY, zl = INFINITY;
  uint16_t *mine = reinterpret_cast<uint16_t *>(sh.hist) + tid * QUEUE;   // pieces of this thread with such tokens: listed
  int queued = 0;                                                         // behind the pass, which waits for nothing so
  auto list_piece = [&](const float (&z)[VEC], int i0) {
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (z[e] >= bound && z[e] > -INFINITY) list_token(order_bits(z[e]), i0 + e, sh);
  };
  auto look = [&](const float (&z)[VEC], int i0) {
    float m = z[0];
#pragma unroll
    for (int e = 1; e < VEC; ++e) m = fmaxf(m, z[e]);
    zm = fmaxf(zm, m);
    if (sampled) {
      if (m >= bound && m > -INFINITY) {
        if (queued < QUEUE) mine[queued++] = (uint16_t)((i0 - row.head) / VEC);
        else list_piece(z, i0);
      }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) zl = fminf(zl, z[e] > -INFINITY ? z[e] : INFINITY);
    }
  };
#pragma unroll
  for (int b = 0; b < SAMPLE; ++b) {
    const int j = b * apart + tid;
    if (j < row.pieces) {
      float z[VEC];
      Row<DT>::unpack(x[b], z);
      look(z, row.head + j * VEC);
    }
  }
  if (apart > SM_THREADS)
#pragma unroll 1
    for (int b = 0; b < SAMPLE; ++b) row.template each_piece<LOOK>(b * apart + SM_THREADS + tid, min((b + 1) * apart, row.pieces), SM_THREADS, look);
  if (sampled) {
#pragma unroll
    for (int b = 0; b < QUEUE; ++b)
      if (b < queued) x[b] = row.piece(mine[b]);
    int hits = 0;
#pragma unroll
    for (int b = 0; b < QUEUE; ++b) {
      if (b >= queued) break;
      float z[VEC];
      Row<DT>::unpack(x[b], z);
#pragma unroll
      for (int e = 0; e < VEC; ++e) hits += z[e] >= bound && z[e] > -INFINITY;
    }
    int at = hits ? atomicAdd(&sh.n, hits) : 0;
#pragma unroll
    for (int b = 0; b < QUEUE; ++b) {
      if (b >= queued) break;
      float z[VEC];
      Row<DT>::unpack(x[b], z);
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (z[e] >= bound && z[e] > -INFINITY) {
          if (at < LIST_MAX) {
            sh.key[at] = order_bits(z[e]);
            sh.idx[at] = row.head + mine[b] * VEC + e;
          }
          ++at;
        }
    }
  }
  row.each_end([&](const float (&z)[VEC], int i) {
    zm = fmaxf(zm, z[0]);
    if (sampled) list_piece(z, i);
    else zl = fminf(zl, z[0] > -INFINITY ? z[0] : INFINITY);
  });
  const uint32_t best = block_max(order_bits(zm), sh);
  if (best == LOWEST) {
    if (tid == 0) {
      a.tokens[r] = -1;
      if (a.logprobs) a.logprobs[r] = -INFINITY;
    }
    return;
  }
  const float top = from_order(best);
  const Weigher weigh(sh.tab, top, pr.T);
  int token = 0;
  u64 total = 1;
  const int n = sh.n;
  const bool listed = sampled && (sure || n >= k);
  if (listed && n <= (p < 1.0f ? RANKED : RANKED / 2)) {
    token = draw_ranked(n, pr, weigh, V, total, sh);
  } else if (listed && n <= LIST_MAX) {
    Items it;
    take_list(it, n, [&](uint32_t b) { return greedy ? (u64)(b == best) : weigh(from_order(b)); }, sh);
    if (!greedy) {
      const int bits = bits_of(best - order_bits(bound));
      if (k > 0 && k < n) {
        Items count = it;
#pragma unroll
        for (int j = 0; j < LIST_PER; ++j) count.w[j] = j * SM_THREADS + tid < n;
        u64 rest, at;
        const uint32_t d = list_search(count, [&](int j) { return best - count.key[j]; }, bits, (u64)(k - 1), rest, at, sh);
        cut_list(it, best, d, rest, 1, at, V, sh);
      }
      if (p < 1.0f) {
        u64 s = 0;
#pragma unroll
        for (int j = 0; j < LIST_PER; ++j) s += it.w[j];
        const u64 z_k = block_sum(s, sh), limit = pr.top_p_limit(z_k);
        if (limit < z_k) {
          u64 rest, at;
          const uint32_t d = list_search(it, [&](int j) { return best - it.key[j]; }, bits, limit, rest, at, sh);
          cut_list(it, best, d, rest, weigh(from_order(best - d)), at, V, sh);
        }
      }
      const u64 floor_w = (u64)ceil((double)mp * ONE);
#pragma unroll
      for (int j = 0; j < LIST_PER; ++j)
        if (it.w[j] < floor_w) it.w[j] = 0;
    }
    u64 s = 0, rest, at;
#pragma unroll
    for (int j = 0; j < LIST_PER; ++j) s += it.w[j];
    total = block_sum(s, sh);
    token = (int)list_search(it, [&](int j) { return (uint32_t)it.idx[j]; }, bits_of(V - 1), greedy ? 0 : pr.draw_limit(total), rest, at, sh);
    if (greedy) total = (u64)ONE;
  } else {
    const float low = sampled ? -INFINITY : -from_order(block_max(order_bits(-zl), sh));   // (sampled: not looked for)
    if (wide && k == 0 && !greedy) {
      WideRow &w = wide[r];
      if (tid == 0) {
        w.kind = p < 1.0f ? 1 : 2;
        w.n = 0;
        w.best = best;
        w.low = low;
        w.cut = 0;
      }
      return;
    }
    token = wide_row<DT>(row, pr, weigh, best, low, total, sh);
  }
  put_token(a, r, token, row.one(token), top, pr, total);
}

// The wide kernels' workgroups share the chunks of all wide rows: item(r, c) for
// each of this workgroup's.
template <typename F>
__device__ __forceinline__ void each_chunk(const sb_sample_args &a, const WideRow *wide, int kinds, F item) {
  __shared__ int found[SM_THREADS];
  __shared__ int counts[SM_WAVES];
  const int chunks = chunks_of(a.vocab), tid = threadIdx.x, w = tid >> 6;
  int before = 0;   // items of the rows before these
  for (int r0 = 0; r0 < a.rows; r0 += SM_THREADS) {
    const bool on = r0 + tid < a.rows && ((kinds >> wide[min(r0 + tid, a.rows - 1)].kind) & 1);
    const u64 m = __ballot(on);
    __syncthreads();
    if ((tid & 63) == 0) counts[w] = __popcll(m);
    __syncthreads();
    int at = __popcll(m & ((1ull << (tid & 63)) - 1)), n = 0;
    for (int i = 0; i < SM_WAVES; ++i) {
      at += i < w ? counts[i] : 0;
      n += counts[i];
    }
    if (on) found[at] = r0 + tid;
    __syncthreads();
    const int items = n * chunks;
    // Item i of all belongs to workgroup i % gridDim.
    int i = (int)blockIdx.x - before % (int)gridDim.x;
    if (i < 0) i += gridDim.x;
    for (; i < items; i += gridDim.x) item(found[i / chunks], i % chunks);
    before += items;
  }
}

// The draw, from the chunks' totals in sh.tot.
template <int DT>
__device__ __forceinline__ void draw_wide(const sb_sample_args &a, int r, const Params &pr, const Weigher &weigh, const Cut &cut, uint32_t best,
                                          const u64 *tot, Shared &sh) {
  constexpr int VEC = Row<DT>::VEC;
  const int chunks = chunks_of(a.vocab);
  u64 total = 0, t;
  for (int c = 0; c < chunks; ++c) total += tot[c];
  u64 limit = pr.draw_limit(total);
  int c = 0;
  while (c < chunks - 1 && limit >= tot[c]) limit -= tot[c++];
  const unsigned char *row = row_at<DT>(a, r);
  const int token = c * CHUNK + locate<DT>(
      Row<DT>(row + (size_t)c * CHUNK * Row<DT>::ES, min(CHUNK, a.vocab - c * CHUNK)),
      [&](const float (&z)[VEC], int i0, u64 (&x)[VEC]) { kept_weights<VEC>(z, c * CHUNK + i0, weigh, cut, x); },
      [&](u64) { return limit; }, t, sh);
  put_token(a, r, token, Row<DT>(row, a.vocab).one(token), from_order(best), pr, total);
}

// First, of a top-p row's chunk: its weights into the row's bins. Of a row
// without: their sum.
template <int DT>
__global__ __launch_bounds__(SM_THREADS, 4) void k_wide_bins(sb_sample_args a, WideRow *wide) {
  constexpr int VEC = Row<DT>::VEC;
  __shared__ Shared sh;
  const int tid = threadIdx.x;
  fill_table(sh);
  each_chunk(a, wide, 1 << 1 | 1 << 2, [&](int r, int c) {
    WideRow &w = wide[r];
    const int i0 = c * CHUNK;
    const Row<DT> row(row_at<DT>(a, r) + (size_t)i0 * Row<DT>::ES, min(CHUNK, a.vocab - i0));
    const Params pr(a, r);
    const Weigher weigh(sh.tab, from_order(w.best), pr.T);
    Cut cut;
    u64 all;
    if (w.kind == 1) {
      add_bins<DT>(row, i0, weigh, Bins(weigh, w.low, pr.top_p_reach(a.vocab)), cut, false, all, sh);
      __syncthreads();
      if (tid < BINS) bins_at(a, wide, r, c)[tid] = sh.hist[tid];
      return;
    }
    if (pr.mp > 0.0f) cut.raise(min_p_logit(pr, weigh, w.best));
    all = 0;
    row.each([&](const float (&z)[VEC], int j0) {
      u64 x[VEC];
      kept_weights<VEC>(z, i0 + j0, weigh, cut, x);
#pragma unroll
      for (int e = 0; e < VEC; ++e) all += x[e];
      all -= VEC * Weigher::RAW;
    });
    all = block_sum(all, sh);
    if (tid == 0) w.totals[c] = all;
  });
}

// Then, of a top-p row: the bin that the cut is in.
template <int DT>
__global__ __launch_bounds__(SM_THREADS, 4) void k_wide_cut(sb_sample_args a, WideRow *wide) {
  __shared__ Shared sh;
  const int r = blockIdx.x, tid = threadIdx.x;
  WideRow &w = wide[r];
  if (w.kind == 0) return;
  fill_table(sh);
  u64 mine = 0;
  if (w.kind == 1 && tid < BINS) {
#pragma unroll 4
    for (int c = 0; c < chunks_of(a.vocab); ++c) mine += bins_at(a, wide, r, c)[tid];
    sh.hist[tid] = mine;
  }
  const u64 all = block_sum(mine, sh);
  const Params pr(a, r);
  const Weigher weigh(sh.tab, from_order(w.best), pr.T);
  const u64 limit = w.kind == 1 ? pr.top_p_limit(all) : 0;
  uint32_t first = 0, last = 0;
  u64 rest = 0, at;
  const bool cuts = limit < all;   // (without top-p all is 0)
  if (cuts) Bins(weigh, w.low, pr.top_p_reach(a.vocab)).range(weigh, (int)find_bin(limit, rest, at, sh), w.best, first, last);
  const float z_mp = pr.mp > 0.0f ? min_p_logit(pr, weigh, w.best) : -INFINITY;
  if (tid == 0) {
    w.cut = cuts;
    w.first = first;
    w.last = last;
    w.rest = rest;
    w.z_mp = z_mp;
  }
}

// Then, of a top-p row's chunk: the tokens of that bin, and the weights above it.
struct ListShared {   // (room for four workgroups a unit)
  double tab[TAB];
  u64 part[SM_WAVES];
  uint32_t key[LIST_MAX];
  uint16_t idx[LIST_MAX];   // within the chunk
  int n;
};
static_assert(CHUNK <= 1 << 16, "a chunk's indexes in 16 bits");
template <int DT>
__global__ __launch_bounds__(SM_THREADS, 8) void k_wide_list(sb_sample_args a, WideRow *wide) {
  constexpr int VEC = Row<DT>::VEC;
  __shared__ ListShared sh;
  __shared__ int base;
  const int tid = threadIdx.x;
  fill_table(sh);
  each_chunk(a, wide, 1 << 1, [&](int r, int c) {
    WideRow &w = wide[r];
    const int i0 = c * CHUNK;
    const Row<DT> row(row_at<DT>(a, r) + (size_t)i0 * Row<DT>::ES, min(CHUNK, a.vocab - i0));
    const Params pr(a, r);
    const Weigher weigh(sh.tab, from_order(w.best), pr.T);
    const bool cuts = w.cut, any_above = !cuts || w.last < w.best;
    // Logits from z_lo to z_hi are listed, those above weighed.
    const float z_lo = cuts ? from_order(w.first) : INFINITY, z_hi = cuts ? from_order(w.last) : -INFINITY;
    Cut above;
    if (cuts) above.raise(from_order(min(w.last + 1, w.best)));
    above.raise(w.z_mp);
    const float from = any_above ? fminf(z_lo, above.lo) : z_lo;
    if (tid == 0) sh.n = 0;
    __syncthreads();
    u64 sum = 0;
    row.each([&](const float (&z)[VEC], int j0) {
      float m = z[0];
#pragma unroll
      for (int e = 1; e < VEC; ++e) m = fmaxf(m, z[e]);
      if (!(m >= from)) return;
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (z[e] >= z_lo && z[e] <= z_hi) {
          const int at = atomicAdd(&sh.n, 1);
          if (at < LIST_MAX) {
            sh.key[at] = order_bits(z[e]);
            sh.idx[at] = (uint16_t)(j0 + e);
          }
        }
      if (!any_above) return;
      u64 x[VEC];
      kept_weights<VEC>(z, i0 + j0, weigh, above, x);
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum += x[e];
      sum -= VEC * Weigher::RAW;
    });
    sum = block_sum(sum, sh);
    const int m = sh.n;
    if (tid == 0) {
      w.totals[c] = sum;
      base = m ? atomicAdd(&w.n, m) : 0;
    }
    __syncthreads();
    for (int j = tid; j < min(m, LIST_MAX); j += SM_THREADS)
      if (base + j < LIST_MAX) {
        w.key[base + j] = sh.key[j];
        w.idx[base + j] = i0 + sh.idx[j];
      }
  });
}

// Last, of a wide row: its cut and its draw.
template <int DT>
__global__ __launch_bounds__(SM_THREADS, 4) void k_wide_draw(sb_sample_args a, WideRow *wide) {
  __shared__ Shared sh;
  __shared__ u64 tot[CHUNKS_MAX];
  const int r = blockIdx.x, tid = threadIdx.x, V = a.vocab, chunks = chunks_of(V);
  const WideRow &w = wide[r];
  if (w.kind == 0) return;
  fill_table(sh);
  if (tid < chunks) tot[tid] = w.totals[tid];
  const Params pr(a, r);
  const uint32_t best = w.best, last = w.last;
  const Weigher weigh(sh.tab, from_order(best), pr.T);
  Cut cut;
  if (w.cut && w.n > LIST_MAX) {
    __syncthreads();
    u64 total;
    const Row<DT> whole(row_at<DT>(a, r), V);
    const int token = wide_row<DT>(whole, pr, weigh, best, w.low, total, sh);
    put_token(a, r, token, whole.one(token), from_order(best), pr, total);
    return;
  }
  if (w.cut) {
    Items it;
    for (int j = tid; j < w.n; j += SM_THREADS) {
      sh.key[j] = w.key[j];
      sh.idx[j] = w.idx[j];
    }
    __syncthreads();
    if (w.n <= RANKED) {
      const Ranked me = rank_list(w.n, [&](uint32_t b) { return weigh(from_order(b)); }, sh);
      if (me.w && me.before <= w.rest) {
        if (from_order(me.key) >= w.z_mp) atomicAdd(&tot[me.idx / CHUNK], me.w);
        if (w.rest < me.before + me.w) {
          sh.digit = me.key;
          sh.token = me.idx;
        }
      }
      __syncthreads();
      cut.lo = from_order(sh.digit);
      cut.last = sh.token;
    } else {
      take_list(it, w.n, [&](uint32_t b) { return weigh(from_order(b)); }, sh);
      u64 rest, at;
      const uint32_t d = list_search(it, [&](int j) { return last - it.key[j]; }, bits_of(last - w.first), w.rest, rest, at, sh);
      const int end = cut_list(it, last, d, rest, weigh(from_order(last - d)), at, V, sh);
      cut.lo = from_order(last - d);
      if (end < V) cut.last = end;
#pragma unroll
      for (int j = 0; j < LIST_PER; ++j)
        if (it.w[j] && from_order(it.key[j]) >= w.z_mp) atomicAdd(&tot[it.idx[j] / CHUNK], it.w[j]);
    }
  }
  __syncthreads();
  cut.raise(w.z_mp);
  draw_wide<DT>(a, r, pr, weigh, cut, best, tot, sh);
}

template <int DT>
hipError_t launch(const sb_sample_args &a, void *workspace, int n_cu, hipStream_t s) {
  WideRow *wide = static_cast<WideRow *>(workspace);
  hipLaunchKernelGGL(k_sample<DT>, dim3(a.rows), dim3(SM_THREADS), 0, s, a, wide);
  if (wide) {
    const long long chunks = (long long)chunks_of(a.vocab) * a.rows;
    hipLaunchKernelGGL(k_wide_bins<DT>, dim3((unsigned)std::min(chunks, 2LL * n_cu)), dim3(SM_THREADS), 0, s, a, wide);
    hipLaunchKernelGGL(k_wide_cut<DT>, dim3(a.rows), dim3(SM_THREADS), 0, s, a, wide);
    if (a.top_p) hipLaunchKernelGGL(k_wide_list<DT>, dim3((unsigned)std::min(chunks, 4LL * n_cu)), dim3(SM_THREADS), 0, s, a, wide);
    hipLaunchKernelGGL(k_wide_draw<DT>, dim3(a.rows), dim3(SM_THREADS), 0, s, a, wide);
  }
  return hipGetLastError();
}

}  // namespace

// Bytes of the wide kernels' workspace. They are four launches more, and pay off
// where one workgroup would pass over a long row three times while others have
// nothing left to do. Rows of which a part has top-k, without and with them:
// 320 of 32000 logits 52 and 68 us, 64 of 64000 79 and 63, 512 of 64000 99 and
// 96, 512 of 128000 195 and 138. One row of 128000 with top-p: 140 and 50, with
// top-k, too, 20 and 27: of a few rows, which may all have top-k, only those of
// calls with top-p bring it.
int64_t sample_workspace(const sb_sample_args &a) {
  if (a.vocab <= 3 * CHUNK || a.rows < 1 || (a.rows < 16 && !a.top_p)) return 0;
  return a.rows * (int64_t)(sizeof(WideRow) + (size_t)chunks_of(a.vocab) * BINS * 8);
}

hipError_t launch_sample(const sb_sample_args &a, void *workspace, int n_cu, hipStream_t s) {
  if (a.dtype == SB_F32) return launch<SB_F32>(a, workspace, n_cu, s);
  return a.dtype == SB_BF16 ? launch<SB_BF16>(a, workspace, n_cu, s) : launch<SB_F16>(a, workspace, n_cu, s);
}

}  // namespace sb
