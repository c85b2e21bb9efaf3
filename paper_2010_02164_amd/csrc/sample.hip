// One token per row of logits under temperature, top-k, top-p and min-p,
// drawn with a given number. One workgroup per row.
//
// Every filter keeps a prefix of the tokens ranked by (-z, index), so the kept
// tokens are those above one cut (a logit and, among its equals, an index),
// and nothing is sorted: a radix search over the ordered bits of the logits
// finds where a sum of counts (top-k) or of weights (top-p) passes its limit,
// and the draw is the same search over the kept tokens' indexes.
//
// Most rows are read once: a sample of the row (four 16-byte pieces a thread)
// gives a bound that the k-th largest logit hardly ever is below, the pass over
// the row lists the tokens from that bound on, a few hundred, and all searches
// run on the list in registers and LDS; a list of fewer than k tokens sends the
// row the other way. min-p alone bounds the tokens by the sample's largest.
// top-p without top-k needs every weight: a second pass adds them up into bins
// of equal ratio, which names the bin that the cut is in, a third lists that
// bin, a fourth draws; they read caches.
//
// Weights are whole multiples of 2^-44 in 64-bit integers: up to 2^18 of them
// add up without rounding or overflow, in any order, so that partial sums of
// waves and LDS atomics give one result. 44 bits below the largest weight
// keep the sum of 2^18 roundings under 2^-27 of it in the worst case and near
// 2^-36 in practice, below what u (24 bits) tells apart.
#include "serve.h"

namespace sb {
namespace {

typedef unsigned long long u64;
typedef unsigned int u4 __attribute__((ext_vector_type(4)));

constexpr int SM_THREADS = 1024;
constexpr int SM_WAVES = SM_THREADS / 64;
constexpr double ONE = 0x1p44;        // the weight of the largest logit
constexpr int LIST_PER = 4, LIST_MAX = LIST_PER * SM_THREADS;
constexpr int BIN_BITS = 9, BINS = 1 << BIN_BITS;
constexpr int TAB_BITS = 9;           // 2^x by a table of 2^(i / 512) and a cubic
// The largest top-k that is read off the sample: the list then aims at twice
// as many tokens, and 256 more.
constexpr int SAMPLED_K = 1536;
// 16-byte pieces a thread loads at once: of the sample, and of a pass (4 there
// made the code of the passes larger than the instruction cache).
constexpr int SAMPLE = 4, BATCH = 2;

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
  template <typename F>
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
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    each_piece(threadIdx.x, pieces, SM_THREADS, f);
    each_end(f);
  }
};

struct Shared {
  double tab[1 << TAB_BITS];   // 2^(i / 512)
  u64 hist[BINS];
  u64 part[SM_WAVES], ends[2][8];
  uint32_t key[LIST_MAX];      // listed tokens: order bits
  int idx[LIST_MAX];           // and indexes
  u64 rest, at_cut;
  uint32_t digit;
  int n, token;
};

// A row's weights: 2^44 exp((z - top) / T), rounded.
struct Weigher {
  const double *tab;
  double top, c;   // c = log2(e) / T. With a largest logit of +inf: 2^128 and 1, far from all others
  __device__ __forceinline__ Weigher(const double *t, float largest, float T)
      : tab(t), top(largest == INFINITY ? 0x1p128 : (double)largest), c(largest == INFINITY ? 1.0 : 1.4426950408889634074 / (double)T) {}
  // log2 of the weight (of the largest: 0). NaN, and -inf with T = inf: -64.
  __device__ __forceinline__ double log2w(float z) const { return fmin(fmax(((double)z - top) * c, -64.0), 0.0); }
  // x = n / 512 + r with |r| <= 2^-10: 2^x = 2^(n / 512) (1 + r ln 2 + ...);
  // the cubic leaves out (2^-10 ln 2)^4 / 24 = 2^-46.7.
  __device__ __forceinline__ u64 of(double x) const {
    constexpr double MAGIC = 0x1.8p43;   // its last bit is worth 2^-9
    const double t = x + MAGIC;
    const int n = __double2loint(t);
    const double r = x - (t - MAGIC);
    const double y = fma(fma(fma(r, 0.055504108664821580, 0.24022650695910071), r, 0.69314718055994531), r, 1.0);
    const double v = tab[n & ((1 << TAB_BITS) - 1)] * y;
    // Its exponent raised by 44 + n / 512, between -20 and 44.
    const double w = __hiloint2double(__double2hiint(v) + ((44 + (n >> TAB_BITS)) << 20), __double2loint(v));
    return (u64)__double_as_longlong(w + 0x1p52) & 0xFFFFFFFFFFFFFull;   // w <= 2^44, rounded to a whole number
  }
  __device__ __forceinline__ u64 operator()(float z) const { return of(log2w(z)); }
};

// x or 0, by a mask that the compiler does not turn into a branch around x:
// the chains of operations of a piece's tokens are to run side by side.
__device__ __forceinline__ u64 only_if(bool on, u64 x) {
  uint32_t m = on ? 0xFFFFFFFFu : 0u;
  asm("" : "+v"(m));
  return (u64)((uint32_t)x & m) | ((u64)((uint32_t)(x >> 32) & m) << 32);
}

__device__ __forceinline__ u64 wave_scan(u64 v) {   // inclusive
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 y = __shfl_up(v, o, 64);
    if ((int)(threadIdx.x & 63) >= o) v += y;
  }
  return v;
}
__device__ __forceinline__ u64 wave_sum(u64 v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ u64 block_sum(u64 v, Shared &sh) {
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
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
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
// total more than `limit`, which they do. keys < 2^bits; `drop` low bits are
// left out of the search (and of the result).
template <typename K>
__device__ __forceinline__ uint32_t list_search(const Items &it, K key, int bits, int drop, u64 limit, u64 &rest, u64 &at, Shared &sh) {
  uint32_t prefix = 0;
  int shift = bits;
  do {
    const int take = min(BIN_BITS, shift - drop);
    shift -= take;
    clear_bins(sh);
#pragma unroll
    for (int j = 0; j < LIST_PER; ++j) {
      const uint32_t k = key(j);
      if (it.w[j] && (shift + take >= 32 || (k >> (shift + take)) == prefix)) atomicAdd(&sh.hist[(k >> shift) & ((1u << take) - 1)], it.w[j]);
    }
    prefix = (prefix << take) | find_bin(limit, rest, at, sh);
    limit = rest;
  } while (shift > drop);
  return prefix << drop;
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
// which they do; weights(z, i0, w) gives those of a piece. Each wave adds up a
// stretch of pieces (the row's ends are stretches of their own), then all
// threads share the stretch that passes the limit.
template <int DT, typename F, typename L>
__device__ __forceinline__ int locate(const Row<DT> &row, F weights, L limit_of, u64 &total, Shared &sh) {
  constexpr int VEC = Row<DT>::VEC;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int len = (row.pieces + SM_WAVES - 1) / SM_WAVES;   // pieces a wave
  u64 s = 0;
  row.each_piece(min(w * len, row.pieces) + lane, min((w + 1) * len, row.pieces), 64, [&](const float (&z)[VEC], int i0) {
    u64 x[VEC];
    weights(z, i0, x);
#pragma unroll
    for (int e = 0; e < VEC; ++e) s += x[e];
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
    x[0] = wave_scan(x[0]);
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
        if (turn == 1 && run <= limit && limit < run + y[e]) sh.token = row.head + j * VEC + e;
        run += y[e];
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

__device__ __forceinline__ int bits_of(uint32_t x) { return 32 - __clz((int)x); }   // x < 2^bits; 0 for 0

template <int DT>
__global__ __launch_bounds__(SM_THREADS, 4) void k_sample(sb_sample_args a) {
  constexpr int VEC = Row<DT>::VEC;
  __shared__ Shared sh;
  const int r = blockIdx.x, V = a.vocab, tid = threadIdx.x;
  const Row<DT> row(static_cast<const unsigned char *>(a.logits) + (size_t)r * a.row_stride * Row<DT>::ES, V);
  const float T = a.temperature ? a.temperature[r] : 1.0f;
  const int k = a.top_k && a.top_k[r] > 0 && a.top_k[r] < V ? a.top_k[r] : 0;
  const float p = a.top_p && a.top_p[r] < 1.0f ? a.top_p[r] : 1.0f;
  const float mp = a.min_p && a.min_p[r] > 0.0f ? fminf(a.min_p[r], 1.0f) : 0.0f;
  const float u = a.u[r];
  const bool greedy = !(T > 0.0f);
  if (tid < (1 << TAB_BITS)) sh.tab[tid] = exp2(tid * (1.0 / (1 << TAB_BITS)));
  if (tid == 0) sh.n = 0;

  // The sample: SAMPLE pieces a thread, from as many places of the row.
  const int apart = max((row.pieces + SAMPLE - 1) / SAMPLE, SM_THREADS);
  u4 x[SAMPLE];
  float zm = -INFINITY;
#pragma unroll
  for (int b = 0; b < SAMPLE; ++b) {
    const int j = b * apart + tid;
    if (j < row.pieces) {
      x[b] = row.piece(j);
      float z[VEC];
      Row<DT>::unpack(x[b], z);
#pragma unroll
      for (int e = 0; e < VEC; ++e) zm = fmaxf(zm, z[e]);
    }
  }
  const uint32_t seen = block_max(order_bits(zm), sh);   // (its barriers also publish tab and n)
  // Whether the tokens that matter are read off the sample, and from which on.
  const bool sampled = greedy || (k > 0 && k <= SAMPLED_K) || (k == 0 && p == 1.0f && mp > 0.0f);
  float bound = -INFINITY;
  bool sure = true;   // nothing that matters lies below the bound
  if (greedy) {
    bound = from_order(seen);
  } else if (sampled) {
    if (k > 0) {
      Items it;
      it.key[0] = seen - order_bits(zm);
      it.w[0] = 1;
#pragma unroll
      for (int j = 1; j < LIST_PER; ++j) it.w[j] = 0, it.key[j] = 0;
      // Read off the sample as the k-th largest is off the row, or a lower
      // one than that (2 k + 256 tokens in the row by the sample's share) where
      // that lists fewer: no bound in itself, so the list is counted.
      const int want = min(k, (int)((float)(2 * k + 256) * (float)(min(SAMPLE * SM_THREADS, row.pieces) * VEC) / (float)V) + 1);
      sure = want == k;
      // 18 bits of it: rounded away from the largest, which keeps it a bound.
      u64 rest, at;
      const uint32_t d = list_search(it, [&](int j) { return it.key[j]; }, 32, 14, (u64)(want - 1), rest, at, sh) | 0x3FFFu;
      bound = from_order(seen - min(d, seen - LOWEST));
    }
    // min-p keeps z >= top + T ln(min_p), top at least the sample's (less a
    // little for the rounding here).
    if (p == 1.0f && mp > 0.0f && from_order(seen) < INFINITY) {
      const double b = (double)from_order(seen) + (double)T * log((double)mp);
      const float bf = (float)(b - 1e-6 * fabs(b) - 1e-30);
      sure |= bf >= bound;
      bound = fmaxf(bound, bf);
    }
  }

  // The pass over the row: its largest logit, its smallest finite one, and
  // the tokens from the bound on.
  zm = -INFINITY;
  float zl = INFINITY;
  auto look = [&](const float (&z)[VEC], int i0) {
    float m = z[0];
#pragma unroll
    for (int e = 1; e < VEC; ++e) m = fmaxf(m, z[e]);
    zm = fmaxf(zm, m);
    if (sampled) {
      if (m >= bound && m > -INFINITY) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (z[e] >= bound && z[e] > -INFINITY) list_token(order_bits(z[e]), i0 + e, sh);
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
    for (int b = 0; b < SAMPLE; ++b) row.each_piece(b * apart + SM_THREADS + tid, min((b + 1) * apart, row.pieces), SM_THREADS, look);
  row.each_end(look);
  const uint32_t best = block_max(order_bits(zm), sh);
  if (best == LOWEST) {
    if (tid == 0) {
      a.tokens[r] = -1;
      if (a.logprobs) a.logprobs[r] = -INFINITY;
    }
    return;
  }
  const float top = from_order(best);
  const Weigher weigh(sh.tab, top, T);
  const u64 floor_w = mp > 0.0f ? (u64)ceil((double)mp * ONE) : 0;
  const float uc = u > 0.0f ? fminf(u, 1.0f) : 0.0f;
  auto draw_limit = [=](u64 total) { return min((u64)((double)uc * (double)total), total - 1); };
  // Kept where the weights ranked before total less than p z_k, so at most
  // this: the cut is where they first total more.
  auto top_p_limit = [=](u64 z_k) { return (u64)fmax(ceil((double)p * (double)z_k), 1.0) - 1; };

  int token = 0;
  u64 total = 1;
  const int n = sh.n;
  if (sampled && n <= LIST_MAX && (sure || n >= k)) {
    Items it;
    take_list(it, n, [&](uint32_t b) { return greedy ? (u64)(b == best) : weigh(from_order(b)); }, sh);
    if (!greedy) {
      const int bits = bits_of(best - order_bits(bound));
      // Leaves the weights of those up to the cut, of its equals the first
      // `rest` / (what each adds) + 1.
      auto cut_at = [&](uint32_t d, u64 before, u64 each, u64 at) {
        int last = V;
        if (at > before + each) {   // not all of its equals stay
          Items eq = it;
#pragma unroll
          for (int j = 0; j < LIST_PER; ++j) eq.w[j] = it.w[j] && best - it.key[j] == d;
          u64 rest, a2;
          last = (int)list_search(eq, [&](int j) { return (uint32_t)eq.idx[j]; }, bits_of(V - 1), 0, before / each, rest, a2, sh);
        }
#pragma unroll
        for (int j = 0; j < LIST_PER; ++j) {
          const uint32_t dj = best - it.key[j];
          if (dj > d || (dj == d && it.idx[j] > last)) it.w[j] = 0;
        }
      };
      if (k > 0 && k < n) {
        Items count = it;
#pragma unroll
        for (int j = 0; j < LIST_PER; ++j) count.w[j] = j * SM_THREADS + tid < n;
        u64 rest, at;
        const uint32_t d = list_search(count, [&](int j) { return best - count.key[j]; }, bits, 0, (u64)(k - 1), rest, at, sh);
        cut_at(d, rest, 1, at);
      }
      if (p < 1.0f) {
        u64 s = 0;
#pragma unroll
        for (int j = 0; j < LIST_PER; ++j) s += it.w[j];
        const u64 z_k = block_sum(s, sh), limit = top_p_limit(z_k);
        if (limit < z_k) {
          u64 rest, at;
          const uint32_t d = list_search(it, [&](int j) { return best - it.key[j]; }, bits, 0, limit, rest, at, sh);
          cut_at(d, rest, weigh(from_order(best - d)), at);
        }
      }
#pragma unroll
      for (int j = 0; j < LIST_PER; ++j)
        if (it.w[j] < floor_w) it.w[j] = 0;
    }
    u64 s = 0, rest, at;
#pragma unroll
    for (int j = 0; j < LIST_PER; ++j) s += it.w[j];
    total = block_sum(s, sh);
    token = (int)list_search(it, [&](int j) { return (uint32_t)it.idx[j]; }, bits_of(V - 1), 0, greedy ? 0 : draw_limit(total), rest, at, sh);
    if (greedy) total = (u64)ONE;
  } else {
    // Kept: order bits above `cut`, or equal to it with an index up to `cut_i`.
    uint32_t cut = LOWEST;
    float cut_z = -INFINITY;
    int cut_i = -1;
    const float low = sampled ? -INFINITY : -from_order(block_max(order_bits(-zl), sh));   // (the full list: not looked for)
    auto kept = [&](int i, float z) { return (z > cut_z) | ((z == cut_z) & (i <= cut_i)); };   // (NaN: no)
    // Top-k by counts, top-p by weights, then the draw: one code for all, its
    // passes being much of the kernel's.
#pragma unroll 1
    for (int stage = greedy ? 2 : 0; stage < 3; ++stage) {
      const bool count = stage == 0;
      uint32_t bits = 0;
      u64 limit = 0;
      if (stage < 2) {
        if (count ? k == 0 : p == 1.0f) continue;
        // Bins of equal ratio, from the largest weight down to the smallest
        // one there is, or that can matter; what is below in the last. Weights
        // below (1 - p) / V of the largest total less than 1 - p of all: the
        // cut is not among them (two octaves to spare for rounding).
        const double reach = count ? 64.0 : fmin(2.0 + log2((double)V / fmax(1.0 - (double)p, 1e-9)), 64.0);
        const double range = fmin(fmax(-weigh.log2w(low), 1e-4), reach), scale = (BINS - 2) / range;
        auto bin = [&](double x) { return min(__double2loint(fma(x, -scale, 0x1.8p52)), BINS - 1); };   // to the nearest
        clear_bins(sh);
        u64 below = 0, all = 0;
        row.each([&](const float (&z)[VEC], int i0) {
          u64 w[VEC];
          int at[VEC];
#pragma unroll
          for (int e = 0; e < VEC; ++e) {   // no branches here: the tokens' chains of operations run side by side
            const double xw = weigh.log2w(z[e]);
            w[e] = only_if(kept(i0 + e, z[e]), count ? 1 : weigh.of(xw));
            at[e] = bin(xw);
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
        if (tid == 0) sh.hist[BINS - 1] = below;
        limit = count ? (u64)(k - 1) : top_p_limit(all);
        if (limit >= all) continue;
        u64 rest, at;
        const int target = (int)find_bin(limit, rest, at, sh);
        if (tid == 0) sh.n = 0;
        // The bin's logits: bins fall as logits rise, so each end is bisected.
        auto first_in = [&](int most) {   // the lowest order bits with a bin up to `most`
          uint32_t lo = LOWEST, hi = best;   // (best is in bin 0)
          while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (bin(weigh.log2w(from_order(mid))) <= most) hi = mid;
            else lo = mid + 1;
          }
          return hi;
        };
        const float z_lo = from_order(max(first_in(target), max(cut, LOWEST + 1)));
        const float z_hi = target > 0 ? from_order(first_in(target - 1) - 1) : top;
        __syncthreads();
        row.each([&](const float (&z)[VEC], int i0) {
          float m = z[0];
#pragma unroll
          for (int e = 1; e < VEC; ++e) m = fmaxf(m, z[e]);
          if (!(m >= z_lo)) return;
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (z[e] >= z_lo && z[e] <= z_hi && (z[e] != cut_z || i0 + e <= cut_i)) list_token(order_bits(z[e]), i0 + e, sh);
        });
        __syncthreads();
        const int m = sh.n;
        if (m <= LIST_MAX) {
          Items it;
          take_list(it, m, [&](uint32_t b) { return count ? (u64)1 : weigh(from_order(b)); }, sh);
          bits = best - list_search(it, [&](int j) { return best - it.key[j]; }, 32, 0, rest, rest, at, sh);
        } else {
          bits = row_search<DT>(row, limit, [&](float z) { return z >= cut_z && z > -INFINITY ? count ? (u64)1 : weigh(z) : 0; }, rest, at, sh);
        }
        const u64 each = count ? 1 : weigh(from_order(bits));
        if (at <= rest + each) {   // all of the cut's equals stay
          if (bits > cut) cut_i = V;
          cut = bits;
          cut_z = from_order(cut);
          continue;
        }
        limit = rest / each;   // the first so many of them, and one
      } else if (greedy) {
        bits = best;
      }
      const int found = locate<DT>(
          row,
          [&](const float (&z)[VEC], int i0, u64 (&w)[VEC]) {
            float m = z[0];
#pragma unroll
            for (int e = 1; e < VEC; ++e) m = fmaxf(m, z[e]);
#pragma unroll
            for (int e = 0; e < VEC; ++e) w[e] = bits && order_bits(z[e]) == bits;
            if (bits || m < cut_z) return;   // a wave without kept tokens takes no weights
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              const u64 x = weigh(z[e]);
              w[e] = only_if(kept(i0 + e, z[e]) & (x >= floor_w), x);
            }
          },
          [&](u64 t) { return bits ? limit : draw_limit(t); }, total, sh);
      if (stage == 2) {
        token = found;
      } else {
        cut_i = bits > cut ? found : min(cut_i, found);
        cut = bits;
        cut_z = from_order(cut);
      }
    }
    if (greedy) total = (u64)ONE;
  }
  if (tid == 0) {
    a.tokens[r] = token;
    const double z = row.one(token);
    const double xt = greedy || top == INFINITY ? 0.0 : (z - (double)top) / (double)T;
    if (a.logprobs) a.logprobs[r] = (float)(xt - log((double)total / ONE));
  }
}

}  // namespace

hipError_t launch_sample(const sb_sample_args &a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  switch (a.dtype) {
    case SB_F32: hipLaunchKernelGGL(k_sample<SB_F32>, dim3(a.rows), dim3(SM_THREADS), 0, s, a); break;
    case SB_BF16: hipLaunchKernelGGL(k_sample<SB_BF16>, dim3(a.rows), dim3(SM_THREADS), 0, s, a); break;
    default: hipLaunchKernelGGL(k_sample<SB_F16>, dim3(a.rows), dim3(SM_THREADS), 0, s, a); break;
  }
  return hipGetLastError();
}

}  // namespace sb
