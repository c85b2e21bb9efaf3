// One token per row of logits under temperature, top-k, top-p and min-p,
// drawn with a given number.
//
// Every filter keeps a prefix of the tokens ranked by (-z, index), so the kept
// tokens are those above one cut (a logit and, among its equals, an index),
// and nothing has to be sorted: a radix search over the ordered bits of the
// logits finds where a sum of counts (top-k) or of weights (top-p) passes its
// limit. The draw then runs over the kept tokens in index order.
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

constexpr int SM_THREADS = 1024;
constexpr int SM_WAVES = SM_THREADS / 64;
constexpr double ONE = 0x1p44;   // the weight of the largest logit

template <int DT>
__device__ __forceinline__ float load_logit(const void *row, int i) {
  if constexpr (DT == SB_F32) return static_cast<const float *>(row)[i];
  else return Half<DT>::to_float(static_cast<const uint16_t *>(row)[i]);
}

// The bits of z in an order that ascends with it; NaN counts as -inf.
__device__ __forceinline__ uint32_t order_bits(float z) {
  if (!(z >= -INFINITY)) z = -INFINITY;
  const uint32_t b = __float_as_uint(z + 0.0f);   // -0 is 0
  return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}

// A row's weights: 2^44 exp((z - top) / T), rounded.
struct Weigher {
  double top, c;   // c = log2(e) / T
  __device__ __forceinline__ u64 operator()(float z) const {
    const double x = fmin(fmax(((double)z - top) * c, -64.0), 0.0);   // NaN, and -inf with T = inf: -64
    return (u64)rint(exp2(x) * ONE);
  }
};

__device__ __forceinline__ u64 wave_scan(u64 v) {   // inclusive
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 y = __shfl_up(v, o, 64);
    if ((int)(threadIdx.x & 63) >= o) v += y;
  }
  return v;
}

struct Shared {
  u64 hist[256];
  u64 part[SM_WAVES];
  u64 rest;          // search: what of the limit is left within the digit
  uint32_t digit;
  int token;
};

__device__ __forceinline__ u64 block_sum(u64 v, Shared &sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = v;
  __syncthreads();
  u64 s = 0;
#pragma unroll
  for (int i = 0; i < SM_WAVES; ++i) s += sh.part[i];
  return s;
}

// The logit (as order bits) at which the weights, added from the largest logit
// down, first total more than `limit`, which they do; `rest`: limit less what
// lies above that logit. weight(bits, z) is a token's weight.
template <int DT, typename F>
__device__ __forceinline__ uint32_t radix_search(const void *row, int V, u64 limit, F weight, u64 &rest, Shared &sh) {
  uint32_t prefix = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    for (int i = threadIdx.x; i < 256; i += SM_THREADS) sh.hist[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < V; i += SM_THREADS) {
      const float z = load_logit<DT>(row, i);
      const uint32_t b = order_bits(z);
      if (shift == 24 || (b >> (shift + 8)) == prefix) {
        const u64 w = weight(b, z);
        if (w) atomicAdd(&sh.hist[(b >> shift) & 255u], w);
      }
    }
    __syncthreads();
    if (threadIdx.x < 64) {   // four digits a lane, from 255 down
      const int d0 = 255 - 4 * (int)threadIdx.x;
      u64 s = 0;
      for (int j = 0; j < 4; ++j) s += sh.hist[d0 - j];
      u64 before = wave_scan(s) - s;
      for (int j = 0; j < 4; ++j) {
        const u64 h = sh.hist[d0 - j];
        if (before <= limit && limit < before + h) {
          sh.digit = (uint32_t)(d0 - j);
          sh.rest = limit - before;
        }
        before += h;
      }
    }
    __syncthreads();
    prefix = (prefix << 8) | sh.digit;
    limit = sh.rest;
  }
  rest = limit;
  return prefix;
}

// The smallest index up to which the weights total more than `limit`, which
// they do. Each wave adds up a stretch of the row; the one that passes the
// limit walks its stretch again.
template <int DT, typename F>
__device__ __forceinline__ int locate(const void *row, int V, u64 limit, F weight, Shared &sh) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int len = (V + SM_THREADS - 1) / SM_THREADS * 64;
  const int lo = min(w * len, V), hi = min(lo + len, V);
  u64 s = 0;
  for (int i = lo + lane; i < hi; i += 64) s += weight(i, load_logit<DT>(row, i));
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  __syncthreads();
  if (lane == 0) sh.part[w] = s;
  __syncthreads();
  u64 before = 0;
  for (int i = 0; i < w; ++i) before += sh.part[i];
  if (before <= limit && limit < before + s) {
    for (int i0 = lo; i0 < hi; i0 += 64) {
      const int i = i0 + lane;
      const u64 x = wave_scan(i < hi ? weight(i, load_logit<DT>(row, i)) : 0);
      const u64 m = __ballot(before + x > limit);
      if (m) {
        if (lane == 0) sh.token = i0 + __builtin_ctzll(m);
        break;
      }
      before += __shfl(x, 63, 64);
    }
  }
  __syncthreads();
  return sh.token;
}

template <int DT>
__global__ __launch_bounds__(SM_THREADS) void k_sample(sb_sample_args a) {
  __shared__ Shared sh;
  const int r = blockIdx.x, V = a.vocab;
  const size_t es = DT == SB_F32 ? 4 : 2;
  const void *row = static_cast<const unsigned char *>(a.logits) + (size_t)r * a.row_stride * es;

  uint32_t best = 0;
  for (int i = threadIdx.x; i < V; i += SM_THREADS) best = max(best, order_bits(load_logit<DT>(row, i)));
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) best = max(best, (uint32_t)__shfl_xor((int)best, o, 64));
  if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = best;
  __syncthreads();
  for (int i = 0; i < SM_WAVES; ++i) best = max(best, (uint32_t)sh.part[i]);
  const uint32_t lowest = order_bits(-INFINITY);
  if (best == lowest) {
    if (threadIdx.x == 0) {
      a.tokens[r] = -1;
      if (a.logprobs) a.logprobs[r] = -INFINITY;
    }
    return;
  }
  const float top = __uint_as_float(best ^ (best >> 31 ? 0x80000000u : 0xFFFFFFFFu));
  const float T = a.temperature ? a.temperature[r] : 1.0f;

  // Kept: order bits above `cut`, or equal to it with an index up to `cut_i`.
  uint32_t cut = 0;
  int cut_i = V;
  double total = 1.0, x_tok = 0.0;
  int token;
  if (!(T > 0.0f)) {
    token = locate<DT>(row, V, 0, [=](int, float z) { return (u64)(order_bits(z) == best); }, sh);
  } else {
    // (The largest logit +inf: 10^300 instead, below which all others weigh nothing.)
    const Weigher weigh{top == INFINITY ? 1e300 : (double)top, 1.4426950408889634074 / (double)T};
    const int k = a.top_k ? a.top_k[r] : 0;
    const float p = a.top_p ? a.top_p[r] : 1.0f, mp = a.min_p ? a.min_p[r] : 0.0f;
    auto kept = [&](int i, uint32_t b) { return b > cut || (b == cut && i <= cut_i); };
    // Of the tokens equal to the cut the first `rest` + 1 stay.
    auto cut_at = [&](uint32_t bits, u64 rest) {
      const int last = locate<DT>(row, V, rest, [=](int, float z) { return (u64)(order_bits(z) == bits); }, sh);
      if (bits > cut) cut_i = last;
      else if (bits == cut) cut_i = min(cut_i, last);
      cut = max(cut, bits);
    };
    if (k > 0 && k < V) {
      u64 rest;
      const uint32_t bits = radix_search<DT>(row, V, (u64)(k - 1), [](uint32_t, float) { return (u64)1; }, rest, sh);
      cut_at(bits, rest);
    }
    if (p < 1.0f) {
      u64 z_k = 0;
      for (int i = threadIdx.x; i < V; i += SM_THREADS) {
        const float z = load_logit<DT>(row, i);
        z_k += kept(i, order_bits(z)) ? weigh(z) : 0;
      }
      z_k = block_sum(z_k, sh);
      // Kept where the weights ranked before total less than p z_k, so at
      // most `limit`: the cut is where they first total more.
      const u64 limit = (u64)fmax(ceil((double)p * (double)z_k), 1.0) - 1;
      if (limit < z_k) {
        // (Ties at the top-k cut weigh the same, so leaving out the kept ones'
        // equals behind cut_i changes no sum before the last kept one.)
        u64 rest;
        const uint32_t bits = radix_search<DT>(row, V, limit, [=](uint32_t b, float z) { return b >= cut ? weigh(z) : 0; }, rest, sh);
        const float z = __uint_as_float(bits ^ (bits >> 31 ? 0x80000000u : 0xFFFFFFFFu));
        cut_at(bits, rest / weigh(z));
      }
    }
    const u64 floor_w = mp > 0.0f ? (u64)ceil((double)fminf(mp, 1.0f) * ONE) : 0;
    auto weight = [&](int i, float z) {
      const u64 w = weigh(z);
      return kept(i, order_bits(z)) && w >= floor_w ? w : 0;
    };
    u64 z_all = 0;
    for (int i = threadIdx.x; i < V; i += SM_THREADS) z_all += weight(i, load_logit<DT>(row, i));
    z_all = block_sum(z_all, sh);
    const float u = a.u[r];
    const u64 limit = min((u64)((double)(u > 0.0f ? fminf(u, 1.0f) : 0.0f) * (double)z_all), z_all - 1);
    token = locate<DT>(row, V, limit, weight, sh);
    total = (double)z_all / ONE;
    const float z = load_logit<DT>(row, token);
    x_tok = top == INFINITY ? 0.0 : ((double)z - (double)top) / (double)T;
  }
  if (threadIdx.x == 0) {
    a.tokens[r] = token;
    if (a.logprobs) a.logprobs[r] = (float)(x_tok - log(total));
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
