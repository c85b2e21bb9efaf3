// Causal attention of new tokens over a paged cache, grouped heads, with an
// optional sliding window and first tokens that stay visible.
//
// The q_heads / kv_heads = G query heads of one key/value head and the
// request's m queries are G m rows over the same keys (row i G + g: query i,
// head g of the group), so one pass over the keys serves them all. Scores are
// taken transposed, S^T = K Q^T: a lane then holds scores of one row only, the
// running maximum and sum of its softmax are one register each, and its
// weights lie just as the second product O^T = V^T P^T wants its right operand
// (the keys of a product may come in any order, as long as both operands have
// the same). V^T is read from row-major V in LDS with the transposing read.
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

#include "serve.h"

namespace sb {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef unsigned int u4 __attribute__((ext_vector_type(4)));
typedef unsigned int u2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));

constexpr int FEW_ROWS = 16, FEW_KEYS = 32;
constexpr int MANY_ROWS = 128, MANY_KEYS = 64;
constexpr int AT_THREADS = 256, AT_WAVES = 4;
constexpr double LOG2E = 1.4426950408889634074;

template <int DT>
__device__ __forceinline__ f4 mfma16(const u4 &x, const u4 &y, const f4 &c) {
  typedef typename Half<DT>::v8 v8;
  if constexpr (DT == SB_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, x), __builtin_bit_cast(v8, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, x), __builtin_bit_cast(v8, y), c, 0, 0, 0);
}
template <int DT>
__device__ __forceinline__ f16v mfma32(const u4 &x, const u4 &y, const f16v &c) {
  typedef typename Half<DT>::v8 v8;
  if constexpr (DT == SB_BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, x), __builtin_bit_cast(v8, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, x), __builtin_bit_cast(v8, y), c, 0, 0, 0);
}

// Four rows of 16 values each, transposed: lane l of each 16 lanes points at
// row l / 4, values 4 (l % 4) .. + 3, and gets value l of the four rows.
__device__ __forceinline__ u2 read_transposed(const unsigned char *p) {
  const s4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)(p));
  return __builtin_bit_cast(u2, v);
}

// v of lane at / 4.
__device__ __forceinline__ long long from_lane(long long v, int at) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_ds_bpermute(at, (int)v), hi = (uint32_t)__builtin_amdgcn_ds_bpermute(at, (int)(v >> 32));
  return (long long)(((unsigned long long)hi << 32) | lo);
}

// Orders a wave's own LDS writes before its later reads by other lanes.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Eight values with NaN and infinities as 0; `bad` if there were any.
template <int DT>
__device__ __forceinline__ u4 finite_only(const u4 &x, bool &bad) {
  constexpr uint32_t E = DT == SB_BF16 ? 0x7F80u : 0x7C00u;   // exponent bits, all set in NaN and infinities
  u4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (x[i] & E) == E, hi = (x[i] & (E << 16)) == (E << 16);
    y[i] = x[i] & ((lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u));
    bad |= lo || hi;
  }
  return y;
}

// A hidden key's weight is 0, and 0 times what stands there would be NaN where
// that is NaN or infinite. In a tile whose keys some rows see and others do
// not, such values are therefore taken out of V, and a product of two
// indicators (ones where V is not finite, ones where a weight is not 0) says
// which results become NaN instead. That code is apart: the loops over the
// keys stop at such a tile and are run again with it from the start, so that
// it takes no registers from them (at heads of 256 the one for prompts is out of
// registers all the same and reloads about 8 a tile).
template <int DT>
__device__ __forceinline__ uint32_t ones_where(bool lo, bool hi) {
  constexpr uint32_t ONE16 = DT == SB_BF16 ? 0x3F80u : 0x3C00u;
  return (lo ? ONE16 : 0u) | (hi ? ONE16 << 16 : 0u);
}
template <int DT>
__device__ __forceinline__ u4 not_finite(const u4 &x) {
  constexpr uint32_t E = DT == SB_BF16 ? 0x7F80u : 0x7C00u;
  u4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = ones_where<DT>((x[i] & E) == E, (x[i] & (E << 16)) == (E << 16));
  return y;
}
template <int DT>
__device__ __forceinline__ u4 not_zero(const u4 &x) {
  u4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = ones_where<DT>((x[i] & 0xFFFFu) != 0, (x[i] >> 16) != 0);
  return y;
}

// Weights go into the second product in the cache's type, and times 2^raise (the
// sums likewise, so that it cancels): fp16 has nothing between 0 and 2^-24, and
// 100000 keys of 2^-25 each total 0.003 of one large one. `most`: how far above 1
// (as a power of 2) a weight may be; the largest stays below fp16's 65504. bf16
// has fp32's exponents.
template <int DT>
constexpr float raise(int most) {
  return DT == SB_F16 ? 15.0f - most : 0.0f;
}

// The rows and keys of one workgroup's pass. The keys its rows see are the
// first `ns` of the request and those from `lo` on, n_vis in all.
struct Span {
  int q0, m, n;      // first query, queries and cached tokens of the request
  int rows, r0;      // G m, first row of this pass
  int ns, lo, n_vis;
  int p_first, p_last;   // positions of the first and last of these rows
  __device__ __forceinline__ int key(int u) const { return u < ns ? u : lo + (u - ns); }
  // Whether all rows see all keys of a tile from k_first to k_last.
  __device__ __forceinline__ bool all_see(const sb_attention_args &a, int k_first, int k_last) const {
    return k_last <= p_first && (a.window == 0 || k_first > p_last - a.window || k_last < a.sinks);
  }
};

__device__ __forceinline__ void span_request(const sb_attention_args &a, int b, Span &s) {
  // Starts outside q, or behind the next one, leave the request no rows. (A
  // difference of unclipped ones, or G times a negative m, could pass 2^31.)
  s.q0 = min(max(a.q_start[b], 0), a.n_tokens);
  s.m = min(max(a.q_start[b + 1], s.q0), a.n_tokens) - s.q0;
  s.n = (int)min((long long)max(a.lens[b], 0), (long long)a.max_pages * a.page_size);
  s.rows = s.m * (a.q_heads / a.kv_heads);
}

__device__ __forceinline__ void span_rows(const sb_attention_args &a, int r0, int count, Span &s) {
  const int G = a.q_heads / a.kv_heads;
  s.r0 = r0;
  s.p_first = s.n - s.m + r0 / G;
  s.p_last = s.n - s.m + min(r0 + count - 1, s.rows - 1) / G;
  s.lo = a.window > 0 ? max(max(s.p_first, 0) - a.window + 1, 0) : 0;   // (the window may be anything up to 2^31)
  s.ns = min(a.sinks, s.lo);
  s.n_vis = max(s.p_last + 1 - s.lo + s.ns, 0);
}

// A key's page, -1 if there is none; `place` within it. (key + 1/2) / size is
// further from a whole number than the product with the reciprocal is off.
__device__ __forceinline__ int page_of(const sb_attention_args &a, const int *table, double inv_page, int key, int &place) {
  const int c = (int)(((double)key + 0.5) * inv_page);
  place = key - c * a.page_size;
  const int page = table[c];
  return (unsigned)page < (unsigned)a.n_pages ? page : -1;
}

__device__ __forceinline__ bool sees(const sb_attention_args &a, int p, int key) {
  return (key <= p) & ((a.window == 0) | (key > max(p, 0) - a.window) | (key < a.sinks));   // (no branches)
}

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

// One wave's pass over its tiles t0, t0 + 4, ... < t_end: the 16 rows' sums, their
// maxima and this lane's share of the weights' sums. False where it stopped.
template <int DT, int D, bool CAREFUL>
__device__ __forceinline__ bool few_keys(const sb_attention_args &a, const Span &s, const int *table, const uint16_t *kc, const uint16_t *vc,
                                         const u4 (&q)[D / 32], int p, bool real, int t0, int t_end, unsigned char *lds, f4 (&o)[D / 16],
                                         float &mx, float &sum) {
  constexpr int VS = 2 * D + 32;            // bytes of a V row in LDS: 8 rows of 32 bytes in different banks
  constexpr int KS = D / 32, NV = D / 16;   // products per score, 16-byte pieces of V per lane
  constexpr int DT16 = D / 16;
  constexpr int V_STEP = 64 / (D / 8);      // rows of V that the lanes bring at once
  const int lane = threadIdx.x & 63, g4 = lane >> 4, l16 = lane & 15, v_row = lane / (D / 8), v_col = lane % (D / 8);
  const double inv_page = 1.0 / a.page_size;
  const float c = (float)(a.scale * LOG2E);
  mx = -INFINITY;
  sum = 0.0f;
#pragma unroll
  for (int x = 0; x < DT16; ++x) o[x] = f4{0, 0, 0, 0};
  // Where a tile's keys lie (lane l: key l % 32), looked up a tile ahead. Its
  // rows are loaded when they are needed: few registers, and so many waves to
  // have loads in flight, did better than loads ahead (286 against 306 us).
  auto find = [&](int t, int &place) {
    const int u = t * FEW_KEYS + (lane & 31);
    return t < t_end && u < s.n_vis ? page_of(a, table, inv_page, s.key(u), place) : -1;
  };
  auto load_k = [&](u4 (&k)[2][KS], int page, int place) {
    const long long at = page >= 0 ? page * a.kc_page + place * a.kc_slot : 0;   // (keys that are not there: any that is)
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const uint16_t *src = kc + from_lane(at, l16 * 4 + hf * 64) + 8 * g4;
#pragma unroll
      for (int x = 0; x < KS; ++x) k[hf][x] = *reinterpret_cast<const u4 *>(src + 32 * x);
    }
  };
  auto load_v = [&](u4 (&v)[NV], int page, int place) {
    const long long at = page >= 0 ? page * a.vc_page + place * a.vc_slot : 0;
#pragma unroll
    for (int x = 0; x < NV; ++x) v[x] = *reinterpret_cast<const u4 *>(vc + from_lane(at, v_row * 4 + x * (4 * V_STEP)) + v_col * 8);
  };
  int next_place = 0, next = find(t0, next_place);
  for (int t = t0; t < t_end; t += AT_WAVES) {
    const int page = next, place = next_place;
    const uint32_t there = (uint32_t)__ballot(page >= 0);
    u4 k[2][KS], v[NV];
    load_k(k, page, place);
    next = find(t + AT_WAVES, next_place);
    const bool plain = there == 0xFFFFFFFFu && s.all_see(a, s.key(t * FEW_KEYS), s.key(t * FEW_KEYS + FEW_KEYS - 1));
    f4 sc[2] = {f4{0, 0, 0, 0}, f4{0, 0, 0, 0}};
#pragma unroll
    for (int x = 0; x < KS; ++x)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) sc[hf] = mfma16<DT>(k[hf][x], q[x], sc[hf]);
    load_v(v, page, place);
    // Lane: keys 16 hf + 4 g4 + j of row l16, as scalars from here on (masks
    // written into the products' vectors have been compiled wrongly).
    float e[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) e[x] = sc[x >> 2][x & 3] * c;
    if (!plain) {
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int at = 16 * (x >> 2) + 4 * g4 + (x & 3);
        const bool on = real & (((there >> at) & 1u) != 0) & sees(a, p, s.key(t * FEW_KEYS + at));
        e[x] = on ? e[x] : -INFINITY;
      }
    }
    float tm = e[0];
#pragma unroll
    for (int x = 1; x < 8; ++x) tm = fmaxf(tm, e[x]);
    tm = fmaxf(tm, __shfl_xor(tm, 16, 64));
    tm = fmaxf(tm, __shfl_xor(tm, 32, 64));
    const float mn = fmaxf(mx, tm), top = mn == -INFINITY ? 0.0f : mn, base = top - raise<DT>(0);
    const float shrink = __builtin_amdgcn_exp2f(mx - top);
    mx = mn;
    float ts = 0.0f;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      e[x] = __builtin_amdgcn_exp2f(e[x] - base);
      ts += e[x];
    }
    sum = sum * shrink + ts;
    // Each weight in two parts, the rounded one and what that leaves: reading the
    // cache binds here, and the second product costs nothing (238.3 us a batch's
    // step, without 238.4).
    u4 pk, pl;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      pk[x] = Half<DT>::pack(e[2 * x], e[2 * x + 1]);
      pl[x] = Half<DT>::pack(e[2 * x] - Half<DT>::to_float(pk[x] & 0xFFFFu), e[2 * x + 1] - Half<DT>::to_float(pk[x] >> 16));
    }
    bool bad = false;
#pragma unroll
    for (int x = 0; x < NV; ++x) {
      if (!plain) {
        if (!((there >> (v_row + x * V_STEP)) & 1u)) v[x] = u4{0, 0, 0, 0};
        finite_only<DT>(v[x], bad);
      }
      *reinterpret_cast<u4 *>(lds + v_row * VS + v_col * 16 + x * (V_STEP * VS)) = v[x];
    }
    if (!CAREFUL && __any(bad)) return false;
    wave_lds_fence();
    const unsigned char *vt = lds + (4 * g4 + (l16 >> 2)) * VS + (l16 & 3) * 8;
    if (CAREFUL && !plain) {
      const u4 pn = not_zero<DT>(pk);
#pragma unroll
      for (int x = 0; x < DT16; ++x) {
        const u2 v0 = read_transposed(vt + 32 * x), v1 = read_transposed(vt + 16 * VS + 32 * x);
        const f4 hit = mfma16<DT>(not_finite<DT>(u4{v0[0], v0[1], v1[0], v1[1]}), pn, f4{0, 0, 0, 0});
#pragma unroll
        for (int j = 0; j < 4; ++j) o[x][j] = hit[j] > 0.0f ? NAN : o[x][j];
      }
      wave_lds_fence();
      for (int piece = lane; piece < FEW_KEYS * (D / 8); piece += 64) {
        u4 *at = reinterpret_cast<u4 *>(lds + piece / (D / 8) * VS + piece % (D / 8) * 16);
        *at = finite_only<DT>(*at, bad);
      }
      wave_lds_fence();
    }
#pragma unroll
    for (int x = 0; x < DT16; ++x) {
      const u2 v0 = read_transposed(vt + 32 * x), v1 = read_transposed(vt + 16 * VS + 32 * x);
      const u4 vv = {v0[0], v0[1], v1[0], v1[1]};
      o[x] = mfma16<DT>(vv, pl, mfma16<DT>(vv, pk, o[x] * shrink));
    }
    wave_lds_fence();
  }
  return true;
}

// Workgroups of k_attn_few that a compute unit is to hold at once, for loads in
// flight: as many as the registers of a wave's tile allow.
constexpr int few_groups(int D) { return D == 64 ? 3 : D == 128 ? 2 : 1; }

// Tiles of the request's rows r0 .. (one where they see nothing: somebody has
// to say so).
__device__ __forceinline__ int unit_tiles(const Span &s) { return max((s.n_vis + FEW_KEYS - 1) / FEW_KEYS, 1); }

template <int D>
struct FewShared {
  static constexpr int VS = 2 * D + 32;
  alignas(16) unsigned char v[AT_WAVES][FEW_KEYS * VS];
  float2 stats[AT_WAVES][FEW_ROWS];
  static_assert(FEW_KEYS * VS >= FEW_ROWS * D * 4, "the waves' sums fit where V was");
};

// Tiles t_begin .. t_end of the span's rows: their result, or, as a share, part
// `part` of it (below 0: the result).
template <int DT, int D>
__device__ __forceinline__ void few_unit(const sb_attention_args &a, const Span &s, int b, int hk, int t_begin, int t_end, int part, int groups,
                                         int units, void *work, FewShared<D> &sh) {
  constexpr int DT16 = D / 16, KS = D / 32;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, g4 = lane >> 4, l16 = lane & 15;
  const int G = a.q_heads / a.kv_heads;
  const int *table = a.table + b * a.table_stride;
  const uint16_t *kc = static_cast<const uint16_t *>(a.k_cache) + hk * a.kc_head;
  const uint16_t *vc = static_cast<const uint16_t *>(a.v_cache) + hk * a.vc_head;
  const int row = s.r0 + l16, i = row / G, p = s.n - s.m + i;
  const bool real = row < s.rows;
  u4 q[KS];
#pragma unroll
  for (int x = 0; x < KS; ++x) {
    const uint16_t *src = static_cast<const uint16_t *>(a.q) + (s.q0 + i) * a.q_token + (hk * G + row - i * G) * a.q_head;
    q[x] = real ? *reinterpret_cast<const u4 *>(src + 32 * x + 8 * g4) : u4{0, 0, 0, 0};
  }
  f4 o[DT16];
  float mx, sum;
  if (!few_keys<DT, D, false>(a, s, table, kc, vc, q, p, real, t_begin + w, t_end, &sh.v[w][0], o, mx, sum))
    few_keys<DT, D, true>(a, s, table, kc, vc, q, p, real, t_begin + w, t_end, &sh.v[w][0], o, mx, sum);
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);
  // The four waves' parts: sums side by side where V was.
  float *os = reinterpret_cast<float *>(&sh.v[w][0]);
#pragma unroll
  for (int x = 0; x < DT16; ++x) *reinterpret_cast<f4 *>(os + l16 * D + 16 * x + 4 * g4) = o[x];
  if (g4 == 0) sh.stats[w][l16] = make_float2(mx, sum);
  __syncthreads();
  for (int e = threadIdx.x; e < FEW_ROWS * D / 4; e += AT_THREADS) {
    const int rr = e / (D / 4), col = (e - rr * (D / 4)) * 4, rw = s.r0 + rr;
    if (rw >= s.rows) continue;
    float m4 = -INFINITY, l4 = 0.0f;
    f4 acc = {0, 0, 0, 0};
#pragma unroll
    for (int x = 0; x < AT_WAVES; ++x) m4 = fmaxf(m4, sh.stats[x][rr].x);
    const float base = m4 == -INFINITY ? 0.0f : m4;
#pragma unroll
    for (int x = 0; x < AT_WAVES; ++x) {
      const float f = __builtin_amdgcn_exp2f(sh.stats[x][rr].x - base);
      l4 += f * sh.stats[x][rr].y;
      acc += f * *reinterpret_cast<const f4 *>(reinterpret_cast<const float *>(&sh.v[x][0]) + rr * D + col);
    }
    if (part < 0) {
      const int qi = rw / G;
      const float inv = l4 == 0.0f ? 0.0f : 1.0f / l4;
      uint16_t *dst = static_cast<uint16_t *>(a.out) + (s.q0 + qi) * a.out_token + (hk * G + rw - qi * G) * a.out_head + col;
      *reinterpret_cast<u2 *>(dst) = u2{Half<DT>::pack(acc[0] * inv, acc[1] * inv), Half<DT>::pack(acc[2] * inv, acc[3] * inv)};
    } else {
      *reinterpret_cast<f4 *>(part_sums<D>(a, work, groups, units, hk, part) + rr * D + col) = acc;
      if (col == 0) part_stats<D>(a, work, groups, units, hk, part)[rr] = make_float2(m4, l4);
    }
  }
  __syncthreads();
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
      few_unit<DT, D>(a, s, j, hk, 0, unit_tiles(s), -1, 0, 0, nullptr, sh);
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
      t += unit_tiles(s);
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
      const int tiles = unit_tiles(s);
      const long long next = at + tiles;
      if (next > begin) {
        const int t0 = (int)max(begin - at, 0LL), t1 = u < units ? (int)min(end - at, (long long)tiles) : tiles;
        const bool whole = t0 == 0 && t1 == tiles;
        if (u < units && t0 == 0 && hk == 0 && threadIdx.x == 0)
          unit_infos(work)[u] = UnitInfo{j + u, whole ? 1 : (int)min(divide(next - 1, per), groups - 1LL) - j + 1, b, r0};
        if (u < units || t0 == 0) few_unit<DT, D>(a, s, b, hk, t0, t1, whole ? -1 : j + u, groups, units, work, sh);
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

// What the waves of k_attn_many share: two tiles of K and V, one worked on
// while the other is filled.
template <int D>
struct ManyShared {
  static constexpr int KSTR = 2 * D + 16, VSTR = 2 * D + 32;   // bytes of a K and a V row
  alignas(16) unsigned char k[2][MANY_KEYS * KSTR];
  alignas(16) unsigned char v[2][MANY_KEYS * VSTR];
  longlong2 at[2][MANY_KEYS];         // where a tile's rows of K and V lie; none (below 0): nowhere
  unsigned char none[2][MANY_KEYS];   // 1: the key's page is outside the cache; looked at only if
  int odd[2];                         // bit 0 says that there are such, bit 1: values that are not
                                      // finite, in a tile that not all rows see
};

// The workgroup's pass over `tiles` tiles from t_first on: the lane's row's sums,
// what its exponentials are taken against, and its keys' share of the weights'
// sum. False where it stopped.
template <int DT, int D, bool CAREFUL>
__device__ __forceinline__ bool many_keys(const sb_attention_args &a, const Span &s, const int *table, const uint16_t *kc, const uint16_t *vc,
                                          const u4 (&q)[D / 16], int p, bool real, int t_first, int tiles, ManyShared<D> &sh,
                                          f16v (&o)[D / 32], float &ref, float &sum) {
  constexpr int KSTR = ManyShared<D>::KSTR, VSTR = ManyShared<D>::VSTR;
  constexpr int PC = MANY_KEYS * (D / 8) / AT_THREADS;   // 16-byte pieces of K (and V) a thread brings,
  constexpr int RSTEP = AT_THREADS / (D / 8);            // their rows so far apart
  constexpr int KS = D / 16, DB = D / 32;
  const int lane = threadIdx.x & 63, l32 = lane & 31, h2 = lane >> 5;
  const int row0 = threadIdx.x / (D / 8), col = threadIdx.x % (D / 8);
  const double inv_page = 1.0 / a.page_size;
  const float c = a.scale == 0.0f ? 1.0f : (float)(fabs((double)a.scale) * LOG2E);
#pragma unroll
  for (int x = 0; x < DB; ++x)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[x][e] = 0.0f;
  // `ref`: what the exponentials are taken against, a score the row has had. It
  // moves to a larger one only when that would be over 2^GROW of it.
  constexpr int GROW = 8;
  ref = -INFINITY;
  sum = 0.0f;

  // A tile's way: its pages are looked up four tiles ahead, by one wave, a key
  // a lane; the places of its rows are written to LDS three ahead, its rows
  // loaded two ahead and written to LDS one ahead. Keys behind the last one
  // are the last one again, which no row sees there.
  u4 kr[PC], vr[PC];
  int page = 0, place = 0;
  uint32_t gone = 0;   // bit x: piece x in the registers has no page
  const int base_u = t_first * MANY_KEYS, wave = threadIdx.x >> 6;
  auto look_up = [&](int t) {
    if (wave == (t & 3)) page = page_of(a, table, inv_page, s.key(min(base_u + t * MANY_KEYS + lane, s.n_vis - 1)), place);
  };
  auto put_at = [&](int t) {
    if (wave == (t & 3))
      sh.at[t & 1][lane] = page < 0 ? longlong2{-1, -1} : longlong2{page * a.kc_page + place * a.kc_slot, page * a.vc_page + place * a.vc_slot};
  };
  auto load = [&](int t) {
    gone = 0;
#pragma unroll
    for (int x = 0; x < PC; ++x) {
      const longlong2 at = sh.at[t & 1][row0 + x * RSTEP];
      kr[x] = *reinterpret_cast<const u4 *>(kc + max(at.x, 0LL) + col * 8);   // (any row for none)
      vr[x] = *reinterpret_cast<const u4 *>(vc + max(at.y, 0LL) + col * 8);
      gone |= (at.x < 0 ? 1u : 0u) << x;
    }
  };
  auto write = [&](int t) {
    const bool shared = s.all_see(a, s.key(base_u + t * MANY_KEYS), s.key(base_u + t * MANY_KEYS + MANY_KEYS - 1));
    const int to = t & 1;
    bool bad = false;
    if (gone) {
#pragma unroll
      for (int x = 0; x < PC; ++x)
        if ((gone >> x) & 1u) vr[x] = u4{0, 0, 0, 0};
    }
#pragma unroll
    for (int x = 0; x < PC; ++x) {
      const int kk = row0 + x * RSTEP;
      *reinterpret_cast<u4 *>(&sh.k[to][kk * KSTR + col * 16]) = kr[x];
      *reinterpret_cast<u4 *>(&sh.v[to][kk * VSTR + col * 16]) = vr[x];
      if (!CAREFUL && !shared) finite_only<DT>(vr[x], bad);
    }
    if (gone || bad) {
#pragma unroll
      for (int x = 0; x < PC; ++x) sh.none[to][row0 + x * RSTEP] = (gone >> x) & 1u;
      atomicOr(&sh.odd[to], (gone ? 1 : 0) | (bad ? 2 : 0));
    }
  };
  __syncthreads();
  if (threadIdx.x < 2) sh.odd[threadIdx.x] = 0;
  for (int x = threadIdx.x; x < 2 * MANY_KEYS; x += AT_THREADS) (&sh.none[0][0])[x] = 0;
  __syncthreads();
  if (tiles > 0) {
    for (int t = 0; t < 3; ++t) {   // the first three tiles' places; tile 0 all the way
      if (t == 2) {
        load(0);
        write(0);
        __syncthreads();
      }
      look_up(t);
      put_at(t);
      __syncthreads();
    }
    load(1);
    look_up(3);
  }
  for (int t = 0; t < tiles; ++t) {
    __syncthreads();   // tile t is there, the places of tile t + 2 are, and the other buffer has been read
    const int odd = sh.odd[t & 1], u0 = base_u + t * MANY_KEYS;
    if (!CAREFUL && (odd & 2)) return false;
    if (t + 1 < tiles) {
      write(t + 1);
      load(t + 2);
      put_at(t + 3);
      look_up(t + 4);
    }
    const unsigned char *sk = sh.k[t & 1], *sv = sh.v[t & 1];
    const bool shared = s.all_see(a, s.key(u0), s.key(u0 + MANY_KEYS - 1));
    // Operands come from LDS AHEAD products before they are needed.
    constexpr int AHEAD = 4;
    f16v sc[2];
    {
      const unsigned char *kp = &sk[l32 * KSTR + 16 * h2];
      u4 kf[AHEAD];
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) kf[x] = *reinterpret_cast<const u4 *>(kp + (x & 1) * 32 * KSTR + 32 * (x >> 1));
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[0][e] = sc[1][e] = 0.0f;
#pragma unroll
      for (int x = 0; x < 2 * KS; ++x) {
        sc[x & 1] = mfma32<DT>(kf[x % AHEAD], q[x >> 1], sc[x & 1]);
        const int y = x + AHEAD;
        if (y < 2 * KS) kf[x % AHEAD] = *reinterpret_cast<const u4 *>(kp + (y & 1) * 32 * KSTR + 32 * (y >> 1));
      }
    }
    const unsigned char *vt = &sv[(4 * h2 + ((lane & 15) >> 2)) * VSTR + ((lane >> 4) & 1) * 32 + (lane & 3) * 8];
    auto v_frag = [&](int x) {   // of product x: keys 16 (x / DB) .. + 15, values 32 (x % DB) .. + 31
      const unsigned char *at = vt + 16 * (x / DB) * VSTR + 64 * (x % DB);
      const u2 v0 = read_transposed(at), v1 = read_transposed(at + 8 * VSTR);
      return u4{v0[0], v0[1], v1[0], v1[1]};
    };
    u4 vf[AHEAD];
    if (!CAREFUL) {
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) vf[x] = v_frag(x);
    }
    // Lane: keys 32 (x / 16) + 8 (x % 16 / 4) + 4 h2 + x % 4 of row l32, as
    // scalars from here on (masks written into the products' vectors have been
    // compiled wrongly).
    float e[32];
#pragma unroll
    for (int x = 0; x < 32; ++x) e[x] = sc[x >> 4][x & 15];
    if (!shared) {
#pragma unroll
      for (int x = 0; x < 32; ++x)
        e[x] = sees(a, p, s.key(u0 + 32 * (x >> 4) + 8 * ((x & 15) >> 2) + 4 * h2 + (x & 3))) ? e[x] : -INFINITY;
    }
    if (odd & 1) {
#pragma unroll
      for (int x = 0; x < 32; ++x)
        e[x] = sh.none[t & 1][32 * (x >> 4) + 8 * ((x & 15) >> 2) + 4 * h2 + (x & 3)] ? -INFINITY : e[x];
    }
    float tm = e[0];
#pragma unroll
    for (int x = 1; x < 32; ++x) tm = fmaxf(tm, e[x]);
    tm = fmaxf(tm, __shfl_xor(tm, 32, 64));
    if (__any(tm > ref && !(c * (tm - ref) <= GROW))) {
      const float mn = fmaxf(ref, tm);
      const float shrink = ref == mn ? 1.0f : __builtin_amdgcn_exp2f(c * (ref - mn));
      ref = mn;
      sum *= shrink;
#pragma unroll
      for (int x = 0; x < DB; ++x) o[x] *= shrink;
    }
    // (One part a weight: a second product with what its rounding leaves made the
    // three prompts' 391 us into 483.)
    const float base = ref == -INFINITY ? 0.0f : fmaf(ref, c, -raise<DT>(GROW));
    float ts[2] = {0.0f, 0.0f};
    u4 pk[4];
#pragma unroll
    for (int x = 0; x < 32; x += 2) {
      const float f = __builtin_amdgcn_exp2f(fmaf(e[x], c, -base)), g = __builtin_amdgcn_exp2f(fmaf(e[x + 1], c, -base));
      ts[0] += f;
      ts[1] += g;
      pk[x >> 3][(x & 7) >> 1] = Half<DT>::pack(f, g);
    }
    sum += ts[0] + ts[1];
    if (CAREFUL && !shared) {
#pragma unroll
      for (int x = 0; x < DB; ++x) {
        f16v hit;
#pragma unroll
        for (int e = 0; e < 16; ++e) hit[e] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          const u2 v0 = read_transposed(vt + 16 * ks * VSTR + 64 * x), v1 = read_transposed(vt + (16 * ks + 8) * VSTR + 64 * x);
          hit = mfma32<DT>(not_finite<DT>(u4{v0[0], v0[1], v1[0], v1[1]}), not_zero<DT>(pk[ks]), hit);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) o[x][e] = hit[e] > 0.0f ? NAN : o[x][e];
      }
      bool bad = false;
      __syncthreads();
      for (int piece = threadIdx.x; piece < MANY_KEYS * (D / 8); piece += AT_THREADS) {
        u4 *at = reinterpret_cast<u4 *>(&sh.v[t & 1][piece / (D / 8) * VSTR + piece % (D / 8) * 16]);
        *at = finite_only<DT>(*at, bad);
      }
      __syncthreads();
    }
    if (CAREFUL) {
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) vf[x] = v_frag(x);
    }
#pragma unroll
    for (int x = 0; x < 4 * DB; ++x) {
      o[x % DB] = mfma32<DT>(vf[x % AHEAD], pk[x / DB], o[x % DB]);
      if (x + AHEAD < 4 * DB) vf[x % AHEAD] = v_frag(x + AHEAD);
    }
    if (odd) {   // for the tile that comes into this buffer
      __syncthreads();
      for (int x = threadIdx.x; x < MANY_KEYS; x += AT_THREADS) sh.none[t & 1][x] = 0;
      if (threadIdx.x == 0) sh.odd[t & 1] = 0;
    }
  }
  return true;
}

// The rows of place `tile` of the grid: request b's tiles start at
// q_start[b] G / 128 + b, which leaves at least one place a tile. Returns the
// request, -1 where the place is empty.
__device__ __forceinline__ int span_tile(const sb_attention_args &a, int tile, Span &s) {
  const int G = a.q_heads / a.kv_heads;
  int b = 0, bh = a.n_requests;
  while (bh - b > 1) {
    const int mid = (b + bh) >> 1;
    if ((long long)a.q_start[mid] * G / MANY_ROWS + mid <= tile) b = mid;
    else bh = mid;
  }
  span_request(a, b, s);
  const long long r0 = (tile - ((long long)a.q_start[b] * G / MANY_ROWS + b)) * MANY_ROWS;
  if (r0 < 0 || r0 >= s.rows) return -1;
  span_rows(a, (int)r0, MANY_ROWS, s);
  return b;
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
  const int row = r0 + 32 * w + l32, i = row / G, p = s.n - s.m + i;
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
  if (!many_keys<DT, D, false>(a, s, table, kc, vc, q, p, real, t0, count, sh, o, ref, sum))
    many_keys<DT, D, true>(a, s, table, kc, vc, q, p, real, t0, count, sh, o, ref, sum);
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
