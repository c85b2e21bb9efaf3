// Rotary positions of a step's queries and keys, and the write of its keys
// and values into the paged cache.
//
// One pass: 16-byte loads, the rotation in registers, 16-byte stores; q, k and
// v are read once and written once, so the kernel is bound by memory. The
// angle of a (token, pair) is the same for every head, so a workgroup takes
// its tokens' cosines and sines once and keeps them in LDS. Angles are in
// turns: position * inv_freq / 2 pi is taken and brought to [-1/2, 1/2] in
// fp64 (at position 10^6 an fp32 angle would be off by 0.03 radians), the
// cosine and sine of the rest in fp32. 16000 tokens, 32 + 8 heads of 128: 73 us,
// 5.4 TB/s (a copy of twice that size: 4.9); one token: 2.9 us.
#include "serve.h"

namespace sb {
namespace {

typedef unsigned int u4 __attribute__((ext_vector_type(4)));

constexpr int ROPE_THREADS = 256;

template <int DT>
__device__ __forceinline__ void unpack(const u4 &x, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = Half<DT>::to_float(x[i] & 0xFFFFu);
    f[2 * i + 1] = Half<DT>::to_float(x[i] >> 16);
  }
}

template <int DT>
__device__ __forceinline__ u4 repack(const float (&f)[8]) {
  return u4{Half<DT>::pack(f[0], f[1]), Half<DT>::pack(f[2], f[3]), Half<DT>::pack(f[4], f[5]), Half<DT>::pack(f[6], f[7])};
}

// TB tokens a workgroup. A task is one 16-byte piece of a head (for rotated
// pairs of the half layout: its two pieces), for all TB tokens.
template <int DT, int LAYOUT, int TB>
__global__ __launch_bounds__(ROPE_THREADS) void k_rope(sb_rope_args a) {
  extern __shared__ float2 turn[];   // [TB][n_pairs] cos, sin
  __shared__ long long s_slot[TB];
  const int t0 = blockIdx.x * TB, np = a.n_pairs;
  const long long n_slots = (long long)a.n_pages * a.page_size;
  if (threadIdx.x < TB) {
    const int t = t0 + threadIdx.x;
    const long long s = t < a.n_tokens ? a.slots[t] : -1;
    s_slot[threadIdx.x] = s < n_slots ? s : -1;
  }
  for (int i = threadIdx.x; i < TB * np; i += ROPE_THREADS) {
    const int tb = i / np, t = min(t0 + tb, a.n_tokens - 1);
    const double turns = (double)a.positions[t] * a.inv_freq[i - tb * np] * 0.15915494309189533577;
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    turn[i] = make_float2(a.mscale * c, a.mscale * s);
  }
  __syncthreads();
  const int per_copy = a.head_dim / 8;
  const int pairs8 = LAYOUT == SB_ROPE_HALF ? np / 8 : np / 4;          // rotated pieces (or pairs of pieces) of a head
  const int per_rot = LAYOUT == SB_ROPE_HALF ? per_copy - pairs8 : per_copy;
  const int n_q = a.q_heads * per_rot, n_k = a.kv_heads * per_rot, n_v = a.kv_heads * per_copy;
  for (int i = threadIdx.x; i < n_q + n_k + n_v; i += ROPE_THREADS) {
    const int kind = i < n_q ? 0 : i < n_q + n_k ? 1 : 2;
    const int j = i - (kind == 0 ? 0 : kind == 1 ? n_q : n_q + n_k);
    const int per = kind == 2 ? per_copy : per_rot;
    const int h = j / per, c = j - h * per;
    const bool rotated = kind != 2 && c < pairs8;
    // Column of the (first) piece.
    const int col = kind != 2 && LAYOUT == SB_ROPE_HALF && !rotated ? (c + pairs8) * 8 : c * 8;
    const uint16_t *src = static_cast<const uint16_t *>(kind == 0 ? a.q : kind == 1 ? a.k : a.v);
    const long long s_tok = kind == 0 ? a.q_token : kind == 1 ? a.k_token : a.v_token;
    src += h * (kind == 0 ? a.q_head : kind == 1 ? a.k_head : a.v_head) + col;
    u4 x[TB], y[TB];
#pragma unroll
    for (int tb = 0; tb < TB; ++tb) {
      if (s_slot[tb] < 0) continue;
      const uint16_t *p = src + (t0 + tb) * s_tok;
      x[tb] = *reinterpret_cast<const u4 *>(p);
      if (LAYOUT == SB_ROPE_HALF && rotated) y[tb] = *reinterpret_cast<const u4 *>(p + np);
    }
#pragma unroll
    for (int tb = 0; tb < TB; ++tb) {
      const long long slot = s_slot[tb];
      if (slot < 0) continue;
      if (rotated) {
        float f[8];
        unpack<DT>(x[tb], f);
        if constexpr (LAYOUT == SB_ROPE_HALF) {
          float g[8];
          unpack<DT>(y[tb], g);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 cs = turn[tb * np + c * 8 + e];
            const float u = f[e], v = g[e];
            f[e] = u * cs.x - v * cs.y;
            g[e] = u * cs.y + v * cs.x;
          }
          y[tb] = repack<DT>(g);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 cs = turn[tb * np + c * 4 + e];
            const float u = f[2 * e], v = f[2 * e + 1];
            f[2 * e] = u * cs.x - v * cs.y;
            f[2 * e + 1] = u * cs.y + v * cs.x;
          }
        }
        x[tb] = repack<DT>(f);
      }
      uint16_t *p;
      if (kind == 0) {
        p = static_cast<uint16_t *>(a.q_out) + (t0 + tb) * a.out_token + h * a.out_head + col;
      } else {
        const int page = (int)(slot / a.page_size), place = (int)(slot - (long long)page * a.page_size);
        p = kind == 1 ? static_cast<uint16_t *>(a.k_cache) + page * a.kc_page + place * a.kc_slot + h * a.kc_head + col
                      : static_cast<uint16_t *>(a.v_cache) + page * a.vc_page + place * a.vc_slot + h * a.vc_head + col;
      }
      *reinterpret_cast<u4 *>(p) = x[tb];
      if (LAYOUT == SB_ROPE_HALF && rotated) *reinterpret_cast<u4 *>(p + np) = y[tb];
    }
  }
}

template <int DT, int LAYOUT>
hipError_t launch(const sb_rope_args &a, int n_cu, hipStream_t s) {
  // Four tokens a workgroup where one leaves it threads without a piece and there
  // are tokens enough for all units (16000 tokens, 24 + 4 heads of 64: 24.9 us, by
  // single tokens 26.6; 16 + 4 of 128: 35.3 and 32.5; 32 + 8 of 128: 83 and 73;
  // 1024 tokens, 16 + 4 of 64: 5.4 and 4.2).
  const long long pieces = ((long long)a.q_heads + 2 * a.kv_heads) * (a.head_dim / 8);
  if (a.n_tokens >= 16 * n_cu && pieces <= ROPE_THREADS)
    hipLaunchKernelGGL((k_rope<DT, LAYOUT, 4>), dim3((a.n_tokens + 3) / 4), dim3(ROPE_THREADS), 4 * a.n_pairs * sizeof(float2), s, a);
  else
    hipLaunchKernelGGL((k_rope<DT, LAYOUT, 1>), dim3(a.n_tokens), dim3(ROPE_THREADS), a.n_pairs * sizeof(float2), s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const sb_rope_args &a, int n_cu, hipStream_t s) {
  if (a.n_tokens == 0) return hipSuccess;
  if (a.dtype == SB_BF16)
    return a.layout == SB_ROPE_HALF ? launch<SB_BF16, SB_ROPE_HALF>(a, n_cu, s) : launch<SB_BF16, SB_ROPE_INTERLEAVED>(a, n_cu, s);
  return a.layout == SB_ROPE_HALF ? launch<SB_F16, SB_ROPE_HALF>(a, n_cu, s) : launch<SB_F16, SB_ROPE_INTERLEAVED>(a, n_cu, s);
}

}  // namespace sb
