// Products in 8-bit integers: rows quantised with a scale each, and their
// product with quantised weights.
//
// k_quantize: a row a workgroup (or a wave, for short ones), its values kept in
// registers between the pass that finds the largest and the one that divides.
//
// k_linear: sums of int8 products by the matrix unit, exact in 32-bit integers,
// so that they may be split and joined in any order.
#include <hip/hip_runtime.h>

#include "serve.h"

namespace sb {
namespace {

typedef unsigned int u4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i16v __attribute__((ext_vector_type(16)));

constexpr int QT_THREADS = 256;
constexpr int QT_PIECE = 16;   // codes a thread makes at a time

// 16 values of a row from column at, 0 behind the last one.
template <int DT, bool WIDE>
__device__ __forceinline__ void load_values(const void *row, int at, int cols, float (&v)[QT_PIECE]) {
  if (WIDE && at + QT_PIECE <= cols) {
    if constexpr (DT == SB_F32) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const u4 p = *reinterpret_cast<const u4 *>(static_cast<const float *>(row) + at + 4 * x);
#pragma unroll
        for (int y = 0; y < 4; ++y) v[4 * x + y] = __uint_as_float(p[y]);
      }
    } else {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const u4 p = *reinterpret_cast<const u4 *>(static_cast<const uint16_t *>(row) + at + 8 * x);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          v[8 * x + 2 * y] = Half<DT>::to_float(p[y] & 0xFFFFu);
          v[8 * x + 2 * y + 1] = Half<DT>::to_float(p[y] >> 16);
        }
      }
    }
    return;
  }
#pragma unroll
  for (int x = 0; x < QT_PIECE; ++x) {
    v[x] = 0.0f;
    if (at + x < cols) {
      if constexpr (DT == SB_F32) v[x] = static_cast<const float *>(row)[at + x];
      else v[x] = Half<DT>::to_float(static_cast<const uint16_t *>(row)[at + x]);
    }
  }
}

// The whole number next to y / s, |y| <= 127.5 s. The product with the rounded
// reciprocal is off by less than one; which side of the borders (n +- 1/2) s y
// lies on is the sign of one fused operation, which rounding does not change.
__device__ __forceinline__ int nearest(float y, float s, float inv) {
  float n = rintf(y * inv);
  const float above = fmaf(-(n + 0.5f), s, y), below = fmaf(-(n - 0.5f), s, y);
  const bool odd = ((int)n & 1) != 0;
  if (above > 0.0f || (above == 0.0f && odd)) n += 1.0f;
  else if (below < 0.0f || (below == 0.0f && odd)) n -= 1.0f;
  return (int)fminf(fmaxf(n, -127.0f), 127.0f);
}

// ROWS rows a workgroup; PIECES pieces a thread stay in registers, those of longer
// rows are read twice.
template <int DT, int ROWS, int PIECES>
__global__ __launch_bounds__(QT_THREADS) void k_quantize(sb_quantize_args a, int wide) {
  constexpr int T = QT_THREADS / ROWS;   // threads a row
  __shared__ uint32_t tops[QT_THREADS / 64];
  const int t = threadIdx.x % T;
  const long long r = (long long)blockIdx.x * ROWS + threadIdx.x / T;
  const bool real = r < a.rows;
  const int pieces = (a.cols + QT_PIECE - 1) / QT_PIECE;
  const char *row = static_cast<const char *>(a.x) + (real ? r : 0) * a.x_row * (DT == SB_F32 ? 4 : 2);
  float v[PIECES][QT_PIECE];
  uint32_t top = 0;   // sizes compare as their codes do, NaN above infinity above all numbers
  auto load = [&](int piece, float (&to)[QT_PIECE]) {
    if (wide) load_values<DT, true>(row, piece * QT_PIECE, a.cols, to);
    else load_values<DT, false>(row, piece * QT_PIECE, a.cols, to);
  };
  auto look = [&](const float (&from)[QT_PIECE]) {
#pragma unroll
    for (int x = 0; x < QT_PIECE; ++x) top = max(top, __float_as_uint(from[x]) & 0x7FFFFFFFu);
  };
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    if (t + p * T < pieces) {
      load(t + p * T, v[p]);
      look(v[p]);
    }
  }
  for (int piece = t + PIECES * T; piece < pieces; piece += T) {
    float w[QT_PIECE];
    load(piece, w);
    look(w);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  if (T > 64) {
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < QT_THREADS / 64; ++w) top = max(top, tops[w]);
  }
  if (!real) return;
  const bool bad = top >= 0x7F800000u;
  const float scale = bad ? __uint_as_float(0x7FC00000u) : __uint_as_float(top) / 127.0f;
  if (t == 0) a.scales[r] = scale;
  // Small rows are taken 2^64 times as large, scale and values: their quotients
  // are the same, and nothing falls out of fp32's range.
  const float up = scale < 0x1p-80f ? 0x1p64f : 1.0f, s = scale * up;
  const bool none = bad || scale == 0.0f;
  const float inv = none ? 0.0f : 1.0f / s;
  u4 *dst = reinterpret_cast<u4 *>(static_cast<int8_t *>(a.codes) + r * a.codes_row);
  auto store = [&](int piece, const float (&from)[QT_PIECE]) {
    u4 out = {0, 0, 0, 0};
    if (!none) {
#pragma unroll
      for (int x = 0; x < QT_PIECE; ++x) out[x >> 2] |= ((uint32_t)nearest(from[x] * up, s, inv) & 0xFFu) << (8 * (x & 3));
    }
    dst[piece] = out;
  };
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
    if (t + p * T < pieces) store(t + p * T, v[p]);
  for (int piece = t + PIECES * T; piece < pieces; piece += T) {
    float w[QT_PIECE];
    load(piece, w);
    store(piece, w);
  }
}

template <int DT>
hipError_t quantize(const sb_quantize_args &a, hipStream_t s) {
  const int unit = DT == SB_F32 ? 4 : 8;
  const int wide = reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && (a.rows == 1 || a.x_row % unit == 0);
  if (a.cols <= 64 * QT_PIECE)
    hipLaunchKernelGGL((k_quantize<DT, 4, 1>), dim3((unsigned)((a.rows + 3LL) / 4)), dim3(QT_THREADS), 0, s, a, wide);
  else
    hipLaunchKernelGGL((k_quantize<DT, 1, 2>), dim3((unsigned)a.rows), dim3(QT_THREADS), 0, s, a, wide);
  return hipGetLastError();
}

// -- products ------------------------------------------------------------------

// A scale in parts: 1 <= |part| < 2 and a power of two, so that a sum times two
// scales passes no border of fp32 on the way.
struct Scale {
  float part;
  int power;
  __device__ __forceinline__ explicit Scale(float s) : part(__builtin_amdgcn_frexp_mantf(s)), power(__builtin_amdgcn_frexp_expf(s)) {}
};

template <int DT>
__device__ __forceinline__ float scaled(int sum, float sx, float sw, float bias) {
  if constexpr (DT == SB_F32) return (float)((double)sum * sx * sw + bias);
  const Scale x(sx), w(sw);
  return __builtin_amdgcn_ldexpf((float)sum * (x.part * w.part), x.power + w.power) + bias;
}

// 64 x 64 results a workgroup, 32 x 32 a wave, straight from memory.
template <int DT>
__global__ __launch_bounds__(256) void k_linear(sb_linear_args a) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l32 = lane & 31, h2 = lane >> 5;
  const int n0 = blockIdx.x * 64 + (w & 1) * 32, m0 = blockIdx.y * 64 + (w >> 1) * 32;
  const int n = min(n0 + l32, a.channels - 1), m = min(m0 + l32, a.rows - 1);
  const char *wr = static_cast<const char *>(a.w) + n * a.w_row, *xr = static_cast<const char *>(a.x) + m * a.x_row;
  i16v c;
#pragma unroll
  for (int e = 0; e < 16; ++e) c[e] = 0;
  for (int k = 16 * h2; k < a.depth + 16 * h2; k += 32) {
    i4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
    if (k < a.depth) {
      x = *reinterpret_cast<const i4 *>(wr + k);
      y = *reinterpret_cast<const i4 *>(xr + k);
    }
    c = __builtin_amdgcn_mfma_i32_32x32x32_i8(x, y, c, 0, 0, 0);
  }
  const int row = m0 + l32;
  if (row >= a.rows) return;
  const float sx = a.x_scale[row];
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int col = n0 + 8 * (e >> 2) + 4 * h2 + (e & 3);
    if (col >= a.channels) continue;
    const float v = scaled<DT>(c[e], sx, a.w_scale[col], a.bias ? a.bias[col] : 0.0f);
    if constexpr (DT == SB_F32) static_cast<float *>(a.out)[row * a.out_row + col] = v;
    else static_cast<uint16_t *>(a.out)[row * a.out_row + col] = (uint16_t)Half<DT>::pack(v, v);
  }
}

template <int DT>
hipError_t linear(const sb_linear_args &a, int n_cu, void *work, hipStream_t s) {
  hipLaunchKernelGGL((k_linear<DT>), dim3((unsigned)((a.channels + 63LL) / 64), (unsigned)((a.rows + 63LL) / 64)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(const sb_quantize_args &a, hipStream_t s) {
  return a.dtype == SB_F32 ? quantize<SB_F32>(a, s) : a.dtype == SB_BF16 ? quantize<SB_BF16>(a, s) : quantize<SB_F16>(a, s);
}

int64_t linear_workspace(const sb_linear_args &a, int n_cu) { return 0; }

hipError_t launch_linear(const sb_linear_args &a, int n_cu, void *work, hipStream_t s) {
  return a.dtype == SB_F32 ? linear<SB_F32>(a, n_cu, work, s)
                           : a.dtype == SB_BF16 ? linear<SB_BF16>(a, n_cu, work, s) : linear<SB_F16>(a, n_cu, work, s);
}

}  // namespace sb
