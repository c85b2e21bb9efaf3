// Products in 8-bit integers: rows quantised with a scale each, and their
// product with quantised weights. Sums of int8 products by the matrix unit are exact
// in 32-bit integers, so that they may be split and joined in any order.
//
// k_quantize: a row a workgroup (or a wave, for short rows and for many), its values
// kept in registers between the pass that finds the largest and the one that
// divides. 8000 rows of 4096 in bf16: 26 us, 3.8 TB/s.
// k_linear_few: up to 64 rows, bound by reading the weights (in a graph, one after the
// other): 1 x 4096 x 4096 4.8 us, 3.5 TB/s; 61 x 6144 x 4096 13.8 us, where every 32
// channels read all of x again from L2.
// k_linear_tiles: more rows, bound by the matrix unit and what feeds it: 8000 x 8192 x
// 4096 255 to 264 us, 2030 to 2100 TOPS (the unit alone makes 4120; a library product 2170),
// of which, in trials without them, waits for loads take 30, writes to LDS 25. k_linear_join: the
// sums of tiles whose depth was split.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "serve.h"
#include "serve_plan.h"
#include "wave.h"

namespace sb {
namespace {

typedef unsigned int u2 __attribute__((ext_vector_type(2)));
typedef unsigned int u4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i16v __attribute__((ext_vector_type(16)));

constexpr int QT_THREADS = 256;
constexpr int QT_PIECE = 16;   // codes a thread makes at a time

typedef uint32_t at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t at4 __attribute__((ext_vector_type(4), aligned(4)));

// 16 values of a row from column at, 0 behind the last one. Loads of 16 bytes need
// no more than their values' alignment.
template <int DT>
__device__ __forceinline__ void load_values(const void *row, int at, int cols, float (&v)[QT_PIECE]) {
  typedef typename std::conditional<DT == SB_F32, at4, at2>::type any4;
  constexpr int SIZE = DT == SB_F32 ? 4 : 2;
  if (at + QT_PIECE <= cols) {
    const any4 *src = reinterpret_cast<const any4 *>(static_cast<const char *>(row) + (long long)at * SIZE);
#pragma unroll
    for (int x = 0; x < SIZE; ++x) {
      const any4 p = src[x];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        if constexpr (DT == SB_F32) {
          v[4 * x + y] = __uint_as_float(p[y]);
        } else {
          v[8 * x + 2 * y] = Half<DT>::to_float(p[y] & 0xFFFFu);
          v[8 * x + 2 * y + 1] = Half<DT>::to_float(p[y] >> 16);
        }
      }
    }
    return;
  }
#pragma unroll
  for (int x = 0; x < QT_PIECE; ++x) {
    const int i = min(at + x, cols - 1);   // (no branches: all loads at once)
    float f;
    if constexpr (DT == SB_F32) f = static_cast<const float *>(row)[i];
    else f = Half<DT>::to_float(static_cast<const uint16_t *>(row)[i]);
    v[x] = at + x < cols ? f : 0.0f;
  }
}

// The whole number next to y / s, |y| <= 190 s. The product with the rounded
// reciprocal is off by less than one; which side of the borders (n +- 1/2) s y
// lies on is the sign of one fused operation, which rounding does not change.
__device__ __forceinline__ int nearest(float y, float s, float inv) {
  const float n = rintf(y * inv), above = fmaf(-(n + 0.5f), s, y), below = fmaf(-(n - 0.5f), s, y);
  const int odd = (int)n & 1;
  int c = (int)n;
  c += (above > 0.0f) | ((above == 0.0f) & odd);
  c -= (below < 0.0f) | ((below == 0.0f) & odd);
  return min(max(c, -127), 127);
}

// The codes of 16 values. With the product plus 1.5 2^23, whose last place is 1, a
// sum's low byte is the code; the product is off by at most 190 2^-22 < 2^-14, and
// only where it comes so near to a border are the codes found the long way (one
// of 1000 values in 30 does in a wave: 82 us for 8000 rows of 4096 where all went
// the long way).
__device__ __forceinline__ u4 codes_of(const float (&v)[QT_PIECE], float up, float s, float inv) {
  constexpr float SHIFT = 12582912.0f;
  u4 out;
  float far = up > 1.0f ? 1.0f : 0.0f;   // (small scales may be rounded to few bits: quotients pass 127)
#pragma unroll
  for (int x = 0; x < QT_PIECE; x += 4) {
    uint32_t bits[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const float value = v[x + y] * up, sum = fmaf(value, inv, SHIFT);
      far = fmaxf(far, fabsf(fmaf(value, inv, SHIFT - sum)));
      bits[y] = __float_as_uint(sum);
    }
    const uint32_t lo = __builtin_amdgcn_perm(bits[1], bits[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(bits[3], bits[2], 0x0C0C0400u);
    out[x >> 2] = lo | hi << 16;
  }
  if (far > 0.5f - 0x1p-14f) {
#pragma unroll
    for (int x = 0; x < QT_PIECE; x += 4) {
      __builtin_amdgcn_sched_barrier(0);   // (4 at a time: few registers)
      out[x >> 2] = 0;
#pragma unroll
      for (int y = 0; y < 4; ++y) out[x >> 2] |= ((uint32_t)nearest(v[x + y] * up, s, inv) & 0xFFu) << (8 * y);
    }
  }
  return out;
}

template <int S>
__device__ __forceinline__ uint32_t max_stage(uint32_t v) {
  uint32_t x, y;
  stage32<S>(v, x, y);
  return max(x, y);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  return max_stage<5>(max_stage<4>(max_stage<3>(max_stage<2>(max_stage<1>(max_stage<0>(v))))));
}

// ROWS rows a workgroup; PIECES pieces a thread stay in registers, those of longer
// rows are read twice.
template <int DT, int ROWS, int PIECES>
__global__ __launch_bounds__(QT_THREADS) void k_quantize(sb_quantize_args a) {
  constexpr int T = QT_THREADS / ROWS;   // threads a row
  __shared__ uint32_t tops[QT_THREADS / 64];
  const int t = threadIdx.x % T;
  const long long r = (long long)blockIdx.x * ROWS + threadIdx.x / T;
  const bool real = r < a.rows;
  const int pieces = (a.cols + QT_PIECE - 1) / QT_PIECE;
  const char *row = static_cast<const char *>(a.x) + (real ? r : 0) * a.x_row * (DT == SB_F32 ? 4 : 2);
  float v[PIECES][QT_PIECE];
  uint32_t top = 0;   // sizes compare as their codes do, NaN above infinity above all numbers
  auto load = [&](int piece, float (&to)[QT_PIECE]) { load_values<DT>(row, piece * QT_PIECE, a.cols, to); };
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
  top = wave_max(top);
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
    dst[piece] = none ? u4{0, 0, 0, 0} : codes_of(from, up, s, inv);
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
  // Rows enough to fill the card go by waves, which do not wait for each other.
  const int wave = 64 * QT_PIECE;
  if (a.cols <= wave)
    hipLaunchKernelGGL((k_quantize<DT, 4, 1>), dim3((unsigned)((a.rows + 3LL) / 4)), dim3(QT_THREADS), 0, s, a);
  else if (a.rows >= 2048 && a.cols <= 4 * wave)
    hipLaunchKernelGGL((k_quantize<DT, 4, 4>), dim3((unsigned)((a.rows + 3LL) / 4)), dim3(QT_THREADS), 0, s, a);
  else if (a.cols <= 4 * wave)
    hipLaunchKernelGGL((k_quantize<DT, 1, 1>), dim3((unsigned)a.rows), dim3(QT_THREADS), 0, s, a);
  else
    hipLaunchKernelGGL((k_quantize<DT, 1, 4>), dim3((unsigned)a.rows), dim3(QT_THREADS), 0, s, a);
  return hipGetLastError();
}

// -- products ------------------------------------------------------------------

// A scale in parts: 1/2 <= |part| < 1 (0 for 0) and a power of two, so that a sum times
// two scales passes no border of fp32 on the way.
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

// W channels of a row side by side, those that there are. wide: rows of 16 bytes
// and more start at multiples of 16. (Rows of an odd number of channels go a value a
// store: 200 x 32001 x 1000 in fp32 37 us, of 32000 19; 8000 x 8193 x 4096 in bf16 444,
// of 8192 255.)
template <int DT, int W>
__device__ __forceinline__ void store_side_by_side(const sb_linear_args &a, int m, int n, const float (&v)[W], bool wide) {
  const long long at = m * a.out_row + n;
  if (wide && n + W <= a.channels) {
    if constexpr (DT == SB_F32) {
#pragma unroll
      for (int y = 0; y < W; y += 4) *reinterpret_cast<f4 *>(static_cast<float *>(a.out) + at + y) = f4{v[y], v[y + 1], v[y + 2], v[y + 3]};
    } else {
      uint32_t p[W / 2];
#pragma unroll
      for (int y = 0; y < W; y += 2) p[y >> 1] = Half<DT>::pack(v[y], v[y + 1]);
      if constexpr (W == 8) *reinterpret_cast<u4 *>(static_cast<uint16_t *>(a.out) + at) = u4{p[0], p[1], p[2], p[3]};
      else *reinterpret_cast<u2 *>(static_cast<uint16_t *>(a.out) + at) = u2{p[0], p[1]};
    }
    return;
  }
#pragma unroll
  for (int y = 0; y < W; ++y) {
    if (n + y >= a.channels) continue;
    if constexpr (DT == SB_F32) static_cast<float *>(a.out)[at + y] = v[y];
    else static_cast<uint16_t *>(a.out)[at + y] = (uint16_t)Half<DT>::pack(v[y], v[y]);
  }
}

// -- few rows: the weights straight to the matrix unit ---------------------------
//
// Up to 64 rows of x: reading the weights binds. A workgroup takes 16 channels, its
// waves a stretch of the depth each, in pieces of 64 that are loaded as the matrix
// unit wants them (lane: channel l % 16, values 16 (l / 16) .. + 15); the waves'
// sums meet in LDS.

template <int DT, int MT, int NT>
__global__ __launch_bounds__(64 * FEW_WAVES) void k_linear_few(sb_linear_args a, bool wide) {
  constexpr int BATCH = MT == 1 ? 8 : 4;   // pieces in flight
  static_assert(FEW_WAVES >= MT * NT, "a thread for every 4 results");
  __shared__ alignas(16) int sums[FEW_WAVES][16 * MT][16 * NT];   // [wave][row of x][channel]
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l16 = lane & 15, g4 = lane >> 4, n0 = blockIdx.x * (16 * NT);
  const unsigned char *wp[NT], *xp[MT];
#pragma unroll
  for (int j = 0; j < NT; ++j) wp[j] = static_cast<const unsigned char *>(a.w) + min(n0 + 16 * j + l16, a.channels - 1) * a.w_row;
#pragma unroll
  for (int i = 0; i < MT; ++i) xp[i] = static_cast<const unsigned char *>(a.x) + min(16 * i + l16, a.rows - 1) * a.x_row;
  // What the results are scaled by is loaded ahead.
  const int m = threadIdx.x / (4 * NT), at4 = threadIdx.x % (4 * NT) * 4, n = n0 + at4;
  const bool mine = m < min(a.rows, 16 * MT);
  float sx = 0.0f, sw[4], bias[4];
  if (mine) {
    sx = a.x_scale[m];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const int at = min(n + y, a.channels - 1);
      sw[y] = a.w_scale[at];
      bias[y] = a.bias ? a.bias[at] : 0.0f;
    }
  }
  i4 c[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) c[i][j] = i4{0, 0, 0, 0};
  const int steps = (a.depth + FEW_STEP - 1) / FEW_STEP, each = (steps + FEW_WAVES - 1) / FEW_WAVES;
  const int end = min(min(w * each + each, steps) * FEW_STEP, a.depth);
  auto batch = [&](int k0, auto whole) {   // BATCH pieces; not whole: those before the end
    i4 wv[BATCH][NT], xv[BATCH][MT];
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const int k = k0 + u * FEW_STEP + 16 * g4, at = decltype(whole)::value ? k : min(k, a.depth - 16);
#pragma unroll
      for (int j = 0; j < NT; ++j) wv[u][j] = *reinterpret_cast<const i4 *>(wp[j] + at);
#pragma unroll
      for (int i = 0; i < MT; ++i) xv[u][i] = *reinterpret_cast<const i4 *>(xp[i] + at);
    }
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const int k = k0 + u * FEW_STEP + 16 * g4;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        if (!decltype(whole)::value && k >= end) wv[u][j] = i4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < MT; ++i) c[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[u][j], xv[u][i], c[i][j], 0, 0, 0);
      }
    }
  };
  int k = w * each * FEW_STEP;
  for (; k + BATCH * FEW_STEP <= end; k += BATCH * FEW_STEP) batch(k, std::true_type());
  if (k < end) batch(k, std::false_type());
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) *reinterpret_cast<i4 *>(&sums[w][16 * i + l16][16 * j + 4 * g4]) = c[i][j];
  __syncthreads();
  if (!mine) return;
  i4 total = {0, 0, 0, 0};
#pragma unroll
  for (int x = 0; x < FEW_WAVES; ++x) total += *reinterpret_cast<const i4 *>(&sums[x][m][at4]);
  float v[4];
#pragma unroll
  for (int y = 0; y < 4; ++y) v[y] = scaled<DT>(total[y], sx, sw[y], bias[y]);
  store_side_by_side<DT, 4>(a, m, n, v, wide);
}

// -- many rows: tiles in LDS -----------------------------------------------------
//
// A workgroup of 2 x 2 waves makes 64 MT rows of x by 64 NT channels, 128 values of
// the depth at a time. LDS has two such tiles of both operands, one worked on
// while the other is filled from registers that were loaded a tile before. In
// LDS a row is 128 bytes, its 16-byte pieces at place piece ^ (a number of the
// row), so that the lanes of an operand's read, which take one piece of rows that
// follow each other, use all banks. The matrix unit's rows are channels: a lane
// then has 4 channels of one row of x side by side, and 8 with the next product's,
// since the channels are dealt out to products in turns of 4.

template <int MT, int NT>
struct TileShared {
  alignas(16) unsigned char x[2][64 * MT * TILE_K];
  alignas(16) unsigned char w[2][64 * NT * TILE_K];
  alignas(16) float x_scale[64 * MT], w_scale[64 * NT], bias[64 * NT];   // (read from memory at the end they took a quarter of the time)
};

__device__ __forceinline__ int x_place(int row, int piece) { return row * TILE_K + ((piece ^ (row & 7)) << 4); }
__device__ __forceinline__ int w_place(int row, int piece) { return row * TILE_K + ((piece ^ ((row & 3) | ((row >> 1) & 4))) << 4); }

// Spreads READS reads and WRITES writes of LDS and LOADS loads over PRODUCTS products
// of the matrix unit, which all came before it.
template <int PRODUCTS, int READS, int WRITES, int LOADS, int X = 0>
__device__ __forceinline__ void interleave() {
  if constexpr (X < PRODUCTS) {
    // (Reads in the first half: the products behind them wait for them.)
    constexpr int H = (PRODUCTS + 1) / 2, Y = X < H ? X + 1 : H;
    constexpr int r = READS * Y / H - READS * (X < H ? X : H) / H, w = WRITES * (X + 1) / PRODUCTS - WRITES * X / PRODUCTS;
    constexpr int l = LOADS * (X + 1) / PRODUCTS - LOADS * X / PRODUCTS;
    if constexpr (r > 0) __builtin_amdgcn_sched_group_barrier(0x100, r, 0);
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if constexpr (w > 0) __builtin_amdgcn_sched_group_barrier(0x200, w, 0);
    if constexpr (l > 0) __builtin_amdgcn_sched_group_barrier(0x020, l, 0);
    interleave<PRODUCTS, READS, WRITES, LOADS, X + 1>();
  } else {
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Which tile is number p: blocks of GROUP tiles of rows by all of channels, so that
// those that follow each other share operands.
__device__ __forceinline__ void tile_place(int p, int tiles_m, int tiles_n, int &m, int &n) {
  constexpr int GROUP = 4;
  const int g = p / (GROUP * tiles_n), in = p - g * (GROUP * tiles_n), high = min(tiles_m - g * GROUP, GROUP);
  m = g * GROUP + in % high;
  n = in / high;
}

template <int DT, int MT, int NT, bool SPLIT>
__global__ __launch_bounds__(256, MT * NT <= 4 ? 2 : 1) void k_linear_tiles(sb_linear_args a, int tiles_m, int tiles_n, bool wide, int split_into,
                                                                            void *work) {
  constexpr int BM = 64 * MT, BN = 64 * NT, KS = TILE_K / 32;
  constexpr int XP = BM * 8 / 256, WP = BN * 8 / 256;   // 16-byte pieces of a tile that a thread brings
  __shared__ TileShared<MT, NT> sh;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l32 = lane & 31, h2 = lane >> 5;
  // Workgroups go to the 8 XCDs in turn: each gets tiles that follow each other (or all
  // splits of few).
  const int splits = SPLIT ? split_into : 1, all = tiles_m * tiles_n * splits, xcd = blockIdx.x & 7, per = all >> 3, more = all & 7;
  const int y = xcd * per + min(xcd, more) + (int)(blockIdx.x >> 3), p = y / splits, split = y - p * splits;
  int m0, n0;
  tile_place(p, tiles_m, tiles_n, m0, n0);
  m0 *= BM;
  n0 *= BN;
  const int row0 = threadIdx.x >> 3, piece = threadIdx.x & 7;
  if (threadIdx.x < BM) sh.x_scale[threadIdx.x] = a.x_scale[min(m0 + (int)threadIdx.x, a.rows - 1)];
  if (threadIdx.x < BN) {
    const int n = min(n0 + (int)threadIdx.x, a.channels - 1);
    sh.w_scale[threadIdx.x] = a.w_scale[n];
    sh.bias[threadIdx.x] = a.bias ? a.bias[n] : 0.0f;
  }
  const unsigned char *xs[XP], *ws[WP];
#pragma unroll
  for (int i = 0; i < XP; ++i) xs[i] = static_cast<const unsigned char *>(a.x) + min(m0 + row0 + 32 * i, a.rows - 1) * a.x_row + 16 * piece;
#pragma unroll
  for (int i = 0; i < WP; ++i) ws[i] = static_cast<const unsigned char *>(a.w) + min(n0 + row0 + 32 * i, a.channels - 1) * a.w_row + 16 * piece;
  u4 xr[XP], wr[WP];
  const int all_steps = (a.depth + TILE_K - 1) / TILE_K, each = (all_steps + splits - 1) / splits;
  const int step0 = min(split * each, all_steps), steps = min(each, all_steps - step0), k0 = step0 * TILE_K;   // (steps 0: nothing is left)
  auto load_x = [&](int k) {
    const int at = min(k0 + k, a.depth - 16 - 16 * piece);   // (behind the last value: any that is)
#pragma unroll
    for (int i = 0; i < XP; ++i) xr[i] = *reinterpret_cast<const u4 *>(xs[i] + at);
  };
  auto load_w = [&](int k) {
    const int at = min(k0 + k, a.depth - 16 - 16 * piece);
#pragma unroll
    for (int i = 0; i < WP; ++i) wr[i] = *reinterpret_cast<const u4 *>(ws[i] + at);
  };
  auto write_x = [&](int k, int to, auto last) {   // of the last tile, zeros behind the last value
    const unsigned int keep = !decltype(last)::value || k0 + k + 16 * piece < a.depth ? ~0u : 0u;
#pragma unroll
    for (int i = 0; i < XP; ++i) *reinterpret_cast<u4 *>(&sh.x[to][x_place(row0 + 32 * i, piece)]) = xr[i] & keep;
  };
  auto write_w = [&](int to) {
#pragma unroll
    for (int i = 0; i < WP; ++i) *reinterpret_cast<u4 *>(&sh.w[to][w_place(row0 + 32 * i, piece)]) = wr[i];
  };
  const int xrow = (w >> 1) * 32 * MT + l32, wrow = (w & 1) * 32 * NT + (l32 >> 2) * 8 + (l32 & 3);
  i4 xf[2][MT], wf[2][NT];
  auto fetch = [&](int from, int ks, int to) {
#pragma unroll
    for (int i = 0; i < MT; ++i) xf[to][i] = *reinterpret_cast<const i4 *>(&sh.x[from][x_place(xrow + 32 * i, 2 * ks + h2)]);
#pragma unroll
    for (int j = 0; j < NT; ++j) wf[to][j] = *reinterpret_cast<const i4 *>(&sh.w[from][w_place(wrow + 64 * (j >> 1) + 4 * (j & 1), 2 * ks + h2)]);
  };
  i16v c[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) c[i][j][e] = 0;
  auto multiply = [&](int from) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) c[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[from][j], xf[from][i], c[i][j], 0, 0, 0);
  };
  // A step's work: operands come from LDS 32 values before their products; in between
  // the next step's go to LDS (WRITE) and those of the one after it are loaded (LOAD).
  auto tile = [&](int t, auto write_next, auto load_next) {
    constexpr bool WRITE = decltype(write_next)::value, LOAD = decltype(load_next)::value;
    const int cur = t & 1, next = cur ^ 1;
    fetch(cur, 1, 1);
    if constexpr (WRITE) write_x((t + 1) * TILE_K, next, std::bool_constant<!LOAD>());
    multiply(0);
    interleave<MT * NT, MT + NT, WRITE ? XP : 0, 0>();
    fetch(cur, 2, 0);
    if constexpr (LOAD) load_x((t + 2) * TILE_K);
    if constexpr (WRITE) write_w(next);
    multiply(1);
    interleave<MT * NT, MT + NT, WRITE ? WP : 0, LOAD ? XP : 0>();
    fetch(cur, 3, 1);
    if constexpr (LOAD) load_w((t + 2) * TILE_K);
    multiply(0);
    interleave<MT * NT, MT + NT, 0, LOAD ? WP : 0>();
    if constexpr (WRITE) {   // all of this step's is in registers, the next one's in LDS
      __syncthreads();
      fetch(next, 0, 0);
    }
    multiply(1);
    interleave<MT * NT, WRITE ? MT + NT : 0, 0, 0>();
  };
  const std::true_type yes;
  const std::false_type no;
  load_x(0);
  load_w(0);
  write_x(0, 0, yes);
  write_w(0);
  load_x(TILE_K);
  load_w(TILE_K);
  __syncthreads();
  fetch(0, 0, 0);
  int t = 0;
  for (; t + 2 < steps; ++t) tile(t, yes, yes);
  if (t + 1 < steps) tile(t++, yes, no);
  tile(t, no, no);
  if constexpr (SPLIT) {   // sums as the threads hold them; k_linear_join adds them up
    i4 *dst = static_cast<i4 *>(work) + ((long long)p * splits + split) * (MT * NT * 4) * 256 + threadIdx.x;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 16; e += 4) dst[((i * NT + j) * 4 + (e >> 2)) * 256] = i4{c[i][j][e], c[i][j][e + 1], c[i][j][e + 2], c[i][j][e + 3]};
    return;
  }
  // Lane: row m, of products j and j + 1 channels 8 (2 (e / 4) + h2) + 4 (j % 2) + e % 4.
#pragma unroll
  for (int j = 0; j < NT; j += 2) {
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int at = (w & 1) * 32 * NT + 64 * (j >> 1) + 8 * (2 * (e >> 2) + h2), n = n0 + at;
      float sw[8], bias[8];
#pragma unroll
      for (int y = 0; y < 8; y += 4) {
        const f4 s4 = *reinterpret_cast<const f4 *>(&sh.w_scale[at + y]), b4 = *reinterpret_cast<const f4 *>(&sh.bias[at + y]);
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          sw[y + z] = s4[z];
          bias[y + z] = b4[z];
        }
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int row = (w >> 1) * 32 * MT + 32 * i + l32, m = m0 + row;
        if (m >= a.rows) continue;
        const float sx = sh.x_scale[row];
        float v[8];
#pragma unroll
        for (int y = 0; y < 8; ++y) v[y] = scaled<DT>(c[i][j + (y >> 2)][e + (y & 3)], sx, sw[y], bias[y]);
        store_side_by_side<DT, 8>(a, m, n, v, wide);
      }
    }
  }
}

// The sums of a tile's splits, scaled: a workgroup 8 of each thread's.
template <int DT, int MT, int NT>
__global__ __launch_bounds__(256) void k_linear_join(sb_linear_args a, int tiles_m, int tiles_n, bool wide, int splits, const void *work) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l32 = lane & 31, h2 = lane >> 5, p = blockIdx.x;
  const int e = (int)blockIdx.y & 3, i = (int)(blockIdx.y >> 2) % MT, j = (int)(blockIdx.y >> 2) / MT * 2;
  int m0, n0;
  tile_place(p, tiles_m, tiles_n, m0, n0);
  const int m = m0 * 64 * MT + (w >> 1) * 32 * MT + 32 * i + l32, n = n0 * 64 * NT + (w & 1) * 32 * NT + 64 * (j >> 1) + 8 * (2 * e + h2);
  const float sx = a.x_scale[min(m, a.rows - 1)];
  float sw[8], bias[8];
#pragma unroll
  for (int y = 0; y < 8; ++y) {
    const int at = min(n + y, a.channels - 1);
    sw[y] = a.w_scale[at];
    bias[y] = a.bias ? a.bias[at] : 0.0f;
  }
  i4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
  const i4 *src = static_cast<const i4 *>(work) + (long long)p * splits * (MT * NT * 4) * 256 + ((i * NT + j) * 4 + e) * 256 + threadIdx.x;
#pragma unroll 8
  for (int x = 0; x < splits; ++x, src += MT * NT * 4 * 256) {
    lo += src[0];
    hi += src[4 * 256];
  }
  if (m >= a.rows) return;
  float v[8];
#pragma unroll
  for (int y = 0; y < 8; ++y) v[y] = scaled<DT>(y < 4 ? lo[y & 3] : hi[y & 3], sx, sw[y], bias[y]);
  store_side_by_side<DT, 8>(a, m, n, v, wide);
}

template <int DT>
hipError_t linear(const sb_linear_args &a, int n_cu, void *work, hipStream_t s) {
  const bool wide = (a.out_row * (DT == SB_F32 ? 4 : 2)) % 16 == 0 && reinterpret_cast<uintptr_t>(a.out) % 16 == 0;
  const LinearPlan p = linear_plan(a, n_cu);
  if (p.tile == 0) {
    const auto few = [&](auto kernel, int channels) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)((a.channels + channels - 1) / channels)), dim3(64 * FEW_WAVES), 0, s, a, wide);
      return hipGetLastError();
    };
    if (a.rows <= 16) return few(k_linear_few<DT, 1, 1>, 16);
    if (a.rows <= 32) return few(k_linear_few<DT, 2, 2>, 32);
    return few(k_linear_few<DT, 4, 2>, 32);
  }
  const dim3 grid((unsigned)((long long)p.m * p.n * p.splits));
  const auto tiles = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, p.m, p.n, wide, p.splits, work);
    return hipGetLastError();
  };
  if (p.tile == 256) return tiles(k_linear_tiles<DT, 4, 4, false>);
  if (p.splits == 1) return tiles(k_linear_tiles<DT, 2, 2, false>);
  const hipError_t e = tiles(k_linear_tiles<DT, 2, 2, true>);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_linear_join<DT, 2, 2>), dim3((unsigned)(p.m * p.n), 8), dim3(256), 0, s, a, p.m, p.n, wide, p.splits, work);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(const sb_quantize_args &a, hipStream_t s) {
  return a.dtype == SB_F32 ? quantize<SB_F32>(a, s) : a.dtype == SB_BF16 ? quantize<SB_BF16>(a, s) : quantize<SB_F16>(a, s);
}

int64_t linear_workspace(const sb_linear_args &a, int n_cu) {
  if (a.rows == 0) return 0;
  const LinearPlan p = linear_plan(a, n_cu);
  return p.splits == 1 ? 0 : (int64_t)p.m * p.n * p.splits * 128 * 128 * 4;
}

hipError_t launch_linear(const sb_linear_args &a, int n_cu, void *work, hipStream_t s) {
  return a.dtype == SB_F32 ? linear<SB_F32>(a, n_cu, work, s)
                           : a.dtype == SB_BF16 ? linear<SB_BF16>(a, n_cu, work, s) : linear<SB_F16>(a, n_cu, work, s);
}

}  // namespace sb
