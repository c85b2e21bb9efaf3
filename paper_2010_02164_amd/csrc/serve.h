// Launchers and small device helpers of the serving operators (cached
// decoding and sampled tokens).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/streambeam.h"

namespace sb {

// Text that sb_last_error(NULL) gives on this thread.
void set_call_error(const char *msg);

// Each returns the launch status; the arguments are checked already.
hipError_t launch_plan(const sb_plan_args &a, hipStream_t s);
hipError_t launch_rope(const sb_rope_args &a, int n_cu, hipStream_t s);
hipError_t launch_paged_attention(const sb_attention_args &a, int n_cu, void *work, hipStream_t s);
hipError_t launch_sample(const sb_sample_args &a, void *workspace, int n_cu, hipStream_t s);   // workspace: may be null

hipError_t launch_shared_attention(const sb_shared_args &a, int n_cu, void *work, hipStream_t s);
hipError_t launch_bounds(const sb_bounds_args &a, hipStream_t s);
hipError_t launch_select(const sb_select_args &a, int n_cu, void *work, hipStream_t s);
hipError_t launch_selected_attention(const sb_selected_args &a, int n_cu, void *work, hipStream_t s);
hipError_t launch_quantize(const sb_quantize_args &a, hipStream_t s);
hipError_t launch_linear(const sb_linear_args &a, int n_cu, void *work, hipStream_t s);

// Bytes of workspace of an attention (0: none).
int64_t attention_workspace(const sb_attention_args &a, int n_cu);
int64_t shared_workspace(const sb_shared_args &a, int n_cu);
int64_t selected_workspace(const sb_selected_args &a, int n_cu);
// Bytes of workspace that speed a draw up (0: none would).
int64_t sample_workspace(const sb_sample_args &a);
// Bytes of workspace of a selection.
int64_t select_workspace(const sb_select_args &a);
// Bytes of workspace of a product (0: none).
int64_t linear_workspace(const sb_linear_args &a, int n_cu);

// 16-bit storage types by their dtype code: the value as float, and the
// nearest code of a float (ties to even).
template <int DT>
struct Half;
template <>
struct Half<SB_BF16> {
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  typedef __bf16 v2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ float to_float(uint32_t code) { return __uint_as_float(code << 16); }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const v2 p = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, p);
  }
};
template <>
struct Half<SB_F16> {
  typedef _Float16 v8 __attribute__((ext_vector_type(8)));
  typedef _Float16 v2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ float to_float(uint32_t code) {
    return (float)__builtin_bit_cast(_Float16, (uint16_t)code);
  }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const v2 p = {(_Float16)lo, (_Float16)hi};
    return __builtin_bit_cast(uint32_t, p);
  }
};

// Sums over the lanes up to each, through the lanes' own paths (a shuffle
// through LDS takes about 130 cycles).
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned long long from_before(unsigned long long v) {   // 0 where nothing comes
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xF, false);
  return ((unsigned long long)hi << 32) | lo;
}
__device__ __forceinline__ unsigned long long wave_scan(unsigned long long v) {   // inclusive
  v += from_before<0x111, 0xF>(v);   // within 16 lanes: from 1, 2, 4, 8 before
  v += from_before<0x112, 0xF>(v);
  v += from_before<0x114, 0xF>(v);
  v += from_before<0x118, 0xF>(v);
  v += from_before<0x142, 0xA>(v);   // the last of the first and third 16 to the next
  v += from_before<0x143, 0xC>(v);   // the last of the first 32 to the others
  return v;
}

}  // namespace sb
