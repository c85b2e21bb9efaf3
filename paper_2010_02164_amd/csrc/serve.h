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

// Bytes of workspace of an attention (0: none).
int64_t attention_workspace(const sb_attention_args &a, int n_cu);
// Bytes of workspace that speed a draw up (0: none would).
int64_t sample_workspace(const sb_sample_args &a);

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

}  // namespace sb
