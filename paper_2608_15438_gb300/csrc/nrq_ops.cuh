// Device and host helpers shared by the encoder operators (neuroute_ops.h):
// element types, vector access, activations, the 8-bit form.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "neuroute_ops.h"
#include "nr_internal.cuh"

constexpr int kOpsGroup = 32;  // columns that share a checkpoint's scale

// ------------------------------------------------------------ element types
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// one element of a runtime type
__device__ __forceinline__ float load_any(const void *p, int64_t i, int dtype) {
  if (dtype == NR_F32) return static_cast<const float *>(p)[i];
  if (dtype == NR_F16) return to_f32(static_cast<const __half *>(p)[i]);
  return to_f32(static_cast<const __nv_bfloat16 *>(p)[i]);
}
__device__ __forceinline__ void store_any(void *p, int64_t i, int dtype, float v) {
  if (dtype == NR_F32) static_cast<float *>(p)[i] = v;
  else if (dtype == NR_F16) static_cast<__half *>(p)[i] = __float2half_rn(v);
  else static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
}

// ------------------------------------------------------------ activations
// Phi(z) = erfc(-z / sqrt 2) / 2: no cancellation in the negative tail
__device__ __forceinline__ float normal_cdf(float z) { return 0.5f * erfcf(-0.70710678118654752f * z); }

__device__ __forceinline__ float act_value(float z, int act) {
  if (act == NR_ACT_RELU) return z < 0.0f ? 0.0f : z;  // keeps a NaN
  if (act == NR_ACT_GELU) return z == -INFINITY ? 0.0f : z * normal_cdf(z);
  if (act == NR_ACT_SILU) return z == -INFINITY ? 0.0f : z / (1.0f + __expf(-z));
  return z;
}
// the derivative
__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == NR_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
  if (act == NR_ACT_GELU) {
    const float tail = fabsf(z) < 15.0f ? z * __expf(-0.5f * z * z) * 0.39894228040143268f : 0.0f;
    return z != z ? z : normal_cdf(z) + tail;
  }
  if (act == NR_ACT_SILU) {
    if (fabsf(z) > 80.0f) return z > 0.0f ? 1.0f : 0.0f;
    const float s = 1.0f / (1.0f + __expf(-z));
    return fmaf(s * z, 1.0f - s, s);
  }
  return 1.0f;
}

// ------------------------------------------------------------ 8-bit form
// The scale byte e + 133 of a group whose largest |v| has these fp32 bits:
// the exponent field, one more where the mantissa is at least that of 127.5
// (bits + 0x10000 carries exactly there); 255 for infinities and NaN.
__device__ __forceinline__ uint32_t held8_scale(uint32_t top) {
  if (top >= 0x7f800000u) return 255u;
  const uint32_t e = (top + 0x10000u) >> 23;
  return e < 7u ? 7u : e > 254u ? 254u : e;
}
// 2^-e and 2^e of a scale byte, normal numbers both; a scale of 255 reads as NaN
__device__ __forceinline__ float held8_up(uint32_t s) {
  return s == 255u ? 0.0f : __uint_as_float((260u - s) << 23);
}
__device__ __forceinline__ float held8_down(uint32_t s) {
  return s == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float((s - 6u) << 23);
}
__device__ __forceinline__ int held8_code(float v, float up) {
  const int q = __float2int_rn(v * up);  // NaN converts to 0
  return max(-127, min(127, q));
}

// ------------------------------------------------------------ host
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }
inline bool is_16bit(int64_t t) { return t == NR_F16 || t == NR_BF16; }
inline size_t type_bytes(int64_t t) { return t == NR_F32 ? 4 : 2; }
inline bool act_ok(int64_t a) { return a >= NR_ACT_NONE && a <= NR_ACT_SILU; }
constexpr int64_t kOpsMaxRows = ((int64_t)1 << 31) - 1, kOpsMaxCols = ((int64_t)1 << 24) - 1;

// the SM count of a device, looked up once
int nr_ops_sms(int device);
// the device's flag that expired waits set (the address, looked up once)
cudaError_t nr_ops_flag(int device, int **flag);
