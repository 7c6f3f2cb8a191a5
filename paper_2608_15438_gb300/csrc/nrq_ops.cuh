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

// ------------------------------------------------------------ launches that follow one another
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;\n" ::: "memory"); }
__device__ __forceinline__ void grid_launch() { asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory"); }

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

template <typename T>
struct TypeCode;
template <>
struct TypeCode<float> { static constexpr int code = NR_F32; };
template <>
struct TypeCode<__half> { static constexpr int code = NR_F16; };
template <>
struct TypeCode<__nv_bfloat16> { static constexpr int code = NR_BF16; };

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

// ------------------------------------------------------------ eight elements
__device__ __forceinline__ uint32_t pack2(float a, float b, int dtype) {
  if (dtype == NR_F16) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 unpack2(uint32_t v, int dtype) {
  if (dtype == NR_F16) return __half22float2(*reinterpret_cast<const __half2 *>(&v));
  return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&v));
}

// eight consecutive elements from (row pointer index) e on, `count` of them there
__device__ __forceinline__ void load8(const void *p, int64_t e, int dtype, int vec, int count, float (&v)[8]) {
  if (vec && count >= 8) {
    if (dtype == NR_F32) {
      const float4 a = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + e);
      const float4 b = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + e + 4);
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
      const uint4 a = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + e);
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float2 f = unpack2(w[q], dtype);
        v[2 * q] = f.x;
        v[2 * q + 1] = f.y;
      }
    }
    return;
  }
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = q < count ? load_any(p, e + q, dtype) : 0.0f;
}
__device__ __forceinline__ void store8(void *p, int64_t e, int dtype, int vec, int count, const float (&v)[8]) {
  if (vec && count >= 8) {
    if (dtype == NR_F32) {
      float4 *d = reinterpret_cast<float4 *>(static_cast<float *>(p) + e);
      d[0] = make_float4(v[0], v[1], v[2], v[3]);
      d[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + e) =
          make_uint4(pack2(v[0], v[1], dtype), pack2(v[2], v[3], dtype), pack2(v[4], v[5], dtype), pack2(v[6], v[7], dtype));
    }
    return;
  }
#pragma unroll
  for (int q = 0; q < 8; ++q)
    if (q < count) store_any(p, e + q, dtype, v[q]);
}

// ------------------------------------------------------------ rows at any 2-byte address
// Sixteen halves in eight words, from half `by` (0 to 8) on: eight of them.
__device__ __forceinline__ void shift_halves(uint32_t (&w)[8], int by, uint32_t (&o)[4]) {
  if (by & 8) {
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = w[k + 4];
  }
#pragma unroll
  for (int k = 0; k < 6; ++k) w[k] = by & 4 ? w[k + 2] : w[k];
#pragma unroll
  for (int k = 0; k < 5; ++k) w[k] = by & 2 ? w[k + 1] : w[k];
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = __funnelshift_r(w[k], w[k + 1], by & 1 ? 16 : 0);
}
// Eight 16-bit values from p on, of which `count` are there: the two aligned
// 16-byte blocks they lie in (fetch), later shifted into place with zeros after the
// last (settle), so that many fetches are under way at once. A block that
// reaches out of the matrix [lo, hi) is not read; the few values at the matrix's
// first and last bytes that need it are read one by one.
__device__ __forceinline__ uint4 load_if128(const void *p, bool in) {
  uint4 v;
  asm("{\n .reg .pred p;\n setp.ne.b32 p, %5, 0;\n mov.b32 %0, 0;\n mov.b32 %1, 0;\n mov.b32 %2, 0;\n mov.b32 %3, 0;\n"
      " @p ld.global.nc.v4.b32 {%0, %1, %2, %3}, [%4];\n}\n"
      : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
      : "l"(p), "r"((int)in));
  return v;
}
__device__ __forceinline__ void fetch16x8(const void *p, int count, const void *lo, const void *hi, uint32_t (&w)[8]) {
  const char *a = reinterpret_cast<const char *>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15);
  const uint4 x = load_if128(a, count > 0 && a >= lo && a + 16 <= hi), y = load_if128(a + 16, count > 0 && a + 32 <= hi);
  w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w, w[4] = y.x, w[5] = y.y, w[6] = y.z, w[7] = y.w;
}
__device__ __forceinline__ void settle16x8(const void *p, int count, const void *lo, const void *hi, uint32_t (&w)[8]) {
  const char *a = reinterpret_cast<const char *>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15);
  const int s = (int)(reinterpret_cast<uintptr_t>(p) & 15) >> 1;
  uint32_t o[4];
  if (count > 0 && (a < lo || a + 16 + (s + count > 8 ? 16 : 0) > hi)) {
    o[0] = o[1] = o[2] = o[3] = 0u;
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q < count) o[q >> 1] |= (uint32_t)__ldg(static_cast<const uint16_t *>(p) + q) << (16 * (q & 1));
  } else {
    shift_halves(w, s, o);
    if (count < 8) {
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = count >= 2 * k + 2 ? o[k] : count == 2 * k + 1 ? o[k] & 0xffffu : 0u;
    }
  }
  w[0] = o[0], w[1] = o[1], w[2] = o[2], w[3] = o[3];
}
// What a lane of a row stores of its eight 16-bit values: the aligned 16-byte block
// of its predecessor's last s values and its own first 8 - s, and its values
// [from, to) one by one. s: its first value's place in an aligned block; left: the
// row's values from that one on (past the row's end: 0 or less); prev, next: the
// neighbouring lane belongs to the row.
struct Span16x8 {
  bool block;
  int from, to;
};
__host__ __device__ inline Span16x8 span16x8(int s, int left, bool prev, bool next) {
  const int count = left < 0 ? 0 : left < 8 ? left : 8, head = 8 - s;
  Span16x8 w;
  w.block = (prev || s == 0) && count >= head;
  w.from = w.block ? head : 0;
  w.to = s != 0 && next && left - 8 >= head ? head : 8;  // the successor's block holds the lane's last values
  if (w.to > count) w.to = count;
  return w;
}
// Stores the row's values from p on, at most eight, of which `left` are in the row.
// The lanes of `lanes` call it together, each eight values after its predecessor's,
// so that all but the lanes' ends are whole blocks.
__device__ __forceinline__ void store16x8(void *p, int left, const uint32_t (&v)[4], bool prev, bool next, unsigned lanes) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  const int s = (int)(at & 15) >> 1;
  uint32_t w[8], o[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    w[k] = __shfl_up_sync(lanes, v[k], 1);
    w[k + 4] = v[k];
  }
  shift_halves(w, 8 - s, o);
  const Span16x8 h = span16x8(s, left, prev, next);
  if (h.block) *reinterpret_cast<uint4 *>(at - 2 * (uintptr_t)s) = make_uint4(o[0], o[1], o[2], o[3]);
  if (h.from < h.to) {
    uint16_t *d = static_cast<uint16_t *>(p);
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q >= h.from && q < h.to) d[q] = (uint16_t)(v[q >> 1] >> (16 * (q & 1)));
  }
}

// Eight consecutive values of a row as they lie in memory: fetched, then settled
// (vec: by aligned 16-byte accesses, which leaves nothing to settle).
template <typename T>
struct Eight {
  uint32_t r[8];
};
template <typename T>
__device__ __forceinline__ Eight<T> fetch_eight(const T *p, bool vec, int count, const void *lo, const void *hi) {
  Eight<T> o = {};
  if (vec && count == 8) {
    const uint4 a = __ldg(reinterpret_cast<const uint4 *>(p));
    o.r[0] = a.x, o.r[1] = a.y, o.r[2] = a.z, o.r[3] = a.w;
    if (sizeof(T) == 4) {
      const uint4 b = __ldg(reinterpret_cast<const uint4 *>(p) + 1);
      o.r[4] = b.x, o.r[5] = b.y, o.r[6] = b.z, o.r[7] = b.w;
    }
  } else if (sizeof(T) == 4) {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q < count) o.r[q] = __ldg(reinterpret_cast<const uint32_t *>(p) + q);
  } else {
    fetch16x8(p, count, lo, hi, o.r);
  }
  return o;
}
template <typename T>
__device__ __forceinline__ void settle_eight(Eight<T> &o, const T *p, bool vec, int count, const void *lo, const void *hi) {
  if (sizeof(T) == 2 && !(vec && count == 8)) settle16x8(p, count, lo, hi, o.r);
}
template <typename T>
__device__ __forceinline__ float2 pair_of(const Eight<T> &o, int p) {
  if (sizeof(T) == 4)
    return make_float2(__uint_as_float(o.r[2 * p]), __uint_as_float(o.r[2 * p + 1]));
  return unpack2(o.r[p], TypeCode<T>::code);
}

// ------------------------------------------------------------ pairs of fp32
// one instruction for two values
__device__ __forceinline__ unsigned long long bits2(float2 v) { return *reinterpret_cast<unsigned long long *>(&v); }
__device__ __forceinline__ float2 from_bits2(unsigned long long v) { return *reinterpret_cast<float2 *>(&v); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(bits2(a)), "l"(bits2(b)), "l"(bits2(c)));
  return from_bits2(d);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits2(a)), "l"(bits2(b)));
  return from_bits2(d);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  unsigned long long d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits2(a)), "l"(bits2(b)));
  return from_bits2(d);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

__device__ __forceinline__ uint4 pack8(const float2 (&v)[4], int dtype) {
  return make_uint4(pack2(v[0].x, v[0].y, dtype), pack2(v[1].x, v[1].y, dtype), pack2(v[2].x, v[2].y, dtype),
                    pack2(v[3].x, v[3].y, dtype));
}

// ------------------------------------------------------------ activations
__device__ __forceinline__ float exp2_approx(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float rcp_approx(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// The normal distribution's tail Q = Phi(-|z|) and e = exp(-z^2 / 2), by formula
// 7.1.26 of Abramowitz and Stegun, Handbook of Mathematical Functions: with
// x = |z| / sqrt 2 and t = 1 / (1 + 0.3275911 x), erfc(x) = (a1 t + ... + a5
// t^5) exp(-x^2) to 1.5e-7 (Q to half of that). One exponential serves Q and
// the density; CUDA's erfcf and expf took 160 instructions an element, which
// bound the epilogue (290 us for 10000 x 1536 -> 6144, 147 without GELU).
__device__ __forceinline__ void normal_tail(float2 z, float2 &Q, float2 &e) {
  const float2 u = fma2(make_float2(fabsf(z.x), fabsf(z.y)), both(0.23164189f), both(1.0f));  // 0.3275911 / sqrt 2
  const float2 t = make_float2(rcp_approx(u.x), rcp_approx(u.y));
  const float2 h = mul2(mul2(z, z), both(-0.72134752f));  // log2(e) / 2
  e = make_float2(exp2_approx(h.x), exp2_approx(h.y));
  float2 p = fma2(t, both(0.5f * 1.061405429f), both(0.5f * -1.453152027f));
  p = fma2(p, t, both(0.5f * 1.421413741f));
  p = fma2(p, t, both(0.5f * -0.284496736f));
  p = fma2(p, t, both(0.5f * 0.254829592f));
  Q = mul2(mul2(p, t), e);
}
// Infinities go to the limits, NaN stays: factors that multiply a vanishing
// term are bounded first.
__device__ __forceinline__ float2 act_value2(float2 z, int act) {
  const float2 pos = make_float2(z.x < 0.0f ? 0.0f : z.x, z.y < 0.0f ? 0.0f : z.y);
  if (act == NR_ACT_RELU) return pos;
  if (act == NR_ACT_GELU) {  // z Phi(z) = max(z, 0) - |z| Q
    float2 Q, e;
    normal_tail(z, Q, e);
    return fma2(make_float2(-fminf(fabsf(z.x), 20.0f), -fminf(fabsf(z.y), 20.0f)), Q, pos);
  }
  if (act == NR_ACT_SILU) {
    const float2 h = mul2(z, both(-1.44269504f));
    const float2 s = make_float2(rcp_approx(1.0f + exp2_approx(h.x)), rcp_approx(1.0f + exp2_approx(h.y)));
    return mul2(make_float2(fmaxf(z.x, -100.0f), fmaxf(z.y, -100.0f)), s);
  }
  return z;
}
// the derivatives
__device__ __forceinline__ float2 act_slope2(float2 z, int act) {
  if (act == NR_ACT_RELU) return make_float2(z.x > 0.0f ? 1.0f : 0.0f, z.y > 0.0f ? 1.0f : 0.0f);
  if (act == NR_ACT_GELU) {  // Phi(z) + z phi(z)
    float2 Q, e;
    normal_tail(z, Q, e);
    const float2 phi = mul2(e, both(0.39894228f));
    const float2 c = make_float2(z.x < 0.0f ? Q.x : 1.0f - Q.x, z.y < 0.0f ? Q.y : 1.0f - Q.y);
    return fma2(make_float2(fmaxf(fminf(z.x, 20.0f), -20.0f), fmaxf(fminf(z.y, 20.0f), -20.0f)), phi, c);
  }
  if (act == NR_ACT_SILU) {  // s + z s (1 - s)
    const float2 h = mul2(z, both(-1.44269504f));
    const float2 s = make_float2(rcp_approx(1.0f + exp2_approx(h.x)), rcp_approx(1.0f + exp2_approx(h.y)));
    const float2 r = fma2(s, both(-1.0f), both(1.0f));
    const float2 zc = make_float2(fmaxf(fminf(z.x, 100.0f), -100.0f), fmaxf(fminf(z.y, 100.0f), -100.0f));
    return fma2(mul2(zc, s), r, s);
  }
  return both(1.0f);
}
__device__ __forceinline__ float act_value(float z, int act) { return act_value2(make_float2(z, z), act).x; }

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
// What a held number stands for in fp16, where 64 x 2^10 is past the type's end:
// at most the largest finite value. From scale kHeld8F16 (2^10) on; NaN stays.
constexpr uint32_t kHeld8F16 = 143u;
__device__ __forceinline__ float2 held8_in_f16(float2 v) {
  return make_float2(v.x > 65504.0f ? 65504.0f : v.x < -65504.0f ? -65504.0f : v.x,
                     v.y > 65504.0f ? 65504.0f : v.y < -65504.0f ? -65504.0f : v.y);
}
// The codes of four values in a word. Adding 1.5 2^23 rounds to a whole number,
// ties to even, and leaves its two's complement in the low byte (a conversion
// instruction runs at half the rate or less). Only the topmost scale (and 255)
// can pass +-127.
__device__ __forceinline__ uint32_t held8_codes(float2 a, float2 b, float up, uint32_t scale) {
  if (scale >= 254u) {
    a.x = fminf(fmaxf(a.x * up, -127.0f), 127.0f), a.y = fminf(fmaxf(a.y * up, -127.0f), 127.0f);
    b.x = fminf(fmaxf(b.x * up, -127.0f), 127.0f), b.y = fminf(fmaxf(b.y * up, -127.0f), 127.0f);
    up = 1.0f;
  }
  a = fma2(a, both(up), both(12582912.0f));
  b = fma2(b, both(up), both(12582912.0f));
  const uint32_t lo = __byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040);
  const uint32_t hi = __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040);
  return __byte_perm(lo, hi, 0x5410);
}
// the four codes of a word as numbers: the byte + 128 under the exponent of 2^23
__device__ __forceinline__ void held8_numbers(uint32_t codes, float2 &a, float2 &b) {
  const uint32_t u = codes ^ 0x80808080u;
  a.x = __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440)), a.y = __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7441));
  b.x = __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7442)), b.y = __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7443));
  a = add2(a, both(-8388736.0f));
  b = add2(b, both(-8388736.0f));
}

// ------------------------------------------------------------ host
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }
inline bool is_16bit(int64_t t) { return t == NR_F16 || t == NR_BF16; }
inline size_t type_bytes(int64_t t) { return t == NR_F32 ? 4 : 2; }
// whether eight columns of every row are a 16-byte access (two in fp32)
inline bool vec_ok(const void *p, int64_t ld, int64_t dtype) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * (int64_t)type_bytes(dtype) % 16 == 0;
}
// whether a matrix (values of a type, or a checkpoint's codes) lies where the kernels' accesses can reach it
inline bool placed(const void *p, int64_t dtype, bool codes = false) {
  return (reinterpret_cast<uintptr_t>(p) & (codes ? 15 : type_bytes(dtype) - 1)) == 0;
}
inline bool act_ok(int64_t a) { return a >= NR_ACT_NONE && a <= NR_ACT_SILU; }
constexpr int64_t kOpsMaxRows = ((int64_t)1 << 31) - 1, kOpsMaxCols = ((int64_t)1 << 24) - 1;

// the SM count of a device, looked up once; 0: there is no such device
int nr_ops_sms(int device);
// the device's flag that expired waits set (the address, looked up once)
cudaError_t nr_ops_flag(int device, int **flag);

// a launch that may begin before the previous one of the call has ended: its
// kernel waits (grid_wait) before it touches memory
template <typename... K, typename... A>
cudaError_t launch(void (*kernel)(K...), unsigned grid, dim3 block, uint32_t smem, cudaStream_t s, bool follows, A &&...a) {
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3(grid);
  c.blockDim = block;
  c.dynamicSmemBytes = smem;
  c.stream = s;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  c.attrs = &at;
  c.numAttrs = follows ? 1 : 0;
  return cudaLaunchKernelEx(&c, kernel, static_cast<K>(a)...);
}
