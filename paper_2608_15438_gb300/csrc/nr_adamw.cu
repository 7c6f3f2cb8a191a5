// AdamW over many tensors at once (neuroute_ops.h), its averages in 32 or in 8 bits,
// and the norm of all gradients. Bound by memory: 28 bytes a value in fp32 (p, m and v
// read and written, g read), 16.1 with averages in 8 bits. 153e6 values take 658 us in fp32 (6.5 TB/s), 49 and 676 us
// with bf16 gradients, fp32 masters and the norm, and 462 us with averages in 8 bits (5.3 TB/s): there some 70
// instructions a value bind as well, one issued in 61% of cycles. Tensors that do not begin at multiples of 32 bytes are
// read by aligned blocks shifted into place: 65e6 values in fp32 292 us (6.3 TB/s).
//
// Without a norm one launch makes the step: a persistent grid walks chunks of kChunk
// values of all tensors, found by bisection in a table among the kernel's parameters.
// The norm takes a launch before it, whose blocks leave their sums of squares; every block
// of the step adds them up again, in order. The last block to end the step counts it.
#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "nrq_ops.cuh"

namespace {

constexpr int kThreads = 256, kChunk = kThreads * 8, kNormBlocks = 8;  // values a chunk, blocks an SM

struct Entry {
  void *p;
  const void *g;
  int64_t n, at;
  uint32_t first;  // chunk
  float decay;  // without a rate on the device: 1 - lr decay, as the few fp64 units would bind
  int p_dtype, g_dtype;
};
// as many tensors as a launch takes: few, whose table fits 4 KB of parameters, or many
template <int CAP>
struct Table {
  int count;
  uint32_t chunks;
  int aligned;  // everything begins at a multiple of 32 bytes
  Entry e[CAP];
};
constexpr int kFew = 64, kMany = 512;

struct Step {
  float *master;
  void *m, *v;
  uint8_t *m_scale, *v_scale;
  int64_t *step;
  int32_t *ticket;
  const float *lr_at;
  double lr, log_b1, log_b2, max_norm;
  float b1, c1, b2, c2, eps, one;  // c = 1 - b
  float *norm;
  const double *parts;  // sums of squares
  int part_count;
  int counts;  // the launch that ends the step
  int tiny;
  uint32_t key0, key1;
};

__device__ __forceinline__ int64_t round_up32(int64_t n) { return (n + 31) & ~(int64_t)31; }

template <int CAP>
__device__ __forceinline__ int find(const Table<CAP> &T, uint32_t chunk, int hi) {
  int lo = 0;  // the last tensor up to hi that begins at or before the chunk
  if (T.e[hi].first <= chunk) return hi;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (T.e[mid].first <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// ------------------------------------------------------------ averages in 8 bits
__device__ __forceinline__ float2 mul2_cut(float2 a, float2 b) {  // towards zero
  unsigned long long d;
  asm("mul.rz.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits2(a)), "l"(bits2(b)));
  return from_bits2(d);
}
__device__ __forceinline__ float largest(float a, float b, float c) {  // NaN if one is
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float power2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
// The scale byte of a group whose largest magnitude has these fp32 bits: the
// exponent field, one more where the mantissa is at least that of 31/16.
__device__ __forceinline__ uint32_t moment_scale(uint32_t top) {
  if (top >= 0x7f800000u) return 255u;
  const uint32_t e = (top + 0x80000u) >> 23;
  return (e < 19u ? 19u : e > 254u ? 254u : e) - 7u;
}
// Magnitudes brought to the fp32 exponents just above the type's least, so that their
// codes are their upper bits and the steps end where fp32's own do: v by
// 2^-(e + 112), m by 2^-(e + 120), each in two factors, as one may be past fp32's
// range. Products are cut, not rounded, which leaves floor(x / step + d) exact.
template <bool V>
struct Moment {
  float2 up, down;  // the factors, towards codes and back
  __device__ __forceinline__ explicit Moment(uint32_t scale) {
    const int e = (int)scale - 120, half = e >> 1, k = V ? 56 : 60;
    up = make_float2(power2(-half - k), power2(half - e - k));
    down = make_float2(power2(half + k), scale == 255u ? __uint_as_float(0x7fffffffu) : power2(e - half + k));
  }
  __device__ __forceinline__ static uint32_t code(float x, float y, uint32_t d) {  // y: |x| times the factors
    uint32_t c = (__float_as_uint(y) + (d << 3)) >> 19;
    if (V) {
      c = c > 255u ? 255u : c;
      return c == 0u && x > 0.0f ? 1u : c;
    }
    c = c > 127u ? 127u : c;
    return c | (__float_as_uint(x) >> 31 << 7);
  }
  // two codes; d: the values' dithers
  __device__ __forceinline__ uint2 codes(float2 x, uint32_t d0, uint32_t d1) const {
    const float2 y = mul2_cut(mul2_cut(make_float2(fabsf(x.x), fabsf(x.y)), both(up.x)), both(up.y));
    return make_uint2(code(x.x, y.x, d0), code(x.y, y.y, d1));
  }
  __device__ __forceinline__ float2 values(uint32_t c0, uint32_t c1) const {
    float2 y = make_float2(__uint_as_float((V ? c0 : c0 & 127u) << 19), __uint_as_float((V ? c1 : c1 & 127u) << 19));
    y = mul2(mul2(y, both(down.x)), both(down.y));
    if (!V) {
      y.x = __uint_as_float(__float_as_uint(y.x) | (c0 & 128u) << 24);
      y.y = __uint_as_float(__float_as_uint(y.y) | (c1 & 128u) << 24);
    }
    return y;
  }
};
// Philox4x32 with 7 rounds (Salmon, Moraes, Dror, Shaw, SC'11)
__device__ __forceinline__ uint4 philox7(uint64_t i, uint64_t t, uint32_t k0, uint32_t k1) {
  uint4 c = make_uint4((uint32_t)i, (uint32_t)(i >> 32), (uint32_t)t, (uint32_t)(t >> 32));
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c.x, b = (uint64_t)0xCD9E8D57u * c.z;
    c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

// ------------------------------------------------------------ a tensor's values, eight a thread
// as they lie in memory: fetched, then settled (see nrq_ops.cuh). ALIGNED: the tensor begins at a multiple of 32
// bytes, and so does every thread's part of fp32 values.
template <bool ALIGNED>
struct Raw {
  uint32_t w[ALIGNED ? 8 : 12];
};
template <bool ALIGNED, bool WHOLE = false>
__device__ __forceinline__ Raw<ALIGNED> fetch(const void *base, int64_t j, int64_t n, int dtype) {
  Raw<ALIGNED> o;
  const int count = WHOLE || n - j >= 8 ? 8 : (int)(n - j);
  const char *p = static_cast<const char *>(base) + j * (dtype == NR_F32 ? 4 : 2);
  if (ALIGNED && count < 8) {
#pragma unroll
    for (int q = 0; q < 8; ++q) o.w[q] = 0u;
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q < count) {
        if (dtype == NR_F32) o.w[q] = reinterpret_cast<const uint32_t *>(p)[q];
        else o.w[q >> 1] |= (uint32_t) reinterpret_cast<const uint16_t *>(p)[q] << (16 * (q & 1));
      }
  } else if constexpr (ALIGNED) {
    if (dtype == NR_F32) {
      load256(p, o.w);
    } else {
      const uint4 a = *reinterpret_cast<const uint4 *>(p);
      o.w[0] = a.x, o.w[1] = a.y, o.w[2] = a.z, o.w[3] = a.w;
    }
  } else if constexpr (!ALIGNED) {
    if (dtype == NR_F32) {
      fetch32x8(p, count, base, static_cast<const char *>(base) + 4 * n, o.w);
    } else {
      uint32_t h[8];
      fetch16x8(p, count, base, static_cast<const char *>(base) + 2 * n, h);
#pragma unroll
      for (int k = 0; k < 8; ++k) o.w[k] = h[k];
    }
  }
  return o;
}
template <bool ALIGNED, bool WHOLE = false>
__device__ __forceinline__ void settle(Raw<ALIGNED> &o, const void *base, int64_t j, int64_t n, int dtype, float2 (&v)[4]) {
  const int count = WHOLE || n - j >= 8 ? 8 : (int)(n - j);
  const char *p = static_cast<const char *>(base) + j * (dtype == NR_F32 ? 4 : 2);
  if (dtype == NR_F32) {
    if constexpr (!ALIGNED) settle32x8(p, count, base, static_cast<const char *>(base) + 4 * n, o.w);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = make_float2(__uint_as_float(o.w[2 * q]), __uint_as_float(o.w[2 * q + 1]));
    return;
  }
  uint32_t h[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) h[k] = o.w[k];
  if constexpr (!ALIGNED) settle16x8(p, count, base, static_cast<const char *>(base) + 2 * n, h);
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = unpack2(h[q], dtype);
}
// eight values of the fp32 arrays
template <bool ALIGNED>
__device__ __forceinline__ void load_array(const float *p, uint32_t (&w)[8]) {
  if (ALIGNED) {
    load256(p, w);
  } else {
    const uint4 a = reinterpret_cast<const uint4 *>(p)[0], b = reinterpret_cast<const uint4 *>(p)[1];
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
  }
}
template <bool ALIGNED>
__device__ __forceinline__ void store_array(float *p, const float2 (&v)[4]) {
  uint32_t w[8];
  words8(v, w);
  if (ALIGNED) {
    store256(p, w);
  } else {
    reinterpret_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    reinterpret_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}
// all lanes of a warp together
template <bool ALIGNED, bool WHOLE>
__device__ __forceinline__ void put(void *base, int64_t j, int64_t n, int dtype, const float2 (&v)[4]) {
  const int lane = threadIdx.x & 31;
  char *p = static_cast<char *>(base) + j * (dtype == NR_F32 ? 4 : 2);
  const int left = WHOLE || n - j >= 512 ? 512 : (int)(n - j);  // past the end: 0 or less
  if (dtype == NR_F32) {
    uint32_t w[8];
    words8(v, w);
    if (ALIGNED && left >= 8) {
      store256(p, w);
    } else if (ALIGNED) {
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (q < left) reinterpret_cast<uint32_t *>(p)[q] = w[q];
    } else {
      store32x8(p, left, w, lane > 0, lane < 31, 0xffffffffu);
    }
    return;
  }
  const uint4 h = pack8(v, dtype);
  const uint32_t w[4] = {h.x, h.y, h.z, h.w};
  if (ALIGNED && left >= 8) *reinterpret_cast<uint4 *>(p) = h;
  else if (!ALIGNED) store16x8(p, left, w, lane > 0, lane < 31, 0xffffffffu);
  else
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q < left) reinterpret_cast<uint16_t *>(p)[q] = (uint16_t)(w[q >> 1] >> (16 * (q & 1)));
}

// ------------------------------------------------------------ the norm
__device__ __forceinline__ double block_sum(double v, double *shared) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < kThreads / 32; ++w) v += shared[w];
  return v;
}

// Loads of kAtOnce chunks are under way together (one at a time: 2.2 TB/s). Sixteen squares a thread are
// added in fp32, their sums in two fp32 numbers, the second what the first's roundings lose (Knuth's exact sum of
// two): the few fp64 units would bind. Sums that near fp32's end go on in fp64, so that however many gradients
// below 2^60 there are, whose sixteen squares are below 2^124, none is infinite.
template <int CAP, bool ALIGNED>
__global__ void __launch_bounds__(kThreads) square_kernel(const __grid_constant__ Table<CAP> T, double *parts) {
  constexpr int kAtOnce = 4;
  __shared__ double shared[kThreads / 32], past[kThreads];  // a thread's own
  float high = 0.0f, low = 0.0f;
  past[threadIdx.x] = 0.0;
  // an infinity stays one (its second number is NaN)
  const auto sum = [&] { return past[threadIdx.x] + (high < INFINITY ? (double)high + (double)low : (double)high); };
  const auto add = [&](float2 s) {
    const float v = s.x + s.y, next = high + v, of = next - high;
    low += (high - (next - of)) + (v - of);
    high = next;
  };
  for (uint32_t c0 = blockIdx.x * kAtOnce; c0 < T.chunks; c0 += gridDim.x * kAtOnce) {
    if (__builtin_expect(high >= 0x1p126f, 0)) {
      past[threadIdx.x] = sum();
      high = low = 0.0f;
    }
    int k = find(T, c0, T.count - 1);
    const Entry &e = T.e[k];
    const int64_t j = (int64_t)(c0 - e.first) * kChunk;
    if (ALIGNED && j + kAtOnce * kChunk <= e.n) {  // all of one tensor
      uint32_t w[kAtOnce][8];
      float2 s[2] = {both(0.0f), both(0.0f)};
      if (e.g_dtype == NR_F32) {
        const float *g = static_cast<const float *>(e.g) + j + threadIdx.x * 8;
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) load256(g + u * kChunk, w[u]);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          float2 v[4];
          floats8(w[u], v);
#pragma unroll
          for (int q = 0; q < 4; ++q) s[u & 1] = fma2(v[q], v[q], s[u & 1]);
        }
      } else {
        const uint16_t *g = static_cast<const uint16_t *>(e.g) + j + threadIdx.x * 8;
        uint4 a[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) a[u] = *reinterpret_cast<const uint4 *>(g + u * kChunk);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const uint32_t h[4] = {a[u].x, a[u].y, a[u].z, a[u].w};
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float2 v = unpack2(h[q], e.g_dtype);
            s[u & 1] = fma2(v, v, s[u & 1]);
          }
        }
      }
      add(s[0]);
      add(s[1]);
      continue;
    }
    for (uint32_t c = c0; c < c0 + kAtOnce && c < T.chunks; ++c) {
      while (k + 1 < T.count && T.e[k + 1].first <= c) ++k;
      const Entry &f = T.e[k];
      const int64_t i = (int64_t)(c - f.first) * kChunk + threadIdx.x * 8;
      if (i >= f.n) continue;
      Raw<ALIGNED> raw = fetch<ALIGNED>(f.g, i, f.n, f.g_dtype);
      float2 g[4], s = both(0.0f);
      settle<ALIGNED>(raw, f.g, i, f.n, f.g_dtype, g);
#pragma unroll
      for (int q = 0; q < 4; ++q) s = fma2(g[q], g[q], s);
      add(s);
    }
  }
  const double all = block_sum(sum(), shared);
  if (threadIdx.x == 0) parts[blockIdx.x] = all;
}

__global__ void __launch_bounds__(kThreads) norm_kernel(const double *parts, int count, float *norm) {
  __shared__ double shared[kThreads / 32];
  double sum = 0.0;
  grid_wait();
  for (int i = threadIdx.x; i < count; i += kThreads) sum += parts[i];
  sum = block_sum(sum, shared);
  if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

// ------------------------------------------------------------ the step
// rate m / (v^1/2 root + eps) by the hardware's approximations, 2^-22 of it. TINY (tiny_matters): for an eps that a
// root of a v below fp32's normal numbers could matter beside; those that flush them cost eight instructions less.
template <bool TINY>
__device__ __forceinline__ float2 quotient(float2 m, float2 v, float rate, float root, float eps) {
  float2 r;
  if (TINY) asm("sqrt.approx.f32 %0, %2;\n sqrt.approx.f32 %1, %3;\n" : "=f"(r.x), "=f"(r.y) : "f"(v.x), "f"(v.y));
  else asm("sqrt.approx.ftz.f32 %0, %2;\n sqrt.approx.ftz.f32 %1, %3;\n" : "=f"(r.x), "=f"(r.y) : "f"(v.x), "f"(v.y));
  const float2 d = fma2(r, both(root), both(eps));
  if (TINY) asm("rcp.approx.f32 %0, %2;\n rcp.approx.f32 %1, %3;\n" : "=f"(r.x), "=f"(r.y) : "f"(d.x), "f"(d.y));
  else asm("rcp.approx.ftz.f32 %0, %2;\n rcp.approx.ftz.f32 %1, %3;\n" : "=f"(r.x), "=f"(r.y) : "f"(d.x), "f"(d.y));
  return mul2(mul2(m, both(rate)), r);
}

// A thread takes eight consecutive values at a time; four lanes share a group of the 8-bit form. Blocks an SM by the
// registers: 64 a thread and four in fp32; 8 bits want 80 (four blocks spill: 735 us for 655; two with the next
// chunk's loads ahead: 690 for 662; four values a thread and five blocks: 750).
template <int CAP, int BITS, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, ALIGNED && BITS == 32 ? 4 : 3)
    step_kernel(const __grid_constant__ Table<CAP> T, const __grid_constant__ Step S) {
  __shared__ double shared;
  grid_wait();
  float coef = 1.0f;
  if (S.norm) {
    if (threadIdx.x < 32) {  // fp64 units are few
      double sum = 0.0;
#pragma unroll 4
      for (int i = threadIdx.x; i < S.part_count; i += 32) sum += S.parts[i];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (threadIdx.x == 0) {
        shared = sqrt(sum);
        if (blockIdx.x == 0) *S.norm = (float)shared;
      }
    }
    __syncthreads();
    const double norm = shared;
    if (!(norm < (double)INFINITY)) return;
    // at most 1: max_norm / (norm + 1e-6) rounded once
    coef = norm + 1e-6 > S.max_norm ? (float)(S.max_norm / (norm + 1e-6)) : 1.0f;
  }
  const int64_t t = *S.step + 1;
  const float lr = S.lr_at ? *S.lr_at : (float)S.lr;
  const float rate = lr / -expm1f((float)((double)t * S.log_b1));
  const float root = 1.0f / sqrtf(-expm1f((float)((double)t * S.log_b2)));
  const int lane = threadIdx.x & 31;
  // WHOLE: a chunk without the tensor's end in it
  const auto chunk = [&](const Entry &e, uint32_t c, auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
    const int64_t first = (int64_t)(c - e.first) * kChunk, j = first + threadIdx.x * 8, at = e.at + j;
    if (!WHOLE && j - lane * 8 >= e.n) return;  // a whole warp
    // the arrays reach to the next multiple of 32 behind the tensor
    const bool in = WHOLE || j < e.n, held = WHOLE || j < round_up32(e.n);
    const bool master = S.master && e.p_dtype != NR_F32;
    const void *pb = master ? S.master + e.at : e.p;
    const int pt = master ? NR_F32 : e.p_dtype;
    const int64_t pn = master ? round_up32(e.n) : e.n;
    Raw<ALIGNED> rg = {}, rp = {};
    uint32_t rm[8] = {}, rv[8] = {};
    uint32_t sm = 12u, sv = 12u;
    if (in) {
      rg = fetch<ALIGNED, WHOLE>(e.g, j, e.n, e.g_dtype);
      rp = fetch<ALIGNED, WHOLE>(pb, j, pn, pt);
    }
    if (BITS == 32) {
      if (held) {
        load_array<ALIGNED>(static_cast<float *>(S.m) + at, rm);
        load_array<ALIGNED>(static_cast<float *>(S.v) + at, rv);
      }
    } else if (held) {
      const uint2 a = *reinterpret_cast<const uint2 *>(static_cast<uint8_t *>(S.m) + at);
      const uint2 b = *reinterpret_cast<const uint2 *>(static_cast<uint8_t *>(S.v) + at);
      rm[0] = a.x, rm[1] = a.y, rv[0] = b.x, rv[1] = b.y;
      sm = S.m_scale[at >> 5];
      sv = S.v_scale[at >> 5];
    }
    float2 g[4], p[4], m[4], v[4];
    if (in) {
      settle<ALIGNED, WHOLE>(rg, e.g, j, e.n, e.g_dtype, g);
      settle<ALIGNED, WHOLE>(rp, pb, j, pn, pt, p);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) g[q] = p[q] = both(0.0f);
    }
    if (BITS == 32) {
      floats8(rm, m);
      floats8(rv, v);
    } else {
      const Moment<false> M(sm);
      const Moment<true> V(sv);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t a = rm[q >> 1] >> (16 * (q & 1)), b = rv[q >> 1] >> (16 * (q & 1));
        m[q] = M.values(a & 255u, a >> 8 & 255u);
        v[q] = V.values(b & 255u, b >> 8 & 255u);
      }
    }
    // one rounding an operation, as the averages are defined: the sums are multiplications by a one that the compiler
    // does not see, as it makes one instruction of a packed product and sum, which rounds once
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (S.norm) g[q] = mul2(g[q], both(coef));
      m[q] = fma2(mul2(m[q], both(S.b1)), both(S.one), mul2(g[q], both(S.c1)));
      v[q] = fma2(mul2(v[q], both(S.b2)), both(S.one), mul2(mul2(g[q], both(S.c2)), g[q]));
    }
    if (BITS == 8 && !WHOLE && j + 8 > e.n) {  // nothing lies behind the tensor
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (j + 2 * q >= e.n) m[q].x = v[q].x = 0.0f;
        if (j + 2 * q + 1 >= e.n) m[q].y = v[q].y = 0.0f;
      }
    }
    const float keep = S.lr_at ? 1.0f - lr * e.decay : e.decay;
    if (S.tiny) {
#pragma unroll
      for (int q = 0; q < 4; ++q) p[q] = fma2(p[q], both(keep), quotient<true>(m[q], v[q], -rate, root, S.eps));
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) p[q] = fma2(p[q], both(keep), quotient<false>(m[q], v[q], -rate, root, S.eps));
    }
    if (BITS == 32) {
      if (held) {
        store_array<ALIGNED>(static_cast<float *>(S.m) + at, m);
        store_array<ALIGNED>(static_cast<float *>(S.v) + at, v);
      }
    } else {
      float tm = 0.0f, tv = 0.0f;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        tm = largest(tm, fabsf(m[q].x), fabsf(m[q].y));
        tv = largest(tv, v[q].x, v[q].y);
      }
#pragma unroll
      for (int o = 1; o <= 2; o *= 2) {
        tm = largest(tm, __shfl_xor_sync(0xffffffffu, tm, o), 0.0f);
        tv = largest(tv, __shfl_xor_sync(0xffffffffu, tv, o), 0.0f);
      }
      sm = moment_scale(__float_as_uint(tm));
      sv = moment_scale(__float_as_uint(tv));
      const Moment<false> M(sm);
      const Moment<true> V(sv);
      uint32_t cm[2], cv[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 w = philox7(((uint64_t)at >> 2) + h, (uint64_t)t, S.key0, S.key1);
        const uint2 a = M.codes(m[2 * h], w.x & 0xffffu, w.y & 0xffffu), b = M.codes(m[2 * h + 1], w.z & 0xffffu, w.w & 0xffffu);
        const uint2 c2 = V.codes(v[2 * h], w.x >> 16, w.y >> 16), d = V.codes(v[2 * h + 1], w.z >> 16, w.w >> 16);
        cm[h] = a.x | a.y << 8 | b.x << 16 | b.y << 24;
        cv[h] = c2.x | c2.y << 8 | d.x << 16 | d.y << 24;
      }
      if (held) {
        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(S.m) + at) = make_uint2(cm[0], cm[1]);
        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(S.v) + at) = make_uint2(cv[0], cv[1]);
        if ((lane & 3) == 0) {
          S.m_scale[at >> 5] = (uint8_t)sm;
          S.v_scale[at >> 5] = (uint8_t)sv;
        }
      }
    }
    put<ALIGNED, WHOLE>(e.p, j, e.n, e.p_dtype, p);
    if (master && held) store_array<ALIGNED>(S.master + at, p);
  };
  // from the last chunk on: the gradients whose squares were added last are still in L2
  int k = T.count - 1;
  for (uint32_t left = T.chunks - blockIdx.x; left <= T.chunks && left > 0; left -= gridDim.x) {
    const uint32_t c = left - 1;
    k = find(T, c, k);
    const Entry &e = T.e[k];
    if ((int64_t)(c - e.first + 1) * kChunk <= e.n) chunk(e, c, std::true_type());
    else chunk(e, c, std::false_type());
  }
  if (!S.counts) return;
  __syncthreads();
  if (threadIdx.x == 0 && atomicAdd(S.ticket, 1) == (int)gridDim.x - 1) {
    *S.step = t;  // every block has read it
    *S.ticket = 0;
  }
}

// blockIdx.y: 0 m, 1 v
__global__ void __launch_bounds__(kThreads)
    read_kernel(const uint8_t *m, const uint8_t *m_scale, const uint8_t *v, const uint8_t *v_scale, int64_t n, uint4 *ym, uint4 *yv) {
  const int64_t stride = (int64_t)gridDim.x * kThreads * 8;
  const uint8_t *codes = blockIdx.y ? v : m, *scales = blockIdx.y ? v_scale : m_scale;
  uint4 *y = blockIdx.y ? yv : ym;
  for (int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 8; i < n; i += stride) {
    const uint2 c = *reinterpret_cast<const uint2 *>(codes + i);
    const uint32_t s = scales[i >> 5];
    float2 o[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t a = (q < 2 ? c.x : c.y) >> (16 * (q & 1));
      o[q] = blockIdx.y ? Moment<true>(s).values(a & 255u, a >> 8 & 255u) : Moment<false>(s).values(a & 255u, a >> 8 & 255u);
    }
    y[i >> 3] = pack8(o, NR_BF16);
  }
}

// ------------------------------------------------------------ host
constexpr int64_t kMostValues = (int64_t)1 << 40;

bool tensors_ok(const nr_adamw *a, bool norm_only) {
  if (!a || a->count < 0 || a->count > ((int64_t)1 << 20)) return false;
  if (a->count > 0 && (!a->tensors || !a->g || (!norm_only && !a->p))) return false;
  for (int64_t i = 0; i < a->count; ++i) {
    const nr_adamw_tensor &t = a->tensors[i];
    if (t.n < 0 || t.n >= kMostValues) return false;
    if (t.n == 0) continue;
    if (a->g[i] && (t.g_dtype < NR_F32 || t.g_dtype > NR_BF16 || !placed(a->g[i], t.g_dtype))) return false;
    if (norm_only) continue;
    if (!a->p[i] || t.p_dtype < NR_F32 || t.p_dtype > NR_BF16 || !placed(a->p[i], t.p_dtype)) return false;
    if (t.at < 0 || t.at % kOpsGroup != 0 || t.at >= 2 * kMostValues || !(t.decay >= 0.0) || !(t.decay <= FLT_MAX)) return false;
  }
  return true;
}
bool aligned(const void *p, int to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool valid(const nr_adamw *a) {
  if (!tensors_ok(a, false)) return false;
  if (a->bits != 32 && a->bits != 8) return false;
  if (!(a->beta1 >= 0.0 && a->beta1 < 1.0 && a->beta2 >= 0.0 && a->beta2 < 1.0)) return false;
  if (!(a->eps > 0.0) || !(a->max_norm >= 0.0) || !(a->max_norm < INFINITY) || !(fabs(a->lr) <= FLT_MAX)) return false;
  if (!a->step || !a->ticket || (reinterpret_cast<uintptr_t>(a->step) & 7) || !placed(a->ticket, NR_F32) ||
      !placed(a->lr_at, NR_F32) || !placed(a->norm, NR_F32) || (a->max_norm > 0.0 && !a->norm))
    return false;
  bool values = false;  // tensors without any have no averages
  for (int64_t i = 0; i < a->count && !values; ++i) values = a->tensors[i].n > 0;
  if (!values) return true;
  return a->m && a->v && aligned(a->m, 16) && aligned(a->v, 16) && aligned(a->master, 16) &&
         (a->bits == 32 || (a->m_scale && a->v_scale));
}

// the tensors from `from` on that a launch takes
template <int CAP>
int64_t fill(const nr_adamw *a, int64_t from, Table<CAP> &T) {
  T.count = 0;
  T.aligned = aligned(a->master, 32) && (a->bits == 8 || (aligned(a->m, 32) && aligned(a->v, 32)));
  uint64_t chunks = 0;
  int64_t i = from;
  for (; i < a->count && T.count < CAP; ++i) {
    const nr_adamw_tensor &t = a->tensors[i];
    const void *g = a->g[i], *p = a->p ? a->p[i] : nullptr;
    if (t.n == 0 || !g) continue;
    const uint64_t more = (uint64_t)ceil_div(t.n, kChunk);
    if (chunks + more > 0x7fffffffu) break;
    const double decay = a->lr_at ? t.decay : 1.0 - a->lr * t.decay;
    T.e[T.count++] = {const_cast<void *>(p), g, t.n, t.at, (uint32_t)chunks, (float)decay, (int)t.p_dtype, (int)t.g_dtype};
    chunks += more;
    if (!aligned(p, 32) || !aligned(g, 32)) T.aligned = 0;
  }
  T.chunks = (uint32_t)chunks;
  return i;
}
int grid_of(uint32_t chunks, int sms, int per_sm) {
  const int64_t most = (int64_t)sms * per_sm;
  return (int)(chunks < most ? chunks : most);
}

// Whether v below 2^-126, whose root is below 2^-63, can move a denominator by 2^-24 of it: root is (1 - beta2^t)^-1/2,
// largest at the first step.
bool tiny_matters(const nr_adamw *a) { return a->eps < ldexp(1.0, -39) / sqrt(1.0 - a->beta2); }

// blocks' sums of squares -> parts; how many
template <int CAP>
cudaError_t squares(const nr_adamw *a, int sms, double *parts, int &count, cudaStream_t s) {
  Table<CAP> T;
  count = 0;
  for (int64_t i = 0; i < a->count;) {
    i = fill(a, i, T);
    if (T.chunks == 0) continue;
    const int blocks = grid_of(T.chunks, sms, kNormBlocks);
    if (T.aligned) square_kernel<CAP, true><<<blocks, kThreads, 0, s>>>(T, parts + count);
    else square_kernel<CAP, false><<<blocks, kThreads, 0, s>>>(T, parts + count);
    count += blocks;
  }
  return cudaGetLastError();
}
template <int CAP>
cudaError_t steps(const nr_adamw *a, Step S, int sms, cudaStream_t s) {
  Table<CAP> T;
  int64_t i = 0;
  do {
    i = fill(a, i, T);
    // nothing but tensors without gradients behind it?
    bool last = true;
    for (int64_t k = i; k < a->count && last; ++k) last = a->tensors[k].n == 0 || !a->g[k];
    S.counts = last;
    const int blocks = T.chunks ? grid_of(T.chunks, sms, T.aligned && a->bits == 32 ? 4 : 3) : 1;
    const bool follows = S.part_count > 0;
    cudaError_t e;
    if (a->bits == 32)
      e = T.aligned ? launch(step_kernel<CAP, 32, true>, blocks, dim3(kThreads), 0, s, follows, T, S)
                    : launch(step_kernel<CAP, 32, false>, blocks, dim3(kThreads), 0, s, follows, T, S);
    else
      e = T.aligned ? launch(step_kernel<CAP, 8, true>, blocks, dim3(kThreads), 0, s, follows, T, S)
                    : launch(step_kernel<CAP, 8, false>, blocks, dim3(kThreads), 0, s, follows, T, S);
    if (e != cudaSuccess || last) return e;
  } while (i < a->count);
  return cudaSuccess;
}
// room for the sums of all launches
int64_t parts_bytes(const nr_adamw *a, int sms) {
  return round_up((a->count / kFew + 2) * (int64_t)sms * kNormBlocks * (int64_t)sizeof(double), 256);
}

}  // namespace

extern "C" int64_t nr_adamw_workspace(const nr_adamw *a, int device) {
  if (!tensors_ok(a, true)) return NR_ERR_INVALID_ARG;
  const int sms = nr_ops_sms(device);
  return sms < 1 ? NR_ERR_CUDA : parts_bytes(a, sms);
}

extern "C" nr_status nr_adamw_step(const nr_adamw *a, int device, void *ws, int64_t ws_bytes, void *stream) {
  if (!valid(a)) return NR_ERR_INVALID_ARG;
  const int sms = nr_ops_sms(device);
  if (sms < 1) return NR_ERR_CUDA;
  const bool clip = a->max_norm > 0.0;
  if (clip && (ws_bytes < parts_bytes(a, sms) || !ws || (reinterpret_cast<uintptr_t>(ws) & 255))) return NR_ERR_INVALID_ARG;
  DeviceGuard g(device);
  if (!g.ok) return NR_ERR_CUDA;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  Step S = {};
  S.master = a->master;
  S.m = a->m;
  S.v = a->v;
  S.m_scale = static_cast<uint8_t *>(a->m_scale);
  S.v_scale = static_cast<uint8_t *>(a->v_scale);
  S.step = a->step;
  S.ticket = a->ticket;
  S.lr_at = a->lr_at;
  S.lr = a->lr;
  S.log_b1 = log(a->beta1);
  S.log_b2 = log(a->beta2);
  S.max_norm = a->max_norm;
  S.b1 = (float)a->beta1;
  S.c1 = (float)(1.0 - a->beta1);
  S.b2 = (float)a->beta2;
  S.c2 = (float)(1.0 - a->beta2);
  S.eps = fmaxf((float)a->eps, 1.17549435e-38f);  // its reciprocal is in fp32's range
  S.one = 1.0f;
  S.tiny = tiny_matters(a);
  S.key0 = (uint32_t)a->seed;
  S.key1 = (uint32_t)((uint64_t)a->seed >> 32);
  cudaError_t e = cudaSuccess;
  if (clip) {
    S.norm = a->norm;
    S.parts = static_cast<double *>(ws);
    e = a->count <= kFew ? squares<kFew>(a, sms, static_cast<double *>(ws), S.part_count, s)
                         : squares<kMany>(a, sms, static_cast<double *>(ws), S.part_count, s);
  }
  if (e == cudaSuccess) e = a->count <= kFew ? steps<kFew>(a, S, sms, s) : steps<kMany>(a, S, sms, s);
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}

extern "C" nr_status nr_grad_norm(const nr_adamw *a, float *norm, int device, void *ws, int64_t ws_bytes, void *stream) {
  if (!tensors_ok(a, true) || !norm || !placed(norm, NR_F32)) return NR_ERR_INVALID_ARG;
  const int sms = nr_ops_sms(device);
  if (sms < 1) return NR_ERR_CUDA;
  if (ws_bytes < parts_bytes(a, sms) || !ws || (reinterpret_cast<uintptr_t>(ws) & 255)) return NR_ERR_INVALID_ARG;
  DeviceGuard g(device);
  if (!g.ok) return NR_ERR_CUDA;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  int count = 0;
  cudaError_t e = a->count <= kFew ? squares<kFew>(a, sms, static_cast<double *>(ws), count, s)
                                   : squares<kMany>(a, sms, static_cast<double *>(ws), count, s);
  if (e == cudaSuccess) e = launch(norm_kernel, 1, dim3(kThreads), 0, s, count > 0, static_cast<double *>(ws), count, norm);
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}

extern "C" nr_status nr_adamw_read(const void *m, const void *m_scale, const void *v, const void *v_scale, int64_t n, void *y_m,
                                   void *y_v, int device, void *stream) {
  if (n < 0 || n % kOpsGroup != 0) return NR_ERR_INVALID_ARG;
  if (n > 0 && (!m || !m_scale || !v || !v_scale || !y_m || !y_v)) return NR_ERR_INVALID_ARG;
  if (n > 0 && !(aligned(m, 16) && aligned(v, 16) && aligned(y_m, 16) && aligned(y_v, 16))) return NR_ERR_INVALID_ARG;
  const int sms = nr_ops_sms(device);
  if (sms < 1) return NR_ERR_CUDA;
  if (n == 0) return NR_OK;
  DeviceGuard g(device);
  if (!g.ok) return NR_ERR_CUDA;
  const int64_t need = ceil_div(n, kThreads * 8), most = (int64_t)sms * 4;
  read_kernel<<<dim3((unsigned)(need < most ? need : most), 2), kThreads, 0, static_cast<cudaStream_t>(stream)>>>(
      static_cast<const uint8_t *>(m), static_cast<const uint8_t *>(m_scale), static_cast<const uint8_t *>(v),
      static_cast<const uint8_t *>(v_scale), n, static_cast<uint4 *>(y_m), static_cast<uint4 *>(y_v));
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}
