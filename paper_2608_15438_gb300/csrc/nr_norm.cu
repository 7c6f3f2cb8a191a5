// Layer norm of residual encoders (neuroute_ops.h).
//   forward   mean = sum x / n, rstd = (sum (x - mean)^2 / n + eps)^-1/2,
//             y = (x - mean) rstd weight + bias
//   backward  xh = (x - mean) rstd, g = dy weight; dx = rstd (g - mean(g) -
//             xh mean(g xh)) + residual gradient; dweight = sum_m dy xh,
//             dbias = sum_m dy
//
// Both are bound by memory: forward reads x and writes y, backward reads dy and
// x (and the residual's gradient) and writes dx, each once. A row is held in the
// registers of some lanes, a warp or a block, so that the statistics' second
// pass (the deviations from the mean, which loses nothing to cancellation) and
// the output need no second read; several rows at a time keep enough bytes in
// flight. Persistent grids walk the rows; in the backward pass each thread
// keeps the parameters' sums of its columns in registers over all its rows, and
// a second kernel adds the blocks' sums in order.
//
// A thread's columns: eight consecutive ones at a time, by 16-byte accesses where
// every matrix allows them and by shifting pairs of aligned ones where 16-bit rows
// do not; in fp32 at other addresses single ones a group's width apart, so that a
// group's accesses stay contiguous. Rows longer than 16384 are read again from memory
// by a block a row, an element a load (the long_ kernels).
//
// Measured (a copy reaches 6.8 TB/s), bf16: forward 262144 x 1536 292 us, 5.5 TB/s;
// backward 455 us, 5.3 TB/s, with a residual's gradient 592 us, 5.4 TB/s. From a
// checkpoint, whose codes become numbers of the type and those fp32, 510 forward and 615
// backward: x's bytes halve, the time does not. 65536 x 1536 in fp32 159 forward, 207 backward (5.1, 5.8
// TB/s). 4096 x 20001 in bf16 156 forward, 893 backward (2.1, 0.6 TB/s).
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "nrq_ops.cuh"

namespace {

// How the matrices lie. kVec: every eight of a row's columns at a 16-byte address.
// kPhase: the matrices' rows start at the same distance from 16-byte addresses, as
// contiguous matrices of one width do, and have at most 4096 columns forward and 8192
// backward less a step (16 bytes' values). Rows a step apart then start
// alike, and a block takes only such rows: its threads hold the aligned sixteen bytes
// of them as in kVec, from `lead` values before a row's first one on, and only a row's
// ends need care (65536 x 1659 in fp16 against kAny: forward 163 us for 282, backward
// 201 for 333; 65536 x 3001 in fp32: 337 for 503, 484 for 875).
// kAny: everything else (65536 x 4095 in bf16: forward 509 us).
enum Lie { kAny, kVec, kPhase };
template <int A, typename T>
constexpr int kStepOf = A == kPhase ? 16 / (int)sizeof(T) : 1;

// values of a type, or a checkpoint's codes and scales
struct Rows {
  const void *p;
  const uint8_t *scale;
  int64_t ld;
  int64_t groups;
};

struct Norm {
  int64_t m, n;
  Rows x;
  const void *weight, *bias;
  int w_dtype;
  float eps;
  void *y;
  int64_t y_ld;
  float *mean, *rstd;
  const void *dy;
  int64_t dy_ld;
  const void *dres;
  int64_t dres_ld;
  void *dx;
  int64_t dx_ld;
  const void *x_end, *dy_end, *dres_end;  // past the matrices' last values
  float *parts;  // [blocks][2][n]: the blocks' sums for dweight, dbias
  int eights;    // a thread's columns come in eights
  int lie;       // Lie
};

// the column of element q of the thread's v-th eight, of a group of TPR threads
// (0: of `width`)
template <int TPR>
__device__ __forceinline__ int column(int eights, int v, int q, int t, int width = TPR) {
  const int w = TPR ? TPR : width;
  return eights ? (v * w + t) * 8 + q : (v * 8 + q) * w + t;
}

// a value if `in`, else 0, in one predicated load
__device__ __forceinline__ uint32_t load_if32(const void *p, bool in) {
  uint32_t v;
  asm("{\n .reg .pred p;\n setp.ne.b32 p, %2, 0;\n mov.b32 %0, 0;\n @p ld.global.nc.b32 %0, [%1];\n}\n"
      : "=r"(v)
      : "l"(p), "r"((int)in));
  return v;
}
__device__ __forceinline__ uint16_t load_if16(const void *p, bool in) {
  uint16_t v;
  asm("{\n .reg .pred p;\n setp.ne.b32 p, %2, 0;\n mov.b16 %0, 0;\n @p ld.global.nc.b16 %0, [%1];\n}\n"
      : "=h"(v)
      : "l"(p), "r"((int)in));
  return v;
}

// (kPhase: row, weights and n count from `lead` values before the row)
template <int TPR, int A, typename T>
__device__ __forceinline__ Eight<T> load_raw(const T *row, int eights, int v, int t, int lead, int n, const void *lo, const void *hi,
                                             int width = TPR) {
  const int c = column<TPR>(eights, v, 0, t, width);
  if (A == kVec) return c < n ? fetch_eight<T>(row + c, true, 8, lo, hi) : Eight<T>{};  // n is a multiple of 8
  if (A == kPhase) {
    Eight<T> o = {};
    // in 16 bits a row's ends are loaded with their neighbours and settled later, but for
    // the matrix's own ends (value by value 307 us for 201 backward at 65536 x 1659);
    // fp32 is 5% faster value by value
    const T *p = row + c;
    if (c < n && ((c >= lead && c + 8 <= n) || (sizeof(T) == 2 && p >= lo && p + 8 <= hi))) {
      o = fetch_eight<T>(p, true, 8, lo, hi);
    } else if (c < n) {
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const bool in = c + q >= lead && c + q < n;
        if (sizeof(T) == 4) o.r[q] = load_if32(p + q, in);
        else o.r[q >> 1] |= (uint32_t)load_if16(p + q, in) << (16 * (q & 1));
      }
    }
    return o;
  }
  if (sizeof(T) == 2) return fetch_eight<T>(row + c, false, min(8, n - c), lo, hi);
  // predicated loads without branches, so that all are under way at once
  Eight<T> o;
  const int st = eights ? 1 : TPR ? TPR : width;
  const T *p = row + c;
#pragma unroll
  for (int q = 0; q < 8; ++q, p += st) o.r[q] = load_if32(p, c + q * st < n);
  return o;
}
template <int TPR, int A, typename T>
__device__ __forceinline__ void settle_raw(Eight<T> &o, const T *row, int v, int t, int lead, int n, const void *lo,
                                           const void *hi, int width = TPR) {
  if (A == kVec || sizeof(T) == 4) return;
  const int c = column<TPR>(1, v, 0, t, width);
  if (A == kPhase) {  // zeros for the neighbouring rows' values
    if (c < lead || c + 8 > n) {
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const bool in = c + q >= lead && c + q < n;
        o.r[q >> 1] &= in ? 0xffffffffu : q & 1 ? 0x0000ffffu : 0xffff0000u;
      }
    }
    return;
  }
  settle_eight<T>(o, row + c, false, min(8, n - c), lo, hi);
}
// x, which may be a checkpoint: then the codes as numbers of T, exactly, and
// their scale (in fp16 near the type's end: the values that they stand for, as
// exact there, and 1)
template <int TPR, typename T>
__device__ __forceinline__ Eight<T> load_held(const Rows &x, int64_t i, int v, int t, int n, float &scale, int width = TPR) {
  Eight<T> o = {};
  scale = 1.0f;
  const int c = column<TPR>(1, v, 0, t, width);
  if (c < n) {
    const uint2 a = __ldg(reinterpret_cast<const uint2 *>(static_cast<const int8_t *>(x.p) + i * x.groups * kOpsGroup + c));
    const uint32_t s = __ldg(x.scale + i * x.groups + (c >> 5));
    scale = held8_down(s);
    float2 p[4];
    held8_numbers(a.x, p[0], p[1]);
    held8_numbers(a.y, p[2], p[3]);
    if (TypeCode<T>::code == NR_F16 && s >= kHeld8F16) {
#pragma unroll
      for (int q = 0; q < 4; ++q) p[q] = held8_in_f16(mul2(p[q], both(scale)));
      scale = 1.0f;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (sizeof(T) == 4) {
        o.r[2 * q] = __float_as_uint(p[q].x);
        o.r[2 * q + 1] = __float_as_uint(p[q].y);
      } else {
        o.r[q] = pack2(p[q].x, p[q].y, TypeCode<T>::code);
      }
    }
  }
  return o;
}
template <int TPR, int A, typename T>
__device__ __forceinline__ void store_row(T *row, int eights, int v, int t, int lead, int n, const float2 (&p)[4], int width = TPR) {
  const float o[8] = {p[0].x, p[0].y, p[1].x, p[1].y, p[2].x, p[2].y, p[3].x, p[3].y};
  const int c = column<TPR>(eights, v, 0, t, width);
  if (A == kVec || (A == kPhase && c >= lead && c + 8 <= n)) {
    if (c < n) store8(row, c, TypeCode<T>::code, 1, 8, o);
    return;
  }
  if (A == kPhase) {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (c + q >= lead && c + q < n) row[c + q] = from_f32<T>(o[q]);
    return;
  }
  if (sizeof(T) == 2) {  // a group's lanes of a warp walk a row in step
    constexpr int kShare = TPR > 0 && TPR < 32 ? TPR : 32;
    const uint4 h = pack8(p, TypeCode<T>::code);
    const uint32_t w[4] = {h.x, h.y, h.z, h.w};
    const int lane = threadIdx.x & 31, at = lane & (kShare - 1);
    const unsigned lanes = kShare == 32 ? 0xffffffffu : ((1u << (kShare & 31)) - 1u) << (lane & ~(kShare - 1));
    store16x8(row + c, n - c, w, at > 0, at < kShare - 1, lanes);
    return;
  }
  const int st = eights ? 1 : TPR ? TPR : width;
#pragma unroll
  for (int q = 0; q < 8; ++q)
    if (c + q * st < n) row[c + q * st] = from_f32<T>(o[q]);
}
// eight of the weights (or biases) as a thread's columns need them
template <int TPR, int A>
__device__ __forceinline__ void load_w(const void *p, int dtype, float none, int eights, int v, int t, int lead, int n,
                                       float2 (&w)[4], int width = TPR) {
  float o[8];
  const int c = column<TPR>(eights, v, 0, t, width);
  const int st = eights ? 1 : TPR ? TPR : width;
  if (!p) {
#pragma unroll
    for (int q = 0; q < 8; ++q) o[q] = none;
  } else if (A == kVec) {
    load8(p, c < n ? c : 0, dtype, 1, 8, o);
  } else if (A == kPhase) {  // once a block
#pragma unroll
    for (int q = 0; q < 8; ++q) o[q] = c + q >= lead && c + q < n ? load_any(p, c + q - lead, dtype) : 0.0f;
  } else if (eights && c + 8 <= n && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {  // rows end anywhere, the weights begin well
    load8(p, c, dtype, 1, 8, o);
  } else if (dtype == NR_F32) {  // one test of the type, all loads under way at once
#pragma unroll
    for (int q = 0; q < 8; ++q) o[q] = __uint_as_float(load_if32(static_cast<const float *>(p) + c + q * st, c + q * st < n));
  } else {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const uint32_t h = load_if16(static_cast<const uint16_t *>(p) + c + q * st, c + q * st < n);
      o[q] = unpack2(h, dtype).x;
    }
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) w[q] = make_float2(o[2 * q], o[2 * q + 1]);
}

// Keeps what was loaded or converted before it from being held in registers for
// reuse after it: the registers buy more rows in flight.
__device__ __forceinline__ void forget() { asm volatile("" ::: "memory"); }
template <typename T>
__device__ __forceinline__ void forget(Eight<T> &o) {
#pragma unroll
  for (int k = 0; k < (sizeof(T) == 4 ? 8 : 4); ++k) asm volatile("" : "+r"(o.r[k]));
}

// ------------------------------------------------------------ sums over a row's threads
// TPR lanes of a warp
template <int TPR, int K>
__device__ __forceinline__ void lane_sums(float (&v)[K]) {
#pragma unroll
  for (int o = TPR / 2; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
}
// A group of whole warps (`width` threads; the block, or one of several side by
// side, whose number is `group`): K sums (a power of two up to 8). A warp halves
// the values it carries at every exchange, so K sums take K + 5 - log2 K
// exchanges at most; the warps' sums are added in order by every thread. `turn`
// alternates between two buffers, so that one barrier a call is enough.
constexpr int kWarpsMax = 16;
template <int K>
struct BlockSums {
  float part[2][kWarpsMax][K < 4 ? 4 : K];
};
template <int K>
__device__ __forceinline__ void block_sums(float (&v)[K], BlockSums<K> &S, int turn, int t, int width, int group) {
  const int lane = t & 31, warps = width >> 5, first = group * warps;
  float u[K];
#pragma unroll
  for (int k = 0; k < K; ++k) u[k] = v[k];
  int o = 16;
#pragma unroll
  for (int h = K / 2; h >= 1; h >>= 1, o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int k = 0; k < h; ++k) {
      const float send = up ? u[k] : u[k + h], keep = up ? u[k + h] : u[k];
      u[k] = keep + __shfl_xor_sync(0xffffffffu, send, o);
    }
  }
  for (; o > 0; o >>= 1) u[0] += __shfl_xor_sync(0xffffffffu, u[0], o);
  constexpr int kLanes = 32 / K;  // lanes that hold the same sum
  if (lane % kLanes == 0) S.part[turn & 1][first + (t >> 5)][lane / kLanes] = u[0];
  if (warps > 1) asm volatile("bar.sync %0, %1;\n" ::"r"(group + 1), "r"(width) : "memory");
  else __syncwarp();
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = 0.0f;
  for (int w = 0; w < warps; ++w)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += S.part[turn & 1][first + w][k];
}

// ------------------------------------------------------------ rows in registers
// R rows from i on of a group of TPR threads (0: the block), V eights a thread:
// centred, with their means and reciprocal deviations, then written. Rows from
// m on are skipped (they hold zeros).
template <int TPR, int V, int R, int A, typename T>
struct Forward {
  // Rows of 16 bits are loaded a turn ahead, so that loads are under way during the
  // sums (2^20 x 128: 105 -> 86 us, 65536 x 4096: 330 -> 280 us; backward, where a
  // row's registers are twice as many, half the rows a turn and the next ones
  // ahead took 573 us for 450 at 262144 x 1536).
  static constexpr bool kAhead = A != kAny && sizeof(T) == 2;
  static constexpr int kStep = kStepOf<A, T>;
  int lead = 0;
  Eight<T> raw[R][V];
  float2 x[R][V][4];
  float mean[R], rstd[R];

  __device__ __forceinline__ void load(const Norm &N, int64_t i, int t, int eights, int width) {
    const T *p = static_cast<const T *>(N.x.p) + i * N.x.ld - lead;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int v = 0; v < V; ++v)
        raw[r][v] = i + r * kStep < N.m ? load_raw<TPR, A, T>(p + r * kStep * N.x.ld, eights, v, t, lead, (int)N.n + lead, N.x.p, N.x_end, width)
                                        : Eight<T>{};
  }
  // rows i on, `next` the turn after's
  template <typename Sums>
  __device__ __forceinline__ void statistics(const Norm &N, int64_t i, int64_t next, int t, int eights, int width, Sums sums) {
    const int n = (int)N.n + lead;
    const float inv = 1.0f / (float)(int)N.n;
    if (A == kPhase || !N.x.scale) {
      const T *p = static_cast<const T *>(N.x.p) + i * N.x.ld;
      if (!kAhead) load(N, i, t, eights, width);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (i + r * kStep < N.m) settle_raw<TPR, A, T>(raw[r][v], p + r * kStep * N.x.ld, v, t, lead, n, N.x.p, N.x_end, width);
#pragma unroll
          for (int q = 0; q < 4; ++q) x[r][v][q] = pair_of<T>(raw[r][v], q);
        }
      if (kAhead) load(N, next, t, eights, width);
    } else {
      float scale[R][V];
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v) raw[r][v] = load_held<TPR, T>(N.x, min(i + r, N.m - 1), v, t, n, scale[r][v], width);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int q = 0; q < 4; ++q) x[r][v][q] = mul2(pair_of<T>(raw[r][v], q), both(scale[r][v]));
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float2 s = both(0.0f);  // zeros past the row's end
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int q = 0; q < 4; ++q) s = add2(s, x[r][v][q]);
      mean[r] = s.x + s.y;
    }
    sums(mean);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mean[r] *= inv;
      float2 s = both(0.0f);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const bool in = column<TPR>(eights, v, 0, t, width) < n;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float2 d = add2(x[r][v][q], both(-mean[r]));
          if (A == kVec) {
            if (!in) d = both(0.0f);
          } else {
            const int c0 = column<TPR>(eights, v, 2 * q, t, width), c1 = column<TPR>(eights, v, 2 * q + 1, t, width);
            if (c0 >= n || (A == kPhase && c0 < lead)) d.x = 0.0f;
            if (c1 >= n || (A == kPhase && c1 < lead)) d.y = 0.0f;
          }
          x[r][v][q] = d;
          s = fma2(d, d, s);
        }
      }
      rstd[r] = s.x + s.y;
    }
    sums(rstd);
#pragma unroll
    for (int r = 0; r < R; ++r) rstd[r] = 1.0f / sqrtf(fmaf(rstd[r], inv, N.eps));
  }

  __device__ __forceinline__ void write(const Norm &N, int64_t i, int v, int t, int eights, int width,
                                        const float2 (&w)[4], const float2 (&b)[4]) {
    T *y = static_cast<T *>(N.y) + i * N.y_ld - lead;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (i + r * kStep >= N.m) break;
      float2 o[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) o[q] = fma2(mul2(x[r][v][q], both(rstd[r])), w[q], b[q]);
      store_row<TPR, A, T>(y + r * kStep * N.y_ld, eights, v, t, lead, (int)N.n + lead, o, width);
    }
  }
  __device__ __forceinline__ void write_statistics(const Norm &N, int64_t i) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (i + r * kStep < N.m) {
        N.mean[i + r * kStep] = mean[r];
        N.rstd[i + r * kStep] = rstd[r];
      }
  }
};

// The same for the backward pass: x and dy stay as they lie in memory, and are
// converted twice.
template <int TPR, int V, int R, int A, typename T>
struct Backward {
  static constexpr int kStep = kStepOf<A, T>;
  Eight<T> x[R][V], dy[R][V];
  float scale[R][V], shift[R], rstd[R];  // xh = x scale + shift
  float s[2 * R];                        // sum g, sum g xh of the thread's columns, then of the rows

  __device__ __forceinline__ void load(const Norm &N, int64_t i, int t, int eights, int lead, int width) {
    const int n = (int)N.n + lead;
    const T *pd = static_cast<const T *>(N.dy) + i * N.dy_ld - lead, *px = static_cast<const T *>(N.x.p) + i * N.x.ld - lead;
    // the residual's gradient into L2 while the sums are made, a line for the eight
    // threads that read it (65536 x 1536 in bf16: 180 -> 162 us; fp32 gained nothing)
    if (A != kAny && sizeof(T) == 2 && N.dres && (t & 7) == 0) {
      const T *pr = static_cast<const T *>(N.dres) + i * N.dres_ld - lead;
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int c = column<TPR>(1, v, 0, t, width);
          if (i + r * kStep < N.m && c < n) asm volatile("prefetch.global.L2 [%0];\n" ::"l"(pr + r * kStep * N.dres_ld + c));
        }
    }
    // one branch around all loads, so that they are under way together; rows past
    // the end hold zeros and add nothing
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int v = 0; v < V; ++v)
        dy[r][v] = i + r * kStep < N.m
                       ? load_raw<TPR, A, T>(pd + r * kStep * N.dy_ld, eights, v, t, lead, n, N.dy, N.dy_end, width)
                       : Eight<T>{};
    if (A != kPhase && N.x.scale) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v) x[r][v] = load_held<TPR, T>(N.x, min(i + r, N.m - 1), v, t, n, scale[r][v], width);
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          x[r][v] = i + r * kStep < N.m
                        ? load_raw<TPR, A, T>(px + r * kStep * N.x.ld, eights, v, t, lead, n, N.x.p, N.x_end, width)
                        : Eight<T>{};
          scale[r][v] = 1.0f;
        }
    }
    if (A != kVec) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (i + r * kStep >= N.m) break;
          settle_raw<TPR, A, T>(dy[r][v], pd + r * kStep * N.dy_ld, v, t, lead, n, N.dy, N.dy_end, width);
          if (A == kPhase || !N.x.scale)
            settle_raw<TPR, A, T>(x[r][v], px + r * kStep * N.x.ld, v, t, lead, n, N.x.p, N.x_end, width);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t j = i + r * kStep;
      shift[r] = j < N.m ? N.mean[j] : 0.0f;
      rstd[r] = j < N.m ? N.rstd[j] : 0.0f;
      s[2 * r] = s[2 * r + 1] = 0.0f;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      shift[r] *= -rstd[r];
#pragma unroll
      for (int v = 0; v < V; ++v) scale[r][v] *= rstd[r];
    }
  }
  __device__ __forceinline__ void add(int v, const float2 (&w)[4], float2 (&dw)[4], float2 (&db)[4]) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float2 s1 = both(0.0f), s2 = both(0.0f);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        // dy is zero past the row's end, and xh finite where the row is
        const float2 d = pair_of<T>(dy[r][v], q), g = mul2(d, w[q]);
        const float2 xh = fma2(pair_of<T>(x[r][v], q), both(scale[r][v]), both(shift[r]));
        s1 = add2(s1, g);
        s2 = fma2(g, xh, s2);
        db[q] = add2(db[q], d);
        dw[q] = fma2(d, xh, dw[q]);
      }
      s[2 * r] += s1.x + s1.y;
      s[2 * r + 1] += s2.x + s2.y;
    }
  }
  __device__ __forceinline__ void write(const Norm &N, int64_t i, int v, int t, int eights, int lead, int width,
                                        const float2 (&w)[4]) {
    const float inv = 1.0f / (float)(int)N.n;
    const int n = (int)N.n + lead;
    const T *res = static_cast<const T *>(N.dres) + i * N.dres_ld - lead;
    T *dx = static_cast<T *>(N.dx) + i * N.dx_ld - lead;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (i + r * kStep >= N.m) break;
      forget(x[r][v]);
      forget(dy[r][v]);
      const float2 m1 = both(-s[2 * r] * inv * rstd[r]), m2 = both(-s[2 * r + 1] * inv * rstd[r]);
      float2 o[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float2 xh = fma2(pair_of<T>(x[r][v], q), both(scale[r][v]), both(shift[r]));
        o[q] = fma2(xh, m2, fma2(mul2(pair_of<T>(dy[r][v], q), w[q]), both(rstd[r]), m1));
      }
      if (N.dres) {
        Eight<T> rr = load_raw<TPR, A, T>(res + r * kStep * N.dres_ld, eights, v, t, lead, n, N.dres, N.dres_end, width);
        settle_raw<TPR, A, T>(rr, res + r * kStep * N.dres_ld, v, t, lead, n, N.dres, N.dres_end, width);
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] = add2(o[q], pair_of<T>(rr, q));
      }
      store_row<TPR, A, T>(dx + r * kStep * N.dx_ld, eights, v, t, lead, n, o, width);
    }
  }
};

// The rows of a block: kStep phases of blocks, each with its rows; `unit` rows a turn.
template <int A, typename T>
struct Walk {
  int64_t first, stride;  // of a block
  int lead;
  __device__ __forceinline__ Walk(const Norm &N, const void *p, int64_t ld, int unit) {
    constexpr int kStep = kStepOf<A, T>;
    const int phase = kStep > 1 ? blockIdx.x % kStep : 0;
    first = phase + (int64_t)(blockIdx.x / kStep) * unit * kStep;
    stride = (int64_t)(gridDim.x / kStep) * unit * kStep;
    lead = kStep > 1 ? (int)((reinterpret_cast<uintptr_t>(p) + (uintptr_t)(phase * ld) * sizeof(T)) & 15) / (int)sizeof(T) : 0;
  }
};

// ------------------------------------------------------------ a row in a warp
// Blocks of 128: groups of TPR lanes hold R rows each, V eights of them a thread.
constexpr int kWarpThreads = 128;

template <int TPR, int V, int A, typename T>
__global__ void __launch_bounds__(kWarpThreads, 4) warp_forward_kernel(const Norm N) {
  constexpr int R = V == 6 ? 1 : V == 3 ? 2 : 4, kGroups = kWarpThreads / TPR;
  const Walk<A, T> W(N, N.x.p, N.x.ld, kGroups * R);
  const int t = threadIdx.x % TPR, lead = W.lead, n = (int)N.n + lead, eights = A != kAny ? 1 : N.eights;
  const int own = threadIdx.x / TPR * R * kStepOf<A, T>;  // the group's first row in the block's
  float2 w[4], b[4];  // V = 1: a thread's own, kept
  if (V == 1) {
    load_w<TPR, A>(N.weight, N.w_dtype, 1.0f, eights, 0, t, lead, n, w);
    load_w<TPR, A>(N.bias, N.w_dtype, 0.0f, eights, 0, t, lead, n, b);
  }
  Forward<TPR, V, R, A, T> F;
  F.lead = lead;
  if (F.kAhead && (A == kPhase || !N.x.scale)) F.load(N, W.first + own, t, eights, TPR);
  // a block's groups take the same number of turns, so that shuffles are complete
  for (int64_t i0 = W.first; i0 < N.m; i0 += W.stride) {
    const int64_t i = i0 + own;
    F.statistics(N, i, i + W.stride, t, eights, TPR, [](float(&v)[R]) { lane_sums<TPR, R>(v); });
    if (V > 1) forget();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (V > 1) {
        load_w<TPR, A>(N.weight, N.w_dtype, 1.0f, eights, v, t, lead, n, w);
        load_w<TPR, A>(N.bias, N.w_dtype, 0.0f, eights, v, t, lead, n, b);
      }
      F.write(N, i, v, t, eights, TPR, w, b);
    }
    if (N.mean && t == 0) F.write_statistics(N, i);
  }
}

// Up to 256 columns: V = 1, four rows a group (two in fp32).
template <int TPR, int A, typename T>
__global__ void __launch_bounds__(kWarpThreads, 4) warp_backward_kernel(const Norm N) {
  constexpr int R = sizeof(T) == 4 ? 2 : 4, kGroups = kWarpThreads / TPR;
  __shared__ float sums[2][TPR * 8];
  const Walk<A, T> W(N, N.dy, N.dy_ld, kGroups * R);
  const int t = threadIdx.x % TPR, group = threadIdx.x / TPR, lead = W.lead, n = (int)N.n + lead;
  const int eights = A != kAny ? 1 : N.eights;
  float2 w[4], dw[4] = {}, db[4] = {};
  load_w<TPR, A>(N.weight, N.w_dtype, 1.0f, eights, 0, t, lead, n, w);
  for (int64_t i0 = W.first; i0 < N.m; i0 += W.stride) {
    const int64_t i = i0 + group * R * kStepOf<A, T>;
    Backward<TPR, 1, R, A, T> G;
    G.load(N, i, t, eights, lead, TPR);
    G.add(0, w, dw, db);
    lane_sums<TPR, 2 * R>(G.s);
    G.write(N, i, 0, t, eights, lead, TPR, w);
  }
  grid_launch();
  if (!N.parts) return;
  float *part = N.parts + (int64_t)blockIdx.x * 2 * N.n;
  for (int g = 0; g < kGroups; ++g) {  // the groups in order
    if (group == g) {
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int c = column<TPR>(eights, 0, q, t);
        float a = q & 1 ? dw[q >> 1].y : dw[q >> 1].x, e = q & 1 ? db[q >> 1].y : db[q >> 1].x;
        if (g > 0) {
          a += sums[0][t * 8 + q];
          e += sums[1][t * 8 + q];
        }
        sums[0][t * 8 + q] = a;
        sums[1][t * 8 + q] = e;
        if (g + 1 == kGroups && c >= lead && c < n) {
          part[c - lead] = a;
          part[N.n + c - lead] = e;
        }
      }
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------ a row in a block
// The block has just the threads that a row's eights need; R rows at a time.
template <int V, int R, int THREADS, int A, typename T>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 3 : V == 4 ? 1 : 2) block_forward_kernel(const Norm N) {
  __shared__ BlockSums<R> S;
  const Walk<A, T> W(N, N.x.p, N.x.ld, R);
  const int t = threadIdx.x, lead = W.lead, n = (int)N.n + lead, eights = A != kAny ? 1 : N.eights, width = blockDim.x;
  float2 w[4], b[4];  // kPhase: a thread's own, kept
  if (A == kPhase) {
    load_w<0, A>(N.weight, N.w_dtype, 1.0f, eights, 0, t, lead, n, w, width);
    load_w<0, A>(N.bias, N.w_dtype, 0.0f, eights, 0, t, lead, n, b, width);
  }
  int turn = 0;
  Forward<0, V, R, A, T> F;
  F.lead = lead;
  if (F.kAhead && (A == kPhase || !N.x.scale)) F.load(N, W.first, t, eights, width);
  for (int64_t i = W.first; i < N.m; i += W.stride) {
    F.statistics(N, i, i + W.stride, t, eights, width, [&](float(&v)[R]) { block_sums<R>(v, S, turn++, t, width, 0); });
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (A != kPhase) {
        load_w<0, A>(N.weight, N.w_dtype, 1.0f, eights, v, t, lead, n, w, width);
        load_w<0, A>(N.bias, N.w_dtype, 0.0f, eights, v, t, lead, n, b, width);
      }
      F.write(N, i, v, t, eights, width, w, b);
    }
    if (N.mean && t == 0) F.write_statistics(N, i);
  }
}

// Backward: with THREADS 384 blockDim.y groups of blockDim.x threads, R rows each,
// so that short rows leave few blocks' sums to add; the groups' are added in order.
template <int V, int R, int THREADS, int A, typename T>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 3 : THREADS == 384 ? 2 : 1) block_backward_kernel(const Norm N) {
  __shared__ BlockSums<2 * R> S;
  extern __shared__ float sums[];  // [2][n], with several groups
  const int group = THREADS == 384 ? threadIdx.y : 0, groups = THREADS == 384 ? blockDim.y : 1;
  const Walk<A, T> W(N, N.dy, N.dy_ld, groups * R);
  const int t = threadIdx.x, lead = W.lead, n = (int)N.n + lead, eights = A != kAny ? 1 : N.eights, width = blockDim.x;
  float2 own[A == kPhase ? V : 1][4];  // weights, kept
  if (A == kPhase) {
#pragma unroll
    for (int v = 0; v < V; ++v) load_w<0, A>(N.weight, N.w_dtype, 1.0f, eights, v, t, lead, n, own[A == kPhase ? v : 0], width);
  }
  float2 dw[V][4] = {}, db[V][4] = {};
  int turn = 0;
  for (int64_t i = W.first + group * R * kStepOf<A, T>; i < N.m; i += W.stride) {
    Backward<0, V, R, A, T> G;
    G.load(N, i, t, eights, lead, width);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float2(&w)[4] = own[A == kPhase ? v : 0];
      if (A != kPhase) load_w<0, A>(N.weight, N.w_dtype, 1.0f, eights, v, t, lead, n, w, width);
      G.add(v, w, dw[v], db[v]);
    }
    block_sums<2 * R>(G.s, S, turn++, t, width, group);
    forget();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float2(&w)[4] = own[A == kPhase ? v : 0];
      if (A != kPhase) load_w<0, A>(N.weight, N.w_dtype, 1.0f, eights, v, t, lead, n, w, width);
      G.write(N, i, v, t, eights, lead, width, w);
    }
  }
  grid_launch();
  if (!N.parts) return;
  float *part = N.parts + (int64_t)blockIdx.x * 2 * N.n;
  for (int g = 0; g < groups; ++g) {
    if (group == g) {
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int c = column<0>(eights, v, q, t, width) - lead;
          if (c < 0 || c >= (int)N.n) continue;
          float a = q & 1 ? dw[v][q >> 1].y : dw[v][q >> 1].x, e = q & 1 ? db[v][q >> 1].y : db[v][q >> 1].x;
          if (g > 0) {
            a += sums[c];
            e += sums[N.n + c];
          }
          float *to = g + 1 < groups ? sums : part;
          to[c] = a;
          to[N.n + c] = e;
        }
    }
    if (groups > 1) __syncthreads();
  }
}

// dweight, dbias: the blocks' sums, 32 columns a block, 32 rows of parts at a time
__global__ void __launch_bounds__(1024)
    norm_params_kernel(const float *parts, int count, int64_t n, void *dweight, void *dbias, int dtype) {
  __shared__ float sums[32][33];
  const int c = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int64_t e = (int64_t)blockIdx.x * 32 + c;  // into [2][n]
  grid_wait();
  float s = 0.0f;
  if (e < 2 * n) {
#pragma unroll 8
    for (int p = r; p < count; p += 32) s += parts[(int64_t)p * 2 * n + e];
  }
  sums[r][c] = s;
  __syncthreads();
  if (r != 0 || e >= 2 * n) return;
  for (int q = 1; q < 32; ++q) s += sums[q][c];
  store_any(e < n ? dweight : dbias, e < n ? e : e - n, dtype, s);
}

// ------------------------------------------------------------ rows past 16384
constexpr int kLong = 16384, kLongThreads = 512;

__device__ __forceinline__ float long_x(const Rows &x, int64_t i, int64_t j, int dtype) {
  if (!x.scale) return load_any(x.p, i * x.ld + j, dtype);
  const float v = (float)static_cast<const int8_t *>(x.p)[i * x.groups * kOpsGroup + j] *
                  held8_down(x.scale[i * x.groups + (j >> 5)]);
  return dtype == NR_F16 ? held8_in_f16(make_float2(v, v)).x : v;
}

__global__ void __launch_bounds__(kLongThreads) long_forward_kernel(const Norm N, int dtype) {
  __shared__ BlockSums<1> S;
  const int64_t i = blockIdx.x;
  float s[1] = {0.0f};
  for (int64_t j = threadIdx.x; j < N.n; j += kLongThreads) s[0] += long_x(N.x, i, j, dtype);
  block_sums<1>(s, S, 0, (int)threadIdx.x, kLongThreads, 0);
  const float mean = s[0] / (float)N.n;
  s[0] = 0.0f;
  for (int64_t j = threadIdx.x; j < N.n; j += kLongThreads) {
    const float d = long_x(N.x, i, j, dtype) - mean;
    s[0] = fmaf(d, d, s[0]);
  }
  block_sums<1>(s, S, 1, (int)threadIdx.x, kLongThreads, 0);
  const float rstd = 1.0f / sqrtf(s[0] / (float)N.n + N.eps);
  for (int64_t j = threadIdx.x; j < N.n; j += kLongThreads) {
    const float w = N.weight ? load_any(N.weight, j, N.w_dtype) : 1.0f, b = N.bias ? load_any(N.bias, j, N.w_dtype) : 0.0f;
    store_any(N.y, i * N.y_ld + j, dtype, fmaf((long_x(N.x, i, j, dtype) - mean) * rstd, w, b));
  }
  if (N.mean && threadIdx.x == 0) {
    N.mean[i] = mean;
    N.rstd[i] = rstd;
  }
}

__global__ void __launch_bounds__(kLongThreads) long_dx_kernel(const Norm N, int dtype) {
  __shared__ BlockSums<2> S;
  const int64_t i = blockIdx.x;
  const float mean = N.mean[i], rstd = N.rstd[i];
  float s[2] = {0.0f, 0.0f};
  for (int64_t j = threadIdx.x; j < N.n; j += kLongThreads) {
    const float g = load_any(N.dy, i * N.dy_ld + j, dtype) * (N.weight ? load_any(N.weight, j, N.w_dtype) : 1.0f);
    s[0] += g;
    s[1] = fmaf(g, (long_x(N.x, i, j, dtype) - mean) * rstd, s[1]);
  }
  block_sums<2>(s, S, 0, (int)threadIdx.x, kLongThreads, 0);
  const float m1 = s[0] / (float)N.n, m2 = s[1] / (float)N.n;
  for (int64_t j = threadIdx.x; j < N.n; j += kLongThreads) {
    const float g = load_any(N.dy, i * N.dy_ld + j, dtype) * (N.weight ? load_any(N.weight, j, N.w_dtype) : 1.0f);
    float d = rstd * (g - m1 - (long_x(N.x, i, j, dtype) - mean) * rstd * m2);
    if (N.dres) d += load_any(N.dres, i * N.dres_ld + j, dtype);
    store_any(N.dx, i * N.dx_ld + j, dtype, d);
  }
}

// 32 columns and every gridDim.y-th eight rows a block -> parts
__global__ void __launch_bounds__(256) long_params_kernel(const Norm N, int dtype) {
  __shared__ float pw[8][33], pb[8][33];
  const int c = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int64_t j = (int64_t)blockIdx.x * 32 + c;
  float w = 0.0f, b = 0.0f;
  if (j < N.n)
    for (int64_t i = (int64_t)blockIdx.y * 8 + r; i < N.m; i += (int64_t)gridDim.y * 8) {
      const float d = load_any(N.dy, i * N.dy_ld + j, dtype);
      b += d;
      w = fmaf(d, (long_x(N.x, i, j, dtype) - N.mean[i]) * N.rstd[i], w);
    }
  pw[r][c] = w;
  pb[r][c] = b;
  __syncthreads();
  if (r != 0 || j >= N.n) return;
  for (int q = 1; q < 8; ++q) {
    w += pw[q][c];
    b += pb[q][c];
  }
  N.parts[(int64_t)blockIdx.y * 2 * N.n + j] = w;
  N.parts[(int64_t)blockIdx.y * 2 * N.n + N.n + j] = b;
}

// ------------------------------------------------------------ host
bool valid(const nr_layer_norm *a, bool backward) {
  if (!a || a->m < 0 || a->m > kOpsMaxRows || a->n < 1 || a->n > kOpsMaxCols) return false;
  if (a->dtype < NR_F32 || a->dtype > NR_BF16 || (a->w_dtype != a->dtype && a->w_dtype != NR_F32)) return false;
  if (a->x_ld < 0 || a->dy_ld < 0 || a->residual_grad_ld < 0 || (a->m > 0 && !a->x)) return false;
  if (a->m > 0 && (!placed(a->x, a->dtype, a->x_scale) || !placed(a->weight, a->w_dtype) || !placed(a->mean, NR_F32) ||
                   !placed(a->rstd, NR_F32)))
    return false;
  if (a->m > 0 && (backward ? !placed(a->dy, a->dtype) || !placed(a->residual_grad, a->dtype) || !placed(a->dx, a->dtype) ||
                                  !placed(a->dweight, a->w_dtype) || !placed(a->dbias, a->w_dtype)
                            : !placed(a->bias, a->w_dtype) || !placed(a->y, a->dtype)))
    return false;
  if (!backward)
    return a->eps > 0.0 && !a->mean == !a->rstd && (a->m == 0 || (a->y && a->y_ld >= a->n));
  return !a->dweight == !a->dbias &&
         (a->m == 0 || (a->dy && a->mean && a->rstd && a->dx && a->dx_ld >= a->n));
}

Norm norm_of(const nr_layer_norm *a, bool backward) {
  Norm N = {};
  N.m = a->m;
  N.n = a->n;
  N.x = {a->x, static_cast<const uint8_t *>(a->x_scale), a->x_ld, ceil_div(a->n, kOpsGroup)};
  N.weight = a->weight;
  N.bias = a->bias;
  N.w_dtype = (int)a->w_dtype;
  // at least the least fp32: an eps below it is positive too (a row without deviation times infinity was NaN)
  N.eps = fmaxf((float)a->eps, 1.40129846e-45f);
  N.y = a->y;
  N.y_ld = a->y_ld;
  N.mean = a->mean;
  N.rstd = a->rstd;
  N.dy = a->dy;
  N.dy_ld = a->dy_ld;
  N.dres = a->residual_grad;
  N.dres_ld = a->residual_grad_ld;
  N.dx = a->dx;
  N.dx_ld = a->dx_ld;
  const int64_t dt = a->dtype;
  bool vec = a->n % 8 == 0 && (a->x_scale || vec_ok(a->x, a->x_ld, dt));
  if (backward)
    vec = vec && vec_ok(a->dy, a->dy_ld, dt) && vec_ok(a->dx, a->dx_ld, dt) &&
          (!a->residual_grad || vec_ok(a->residual_grad, a->residual_grad_ld, dt));
  else
    vec = vec && vec_ok(a->y, a->y_ld, dt);
  vec = vec && vec_ok(a->weight, 8, a->w_dtype) && vec_ok(a->bias, 8, a->w_dtype);
  const int64_t e = (int64_t)type_bytes(dt), step = 16 / e;
  const auto alike = [&](const void *p, int64_t ld) {
    return ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(a->x)) & 15) == 0 && (ld - a->x_ld) % step == 0;
  };
  const bool phase = !vec && !a->x_scale && a->n <= (backward ? 8192 : 4096) - step &&
                     (backward ? alike(a->dy, a->dy_ld) && alike(a->dx, a->dx_ld) &&
                                     (!a->residual_grad || alike(a->residual_grad, a->residual_grad_ld))
                               : alike(a->y, a->y_ld));
  N.lie = vec ? kVec : phase ? kPhase : kAny;
  N.eights = vec || phase || a->x_scale || dt != NR_F32;
  N.x_end = static_cast<const char *>(a->x) + ((a->m - 1) * a->x_ld + a->n) * e;
  N.dy_end = static_cast<const char *>(a->dy) + ((a->m - 1) * a->dy_ld + a->n) * e;
  N.dres_end = static_cast<const char *>(a->residual_grad) + ((a->m - 1) * a->residual_grad_ld + a->n) * e;
  return N;
}

// How a row is held. Warps (tpr lanes a row, v eights a thread): forward up to
// 1536 columns of aligned rows, where a row's sums cost five exchanges and no barrier;
// backward up to 256, as the parameters' sums are 16 registers an eight and
// leave too few rows in flight beyond. Fewer lanes take rows of 64 and 128, so that
// none is idle. Blocks (tpr 0, v eights a thread, `threads` of them): up to
// 16384. Longer rows: threads 0.
struct Shape {
  int tpr, v, threads, groups;  // threads a row's group, groups a block
};
Shape shape_of(const Norm &N, bool small, bool backward) {
  const bool vec = N.lie == kVec;
  const int64_t n = N.n + (N.lie == kPhase ? (small ? 7 : 3) : 0);  // with the values before a row
  if (n <= 256) return {n <= 64 ? 8 : n <= 128 ? 16 : 32, 1, kWarpThreads, 1};
  if (!backward && vec && n <= 768) return {32, 3, kWarpThreads, 1};
  if (!backward && vec && n <= 1536) return {32, 6, kWarpThreads, 1};
  if (n > kLong) return {0, 0, 0, 0};
  // forward with aligned rows: as many eights as leave a block 256 threads, since
  // the rows of three such blocks an SM wait less for each other at the sums'
  // barriers than two of 512 (65536 x 4096: 212 us, 280 by 512 threads)
  const bool wide = backward ? n > 2048 : n > (vec ? 2048 : 4096);
  const int v = n > (vec && small && !backward ? 4096 : 8192) ? 4 : wide ? 2 : 1;
  const int threads = (int)round_up(ceil_div(n, 8 * v), 32);
  // groups side by side up to 384 threads: rows of 387 in fp32 leave 304 blocks'
  // sums instead of 1824 to add (23 us); rows of 1536 ran 15% slower so
  const int groups = backward && threads <= 128 && v == 1 ? 384 / threads : 1;
  return {0, v, threads, groups};
}

// Blocks of a persistent grid: those the registers allow at once, by sizes alone,
// so that the order of the parameters' sums is fixed.
int block_count(const Shape &s, const Norm &N, bool small, bool backward, int sms) {
  const bool vec = N.lie != kAny;
  int per_sm, rows = s.groups;
  if (s.tpr) {
    per_sm = 4;
    rows = kWarpThreads / s.tpr;
  } else if (backward && s.v == 1) {
    per_sm = 768 / (s.threads * s.groups);
  } else {
    const int held = !backward ? s.threads <= 256 ? 768 : s.v < 4 ? 1024 : 512 : s.v == 2 && !vec ? 580 : 512;
    per_sm = held / s.threads;
  }
  const int64_t step = N.lie == kPhase ? small ? 8 : 4 : 1;
  const int64_t need = round_up(ceil_div(N.m, rows), step), most = (int64_t)sms * per_sm / step * step;
  return (int)(need < most ? need : most);
}

// rows at a time of a block with one eight a thread: what 80 registers hold
template <int A, typename T>
constexpr int block_rows() { return A == kVec && sizeof(T) == 2 ? 4 : 2; }

template <int A, typename T>
cudaError_t forward_typed(const Norm &N, const Shape &s, int blocks, cudaStream_t st) {
  const int th = s.threads;
  if (s.tpr == 8) warp_forward_kernel<8, 1, A, T><<<blocks, th, 0, st>>>(N);
  else if (s.tpr == 16) warp_forward_kernel<16, 1, A, T><<<blocks, th, 0, st>>>(N);
  else if (s.tpr && s.v == 1) warp_forward_kernel<32, 1, A, T><<<blocks, th, 0, st>>>(N);
  else if (s.v == 1 && th <= 256) block_forward_kernel<1, block_rows<A, T>(), 256, A, T><<<blocks, th, 0, st>>>(N);
  else if (A != kVec && s.v == 1) block_forward_kernel<1, 2, 512, A == kVec ? kAny : A, T><<<blocks, th, 0, st>>>(N);
  else if (A == kVec && s.tpr && s.v == 3) warp_forward_kernel<32, 3, kVec, T><<<blocks, th, 0, st>>>(N);
  else if (A == kVec && s.tpr) warp_forward_kernel<32, 6, kVec, T><<<blocks, th, 0, st>>>(N);
  else if (A == kVec && s.v == 2 && th <= 256)
    block_forward_kernel<2, sizeof(T) == 2 ? 2 : 1, 256, kVec, T><<<blocks, th, 0, st>>>(N);
  else if (A == kVec && s.v == 4 && th <= 256) block_forward_kernel<4, 1, 256, kVec, T><<<blocks, th, 0, st>>>(N);
  else if (A != kPhase && s.v == 2) block_forward_kernel<2, 1, 512, A == kPhase ? kAny : A, T><<<blocks, th, 0, st>>>(N);
  else if (A != kPhase) block_forward_kernel<4, 1, 512, A == kPhase ? kAny : A, T><<<blocks, th, 0, st>>>(N);
  return cudaGetLastError();
}
template <int A, typename T>
cudaError_t backward_typed(const Norm &N, const Shape &s, int blocks, cudaStream_t st) {
  const int th = s.threads;
  if (s.tpr == 8) warp_backward_kernel<8, A, T><<<blocks, th, 0, st>>>(N);
  else if (s.tpr == 16) warp_backward_kernel<16, A, T><<<blocks, th, 0, st>>>(N);
  else if (s.tpr) warp_backward_kernel<32, A, T><<<blocks, th, 0, st>>>(N);
  else if (s.v == 1 && s.groups == 1)
    block_backward_kernel<1, block_rows<A, T>(), 256, A, T><<<blocks, th, 0, st>>>(N);
  else if (s.v == 1)
    block_backward_kernel<1, block_rows<A, T>(), 384, A, T><<<blocks, dim3(th, s.groups), (size_t)N.n * 8, st>>>(N);
  else if (s.v == 2) block_backward_kernel<2, A == kVec && sizeof(T) == 2 ? 2 : 1, 512, A, T><<<blocks, th, 0, st>>>(N);
  else if (A != kPhase) block_backward_kernel<4, 1, 512, A == kPhase ? kAny : A, T><<<blocks, th, 0, st>>>(N);
  return cudaGetLastError();
}
template <typename T>
cudaError_t launch_typed(const Norm &N, const Shape &s, bool backward, int blocks, cudaStream_t st) {
  if (N.lie == kVec) return backward ? backward_typed<kVec, T>(N, s, blocks, st) : forward_typed<kVec, T>(N, s, blocks, st);
  if (N.lie == kPhase) return backward ? backward_typed<kPhase, T>(N, s, blocks, st) : forward_typed<kPhase, T>(N, s, blocks, st);
  return backward ? backward_typed<kAny, T>(N, s, blocks, st) : forward_typed<kAny, T>(N, s, blocks, st);
}
cudaError_t launch_any(const Norm &N, const Shape &s, bool backward, int64_t dtype, int blocks, cudaStream_t st) {
  if (dtype == NR_F32) return launch_typed<float>(N, s, backward, blocks, st);
  if (dtype == NR_F16) return launch_typed<__half>(N, s, backward, blocks, st);
  return launch_typed<__nv_bfloat16>(N, s, backward, blocks, st);
}
constexpr int kLongParts = 32;

}  // namespace

extern "C" nr_status nr_layer_norm_forward(const nr_layer_norm *a, int device, void *stream) {
  if (!valid(a, false)) return NR_ERR_INVALID_ARG;
  if (a->m == 0) return NR_OK;
  const int sms = nr_ops_sms(device);
  DeviceGuard g(device);
  if (sms < 1 || !g.ok) return NR_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const Norm N = norm_of(a, false);
  const Shape sh = shape_of(N, a->dtype != NR_F32, false);
  cudaError_t e;
  if (sh.threads) {
    e = launch_any(N, sh, false, a->dtype, block_count(sh, N, a->dtype != NR_F32, false, sms), s);
  } else {
    long_forward_kernel<<<(unsigned)a->m, kLongThreads, 0, s>>>(N, (int)a->dtype);
    e = cudaGetLastError();
  }
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}

extern "C" int64_t nr_layer_norm_backward_workspace(const nr_layer_norm *a, int device) {
  if (!valid(a, true)) return NR_ERR_INVALID_ARG;
  const int sms = nr_ops_sms(device);
  if (sms < 1) return NR_ERR_CUDA;
  if (a->m == 0 || !a->dweight) return 0;
  const Norm N = norm_of(a, true);
  const Shape sh = shape_of(N, a->dtype != NR_F32, true);
  const int64_t blocks = sh.threads ? block_count(sh, N, a->dtype != NR_F32, true, sms) : kLongParts;
  return round_up(blocks * 2 * a->n * 4, 256);
}

extern "C" nr_status nr_layer_norm_backward(const nr_layer_norm *a, int device, void *ws, int64_t ws_bytes, void *stream) {
  const int64_t need = nr_layer_norm_backward_workspace(a, device);
  if (need < 0) return (nr_status)need;
  if (ws_bytes < need || (need > 0 && (!ws || (reinterpret_cast<uintptr_t>(ws) & 255))))
    return NR_ERR_INVALID_ARG;
  DeviceGuard g(device);
  if (!g.ok) return NR_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (a->m == 0) {
    if (a->dweight) {
      e = cudaMemsetAsync(a->dweight, 0, (size_t)a->n * type_bytes(a->w_dtype), s);
      if (e == cudaSuccess) e = cudaMemsetAsync(a->dbias, 0, (size_t)a->n * type_bytes(a->w_dtype), s);
    }
    return e == cudaSuccess ? NR_OK : cuda_status(e);
  }
  Norm N = norm_of(a, true);
  N.parts = a->dweight ? static_cast<float *>(ws) : nullptr;
  const Shape sh = shape_of(N, a->dtype != NR_F32, true);
  int parts = kLongParts;
  if (sh.threads) {
    parts = block_count(sh, N, a->dtype != NR_F32, true, nr_ops_sms(device));
    e = launch_any(N, sh, true, a->dtype, parts, s);
  } else {
    long_dx_kernel<<<(unsigned)a->m, kLongThreads, 0, s>>>(N, (int)a->dtype);
    if (N.parts)
      long_params_kernel<<<dim3((unsigned)ceil_div(a->n, 32), kLongParts), 256, 0, s>>>(N, (int)a->dtype);
    e = cudaGetLastError();
  }
  if (e == cudaSuccess && N.parts) {
    e = launch(norm_params_kernel, (unsigned)ceil_div(2 * a->n, 32), dim3(1024), 0, s, true, N.parts, parts, a->n,
               a->dweight, a->dbias, (int)a->w_dtype);
  }
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}
