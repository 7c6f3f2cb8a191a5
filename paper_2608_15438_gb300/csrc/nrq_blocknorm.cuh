// The norms around a block of a residual encoder (nr_block_norm): rows of up to 8192
// columns, worked on in shared memory. Bound by memory: forward reads r, u and the gate and writes y and h,
// backward reads dh, dy, y, u and the gate and writes dr, du and dgate, each once. Of 6.8 TB/s measured:
//   forward   262144 x 1536 bf16 around an fp32 stream 733 us, 6.6 TB/s; 10000 x 1536 bf16 30 us, 5.1 (eleven
//             warps an SM, six rows each: beginning and end)
//   backward  65536 x 1536 bf16 286 us, 5.6 TB/s (an instruction issued in 47% of cycles, twelve warps an SM: their
//             160 registers hold the columns' sums); 30011 x 387 fp32 71 us, 3.9, and 81 written at another pitch: 168
//             registers leave eleven warps, and what a row costs is shared by 387 columns (two warps a row, eight
//             columns a thread, 96 registers: 116 us)
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "nrq_ops.cuh"

namespace blocknorm {

struct Rows {
  void *p;
  int64_t ld;
};
struct Block {
  int64_t m, n;
  int dtype, r_dtype, w_dtype;
  int post, pre, act;
  int gate;  // 0 none, 1 a value a row, 2 full
  float alpha, eps;
  Rows r, u, q, y, h, dh, dy, dr, du, dq;
  const void *scale, *post_w, *post_b, *w, *b;
  float *u_mean, *u_rstd, *y_mean, *y_rstd;  // rows of stats
  float *row_sums;                           // [2][m]: mean g, mean g yh
  float *parts;                              // [4][blocks][n]: dh yh, dh, t a uh, t a
  void *dscale, *dpost_w, *dpost_b, *dw, *db;
};

// ------------------------------------------------------------ gates
// a(q) and its slope; infinities go to the limits, NaN stays
__device__ __forceinline__ float logistic(float q) { return rcp_approx(1.0f + exp2_approx(q * -1.44269504f)); }
__device__ __forceinline__ float gate_value(float q, int act) {
  const float a = logistic(q);
  return act == NR_ACT_SILU ? fmaxf(q, -100.0f) * a : a;
}
__device__ __forceinline__ float gate_slope(float q, int act) {
  const float a = logistic(q), r = 1.0f - a;
  return act == NR_ACT_SILU ? fmaf(fmaxf(fminf(q, 100.0f), -100.0f) * a, r, a) : a * r;
}
__device__ __forceinline__ float2 logistic2(float2 q) {
  const float2 h = mul2(q, both(-1.44269504f));
  const float2 d = add2(make_float2(exp2_approx(h.x), exp2_approx(h.y)), both(1.0f));
  return make_float2(rcp_approx(d.x), rcp_approx(d.y));
}
__device__ __forceinline__ float2 silu2(float2 q, float2 a) {
  return mul2(make_float2(fmaxf(q.x, -100.0f), fmaxf(q.y, -100.0f)), a);
}
__device__ __forceinline__ float2 silu_slope2(float2 q, float2 a) {  // a + q a (1 - a)
  const float2 r = fma2(a, both(-1.0f), both(1.0f));
  return fma2(mul2(make_float2(fmaxf(fminf(q.x, 100.0f), -100.0f), fmaxf(fminf(q.y, 100.0f), -100.0f)), a), r, a);
}

// ------------------------------------------------------------ vectors
__device__ __forceinline__ float vec(const void *p, int64_t j, int dtype, float none) { return p ? load_any(p, j, dtype) : none; }

// ------------------------------------------------------------ rows in shared memory
// A row is taken by TPR lanes of a warp, or by several warps (TPR 0), 8 V columns a
// thread: V eights where all matrices have 16 bits, else 2 V pieces of four, neighbouring threads' pieces side by
// side. Copies of the rows to come are under way (cp.async) while one is worked on: long rows have one stage a
// group, whose next copy starts when the present row is in registers, short and few ones up to four. What a row costs whatever
// its length (addresses, exchanges, statistics: some 200 instructions a warp) is shared by a thread's columns: eight of them,
// six warps a row of 1536, ran at 3.3 TB/s, an instruction issued in 68% of cycles.
//
// kAligned: all rows begin at multiples of 16 bytes and n is one of 8; a thread reads what it has
// copied itself. Else copies bring the aligned 16-byte blocks that a row lies in, and a thread's pieces
// begin `ref` columns before the row, so that they lie at whole pieces' places in the first matrix read (and in
// all others that lie alike, as contiguous ones of one width do); what lies otherwise is shifted
// into place. Rows PW apart begin alike; a block takes such rows only, so that its threads keep their columns. kAlike, for
// matrices read that all lie alike, leaves out the code that shifts (65536 x 1537 forward 306 -> 273 us).
constexpr int kMostStages = 4;
// how rows lie: anyhow, those read alike (nothing read is shifted into place), at multiples of 16 bytes
enum { kAny, kAlike, kAligned };

// a matrix as rows of it are copied
struct Source {
  const char *p, *end;
  int64_t pitch;  // bytes
  int at;         // its place in a stage
};
struct Ring {
  Source s[5];
  int row_bytes;  // of a row's stage
  int columns;    // that the threads of a row have, n or more
  int stages;
  int vectors;    // bytes at which the vectors lie in shared memory, behind the stages
  int present;    // of the vectors, bits: scale post_weight, scale post_bias, weight, bias
};

__device__ __forceinline__ uint32_t shared_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <int N>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wait_copies(int left) {
  if (left >= 3) wait_copies<3>();
  else if (left == 2) wait_copies<2>();
  else if (left == 1) wait_copies<1>();
  else wait_copies<0>();
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }

// ------------------------------------------------------------ pieces of a row
// PW consecutive values as they lie in memory
template <typename E, int PW>
struct Piece {
  static constexpr int kWords = PW * (int)sizeof(E) / 4, kBytes = kWords * 4;
};
template <int WORDS>
__device__ __forceinline__ void shared_words(const char *p, uint32_t *w) {
  if (WORDS == 4) {
    const uint4 v = *reinterpret_cast<const uint4 *>(p);
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  } else {
    const uint2 v = *reinterpret_cast<const uint2 *>(p);
    w[0] = v.x, w[1] = v.y;
  }
}
template <typename E, int PW>
__device__ __forceinline__ void numbers(const uint32_t *w, float2 (&v)[PW / 2]) {
#pragma unroll
  for (int q = 0; q < PW / 2; ++q) {
    if (sizeof(E) == 4) v[q] = make_float2(__uint_as_float(w[2 * q]), __uint_as_float(w[2 * q + 1]));
    else v[q] = unpack2(w[q], TypeCode<E>::code);
  }
}
// the PW values that begin s bytes behind p, s less than their size
template <typename E, int PW>
__device__ __forceinline__ void read_shifted(const char *p, int s, float2 (&v)[PW / 2]) {
  typedef Piece<E, PW> P;
  uint32_t w[2 * P::kWords];
  shared_words<P::kWords>(p, w);
  if (s) {
    shared_words<P::kWords>(p + P::kBytes, w + P::kWords);
    if (P::kWords == 4) {
#pragma unroll
      for (int k = 0; k < 6; ++k) w[k] = s & 8 ? w[k + 2] : w[k];
    }
#pragma unroll
    for (int k = 0; k < P::kWords + 1; ++k) w[k] = s & 4 ? w[k + 1] : w[k];
    if (sizeof(E) == 2) {
#pragma unroll
      for (int k = 0; k < P::kWords; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], s & 2 ? 16 : 0);
    }
  }
  numbers<E, PW>(w, v);
}
template <int WORDS>
__device__ __forceinline__ void write_block(void *at, const uint32_t *o) {
  if (WORDS == 4) *static_cast<uint4 *>(at) = make_uint4(o[0], o[1], o[2], o[3]);
  else *static_cast<uint2 *>(at) = make_uint2(o[0], o[1]);
}
template <typename E, int PW>
__device__ __forceinline__ void words_of(const float2 (&v)[PW / 2], uint32_t *w) {
#pragma unroll
  for (int q = 0; q < PW / 2; ++q) {
    if (sizeof(E) == 4) w[2 * q] = __float_as_uint(v[q].x), w[2 * q + 1] = __float_as_uint(v[q].y);
    else w[q] = pack2(v[q].x, v[q].y, TypeCode<E>::code);
  }
}
// Which of a row's values a thread stores as an aligned block, and which one by one. It has those of columns
// c to c + PW - 1, of which [lo, hi) are the row's, and c lies s values behind an aligned block's begin: that
// block has the predecessor's last s values and its own first PW - s; its last s are in its successor's.
struct SpanOf {
  bool block, rest;  // the block; the successor stores the last s
};
__host__ __device__ inline SpanOf span_of(int pw, int c, int lo, int hi, int s, bool prev, bool next) {
  return {(prev || s == 0) && c - s >= lo && c - s + pw <= hi, s != 0 && next && c + pw - s >= lo && c + 2 * pw - s <= hi};
}
template <typename E, int PW>
__device__ __forceinline__ void write_singly(E *p, int c, int lo, int hi, int s, SpanOf w,
                                             const uint32_t (&own)[Piece<E, PW>::kWords]) {
#pragma unroll
  for (int q = 0; q < PW; ++q)
    if (c + q >= lo && c + q < hi && !(q < PW - s ? w.block : w.rest)) {
      if (sizeof(E) == 4) reinterpret_cast<uint32_t *>(p)[q] = own[sizeof(E) == 4 ? q : 0];
      else reinterpret_cast<uint16_t *>(p)[q] = (uint16_t)(own[sizeof(E) == 4 ? 0 : q >> 1] >> (16 * (q & 1)));
    }
}

// ------------------------------------------------------------ a thread's place in its row
template <int TPR, int V, int PW, int LIE>
struct Place {
  static constexpr bool VEC = LIE == kAligned;
  static constexpr int kPieces = 8 * V / PW, kHalf = PW / 2;
  static constexpr int kStep = (TPR ? TPR : 32) * PW;  // from a thread's piece to its next: a warp has its columns together
  int t, width, n, group, base, full, ref;
  // `first`: row's first column of the first matrix read, of the block's rows
  __device__ __forceinline__ Place(int n_, int width_, const Source &s, int elements, int64_t row) : n(n_) {
    width = TPR ? TPR : width_;
    group = TPR ? threadIdx.x / (TPR ? TPR : 1) : threadIdx.y;
    t = TPR ? threadIdx.x % (TPR ? TPR : 1) : threadIdx.x;
    ref = VEC ? 0 : (int)((reinterpret_cast<uintptr_t>(s.p) + (uintptr_t)(row * s.pitch)) / (unsigned)elements) & (PW - 1);
    const int first = TPR ? 0 : (t >> 5) * (256 * V);  // the warp's first column
    base = first + (TPR ? t : t & 31) * PW;
    full = n + ref > first ? min((n + ref - first) / kStep, kPieces) : 0;  // pieces in the row for all threads
  }
  // a thread's columns count from `ref` before the row's first
  __device__ __forceinline__ int column(int p) const { return base + p * kStep; }
  __device__ __forceinline__ unsigned lanes() const {
    return TPR && TPR < 32 ? ((1u << (TPR & 31)) - 1u) << (threadIdx.x & 31 & ~(TPR - 1)) : 0xffffffffu;
  }
  // the row's columns that the thread's warp has (or the lanes that share it)
  __device__ __forceinline__ int of_warp() const {
    const int first = (t >> 5) * (256 * V);
    return TPR ? n : max(0, min(256 * V, n + ref - first)) - (first == 0 ? ref : 0);
  }
  // Copies row i of a matrix into its stage. No byte past the matrix is read; the block in which
  // it begins comes value by value if it begins inside one.
  template <typename E>
  __device__ __forceinline__ void copy(const Source &s, char *stage, int64_t i) const {
    const char *row = s.p + i * s.pitch;
    if constexpr (VEC) {
      constexpr int kBytes = Piece<E, PW>::kBytes;
      const uint32_t to = shared_address(stage) + s.at + base * (int)sizeof(E);
      const char *from = row + base * (int)sizeof(E);
#pragma unroll
      for (int p = 0; p < kPieces; ++p)
        if (column(p) < n) {
          const int by = p * kStep * (int)sizeof(E);
          if (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(to + by), "l"(from + by) : "memory");
          else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;\n" ::"r"(to + by), "l"(from + by) : "memory");
        }
    } else {
      const int lead = (int)(reinterpret_cast<uintptr_t>(row) & 15), blocks = (lead + n * (int)sizeof(E) + 15) >> 4;
      const char *from = row - lead;
      const uint32_t to = shared_address(stage) + s.at;
      if (from >= s.p && from + 16 * blocks <= s.end) {
#pragma unroll 4
        for (int k = t; k < blocks; k += width)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(to + 16 * k), "l"(from + 16 * k) : "memory");
        return;
      }
      for (int k = t; k < blocks; k += width) {
        const char *a = from + 16 * k;
        if (a >= s.p) {
          const int64_t left = s.end - a;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(to + 16 * k), "l"(a), "r"(left < 16 ? (int)left : 16)
                       : "memory");
        } else {
          for (int b = lead; b < 16 && a + b < s.end; b += (int)sizeof(E))
            *reinterpret_cast<E *>(stage + s.at + 16 * k + b) = *reinterpret_cast<const E *>(a + b);
        }
      }
    }
  }
  // row i in its stage: where the piece at column 0 begins there, and how many bytes behind a piece's place
  struct In {
    const char *p;
    int s;
  };
  template <typename E>
  __device__ __forceinline__ In in(const Source &s, const char *stage, int64_t i) const {
    if constexpr (VEC) return {stage + s.at + base * (int)sizeof(E), 0};
    const int lead = (int)(reinterpret_cast<uintptr_t>(s.p + i * s.pitch) & 15) - ref * (int)sizeof(E);
    const int by = LIE == kAlike ? 0 : lead & (Piece<E, PW>::kBytes - 1);
    return {stage + s.at + (lead - by) + base * (int)sizeof(E), by};
  }
  // stages and vectors in shared memory have room for all of the threads' columns: reads need no bounds, and what
  // they bring from outside the row is cleared (`clip`) where it counts
  template <typename E>
  __device__ __forceinline__ void read(const In &r, int p, float2 (&v)[kHalf]) const {
    const char *at = r.p + p * kStep * (int)sizeof(E);
    if constexpr (LIE != kAny) {
      uint32_t w[Piece<E, PW>::kWords];
      shared_words<Piece<E, PW>::kWords>(at, w);
      numbers<E, PW>(w, v);
    } else {
      read_shifted<E, PW>(at, r.s, v);
    }
  }
  // a row that is written, its pieces in order: where the piece at column 0 is or would be, how many values
  // behind a block's begin, and the words of the last piece
  template <typename E>
  struct Out {
    E *p;
    int s;
    uint32_t last[Piece<E, PW>::kWords];
  };
  template <typename E>
  __device__ __forceinline__ Out<E> out(const Rows &m, int64_t i) const {
    Out<E> o;
    o.p = static_cast<E *>(m.p) + (i * m.ld + base - ref);
    o.s = VEC ? 0 : (int)(reinterpret_cast<uintptr_t>(o.p) & (Piece<E, PW>::kBytes - 1)) / (int)sizeof(E);
    return o;
  }
  template <typename E>
  __device__ __forceinline__ void write(Out<E> &o, int p, const float2 (&v)[kHalf]) const {
    constexpr int kW = Piece<E, PW>::kWords;
    uint32_t own[kW];
    words_of<E, PW>(v, own);
    E *to = o.p + p * kStep;
    if constexpr (VEC) {
      if (column(p) < n) write_block<kW>(to, own);
      return;
    }
    const int c = column(p), hi = n + ref;
    if (o.s == 0) {
      if ((p > 0 && p < full) || (c >= ref && c + PW <= hi)) write_block<kW>(to, own);
      else if (c < hi && c + PW > ref) write_singly<E, PW>(to, c, ref, hi, 0, SpanOf{false, false}, own);
      return;
    }
    // the block from s values before the piece on: the predecessor's are its neighbour's, or the first lane's
    // the last lane's of the piece before
    constexpr int kLanes = TPR ? TPR : 32;
    const int me = threadIdx.x & (kLanes - 1);
    uint32_t b[2 * kW + 1];
#pragma unroll
    for (int k = 0; k < kW; ++k) {
      const uint32_t send = me == kLanes - 1 && p > 0 ? o.last[k] : own[k];
      b[k] = __shfl_sync(lanes(), send, (threadIdx.x & ~(kLanes - 1)) | ((me + kLanes - 1) & (kLanes - 1)));
      b[k + kW] = own[k];
      o.last[k] = own[k];
    }
    b[2 * kW] = 0u;
    const int by = Piece<E, PW>::kBytes - o.s * (int)sizeof(E);
    if (kW == 4) {
#pragma unroll
      for (int k = 0; k < 6; ++k) b[k] = by & 8 ? b[k + 2] : b[k];
    }
#pragma unroll
    for (int k = 0; k < kW + 1; ++k) b[k] = by & 4 ? b[k + 1] : b[k];
    if (sizeof(E) == 2) {
#pragma unroll
      for (int k = 0; k < kW; ++k) b[k] = __funnelshift_r(b[k], b[k + 1], by & 2 ? 16 : 0);
    }
    if (p > 0 && p + 1 < full) {  // this block and its successor's are whole
      write_block<kW>(to - o.s, b);
      return;
    }
    const SpanOf w = span_of(PW, c, ref, hi, o.s, p > 0 || me > 0, p < kPieces - 1 || me < kLanes - 1);
    if (w.block) write_block<kW>(to - o.s, b);
    write_singly<E, PW>(to, c, ref, hi, o.s, w, own);
  }
  // zeros outside the row; of a piece before `full` only values before the row's first are
  __device__ __forceinline__ void clip(float2 (&v)[kHalf], int p) const {
    if (__builtin_expect(p >= full, 0)) {
      const int k = n + ref - column(p);
#pragma unroll
      for (int q = 0; q < kHalf; ++q) {
        if (2 * q >= k) v[q].x = 0.0f;
        if (2 * q + 1 >= k) v[q].y = 0.0f;
      }
    }
    if (!VEC && p == 0) {
      if (base < ref) {
#pragma unroll
        for (int q = 0; q < kHalf; ++q) {
          if (2 * q < ref) v[q].x = 0.0f;
          if (2 * q + 1 < ref) v[q].y = 0.0f;
        }
      }
    }
  }
};

// ------------------------------------------------------------ vectors
// As the rows need them, in fp32: scale post_weight, scale post_bias, weight, bias; those there are lie in
// shared memory one after the other.
struct Vectors {
  const float *at[4];
  // values j to j + 3 of a vector, `none` where it has none
  __device__ __forceinline__ static float4 four(const void *p, int j, int n, int dtype, float none) {
    float4 f = make_float4(none, none, none, none);
    if (!p) return f;
    const char *a = static_cast<const char *>(p) + (int64_t)j * (dtype == NR_F32 ? 4 : 2);
    const bool in = j >= 0 && j + 4 <= n;
    if (in && (reinterpret_cast<uintptr_t>(a) & 15) == 0 && dtype == NR_F32) return __ldg(reinterpret_cast<const float4 *>(a));
    if (in && (reinterpret_cast<uintptr_t>(a) & 7) == 0 && dtype != NR_F32) {
      const uint2 w = __ldg(reinterpret_cast<const uint2 *>(a));
      const float2 x = unpack2(w.x, dtype), y = unpack2(w.y, dtype);
      return make_float4(x.x, x.y, y.x, y.y);
    }
    if (j >= 0 && j < n) f.x = load_any(p, j, dtype);
    if (j + 1 >= 0 && j + 1 < n) f.y = load_any(p, j + 1, dtype);
    if (j + 2 >= 0 && j + 2 < n) f.z = load_any(p, j + 2, dtype);
    if (j + 3 >= 0 && j + 3 < n) f.w = load_any(p, j + 3, dtype);
    return f;
  }
  __device__ __forceinline__ static float4 times(float4 a, float4 b) { return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w); }
  // all threads of the block; a barrier follows
  __device__ __forceinline__ Vectors(const Block &B, const Ring &R, char *shared, int ref) {
    float *to = reinterpret_cast<float *>(shared + R.vectors);
    const int n = (int)B.n;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      at[k] = to;
      if (R.present >> k & 1) to += R.columns;
    }
    // columns outside the row hold zeros
    for (int c = 4 * (threadIdx.y * blockDim.x + threadIdx.x); c < R.columns; c += 4 * blockDim.x * blockDim.y) {
      const int j = c - ref;
      const float4 s = four(B.scale, j, n, B.w_dtype, 1.0f);
      float4 f[4] = {four(B.post_w, j, n, B.w_dtype, 1.0f), four(B.post_b, j, n, B.w_dtype, 0.0f), four(B.w, j, n, B.w_dtype, 1.0f),
                     four(B.b, j, n, B.w_dtype, 0.0f)};
      f[0] = times(f[0], s);
      f[1] = times(f[1], s);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (!(R.present >> k & 1)) continue;
        if (j < 0 || j >= n) f[k].x = 0.0f;
        if (j + 1 < 0 || j + 1 >= n) f[k].y = 0.0f;
        if (j + 2 < 0 || j + 2 >= n) f[k].z = 0.0f;
        if (j + 3 < 0 || j + 3 >= n) f[k].w = 0.0f;
        *reinterpret_cast<float4 *>(const_cast<float *>(at[k]) + c) = f[k];
      }
    }
  }
  // PW of vector k from column c on, zeros past the row
  template <int PW>
  __device__ __forceinline__ void piece(int k, int c, float2 (&v)[PW / 2]) const {
#pragma unroll
    for (int q = 0; q < PW / 4; ++q) {
      const float4 f = *reinterpret_cast<const float4 *>(at[k] + c + 4 * q);
      v[2 * q] = make_float2(f.x, f.y);
      v[2 * q + 1] = make_float2(f.z, f.w);
    }
  }
};

// ------------------------------------------------------------ sums over a row's threads
template <int TPR, int K>
__device__ __forceinline__ void lane_sums(float (&v)[K]) {
#pragma unroll
  for (int o = (TPR ? TPR : 32) / 2; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
}
// Where the warps of a row leave their sums; `turn` alternates between two of them, so that
// one barrier a sum is enough. A row's warps meet at a barrier of their own.
constexpr int kMostWarps = 32;
struct Sums {
  float4 v[2][kMostWarps];
};
template <int TPR>
struct Meeting {
  Sums *sums;
  int width, first, id, turn = 0;  // threads of the row, its first warp in the block, its barrier
  __device__ __forceinline__ bool alone() const { return TPR || width == 32; }
  __device__ __forceinline__ void barrier() const {
    if (alone()) __syncwarp();
    else asm volatile("bar.sync %0, %1;\n" ::"r"(id), "r"(width) : "memory");
  }
  // a warp's four values to all of the row's; then warp w's are part[first + w]
  __device__ __forceinline__ const float4 *share(float4 v) {
    float4 *part = sums->v[turn & 1] + first;
    ++turn;
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    barrier();
    return part;
  }
  template <int K>
  __device__ __forceinline__ void row_sums(float (&v)[K]) {
    lane_sums<TPR, K>(v);
    if (alone()) return;
    const float4 *part = share(make_float4(v[0], K > 1 ? v[K > 1 ? 1 : 0] : 0.0f, K > 2 ? v[K > 2 ? 2 : 0] : 0.0f, 0.0f));
    float4 s = part[0];
    for (int w = 1; w < width >> 5; ++w) {
      const float4 o = part[w];
      s.x += o.x, s.y += o.y, s.z += o.z;
    }
    v[0] = s.x;
    if (K > 1) v[K > 1 ? 1 : 0] = s.y;
    if (K > 2) v[K > 2 ? 2 : 0] = s.z;
  }
  // The mean and the sum of squared deviations of a row from those of its warps' parts: M2 = sum
  // M2_w + n_w (mean_w - mean)^2 (Chan, Golub, LeVeque), which loses nothing to cancellation.
  __device__ __forceinline__ void join(float &mean, float &m2, float n_warp, float inv) {
    const float4 *part = share(make_float4(mean, m2, n_warp, 0.0f));
    mean = 0.0f;
    for (int w = 0; w < width >> 5; ++w) mean = fmaf(part[w].x, part[w].z, mean);
    mean *= inv;
    m2 = 0.0f;
    for (int w = 0; w < width >> 5; ++w) {
      const float4 o = part[w];
      m2 += fmaf(o.z * (o.x - mean), o.x - mean, o.y);
    }
  }
};

// The stages of a group's rows. A row's stage takes the copies of the row `stages` turns later as
// soon as its values are in registers.
template <int TPR, bool VEC>
struct Turns {
  char *ring;
  int64_t first, stride;  // the group's rows
  int it = 0;
  template <typename Copy>
  __device__ __forceinline__ void begin(const Ring &R, const Copy &copy) const {
    for (int s = 0; s < R.stages; ++s) {
      copy(first + s * stride, ring + s * R.row_bytes);
      commit_copies();
    }
  }
  // the stage of the turn's row, once it is there
  __device__ __forceinline__ const char *next(const Ring &R, const Meeting<TPR> &M) const {
    wait_copies(R.stages - 1);
    if (!VEC) M.barrier();  // threads read what others have copied
    return ring + it * R.row_bytes;
  }
  // row i has been read
  template <typename Copy>
  __device__ __forceinline__ void release(const Ring &R, int64_t i, const Meeting<TPR> &M, const Copy &copy) {
    if (!VEC) M.barrier();
    copy(i + R.stages * stride, ring + it * R.row_bytes);
    commit_copies();
    it = it + 1 < R.stages ? it + 1 : 0;
  }
};

// Steps that a call may lack are loops over the thread's pieces of their own, so that a step
// costs one branch a row.
#define NR_PIECES(p) _Pragma("unroll") for (int p = 0; p < N; ++p)
#define NR_PAIRS(q) _Pragma("unroll") for (int q = 0; q < H; ++q)

// Blocks of blockDim.y rows' groups of blockDim.x threads (TPR: of blockDim.x / TPR).
template <int TPR, int V, int LIE, typename S, typename T>
__global__ void __launch_bounds__(TPR == 0 && V == 1 ? 1024 : V <= 2 ? 256 : 512, TPR == 0 && V == 1 || V > 2 ? 1 : 4)
    forward_kernel(const __grid_constant__ Block B, const __grid_constant__ Ring R) {
  constexpr int PW = sizeof(S) == 2 ? 8 : 4, H = PW / 2, N = 8 * V / PW;
  extern __shared__ uint4 shared_ring[];
  __shared__ Sums sums;
  char *shared = reinterpret_cast<char *>(shared_ring);
  constexpr bool VEC = LIE == kAligned;
  constexpr int kEvery = VEC ? 1 : PW;  // every which row a block takes
  const int phase = blockIdx.x % kEvery;
  const Place<TPR, V, PW, LIE> at((int)B.n, blockDim.x, R.s[0], sizeof(S), phase);
  const int groups = TPR ? blockDim.x / (TPR ? TPR : 1) : blockDim.y;
  const float inv = 1.0f / (float)(int)B.n, n_warp = (float)at.of_warp(), inv_warp = n_warp > 0.0f ? 1.0f / n_warp : 0.0f;
  const int64_t row0 = phase + (int64_t)(blockIdx.x / kEvery) * groups * kEvery;  // the block's first
  Turns<TPR, VEC> turns{shared + at.group * R.stages * R.row_bytes, row0 + at.group * kEvery, (int64_t)(gridDim.x / kEvery) * groups * kEvery};
  Meeting<TPR> meet{&sums, at.width, TPR ? 0 : at.group * (at.width >> 5), at.group + 1};
  const bool gate = B.gate == 2, u = B.u.p != nullptr;
  const auto copy = [&](int64_t i, char *stage) {
    if (i >= B.m) return;
    at.template copy<S>(R.s[0], stage, i);
    if (u) at.template copy<T>(R.s[1], stage, i);
    if (gate) at.template copy<T>(R.s[2], stage, i);
  };
  turns.begin(R, copy);
  const Vectors X(B, R, shared, at.ref);
  __syncthreads();
  float q_next = 0.0f;  // the next row's gate, if it has one
  if (B.gate == 1 && turns.first < B.m) q_next = load_any(B.q.p, turns.first * B.q.ld, B.dtype);
  // a block's groups take the same number of turns, so that shuffles are complete
  for (int64_t i0 = row0; i0 < B.m; i0 += turns.stride) {
    const int64_t i = i0 + at.group * kEvery;
    const bool in = i < B.m;
    const char *row = turns.next(R, meet);
    float2 y[N][H];
    const float q_row = q_next;
    if (B.gate == 1 && i + turns.stride < B.m) q_next = load_any(B.q.p, (i + turns.stride) * B.q.ld, B.dtype);
    // the mean (layer) and reciprocal deviation of the row in y, which becomes its deviations from the mean
    const auto statistics = [&](int kind, float &mean, float &rstd) {
      float2 s = both(0.0f);
      float v[1];
      if (kind == NR_NORM_LAYER) {
        NR_PIECES(p) NR_PAIRS(q) s = add2(s, y[p][q]);
        v[0] = s.x + s.y;
        lane_sums<TPR, 1>(v);
        mean = v[0] * (meet.alone() ? inv : inv_warp);
        s = both(0.0f);
        NR_PIECES(p) {
          NR_PAIRS(q) y[p][q] = add2(y[p][q], both(-mean));
          at.clip(y[p], p);
        }
        NR_PIECES(p) NR_PAIRS(q) s = fma2(y[p][q], y[p][q], s);
        v[0] = s.x + s.y;
        lane_sums<TPR, 1>(v);
        if (!meet.alone()) {
          const float own = mean;
          meet.join(mean, v[0], n_warp, inv);
          NR_PIECES(p) {
            NR_PAIRS(q) y[p][q] = add2(y[p][q], both(own - mean));
            at.clip(y[p], p);
          }
        }
      } else {
        NR_PIECES(p) NR_PAIRS(q) s = fma2(y[p][q], y[p][q], s);
        v[0] = s.x + s.y;
        meet.template row_sums<1>(v);
      }
      rstd = 1.0f / sqrtf(fmaf(v[0], inv, B.eps));
    };
    float um = 0.0f, ur = 1.0f, ym = 0.0f, yr = 1.0f;
    const auto rr = at.template in<S>(R.s[0], row, i);
    if (u) {
      const auto ru = at.template in<T>(R.s[1], row, i);
      NR_PIECES(p) {
        at.template read<T>(ru, p, y[p]);
        at.clip(y[p], p);
      }
      if (B.post != NR_NORM_NONE) {
        statistics(B.post, um, ur);
        NR_PIECES(p) NR_PAIRS(q) y[p][q] = mul2(y[p][q], both(ur));
      }
      if (R.present & 1) NR_PIECES(p) {
          float2 f[H];
          X.template piece<PW>(0, at.column(p), f);
          NR_PAIRS(q) y[p][q] = mul2(y[p][q], f[q]);
        }
      if (R.present & 2) NR_PIECES(p) {
          float2 f[H];
          X.template piece<PW>(1, at.column(p), f);
          NR_PAIRS(q) y[p][q] = add2(y[p][q], f[q]);
        }
      if (gate) {
        const auto rq = at.template in<T>(R.s[2], row, i);
        if (B.act == NR_ACT_SILU) NR_PIECES(p) {
            float2 f[H];
            at.template read<T>(rq, p, f);
            NR_PAIRS(q) y[p][q] = mul2(y[p][q], silu2(f[q], logistic2(f[q])));
          }
        else NR_PIECES(p) {
            float2 f[H];
            at.template read<T>(rq, p, f);
            NR_PAIRS(q) y[p][q] = mul2(y[p][q], logistic2(f[q]));
          }
      } else if (B.gate == 1) {
        const float a = gate_value(q_row, B.act);
        NR_PIECES(p) NR_PAIRS(q) y[p][q] = mul2(y[p][q], both(a));
      }
      auto to = at.template out<S>(B.y, i);
      NR_PIECES(p) {
        float2 f[H];
        at.template read<S>(rr, p, f);
        NR_PAIRS(q) y[p][q] = fma2(f[q], both(B.alpha), y[p][q]);
        at.clip(y[p], p);
        if (in) at.template write<S>(to, p, y[p]);
      }
    } else {
      NR_PIECES(p) {
        at.template read<S>(rr, p, y[p]);
        at.clip(y[p], p);
      }
    }
    turns.release(R, i, meet, copy);
    if (B.pre != NR_NORM_NONE) {
      statistics(B.pre, ym, yr);
      NR_PIECES(p) NR_PAIRS(q) y[p][q] = mul2(y[p][q], both(yr));
      if (R.present & 4) NR_PIECES(p) {
          float2 f[H];
          X.template piece<PW>(2, at.column(p), f);
          NR_PAIRS(q) y[p][q] = mul2(y[p][q], f[q]);
        }
      if (R.present & 8) NR_PIECES(p) {
          float2 f[H];
          X.template piece<PW>(3, at.column(p), f);
          NR_PAIRS(q) y[p][q] = add2(y[p][q], f[q]);
        }
      auto to = at.template out<T>(B.h, i);
      if (in) NR_PIECES(p) at.template write<T>(to, p, y[p]);
    }
    if (in && at.t == 0) {
      if (B.u_mean) B.u_mean[i] = um;
      if (B.u_rstd) B.u_rstd[i] = ur;
      if (B.y_mean) B.y_mean[i] = ym;
      if (B.y_rstd) B.y_rstd[i] = yr;
    }
  }
}

// The statistics and gate of a row, loaded a turn ahead
struct Row {
  float um, ur, ym, yr, q;
  __device__ __forceinline__ Row(const Block &B, int64_t i) {
    const bool in = i < B.m;
    um = in && B.u_mean ? B.u_mean[i] : 0.0f;
    ur = in && B.u_rstd ? B.u_rstd[i] : 1.0f;
    ym = in && B.y_mean ? B.y_mean[i] : 0.0f;
    yr = in && B.y_rstd ? B.y_rstd[i] : 1.0f;
    q = in && B.gate == 1 ? load_any(B.q.p, i * B.q.ld, B.dtype) : 0.0f;
  }
};

// BIAS: the sums of dh and of t a are wanted too
template <int TPR, int V, int LIE, bool BIAS, int THREADS, typename S, typename T>
__global__ void __launch_bounds__(THREADS, V == 1 ? 2 : 1)
    backward_kernel(const __grid_constant__ Block B, const __grid_constant__ Ring R) {
  constexpr int PW = sizeof(S) == 2 ? 8 : 4, H = PW / 2, N = 8 * V / PW, NB = BIAS ? N : 1;
  extern __shared__ uint4 shared_ring[];
  __shared__ Sums sums;
  char *shared = reinterpret_cast<char *>(shared_ring);
  constexpr bool VEC = LIE == kAligned;
  constexpr int kEvery = VEC ? 1 : PW;  // every which row a block takes
  const int phase = blockIdx.x % kEvery;
  // the first matrix read, which there always is: y with a norm before the next block, else dy
  const Place<TPR, V, PW, LIE> at((int)B.n, blockDim.x, B.pre != NR_NORM_NONE ? R.s[1] : R.s[2], sizeof(S), phase);
  const int groups = TPR ? blockDim.x / (TPR ? TPR : 1) : blockDim.y;
  const float inv = 1.0f / (float)(int)B.n;
  const int64_t row0 = phase + (int64_t)(blockIdx.x / kEvery) * groups * kEvery;  // the block's first
  Turns<TPR, VEC> turns{shared + at.group * R.stages * R.row_bytes, row0 + at.group * kEvery, (int64_t)(gridDim.x / kEvery) * groups * kEvery};
  Meeting<TPR> meet{&sums, at.width, TPR ? 0 : at.group * (at.width >> 5), at.group + 1};
  const bool gate = B.gate == 2, u = B.u.p != nullptr, pre = B.pre != NR_NORM_NONE, dy = B.dy.p != nullptr;
  const auto copy = [&](int64_t i, char *stage) {
    if (i >= B.m) return;
    if (pre) {
      at.template copy<T>(R.s[0], stage, i);
      at.template copy<S>(R.s[1], stage, i);
    }
    if (dy) at.template copy<S>(R.s[2], stage, i);
    if (u) at.template copy<T>(R.s[3], stage, i);
    if (gate) at.template copy<T>(R.s[4], stage, i);
  };
  turns.begin(R, copy);
  const Vectors X(B, R, shared, at.ref);
  __syncthreads();
  float2 sw[N][H], sA[N][H], sb[NB][H], sB[NB][H];  // the columns' sums: dh yh, t a uh, dh, t a
  NR_PIECES(p) NR_PAIRS(q) {
    sw[p][q] = sA[p][q] = both(0.0f);
    if (BIAS) sb[BIAS ? p : 0][q] = sB[BIAS ? p : 0][q] = both(0.0f);
  }
  Row ahead(B, turns.first);
  for (int64_t i0 = row0; i0 < B.m; i0 += turns.stride) {
    const int64_t i = i0 + at.group * kEvery;
    const bool in = i < B.m;
    const char *row = turns.next(R, meet);
    const Row now = ahead;
    ahead = Row(B, i + turns.stride);
    float2 t[N][H], b[N][H];  // g and yh, then t, then e and uh
    if (pre) {
      const auto rh = at.template in<T>(R.s[0], row, i);
      const auto ry = at.template in<S>(R.s[1], row, i);
      NR_PIECES(p) {
        at.template read<T>(rh, p, t[p]);
        at.clip(t[p], p);
        at.template read<S>(ry, p, b[p]);
        NR_PAIRS(q) b[p][q] = mul2(add2(b[p][q], both(-now.ym)), both(now.yr));
        at.clip(b[p], p);
      }
      if (in) {  // groups behind the last row hold what lies in their stage
        NR_PIECES(p) NR_PAIRS(q) sw[p][q] = fma2(t[p][q], b[p][q], sw[p][q]);
        if (BIAS) NR_PIECES(p) NR_PAIRS(q) sb[BIAS ? p : 0][q] = add2(sb[BIAS ? p : 0][q], t[p][q]);
      }
      if (R.present & 4) NR_PIECES(p) {
          float2 f[H];
          X.template piece<PW>(2, at.column(p), f);
          NR_PAIRS(q) t[p][q] = mul2(t[p][q], f[q]);
        }
      float2 s1 = both(0.0f), s2 = both(0.0f);
      NR_PIECES(p) NR_PAIRS(q) s2 = fma2(t[p][q], b[p][q], s2);
      if (B.pre == NR_NORM_LAYER) {
        NR_PIECES(p) NR_PAIRS(q) s1 = add2(s1, t[p][q]);
        float v[2] = {s2.x + s2.y, s1.x + s1.y};
        meet.template row_sums<2>(v);
        const float m1 = v[1] * inv * now.yr, m2 = v[0] * inv * now.yr;
        NR_PIECES(p) NR_PAIRS(q) t[p][q] = fma2(b[p][q], both(-m2), fma2(t[p][q], both(now.yr), both(-m1)));
      } else {
        float v[1] = {s2.x + s2.y};
        meet.template row_sums<1>(v);
        const float m2 = v[0] * inv * now.yr;
        NR_PIECES(p) NR_PAIRS(q) t[p][q] = fma2(b[p][q], both(-m2), mul2(t[p][q], both(now.yr)));
      }
    } else {
      NR_PIECES(p) NR_PAIRS(q) t[p][q] = both(0.0f);
    }
    if (dy) {
      const auto rd = at.template in<S>(R.s[2], row, i);
      NR_PIECES(p) {
        float2 o[H];
        at.template read<S>(rd, p, o);
        NR_PAIRS(q) t[p][q] = add2(t[p][q], o[q]);
      }
    }
    if (in) {
      auto to = at.template out<S>(B.dr, i);
      if (B.alpha == 1.0f) NR_PIECES(p) at.template write<S>(to, p, t[p]);
      else NR_PIECES(p) {
          float2 o[H];
          NR_PAIRS(q) o[q] = mul2(t[p][q], both(B.alpha));
          at.template write<S>(to, p, o);
        }
    }
    if (!u) {
      turns.release(R, i, meet, copy);
      continue;
    }
    const auto ru = at.template in<T>(R.s[3], row, i);
    NR_PIECES(p) {
      at.clip(t[p], p);
      at.template read<T>(ru, p, b[p]);
    }
    if (B.post != NR_NORM_NONE) NR_PIECES(p) NR_PAIRS(q) b[p][q] = mul2(add2(b[p][q], both(-now.um)), both(now.ur));
    NR_PIECES(p) at.clip(b[p], p);
    float2 s1 = both(0.0f), s2 = both(0.0f), s3 = both(0.0f);
    if (B.gate) {  // dq = t scale c a'(q), and t becomes t a(q)
      const auto rq = gate ? at.template in<T>(R.s[4], row, i) : at.template in<T>(R.s[3], row, i);
      const float a_row = B.gate == 1 ? gate_value(now.q, B.act) : 1.0f;
      auto to = at.template out<T>(B.dq, i);
      NR_PIECES(p) {
        float2 c[H], f[H];
        if (R.present & 1) {
          X.template piece<PW>(0, at.column(p), f);
          NR_PAIRS(q) c[q] = mul2(b[p][q], f[q]);
        } else {
          NR_PAIRS(q) c[q] = b[p][q];
        }
        if (R.present & 2) {
          X.template piece<PW>(1, at.column(p), f);
          NR_PAIRS(q) c[q] = add2(c[q], f[q]);
        }
        NR_PAIRS(q) c[q] = mul2(c[q], t[p][q]);
        if (gate) {
          at.template read<T>(rq, p, f);
          at.clip(f, p);
          if (B.act == NR_ACT_SILU) {
            NR_PAIRS(q) {
              const float2 a = logistic2(f[q]);
              c[q] = mul2(c[q], silu_slope2(f[q], a));
              t[p][q] = mul2(t[p][q], silu2(f[q], a));
            }
          } else {
            NR_PAIRS(q) {
              const float2 a = logistic2(f[q]);
              c[q] = mul2(c[q], mul2(a, fma2(a, both(-1.0f), both(1.0f))));
              t[p][q] = mul2(t[p][q], a);
            }
          }
          if (in) at.template write<T>(to, p, c);
        } else {
          NR_PAIRS(q) {
            s3 = add2(s3, c[q]);
            t[p][q] = mul2(t[p][q], both(a_row));
          }
        }
      }
    }
    turns.release(R, i, meet, copy);
    if (in) {
      NR_PIECES(p) NR_PAIRS(q) sA[p][q] = fma2(t[p][q], b[p][q], sA[p][q]);
      if (BIAS) NR_PIECES(p) NR_PAIRS(q) sB[BIAS ? p : 0][q] = add2(sB[BIAS ? p : 0][q], t[p][q]);
    }
    if (R.present & 1) NR_PIECES(p) {
        float2 f[H];
        X.template piece<PW>(0, at.column(p), f);
        NR_PAIRS(q) t[p][q] = mul2(t[p][q], f[q]);
      }
    if (B.post != NR_NORM_NONE || B.gate == 1) {
      NR_PIECES(p) NR_PAIRS(q) {
        s1 = add2(s1, t[p][q]);
        s2 = fma2(t[p][q], b[p][q], s2);
      }
      float v[3] = {s1.x + s1.y, s2.x + s2.y, s3.x + s3.y};
      meet.template row_sums<3>(v);
      if (in && B.gate == 1 && at.t == 0) static_cast<T *>(B.dq.p)[i * B.dq.ld] = from_f32<T>(v[2] * gate_slope(now.q, B.act));
      if (B.post != NR_NORM_NONE) {
        const float e1 = B.post == NR_NORM_LAYER ? v[0] * inv * now.ur : 0.0f, e2 = v[1] * inv * now.ur;
        NR_PIECES(p) NR_PAIRS(q) t[p][q] = fma2(b[p][q], both(-e2), fma2(t[p][q], both(now.ur), both(-e1)));
      }
    }
    if (in) {
      auto to = at.template out<T>(B.du, i);
      NR_PIECES(p) at.template write<T>(to, p, t[p]);
    }
  }
  wait_copies<0>();
  grid_launch();
  if (!B.parts) return;
  // the block's sums: its groups' side by side in shared memory, then added in order
  constexpr int K = BIAS ? 4 : 2;  // dh yh, t a uh, dh, t a
  float *mine = reinterpret_cast<float *>(shared_ring) + (int64_t)at.group * K * at.n;
  const auto part = [&](int k) { return B.parts + ((int64_t)(k == 0 ? 0 : k == 1 ? 2 : k == 2 ? 1 : 3) * gridDim.x + blockIdx.x) * B.n; };
  __syncthreads();
  const auto put = [&](const float2 &f, int k, int c) {
    float *to = groups > 1 ? mine + k * at.n : part(k);
    if (c >= 0 && c < at.n) to[c] = f.x;
    if (c + 1 >= 0 && c + 1 < at.n) to[c + 1] = f.y;
  };
  NR_PIECES(p) NR_PAIRS(q) {
    const int c = at.column(p) - at.ref + 2 * q;
    put(sw[p][q], 0, c);
    put(sA[p][q], 1, c);
    if (BIAS) {
      put(sb[BIAS ? p : 0][q], 2, c);
      put(sB[BIAS ? p : 0][q], 3, c);
    }
  }
  if (groups == 1) return;
  __syncthreads();
  const float *all = reinterpret_cast<const float *>(shared_ring);
  for (int k = 0; k < K; ++k)
    for (int c = threadIdx.y * blockDim.x + threadIdx.x; c < at.n; c += blockDim.x * blockDim.y) {
      float sum = all[k * at.n + c];
      for (int g = 1; g < groups; ++g) sum += all[(g * K + k) * at.n + c];
      part(k)[c] = sum;
    }
}
#undef NR_PIECES
#undef NR_PAIRS

// ------------------------------------------------------------ launches
// How rows are taken: tpr lanes, or x threads (tpr 0) with v eights each, y rows' groups a block. x 0: not here.
struct Plan {
  int tpr, v, x, y, lie, bias, blocks, bytes;
  Ring ring;
};

typedef void (*Kernel)(Block, Ring);
template <typename S, typename T>
Kernel forward_of(const Plan &P);
template <typename S, typename T>
Kernel backward_of(const Plan &P);

#define NR_BLOCKNORM_KERNELS(S, T)                                                                       \
  template <int LIE>                                                                                     \
  static Kernel forward_##S##_##T(const Plan &P) {                                                       \
    if (P.tpr == 8) return forward_kernel<8, 1, LIE, S, T>;                                              \
    if (P.tpr == 16) return forward_kernel<16, 1, LIE, S, T>;                                            \
    if (P.tpr == 32) {                                                                                   \
      return P.v == 1   ? forward_kernel<32, 1, LIE, S, T>                                               \
             : P.v == 2 ? forward_kernel<32, 2, LIE, S, T>                                               \
             : P.v == 3 ? forward_kernel<32, 3, LIE, S, T>                                               \
             : P.v == 4 ? forward_kernel<32, 4, LIE, S, T>                                               \
                        : forward_kernel<32, 6, LIE, S, T>;                                              \
    }                                                                                                    \
    return P.v == 1   ? forward_kernel<0, 1, LIE, S, T>                                                  \
           : P.v == 3 ? forward_kernel<0, 3, LIE, S, T>                                                  \
                      : forward_kernel<0, 4, LIE, S, T>;                                                 \
  }                                                                                                      \
  template <int LIE, bool BIAS>                                                                          \
  static Kernel backward_##S##_##T(const Plan &P) {                                                      \
    if (P.tpr == 8) return backward_kernel<8, 1, LIE, BIAS, 256, S, T>;                                  \
    if (P.tpr == 16) return backward_kernel<16, 1, LIE, BIAS, 256, S, T>;                                \
    if (P.tpr == 32) return P.v == 1 ? backward_kernel<32, 1, LIE, BIAS, 256, S, T> : backward_kernel<32, 2, LIE, BIAS, 384, S, T>; \
    if constexpr (BIAS) { if (P.x > 384) return backward_kernel<0, 2, LIE, true, 512, S, T>; }           \
    return backward_kernel<0, BIAS ? 2 : 3, LIE, BIAS, 384, S, T>;                                       \
  }                                                                                                      \
  template <>                                                                                            \
  Kernel forward_of<S, T>(const Plan &P) {                                                               \
    return P.lie == kAligned ? forward_##S##_##T<kAligned>(P)                                            \
           : P.lie == kAlike ? forward_##S##_##T<kAlike>(P)                                              \
                             : forward_##S##_##T<kAny>(P);                                               \
  }                                                                                                      \
  template <>                                                                                            \
  Kernel backward_of<S, T>(const Plan &P) {                                                              \
    if (P.bias)                                                                                          \
      return P.lie == kAligned ? backward_##S##_##T<kAligned, true>(P)                                   \
             : P.lie == kAlike ? backward_##S##_##T<kAlike, true>(P)                                     \
                               : backward_##S##_##T<kAny, true>(P);                                      \
    return P.lie == kAligned ? backward_##S##_##T<kAligned, false>(P)                                    \
           : P.lie == kAlike ? backward_##S##_##T<kAlike, false>(P)                                      \
                             : backward_##S##_##T<kAny, false>(P);                                       \
  }

}  // namespace blocknorm
