// The linear layer of residual encoders (neuroute_ops.h):
//   forward   z = x w^T + bias, y = act(z) + residual
//   backward  dz = dy act'(z); dx = dz w, dw = dz^T x, dbias = sum of dz's rows
//
// Every product is one launch of product_kernel, C[i, j] = sum_t A[i, t] B[j, t]
// on tcgen05 with fp32 sums in tensor memory; A and B lie in memory either with t
// contiguous (x and w forward; dz for dx) or with their own index contiguous
// (w for dx; dz and x for dw), which the tensor maps and the operands'
// descriptors tell apart, so nothing is transposed.
//
// product_kernel is persistent and warp-specialised. A work item is a tile of C
// (128 rows a CTA, up to 256 columns) and a range of t, walked 64 values of t at
// a time through a ring of shared-memory stages:
//   producer  one thread: tensor copies of A's and B's slices, 128-byte swizzle,
//             zeros past the operands' ends
//   MMA       one thread: four MMAs of 16 values of t a stage into one of two
//             accumulators, so that the next item starts under the epilogue
//   epilogue  eight warps: accumulator -> registers -> 32 x 32 fp32 blocks in
//             shared memory, read back eight columns a thread with a row's
//             threads side by side, so that the global accesses of bias,
//             residual, z and y run along rows
// A pair of CTAs on two SMs (CG = 2) shares a tile of 256 rows: each holds its
// rows of A and half of B's columns, the first issues the MMAs for both, and a
// B slice is read once for 256 rows. Few tiles with a long t are split along t;
// the parts' sums go to scratch and finish_kernel adds them in order.
// Every wait is bounded: one that expires stops all roles of its CTA, which
// lets copies in flight land, frees its tensor memory and sets the flag that
// nr_ops_status reports.
//
// Up to eight rows run on CUDA cores instead (rows_kernel): the weights are
// read once, which is all the time such a call can take.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include "nrq_ops.cuh"
#include "nrq_tc.cuh"

namespace {

// ------------------------------------------------------------ epilogue
// What becomes of the sums s[i, j]: z = s + bias, y = act(z) + residual.
struct Epilogue {
  const void *bias;
  int bias_dtype, act;
  const void *residual;  // of type dtype
  int64_t residual_ld;
  void *y;
  int64_t y_ld;
  void *z;  // of type dtype, or int8 codes
  int64_t z_ld;
  uint8_t *z_scale;
  int64_t n;
  int dtype, y_dtype;
  int y_vec, z_vec, residual_vec, bias_vec;  // eight columns a 16-byte access (32 bytes in fp32)
};

// z of eight columns in 8 bits: the four threads of a group of 32 columns together
// (lanes 4 a .. 4 a + 3 of a warp, in column order); count: columns there
__device__ __forceinline__ void hold8(const Epilogue &E, int64_t i, int j, bool row_ok, int count, const float2 (&v)[4]) {
  float2 u[4];
  uint32_t top = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    u[q] = make_float2(2 * q < count ? v[q].x : 0.0f, 2 * q + 1 < count ? v[q].y : 0.0f);
    top = max(top, max(__float_as_uint(u[q].x) & 0x7fffffffu, __float_as_uint(u[q].y) & 0x7fffffffu));
  }
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const uint32_t sc = held8_scale(top);
  const float up = held8_up(sc);
  const int groups = ((int)E.n + kOpsGroup - 1) / kOpsGroup;
  if (row_ok && j < groups * kOpsGroup) {
    *reinterpret_cast<uint2 *>(static_cast<int8_t *>(E.z) + i * groups * kOpsGroup + j) =
        make_uint2(held8_codes(u[0], u[1], up, sc), held8_codes(u[2], u[3], up, sc));
    if ((j & (kOpsGroup - 1)) == 0) E.z_scale[i * groups + (j >> 5)] = (uint8_t)sc;
  }
}
__device__ __forceinline__ void add_raw(float2 (&v)[4], const uint4 &r, int dtype) {
  v[0] = add2(v[0], unpack2(r.x, dtype)), v[1] = add2(v[1], unpack2(r.y, dtype));
  v[2] = add2(v[2], unpack2(r.z, dtype)), v[3] = add2(v[3], unpack2(r.w, dtype));
}
__device__ __forceinline__ uint4 pack8(const float2 (&v)[4], int dtype) {
  return make_uint4(pack2(v[0].x, v[0].y, dtype), pack2(v[1].x, v[1].y, dtype), pack2(v[2].x, v[2].y, dtype),
                    pack2(v[3].x, v[3].y, dtype));
}

// Finishes s[i, j .. j + 7] (j a multiple of 8; bias: those columns'), row_ok
// false for rows past the end; called as hold8 is.
__device__ __forceinline__ void finish8(const Epilogue &E, int64_t i, int j, bool row_ok, float2 (&v)[4],
                                        const float2 (&bias)[4]) {
  const int count = row_ok ? min(8, (int)E.n - j) : 0;  // may be negative
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = add2(v[q], bias[q]);
  if (E.z) {
    if (E.z_scale) {
      hold8(E, i, j, row_ok, count, v);
    } else if (count > 0) {
      const float o[8] = {v[0].x, v[0].y, v[1].x, v[1].y, v[2].x, v[2].y, v[3].x, v[3].y};
      store8(E.z, i * E.z_ld + j, E.dtype, E.z_vec, count, o);
    }
  }
  if (count <= 0) return;
  if (E.act != NR_ACT_NONE) {
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = act_value2(v[q], E.act);
  }
  if (E.residual) {
    float r[8];
    load8(E.residual, i * E.residual_ld + j, E.dtype, E.residual_vec, count, r);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = add2(v[q], make_float2(r[2 * q], r[2 * q + 1]));
  }
  const float o[8] = {v[0].x, v[0].y, v[1].x, v[1].y, v[2].x, v[2].y, v[3].x, v[3].y};
  store8(E.y, i * E.y_ld + j, E.y_dtype, E.y_vec, count, o);
}

__device__ __forceinline__ void bias8(const Epilogue &E, int j, float2 (&b)[4]) {
  if (E.bias && E.bias_vec && j + 8 <= (int)E.n) {
    float o[8];
    load8(E.bias, j, E.bias_dtype, 1, 8, o);
#pragma unroll
    for (int q = 0; q < 4; ++q) b[q] = make_float2(o[2 * q], o[2 * q + 1]);
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    b[q].x = E.bias && j + 2 * q < (int)E.n ? load_any(E.bias, j + 2 * q, E.bias_dtype) : 0.0f;
    b[q].y = E.bias && j + 2 * q + 1 < (int)E.n ? load_any(E.bias, j + 2 * q + 1, E.bias_dtype) : 0.0f;
  }
}

// A warp's 32 x 32 block of sums: from tensor memory (a thread a row) through
// shared memory to eight columns of four rows a thread, so that the global
// accesses run along rows. 16-byte piece q of row r lies at piece q ^ (r % 8): both
// the rows' threads and the eight columns' touch all banks.
__device__ __forceinline__ void stage_write(float *stage, int lane, const uint32_t (&v)[32]) {
#pragma unroll
  for (int q = 0; q < 8; ++q)
    *reinterpret_cast<uint4 *>(stage + lane * 32 + ((q ^ (lane & 7)) << 2)) =
        make_uint4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
}
__device__ __forceinline__ void stage_read(const float *stage, int lane, int u, float2 (&v)[4]) {
  const int seg = lane & 3, r8 = lane >> 2;
  const float4 lo = *reinterpret_cast<const float4 *>(stage + (u * 8 + r8) * 32 + (((2 * seg) ^ r8) << 2));
  const float4 hi = *reinterpret_cast<const float4 *>(stage + (u * 8 + r8) * 32 + (((2 * seg + 1) ^ r8) << 2));
  v[0] = make_float2(lo.x, lo.y), v[1] = make_float2(lo.z, lo.w);
  v[2] = make_float2(hi.x, hi.y), v[3] = make_float2(hi.z, hi.w);
}

// A whole block (32 rows and columns there, every matrix in vectors, y 16-bit) from
// row i, column j of the thread's eight: no bounds, one test a step for all rows.
__device__ __forceinline__ void finish_block(const Epilogue &E, int64_t i, int j, const float *stage, int lane,
                                             const float2 (&b)[4], const uint4 (&res)[4]) {
  float2 v[4][4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    stage_read(stage, lane, u, v[u]);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[u][q] = add2(v[u][q], b[q]);
  }
  if (E.z) {
    if (E.z_scale) {
#pragma unroll
      for (int u = 0; u < 4; ++u) hold8(E, i + 8 * u, j, true, 8, v[u]);
    } else {
      uint16_t *z = static_cast<uint16_t *>(E.z) + i * E.z_ld + j;
#pragma unroll
      for (int u = 0; u < 4; ++u) *reinterpret_cast<uint4 *>(z + 8 * u * E.z_ld) = pack8(v[u], E.dtype);
    }
  }
#define NR_BLOCK_ACT(A)                                  \
  _Pragma("unroll") for (int u = 0; u < 4; ++u)          \
  _Pragma("unroll") for (int q = 0; q < 4; ++q) v[u][q] = act_value2(v[u][q], A);
  if (E.act == NR_ACT_GELU) {
    NR_BLOCK_ACT(NR_ACT_GELU)
  } else if (E.act == NR_ACT_SILU) {
    NR_BLOCK_ACT(NR_ACT_SILU)
  } else if (E.act == NR_ACT_RELU) {
    NR_BLOCK_ACT(NR_ACT_RELU)
  }
#undef NR_BLOCK_ACT
  if (E.residual) {
#pragma unroll
    for (int u = 0; u < 4; ++u) add_raw(v[u], res[u], E.dtype);
  }
  uint16_t *y = static_cast<uint16_t *>(E.y) + i * E.y_ld + j;
#pragma unroll
  for (int u = 0; u < 4; ++u) *reinterpret_cast<uint4 *>(y + 8 * u * E.y_ld) = pack8(v[u], E.dtype);
}

// ------------------------------------------------------------ products on tensor cores
constexpr int kRows = 128;            // rows of C a CTA
constexpr int kSlice = 64;            // values of t a stage: 128 bytes
constexpr int kEpiWarps = 8;
constexpr int kWarpProd = 0, kWarpMma = 1, kWarpEpi = 2;
constexpr int kThreads = 32 * (kWarpEpi + kEpiWarps);
constexpr int kStagesMax = 8;
constexpr uint32_t kABytes = kRows * kSlice * 2;
constexpr uint32_t kStaging = 32 * 32 * 4;  // a warp's 32 x 32 block of sums
constexpr int64_t kWaitNs = 1000000000;

struct Bars {
  uint64_t full[kStagesMax], empty[kStagesMax], accfull[2], accempty[2], drain;
  uint32_t tmem_slot;
  int abort;
};

struct Product {
  int64_t rows;          // of C
  int tiles_m, tiles_n;  // tiles of 128 CG rows, of nt columns
  int nt, stages;
  int slices, splits;    // of 64 values of t; parts of them
  int a_outer, b_outer;  // the operand's own index is the contiguous one
  uint32_t idesc;
  int partial;           // part s's sums go to y + s rows y_ld, nothing else
  int64_t wait_ns;
};

// an item's tile and part. Tiles run down bands of 8 tile rows, so that the
// tiles in flight share their slices of A and B in L2.
__device__ __forceinline__ void item_of(const Product &P, int item, int &tm, int &tn, int &part) {
  const int tiles = P.tiles_m * P.tiles_n;
  part = item / tiles;
  const int t = item - part * tiles;
  constexpr int kBand = 8;
  const int band = t / (kBand * P.tiles_n), in = t - band * kBand * P.tiles_n;
  const int height = min(kBand, P.tiles_m - band * kBand);
  tn = in / height;
  tm = band * kBand + in - tn * height;
}

template <int CG>
__global__ void __cluster_dims__(CG, 1, 1) __launch_bounds__(kThreads, 1)
    product_kernel(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mb, const Product P,
                   const Epilogue E, int *flag) {
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char *smem = smem_raw + (base - tc::smem_u32(smem_raw));
  const int nb = P.nt / CG;  // rows of B this CTA holds
  const uint32_t stage_bytes = kABytes + (uint32_t)nb * kSlice * 2;
  const uint32_t o_staging = (uint32_t)P.stages * stage_bytes, o_bars = o_staging + kEpiWarps * kStaging;
  Bars &B = *reinterpret_cast<Bars *>(smem + o_bars);
  volatile int *abort = &B.abort;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = CG == 2 ? tc::cluster_rank() : 0u;
  const int items = P.tiles_m * P.tiles_n * P.splits, first = blockIdx.x / CG, step = gridDim.x / CG;
  uint32_t cols = 32;
  while (cols < 2u * (uint32_t)P.nt) cols <<= 1;

  if (warp == kWarpMma) tc::alloc<CG>(tc::smem_u32(&B.tmem_slot), cols);
  if (tid == 0) {
    for (int i = 0; i < P.stages; ++i) {
      tc::bar_init(tc::smem_u32(&B.full[i]), 1);
      tc::bar_init(tc::smem_u32(&B.empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::bar_init(tc::smem_u32(&B.accfull[i]), 1);
      tc::bar_init(tc::smem_u32(&B.accempty[i]), CG * kEpiWarps);
    }
    tc::bar_init(tc::smem_u32(&B.drain), 1);
    B.abort = 0;
    tc::fence_bar_init();
  }
  tc::fence_before();
  __syncthreads();
  if (CG == 2) tc::cluster_sync();
  tc::fence_after();
  const uint32_t tmem = B.tmem_slot;
  const uint32_t nstages = (uint32_t)P.stages;

  if (warp == kWarpProd) {
    if (lane == 0) {
      uint32_t st = 0, phase = 1;  // the stage's wait parity: free at first
      bool ok = true;
      for (int item = first; item < items && ok; item += step) {
        int tm, tn, part;
        item_of(P, item, tm, tn, part);
        const int i0 = (tm * CG + (int)rank) * kRows, j0 = tn * P.nt + (int)rank * nb;
        const int s0 = (int)((int64_t)P.slices * part / P.splits), s1 = (int)((int64_t)P.slices * (part + 1) / P.splits);
        for (int s = s0; s < s1; ++s) {
          if (!tc::bar_wait(tc::smem_u32(&B.empty[st]), phase, abort, P.wait_ns)) {
            ok = false;
            break;
          }
          // the pair's bytes are counted on the first CTA's barrier
          uint32_t bar = tc::smem_u32(&B.full[st]);
          if (rank == 0) tc::bar_expect(bar, CG * stage_bytes);
          if (CG == 2) bar = tc::map_rank(bar, 0);
          const uint32_t sa = base + st * stage_bytes, sb = sa + kABytes;
          const int t0 = s * kSlice;
          if (P.a_outer) {
            for (int q = 0; q < kRows / 64; ++q) tc::load_2d<CG>(sa + (uint32_t)q * 8192u, &ma, i0 + q * 64, t0, bar);
          } else {
            tc::load_2d<CG>(sa, &ma, t0, i0, bar);
          }
          if (P.b_outer) {
            for (int q = 0; q < nb / 64; ++q) tc::load_2d<CG>(sb + (uint32_t)q * 8192u, &mb, j0 + q * 64, t0, bar);
          } else {
            tc::load_2d<CG>(sb, &mb, t0, j0, bar);
          }
          if (++st == nstages) st = 0, phase ^= 1u;
        }
      }
    }
    __syncwarp();
  } else if (warp == kWarpMma) {
    if (lane == 0 && rank == 0) {
      uint32_t it = 0, st = 0, phase = 0;
      bool ok = true;
      // 16 values of t: 32 bytes along 128-byte rows, or 16 rows of 128 bytes
      // (descriptors count in 16 bytes)
      const uint64_t step_a = P.a_outer ? 128u : 2u, step_b = P.b_outer ? 128u : 2u, step_st = stage_bytes >> 4;
      const uint64_t da0 = tc::desc128(base, 8192u), db0 = tc::desc128(base + kABytes, 8192u);
      uint64_t da = da0, db = db0;
      // The next stage's barrier is awaited in the middle of a stage's MMAs: the
      // tensor pipe holds about two MMAs, which cover the wait there but not
      // one between stages (720 against 512 cycles a stage of 256 x 256).
      for (int item = first; item < items && ok; item += step, ++it) {
        int tm, tn, part;
        item_of(P, item, tm, tn, part);
        const int s0 = (int)((int64_t)P.slices * part / P.splits), s1 = (int)((int64_t)P.slices * (part + 1) / P.splits);
        const uint32_t a = it & 1u, d = tmem + a * (uint32_t)P.nt;
        if (!tc::bar_wait(tc::smem_u32(&B.accempty[a]), ((it >> 1) & 1u) ^ 1u, abort, P.wait_ns) ||
            !tc::bar_wait(tc::smem_u32(&B.full[st]), phase, abort, P.wait_ns))
          break;
        tc::fence_after();
        for (int left = s1 - s0; left > 0; --left) {
          const uint32_t bar = tc::smem_u32(&B.empty[st]);
          const bool wrap = st + 1 == nstages;
          tc::mma<CG>(d, da, db, P.idesc, left != s1 - s0);
          tc::mma<CG>(d, da + step_a, db + step_b, P.idesc, 1u);
          st = wrap ? 0u : st + 1;
          phase ^= wrap ? 1u : 0u;
          ok = left == 1 || tc::bar_wait(tc::smem_u32(&B.full[st]), phase, abort, P.wait_ns);
          tc::fence_after();
          tc::mma<CG>(d, da + 2 * step_a, db + 2 * step_b, P.idesc, 1u);
          tc::mma<CG>(d, da + 3 * step_a, db + 3 * step_b, P.idesc, 1u);
          tc::commit<CG>(bar);
          if (!ok) break;
          da = wrap ? da0 : da + step_st;
          db = wrap ? db0 : db + step_st;
        }
        if (ok) tc::commit<CG>(tc::smem_u32(&B.accfull[a]));
      }
      // every MMA is complete before tensor memory is freed or the pair ends
      tc::commit<CG>(tc::smem_u32(&B.drain));
      const uint64_t t0 = tc::now_ns();
      while (!tc::bar_try(tc::smem_u32(&B.drain), 0) && tc::now_ns() - t0 < (uint64_t)kWaitNs) {
      }
    }
    __syncwarp();
  } else {
    const int ew = warp - kWarpEpi;
    const int lg = warp & 3;  // the quarter of the lanes this warp may read
    const uint32_t lane_base = (uint32_t)(lg * 32) << 16;
    float *stage = reinterpret_cast<float *>(smem + o_staging + (uint32_t)ew * kStaging);
    const int seg = lane & 3, r8 = lane >> 2, n = (int)E.n;
    const bool vectors = E.y_vec && E.y_dtype != NR_F32 && (!E.z || E.z_scale || E.z_vec) && (!E.residual || E.residual_vec) &&
                         !P.partial;
    const uint32_t accempty0 = tc::map_rank(tc::smem_u32(&B.accempty[0]), 0);
    uint32_t it = 0;
    for (int item = first; item < items; item += step, ++it) {
      int tm, tn, part;
      item_of(P, item, tm, tn, part);
      const uint32_t a = it & 1u;
      const int64_t i0 = ((int64_t)tm * CG + rank) * kRows + lg * 32;
      // the two warps of a lane quarter take its chunks of 32 columns in turn
      const int c0 = tn * P.nt + (ew >> 2) * 32, c1 = i0 < P.rows ? min(n, (tn + 1) * P.nt) : 0;
      if (__all_sync(0xffffffffu, tc::bar_wait(tc::smem_u32(&B.accfull[a]), (it >> 1) & 1u, abort, P.wait_ns)) == 0) break;
      tc::fence_after();
      const uint32_t acc = tmem + lane_base + a * (uint32_t)P.nt - (uint32_t)(tn * P.nt);
      for (int c = c0; c < c1; c += 64) {
        uint32_t v[32];
        __syncwarp();  // the block's previous readers are done
        tc::ld32(acc + (uint32_t)c, v);
        const int j = c + seg * 8;
        const bool whole = vectors && c + 32 <= n && i0 + 32 <= P.rows;
        // meanwhile, what the read-back needs
        float2 b[4];
        uint4 res[4];
        if (E.bias) {
          bias8(E, j, b);
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) b[q] = both(0.0f);
        }
        if (E.residual && whole) {
          const uint16_t *p = static_cast<const uint16_t *>(E.residual) + (i0 + r8) * E.residual_ld + j;
#pragma unroll
          for (int u = 0; u < 4; ++u) res[u] = __ldg(reinterpret_cast<const uint4 *>(p + 8 * u * E.residual_ld));
        }
        tc::wait_ld();
        stage_write(stage, lane, v);
        __syncwarp();
        if (whole) {
          finish_block(E, i0 + r8, j, stage, lane, b, res);
        } else {
#pragma unroll 1
          for (int u = 0; u < 4; ++u) {
            float2 s[4];
            stage_read(stage, lane, u, s);
            const int64_t i = i0 + u * 8 + r8;
            if (!P.partial) {
              finish8(E, i, j, i < P.rows, s, b);
            } else if (i < P.rows && j < n) {  // the pitch is a multiple of 8
              float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(E.y) + ((int64_t)part * P.rows + i) * E.y_ld + j);
              p[0] = make_float4(s[0].x, s[0].y, s[1].x, s[1].y);
              p[1] = make_float4(s[2].x, s[2].y, s[3].x, s[3].y);
            }
          }
        }
      }
      tc::fence_before();
      __syncwarp();
      if (lane == 0) tc::bar_arrive_cluster(accempty0 + a * 8u);
    }
  }
  tc::fence_before();
  __syncthreads();
  if (tid == 0 && B.abort) {
    atomicCAS(flag, 0, NR_DEV_TIMEOUT);
    // no MMA waits for the copies in flight any more: a millisecond lets them land
    const uint64_t t0 = tc::now_ns();
    while (tc::now_ns() - t0 < 1000000u) {
    }
  }
  __syncthreads();
  if (CG == 2) tc::cluster_sync();  // no MMA or arrival of the pair is under way any more
  if (warp == kWarpMma) {
    tc::fence_after();
    tc::dealloc<CG>(tmem, cols);
  }
}

// adds the parts' sums in order and finishes them: a thread eight columns, the
// columns padded to whole groups of 32
__global__ void __launch_bounds__(256)
    finish_kernel(const float *parts, int splits, int64_t part_ld, int64_t rows, const Epilogue E) {
  const int64_t segs = (E.n + kOpsGroup - 1) / kOpsGroup * 4;
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t i = e / segs, j = (e - i * segs) * 8;
  const bool row_ok = i < rows;
  float2 v[4] = {}, b[4];
  if (row_ok && j < E.n) {
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
      const float4 *p = reinterpret_cast<const float4 *>(parts + ((int64_t)s * rows + i) * part_ld + j);
      const float4 lo = __ldg(p), hi = __ldg(p + 1);
      v[0] = add2(v[0], make_float2(lo.x, lo.y)), v[1] = add2(v[1], make_float2(lo.z, lo.w));
      v[2] = add2(v[2], make_float2(hi.x, hi.y)), v[3] = add2(v[3], make_float2(hi.z, hi.w));
    }
  }
  bias8(E, (int)j, b);
  finish8(E, i, (int)j, row_ok, v, b);
}

// ------------------------------------------------------------ few rows, on CUDA cores
// A warp holds MR rows against NR columns of C and KS warps share the columns,
// each a part of t; x's values are converted once for NR weights.
constexpr int kRowsThreads = 256;
template <int MR, int NR, typename T>
__global__ void __launch_bounds__(kRowsThreads)
    rows_kernel(const T *__restrict__ x, int64_t x_ld, const T *__restrict__ w, int64_t w_ld, int m, int64_t n, int64_t k,
                int ks, int vec, const Epilogue E) {
  __shared__ float part[kRowsThreads / 32][MR * NR];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int kp = warp % ks;
  const int64_t j0 = ((int64_t)blockIdx.x * (kRowsThreads / 32 / ks) + warp / ks) * NR;
  float acc[MR][NR] = {};
  const T *xr[MR], *wr[NR];
#pragma unroll
  for (int r = 0; r < MR; ++r) xr[r] = x + (int64_t)min(r, m - 1) * x_ld;
#pragma unroll
  for (int c = 0; c < NR; ++c) wr[c] = w + min(j0 + c, n - 1) * w_ld;
  if (j0 < n) {
    if (vec) {
      const int64_t k8 = k / 8;
#pragma unroll 2
      for (int64_t t = kp * 32 + lane; t < k8; t += ks * 32) {
        uint4 wv[NR];
#pragma unroll
        for (int c = 0; c < NR; ++c) wv[c] = __ldg(reinterpret_cast<const uint4 *>(wr[c]) + t);
        uint4 xv[MR];
#pragma unroll
        for (int r = 0; r < MR; ++r) xv[r] = __ldg(reinterpret_cast<const uint4 *>(xr[r]) + t);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          float xf[MR], wf[NR];
#pragma unroll
          for (int r = 0; r < MR; ++r) xf[r] = to_f32(reinterpret_cast<const T *>(&xv[r])[q]);
#pragma unroll
          for (int c = 0; c < NR; ++c) wf[c] = to_f32(reinterpret_cast<const T *>(&wv[c])[q]);
#pragma unroll
          for (int r = 0; r < MR; ++r)
#pragma unroll
            for (int c = 0; c < NR; ++c) acc[r][c] = fmaf(xf[r], wf[c], acc[r][c]);
        }
      }
    }
    for (int64_t t = (vec ? k / 8 * 8 : 0) + kp * 32 + lane; t < k; t += ks * 32) {
      float wf[NR];
#pragma unroll
      for (int c = 0; c < NR; ++c) wf[c] = to_f32(wr[c][t]);
#pragma unroll
      for (int r = 0; r < MR; ++r) {
        const float xf = to_f32(xr[r][t]);
#pragma unroll
        for (int c = 0; c < NR; ++c) acc[r][c] = fmaf(xf, wf[c], acc[r][c]);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < MR; ++r)
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      float v = acc[r][c];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (lane == 0) part[warp][r * NR + c] = v;
    }
  __syncthreads();
  if (kp != 0 || lane >= MR * NR) return;
  const int r = lane / NR;
  const int64_t j = j0 + lane % NR;
  if (r >= m || j >= n) return;
  float z = 0.0f;
  for (int p = 0; p < ks; ++p) z += part[warp + p][lane];
  if (E.bias) z += load_any(E.bias, j, E.bias_dtype);
  if (E.z) store_any(E.z, r * E.z_ld + j, E.z_scale ? (int)NR_F32 : E.dtype, z);
  float y = act_value(z, E.act);
  if (E.residual) y += load_any(E.residual, r * E.residual_ld + j, E.dtype);
  store_any(E.y, r * E.y_ld + j, E.y_dtype, y);
}

// ------------------------------------------------------------ dz and dbias
// z: values of a type, or a checkpoint's codes and scales
struct Saved {
  const void *p;
  const uint8_t *scale;
  int64_t ld;
  int64_t groups;
  int vec;
};
__device__ __forceinline__ void saved8(const Saved &s, int64_t i, int64_t j, int dtype, int count, float (&v)[8]) {
  if (!s.scale) {
    load8(s.p, i * s.ld + j, dtype, s.vec, count, v);
    return;
  }
  const uint2 c = *reinterpret_cast<const uint2 *>(static_cast<const int8_t *>(s.p) + i * s.groups * kOpsGroup + j);
  const float down = held8_down(s.scale[i * s.groups + (j >> 5)]);
  float2 p[4];
  held8_numbers(c.x, p[0], p[1]);
  held8_numbers(c.y, p[2], p[3]);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    v[2 * q] = p[q].x * down;
    v[2 * q + 1] = p[q].y * down;
  }
}

// dz = dy act'(z) rounded to dtype (unless dz is null), and the column sums of
// the unrounded values over this block's rows -> parts[blockIdx.y] (unless
// null). A block takes 256 columns, eight a lane, and its eight warps its rows
// in turn.
__global__ void __launch_bounds__(256)
    dz_kernel(const void *dy, int dy_dtype, int64_t dy_ld, int dy_vec, const Saved z, int act, int64_t m, int64_t n,
              int rows_per_block, int dtype, uint16_t *dz, int64_t dz_ld, float *parts) {
  __shared__ float sums[8][32 * 9];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t j = (int64_t)blockIdx.x * 256 + lane * 8;
  const int count = (int)min((int64_t)8, n - j);
  const int64_t i0 = (int64_t)blockIdx.y * rows_per_block, i1 = min(m, i0 + rows_per_block);
  float acc[8] = {};
  if (count > 0) {
#pragma unroll 2
    for (int64_t i = i0 + warp; i < i1; i += 8) {
      float v[8];
      load8(dy, i * dy_ld + j, dy_dtype, dy_vec, count, v);
      if (act != NR_ACT_NONE) {
        float s[8];
        saved8(z, i, j, dtype, count, s);
#pragma unroll
        for (int q = 0; q < 8; q += 2) {
          const float2 d = mul2(make_float2(v[q], v[q + 1]), act_slope2(make_float2(s[q], s[q + 1]), act));
          v[q] = d.x;
          v[q + 1] = d.y;
        }
      }
      if (dz) store8(dz, i * dz_ld + j, dtype, 1, 8, v);  // the pitch is a multiple of 8
#pragma unroll
      for (int q = 0; q < 8; ++q) acc[q] += v[q];
    }
  }
  if (!parts) return;
#pragma unroll
  for (int q = 0; q < 8; ++q) sums[warp][lane * 9 + q] = acc[q];
  __syncthreads();
  const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (col >= n) return;
  float s = 0.0f;
#pragma unroll
  for (int w = 0; w < 8; ++w) s += sums[w][(threadIdx.x >> 3) * 9 + (threadIdx.x & 7)];
  parts[(int64_t)blockIdx.y * n + col] = s;
}

// dbias[j] = the sum of parts[.][j]: 32 columns a block, eight rows of parts at a time
__global__ void __launch_bounds__(256) dbias_kernel(const float *parts, int count, int64_t n, void *dbias, int dtype) {
  __shared__ float sums[8][33];
  const int c = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int64_t j = (int64_t)blockIdx.x * 32 + c;
  float s = 0.0f;
  if (j < n) {
#pragma unroll 4
    for (int p = r; p < count; p += 8) s += parts[(int64_t)p * n + j];
  }
  sums[r][c] = s;
  __syncthreads();
  if (r != 0 || j >= n) return;
  for (int q = 1; q < 8; ++q) s += sums[q][c];
  store_any(dbias, j, dtype, s);
}

// rows of 16-bit values at any pitch and alignment -> pitch d_ld (a multiple of 8)
__global__ void __launch_bounds__(256)
    pack_kernel(const uint16_t *__restrict__ s, int64_t s_ld, int64_t rows, int64_t cols, uint16_t *d, int64_t d_ld) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t segs = d_ld / 8, i = e / segs, j = (e - i * segs) * 8;
  if (i >= rows) return;
  uint32_t v[4] = {};
#pragma unroll
  for (int q = 0; q < 8; ++q)
    if (j + q < cols) v[q >> 1] |= (uint32_t)s[i * s_ld + j + q] << (16 * (q & 1));
  *reinterpret_cast<uint4 *>(d + i * d_ld + j) = make_uint4(v[0], v[1], v[2], v[3]);
}

// ------------------------------------------------------------ host
// The driver's tensor-map encoder, looked up once through the runtime.
PFN_cuTensorMapEncodeTiled_v12000 map_encoder() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      p = nullptr;
    }
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  }();
  return fn;
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// an operand of a product: `rows` x `cols` 16-bit values, row-major; outer:
// its rows are the products' index t
struct Operand {
  const void *p;
  int64_t ld, rows, cols;
  bool outer;
};
// tensor copies need 16-byte rows that do not overlap
bool mappable(const Operand &o) { return aligned16(o.p) && o.ld % 8 == 0 && o.ld >= o.cols; }

bool make_map(CUtensorMap *m, const Operand &o, int dtype, int box_rows) {
  const PFN_cuTensorMapEncodeTiled_v12000 encode = map_encoder();
  if (!encode) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows}, strides[1] = {(cuuint64_t)o.ld * 2u};
  const cuuint32_t box[2] = {64u, (cuuint32_t)box_rows}, es[2] = {1u, 1u};
  return encode(m, dtype == NR_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
                const_cast<void *>(o.p), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// how a product is cut: CTAs a tile, columns a tile, parts of t
struct Cut {
  int cg, nt, splits;
};

uint32_t stage_bytes(const Cut &c) { return kABytes + (uint32_t)(c.nt / c.cg) * kSlice * 2; }
constexpr uint32_t kSmemMax = 232448;
int stage_count(const Cut &c) {
  const uint32_t fixed = 1024u + kEpiWarps * kStaging + (uint32_t)sizeof(Bars);
  const int s = (int)((kSmemMax - fixed) / stage_bytes(c));
  return s < kStagesMax ? s : kStagesMax;
}

// The cut with the least estimated time, in cycles of an SM: a slice of a tile
// costs its MMAs (128 x nt x 64 products at 8192 flop a cycle) or the copy of
// its operands (48 bytes a cycle an SM), whichever is longer; an item 1500
// cycles more; parts of t their sums' way through L2 (2 KB a cycle over the GPU).
Cut choose(int64_t rows, int64_t n, int64_t slices, bool b_outer, int sms) {
  Cut best = {1, 64, 1};
  double least = 1e30;
  for (int cg = 1; cg <= 2; ++cg)
    for (int nt = 32; nt <= 256; nt *= 2) {
      if (cg == 2 && (nt < 128 || rows <= kRows)) continue;
      if (b_outer && nt / cg < 64) continue;
      if (nt > 32 && nt / 2 >= n && !(b_outer && nt / cg == 64)) continue;  // half of it would do
      const Cut c0 = {cg, nt, 1};
      const double tiles = (double)ceil_div(rows, (int64_t)kRows * cg) * (double)ceil_div(n, nt);
      const double feed = stage_bytes(c0) / 48.0, mma = 2.0 * nt, slot = sms / cg;
      for (int sp = 1; sp <= 32 && (sp == 1 || slices / sp >= 4); ++sp) {
        const double items = tiles * sp, waves = (double)ceil_div((int64_t)items, (int64_t)slot);
        double t = waves * ((double)ceil_div(slices, sp) * (feed > mma ? feed : mma) + 1500.0);
        if (sp > 1) t += 4000.0 + 8.0 * (double)rows * (double)n * sp / 2048.0;
        if (t < least) {
          least = t;
          best = {cg, nt, sp};
        }
      }
    }
  return best;
}

int64_t parts_bytes(const Cut &c, int64_t rows, int64_t n) {
  return c.splits > 1 ? round_up(c.splits * rows * round_up(n, 8) * 4, 256) : 0;
}

int64_t wait_limit = kWaitNs;  // nr_ops_wait_limit

template <int CG>
cudaError_t launch_product(const CUtensorMap &ma, const CUtensorMap &mb, const Product &P, const Epilogue &E, uint32_t smem,
                           int grid, int device, int *flag, cudaStream_t s) {
  static bool ready[64];  // the attribute is set once a device
  if (!ready[device]) {
    const cudaError_t e =
        cudaFuncSetAttribute(product_kernel<CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMax);
    if (e != cudaSuccess) return e;
    ready[device] = true;
  }
  product_kernel<CG><<<grid, kThreads, smem, s>>>(ma, mb, P, E, flag);
  return cudaGetLastError();
}

// C [rows x E.n] = A B^T over t < inner, through E; parts: scratch of parts_bytes(c, rows, E.n)
nr_status product(const Operand &A, const Operand &B, int64_t rows, int64_t inner, const Cut &c, const Epilogue &E,
                  void *parts, int device, cudaStream_t s) {
  int *flag = nullptr;
  cudaError_t e = nr_ops_flag(device, &flag);
  if (e != cudaSuccess) return cuda_status(e);
  CUtensorMap ma, mb;
  if (!make_map(&ma, A, E.dtype, A.outer ? kSlice : kRows) ||
      !make_map(&mb, B, E.dtype, B.outer ? kSlice : c.nt / c.cg))
    return NR_ERR_CUDA;
  Product P = {};
  P.rows = rows;
  P.tiles_m = (int)ceil_div(rows, (int64_t)kRows * c.cg);
  P.tiles_n = (int)ceil_div(E.n, c.nt);
  P.nt = c.nt;
  P.stages = stage_count(c);
  P.slices = (int)ceil_div(inner, kSlice);
  P.splits = c.splits;
  P.a_outer = A.outer;
  P.b_outer = B.outer;
  P.idesc = tc::idesc_f16(kRows * c.cg, c.nt, E.dtype == NR_BF16, A.outer, B.outer);
  P.partial = c.splits > 1;
  P.wait_ns = wait_limit;
  Epilogue X = E;
  if (P.partial) {
    X.y = parts;
    X.y_ld = round_up(E.n, 8);
  }
  const int64_t items = (int64_t)P.tiles_m * P.tiles_n * P.splits, slots = nr_ops_sms(device) / c.cg;
  if (items > (int64_t)1 << 30) return NR_ERR_INVALID_ARG;
  const int grid = (int)(items < slots ? items : slots) * c.cg;
  const uint32_t smem = 1024u + (uint32_t)P.stages * stage_bytes(c) + kEpiWarps * kStaging + (uint32_t)sizeof(Bars);
  e = c.cg == 1 ? launch_product<1>(ma, mb, P, X, smem, grid, device, flag, s)
                : launch_product<2>(ma, mb, P, X, smem, grid, device, flag, s);
  if (e == cudaSuccess && P.partial) {
    const int64_t threads = rows * ceil_div(E.n, kOpsGroup) * 4;
    finish_kernel<<<(unsigned)ceil_div(threads, 256), 256, 0, s>>>(static_cast<const float *>(parts), c.splits, X.y_ld,
                                                                   rows, E);
    e = cudaGetLastError();
  }
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}

cudaError_t pack(const void *src, int64_t ld, int64_t rows, int64_t cols, void *dst, cudaStream_t s) {
  const int64_t d_ld = round_up(cols, 8);
  pack_kernel<<<(unsigned)ceil_div(rows * (d_ld / 8), 256), 256, 0, s>>>(static_cast<const uint16_t *>(src), ld, rows,
                                                                         cols, static_cast<uint16_t *>(dst), d_ld);
  return cudaGetLastError();
}

bool valid(const nr_linear *a, bool backward) {
  if (!a || a->m < 0 || a->m > kOpsMaxRows || a->k < 1 || a->k > kOpsMaxCols || a->n < 1 || a->n > kOpsMaxCols)
    return false;
  if (!is_16bit(a->dtype) || (a->y_dtype != a->dtype && a->y_dtype != NR_F32) ||
      (a->bias_dtype != a->dtype && a->bias_dtype != NR_F32) || !act_ok(a->act) || !act_ok(a->x_act))
    return false;
  if (a->x_ld < 0 || a->w_ld < 0 || a->residual_ld < 0 || a->dy_ld < 0) return false;
  if (a->m > 0 && (!a->x || !a->w)) return false;
  if (!backward) {
    if (a->x_scale || a->x_act) return false;
    if (a->m > 0 && (!a->y || a->y_ld < a->n || (a->z && !a->z_scale && a->z_ld < a->n))) return false;
    return !(a->z_scale && !a->z);
  }
  if (a->x_act && !a->x_scale) return false;
  if (a->m > 0 && (!a->dy || (a->act != NR_ACT_NONE && !a->z))) return false;
  return !(a->m > 0 && a->dx && a->dx_ld < a->k);
}

// the scratch of a call, in order; offsets of -1: not needed
struct Scratch {
  int64_t at = 0;
  int64_t take(int64_t bytes) {
    const int64_t o = at;
    at += round_up(bytes, 256);
    return o;
  }
};

constexpr int kFewRows = 8;
constexpr int64_t kRowsWarps = 16;  // warps an SM that keep enough of the weights in flight

struct ForwardPlan {
  bool few;
  Operand x, w;
  int64_t x_at = -1, w_at = -1, parts_at = -1, z_at = -1, bytes = 0;
  Cut cut = {1, 32, 1};
};
ForwardPlan plan_forward(const nr_linear *a, int device) {
  ForwardPlan f;
  f.few = a->m <= kFewRows;
  f.x = {a->x, a->x_ld, a->m, a->k, false};
  f.w = {a->w, a->w_ld, a->n, a->k, false};
  Scratch s;
  if (f.few) {
    if (a->z_scale) f.z_at = s.take(a->m * a->n * 4);  // z in fp32, to be held in 8 bits
    f.bytes = s.at;
    return f;
  }
  if (!mappable(f.x)) f.x_at = s.take(a->m * round_up(a->k, 8) * 2);
  if (!mappable(f.w)) f.w_at = s.take(a->n * round_up(a->k, 8) * 2);
  f.cut = choose(a->m, a->n, ceil_div(a->k, kSlice), false, nr_ops_sms(device));
  if (f.cut.splits > 1) f.parts_at = s.take(parts_bytes(f.cut, a->m, a->n));
  f.bytes = s.at;
  return f;
}

template <int MR, typename T>
void launch_rows(const nr_linear *a, const Epilogue &E, int sms, cudaStream_t s) {
  const T *x = static_cast<const T *>(a->x), *w = static_cast<const T *>(a->w);
  const int vec = vec_ok(a->x, a->x_ld, a->dtype) && vec_ok(a->w, a->w_ld, a->dtype);
  const int64_t want = sms * kRowsWarps;
  // four columns a warp where that fills the GPU, else one and t split over warps
  const int nr = a->n >= 4 * want ? 4 : 1;
  int ks = 1;
  while (ks < kRowsThreads / 32 && ceil_div(a->n, nr) * ks < want && a->k / (ks * 2) >= 256) ks *= 2;
  const unsigned blocks = (unsigned)ceil_div(ceil_div(a->n, nr), kRowsThreads / 32 / ks);
  if (nr == 4)
    rows_kernel<MR, 4, T><<<blocks, kRowsThreads, 0, s>>>(x, a->x_ld, w, a->w_ld, (int)a->m, a->n, a->k, ks, vec, E);
  else
    rows_kernel<MR, 1, T><<<blocks, kRowsThreads, 0, s>>>(x, a->x_ld, w, a->w_ld, (int)a->m, a->n, a->k, ks, vec, E);
}
template <typename T>
void launch_rows_any(const nr_linear *a, const Epilogue &E, int sms, cudaStream_t s) {
  if (a->m == 1) launch_rows<1, T>(a, E, sms, s);
  else if (a->m == 2) launch_rows<2, T>(a, E, sms, s);
  else if (a->m <= 4) launch_rows<4, T>(a, E, sms, s);
  else launch_rows<8, T>(a, E, sms, s);
}

// rows a block of dz_kernel takes: enough blocks for the GPU, at most 256 parts to add
int dz_rows(int64_t m, int64_t n, int sms) {
  const int64_t want = ceil_div((int64_t)sms * 8, ceil_div(n, 256));
  const int64_t blocks = want < 256 ? want : 256;
  const int64_t r = round_up(ceil_div(m, blocks), 8);
  return (int)(r < 8 ? 8 : r);
}

struct BackwardPlan {
  bool make_dz;  // else dy serves as it is
  Operand dz, x, w;
  int rows = 0, blocks = 0;
  int64_t dz_at = -1, x_at = -1, w_at = -1, sums_at = -1, dx_at = -1, dw_at = -1, bytes = 0;
  Cut dx = {1, 64, 1}, dw = {1, 64, 1};
};
BackwardPlan plan_backward(const nr_linear *a, int device) {
  BackwardPlan b;
  Scratch s;
  const int sms = nr_ops_sms(device);
  const int64_t m = a->m, n = a->n, k = a->k;
  b.dz = {a->dy, a->dy_ld, m, n, false};
  b.x = {a->x, a->x_ld, m, k, true};
  b.w = {a->w, a->w_ld, n, k, true};
  b.make_dz = a->act != NR_ACT_NONE || a->y_dtype != a->dtype || !mappable(b.dz);
  if (m == 0) return b;
  if (b.make_dz && (a->dx || a->dw)) {
    b.dz_at = s.take(m * round_up(n, 8) * 2);
    b.dz.ld = round_up(n, 8);
  }
  b.rows = dz_rows(m, n, sms);
  b.blocks = (int)ceil_div(m, b.rows);
  if (a->dbias) b.sums_at = s.take((int64_t)b.blocks * n * 4);
  if (a->dw && (a->x_scale || !mappable(b.x))) {
    b.x_at = s.take(m * round_up(k, 8) * 2);
    b.x.ld = round_up(k, 8);
  }
  if (a->dx && !mappable(b.w)) {
    b.w_at = s.take(n * round_up(k, 8) * 2);
    b.w.ld = round_up(k, 8);
  }
  // the two products run one after the other and share the parts' scratch
  int64_t parts = 0;
  if (a->dx) {
    b.dx = choose(m, k, ceil_div(n, kSlice), true, sms);
    parts = parts_bytes(b.dx, m, k);
  }
  if (a->dw) {
    b.dw = choose(n, k, ceil_div(m, kSlice), true, sms);
    const int64_t p = parts_bytes(b.dw, n, k);
    parts = p > parts ? p : parts;
  }
  if (parts) b.dx_at = b.dw_at = s.take(parts);
  b.bytes = s.at;
  return b;
}

void *at(void *ws, int64_t o) { return o < 0 ? nullptr : static_cast<char *>(ws) + o; }

}  // namespace

extern "C" int64_t nr_linear_forward_workspace(const nr_linear *a, int device) {
  return valid(a, false) ? plan_forward(a, device).bytes : -1;
}

extern "C" nr_status nr_linear_forward(const nr_linear *a, int device, void *ws, int64_t ws_bytes, void *stream) {
  if (!valid(a, false)) return NR_ERR_INVALID_ARG;
  if (a->m == 0) return NR_OK;
  ForwardPlan f = plan_forward(a, device);
  if (ws_bytes < f.bytes || (f.bytes > 0 && (!ws || (reinterpret_cast<uintptr_t>(ws) & 255)))) return NR_ERR_INVALID_ARG;
  DeviceGuard g(device);
  if (!g.ok) return NR_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Epilogue E = {};
  E.bias = a->bias;
  E.bias_dtype = (int)a->bias_dtype;
  E.act = (int)a->act;
  E.residual = a->residual;
  E.residual_ld = a->residual_ld;
  E.y = a->y;
  E.y_ld = a->y_ld;
  E.z = a->z;
  E.z_ld = a->z_ld;
  E.z_scale = static_cast<uint8_t *>(a->z_scale);
  E.n = a->n;
  E.dtype = (int)a->dtype;
  E.y_dtype = (int)a->y_dtype;
  E.y_vec = vec_ok(a->y, a->y_ld, a->y_dtype);
  E.z_vec = vec_ok(a->z, a->z_ld, a->dtype);
  E.residual_vec = vec_ok(a->residual, a->residual_ld, a->dtype);
  E.bias_vec = vec_ok(a->bias, 8, a->bias_dtype);
  if (f.few) {
    if (a->z_scale) {
      E.z = at(ws, f.z_at);
      E.z_ld = a->n;
    }
    if (a->dtype == NR_F16) launch_rows_any<__half>(a, E, nr_ops_sms(device), s);
    else launch_rows_any<__nv_bfloat16>(a, E, nr_ops_sms(device), s);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_status(e);
    return a->z_scale ? nr_checkpoint8_write(E.z, NR_F32, a->m, a->n, a->n, a->z, a->z_scale, device, stream) : NR_OK;
  }
  cudaError_t e = cudaSuccess;
  if (f.x_at >= 0) {
    e = pack(a->x, a->x_ld, a->m, a->k, at(ws, f.x_at), s);
    f.x.p = at(ws, f.x_at);
    f.x.ld = round_up(a->k, 8);
  }
  if (e == cudaSuccess && f.w_at >= 0) {
    e = pack(a->w, a->w_ld, a->n, a->k, at(ws, f.w_at), s);
    f.w.p = at(ws, f.w_at);
    f.w.ld = round_up(a->k, 8);
  }
  if (e != cudaSuccess) return cuda_status(e);
  return product(f.x, f.w, a->m, a->k, f.cut, E, at(ws, f.parts_at), device, s);
}

extern "C" int64_t nr_linear_backward_workspace(const nr_linear *a, int device) {
  return valid(a, true) ? plan_backward(a, device).bytes : -1;
}

extern "C" nr_status nr_linear_backward(const nr_linear *a, int device, void *ws, int64_t ws_bytes, void *stream) {
  if (!valid(a, true)) return NR_ERR_INVALID_ARG;
  BackwardPlan b = plan_backward(a, device);
  if (ws_bytes < b.bytes || (b.bytes > 0 && (!ws || (reinterpret_cast<uintptr_t>(ws) & 255)))) return NR_ERR_INVALID_ARG;
  DeviceGuard g(device);
  if (!g.ok) return NR_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int dt = (int)a->dtype;
  const int64_t m = a->m, n = a->n, k = a->k;
  cudaError_t e = cudaSuccess;
  if (m == 0) {
    if (a->dw) e = cudaMemsetAsync(a->dw, 0, (size_t)(n * k) * 2, s);
    if (e == cudaSuccess && a->dbias) e = cudaMemsetAsync(a->dbias, 0, (size_t)n * type_bytes(a->bias_dtype), s);
    return e == cudaSuccess ? NR_OK : cuda_status(e);
  }
  if (b.dz_at >= 0 || a->dbias) {
    const int vec = a->y_dtype == NR_F32 ? vec_ok(a->dy, a->dy_ld, NR_F32) : vec_ok(a->dy, a->dy_ld, dt);
    const Saved z = {a->z, static_cast<const uint8_t *>(a->z_scale), a->z_ld, ceil_div(n, kOpsGroup),
                     vec_ok(a->z, a->z_ld, dt)};
    float *sums = static_cast<float *>(at(ws, b.sums_at));
    dz_kernel<<<dim3((unsigned)ceil_div(n, 256), (unsigned)b.blocks), 256, 0, s>>>(
        a->dy, (int)a->y_dtype, a->dy_ld, vec, z, (int)a->act, m, n, b.rows, dt,
        static_cast<uint16_t *>(at(ws, b.dz_at)), b.dz.ld, sums);
    if (a->dbias)
      dbias_kernel<<<(unsigned)ceil_div(n, 32), 256, 0, s>>>(sums, b.blocks, n, a->dbias, (int)a->bias_dtype);
    e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_status(e);
    if (b.dz_at >= 0) b.dz.p = at(ws, b.dz_at);
  }
  Epilogue E = {};
  E.dtype = E.y_dtype = dt;
  E.n = k;
  if (a->dx) {
    if (b.w_at >= 0) {
      e = pack(a->w, a->w_ld, n, k, at(ws, b.w_at), s);
      if (e != cudaSuccess) return cuda_status(e);
      b.w.p = at(ws, b.w_at);
    }
    E.y = a->dx;
    E.y_ld = a->dx_ld;
    E.y_vec = vec_ok(E.y, E.y_ld, dt);
    const nr_status st = product(b.dz, b.w, m, n, b.dx, E, at(ws, b.dx_at), device, s);
    if (st != NR_OK) return st;
  }
  if (a->dw) {
    if (b.x_at >= 0) {
      if (a->x_scale) {
        const nr_status st =
            nr_checkpoint8_read(a->x, a->x_scale, m, k, (int)a->x_act, at(ws, b.x_at), dt, b.x.ld, device, stream);
        if (st != NR_OK) return st;
      } else {
        e = pack(a->x, a->x_ld, m, k, at(ws, b.x_at), s);
        if (e != cudaSuccess) return cuda_status(e);
      }
      b.x.p = at(ws, b.x_at);
    }
    E.y = a->dw;
    E.y_ld = k;
    E.y_vec = vec_ok(E.y, E.y_ld, dt);
    Operand dzt = b.dz;
    dzt.outer = true;
    return product(dzt, b.x, n, m, b.dw, E, at(ws, b.dw_at), device, s);
  }
  return NR_OK;
}

extern "C" nr_status nr_ops_wait_limit(int64_t us) {
  wait_limit = us == 0 ? kWaitNs : us < 0 ? (int64_t)-1 : us * 1000;
  return NR_OK;
}
