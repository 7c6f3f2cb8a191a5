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
// Measured, bf16: 65536 x 6144 -> 1536 690 to 730 us, 1.7 PFLOP/s (a library's
// product reaches 1.9); 10000 x 1536 -> 6144 121 us, 154 with GELU and z kept, 173
// with z in 8 bits, 145 for 136 in the same run with fp32 outputs, whose blocks all
// take the edges' path. A stage takes 600 cycles where its MMAs need 512, and 512
// without its copies; but no one rate is filled: of a plain launch's cycles the
// tensor pipe is active in 72% (64% with GELU and z), shared memory's banks are read
// in 21% and written in 21%, L2 is busy to 47%.
//
// Up to eight rows run on CUDA cores instead (rows_kernel), which read the weights
// once: one to four rows take little more than that, five to eight the code of eight
// rows. GPU time in us for one, four, five to eight rows, and nine on the tensor
// cores: 1536 -> 6144 6.0, 8.1, 15.0 and 12.1; 6144 -> 1536 4.8, 8.1, 13.4 and 13.6;
// 1536 -> 512 2.6, 3.4, 4.6 and 8.3; 512 -> 512 2.3, 2.8, 3.4 and 6.2. So five to
// eight rows lose to the tensor cores in wide layers and gain in narrow ones.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "nrq_ops.cuh"
#include "nrq_tc.cuh"

namespace {

// ------------------------------------------------------------ epilogue
// What becomes of the sums s[i, j]: z = s + bias, y = act(z) + residual.
struct Epilogue {
  const void *bias;
  int bias_dtype, act;
  const void *residual, *residual_end;  // of type dtype; past its last value
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
// eight 16-bit values of a row that has `left` from p on, the four threads of 32
// columns together (lanes 4 a .. 4 a + 3 of a warp); vec: at 16-byte addresses
__device__ __forceinline__ void store_any16(uint16_t *p, int vec, int left, const float2 (&v)[4], int dtype) {
  const int lane = threadIdx.x & 31;
  const uint4 o = pack8(v, dtype);
  if (vec && left >= 8) {
    *reinterpret_cast<uint4 *>(p) = o;
    return;
  }
  const uint32_t w[4] = {o.x, o.y, o.z, o.w};
  if (vec) {  // a row's end, which is this lane's alone
#pragma unroll
    for (int q = 0; q < 7; ++q)
      if (q < left) p[q] = (uint16_t)(w[q >> 1] >> (16 * (q & 1)));
    return;
  }
  store16x8(p, left, w, (lane & 3) > 0, (lane & 3) < 3, 0xfu << (lane & 28));
}

// Finishes s[i, j .. j + 7] (j a multiple of 8; bias: those columns'), row_ok
// false for rows past the end; called as hold8 is.
__device__ __forceinline__ void finish8(const Epilogue &E, int64_t i, int j, bool row_ok, float2 (&v)[4],
                                        const float2 (&bias)[4]) {
  const int left = row_ok ? (int)E.n - j : 0, count = max(0, min(8, left));
  const uint16_t *pr = static_cast<const uint16_t *>(E.residual) + i * E.residual_ld + j;
  uint32_t res[8];
  if (E.residual) fetch16x8(pr, count, E.residual, E.residual_end, res);
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = add2(v[q], bias[q]);
  if (E.z) {
    if (E.z_scale) hold8(E, i, j, row_ok, count, v);
    else store_any16(static_cast<uint16_t *>(E.z) + i * E.z_ld + j, E.z_vec, left, v, E.dtype);
  }
  if (E.act != NR_ACT_NONE) {
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = act_value2(v[q], E.act);
  }
  if (E.residual) {
    settle16x8(pr, count, E.residual, E.residual_end, res);
    add_raw(v, make_uint4(res[0], res[1], res[2], res[3]), E.dtype);
  }
  if (E.y_dtype == NR_F32) {
    const float o[8] = {v[0].x, v[0].y, v[1].x, v[1].y, v[2].x, v[2].y, v[3].x, v[3].y};
    if (count > 0) store8(E.y, i * E.y_ld + j, NR_F32, E.y_vec, count, o);
  } else {
    store_any16(static_cast<uint16_t *>(E.y) + i * E.y_ld + j, E.y_vec, left, v, E.dtype);
  }
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

// eight 16-bit values of a row: the four threads of 32 columns together
template <bool VEC>
__device__ __forceinline__ void store_block(uint16_t *p, bool there, int lane, const float2 (&v)[4], int dtype) {
  const uint4 o = pack8(v, dtype);
  if (VEC) {
    if (there) *reinterpret_cast<uint4 *>(p) = o;
  } else {
    const uint32_t w[4] = {o.x, o.y, o.z, o.w};
    store16x8(p, there ? 32 - 8 * (lane & 3) : 0, w, (lane & 3) > 0, (lane & 3) < 3, 0xfu << (lane & 28));
  }
}

// A block with its 32 columns there and y 16-bit, from row i, column j of the
// thread's eight of four rows, of which those below `left` rows on are there: one
// test a step for all rows. VEC: every matrix takes
// 16-byte accesses, and res holds the residual, loaded ahead.
template <bool VEC>
__device__ __forceinline__ void finish_block(const Epilogue &E, int64_t i, int left, int j, const float *stage, int lane,
                                             const float2 (&b)[4], const uint4 (&res)[4]) {
  float2 v[4][4];
  uint32_t far[4][8];
  const uint16_t *pr = static_cast<const uint16_t *>(E.residual) + i * E.residual_ld + j;
  if (!VEC && E.residual) {
#pragma unroll
    for (int u = 0; u < 4; ++u) fetch16x8(pr + 8 * u * E.residual_ld, 8 * u < left ? 8 : 0, E.residual, E.residual_end, far[u]);
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    stage_read(stage, lane, u, v[u]);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[u][q] = add2(v[u][q], b[q]);
  }
  if (E.z) {
    if (E.z_scale) {
#pragma unroll
      for (int u = 0; u < 4; ++u) hold8(E, i + 8 * u, j, 8 * u < left, 8, v[u]);
    } else {
      uint16_t *z = static_cast<uint16_t *>(E.z) + i * E.z_ld + j;
#pragma unroll
      for (int u = 0; u < 4; ++u) store_block<VEC>(z + 8 * u * E.z_ld, 8 * u < left, lane, v[u], E.dtype);
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
    for (int u = 0; u < 4; ++u) {
      if (VEC) {
        add_raw(v[u], res[u], E.dtype);
      } else {
        settle16x8(pr + 8 * u * E.residual_ld, 8 * u < left ? 8 : 0, E.residual, E.residual_end, far[u]);
        add_raw(v[u], make_uint4(far[u][0], far[u][1], far[u][2], far[u][3]), E.dtype);
      }
    }
  }
  uint16_t *y = static_cast<uint16_t *>(E.y) + i * E.y_ld + j;
#pragma unroll
  for (int u = 0; u < 4; ++u) store_block<VEC>(y + 8 * u * E.y_ld, 8 * u < left, lane, v[u], E.dtype);
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

// One product, and how it is cut.
struct Product {
  int64_t rows;          // of C
  int tiles_m, tiles_n;  // tiles of 128 CG rows, of nt columns
  int nt;
  int slices, splits;    // of 64 values of t; parts of them
  int a_outer, b_outer;  // the operand's own index is the contiguous one
  uint32_t idesc;
  float *parts;          // splits > 1: part s's sums go to parts + s rows parts_ld
  int64_t parts_ld;
  Epilogue E;
};

// A launch: one product, or two that share the GPU (the second's tiles fill what the
// first's leave idle).
struct Job {
  Product p[2];
  int items0, items;     // work items of the first, of both
  int nt, stages;        // the wider tile's columns
  uint32_t stage_bytes;
  int *flag;
  int64_t wait_ns;
};

// Items go to the CTAs (pairs), the longer first, in turns that run forwards and
// backwards. A last, short turn falls to those that had the shorter items of the turn
// before if the number of turns is odd, and to those that had the longer ones if it
// is even (both products of 4096 rows of 1536 -> 6144: 320 slices on one pair where
// the mean is 242.5).
__device__ __forceinline__ int item_at(int turn, int slot, int slots) {
  return turn * slots + ((turn & 1) ? slots - 1 - slot : slot);
}

// an item's tile and part. Tiles run down bands of 8 tile rows, so that the
// tiles in flight share their slices of A and B in L2.
__device__ __forceinline__ void item_of(const Product &P, int item, int &tm, int &tn, int &part) {
  const int tiles = P.tiles_m * P.tiles_n;
  part = P.splits > 1 ? item / tiles : 0;
  const int t = item - part * tiles;
  constexpr int kBand = 8;
  const int band = t / (kBand * P.tiles_n), in = t - band * kBand * P.tiles_n;
  const int height = min(kBand, P.tiles_m - band * kBand);
  tn = in / height;
  tm = band * kBand + in - tn * height;
}

// A part's slices. Splits are rare: the divisions, hundreds of cycles between
// two tiles' MMAs, are left out without them.
__device__ __forceinline__ void slices_of(const Product &P, int part, int &s0, int &s1) {
  s0 = 0, s1 = P.slices;
  if (P.splits > 1) {  // slices and parts: at most 2^25 and 32
    s0 = P.slices / P.splits * part + min(part, P.slices % P.splits);
    s1 = s0 + P.slices / P.splits + (part < P.slices % P.splits ? 1 : 0);
  }
}

template <int CG>
__global__ void __cluster_dims__(CG, 1, 1) __launch_bounds__(kThreads, 1)
    product_kernel(const __grid_constant__ CUtensorMap ma0, const __grid_constant__ CUtensorMap mb0,
                   const __grid_constant__ CUtensorMap ma1, const __grid_constant__ CUtensorMap mb1,
                   const __grid_constant__ Job J) {
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char *smem = smem_raw + (base - tc::smem_u32(smem_raw));
  const uint32_t o_staging = (uint32_t)J.stages * J.stage_bytes, o_bars = o_staging + kEpiWarps * kStaging;
  Bars &B = *reinterpret_cast<Bars *>(smem + o_bars);
  volatile int *abort = &B.abort;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = CG == 2 ? tc::cluster_rank() : 0u;
  const int slot = blockIdx.x / CG, slots = gridDim.x / CG;
  const int64_t limit = J.wait_ns;
  uint32_t cols = 32;
  while (cols < 2u * (uint32_t)J.nt) cols <<= 1;

  if (warp == kWarpMma) tc::alloc<CG>(tc::smem_u32(&B.tmem_slot), cols);
  if (tid == 0) {
    for (int i = 0; i < J.stages; ++i) {
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
  const uint32_t nstages = (uint32_t)J.stages;
  grid_wait();  // what the previous launch of this call wrote is there
  grid_launch();

  // The roles below take the first product's items, then the second's, in code of
  // their own: a product picked by index would keep its constants out of the
  // uniform registers that copies and MMAs are issued from (up to a third slower).
  if (warp == kWarpProd) {
    if (lane == 0) {
      uint32_t st = 0, phase = 1;  // the stage's wait parity: free at first
      int turn = 0;
      bool ok = true;
      auto produce = [&](const Product &P, const CUtensorMap *ma, const CUtensorMap *mb, int from, int to) {
        const int nb = P.nt / CG;  // rows of B this CTA holds
        const uint32_t bytes = kABytes + (uint32_t)nb * kSlice * 2;
        for (; ok; ++turn) {
          const int item = item_at(turn, slot, slots);
          if (item >= to) break;
          int tm, tn, part;
          item_of(P, item - from, tm, tn, part);
          const int i0 = (tm * CG + (int)rank) * kRows, j0 = tn * P.nt + (int)rank * nb;
          int s0, s1;
          slices_of(P, part, s0, s1);
          for (int s = s0; s < s1; ++s) {
            if (!tc::bar_wait(tc::smem_u32(&B.empty[st]), phase, abort, limit)) {
              ok = false;
              break;
            }
            // the pair's bytes are counted on the first CTA's barrier
            uint32_t bar = tc::smem_u32(&B.full[st]);
            if (rank == 0) tc::bar_expect(bar, CG * bytes);
            if (CG == 2) bar = tc::map_rank(bar, 0);
            const uint32_t sa = base + st * J.stage_bytes, sb = sa + kABytes;
            const int t0 = s * kSlice;
            if (P.a_outer) {
              for (int q = 0; q < kRows / 64; ++q) tc::load_2d<CG>(sa + (uint32_t)q * 8192u, ma, i0 + q * 64, t0, bar);
            } else {
              tc::load_2d<CG>(sa, ma, t0, i0, bar);
            }
            if (P.b_outer) {
              for (int q = 0; q < nb / 64; ++q) tc::load_2d<CG>(sb + (uint32_t)q * 8192u, mb, j0 + q * 64, t0, bar);
            } else {
              tc::load_2d<CG>(sb, mb, t0, j0, bar);
            }
            if (++st == nstages) st = 0, phase ^= 1u;
          }
        }
      };
      produce(J.p[0], &ma0, &mb0, 0, J.items0);
      produce(J.p[1], &ma1, &mb1, J.items0, J.items);
    }
    __syncwarp();
  } else if (warp == kWarpMma) {
    if (lane == 0 && rank == 0) {
      uint32_t it = 0, st = 0, phase = 0;
      int turn = 0;
      bool ok = true;
      const uint64_t step_st = J.stage_bytes >> 4;  // descriptors count in 16 bytes
      const uint64_t da0 = tc::desc128(base, 8192u), db0 = tc::desc128(base + kABytes, 8192u);
      uint64_t da = da0, db = db0;
      // The next stage's barrier is awaited in the middle of a stage's MMAs: the
      // tensor pipe holds about two MMAs, which cover the wait there but not
      // one between stages (720 against 512 cycles a stage of 256 x 256).
      auto multiply = [&](const Product &P, int from, int to) {
        // 16 values of t: 32 bytes along 128-byte rows, or 16 rows of 128 bytes
        const uint64_t step_a = P.a_outer ? 128u : 2u, step_b = P.b_outer ? 128u : 2u;
        for (; ok; ++turn) {
          const int item = item_at(turn, slot, slots);
          if (item >= to) break;
          int s0, s1;
          slices_of(P, P.splits > 1 ? (item - from) / (P.tiles_m * P.tiles_n) : 0, s0, s1);
          const uint32_t a = it & 1u, d = tmem + a * (uint32_t)J.nt;
          if (!tc::bar_wait(tc::smem_u32(&B.accempty[a]), ((it >> 1) & 1u) ^ 1u, abort, limit) ||
              !tc::bar_wait(tc::smem_u32(&B.full[st]), phase, abort, limit)) {
            ok = false;
            break;
          }
          tc::fence_after();
          for (int left = s1 - s0; left > 0; --left) {
            const uint32_t bar = tc::smem_u32(&B.empty[st]);
            const bool wrap = st + 1 == nstages;
            tc::mma<CG>(d, da, db, P.idesc, left != s1 - s0);
            tc::mma<CG>(d, da + step_a, db + step_b, P.idesc, 1u);
            st = wrap ? 0u : st + 1;
            phase ^= wrap ? 1u : 0u;
            ok = left == 1 || tc::bar_wait(tc::smem_u32(&B.full[st]), phase, abort, limit);
            tc::fence_after();
            tc::mma<CG>(d, da + 2 * step_a, db + 2 * step_b, P.idesc, 1u);
            tc::mma<CG>(d, da + 3 * step_a, db + 3 * step_b, P.idesc, 1u);
            tc::commit<CG>(bar);
            if (!ok) break;
            da = wrap ? da0 : da + step_st;
            db = wrap ? db0 : db + step_st;
          }
          if (ok) tc::commit<CG>(tc::smem_u32(&B.accfull[a]));
          ++it;
        }
      };
      multiply(J.p[0], 0, J.items0);
      multiply(J.p[1], J.items0, J.items);
      tc::commit<CG>(tc::smem_u32(&B.drain));
    }
    __syncwarp();
  } else {
    const int ew = warp - kWarpEpi;
    const int lg = warp & 3;  // the quarter of the lanes this warp may read
    const uint32_t lane_base = (uint32_t)(lg * 32) << 16;
    float *stage = reinterpret_cast<float *>(smem + o_staging + (uint32_t)ew * kStaging);
    const int seg = lane & 3, r8 = lane >> 2;
    const uint32_t accempty0 = tc::map_rank(tc::smem_u32(&B.accempty[0]), 0);
    uint32_t it = 0;
    for (int turn = 0;; ++turn) {
      const int item = item_at(turn, slot, slots);
      if (item >= J.items) break;  // later turns are past the end too
      const bool second = item >= J.items0;
      const Product &P = J.p[second];
      const Epilogue E = P.E;  // in registers
      const int n = (int)E.n;
      const int64_t rows = P.rows;
      const bool partial = P.splits > 1;
      int tm, tn, part;
      item_of(P, second ? item - J.items0 : item, tm, tn, part);
      const uint32_t a = it & 1u;
      const int64_t i0 = ((int64_t)tm * CG + rank) * kRows + lg * 32;
      const bool blocks = E.y_dtype != NR_F32 && !partial;
      const int left = (int)min(rows - i0, (int64_t)32) - r8;  // rows from the thread's first on
      const bool vectors = E.y_vec && (!E.z || E.z_scale || E.z_vec) && (!E.residual || E.residual_vec);
      // the two warps of a lane quarter take its chunks of 32 columns in turn
      const int c0 = tn * P.nt + (ew >> 2) * 32, c1 = i0 < rows ? min(n, (tn + 1) * P.nt) : 0;
      if (E.residual && blocks && i0 + lane < rows) {  // the residual's way from memory, while the sums are made
        const uint16_t *p = static_cast<const uint16_t *>(E.residual) + (i0 + lane) * E.residual_ld;
        for (int c = c0; c < c1; c += 64) asm volatile("prefetch.global.L2 [%0];\n" ::"l"(p + c));
      }
      if (__all_sync(0xffffffffu, tc::bar_wait(tc::smem_u32(&B.accfull[a]), (it >> 1) & 1u, abort, limit)) == 0) break;
      tc::fence_after();
      const uint32_t acc = tmem + lane_base + a * (uint32_t)J.nt - (uint32_t)(tn * P.nt);
      for (int c = c0; c < c1; c += 64) {
        uint32_t v[32];
        __syncwarp();
        tc::ld32(acc + (uint32_t)c, v);
        const int j = c + seg * 8;
        const bool whole = blocks && c + 32 <= n;
        // what the read-back needs, while the sums arrive
        float2 b[4];
        uint4 res[4];
        if (E.bias) {
          bias8(E, j, b);
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) b[q] = both(0.0f);
        }
        if (E.residual && whole && vectors) {
          const uint16_t *p = static_cast<const uint16_t *>(E.residual) + (i0 + r8) * E.residual_ld + j;
#pragma unroll
          for (int u = 0; u < 4; ++u) res[u] = load_if128(p + 8 * u * E.residual_ld, 8 * u < left);
        }
        tc::wait_ld(v);
        __syncwarp();  // the block's previous readers are done
        stage_write(stage, lane, v);
        __syncwarp();
        if (whole && vectors) {
          finish_block<true>(E, i0 + r8, left, j, stage, lane, b, res);
        } else if (whole) {
          finish_block<false>(E, i0 + r8, left, j, stage, lane, b, res);
        } else {
#pragma unroll 1
          for (int u = 0; u < 4; ++u) {
            float2 s[4];
            stage_read(stage, lane, u, s);
            const int64_t i = i0 + u * 8 + r8;
            if (!partial) {
              finish8(E, i, j, i < rows, s, b);
            } else if (i < rows && j < n) {  // the pitch is a multiple of 8
              float4 *p = reinterpret_cast<float4 *>(P.parts + ((int64_t)part * rows + i) * P.parts_ld + j);
              p[0] = make_float4(s[0].x, s[0].y, s[1].x, s[1].y);
              p[1] = make_float4(s[2].x, s[2].y, s[3].x, s[3].y);
            }
          }
        }
      }
      tc::fence_before();
      __syncwarp();
      if (lane == 0) tc::bar_arrive_cluster(accempty0 + a * 8u);
      ++it;
    }
  }
  tc::fence_before();
  __syncthreads();
  if (tid == 0) {
    // Every MMA is complete before tensor memory is freed; and commits arrive on both
    // CTAs' barriers, the drain's last, so neither leaves before it has them.
    const uint64_t t0 = tc::now_ns();
    while (!tc::bar_try(tc::smem_u32(&B.drain), 0) && tc::now_ns() - t0 < (uint64_t)kWaitNs) {
    }
  }
  if (tid == 0 && B.abort) {
    atomicCAS(J.flag, 0, NR_DEV_TIMEOUT);
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

// What is left after the products, in one launch: block ranges add the parts'
// sums of a split product in order and finish them (a thread eight columns,
// padded to whole groups of 32), and the rows of column sums that dz_kernel
// left into dbias (eight columns a block, 32 rows at a time).
struct Finish {
  Product p[2];
  int blocks[2];  // of each product; 0: not split
  const float *sums;
  int sums_rows;
  int64_t sums_n;
  void *dbias;
  int dbias_dtype;
};
__global__ void __launch_bounds__(256) finish_kernel(const __grid_constant__ Finish F) {
  __shared__ float sums[32][9];
  grid_wait();
  int block = (int)blockIdx.x;
  const int which = block < F.blocks[0] ? 0 : 1;
  if (which) block -= F.blocks[0];
  if (which == 0 || block < F.blocks[1]) {
    const Product &P = F.p[which];
    const Epilogue &E = P.E;
    const int segs = ((int)E.n + kOpsGroup - 1) / kOpsGroup * 4;
    const int64_t e = (int64_t)block * 256 + threadIdx.x;
    const int64_t i = e / segs;
    const int j = (int)(e - i * segs) * 8;
    const bool row_ok = i < P.rows;
    float2 v[4] = {}, b[4];
    if (row_ok && j < (int)E.n) {
#pragma unroll 4
      for (int s = 0; s < P.splits; ++s) {
        const float4 *p = reinterpret_cast<const float4 *>(P.parts + ((int64_t)s * P.rows + i) * P.parts_ld + j);
        const float4 lo = p[0], hi = p[1];
        v[0] = add2(v[0], make_float2(lo.x, lo.y)), v[1] = add2(v[1], make_float2(lo.z, lo.w));
        v[2] = add2(v[2], make_float2(hi.x, hi.y)), v[3] = add2(v[3], make_float2(hi.z, hi.w));
      }
    }
    bias8(E, j, b);
    finish8(E, i, j, row_ok, v, b);
    return;
  }
  block -= F.blocks[1];
  const int c = threadIdx.x & 7, r = threadIdx.x >> 3;
  const int64_t j = (int64_t)block * 8 + c;
  float s = 0.0f;
  if (j < F.sums_n) {
#pragma unroll 8
    for (int p = r; p < F.sums_rows; p += 32) s += F.sums[(int64_t)p * F.sums_n + j];
  }
  sums[r][c] = s;
  __syncthreads();
  if (r != 0 || j >= F.sums_n) return;
  for (int q = 1; q < 32; ++q) s += sums[q][c];
  store_any(F.dbias, j, F.dbias_dtype, s);
}

// ------------------------------------------------------------ few rows, on CUDA cores
// Bound by reading the weights up to four rows (19 MB of them in 6.0 us at one row, from
// L2), by conversions and products from five on.
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
  float2 acc2[MR][NR] = {};
  const T *xr[MR], *wr[NR];
#pragma unroll
  for (int r = 0; r < MR; ++r) xr[r] = x + (int64_t)min(r, m - 1) * x_ld;
#pragma unroll
  for (int c = 0; c < NR; ++c) wr[c] = w + min(j0 + c, n - 1) * w_ld;
  if (j0 < n) {
    if (vec) {
      const int64_t k8 = k / 8;
      // U of the weights' loads under way at once (past the row's end: zeros)
      constexpr int U = NR == 1 ? 4 : 2;
      for (int64_t t0 = kp * 32 + lane; t0 < k8; t0 += (int64_t)U * ks * 32) {
        uint4 wv[U][NR];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int c = 0; c < NR; ++c)
            wv[u][c] = load_if128(reinterpret_cast<const uint4 *>(wr[c]) + t0 + u * ks * 32, t0 + u * ks * 32 < k8);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          uint4 xv[MR];
#pragma unroll
          for (int r = 0; r < MR; ++r)
            xv[r] = load_if128(reinterpret_cast<const uint4 *>(xr[r]) + t0 + u * ks * 32, t0 + u * ks * 32 < k8);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float2 xf[MR], wf[NR];
#pragma unroll
            for (int r = 0; r < MR; ++r) xf[r] = unpack2(reinterpret_cast<const uint32_t *>(&xv[r])[q], TypeCode<T>::code);
#pragma unroll
            for (int c = 0; c < NR; ++c) wf[c] = unpack2(reinterpret_cast<const uint32_t *>(&wv[u][c])[q], TypeCode<T>::code);
#pragma unroll
            for (int r = 0; r < MR; ++r)
#pragma unroll
              for (int c = 0; c < NR; ++c) acc2[r][c] = fma2(xf[r], wf[c], acc2[r][c]);
          }
        }
      }
#pragma unroll
      for (int r = 0; r < MR; ++r)
#pragma unroll
        for (int c = 0; c < NR; ++c) acc[r][c] = acc2[r][c].x + acc2[r][c].y;
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

// ------------------------------------------------------------ dz and the column sums
// z: values of a type, or a checkpoint's codes and scales
struct Saved {
  const void *p;
  const uint8_t *scale;
  int64_t ld;
  int groups;
};

// dz = dy act'(z) rounded to T (unless dz is null), and the column sums of the
// unrounded values over a block's rows -> sums[blockIdx.y] (unless null). Rounded, as
// the tensor cores multiply 16-bit operands of one type and dx and dw have w and x of T
// beside it: dz as a sum of two such terms would double both products. An fp32 dy is
// rounded there too. In bf16 the rounding takes their error from 0.0017 of the norm,
// which is their own rounding's, to 0.0023.
// Bound by memory with z in 16 bits: dy and z read, dz written (4096 x 6144 with GELU 24
// us, 6.2 TB/s); with z in 8 bits by the arithmetic (16384 x 6144 104 us, 4.9 TB/s, and 95
// without writing dz, an instruction issued in 69% of cycles). A block's threads: x over columns,
// eight each, y over rows; a thread takes four rows at a time (two at other addresses,
// which take twice the registers), all loads first. VEC: n is a multiple of 8 and dy and
// z take 16-byte accesses.
constexpr int kDzRows = 4;
template <bool VEC, typename D, typename T>
__global__ void __launch_bounds__(256, 3)
    dz_kernel(const D *dy, int64_t dy_ld, const Saved z, int act, int64_t m, int n, int rows_per_block, T *dz,
              int64_t dz_ld, float *sums) {
  constexpr int R = VEC ? kDzRows : kDzRows / 2;
  __shared__ float part[256 * 8];
  const int j = (blockIdx.x * blockDim.x + threadIdx.x) * 8, count = max(0, min(8, n - j));
  const int64_t i1 = min(m, ((int64_t)blockIdx.y + 1) * rows_per_block);
  float2 acc[4] = {};
  const int step = blockDim.y;
  grid_launch();
  for (int64_t i0 = (int64_t)blockIdx.y * rows_per_block + threadIdx.y; i0 < i1 && count > 0; i0 += R * step) {
    Eight<D> v[R];
    Eight<T> s[R];
    float down[R];
    const int there = VEC ? 8 : count;
    const void *dy_end = dy + (m - 1) * dy_ld + n, *z_end = static_cast<const T *>(z.p) + (m - 1) * z.ld + n;
#pragma unroll
    for (int u = 0; u < R; ++u) v[u] = fetch_eight<D>(dy + min(i0 + u * step, i1 - 1) * dy_ld + j, VEC, there, dy, dy_end);
    if (act != NR_ACT_NONE) {
      if (!z.scale) {
#pragma unroll
        for (int u = 0; u < R; ++u)
          s[u] = fetch_eight<T>(static_cast<const T *>(z.p) + min(i0 + u * step, i1 - 1) * z.ld + j, VEC, there, z.p, z_end);
      } else {
#pragma unroll
        for (int u = 0; u < R; ++u) {
          const int64_t i = min(i0 + u * step, i1 - 1);
          const uint2 c = __ldg(reinterpret_cast<const uint2 *>(static_cast<const int8_t *>(z.p) + i * z.groups * kOpsGroup + j));
          s[u].r[0] = c.x, s[u].r[1] = c.y;
          down[u] = held8_down(__ldg(z.scale + i * z.groups + (j >> 5)));
        }
      }
    }
#pragma unroll
    for (int u = 0; u < R; ++u) {
      const int64_t i = i0 + u * step;
      if (i >= i1) break;
      settle_eight<D>(v[u], dy + i * dy_ld + j, VEC, there, dy, dy_end);
      if (act != NR_ACT_NONE && !z.scale)
        settle_eight<T>(s[u], static_cast<const T *>(z.p) + i * z.ld + j, VEC, there, z.p, z_end);
      float2 d[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) d[q] = pair_of<D>(v[u], q);
      if (act != NR_ACT_NONE) {
        float2 p[4];
        if (z.scale) {
          held8_numbers(s[u].r[0], p[0], p[1]);
          held8_numbers(s[u].r[1], p[2], p[3]);
#pragma unroll
          for (int q = 0; q < 4; ++q) p[q] = mul2(p[q], both(down[u]));
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) p[q] = pair_of<T>(s[u], q);
        }
        // one test of the activation for the eight
#define NR_SLOPE(A)                   \
  _Pragma("unroll") for (int q = 0; q < 4; ++q) d[q] = mul2(d[q], act_slope2(p[q], A));
        if (act == NR_ACT_GELU) {
          NR_SLOPE(NR_ACT_GELU)
        } else if (act == NR_ACT_SILU) {
          NR_SLOPE(NR_ACT_SILU)
        } else {
          NR_SLOPE(NR_ACT_RELU)
        }
#undef NR_SLOPE
      }
      // the pitch is a multiple of 8
      if (dz) *reinterpret_cast<uint4 *>(dz + i * dz_ld + j) = pack8(d, TypeCode<T>::code);
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[q] = add2(acc[q], d[q]);
    }
  }
  if (!sums) return;
  const int bx = blockDim.x * 8;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    *reinterpret_cast<float2 *>(part + threadIdx.y * bx + threadIdx.x * 8 + 2 * q) = acc[q];
  __syncthreads();
  const int t = threadIdx.y * blockDim.x + threadIdx.x, col = blockIdx.x * bx + t;
  if (t >= bx || col >= n) return;
  float s = 0.0f;
  for (int r = 0; r < (int)blockDim.y; ++r) s += part[r * bx + t];
  sums[(int64_t)blockIdx.y * n + col] = s;
}

// rows of 16-bit values at any pitch and alignment -> pitch d_ld (a multiple of
// 8), for up to two matrices a launch
struct Pack {
  const uint16_t *s[2];
  uint16_t *d[2];
  int64_t s_ld[2], rows[2];
  int cols[2], d_ld[2];
  int64_t blocks0;
};
__global__ void __launch_bounds__(256) pack_kernel(const Pack K) {
  grid_launch();
  const int which = (int64_t)blockIdx.x >= K.blocks0;
  const int64_t e = ((int64_t)blockIdx.x - (which ? K.blocks0 : 0)) * 256 + threadIdx.x;
  const int segs = K.d_ld[which] / 8, cols = K.cols[which];
  const int64_t i = e / segs;
  const int j = (int)(e - i * segs) * 8;
  if (i >= K.rows[which]) return;
  const uint16_t *s = K.s[which];
  const uint16_t *p = s + i * K.s_ld[which] + j, *end = s + (K.rows[which] - 1) * K.s_ld[which] + cols;
  uint32_t v[8];
  fetch16x8(p, min(8, cols - j), s, end, v);
  settle16x8(p, min(8, cols - j), s, end, v);
  *reinterpret_cast<uint4 *>(K.d[which] + i * K.d_ld[which] + j) = make_uint4(v[0], v[1], v[2], v[3]);
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

constexpr uint32_t kSmemMax = 232448;
uint32_t cut_bytes(const Cut &c) { return kABytes + (uint32_t)(c.nt / c.cg) * kSlice * 2; }

// The cut with the least estimated time, in cycles of an SM: a slice of a tile
// costs its MMAs (128 x nt x 64 products at 8192 flop a cycle, of which 0.85
// was reached) or the copy of its operands (56 bytes a cycle an SM), whichever is
// longer; an item 1500 cycles more; parts of t their sums' way through L2 (2 KB a
// cycle over the GPU) and the launch that adds them. cg 0: either.
Cut choose(int64_t rows, int64_t n, int64_t slices, bool b_outer, int cg_only, int sms, float *cost = nullptr) {
  static const int kSplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
  Cut best = {1, 64, 1};
  float least = 1e30f;
  for (int cg = 1; cg <= 2; ++cg) {
    if (cg_only ? cg != cg_only : cg == 2 && rows <= kRows) continue;
    const int64_t tm = ceil_div(rows, (int64_t)kRows * cg), slot = sms / cg;
    if (slot < 1) continue;
    for (int nt = 32; nt <= 256; nt *= 2) {
      if (cg == 2 && nt < 128) continue;
      if (b_outer && nt / cg < 64) continue;
      if (nt > 32 && nt / 2 >= n && !(b_outer && nt / cg == 64) && !(cg == 2 && nt == 128)) continue;  // half of it would do
      const int64_t tiles = tm * ceil_div(n, nt);
      const float feed = (float)cut_bytes({cg, nt, 1}) / 56.0f, mma = 2.35f * (float)nt, each = feed > mma ? feed : mma;
      for (int sp : kSplits) {
        if (sp > 1 && (slices / sp < 4 || tiles * (sp - 1) > 4 * slot)) break;
        const float waves = (float)ceil_div(tiles * sp, slot);
        float t = waves * ((float)ceil_div(slices, sp) * each + 1500.0f);
        if (sp > 1) t += 4000.0f + 8.0f * (float)rows * (float)n * (float)sp / 2048.0f;
        if (t < least) {
          least = t;
          best = {cg, nt, sp};
        }
      }
    }
  }
  if (cost) *cost = least;
  return best;
}

int64_t parts_bytes(const Cut &c, int64_t rows, int64_t n) {
  return c.splits > 1 ? round_up(c.splits * rows * round_up(n, 8) * 4, 256) : 0;
}

std::atomic<int64_t> wait_limit{kWaitNs};  // nr_ops_wait_limit, from any thread

// an operand pair, its cut and what becomes of C
struct Task {
  Operand A, B;
  int64_t rows, inner;
  Cut c;
  Epilogue E;
  float *parts;  // scratch of parts_bytes(c, rows, E.n)
};

template <int CG>
cudaError_t launch_product(const CUtensorMap (&m)[4], const Job &J, uint32_t smem, int grid, int device, bool follows,
                           cudaStream_t s) {
  static std::atomic<bool> ready[64];  // the attribute is set once a device (twice by threads that race)
  if (!ready[device]) {
    const cudaError_t e =
        cudaFuncSetAttribute(product_kernel<CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMax);
    if (e != cudaSuccess) return e;
    ready[device] = true;
  }
  return launch(product_kernel<CG>, (unsigned)grid, dim3(kThreads), smem, s, follows, m[0], m[1], m[2], m[3], J);
}

// The products of one or two tasks (of the same CTAs a tile) in one launch, and
// what is left to finish, with the column sums' last addition, in another.
// follows: the call has launched before.
nr_status products(Task *t, int count, Finish &F, int device, bool follows, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  // the longer items first: the last turn is then a short one (36696 x 496 -> 170
  // backward 87 -> 74 us)
  if (count == 2 && ceil_div(t[1].inner, t[1].c.splits) * t[1].c.nt > ceil_div(t[0].inner, t[0].c.splits) * t[0].c.nt) {
    const Task first = t[1];
    t[1] = t[0];
    t[0] = first;
  }
  Job J = {};
  if (count > 0) {
    e = nr_ops_flag(device, &J.flag);
    if (e != cudaSuccess) return cuda_status(e);
    CUtensorMap maps[4];
    const int cg = t[0].c.cg;
    for (int q = 0; q < count; ++q) {
      const Task &k = t[q];
      if (!make_map(&maps[2 * q], k.A, k.E.dtype, k.A.outer ? kSlice : kRows) ||
          !make_map(&maps[2 * q + 1], k.B, k.E.dtype, k.B.outer ? kSlice : k.c.nt / cg))
        return NR_ERR_CUDA;
      Product &P = J.p[q];
      P.rows = k.rows;
      P.tiles_m = (int)ceil_div(k.rows, (int64_t)kRows * cg);
      P.tiles_n = (int)ceil_div(k.E.n, k.c.nt);
      P.nt = k.c.nt;
      P.slices = (int)ceil_div(k.inner, kSlice);
      P.splits = k.c.splits;
      P.a_outer = k.A.outer;
      P.b_outer = k.B.outer;
      P.idesc = tc::idesc_f16(kRows * cg, k.c.nt, k.E.dtype == NR_BF16, k.A.outer, k.B.outer);
      P.parts = k.parts;
      P.parts_ld = round_up(k.E.n, 8);
      P.E = k.E;
      const int64_t items = (int64_t)P.tiles_m * P.tiles_n * P.splits;
      if (items > (int64_t)1 << 29) return NR_ERR_INVALID_ARG;
      J.items += (int)items;
      if (q == 0) J.items0 = (int)items;
      if (k.c.nt > J.nt) J.nt = k.c.nt;
      if (cut_bytes(k.c) > J.stage_bytes) J.stage_bytes = cut_bytes(k.c);
      if (P.splits > 1) {
        F.p[q] = P;
        F.blocks[q] = (int)ceil_div(k.rows * ceil_div(k.E.n, kOpsGroup) * 4, 256);
      }
    }
    if (count == 1) maps[2] = maps[0], maps[3] = maps[1];
    const uint32_t fixed = 1024u + kEpiWarps * kStaging + (uint32_t)sizeof(Bars);
    J.stages = (int)((kSmemMax - fixed) / J.stage_bytes);
    if (J.stages > kStagesMax) J.stages = kStagesMax;
    J.wait_ns = wait_limit;
    const int slots = nr_ops_sms(device) / cg;
    const int grid = (J.items < slots ? J.items : slots) * cg;
    const uint32_t smem = fixed + (uint32_t)J.stages * J.stage_bytes;
    e = cg == 1 ? launch_product<1>(maps, J, smem, grid, device, follows, s)
                : launch_product<2>(maps, J, smem, grid, device, follows, s);
    follows = true;
  }
  const int64_t blocks = (int64_t)F.blocks[0] + F.blocks[1] + (F.dbias ? ceil_div(F.sums_n, 8) : 0);
  if (e == cudaSuccess && blocks > 0) e = launch(finish_kernel, (unsigned)blocks, dim3(256), 0, s, follows, F);
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}

// one or two matrices into aligned rows
cudaError_t pack(Operand *o, void *const *dst, int count, cudaStream_t s) {
  Pack K = {};
  int64_t blocks = 0;
  for (int q = 0; q < count; ++q) {
    K.s[q] = static_cast<const uint16_t *>(o[q].p);
    K.d[q] = static_cast<uint16_t *>(dst[q]);
    K.s_ld[q] = o[q].ld;
    K.rows[q] = o[q].rows;
    K.cols[q] = (int)o[q].cols;
    K.d_ld[q] = (int)round_up(o[q].cols, 8);
    blocks += ceil_div(o[q].rows * (K.d_ld[q] / 8), 256);
    if (q == 0) K.blocks0 = blocks;
    o[q].p = dst[q];
    o[q].ld = K.d_ld[q];
  }
  pack_kernel<<<(unsigned)blocks, 256, 0, s>>>(K);
  return cudaGetLastError();
}

bool valid(const nr_linear *a, bool backward) {
  if (!a || a->m < 0 || a->m > kOpsMaxRows || a->k < 1 || a->k > kOpsMaxCols || a->n < 1 || a->n > kOpsMaxCols)
    return false;
  if (!is_16bit(a->dtype) || (a->y_dtype != a->dtype && a->y_dtype != NR_F32) ||
      (a->bias_dtype != a->dtype && a->bias_dtype != NR_F32) || !act_ok(a->act) || !act_ok(a->x_act))
    return false;
  if (a->x_ld < 0 || a->w_ld < 0 || a->residual_ld < 0 || a->dy_ld < 0) return false;
  if (a->m > 0 && (!a->x || !a->w || !placed(a->x, a->dtype, a->x_scale) || !placed(a->w, a->dtype))) return false;
  if (!backward) {
    if (a->x_scale || a->x_act) return false;
    if (a->m > 0 && (!a->y || a->y_ld < a->n || (a->z && !a->z_scale && a->z_ld < a->n))) return false;
    if (a->m > 0 && (!placed(a->y, a->y_dtype) || !placed(a->z, a->dtype, a->z_scale) || !placed(a->residual, a->dtype) ||
                     !placed(a->bias, a->bias_dtype)))
      return false;
    return !(a->z_scale && !a->z);
  }
  if (a->x_act && !a->x_scale) return false;
  if (a->m > 0 && (!a->dy || (a->act != NR_ACT_NONE && !a->z))) return false;
  if (a->act != NR_ACT_NONE && !a->z_scale && a->z_ld < 0) return false;
  if (a->m > 0 && (!placed(a->dy, a->y_dtype) || (a->act != NR_ACT_NONE && !placed(a->z, a->dtype, a->z_scale)) ||
                   !placed(a->dx, a->dtype) || !placed(a->dw, a->dtype) || !placed(a->dbias, a->bias_dtype)))
    return false;
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

constexpr int kFewRows = 8;  // on CUDA cores up to here (figures at the top)
constexpr int64_t kRowsWarps = 16;  // warps an SM that keep enough of the weights in flight

struct ForwardPlan {
  bool few;
  Operand x, w;
  int64_t x_at = -1, w_at = -1, parts_at = -1, z_at = -1, bytes = 0;
  Cut cut = {1, 32, 1};
};
ForwardPlan plan_forward(const nr_linear *a, int sms) {
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
  f.cut = choose(a->m, a->n, ceil_div(a->k, kSlice), false, 0, sms);
  if (f.cut.splits > 1) f.parts_at = s.take(parts_bytes(f.cut, a->m, a->n));
  f.bytes = s.at;
  return f;
}

template <int MR, typename T>
void launch_rows(const nr_linear *a, const Epilogue &E, int sms, cudaStream_t s) {
  const T *x = static_cast<const T *>(a->x), *w = static_cast<const T *>(a->w);
  const int vec = vec_ok(a->x, a->x_ld, a->dtype) && vec_ok(a->w, a->w_ld, a->dtype);
  const int64_t want = sms * kRowsWarps;
  // Four columns a warp where that fills the GPU, with t in parts for four rows and
  // more, whose conversions for one column cost more than its products (1536 ->
  // 6144: four rows 11.0 -> 8.4 us, eight 18.2 -> 15.6). Else one column, and t split
  // over warps.
  const int nr = a->n >= 4 * want || (MR >= 4 && a->n * (a->k / 512) >= 4 * want && a->n >= want) ? 4 : 1;
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

// dz_kernel's blocks: threads across up to 256 columns, rows of few columns share a
// block; enough blocks for the GPU, at most 1024 rows of column sums to add
struct DzCut {
  dim3 block;
  int gx, gy, rows;
};
DzCut cut_dz(int64_t m, int64_t n, int sms) {
  DzCut c;
  unsigned bx = 4;
  while (bx < 32 && (int64_t)bx * 8 < n) bx *= 2;
  c.block = dim3(bx, 256 / bx);
  c.gx = (int)ceil_div(n, (int64_t)bx * 8);
  const int64_t most = ceil_div((int64_t)sms * 6, c.gx);
  const int64_t step = kDzRows * (int64_t)c.block.y;
  c.rows = (int)round_up(ceil_div(m, most < 1024 ? most : 1024), step);
  c.gy = (int)ceil_div(m, c.rows);
  return c;
}

struct BackwardPlan {
  bool make_dz;  // else dy serves as it is
  Operand dz, x, w;
  DzCut cut;
  int64_t dz_at = -1, x_at = -1, w_at = -1, sums_at = -1, dx_at = -1, dw_at = -1, bytes = 0;
  Cut dx = {1, 64, 1}, dw = {1, 64, 1};
};
BackwardPlan plan_backward(const nr_linear *a, int sms) {
  BackwardPlan b;
  Scratch s;
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
  b.cut = cut_dz(m, n, sms);
  if (a->dbias) b.sums_at = s.take((int64_t)b.cut.gy * n * 4);
  if (a->dw && (a->x_scale || !mappable(b.x))) {
    b.x_at = s.take(m * round_up(k, 8) * 2);
    if (a->x_scale) b.x.ld = round_up(k, 8);
  }
  if (a->dx && !mappable(b.w)) b.w_at = s.take(n * round_up(k, 8) * 2);
  // both in one launch, so of the same CTAs a tile
  float cost[2] = {0.0f, 0.0f};
  const int only = a->dx && a->dw ? 2 : 0;
  const int64_t sx = ceil_div(n, kSlice), sw = ceil_div(m, kSlice);
  if (a->dx) b.dx = choose(m, k, sx, true, only, sms, &cost[0]);
  if (a->dw) b.dw = choose(n, k, sw, true, only, sms, &cost[1]);
  if (only) {
    float c1[2];
    const Cut dx1 = choose(m, k, sx, true, 1, sms, &c1[0]), dw1 = choose(n, k, sw, true, 1, sms, &c1[1]);
    if (c1[0] + c1[1] < cost[0] + cost[1]) b.dx = dx1, b.dw = dw1;
  }
  if (a->dx && b.dx.splits > 1) b.dx_at = s.take(parts_bytes(b.dx, m, k));
  if (a->dw && b.dw.splits > 1) b.dw_at = s.take(parts_bytes(b.dw, n, k));
  b.bytes = s.at;
  return b;
}

template <bool VEC, typename D, typename T>
void launch_dz(const nr_linear *a, const BackwardPlan &b, const Saved &z, void *dz, float *sums, cudaStream_t s) {
  dz_kernel<VEC, D, T><<<dim3((unsigned)b.cut.gx, (unsigned)b.cut.gy), b.cut.block, 0, s>>>(
      static_cast<const D *>(a->dy), a->dy_ld, z, (int)a->act, a->m, (int)a->n, b.cut.rows, static_cast<T *>(dz), b.dz.ld,
      sums);
}
template <typename T>
void launch_dz_any(const nr_linear *a, const BackwardPlan &b, const Saved &z, void *dz, float *sums, cudaStream_t s) {
  const bool vec = a->n % 8 == 0 && vec_ok(a->dy, a->dy_ld, a->y_dtype) &&
                   (a->act == NR_ACT_NONE || z.scale || vec_ok(a->z, a->z_ld, a->dtype));
  if (a->y_dtype == NR_F32)
    vec ? launch_dz<true, float, T>(a, b, z, dz, sums, s) : launch_dz<false, float, T>(a, b, z, dz, sums, s);
  else
    vec ? launch_dz<true, T, T>(a, b, z, dz, sums, s) : launch_dz<false, T, T>(a, b, z, dz, sums, s);
}

void *at(void *ws, int64_t o) { return o < 0 ? nullptr : static_cast<char *>(ws) + o; }

}  // namespace

extern "C" int64_t nr_linear_forward_workspace(const nr_linear *a, int device) {
  if (!valid(a, false)) return NR_ERR_INVALID_ARG;
  const int sms = nr_ops_sms(device);
  return sms > 0 ? plan_forward(a, sms).bytes : (int64_t)NR_ERR_CUDA;
}

extern "C" nr_status nr_linear_forward(const nr_linear *a, int device, void *ws, int64_t ws_bytes, void *stream) {
  if (!valid(a, false)) return NR_ERR_INVALID_ARG;
  if (a->m == 0) return NR_OK;
  const int sms = nr_ops_sms(device);
  if (sms < 1) return NR_ERR_CUDA;
  ForwardPlan f = plan_forward(a, sms);
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
  E.residual_end = static_cast<const uint16_t *>(a->residual) + (a->m - 1) * a->residual_ld + a->n;
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
    if (a->dtype == NR_F16) launch_rows_any<__half>(a, E, sms, s);
    else launch_rows_any<__nv_bfloat16>(a, E, sms, s);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_status(e);
    return a->z_scale ? nr_checkpoint8_write(E.z, NR_F32, a->m, a->n, a->n, a->z, a->z_scale, device, stream) : NR_OK;
  }
  Operand o[2];
  void *dst[2];
  int packs = 0;
  if (f.x_at >= 0) o[packs] = f.x, dst[packs++] = at(ws, f.x_at);
  if (f.w_at >= 0) o[packs] = f.w, dst[packs++] = at(ws, f.w_at);
  if (packs) {
    const cudaError_t e = pack(o, dst, packs, s);
    if (e != cudaSuccess) return cuda_status(e);
    if (f.x_at >= 0) f.x = o[0];
    if (f.w_at >= 0) f.w = o[packs - 1];
  }
  Finish F = {};
  Task t = {f.x, f.w, a->m, a->k, f.cut, E, static_cast<float *>(at(ws, f.parts_at))};
  return products(&t, 1, F, device, packs > 0, s);
}

extern "C" int64_t nr_linear_backward_workspace(const nr_linear *a, int device) {
  if (!valid(a, true)) return NR_ERR_INVALID_ARG;
  const int sms = nr_ops_sms(device);
  return sms > 0 ? plan_backward(a, sms).bytes : (int64_t)NR_ERR_CUDA;
}

extern "C" nr_status nr_linear_backward(const nr_linear *a, int device, void *ws, int64_t ws_bytes, void *stream) {
  if (!valid(a, true)) return NR_ERR_INVALID_ARG;
  const int sms = nr_ops_sms(device);
  if (sms < 1) return NR_ERR_CUDA;
  BackwardPlan b = plan_backward(a, sms);
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
  bool follows = false;  // a launch of this call has been made
  if (a->dw && a->x_scale) {
    const nr_status st =
        nr_checkpoint8_read(a->x, a->x_scale, m, k, (int)a->x_act, at(ws, b.x_at), dt, b.x.ld, device, stream);
    if (st != NR_OK) return st;
    b.x.p = at(ws, b.x_at);
  }
  Operand o[2];
  void *dst[2];
  int packs = 0;
  const bool pack_x = a->dw && !a->x_scale && b.x_at >= 0, pack_w = a->dx && b.w_at >= 0;
  if (pack_x) o[packs] = b.x, dst[packs++] = at(ws, b.x_at);
  if (pack_w) o[packs] = b.w, dst[packs++] = at(ws, b.w_at);
  if (packs) {
    e = pack(o, dst, packs, s);
    if (e != cudaSuccess) return cuda_status(e);
    if (pack_x) b.x = o[0];
    if (pack_w) b.w = o[packs - 1];
  }
  Finish F = {};
  if (b.dz_at >= 0 || a->dbias) {
    const Saved z = {a->z, static_cast<const uint8_t *>(a->z_scale), a->z_ld, (int)ceil_div(n, kOpsGroup)};
    float *sums = static_cast<float *>(at(ws, b.sums_at));
    if (dt == NR_F16) launch_dz_any<__half>(a, b, z, at(ws, b.dz_at), sums, s);
    else launch_dz_any<__nv_bfloat16>(a, b, z, at(ws, b.dz_at), sums, s);
    e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_status(e);
    if (b.dz_at >= 0) b.dz.p = at(ws, b.dz_at);
    follows = true;
    if (a->dbias) {
      F.sums = sums;
      F.sums_rows = b.cut.gy;
      F.sums_n = n;
      F.dbias = a->dbias;
      F.dbias_dtype = (int)a->bias_dtype;
    }
  }
  Task t[2];
  int count = 0;
  Epilogue E = {};
  E.dtype = E.y_dtype = dt;
  E.n = k;
  if (a->dx) {
    E.y = a->dx;
    E.y_ld = a->dx_ld;
    E.y_vec = vec_ok(E.y, E.y_ld, dt);
    t[count++] = {b.dz, b.w, m, n, b.dx, E, static_cast<float *>(at(ws, b.dx_at))};
  }
  if (a->dw) {
    E.y = a->dw;
    E.y_ld = k;
    E.y_vec = vec_ok(E.y, E.y_ld, dt);
    Operand dzt = b.dz;
    dzt.outer = true;
    t[count++] = {dzt, b.x, n, m, b.dw, E, static_cast<float *>(at(ws, b.dw_at))};
  }
  return products(t, count, F, device, follows, s);
}

extern "C" nr_status nr_ops_wait_limit(int64_t us) {
  if (us > 60000000) return NR_ERR_INVALID_ARG;
  wait_limit = us == 0 ? kWaitNs : us < 0 ? (int64_t)-1 : us * 1000;
  return NR_OK;
}
