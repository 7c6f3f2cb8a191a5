// 8-bit activation checkpoints (neuroute_ops.h): groups of 32 columns of a row
// share a power-of-two scale. Bound by memory in both directions: a value's 2 or 4
// bytes one way and 1 + 1/32 the other. Measured at 262144 x 1536 in bf16: written in
// 255 us (4.8 TB/s), read in 223 (5.5 TB/s); 65536 x 6144 both in 415 us, 5.9 TB/s.
// Odd widths shift and share aligned blocks: 200000 x 771 written in 208 us, read in 151
// (2.3, 3.1 TB/s).
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "nrq_ops.cuh"

namespace {

constexpr int kThreads = 256, kBlocks = 6, kBatch = 4;  // blocks an SM, rows at a time

// the fp32 bits of the largest magnitude: 16-bit types are ordered like their
// bits without the sign
template <typename T>
__device__ __forceinline__ uint32_t largest(const Eight<T> &o) {
  if (sizeof(T) == 4) {
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) top = max(top, o.r[q] & 0x7fffffffu);
    return top;
  }
  uint32_t top = o.r[0] & 0x7fff7fffu;
#pragma unroll
  for (int q = 1; q < 4; ++q) top = __vmaxu2(top, o.r[q] & 0x7fff7fffu);
  top = max(top & 0xffffu, top >> 16);
  return __float_as_uint(unpack2(top, TypeCode<T>::code).x);
}
// Threads of a block: x along a row (eight columns each, four threads a group),
// y over rows; a thread takes kBatch rows at a time, all their loads first.
// VEC: n is a multiple of 8 and the rows take 16-byte accesses.
template <bool VEC, typename T>
__global__ void __launch_bounds__(kThreads)
    write8_kernel(const T *x, int64_t m, int n, int groups, int64_t x_ld, int8_t *codes, uint8_t *scales) {
  const T *end = x + (m - 1) * x_ld + n;
  const int j = (blockIdx.x * blockDim.x + threadIdx.x) * 8;
  const int count = max(0, min(8, n - j));
  const bool in = j < groups * kOpsGroup;
  const int64_t step = (int64_t)gridDim.y * blockDim.y;
  const unsigned lanes = 0xfu << ((threadIdx.y * blockDim.x + threadIdx.x) & 28);
  for (int64_t i0 = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; i0 < m; i0 += step * kBatch) {
    Eight<T> v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      v[u] = VEC && count <= 0 ? Eight<T>{} : fetch_eight<T>(x + min(i0 + u * step, m - 1) * x_ld + j, VEC, VEC ? 8 : count, x, end);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int64_t i = i0 + u * step;
      if (!VEC) settle_eight<T>(v[u], x + min(i, m - 1) * x_ld + j, VEC, count, x, end);
      uint32_t top = largest<T>(v[u]);
      top = max(top, __shfl_xor_sync(lanes, top, 1));
      top = max(top, __shfl_xor_sync(lanes, top, 2));
      const uint32_t s = held8_scale(top);
      const float up = held8_up(s);
      if (!in || i >= m) continue;
      *reinterpret_cast<uint2 *>(codes + i * groups * kOpsGroup + j) =
          make_uint2(held8_codes(pair_of<T>(v[u], 0), pair_of<T>(v[u], 1), up, s),
                     held8_codes(pair_of<T>(v[u], 2), pair_of<T>(v[u], 3), up, s));
      if ((threadIdx.x & 3) == 0) scales[i * groups + (j >> 5)] = (uint8_t)s;
    }
  }
}

template <bool VEC, typename T>
__global__ void __launch_bounds__(kThreads)
    read8_kernel(const int8_t *codes, const uint8_t *scales, int64_t m, int n, int groups, int act, T *y, int64_t y_ld) {
  const int j = (blockIdx.x * blockDim.x + threadIdx.x) * 8, count = max(0, min(8, n - j));
  const int64_t step = (int64_t)gridDim.y * blockDim.y;
  // the lanes of a warp that share a row, for stores at any address
  const int lane = (threadIdx.y * blockDim.x + threadIdx.x) & 31, share = min((int)blockDim.x, 32);
  const unsigned lanes = share == 32 ? 0xffffffffu : ((1u << share) - 1u) << (lane & ~(share - 1));
  const bool prev = (lane & (share - 1)) != 0, next = (lane & (share - 1)) != share - 1;
  const int jc = min(j, groups * kOpsGroup - 8);  // lanes past the row load its last eight
  for (int64_t i0 = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; i0 < m; i0 += step * kBatch) {
    uint2 c[kBatch];
    uint32_t s[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int64_t i = min(i0 + u * step, m - 1);
      c[u] = __ldg(reinterpret_cast<const uint2 *>(codes + i * groups * kOpsGroup + jc));
      s[u] = __ldg(scales + i * groups + (jc >> 5));
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int64_t i = i0 + u * step;
      if (i >= m) break;
      const float down = held8_down(s[u]);
      float2 p[4];
      held8_numbers(c[u].x, p[0], p[1]);
      held8_numbers(c[u].y, p[2], p[3]);
#pragma unroll
      for (int q = 0; q < 4; ++q) p[q] = mul2(p[q], both(down));
      if (act != NR_ACT_NONE) {
#pragma unroll
        for (int q = 0; q < 4; ++q) p[q] = act_value2(p[q], act);
      }
      if (TypeCode<T>::code == NR_F16 && s[u] >= kHeld8F16) {
#pragma unroll
        for (int q = 0; q < 4; ++q) p[q] = held8_in_f16(p[q]);
      }
      const float v[8] = {p[0].x, p[0].y, p[1].x, p[1].y, p[2].x, p[2].y, p[3].x, p[3].y};
      if (VEC || sizeof(T) == 4) {
        if (count > 0) store8(y + i * y_ld, j, TypeCode<T>::code, VEC, VEC ? 8 : count, v);
      } else {
        const uint4 h = pack8(p, TypeCode<T>::code);
        const uint32_t w[4] = {h.x, h.y, h.z, h.w};
        store16x8(y + i * y_ld + j, n - j, w, prev, next, lanes);
      }
    }
  }
}

// the block's shape and the grid: rows of few columns share a block
void cut(int64_t m, int64_t n, int sms, dim3 &grid, dim3 &block) {
  const int64_t segs = ceil_div(n, kOpsGroup) * 4;
  unsigned bx = 4;
  while (bx < (unsigned)kThreads && bx < segs) bx *= 2;
  block = dim3(bx, kThreads / bx);
  const int64_t gx = ceil_div(segs, bx), rows = ceil_div(m, block.y), most = ceil_div((int64_t)sms * kBlocks, gx);
  grid = dim3((unsigned)gx, (unsigned)(rows < most ? rows : most));
}

bool valid(const void *codes, const void *scales, const void *v, int64_t m, int64_t n, int dtype) {
  if (m < 0 || m > kOpsMaxRows || n < 1 || n > kOpsMaxCols || dtype < NR_F32 || dtype > NR_BF16) return false;
  return m == 0 || (codes && scales && v && placed(codes, dtype, true) && placed(v, dtype));
}

}  // namespace

extern "C" nr_status nr_checkpoint8_write(const void *x, int dtype, int64_t m, int64_t n, int64_t x_ld, void *codes,
                                          void *scales, int device, void *stream) {
  if (!valid(codes, scales, x, m, n, dtype) || x_ld < 0) return NR_ERR_INVALID_ARG;
  if (m == 0) return NR_OK;
  const int sms = nr_ops_sms(device);
  DeviceGuard g(device);
  if (sms < 1 || !g.ok) return NR_ERR_CUDA;
  const int64_t groups = ceil_div(n, kOpsGroup);
  dim3 grid, block;
  cut(m, n, sms, grid, block);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool vec = n % 8 == 0 && vec_ok(x, x_ld, dtype);
  int8_t *c = static_cast<int8_t *>(codes);
  uint8_t *sc = static_cast<uint8_t *>(scales);
#define NR_WRITE8(T)                                                                                             \
  if (vec) write8_kernel<true, T><<<grid, block, 0, s>>>(static_cast<const T *>(x), m, (int)n, (int)groups, x_ld, c, sc); \
  else write8_kernel<false, T><<<grid, block, 0, s>>>(static_cast<const T *>(x), m, (int)n, (int)groups, x_ld, c, sc);
  if (dtype == NR_F32) {
    NR_WRITE8(float)
  } else if (dtype == NR_F16) {
    NR_WRITE8(__half)
  } else {
    NR_WRITE8(__nv_bfloat16)
  }
#undef NR_WRITE8
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}

extern "C" nr_status nr_checkpoint8_read(const void *codes, const void *scales, int64_t m, int64_t n, int act, void *y,
                                         int dtype, int64_t y_ld, int device, void *stream) {
  if (!valid(codes, scales, y, m, n, dtype) || !act_ok(act) || y_ld < n) return NR_ERR_INVALID_ARG;
  if (m == 0) return NR_OK;
  const int sms = nr_ops_sms(device);
  DeviceGuard g(device);
  if (sms < 1 || !g.ok) return NR_ERR_CUDA;
  const int64_t groups = ceil_div(n, kOpsGroup);
  dim3 grid, block;
  cut(m, n, sms, grid, block);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool vec = n % 8 == 0 && vec_ok(y, y_ld, dtype);
  const int8_t *c = static_cast<const int8_t *>(codes);
  const uint8_t *sc = static_cast<const uint8_t *>(scales);
#define NR_READ8(T)                                                                                            \
  if (vec) read8_kernel<true, T><<<grid, block, 0, s>>>(c, sc, m, (int)n, (int)groups, act, static_cast<T *>(y), y_ld); \
  else read8_kernel<false, T><<<grid, block, 0, s>>>(c, sc, m, (int)n, (int)groups, act, static_cast<T *>(y), y_ld);
  if (dtype == NR_F32) {
    NR_READ8(float)
  } else if (dtype == NR_F16) {
    NR_READ8(__half)
  } else {
    NR_READ8(__nv_bfloat16)
  }
#undef NR_READ8
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}

// ------------------------------------------------------------ devices
namespace {
constexpr int kOpsDevices = 64;
__device__ int ops_flag;
}  // namespace

int nr_ops_sms(int device) {
  static std::atomic<int> sms[kOpsDevices];  // 0: not looked up yet; threads that race write the same value
  if (device < 0 || device >= kOpsDevices) return 0;
  if (sms[device] == 0) {
    int v = 0;
    if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || v < 1) {
      cudaGetLastError();
      return 0;
    }
    sms[device] = v;
  }
  return sms[device];
}

cudaError_t nr_ops_flag(int device, int **flag) {
  static std::atomic<int *> flags[kOpsDevices];
  if (device < 0 || device >= kOpsDevices) return cudaErrorInvalidDevice;
  if (!flags[device]) {
    void *p = nullptr;
    const cudaError_t e = cudaGetSymbolAddress(&p, ops_flag);  // of the current device
    if (e != cudaSuccess) return e;
    flags[device] = static_cast<int *>(p);
  }
  *flag = flags[device];
  return cudaSuccess;
}

extern "C" nr_status nr_ops_status(int device) {
  DeviceGuard g(device);
  if (!g.ok) return NR_ERR_CUDA;
  int *flag = nullptr, v = 0;
  cudaError_t e = nr_ops_flag(device, &flag);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpy(&v, flag, sizeof(int), cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && v != 0) {
    e = cudaMemset(flag, 0, sizeof(int));
    if (e == cudaSuccess) return NR_ERR_DEVICE_CHECK;
  }
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}
