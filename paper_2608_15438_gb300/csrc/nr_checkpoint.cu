// 8-bit activation checkpoints (neuroute_ops.h): groups of 32 columns of a row
// share a power-of-two scale. A thread holds a group.
#include <cuda_runtime.h>
#include <stdint.h>

#include "nrq_ops.cuh"

namespace {

__global__ void __launch_bounds__(256)
    write8_kernel(const void *x, int dtype, int64_t m, int64_t n, int64_t groups, int64_t x_ld,
                  int8_t *codes, uint8_t *scales) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= m * groups) return;
  const int64_t i = e / groups, c0 = (e - i * groups) * kOpsGroup;
  float v[kOpsGroup];
  uint32_t top = 0;
#pragma unroll
  for (int c = 0; c < kOpsGroup; ++c) {
    v[c] = c0 + c < n ? load_any(x, i * x_ld + c0 + c, dtype) : 0.0f;
    top = max(top, __float_as_uint(v[c]) & 0x7fffffffu);
  }
  const uint32_t s = held8_scale(top);
  const float up = held8_up(s);
  scales[e] = (uint8_t)s;
#pragma unroll
  for (int c = 0; c < kOpsGroup; ++c) codes[e * kOpsGroup + c] = (int8_t)held8_code(v[c], up);
}

__global__ void __launch_bounds__(256)
    read8_kernel(const int8_t *codes, const uint8_t *scales, int64_t m, int64_t n, int64_t groups, int act,
                 void *y, int dtype, int64_t y_ld) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= m * groups) return;
  const int64_t i = e / groups, c0 = (e - i * groups) * kOpsGroup;
  const float down = held8_down(scales[e]);
#pragma unroll
  for (int c = 0; c < kOpsGroup; ++c) {
    if (c0 + c >= n) break;
    float v = act_value((float)codes[e * kOpsGroup + c] * down, act);
    if (dtype == NR_F16 && fabsf(v) > 65504.0f) v = copysignf(65504.0f, v);
    store_any(y, i * y_ld + c0 + c, dtype, v);
  }
}

bool valid(const void *codes, const void *scales, const void *v, int64_t m, int64_t n, int dtype) {
  if (m < 0 || m > kOpsMaxRows || n < 1 || n > kOpsMaxCols || dtype < NR_F32 || dtype > NR_BF16) return false;
  return m == 0 || (codes && scales && v && (reinterpret_cast<uintptr_t>(codes) & 15) == 0);
}

}  // namespace

extern "C" nr_status nr_checkpoint8_write(const void *x, int dtype, int64_t m, int64_t n, int64_t x_ld, void *codes,
                                          void *scales, int device, void *stream) {
  if (!valid(codes, scales, x, m, n, dtype) || x_ld < 0) return NR_ERR_INVALID_ARG;
  if (m == 0) return NR_OK;
  DeviceGuard g(device);
  if (!g.ok) return NR_ERR_CUDA;
  const int64_t groups = ceil_div(n, kOpsGroup);
  write8_kernel<<<(unsigned)ceil_div(m * groups, 256), 256, 0, static_cast<cudaStream_t>(stream)>>>(
      x, dtype, m, n, groups, x_ld, static_cast<int8_t *>(codes), static_cast<uint8_t *>(scales));
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}

extern "C" nr_status nr_checkpoint8_read(const void *codes, const void *scales, int64_t m, int64_t n, int act, void *y,
                                         int dtype, int64_t y_ld, int device, void *stream) {
  if (!valid(codes, scales, y, m, n, dtype) || !act_ok(act) || y_ld < n) return NR_ERR_INVALID_ARG;
  if (m == 0) return NR_OK;
  DeviceGuard g(device);
  if (!g.ok) return NR_ERR_CUDA;
  const int64_t groups = ceil_div(n, kOpsGroup);
  read8_kernel<<<(unsigned)ceil_div(m * groups, 256), 256, 0, static_cast<cudaStream_t>(stream)>>>(
      static_cast<const int8_t *>(codes), static_cast<const uint8_t *>(scales), m, n, groups, act, y, dtype, y_ld);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}

// ------------------------------------------------------------ devices
namespace {
constexpr int kOpsDevices = 64;
__device__ int ops_flag;
}  // namespace

int nr_ops_sms(int device) {
  static int sms[kOpsDevices];  // 0: not looked up yet; a race writes the same value
  if (device < 0 || device >= kOpsDevices) return 1;
  if (sms[device] == 0) {
    int v = 0;
    if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || v < 1) {
      cudaGetLastError();
      return 1;
    }
    sms[device] = v;
  }
  return sms[device];
}

cudaError_t nr_ops_flag(int device, int **flag) {
  static int *flags[kOpsDevices];
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
