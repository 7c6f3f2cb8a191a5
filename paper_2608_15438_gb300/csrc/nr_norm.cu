// Layer norm of residual encoders (neuroute_ops.h), simple form: a block a row;
// the parameters' gradients by a block for every 32 columns.
#include <cuda_runtime.h>
#include <stdint.h>

#include "nrq_ops.cuh"

namespace {

constexpr int kThreads = 256;

// values of a type, or a checkpoint's codes and scales
struct Rows {
  const void *p;
  const uint8_t *scale;
  int64_t ld;
  int dtype;
  int64_t groups;
};
__device__ __forceinline__ float row_at(const Rows &s, int64_t i, int64_t j) {
  if (!s.scale) return load_any(s.p, i * s.ld + j, s.dtype);
  return (float)static_cast<const int8_t *>(s.p)[i * s.groups * kOpsGroup + j] *
         held8_down(s.scale[i * s.groups + j / kOpsGroup]);
}

__device__ __forceinline__ float block_sum(float v) {
  __shared__ float part[kThreads / 32];
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0f;
  for (int w = 0; w < kThreads / 32; ++w) v += part[w];
  return v;
}

__global__ void __launch_bounds__(kThreads)
    norm_forward_kernel(Rows x, int64_t n, const void *weight, const void *bias, int w_dtype, float eps, void *y,
                        int64_t y_ld, int dtype, float *mean_out, float *rstd_out) {
  const int64_t i = blockIdx.x;
  float s = 0.0f;
  for (int64_t j = threadIdx.x; j < n; j += kThreads) s += row_at(x, i, j);
  const float mean = block_sum(s) / (float)n;
  s = 0.0f;
  for (int64_t j = threadIdx.x; j < n; j += kThreads) {
    const float d = row_at(x, i, j) - mean;
    s = fmaf(d, d, s);
  }
  const float rstd = 1.0f / sqrtf(block_sum(s) / (float)n + eps);
  for (int64_t j = threadIdx.x; j < n; j += kThreads) {
    const float g = weight ? load_any(weight, j, w_dtype) : 1.0f, b = bias ? load_any(bias, j, w_dtype) : 0.0f;
    store_any(y, i * y_ld + j, dtype, fmaf((row_at(x, i, j) - mean) * rstd, g, b));
  }
  if (mean_out && threadIdx.x == 0) {
    mean_out[i] = mean;
    rstd_out[i] = rstd;
  }
}

__global__ void __launch_bounds__(kThreads)
    norm_dx_kernel(const void *dy, int64_t dy_ld, Rows x, int64_t n, const void *weight, int w_dtype,
                   const float *mean, const float *rstd, const void *dres, int64_t dres_ld, void *dx, int64_t dx_ld,
                   int dtype) {
  const int64_t i = blockIdx.x;
  const float mu = mean[i], rs = rstd[i];
  float s1 = 0.0f, s2 = 0.0f;
  for (int64_t j = threadIdx.x; j < n; j += kThreads) {
    const float g = load_any(dy, i * dy_ld + j, dtype) * (weight ? load_any(weight, j, w_dtype) : 1.0f);
    s1 += g;
    s2 = fmaf(g, (row_at(x, i, j) - mu) * rs, s2);
  }
  const float m1 = block_sum(s1) / (float)n, m2 = block_sum(s2) / (float)n;
  for (int64_t j = threadIdx.x; j < n; j += kThreads) {
    const float g = load_any(dy, i * dy_ld + j, dtype) * (weight ? load_any(weight, j, w_dtype) : 1.0f);
    float d = rs * (g - m1 - (row_at(x, i, j) - mu) * rs * m2);
    if (dres) d += load_any(dres, i * dres_ld + j, dtype);
    store_any(dx, i * dx_ld + j, dtype, d);
  }
}

__global__ void __launch_bounds__(256)
    norm_dparam_kernel(const void *dy, int64_t dy_ld, Rows x, int64_t m, int64_t n, const float *mean,
                       const float *rstd, int dtype, void *dweight, void *dbias, int w_dtype) {
  __shared__ float pw[8][33], pb[8][33];
  const int c = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int64_t j = (int64_t)blockIdx.x * 32 + c;
  float w = 0.0f, b = 0.0f;
  if (j < n)
    for (int64_t i = r; i < m; i += 8) {
      const float v = load_any(dy, i * dy_ld + j, dtype);
      b += v;
      w = fmaf(v, (row_at(x, i, j) - mean[i]) * rstd[i], w);
    }
  pw[r][c] = w;
  pb[r][c] = b;
  __syncthreads();
  if (r == 0 && j < n) {
    for (int q = 1; q < 8; ++q) {
      w += pw[q][c];
      b += pb[q][c];
    }
    store_any(dweight, j, w_dtype, w);
    store_any(dbias, j, w_dtype, b);
  }
}

bool valid(const nr_layer_norm *a, bool backward) {
  if (!a || a->m < 0 || a->m > kOpsMaxRows || a->n < 1 || a->n > kOpsMaxCols) return false;
  if (a->dtype < NR_F32 || a->dtype > NR_BF16 || (a->w_dtype != a->dtype && a->w_dtype != NR_F32)) return false;
  if (a->x_ld < 0 || a->dy_ld < 0 || a->residual_grad_ld < 0 || (a->m > 0 && !a->x)) return false;
  if (!backward)
    return a->eps > 0.0 && !a->mean == !a->rstd && (a->m == 0 || (a->y && a->y_ld >= a->n));
  return !a->dweight == !a->dbias &&
         (a->m == 0 || (a->dy && a->mean && a->rstd && a->dx && a->dx_ld >= a->n));
}

Rows rows_of(const nr_layer_norm *a) {
  return {a->x, static_cast<const uint8_t *>(a->x_scale), a->x_ld, (int)a->dtype, ceil_div(a->n, kOpsGroup)};
}

}  // namespace

extern "C" nr_status nr_layer_norm_forward(const nr_layer_norm *a, int device, void *stream) {
  if (!valid(a, false)) return NR_ERR_INVALID_ARG;
  if (a->m == 0) return NR_OK;
  DeviceGuard g(device);
  if (!g.ok) return NR_ERR_CUDA;
  norm_forward_kernel<<<(unsigned)a->m, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(
      rows_of(a), a->n, a->weight, a->bias, (int)a->w_dtype, (float)a->eps, a->y, a->y_ld, (int)a->dtype, a->mean,
      a->rstd);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}

extern "C" int64_t nr_layer_norm_backward_workspace(const nr_layer_norm *a, int) { return valid(a, true) ? 0 : -1; }

extern "C" nr_status nr_layer_norm_backward(const nr_layer_norm *a, int device, void *, int64_t, void *stream) {
  if (!valid(a, true)) return NR_ERR_INVALID_ARG;
  DeviceGuard g(device);
  if (!g.ok) return NR_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a->m == 0) {
    cudaError_t e = cudaSuccess;
    if (a->dweight) {
      e = cudaMemsetAsync(a->dweight, 0, (size_t)a->n * type_bytes(a->w_dtype), s);
      if (e == cudaSuccess) e = cudaMemsetAsync(a->dbias, 0, (size_t)a->n * type_bytes(a->w_dtype), s);
    }
    return e == cudaSuccess ? NR_OK : cuda_status(e);
  }
  norm_dx_kernel<<<(unsigned)a->m, kThreads, 0, s>>>(a->dy, a->dy_ld, rows_of(a), a->n, a->weight, (int)a->w_dtype,
                                                     a->mean, a->rstd, a->residual_grad, a->residual_grad_ld, a->dx,
                                                     a->dx_ld, (int)a->dtype);
  if (a->dweight)
    norm_dparam_kernel<<<(unsigned)ceil_div(a->n, 32), 256, 0, s>>>(a->dy, a->dy_ld, rows_of(a), a->m, a->n, a->mean,
                                                                    a->rstd, (int)a->dtype, a->dweight, a->dbias,
                                                                    (int)a->w_dtype);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}
