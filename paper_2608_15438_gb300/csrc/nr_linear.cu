// The linear layer of residual encoders (neuroute_ops.h):
//   forward   z = x w^T + bias, y = act(z) + residual
//   backward  dz = dy act'(z); dx = dz w, dw = dz^T x, dbias = sum of dz's rows
//
// Simple form: one matrix product kernel on CUDA cores that reads both
// operands through two strides each, so that every product above is one
// launch of it; dz, the input's 8-bit form and the column sums are kernels of
// their own around it.
#include <cuda_runtime.h>
#include <stdint.h>

#include "nrq_ops.cuh"

namespace {

// C[i, j] = sum_t A[i, t] B[j, t], A[i, t] at a + i * ai + t * at (elements)
struct Operand {
  const void *p;
  int64_t row, inner;
};

// what becomes of the sums: y = act(sum + bias) + residual, and z = sum + bias
struct Epilogue {
  const void *bias;
  int bias_dtype, act;
  const void *residual;  // of the product's type
  int64_t residual_ld;
  void *y;
  int y_dtype;
  int64_t y_ld;
  void *z;
  int z_dtype;
  int64_t z_ld;
};

constexpr int kTile = 64, kSlab = 16;

template <typename T>
__global__ void __launch_bounds__(256)
    product_kernel(Operand A, Operand B, int64_t m, int64_t n, int64_t k, int dtype, Epilogue E) {
  __shared__ float sa[kSlab][kTile + 1], sb[kSlab][kTile + 1];
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int64_t i0 = (int64_t)blockIdx.x * kTile, j0 = (int64_t)blockIdx.y * kTile;
  const T *a = static_cast<const T *>(A.p), *b = static_cast<const T *>(B.p);
  float acc[4][4] = {};
  for (int64_t t0 = 0; t0 < k; t0 += kSlab) {
    for (int e = tid; e < kTile * kSlab; e += 256) {
      // the index that runs over consecutive addresses runs over the lanes
      const int ra = A.inner == 1 ? e / kSlab : e % kTile, ta = A.inner == 1 ? e % kSlab : e / kTile;
      const int rb = B.inner == 1 ? e / kSlab : e % kTile, tb = B.inner == 1 ? e % kSlab : e / kTile;
      sa[ta][ra] = i0 + ra < m && t0 + ta < k ? to_f32(a[(i0 + ra) * A.row + (t0 + ta) * A.inner]) : 0.0f;
      sb[tb][rb] = j0 + rb < n && t0 + tb < k ? to_f32(b[(j0 + rb) * B.row + (t0 + tb) * B.inner]) : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kSlab; ++t)
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[u][v] = fmaf(sa[t][ty + 16 * u], sb[t][tx + 16 * v], acc[u][v]);
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int64_t i = i0 + ty + 16 * u, j = j0 + tx + 16 * v;
      if (i >= m || j >= n) continue;
      float z = acc[u][v];
      if (E.bias) z += load_any(E.bias, j, E.bias_dtype);
      if (E.z) store_any(E.z, i * E.z_ld + j, E.z_dtype, z);
      float y = act_value(z, E.act);
      if (E.residual) y += load_any(E.residual, i * E.residual_ld + j, dtype);
      store_any(E.y, i * E.y_ld + j, E.y_dtype, y);
    }
}

// z's element (i, j): values of a type, or a checkpoint's codes and scales
struct Saved {
  const void *p;
  const uint8_t *scale;
  int64_t ld;
  int dtype;
  int64_t groups;
};
__device__ __forceinline__ float saved_at(const Saved &s, int64_t i, int64_t j) {
  if (!s.scale) return load_any(s.p, i * s.ld + j, s.dtype);
  const float q = (float)static_cast<const int8_t *>(s.p)[i * s.groups * kOpsGroup + j];
  return q * held8_down(s.scale[i * s.groups + j / kOpsGroup]);
}

// dz = dy act'(z), rounded to dtype
__global__ void dz_kernel(const void *dy, int dy_dtype, int64_t dy_ld, Saved z, int act, int64_t m, int64_t n,
                          void *dz, int dtype) {
  const int64_t e = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (e >= m * n) return;
  const int64_t i = e / n, j = e - i * n;
  float v = load_any(dy, i * dy_ld + j, dy_dtype);
  if (act != NR_ACT_NONE) v *= act_slope(saved_at(z, i, j), act);
  store_any(dz, e, dtype, v);
}

// dbias[j] = sum_i dy[i, j] act'(z[i, j]): 32 columns a block, 8 row lanes
__global__ void __launch_bounds__(256)
    dbias_kernel(const void *dy, int dy_dtype, int64_t dy_ld, Saved z, int act, int64_t m, int64_t n,
                 void *dbias, int dtype) {
  __shared__ float part[8][33];
  const int c = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int64_t j = (int64_t)blockIdx.x * 32 + c;
  float s = 0.0f;
  if (j < n)
    for (int64_t i = r; i < m; i += 8) {
      float v = load_any(dy, i * dy_ld + j, dy_dtype);
      if (act != NR_ACT_NONE) v *= act_slope(saved_at(z, i, j), act);
      s += v;
    }
  part[r][c] = s;
  __syncthreads();
  if (r == 0 && j < n) {
    for (int q = 1; q < 8; ++q) s += part[q][c];
    store_any(dbias, j, dtype, s);
  }
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

template <typename T>
void product(Operand A, Operand B, int64_t m, int64_t n, int64_t k, int dtype, const Epilogue &E, cudaStream_t s) {
  const dim3 grid((unsigned)ceil_div(m, kTile), (unsigned)ceil_div(n, kTile));
  product_kernel<T><<<grid, 256, 0, s>>>(A, B, m, n, k, dtype, E);
}
void product_any(Operand A, Operand B, int64_t m, int64_t n, int64_t k, int dtype, const Epilogue &E, cudaStream_t s) {
  if (dtype == NR_F16) product<__half>(A, B, m, n, k, dtype, E, s);
  else product<__nv_bfloat16>(A, B, m, n, k, dtype, E, s);
}

Saved saved_z(const nr_linear *a) {
  return {a->z, static_cast<const uint8_t *>(a->z_scale), a->z_ld, (int)a->dtype, ceil_div(a->n, kOpsGroup)};
}

}  // namespace

extern "C" int64_t nr_linear_forward_workspace(const nr_linear *a, int) {
  if (!valid(a, false)) return -1;
  return a->z_scale ? round_up(a->m * a->n * 4, 256) : 0;
}

extern "C" nr_status nr_linear_forward(const nr_linear *a, int device, void *ws, int64_t ws_bytes, void *stream) {
  const int64_t need = nr_linear_forward_workspace(a, device);
  if (need < 0 || ws_bytes < need || (need > 0 && !ws)) return NR_ERR_INVALID_ARG;
  if (a->m == 0) return NR_OK;
  DeviceGuard g(device);
  if (!g.ok) return NR_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool held = a->z_scale != nullptr;
  const Epilogue E = {a->bias, (int)a->bias_dtype, (int)a->act, a->residual, a->residual_ld, a->y, (int)a->y_dtype,
                      a->y_ld, held ? ws : a->z, held ? (int)NR_F32 : (int)a->dtype, held ? a->n : a->z_ld};
  product_any({a->x, a->x_ld, 1}, {a->w, a->w_ld, 1}, a->m, a->n, a->k, (int)a->dtype, E, s);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return cuda_status(e);
  return held ? nr_checkpoint8_write(ws, NR_F32, a->m, a->n, a->n, a->z, a->z_scale, device, stream) : NR_OK;
}

extern "C" int64_t nr_linear_backward_workspace(const nr_linear *a, int) {
  if (!valid(a, true)) return -1;
  return round_up(a->m * a->n * 2, 256) + (a->x_scale ? round_up(a->m * a->k * 2, 256) : 0);
}

extern "C" nr_status nr_linear_backward(const nr_linear *a, int device, void *ws, int64_t ws_bytes, void *stream) {
  const int64_t need = nr_linear_backward_workspace(a, device);
  if (need < 0 || ws_bytes < need || (need > 0 && !ws)) return NR_ERR_INVALID_ARG;
  DeviceGuard g(device);
  if (!g.ok) return NR_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int dt = (int)a->dtype;
  if (a->m == 0) {
    cudaError_t e = cudaSuccess;
    if (a->dw) e = cudaMemsetAsync(a->dw, 0, (size_t)(a->n * a->k) * 2, s);
    if (e == cudaSuccess && a->dbias) e = cudaMemsetAsync(a->dbias, 0, (size_t)a->n * type_bytes(a->bias_dtype), s);
    return e == cudaSuccess ? NR_OK : cuda_status(e);
  }
  const Saved z = saved_z(a);
  void *dz = ws;
  const int64_t count = a->m * a->n;
  dz_kernel<<<(unsigned)ceil_div(count, 256), 256, 0, s>>>(a->dy, (int)a->y_dtype, a->dy_ld, z, (int)a->act, a->m,
                                                           a->n, dz, dt);
  if (a->dbias)
    dbias_kernel<<<(unsigned)ceil_div(a->n, 32), 256, 0, s>>>(a->dy, (int)a->y_dtype, a->dy_ld, z, (int)a->act, a->m,
                                                              a->n, a->dbias, (int)a->bias_dtype);
  const void *x = a->x;
  int64_t x_ld = a->x_ld;
  if (a->x_scale && a->dw) {
    void *xv = static_cast<char *>(ws) + round_up(count * 2, 256);
    const nr_status st = nr_checkpoint8_read(a->x, a->x_scale, a->m, a->k, (int)a->x_act, xv, dt, a->k, device, stream);
    if (st != NR_OK) return st;
    x = xv;
    x_ld = a->k;
  }
  Epilogue E = {};
  if (a->dx) {
    E.y = a->dx;
    E.y_dtype = dt;
    E.y_ld = a->dx_ld;
    product_any({dz, a->n, 1}, {a->w, 1, a->w_ld}, a->m, a->k, a->n, dt, E, s);
  }
  if (a->dw) {
    E.y = a->dw;
    E.y_dtype = dt;
    E.y_ld = a->k;
    product_any({dz, 1, a->n}, {x, 1, x_ld}, a->n, a->k, a->m, dt, E, s);
  }
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}
