// The norms after and before a block of a residual encoder, fused with the block's
// gate and residual scale (neuroute_ops.h: nr_block_norm): the C entries, rows of any length, and the parameters'
// gradients. Rows of up to 8192 columns are worked on in shared memory (nrq_blocknorm.cuh).
#include <float.h>
#include <math.h>

#include <atomic>

#include "nrq_blocknorm.cuh"

namespace {

using namespace blocknorm;

// ------------------------------------------------------------ rows of any length, read again from memory
constexpr int kLongThreads = 512;
template <int K>
__device__ __forceinline__ void long_sums(float (&v)[K], float (*shared)[K]) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  __syncthreads();  // the last sums have been read
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) shared[threadIdx.x >> 5][k] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = 0.0f;
  for (int w = 0; w < kLongThreads / 32; ++w)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += shared[w][k];
}

// c of a row's column, and y
__device__ __forceinline__ float long_c(const Block &B, int64_t i, int64_t j, float mean, float rstd) {
  const float uh = (load_any(B.u.p, i * B.u.ld + j, B.dtype) - mean) * rstd;
  return fmaf(uh, vec(B.post_w, j, B.w_dtype, 1.0f), vec(B.post_b, j, B.w_dtype, 0.0f));
}
__device__ __forceinline__ float long_y(const Block &B, int64_t i, int64_t j, float mean, float rstd) {
  const float r = load_any(B.r.p, i * B.r.ld + j, B.r_dtype);
  if (!B.u.p) return r;
  float f = vec(B.scale, j, B.w_dtype, 1.0f);
  if (B.gate) f *= gate_value(load_any(B.q.p, i * B.q.ld + (B.gate == 2 ? j : 0), B.dtype), B.act);
  return fmaf(long_c(B, i, j, mean, rstd), f, B.alpha * r);
}

__global__ void __launch_bounds__(kLongThreads) long_forward_kernel(const Block B) {
  __shared__ float shared[kLongThreads / 32][1];
  const float inv = 1.0f / (float)B.n;
  for (int64_t i = blockIdx.x; i < B.m; i += gridDim.x) {
    float um = 0.0f, ur = 1.0f, ym = 0.0f, yr = 1.0f, s[1];
    if (B.post == NR_NORM_LAYER) {
      s[0] = 0.0f;
      for (int64_t j = threadIdx.x; j < B.n; j += kLongThreads) s[0] += load_any(B.u.p, i * B.u.ld + j, B.dtype);
      long_sums<1>(s, shared);
      um = s[0] * inv;
    }
    if (B.post != NR_NORM_NONE) {
      s[0] = 0.0f;
      for (int64_t j = threadIdx.x; j < B.n; j += kLongThreads) {
        const float d = load_any(B.u.p, i * B.u.ld + j, B.dtype) - um;
        s[0] = fmaf(d, d, s[0]);
      }
      long_sums<1>(s, shared);
      ur = 1.0f / sqrtf(fmaf(s[0], inv, B.eps));
    }
    if (B.pre == NR_NORM_LAYER) {
      s[0] = 0.0f;
      for (int64_t j = threadIdx.x; j < B.n; j += kLongThreads) s[0] += long_y(B, i, j, um, ur);
      long_sums<1>(s, shared);
      ym = s[0] * inv;
    }
    if (B.pre != NR_NORM_NONE) {
      s[0] = 0.0f;
      for (int64_t j = threadIdx.x; j < B.n; j += kLongThreads) {
        const float d = long_y(B, i, j, um, ur) - ym;
        s[0] = fmaf(d, d, s[0]);
      }
      long_sums<1>(s, shared);
      yr = 1.0f / sqrtf(fmaf(s[0], inv, B.eps));
    }
    for (int64_t j = threadIdx.x; j < B.n; j += kLongThreads) {
      const float y = long_y(B, i, j, um, ur);
      if (B.u.p) store_any(B.y.p, i * B.y.ld + j, B.r_dtype, y);
      if (B.pre != NR_NORM_NONE)
        store_any(B.h.p, i * B.h.ld + j, B.dtype, fmaf((y - ym) * yr, vec(B.w, j, B.w_dtype, 1.0f), vec(B.b, j, B.w_dtype, 0.0f)));
    }
    if (threadIdx.x == 0) {
      if (B.u_mean) B.u_mean[i] = um;
      if (B.u_rstd) B.u_rstd[i] = ur;
      if (B.y_mean) B.y_mean[i] = ym;
      if (B.y_rstd) B.y_rstd[i] = yr;
    }
  }
}

// the gradient of y that reaches column j, with the row's means of g and g yh
__device__ __forceinline__ float long_t(const Block &B, int64_t i, int64_t j, float m1, float m2, float &dh, float &yh) {
  float t = B.dy.p ? load_any(B.dy.p, i * B.dy.ld + j, B.r_dtype) : 0.0f;
  dh = yh = 0.0f;
  if (B.pre != NR_NORM_NONE) {
    const float rstd = B.y_rstd[i];
    dh = load_any(B.dh.p, i * B.dh.ld + j, B.dtype);
    yh = (load_any(B.y.p, i * B.y.ld + j, B.r_dtype) - (B.y_mean ? B.y_mean[i] : 0.0f)) * rstd;
    t += rstd * (dh * vec(B.w, j, B.w_dtype, 1.0f) - m1 - yh * m2);
  }
  return t;
}

__global__ void __launch_bounds__(kLongThreads) long_rows_kernel(const Block B) {
  __shared__ float shared[kLongThreads / 32][2];
  __shared__ float shared1[kLongThreads / 32][1];
  const float inv = 1.0f / (float)B.n;
  for (int64_t i = blockIdx.x; i < B.m; i += gridDim.x) {
    float s[2] = {0.0f, 0.0f}, dh, yh;
    if (B.pre != NR_NORM_NONE) {
      const float mean = B.y_mean ? B.y_mean[i] : 0.0f, rstd = B.y_rstd[i];
      for (int64_t j = threadIdx.x; j < B.n; j += kLongThreads) {
        const float g = load_any(B.dh.p, i * B.dh.ld + j, B.dtype) * vec(B.w, j, B.w_dtype, 1.0f);
        s[0] += g;
        s[1] = fmaf(g, (load_any(B.y.p, i * B.y.ld + j, B.r_dtype) - mean) * rstd, s[1]);
      }
      long_sums<2>(s, shared);
    }
    const float m1 = B.pre == NR_NORM_LAYER ? s[0] * inv : 0.0f, m2 = s[1] * inv;
    if (B.row_sums && threadIdx.x == 0) {
      B.row_sums[i] = m1;
      B.row_sums[B.m + i] = m2;
    }
    const float um = B.u_mean ? B.u_mean[i] : 0.0f, ur = B.u_rstd ? B.u_rstd[i] : 1.0f;
    float qrow = 0.0f, gate = 1.0f;
    if (B.gate == 1) qrow = load_any(B.q.p, i * B.q.ld, B.dtype), gate = gate_value(qrow, B.act);
    float e1 = 0.0f, e2 = 0.0f;
    if (B.post != NR_NORM_NONE) {
      s[0] = s[1] = 0.0f;
      for (int64_t j = threadIdx.x; j < B.n; j += kLongThreads) {
        const float t = long_t(B, i, j, m1, m2, dh, yh);
        if (B.gate == 2) gate = gate_value(load_any(B.q.p, i * B.q.ld + j, B.dtype), B.act);
        const float e = t * gate * vec(B.scale, j, B.w_dtype, 1.0f) * vec(B.post_w, j, B.w_dtype, 1.0f);
        s[0] += e;
        s[1] = fmaf(e, (load_any(B.u.p, i * B.u.ld + j, B.dtype) - um) * ur, s[1]);
      }
      long_sums<2>(s, shared);
      e1 = B.post == NR_NORM_LAYER ? s[0] * inv : 0.0f;
      e2 = s[1] * inv;
    }
    float dq[1] = {0.0f};
    for (int64_t j = threadIdx.x; j < B.n; j += kLongThreads) {
      const float t = long_t(B, i, j, m1, m2, dh, yh);
      store_any(B.dr.p, i * B.dr.ld + j, B.r_dtype, B.alpha * t);
      if (!B.u.p) continue;
      float q = qrow;
      if (B.gate == 2) q = load_any(B.q.p, i * B.q.ld + j, B.dtype), gate = gate_value(q, B.act);
      const float uh = (load_any(B.u.p, i * B.u.ld + j, B.dtype) - um) * ur, ts = t * vec(B.scale, j, B.w_dtype, 1.0f);
      const float pw = vec(B.post_w, j, B.w_dtype, 1.0f);
      store_any(B.du.p, i * B.du.ld + j, B.dtype, ur * (ts * gate * pw - e1 - uh * e2));
      if (B.gate) {
        const float d = ts * fmaf(uh, pw, vec(B.post_b, j, B.w_dtype, 0.0f)) * gate_slope(q, B.act);
        if (B.gate == 2) store_any(B.dq.p, i * B.dq.ld + j, B.dtype, d);
        dq[0] += d;
      }
    }
    if (B.gate == 1) {
      long_sums<1>(dq, shared1);
      if (threadIdx.x == 0) store_any(B.dq.p, i * B.dq.ld, B.dtype, dq[0]);
    }
  }
}

// 32 columns and every gridDim.y-th eight rows a block -> parts
__global__ void __launch_bounds__(256) long_params_kernel(const Block B) {
  __shared__ float part[4][8][33];
  const int c = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int64_t j = (int64_t)blockIdx.x * 32 + c;
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (j < B.n)
    for (int64_t i = (int64_t)blockIdx.y * 8 + r; i < B.m; i += (int64_t)gridDim.y * 8) {
      float dh, yh;
      float t = long_t(B, i, j, B.row_sums[i], B.row_sums[B.m + i], dh, yh);
      s[0] = fmaf(dh, yh, s[0]);
      s[1] += dh;
      if (B.u.p) {
        if (B.gate) t *= gate_value(load_any(B.q.p, i * B.q.ld + (B.gate == 2 ? j : 0), B.dtype), B.act);
        const float uh = (load_any(B.u.p, i * B.u.ld + j, B.dtype) - (B.u_mean ? B.u_mean[i] : 0.0f)) * (B.u_rstd ? B.u_rstd[i] : 1.0f);
        s[2] = fmaf(t, uh, s[2]);
        s[3] += t;
      }
    }
  for (int k = 0; k < 4; ++k) part[k][r][c] = s[k];
  __syncthreads();
  if (r >= 4 || j >= B.n) return;
  float v = 0.0f;
  for (int q = 0; q < 8; ++q) v += part[r][q][c];
  B.parts[((int64_t)r * gridDim.y + blockIdx.y) * B.n + j] = v;
}

// The parameters' gradients: the blocks' four sums of 8 columns, 32 rows of parts at a time
__global__ void __launch_bounds__(1024) params_kernel(const Block B, int count) {
  __shared__ float part[32][33], v[32];
  const int c = threadIdx.x & 31, r = threadIdx.x >> 5, k = c >> 3;
  const int64_t j = (int64_t)blockIdx.x * 8 + (c & 7);
  grid_wait();
  float s = 0.0f;
  // the sums of dh and of t a are there where they are wanted
  if (j < B.n && (!(k & 1) || (k == 1 ? B.db != nullptr : B.post_b || B.dpost_b))) {
    const float *p = B.parts + (int64_t)k * count * B.n + j;
#pragma unroll 8
    for (int i = r; i < count; i += 32) s += p[(int64_t)i * B.n];
  }
  part[r][c] = s;
  __syncthreads();
  if (r != 0) return;
  for (int q = 1; q < 32; ++q) s += part[q][c];
  v[c] = s;
  __syncwarp();
  if (k != 0 || j >= B.n) return;
  const float A = v[16 + c], S = v[24 + c], scale = vec(B.scale, j, B.w_dtype, 1.0f);
  if (B.dw) store_any(B.dw, j, B.w_dtype, v[c]);
  if (B.db) store_any(B.db, j, B.w_dtype, v[8 + c]);
  if (B.dpost_w) store_any(B.dpost_w, j, B.w_dtype, scale * A);
  if (B.dpost_b) store_any(B.dpost_b, j, B.w_dtype, scale * S);
  if (B.dscale) store_any(B.dscale, j, B.w_dtype, fmaf(vec(B.post_w, j, B.w_dtype, 1.0f), A, vec(B.post_b, j, B.w_dtype, 0.0f) * S));
}

// ------------------------------------------------------------ host
int stats_rows(const nr_block_norm *a) { return (int)(a->post + a->pre); }  // none 0, RMS 1, layer 2
bool matrix_ok(const void *p, int64_t ld, int64_t dtype, int64_t least_ld) { return p && placed(p, dtype) && ld >= least_ld; }

bool valid(const nr_block_norm *a, bool backward) {
  if (!a || a->m < 0 || a->m > kOpsMaxRows || a->n < 1 || a->n > kOpsMaxCols) return false;
  if (a->dtype < NR_F32 || a->dtype > NR_BF16 || (a->r_dtype != a->dtype && a->r_dtype != NR_F32) ||
      (a->w_dtype != a->dtype && a->w_dtype != NR_F32))
    return false;
  if (a->post < NR_NORM_NONE || a->post > NR_NORM_LAYER || a->pre < NR_NORM_NONE || a->pre > NR_NORM_LAYER) return false;
  if (a->gate && ((a->gate_act != NR_ACT_SIGMOID && a->gate_act != NR_ACT_SILU) || (a->gate_cols != 1 && a->gate_cols != a->n)))
    return false;
  if (!(fabs(a->alpha) <= FLT_MAX)) return false;
  const void *vectors[] = {a->scale, a->post_weight, a->post_bias, a->weight, a->bias, a->dscale, a->dpost_weight, a->dpost_bias,
                           a->dweight, a->dbias};
  for (const void *p : vectors)
    if (!placed(p, a->w_dtype)) return false;
  // parts without what they belong to
  if (a->post == NR_NORM_NONE && (a->post_weight || a->post_bias || a->dpost_weight || a->dpost_bias)) return false;
  if (a->pre == NR_NORM_NONE && (a->weight || a->bias || a->dweight || a->dbias)) return false;
  if (!placed(a->stats, NR_F32)) return false;
  if (a->m > 0 && !a->u) {
    if (a->gate || a->scale || a->post != NR_NORM_NONE || a->pre == NR_NORM_NONE || a->alpha != 1.0 || a->dscale) return false;
  }
  if (!backward && !(a->eps > 0.0)) return false;
  if (a->m == 0) return true;
  if (a->u && !matrix_ok(a->u, a->u_ld, a->dtype, 0)) return false;
  if (a->gate && !matrix_ok(a->gate, a->gate_ld, a->dtype, 0)) return false;
  if (!backward) {
    if (!matrix_ok(a->r, a->r_ld, a->r_dtype, 0)) return false;
    if (a->u && !matrix_ok(a->y, a->y_ld, a->r_dtype, a->n)) return false;
    return a->pre == NR_NORM_NONE || matrix_ok(a->h, a->h_ld, a->dtype, a->n);
  }
  if (stats_rows(a) && !a->stats) return false;
  if (a->pre != NR_NORM_NONE && (!matrix_ok(a->dh, a->dh_ld, a->dtype, 0) || !matrix_ok(a->y, a->y_ld, a->r_dtype, 0))) return false;
  if (a->dy ? !matrix_ok(a->dy, a->dy_ld, a->r_dtype, 0) : a->pre == NR_NORM_NONE) return false;
  if (!matrix_ok(a->dr, a->dr_ld, a->r_dtype, a->n)) return false;
  if (a->u && !matrix_ok(a->du, a->du_ld, a->dtype, a->n)) return false;
  return !a->gate || matrix_ok(a->dgate, a->dgate_ld, a->dtype, a->gate_cols);
}

Block block_of(const nr_block_norm *a, bool backward) {
  Block B = {};
  const auto rows = [](const void *p, int64_t ld) { return Rows{const_cast<void *>(p), ld}; };
  B.m = a->m;
  B.n = a->n;
  B.dtype = (int)a->dtype;
  B.r_dtype = (int)a->r_dtype;
  B.w_dtype = (int)a->w_dtype;
  B.post = (int)a->post;
  B.pre = (int)a->pre;
  B.act = (int)a->gate_act;
  B.gate = !a->gate ? 0 : a->gate_cols == 1 && a->n != 1 ? 1 : 2;
  B.alpha = (float)a->alpha;
  B.eps = fmaxf((float)a->eps, 1.40129846e-45f);  // at least the least fp32: an eps below it is positive too
  B.u = rows(a->u, a->u_ld);
  B.q = rows(a->gate, a->gate_ld);
  B.y = rows(a->y, a->y_ld);
  B.scale = a->scale;
  B.post_w = a->post_weight;
  B.post_b = a->post_bias;
  B.w = a->weight;
  B.b = a->bias;
  if (a->stats) {
    float *at = a->stats;
    if (B.post == NR_NORM_LAYER) B.u_mean = at, at += a->m;
    if (B.post != NR_NORM_NONE) B.u_rstd = at, at += a->m;
    if (B.pre == NR_NORM_LAYER) B.y_mean = at, at += a->m;
    if (B.pre != NR_NORM_NONE) B.y_rstd = at;
  }
  if (!backward) {
    B.r = rows(a->r, a->r_ld);
    B.h = rows(a->h, a->h_ld);
    return B;
  }
  B.dh = rows(a->dh, a->dh_ld);
  B.dy = rows(a->dy, a->dy_ld);
  B.dr = rows(a->dr, a->dr_ld);
  B.du = rows(a->du, a->du_ld);
  B.dq = rows(a->dgate, a->dgate_ld);
  B.dscale = a->dscale;
  B.dpost_w = a->dpost_weight;
  B.dpost_b = a->dpost_bias;
  B.dw = a->dweight;
  B.db = a->dbias;
  return B;
}
bool has_params(const nr_block_norm *a) { return a->dscale || a->dpost_weight || a->dpost_bias || a->dweight || a->dbias; }

constexpr int kLongParts = 32, kLongBlocks = 4;  // blocks an SM
// bytes of shared memory an SM, of which a block needs so many besides its stages, and the most that a block's may take
constexpr int kShared = 228 * 1024, kSharedOwn = 2048, kSharedMost = 226 * 1024;

// Forward a warp takes rows of up to 1536 columns and several warps longer ones, three or four eights a
// thread, whichever leaves fewer columns unused. Backward, where a column's sums are two or four registers, a warp takes
// 512 columns, and threads of longer rows three eights or two. Rows longer than 8192, counted with the columns
// that lie before them (odd widths from 8186 on, 8190 around an fp32 stream), and those whose stage does not fit beside the
// vectors (fp32 backward with a full gate: from 7176 columns with layer norms and biases, 7688 with RMS norms), are read
// again from memory (x 0). That is dear: 1.3e8 values in bf16 with RMS norms and a gate, 8192 columns 218 us forward and
// 464 backward, 8193 columns 2274 and 6292; fp32 backward 629 us at 7168 columns, 5453 at 8184.
Plan plan_of(const Block &B, bool backward, int sms) {
  Plan P = {};
  // the matrices read, as the kernels number them, and those written
  const Rows *rows[5] = {&B.r, &B.u, B.gate == 2 ? &B.q : nullptr, nullptr, nullptr};
  int types[5] = {B.r_dtype, B.dtype, B.dtype, B.dtype, B.dtype};
  if (backward) {
    rows[0] = B.pre ? &B.dh : nullptr, rows[1] = B.pre ? &B.y : nullptr, rows[2] = &B.dy, rows[3] = &B.u;
    rows[4] = B.gate == 2 ? &B.q : nullptr;
    types[0] = B.dtype, types[1] = types[2] = B.r_dtype;
  }
  const Rows *outs[3] = {backward ? &B.dr : &B.y, backward ? &B.du : &B.h, backward && B.gate == 2 ? &B.dq : nullptr};
  bool aligned = B.n % 8 == 0, same = true;
  int alike = B.r_dtype == NR_F32 ? 4 : 8;  // rows so far apart begin alike
  int64_t place = -1, pitch = 0;            // the first matrix's, in values, of `alike`
  for (int k = 0; k < 5; ++k) {
    if (!rows[k] || !rows[k]->p) continue;
    const int64_t begins = (int64_t)(reinterpret_cast<uintptr_t>(rows[k]->p) / (unsigned)type_bytes(types[k])) % alike;
    aligned = aligned && vec_ok(rows[k]->p, rows[k]->ld, types[k]);
    if (place < 0) place = begins, pitch = rows[k]->ld % alike;
    same = same && begins == place && rows[k]->ld % alike == pitch;
  }
  for (int k = 0; k < 3; ++k)
    aligned = aligned && (!outs[k] || !outs[k]->p || vec_ok(outs[k]->p, outs[k]->ld, k == 0 ? B.r_dtype : B.dtype));
  P.lie = aligned ? kAligned : same ? kAlike : kAny;
  if (aligned) alike = 1;
  if (B.n + alike - 1 > 8192) return P;
  const int n = (int)B.n, most = n + alike - 1, units = (int)ceil_div(most, 256);  // columns with those before the row
  P.bias = backward && (B.b || B.db || B.post_b || B.dpost_b);  // by the vectors too: leaving gradients out changes no other
  P.tpr = most <= 64 ? 8 : most <= 128 ? 16 : most <= (backward ? 512 : 1536) ? 32 : 0;
  if (units <= 2) P.v = units;
  else if (backward) P.v = P.bias ? 2 : 3;
  else if (P.tpr) P.v = units <= 4 ? units : 6;
  else P.v = ceil_div(units, 3) * 3 < ceil_div(units, 4) * 4 ? 3 : 4;
  // few rows forward, as single queries are: a warp for every 256 columns (1 x 1536: 3.7 us for 7.7)
  const bool few_rows = !backward && units > 1 && B.m <= 2 * (int64_t)sms;
  if (few_rows) P.tpr = 0, P.v = 1;
  const int warps = P.tpr ? 1 : (int)ceil_div(units, P.v);
  // blocks an SM and warps a block that the registers allow
  int per_sm = P.v > 1 && (backward || P.v > 2) ? 1 : backward ? 2 : 4;
  if (few_rows) per_sm = warps <= 16 ? 2 : 1;
  const int most_warps = few_rows ? warps : per_sm > 1 ? 8 : !backward ? 16 : warps > 12 ? 16 : 12;
  int groups = P.tpr ? most_warps * 32 / P.tpr : most_warps / warps;
  P.ring.columns = (P.tpr ? P.tpr : 32 * warps) * 8 * P.v;
  int at = 0;
  for (int k = 0; k < 5; ++k) {
    if (!rows[k] || !rows[k]->p) continue;
    const int64_t e = (int64_t)type_bytes(types[k]);
    const char *p = static_cast<const char *>(rows[k]->p);
    // up to 16 bytes before the row and a piece behind it are read, if it does not begin at a piece's place; whole lines
    // of shared memory (16 bytes behind a line's begin copies and reads took 350 us for 290 backward at 65536 x 1536)
    at = (int)round_up(at + 16, 128);
    P.ring.s[k] = {p, p + ((B.m - 1) * rows[k]->ld + B.n) * e, rows[k]->ld * e, at};
    at += (int)(P.ring.columns * e) + 32;
  }
  at = (int)round_up(at, 128);
  P.ring.row_bytes = at;
  const bool u = B.u.p != nullptr;
  P.ring.present = (u && (B.scale || B.post_w) ? 1 : 0) | (u && B.post_b ? 2 : 0) | (B.w ? 4 : 0) | (!backward && B.b ? 8 : 0);
  const int vectors = __builtin_popcount(P.ring.present) * P.ring.columns * 4;
  const auto room = [](int blocks) { return kShared / blocks - kSharedOwn < kSharedMost ? kShared / blocks - kSharedOwn : kSharedMost; };
  while (per_sm > 1 && room(per_sm) - vectors < groups * at) --per_sm;
  if (room(per_sm) - vectors < groups * at) groups = (room(per_sm) - vectors) / at;
  if (P.tpr && P.tpr < 32) groups = groups / (32 / P.tpr) * (32 / P.tpr);  // whole warps
  if (groups < 1) return Plan{};
  // Copies under way at once, bytes an SM: more of them do not feed DRAM better. 65536 x 1536, us by 80, 112 and
  // 200 KB: forward bf16 179, 167, 180, around an fp32 stream 189, 200, 208 (of 4096 columns 213, 192, 192), backward
  // 376, 286, 308; 400000 x 64 backward 88, 88, 74.
  const int under_way = 1024 * (backward ? P.v == 1 ? 200 : 160 : P.tpr && B.r_dtype != B.dtype ? 80 : 112);
  const int few = few_rows ? 1 : P.tpr && P.tpr < 32 ? groups : P.tpr ? 8 : (int)ceil_div(8, warps);  // groups of eight warps
  if (per_sm == 1)
    while (groups > few && groups * at > under_way) --groups;
  // rows are dealt out evenly: as many a turn as leave the fewest places of the last turn empty
  const int64_t rows_sm = ceil_div(B.m, (int64_t)sms * per_sm);
  if (P.tpr == 0 || P.tpr == 32) {
    int best = groups;
    for (int g = groups; 4 * g >= 3 * groups && g >= 1; --g)
      if (ceil_div(rows_sm, g) * g < ceil_div(rows_sm, best) * best) best = g;
    groups = rows_sm < groups ? (int)rows_sm : best;
  }
  const int fit = (room(per_sm) - vectors) / (groups * at), deep = under_way / (per_sm * groups * at);
  P.ring.stages = deep < 1 ? 1 : deep < fit ? deep : fit;
  if (P.ring.stages > kMostStages) P.ring.stages = kMostStages;
  P.x = P.tpr ? groups * P.tpr : 32 * warps;
  P.y = P.tpr ? 1 : groups;
  P.ring.vectors = P.ring.stages * groups * at;
  P.bytes = P.ring.vectors + vectors;
  if (backward && groups > 1 && P.bytes < groups * n * (P.bias ? 16 : 8)) P.bytes = groups * n * (P.bias ? 16 : 8);  // their sums
  const int64_t need = ceil_div(ceil_div(B.m, alike), groups) * alike, all = (int64_t)sms * per_sm / alike * alike;
  P.blocks = (int)(need < all ? need : all);
  return P;
}

Kernel kernel_of(const Block &B, const Plan &P, bool backward) {
  if (B.dtype == NR_F32) return backward ? backward_of<float, float>(P) : forward_of<float, float>(P);
  if (B.dtype == NR_F16) {
    if (B.r_dtype == NR_F32) return backward ? backward_of<float, __half>(P) : forward_of<float, __half>(P);
    return backward ? backward_of<__half, __half>(P) : forward_of<__half, __half>(P);
  }
  if (B.r_dtype == NR_F32) return backward ? backward_of<float, __nv_bfloat16>(P) : forward_of<float, __nv_bfloat16>(P);
  return backward ? backward_of<__nv_bfloat16, __nv_bfloat16>(P) : forward_of<__nv_bfloat16, __nv_bfloat16>(P);
}
// Lets a kernel's blocks have more shared memory than without asking, once on each device: a table of
// those that do, filled by whoever comes first (threads that race ask twice).
cudaError_t allow_shared(Kernel k, int device) {
  constexpr int kSlots = 1024;
  static std::atomic<uintptr_t> seen[kSlots];
  const uintptr_t key = (reinterpret_cast<uintptr_t>(k) << 6) | (uintptr_t)device;
  for (int i = 0, at = (int)((key ^ key >> 10 ^ key >> 20) % kSlots); i < 16; ++i, at = (at + 1) % kSlots) {
    const uintptr_t have = seen[at].load(std::memory_order_acquire);
    if (have == key) return cudaSuccess;
    if (have) continue;
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedMost);
    if (e == cudaSuccess) seen[at].store(key, std::memory_order_release);
    return e;
  }
  return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedMost);
}
cudaError_t start(const Block &B, const Plan &P, bool backward, int device, cudaStream_t s) {
  const Kernel k = kernel_of(B, P, backward);
  if (P.bytes > 48 * 1024 - kSharedOwn) {
    const cudaError_t e = allow_shared(k, device);
    if (e != cudaSuccess) return e;
  }
  k<<<P.blocks, dim3(P.x, P.y), P.bytes, s>>>(B, P.ring);
  return cudaGetLastError();
}

}  // namespace

extern "C" nr_status nr_block_norm_forward(const nr_block_norm *a, int device, void *stream) {
  if (!valid(a, false)) return NR_ERR_INVALID_ARG;
  if (a->m == 0) return NR_OK;
  const int sms = nr_ops_sms(device);
  DeviceGuard g(device);
  if (sms < 1 || !g.ok) return NR_ERR_CUDA;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const Block B = block_of(a, false);
  const Plan P = plan_of(B, false, sms);
  cudaError_t e;
  if (P.x) {
    e = start(B, P, false, device, s);
  } else {
    const int64_t most = (int64_t)sms * kLongBlocks;
    long_forward_kernel<<<(unsigned)(a->m < most ? a->m : most), kLongThreads, 0, s>>>(B);
    e = cudaGetLastError();
  }
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}

extern "C" int64_t nr_block_norm_backward_workspace(const nr_block_norm *a, int device) {
  if (!valid(a, true)) return NR_ERR_INVALID_ARG;
  const int sms = nr_ops_sms(device);
  if (sms < 1) return NR_ERR_CUDA;
  if (a->m == 0 || !has_params(a)) return 0;
  const Block B = block_of(a, true);
  const Plan P = plan_of(B, true, sms);
  if (P.x) return round_up((int64_t)P.blocks * 4 * a->n * 4, 256);
  return round_up(a->m * 8, 256) + round_up((int64_t)kLongParts * 4 * a->n * 4, 256);
}

extern "C" nr_status nr_block_norm_backward(const nr_block_norm *a, int device, void *ws, int64_t ws_bytes, void *stream) {
  const int64_t need = nr_block_norm_backward_workspace(a, device);
  if (need < 0) return (nr_status)need;
  if (ws_bytes < need || (need > 0 && (!ws || (reinterpret_cast<uintptr_t>(ws) & 255)))) return NR_ERR_INVALID_ARG;
  DeviceGuard g(device);
  if (!g.ok) return NR_ERR_CUDA;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (a->m == 0) {
    void *const out[] = {a->dscale, a->dpost_weight, a->dpost_bias, a->dweight, a->dbias};
    for (void *p : out)
      if (p && e == cudaSuccess) e = cudaMemsetAsync(p, 0, (size_t)a->n * type_bytes(a->w_dtype), s);
    return e == cudaSuccess ? NR_OK : cuda_status(e);
  }
  Block B = block_of(a, true);
  const Plan P = plan_of(B, true, nr_ops_sms(device));
  int parts = kLongParts;
  if (P.x) {
    parts = P.blocks;
    if (need > 0) B.parts = static_cast<float *>(ws);
    e = start(B, P, true, device, s);
  } else {
    const int64_t most = (int64_t)nr_ops_sms(device) * kLongBlocks;
    if (need > 0) {
      B.row_sums = static_cast<float *>(ws);
      B.parts = reinterpret_cast<float *>(static_cast<char *>(ws) + round_up(a->m * 8, 256));
    }
    long_rows_kernel<<<(unsigned)(a->m < most ? a->m : most), kLongThreads, 0, s>>>(B);
    if (need > 0) long_params_kernel<<<dim3((unsigned)ceil_div(a->n, 32), kLongParts), 256, 0, s>>>(B);
    e = cudaGetLastError();
  }
  if (e == cudaSuccess && need > 0) e = launch(params_kernel, (unsigned)ceil_div(a->n, 8), dim3(1024), 0, s, true, B, parts);
  return e == cudaSuccess ? NR_OK : cuda_status(e);
}
