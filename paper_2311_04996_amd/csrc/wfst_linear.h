// The matrix product x w^T with what follows it in its epilogue: bias, activation, scale and residual (wfst_linear), or
// bias, log-softmax and log priors (wfst_loglikes).
#ifndef WFST_LINEAR_H_
#define WFST_LINEAR_H_

#include "wfst_elements.h"

namespace wfst_ops {

struct LinearArgs {
  const void *x, *w, *bias, *residual;
  void *y;
  int64_t rows, x_stride, w_stride, residual_stride, y_stride;
  int32_t k, n, bias_dtype, out_dtype, activation;
  float scale;
};

// relu, silu and gelu as the header defines them; a NaN stays one
__device__ __forceinline__ float activate(float z, int act) {
  if (act == 1) return z < 0.0f ? 0.0f : z;
  if (act == 2) return z / (1.0f + exp_fast(-z));
  if (act == 3) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
  return z;
}

// 64 x 64 results per workgroup of 256, 4 x 4 per lane, 16 columns of x and w at a time through LDS
template <class E>
__global__ __launch_bounds__(256) void linear_kernel(LinearArgs a) {
  __shared__ float xs[16][65], ws[16][65];
  const typename E::T *x = static_cast<const typename E::T *>(a.x), *w = static_cast<const typename E::T *>(a.w);
  const int tiles_n = (a.n + 63) / 64;
  const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * 64;
  const int n0 = (int)(blockIdx.x % tiles_n) * 64;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float acc[4][4] = {};
  for (int k0 = 0; k0 < a.k; k0 += 16) {
    for (int i = threadIdx.x; i < 64 * 16; i += 256) {
      const int r = i / 16, c = i % 16;
      xs[c][r] = m0 + r < a.rows && k0 + c < a.k ? E::get(x[(m0 + r) * a.x_stride + k0 + c]) : 0.0f;
      ws[c][r] = n0 + r < a.n && k0 + c < a.k ? E::get(w[(n0 + r) * a.w_stride + k0 + c]) : 0.0f;
    }
    __syncthreads();
    for (int c = 0; c < 16; ++c)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_fmaf(xs[c][ty + 16 * i], ws[c][tx + 16 * j], acc[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t m = m0 + ty + 16 * i;
      const int n = n0 + tx + 16 * j;
      if (m >= a.rows || n >= a.n) continue;
      float z = acc[i][j];
      if (a.bias) z += load_as(a.bias, n, a.bias_dtype);
      z = a.scale * activate(z, a.activation);
      if (a.residual) z += load_as(a.residual, m * a.residual_stride + n, a.out_dtype);
      store_as(a.y, m * a.y_stride + n, a.out_dtype, z);
    }
}

struct LoglikesArgs {
  const void *x, *w, *bias;
  const float *log_prior;
  const int32_t *lengths;
  void *out;
  int64_t x_seq_stride, x_stride, w_stride, out_seq_stride, out_stride;
  int32_t seqs, frames, k, v, bias_dtype, out_dtype;
};

// one workgroup of 256 per frame: a lane's class at a time, then the row's maximum and sum through LDS
template <class E>
__global__ __launch_bounds__(256) void loglikes_kernel(LoglikesArgs a) {
  __shared__ float z[2048], part[256];
  const int64_t row = blockIdx.x;
  const int s = (int)(row / a.frames), t = (int)(row % a.frames);
  if (a.lengths && t >= a.lengths[s]) return;
  const typename E::T *x = static_cast<const typename E::T *>(a.x) + s * a.x_seq_stride + t * a.x_stride;
  float m = -__builtin_inff();
  for (int c = threadIdx.x; c < a.v; c += 256) {
    const typename E::T *w = static_cast<const typename E::T *>(a.w) + c * a.w_stride;
    float acc = 0.0f;
    for (int k = 0; k < a.k; ++k) acc = __builtin_fmaf(E::get(x[k]), E::get(w[k]), acc);
    if (a.bias) acc += load_as(a.bias, c, a.bias_dtype);
    z[c] = acc;
    m = fmaxf(m, acc);
  }
  part[threadIdx.x] = m;
  __syncthreads();
  for (int i = 0; i < 256; ++i) m = fmaxf(m, part[i]);
  __syncthreads();
  float sum = 0.0f;
  for (int c = threadIdx.x; c < a.v; c += 256) sum += exp_fast(z[c] - m);
  part[threadIdx.x] = sum;
  __syncthreads();
  sum = 0.0f;
  for (int i = 0; i < 256; ++i) sum += part[i];
  const float ls = logf(sum);
  for (int c = threadIdx.x; c < a.v; c += 256) {
    float l = z[c] - m - ls;
    if (a.log_prior) l -= a.log_prior[c];
    store_as(a.out, s * a.out_seq_stride + t * a.out_stride + c, a.out_dtype, l);
  }
}

}  // namespace wfst_ops

#endif  // WFST_LINEAR_H_
