// Layer norm of rows, forward and backward.  For a row x of D elements, with
// mean m, variance v = mean (x - m)^2 and r = 1 / sqrt(v + eps):
//   y = (x - m) r gamma + beta
// and with h = (x - m) r, g = dy gamma:
//   dx = r (g - mean g - h mean (g h)),  dgamma = sum_rows dy h,  dbeta = sum_rows dy.
// Statistics and sums are fp32; the variance is taken about the mean in a
// second pass, so a large mean costs no digits.
#include "wr_ops.h"

namespace {

struct NormArgs {
  const void* x;
  int64_t n, x_stride;
  int d;
  const void *gamma, *beta;
  float eps;
  void* y;
  int64_t y_stride;
  float *mean, *rstd;
};

template <class T, class W>
__global__ __launch_bounds__(256) void wr_norm_kernel(NormArgs a) {
  __shared__ float red[2][4];
  const W *gamma = (const W*)a.gamma, *beta = (const W*)a.beta;
  for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x) {
    const T* x = (const T*)a.x + i * a.x_stride;
    T* y = (T*)a.y + i * a.y_stride;
    float s = 0.0f;
    for (int c = threadIdx.x; c < a.d; c += 256) s += (float)x[c];
    const float m = block_sum<4>(s, red[0]) / (float)a.d;
    s = 0.0f;
    for (int c = threadIdx.x; c < a.d; c += 256) {
      const float q = (float)x[c] - m;
      s += q * q;
    }
    const float r = 1.0f / sqrtf(block_sum<4>(s, red[1]) / (float)a.d + a.eps);
    for (int c = threadIdx.x; c < a.d; c += 256)
      y[c] = (T)(((float)x[c] - m) * r * (gamma ? (float)gamma[c] : 1.0f) + (beta ? (float)beta[c] : 0.0f));
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[i] = m;
      if (a.rstd) a.rstd[i] = r;
    }
  }
}

struct NormGradArgs {
  const void *dy, *x;
  int64_t n, dy_stride, x_stride;
  int d;
  const void* gamma;
  const float *mean, *rstd;
  void* dx;
  int64_t dx_stride;
  float *dgamma, *dbeta;
};

template <class T, class W>
__global__ __launch_bounds__(256) void wr_norm_dx_kernel(NormGradArgs a) {
  __shared__ float red[2][4];
  const W* gamma = (const W*)a.gamma;
  for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x) {
    const T *x = (const T*)a.x + i * a.x_stride, *dy = (const T*)a.dy + i * a.dy_stride;
    T* dx = (T*)a.dx + i * a.dx_stride;
    const float m = a.mean[i], r = a.rstd[i];
    float s0 = 0.0f, s1 = 0.0f;
    for (int c = threadIdx.x; c < a.d; c += 256) {
      const float g = (float)dy[c] * (gamma ? (float)gamma[c] : 1.0f);
      s0 += g;
      s1 += g * (((float)x[c] - m) * r);
    }
    const float m0 = block_sum<4>(s0, red[0]) / (float)a.d, m1 = block_sum<4>(s1, red[1]) / (float)a.d;
    for (int c = threadIdx.x; c < a.d; c += 256) {
      const float g = (float)dy[c] * (gamma ? (float)gamma[c] : 1.0f);
      dx[c] = (T)(r * (g - m0 - ((float)x[c] - m) * r * m1));
    }
  }
}

// 64 columns a block, four rows at a time.
template <class T>
__global__ __launch_bounds__(256) void wr_norm_dw_kernel(NormGradArgs a) {
  __shared__ float red[2][256];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63);
  float s0 = 0.0f, s1 = 0.0f;
  if (c < a.d)
    for (int64_t i = threadIdx.x >> 6; i < a.n; i += 4) {
      const float dy = (float)((const T*)a.dy)[i * a.dy_stride + c];
      s0 += dy * (((float)((const T*)a.x)[i * a.x_stride + c] - a.mean[i]) * a.rstd[i]);
      s1 += dy;
    }
  red[0][threadIdx.x] = s0;
  red[1][threadIdx.x] = s1;
  __syncthreads();
  if (threadIdx.x < 64 && c < a.d) {
    const float* q = red[0] + threadIdx.x;
    if (a.dgamma) a.dgamma[c] = (q[0] + q[64]) + (q[128] + q[192]);
    q = red[1] + threadIdx.x;
    if (a.dbeta) a.dbeta[c] = (q[0] + q[64]) + (q[128] + q[192]);
  }
}

wavernn_status check_norm(int dtype, int w_dtype, int64_t n, int32_t d) {
  if (!wr_dtype_ok(dtype) || !wr_dtype_ok(w_dtype)) return wr_fail(WAVERNN_E_INVALID, "bad dtype");
  if (w_dtype != dtype && w_dtype != WAVERNN_F32)
    return wr_fail(WAVERNN_E_INVALID, "gamma's and beta's dtype must be the rows' or F32");
  if (n < 0 || n > INT32_MAX) return wr_fail(WAVERNN_E_INVALID, "n_rows %lld out of range", (long long)n);
  if (d < 1) return wr_fail(WAVERNN_E_INVALID, "dim %d: must be positive", d);
  return WAVERNN_OK;
}

}  // namespace

extern "C" {

wavernn_status wavernn_layer_norm(int32_t dtype, const void* x_dev, int64_t n_rows, int32_t dim, int64_t x_stride,
                                  int32_t w_dtype, const void* gamma_dev, const void* beta_dev, float eps, void* y_dev,
                                  int64_t y_stride, float* mean_dev, float* rstd_dev, void* stream) {
  wavernn_status s;
  if ((s = check_norm(dtype, w_dtype, n_rows, dim)) != WAVERNN_OK) return s;
  if (!(eps > 0.0f)) return wr_fail(WAVERNN_E_INVALID, "eps must be positive");
  if ((s = wr_check_rows("x", x_dev, dtype, n_rows, dim, x_stride, false)) != WAVERNN_OK) return s;
  if ((s = wr_check_rows("y", y_dev, dtype, n_rows, dim, y_stride, true)) != WAVERNN_OK) return s;
  if (!wr_aligned(gamma_dev, wr_dtype_bytes(w_dtype)) || !wr_aligned(beta_dev, wr_dtype_bytes(w_dtype)))
    return wr_fail(WAVERNN_E_INVALID, "gamma or beta is not aligned to its elements");
  if (x_dev == y_dev && x_stride != y_stride) return wr_fail(WAVERNN_E_INVALID, "y in place of x needs the same row stride");
  if (n_rows == 0) return WAVERNN_OK;
  NormArgs a{x_dev, n_rows, x_stride, dim, gamma_dev, beta_dev, eps, y_dev, y_stride, mean_dev, rstd_dev};
  const int64_t grid = std::min<int64_t>(n_rows, WR_OP_BLOCKS);
  WR_DISPATCH(dtype, T, if (w_dtype == WAVERNN_F32) WR_LAUNCH((wr_norm_kernel<T, float>), grid, 256, 0, stream, a);
              else WR_LAUNCH((wr_norm_kernel<T, T>), grid, 256, 0, stream, a));
  return WAVERNN_OK;
}

int64_t wavernn_layer_norm_grad_workspace(int64_t n_rows, int32_t dim) {
  if (n_rows < 0 || n_rows > INT32_MAX || dim < 1) return -1;
  return 0;
}

wavernn_status wavernn_layer_norm_grad(int32_t dtype, const void* dy_dev, int64_t dy_stride, const void* x_dev,
                                       int64_t x_stride, int64_t n_rows, int32_t dim, int32_t w_dtype,
                                       const void* gamma_dev, const float* mean_dev, const float* rstd_dev, void* dx_dev,
                                       int64_t dx_stride, float* dgamma_dev, float* dbeta_dev, void* workspace_dev,
                                       int64_t workspace_bytes, void* stream) {
  wavernn_status s;
  if ((s = check_norm(dtype, w_dtype, n_rows, dim)) != WAVERNN_OK) return s;
  if ((s = wr_check_rows("dy", dy_dev, dtype, n_rows, dim, dy_stride, false)) != WAVERNN_OK) return s;
  if ((s = wr_check_rows("x", x_dev, dtype, n_rows, dim, x_stride, false)) != WAVERNN_OK) return s;
  if (dx_dev && (s = wr_check_rows("dx", dx_dev, dtype, n_rows, dim, dx_stride, true)) != WAVERNN_OK) return s;
  if (n_rows > 0 && (!mean_dev || !rstd_dev)) return wr_fail(WAVERNN_E_INVALID, "mean or rstd is null");
  if (!wr_aligned(gamma_dev, wr_dtype_bytes(w_dtype)))
    return wr_fail(WAVERNN_E_INVALID, "gamma is not aligned to its elements");
  if (dx_dev && ((dx_dev == dy_dev && dx_stride != dy_stride) || (dx_dev == x_dev && dx_stride != x_stride)))
    return wr_fail(WAVERNN_E_INVALID, "dx in place of dy or x needs the same row stride");
  const int64_t need = dgamma_dev || dbeta_dev ? wavernn_layer_norm_grad_workspace(n_rows, dim) : 0;
  if (need > 0 && (!workspace_dev || workspace_bytes < need || !wr_aligned(workspace_dev, 16)))
    return wr_fail(WAVERNN_E_INVALID, "workspace: %lld bytes needed, 16-byte aligned", (long long)need);
  NormGradArgs a{dy_dev, x_dev, n_rows, dy_stride, x_stride, dim, gamma_dev, mean_dev, rstd_dev, dx_dev, dx_stride,
                 dgamma_dev, dbeta_dev};
  if (dgamma_dev || dbeta_dev)   // before dx, which may replace dy or x
    WR_DISPATCH(dtype, T, WR_LAUNCH((wr_norm_dw_kernel<T>), (dim + 63) / 64, 256, 0, stream, a));
  if (dx_dev && n_rows > 0) {
    const int64_t grid = std::min<int64_t>(n_rows, WR_OP_BLOCKS);
    WR_DISPATCH(dtype, T, if (w_dtype == WAVERNN_F32) WR_LAUNCH((wr_norm_dx_kernel<T, float>), grid, 256, 0, stream, a);
                else WR_LAUNCH((wr_norm_dx_kernel<T, T>), grid, 256, 0, stream, a));
  }
  return WAVERNN_OK;
}

}  // extern "C"
