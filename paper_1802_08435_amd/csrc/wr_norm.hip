// Layer norm of rows, forward and backward.  For a row x of D elements, with
// mean m, variance v = mean (x - m)^2 and r = 1 / sqrt(v + eps):
//   y = (x - m) r gamma + beta
// and with h = (x - m) r, g = dy gamma:
//   dx = r (g - mean g - h mean (g h)),  dgamma = sum_rows dy h,  dbeta = sum_rows dy.
// Statistics and sums are fp32.  The sum's mean m' is off by some roundings of the row's size, which for a
// row far from 0 could be more than its spread (a constant row at 3e5 could come out as +-1 for 0), so
// forward the differences c = x - m' are centred once more: m = m' + mean c, v = mean c^2 - (mean c)^2,
// y = (c - mean c) r gamma + beta.  Backward x - m is as good as the mean given, half an fp32 step of it.
//
// Both are bound by memory (forward one read and one write of the rows,
// backward two and one), so a row is read once and kept in registers between its
// sums: RT threads a row (16 for narrow rows, so that 16 share a block, a wave,
// or a block) with E vectors of 16 bytes each.  Blocks keep gamma and beta in registers and
// take row after row; backward they also keep their columns' part of dgamma and dbeta,
// which a second launch adds in the order of the blocks.  Rows past the widest
// of these (2,048 vectors) are read from memory again for each sum (with 1,024 threads of four vectors the
// registers spill in 16 bits: 1,024 x 20,000 bf16 106 us, 25 so; fp32 2,048 x 16,384 66 and 82, 512 x 10,000 13.5 and 12.3).
// 16,384 x 4,096 bf16 forward 48 us (5.6 TB/s), 16,384 x 2,048 backward 38 and 5 for the
// parts (5.3 TB/s); a large copy 4.7.
#include "wr_ops.h"

namespace {

// Vectors of a row, threads on it, vectors a thread: the first line with room.
struct NormShape {
  int vecs, rt, e;
};
constexpr NormShape kShapes[] = {{16, 16, 1},  {64, 64, 1},    {128, 64, 2},   {256, 64, 4},
                                 {512, 256, 2}, {1024, 512, 2}, {2048, 512, 4}};

#define NORM_BLOCKS 2048       // forward: eight blocks of 256 threads a CU
#define NORM_GRAD_BT 512       // backward: threads of a block, where a row takes fewer

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

// Sum over the wave's lanes of a row, in every one of them: within 16 lanes by rotations, which need no LDS and
// pair the same operands as exchanges would (65,536 x 256 fp32 forward 22.4 us, by exchanges 23.7).
template <int N>
__device__ __forceinline__ float rotate_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + N, 0xf, 0xf, true));
}
template <int RT>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (RT > 32) v += __shfl_xor(v, 32, 64);
  if constexpr (RT > 16) v += __shfl_xor(v, 16, 64);
  return rotate_add<1>(rotate_add<2>(rotate_add<4>(rotate_add<8>(v))));
}
// Sums of K values over the RT threads of a row; `s` (RT > 64): [waves of the block][K], another one for the next sum.
template <int RT, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float* s) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = group_sum<RT>(v[k]);
  if constexpr (RT > 64) {
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) s[(threadIdx.x >> 6) * K + k] = v[k];
    __syncthreads();
    s += threadIdx.x / RT * (RT / 64) * K;   // this row's waves
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = s[k];
#pragma unroll
      for (int w = 1; w < RT / 64; ++w) v[k] += s[w * K + k];
    }
  }
}

// 1 / sqrt(variance + eps) from the mean square and the mean of the differences.
__device__ __forceinline__ float norm_rstd(float square, float dm, float eps) {
  const float v = square - (square > 3.0e38f ? 0.0f : dm * dm);   // (past fp32's range both may be infinite)
  return 1.0f / sqrtf((v < 0.0f ? 0.0f : v) + eps);               // (a NaN stays)
}

// Columns of thread t's vector e: where it begins, how many of its first elements are not its own
// (all VW past the row), and how many there are to load and store (0 past the row, the row's if it
// is shorter than a vector).
template <int RT, int VW>
struct NormCols {
  int c, skip, count;
  __device__ __forceinline__ NormCols(int e, int t, int d) {
    const int c0 = (e * RT + t) * VW;
    c = d < VW ? 0 : vec_begin<VW>(c0, d);
    skip = c0 >= d ? VW : c0 - c;
    count = c0 >= d ? 0 : d < VW ? d : VW;
  }
  // A sum over the vector's own elements: add(k, s) is s with element k added.
  template <class F>
  __device__ __forceinline__ float sum(F add) const {
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < VW; ++k) s = add(k, s);
    if (skip > 0 || count < VW) {   // (no lane of most waves)
      s = 0.0f;
#pragma unroll
      for (int k = 0; k < VW; ++k) s = k >= skip && k < count ? add(k, s) : s;
    }
    return s;
  }
};

template <class T, class W, int RT, int E>
__global__ __launch_bounds__(RT < 256 ? 256 : RT) void wr_norm_kernel(NormArgs a) {
  constexpr int VW = 16 / sizeof(T), BT = RT < 256 ? 256 : RT, G = BT / RT;
  __shared__ float red[2][BT / 64 * 2];
  const int t = threadIdx.x % RT;
  const float inv_d = 1.0f / (float)a.d;
  Raw<W, VW> ga[E], be[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const NormCols<RT, VW> q(e, t, a.d);
    ga[e] = load_raw<W, VW>((const W*)a.gamma + q.c, a.gamma ? q.count : 0, (W)1.0f);
    be[e] = load_raw<W, VW>((const W*)a.beta + q.c, a.beta ? q.count : 0);
  }
  for (int64_t i0 = (int64_t)blockIdx.x * G; i0 < a.n; i0 += (int64_t)gridDim.x * G) {
    const int64_t i = i0 + threadIdx.x / RT;
    const bool on = i < a.n;   // (only the last rows of a block that shares rows; its sums stay in the group)
    const T* x = (const T*)a.x + i * a.x_stride;
    T* y = (T*)a.y + i * a.y_stride;
    Raw<T, VW> raw[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const NormCols<RT, VW> q(e, t, a.d);
      raw[e] = load_raw<T, VW>(x + q.c, on ? q.count : 0);
    }
    float v[E][VW], s[1] = {0.0f};
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const NormCols<RT, VW> q(e, t, a.d);
#pragma unroll
      for (int k = 0; k < VW; ++k) v[e][k] = (float)raw[e][k];
      s[0] += q.sum([&](int k, float s) { return s + v[e][k]; });
    }
    row_sums<RT, 1>(s, red[0]);
    const float m = s[0] * inv_d;
    float c[2] = {0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const NormCols<RT, VW> q(e, t, a.d);
#pragma unroll
      for (int k = 0; k < VW; ++k) v[e][k] -= m;
      c[0] += q.sum([&](int k, float s) { return s + v[e][k]; });
      c[1] += q.sum([&](int k, float s) { return __builtin_fmaf(v[e][k], v[e][k], s); });
    }
    row_sums<RT, 2>(c, red[1]);
    const float dm = c[0] * inv_d, r = norm_rstd(c[1] * inv_d, dm, a.eps);
    if (on) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const NormCols<RT, VW> q(e, t, a.d);
#pragma unroll
        for (int k = 0; k < VW; ++k) v[e][k] = __builtin_fmaf((v[e][k] - dm) * r, (float)ga[e][k], (float)be[e][k]);
        store_part<T, VW>(y + q.c, v[e], q.count);
      }
      if (t == 0) {
        if (a.mean) a.mean[i] = m + dm;
        if (a.rstd) a.rstd[i] = r;
      }
    }
  }
}

// Rows of any width, read three times.
template <class T, class W>
__global__ __launch_bounds__(1024) void wr_norm_wide_kernel(NormArgs a) {
  constexpr int VW = 16 / sizeof(T), RT = 1024;
  __shared__ float red[2][RT / 64 * 2];
  for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x) {
    const T* x = (const T*)a.x + i * a.x_stride;
    T* y = (T*)a.y + i * a.y_stride;
    float s[1] = {0.0f}, v[VW];
    for (int64_t c = threadIdx.x * VW; c < a.d; c += RT * VW) {
      load_part<T, VW>(x + c, v, (int)(a.d - c));
#pragma unroll
      for (int k = 0; k < VW; ++k) s[0] += v[k];
    }
    row_sums<RT, 1>(s, red[0]);
    const float m = s[0] / (float)a.d;
    float cs[2] = {0.0f, 0.0f};
    for (int64_t c = threadIdx.x * VW; c < a.d; c += RT * VW) {
      load_part<T, VW>(x + c, v, (int)(a.d - c));
#pragma unroll
      for (int k = 0; k < VW; ++k)
        if (c + k < a.d) cs[0] += v[k] - m, cs[1] = __builtin_fmaf(v[k] - m, v[k] - m, cs[1]);
    }
    row_sums<RT, 2>(cs, red[1]);
    const float dm = cs[0] / (float)a.d, r = norm_rstd(cs[1] / (float)a.d, dm, a.eps);
    for (int64_t c = threadIdx.x * VW; c < a.d; c += RT * VW) {
      const int count = (int)(a.d - c);
      float ga[VW], be[VW];
#pragma unroll
      for (int k = 0; k < VW; ++k) ga[k] = 1.0f, be[k] = 0.0f;
      if (a.gamma) load_part<W, VW>((const W*)a.gamma + c, ga, count);
      if (a.beta) load_part<W, VW>((const W*)a.beta + c, be, count);
      load_part<T, VW>(x + c, v, count);
#pragma unroll
      for (int k = 0; k < VW; ++k) v[k] = __builtin_fmaf((v[k] - m - dm) * r, ga[k], be[k]);
      store_part<T, VW>(y + c, v, count);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[i] = m + dm;
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
  float* part;   // [parts][2][d]
  int parts;
};

// dx, and with WG this block's part of dgamma and dbeta.
template <class T, class W, int RT, int E, bool WG>
__global__ __launch_bounds__(RT < NORM_GRAD_BT ? NORM_GRAD_BT : RT) void wr_norm_grad_kernel(NormGradArgs a) {
  constexpr int VW = 16 / sizeof(T), BT = RT < NORM_GRAD_BT ? NORM_GRAD_BT : RT, G = BT / RT;
  __shared__ float red[2][BT / 64 * 2];
  const int t = threadIdx.x % RT;
  const float inv_d = 1.0f / (float)a.d;
  Raw<W, VW> ga[E];
  float dg[E][VW], db[E][VW];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const NormCols<RT, VW> q(e, t, a.d);
    ga[e] = load_raw<W, VW>((const W*)a.gamma + q.c, a.gamma ? q.count : 0, (W)1.0f);
#pragma unroll
    for (int k = 0; k < VW; ++k) dg[e][k] = db[e][k] = 0.0f;
  }
  int turn = 0;
  for (int64_t i0 = (int64_t)blockIdx.x * G; i0 < a.n; i0 += (int64_t)gridDim.x * G, turn ^= 1) {
    const int64_t i = i0 + threadIdx.x / RT;
    const bool on = i < a.n;
    Raw<T, VW> rx[E], ry[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const NormCols<RT, VW> q(e, t, a.d);
      rx[e] = load_raw<T, VW>((const T*)a.x + i * a.x_stride + q.c, on ? q.count : 0);
      ry[e] = load_raw<T, VW>((const T*)a.dy + i * a.dy_stride + q.c, on ? q.count : 0);
    }
    const float m = on ? a.mean[i] : 0.0f, r = on ? a.rstd[i] : 0.0f;
    float h[E][VW], g[E][VW], s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const NormCols<RT, VW> q(e, t, a.d);
#pragma unroll
      for (int k = 0; k < VW; ++k) {
        h[e][k] = ((float)rx[e][k] - m) * r;
        g[e][k] = (float)ry[e][k];
        if constexpr (WG) {   // (each thread sums all its columns: a column of two threads comes out the same in both)
          dg[e][k] = __builtin_fmaf(g[e][k], h[e][k], dg[e][k]);
          db[e][k] += g[e][k];
        }
        g[e][k] *= (float)ga[e][k];
      }
      s[0] += q.sum([&](int k, float s) { return s + g[e][k]; });
      s[1] += q.sum([&](int k, float s) { return __builtin_fmaf(g[e][k], h[e][k], s); });
    }
    row_sums<RT, 2>(s, red[turn]);
    if (on && a.dx) {
      const float m0 = s[0] * inv_d, m1 = s[1] * inv_d;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const NormCols<RT, VW> q(e, t, a.d);
#pragma unroll
        for (int k = 0; k < VW; ++k) g[e][k] = r * (g[e][k] - __builtin_fmaf(h[e][k], m1, m0));
        store_part<T, VW>((T*)a.dx + i * a.dx_stride + q.c, g[e], q.count);
      }
    }
  }
  if constexpr (WG) {
    // (a single block's part is the whole)
    float* pg = a.parts > 1 ? a.part + (int64_t)blockIdx.x * 2 * a.d : a.dgamma;
    float* pb = a.parts > 1 ? pg + a.d : a.dbeta;
    if constexpr (G > 1) {   // the block's groups, in order
      __shared__ float sum[2][VW][BT];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < VW; ++k) sum[0][k][threadIdx.x] = dg[e][k], sum[1][k][threadIdx.x] = db[e][k];
        __syncthreads();
        if (threadIdx.x < RT) {
#pragma unroll
          for (int k = 0; k < VW; ++k)
#pragma unroll
            for (int q = 1; q < G; ++q) {
              dg[e][k] += sum[0][k][q * RT + t];
              db[e][k] += sum[1][k][q * RT + t];
            }
        }
      }
      if (threadIdx.x >= RT) return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const NormCols<RT, VW> q(e, t, a.d);
      store_part<float, VW>(pg + q.c, dg[e], pg ? q.count : 0);
      store_part<float, VW>(pb + q.c, db[e], pb ? q.count : 0);
    }
  }
}

template <class T, class W>
__global__ __launch_bounds__(1024) void wr_norm_grad_wide_kernel(NormGradArgs a) {
  constexpr int VW = 16 / sizeof(T), RT = 1024;
  __shared__ float red[2][RT / 64 * 2];
  int turn = 0;
  for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x, turn ^= 1) {
    const T *x = (const T*)a.x + i * a.x_stride, *dy = (const T*)a.dy + i * a.dy_stride;
    const float m = a.mean[i], r = a.rstd[i];
    float s[2] = {0.0f, 0.0f}, h[VW], g[VW], ga[VW];
    auto read = [&](int64_t c) {
      const int count = (int)(a.d - c);
#pragma unroll
      for (int k = 0; k < VW; ++k) ga[k] = 1.0f;
      if (a.gamma) load_part<W, VW>((const W*)a.gamma + c, ga, count);
      load_part<T, VW>(x + c, h, count);
      load_part<T, VW>(dy + c, g, count);
#pragma unroll
      for (int k = 0; k < VW; ++k) h[k] = (h[k] - m) * r, g[k] *= ga[k];
    };
    for (int64_t c = threadIdx.x * VW; c < a.d; c += RT * VW) {
      read(c);
#pragma unroll
      for (int k = 0; k < VW; ++k) s[0] += g[k], s[1] = __builtin_fmaf(g[k], h[k], s[1]);
    }
    row_sums<RT, 2>(s, red[turn]);
    const float m0 = s[0] / (float)a.d, m1 = s[1] / (float)a.d;
    for (int64_t c = threadIdx.x * VW; c < a.d; c += RT * VW) {
      read(c);
#pragma unroll
      for (int k = 0; k < VW; ++k) g[k] = r * (g[k] - __builtin_fmaf(h[k], m1, m0));
      store_part<T, VW>((T*)a.dx + i * a.dx_stride + c, g, (int)(a.d - c));
    }
  }
}

// dgamma's and dbeta's parts of wide rows: block (x, y) takes 1,024 columns of every gridDim.y-th row.
template <class T>
__global__ __launch_bounds__(256) void wr_norm_wide_dw_kernel(NormGradArgs a) {
  const int64_t c = (int64_t)blockIdx.x * 1024 + threadIdx.x * 4;
  if (c >= a.d) return;
  const int count = (int)std::min<int64_t>(4, a.d - c);
  float dg[4] = {}, db[4] = {}, x[4], dy[4];
#pragma unroll 4
  for (int64_t i = blockIdx.y; i < a.n; i += gridDim.y) {
    const float m = a.mean[i], r = a.rstd[i];
    load_part<T, 4>((const T*)a.x + i * a.x_stride + c, x, count);
    load_part<T, 4>((const T*)a.dy + i * a.dy_stride + c, dy, count);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      dg[k] = __builtin_fmaf(dy[k], (x[k] - m) * r, dg[k]);
      db[k] += dy[k];
    }
  }
  float* pg = a.parts > 1 ? a.part + (int64_t)blockIdx.y * 2 * a.d : a.dgamma;
  float* pb = a.parts > 1 ? pg + a.d : a.dbeta;
  store_part<float, 4>(pg + c, dg, pg ? count : 0);
  store_part<float, 4>(pb + c, db, pb ? count : 0);
}

// The parts of 64 sums added: each of 16 waves every 16th part, then the waves in order.  (Blocks stride over
// the sums: a block each would pass the grid limit from 2^27 columns on.)
__global__ __launch_bounds__(1024) void wr_norm_parts_kernel(NormGradArgs a) {
  __shared__ float sum[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t n = 2 * (int64_t)a.d;
  for (int64_t c0 = (int64_t)blockIdx.x * 64; c0 < n; c0 += (int64_t)gridDim.x * 64) {
    const int64_t c = c0 + lane;
    float s = 0.0f;
    if (c < n)
#pragma unroll 8
      for (int p = w; p < a.parts; p += 16) s += a.part[(int64_t)p * n + c];
    sum[w][lane] = s;
    __syncthreads();
    if (w == 0 && c < n) {
#pragma unroll
      for (int q = 1; q < 16; ++q) s += sum[q][lane];
      float* o = c < a.d ? a.dgamma : a.dbeta;
      if (o) o[c < a.d ? c : c - a.d] = s;
    }
    __syncthreads();
  }
}

wavernn_status check_norm(int dtype, int w_dtype, int64_t n, int32_t d) {
  if (!wr_dtype_ok(dtype) || !wr_dtype_ok(w_dtype)) return wr_fail(WAVERNN_E_INVALID, "bad dtype");
  if (w_dtype != dtype && w_dtype != WAVERNN_F32)
    return wr_fail(WAVERNN_E_INVALID, "gamma's and beta's dtype must be the rows' or F32");
  if (n < 0 || n > INT32_MAX) return wr_fail(WAVERNN_E_INVALID, "n_rows %lld out of range", (long long)n);
  if (d < 1 || d > (1 << 30)) return wr_fail(WAVERNN_E_INVALID, "dim %d not in [1, 2^30]", d);
  return WAVERNN_OK;
}

// Index into kShapes for rows of `vecs` vectors, or the number of shapes (wide rows).
int norm_shape(int64_t vecs) {
  int i = 0;
  while (i < (int)(sizeof kShapes / sizeof kShapes[0]) && vecs > kShapes[i].vecs) ++i;
  return i;
}
// Runs `body` with the shape's RT and E, `wide` if the rows are wider than all of them.
#define NORM_SHAPE(i, RT, E, wide, ...)                              \
  switch (i) {                                                       \
    case 0: { constexpr int RT = kShapes[0].rt, E = kShapes[0].e; __VA_ARGS__; } break; \
    case 1: { constexpr int RT = kShapes[1].rt, E = kShapes[1].e; __VA_ARGS__; } break; \
    case 2: { constexpr int RT = kShapes[2].rt, E = kShapes[2].e; __VA_ARGS__; } break; \
    case 3: { constexpr int RT = kShapes[3].rt, E = kShapes[3].e; __VA_ARGS__; } break; \
    case 4: { constexpr int RT = kShapes[4].rt, E = kShapes[4].e; __VA_ARGS__; } break; \
    case 5: { constexpr int RT = kShapes[5].rt, E = kShapes[5].e; __VA_ARGS__; } break; \
    case 6: { constexpr int RT = kShapes[6].rt, E = kShapes[6].e; __VA_ARGS__; } break; \
    default: wide;                                                   \
  }

template <class T, class W>
wavernn_status run_norm(NormArgs& a, void* stream) {
  const int64_t vecs = ((int64_t)a.d * sizeof(T) + 15) / 16;
  NORM_SHAPE(norm_shape(vecs), RT, E, WR_LAUNCH((wr_norm_wide_kernel<T, W>), std::min<int64_t>(a.n, NORM_BLOCKS), 1024, 0, stream, a),
             constexpr int BT = RT < 256 ? 256 : RT;
             const int64_t blocks = (a.n + BT / RT - 1) / (BT / RT);
             WR_LAUNCH((wr_norm_kernel<T, W, RT, E>), std::min<int64_t>(blocks, NORM_BLOCKS), BT, 0, stream, a));
  return WAVERNN_OK;
}

// Parts of dgamma and dbeta of a call (dtype's bytes matter to the shape), a block each: one a CU where a
// thread keeps 16 columns, two where fewer (20,000 x 257 fp32, 8 columns: 16.7 us with 512 parts, 20.0 with 256;
// 20,000 x 768 bf16, 16 columns: 27.7 and 24.9, the parts being large), and two rows for each group of threads at
// least (1,999 x 1,001 fp16, 125 parts, 12.9 us; with four rows 14.5, with one 12.4; 100 x 8,192 fp32 11.0, 13.0 and 11.7).
int norm_parts(int64_t n, int32_t d, int bytes) {
  const int i = norm_shape(((int64_t)d * bytes + 15) / 16);
  const bool wide = i >= (int)(sizeof kShapes / sizeof kShapes[0]);
  const int rt = wide ? NORM_GRAD_BT : kShapes[i].rt, g = rt < NORM_GRAD_BT ? NORM_GRAD_BT / rt : 1;
  return (int)std::min<int64_t>(!wide && kShapes[i].e * 16 / bytes >= 16 ? 256 : 512, std::max<int64_t>(1, (n + 2 * g - 1) / (2 * g)));
}

template <class T, class W>
wavernn_status run_norm_grad(NormGradArgs& a, void* stream) {
  const int64_t vecs = ((int64_t)a.d * sizeof(T) + 15) / 16;
  const bool wg = a.dgamma || a.dbeta;
  a.parts = norm_parts(a.n, a.d, sizeof(T));
  if (a.n > 0) {
    NORM_SHAPE(norm_shape(vecs), RT, E,
               if (wg) {   // before dx, which may replace dy or x
                 void* argv[] = {&a};
                 const hipError_t e = hipLaunchKernel((const void*)wr_norm_wide_dw_kernel<T>,
                                                      dim3((unsigned)((a.d + 1023LL) / 1024), (unsigned)a.parts), dim3(256),
                                                      argv, 0, (hipStream_t)stream);
                 if (e != hipSuccess) return wr_fail(WAVERNN_E_HIP, "launch of wr_norm_wide_dw_kernel: %s", hipGetErrorString(e));
               }
               if (a.dx) WR_LAUNCH((wr_norm_grad_wide_kernel<T, W>), std::min<int64_t>(a.n, NORM_BLOCKS), 1024, 0, stream, a),
               constexpr int BT = RT < NORM_GRAD_BT ? NORM_GRAD_BT : RT;
               if (wg) WR_LAUNCH((wr_norm_grad_kernel<T, W, RT, E, true>), a.parts, BT, 0, stream, a);
               else WR_LAUNCH((wr_norm_grad_kernel<T, W, RT, E, false>),
                              std::min<int64_t>((a.n + BT / RT - 1) / (BT / RT), NORM_BLOCKS), BT, 0, stream, a));
  } else {
    a.parts = 0;
  }
  if (wg && a.parts != 1)
    WR_LAUNCH(wr_norm_parts_kernel, std::min<int64_t>((2 * (int64_t)a.d + 63) / 64, WR_OP_BLOCKS), 1024, 0, stream, a);
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
  WR_DISPATCH(dtype, T, return w_dtype == WAVERNN_F32 ? run_norm<T, float>(a, stream) : run_norm<T, T>(a, stream));
}

int64_t wavernn_layer_norm_grad_workspace(int64_t n_rows, int32_t dim) {
  if (n_rows < 0 || n_rows > INT32_MAX || dim < 1 || dim > (1 << 30)) return -1;
  const int parts = std::max(norm_parts(n_rows, dim, 2), norm_parts(n_rows, dim, 4));
  return n_rows > 0 && parts > 1 ? (int64_t)8 * dim * parts : 0;
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
  if (!dx_dev && !dgamma_dev && !dbeta_dev) return WAVERNN_OK;
  const int64_t need = dgamma_dev || dbeta_dev ? wavernn_layer_norm_grad_workspace(n_rows, dim) : 0;
  if (need > 0 && (!workspace_dev || workspace_bytes < need || !wr_aligned(workspace_dev, 16)))
    return wr_fail(WAVERNN_E_INVALID, "workspace: %lld bytes needed, 16-byte aligned", (long long)need);
  NormGradArgs a{dy_dev, x_dev, n_rows, dy_stride, x_stride, dim, gamma_dev, mean_dev, rstd_dev, dx_dev, dx_stride,
                 dgamma_dev, dbeta_dev, (float*)workspace_dev, 0};
  WR_DISPATCH(dtype, T, return w_dtype == WAVERNN_F32 ? run_norm_grad<T, float>(a, stream) : run_norm_grad<T, T>(a, stream));
}

}  // extern "C"
