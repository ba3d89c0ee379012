// Log probabilities of given tokens with the entropy and the top alternatives
// of their distributions, and the gradient of all of them with respect to the
// logits.  For a row z of V logits with m = max z, s = sum e^(z - m):
//   lse = m + log s,  logp = z_t - lse,
//   H = -sum p log p = log s - sum (z - m) e^(z - m) / s
// (both terms of H are >= 0, so nothing cancels), and the top K by (z
// descending, number ascending).  Sums are fp32.
//   dz_j = [j = t] g_logp + sum_k [j = top_k] g_top_k
//        + p_j (g_lse - g_logp - sum_k g_top_k) - g_H p_j (log p_j + H)
#include <math.h>

#include "wr_kern.h"
#include "wr_logp.h"
#include "wr_ops.h"

namespace {

// The token of a row; negative: the row is padding.
__device__ __forceinline__ int64_t row_token(const LogpArgs& a, int64_t row) {
  switch (a.kind) {
    case WR_TOK_NONE: return 0;
    case WR_TOK_I32: return ((const int32_t*)a.tokens)[row];
    case WR_TOK_I64: return ((const int64_t*)a.tokens)[row];
    case WR_TOK_HIGH: return ((const uint16_t*)a.tokens)[row] >> 8;
    case WR_TOK_LOW: return ((const uint16_t*)a.tokens)[row] & 255;
    default: {   // nibbles: rows 2 i and 2 i + 1 are the high and low nibble of byte i
      const int u = ((const uint16_t*)a.tokens)[row >> 1], b = a.kind == WR_TOK_HIGH4 ? u >> 8 : u & 255;
      return row & 1 ? b & 15 : b >> 4;
    }
  }
}
// Where a row's results go: [sample][coarse, fine] for bytes, [sample][4] for nibbles.
__device__ __forceinline__ int64_t row_out(const LogpArgs& a, int64_t row) {
  switch (a.kind) {
    case WR_TOK_HIGH: return 2 * row;
    case WR_TOK_LOW: return 2 * row + 1;
    case WR_TOK_HIGH4: return 2 * row - (row & 1);
    case WR_TOK_LOW4: return 2 * row - (row & 1) + 2;
    default: return row;
  }
}

// Order of the alternatives as whole numbers: a logit's rank in the upper half
// (NaN above all, -0 equal to +0), its number complemented in the lower, so
// that no two classes compare equal.
__device__ __forceinline__ u64 top_key(float z, int j) {
  uint32_t u = __float_as_uint(z + 0.0f);
  u = z != z ? 0xfffffffeu : (u >> 31) ? ~u : u | 0x80000000u;
  return (u64)u << 32 | (uint32_t)~j;
}
__device__ __forceinline__ float key_value(u64 k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return __uint_as_float(u == 0xfffffffeu ? 0x7fc00000u : (u >> 31) ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_class(u64 k) { return (int)~(uint32_t)k; }

__device__ __forceinline__ u64 shfl_max(u64 v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const u64 w = __shfl_xor(v, o, 64);
    v = w > v ? w : v;
  }
  return v;
}

// Running maximum, sum of e^(z - m) and sum of (z - m) e^(z - m).
struct Soft {
  float m, s, w;
};
// Differences are held above this where they multiply a weight that is zero
// (masked classes, the type's lowest value), so that no 0 * inf arises.
#define WR_FAR -1e20f
__device__ __forceinline__ float soft_base(float m) { return m == -__builtin_inff() ? 0.0f : m; }
// The state against a maximum m2 >= a.m.
__device__ __forceinline__ Soft soft_at(Soft a, float m2) {
  if (a.s == 0.0f) return Soft{m2, 0.0f, 0.0f};
  const float d = fmaxf(a.m - soft_base(m2), WR_FAR), c = fexp(d);
  return Soft{m2, a.s * c, (a.w + d * a.s) * c};
}
__device__ __forceinline__ Soft soft_join(Soft a, Soft b) {
  const float m = fmaxf(a.m, b.m);
  a = soft_at(a, m);
  b = soft_at(b, m);
  return Soft{m, a.s + b.s, a.w + b.w};
}
__device__ __forceinline__ void soft_add(Soft& a, float z) {
  if (z > a.m) a = soft_at(a, z);
  const float d = z - soft_base(a.m), e = fexp(d);
  a.s += e;
  a.w += fmaxf(d, WR_FAR) * e;   // (a masked class: e = 0 and no 0 * inf)
}

// One block a row, any number of classes.
template <class T>
__global__ __launch_bounds__(256) void wr_logp_kernel(LogpArgs a) {
  __shared__ Soft ss[4];
  __shared__ u64 sk[4];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const int64_t t = row_token(a, row), o = row_out(a, row);
    if (t < 0) {
      if (tid == 0) {
        if (a.logp) a.logp[o] = 0.0f;
        if (a.entropy) a.entropy[o] = 0.0f;
        if (a.lse) a.lse[o] = 0.0f;
      }
      if (tid < a.top) a.top_logp[o * a.top + tid] = 0.0f, a.top_idx[o * a.top + tid] = -1;
      continue;
    }
    const T* z = (const T*)a.logits + row * a.stride;
    Soft q{-__builtin_inff(), 0.0f, 0.0f};
    for (int j = tid; j < a.v; j += 256) soft_add(q, (float)z[j]);
    for (int d = 32; d >= 1; d >>= 1)
      q = soft_join(q, Soft{__shfl_xor(q.m, d, 64), __shfl_xor(q.s, d, 64), __shfl_xor(q.w, d, 64)});
    __syncthreads();   // the previous row's results are read
    if (lane == 0) ss[wave] = q;
    __syncthreads();
    q = soft_join(soft_join(ss[0], ss[1]), soft_join(ss[2], ss[3]));
    const float lse = soft_base(q.m) + logf(q.s);
    if (tid == 0) {
      if (a.logp) a.logp[o] = t < a.v ? (float)z[t] - (q.s == 0.0f ? 0.0f : lse) : __builtin_nanf("");
      if (a.entropy) a.entropy[o] = q.s == 0.0f ? 0.0f : logf(q.s) - q.w / q.s;
      if (a.lse) a.lse[o] = lse;
    }
    u64 prev = ~0ull;
    for (int k = 0; k < a.top; ++k) {
      u64 best = 0;
      for (int j = tid; j < a.v; j += 256) {
        const u64 key = top_key((float)z[j], j);
        if (key < prev && key > best) best = key;
      }
      best = shfl_max(best);
      __syncthreads();
      if (lane == 0) sk[wave] = best;
      __syncthreads();
      for (int i = 0; i < 4; ++i) best = sk[i] > best ? sk[i] : best;
      if (tid == 0) {
        a.top_idx[o * a.top + k] = key_class(best);
        a.top_logp[o * a.top + k] = key_value(best) - (q.s == 0.0f ? 0.0f : lse);
      }
      prev = best;
    }
  }
}

template <class T>
__global__ __launch_bounds__(256) void wr_logp_grad_kernel(LogpGradArgs a) {
  for (int64_t row = blockIdx.x; row < a.f.n; row += gridDim.x) {
    const int64_t t = row_token(a.f, row);
    const T* z = (const T*)a.f.logits + row * a.f.stride;
    T* dz = (T*)a.dlogits + row * a.dstride;
    const float lse = t < 0 ? 0.0f : a.lse_in[row];
    if (t < 0 || lse == -__builtin_inff()) {   // padding, or every class masked
      for (int j = threadIdx.x; j < a.f.v; j += 256) dz[j] = (T)0.0f;
      continue;
    }
    float gl = a.g_logp ? a.g_logp[row] : 0.0f, gp = (a.g_lse ? a.g_lse[row] : 0.0f) - gl;
    const float gh = a.g_entropy ? a.g_entropy[row] : 0.0f, h = a.g_entropy ? a.entropy_in[row] : 0.0f;
    if (a.g_logp && t >= a.f.v) gp = __builtin_nanf("");
    for (int k = 0; k < a.f.top; ++k)
      if (a.f.top_idx[row * a.f.top + k] >= 0) gp -= a.g_top[row * a.f.top + k];
    for (int j = threadIdx.x; j < a.f.v; j += 256) {
      const float lp = (float)z[j] - lse, p = fexp(lp);
      float g = p * (gp - gh * (fmaxf(lp, WR_FAR) + h));
      if (j == t) g += gl;
      for (int k = 0; k < a.f.top; ++k)
        if (a.f.top_idx[row * a.f.top + k] == j) g += a.g_top[row * a.f.top + k];
      dz[j] = (T)g;
    }
  }
}

wavernn_status check_logits(const char* name, int dtype, const void* p, int64_t n, int32_t v, int64_t stride, bool output) {
  if (!wr_dtype_ok(dtype)) return wr_fail(WAVERNN_E_INVALID, "bad dtype %d", dtype);
  if (n < 0 || n > INT32_MAX) return wr_fail(WAVERNN_E_INVALID, "n_rows %lld out of range", (long long)n);
  if (v < 1) return wr_fail(WAVERNN_E_INVALID, "n_classes %d: must be positive", v);
  return wr_check_rows(name, p, dtype, n, v, stride, output);
}
wavernn_status check_tokens(const void* tokens, int bytes, int* kind) {
  if (tokens && bytes != 4 && bytes != 8) return wr_fail(WAVERNN_E_INVALID, "token_bytes %d: must be 4 or 8", bytes);
  if (!wr_aligned(tokens, tokens ? bytes : 1)) return wr_fail(WAVERNN_E_INVALID, "tokens are not aligned to their elements");
  *kind = !tokens ? WR_TOK_NONE : bytes == 4 ? WR_TOK_I32 : WR_TOK_I64;
  return WAVERNN_OK;
}

}  // namespace

wavernn_status wr_logp_launch(int dtype, LogpArgs& a, void* stream) {
  if (a.n == 0) return WAVERNN_OK;
  const int64_t grid = std::min<int64_t>(a.n, WR_OP_BLOCKS);
  WR_DISPATCH(dtype, T, WR_LAUNCH((wr_logp_kernel<T>), grid, 256, 0, stream, a));
  return WAVERNN_OK;
}

extern "C" {

int64_t wavernn_token_logprobs_workspace(int64_t n_rows, int32_t n_classes, int32_t top) {
  if (n_rows < 0 || n_rows > INT32_MAX || n_classes < 1 || top < 0 || top > WAVERNN_MAX_TOP || top > n_classes) return -1;
  return 0;
}

wavernn_status wavernn_token_logprobs(int32_t dtype, const void* logits_dev, int64_t n_rows, int32_t n_classes,
                                      int64_t row_stride, const void* tokens_dev, int32_t token_bytes, int32_t top,
                                      float* logp_dev, float* entropy_dev, float* lse_dev, float* top_logp_dev,
                                      int32_t* top_idx_dev, void* workspace_dev, int64_t workspace_bytes, void* stream) {
  LogpArgs a = {};
  wavernn_status s;
  if ((s = check_logits("logits", dtype, logits_dev, n_rows, n_classes, row_stride, false)) != WAVERNN_OK) return s;
  if ((s = check_tokens(tokens_dev, token_bytes, &a.kind)) != WAVERNN_OK) return s;
  if (logp_dev && !tokens_dev && n_rows > 0) return wr_fail(WAVERNN_E_INVALID, "logp without tokens");
  if (top < 0 || top > WAVERNN_MAX_TOP || top > n_classes)
    return wr_fail(WAVERNN_E_INVALID, "top %d not in [0, min(%d, n_classes)]", top, WAVERNN_MAX_TOP);
  if (top > 0 && n_rows > 0 && (!top_logp_dev || !top_idx_dev)) return wr_fail(WAVERNN_E_INVALID, "top_logp or top_idx is null");
  const int64_t need = wavernn_token_logprobs_workspace(n_rows, n_classes, top);
  if (need > 0 && (!workspace_dev || workspace_bytes < need || !wr_aligned(workspace_dev, 16)))
    return wr_fail(WAVERNN_E_INVALID, "workspace: %lld bytes needed, 16-byte aligned", (long long)need);
  a.logits = logits_dev;
  a.n = n_rows;
  a.v = n_classes;
  a.stride = row_stride;
  a.tokens = tokens_dev;
  a.top = top;
  a.logp = logp_dev;
  a.entropy = entropy_dev;
  a.lse = lse_dev;
  a.top_logp = top_logp_dev;
  a.top_idx = top_idx_dev;
  return wr_logp_launch(dtype, a, stream);
}

wavernn_status wavernn_token_logprobs_grad(int32_t dtype, const void* logits_dev, int64_t n_rows, int32_t n_classes,
                                           int64_t row_stride, const void* tokens_dev, int32_t token_bytes,
                                           const float* lse_dev, const float* entropy_dev, const float* g_logp_dev,
                                           const float* g_entropy_dev, const float* g_lse_dev, int32_t top,
                                           const int32_t* top_idx_dev, const float* g_top_dev, void* dlogits_dev,
                                           int64_t dlogits_stride, void* stream) {
  LogpGradArgs a = {};
  wavernn_status s;
  if ((s = check_logits("logits", dtype, logits_dev, n_rows, n_classes, row_stride, false)) != WAVERNN_OK) return s;
  if ((s = check_logits("dlogits", dtype, dlogits_dev, n_rows, n_classes, dlogits_stride, true)) != WAVERNN_OK) return s;
  if ((s = check_tokens(tokens_dev, token_bytes, &a.f.kind)) != WAVERNN_OK) return s;
  if (n_rows == 0) return WAVERNN_OK;
  if (!lse_dev) return wr_fail(WAVERNN_E_INVALID, "lse is null");
  if (g_logp_dev && !tokens_dev) return wr_fail(WAVERNN_E_INVALID, "g_logp without tokens");
  if (g_entropy_dev && !entropy_dev) return wr_fail(WAVERNN_E_INVALID, "g_entropy without entropy");
  if (top < 0 || top > WAVERNN_MAX_TOP || top > n_classes)
    return wr_fail(WAVERNN_E_INVALID, "top %d not in [0, min(%d, n_classes)]", top, WAVERNN_MAX_TOP);
  if (top > 0 && (!top_idx_dev || !g_top_dev)) return wr_fail(WAVERNN_E_INVALID, "top_idx or g_top is null");
  if (dlogits_dev == logits_dev && dlogits_stride != row_stride)
    return wr_fail(WAVERNN_E_INVALID, "dlogits in place of logits needs the same row stride");
  a.f.logits = logits_dev;
  a.f.n = n_rows;
  a.f.v = n_classes;
  a.f.stride = row_stride;
  a.f.tokens = tokens_dev;
  a.f.top = top;
  a.f.top_idx = (int32_t*)top_idx_dev;
  a.lse_in = lse_dev;
  a.entropy_in = entropy_dev;
  a.g_logp = g_logp_dev;
  a.g_entropy = g_entropy_dev;
  a.g_lse = g_lse_dev;
  a.g_top = g_top_dev;
  a.dlogits = dlogits_dev;
  a.dstride = dlogits_stride;
  const int64_t grid = std::min<int64_t>(n_rows, WR_OP_BLOCKS);
  WR_DISPATCH(dtype, T, WR_LAUNCH((wr_logp_grad_kernel<T>), grid, 256, 0, stream, a));
  return WAVERNN_OK;
}

}  // extern "C"
