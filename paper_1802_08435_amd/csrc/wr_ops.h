// Shared by the operators on callers' tensors (wr_logp.hip, wr_embed.hip,
// wr_norm.hip): element types, row access, argument checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <algorithm>

#include "wavernn.h"

// Sets wavernn_last_error and returns s (wr_host.hip).
wavernn_status wr_fail(wavernn_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

#define WR_LAUNCH(kernel, grid, block, lds, stream, args)                                                      \
  do {                                                                                                         \
    void* argv_[] = {&args};                                                                                   \
    hipError_t e_ = hipLaunchKernel((const void*)(kernel), dim3((unsigned)(grid)), dim3(block), argv_, (lds),   \
                                    (hipStream_t)(stream));                                                    \
    if (e_ != hipSuccess) return wr_fail(WAVERNN_E_HIP, "launch of " #kernel ": %s", hipGetErrorString(e_));    \
  } while (0)

// Blocks of a launch whose kernels stride over their rows: enough to fill the
// card many times over, far below the grid limit of 2^32 - 1 threads.
#define WR_OP_BLOCKS 65536

inline bool wr_dtype_ok(int t) { return t == WAVERNN_F32 || t == WAVERNN_BF16 || t == WAVERNN_F16; }
inline int wr_dtype_bytes(int t) { return t == WAVERNN_F32 ? 4 : 2; }
inline bool wr_aligned(const void* p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

// The sizes and pointer of one matrix of rows: n rows of `width` elements, `stride` elements apart.
inline wavernn_status wr_check_rows(const char* name, const void* p, int dtype, int64_t n, int64_t width, int64_t stride,
                                    bool output) {
  if (n > 0 && !p) return wr_fail(WAVERNN_E_INVALID, "%s is null", name);
  if (!wr_aligned(p, wr_dtype_bytes(dtype))) return wr_fail(WAVERNN_E_INVALID, "%s is not aligned to its elements", name);
  if (stride < 0 || stride > INT32_MAX) return wr_fail(WAVERNN_E_INVALID, "%s: row stride %lld out of range", name, (long long)stride);
  if (output && n > 1 && stride < width)
    return wr_fail(WAVERNN_E_INVALID, "%s: row stride %lld below the row's %lld elements", name, (long long)stride, (long long)width);
  return WAVERNN_OK;
}

// Runs `body` with T the element type of dtype t.
#define WR_DISPATCH(t, T, ...)                                        \
  do {                                                                \
    if ((t) == WAVERNN_F32) { using T = float; __VA_ARGS__; }         \
    else if ((t) == WAVERNN_BF16) { using T = __bf16; __VA_ARGS__; }  \
    else { using T = _Float16; __VA_ARGS__; }                         \
  } while (0)

// A whole number of a list of 4- or 8-byte ones.
__device__ __forceinline__ int64_t wr_id(const void* ids, int bytes, int64_t i) {
  return bytes == 8 ? ((const int64_t*)ids)[i] : (int64_t)((const int32_t*)ids)[i];
}

// N adjacent elements from or to any address aligned to an element: whole
// vectors as one access (the hardware takes them at any alignment; at an odd
// one an access touches two cache lines now and then), the first `count` of a
// row's last vector one by one.  load_raw leaves the elements as they are, with
// `fill` past the count, so that the loads of several vectors are under way
// before the first is waited for: a conversion right behind a load that not every lane
// makes would wait for it there.
template <class T, int N>
struct RawVec {
  typedef T type __attribute__((ext_vector_type(N)));
};
template <class T, int N>
using Raw = typename RawVec<T, N>::type;
template <class T, int N>
__device__ __forceinline__ Raw<T, N> load_raw(const T* p, int count, T fill = (T)0.0f) {
  Raw<T, N> x;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = fill;
  if (count >= N) {
    __builtin_memcpy(&x, p, sizeof x);
  } else if (count > 0) {
    T y[N];
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = p[i < count ? i : count - 1];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = i < count ? y[i] : fill;
  }
  return x;
}
// Where a thread's vector at column c of a row of d elements begins: a row's last vector, if it is not
// whole, is the last N elements, so that every load and store is of a whole vector.  Some columns are
// then another thread's too: both come to the same values, and sums leave out the first
// c - vec_begin of the vector (all of it past the row).  Only for d >= N.
template <int N>
__device__ __forceinline__ int vec_begin(int c, int d) { return c <= d - N ? c : d - N; }
template <class T, int N>
__device__ __forceinline__ void load_part(const T* p, float (&f)[N], int count) {
  const Raw<T, N> x = load_raw<T, N>(p, count);
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = (float)x[i];
}
template <class T, int N>
__device__ __forceinline__ void store_vec(T* p, const float (&f)[N]) {
  Raw<T, N> x;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = (T)f[i];
  __builtin_memcpy(p, &x, sizeof x);
}
template <class T, int N>
__device__ __forceinline__ void store_part(T* p, const float (&f)[N], int count) {
  if (count >= N) return store_vec<T, N>(p, f);
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < count) p[i] = (T)f[i];
}
// Elements of a 16-byte vector of the narrower of two types.
template <class T, class U>
constexpr int vec_of() { return 16 / (int)(sizeof(T) < sizeof(U) ? sizeof(T) : sizeof(U)); }

// Threads of a block of 256 on one row of `vecs` vectors: a power of two, so that small rows share a block.
inline int wr_row_threads(int64_t vecs) {
  int t = 1;
  while (t < 256 && t < vecs) t *= 2;
  return t;
}
