// Rows of a table by number, scaled, and the table's gradient.
//   out_i = s E[id_i],   dE[v] = s sum over the i with id_i = v of dout_i
// A negative number is padding: a row of zeros, no part of any gradient.  A
// number past the table is a mistake that shows: a row of NaN (and no gradient).
#include "wr_ops.h"

namespace {

struct EmbedArgs {
  const void* table;
  int64_t v, table_stride;
  int dim;
  const void* ids;
  int id_bytes;
  int64_t n;
  float scale;
  void* out;
  int64_t out_stride;
};

template <class T, class U>
__global__ __launch_bounds__(256) void wr_embed_kernel(EmbedArgs a) {
  for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x) {
    const int64_t id = wr_id(a.ids, a.id_bytes, i);
    U* o = (U*)a.out + i * a.out_stride;
    const T* r = (const T*)a.table + (id >= 0 && id < a.v ? id : 0) * a.table_stride;
    for (int c = threadIdx.x; c < a.dim; c += 256)
      o[c] = id < 0 ? (U)0.0f : id >= a.v ? (U)__builtin_nanf("") : (U)((float)r[c] * a.scale);
  }
}

struct EmbedGradArgs {
  const void* dout;
  int64_t n, dout_stride;
  int dim;
  const void* ids;
  int id_bytes;
  int64_t v;
  float scale;
  void* dtable;
};

// One block a row of the table: it looks for the row's number among all ids.
template <class T, class U>
__global__ __launch_bounds__(256) void wr_embed_grad_kernel(EmbedGradArgs a) {
  __shared__ int64_t found[256];
  __shared__ int count;
  const int tid = threadIdx.x;
  for (int64_t v = blockIdx.x; v < a.v; v += gridDim.x)
    for (int c0 = 0; c0 < a.dim; c0 += 256) {
      float acc = 0.0f;
      for (int64_t i0 = 0; i0 < a.n; i0 += 256) {
        const bool hit = i0 + tid < a.n && wr_id(a.ids, a.id_bytes, i0 + tid) == v;
        __syncthreads();
        found[tid] = hit;
        __syncthreads();
        if (tid == 0) {
          int k = 0;
          for (int j = 0; j < 256; ++j)
            if (found[j]) found[k++] = i0 + j;
          count = k;
        }
        __syncthreads();
        if (c0 + tid < a.dim)
          for (int k = 0; k < count; ++k) acc += (float)((const T*)a.dout)[found[k] * a.dout_stride + c0 + tid];
      }
      if (c0 + tid < a.dim) ((U*)a.dtable)[v * a.dim + c0 + tid] = (U)(acc * a.scale);
    }
}

wavernn_status check_ids(const void* ids, int bytes, int64_t n) {
  if (n < 0 || n > INT32_MAX) return wr_fail(WAVERNN_E_INVALID, "n_ids %lld out of range", (long long)n);
  if (bytes != 4 && bytes != 8) return wr_fail(WAVERNN_E_INVALID, "id_bytes %d: must be 4 or 8", bytes);
  if (n > 0 && !ids) return wr_fail(WAVERNN_E_INVALID, "ids is null");
  if (!wr_aligned(ids, bytes)) return wr_fail(WAVERNN_E_INVALID, "ids are not aligned to their elements");
  return WAVERNN_OK;
}
wavernn_status check_embed(int in_dtype, int out_dtype, int64_t n_table, int32_t dim) {
  if (!wr_dtype_ok(in_dtype) || !wr_dtype_ok(out_dtype)) return wr_fail(WAVERNN_E_INVALID, "bad dtype");
  if (out_dtype != in_dtype && out_dtype != WAVERNN_F32)
    return wr_fail(WAVERNN_E_INVALID, "the result's dtype must be the input's or F32");
  if (n_table < 1 || n_table > INT32_MAX) return wr_fail(WAVERNN_E_INVALID, "n_table %lld out of range", (long long)n_table);
  if (dim < 1) return wr_fail(WAVERNN_E_INVALID, "dim %d: must be positive", dim);
  return WAVERNN_OK;
}

}  // namespace

extern "C" {

wavernn_status wavernn_embed(int32_t table_dtype, const void* table_dev, int64_t n_table, int32_t dim,
                             int64_t table_stride, const void* ids_dev, int32_t id_bytes, int64_t n_ids, float scale,
                             int32_t out_dtype, void* out_dev, int64_t out_stride, void* stream) {
  wavernn_status s;
  if ((s = check_embed(table_dtype, out_dtype, n_table, dim)) != WAVERNN_OK) return s;
  if ((s = check_ids(ids_dev, id_bytes, n_ids)) != WAVERNN_OK) return s;
  if ((s = wr_check_rows("table", table_dev, table_dtype, n_table, dim, table_stride, false)) != WAVERNN_OK) return s;
  if ((s = wr_check_rows("out", out_dev, out_dtype, n_ids, dim, out_stride, true)) != WAVERNN_OK) return s;
  if (n_ids == 0) return WAVERNN_OK;
  EmbedArgs a{table_dev, n_table, table_stride, dim, ids_dev, id_bytes, n_ids, scale, out_dev, out_stride};
  const int64_t grid = std::min<int64_t>(n_ids, WR_OP_BLOCKS);
  WR_DISPATCH(table_dtype, T, if (out_dtype == WAVERNN_F32) WR_LAUNCH((wr_embed_kernel<T, float>), grid, 256, 0, stream, a);
              else WR_LAUNCH((wr_embed_kernel<T, T>), grid, 256, 0, stream, a));
  return WAVERNN_OK;
}

int64_t wavernn_embed_grad_workspace(int64_t n_ids, int32_t dim, int64_t n_table) {
  if (n_ids < 0 || n_ids > INT32_MAX || dim < 1 || n_table < 1 || n_table > INT32_MAX) return -1;
  return 0;
}

wavernn_status wavernn_embed_grad(int32_t dout_dtype, const void* dout_dev, int64_t n_ids, int32_t dim,
                                  int64_t dout_stride, const void* ids_dev, int32_t id_bytes, int64_t n_table,
                                  float scale, int32_t out_dtype, void* dtable_dev, void* workspace_dev,
                                  int64_t workspace_bytes, void* stream) {
  wavernn_status s;
  if ((s = check_embed(dout_dtype, out_dtype, n_table, dim)) != WAVERNN_OK) return s;
  if ((s = check_ids(ids_dev, id_bytes, n_ids)) != WAVERNN_OK) return s;
  if ((s = wr_check_rows("dout", dout_dev, dout_dtype, n_ids, dim, dout_stride, false)) != WAVERNN_OK) return s;
  if ((s = wr_check_rows("dtable", dtable_dev, out_dtype, n_table, dim, dim, true)) != WAVERNN_OK) return s;
  const int64_t need = wavernn_embed_grad_workspace(n_ids, dim, n_table);
  if (need > 0 && (!workspace_dev || workspace_bytes < need || !wr_aligned(workspace_dev, 16)))
    return wr_fail(WAVERNN_E_INVALID, "workspace: %lld bytes needed, 16-byte aligned", (long long)need);
  EmbedGradArgs a{dout_dev, n_ids, dout_stride, dim, ids_dev, id_bytes, n_table, scale, dtable_dev};
  const int64_t grid = std::min<int64_t>(n_table, WR_OP_BLOCKS);
  WR_DISPATCH(dout_dtype, T, if (out_dtype == WAVERNN_F32) WR_LAUNCH((wr_embed_grad_kernel<T, float>), grid, 256, 0, stream, a);
              else WR_LAUNCH((wr_embed_grad_kernel<T, T>), grid, 256, 0, stream, a));
  return WAVERNN_OK;
}

}  // extern "C"
