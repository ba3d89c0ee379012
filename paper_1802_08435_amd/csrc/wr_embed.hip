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
  int row_threads;
};

// Each group of row_threads threads copies EMBED_ROWS rows at a time, their loads in flight together.  Bound by
// memory: 16,384 rows of 4,096 bf16 from 65,536 39.7 us, 5.4 TB/s (one row a block, its loads one by one: 96).
#define EMBED_ROWS 4

template <class T, class U>
__global__ __launch_bounds__(256) void wr_embed_kernel(EmbedArgs a) {
  constexpr int VW = vec_of<T, U>(), R = EMBED_ROWS;
  const int rt = a.row_threads, t = threadIdx.x % rt;
  const int64_t step = (int64_t)gridDim.x * (256 / rt) * R;
  for (int64_t i0 = ((int64_t)blockIdx.x * (256 / rt) + threadIdx.x / rt) * R; i0 < a.n; i0 += step) {
    int64_t id[R];
#pragma unroll
    for (int k = 0; k < R; ++k) id[k] = i0 + k < a.n ? wr_id(a.ids, a.id_bytes, i0 + k) : -1;
    for (int c0 = t * VW; c0 < a.dim; c0 += rt * VW) {
      const int c = a.dim < VW ? 0 : vec_begin<VW>(c0, a.dim), count = a.dim - c;
      Raw<T, VW> x[R];
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const bool in = id[k] >= 0 && id[k] < a.v;
        x[k] = load_raw<T, VW>((const T*)a.table + (in ? id[k] : 0) * a.table_stride + c, in ? count : 0);
      }
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if (i0 + k >= a.n) break;
        const float scale = id[k] < 0 ? 0.0f : id[k] < a.v ? a.scale : __builtin_nanf("");
        float f[VW];
#pragma unroll
        for (int i = 0; i < VW; ++i) f[i] = (float)x[k][i] * scale;
        store_part<U, VW>((U*)a.out + (i0 + k) * a.out_stride + c, f, count);
      }
    }
  }
}

// ---- the table's gradient ----------------------------------------------------
// The positions are sorted by number (stably, so by position within a number)
// and each run of one number is summed: nothing is added atomically, so the
// result is the same every time.  Padding and numbers outside the table sort
// as number n_table, behind all others.
//
// Sort: least significant digit first, digits of up to 9 bits (so 2 passes to
// 262,143 rows, 1 to 511).  A wave ranks 64 numbers at a time: the lanes that
// hold the same digit find each other by ballots, and the wave's count of that
// digit, in LDS, is the base of their ranks.  Up to 4,096 ids one block does all
// passes in LDS; more take tiles of SORT_TILE ids, at most 256 tiles, and two launches a
// pass (digit counts of every tile, then the scatter), or one where each tile's block can count
// all ids itself (up to SORT_SELF tiles).
//
// The sort leaves the memory idle, so further blocks of its launches clear the table
// meanwhile, all of it: which rows stay without a number is not known yet.
//
// Sum: chunks of sorted positions, one group of threads a chunk, each thread one
// vector of columns, EG_AHEAD rows in flight.  A run inside a chunk is written to
// the table; the parts of a run that crosses chunks go to the workspace
// (slot 0: the chunk's beginning, slot 1: its end), and one more launch adds them
// in chunk order.
//
// 16,384 bf16 rows of 1,024 into 50,021 fp32 (205 MB to write, 33 to read), uneven ids: 71 us a call among
// others, of it the two passes with the clear 34 to 38, the sums 17, the frequent numbers' parts 8.
#define SORT_THREADS 1024
#define SORT_WAVES 16
#define SORT_BITS 9
#define SORT_BINS 512
#define SORT_SMALL 4096
#define SORT_TILE 2048
#define SORT_TILES 256
// Whole calls replayed in a graph, bf16 rows of 1,024 into 50,021 fp32: 16,384 even ids (8 tiles) 80.9 us with
// counts, 78.0 so, uneven ones 75.2 and 73.7; 24,576 (12 tiles) 93.6 and 92.7, uneven 85.3 and 87.9; 32,768 (16) 95.8 and
// 102.8.  Rows of 8, where the sort is most of the call: 24,576 41.0 and 43.9, 32,768 40.2 and 48.4.
#define SORT_SELF 8
#define EG_AHEAD 8
#define EG_CHUNK_MIN 8      // positions of a chunk: doubled up to 64 while that leaves 1,024 blocks of a thread for four columns
                            // (four a CU; half as many where a thread takes eight, with 16-bit types), and 64 KiB of LDS are enough
#define EG_CHUNK_MAX 64
#define EG_CLEAR 16384      // bytes that a block clears at a time
#define EG_CLEAR_BLOCKS 512

struct EmbedGradArgs {
  const void* dout;
  int64_t dout_stride;
  int n, dim;
  const void* ids;
  int id_bytes;
  int v;
  float scale;
  void* dtable;
  bool few;                     // few rows: no sort; tiles segments of `tile` ids
  int passes, bits;             // of the sort
  int tiles, tile;              // of the sort's launches; ids of a tile (a multiple of SORT_TILE)
  uint32_t *key[2], *pos[2];    // [n] each; [1] absent with n <= SORT_SMALL
  uint32_t* hist;               // [tiles][SORT_BINS]
  int src, shift;               // of one pass: buffer read (-1: the ids), digit's lowest bit
  const uint32_t *skey, *spos;  // sorted
  float* part;                  // [chunks][2][dim]; few rows: [tiles][v][dim]
  int chunk, chunks;            // positions of a chunk
  int row_threads;              // threads on a row (256 / row_threads chunks a block)
  int sort_blocks;              // of a sort's launch; the ones behind them clear bytes clear0 .. clear1 of dtable
  int64_t clear0, clear1;
};

__device__ __forceinline__ uint32_t sort_key(const EmbedGradArgs& a, int i) {
  const int64_t id = wr_id(a.ids, a.id_bytes, i);
  return id >= 0 && id < a.v ? (uint32_t)id : (uint32_t)a.v;
}

// Rank of this lane's digit among the lanes before it that hold the same one, and their base in the wave's
// counts `cnt`, which grow by this round's.  Lanes without a number pass valid = false.
__device__ __forceinline__ int wave_rank(uint16_t* cnt, int digit, int bits, bool valid) {
  const uint64_t on = __ballot(valid);
  uint32_t lo = (uint32_t)on, hi = (uint32_t)(on >> 32);
  for (int b = 0; b < bits; ++b) {
    const uint32_t mine = 0u - ((uint32_t)digit >> b & 1u);   // all ones where this lane's bit is set
    const uint64_t m = __ballot(mine != 0);
    lo &= ~((uint32_t)m ^ mine);
    hi &= ~((uint32_t)(m >> 32) ^ mine);
  }
  const uint64_t same = (uint64_t)hi << 32 | lo;
  const int lane = threadIdx.x & 63, below = __popcll(same & ((1ull << lane) - 1));
  int base = 0;
  if (valid) base = cnt[digit];
  __builtin_amdgcn_wave_barrier();
  if (valid && below == 0) cnt[digit] = (uint16_t)(base + __popcll(same));
  __builtin_amdgcn_wave_barrier();
  return base + below;
}
// After every wave counted its digits: cnt[w][d] becomes the count of d in the waves before w,
// total[d] the block's.
__device__ __forceinline__ void wave_bases(uint16_t (*cnt)[SORT_BINS], uint32_t* total) {
  const int d = threadIdx.x;
  if (d < SORT_BINS) {
    int run = 0;
#pragma unroll
    for (int w = 0; w < SORT_WAVES; ++w) {
      const int c = cnt[w][d];
      cnt[w][d] = (uint16_t)run;
      run += c;
    }
    total[d] = run;
  }
}
// x[d] becomes the sum of the x[e] with e < d.  Every thread calls it; `tmp`: 16 words.
__device__ __forceinline__ void scan_bins(uint32_t* x, uint32_t* tmp) {
  const int d = threadIdx.x, lane = d & 63;
  uint32_t v = 0, s = 0;
  if (d < SORT_BINS) {
    v = s = x[d];
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const uint32_t t = __shfl_up(s, o, 64);
      if (lane >= o) s += t;
    }
    if (lane == 63) tmp[d >> 6] = s;
  }
  __syncthreads();
  if (d < SORT_BINS) {
    for (int w = 0; w < (d >> 6); ++w) s += tmp[w];
    x[d] = s - v;
  }
  __syncthreads();
}

// Clears this block's part of the table (any alignment; whole 16-byte pieces and the ends by element).
__device__ void clear_part(const EmbedGradArgs& a) {
  const int64_t step = (int64_t)(gridDim.x - a.sort_blocks) * EG_CLEAR;
  for (int64_t b0 = a.clear0 + (int64_t)(blockIdx.x - a.sort_blocks) * EG_CLEAR; b0 < a.clear1; b0 += step) {
    unsigned char* p = (unsigned char*)a.dtable + b0;
    const int n = (int)std::min<int64_t>(EG_CLEAR, a.clear1 - b0);
    for (int i = threadIdx.x * 16; i < n; i += SORT_THREADS * 16) {
      if (i + 16 <= n) {
        const uint4 z = {0, 0, 0, 0};
        __builtin_memcpy(p + i, &z, 16);
      } else {
        for (int j = i; j < n; j += 2) *(uint16_t*)(p + j) = 0;
      }
    }
  }
}

// All passes by one block, n <= E SORT_THREADS.
template <int E>
__global__ __launch_bounds__(SORT_THREADS) void wr_sort_small_kernel(EmbedGradArgs a) {
  __shared__ uint16_t cnt[SORT_WAVES][SORT_BINS];
  __shared__ uint32_t keys[E * SORT_THREADS];
  __shared__ uint16_t poss[E * SORT_THREADS];
  __shared__ uint32_t base[SORT_BINS], tmp[16];
  if ((int)blockIdx.x >= a.sort_blocks) return clear_part(a);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  uint32_t k[E];
  int p[E], r[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    p[e] = wave * 64 * E + e * 64 + lane;
    k[e] = p[e] < a.n ? sort_key(a, p[e]) : 0;
  }
  for (int pass = 0; pass < a.passes; ++pass) {
    const int shift = pass * a.bits;
    for (int i = tid; i < SORT_WAVES * SORT_BINS / 2; i += SORT_THREADS) ((uint32_t*)cnt)[i] = 0;
    __syncthreads();
    const uint32_t mask = (1u << a.bits) - 1;
#pragma unroll
    for (int e = 0; e < E; ++e)
      r[e] = wave_rank(cnt[wave], (k[e] >> shift) & mask, a.bits, wave * 64 * E + e * 64 + lane < a.n);
    __syncthreads();
    wave_bases(cnt, base);
    __syncthreads();
    scan_bins(base, tmp);
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (wave * 64 * E + e * 64 + lane < a.n) {
        const int d = (k[e] >> shift) & mask, to = base[d] + cnt[wave][d] + r[e];
        keys[to] = k[e];
        poss[to] = (uint16_t)p[e];
      }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = wave * 64 * E + e * 64 + lane;
      if (i < a.n) k[e] = keys[i], p[e] = poss[i];
    }
    __syncthreads();
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = wave * 64 * E + e * 64 + lane;
    if (i < a.n) a.key[0][i] = k[e], a.pos[0][i] = (uint32_t)p[e];
  }
}

// Counts of the pass's digits in each tile.
__global__ __launch_bounds__(SORT_THREADS) void wr_sort_count_kernel(EmbedGradArgs a) {
  __shared__ uint32_t h[SORT_BINS];
  if ((int)blockIdx.x >= a.sort_blocks) return clear_part(a);
  const uint32_t mask = (1u << a.bits) - 1;
  if (threadIdx.x < SORT_BINS) h[threadIdx.x] = 0;
  __syncthreads();
  const int64_t i0 = (int64_t)blockIdx.x * a.tile;
  const int64_t i1 = std::min<int64_t>(a.n, i0 + a.tile);
  for (int64_t i = i0 + threadIdx.x; i < i1; i += SORT_THREADS)
    atomicAdd(&h[((a.src < 0 ? sort_key(a, (int)i) : a.key[a.src][i]) >> a.shift) & mask], 1u);
  __syncthreads();
  if (threadIdx.x < SORT_BINS) a.hist[(int64_t)blockIdx.x * SORT_BINS + threadIdx.x] = h[threadIdx.x];
}

// One tile's numbers to their places by the pass's digit.
__global__ __launch_bounds__(SORT_THREADS) void wr_sort_scatter_kernel(EmbedGradArgs a) {
  constexpr int E = SORT_TILE / SORT_THREADS;
  __shared__ uint16_t cnt[SORT_WAVES][SORT_BINS];
  __shared__ uint32_t base[SORT_BINS], before[2][SORT_BINS], total[2][SORT_BINS], tmp[16];
  if ((int)blockIdx.x >= a.sort_blocks) return clear_part(a);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const uint32_t mask = (1u << a.bits) - 1;
  uint32_t k[E], p[E];
  auto read = [&](int64_t i0) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int64_t i = i0 + wave * 64 * E + e * 64 + lane;
      const bool in = i < a.n;
      k[e] = in ? (a.src < 0 ? sort_key(a, (int)i) : a.key[a.src][i]) : 0;
      p[e] = in ? (a.src < 0 ? (uint32_t)i : a.pos[a.src][i]) : 0;
    }
  };
  read((int64_t)blockIdx.x * a.tile);
  // this tile's first place of each digit: all smaller digits, and this one in the tiles before
  if (a.tiles <= SORT_SELF) {
    for (int i = tid; i < 4 * SORT_BINS; i += SORT_THREADS) (i < 2 * SORT_BINS ? before[0] : total[0])[i % (2 * SORT_BINS)] = 0;
    __syncthreads();
    const int first = (int)blockIdx.x * a.tile;
    for (int i0 = tid; i0 < a.n; i0 += SORT_THREADS * 4) {
      uint32_t x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * SORT_THREADS;
        x[u] = i < a.n ? (a.src < 0 ? sort_key(a, i) : a.key[a.src][i]) : 0;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * SORT_THREADS;
        if (i < a.n) atomicAdd(i < first ? &before[0][(x[u] >> a.shift) & mask] : &total[0][(x[u] >> a.shift) & mask], 1u);
      }
    }
    __syncthreads();
    if (tid < SORT_BINS) total[0][tid] += before[0][tid];
  } else {
    const int d = tid & (SORT_BINS - 1), half = tid / SORT_BINS;
    uint32_t b = 0, t = 0;
#pragma unroll 8
    for (int i = half; i < a.tiles; i += 2) {
      const uint32_t c = a.hist[(int64_t)i * SORT_BINS + d];
      t += c;
      if (i < (int)blockIdx.x) b += c;
    }
    before[half][d] = b;
    total[half][d] = t;
  }
  __syncthreads();
  if (tid < SORT_BINS) base[tid] = total[0][tid] + total[1][tid];
  __syncthreads();
  scan_bins(base, tmp);
  if (tid < SORT_BINS) base[tid] += before[0][tid] + before[1][tid];
  const int dst = a.src < 0 ? 0 : 1 - a.src;
  for (int t0 = 0; t0 < a.tile; t0 += SORT_TILE) {
    const int64_t i0 = (int64_t)blockIdx.x * a.tile + t0;
    if (i0 >= a.n) break;
    for (int i = tid; i < SORT_WAVES * SORT_BINS / 2; i += SORT_THREADS) ((uint32_t*)cnt)[i] = 0;
    __syncthreads();
    if (t0 > 0) read(i0);
    int r[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
      r[e] = wave_rank(cnt[wave], (k[e] >> a.shift) & mask, a.bits, i0 + wave * 64 * E + e * 64 + lane < a.n);
    __syncthreads();
    wave_bases(cnt, total[0]);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (i0 + wave * 64 * E + e * 64 + lane < a.n) {
        const int d = (k[e] >> a.shift) & mask;
        const uint32_t to = base[d] + cnt[wave][d] + r[e];
        a.key[dst][to] = k[e];
        a.pos[dst][to] = p[e];
      }
    __syncthreads();
    if (tid < SORT_BINS) base[tid] += total[0][tid];
    __syncthreads();
  }
}

// LDS: the numbers and positions of the block's chunks.
template <class T, class U>
__global__ __launch_bounds__(256) void wr_embed_sum_kernel(EmbedGradArgs a) {
  extern __shared__ uint32_t at[];
  constexpr int VW = vec_of<T, U>();
  const int rt = a.row_threads, t = threadIdx.x % rt, per = 256 / rt * a.chunk;
  U* table = (U*)a.dtable;
  for (int64_t b0 = (int64_t)blockIdx.x * per; b0 < a.n; b0 += (int64_t)gridDim.x * per) {
    __syncthreads();
    for (int i = threadIdx.x; i < per && b0 + i < a.n; i += 256) at[i] = a.skey[b0 + i], at[per + i] = a.spos[b0 + i];
    __syncthreads();
    const int l0 = threadIdx.x / rt * a.chunk;            // this group's chunk, in LDS
    const int64_t p0 = b0 + l0;
    if (p0 >= a.n) continue;
    const int m = (int)std::min<int64_t>(a.chunk, a.n - p0);
    const int64_t c = p0 / a.chunk;
    const uint32_t *key = at + l0, *pos = at + per + l0;
    const uint32_t first = key[0], last = key[m - 1], v = (uint32_t)a.v;
    const bool from = p0 > 0 && a.skey[p0 - 1] == first, on = p0 + m < a.n && a.skey[p0 + m] == last;
    for (int c0 = t * VW; c0 < a.dim; c0 += rt * VW) {
      const int col = a.dim < VW ? 0 : vec_begin<VW>(c0, a.dim), count = a.dim - col;
      float acc[VW];
      uint32_t cur = first;
      auto flush = [&](uint32_t id, bool at_end) {
        if (id >= v) return;
        if (id == first && from) store_part<float, VW>(a.part + (2 * c) * a.dim + col, acc, count);
        else if (at_end && on) store_part<float, VW>(a.part + (2 * c + 1) * a.dim + col, acc, count);
        else {
#pragma unroll
          for (int i = 0; i < VW; ++i) acc[i] *= a.scale;
          store_part<U, VW>(table + (int64_t)id * a.dim + col, acc, count);
        }
      };
#pragma unroll
      for (int i = 0; i < VW; ++i) acc[i] = 0.0f;
      for (int p = 0; p < m; p += EG_AHEAD) {
        Raw<T, VW> x[EG_AHEAD];
#pragma unroll
        for (int u = 0; u < EG_AHEAD; ++u) {
          const bool in = p + u < m && key[p + u] < v;
          x[u] = load_raw<T, VW>((const T*)a.dout + (in ? (int64_t)pos[p + u] : 0) * a.dout_stride + col, in ? count : 0);
        }
#pragma unroll
        for (int u = 0; u < EG_AHEAD; ++u) {
          if (p + u >= m) break;
          const uint32_t id = key[p + u];
          if (id != cur) {
            flush(cur, false);
            cur = id;
#pragma unroll
            for (int i = 0; i < VW; ++i) acc[i] = 0.0f;
          }
          if (id < v)
#pragma unroll
            for (int i = 0; i < VW; ++i) acc[i] += (float)x[u][i];
        }
      }
      flush(cur, true);
    }
  }
}

// Runs that cross chunks: block (c, s) adds, for up to 256 columns, the parts of the run that begins in chunk c and
// goes on, in chunk order (each group of threads every groups-th part, then the groups in order).
template <class U>
__global__ __launch_bounds__(256) void wr_embed_join_kernel(EmbedGradArgs a) {
  __shared__ float sums[256][4];
  const int rt = a.row_threads, groups = 256 / rt, g = threadIdx.x / rt, t = threadIdx.x % rt;
  for (int64_t c = blockIdx.x; c + 1 < a.chunks; c += gridDim.x) {
    const int64_t p0 = c * a.chunk, p1 = p0 + a.chunk;
    const uint32_t id = a.skey[p1 - 1], next = a.skey[p1], head = a.skey[p0], prev = p0 > 0 ? a.skey[p0 - 1] : ~0u;
    if (id >= (uint32_t)a.v || next != id || (head == id && prev == id)) continue;
    int64_t more = 0;   // chunks after c that begin with the number
    for (;;) {
      const int64_t p = (c + 1 + more + threadIdx.x) * a.chunk;
      const int k = __syncthreads_count(p < a.n && a.skey[p] == id);
      more += k;
      if (k < 256) break;
    }
    const int64_t col = ((int64_t)blockIdx.y * rt + t) * 4;
    const int count = (int)std::min<int64_t>(4, a.dim - col);
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t j0 = g; j0 <= more; j0 += EG_AHEAD * groups) {
      Raw<float, 4> x[EG_AHEAD];
#pragma unroll
      for (int u = 0; u < EG_AHEAD; ++u) {
        const int64_t j = j0 + u * groups;
        x[u] = load_raw<float, 4>(a.part + (2 * (c + (j <= more ? j : 0)) + (j == 0)) * a.dim + col, j <= more ? count : 0);
      }
#pragma unroll
      for (int u = 0; u < EG_AHEAD; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] += x[u][i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[threadIdx.x][i] = acc[i];
    __syncthreads();
    if (g == 0 && count > 0) {
      for (int k = 1; k < groups; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] += sums[k * rt + t][i];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] *= a.scale;
      store_part<U, 4>((U*)a.dtable + (int64_t)id * a.dim + col, acc, count);
    }
  }
}

// ---- few rows ----------------------------------------------------------------
// A table of up to EF_ROWS rows (bytes, labels), with up to EF_WORK ids compared: block (v, s) looks
// for number v among the ids of segment s itself, which takes no sort, and sums the rows it finds; with
// several segments one more launch adds their sums in order.  12,800 rows of 64 into 97: 20 us by the
// sort (four launches), 12 so; 100,000 rows of 16 into 256, past EF_WORK: 74 so, 33 by the sort.
#define EF_ROWS 256
#define EF_WORK (4 << 20)  // ids times rows
#define EF_SEG 2048        // ids of a segment: 8 a thread; more (up to 8,192) past 64 segments
#define EF_SEG_MAX 8192
#define EF_SEGS 64

template <class T, class U>
__global__ __launch_bounds__(256) void wr_embed_few_kernel(EmbedGradArgs a) {
  constexpr int VW = vec_of<T, U>();
  __shared__ uint16_t found[EF_SEG_MAX];   // each wave's hits, in order, in its quarter of the segment
  __shared__ int hits[4];
  __shared__ float sums[256][VW + 1];      // (padded against bank conflicts)
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, v = blockIdx.x;
  const int64_t i0 = (int64_t)blockIdx.y * a.tile;
  const int quarter = a.tile / 4;
  int n = 0;
  for (int j = 0; j < quarter; j += 64) {
    const int64_t i = i0 + wave * quarter + j + lane;
    const bool hit = i < a.n && wr_id(a.ids, a.id_bytes, i) == v;
    const uint64_t m = __ballot(hit);
    if (hit) found[wave * quarter + n + __popcll(m & ((1ull << lane) - 1))] = (uint16_t)(wave * quarter + j + lane);
    n += __popcll(m);
  }
  if (lane == 0) hits[wave] = n;
  __syncthreads();
  const int h0 = hits[0], h1 = h0 + hits[1], h2 = h1 + hits[2], total = h2 + hits[3];
  const int rt = a.row_threads, groups = 256 / rt, g = tid / rt, t = tid % rt;
  for (int b0 = 0; b0 < a.dim; b0 += rt * VW) {
    const int c0 = b0 + t * VW, col = a.dim < VW ? 0 : vec_begin<VW>(c0, a.dim), count = c0 < a.dim ? a.dim - col : 0;
    float acc[VW];
#pragma unroll
    for (int k = 0; k < VW; ++k) acc[k] = 0.0f;
    for (int j0 = g; j0 < total; j0 += EG_AHEAD * groups) {
      Raw<T, VW> x[EG_AHEAD];
#pragma unroll
      for (int u = 0; u < EG_AHEAD; ++u) {
        const int j = j0 + u * groups;
        const int q = j < h0 ? j : j < h1 ? quarter + j - h0 : j < h2 ? 2 * quarter + j - h1 : 3 * quarter + j - h2;
        x[u] = load_raw<T, VW>((const T*)a.dout + (j < total ? i0 + found[q] : 0) * a.dout_stride + col, j < total ? count : 0);
      }
#pragma unroll
      for (int u = 0; u < EG_AHEAD; ++u)
#pragma unroll
        for (int k = 0; k < VW; ++k) acc[k] += (float)x[u][k];
    }
    if (groups > 1) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < VW; ++k) sums[tid][k] = acc[k];
      __syncthreads();
      if (g == 0)
        for (int q = 1; q < groups; ++q)
#pragma unroll
          for (int k = 0; k < VW; ++k) acc[k] += sums[q * rt + t][k];
    }
    if (g == 0 && count > 0) {
      if (a.tiles > 1) {
        store_part<float, VW>(a.part + ((int64_t)blockIdx.y * a.v + v) * a.dim + col, acc, count);
      } else {
#pragma unroll
        for (int k = 0; k < VW; ++k) acc[k] *= a.scale;
        store_part<U, VW>((U*)a.dtable + (int64_t)v * a.dim + col, acc, count);
      }
    }
  }
}

template <class U>
__global__ __launch_bounds__(256) void wr_embed_few_join_kernel(EmbedGradArgs a) {
  const int64_t cells = (int64_t)a.v * a.dim;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < cells; i += (int64_t)gridDim.x * 1024) {
    const int count = (int)std::min<int64_t>(4, cells - i);
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = 0; s0 < a.tiles; s0 += EG_AHEAD) {
      Raw<float, 4> x[EG_AHEAD];
#pragma unroll
      for (int u = 0; u < EG_AHEAD; ++u)
        x[u] = load_raw<float, 4>(a.part + (s0 + u < a.tiles ? s0 + u : 0) * cells + i, s0 + u < a.tiles ? count : 0);
#pragma unroll
      for (int u = 0; u < EG_AHEAD; ++u)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] += x[u][k];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] *= a.scale;
    store_part<U, 4>((U*)a.dtable + i, acc, count);
  }
}

// Sizes of a call and its workspace's layout; returns the workspace's bytes.
int64_t plan_embed_grad(int64_t n, int32_t dim, int64_t v, EmbedGradArgs* a, unsigned char* ws) {
  a->few = v <= EF_ROWS && n * v <= EF_WORK && n <= (int64_t)EF_SEGS * EF_SEG_MAX;
  if (a->few) {
    a->tile = EF_SEG;
    while (n > (int64_t)EF_SEGS * a->tile) a->tile *= 2;
    a->tiles = (int)std::max<int64_t>(1, (n + a->tile - 1) / a->tile);
    a->part = (float*)ws;
    return a->tiles > 1 ? (int64_t)4 * a->tiles * v * dim : 0;
  }
  int bits = 1;
  while (bits < 32 && (v >> bits)) ++bits;   // keys 0 .. v
  a->passes = (bits + SORT_BITS - 1) / SORT_BITS;
  a->bits = (bits + a->passes - 1) / a->passes;
  a->tile = SORT_TILE;
  while ((n + a->tile - 1) / a->tile > SORT_TILES) a->tile += SORT_TILE;
  a->tiles = (int)((n + a->tile - 1) / a->tile);
  // (by vectors of 4 elements, whatever the types, so that the workspace is known from the sizes)
  const int64_t rt = wr_row_threads(((int64_t)dim + 3) / 4);
  a->chunk = EG_CHUNK_MIN;
  while (a->chunk < EG_CHUNK_MAX && n * rt / 256 / (2 * a->chunk) >= 1024 && 2 * a->chunk * 512 <= 8192 * rt) a->chunk *= 2;
  a->chunks = (int)((n + a->chunk - 1) / a->chunk);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    unsigned char* p = ws + at;
    at += (bytes + 15) / 16 * 16;
    return p;
  };
  const bool small = n <= SORT_SMALL;
  for (int i = 0; i < (small ? 1 : 2); ++i) {
    a->key[i] = (uint32_t*)take(4 * n);
    a->pos[i] = (uint32_t*)take(4 * n);
  }
  if (!small) a->hist = (uint32_t*)take((int64_t)4 * a->tiles * SORT_BINS);
  if (a->chunks > 1) a->part = (float*)take((int64_t)8 * a->chunks * dim);
  return at;
}

template <class T, class U>
wavernn_status run_embed_grad(EmbedGradArgs& a, void* stream) {
  if (a.few) {
    constexpr int VW = vec_of<T, U>();
    // (16 threads a row at least: a block finds few rows, and its groups are added one by one)
    a.row_threads = std::max(16, wr_row_threads(((int64_t)a.dim + VW - 1) / VW));
    void* argv[] = {&a};
    const hipError_t e = hipLaunchKernel((const void*)wr_embed_few_kernel<T, U>, dim3(a.v, a.tiles), dim3(256), argv, 0,
                                         (hipStream_t)stream);
    if (e != hipSuccess) return wr_fail(WAVERNN_E_HIP, "launch of wr_embed_few_kernel: %s", hipGetErrorString(e));
    if (a.tiles > 1)
      WR_LAUNCH((wr_embed_few_join_kernel<U>), std::min<int64_t>(((int64_t)a.v * a.dim + 1023) / 1024, 1 << 16), 256, 0, stream, a);
    return WAVERNN_OK;
  }
  int last = 0;
  const bool small = a.n <= SORT_SMALL;
  const bool counts = a.tiles > SORT_SELF;
  const int launches = small ? 1 : counts ? 2 * a.passes : a.passes;
  const int64_t bytes = (int64_t)a.v * a.dim * sizeof(U);
  auto clear = [&](int i) {   // launch i's share of the table, in 16-byte pieces; its blocks
    a.clear0 = bytes / 16 * i / launches * 16;
    a.clear1 = i + 1 == launches ? bytes : bytes / 16 * (i + 1) / launches * 16;
    // two blocks of 1,024 threads fit a CU: as many as run at once
    return a.sort_blocks + std::min<int64_t>((a.clear1 - a.clear0 + EG_CLEAR - 1) / EG_CLEAR,
                                             std::max(EG_CLEAR_BLOCKS - a.sort_blocks, 256));
  };
  if (small) {
    a.sort_blocks = 1;
    if (a.n <= SORT_THREADS) WR_LAUNCH((wr_sort_small_kernel<1>), clear(0), SORT_THREADS, 0, stream, a);
    else WR_LAUNCH((wr_sort_small_kernel<SORT_SMALL / SORT_THREADS>), clear(0), SORT_THREADS, 0, stream, a);
  } else {
    a.sort_blocks = a.tiles;
    for (int pass = 0; pass < a.passes; ++pass) {
      a.src = pass == 0 ? -1 : (pass - 1) & 1;
      a.shift = pass * a.bits;
      if (counts) WR_LAUNCH(wr_sort_count_kernel, clear(2 * pass), SORT_THREADS, 0, stream, a);
      WR_LAUNCH(wr_sort_scatter_kernel, clear(counts ? 2 * pass + 1 : pass), SORT_THREADS, 0, stream, a);
    }
    last = (a.passes - 1) & 1;
  }
  if (a.n == 0) return WAVERNN_OK;
  a.skey = a.key[last];
  a.spos = a.pos[last];
  constexpr int VW = vec_of<T, U>();
  a.row_threads = wr_row_threads(((int64_t)a.dim + VW - 1) / VW);
  const int per = 256 / a.row_threads * a.chunk;
  WR_LAUNCH((wr_embed_sum_kernel<T, U>), std::min<int64_t>(((int64_t)a.n + per - 1) / per, 1 << 20), 256, 8 * per, stream, a);
  if (a.chunks > 1) {
    a.row_threads = std::min(64, wr_row_threads(((int64_t)a.dim + 3) / 4));
    void* argv[] = {&a};
    const unsigned slices = (unsigned)(((int64_t)a.dim + 4 * a.row_threads - 1) / (4 * a.row_threads));
    const unsigned blocks = (unsigned)std::min<int64_t>(a.chunks - 1, 1 << 16);
    const hipError_t e = hipLaunchKernel((const void*)wr_embed_join_kernel<U>, dim3(blocks, slices), dim3(256), argv, 0,
                                         (hipStream_t)stream);
    if (e != hipSuccess) return wr_fail(WAVERNN_E_HIP, "launch of wr_embed_join_kernel: %s", hipGetErrorString(e));
  }
  return WAVERNN_OK;
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
  if (dim < 1 || dim > (1 << 20)) return wr_fail(WAVERNN_E_INVALID, "dim %d not in [1, 2^20]", dim);
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
  EmbedArgs a{table_dev, n_table, table_stride, dim, ids_dev, id_bytes, n_ids, scale, out_dev, out_stride, 0};
  const int vw = 16 / std::min(wr_dtype_bytes(table_dtype), wr_dtype_bytes(out_dtype));
  a.row_threads = wr_row_threads(((int64_t)dim + vw - 1) / vw);
  const int64_t rows = 256 / a.row_threads * EMBED_ROWS, grid = std::min<int64_t>((n_ids + rows - 1) / rows, WR_OP_BLOCKS);
  WR_DISPATCH(table_dtype, T, if (out_dtype == WAVERNN_F32) WR_LAUNCH((wr_embed_kernel<T, float>), grid, 256, 0, stream, a);
              else WR_LAUNCH((wr_embed_kernel<T, T>), grid, 256, 0, stream, a));
  return WAVERNN_OK;
}

int64_t wavernn_embed_grad_workspace(int64_t n_ids, int32_t dim, int64_t n_table) {
  if (n_ids < 0 || n_ids > INT32_MAX || dim < 1 || dim > (1 << 20) || n_table < 1 || n_table > INT32_MAX) return -1;
  EmbedGradArgs a = {};
  return plan_embed_grad(n_ids, dim, n_table, &a, nullptr);
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
  EmbedGradArgs a = {};
  plan_embed_grad(n_ids, dim, n_table, &a, (unsigned char*)workspace_dev);
  a.dout = dout_dev;
  a.dout_stride = dout_stride;
  a.n = (int)n_ids;
  a.dim = dim;
  a.ids = ids_dev;
  a.id_bytes = id_bytes;
  a.v = (int)n_table;
  a.scale = scale;
  a.dtable = dtable_dev;
  WR_DISPATCH(dout_dtype, T, return out_dtype == WAVERNN_F32 ? run_embed_grad<T, float>(a, stream)
                                                             : run_embed_grad<T, T>(a, stream));
}

}  // extern "C"
