// Log probabilities of given tokens with the entropy and the top alternatives
// of their distributions, and the gradient of all of them with respect to the
// logits.  For a row z of V logits with m = max z, s = sum e^(z - m):
//   lse = m + log s,  logp = (z_t - m) - log s,
//   H = -sum p log p = log s - sum (z - m) e^(z - m) / s
// (both terms of H are >= 0, so nothing cancels), and the top K by (z
// descending, number ascending).  Sums are fp32.  A log probability is formed
// without lse, whose rounding is the logits' size: at logits near 50 steps of 3.8e-6,
// which would leave a probable token's -1e-5 one digit.
//   dz_j = [j = t] g_logp + sum_k [j = top_k] g_top_k
//        + p_j (g_lse - g_logp - sum_k g_top_k) - g_H p_j (log p_j + H)
#include <math.h>

#include "wr_kern.h"
#include "wr_logp.h"
#include "wr_ops.h"

#define LR_CAP 64          // classes of a short row that are ranked
#define LOGP_BLOCKS 2048   // eight blocks of 256 threads a CU
#define LW_SPLITS 128      // most segments of a row
#define LW_SEG 8192        // fewest classes of one (but for rounding)

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

// Order of the alternatives as whole numbers: a logit's rank (its bits with the sign turned
// round, -0 as +0, every NaN as the one above +inf) in the upper half, its number complemented in the
// lower, so that no two classes compare equal.  0 is below every logit.
__device__ __forceinline__ float plain_nan(float z) { return z != z ? __builtin_nanf("") : z; }
__device__ __forceinline__ uint32_t rank_of(float z) {   // z not NaN, or plain_nan's
  const int u = (int)__float_as_uint(z + 0.0f);
  return (uint32_t)(u ^ (u >> 31 | (int)0x80000000));
}
__device__ __forceinline__ uint32_t top_rank(float z) { return rank_of(plain_nan(z)); }
__device__ __forceinline__ u64 top_key(float z, int j) { return (u64)top_rank(z) << 32 | (uint32_t)~j; }
__device__ __forceinline__ float key_value(u64 k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return __uint_as_float((u >> 31) ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_class(u64 k) { return (int)~(uint32_t)k; }

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
  const float d = fmaxf(a.m - soft_base(m2), WR_FAR), c = fexp(d);
  return Soft{m2, a.s * c, __builtin_fmaf(d, a.s, a.w) * c};
}
__device__ __forceinline__ Soft soft_join(Soft a, Soft b) {
  const float m = fmaxf(a.m, b.m);
  a = soft_at(a, m);
  b = soft_at(b, m);
  return Soft{m, a.s + b.s, a.w + b.w};
}
// One logit, z <= its maximum (base = soft_base(m)).
__device__ __forceinline__ void soft_term(float z, float base, float& s, float& w) {
  const float d = z - base, e = fexp(d);
  s += e;
  w = __builtin_fmaf(fmaxf(d, WR_FAR), e, w);
}
// A row's log probabilities: the logit less the maximum, less log s.  Nothing more where every class is masked
// (q.s = 0), nor where the maximum is a mask's finite value, past WR_MASK in size (the type's lowest): lse is that value
// itself there, in 64 bits too, and z - lse is 0.
#define WR_MASK 1e30f
struct LogP {
  float base, logs;
  __device__ __forceinline__ float operator()(float z) const { return (z - base) - logs; }
};
__device__ __forceinline__ LogP soft_logp(Soft q) {
  const bool none = q.s == 0.0f || (fabsf(q.m) > WR_MASK && q.s == q.s);
  return LogP{soft_base(q.m), none ? 0.0f : logf(q.s)};
}
__device__ __forceinline__ float soft_entropy(Soft q) { return q.s == 0.0f ? 0.0f : logf(q.s) - q.w / q.s; }

template <class T>
__device__ __forceinline__ void put_row(const LogpArgs& a, int64_t o, int64_t t, const T* z, Soft q, LogP lp) {
  if (a.logp) a.logp[o] = t < a.v ? lp((float)z[t]) : __builtin_nanf("");
  if (a.entropy) a.entropy[o] = soft_entropy(q);
  if (a.lse) a.lse[o] = q.s == 0.0f ? -__builtin_inff() : lp.base + lp.logs;
}
__device__ __forceinline__ void put_padding(const LogpArgs& a, int64_t o, int i) {
  if (i == 0) {
    if (a.logp) a.logp[o] = 0.0f;
    if (a.entropy) a.entropy[o] = 0.0f;
    if (a.lse) a.lse[o] = 0.0f;
  }
  if (i < a.top) a.top_logp[o * a.top + i] = 0.0f, a.top_idx[o * a.top + i] = -1;
}

// ---- a group of lanes a row ----------------------------------------------------
// Reductions over RT = 16 lanes by rotations within a row of 16 (every lane gets the result, in the same bits, as
// each step only exchanges the operands of a commutative operation), over 32 and 64 by joining the rows' results.
template <int N>
__device__ __forceinline__ int rotate16(int v) { return __builtin_amdgcn_update_dpp(0, v, 0x120 + N, 0xf, 0xf, true); }
template <int RT, class F>
__device__ __forceinline__ int group_reduce(int v, F f) {
  v = f(v, rotate16<8>(v));
  v = f(v, rotate16<4>(v));
  v = f(v, rotate16<2>(v));
  v = f(v, rotate16<1>(v));
  if constexpr (RT == 32) v = f(v, __shfl_xor(v, 16, 64));
  if constexpr (RT == 64)
    v = f(f(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)),
          f(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
  return v;
}
template <int RT>
__device__ __forceinline__ float group_fmax(float v) {
  return __int_as_float(group_reduce<RT>(__float_as_int(v), [](int a, int b) {
    return __float_as_int(fmaxf(__int_as_float(a), __int_as_float(b)));
  }));
}
template <int RT>
__device__ __forceinline__ float group_fsum(float v) {
  return __int_as_float(group_reduce<RT>(__float_as_int(v), [](int a, int b) {
    return __float_as_int(__int_as_float(a) + __int_as_float(b));
  }));
}
template <int RT>
__device__ __forceinline__ uint32_t group_umax(uint32_t v) {
  return (uint32_t)group_reduce<RT>((int)v, [](int a, int b) { return (int)((uint32_t)a > (uint32_t)b ? (uint32_t)a : (uint32_t)b); });
}
template <int RT>
__device__ __forceinline__ uint32_t group_umin(uint32_t v) {
  return (uint32_t)group_reduce<RT>((int)v, [](int a, int b) { return (int)((uint32_t)a < (uint32_t)b ? (uint32_t)a : (uint32_t)b); });
}

// One vector's classes c, c + 1, ... by their order among the alternatives (NaN as plain_nan's).  Ones below
// `own` are another vector's and have key 0; ones past the row are -inf with numbers past every other, so they
// come last (fp32: key 0 for c >= v, if v is given).  sort() puts them in order, pop() takes the first away.
template <class T>
struct TopVec {   // 16-bit logits: rank and number in one word, all different, sorted by a merge network (Batcher, 1968)
  uint32_t key[8];
  __device__ __forceinline__ void keys(const float (&z)[8], int c, int own, int) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      uint32_t u;
      if constexpr (__is_same(T, __bf16)) u = rank_of(z[k]) & 0xffff0000u;   // a bf16's bits are a float's upper half
      else {
        const int h = (int)__builtin_bit_cast(uint16_t, (_Float16)(z[k] + 0.0f)) << 16;
        u = (uint32_t)(h ^ (h >> 31 | (int)0x80000000)) & 0xffff0000u;
      }
      key[k] = u | (uint32_t)(0xffff - (c + k));
    }
    if (c < own)
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c + k < own) key[k] = 0;
  }
  __device__ __forceinline__ void sort() {
    constexpr int net[19][2] = {{0, 1}, {2, 3}, {4, 5}, {6, 7}, {0, 2}, {1, 3}, {4, 6}, {5, 7}, {1, 2}, {5, 6},
                                {0, 4}, {1, 5}, {2, 6}, {3, 7}, {2, 4}, {3, 5}, {1, 2}, {3, 4}, {5, 6}};
#pragma unroll
    for (int i = 0; i < 19; ++i) {
      const uint32_t x = key[net[i][0]], y = key[net[i][1]];
      key[net[i][0]] = x > y ? x : y;
      key[net[i][1]] = x > y ? y : x;
    }
  }
  __device__ __forceinline__ uint32_t at(int) const { return 0; }   // (in the key)
  __device__ __forceinline__ void pop(bool on) {
#pragma unroll
    for (int k = 0; k < 7; ++k) key[k] = on ? key[k + 1] : key[k];
    if (on) key[7] = 0;
  }
  static __device__ __forceinline__ int number(uint32_t key, uint32_t) { return 0xffff - (int)(key & 0xffffu); }
  static __device__ __forceinline__ float value(uint32_t key) {
    if constexpr (__is_same(T, __bf16)) return key_value((u64)(key & 0xffff0000u) << 32 | ((key >> 31) ? 0ull : 0xffffull << 32));
    const uint32_t u = key >> 16;
    return (float)__builtin_bit_cast(_Float16, (uint16_t)((u >> 15) ? u & 0x7fffu : ~u));
  }
};
template <>
struct TopVec<float> {   // sorted by neighbours' exchanges, which keep equal logits in their order
  uint32_t key[4], k_[4];
  __device__ __forceinline__ void keys(const float (&z)[4], int c, int own, int v) {
#pragma unroll
    for (int k = 0; k < 4; ++k) key[k] = rank_of(z[k]);
    if (c < own)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + k < own) key[k] = 0;
    if (v < 1 << 30)   // (the same for all lanes)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + k >= v) key[k] = 0;
  }
  __device__ __forceinline__ void sort() {
#pragma unroll
    for (int k = 0; k < 4; ++k) k_[k] = k;
    constexpr int net[6] = {0, 2, 1, 0, 2, 1};
#pragma unroll
    for (int i = 0; i < 6; ++i) {
      const int x = net[i], y = x + 1;
      const bool swap = key[y] > key[x];
      const uint32_t a = key[x], b = k_[x];
      key[x] = swap ? key[y] : a, k_[x] = swap ? k_[y] : b;
      key[y] = swap ? a : key[y], k_[y] = swap ? b : k_[y];
    }
  }
  __device__ __forceinline__ uint32_t at(int c) const { return (uint32_t)c + k_[0]; }
  __device__ __forceinline__ void pop(bool on) {
#pragma unroll
    for (int k = 0; k < 3; ++k) key[k] = on ? key[k + 1] : key[k], k_[k] = on ? k_[k + 1] : k_[k];
    if (on) key[3] = 0;
  }
  static __device__ __forceinline__ int number(uint32_t, uint32_t at) { return (int)at; }
  static __device__ __forceinline__ float value(uint32_t key) { return key_value((u64)key << 32); }
};

// Sum of v over the group's lanes up to this one, and the last lane's.
template <int RT>
__device__ __forceinline__ int group_scan(int v, int* last) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);   // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  const int lane = threadIdx.x & 63;
  if constexpr (RT >= 32) {
    const int t = __shfl(v, (lane & 32) + 15, 64);
    if (lane & 16) v += t;
  }
  if constexpr (RT == 64) {
    const int t = __builtin_amdgcn_readlane(v, 31);
    if (lane & 32) v += t;
  }
  *last = __shfl(v, lane | (RT - 1), 64);
  return v;
}

// Rows of up to RT * E vectors of 16 bytes, in registers: class (e RT + lane) VW + k.
// Alternatives: each vector is sorted for itself, and then they are drawn one by one,
// each lane offering its best class left.  With 16 lanes a row four rows share every
// reduction of a wave.  Where a lane holds four fp32 vectors and up to RT / 2 alternatives
// are wanted, less is to be done without sorting (48,000 x 256 with five: 18.7 us
// drawn, 16.6 so; 12,000 x 1,024 with 20: 38 and 24; but bf16, 48,000 x 256 with five, 14.3 and 15.4): the top-th
// largest of the lanes' best classes is no larger than the top-th largest class, and few
// classes reach it; those are listed in LDS and ranked among each other, unless they are
// more than LR_CAP (many equal ones).
//
// 48,000 x 256 fp32 (52 MB, 11 us at a copy's rate): 10.7 us without alternatives, 15.7 with
// five, bound by vector instructions then.  Widths between the shapes have their own:
// 24,000 x 512 fp32 with five, in half of the shape for 1,024, took 34 us for 17.
template <class T, int RT, int E, bool TAIL>
__global__ __launch_bounds__(256) void wr_logp_rows_kernel(LogpArgs a) {
  constexpr int VW = 16 / sizeof(T), KR = (WAVERNN_MAX_TOP + RT - 1) / RT;
  constexpr bool packed = sizeof(T) == 2;
  constexpr bool LIST = !packed && E == 4;
  __shared__ u64 lists[LIST ? 256 / RT : 1][LIST ? LR_CAP : 1];
  const int lane = threadIdx.x % RT;
  u64* list = lists[LIST ? threadIdx.x / RT : 0];
  const int64_t step = (int64_t)gridDim.x * (256 / RT);
  for (int64_t row = (int64_t)blockIdx.x * (256 / RT) + threadIdx.x / RT; row < a.n; row += step) {
    const int64_t t = row_token(a, row), o = row_out(a, row);
    if (t < 0) {
      for (int i = lane; i == lane || i < a.top; i += RT) put_padding(a, o, i);
      continue;
    }
    const T* zr = (const T*)a.logits + row * a.stride;
    Raw<T, VW> raw[E];
    int c[E];   // the first class of each vector; a row's last one may begin with another lane's classes
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c0 = (e * RT + lane) * VW;
      c[e] = !TAIL || a.v < VW || c0 >= a.v ? c0 : vec_begin<VW>(c0, a.v);
      raw[e] = load_raw<T, VW>(zr + c[e], a.v - c[e], (T)-__builtin_inff());
    }
    float z[E][VW];
    Soft q{-__builtin_inff(), 0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < E; ++e) {
#pragma unroll
      for (int k = 0; k < VW; ++k) z[e][k] = (float)raw[e][k];
      if (TAIL && c[e] < (e * RT + lane) * VW)   // (no lane of most waves)
#pragma unroll
        for (int k = 0; k < VW; ++k)
          if (c[e] + k < (e * RT + lane) * VW) z[e][k] = -__builtin_inff();
#pragma unroll
      for (int k = 0; k < VW; ++k) q.m = fmaxf(q.m, z[e][k]);
    }
    q.m = group_fmax<RT>(q.m);
    const float base = soft_base(q.m);
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int k = 0; k < VW; ++k) soft_term(z[e][k], base, q.s, q.w);
    q.s = group_fsum<RT>(q.s);
    q.w = group_fsum<RT>(q.w);
    const LogP lp = soft_logp(q);
    if (lane == 0) put_row(a, o, t, zr, q, lp);
    if (a.top == 0) continue;
    TopVec<T> vec[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (q.s != q.s)
#pragma unroll
        for (int k = 0; k < VW; ++k) z[e][k] = plain_nan(z[e][k]);
      vec[e].keys(z[e], c[e], TAIL ? (e * RT + lane) * VW : c[e], LIST && a.v < RT * E * VW ? a.v : 1 << 30);
    }
    if (LIST && a.top <= RT / 2) {
      uint32_t left = 0, low = 0;
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int k = 0; k < VW; ++k) left = max(left, vec[e].key[k]);
      for (int i = 0; i < a.top; ++i) {   // (lanes whose best are equal go at once, which lowers the bound at most)
        low = group_umax<RT>(left);
        left = left == low ? 0 : left;
      }
      low = max(low, 1u);
      int mine = 0, n;
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int k = 0; k < VW; ++k) mine += vec[e].key[k] >= low;
      int to = group_scan<RT>(mine, &n) - mine;
      if (n <= LR_CAP) {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int k = 0; k < VW; ++k)
            if (vec[e].key[k] >= low) list[to++] = (u64)vec[e].key[k] << 32 | (uint32_t)~(c[e] + k);
        __builtin_amdgcn_wave_barrier();   // (a group lies in one wave, whose LDS accesses are in order)
        for (int i = lane; i < n; i += RT) {
          const u64 w = list[i];
          int r = 0;
          for (int j0 = 0; j0 < n; j0 += 4) {   // (LR_CAP is a multiple of 4)
            u64 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = list[j0 + j];
#pragma unroll
            for (int j = 0; j < 4; ++j) r += j0 + j < n && x[j] > w;
          }
          if (r < a.top) {
            a.top_idx[o * a.top + r] = key_class(w);
            a.top_logp[o * a.top + r] = lp(key_value(w));
          }
        }
        __builtin_amdgcn_wave_barrier();
        continue;
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) vec[e].sort();
    uint32_t won[KR] = {}, won_at[KR] = {};
    for (int i = 0; i < a.top; ++i) {
      uint32_t best = vec[0].key[0], at = vec[0].at(c[0]);
#pragma unroll
      for (int e = 1; e < E; ++e) {
        const bool more = vec[e].key[0] > best;
        best = more ? vec[e].key[0] : best;
        if constexpr (!packed) at = more ? vec[e].at(c[e]) : at;
      }
      const uint32_t m = group_umax<RT>(best);
      uint32_t j = 0;
      if constexpr (!packed) j = group_umin<RT>(best == m ? at : 0xffffffffu);
#pragma unroll
      for (int r = 0; r < KR; ++r)
        if (lane + r * RT == i) won[r] = m, won_at[r] = j;
#pragma unroll
      for (int e = 0; e < E; ++e) vec[e].pop(packed ? vec[e].key[0] == m : vec[e].at(c[e]) == j);
    }
#pragma unroll
    for (int r = 0; r < KR; ++r)
      if (lane + r * RT < a.top) {
        a.top_idx[o * a.top + lane + r * RT] = TopVec<T>::number(won[r], won_at[r]);
        a.top_logp[o * a.top + lane + r * RT] = lp(TopVec<T>::value(won[r]));
      }
  }
}

// ---- a block a row, or a block a segment of a row --------------------------------
// One pass over the row, four vectors a thread in flight, with the running maximum and
// sums of each thread; the alternatives are then looked for where they can be.  Each quad of lanes
// keeps the largest logit it saw.  The top-th largest of the 64 quads' values, `low`, is no
// larger than the top-th largest logit, so only quads that reach it can hold an
// alternative: their vectors (for few alternatives a small part of the row) are read once more,
// from cache, and the classes that reach `low` are ranked among each other.
// Bound by memory: 4,096 x 65,536 bf16 105 us without alternatives (5.1 TB/s; a copy reaches
// 4.7), 122 with eight, each on its own; 145 in a training step, behind the gradient's 537 MB of writes.
#define LW_U 4        // vectors in flight
#define LW_CAP 1024   // classes ranked

struct LogpShared {
  Soft soft[4];
  uint32_t quad[64];
  int count, need;
  u64 list[LW_CAP];
  u64 wave_best[4];
  int wave_count[4];
  uint8_t quads[4][64];   // each wave's list of the quads to look into
};

// What is found of a row or segment: kept for the join if the row has several.
struct LogpPart {
  Soft q;
  float pad;
};

// Writes alternative k (0 <= k < top) of the row or segment.
__device__ __forceinline__ void put_top(const LogpArgs& a, int64_t o, int64_t part, int k, u64 key, LogP lp) {
  if (a.splits > 1) {
    a.part_keys[part * a.top + k] = key;
  } else {
    a.top_idx[o * a.top + k] = key_class(key);
    a.top_logp[o * a.top + k] = lp(key_value(key));
  }
}
// The `top` largest of the n classes listed, in order, by counting the larger ones.
__device__ __forceinline__ void put_ranked(const LogpArgs& a, LogpShared& sh, int n, int64_t o, int64_t part, LogP lp) {
  for (int i = threadIdx.x; i < n; i += 256) {
    const u64 key = sh.list[i];
    int r = 0;
    for (int j0 = 0; j0 < n; j0 += 8) {   // (eight reads under way together; LW_CAP is a multiple of 8)
      u64 x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = sh.list[j0 + j];
#pragma unroll
      for (int j = 0; j < 8; ++j) r += j0 + j < n && x[j] > key;
    }
    if (r < a.top) put_top(a, o, part, r, key, lp);
  }
}

// The alternatives of classes j0 .. j0 + nj - 1, whose vectors the block's threads took in turn.
template <class T>
__device__ __forceinline__ void find_top(const LogpArgs& a, LogpShared& sh, const T* z0, int j0, int nj, int vecs, int64_t o,
                                         int64_t part, LogP lp) {
  constexpr int VW = 16 / sizeof(T);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  // every wave finds the top-th largest quad for itself, bit by bit
  const uint32_t mine = sh.quad[lane];
  uint32_t low = 0;
  for (int b = 31; b >= 0; --b) {
    const uint32_t tryit = low | 1u << b;
    if (__popcll(__ballot(mine >= tryit)) >= a.top) low = tryit;
  }
  const u64 quads = __ballot(mine >= low && mine > 0);
  const int nq = __popcll(quads);
  if (quads >> lane & 1) sh.quads[wave][__popcll(quads & ((1ull << lane) - 1))] = (uint8_t)lane;
  __builtin_amdgcn_wave_barrier();
  // reads the vectors of those quads: thread tid takes lane tid % 4 of quad number tid / 4, and so on
  auto scan = [&](auto&& take) {
    const int rounds = (vecs + 255) / 256;   // vectors of a thread
    for (int x = tid >> 2; x < nq * rounds; x += 64) {
      const int vec = x / nq * 256 + sh.quads[wave][x % nq] * 4 + (tid & 3);
      if (vec >= vecs) continue;
      float z[VW];
      const int c = vec * VW, count = nj - c;
      load_part<T, VW>(z0 + c, z, count);
#pragma unroll
      for (int k = 0; k < VW; ++k)
        if (k < count) take(z[k], j0 + c + k);
    }
  };
  scan([&](float z, int j) {
    if (top_rank(z) >= low) {
      const int at = atomicAdd(&sh.count, 1);
      if (at < LW_CAP) sh.list[at] = top_key(z, j);
    }
  });
  __syncthreads();
  int n = sh.count;
  if (n <= LW_CAP) return put_ranked(a, sh, n, o, part, lp);
  // Too many equal or close classes.  Those above `low` alone, and then the first that equal it:
  __syncthreads();
  if (tid == 0) sh.count = 0;
  __syncthreads();
  scan([&](float z, int j) {
    if (top_rank(z) > low) {
      const int at = atomicAdd(&sh.count, 1);
      if (at < LW_CAP) sh.list[at] = top_key(z, j);
    }
  });
  __syncthreads();
  n = sh.count;
  if (n <= LW_CAP) {
    put_ranked(a, sh, n, o, part, lp);
    int have = n;
    for (int i0 = 0; have < a.top && i0 < vecs; i0 += 256) {
      float z[VW];
      const int c = (i0 + tid) * VW, count = i0 + tid < vecs ? min(nj - c, VW) : 0;
      load_part<T, VW>(z0 + c, z, count);
      int mineq = 0;
#pragma unroll
      for (int k = 0; k < VW; ++k) mineq += k < count && top_rank(z[k]) == low;
      int before = mineq;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int x = __shfl_up(before, d, 64);
        if (lane >= d) before += x;
      }
      if (lane == 63) sh.wave_count[wave] = before;
      __syncthreads();
      int r = have + before - mineq;
      for (int w = 0; w < 4; ++w) {
        if (w < wave) r += sh.wave_count[w];
        have += sh.wave_count[w];
      }
#pragma unroll
      for (int k = 0; k < VW; ++k)
        if (k < count && top_rank(z[k]) == low) {
          if (r < a.top) put_top(a, o, part, r, top_key(z[k], j0 + c + k), lp);
          ++r;
        }
      __syncthreads();
    }
    return;
  }
  // One after another: the largest class below the last one found.
  u64 prev = ~0ull;
  for (int k = 0; k < a.top; ++k) {
    u64 best = 0;
    scan([&](float z, int j) {
      const u64 key = top_key(z, j);
      if (key < prev && key > best) best = key;
    });
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
      const u64 x = __shfl_xor(best, d, 64);
      best = x > best ? x : best;
    }
    __syncthreads();
    if (lane == 0) sh.wave_best[wave] = best;
    __syncthreads();
    for (int w = 0; w < 4; ++w) best = sh.wave_best[w] > best ? sh.wave_best[w] : best;
    if (tid == 0) put_top(a, o, part, k, best, lp);
    prev = best;
  }
}

template <class T>
__global__ __launch_bounds__(256) void wr_logp_kernel(LogpArgs a) {
  constexpr int VW = 16 / sizeof(T);
  __shared__ LogpShared sh;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int64_t items = a.n * a.splits;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t row = a.splits > 1 ? item / a.splits : item;
    const int64_t t = row_token(a, row), o = row_out(a, row);
    if (t < 0) {
      if (a.splits == 1) put_padding(a, o, tid);
      continue;
    }
    const T* zr = (const T*)a.logits + row * a.stride;
    // classes j0 .. j1 - 1 of the row, thread t's vectors t, t + 256, ... of them
    const int j0 = a.splits > 1 ? (int)(item % a.splits) * a.seg : 0;
    const int j1 = a.splits > 1 ? (int)std::min<int64_t>(a.v, (int64_t)j0 + a.seg) : a.v;
    const T* z0 = zr + j0;
    const int nj = j1 - j0, vecs = (nj + VW - 1) / VW;
    Soft q{-__builtin_inff(), 0.0f, 0.0f};
    for (int i = tid; i < vecs; i += 256 * LW_U) {
      Raw<T, VW> z[LW_U];
      float m = q.m;
#pragma unroll
      for (int u = 0; u < LW_U; ++u) {
        const int64_t c = (int64_t)(i + u * 256) * VW;
        z[u] = load_raw<T, VW>(z0 + c, i + u * 256 < vecs ? nj - (int)c : 0, (T)-__builtin_inff());
      }
#pragma unroll
      for (int u = 0; u < LW_U; ++u)
#pragma unroll
        for (int k = 0; k < VW; ++k) m = fmaxf(m, (float)z[u][k]);
      if (m > q.m) q = soft_at(q, m);
      const float base = soft_base(m);
#pragma unroll
      for (int u = 0; u < LW_U; ++u)
#pragma unroll
        for (int k = 0; k < VW; ++k) soft_term((float)z[u][k], base, q.s, q.w);
    }
    const float best = q.m;
    const bool nan = q.s != q.s;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1)
      q = soft_join(q, Soft{__shfl_xor(q.m, d, 64), __shfl_xor(q.s, d, 64), __shfl_xor(q.w, d, 64)});
    if (lane == 0) sh.soft[wave] = q;
    if (a.top > 0) {
      uint32_t r = tid < vecs ? top_rank(best) : 0;
      if (nan)   // a NaN, which comes first among the alternatives and which the maximum passes over, or +inf
        for (int i = tid; i < vecs; i += 256)
          for (int j = i * VW; j < min(nj, (i + 1) * VW); ++j) r = max(r, top_rank((float)z0[j]));
      r = max(r, (uint32_t)__builtin_amdgcn_update_dpp((int)r, (int)r, 0xb1, 0xf, 0xf, false));   // quad: lanes 1 0 3 2
      r = max(r, (uint32_t)__builtin_amdgcn_update_dpp((int)r, (int)r, 0x4e, 0xf, 0xf, false));   // quad: lanes 2 3 0 1
      if ((lane & 3) == 0) sh.quad[tid >> 2] = r;
      if (tid == 0) sh.count = 0;
    }
    __syncthreads();
    q = soft_join(soft_join(sh.soft[0], sh.soft[1]), soft_join(sh.soft[2], sh.soft[3]));
    if (tid == 0) {
      if (a.splits == 1) put_row(a, o, t, zr, q, soft_logp(q));
      else ((LogpPart*)a.part)[item].q = q;
    }
    if (a.top > 0) {
      const LogP lp = a.splits == 1 ? soft_logp(q) : LogP{};   // (segments keep the logits)
      find_top<T>(a, sh, z0, j0, nj, vecs, o, item, lp);
    }
    __syncthreads();
  }
}

// Joins the segments of each row.
template <class T>
__global__ __launch_bounds__(256) void wr_logp_join_kernel(LogpArgs a) {
  __shared__ LogpShared sh;
  const int tid = threadIdx.x, lane = tid & 63;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const int64_t t = row_token(a, row), o = row_out(a, row);
    if (t < 0) {
      put_padding(a, o, tid);
      continue;
    }
    const LogpPart* part = (const LogpPart*)a.part + row * a.splits;
    Soft q{-__builtin_inff(), 0.0f, 0.0f};
    for (int i = lane; i < a.splits; i += 64) q = soft_join(q, part[i].q);   // every wave the same
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1)
      q = soft_join(q, Soft{__shfl_xor(q.m, d, 64), __shfl_xor(q.s, d, 64), __shfl_xor(q.w, d, 64)});
    const LogP lp = soft_logp(q);
    if (tid == 0) put_row(a, o, t, (const T*)a.logits + row * a.stride, q, lp);
    if (a.top == 0) continue;
    // Each segment's classes come in order, so the top-th largest of their first few (enough that there are
    // `top` of them) is a lower bound, and what reaches it is ranked: with a bound from the best ones alone
    // it is reached in at most `top` segments, at most top^2 classes.
    const u64* keys = a.part_keys + row * a.splits * a.top;
    const int first = (a.top + a.splits - 1) / a.splits, heads = first * a.splits;   // heads < 2 top or = splits
    if (tid < heads) sh.list[tid] = keys[tid / first * a.top + tid % first];
    if (tid == 0) sh.count = 0;
    __syncthreads();
    if (tid < heads) {
      const u64 mine = sh.list[tid];
      int r = 0;
#pragma unroll 8
      for (int j = 0; j < heads; ++j) r += sh.list[j] > mine;
      if (r == a.top - 1) sh.wave_best[0] = mine;
    }
    __syncthreads();
    const u64 low = sh.wave_best[0];
    __syncthreads();
    for (int i = tid; i < a.splits * a.top; i += 256) {
      const u64 key = keys[i];
      if (key >= low) sh.list[atomicAdd(&sh.count, 1)] = key;
    }
    __syncthreads();
    LogpArgs b = a;
    b.splits = 1;
    put_ranked(b, sh, sh.count, o, 0, lp);
    __syncthreads();
  }
}

// ---- gradient ----------------------------------------------------------------
// One thread a vector, LG_U vectors in flight; rows of up to 256 LG_U vectors share
// blocks or take one, wider ones take a block for every 256 LG_U vectors.  Bound by
// memory: 4,096 x 65,536 bf16 183 us, 5.7 TB/s read and written.
#define LG_U 4

template <class T>
__global__ __launch_bounds__(256) void wr_logp_grad_kernel(LogpGradArgs a) {
  constexpr int VW = 16 / sizeof(T);
  const int rt = a.row_threads, t0 = threadIdx.x % rt, v = a.f.v;
  const int64_t items = a.f.n * a.splits, step = (int64_t)gridDim.x * (256 / rt);
  for (int64_t item = (int64_t)blockIdx.x * (256 / rt) + threadIdx.x / rt; item < items; item += step) {
    const int64_t row = a.splits > 1 ? item / a.splits : item;
    const int seg = a.splits > 1 ? (int)(item % a.splits) : 0;
    const int64_t t = row_token(a.f, row);
    const T* z = (const T*)a.f.logits + row * a.f.stride;
    T* dz = (T*)a.dlogits + row * a.dstride;
    Raw<T, VW> raw[LG_U];
    const int64_t i0 = ((int64_t)seg * LG_U * rt + t0) * VW;
#pragma unroll
    for (int u = 0; u < LG_U; ++u) {
      const int64_t j = i0 + (int64_t)u * rt * VW;
      raw[u] = load_raw<T, VW>(z + j, t < 0 || j >= v ? 0 : (int)(v - j));
    }
    const float lse = t < 0 ? 0.0f : a.lse_in[row];
    const bool zero = t < 0 || lse == -__builtin_inff();   // padding, or every class masked
    const float gl = a.g_logp && !zero ? a.g_logp[row] : 0.0f;
    const float gh = a.g_entropy && !zero ? a.g_entropy[row] : 0.0f, h = a.g_entropy && !zero ? a.entropy_in[row] : 0.0f;
    float gp = (a.g_lse && !zero ? a.g_lse[row] : 0.0f) - gl;
    if (a.g_logp && t >= v) gp = __builtin_nanf("");
    const int32_t* ti = a.f.top_idx + row * a.f.top;
    const float* tg = a.g_top + row * a.f.top;
    if (!zero)
      for (int k = 0; k < a.f.top; ++k)
        if (ti[k] >= 0 && ti[k] < v) gp -= tg[k];
#pragma unroll
    for (int u = 0; u < LG_U; ++u) {
      const int64_t j = i0 + (int64_t)u * rt * VW;
      if (j >= v) break;
      float x[VW];
#pragma unroll
      for (int k = 0; k < VW; ++k) x[k] = zero ? 0.0f : (float)raw[u][k];
      if (!zero) {
#pragma unroll
        for (int k = 0; k < VW; ++k) {
          const float lp = x[k] - lse;
          x[k] = fexp(lp) * (gp - gh * (fmaxf(lp, WR_FAR) + h));
        }
        if (t >= j && t < j + VW)
#pragma unroll
          for (int k = 0; k < VW; ++k)
            if (t == j + k) x[k] += gl;
        for (int i = 0; i < a.f.top; ++i)
          if (ti[i] >= j && ti[i] < j + VW)
#pragma unroll
            for (int k = 0; k < VW; ++k)
              if (ti[i] == j + k) x[k] += tg[i];
      }
      store_part<T, VW>(dz + j, x, (int)(v - j));
    }
  }
}

wavernn_status check_logits(const char* name, int dtype, const void* p, int64_t n, int32_t v, int64_t stride, bool output) {
  if (!wr_dtype_ok(dtype)) return wr_fail(WAVERNN_E_INVALID, "bad dtype %d", dtype);
  if (n < 0 || n > INT32_MAX) return wr_fail(WAVERNN_E_INVALID, "n_rows %lld out of range", (long long)n);
  if (v < 1 || v > (1 << 30)) return wr_fail(WAVERNN_E_INVALID, "n_classes %d not in [1, 2^30]", v);
  return wr_check_rows(name, p, dtype, n, v, stride, output);
}
wavernn_status check_tokens(const void* tokens, int bytes, int* kind) {
  if (tokens && bytes != 4 && bytes != 8) return wr_fail(WAVERNN_E_INVALID, "token_bytes %d: must be 4 or 8", bytes);
  if (!wr_aligned(tokens, tokens ? bytes : 1)) return wr_fail(WAVERNN_E_INVALID, "tokens are not aligned to their elements");
  *kind = !tokens ? WR_TOK_NONE : bytes == 4 ? WR_TOK_I32 : WR_TOK_I64;
  return WAVERNN_OK;
}

}  // namespace

// Segments of a row: one, unless there are too few rows for the card (a row each for fewer than 512
// blocks, two a CU) and they are long: then as many as give 1,024 blocks, of LW_SEG classes at least.
// (1 x 65,536 with top 8, us: segments of 4,096 9.3, of 8,192 9.9, of 16,384 11.3; but 1 x 5,000 in two segments
// 8.9 and whole 5.6.  A block of 1,024 threads a row: 13.3.)
static int logp_splits(int64_t n, int32_t v) {
  if (n < 1 || n >= 512) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>({LW_SPLITS, 1024 / n, ((int64_t)v + LW_SEG - 1) / LW_SEG}));
}

template <class T, bool TAIL>
static wavernn_status rows_launch(LogpArgs& a, int vecs, void* stream) {
  auto blocks = [&](int rows) { return std::min<int64_t>((a.n + rows - 1) / rows, LOGP_BLOCKS); };
  if (vecs <= 16) WR_LAUNCH((wr_logp_rows_kernel<T, 16, 1, TAIL>), blocks(16), 256, 0, stream, a);
  else if (vecs <= 32) WR_LAUNCH((wr_logp_rows_kernel<T, 16, 2, TAIL>), blocks(16), 256, 0, stream, a);
  else if (vecs <= 64) WR_LAUNCH((wr_logp_rows_kernel<T, 16, 4, TAIL>), blocks(16), 256, 0, stream, a);
  else if (vecs <= 128) WR_LAUNCH((wr_logp_rows_kernel<T, 32, 4, TAIL>), blocks(8), 256, 0, stream, a);
  else if (vecs <= 256) WR_LAUNCH((wr_logp_rows_kernel<T, 64, 4, TAIL>), blocks(4), 256, 0, stream, a);
  else WR_LAUNCH((wr_logp_rows_kernel<T, 64, 8, TAIL>), blocks(4), 256, 0, stream, a);
  return WAVERNN_OK;
}
template <class T>
static wavernn_status logp_launch(LogpArgs& a, void* stream) {
  constexpr int VW = 16 / sizeof(T);
  const int vecs = (int)(((int64_t)a.v + VW - 1) / VW);
  if (vecs <= 512) return a.v % VW ? rows_launch<T, true>(a, vecs, stream) : rows_launch<T, false>(a, vecs, stream);
  a.splits = a.part ? logp_splits(a.n, a.v) : 1;
  a.seg = (int)(((int64_t)a.v + a.splits - 1) / a.splits + 7) / 8 * 8;
  a.part_keys = (u64*)((LogpPart*)a.part + a.n * a.splits);
  WR_LAUNCH((wr_logp_kernel<T>), std::min<int64_t>(a.n * a.splits, LOGP_BLOCKS), 256, 0, stream, a);
  if (a.splits > 1) WR_LAUNCH((wr_logp_join_kernel<T>), a.n, 256, 0, stream, a);
  return WAVERNN_OK;
}
wavernn_status wr_logp_launch(int dtype, LogpArgs& a, void* stream) {
  if (a.n == 0) return WAVERNN_OK;
  WR_DISPATCH(dtype, T, return logp_launch<T>(a, stream));
}

extern "C" {

int64_t wavernn_token_logprobs_workspace(int64_t n_rows, int32_t n_classes, int32_t top) {
  if (n_rows < 0 || n_rows > INT32_MAX || n_classes < 1 || n_classes > (1 << 30) || top < 0 || top > WAVERNN_MAX_TOP || top > n_classes) return -1;
  const int s = logp_splits(n_rows, n_classes);
  return s > 1 ? n_rows * s * (int64_t)(sizeof(LogpPart) + 8 * top) : 0;
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
  a.part = need > 0 ? workspace_dev : nullptr;
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
  const int64_t vecs = ((int64_t)n_classes * wr_dtype_bytes(dtype) + 15) / 16;
  a.row_threads = wr_row_threads((vecs + LG_U - 1) / LG_U);
  a.splits = (int)((vecs + 256 * LG_U - 1) / (256 * LG_U));
  const int64_t per = 256 / a.row_threads, grid = std::min<int64_t>((n_rows * a.splits + per - 1) / per, WR_OP_BLOCKS);
  WR_DISPATCH(dtype, T, WR_LAUNCH((wr_logp_grad_kernel<T>), grid, 256, 0, stream, a));
  return WAVERNN_OK;
}

}  // extern "C"
