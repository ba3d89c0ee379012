// Arguments of the log-probability kernels (wr_logp.hip), also launched by the
// scoring entry points (wr_host.hip).
#pragma once
#include <stdint.h>

#include "wavernn.h"

// Where a row's token comes from.
enum {
  WR_TOK_NONE = 0,    // no tokens: no row is padding
  WR_TOK_I32, WR_TOK_I64,
  WR_TOK_HIGH,        // 16-bit samples: the coarse byte of sample `row`
  WR_TOK_LOW,         // its fine byte
  WR_TOK_HIGH4,       // rows 2 i, 2 i + 1: the high and low nibble of sample i's coarse byte
  WR_TOK_LOW4         // of its fine byte
};

struct LogpArgs {
  const void* logits;   // [n] rows of v elements, stride apart
  int64_t n, stride;
  int v;
  const void* tokens;
  int kind;
  int top;
  float *logp, *entropy, *lse;   // [n] each, or null
  float* top_logp;               // [n][top]
  int32_t* top_idx;              // [n][top]
  // rows of several segments (set by the launch; part: the caller's workspace, or null)
  void* part;                    // [n][splits] maximum and sums of a segment
  unsigned long long* part_keys; // [n][splits][top] its alternatives
  int splits, seg;               // segments of a row, classes of one
};

struct LogpGradArgs {
  LogpArgs f;                    // the forward call's inputs (its outputs unused but for top_idx)
  const float *lse_in, *entropy_in, *g_logp, *g_entropy, *g_lse;   // [n], null where not used (lse always)
  const float* g_top;            // [n][f.top]
  void* dlogits;
  int64_t dstride;
  int row_threads, splits;       // threads on a row or segment, segments of a row
};

wavernn_status wr_logp_launch(int dtype, LogpArgs& a, void* stream);
