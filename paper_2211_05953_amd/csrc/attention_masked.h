// What the kernels of masked attention share: arguments, spans, the score's way from a dot product to an exponent.
#pragma once
#include <float.h>
#include <limits.h>

#include "../../include/bf_ops.h"
#include "common.h"

namespace bf {

// A row's keys are one interval [lo, hi): a document, cut at the diagonal or at the prefix.  The spans buffer holds them for
// every row, then one summary for every 64 rows of a sequence, from which tiles are skipped or taken without a mask.
constexpr int SPAN_ROWS = 64;
struct SpanBlock { int lo_min, hi_max, lo_max, hi_min; };  // over the rows of the block; no key at all: hi_max = 0

inline size_t up4(size_t n) { return (n + 3) / 4 * 4; }  // the blocks are 16-byte aligned
inline size_t span_blocks(int S_seq) { return (size_t)((S_seq + SPAN_ROWS - 1) / SPAN_ROWS); }

struct MaskedArgs {
  int S_mb, S_seq, N_heads, N_kv, S_head;
  float scale, cap;  // cap: 0 for none
  size_t ldq, ldk, ldv, ldo;  // elements from a token to the next
  const void *q, *k, *v;
  const int2* span;          // [S_mb][S_seq]
  const SpanBlock* block;    // [S_mb][span_blocks]
  const float* slope;        // [N_heads] or null
  void* ctx;
  float* lse;                // may be null (forward)
  // backward
  const void* dctx;
  void *dq, *dk, *dv;
  float* delta;              // [S_mb][N_heads][S_seq]
  float* planes;             // fp32 shares of dk and dv, see attention_masked_bwd
  int splits;                // of a key / value head's query heads
  bool vec;                  // rows are whole 16-byte chunks
};

bf_status attention_masked_fwd_mfma(const MaskedArgs& a, hipStream_t st);
bf_status attention_masked_bwd_mfma(const MaskedArgs& a, hipStream_t st);
bf_status attention_masked_fwd_f32(const MaskedArgs& a, hipStream_t st);
bf_status attention_masked_bwd_f32(const MaskedArgs& a, hipStream_t st);

}  // namespace bf
