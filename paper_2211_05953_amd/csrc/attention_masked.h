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

// tanh to 3 ulp without a branch: a polynomial fitted to tanh(x) / x up to 0.55 (7e-9 off), 1 - 2 / (1 + e^2x) beyond, where the
// difference costs no bits.  The library's function, inlined for every register of a tile, made the fp32 kernels long enough to
// wait for their own instructions (500 queries: dQ 71.2 us and 69.0 with this, keys 120.6 and 106.0).
__device__ __forceinline__ float tanh_f(float x) {
  const float y = fabsf(x), u = x * x;
  const float near = fmaf(x * u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, -0.00627260751f, 0.0210702536f), -0.0538518654f), 0.133325804f), -0.333333173f), x);
  const float e = __builtin_amdgcn_exp2f(y * (2.f * 1.4426950408889634f));
  return y < 0.55f ? near : copysignf(fmaf(-2.f, __builtin_amdgcn_rcpf(e + 1.f), 1.f), x);
}

// (the inverse of a cap below 2^-128 is held to what fp32 has: a score of 0 stays 0, any other saturates all the same)
__device__ __forceinline__ float inverse_cap(float cap) { return fminf(1.f / cap, FLT_MAX); }

bf_status attention_masked_fwd_mfma(const MaskedArgs& a, hipStream_t st);
bf_status attention_masked_bwd_mfma(const MaskedArgs& a, hipStream_t st);
bf_status attention_masked_fwd_f32(const MaskedArgs& a, hipStream_t st);
bf_status attention_masked_bwd_f32(const MaskedArgs& a, hipStream_t st);

}  // namespace bf
