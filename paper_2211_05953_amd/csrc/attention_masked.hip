// Attention under masks that are an interval of keys per row (documents, prefixes, causal or not), with scores capped by a
// tanh, a bias that falls with distance, and query heads that share key / value heads: spans, dispatch, and the plain kernels.
//
//   c_ij = cap tanh(scale q_i.k_j / cap)   (or scale q_i.k_j),   b_ij = c_ij - slope |i - j|
//   P = softmax of b over j in [lo_i, hi_i),   ctx = P V,   lse = log-sum-exp of b
//   dB = P (dctx V^T - delta),  delta_i = dctx_i . ctx_i = sum_j P_ij dP_ij,  dP = dctx V^T,   dS = dB (1 - tanh^2) scale
//   dq = dS K,   dk = dS^T Q,   dv = P^T dctx,   dk and dv summed over the query heads of a key / value head
// A row with one key has dB = 0 (its P is 1 whatever the score), taken as exactly that; a row with none has ctx = 0,
// lse = -inf and no gradient.
#include "attention_masked.h"

#include <math.h>

#include "../../include/bf_ops.h"

namespace bf {

namespace {

constexpr int NT = 256;

bf_status launched() {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_error("attention_masked: launch failed: %s", hipGetErrorString(e)); return BF_EDEVICE; }
  return BF_OK;
}

// ---- spans -----------------------------------------------------------------------------------------
// 1024 tokens a workgroup.  The first token of a document is a scan over the boundaries in front: in registers inside a wave, over
// the workgroup's waves in LDS, and in front of the workgroup's first token a search backwards, 4096 ids at a time; its end
// likewise from behind.
constexpr int TOKENS = 1024;

__global__ __launch_bounds__(TOKENS) void spans_kernel(int S, int causal, const int32_t* __restrict__ doc, const int32_t* __restrict__ prefix,
                                                       int2* __restrict__ span, SpanBlock* __restrict__ block, int blocks) {
  __shared__ int begin_s[TOKENS / 64], end_s[TOKENS / 64], found[2];
  const int b = blockIdx.y, t0 = blockIdx.x * TOKENS, tid = threadIdx.x, lane = tid & 63, w = tid >> 6, i = t0 + tid;
  int begin = 0, end = S;
  bool pad = false;
  if (doc) {
    const int32_t* d = doc + (size_t)b * S;
    const int mine = i < S ? d[i] : 0;
    pad = mine < 0;
    // the document's first token: the last boundary at or in front of i
    int at = i < S && (i == 0 || d[i - 1] != mine) ? i : -1;
    // one past its last: the first boundary behind i
    int to = i < S && (i == S - 1 || d[i + 1] != mine) ? i + 1 : INT_MAX;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int p = __shfl_up(at, o, 64), n = __shfl_down(to, o, 64);
      if (lane >= o) at = max(at, p);
      if (lane + o < 64) to = min(to, n);
    }
    if (lane == 63) begin_s[w] = at;
    if (lane == 0) end_s[w] = to;
    if (tid == 0) { found[0] = -1; found[1] = INT_MAX; }
    __syncthreads();
    // in front of the workgroup's tokens, and behind them
    for (int hi = t0; hi > 0; hi -= 4 * TOKENS) {
      int f = -1;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int x = hi - 1 - (k * TOKENS + tid);
        if (x >= 0 && (x == 0 || d[x - 1] != d[x])) f = max(f, x);
      }
      if (f >= 0) atomicMax(&found[0], f);
      __syncthreads();
      const bool done = found[0] >= 0;
      __syncthreads();
      if (done) break;
    }
    for (int lo = t0 + TOKENS; lo < S; lo += 4 * TOKENS) {
      int f = INT_MAX;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int x = lo + k * TOKENS + tid;
        if (x < S && (x == S - 1 || d[x + 1] != d[x])) f = min(f, x + 1);
      }
      if (f < INT_MAX) atomicMin(&found[1], f);
      __syncthreads();
      const bool done = found[1] < INT_MAX;
      __syncthreads();
      if (done) break;
    }
    begin = at;
    end = to;
    for (int k = 0; k < w; ++k) begin = max(begin, begin_s[k]);
    for (int k = w + 1; k < TOKENS / 64; ++k) end = min(end, end_s[k]);
    if (begin < 0) begin = found[0];
    if (end == INT_MAX) end = found[1];
  }
  if (causal) end = min(end, max(i + 1, prefix ? prefix[b] : 0));
  if (pad) begin = end = 0;
  const bool row = i < S;
  if (row) span[(size_t)b * S + i] = make_int2(begin, end);
  // the wave's 64 rows are one block
  const bool any = row && end > begin;
  SpanBlock x{any ? begin : INT_MAX, any ? end : 0, row ? (any ? begin : INT_MAX) : 0, row ? (any ? end : 0) : INT_MAX};
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    x.lo_min = min(x.lo_min, __shfl_xor(x.lo_min, o, 64));
    x.hi_max = max(x.hi_max, __shfl_xor(x.hi_max, o, 64));
    x.lo_max = max(x.lo_max, __shfl_xor(x.lo_max, o, 64));
    x.hi_min = min(x.hi_min, __shfl_xor(x.hi_min, o, 64));
  }
  const int at = t0 / SPAN_ROWS + w;
  if (lane == 0 && at < blocks) block[(size_t)b * blocks + at] = x;
}

// ---- plain kernels: one wave per row, any head size up to 1024 -------------------------------------
// Scalar products, a lane to a key: 500 tokens, 8 heads of 256 over 4, causal, bf16: forward 338 us (3 TFLOP/s), backward 2765.  For the sizes that the
// matrix-core kernels have no form for, and to check them against.
constexpr int PLAIN_HEAD = 1024, PER = PLAIN_HEAD / 64;

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// a score from a dot product; slack: the derivative of the cap there
__device__ __forceinline__ float score_of(float dot, const MaskedArgs& a, float slope, int i, int j, float& slack) {
  float s = dot * a.scale;
  slack = 1.f;
  if (a.cap > 0.f) {
    const float t = tanhf(s / a.cap);
    s = a.cap * t;
    slack = 1.f - t * t;
  }
  return s - slope * fabsf((float)(i - j));
}

// what probabilities are taken from again: a row without a finite score has none
__device__ __forceinline__ float lse_of(float lse) { return lse == -INFINITY ? INFINITY : lse; }

template <typename T>
__device__ __forceinline__ float dot_row(const float* x, const T* y, int d) {
  float s = 0.f;
  for (int c = 0; c < d; ++c) s = fmaf(x[c], (float)y[c], s);
  return s;
}

template <typename T>
__global__ __launch_bounds__(64) void plain_fwd_kernel(MaskedArgs a) {
  __shared__ float q_s[PLAIN_HEAD];
  const int lane = threadIdx.x, i = blockIdx.x, head = blockIdx.y % a.N_heads, b = blockIdx.y / a.N_heads, d = a.S_head;
  const int kv = head / (a.N_heads / a.N_kv);
  const size_t row = (size_t)b * a.S_seq + i;
  const T* q = (const T*)a.q + row * a.ldq + (size_t)head * d;
  for (int c = lane; c < d; c += 64) q_s[c] = (float)q[c];
  __syncthreads();
  const int2 sp = a.span[row];
  const int lo = max(sp.x, 0), hi = min(sp.y, a.S_seq);
  const float slope = a.slope ? a.slope[head] : 0.f;
  float m = -FLT_MAX, l = 0.f, o[PER];
  for (int c = 0; c < PER; ++c) o[c] = 0.f;
  for (int j0 = lo; j0 < hi; j0 += 64) {
    const int j = j0 + lane;
    float slack, s = -INFINITY;
    if (j < hi) s = score_of(dot_row(q_s, (const T*)a.k + ((size_t)b * a.S_seq + j) * a.ldk + (size_t)kv * d, d), a, slope, i, j, slack);
    const float mx = fmaxf(m, wave_max(s)), alpha = expf(m - mx);
    const float p = j < hi ? expf(s - mx) : 0.f;
    l = l * alpha + wave_sum(p);
    m = mx;
    for (int c = 0; c < PER; ++c) o[c] *= alpha;
    for (int k = 0; k < 64 && j0 + k < hi; ++k) {
      const float pk = __shfl(p, k, 64);
      const T* v = (const T*)a.v + ((size_t)b * a.S_seq + j0 + k) * a.ldv + (size_t)kv * d;
      for (int c = 0; c * 64 + lane < d; ++c) o[c] = fmaf(pk, (float)v[c * 64 + lane], o[c]);
    }
  }
  T* out = (T*)a.ctx + row * a.ldo + (size_t)head * d;
  for (int c = 0; c * 64 + lane < d; ++c) out[c * 64 + lane] = (T)(l > 0.f || l != l ? o[c] / l : 0.f);
  if (lane == 0 && a.lse) a.lse[((size_t)b * a.N_heads + head) * a.S_seq + i] = l == 0.f ? -INFINITY : m + logf(l);
}

// delta: fp32 dctx . ctx; bf16 the sum of P dP as it is, since ctx was rounded when it was stored, which would enter every score gradient of
// a row of few keys as far as their own rounding.  A span of up to 64 keys keeps P and dP for what follows
// (backward, us, and with the stored ctx: 256 x 16 heads of 128, 4 tokens 188 / 186; 8 heads of 256 over 4, 500 tokens 2765 / 2637).
template <typename T>
__global__ __launch_bounds__(64) void plain_dq_kernel(MaskedArgs a) {
  __shared__ float q_s[PLAIN_HEAD], do_s[PLAIN_HEAD];
  constexpr bool STORED = sizeof(T) == 4;
  const int lane = threadIdx.x, i = blockIdx.x, head = blockIdx.y % a.N_heads, b = blockIdx.y / a.N_heads, d = a.S_head;
  const int kv = head / (a.N_heads / a.N_kv);
  const size_t row = (size_t)b * a.S_seq + i, st = ((size_t)b * a.N_heads + head) * a.S_seq + i;
  const T* q = (const T*)a.q + row * a.ldq + (size_t)head * d;
  const T* dc = (const T*)a.dctx + row * a.ldo + (size_t)head * d;
  const T* ctx = (const T*)a.ctx + row * a.ldo + (size_t)head * d;
  float dl = 0.f;
  for (int c = lane; c < d; c += 64) {
    q_s[c] = (float)q[c];
    do_s[c] = (float)dc[c];
    if (STORED) dl = fmaf((float)dc[c], (float)ctx[c], dl);
  }
  __syncthreads();
  const int2 sp = a.span[row];
  const int lo = max(sp.x, 0), hi = min(sp.y, a.S_seq);
  const float slope = a.slope ? a.slope[head] : 0.f, lse = lse_of(a.lse[st]);
  float p = 0.f, dp = 0.f, slack = 0.f;
  auto key = [&](int j) {
    p = dp = 0.f;
    if (j >= hi) return;
    const size_t at = (size_t)b * a.S_seq + j;
    p = expf(score_of(dot_row(q_s, (const T*)a.k + at * a.ldk + (size_t)kv * d, d), a, slope, i, j, slack) - lse);
    dp = dot_row(do_s, (const T*)a.v + at * a.ldv + (size_t)kv * d, d);
  };
  if (!STORED)
    for (int j0 = lo; j0 < hi; j0 += 64) {
      key(j0 + lane);
      dl = fmaf(p, dp, dl);
    }
  dl = wave_sum(dl);
  if (lane == 0) a.delta[st] = dl;
  float o[PER];
  for (int c = 0; c < PER; ++c) o[c] = 0.f;
  for (int j0 = lo; j0 < hi && hi - lo > 1; j0 += 64) {
    if (STORED || hi - lo > 64) key(j0 + lane);
    const float ds = j0 + lane < hi ? p * (dp - dl) * slack : 0.f;
    for (int k = 0; k < 64 && j0 + k < hi; ++k) {
      const float dk = __shfl(ds, k, 64);
      const T* kr = (const T*)a.k + ((size_t)b * a.S_seq + j0 + k) * a.ldk + (size_t)kv * d;
      for (int c = 0; c * 64 + lane < d; ++c) o[c] = fmaf(dk, (float)kr[c * 64 + lane], o[c]);
    }
  }
  T* out = (T*)a.dq + row * a.ldq + (size_t)head * d;
  for (int c = 0; c * 64 + lane < d; ++c) out[c * 64 + lane] = (T)(o[c] * a.scale);
}

template <typename T>
__global__ __launch_bounds__(64) void plain_dkv_kernel(MaskedArgs a) {
  __shared__ float k_s[PLAIN_HEAD], v_s[PLAIN_HEAD];
  const int lane = threadIdx.x, j = blockIdx.x, kv = blockIdx.y % a.N_kv, b = blockIdx.y / a.N_kv, d = a.S_head, group = a.N_heads / a.N_kv;
  const size_t key = (size_t)b * a.S_seq + j;
  const T* k = (const T*)a.k + key * a.ldk + (size_t)kv * d;
  const T* v = (const T*)a.v + key * a.ldv + (size_t)kv * d;
  for (int c = lane; c < d; c += 64) {
    k_s[c] = (float)k[c];
    v_s[c] = (float)v[c];
  }
  __syncthreads();
  float dk[PER], dv[PER];
  for (int c = 0; c < PER; ++c) dk[c] = dv[c] = 0.f;
  const int blocks = (a.S_seq + SPAN_ROWS - 1) / SPAN_ROWS;
  for (int g = 0; g < group; ++g) {
    const int head = kv * group + g;
    const float slope = a.slope ? a.slope[head] : 0.f;
    const size_t st = ((size_t)b * a.N_heads + head) * a.S_seq;
    for (int t = 0; t < blocks; ++t) {
      const SpanBlock x = a.block[(size_t)b * blocks + t];
      if (j < x.lo_min || j >= x.hi_max) continue;
      const int i = t * SPAN_ROWS + lane;
      float p = 0.f, ds = 0.f;
      bool in = false;
      if (i < a.S_seq) {
        const int2 sp = a.span[(size_t)b * a.S_seq + i];
        in = j >= sp.x && j < sp.y;
        if (in) {
          const size_t row = (size_t)b * a.S_seq + i;
          float slack;
          const float s = score_of(dot_row(k_s, (const T*)a.q + row * a.ldq + (size_t)head * d, d), a, slope, i, j, slack);
          p = expf(s - lse_of(a.lse[st + i]));
          if (sp.y - sp.x > 1) ds = p * (dot_row(v_s, (const T*)a.dctx + row * a.ldo + (size_t)head * d, d) - a.delta[st + i]) * slack;
        }
      }
      const unsigned long long who = __ballot(in);
      for (int r = 0; r < SPAN_ROWS; ++r) {
        if (!(who >> r & 1)) continue;
        const float pr = __shfl(p, r, 64), dr = __shfl(ds, r, 64);
        const size_t row = (size_t)b * a.S_seq + t * SPAN_ROWS + r;
        const T* qr = (const T*)a.q + row * a.ldq + (size_t)head * d;
        const T* dr_ = (const T*)a.dctx + row * a.ldo + (size_t)head * d;
        for (int c = 0; c * 64 + lane < d; ++c) {
          dk[c] = fmaf(dr, (float)qr[c * 64 + lane], dk[c]);
          dv[c] = fmaf(pr, (float)dr_[c * 64 + lane], dv[c]);
        }
      }
    }
  }
  T* ok = (T*)a.dk + key * a.ldk + (size_t)kv * d;
  T* ov = (T*)a.dv + key * a.ldv + (size_t)kv * d;
  for (int c = 0; c * 64 + lane < d; ++c) {
    ok[c * 64 + lane] = (T)(dk[c] * a.scale);
    ov[c * 64 + lane] = (T)dv[c];
  }
}

bool cfg_ok(const char* who, const bf_attn_config* c) {
  if (!c) { set_error("%s: the configuration is null", who); return false; }
  if ((c->dtype != BF_FP32 && c->dtype != BF_BF16) || (c->kernels != BF_KERNELS_AUTO && c->kernels != BF_KERNELS_PLAIN)) {
    set_error("%s: unknown dtype %d or kernels %d", who, c->dtype, c->kernels);
    return false;
  }
  if (c->S_mb < 1 || c->S_seq < 1 || c->N_heads < 1 || c->N_kv_heads < 1 || c->N_heads % c->N_kv_heads || c->S_head < 1 || c->S_head > PLAIN_HEAD ||
      c->S_seq > (1 << 24) || (long long)c->S_mb * c->N_heads > 65535 || (long long)c->S_mb * c->S_seq > (1ll << 31)) {
    set_error("%s: bad sizes (S_mb %d, S_seq %d, %d heads over %d key / value heads of %d)", who, c->S_mb, c->S_seq, c->N_heads, c->N_kv_heads, c->S_head);
    return false;
  }
  const int64_t rq = (int64_t)c->N_heads * c->S_head, rk = (int64_t)c->N_kv_heads * c->S_head;
  if ((c->ld_q && c->ld_q < rq) || (c->ld_k && c->ld_k < rk) || (c->ld_v && c->ld_v < rk) || (c->ld_ctx && c->ld_ctx < rq)) {
    set_error("%s: a token's row is longer than the step to the next", who);
    return false;
  }
  // (the scale enters exponents of two: times log2(e), and the cap's tanh twice that, it has to be a finite fp32 number)
  if (!(c->scale >= 0.f && c->scale <= 0x1p126f) || !(c->cap >= 0.f && c->cap <= FLT_MAX)) {
    set_error("%s: scale must be 0 to 2^126, cap finite and not negative", who);
    return false;
  }
  return true;
}

MaskedArgs args_of(const bf_attn_config& c, const void* q, const void* k, const void* v, const int32_t* spans, const float* slopes, const void* ctx, float* lse) {
  MaskedArgs a{};
  a.S_mb = c.S_mb; a.S_seq = c.S_seq; a.N_heads = c.N_heads; a.N_kv = c.N_kv_heads; a.S_head = c.S_head;
  a.scale = c.scale > 0.f ? c.scale : 1.0f / sqrtf((float)c.S_head);
  a.cap = c.cap;
  const size_t rq = (size_t)c.N_heads * c.S_head, rk = (size_t)c.N_kv_heads * c.S_head;
  a.ldq = c.ld_q ? c.ld_q : rq; a.ldk = c.ld_k ? c.ld_k : rk; a.ldv = c.ld_v ? c.ld_v : rk; a.ldo = c.ld_ctx ? c.ld_ctx : rq;
  a.q = q; a.k = k; a.v = v;
  a.span = (const int2*)spans;
  a.block = (const SpanBlock*)(spans + up4((size_t)c.S_mb * c.S_seq * 2));
  a.slope = slopes;
  a.ctx = (void*)ctx;
  a.lse = lse;
  return a;
}

// rows of whole 16-byte chunks that start at multiples of 4 bytes, in every tensor
bool chunks(const bf_attn_config& c, const MaskedArgs& a, uintptr_t al) {
  if (c.dtype == BF_FP32) return a.S_head % 4 == 0;
  return (al & 3) == 0 && a.S_head % 8 == 0 && ((a.ldq | a.ldk | a.ldv | a.ldo) & 1) == 0;
}

// The matrix-core kernels: heads up to 128, and 32-bit offsets into a tile of 64 rows.  Not up to four tokens without shared heads, where
// the plain kernels are faster (forward and backward in bf16, heads of 128, us: 4 x 16 of 4 tokens 35 against 40, 256 x 16 214 against
// 299; of 8 39 against 39 and 491 against 307) and keep dS, which sums of one or two terms would round in full view, in fp32.
bool matrix(const bf_attn_config& c) {
  const int64_t far = 1 << 22;
  if (c.S_seq <= 4 && c.N_heads == c.N_kv_heads) return false;
  return c.kernels == BF_KERNELS_AUTO && c.S_head <= 128 && c.ld_q <= far && c.ld_k <= far && c.ld_v <= far && c.ld_ctx <= far &&
         (int64_t)c.N_heads * c.S_head <= far;
}

// A launch has fewer than 2^32 threads along its grid: 256 to 128 queries of a head, 512 to 128 keys (no more of those workgroups than of
// the queries').
bool launches_fit(const char* who, const bf_attn_config& c, bool backward) {
  const long long wgs = (long long)((c.S_seq + 127) / 128) * c.S_mb * c.N_heads;
  if (!matrix(c) || wgs < (backward ? 1 << 23 : 1 << 24)) return true;
  set_error("%s: %d x %d tokens of %d heads are more than a launch holds", who, c.S_mb, c.S_seq, c.N_heads);
  return false;
}

// Shares of a key / value head's query heads in the dK / dV pass
int splits_of(const bf_attn_config& c) {
  if (!matrix(c)) return 1;
  const int group = c.N_heads / c.N_kv_heads;
  const long wgs = (long)((c.S_seq + 127) / 128) * c.N_kv_heads * c.S_mb;
  int s = 1;
  for (int k = 2; k <= group; ++k)
    if (group % k == 0 && wgs * s < 1024) s = k;
  return s;
}

bool element_aligned(int dtype, uintptr_t p) { return (p & (dtype == BF_BF16 ? 1 : 3)) == 0; }

bool word_aligned(uintptr_t p) { return (p & 3) == 0; }

}  // namespace

size_t attention_spans_elems(int S_mb, int S_seq) {
  if (S_mb < 1 || S_seq < 1 || S_seq > (1 << 24) || (long long)S_mb * S_seq > (1ll << 31)) return 0;
  return up4((size_t)S_mb * S_seq * 2) + (size_t)S_mb * span_blocks(S_seq) * 4;
}

bf_status attention_spans(int S_mb, int S_seq, int causal, const int32_t* doc, const int32_t* prefix, int32_t* spans, hipStream_t st) {
  if (!attention_spans_elems(S_mb, S_seq) || S_mb > 65535) { set_error("bf_op_attention_spans: bad sizes"); return BF_EINVAL; }
  if (!spans || ((uintptr_t)spans & 15)) { set_error("bf_op_attention_spans: spans is null or not 16-byte aligned"); return BF_EINVAL; }
  if (!word_aligned((uintptr_t)doc | (uintptr_t)prefix)) { set_error("bf_op_attention_spans: doc or prefix is not aligned to its elements"); return BF_EINVAL; }
  spans_kernel<<<dim3((S_seq + TOKENS - 1) / TOKENS, S_mb), TOKENS, 0, st>>>(S_seq, causal != 0, doc, prefix, (int2*)spans,
                                                                            (SpanBlock*)(spans + up4((size_t)S_mb * S_seq * 2)), (int)span_blocks(S_seq));
  return launched();
}

bf_status attention_masked_fwd(const bf_attn_config* c, const void* q, const void* k, const void* v, const int32_t* spans, const float* slopes, void* ctx,
                               float* lse, hipStream_t st) {
  const char* who = "bf_op_attention_masked_fwd";
  if (!cfg_ok(who, c) || !launches_fit(who, *c, false)) return BF_EINVAL;
  if (!q || !k || !v || !spans || !ctx) { set_error("%s: null pointer", who); return BF_EINVAL; }
  if (!element_aligned(c->dtype, (uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)ctx) || ((uintptr_t)spans & 15) ||
      !word_aligned((uintptr_t)slopes | (uintptr_t)lse)) {
    set_error("%s: a tensor is not aligned to its elements, or spans not to 16 bytes", who);
    return BF_EINVAL;
  }
  MaskedArgs a = args_of(*c, q, k, v, spans, slopes, ctx, lse);
  a.vec = chunks(*c, a, (uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)ctx);
  if (matrix(*c)) return c->dtype == BF_BF16 ? attention_masked_fwd_mfma(a, st) : attention_masked_fwd_f32(a, st);
  const dim3 grid(c->S_seq, c->S_mb * c->N_heads);
  if (c->dtype == BF_BF16) plain_fwd_kernel<bf16_t><<<grid, 64, 0, st>>>(a);
  else plain_fwd_kernel<float><<<grid, 64, 0, st>>>(a);
  return launched();
}

size_t attention_masked_bwd_work_bytes(const bf_attn_config* c) {
  const char* who = "bf_op_attention_masked_bwd_work_bytes";
  if (!cfg_ok(who, c) || !launches_fit(who, *c, true)) return 0;
  const size_t delta = ((size_t)c->S_mb * c->N_heads * c->S_seq * 4 + 255) / 256 * 256;
  const int splits = splits_of(*c);
  return delta + (splits > 1 ? (size_t)splits * 2 * c->S_mb * c->S_seq * c->N_kv_heads * c->S_head * 4 : 0);
}

bf_status attention_masked_bwd(const bf_attn_config* c, const void* q, const void* k, const void* v, const int32_t* spans, const float* slopes, const void* ctx,
                               const float* lse, const void* dctx, void* dq, void* dk, void* dv, void* work, size_t work_bytes, hipStream_t st) {
  const char* who = "bf_op_attention_masked_bwd";
  if (!cfg_ok(who, c) || !launches_fit(who, *c, true)) return BF_EINVAL;
  if (!q || !k || !v || !spans || !ctx || !lse || !dctx || !dq || !dk || !dv) { set_error("%s: null pointer", who); return BF_EINVAL; }
  const uintptr_t al = (uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)ctx | (uintptr_t)dctx | (uintptr_t)dq | (uintptr_t)dk | (uintptr_t)dv;
  if (!element_aligned(c->dtype, al) || ((uintptr_t)spans & 15) || !word_aligned((uintptr_t)slopes | (uintptr_t)lse)) {
    set_error("%s: a tensor is not aligned to its elements, or spans not to 16 bytes", who);
    return BF_EINVAL;
  }
  const size_t need = attention_masked_bwd_work_bytes(c);
  if (!work || ((uintptr_t)work & 255) || work_bytes < need) { set_error("%s: needs %zu bytes of 256-byte aligned scratch", who, need); return BF_EINVAL; }
  MaskedArgs a = args_of(*c, q, k, v, spans, slopes, ctx, (float*)lse);
  a.dctx = dctx;
  a.dq = dq; a.dk = dk; a.dv = dv;
  a.delta = (float*)work;
  a.splits = splits_of(*c);
  a.planes = (float*)((char*)work + ((size_t)c->S_mb * c->N_heads * c->S_seq * 4 + 255) / 256 * 256);
  a.vec = chunks(*c, a, al);
  if (matrix(*c)) return c->dtype == BF_BF16 ? attention_masked_bwd_mfma(a, st) : attention_masked_bwd_f32(a, st);
  const dim3 grid(c->S_seq, c->S_mb * c->N_heads), grid_kv(c->S_seq, c->S_mb * c->N_kv_heads);
  if (c->dtype == BF_BF16) {
    plain_dq_kernel<bf16_t><<<grid, 64, 0, st>>>(a);
    plain_dkv_kernel<bf16_t><<<grid_kv, 64, 0, st>>>(a);
  } else {
    plain_dq_kernel<float><<<grid, 64, 0, st>>>(a);
    plain_dkv_kernel<float><<<grid_kv, 64, 0, st>>>(a);
  }
  return launched();
}

}  // namespace bf
