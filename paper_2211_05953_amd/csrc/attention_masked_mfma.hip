// Masked attention on the bf16 matrix cores, heads up to 128 (padded with zeros to 64 or 128 in LDS and registers).
//
// Layouts, LDS swizzle and the transposed score tiles are those of attention_mfma.hip: a lane owns one softmax row of a
// forward or dQ tile and one key of a dK / dV tile, and its score registers are, rounded, the next product's operand.  What the
// masks add: a workgroup walks only the tiles that its rows' spans reach; a wave skips a tile that none of its 32 rows sees
// and applies no mask to one that all of them see whole; the others are masked by selection, after the score and before
// anything is summed.  A tile that is masked in part and holds an infinity or a NaN takes a product for every column, over
// the rows that the column sees (zero times infinity is a NaN in a matrix instruction).
#include <float.h>
#include <math.h>

#include <type_traits>
#include <utility>

#include "attention_masked.h"
#include "attention_tiles.h"

namespace bf {

namespace {

template <typename F, int... I>
__device__ __forceinline__ void static_for_(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) { static_for_(f, std::make_integer_sequence<int, N>{}); }

// ---- loads and stores of token rows, shorter than D or not.  Through buffer descriptors that end where the rows do: a lane keeps one
// 32-bit offset, and what lies past the end, or past a short row, reads as zeros and is not written.  No branches: short
// launches wait for their instructions, about 1 us for 600 bytes that run once.
// VEC: rows of whole 16-byte chunks that start at multiples of 4 bytes; else element by element.
constexpr uint32_t NOWHERE = 0x7fffff00u;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const void* g, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)g, 0, (int)bytes, 0x00020000);
}

// eight elements at byte offset `off`, `left` of them inside the row (VEC: all or none)
template <bool VEC>
__device__ __forceinline__ u32x4 load_chunk(__amdgpu_buffer_rsrc_t rsrc, uint32_t off, int left) {
  if (VEC) return __builtin_amdgcn_raw_buffer_load_b128(rsrc, off, 0, 0);
  u32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t lo = __builtin_amdgcn_raw_buffer_load_b16(rsrc, 2 * e < left ? off + 4 * e : NOWHERE, 0, 0);
    const uint32_t hi = __builtin_amdgcn_raw_buffer_load_b16(rsrc, 2 * e + 1 < left ? off + 4 * e + 2 : NOWHERE, 0, 0);
    v[e] = lo | hi << 16;
  }
  return v;
}

template <int ROWS, int D, int NT, bool VEC>
struct Tile : TileRegs<ROWS, D, NT> {
  static constexpr int CH = TileRegs<ROWS, D, NT>::CH, STEP = NT / (D / 8);  // rows between a thread's chunks
  uint32_t off;
  int left;
  __device__ __forceinline__ void init(size_t ld, int tid, int d) {
    const int col = tid % (D / 8) * 8;
    left = d - col;
    off = VEC && left <= 0 ? NOWHERE : (uint32_t)(tid / (D / 8) * ld + col) * 2;
  }
  // g: the tile's first row, `valid` >= 1 of which are there (uniform)
  __device__ __forceinline__ void fetch(const bf16_t* __restrict__ g, size_t ld, int valid, int d) {
    const auto rsrc = rows_at(g, (uint32_t)(((valid < ROWS ? valid : ROWS) - 1) * ld + d) * 2);
    const uint32_t step = (uint32_t)(STEP * ld * 2);
#pragma unroll
    for (int i = 0; i < CH; ++i) this->v[i] = load_chunk<VEC>(rsrc, off + i * step, left);
  }
};

// rows: the workgroup's first row and its bytes from there (uniform); off: the lane's row
template <int D, bool VEC>
__device__ __forceinline__ void load_row(__amdgpu_buffer_rsrc_t rows, uint32_t off, int lane, int d, bf16x8 (&f)[D / 16]) {
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    const int c = kk * 16 + 8 * (lane >> 5);
    f[kk] = __builtin_bit_cast(bf16x8, load_chunk<VEC>(rows, !VEC || c < d ? off + 2 * c : NOWHERE, d - c));
  }
}

template <int D, bool VEC>
__device__ __forceinline__ void store_row(const f32x16 (&acc)[D / 32], __amdgpu_buffer_rsrc_t rows, uint32_t off, int lane, float mul, int d) {
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const int c = dt * 32 + q4 * 8 + (lane >> 5) * 4;
      bf16x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (__bf16)(acc[dt][q4 * 4 + e] * mul);
      typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2;
      const u32x2 u = __builtin_bit_cast(u32x2, o);
      if (VEC) {
        __builtin_amdgcn_raw_buffer_store_b64(u, rows, c < d ? off + 2 * c : NOWHERE, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          __builtin_amdgcn_raw_buffer_store_b16((short)(u[e >> 1] >> 16 * (e & 1)), rows, c + e < d ? off + 2 * (c + e) : NOWHERE, 0, 0);
      }
    }
}

// bytes of up to n rows, those that are there of them
__device__ __forceinline__ uint32_t row_bytes(int n, int there, size_t ld, int d) { return (uint32_t)(((there < n ? there : n) - 1) * ld + d) * 2; }

// ---- from a dot product to an exponent of two.  Without cap and bias the dot products stay as they are and the factor enters with
// the exponential (one fma).  CAP 1: tanh x = 1 - 2 r with r = 1 / (1 + e^2x), on the hardware exponential and reciprocal (1 ulp
// each); its derivative 1 - tanh^2 is 4 r (1 - r).  That is off by 1.2e-7 of the cap, not of the score: caps past 2^10, where it
// would show beside P's rounding (cap 1e4: 1.2e-3 of a probability, 1e6: a tenth), take CAP 2, a tanh as exact for small scores as for large
// (8192 tokens, 16 heads of 128 over 4, forward and backward, us: 405 + 1868 and 538 + 2851).  So do caps so small that e2x is no fp32 number.
struct ScoreFactors {
  float c2;      // factor of an exponent: 1 where the score carries it already
  float e2x;     // dot product to 2 x log2(e), x the tanh's argument
  float capl;    // cap log2(e)
  float mul;     // dot product to score (bias without cap)
  float slopel;  // slope log2(e)
  float scale, cap, inv_cap;  // CAP 2
};

constexpr float CAP_FAST = 1024.f;

template <int CAP, bool BIAS>
__device__ __forceinline__ ScoreFactors factors(const MaskedArgs& a, int head) {
  ScoreFactors f;
  f.c2 = CAP || BIAS ? 1.f : a.scale * LOG2E;
  f.mul = a.scale * LOG2E;
  f.capl = a.cap * LOG2E;
  f.e2x = CAP ? 2.f * LOG2E * a.scale / a.cap : 0.f;
  f.scale = a.scale;
  f.cap = a.cap;
  f.inv_cap = CAP == 2 ? inverse_cap(a.cap) : 0.f;
  f.slopel = BIAS && (CAP != 2 || a.slope) ? a.slope[head] * LOG2E : 0.f;  // (CAP 2 has no form without the bias)
  return f;
}

// dist: i - j as a float.  r: what slack_of takes (CAP)
template <int CAP, bool BIAS>
__device__ __forceinline__ float exponent(float dot, float dist, const ScoreFactors& f, float& r) {
  float t = dot;
  if (CAP == 1) {
    r = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(dot * f.e2x));
    t = fmaf(r, -2.f * f.capl, f.capl);
  } else if (CAP == 2) {
    r = tanh_f(dot * f.scale * f.inv_cap);
    t = f.cap * r * LOG2E;
  } else if (BIAS) {
    t *= f.mul;
  }
  if (BIAS) t = fmaf(-f.slopel, fabsf(dist), t);
  return t;
}

// the cap's derivative
template <int CAP>
__device__ __forceinline__ float slack_of(float r) { return CAP == 1 ? 4.f * r * (1.f - r) : fmaf(-r, r, 1.f); }

// acc += tile^T p over a tile that is masked in part and holds an infinity or a NaN: column by column of p, with the tile's
// rows that the column does not see taken as zeros.  rows_of(c): bit r is set where column c sees row r of the tile (uniform).
template <int D, typename FA, typename F>
__device__ __forceinline__ void accumulate_seen(f32x16 (&acc)[D / 32], const bf16x8 (&p)[4], int row0, int subs, const bf16_t* tile, const FA& fa, int lane,
                                                F rows_of) {
#pragma unroll 1
  for (int c = 0; c < 32; ++c) {
    const uint64_t seen = rows_of(c);
    if (seen == 0) continue;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
      f32x16 sum = zero16();
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (k >= subs) continue;
        bf16x8 v = fa.frag_t(tile, row0 + 16 * k, dt);
        const uint32_t bits = (uint32_t)(seen >> (row0 + 16 * k + 4 * (lane >> 5)));  // rows 8 (e / 4) + e % 4 from there on
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = bits >> (8 * (e >> 2) + (e & 3)) & 1 ? v[e] : (bf16_t)0.f;
        sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[k], sum, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[dt][r] = (lane & 31) == c ? acc[dt][r] + sum[r] : acc[dt][r];
    }
  }
}

// the rows of a tile at k0 that lie in [lo, hi)
__device__ __forceinline__ uint64_t interval_bits(int k0, int lo, int hi) {
  const int a = min(max(lo - k0, 0), 64), b = min(max(hi - k0, 0), 64);
  if (a >= b) return 0;
  return (~0ull >> (64 - (b - a))) << a;
}

// a wave's spans: which tiles it needs, and which of them whole.  Rows past the end count as neither.
struct WaveSpan {
  int lo_min, hi_max, lo_max, hi_min;
  __device__ __forceinline__ void init(int2 sp, bool row) {
    const bool any = sp.y > sp.x;
    lo_min = row && any ? sp.x : INT_MAX;
    hi_max = row && any ? sp.y : 0;
    lo_max = !row ? 0 : any ? sp.x : INT_MAX;
    hi_min = !row ? INT_MAX : any ? sp.y : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {  // lanes l and l + 32 hold the same row
      lo_min = min(lo_min, __shfl_xor(lo_min, o, 64));
      hi_max = max(hi_max, __shfl_xor(hi_max, o, 64));
      lo_max = max(lo_max, __shfl_xor(lo_max, o, 64));
      hi_min = min(hi_min, __shfl_xor(hi_min, o, 64));
    }
    lo_min = __builtin_amdgcn_readfirstlane(lo_min);
    hi_max = __builtin_amdgcn_readfirstlane(hi_max);
    lo_max = __builtin_amdgcn_readfirstlane(lo_max);
    hi_min = __builtin_amdgcn_readfirstlane(hi_min);
  }
  __device__ __forceinline__ bool skips(int k, int n) const { return k >= hi_max || k + n <= lo_min; }
  __device__ __forceinline__ bool whole(int k, int n) const { return k >= lo_max && k + n <= hi_min; }
};

// of the query block's rows together
template <int ROWS>
__device__ __forceinline__ SpanBlock rows_of_block(const MaskedArgs& a, int b, int q0) {
  const int blocks = (a.S_seq + SPAN_ROWS - 1) / SPAN_ROWS, at = q0 / SPAN_ROWS;
  SpanBlock x = a.block[(size_t)b * blocks + at];
#pragma unroll
  for (int k = 1; k < ROWS / SPAN_ROWS; ++k)
    if (at + k < blocks) {
      const SpanBlock y = a.block[(size_t)b * blocks + at + k];
      x = {min(x.lo_min, y.lo_min), max(x.hi_max, y.hi_max), max(x.lo_max, y.lo_max), min(x.hi_min, y.hi_min)};
    }
  x.hi_max = min(x.hi_max, a.S_seq);
  return x;
}

// query block, head and sequence of a workgroup of a 1-D grid: the last query blocks first (under a causal mask the longest), and
// neighbouring workgroups on different key / value heads, so that the query heads of one of them meet in one XCD's L2
struct QueryBlock { int q0, head, kv, b; };
__device__ __forceinline__ QueryBlock query_block(const MaskedArgs& a, int idx, int rows) {
  const int nhb = a.N_heads * a.S_mb, blocks = (a.S_seq + rows - 1) / rows, group = a.N_heads / a.N_kv;
  const int x = idx % nhb, hx = x % a.N_heads;
  QueryBlock w;
  w.q0 = (blocks - 1 - idx / nhb) * rows;
  w.b = x / a.N_heads;
  w.kv = hx % a.N_kv;
  w.head = w.kv * group + hx / a.N_kv;
  return w;
}

// ------------------------------------------------------------------------------ forward
// SEEN: tiles that are masked in part by accumulate_seen.  Without it, returns whether one of those held a non-finite V.
// 64 heads of 128, 2048 tokens, causal: 113 us, 0.61 PFLOP/s of the unmasked half's products, matrix cores busy 20 % of the time: bound by each
// wave's chain of product, exponential, product, two workgroups of four waves to a compute unit.
template <int D, int ROWS, bool VEC, int CAP, bool BIAS, bool SEEN>
__device__ __forceinline__ bool fwd_rows(const MaskedArgs& a, bf16_t (&KVs)[2][2][BLK * D]) {
  constexpr int NT = 2 * ROWS;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const QueryBlock wb = query_block(a, blockIdx.x, ROWS);
  const int S = a.S_seq, d = a.S_head, q = wb.q0 + 32 * w + (lane & 31), ql = min(q, S - 1);
  const size_t seq = (size_t)wb.b * S;
  const bf16_t* kbase = (const bf16_t*)a.k + seq * a.ldk + (size_t)wb.kv * d;
  const bf16_t* vbase = (const bf16_t*)a.v + seq * a.ldv + (size_t)wb.kv * d;
  // (S_head 128: precomputed offsets would spill)
  typename std::conditional<D == 64, FragAddr<D>, FragAddrXor<D>>::type fa;
  fa.init(lane);
  bf16x8 qf[D / 16];
  // (rows past the end read zeros)
  const int r0 = 32 * w + (lane & 31);
  load_row<D, VEC>(rows_at((const bf16_t*)a.q + (seq + wb.q0) * a.ldq + (size_t)wb.head * d, row_bytes(ROWS, S - wb.q0, a.ldq, d)), (uint32_t)(r0 * a.ldq) * 2, lane,
                   d, qf);
  int2 sp = a.span[seq + ql];
  sp.x = max(sp.x, 0);
  sp.y = min(sp.y, S);
  WaveSpan ws;
  ws.init(sp, q < S);
  const SpanBlock wg = rows_of_block<ROWS>(a, wb.b, wb.q0);
  const ScoreFactors f = factors<CAP, BIAS>(a, wb.head);
  f32x16 o[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) o[dt] = zero16();
  // (a maximum of the lowest finite value, that its factor leaves finite: a row that has met only -inf adds exactly 0, no NaN)
  float m = f.c2 > 1.f ? -FLT_MAX / f.c2 : -FLT_MAX, l = 0.f;

  const int jbeg = wg.hi_max > 0 ? max(wg.lo_min, 0) / BLK : 0, jend = (wg.hi_max + BLK - 1) / BLK;
  Tile<BLK, D, NT, VEC> kr, vr;
  bool bad = false;
  kr.init(a.ldk, tid, d);
  vr.init(a.ldv, tid, d);
  // the next tile's K is on its way during the first half of a tile's work, its V during the second, in the same registers
  auto fetch_k = [&](int j) { kr.fetch(kbase + (size_t)j * BLK * a.ldk, a.ldk, S - j * BLK, d); };
  auto fetch_v = [&](int j) { vr.fetch(vbase + (size_t)j * BLK * a.ldv, a.ldv, S - j * BLK, d); };
  auto note = [&](int j) {
    const int kb = j * BLK;
    if (!SEEN && !(kb >= wg.lo_max && kb + BLK <= wg.hi_min)) bad |= vr.non_finite();
  };
  typedef std::integral_constant<int, 0> I0;
  typedef std::integral_constant<int, 1> I1;
  if (jbeg < jend) {
    fetch_k(jbeg);
    fetch_v(jbeg);
    kr.store(KVs[0][0], tid);
    vr.store(KVs[0][1], tid);
    note(jbeg);
  }
  __syncthreads();
  // one key tile; PAR, its LDS stage, is a compile-time constant (the loop is unrolled by two)
  auto body = [&](int j, auto parc) {
    constexpr int PAR = decltype(parc)::value;
    if constexpr (D == 128) fa.loop();
    const bf16_t* Ks = KVs[PAR][0];
    const bf16_t* Vs = KVs[PAR][1];
    const int kb = j * BLK;
    const bool next = j + 1 < jend, work = !ws.skips(kb, BLK), part = !ws.whole(kb, BLK);
    if (next) fetch_k(j + 1);
    f32x16 s[2] = {zero16(), zero16()};
    if (work) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa.frag_k(Ks, 32 * t, kk), qf[kk], s[t], 0, 0, 0);
    mfma_lds_pipeline<2 * (D / 16), 1, 4>();
    if (CAP || BIAS) {
      const float dist = (float)(q - kb - 4 * (lane >> 5));
      float r_;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = exponent<CAP, BIAS>(s[t][r], dist - (float)(32 * t + (r >> 2) * 8 + (r & 3)), f, r_);
    }
    if (part) {
      const int lo = sp.x - kb, n = sp.y - sp.x;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if ((unsigned)(32 * t + acc_row(r, lane) - lo) >= (unsigned)n) s[t][r] = -INFINITY;
    }
    float mx = m;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[t][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float nmx = -mx * f.c2;
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(CAP || BIAS ? s[t][r] + nmx : fmaf(s[t][r], f.c2, nmx));
        s[t][r] = p;
        sum += p;
      }
    if (__builtin_amdgcn_ballot_w64(mx > m) != 0) {  // some row's maximum moved
      const float alpha = __builtin_amdgcn_exp2f(CAP || BIAS ? m + nmx : fmaf(m, f.c2, nmx));
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
      m = mx;
    }
    l += sum;
    }
    bf16x8 pb[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) pb[k] = pack8(s[k >> 1], k & 1);
    if (next) {
      kr.store(KVs[PAR ^ 1][0], tid);
      fetch_v(j + 1);
    }
    if (work) {
      if (SEEN && part) {
        accumulate_seen<D>(o, pb, 0, 4, Vs, fa, lane, [&](int c) {
          return interval_bits(kb, __builtin_amdgcn_readlane(sp.x, c), __builtin_amdgcn_readlane(sp.y, c));
        });
      } else {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int dt = 0; dt < D / 32; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa.frag_t(Vs, 16 * k, dt), pb[k], o[dt], 0, 0, 0);
        mfma_lds_pipeline<4 * (D / 32), 2, 4>();
      }
    }
    if (next) {
      vr.store(KVs[PAR ^ 1][1], tid);
      note(j + 1);
    }
    __syncthreads();
  };
  for (int j = jbeg; j < jend; j += 2) {
    body(j, I0{});
    if (j + 1 < jend) body(j + 1, I1{});
  }
  if (!SEEN && __syncthreads_or(bad)) return true;
  l += __shfl_xor(l, 32, 64);
  store_row<D, VEC>(o, rows_at((bf16_t*)a.ctx + (seq + wb.q0) * a.ldo + (size_t)wb.head * d, row_bytes(ROWS, S - wb.q0, a.ldo, d)), (uint32_t)(r0 * a.ldo) * 2, lane,
                    l == 0.f ? 0.f : 1.0f / l, d);
  if (lane < 32 && q < S && a.lse)
    a.lse[((size_t)wb.b * a.N_heads + wb.head) * S + q] = l == 0.f ? -INFINITY : m * (CAP || BIAS ? LN2 : a.scale) + logf(l);
  return false;
}

// The second way is a pass of its own, and a function: in the first one's loop, or behind it in the same body, what it needs
// pushes the first one's registers out.
template <int D, int ROWS, bool VEC, int CAP, bool BIAS>
__device__ __attribute__((noinline)) void fwd_rows_seen(MaskedArgs a, bf16_t (&KVs)[2][2][BLK * D]) {
  fwd_rows<D, ROWS, VEC, CAP, BIAS, true>(a, KVs);
}

template <int D, int ROWS, bool VEC, int CAP, bool BIAS>
__global__ __launch_bounds__(2 * ROWS, 2) void masked_fwd_kernel(MaskedArgs a) {
  __shared__ __attribute__((aligned(16))) bf16_t KVs[2][2][BLK * D];
  if (fwd_rows<D, ROWS, VEC, CAP, BIAS, false>(a, KVs)) fwd_rows_seen<D, ROWS, VEC, CAP, BIAS>(a, KVs);
}

// ------------------------------------------------------------------- backward, dQ pass
// Walks the keys twice.  First for delta = sum of P dP, in fp32 and kept for the dK / dV pass; then for dS = P (dP - delta) and
// dQ = dS K.  The usual delta = dctx . ctx takes a ctx that was rounded when it was stored, which puts as large an error on every score
// gradient of the row as their own rounding does where few keys share a row (8192 tokens, 16 heads of 128, sharp rows: dQ and dK
// 2.8e-3 off in the 2-norm, 2.3e-3 so, the results' own rounding 1.7e-3); it is two products and no sums, against three and their sums, 35 % of the pass.
// 64 heads of 128, 2048 tokens, causal: 209 us, matrix cores busy 41 %; 0.82 PFLOP/s with the first walk's products, 0.49 without.
template <int D, int ROWS, bool VEC, int CAP, bool BIAS, bool SEEN>
__device__ __forceinline__ bool dq_rows(const MaskedArgs& a, bf16_t (&KVs)[2][2][BLK * D]) {
  constexpr int NT = 2 * ROWS;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const QueryBlock wb = query_block(a, blockIdx.x, ROWS);
  const int S = a.S_seq, d = a.S_head, q = wb.q0 + 32 * w + (lane & 31), ql = min(q, S - 1);
  const size_t seq = (size_t)wb.b * S;
  const bf16_t* kbase = (const bf16_t*)a.k + seq * a.ldk + (size_t)wb.kv * d;
  const bf16_t* vbase = (const bf16_t*)a.v + seq * a.ldv + (size_t)wb.kv * d;

  // (S_head 128: precomputed offsets would spill)
  typename std::conditional<D == 64, FragAddr<D>, FragAddrXor<D>>::type fa;
  fa.init(lane);
  bf16x8 qf[D / 16], dof[D / 16];
  const int r0 = 32 * w + (lane & 31);
  load_row<D, VEC>(rows_at((const bf16_t*)a.q + (seq + wb.q0) * a.ldq + (size_t)wb.head * d, row_bytes(ROWS, S - wb.q0, a.ldq, d)), (uint32_t)(r0 * a.ldq) * 2, lane,
                   d, qf);
  load_row<D, VEC>(rows_at((const bf16_t*)a.dctx + (seq + wb.q0) * a.ldo + (size_t)wb.head * d, row_bytes(ROWS, S - wb.q0, a.ldo, d)), (uint32_t)(r0 * a.ldo) * 2,
                   lane, d, dof);
  const size_t st = ((size_t)wb.b * a.N_heads + wb.head) * S + ql;
  // (a row without a finite score has no probabilities)
  const float lse = a.lse[st], lse2 = lse == -INFINITY ? INFINITY : lse * LOG2E;
  int2 sp = a.span[seq + ql];
  sp.x = max(sp.x, 0);
  sp.y = min(sp.y, S);
  WaveSpan ws;
  ws.init(sp, q < S);
  const SpanBlock wg = rows_of_block<ROWS>(a, wb.b, wb.q0);
  const ScoreFactors f = factors<CAP, BIAS>(a, wb.head);
  f32x16 dq[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) dq[dt] = zero16();

  const int jbeg = wg.hi_max > 0 ? max(wg.lo_min, 0) / BLK : 0, jend = (wg.hi_max + BLK - 1) / BLK;
  Tile<BLK, D, NT, VEC> kr, vr;
  bool bad = false;
  kr.init(a.ldk, tid, d);
  vr.init(a.ldv, tid, d);
  // the next tile's K is on its way during the first half of a tile's work, its V during the second, in the same registers
  auto fetch_k = [&](int j) { kr.fetch(kbase + (size_t)j * BLK * a.ldk, a.ldk, S - j * BLK, d); };
  auto fetch_v = [&](int j) { vr.fetch(vbase + (size_t)j * BLK * a.ldv, a.ldv, S - j * BLK, d); };
  auto note = [&](int j) {
    const int kb = j * BLK;
    if (!SEEN && !(kb >= wg.lo_max && kb + BLK <= wg.hi_min)) bad |= kr.non_finite();
  };
  float delta = 0.f;
  auto walk = [&](auto second) {
    constexpr bool GRAD = decltype(second)::value;
    if (jbeg < jend) {
      fetch_k(jbeg);
      fetch_v(jbeg);
      kr.store(KVs[0][0], tid);
      vr.store(KVs[0][1], tid);
      if (GRAD) note(jbeg);
    }
    __syncthreads();
    auto body = [&](int j, auto par) {
      const int p = par;
      if constexpr (D == 128) fa.loop();
      const bf16_t* Ks = KVs[p][0];
      const bf16_t* Vs = KVs[p][1];
      const int kb = j * BLK;
      const bool next = j + 1 < jend, work = !ws.skips(kb, BLK), part = !ws.whole(kb, BLK);
      if (next) fetch_k(j + 1);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (t == 1 && next) {
          kr.store(KVs[p ^ 1][0], tid);
          if (GRAD) note(j + 1);
          fetch_v(j + 1);
        }
        if (!work) continue;
        f32x16 s = zero16(), dp = zero16();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa.frag_k(Ks, 32 * t, kk), qf[kk], s, 0, 0, 0);
          dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa.frag_k(Vs, 32 * t, kk), dof[kk], dp, 0, 0, 0);
        }
        mfma_lds_pipeline<2 * (D / 16), 1, 4>();
        // p = exp(score - lse); dS = p (dP - delta) times the cap's derivative (the factor 1/sqrt(d) is applied once, to dQ)
        const float dist = (float)(q - kb - 32 * t - 4 * (lane >> 5));
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float c = 0.f;
          const float e = exponent<CAP, BIAS>(s[r], dist - (float)((r >> 2) * 8 + (r & 3)), f, c);
          const float pr = __builtin_amdgcn_exp2f(CAP || BIAS ? e - lse2 : fmaf(e, f.c2, -lse2));
          if (GRAD) {
            s[r] = pr * (dp[r] - delta);
            if (CAP) s[r] *= slack_of<CAP>(c);
          } else {
            s[r] = pr * dp[r];
          }
        }
        if (part) {
          const int lo = sp.x - kb - 32 * t, n = sp.y - sp.x;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if ((unsigned)(acc_row(r, lane) - lo) >= (unsigned)n) s[r] = 0.f;
        }
        if constexpr (!GRAD) {
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int r = 0; r < 16; ++r) sum[r & 3] += s[r];
          delta += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        } else {
          const bf16x8 dsb[4] = {pack8(s, 0), pack8(s, 1)};
          if (SEEN && part) {
            accumulate_seen<D>(dq, dsb, 32 * t, 2, Ks, fa, lane, [&](int c) {
              return interval_bits(kb, __builtin_amdgcn_readlane(sp.x, c), __builtin_amdgcn_readlane(sp.y, c));
            });
            continue;
          }
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
              dq[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa.frag_t(Ks, 32 * t + 16 * k2, dt), dsb[k2], dq[dt], 0, 0, 0);
          mfma_lds_pipeline<2 * (D / 32), 2, 4>();
        }
      }
      if (next) vr.store(KVs[p ^ 1][1], tid);
      __syncthreads();
    };
    if constexpr (D == 64) {
      // unrolled by two: the LDS stage (and with it every fragment address) is a compile-time constant
      for (int j = jbeg; j < jend; j += 2) {
        body(j, std::integral_constant<int, 0>{});
        if (j + 1 < jend) body(j + 1, std::integral_constant<int, 1>{});
      }
    } else {
      for (int j = jbeg; j < jend; ++j) body(j, (j - jbeg) & 1);
    }
  };
  walk(std::false_type{});
  delta += __shfl_xor(delta, 32, 64);  // lanes l and l + 32 hold the two halves of a row
  if (lane < 32 && q < S) a.delta[st] = delta;
  walk(std::true_type{});
  if (!SEEN && __syncthreads_or(bad)) return true;
  if (sp.y - sp.x <= 1) {  // one key: its probability is 1 whatever the score
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) dq[dt] = zero16();
  }
  store_row<D, VEC>(dq, rows_at((bf16_t*)a.dq + (seq + wb.q0) * a.ldq + (size_t)wb.head * d, row_bytes(ROWS, S - wb.q0, a.ldq, d)), (uint32_t)(r0 * a.ldq) * 2, lane,
                    a.scale, d);
  return false;
}

template <int D, int ROWS, bool VEC, int CAP, bool BIAS>
__device__ __attribute__((noinline)) void dq_rows_seen(MaskedArgs a, bf16_t (&KVs)[2][2][BLK * D]) {
  dq_rows<D, ROWS, VEC, CAP, BIAS, true>(a, KVs);
}

template <int D, int ROWS, bool VEC, int CAP, bool BIAS>
__global__ __launch_bounds__(2 * ROWS, 2) void masked_dq_kernel(MaskedArgs a) {
  __shared__ __attribute__((aligned(16))) bf16_t KVs[2][2][BLK * D];
  if (dq_rows<D, ROWS, VEC, CAP, BIAS, false>(a, KVs)) dq_rows_seen<D, ROWS, VEC, CAP, BIAS>(a, KVs);
}

// ----------------------------------------------------------------- backward, dK / dV pass
// 8 waves per 128 keys, in pairs that share 32 keys.  Of a tile of 64 queries each wave of a pair takes 32: their scores, dP, P and
// dS.  Wave 0 of the pair sums dV = P^T dctx, wave 1 dK = dS^T Q, each over all 64 queries: they hand each other, through LDS and
// lane to lane, what the other sums, rounded as its product's operand.  The sums run one tile behind, so that a tile's products
// have its successor's exponentials beside them, and a tile has one barrier; three LDS stages.
// (One wave for the scores and P of both halves, the other for dP and dS, in fp32 through LDS and two barriers: 64 heads of 128,
// 2048 tokens, causal 283 us, here 272, 0.51 PFLOP/s of the unmasked half's products; 2 x 16 heads of packed documents 119 and 94;
// 8192 tokens with capped scores 967 and 1027, where each wave's exponentials and not the barriers set the time: one form for all, as the others gain
// more.)  Heads of 128 leave 8 registers in scratch around the loop's products, 16 and more where rows are no 16-byte chunks.
// A workgroup walks the query tiles whose spans reach its keys, for every query head of its share of the key / value head's
// group, one after the other in one chain of sums.
constexpr int NTHR_DKV = 512;

template <int D>
struct DkvShared {
  bf16_t QOs[3][2][BLK * D];  // Q and dctx tiles
  float stat[3][2][BLK];      // lse * log2(e) and delta of the tile's queries
  int span[3][2][BLK];        // their spans
  bf16x8 hand[2][4][2][2][64];  // [tile parity][pair][from wave][operand][lane]
  int range[2];
};

// Addresses of fragments in the three stages, in elements from the first.  Chunk and key of a row occupy other bits than tile, stage and
// row blocks, so an address is a register XOR a constant, one instruction, and the rest an immediate.
template <int D>
struct DkvAddr {
  static constexpr int TILE = BLK * D;
  int k, own, other;  // frag_k of the wave's half, frag_t of its own half and of its partner's
  __device__ __forceinline__ void init(int lane, int role) {
    const int tt = lane & 15, blk = lane >> 4;
    const int t0 = swz<D>(4 * (blk >> 1) + (tt >> 2), 16 * (blk & 1) + 4 * (tt & 3)) + (role ? 0 : TILE);  // wave 0 sums over dctx, wave 1 over Q
    k = swz<D>(lane & 31, 8 * (lane >> 5)) + 32 * D * role;
    own = t0 + 32 * D * role;
    other = t0 + 32 * D * (1 - role);
  }
  // Q (tensor 0) or dctx (1): contraction over the head dimensions
  static __device__ __forceinline__ bf16x8 frag_k(const bf16_t* lds, int at, int tensor, int kk) {
    return *reinterpret_cast<const bf16x8*>(lds + tensor * TILE + (at ^ (16 * kk)));
  }
  static __device__ __forceinline__ bf16x8 frag_t(const bf16_t* lds, int at, int k2, int dt) {
    typedef s16x4 __attribute__((address_space(3))) * lds_v4;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4)(lds + 16 * k2 * D + (at ^ (32 * dt))));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4)(lds + (16 * k2 + 8) * D + (at ^ (32 * dt) ^ 16)));
    return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

template <int D, bool VEC, int CAP, bool BIAS, bool SEEN>
__device__ __forceinline__ bool dkv_keys(const MaskedArgs& a, DkvShared<D>& sh) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, kg = w & 3;
  const int role = __builtin_amdgcn_readfirstlane(w >> 2);
  const int S = a.S_seq, d = a.S_head, group = a.N_heads / a.N_kv, heads = group / a.splits;
  const int per = a.N_kv * a.splits * a.S_mb, x = blockIdx.x % per;
  const int k0 = blockIdx.x / per * WG_ROWS;  // earliest keys first: under a causal mask they see the most queries
  const int kv = x % a.N_kv, split = x / a.N_kv % a.splits, b = x / (a.N_kv * a.splits);
  const size_t seq = (size_t)b * S;
  const int kw = k0 + 32 * kg, key = kw + (lane & 31);
  const int blocks = (S + SPAN_ROWS - 1) / SPAN_ROWS;
  const SpanBlock* tb = a.block + (size_t)b * blocks;

  // the query tiles that see any of these keys lie between the first and the last of them
  if (tid < 2) sh.range[tid] = tid ? 0 : INT_MAX;
  __syncthreads();
  for (int j = tid; j < blocks; j += NTHR_DKV) {
    const SpanBlock y = tb[j];
    if (y.hi_max > k0 && y.lo_min < k0 + WG_ROWS) { atomicMin(&sh.range[0], j); atomicMax(&sh.range[1], j + 1); }
  }
  __syncthreads();
  const int jbeg = sh.range[0], jend = sh.range[1], tiles = jend > jbeg ? jend - jbeg : 0, total = tiles * heads;

  DkvAddr<D> fa;
  fa.init(lane, role);
  const bf16_t* lds = &sh.QOs[0][0][0];
  bf16x8 kf[D / 16], vf[D / 16];
  const uint32_t kr = (uint32_t)(32 * kg + (lane & 31)) * 2;
  load_row<D, VEC>(rows_at((const bf16_t*)a.k + (seq + k0) * a.ldk + (size_t)kv * d, row_bytes(WG_ROWS, S - k0, a.ldk, d)), kr * (uint32_t)a.ldk, lane, d, kf);
  load_row<D, VEC>(rows_at((const bf16_t*)a.v + (seq + k0) * a.ldv + (size_t)kv * d, row_bytes(WG_ROWS, S - k0, a.ldv, d)), kr * (uint32_t)a.ldv, lane, d, vf);
  f32x16 acc[D / 32];  // dV (wave 0 of a pair) or dK, transposed: rows = head dims, column = key
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) acc[dt] = zero16();

  Tile<BLK, D, NTHR_DKV, VEC> qr, dor;
  qr.init(a.ldq, tid, d);
  dor.init(a.ldo, tid, d);
  bool bad = false;
  float lnext = 0.f, dnext = 0.f;
  typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2;
  u32x2 snext{0, 0};
  const int head0 = kv * group + split * heads;
  int fh = 0, fj = jbeg;  // of the next fetch
  // (the tiles' summaries come through vector loads, a tile ahead: scalar ones would be waited for with the next LDS access)
  const auto tiles_at = rows_at(tb, (uint32_t)blocks * 16);
  u32x4 bnext{0, 0, 0, 0};
  SpanBlock ynext{INT_MAX, 0, INT_MAX, 0};
  auto fetch = [&]() {
    const int head = head0 + fh;
    bnext = __builtin_amdgcn_raw_buffer_load_b128(tiles_at, (uint32_t)fj * 16 + 0 * lane, 0, 0);
    qr.fetch((const bf16_t*)a.q + (seq + (size_t)fj * BLK) * a.ldq + (size_t)head * d, a.ldq, S - fj * BLK, d);
    dor.fetch((const bf16_t*)a.dctx + (seq + (size_t)fj * BLK) * a.ldo + (size_t)head * d, a.ldo, S - fj * BLK, d);
    if (w == 0) {
      // (as they come: arithmetic on them here would wait for the tiles)
      const size_t st = ((size_t)b * a.N_heads + head) * S + (size_t)fj * BLK;
      const int left = min(S - fj * BLK, BLK);
      lnext = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rows_at(a.lse + st, left * 4), lane * 4, 0, 0));
      dnext = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rows_at(a.delta + st, left * 4), lane * 4, 0, 0));
      snext = __builtin_amdgcn_raw_buffer_load_b64(rows_at(a.span + seq + (size_t)fj * BLK, left * 8), lane * 8, 0, 0);  // past the end: none
    }
    if (++fj == jend) { fj = jbeg; ++fh; }
  };
  int pj = jbeg;  // of the next store
  auto put = [&](int stage) {
    qr.store(sh.QOs[stage][0], tid);
    dor.store(sh.QOs[stage][1], tid);
    if (w == 0) {
      // past the end, and for rows without a finite score, exp2(score - inf) = 0
      sh.stat[stage][0][lane] = pj * BLK + lane < S && lnext != -INFINITY ? lnext * LOG2E : INFINITY;
      sh.stat[stage][1][lane] = dnext;
      sh.span[stage][0][lane] = (int)snext[0];
      sh.span[stage][1][lane] = (int)snext[1];
    }
    ynext = {__builtin_amdgcn_readfirstlane((int)bnext[0]), __builtin_amdgcn_readfirstlane((int)bnext[1]), __builtin_amdgcn_readfirstlane((int)bnext[2]),
             __builtin_amdgcn_readfirstlane((int)bnext[3])};
    const bool whole = k0 >= ynext.lo_max && k0 + WG_ROWS <= ynext.hi_min && (pj + 1) * BLK <= S;
    if (!SEEN && !whole) bad |= qr.non_finite() || dor.non_finite();
    if (++pj == jend) pj = jbeg;
  };
  if (total > 0) {
    fetch();
    put(0);
  }
  if (total > 1) fetch();
  __syncthreads();
  int j = jbeg, hx = 0, stage = 0, before = 2;  // stages of this tile and of the one before
  bool sum_before = false, part_before = false;
  bf16x8 mine[2];  // the wave's own operand of the tile before
  mine[0] = mine[1] = bf16x8{};
  ScoreFactors f = factors<CAP, BIAS>(a, head0);
  for (int it = 0; it <= total; ++it) {
    const bool here = it < total;
    const int after = stage == 2 ? 0 : stage + 1;
    const SpanBlock y = ynext;
    if (it + 1 < total) put(after);
    if (it + 2 < total) fetch();
    const int qb = j * BLK;
    const bool work = here && !(kw >= S || y.hi_max <= kw || y.lo_min >= kw + 32);
    const bool part = !(kw >= y.lo_max && kw + 32 <= y.hi_min && qb + BLK <= S);
    // what the partner left of the tile before
    bf16x8 theirs[2];
    if (sum_before) {
      theirs[0] = sh.hand[(it & 1) ^ 1][kg][role ^ 1][0][lane];
      theirs[1] = sh.hand[(it & 1) ^ 1][kg][role ^ 1][1][lane];
    }
    auto sums = [&]() {
      const int at = before * 2 * DkvAddr<D>::TILE, own = fa.own + at, other = fa.other + at;
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(DkvAddr<D>::frag_t(lds, own, k2, dt), mine[k2], acc[dt], 0, 0, 0);
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(DkvAddr<D>::frag_t(lds, other, k2, dt), theirs[k2], acc[dt], 0, 0, 0);
    };
    if (SEEN && sum_before && part_before) {
      const int* lo_s = sh.span[before][0];
      const int* hi_s = sh.span[before][1];
      bf16x8 p[4];
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) {
        p[k2] = role ? theirs[k2] : mine[k2];
        p[2 + k2] = role ? mine[k2] : theirs[k2];
      }
      FragAddrXor<D> fx;
      fx.init(lane);
      accumulate_seen<D>(acc, p, 0, 4, sh.QOs[before][role ? 0 : 1], fx, lane,
                         [&](int c) { return __builtin_amdgcn_ballot_w64(kw + c >= lo_s[lane] && kw + c < hi_s[lane]); });
    } else if (sum_before && !work) {
      sums();
    }
    if (work) {
      const int at = fa.k + stage * 2 * DkvAddr<D>::TILE, h0 = 32 * role;
      f32x16 s = zero16(), dp = zero16();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(DkvAddr<D>::frag_k(lds, at, 0, kk), kf[kk], s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(DkvAddr<D>::frag_k(lds, at, 1, kk), vf[kk], dp, 0, 0, 0);
      }
      mfma_lds_pipeline<2 * (D / 16), 1, 4>();
      const float dist = (float)(qb + h0 + 4 * (lane >> 5) - key);
      // P = exp(score - lse), dS = P (dP - delta) times the cap's derivative (the factor 1/sqrt(d) is applied once, to dK)
      const float *ls_s = sh.stat[stage][0] + h0, *dl_s = sh.stat[stage][1] + h0;
      f32x4 ls, dl, ls2 = *reinterpret_cast<const f32x4*>(&ls_s[acc_row(0, lane)]), dl2 = *reinterpret_cast<const f32x4*>(&dl_s[acc_row(0, lane)]);
      auto grad = [&](auto rc) {
        constexpr int r = decltype(rc)::value, q4 = r >> 2, e = r & 3;
        if constexpr (e == 0) {  // the next four rows' statistics are on their way
          ls = ls2;
          dl = dl2;
          if constexpr (q4 < 3) {
            ls2 = *reinterpret_cast<const f32x4*>(&ls_s[acc_row(4 * q4 + 4, lane)]);
            dl2 = *reinterpret_cast<const f32x4*>(&dl_s[acc_row(4 * q4 + 4, lane)]);
          }
        }
        float c = 0.f;
        const float ex = exponent<CAP, BIAS>(s[r], dist + (float)(8 * q4 + e), f, c);
        s[r] = __builtin_amdgcn_exp2f(CAP || BIAS ? ex - ls[e] : fmaf(ex, f.c2, -ls[e]));
        dp[r] = s[r] * (dp[r] - dl[e]);
        if (CAP) dp[r] *= slack_of<CAP>(c);
      };
      if (sum_before && !(SEEN && part_before)) {
        // The tile before's products beside this one's exponentials, in an order fixed by hand: a step is one product, the fragment
        // AHEAD steps further on, and a share of the vector work.  (Left to itself the scheduler waits for every fragment and
        // puts the vector work behind: 290 us where this took 279.)
        constexpr int STEPS = 4 * (D / 32), AHEAD = 3, PER = 16 / STEPS;
        const int tile = before * 2 * DkvAddr<D>::TILE, own = fa.own + tile, other = fa.other + tile;
        bf16x8 ring[AHEAD + 1];
        auto load = [&](auto ic) {
          constexpr int i = decltype(ic)::value, h = i / (2 * (D / 32)), k2 = i / (D / 32) % 2, dt = i % (D / 32);
          ring[i % (AHEAD + 1)] = DkvAddr<D>::frag_t(lds, h ? other : own, k2, dt);
        };
        __builtin_amdgcn_sched_barrier(0);
        static_for<AHEAD>([&](auto ic) { load(ic); });
        static_for<STEPS>([&](auto ic) {
          constexpr int i = decltype(ic)::value, h = i / (2 * (D / 32)), k2 = i / (D / 32) % 2, dt = i % (D / 32);
          if constexpr (i + AHEAD < STEPS) load(std::integral_constant<int, i + AHEAD>{});
          acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[i % (AHEAD + 1)], h ? theirs[k2] : mine[k2], acc[dt], 0, 0, 0);
          static_for<PER>([&](auto rc) { grad(std::integral_constant<int, i * PER + decltype(rc)::value>{}); });
          __builtin_amdgcn_sched_barrier(0);
        });
      } else {
        static_for<16>([&](auto rc) { grad(rc); });
      }
      if (part) {
        const int* lo_s = sh.span[stage][0] + h0;
        const int* hi_s = sh.span[stage][1] + h0;
        // (a row of one key has no score gradient; it is never part of a tile taken whole)
        auto mask = [&](int r, int lo, int hi) {
          const bool out = (unsigned)(key - lo) >= (unsigned)(hi - lo);
          s[r] = out ? 0.f : s[r];
          dp[r] = (unsigned)out | (unsigned)(hi - lo == 1) ? 0.f : dp[r];
        };
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const int4 lo = *reinterpret_cast<const int4*>(&lo_s[acc_row(4 * q4, lane)]);
          const int4 hi = *reinterpret_cast<const int4*>(&hi_s[acc_row(4 * q4, lane)]);
          mask(4 * q4, lo.x, hi.x);
          mask(4 * q4 + 1, lo.y, hi.y);
          mask(4 * q4 + 2, lo.z, hi.z);
          mask(4 * q4 + 3, lo.w, hi.w);
        }
      }
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) {
        const bf16x8 p = pack8(s, k2), g = pack8(dp, k2);
        mine[k2] = role ? g : p;
        sh.hand[it & 1][kg][role][k2][lane] = role ? p : g;
      }
    }
    sum_before = work;
    part_before = part;
    before = stage;
    stage = after;
    if (++j == jend) {
      j = jbeg;
      if (++hx < heads && BIAS) f = factors<CAP, BIAS>(a, head0 + hx);
    }
    __syncthreads();
  }
  if (!SEEN && __syncthreads_or(bad)) return true;
  const float mul = role ? a.scale : 1.f;
  if (a.splits > 1) {
    if (key >= S) return false;
    // this share's plane: [split][dk, dv][token][key / value head][d]
    const size_t width = (size_t)a.N_kv * d, plane = (size_t)a.S_mb * S * width;
    float* out = a.planes + (2 * (size_t)split + (role ? 0 : 1)) * plane + (seq + key) * width + (size_t)kv * d;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int c = dt * 32 + acc_row(r, lane);
        if (c < d) out[c] = acc[dt][r] * mul;
      }
    return false;
  }
  bf16_t* out = role ? (bf16_t*)a.dk + (seq + k0) * a.ldk : (bf16_t*)a.dv + (seq + k0) * a.ldv;
  const size_t ldg = role ? a.ldk : a.ldv;
  store_row<D, VEC>(acc, rows_at(out + (size_t)kv * d, row_bytes(WG_ROWS, S - k0, ldg, d)), kr * (uint32_t)ldg, lane, mul, d);
  return false;
}

template <int D, bool VEC, int CAP, bool BIAS>
__device__ __attribute__((noinline)) void dkv_keys_seen(MaskedArgs a, DkvShared<D>& sh) {
  dkv_keys<D, VEC, CAP, BIAS, true>(a, sh);
}

template <int D, bool VEC, int CAP, bool BIAS>
__global__ __launch_bounds__(NTHR_DKV, 2) void masked_dkv_kernel(MaskedArgs a) {
  __shared__ __attribute__((aligned(16))) DkvShared<D> sh;
  if (dkv_keys<D, VEC, CAP, BIAS, false>(a, sh)) dkv_keys_seen<D, VEC, CAP, BIAS>(a, sh);
}

// dk, dv = the shares' planes, added in ascending order
__global__ __launch_bounds__(256) void masked_join_kernel(MaskedArgs a) {
  const size_t width = (size_t)a.N_kv * a.S_head, plane = (size_t)a.S_mb * a.S_seq * width, n = 2 * plane;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
    float t = 0.f;
    for (int k = 0; k < a.splits; ++k) t += a.planes[(size_t)k * n + i];
    const bool v = i >= plane;
    const size_t e = v ? i - plane : i, row = e / width, c = e - row * width;
    if (v) ((bf16_t*)a.dv)[row * a.ldv + c] = (bf16_t)t;
    else ((bf16_t*)a.dk)[row * a.ldk + c] = (bf16_t)t;
  }
}

bf_status launched() {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_error("attention_masked_mfma: launch failed: %s", hipGetErrorString(e)); return BF_EDEVICE; }
  return BF_OK;
}

inline unsigned query_grid(const MaskedArgs& a, int rows) { return (unsigned)((a.S_seq + rows - 1) / rows) * (unsigned)(a.N_heads * a.S_mb); }

template <int D, bool VEC, int CAP, bool BIAS>
void run(const MaskedArgs& a, bool backward, hipStream_t st) {
  constexpr int ROWS = 128;
  if (!backward) {
    masked_fwd_kernel<D, ROWS, VEC, CAP, BIAS><<<query_grid(a, ROWS), 2 * ROWS, 0, st>>>(a);
    return;
  }
  masked_dq_kernel<D, ROWS, VEC, CAP, BIAS><<<query_grid(a, ROWS), 2 * ROWS, 0, st>>>(a);
  const unsigned grid = (unsigned)((a.S_seq + WG_ROWS - 1) / WG_ROWS) * (unsigned)(a.N_kv * a.splits * a.S_mb);
  masked_dkv_kernel<D, VEC, CAP, BIAS><<<grid, NTHR_DKV, 0, st>>>(a);
  if (a.splits > 1) masked_join_kernel<<<2048, 256, 0, st>>>(a);
}

template <int D, bool VEC>
void by_score(const MaskedArgs& a, bool backward, hipStream_t st) {
  // (see ScoreFactors)
  if (a.cap > CAP_FAST || (a.cap > 0.f && 2.0 * LOG2E * a.scale / a.cap > FLT_MAX)) run<D, VEC, 2, true>(a, backward, st);
  else if (a.cap > 0.f && a.slope) run<D, VEC, 1, true>(a, backward, st);
  else if (a.cap > 0.f) run<D, VEC, 1, false>(a, backward, st);
  else if (a.slope) run<D, VEC, 0, true>(a, backward, st);
  else run<D, VEC, 0, false>(a, backward, st);
}

bf_status by_head(const MaskedArgs& a, bool backward, hipStream_t st) {
  if (a.S_head <= 64) a.vec ? by_score<64, true>(a, backward, st) : by_score<64, false>(a, backward, st);
  else a.vec ? by_score<128, true>(a, backward, st) : by_score<128, false>(a, backward, st);
  return launched();
}

}  // namespace

bf_status attention_masked_fwd_mfma(const MaskedArgs& a, hipStream_t st) { return by_head(a, false, st); }
bf_status attention_masked_bwd_mfma(const MaskedArgs& a, hipStream_t st) { return by_head(a, true, st); }

}  // namespace bf
