// Masked attention in fp32 on the fp32 matrix cores (v_mfma_f32_32x32x2_f32), heads up to 128 (padded with zeros to 64 or 128).
//
// The passes are those of attention_masked_mfma.hip on tiles of 32 keys (queries), with dQ in one walk: ctx is fp32, and delta = dctx . ctx
// as exact as any.  An instruction contracts over two values,
// one from each half of the wave.  Over head dimensions a lane holds four in a row, dimensions 8 c + 4 (lane / 32) .. + 3, for four
// instructions.  Over the tile's rows instruction r takes rows (r / 4) 8 + r % 4 and the same + 4: register r of a score tile is then
// the other operand as it stands.  157 TFLOP/s against 2.5 PFLOP/s in bf16: the matrix cores bound everything here (64 cycles an
// instruction, one 4- or 16-byte LDS read for one or four of them).
#include <float.h>
#include <math.h>

#include <type_traits>

#include "attention_masked.h"

namespace bf {

namespace {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;

constexpr float LOG2E = 1.4426950408889634f;
constexpr int BLK = 32;    // rows of a streamed tile
constexpr int ROWS = 128;  // queries (keys) of a workgroup, 32 to a wave
constexpr uint32_t NOWHERE = 0x7fffff00u;

// a tile row's length: rows eight apart share banks in a 16-byte read, and the two rows of a 4-byte read do not
template <int D> constexpr int LD = D + 8;

__device__ __forceinline__ int acc_row(int r, int lane) { return (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3); }

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}

// Rows go through buffer descriptors that end with the last row there is: what lies past it, or past a short row, reads as zeros and
// is not written, without branches (a short launch waits for its instructions).  VEC: rows of whole 16-byte chunks that start at
// multiples of 4 bytes; else element by element.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const void* g, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)g, 0, (int)bytes, 0x00020000);
}
// bytes of up to 32 rows, those that are there of them
__device__ __forceinline__ uint32_t row_bytes(int there, size_t ld, int d) {
  return there < 1 ? 0 : (uint32_t)(((there < 32 ? there : 32) - 1) * ld + d) * 4;
}

template <int D, int NT, bool VEC>
struct Tile {
  static constexpr int CH = BLK * D / 4 / NT, STEP = NT / (D / 4);
  u32x4 v[CH];
  uint32_t off;
  int col;
  __device__ __forceinline__ void init(size_t ld, int tid, int d) {
    col = tid % (D / 4) * 4;
    off = (uint32_t)(tid / (D / 4) * ld + col) * 4;
    if (VEC && col >= d) off = NOWHERE;
  }
  __device__ __forceinline__ void fetch(const float* __restrict__ g, size_t ld, int valid, int d) {
    const auto rsrc = rows_at(g, row_bytes(valid, ld, d));
    const uint32_t step = (uint32_t)(STEP * ld * 4);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      if (VEC) {
        v[i] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, off + i * step, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i][e] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, col + e < d ? off + i * step + 4 * e : NOWHERE, 0, 0);
      }
    }
  }
  __device__ __forceinline__ void store(float* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < CH; ++i) *reinterpret_cast<u32x4*>(lds + (tid / (D / 4) + i * STEP) * LD<D> + col) = v[i];
  }
  __device__ __forceinline__ bool non_finite() const {
    bool any = false;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) any |= (v[i][e] & 0x7fffffffu) >= 0x7f800000u;
    return any;
  }
};

// A token's row as the operand of a contraction over head dimensions.  rows: the wave's 32 (uniform); off: the lane's
template <int D, bool VEC>
__device__ __forceinline__ void load_row(__amdgpu_buffer_rsrc_t rows, uint32_t off, int lane, int d, f32x4 (&f)[D / 8]) {
#pragma unroll
  for (int c = 0; c < D / 8; ++c) {
    const int at = 8 * c + 4 * (lane >> 5);
    if (VEC) {
      f[c] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, at < d ? off + 4 * at : NOWHERE, 0, 0));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) f[c][e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rows, at + e < d ? off + 4 * (at + e) : NOWHERE, 0, 0));
    }
  }
}

template <int D, bool VEC>
__device__ __forceinline__ void store_row(const f32x16 (&acc)[D / 32], __amdgpu_buffer_rsrc_t rows, uint32_t off, int lane, float mul, int d) {
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const int c = dt * 32 + q4 * 8 + (lane >> 5) * 4;
      f32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = acc[dt][q4 * 4 + e] * mul;
      const u32x4 u = __builtin_bit_cast(u32x4, o);
      if (VEC) {
        __builtin_amdgcn_raw_buffer_store_b128(u, rows, c < d ? off + 4 * c : NOWHERE, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) __builtin_amdgcn_raw_buffer_store_b32(u[e], rows, c + e < d ? off + 4 * (c + e) : NOWHERE, 0, 0);
      }
    }
}

// s += tile (rows) x row^T over the head dimensions
template <int D>
__device__ __forceinline__ void dots(f32x16& s, const float* tile, const f32x4 (&f)[D / 8], int lane, int d) {
#pragma unroll
  for (int c = 0; c < D / 8; ++c) {
    if (8 * c >= d) break;  // (uniform: nothing but zeros from here on)
    const f32x4 t = *reinterpret_cast<const f32x4*>(tile + (lane & 31) * LD<D> + 8 * c + 4 * (lane >> 5));
#pragma unroll
    for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(t[e], f[c][e], s, 0, 0, 0);
  }
}

// acc += tile^T s over the tile's rows
template <int D>
__device__ __forceinline__ void sums(f32x16 (&acc)[D / 32], const f32x16& s, const float* tile, int lane, int d) {
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) {
    if (32 * dt >= d) break;
#pragma unroll
    for (int r = 0; r < 16; ++r)
      acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(tile[acc_row(r, lane) * LD<D> + 32 * dt + (lane & 31)], s[r], acc[dt], 0, 0, 0);
  }
}

// the same, column by column of s over the tile's rows that the column sees (bit r of rows_of(c)): for tiles masked in part that
// hold an infinity or a NaN
template <int D, typename F>
__device__ __forceinline__ void sums_seen(f32x16 (&acc)[D / 32], const f32x16& s, const float* tile, int lane, int d, F rows_of) {
#pragma unroll 1
  for (int c = 0; c < 32; ++c) {
    const uint32_t seen = rows_of(c);
    if (seen == 0) continue;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
      if (32 * dt >= d) break;
      f32x16 sum = zero16();
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = acc_row(r, lane);
        const float t = tile[row * LD<D> + 32 * dt + (lane & 31)];
        sum = __builtin_amdgcn_mfma_f32_32x32x2f32(seen >> row & 1 ? t : 0.f, s[r], sum, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[dt][r] = (lane & 31) == c ? acc[dt][r] + sum[r] : acc[dt][r];
    }
  }
}

__device__ __forceinline__ uint32_t interval_bits(int k0, int lo, int hi) {
  const int a = min(max(lo - k0, 0), 32), b = min(max(hi - k0, 0), 32);
  return a >= b ? 0u : (~0u >> (32 - (b - a))) << a;
}

// a score from a dot product; slack: the cap's derivative there.  (slope 0: no bias; not worth kernels of its own, 2 operations beside
// 64 cycles of the matrix core for each of a dot product's pairs of dimensions)
template <bool CAP>
__device__ __forceinline__ float score_of(float dot, float dist, const MaskedArgs& a, float inv_cap, float slope, float& slack) {
  float s = dot * a.scale;
  if (CAP) {
    const float t = tanh_f(s * inv_cap);
    s = a.cap * t;
    slack = 1.f - t * t;
  }
  return fmaf(-slope, fabsf(dist), s);
}

struct WaveSpan {
  int lo_min, hi_max, lo_max, hi_min;
  __device__ __forceinline__ void init(int2 sp, bool row) {
    const bool any = sp.y > sp.x;
    lo_min = row && any ? sp.x : INT_MAX;
    hi_max = row && any ? sp.y : 0;
    lo_max = !row ? 0 : any ? sp.x : INT_MAX;
    hi_min = !row ? INT_MAX : any ? sp.y : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
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

// KG key groups: 1: the four waves hold 32 rows each and share the tiles, in two LDS stages.  4: they hold the same 32 rows, every wave walks
// every fourth tile through an LDS stage of its own, without barriers, and their sums meet at the end: for launches that
// leave compute units idle.
template <int D, int KG>
struct QueryShared {
  static constexpr int STAGES = KG == 1 ? 2 : 4;
  float K[STAGES][BLK * LD<D>], V[STAGES][BLK * LD<D>];
};

// Forward (GRAD false) and dQ (GRAD true).  SEEN: tiles that are masked in part by sums_seen; without it returns whether one of
// those held a non-finite value that enters a sum.
// 2 x 500 queries, 8 heads of 80 over 2, bias and capped scores: forward 54 us, dQ 60, and the keys 77 (12, 16 and 17 TFLOP/s of 154): 256
// workgroups, each wave a chain of two to four tiles.  A launch of one tile takes 24 us at D 128: rows, instructions, hand-over.  dQ at D 128 on KG 1
// keeps ten registers in scratch inside its loop, and rows that are no 16-byte chunks 20 to 80 in every form of D 128.
template <int D, int KG, bool VEC, bool CAP, bool GRAD, bool SEEN>
__device__ __forceinline__ bool query_rows(const MaskedArgs& a, QueryShared<D, KG>& sh) {
  constexpr int NT = KG == 1 ? 256 : 64, RB = KG == 1 ? ROWS : 32;  // threads that fetch a tile, rows of the workgroup
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, wr = KG == 1 ? w : 0, ft = KG == 1 ? tid : lane;
  const int S = a.S_seq, d = a.S_head, nhb = a.N_heads * a.S_mb, blocks = (S + RB - 1) / RB, group = a.N_heads / a.N_kv;
  const int x = blockIdx.x % nhb, hx = x % a.N_heads, b = x / a.N_heads, kv = hx % a.N_kv, head = kv * group + hx / a.N_kv;
  const int q0 = (blocks - 1 - blockIdx.x / nhb) * RB, q = q0 + 32 * wr + (lane & 31), ql = min(q, S - 1);
  const size_t seq = (size_t)b * S, st = ((size_t)b * a.N_heads + head) * S + ql;
  const float* kbase = (const float*)a.k + seq * a.ldk + (size_t)kv * d;
  const float* vbase = (const float*)a.v + seq * a.ldv + (size_t)kv * d;

  f32x4 qf[D / 8], dof[GRAD ? D / 8 : 1];
  const int w0 = q0 + 32 * wr;  // the wave's first row
  const auto rows_of = [&](const void* t, size_t ld) { return rows_at((const float*)t + (seq + w0) * ld + (size_t)head * d, row_bytes(S - w0, ld, d)); };
  const uint32_t qat = (uint32_t)((lane & 31) * a.ldq) * 4, oat = (uint32_t)((lane & 31) * a.ldo) * 4;
  load_row<D, VEC>(rows_of(a.q, a.ldq), qat, lane, d, qf);
  float lse = 0.f, dl = 0.f;
  if constexpr (GRAD) {
    load_row<D, VEC>(rows_of(a.dctx, a.ldo), oat, lane, d, dof);
    f32x4 cf[D / 8];
    load_row<D, VEC>(rows_of(a.ctx, a.ldo), oat, lane, d, cf);
#pragma unroll
    for (int c = 0; c < D / 8; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) dl = fmaf(dof[c][e], cf[c][e], dl);
    dl += __shfl_xor(dl, 32, 64);
    if (lane < 32 && q < S && (KG == 1 || w == 0)) a.delta[st] = dl;
    lse = a.lse[st] == -INFINITY ? INFINITY : a.lse[st];  // (a row without a finite score has no probabilities)
  }
  int2 sp = a.span[seq + ql];
  sp.x = max(sp.x, 0);
  sp.y = min(sp.y, S);
  WaveSpan ws;
  ws.init(sp, q < S);
  const int sb = (S + SPAN_ROWS - 1) / SPAN_ROWS, at = q0 / SPAN_ROWS;
  SpanBlock wg = a.block[(size_t)b * sb + at];
  if (KG > 1) {
    wg = {ws.lo_min, ws.hi_max, ws.lo_max, ws.hi_min};
  } else if (at + 1 < sb) {
    const SpanBlock y = a.block[(size_t)b * sb + at + 1];
    wg = {min(wg.lo_min, y.lo_min), max(wg.hi_max, y.hi_max), max(wg.lo_max, y.lo_max), min(wg.hi_min, y.hi_min)};
  }
  wg.hi_max = min(wg.hi_max, S);
  const float slope = a.slope ? a.slope[head] : 0.f, inv_cap = CAP ? inverse_cap(a.cap) : 0.f;
  f32x16 o[D / 32];  // ctx, or dQ; transposed: rows = head dims, column = the lane's query
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) o[dt] = zero16();
  float m = -FLT_MAX, l = 0.f;

  const int jbeg = wg.hi_max > 0 ? max(wg.lo_min, 0) / BLK : 0, jend = (wg.hi_max + BLK - 1) / BLK;
  Tile<D, NT, VEC> kr, vr;
  kr.init(a.ldk, ft, d);
  vr.init(a.ldv, ft, d);
  bool bad = false;
  auto fetch = [&](int j) {
    kr.fetch(kbase + (size_t)j * BLK * a.ldk, a.ldk, S - j * BLK, d);
    vr.fetch(vbase + (size_t)j * BLK * a.ldv, a.ldv, S - j * BLK, d);
  };
  auto put = [&](int j, int stage) {
    kr.store(sh.K[stage], ft);
    vr.store(sh.V[stage], ft);
    const int kb = j * BLK;
    if (!SEEN && !(kb >= wg.lo_max && kb + BLK <= wg.hi_min)) bad |= GRAD ? kr.non_finite() : vr.non_finite();
  };
  // (one wave's own stage: its LDS accesses are in order)
  auto sync = [&]() {
    if (KG == 1) __syncthreads();
    else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
  const int j0 = KG == 1 ? jbeg : jbeg + w;
  if (j0 < jend) {
    fetch(j0);
    put(j0, KG == 1 ? 0 : w);
  }
  sync();
  for (int j = j0; j < jend; j += KG) {
    const int cur = KG == 1 ? (j - jbeg) & 1 : w, kb = j * BLK;
    const float *K = sh.K[cur], *V = sh.V[cur];
    if (j + KG < jend) fetch(j + KG);
    if (!ws.skips(kb, BLK)) {
      const bool part = !ws.whole(kb, BLK);
      f32x16 s = zero16();
      dots<D>(s, K, qf, lane, d);
      const float dist = (float)(q - kb - 4 * (lane >> 5));
      const int lo = sp.x - kb, n = sp.y - sp.x;
      if constexpr (!GRAD) {
        float mx = m, slack;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = score_of<CAP>(s[r], dist - (float)((r >> 2) * 8 + (r & 3)), a, inv_cap, slope, slack);
          if (part && (unsigned)(acc_row(r, lane) - lo) >= (unsigned)n) s[r] = -INFINITY;
          mx = fmaxf(mx, s[r]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        if (__builtin_amdgcn_ballot_w64(mx > m) != 0) {
          const float alpha = __builtin_amdgcn_exp2f((m - mx) * LOG2E);
          l *= alpha;
#pragma unroll
          for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
          m = mx;
        }
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = __builtin_amdgcn_exp2f((s[r] - m) * LOG2E);
          sum[r & 3] += s[r];
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      } else {
        f32x16 dp = zero16();
        dots<D>(dp, V, dof, lane, d);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float slack = 1.f;
          const float t = score_of<CAP>(s[r], dist - (float)((r >> 2) * 8 + (r & 3)), a, inv_cap, slope, slack);
          s[r] = __builtin_amdgcn_exp2f((t - lse) * LOG2E) * (dp[r] - dl) * slack;
          if (part && (unsigned)(acc_row(r, lane) - lo) >= (unsigned)n) s[r] = 0.f;
        }
      }
      const float* tile = GRAD ? K : V;
      if (SEEN && part)
        sums_seen<D>(o, s, tile, lane, d, [&](int c) { return interval_bits(kb, __builtin_amdgcn_readlane(sp.x, c), __builtin_amdgcn_readlane(sp.y, c)); });
      else sums<D>(o, s, tile, lane, d);
    }
    if (KG > 1) sync();
    if (j + KG < jend) put(j + KG, KG == 1 ? cur ^ 1 : w);
    sync();
  }
  if (!SEEN && __syncthreads_or(bad)) return true;
  l += __shfl_xor(l, 32, 64);
  if constexpr (KG > 1) {
    // the other groups hand over their sums, lane to lane, in the stage that was theirs; added in order
    constexpr int NV = D / 2 + 2;
    static_assert(NV * 64 <= BLK * LD<D>, "the hand-over does not fit");
    if (w > 0) {
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) sh.K[w][(dt * 16 + r) * 64 + lane] = o[dt][r];
      sh.K[w][(NV - 2) * 64 + lane] = m;
      sh.K[w][(NV - 1) * 64 + lane] = l;
    }
    __syncthreads();
    if (w > 0) return false;
#pragma unroll 1
    for (int g = 1; g < KG; ++g) {
      const float* from = sh.K[g] + lane;
      float a0 = 1.f, a1 = 1.f;
      if (!GRAD) {
        const float m1 = from[(NV - 2) * 64], M = fmaxf(m, m1);
        a0 = __builtin_amdgcn_exp2f((m - M) * LOG2E);
        a1 = __builtin_amdgcn_exp2f((m1 - M) * LOG2E);
        l = l * a0 + from[(NV - 1) * 64] * a1;
        m = M;
      }
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = GRAD ? o[dt][r] + from[(dt * 16 + r) * 64] : o[dt][r] * a0 + from[(dt * 16 + r) * 64] * a1;
    }
  }
  if (q >= S) return false;
  if constexpr (GRAD) {
    if (sp.y - sp.x <= 1) {  // one key: its probability is 1 whatever the score
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) o[dt] = zero16();
    }
    store_row<D, VEC>(o, rows_of(a.dq, a.ldq), qat, lane, a.scale, d);
  } else {
    store_row<D, VEC>(o, rows_of(a.ctx, a.ldo), oat, lane, l == 0.f ? 0.f : 1.0f / l, d);
    if (lane < 32 && a.lse) a.lse[st] = l == 0.f ? -INFINITY : m + logf(l);
  }
  return false;
}

// (a function of its own: see attention_masked_mfma.hip)
template <int D, int KG, bool VEC, bool CAP, bool GRAD>
__device__ __attribute__((noinline)) void query_rows_seen(MaskedArgs a, QueryShared<D, KG>& sh) {
  query_rows<D, KG, VEC, CAP, GRAD, true>(a, sh);
}

template <int D, int KG, bool VEC, bool CAP, bool GRAD>
__global__ __launch_bounds__(256, KG == 1 ? 2 : 1) void masked_query_f32_kernel(MaskedArgs a) {
  __shared__ __attribute__((aligned(16))) QueryShared<D, KG> sh;
  if (query_rows<D, KG, VEC, CAP, GRAD, false>(a, sh)) {
    __syncthreads();
    query_rows_seen<D, KG, VEC, CAP, GRAD>(a, sh);
  }
}

// dK / dV: 8 waves in pairs that share 32 keys: the first takes a tile's scores and P and sums dV, the second dP and, from the first's P
// through LDS, dS and sums dK.  QG query groups: 1: 32 keys to a pair, 128 to the workgroup, the tiles in
// two LDS stages.  4: all pairs hold the same 32 keys, each takes every fourth tile through a stage of its own, and their sums
// meet at the end.
constexpr int NTHR_DKV = 512;
template <int D, int QG>
struct KeyShared {
  static constexpr int STAGES = QG == 1 ? 2 : 4;
  float Q[STAGES][BLK * LD<D>], O[STAGES][BLK * LD<D>];
  float stat[STAGES][2][BLK];
  int span[STAGES][2][BLK];
  float P[4][4][64 * 4];  // [pair][register quarter][lane]
  int range[2];
};

template <int D, int QG, bool VEC, bool CAP, bool SEEN>
__device__ __forceinline__ bool key_rows(const MaskedArgs& a, KeyShared<D, QG>& sh) {
  constexpr int KB = QG == 1 ? ROWS : 32, NT = NTHR_DKV / QG;  // keys of the workgroup, threads that fetch a tile
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, pair = w & 3;
  const int kg = QG == 1 ? pair : 0, grp = QG == 1 ? 0 : pair, ft = QG == 1 ? tid : (w >> 2) * 64 + lane;
  const bool dk_role = w >= 4;  // wave-uniform
  const int S = a.S_seq, d = a.S_head, group = a.N_heads / a.N_kv, heads = group / a.splits;
  const int per = a.N_kv * a.splits * a.S_mb, x = blockIdx.x % per, k0 = blockIdx.x / per * KB;
  const int kv = x % a.N_kv, split = x / a.N_kv % a.splits, b = x / (a.N_kv * a.splits);
  const size_t seq = (size_t)b * S;
  const int kw = k0 + 32 * kg, key = kw + (lane & 31);
  const int blocks = (S + SPAN_ROWS - 1) / SPAN_ROWS;
  const SpanBlock* tb = a.block + (size_t)b * blocks;
  if (tid < 2) sh.range[tid] = tid ? 0 : INT_MAX;
  __syncthreads();
  for (int j = tid; j < blocks; j += NTHR_DKV) {
    const SpanBlock y = tb[j];
    if (y.hi_max > k0 && y.lo_min < k0 + KB) { atomicMin(&sh.range[0], j); atomicMax(&sh.range[1], j + 1); }
  }
  __syncthreads();
  // in tiles of 32 queries, two to a block of spans
  const int jbeg = sh.range[0] == INT_MAX ? 0 : 2 * sh.range[0], jend = min(2 * sh.range[1], (S + BLK - 1) / BLK);
  const int tiles = jend > jbeg ? jend - jbeg : 0, total = tiles * heads, head0 = kv * group + split * heads;

  f32x4 kvf[D / 8];  // this wave's K rows (dV role) or V rows (dK role)
  const size_t ldkv = dk_role ? a.ldv : a.ldk;
  load_row<D, VEC>(rows_at((const float*)(dk_role ? a.v : a.k) + (seq + kw) * ldkv + (size_t)kv * d, row_bytes(S - kw, ldkv, d)),
                   (uint32_t)((lane & 31) * ldkv) * 4, lane, d, kvf);
  f32x16 acc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) acc[dt] = zero16();
  Tile<D, NT, VEC> qr, dor;
  qr.init(a.ldq, ft, d);
  dor.init(a.ldo, ft, d);
  bool bad = false;
  float lnext = 0.f, dnext = 0.f;
  int2 snext = make_int2(0, 0);
  // step `it`: query head it / tiles of the share, tile jbeg + it % tiles
  auto fetch = [&](int it) {
    if (it >= total) return;
    const int fj = jbeg + it % tiles, head = head0 + it / tiles;
    qr.fetch((const float*)a.q + (seq + (size_t)fj * BLK) * a.ldq + (size_t)head * d, a.ldq, S - fj * BLK, d);
    dor.fetch((const float*)a.dctx + (seq + (size_t)fj * BLK) * a.ldo + (size_t)head * d, a.ldo, S - fj * BLK, d);
    if (ft < BLK) {
      const int i = fj * BLK + ft;
      const size_t st = ((size_t)b * a.N_heads + head) * S + i;
      // (as it comes: arithmetic on it here would wait for the tiles)
      lnext = i < S ? a.lse[st] : -INFINITY;
      dnext = i < S ? a.delta[st] : 0.f;
      snext = i < S ? a.span[seq + i] : make_int2(0, 0);
    }
  };
  auto put = [&](int it, int stage) {
    if (it >= total) return;
    qr.store(sh.Q[stage], ft);
    dor.store(sh.O[stage], ft);
    if (ft < BLK) {
      sh.stat[stage][0][ft] = lnext == -INFINITY ? INFINITY : lnext;  // no probabilities
      sh.stat[stage][1][ft] = dnext;
      sh.span[stage][0][ft] = snext.x;
      sh.span[stage][1][ft] = snext.y;
    }
    const int pj = jbeg + it % tiles;
    const SpanBlock y = tb[pj >> 1];
    const bool whole = k0 >= y.lo_max && k0 + KB <= y.hi_min && (pj + 1) * BLK <= S;
    if (!SEEN && !whole) bad |= qr.non_finite() || dor.non_finite();
  };
  fetch(grp);
  put(grp, grp);
  __syncthreads();
  const float inv_cap = CAP ? inverse_cap(a.cap) : 0.f;
  // every wave passes the same barriers, whether it has a tile or not
  for (int step = 0; step < total; step += QG) {
    const int it = step + grp, cur = QG == 1 ? it & 1 : grp;
    const bool there = it < total;
    const int j = jbeg + (there ? it % tiles : 0), qb = j * BLK;
    const float slope = a.slope && there ? a.slope[head0 + it / tiles] : 0.f;
    fetch(it + QG);
    const SpanBlock y = tb[j >> 1];
    const bool skip = !there || kw >= S || y.hi_max <= kw || y.lo_min >= kw + 32;
    const bool part = !(kw >= y.lo_max && kw + 32 <= y.hi_min && qb + BLK <= S);
    const int* lo_s = sh.span[cur][0];
    const int* hi_s = sh.span[cur][1];
    f32x16 s = zero16();
    if (!skip) {
      if (!dk_role) {
        dots<D>(s, sh.Q[cur], kvf, lane, d);
        const float dist = (float)(qb + 4 * (lane >> 5) - key);
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const f32x4 ls = *reinterpret_cast<const f32x4*>(&sh.stat[cur][0][acc_row(4 * q4, lane)]);
          f32x4 give;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 4 * q4 + e;
            float slack = 1.f;
            const float t = score_of<CAP>(s[r], dist + (float)(8 * q4 + e), a, inv_cap, slope, slack);
            s[r] = __builtin_amdgcn_exp2f((t - ls[e]) * LOG2E);
            give[e] = s[r] * slack;
            if (part && (key < lo_s[acc_row(r, lane)] || key >= hi_s[acc_row(r, lane)])) s[r] = 0.f;
          }
          *reinterpret_cast<f32x4*>(&sh.P[pair][q4][lane * 4]) = give;
        }
      } else {
        dots<D>(s, sh.O[cur], kvf, lane, d);
      }
    }
    __syncthreads();
    if (!skip) {
      if (dk_role) {
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const f32x4 pr = *reinterpret_cast<const f32x4*>(&sh.P[pair][q4][lane * 4]);
          const f32x4 dl = *reinterpret_cast<const f32x4*>(&sh.stat[cur][1][acc_row(4 * q4, lane)]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 4 * q4 + e;
            s[r] = pr[e] * (s[r] - dl[e]);
            if (part) {
              const int lo = lo_s[acc_row(r, lane)], hi = hi_s[acc_row(r, lane)];
              if (key < lo || key >= hi || hi - lo == 1) s[r] = 0.f;  // (a row of one key has no score gradient)
            }
          }
        }
      }
      const float* tile = dk_role ? sh.Q[cur] : sh.O[cur];
      if (SEEN && part)
        sums_seen<D>(acc, s, tile, lane, d, [&](int c) {
          return (uint32_t)__builtin_amdgcn_ballot_w64(kw + c >= lo_s[lane & 31] && kw + c < hi_s[lane & 31]);
        });
      else sums<D>(acc, s, tile, lane, d);
    }
    if (QG > 1) __syncthreads();  // its own stage is free
    put(it + QG, QG == 1 ? cur ^ 1 : grp);
    __syncthreads();
  }
  if (!SEEN && __syncthreads_or(bad)) return true;
  if constexpr (QG > 1) {
    // the other pairs' sums, lane to lane, in the stages that were theirs; added in order
    static_assert(D / 2 * 64 <= BLK * LD<D>, "the hand-over does not fit");
    float* mine = (dk_role ? sh.Q : sh.O)[pair] + lane;
    if (pair > 0) {
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) mine[(dt * 16 + r) * 64] = acc[dt][r];
    }
    __syncthreads();
    if (pair > 0) return false;
#pragma unroll 1
    for (int g = 1; g < QG; ++g) {
      const float* from = (dk_role ? sh.Q : sh.O)[g] + lane;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[dt][r] += from[(dt * 16 + r) * 64];
    }
  }
  // a share of several: its plane, [split][dk, dv][token][key / value head][d]
  const size_t width = (size_t)a.N_kv * d, plane = (size_t)a.S_mb * S * width, ldg = a.splits > 1 ? width : dk_role ? a.ldk : a.ldv;
  float* out = a.splits > 1 ? a.planes + (2 * (size_t)split + (dk_role ? 0 : 1)) * plane : (float*)(dk_role ? a.dk : a.dv);
  store_row<D, VEC>(acc, rows_at(out + (seq + kw) * ldg + (size_t)kv * d, row_bytes(S - kw, ldg, d)), (uint32_t)((lane & 31) * ldg) * 4, lane,
                    dk_role ? a.scale : 1.f, d);
  return false;
}

template <int D, int QG, bool VEC, bool CAP>
__device__ __attribute__((noinline)) void key_rows_seen(MaskedArgs a, KeyShared<D, QG>& sh) {
  key_rows<D, QG, VEC, CAP, true>(a, sh);
}

template <int D, int QG, bool VEC, bool CAP>
__global__ __launch_bounds__(NTHR_DKV, 2) void masked_key_f32_kernel(MaskedArgs a) {
  __shared__ __attribute__((aligned(16))) KeyShared<D, QG> sh;
  if (key_rows<D, QG, VEC, CAP, false>(a, sh)) {
    __syncthreads();
    key_rows_seen<D, QG, VEC, CAP>(a, sh);
  }
}

__global__ __launch_bounds__(256) void masked_join_f32_kernel(MaskedArgs a) {
  const size_t width = (size_t)a.N_kv * a.S_head, plane = (size_t)a.S_mb * a.S_seq * width, n = 2 * plane;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
    float t = 0.f;
    for (int k = 0; k < a.splits; ++k) t += a.planes[(size_t)k * n + i];
    const bool v = i >= plane;
    const size_t e = v ? i - plane : i, row = e / width, c = e - row * width;
    if (v) ((float*)a.dv)[row * a.ldv + c] = t;
    else ((float*)a.dk)[row * a.ldk + c] = t;
  }
}

// Workgroups of 128 rows below which the rows' keys (the keys' queries) are shared out over the waves instead
constexpr unsigned FEW = 192;

template <int D, bool VEC, bool CAP, bool GRAD>
void query(const MaskedArgs& a, hipStream_t st) {
  const unsigned hb = (unsigned)(a.N_heads * a.S_mb), grid = (unsigned)((a.S_seq + ROWS - 1) / ROWS) * hb;
  if (grid < FEW) masked_query_f32_kernel<D, 4, VEC, CAP, GRAD><<<(unsigned)((a.S_seq + 31) / 32) * hb, 256, 0, st>>>(a);
  else masked_query_f32_kernel<D, 1, VEC, CAP, GRAD><<<grid, 256, 0, st>>>(a);
}

template <int D, bool VEC, bool CAP>
void run(const MaskedArgs& a, bool backward, hipStream_t st) {
  if (!backward) { query<D, VEC, CAP, false>(a, st); return; }
  query<D, VEC, CAP, true>(a, st);
  const unsigned hb = (unsigned)(a.N_kv * a.splits * a.S_mb), grid = (unsigned)((a.S_seq + ROWS - 1) / ROWS) * hb;
  if (grid < FEW) masked_key_f32_kernel<D, 4, VEC, CAP><<<(unsigned)((a.S_seq + 31) / 32) * hb, NTHR_DKV, 0, st>>>(a);
  else masked_key_f32_kernel<D, 1, VEC, CAP><<<grid, NTHR_DKV, 0, st>>>(a);
  if (a.splits > 1) masked_join_f32_kernel<<<2048, 256, 0, st>>>(a);
}

template <int D, bool VEC>
void by_score(const MaskedArgs& a, bool backward, hipStream_t st) {
  if (a.cap > 0.f) run<D, VEC, true>(a, backward, st);
  else run<D, VEC, false>(a, backward, st);
}

bf_status both(const MaskedArgs& a, bool backward, hipStream_t st) {
  if (a.S_head <= 64) a.vec ? by_score<64, true>(a, backward, st) : by_score<64, false>(a, backward, st);
  else a.vec ? by_score<128, true>(a, backward, st) : by_score<128, false>(a, backward, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_error("attention_masked_f32: launch failed: %s", hipGetErrorString(e)); return BF_EDEVICE; }
  return BF_OK;
}

}  // namespace

bf_status attention_masked_fwd_f32(const MaskedArgs& a, hipStream_t st) { return both(a, false, st); }
bf_status attention_masked_bwd_f32(const MaskedArgs& a, hipStream_t st) { return both(a, true, st); }

}  // namespace bf
