// Products of 8-bit operands with a power-of-two scale for each 128 elements along the contraction:
//
//   C[m,n] = sum over blocks b of 2^(sa[b,m] - 127) 2^(sb[b,n] - 127) sum over k in block b of A[m,k] B[n,k]
//
// Both operands are K-contiguous and whole blocks long (see fp8.hip), so forward, input-gradient and weight-gradient products
// of a linear layer are this one layout on forms quantised along the right axis.
//
// bf16 results: v_mfma_scale_f32_16x16x128_f8f6f4.  One instruction takes a block of 16 rows by 16 columns with one scale byte per
// row and column, so the block scales cost no arithmetic.  The accumulators are fp32, but the instruction lines the products of
// a few neighbouring k up before it adds them and drops what falls under them: 1.5e-5 (2-norm, over the result's) on normal
// operands, 8e-5 with outliers of 20 sigma in every block, whatever the length, and the same from the 16x16x32 form: 50 times under
// bf16's own rounding.  fp32 results (main-grads) are held to more than that: their operands are widened in registers to bf16, which holds
// code times scale exactly, and multiplied by v_mfma_f32_16x16x32_bf16 at half the rate.
//
// A workgroup computes BM x BN of C in steps of one block (128 bytes of a row).  Tiles go from memory straight into LDS (16 bytes a lane,
// two stages).  Within an LDS row the 16-byte chunks are XOR-swizzled (conflict-free fragment reads); as the instruction
// that loads into LDS writes lane after lane, the swizzle is in the addresses that the lanes read from.  Any order of k is right as long as
// A and B share it and a block's scale covers it: lane group q takes chunks q and q + 4.
// LDS row 16 i + j of a group of 16 G rows (G = 4: 64 rows) holds row G j + i of it: a lane's scale bytes of G fragments are then
// neighbours in memory (one load, picked apart by the instruction's byte selector), and so are its results of G fragments across (one store).
#include <atomic>
#include <type_traits>

#include "../../include/bf_ops.h"
#include "common.h"

namespace bf {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;

constexpr int BKB = 128;  // bytes of a row per step: one block

struct Fp8Args {
  int M, N, blocks;            // blocks: of the contraction
  const uint8_t *A, *B;        // rows of 128 * blocks bytes
  const uint8_t *sa, *sb;      // [blocks][ldsa], [blocks][ldsb]
  int ldsa, ldsb;
  void* C;
  const float* bias;
  const void* R;
  int accumulate;
  int tiles_m, remap, slice;   // slice: blocks that a workgroup takes; grid.y slices, slice y into plane y of C
};

template <int BM_, int BN_, int WM_, int WN_>
struct Tile8 {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NT = WM * WN * 64;
  static constexpr int TM = BM / WM, TN = BN / WN, MI = TM / 16, NI = TN / 16;
  static constexpr int GA = MI < 4 ? MI : 4, GB = NI < 4 ? NI : 4;  // fragments that share a load of scale bytes
  static constexpr int CA = BM * 8 / NT, CB = BN * 8 / NT;          // 16-byte chunks of a thread
};

// XOR key of an LDS row of 8 chunks: the 16 lanes that a 16-byte read serves in a cycle are quads of lanes 0, 3, 5, 6 (or the others) of a
// half wave, and the key sends their rows to different chunks (bank conflicts measured: none)
__device__ __forceinline__ int kswz8(int row) {
  return ((row >> 1) & 1) | (((row >> 3) & 1) << 1) | ((((row >> 2) ^ (row >> 3)) & 1) << 2);
}

// row of the tile that LDS row r holds
template <int G>
__device__ __forceinline__ int row_of(int r) { return (r / (16 * G)) * (16 * G) + (r % 16) * G + (r / 16) % G; }

template <int G>
__device__ __forceinline__ int load_scales(const uint8_t* p) {
  if constexpr (G == 4) return *reinterpret_cast<const int*>(p);
  else if constexpr (G == 2) return *reinterpret_cast<const uint16_t*>(p);
  else return *p;
}

template <int SEL_A, int SEL_B, int FA, int FB>
__device__ __forceinline__ f32x4 mma_scaled(v8i a, v8i b, f32x4 c, int sa, int sb) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, FA, FB, SEL_A, sa, SEL_B, sb);
}

template <int I, int N, typename F>
__device__ __forceinline__ void unrolled(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    unrolled<I + 1, N>(f);
  }
}

// 16 codes -> 16 bf16 times 2^e (exact)
template <int FMT>
__device__ __forceinline__ void widen(v4i v, float unit, bf16x8 (&o)[2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    bf16x2 p[4];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      if constexpr (FMT == BF_E4M3) {
        p[2 * w] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * h + w], unit, false);
        p[2 * w + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * h + w], unit, true);
      } else {
        p[2 * w] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(v[2 * h + w], unit, false);
        p[2 * w + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(v[2 * h + w], unit, true);
      }
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) { o[h][2 * w] = p[w][0]; o[h][2 * w + 1] = p[w][1]; }
  }
}

// Adds the epilogue's terms to G neighbouring results and stores them.
template <int G, typename TO>
__device__ __forceinline__ void put(float (&v)[G], int row, int col, const Fp8Args& p, TO* C, bool vec) {
  if (row >= p.M || col >= p.N) return;
  const size_t at = (size_t)row * p.N + col;
  const TO* R = reinterpret_cast<const TO*>(p.R);
  if (vec) {  // N is a multiple of G and the tensors are aligned to G elements: whole groups
    typedef TO V __attribute__((ext_vector_type(G)));
    if (p.bias) {
#pragma unroll
      for (int e = 0; e < G; ++e) v[e] += p.bias[col + e];
    }
    if (R) {
      const V r = *reinterpret_cast<const V*>(R + at);
#pragma unroll
      for (int e = 0; e < G; ++e) v[e] += (float)r[e];
    }
    if (p.accumulate) {
      const V r = *reinterpret_cast<const V*>(C + at);
#pragma unroll
      for (int e = 0; e < G; ++e) v[e] += (float)r[e];
    }
    V o;
#pragma unroll
    for (int e = 0; e < G; ++e) o[e] = (TO)v[e];
    *reinterpret_cast<V*>(C + at) = o;
    return;
  }
#pragma unroll
  for (int e = 0; e < G; ++e) {
    if (col + e >= p.N) continue;
    float x = v[e];
    if (p.bias) x += p.bias[col + e];
    if (R) x += (float)R[at + e];
    if (p.accumulate) x += (float)C[at + e];
    C[at + e] = (TO)x;
  }
}

// WIDE: bf16 instructions on widened operands.
template <typename TL, int FA, int FB, bool WIDE, typename TO>
__global__ __launch_bounds__(TL::NT) void gemm_fp8_kernel(Fp8Args p) {
#ifdef __HIP_DEVICE_COMPILE__  // (the host's pass drops the whole kernel over the builtins that load into LDS)
  constexpr int BM = TL::BM, BN = TL::BN, NT = TL::NT, MI = TL::MI, NI = TL::NI, GA = TL::GA, GB = TL::GB, CA = TL::CA, CB = TL::CB;
  // (two arrays and not one: the compiler then knows that reads of a stage need not wait for loads into the other)
  __shared__ __attribute__((aligned(128))) uint8_t stage0[(BM + BN) * BKB];
  __shared__ __attribute__((aligned(128))) uint8_t stage1[(BM + BN) * BKB];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w % TL::WM, wn = w / TL::WM;

  // each XCD (its own L2) a contiguous range of the tile order, which walks groups of 8 row-tiles
  int lin = blockIdx.x;
  if (p.remap) lin = (lin & 7) * (gridDim.x >> 3) + (lin >> 3);
  const int tiles_n = gridDim.x / p.tiles_m;
  int bm, bn;
  if (p.remap && p.tiles_m % 8 == 0) {
    const int in_group = 8 * tiles_n, gi = lin / in_group, rem = lin % in_group;
    bm = gi * 8 + (rem & 7);
    bn = rem >> 3;
  } else {
    bm = lin % p.tiles_m;
    bn = lin / p.tiles_m;
  }
  const int m0 = bm * BM, n0 = bn * BN;
  const int kb0 = blockIdx.y * p.slice, nk = min(p.slice, p.blocks - kb0);
  const size_t ld = (size_t)p.blocks * BKB;
  const uint8_t *ga = p.A + (size_t)m0 * ld + (size_t)kb0 * BKB, *gb = p.B + (size_t)n0 * ld + (size_t)kb0 * BKB;
  TO* C = reinterpret_cast<TO*>(p.C) + (size_t)blockIdx.y * p.M * p.N;

  // Lanes whose row lies behind the matrix read its last row instead: what they compute is not stored.
  const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc((void*)ga, 0, 0x7fffffff, 0x00020000);
  const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc((void*)gb, 0, 0x7fffffff, 0x00020000);
  int off_a[CA], off_b[CB];
#pragma unroll
  for (int i = 0; i < CA; ++i) {
    const int c = i * NT + tid, r = c >> 3, ch = (c & 7) ^ kswz8(r);
    off_a[i] = min(row_of<GA>(r), p.M - 1 - m0) * (int)ld + ch * 16;
  }
#pragma unroll
  for (int i = 0; i < CB; ++i) {
    const int c = i * NT + tid, r = c >> 3, ch = (c & 7) ^ kswz8(r);
    off_b[i] = min(row_of<GB>(r), p.N - 1 - n0) * (int)ld + ch * 16;
  }
  typedef __attribute__((address_space(3))) void* lds_ptr;
  auto issue = [&](uint8_t* st, int kt) {
#pragma unroll
    for (int i = 0; i < CA; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr)(st + (i * NT + w * 64) * 16), 16, off_a[i], kt * BKB, 0, 0);
#pragma unroll
    for (int i = 0; i < CB; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_ptr)(st + BM * BKB + (i * NT + w * 64) * 16), 16, off_b[i], kt * BKB, 0, 0);
  };
  // scale bytes of the lane's rows / columns, G to a load
  constexpr int SA = MI / GA, SB = NI / GB;
  const uint8_t *psa = p.sa + (size_t)kb0 * p.ldsa, *psb = p.sb + (size_t)kb0 * p.ldsb;
  int oa[SA], ob[SB];
#pragma unroll
  for (int s = 0; s < SA; ++s) oa[s] = min(m0 + wm * TL::TM + s * 16 * GA + (lane & 15) * GA, p.ldsa - GA);
#pragma unroll
  for (int s = 0; s < SB; ++s) ob[s] = min(n0 + wn * TL::TN + s * 16 * GB + (lane & 15) * GB, p.ldsb - GB);
  int sca[SA], scb[SB], nsa[SA], nsb[SB];
  auto scales = [&](int kt, int (&a)[SA], int (&b)[SB]) {
    const uint8_t *qa = psa + (size_t)kt * p.ldsa, *qb = psb + (size_t)kt * p.ldsb;
#pragma unroll
    for (int s = 0; s < SA; ++s) a[s] = load_scales<GA>(qa + oa[s]);
#pragma unroll
    for (int s = 0; s < SB; ++s) b[s] = load_scales<GB>(qb + ob[s]);
  };

  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};

  // a fragment's address: lane part (one per chunk) plus a compile-time multiple of 16 rows
  int fo[2];
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) fo[kk] = (lane & 15) * BKB + (((kk * 4 + (lane >> 4)) ^ kswz8(lane & 15)) << 4);
  const int fa = wm * TL::TM * BKB, fb = BM * BKB + wn * TL::TN * BKB;
  auto chunk = [&](const uint8_t* st, int base, int t, int kk) { return *reinterpret_cast<const v4i*>(st + base + t * 16 * BKB + fo[kk]); };
  auto arrived = [] {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };

  issue(stage0, 0);
  scales(0, sca, scb);
  if constexpr (WIDE) {
    // One barrier per block: behind it the tile is there and the other stage is free.
    auto body = [&](uint8_t* cur, uint8_t* nxt, int kt) {
      arrived();
      if (kt + 1 < nk) {
        issue(nxt, kt + 1);
        scales(kt + 1, nsa, nsb);
      }
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        bf16x8 b[NI][2];
        unrolled<0, NI>([&](auto j) {
          const int e = (scb[j / GB] >> (8 * (j % GB))) & 255;
          widen<FB>(chunk(cur, fb, j, kk), __int_as_float(e << 23), b[j]);
        });
        unrolled<0, MI>([&](auto i) {
          const int e = (sca[i / GA] >> (8 * (i % GA))) & 255;
          bf16x8 a[2];
          widen<FA>(chunk(cur, fa, i, kk), __int_as_float(e << 23), a);
#pragma unroll
          for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[h], b[j][h], acc[i][j], 0, 0, 0);
        });
      }
#pragma unroll
      for (int s = 0; s < SA; ++s) sca[s] = nsa[s];
#pragma unroll
      for (int s = 0; s < SB; ++s) scb[s] = nsb[s];
    };
    for (int kt = 0; kt < nk; kt += 2) {
      body(stage0, stage1, kt);
      if (kt + 1 < nk) body(stage1, stage0, kt + 1);
    }
  } else {
    // Four phases to a block, each a half of the wave's A fragments times a half of its B fragments; what the next phase needs
    // is fetched meanwhile.  By the end of the second phase everything of the stage is in registers: the barrier stands
    // there, the loads of the block after next go into the stage behind it, and the last two phases fetch the next block's first halves.
    // (The halves of B swap roles from block to block, so that the one that is fetched first is free.)
    constexpr int MH = MI / 2, NH = NI / 2;
    static_assert(MI % 2 == 0 && NI % 2 == 0, "halves");
    v8i a0[MH], a1[MH], bx[2][NH];
    auto whole = [&](const uint8_t* st, int base, int t) {
      const v4i x = chunk(st, base, t, 0), y = chunk(st, base, t, 1);
      return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto get_a = [&](const uint8_t* st, int half, v8i (&f)[MH]) {
#pragma unroll
      for (int i = 0; i < MH; ++i) f[i] = whole(st, fa, half * MH + i);
    };
    auto get_b = [&](const uint8_t* st, int half) {
#pragma unroll
      for (int j = 0; j < NH; ++j) bx[half][j] = whole(st, fb, half * NH + j);
    };
    auto mma = [&](auto ha, auto hb, v8i (&f)[MH]) {
      unrolled<0, MH>([&](auto i) {
        unrolled<0, NH>([&](auto jj) {
          constexpr int I = decltype(i)::value, J = I & 1 ? NH - 1 - decltype(jj)::value : decltype(jj)::value;  // serpentine: one operand changes
          constexpr int TI = decltype(ha)::value * MH + I, TJ = decltype(hb)::value * NH + J;
          acc[TI][TJ] = mma_scaled<TI % GA, TJ % GB, FA, FB>(f[I], bx[decltype(hb)::value][J], acc[TI][TJ], sca[TI / GA], scb[TJ / GB]);
        });
      });
    };
    typedef std::integral_constant<int, 0> H0;
    typedef std::integral_constant<int, 1> H1;
    // one phase's instructions in turn: an MFMA, then a share of the reads from LDS (0x100)
    auto interleave = [&](auto reads) {
      constexpr int NMMA = MH * NH, NR = decltype(reads)::value, PER = (NR + NMMA - 1) / NMMA;
#pragma unroll
      for (int i = 0; i < NMMA; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (i * PER < NR) __builtin_amdgcn_sched_group_barrier(0x100, PER, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    typedef std::integral_constant<int, 2 * MH> RA;
    typedef std::integral_constant<int, 2 * NH> RB;
    auto body = [&](uint8_t* cur, uint8_t* nxt, int kt, auto first, auto second) {
      constexpr int F = decltype(first)::value, S = decltype(second)::value;
      if (kt + 1 < nk) scales(kt + 1, nsa, nsb);
      get_b(cur, S);
      mma(H0{}, first, a0);
      interleave(RB{});
      get_a(cur, 1, a1);
      mma(H0{}, second, a0);
      interleave(RA{});
      arrived();
      if (kt + 2 < nk) issue(cur, kt + 2);
      get_a(nxt, 0, a0);
      mma(H1{}, second, a1);
      interleave(RA{});
      get_b(nxt, S);
      mma(H1{}, first, a1);
      interleave(RB{});
#pragma unroll
      for (int s = 0; s < SA; ++s) sca[s] = nsa[s];
#pragma unroll
      for (int s = 0; s < SB; ++s) scb[s] = nsb[s];
    };
    arrived();
    if (nk > 1) issue(stage1, 1);
    get_a(stage0, 0, a0);
    get_b(stage0, 0);
    for (int kt = 0; kt < nk; kt += 2) {
      body(stage0, stage1, kt, H0{}, H1{});
      if (kt + 1 < nk) body(stage1, stage0, kt + 1, H1{}, H0{});
    }
  }

  // lane l, register r of a fragment: row 4 (l / 16) + r, column l % 16 of it
  const bool vec = p.N % GB == 0 && (((uintptr_t)p.C | (uintptr_t)p.R) & (GB * sizeof(TO) - 1)) == 0;
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = m0 + wm * TL::TM + i / GA * 16 * GA + (4 * (lane >> 4) + r) * GA + i % GA;
#pragma unroll
      for (int s = 0; s < SB; ++s) {
        float v[GB];
#pragma unroll
        for (int e = 0; e < GB; ++e) v[e] = acc[i][s * GB + e][r];
        put<GB, TO>(v, row, n0 + wn * TL::TN + s * 16 * GB + (lane & 15) * GB, p, C, vec);
      }
    }
#endif
}

// C = the sum of the slices' planes in ascending order, and the epilogue
template <typename TO>
__global__ __launch_bounds__(256) void fp8_finish_kernel(size_t n, int N, int slices, const float* __restrict__ planes, TO* __restrict__ C,
                                                         const float* __restrict__ bias, const TO* __restrict__ R, int accumulate) {
  const size_t stride = (size_t)gridDim.x * 256;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += stride) {
    float x = 0.f;
#pragma unroll 4
    for (int s = 0; s < slices; ++s) x += planes[(size_t)s * n + i];
    if (bias) x += bias[i % N];
    if (R) x += (float)R[i];
    if (accumulate) x += (float)C[i];
    C[i] = (TO)x;
  }
}

typedef Tile8<256, 256, 2, 4> Big8;
typedef Tile8<256, 256, 2, 4> Wide8;  // widened operands: smaller sub-tiles, two waves to a SIMD
typedef Tile8<128, 128, 2, 2> Mid8;
typedef Tile8<64, 64, 2, 2> Small8;

struct Plan { int tile, slices, slice; };  // tile 0: 256 x 256, 1: 128 x 128, 2: 64 x 64

Plan plan_of(int M, int N, int blocks) {
  auto tiles = [&](int e) { return (long)((M + e - 1) / e) * ((N + e - 1) / e); };
  Plan q{tiles(256) >= 192 ? 0 : tiles(128) >= 256 ? 1 : 2, 1, blocks};
  if (q.tile == 2 && tiles(64) < 512 && blocks >= 8) {
    const long want = 1024 / tiles(64), most = blocks / 4;
    const int s = (int)(want < most ? want : most);
    if (s > 1) {
      q.slice = (blocks + s - 1) / s;
      q.slices = (blocks + q.slice - 1) / q.slice;
    }
  }
  return q;
}

template <typename TL, int FA, int FB, bool WIDE, typename TO>
bf_status launch8(Fp8Args a, int slices, hipStream_t st) {
  a.tiles_m = (a.M + TL::BM - 1) / TL::BM;
  const long tiles = (long)a.tiles_m * ((a.N + TL::BN - 1) / TL::BN);
  if (tiles * TL::NT >= (1l << 32)) { set_error("bf_op_fp8_gemm: more than 2^32 threads"); return BF_EINVAL; }
  a.remap = tiles % 8 == 0;
  gemm_fp8_kernel<TL, FA, FB, WIDE, TO><<<dim3((unsigned)tiles, (unsigned)slices), TL::NT, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_error("bf_op_fp8_gemm: launch failed: %s", hipGetErrorString(e)); return BF_EDEVICE; }
  return BF_OK;
}

template <int FA, int FB>
bf_status by_tile(const Fp8Args& a, int tile, int slices, bool wide, bool f32, hipStream_t st) {
  if (wide) switch (tile) {
    case 0: return launch8<Wide8, FA, FB, true, float>(a, slices, st);
    case 1: return launch8<Mid8, FA, FB, true, float>(a, slices, st);
    default: return launch8<Small8, FA, FB, true, float>(a, slices, st);
  }
  if (f32) return launch8<Small8, FA, FB, false, float>(a, slices, st);  // planes
  switch (tile) {
    case 0: return launch8<Big8, FA, FB, false, bf16_t>(a, slices, st);
    case 1: return launch8<Mid8, FA, FB, false, bf16_t>(a, slices, st);
    default: return launch8<Small8, FA, FB, false, bf16_t>(a, slices, st);
  }
}

bool sizes_ok(int M, int N, int K) { return M >= 1 && N >= 1 && K >= 1 && M <= (1 << 21) && N <= (1 << 21) && K <= (1 << 21); }

}  // namespace

size_t fp8_gemm_work_bytes(int M, int N, int K) {
  if (!sizes_ok(M, N, K)) return 0;
  const Plan q = plan_of(M, N, (K + 127) / 128);
  return q.slices > 1 ? (size_t)q.slices * M * N * sizeof(float) : 0;
}

bf_status fp8_gemm(int fa, int fb, int dtype, int M, int N, int K, const void* A, const void* sa, const void* B, const void* sb, void* C, const float* bias,
                   const void* R, int accumulate, void* work, size_t work_bytes, hipStream_t st) {
  if ((fa != BF_E4M3 && fa != BF_E5M2) || (fb != BF_E4M3 && fb != BF_E5M2)) { set_error("bf_op_fp8_gemm: unknown format %d, %d", fa, fb); return BF_EINVAL; }
  if (!sizes_ok(M, N, K)) { set_error("bf_op_fp8_gemm: sizes are 1 to 2^21, got %d x %d x %d", M, N, K); return BF_EINVAL; }
  const size_t es = dtype == BF_BF16 ? 2 : 4;
  if (!A || !B || !sa || !sb || !C) { set_error("bf_op_fp8_gemm: null operand"); return BF_EINVAL; }
  if ((((uintptr_t)A | (uintptr_t)B | (uintptr_t)sa | (uintptr_t)sb) & 15) || (((uintptr_t)C | (uintptr_t)R) & (es - 1)) || ((uintptr_t)bias & 3)) {
    set_error("bf_op_fp8_gemm: codes and scales have to be 16-byte aligned, other tensors to their elements");
    return BF_EINVAL;
  }
  if (accumulate && dtype != BF_FP32) { set_error("bf_op_fp8_gemm: accumulates into fp32 only"); return BF_EINVAL; }
  const int blocks = (K + 127) / 128;
  const Plan q = plan_of(M, N, blocks);
  const bool wide = dtype == BF_FP32, split = q.slices > 1;
  if (split && (!work || ((uintptr_t)work & 255) || work_bytes < (size_t)q.slices * M * N * sizeof(float))) {
    set_error("bf_op_fp8_gemm: needs %zu bytes of 256-byte aligned scratch", (size_t)q.slices * M * N * sizeof(float));
    return BF_EINVAL;
  }
  Fp8Args a{M, N, blocks, (const uint8_t*)A, (const uint8_t*)B, (const uint8_t*)sa, (const uint8_t*)sb, (M + 15) / 16 * 16, (N + 15) / 16 * 16, C, bias, R,
            accumulate, 0, 0, q.slice};
  if (split) {
    a.C = work;
    a.bias = nullptr;
    a.R = nullptr;
    a.accumulate = 0;
  }
  bf_status s;
  if (fa == BF_E4M3) s = fb == BF_E4M3 ? by_tile<0, 0>(a, q.tile, q.slices, wide, split, st) : by_tile<0, 1>(a, q.tile, q.slices, wide, split, st);
  else s = fb == BF_E4M3 ? by_tile<1, 0>(a, q.tile, q.slices, wide, split, st) : by_tile<1, 1>(a, q.tile, q.slices, wide, split, st);
  if (s != BF_OK || !split) return s;
  const size_t n = (size_t)M * N;
  const unsigned grid = (unsigned)((n + 255) / 256 < 4096 ? (n + 255) / 256 : 4096);
  if (dtype == BF_BF16)
    fp8_finish_kernel<bf16_t><<<grid, 256, 0, st>>>(n, N, q.slices, (const float*)work, (bf16_t*)C, bias, (const bf16_t*)R, accumulate);
  else fp8_finish_kernel<float><<<grid, 256, 0, st>>>(n, N, q.slices, (const float*)work, (float*)C, bias, (const float*)R, accumulate);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_error("bf_op_fp8_gemm: launch failed: %s", hipGetErrorString(e)); return BF_EDEVICE; }
  return BF_OK;
}

}  // namespace bf
