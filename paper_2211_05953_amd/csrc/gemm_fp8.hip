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
// code times scale exactly (down to 2^-133, its smallest step), and multiplied by v_mfma_f32_16x16x32_bf16 at half the rate.
//
// A workgroup computes BM x BN of C in steps of one block (128 bytes of a row).  Tiles go from memory straight into LDS (16 bytes a lane,
// two or four stages).  Within an LDS row the 16-byte chunks are XOR-swizzled (conflict-free fragment reads); as the instruction
// that loads into LDS writes lane after lane, the swizzle is in the addresses that the lanes read from.  Any order of k is right as long as
// A and B share it and a block's scale covers it: lane group q takes chunks q and q + 4.
// LDS row 16 i + j of a group of 16 G rows (G = 4: 64 rows) holds row G j + i of it: a lane's scale bytes of G fragments are then
// neighbours in memory (one load, picked apart by the instruction's byte selector), and so are its results of G fragments across (one store).
//
// Large bf16 results: 8192^3 348 us, 3.2 PFLOP/s; 2048 x 32768 x 8192 361, 3.0; 8192 x 32768 x 2048 427, 2.6 (half a gigabyte of results).  Instructions on registers alone reach 4.05 on
// random operands (4.9 on zeros: the clock falls with the power); matrix cores are busy 76 to 80 % at 1.89 to 1.79 GHz, and LDS has no bank conflicts.  fp32: 8192 x 8192 x 2048 213 us, 1.29.
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
  int tiles_m, slice;          // slice: blocks that a workgroup takes; grid.y slices, slice y into plane y of C
  int passing;                 // C does not stay in the caches
};

template <int BM_, int BN_, int WM_, int WN_, int NS_ = 2>
struct Tile8 {
  static constexpr int NS = NS_;  // stages
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
__host__ __device__ __forceinline__ constexpr int row_of(int r) { return (r / (16 * G)) * (16 * G) + (r % 16) * G + (r / 16) % G; }

template <int G>
__device__ __forceinline__ int load_scales(const uint8_t* p) {
  if constexpr (G == 4) return *reinterpret_cast<const int*>(p);
  else if constexpr (G == 2) return *reinterpret_cast<const uint16_t*>(p);
  else return *p;
}

// c += a b with scales, c in place.  (Written out: from the builtin the compiler gives accumulators new registers, and a 128 x 128 sub-tile, whose
// accumulators are half of all registers there are, spends as long on moving them as on products.)
template <int SEL_A, int SEL_B, int FA, int FB>
__device__ __forceinline__ void mma_scaled(const v8i& a, const v8i& b, f32x4& c, int sa, int sb) {
  asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%c5,%c6,0] op_sel_hi:[%c7,%c8,0] cbsz:%c9 blgp:%c10"
               : "+a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb), "n"(SEL_A & 1), "n"(SEL_B & 1), "n"(SEL_A >> 1), "n"(SEL_B >> 1), "n"(FA), "n"(FB));
}

template <int I, int N, typename F>
__device__ __forceinline__ void unrolled(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    unrolled<I + 1, N>(f);
  }
}

// Codes 2 n, 2 n + 1 of eight (two registers) as bf16 times 2^e (exact down to 2^-133), into place n of o
template <int FMT>
__device__ __forceinline__ void widen2(int lo, int hi, float unit, int n, bf16x8& o) {
  bf16x2 p;
  if constexpr (FMT == BF_E4M3) p = n & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(n < 2 ? lo : hi, unit, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(n < 2 ? lo : hi, unit, false);
  else p = n & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(n < 2 ? lo : hi, unit, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(n < 2 ? lo : hi, unit, false);
  o[2 * n] = p[0];
  o[2 * n + 1] = p[1];
}

__device__ __forceinline__ void mma_bf16(const bf16x8& a, const bf16x8& b, f32x4& c) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}

// n neighbouring elements by one load or store; lanes behind the descriptor's end read zero and write nothing.  AUX 2: past the caches
template <int BYTES>
__device__ __forceinline__ auto load_some(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  if constexpr (BYTES == 2) return __builtin_amdgcn_raw_buffer_load_b16(r, off, 0, 0);
  else if constexpr (BYTES == 4) return __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0);
  else if constexpr (BYTES == 8) return __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0);
  else return __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0);
}
template <int AUX, typename V>
__device__ __forceinline__ void store_some(__amdgpu_buffer_rsrc_t r, uint32_t off, V v) {
  if constexpr (sizeof(V) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), r, off, 0, AUX);
  else if constexpr (sizeof(V) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), r, off, 0, AUX);
  else if constexpr (sizeof(V) == 8) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(decltype(load_some<8>(r, off)), v), r, off, 0, AUX);
  else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(decltype(load_some<16>(r, off)), v), r, off, 0, AUX);
}

// WIDE: bf16 instructions on widened operands.
template <typename TL, int FA, int FB, bool WIDE, typename TO>
__global__ __launch_bounds__(TL::NT) void gemm_fp8_kernel(Fp8Args p) {
#ifdef __HIP_DEVICE_COMPILE__  // (the host's pass drops the whole kernel over the builtins that load into LDS)
  static_assert((TL::NT & (TL::NT - 1)) == 0, "a power of two");
  constexpr int BM = TL::BM, BN = TL::BN, NT = TL::NT, MI = TL::MI, NI = TL::NI, GA = TL::GA, GB = TL::GB, CA = TL::CA, CB = TL::CB;
  // (an array for each and not one: the compiler then knows that reads of a stage need not wait for loads into the others)
  constexpr int NS = TL::NS, STAGE = (BM + BN) * BKB + 512;
  static_assert(NS == 2 || NS == 4, "two or four stages");
  __shared__ __attribute__((aligned(128))) uint8_t stage0[STAGE];
  __shared__ __attribute__((aligned(128))) uint8_t stage1[STAGE];
  __shared__ __attribute__((aligned(128))) uint8_t stage2[NS == 4 ? STAGE : 16];
  __shared__ __attribute__((aligned(128))) uint8_t stage3[NS == 4 ? STAGE : 16];
  auto stage = [&](auto i) __attribute__((always_inline)) -> uint8_t* {
    constexpr int S = decltype(i)::value % NS;
    if constexpr (S == 0) return stage0;
    else if constexpr (S == 1) return stage1;
    else if constexpr (S == 2) return stage2;
    else return stage3;
  };
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w % TL::WM, wn = w / TL::WM;

  // Each XCD (its own L2) a contiguous range of the tile order, which walks groups of 8 tiles of the longer side along the shorter one: the larger operand is fetched once.  (2048 x 32768 x 8192
  // 376 us, groups of the rows 391; 8192 x 32768 x 1024 285 and 319; groups of 4 the same on average, of 2 slower.)
  const int tiles_n = gridDim.x / p.tiles_m;
  const bool across = tiles_n > p.tiles_m;
  const int len = across ? tiles_n : p.tiles_m, width = across ? p.tiles_m : tiles_n;
  const int xcd = blockIdx.x & 7, lin = (int)(blockIdx.x >> 3) + xcd * (int)(gridDim.x >> 3) + min(xcd, (int)(gridDim.x & 7));
  const int group = lin / (8 * width), rem = lin - group * 8 * width, size = min(8, len - group * 8), along = group * 8 + rem % size, other = rem / size;
  const int bm = across ? other : along, bn = across ? along : other;
  const int m0 = bm * BM, n0 = bn * BN;
  const int kb0 = blockIdx.y * p.slice, nk = min(p.slice, p.blocks - kb0);
  const size_t ld = (size_t)p.blocks * BKB;
  TO* C = reinterpret_cast<TO*>(p.C) + (size_t)blockIdx.y * p.M * p.N;

  // What is loaded: a tile's operands by 32-bit lane offsets from its first byte.  The descriptors end where the matrices end, and lanes whose row lies
  // behind it get nothing: what they compute is not stored.
  typedef __attribute__((address_space(3))) void* lds_ptr;
  auto rest = [&](int rows) __attribute__((always_inline)) {
    const size_t n = (size_t)rows * ld - (size_t)kb0 * BKB;
    return (int)(n < 0x7fffff00u ? n : 0x7fffff00u);
  };
  const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc((void*)(p.A + (size_t)m0 * ld + (size_t)kb0 * BKB), 0, rest(p.M - m0), 0x00020000);
  const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc((void*)(p.B + (size_t)n0 * ld + (size_t)kb0 * BKB), 0, rest(p.N - n0), 0x00020000);
  int sld = w & 1 ? p.ldsb : p.ldsa;
  const uint8_t* sp = (w & 1 ? p.sb : p.sa) + (size_t)kb0 * sld;
  asm("" : "+s"(sld), "+s"(sp));  // held in registers: a load of arguments in the loop would wait for everything that is read from LDS
  const int off_s = min((w & 1 ? n0 : m0) + 4 * lane, sld - 4);
  // chunk i of a thread is NT / 8 LDS rows, a power of two, further on: the bits of row_of are those of the two parts
  const int ch = (tid & 7) ^ kswz8(tid >> 3);
  const int off_a = row_of<GA>(tid >> 3) * (int)ld + ch * 16, off_b = GA == GB ? off_a : row_of<GB>(tid >> 3) * (int)ld + ch * 16;
  auto issue_chunk = [&](uint8_t* st, int kt, int i) __attribute__((always_inline)) {
    if (i < CA) __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr)(st + (i * NT + w * 64) * 16), 16, off_a + (kt * BKB + row_of<GA>(i * (NT / 8)) * (int)ld), 0, 0, 0);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_ptr)(st + BM * BKB + ((i - CA) * NT + w * 64) * 16), 16, off_b + (kt * BKB + row_of<GB>((i - CA) * (NT / 8)) * (int)ld), 0, 0, 0);
  };
  // The block's scale bytes behind the tiles, 256 of A's rows (even waves, all the same) and 256 of B's (odd ones): every wave has the same number of loads
  // on its way.  Lanes behind the last row repeat its neighbours'.
  constexpr int SCALES = (BM + BN) * BKB;
  auto issue_scales = [&](uint8_t* st, int kt) __attribute__((always_inline)) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void*)(sp + (int64_t)kt * sld), 0, 0x7fffffff, 0x00020000), (lds_ptr)(st + SCALES + (w & 1) * 256), 4, off_s, 0, 0, 0);
  };
  auto issue = [&](uint8_t* st, int kt) __attribute__((always_inline)) {
    issue_scales(st, kt);
#pragma unroll
    for (int i = 0; i < CA + CB; ++i) issue_chunk(st, kt, i);
  };
  // the lane's: G rows / columns to a load
  constexpr int SA = MI / GA, SB = NI / GB;
  int sca[SA], scb[SB];
  auto scales = [&](const uint8_t* st, int (&a)[SA], int (&b)[SB]) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < SA; ++s) a[s] = load_scales<GA>(st + SCALES + wm * TL::TM + s * 16 * GA + (lane & 15) * GA);
#pragma unroll
    for (int s = 0; s < SB; ++s) b[s] = load_scales<GB>(st + SCALES + 256 + wn * TL::TN + s * 16 * GB + (lane & 15) * GB);
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
  auto chunk = [&](const uint8_t* st, int base, int t, int kk) __attribute__((always_inline)) { return *reinterpret_cast<const v4i*>(st + base + t * 16 * BKB + fo[kk]); };
  // All but the wave's last `left` loads are there, for all waves, and their reads of LDS are over.
  auto meet = [](auto left) __attribute__((always_inline)) {
    constexpr int VM = decltype(left)::value;
    static_assert(VM < 64, "the counter's range");
    __builtin_amdgcn_s_waitcnt((VM & 15) | (VM >> 4) << 14 | 7 << 4);  // vmcnt(VM) lgkmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  auto arrived = [&](auto blocks) __attribute__((always_inline)) { meet(std::integral_constant<int, decltype(blocks)::value * (CA + CB + 1)>{}); };  // but the last blocks'
  typedef std::integral_constant<int, 0> H0;
  typedef std::integral_constant<int, 1> H1;

  if constexpr (WIDE) {
    // Two phases to a block, one for each 16-byte chunk of a lane, and two halves to a phase: 8 k of every fragment.  A half widens its B fragments, then its A
    // fragments one by one, each a fragment ahead of the products that it enters; the second reads the next phase's codes into what it leaves free.
    // After the first phase everything of the stage is in registers: the barrier stands there, and the loads of the block after next go into the stage behind it.
    v4i ar[MI], br[NI];
    bf16x8 aw[2], bw[NI];
    auto unit = [](int e, int i) __attribute__((always_inline)) { return __int_as_float(((e >> (8 * i)) & 255) << 23); };
    auto phase = [&](const uint8_t* st, int kk) __attribute__((always_inline)) {
      unrolled<0, 2>([&](auto h) __attribute__((always_inline)) {
        constexpr int H = decltype(h)::value;
        unrolled<0, NI>([&](auto j) __attribute__((always_inline)) {
#pragma unroll
          for (int n = 0; n < 4; ++n) widen2<FB>(br[j][2 * H], br[j][2 * H + 1], unit(scb[j / GB], j % GB), n, bw[j]);
          if (H) br[j] = chunk(st, fb, j, kk);
        });
#pragma unroll
        for (int n = 0; n < 4; ++n) widen2<FA>(ar[0][2 * H], ar[0][2 * H + 1], unit(sca[0], 0), n, aw[0]);
        if (H) ar[0] = chunk(st, fa, 0, kk);
        unrolled<0, MI>([&](auto i) __attribute__((always_inline)) {
          constexpr int I = decltype(i)::value, X = I & 1;
          __builtin_amdgcn_sched_barrier(0);
          asm volatile("s_nop 1");  // between a conversion (for the first one also the sums' zeros) and a matrix instruction that reads it
          float u = 0.f;
          if constexpr (I + 1 < MI) u = unit(sca[(I + 1) / GA], (I + 1) % GA);
          unrolled<0, NI>([&](auto j) __attribute__((always_inline)) {
            constexpr int J = decltype(j)::value;
            mma_bf16(aw[X], bw[J], acc[I][J]);
            if constexpr (I + 1 < MI) {
#pragma unroll
              for (int n = 0; n < 4; ++n)
                if (n * NI / 4 == J) widen2<FA>(ar[I + 1][2 * H], ar[I + 1][2 * H + 1], u, n, aw[1 - X]);
              if (H && J == NI - 1) ar[I + 1] = chunk(st, fa, I + 1, kk);
            }
            __builtin_amdgcn_sched_barrier(0);
          });
        });
      });
    };
    auto body = [&](uint8_t* cur, uint8_t* nxt, int kt) __attribute__((always_inline)) {
      phase(cur, 1);
      arrived(H0{});
      int na[SA], nb[SB];
      scales(nxt, na, nb);
      issue(cur, min(kt + 2, nk - 1));  // (behind the last block: that one again, which nothing reads)
      phase(nxt, 0);
#pragma unroll
      for (int s = 0; s < SA; ++s) sca[s] = na[s];
#pragma unroll
      for (int s = 0; s < SB; ++s) scb[s] = nb[s];
    };
    issue(stage0, 0);
    issue(stage1, min(1, nk - 1));
    arrived(H1{});
    scales(stage0, sca, scb);
#pragma unroll
    for (int j = 0; j < NI; ++j) br[j] = chunk(stage0, fb, j, 0);
#pragma unroll
    for (int i = 0; i < MI; ++i) ar[i] = chunk(stage0, fa, i, 0);
    int kt = 0;
    for (; kt + 2 <= nk; kt += 2) {
      body(stage0, stage1, kt);
      body(stage1, stage0, kt + 1);
    }
    if (kt < nk) body(stage0, stage1, kt);
    // nothing is on its way into LDS when the workgroup ends, and the last results are there
    asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15" ::: "memory");
  } else {
    // Four phases to a block, each a half of the wave's A fragments times a half of its B fragments; what the next phase needs
    // is fetched meanwhile.  The last two phases fetch the next block's first halves.  (The halves of B swap roles from block to block, so that the one that is fetched first is free.)
    // Two stages: the first phase fetches all that is left of the stage, and behind it a barrier gives the stage up to the loads of the block after next; the next stage has to be
    // there half a block later, at a second barrier.  (With one barrier, at half a block, the loads have a quarter of a block less to arrive: 2048 x 32768 x 8192 439 us and not 394, of
    // 2048 x 8192 x 32768 441 and not 407; a third stage for B alone does not give more.)
    // Four: the first two phases fetch it, and one barrier stands behind them.
    constexpr int MH = MI / 2, NH = NI / 2;
    static_assert(MI % 2 == 0 && NI % 2 == 0, "halves");
    v8i a0[MH], a1[MH], bx[2][NH];
    auto whole = [&](const uint8_t* st, int base, int t) __attribute__((always_inline)) {
      const v4i x = chunk(st, base, t, 0), y = chunk(st, base, t, 1);
      return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto read_a = [&](const uint8_t* st, int half, v8i (&f)[MH], int i) __attribute__((always_inline)) { f[i] = whole(st, fa, half * MH + i); };
    auto read_b = [&](const uint8_t* st, int half, int j) __attribute__((always_inline)) { bx[half][j] = whole(st, fb, half * NH + j); };
    // The instructions of a phase in the order that they are issued in: an MFMA, then what `side` has for its place.
    auto phase = [&](auto ha, auto hb, v8i (&f)[MH], auto&& side) __attribute__((always_inline)) {
      unrolled<0, MH * NH>([&](auto n) __attribute__((always_inline)) {
        constexpr int I = decltype(n)::value / NH, JJ = decltype(n)::value % NH, J = I & 1 ? NH - 1 - JJ : JJ;  // serpentine: one operand changes
        constexpr int TI = decltype(ha)::value * MH + I, TJ = decltype(hb)::value * NH + J;
        mma_scaled<TI % GA, TJ % GB, FA, FB>(f[I], bx[decltype(hb)::value][J], acc[TI][TJ], sca[TI / GA], scb[TJ / GB]);
        side(decltype(n)::value);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    // loads of a tile: one after every EACH matrix instructions from the second (third) phase on, or PER after each
    constexpr int NMMA = MH * NH, PHASES = NS == 2 ? 3 : 2, FIT = PHASES * NMMA / (CA + CB), MOST = NS == 2 ? NMMA / 4 : 3, EACH = FIT > MOST ? MOST : FIT < 1 ? 1 : FIT,
                  PER = (CA + CB + PHASES * NMMA - 1) / (PHASES * NMMA);
    static_assert((PHASES * NMMA + EACH - 1) / EACH * PER >= CA + CB, "all of them");
    auto share = [&](uint8_t* st, int kt, int n) __attribute__((always_inline)) {
      if (n % EACH) return;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (n / EACH * PER + i < CA + CB) issue_chunk(st, kt, n / EACH * PER + i);
    };
    // works on block kt in stage U and loads block kt + NS into it (behind the last one: the last again, which nothing reads)
    auto body = [&](auto u, int kt) __attribute__((always_inline)) {
      constexpr int U = decltype(u)::value, S = U & 1 ? 0 : 1;
      const std::integral_constant<int, U & 1> first_half{};
      const std::integral_constant<int, S> second_half{};
      uint8_t *const cur = stage(u), *const nxt = stage(std::integral_constant<int, U + 1>{});
      const int lk = min(kt + NS, nk - 1);
      int na[SA], nb[SB];
      constexpr int START = NS == 2 ? 0 : -NMMA;  // of the loads, in instructions from the second phase on
      // between what is moved in front of a block (scales, in front of the first one the sums' zeros) and a matrix instruction that reads it, which the compiler does not see
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_nop 1");
      __builtin_amdgcn_sched_barrier(0);
      phase(H0{}, first_half, a0, [&](int n) __attribute__((always_inline)) {
        if (n < NH) read_b(cur, S, n);
        if (NS == 2 && n >= NH && n - NH < MH) read_a(cur, 1, a1, n - NH);
      });
      if constexpr (NS == 2) {
        static_assert(NMMA >= NH + MH, "the first phase has a place for each read");
        meet(std::integral_constant<int, 63>{});
        issue_scales(cur, lk);
      }
      phase(H0{}, second_half, a0, [&](int n) __attribute__((always_inline)) {
        if constexpr (NS == 2) share(cur, lk, n);
        else if (n < MH) read_a(cur, 1, a1, n);
      });
      if constexpr (NS == 2) {
        constexpr int GONE = (NMMA + EACH - 1) / EACH * PER;  // loads of the second phase
        meet(std::integral_constant<int, (GONE < CA + CB ? GONE : CA + CB) + 1>{});
        scales(nxt, na, nb);
      } else {
        arrived(std::integral_constant<int, NS - 2>{});
        scales(nxt, na, nb);
        issue_scales(cur, lk);
      }
      phase(H1{}, second_half, a1, [&](int n) __attribute__((always_inline)) {
        if (n < MH) read_a(nxt, 0, a0, n);
        share(cur, lk, START + NMMA + n);
      });
      phase(H1{}, first_half, a1, [&](int n) __attribute__((always_inline)) {
        if (n < NH) read_b(nxt, S, n);
        share(cur, lk, START + 2 * NMMA + n);
      });
#pragma unroll
      for (int s = 0; s < SA; ++s) sca[s] = na[s];
#pragma unroll
      for (int s = 0; s < SB; ++s) scb[s] = nb[s];
    };
    unrolled<0, NS>([&](auto u) __attribute__((always_inline)) { issue(stage(u), min((int)decltype(u)::value, nk - 1)); });
    arrived(std::integral_constant<int, NS - 1>{});
    scales(stage0, sca, scb);
#pragma unroll
    for (int i = 0; i < MH; ++i) read_a(stage0, 0, a0, i);
#pragma unroll
    for (int j = 0; j < NH; ++j) read_b(stage0, 0, j);
    int kt = 0;
    for (; kt + NS <= nk; kt += NS) unrolled<0, NS>([&](auto u) __attribute__((always_inline)) { body(u, kt + decltype(u)::value); });
    unrolled<0, NS - 1>([&](auto u) __attribute__((always_inline)) {
      if (kt + decltype(u)::value < nk) body(u, kt + decltype(u)::value);
    });
    // nothing is on its way into LDS when the workgroup ends, and the last results are there (16 passes and some)
    asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");
  }

  // The epilogue.  Stores go by 32-bit offsets from the wave's first result, columns behind the last at offsets behind the descriptor's end, where rows behind the last are by themselves, so
  // that a result and its bias need no branch for an element.  (With a branch for each group of results, and the bias fetched for each: 2048 x 6144 x 2048 with a bias 35.6 us and not 27, 8192 x 32768 x 2048 634 and not 536.)
  // R and C's own values do: two branches of the whole wave for each access, whose load is waited for, behind the store before it, before the next one starts.  us without / with R / accumulating: into fp32
  // 2048 x 8192 x 2048 55 / 67 / 67, 8192 x 32768 x 2048 855 / 1128 / 1118, 2048 x 2048 x 2048 21 / 24 / 24 (what is read more takes 14, 224 and 3.5 at a copy's rate); in bf16 2048 x 2048 x 8192 30 / 35, 2048 x 8192 x
  // 32768 347 / 372, 2048 x 6144 x 2048 25 / 34, 8192 x 32768 x 2048 428 / 707 (1.7, 7, 5 and 112): there the waiting shows, most where there are few blocks to a result.
  const int mw = m0 + wm * TL::TM, nw = n0 + wn * TL::TN;
  if (mw >= p.M || nw >= p.N) return;
  const size_t from = (size_t)mw * p.N + nw, left = ((size_t)p.M * p.N - from) * sizeof(TO);
  const int bytes = (int)(left < 0x7fffff00u ? left : 0x7fffff00u);
  const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc((void*)(C + from), 0, bytes, 0x00020000);
  const __amdgpu_buffer_rsrc_t rr = __builtin_amdgcn_make_buffer_rsrc((void*)(p.R ? reinterpret_cast<const TO*>(p.R) + from : C + from), 0, bytes, 0x00020000);
  // lane l, register r of a fragment: row 4 (l / 16) + r, column l % 16 of it
  const int lc = (lane & 15) * GB;
  float bias[SB][GB];
#pragma unroll
  for (int s = 0; s < SB; ++s)
#pragma unroll
    for (int e = 0; e < GB; ++e) bias[s][e] = -0.f;  // a sum with it is the other term
  if (p.bias) {
#pragma unroll
    for (int s = 0; s < SB; ++s)
#pragma unroll
      for (int e = 0; e < GB; ++e) bias[s][e] = p.bias[min(nw + s * 16 * GB + lc + e, p.N - 1)];
  }
  // E: neighbouring elements of an access, MORE: R or C's own values are added, AUX: of the stores
  auto write = [&](auto elems, auto more, auto aux) __attribute__((always_inline)) {
    constexpr int E = decltype(elems)::value;
    typedef TO V __attribute__((ext_vector_type(E)));
    uint32_t n = p.N, col[SB][GB / E];
    asm("" : "+s"(n));  // nothing of a form of the epilogue is kept for the others
#pragma unroll
    for (int s = 0; s < SB; ++s)
#pragma unroll
      for (int e = 0; e < GB; e += E) col[s][e / E] = nw + s * 16 * GB + lc + e < p.N ? (4 * (lane >> 4) * GA * n + s * 16 * GB + lc + e) * (uint32_t)sizeof(TO) : 0x80000000u;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint32_t line = (uint32_t)(i / GA * 16 * GA + r * GA + i % GA) * n * sizeof(TO);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < SB; ++s)
#pragma unroll
          for (int e = 0; e < GB; e += E) {
            const uint32_t at = col[s][e / E] + line;
            float v[E];
#pragma unroll
            for (int k = 0; k < E; ++k) v[k] = acc[i][s * GB + e + k][r] + bias[s][e + k];
            if constexpr (decltype(more)::value) {
              if (p.R) {
                const V x = __builtin_bit_cast(V, load_some<sizeof(V)>(rr, at));
#pragma unroll
                for (int k = 0; k < E; ++k) v[k] += (float)x[k];
              }
              if (p.accumulate) {
                const V x = __builtin_bit_cast(V, load_some<sizeof(V)>(rc, at));
#pragma unroll
                for (int k = 0; k < E; ++k) v[k] += (float)x[k];
              }
            }
            V o;
#pragma unroll
            for (int k = 0; k < E; ++k) o[k] = (TO)v[k];
            store_some<decltype(aux)::value>(rc, at, o);
          }
      }
  };
  typedef std::integral_constant<int, 2> Past;
  const bool vec = p.N % GB == 0 && (((uintptr_t)p.C | (uintptr_t)p.R) & (GB * sizeof(TO) - 1)) == 0, more = p.R || p.accumulate;
  const std::integral_constant<int, GB> elems{};
  if constexpr (!WIDE && std::is_same<TO, float>::value) {  // planes: only the product
    if (vec) write(elems, H0{}, H0{});
    else write(H1{}, H0{}, H0{});
  } else if (!vec) write(H1{}, H1{}, H0{});
  else if (more) write(elems, H1{}, H0{});
  else if (p.passing) write(elems, H0{}, Past{});
  else write(elems, H0{}, H0{});
#endif
}

// C = the sum of the slices' planes in ascending order, and the epilogue; V neighbouring columns to a thread
template <typename TO, int V>
__global__ __launch_bounds__(256) void fp8_finish_kernel(uint32_t groups, uint32_t across, size_t plane, int slices, const float* __restrict__ planes,
                                                         TO* C, const float* __restrict__ bias, const TO* R, int accumulate) {
  typedef float F __attribute__((ext_vector_type(V)));
  typedef TO O __attribute__((ext_vector_type(V)));
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < groups; i += gridDim.x * 256) {
    const size_t at = (size_t)i * V;
    F x = *reinterpret_cast<const F*>(planes + at);
#pragma unroll 4
    for (int s = 1; s < slices; ++s) x += *reinterpret_cast<const F*>(planes + s * plane + at);
    if (bias) {
      const uint32_t col = i % across * V;
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] += bias[col + e];
    }
    O o;
    if (R) {
      o = *reinterpret_cast<const O*>(R + at);
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] += (float)o[e];
    }
    if (accumulate) {
      o = *reinterpret_cast<const O*>(C + at);
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] += (float)o[e];
    }
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = (TO)x[e];
    *reinterpret_cast<O*>(C + at) = o;
  }
}

typedef Tile8<256, 256, 4, 2> Big8;
// Long contractions: half the waves, each with all of a SIMD's registers, read a third less from LDS, whose power goes to the clock; with few blocks one wave waits alone for the first loads and at the epilogue.  What
// four waves take more (+) or less than eight, in %, at 8 / 12 / 16 / 20 / 24 / 32 / 40 / 64 / 128 blocks: 2304 x 4096 results +3.1 +1.8 +1.6 +1.5 +1.3 -1.1 +1.3 +0.1 -0.4; 2048 x 6144 +2.4 +0.9 +0.2 +1.7 -0.1 -0.7
// -0.8 -1.1 -2.8; 4096 x 4096 +2.0 +1.0 +0.3 -0.4 -1.5 -1.3 -1.6 -1.5 -3.0; 5000 x 4000 +1.5 +0.8 +0.5 -0.5 -0.7 -0.7 -0.9 -1.7 -2.1; 4096 x 8192 -2.6 -2.0 -1.8 -1.4 -1.2 -2.3 -1.2 -2.1 -2.2; 16384 x 2048 +7.6
// +6.7 +5.3 +3.7 +2.9 +1.6 +1.4 -1.1 -1.4; 8192 x 8192 -6.5 -1.9 -1.5 -0.5 -2.0 -1.2 -1.8 -1.8 -2.3; 2048 x 32768 -2.6 +0.1 +0.2 -0.2 -1.6 -1.2 -1.6 -1.7 -2.2; 8192 x 32768 +0.1 +0.5 -0.7 -1.2 -0.7 -1.5
// -1.7 -2.7 -2.0.  Their mean is +0.5 at 16, +0.3 at 20, -0.4 at 24 and -0.9 at 32.
typedef Tile8<256, 256, 2, 2> Long8;
constexpr int LONG_BLOCKS = 24;
typedef Tile8<256, 256, 2, 4> Wide8;  // widened operands: smaller sub-tiles, two waves to a SIMD
typedef Tile8<128, 128, 2, 2, 4> Mid8;
typedef Tile8<128, 128, 2, 2> WideMid8;
typedef Tile8<64, 64, 2, 2> WideSmall8;
typedef Tile8<64, 64, 2, 2, 4> Small8;

struct Plan { int tile, slices, slice; };  // tile 0: 256 x 256, 1: 128 x 128, 2: 64 x 64

// The tile, and the slices that the contraction is cut into, of the least estimated time.  A round of workgroups over the chip takes START + blocks x BLOCK us; one that takes
// only some of its SLOTS that share of BLOCK, but LEAST at least.  A split costs a second kernel and the planes' way to memory and back.  Fitted to 30 shapes from 1 x 256 x 250 to
// 256 x 8192 x 32768 on all tiles and splits, in both types, with eight waves to a 256 x 256 tile throughout.  With the kernels there are now the choice is the best or within 10 % of it for 58 of the 60 (into fp32: 1 x 2048
// x 2048 7.9 us, 6.6 in four slices; 8192 x 2048 x 300 22.9, 20.6 on 128 x 128 tiles).  us, 64 x 64 / 128 x 128 / 256 x 256, bf16 results: 200 x 3000 x 1000 4.6 / 6.6 / 12.9; 1000 x 4004 x 1000 11.4 / 8.2 / 13.6;
// 2048 x 2048 x 8192 50 / 30 / 67; 2048 x 6144 x 2048 45 / 31 / 25.
// Splits: 1 x 8192 x 8192 into fp32 30 in one, 15 in 4 slices; 256 x 8192 x 32768 into fp32 179 on 64 x 64 tiles, 128 in 4 slices on 128 x 128; most shapes lose by them
// (1000 x 1000 x 4096 9.1 in one, 16 in two).
constexpr double BASE_US = 2.5, SPLIT_US = 6.0, PLANE_BYTES_US = 9e6;
struct TileCost { int edge, slots; double start, block, least; };
constexpr TileCost COST[2][3] = {{{256, 256, 4.0, 1.42, 0.92}, {128, 256, 1.8, 0.41, 0.3}, {64, 512, 0.8, 0.36, 0.17}},    // 8-bit instructions
                                 {{256, 256, 4.0, 3.3, 2.4}, {128, 512, 2.0, 1.75, 0.95}, {64, 1024, 0.8, 1.15, 0.41}}};  // widened operands
// Operands and result larger together than the 256 MiB memory-side cache, by half: the result goes past the caches, whose lines the operands then keep.  us, in the caches and past them:
// 32768 x 8192 x 2048 465 and 430, 8192 x 32768 x 1024 283 and 252, 2048 x 32768 x 8192 370 and 360, 8192 x 16384 x 4096 390 and 391.  Not results that something is added to, which were just read.
constexpr size_t PASSING_BYTES = (size_t)384 << 20;
constexpr size_t MAX_PLANES = (size_t)1 << 28;

Plan plan_of(int M, int N, int blocks, bool wide) {
  Plan best{};
  double best_t = 0;
  for (int t = 0; t < 3; ++t) {
    const TileCost& c = COST[wide][t];
    const double tiles = (double)((M + c.edge - 1) / c.edge) * ((N + c.edge - 1) / c.edge);
    for (int s = 1; s <= 16 && s <= blocks; s *= 2) {
      const int slice = (blocks + s - 1) / s, slices = (blocks + slice - 1) / slice;
      const double planes = 4.0 * M * N * slices, wgs = tiles * slices;
      if (slices != s || (s > 1 && (wgs > 4 * c.slots || planes > (double)MAX_PLANES))) break;
      const double full = (double)(long)(wgs / c.slots), part = wgs / c.slots - full;
      double us = BASE_US + full * (c.start + slice * c.block) + (s > 1 ? SPLIT_US + 2 * planes / PLANE_BYTES_US : 0);
      if (part > 0) us += c.start + slice * (c.block * part > c.least ? c.block * part : c.least);
      if (s > 1) us *= 1.1;  // a split has to win by more than the estimate may be off
      if (!best.slices || us < best_t) { best = {t, slices, slice}; best_t = us; }
    }
  }
  return best;
}

// whether a 256 x 256 tile of 8-bit instructions that writes its result itself is the one of four waves
bool is_long(int slice, int slices) { return slices == 1 && slice >= LONG_BLOCKS; }

template <typename TL, int FA, int FB, bool WIDE, typename TO>
bf_status launch8(Fp8Args a, int slices, hipStream_t st) {
  a.tiles_m = (a.M + TL::BM - 1) / TL::BM;
  const long tiles = (long)a.tiles_m * ((a.N + TL::BN - 1) / TL::BN);
  if (tiles * TL::NT >= (1l << 32)) { set_error("bf_op_fp8_gemm: more than 2^32 threads"); return BF_EINVAL; }
  gemm_fp8_kernel<TL, FA, FB, WIDE, TO><<<dim3((unsigned)tiles, (unsigned)slices), TL::NT, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_error("bf_op_fp8_gemm: launch failed: %s", hipGetErrorString(e)); return BF_EDEVICE; }
  return BF_OK;
}

template <int FA, int FB>
bf_status by_tile(const Fp8Args& a, int tile, int slices, bool wide, bool f32, hipStream_t st) {
  if (wide) switch (tile) {
    case 0: return launch8<Wide8, FA, FB, true, float>(a, slices, st);
    case 1: return launch8<WideMid8, FA, FB, true, float>(a, slices, st);
    default: return launch8<WideSmall8, FA, FB, true, float>(a, slices, st);
  }
  if (f32) switch (tile) {  // planes
    case 0: return launch8<Big8, FA, FB, false, float>(a, slices, st);
    case 1: return launch8<Mid8, FA, FB, false, float>(a, slices, st);
    default: return launch8<Small8, FA, FB, false, float>(a, slices, st);
  }
  switch (tile) {
    case 0: return is_long(a.slice, slices) ? launch8<Long8, FA, FB, false, bf16_t>(a, slices, st) : launch8<Big8, FA, FB, false, bf16_t>(a, slices, st);
    case 1: return launch8<Mid8, FA, FB, false, bf16_t>(a, slices, st);
    default: return launch8<Small8, FA, FB, false, bf16_t>(a, slices, st);
  }
}

template <typename TO, int V>
void launch_finish(int M, int N, int slices, const float* planes, void* C, const float* bias, const void* R, int accumulate, hipStream_t st) {
  const size_t n = (size_t)M * N, groups = n / V;  // (splits are of few tiles: under 2^32)
  const unsigned grid = (unsigned)((groups + 255) / 256 < 2048 ? (groups + 255) / 256 : 2048);
  fp8_finish_kernel<TO, V><<<grid, 256, 0, st>>>((uint32_t)groups, (uint32_t)(N / V), n, slices, planes, (TO*)C, bias, (const TO*)R, accumulate);
}

bf_status finish(int dtype, int M, int N, int slices, const float* planes, void* C, const float* bias, const void* R, int accumulate, hipStream_t st) {
  const bool four = N % 4 == 0 && (((uintptr_t)C | (uintptr_t)R) & (dtype == BF_BF16 ? 7 : 15)) == 0;
  if (dtype == BF_BF16) {
    if (four) launch_finish<bf16_t, 4>(M, N, slices, planes, C, bias, R, accumulate, st);
    else launch_finish<bf16_t, 1>(M, N, slices, planes, C, bias, R, accumulate, st);
  } else {
    if (four) launch_finish<float, 4>(M, N, slices, planes, C, bias, R, accumulate, st);
    else launch_finish<float, 1>(M, N, slices, planes, C, bias, R, accumulate, st);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_error("bf_op_fp8_gemm: launch failed: %s", hipGetErrorString(e)); return BF_EDEVICE; }
  return BF_OK;
}

bool sizes_ok(int M, int N, int K) { return M >= 1 && N >= 1 && K >= 1 && M <= (1 << 21) && N <= (1 << 21) && K <= (1 << 21); }

}  // namespace

size_t fp8_gemm_work_bytes(int dtype, int M, int N, int K) {
  if (!sizes_ok(M, N, K) || (dtype != BF_BF16 && dtype != BF_FP32)) return 0;
  const Plan q = plan_of(M, N, (K + 127) / 128, dtype == BF_FP32);
  return q.slices > 1 ? (size_t)q.slices * M * N * sizeof(float) : 0;
}

bool fp8_gemm_tile(int dtype, int M, int N, int K, int* edge, int* waves, int* slices) {
  *edge = *waves = *slices = 0;
  if (!sizes_ok(M, N, K) || (dtype != BF_BF16 && dtype != BF_FP32)) return false;
  const bool wide = dtype == BF_FP32;
  const Plan q = plan_of(M, N, (K + 127) / 128, wide);
  const int nt[3] = {wide ? Wide8::NT : is_long(q.slice, q.slices) ? Long8::NT : Big8::NT, wide ? WideMid8::NT : Mid8::NT, wide ? WideSmall8::NT : Small8::NT};
  *edge = COST[wide][q.tile].edge;
  *waves = nt[q.tile] / 64;
  *slices = q.slices;
  return true;
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
  const bool wide = dtype == BF_FP32;
  const Plan q = plan_of(M, N, blocks, wide);
  const bool split = q.slices > 1;
  const size_t need = split ? (size_t)q.slices * M * N * sizeof(float) : 0;
  if (need && (!work || ((uintptr_t)work & 255) || work_bytes < need)) {
    set_error("bf_op_fp8_gemm: needs %zu bytes of 256-byte aligned scratch", need);
    return BF_EINVAL;
  }
  Fp8Args a{M, N, blocks, (const uint8_t*)A, (const uint8_t*)B, (const uint8_t*)sa, (const uint8_t*)sb, (M + 15) / 16 * 16, (N + 15) / 16 * 16, C, bias, R,
            accumulate, 0, q.slice, 0};
  a.passing = (double)(M + (double)N) * blocks * 128 + (double)M * N * es > (double)PASSING_BYTES;
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
  return finish(dtype, M, N, q.slices, (const float*)work, C, bias, R, accumulate, st);
}

}  // namespace bf
