// The 8-bit form of a matrix: e4m3 or e5m2 codes with one power-of-two scale for each 128 elements, along its rows, down its columns, or both.
//
// e = the smallest integer >= -127 with amax <= top 2^e (top = 1.75 2^8 or 1.75 2^15), code = x 2^-e rounded to nearest even.  Dividing by a power of two is exact, so a
// code has one rounding; the scaled conversions do both (v_cvt_scalef32_pk_fp8_bf16 and its like).  amax is taken over finite values; others get the NaN code.
//
// HBM traffic: an element is read once (2 or 4 bytes) and written once or twice (1 byte each).  A workgroup has a tile of 128 x 128, whole blocks either
// way: a thread 8 rows x 8 columns of it, a row of the tile is 16 lanes.  Rows' maxima meet by lane rotations, columns' in LDS; the codes down the
// columns turn round in LDS, so that both forms leave in whole 128-byte lines.  8192 x 32768 in bf16: both ways 211 us, 5.1 TB/s, along the rows alone 151 us, 5.3 (a copy reaches 5.2
// to 5.6); 2048 x 8192 12.4 and 8.5 us; 1 x 8192 2.9 us.  (In fp32 arithmetic, element by element, 250, 191, 17, 12 and 5.4: three to four instructions an element in place of twenty.)
#include "../../include/bf_ops.h"
#include "common.h"

namespace bf {

namespace {

constexpr int NT = 256, BLK = 128;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// A thread's 8 x 8 elements, and what is taken of them; magnitudes as bits, shifted to those of fp32.  bf16 stays in pairs of neighbours in a row: two elements
// to a register and an instruction.
template <typename T> struct Part;

template <> struct Part<float> {
  typedef float V __attribute__((vector_size(32), aligned(4)));  // eight elements, as aligned as one
  float x[8][8];
  __device__ __forceinline__ void put(int p, const V& t, bool in) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[p][k] = in ? t[k] : 0.f;
  }
  __device__ __forceinline__ void put1(int p, int k, float t, bool in) { x[p][k] = in ? t : 0.f; }
  static __device__ __forceinline__ uint32_t bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
  __device__ __forceinline__ void maxima(uint32_t (&rm)[8], uint32_t (&cm)[8]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) cm[k] = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      rm[p] = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        rm[p] = max(rm[p], bits(x[p][k]));
        cm[k] = max(cm[k], bits(x[p][k]));
      }
    }
  }
  // infinities and NaN: NaN, and out of the maxima
  __device__ __forceinline__ void without_infinite(uint32_t (&rm)[8], uint32_t (&cm)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) cm[k] = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      rm[p] = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const bool bad = bits(x[p][k]) >= 0x7f800000u;
        const uint32_t b = bad ? 0u : bits(x[p][k]);
        x[p][k] = bad ? __uint_as_float(0x7fc00000u) : x[p][k];
        rm[p] = max(rm[p], b);
        cm[k] = max(cm[k], b);
      }
    }
  }
  // codes of four neighbours along a row / down a column, divided by `unit`
  template <int FMT>
  __device__ __forceinline__ uint32_t along(int p, int k, float unit) const { return four<FMT>(x[p][k], x[p][k + 1], x[p][k + 2], x[p][k + 3], unit); }
  template <int FMT>
  __device__ __forceinline__ uint32_t down(int p, int k, float unit) const { return four<FMT>(x[p][k], x[p + 1][k], x[p + 2][k], x[p + 3][k], unit); }
  template <int FMT>
  static __device__ __forceinline__ uint32_t four(float a, float b, float c, float d, float unit) {
    s16x2 o = {0, 0};
    if constexpr (FMT == BF_E4M3) {
      o = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(o, a, b, unit, false);
      o = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(o, c, d, unit, true);
    } else {
      o = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(o, a, b, unit, false);
      o = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(o, c, d, unit, true);
    }
    return __builtin_bit_cast(uint32_t, o);
  }
};

template <> struct Part<bf16_t> {
  typedef uint32_t V __attribute__((vector_size(16), aligned(2)));
  uint32_t x[8][4];
  __device__ __forceinline__ void put(int p, const V& t, bool in) {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[p][k] = in ? t[k] : 0u;
  }
  __device__ __forceinline__ void put1(int p, int k, bf16_t t, bool in) {
    const uint32_t b = in ? __builtin_bit_cast(uint16_t, t) : 0u;
    x[p][k / 2] = k & 1 ? x[p][k / 2] | b << 16 : b;
  }
  static __device__ __forceinline__ u16x2 bits(uint32_t v) { return __builtin_bit_cast(u16x2, v & 0x7fff7fffu); }
  static __device__ __forceinline__ u16x2 most(u16x2 a, u16x2 b) { return __builtin_elementwise_max(a, b); }
  __device__ __forceinline__ void maxima(uint32_t (&rm)[8], uint32_t (&cm)[8]) const {
    u16x2 c[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = (u16x2){0, 0};
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      u16x2 r = {0, 0};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const u16x2 b = bits(x[p][k]);
        r = most(r, b);
        c[k] = most(c[k], b);
      }
      rm[p] = (uint32_t)max(r[0], r[1]) << 16;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) { cm[2 * k] = (uint32_t)c[k][0] << 16; cm[2 * k + 1] = (uint32_t)c[k][1] << 16; }
  }
  __device__ __forceinline__ void without_infinite(uint32_t (&rm)[8], uint32_t (&cm)[8]) {
#pragma unroll
    for (int p = 0; p < 8; ++p)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if ((x[p][k] & 0x7f80u) == 0x7f80u) x[p][k] = (x[p][k] & 0xffff0000u) | 0x7fc0u;
        if ((x[p][k] & 0x7f800000u) == 0x7f800000u) x[p][k] = (x[p][k] & 0xffffu) | 0x7fc00000u;
      }
#pragma unroll
    for (int k = 0; k < 8; ++k) cm[k] = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      rm[p] = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t b = (k & 1 ? x[p][k / 2] >> 16 : x[p][k / 2]) & 0x7fffu, f = b >= 0x7f80u ? 0u : b << 16;
        rm[p] = max(rm[p], f);
        cm[k] = max(cm[k], f);
      }
    }
  }
  template <int FMT>
  __device__ __forceinline__ uint32_t along(int p, int k, float unit) const { return four<FMT>(x[p][k / 2], x[p][k / 2 + 1], unit); }
  template <int FMT>
  __device__ __forceinline__ uint32_t down(int p, int k, float unit) const {
    const uint32_t sel = k & 1 ? 0x07060302u : 0x05040100u;  // the upper or the lower halves of two registers
    return four<FMT>(__builtin_amdgcn_perm(x[p + 1][k / 2], x[p][k / 2], sel), __builtin_amdgcn_perm(x[p + 3][k / 2], x[p + 2][k / 2], sel), unit);
  }
  template <int FMT>
  static __device__ __forceinline__ uint32_t four(uint32_t a, uint32_t b, float unit) {
    s16x2 o = {0, 0};
    if constexpr (FMT == BF_E4M3) {
      o = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, __builtin_bit_cast(bf16x2, a), unit, false);
      o = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, __builtin_bit_cast(bf16x2, b), unit, true);
    } else {
      o = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(o, __builtin_bit_cast(bf16x2, a), unit, false);
      o = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(o, __builtin_bit_cast(bf16x2, b), unit, true);
    }
    return __builtin_bit_cast(uint32_t, o);
  }
};

// maximum over the 16 lanes of a row
__device__ __forceinline__ uint32_t max16(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x128, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x124, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x122, 0xf, 0xf, false));
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x121, 0xf, 0xf, false));
}

template <int FMT>
__device__ __forceinline__ int exponent_of(uint32_t amax) {
  if (amax == 0) return 0;
  const int e = (int)(amax >> 23) - 127 - (FMT == BF_E4M3 ? 8 : 15) + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(e, -127);
}

// 2^e, whose exponent is what the conversions divide by
__device__ __forceinline__ float unit_of(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

template <typename T, int FMT>
__global__ __launch_bounds__(NT) void fp8_quantize_kernel(int rows, int cols, const T* __restrict__ x, size_t ld, uint8_t* __restrict__ q,
                                                          uint8_t* __restrict__ scale, uint8_t* __restrict__ qt, uint8_t* __restrict__ scale_t, int by_xcd) {
  __shared__ __attribute__((aligned(16))) uint8_t turn[BLK * BLK];
  __shared__ uint32_t cmax[4][BLK];
  const int tid = threadIdx.x, tc = tid & 15, tr = tid >> 4;
  int bx = blockIdx.x, by = blockIdx.y;
  if (by_xcd) {  // each XCD a contiguous range of pairs of tiles, one below the other (the host sees to even numbers)
    const uint32_t per = gridDim.x * gridDim.y >> 3, id = by * gridDim.x + bx, lin = (id & 7) * per + (id >> 3), pair = 2 * gridDim.x;
    by = lin / pair * 2 + (lin & 1);
    bx = lin % pair >> 1;
  }
  const int r0 = by * BLK, c0 = bx * BLK, row = r0 + tr * 8, col = c0 + tc * 8;
  const size_t ldq = ((size_t)cols + BLK - 1) / BLK * BLK, ldt = ((size_t)rows + BLK - 1) / BLK * BLK;
  const int rows16 = (rows + 15) / 16 * 16, cols16 = (cols + 15) / 16 * 16;

  Part<T> v;
  const T* src = x + col;
  if (col + 8 <= cols) {
#pragma unroll
    for (int p = 0; p < 8; ++p) v.put(p, *reinterpret_cast<const typename Part<T>::V*>(src + (size_t)min(row + p, rows - 1) * ld), row + p < rows);
  } else {  // the end of a row, element by element; what lies behind is zero
#pragma unroll
    for (int p = 0; p < 8; ++p)
#pragma unroll
      for (int k = 0; k < 8; ++k) v.put1(p, k, x[(size_t)min(row + p, rows - 1) * ld + min(col + k, cols - 1)], row + p < rows && col + k < cols);
  }
  uint32_t cm[8], rm[8], top = 0;
  v.maxima(rm, cm);
#pragma unroll
  for (int p = 0; p < 8; ++p) top = max(top, rm[p]);
  if (top >= 0x7f800000u) v.without_infinite(rm, cm);
  if (q) {
    uint64_t sb = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int e = exponent_of<FMT>(max16(rm[p]));
      const float u = unit_of(e);
      sb |= (uint64_t)(uint32_t)(e + 127) << (8 * p);
      uint2 o;
      o.x = v.template along<FMT>(p, 0, u);
      o.y = v.template along<FMT>(p, 4, u);
      if (row + p < rows) *reinterpret_cast<uint2*>(q + (size_t)(row + p) * ldq + col) = o;
    }
    if (tc == 0 && row < rows16) *reinterpret_cast<uint64_t*>(scale + (size_t)bx * rows16 + row) = sb;
  }
  if (!qt) return;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    cm[k] = max(cm[k], (uint32_t)__shfl_xor((int)cm[k], 16, 64));
    cm[k] = max(cm[k], (uint32_t)__shfl_xor((int)cm[k], 32, 64));
  }
  if ((tid & 63) < 16) {
#pragma unroll
    for (int k = 0; k < 8; ++k) cmax[tid >> 6][tc * 8 + k] = cm[k];
  }
  __syncthreads();
  uint64_t sb = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int c = tc * 8 + k;
    const int e = exponent_of<FMT>(max(max(cmax[0][c], cmax[1][c]), max(cmax[2][c], cmax[3][c])));
    const float u = unit_of(e);
    sb |= (uint64_t)(uint32_t)(e + 127) << (8 * k);
    uint2 o;
    o.x = v.template down<FMT>(0, k, u);
    o.y = v.template down<FMT>(4, k, u);
    // the 32 lanes that write in a cycle (16 columns, 8 apart, by 2 groups of rows) on different banks: chunks of 16 bytes XORed with
    // the column group, neighbouring columns swapped in the upper half.  (What conflicts there are, 30 % of the accesses' cycles, are those of cmax, which a row's 16 lanes write and read
    // eight words apart.)
    *reinterpret_cast<uint2*>(turn + (c ^ ((c >> 6) & 1)) * BLK + (((tr >> 1) ^ (tc & 7)) << 4) + (tr & 1) * 8) = o;
  }
  if (tr == 0 && col < cols16) *reinterpret_cast<uint64_t*>(scale_t + (size_t)by * cols16 + col) = sb;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = i * 32 + (tid >> 3), ch = tid & 7;
    if (c0 + c >= cols) continue;
    const uint4 o = *reinterpret_cast<const uint4*>(turn + (c ^ ((c >> 6) & 1)) * BLK + ((ch ^ ((c >> 3) & 7)) << 4));
    *reinterpret_cast<uint4*>(qt + (size_t)(c0 + c) * ldt + r0 + ch * 16) = o;
  }
}

}  // namespace

bf_status fp8_quantize(int dtype, int format, int rows, int cols, const void* x, size_t ld, void* q, void* scale, void* qt, void* scale_t, hipStream_t st) {
  if (format != BF_E4M3 && format != BF_E5M2) { set_error("bf_op_fp8_quantize: unknown format %d", format); return BF_EINVAL; }
  if (rows < 1 || cols < 1 || rows > (1 << 21) || cols > (1 << 21)) { set_error("bf_op_fp8_quantize: sizes are 1 to 2^21, got %d x %d", rows, cols); return BF_EINVAL; }
  if (!ld) ld = cols;
  if (ld < (size_t)cols || ld > ((size_t)1 << 40)) { set_error("bf_op_fp8_quantize: rows of %d elements %zu apart", cols, ld); return BF_EINVAL; }
  const size_t es = dtype == BF_BF16 ? 2 : 4;
  if (!x || ((uintptr_t)x & (es - 1))) { set_error("bf_op_fp8_quantize: x is null or not aligned to its elements"); return BF_EINVAL; }
  if (!q != !scale || !qt != !scale_t || (!q && !qt)) { set_error("bf_op_fp8_quantize: q goes with scale and qt with scale_t, and one pair at least is needed"); return BF_EINVAL; }
  if (((uintptr_t)q | (uintptr_t)scale | (uintptr_t)qt | (uintptr_t)scale_t) & 15) { set_error("bf_op_fp8_quantize: codes and scales have to be 16-byte aligned"); return BF_EINVAL; }
  const dim3 grid((cols + BLK - 1) / BLK, (rows + BLK - 1) / BLK);
  // More bytes than the 256 MiB memory-side cache by half, and lines down the columns among them: neighbouring tiles on one XCD (8192 x 32768 bf16 both ways 226 -> 211 us, down the
  // columns alone 175 -> 156; 2048 x 32768, which fits, 43.5 -> 45.4, along the rows alone 151 -> 150)
  const int by_xcd = qt && (double)rows * cols * (es + 1 + (q ? 1 : 0)) > (double)((size_t)384 << 20) && grid.y % 2 == 0 && (uint64_t)grid.x * grid.y % 8 == 0;
  auto go = [&](auto kern, auto* xs) { kern<<<grid, NT, 0, st>>>(rows, cols, xs, ld, (uint8_t*)q, (uint8_t*)scale, (uint8_t*)qt, (uint8_t*)scale_t, by_xcd); };
  if (dtype == BF_BF16) {
    if (format == BF_E4M3) go(fp8_quantize_kernel<bf16_t, BF_E4M3>, (const bf16_t*)x);
    else go(fp8_quantize_kernel<bf16_t, BF_E5M2>, (const bf16_t*)x);
  } else {
    if (format == BF_E4M3) go(fp8_quantize_kernel<float, BF_E4M3>, (const float*)x);
    else go(fp8_quantize_kernel<float, BF_E5M2>, (const float*)x);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_error("bf_op_fp8_quantize: launch failed: %s", hipGetErrorString(e)); return BF_EDEVICE; }
  return BF_OK;
}

}  // namespace bf
