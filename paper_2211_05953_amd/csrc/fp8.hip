// The 8-bit form of a matrix: e4m3 or e5m2 codes with one power-of-two scale for each 128 elements, along its rows, down its columns, or both.
//
// e = the smallest integer >= -127 with amax <= top 2^e (top = 1.75 2^8 or 1.75 2^15), code = x 2^-e rounded to nearest even.  x 2^-e is exact, so a
// code has one rounding.  amax is taken over finite values; others get the NaN code.
//
// HBM traffic: an element is read once (2 or 4 bytes) and written once or twice (1 byte each).  A workgroup has a tile of 128 x 128, whole blocks either
// way: a thread 8 rows x 8 columns of it, a row of the tile is 16 lanes.  Rows' maxima meet by lane rotations, columns' in LDS; the codes down the
// columns turn round in LDS, so that both forms leave in whole 128-byte lines.
#include "../../include/bf_ops.h"
#include "common.h"

namespace bf {

namespace {

constexpr int NT = 256, BLK = 128;

template <typename T> struct Row8;  // eight elements, as aligned as one
template <> struct Row8<bf16_t> { typedef bf16_t V __attribute__((vector_size(16), aligned(2))); };
template <> struct Row8<float> { typedef float V __attribute__((vector_size(32), aligned(4))); };

__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}

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

// 2^-e for e in -127..121
__device__ __forceinline__ float inverse_of(int e) { return __uint_as_float((uint32_t)(127 - e) << 23); }

template <int FMT>
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int o = 0;
  if constexpr (FMT == BF_E4M3) {
    o = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, o, false);
    o = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, o, true);
  } else {
    o = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, o, false);
    o = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, o, true);
  }
  return (uint32_t)o;
}

template <typename T, int FMT>
__global__ __launch_bounds__(NT) void fp8_quantize_kernel(int rows, int cols, const T* __restrict__ x, size_t ld, uint8_t* __restrict__ q,
                                                          uint8_t* __restrict__ scale, uint8_t* __restrict__ qt, uint8_t* __restrict__ scale_t) {
  __shared__ __attribute__((aligned(16))) uint8_t turn[BLK * BLK];
  __shared__ uint32_t cmax[4][BLK];
  const int tid = threadIdx.x, tc = tid & 15, tr = tid >> 4;
  const int r0 = blockIdx.y * BLK, c0 = blockIdx.x * BLK, row = r0 + tr * 8, col = c0 + tc * 8;
  const size_t ldq = ((size_t)cols + BLK - 1) / BLK * BLK, ldt = ((size_t)rows + BLK - 1) / BLK * BLK;
  const int rows16 = (rows + 15) / 16 * 16, cols16 = (cols + 15) / 16 * 16;

  float v[8][8];
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const T* src = x + (size_t)(row + p) * ld + col;
    if (row + p < rows && col + 8 <= cols) {
      const typename Row8<T>::V t = *reinterpret_cast<const typename Row8<T>::V*>(src);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[p][k] = (float)t[k];
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[p][k] = row + p < rows && col + k < cols ? (float)src[k] : 0.f;
    }
  }
  // infinities and NaN: out of the maxima, and NaN in whatever they are scaled by
  uint32_t cm[8] = {0, 0, 0, 0, 0, 0, 0, 0}, rm[8];
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    rm[p] = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t b = finite_bits(v[p][k]);
      rm[p] = max(rm[p], b);
      cm[k] = max(cm[k], b);
      v[p][k] = (__float_as_uint(v[p][k]) & 0x7f800000u) == 0x7f800000u ? __uint_as_float(0x7fc00000u) : v[p][k];
    }
  }
  if (q) {
    uint64_t sb = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int e = exponent_of<FMT>(max16(rm[p]));
      const float u = inverse_of(e);
      sb |= (uint64_t)(uint32_t)(e + 127) << (8 * p);
      uint2 o;
      o.x = codes4<FMT>(v[p][0] * u, v[p][1] * u, v[p][2] * u, v[p][3] * u);
      o.y = codes4<FMT>(v[p][4] * u, v[p][5] * u, v[p][6] * u, v[p][7] * u);
      if (row + p < rows) *reinterpret_cast<uint2*>(q + (size_t)(row + p) * ldq + col) = o;
    }
    if (tc == 0 && row < rows16) *reinterpret_cast<uint64_t*>(scale + (size_t)blockIdx.x * rows16 + row) = sb;
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
    const float u = inverse_of(e);
    sb |= (uint64_t)(uint32_t)(e + 127) << (8 * k);
    uint2 o;
    o.x = codes4<FMT>(v[0][k] * u, v[1][k] * u, v[2][k] * u, v[3][k] * u);
    o.y = codes4<FMT>(v[4][k] * u, v[5][k] * u, v[6][k] * u, v[7][k] * u);
    // the 32 lanes that write in a cycle (16 columns, 8 apart, by 2 groups of rows) on different banks: chunks of 16 bytes XORed with
    // the column group, neighbouring columns swapped in the upper half
    *reinterpret_cast<uint2*>(turn + (c ^ ((c >> 6) & 1)) * BLK + (((tr >> 1) ^ (tc & 7)) << 4) + (tr & 1) * 8) = o;
  }
  if (tr == 0 && col < cols16) *reinterpret_cast<uint64_t*>(scale_t + (size_t)blockIdx.y * cols16 + col) = sb;
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
  auto go = [&](auto kern, auto* xs) { kern<<<grid, NT, 0, st>>>(rows, cols, xs, ld, (uint8_t*)q, (uint8_t*)scale, (uint8_t*)qt, (uint8_t*)scale_t); };
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
