// Softmax cross entropy of a linear layer over a large vocabulary, in pieces of the vocabulary: z = y W^T is never kept.
//
//   lse_t = log sum_v exp z_tv,   row_loss_t = (lse_t - z_t,label) scale,   dz = scale (exp(z - lse) - onehot)
//   dy = dz W,   dW = dz^T y
//
// Forward: the product's epilogue reduces each tile of logits to a maximum and a sum of exponentials per row (and picks the
// label's logit); a second kernel merges the tiles in their order.  No logit reaches HBM.  Backward: piece by piece of the
// vocabulary, the product again with dz as its epilogue, then the two gradient products on that piece: 6 T h V operations
// beside the forward pass's 2.
// 2048 rows, 2048 x 50304, us in kernels: forward 402 (1.05 PFLOP/s), logits again 495, dW in three parts 1016 (1.25), dy 410.  8192 x 50304:
// 1292 (1.31), 1379, 2766 in two parts (1.22), 1328.  Bound by the products: their rates are those of the same products elsewhere.
//
// Precision.  dW is an fp32 main-grad: dz enters its product as two or three bf16 parts (parts_of).  dy is stored in bf16: dz enters in
// one part, rounded once more than the result, as every bf16 tensor between kernels here, or of few rows in two (dy_parts_of).
//
// Rows whose label is outside the vocabulary have no loss and no gradient, whatever their y holds: dz is set to zero, and dW's
// product reads a copy of y in which those rows are zero (a zero times an infinity is a NaN).
#include <float.h>
#include <math.h>

#include "../../include/bf_ops.h"
#include "common.h"

namespace bf {

namespace {

constexpr int NT = 256;
constexpr float LOG2E = 1.4426950408889634f;

inline size_t up(size_t n, size_t m) { return (n + m - 1) / m * m; }

bf_status launched() {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_error("vocab_loss: launch failed: %s", hipGetErrorString(e)); return BF_EDEVICE; }
  return BF_OK;
}

// (m, s) and (m2, s2): maxima, and sums of exponentials relative to them
__device__ __forceinline__ void merge(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  s = s * __builtin_amdgcn_exp2f((m - top) * LOG2E) + s2 * __builtin_amdgcn_exp2f((m2 - top) * LOG2E);
  m = top;
}

// 32 rows a workgroup, 8 threads to a row, each over every eighth tile in ascending order.  run (or NULL): what earlier pieces' tiles came
// to (unless first), and where these go with them (unless last)
__global__ __launch_bounds__(NT) void lse_merge_kernel(int rows, int tiles, const float2* __restrict__ part, const float* __restrict__ at_label,
                                                       const int32_t* __restrict__ label, int S_voc, float scale, float* __restrict__ lse,
                                                       float* __restrict__ row_loss, float2* __restrict__ run, int first, int last) {
  __shared__ float2 red[8][32];
  const int r = threadIdx.x & 31, g = threadIdx.x >> 5, row = blockIdx.x * 32 + r;
  float m = -FLT_MAX, s = 0.f;
  if (row < rows) {
#pragma unroll 4
    for (int k = g; k < tiles; k += 8) {
      const float2 p = part[(size_t)k * rows + row];
      merge(m, s, p.x, p.y);
    }
  }
  red[g][r] = make_float2(m, s);
  __syncthreads();
  if (g || row >= rows) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) merge(m, s, red[k][r].x, red[k][r].y);
  if (run && !first) merge(m, s, run[row].x, run[row].y);
  if (run && !last) {
    run[row] = make_float2(m, s);
    return;
  }
  const float l = m + logf(s);
  lse[row] = l;
  const int v = label[row];
  row_loss[row] = v >= 0 && v < S_voc ? (l - at_label[row]) * scale : 0.f;
}

__global__ __launch_bounds__(1024) void loss_sum_kernel(int rows, const float* __restrict__ row_loss, float* __restrict__ out) {
  double s = 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < rows; i += 1024) s += (double)row_loss[i];
  __shared__ double red[16];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x) return;
  for (int k = 1; k < 16; ++k) s += red[k];
  out[0] = (float)s;
}

// dst = src, rows without a label in the vocabulary as zeros
__global__ __launch_bounds__(NT) void labelled_rows_kernel(int h, const float* __restrict__ src, const int32_t* __restrict__ label, int S_voc,
                                                           float* __restrict__ dst) {
  const size_t row = blockIdx.x;
  const int v = label[row];
  const bool known = v >= 0 && v < S_voc;
  for (int c = threadIdx.x; c < h; c += NT) dst[row * h + c] = known ? src[row * h + c] : 0.f;
}

// the same for rows of whole 16-byte chunks of bf16
__global__ __launch_bounds__(NT) void labelled_rows16_kernel(int chunks, const uint4* __restrict__ src, const int32_t* __restrict__ label, int S_voc,
                                                             uint4* __restrict__ dst) {
  const size_t row = blockIdx.x;
  const int v = label[row];
  const bool known = v >= 0 && v < S_voc;
  for (int c = threadIdx.x; c < chunks; c += NT) dst[row * chunks + c] = known ? src[row * chunks + c] : make_uint4(0, 0, 0, 0);
}

// rows that are none: lengthened with zeros.  label: as above, or NULL: every row
typedef bf16_t V8 __attribute__((vector_size(16)));
__global__ __launch_bounds__(NT) void pad_rows_kernel(size_t n8, int h, int chunks, const bf16_t* __restrict__ src, const int32_t* __restrict__ label,
                                                      int S_voc, V8* __restrict__ dst) {
  for (size_t i = (size_t)blockIdx.x * NT + threadIdx.x; i < n8; i += (size_t)gridDim.x * NT) {
    const size_t row = i / chunks;
    const int c = (int)(i - row * chunks) * 8;
    const bool known = !label || (label[row] >= 0 && label[row] < S_voc);
    V8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = known && c + e < h ? src[row * h + c + e] : (bf16_t)0.f;
    dst[i] = o;
  }
}

// dw = (accumulate ? dw : 0) + a piece of lengthened rows
__global__ __launch_bounds__(NT) void cut_rows_kernel(size_t n, int h, int ld, const float* __restrict__ src, int accumulate, float* __restrict__ dw) {
  for (size_t i = (size_t)blockIdx.x * NT + threadIdx.x; i < n; i += (size_t)gridDim.x * NT) {
    const size_t row = i / h, c = i - row * h;
    const float v = src[row * ld + c];
    dw[i] = accumulate ? dw[i] + v : v;
  }
}

__global__ __launch_bounds__(NT) void add_kernel(size_t n, const float* __restrict__ src, float* __restrict__ dst) {
  for (size_t i = (size_t)blockIdx.x * NT + threadIdx.x; i < n; i += (size_t)gridDim.x * NT) dst[i] += src[i];
}

inline unsigned grid_for(size_t n) {
  const size_t g = (n + NT - 1) / NT;
  return (unsigned)(g < 1 ? 1 : g > 4096 ? 4096 : g);
}

// ---- fp32 logits, a piece at a time
// statistics of a row of the piece, merged into what earlier pieces left
__global__ __launch_bounds__(NT) void piece_lse_kernel(int rows, int cols, const float* __restrict__ z, const int32_t* __restrict__ label, int col0,
                                                       int first, float2* __restrict__ stat, float* __restrict__ at_label) {
  const int row = blockIdx.x;
  const float* zr = z + (size_t)row * cols;
  float m = -FLT_MAX, s = 0.f;
  for (int c = threadIdx.x; c < cols; c += NT) m = fmaxf(m, zr[c]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  __shared__ float red[2][NT / 64];
  if ((threadIdx.x & 63) == 0) red[0][threadIdx.x >> 6] = m;
  __syncthreads();
  m = fminf(fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3])), FLT_MAX);
  for (int c = threadIdx.x; c < cols; c += NT) s += expf(zr[c] - m);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) red[1][threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x) return;
  s = red[1][0] + red[1][1] + red[1][2] + red[1][3];
  if (!first) merge(m, s, stat[row].x, stat[row].y);
  stat[row] = make_float2(m, s);
  const int at = label[row] - col0;
  if (at >= 0 && at < cols) at_label[row] = zr[at];
}

__global__ __launch_bounds__(NT) void piece_dz_kernel(int cols, float* __restrict__ z, const int32_t* __restrict__ label, const float* __restrict__ lse,
                                                      int col0, int S_voc, float scale) {
  const size_t row = blockIdx.x;
  float* zr = z + row * (size_t)cols;
  const int v = label[row], at = v - col0;
  const bool known = v >= 0 && v < S_voc;
  const float l = lse[row];
  for (int c = threadIdx.x; c < cols; c += NT) zr[c] = known ? (expf(zr[c] - l) - (c == at ? 1.f : 0.f)) * scale : 0.f;
}

// ---- sizes ---------------------------------------------------------------------------------------
constexpr size_t PIECE_BYTES = (size_t)256 << 20;  // of dz: what the memory-side cache holds, and little beside 288 GB

// dz's parts in dw's product.  Error of dw in the 2-norm and gradient's time, 2048 rows, 16384 columns: two parts 1.6e-6 to 1.75e-6 whatever
// S_hidden; three, which leave the fp32 error of the logits and of the sums, 5.8e-7 at 1024 (388 us, two 320), 7.4e-7 at 4096 (1140, 925), 8.4e-7 at
// 6144 (1697, 1383), 8.8e-7 at 7168 (1950, 1568), 9.3e-7 at 8192 (2162, 1763).  So the third part costs a fifth of the gradient at any size, and
// is taken while it makes dw twice as exact, which ends between 7168 and 8192.  Up to some 200 rows dw's product is the writing of dw, and the
// third part costs nothing.
inline int parts_of(int rows, int h) { return rows <= 256 || h < 8192 ? 3 : 2; }

// dy is stored in bf16, and dz's rounding in one part is one more: 1.95e-3 off in the 2-norm at any number of rows, 1.66e-3, a rounding alone, with
// two.  Of few rows the largest dz, the label's, may fall where bf16 is coarsest for all of them: at most over 60 draws 3.3e-3 (1.9e-3 with two parts) for
// one row, 2.5e-3 for four, 2.2e-3 for 16, 2.0e-3 for 64 and more.  Two parts cost 13 % of the gradient up to 64 rows, where reading w bounds
// the product, 23 % at 128, 27 % at 256 (2048 x 16384: 142 us, 180), and then buy the mean's seventh alone: 16 % at 300, 11 % at 1024.
// One part is taken without the scale, which enters with dy's rounding: a label of small probability is then -1, whose rounding is none, and not
// -scale, whose rounding all rows share (1720 rows of 64: 2.8e-3 off, 2.0e-3 so).  Its plane costs 2 to 4 % of the gradient.
inline int dy_parts_of(int rows) { return rows <= 256 ? 2 : 1; }
inline int planes_of(int rows, int h) { return parts_of(rows, h) + (dy_parts_of(rows) == 1); }

// dy = factor * the sum of its slices' planes, in their order, of the h first of a plane's 8 * chunks columns
template <bool CUT>
__global__ __launch_bounds__(NT) void dy_finish_kernel(size_t n8, int h, int chunks, int slices, const float4* __restrict__ planes, float factor,
                                                       bf16_t* __restrict__ dy) {
  for (size_t i = (size_t)blockIdx.x * NT + threadIdx.x; i < n8; i += (size_t)gridDim.x * NT) {
    float4 a = planes[2 * i], b = planes[2 * i + 1];
    for (int k = 1; k < slices; ++k) {
      const float4 c = planes[2 * (k * n8 + i)], d = planes[2 * (k * n8 + i) + 1];
      a.x += c.x; a.y += c.y; a.z += c.z; a.w += c.w;
      b.x += d.x; b.y += d.y; b.z += d.z; b.w += d.w;
    }
    const V8 o = {(bf16_t)(a.x * factor), (bf16_t)(a.y * factor), (bf16_t)(a.z * factor), (bf16_t)(a.w * factor),
                  (bf16_t)(b.x * factor), (bf16_t)(b.y * factor), (bf16_t)(b.z * factor), (bf16_t)(b.w * factor)};
    if (!CUT) {
      reinterpret_cast<V8*>(dy)[i] = o;
    } else {
      const size_t row = i / chunks;
      const int c = (int)(i - row * chunks) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < h) dy[row * h + c + e] = o[e];
    }
  }
}

struct Plan {
  bool matrix;   // bf16 matrix cores, else fp32 products
  int piece;     // columns of the largest piece
  int unit;      // pieces are multiples of this, but for the last one
  bool pad;      // lengthened rows
  int h;         // row length of the products
  bool merge;    // bf16 forward: statistics merged piece by piece, so that they do not grow with the vocabulary
  // offsets into the scratch: copy of y, lengthened piece of W and its dw, z / dz, planes of dy, statistics (or a piece's dy), those of
  // earlier pieces, labels' logits
  size_t y, w, dw, z, dy, stat, run, lab, total;
  int slices;
};

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

bool sizes_ok(int dtype, int rows, int h, int V, int piece) {
  return (dtype == BF_FP32 || dtype == BF_BF16) && rows >= 1 && h >= 1 && V >= 1 && piece >= 0 && rows <= (1 << 21) && h <= (1 << 21) && V <= (1 << 21);
}

// columns of the piece at c0
int cols_at(const Plan& p, int c0, int V) {
  const int left = V - c0;
  if (left >= p.piece) return p.piece;
  return p.matrix && left > p.unit ? left / p.unit * p.unit : left;
}

// bf16 rows that are not whole 16-byte chunks, or do not start at one, are lengthened: copies of y and of a piece of w, the piece's dw and
// dy's planes in the scratch (142 rows of 170, 58496 columns, loss and gradient: as fp32 products 1358 us, so 186; 138 for rows of 176, which are whole chunks).  Where the tensors start is not known when the scratch is sized: the larger of the two
Plan plan_for(bool pad, int dtype, int rows, int h_given, int V, int piece, bool backward) {
  Plan p{};
  const bool matrix = dtype == BF_BF16;
  const int h = matrix ? (int)up(h_given, 8) : h_given;
  p.matrix = matrix;
  p.pad = pad;
  p.h = h;
  const size_t per_col = (size_t)rows * (matrix ? 2 * (size_t)planes_of(rows, h) : 4);
  size_t cols = piece ? (size_t)piece : PIECE_BYTES / per_col;
  if (cols < 1024 && !piece) cols = 1024;
  // fp32 dy: a product's sum over the columns is one chain in fp32, so it is cut (50304 columns in one: 1.1e-6 off, 6e-7 cut)
  if (!matrix && backward && !piece && cols > 4096) cols = 4096;
  p.unit = 8;
  if (matrix) {
    // a forward product keeps nothing: the vocabulary in one, but for the 2^32 threads of a launch (512 to 256 x 256, 256 to 128 x 128 logits)
    const size_t most = ((size_t)1 << 37) / rows / 256 * 256;
    if (!backward && (!piece || cols > most)) cols = !piece && (size_t)V < most ? (size_t)V : most;
    // whole rounds of tiles and a rest: 2048 x 2048 x 50304 in pieces of 25600 (3.1 rounds of 256 x 256) and of 24576 (3), us for logits and dw of
    // one: 250 + 429 and 208 + 350
    const int round = gemm_mfma_logits_round(rows, h);
    if (!piece && round) {
      if (cols >= (size_t)round) p.unit = round;
    } else if (backward && !piece && cols < (size_t)V) {
      cols = up((V + (V + cols - 1) / cols - 1) / ((V + cols - 1) / cols), 512);  // pieces of about the same size
    }
    cols = p.unit == 8 ? up(cols, 8) : cols / p.unit * p.unit;
  }
  if (pad && !piece && cols > PIECE_BYTES / 4 / h) cols = PIECE_BYTES / 4 / h < 1024 ? 1024 : PIECE_BYTES / 4 / h / 8 * 8;
  if (cols > (size_t)V) cols = (size_t)V;
  if (p.unit > 8 && cols >= (size_t)p.unit) cols = cols / p.unit * p.unit;
  p.piece = (int)cols;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += up(bytes, 256); return o; };
  if (matrix) {
    if (pad) {
      p.w = take(cols * h * 2);
      if (backward) p.dw = take(cols * h * 4);
      else p.y = take((size_t)rows * h * 2);
    }
    if (backward) {
      p.slices = gemm_mfma_logits_dy_slices(rows, p.piece, h);
      p.y = take((size_t)rows * h * 2);
      p.z = take((size_t)rows * up(cols, 8) * 2 * planes_of(rows, h));
      p.dy = take((size_t)p.slices * rows * h * 4);
    } else {
      size_t tiles = 0;
      p.merge = piece != 0;
      if (p.merge) tiles = (cols + 63) / 64;  // of any piece: the smallest tile is 64 wide
      else for (int c0 = 0, n; c0 < V; c0 += n) tiles += gemm_mfma_logits_tiles(rows, n = cols_at(p, c0, V));
      p.stat = take(tiles * rows * 8);
      if (p.merge) p.run = take((size_t)rows * 8);
      p.lab = take((size_t)rows * 4);
    }
  } else {
    p.y = take((size_t)rows * h * 4);
    p.z = take((size_t)rows * cols * 4);
    if (backward) {
      p.stat = take(p.piece < V ? (size_t)rows * h * 4 : 0);  // a later piece's share of dy
    } else {
      p.stat = take((size_t)rows * 8);
      p.lab = take((size_t)rows * 4);
    }
  }
  p.total = at;
  return p;
}

bf_status pad_rows(size_t n, int h, int h8, const bf16_t* src, const int32_t* label, int V, void* dst, hipStream_t st) {
  const size_t n8 = n * (h8 / 8);
  pad_rows_kernel<<<grid_for(n8), NT, 0, st>>>(n8, h, h8 / 8, src, label, V, (V8*)dst);
  return launched();
}

bf_status product(int layout, int epi, GemmArgs a, hipStream_t st) { return gemm(BF_FP32, BF_KERNELS_AUTO, layout, epi, a, st); }

}  // namespace

size_t vocab_loss_work_bytes(int dtype, int rows, int h, int V, int piece, int backward) {
  if (!sizes_ok(dtype, rows, h, V, piece)) return 0;
  size_t n = plan_for(false, dtype, rows, h, V, piece, backward != 0).total;
  if (dtype == BF_BF16) {
    const size_t m = plan_for(true, dtype, rows, h, V, piece, backward != 0).total;
    n = n > m ? n : m;
  }
  return n;
}

static bf_status check_args(const char* who, int dtype, int rows, int h, int V, int piece, const void* y, const void* w, const int32_t* label, const void* a,
                            const void* b, const void* c, float scale, const void* work, size_t work_bytes, int backward) {
  if (!sizes_ok(dtype, rows, h, V, piece)) { set_error("%s: bad type or sizes (1 .. 2^21)", who); return BF_EINVAL; }
  if (!y || !w || !label || !a || !b || !c) { set_error("%s: null pointer", who); return BF_EINVAL; }
  // (a, b and c: fp32, but for a backward call's b, which is dy)
  const uintptr_t wide = (uintptr_t)label | (uintptr_t)a | (uintptr_t)c | (backward ? 0 : (uintptr_t)b), stored = (uintptr_t)y | (uintptr_t)w | (backward ? (uintptr_t)b : 0);
  if ((wide & 3) || (stored & (dtype == BF_BF16 ? 1 : 3))) { set_error("%s: a tensor is not aligned to its elements", who); return BF_EINVAL; }
  if (!(fabsf(scale) <= FLT_MAX)) { set_error("%s: scale is not finite", who); return BF_EINVAL; }
  const size_t need = vocab_loss_work_bytes(dtype, rows, h, V, piece, backward);
  if (!work || ((uintptr_t)work & 255) || work_bytes < need) { set_error("%s: needs %zu bytes of 256-byte aligned scratch", who, need); return BF_EINVAL; }
  return BF_OK;
}

bf_status vocab_loss_fwd(int dtype, int rows, int h, int V, int piece, const void* y, const void* w, const int32_t* label, float scale, float* lse,
                         float* row_loss, float* loss, void* work, size_t work_bytes, hipStream_t st) {
  bf_status s = check_args("bf_op_vocab_loss_fwd", dtype, rows, h, V, piece, y, w, label, lse, row_loss, loss, scale, work, work_bytes, 0);
  if (s != BF_OK) return s;
  const Plan p = plan_for(h % 8 || !aligned16(y) || !aligned16(w), dtype, rows, h, V, piece, false);
  char* ws = (char*)work;
  float* stat = (float*)(ws + p.stat);
  int tiles = 1;
  bool pieces = false;  // some of the vocabulary is in `run` already
  float* at_label = (float*)(ws + p.lab);
  float2* run = p.matrix && p.merge ? (float2*)(ws + p.run) : nullptr;
  if (p.matrix) {
    LogitArgs l;
    l.label = label;
    l.at_label = at_label;
    tiles = 0;
    const void* ym = y;
    if (p.pad) {
      s = pad_rows(rows, h, p.h, (const bf16_t*)y, nullptr, V, ws + p.y, st);
      if (s != BF_OK) return s;
      ym = ws + p.y;
    }
    for (int c0 = 0, n; c0 < V; c0 += n) {
      int done = 0;
      n = cols_at(p, c0, V);
      l.part = stat + (size_t)tiles * rows * 2;
      l.col0 = c0;
      const void* wp = (const bf16_t*)w + (size_t)c0 * h;
      if (p.pad) {
        s = pad_rows(n, h, p.h, (const bf16_t*)wp, nullptr, V, ws + p.w, st);
        if (s != BF_OK) return s;
        wp = ws + p.w;
      }
      s = gemm_mfma_logits_lse(rows, n, p.h, ym, wp, l, &done, st);
      if (s != BF_OK) return s;
      tiles += done;
      if (run && c0 + n < V) {
        lse_merge_kernel<<<(rows + 31) / 32, NT, 0, st>>>(rows, tiles, (const float2*)stat, at_label, label, V, scale, lse, row_loss, run, c0 == 0, 0);
        s = launched();
        if (s != BF_OK) return s;
        tiles = 0;
        pieces = true;
      }
    }
  } else {
    float* z = (float*)(ws + p.z);
    const float* yf = (const float*)y;
    for (int c0 = 0, n; c0 < V; c0 += n) {
      const int cols = n = cols_at(p, c0, V);
      const float* wf = (const float*)w + (size_t)c0 * h;
      s = product(L_NT, E_NONE, GemmArgs{rows, cols, h, yf, wf, z, nullptr, nullptr, nullptr, 0}, st);
      if (s != BF_OK) return s;
      piece_lse_kernel<<<rows, NT, 0, st>>>(rows, cols, z, label, c0, c0 == 0, (float2*)stat, at_label);
      s = launched();
      if (s != BF_OK) return s;
    }
  }
  lse_merge_kernel<<<(rows + 31) / 32, NT, 0, st>>>(rows, tiles, (const float2*)stat, at_label, label, V, scale, lse, row_loss, run, !pieces, 1);
  s = launched();
  if (s != BF_OK) return s;
  loss_sum_kernel<<<1, 1024, 0, st>>>(rows, row_loss, loss);
  return launched();
}

bf_status vocab_loss_bwd(int dtype, int rows, int h, int V, int piece, const void* y, const void* w, const int32_t* label, const float* lse, float scale,
                         void* dy, float* dw, int accumulate, void* work, size_t work_bytes, hipStream_t st) {
  bf_status s = check_args("bf_op_vocab_loss_bwd", dtype, rows, h, V, piece, y, w, label, lse, dy, dw, scale, work, work_bytes, 1);
  if (s != BF_OK) return s;
  const bool al = aligned16(y) && aligned16(w) && aligned16(dy) && aligned16(dw);
  const Plan p = plan_for(h % 8 || !al, dtype, rows, h, V, piece, true);
  char* ws = (char*)work;
  if (p.matrix) {
    bf16_t* yc = (bf16_t*)(ws + p.y);
    float* planes = (float*)(ws + p.dy);
    const bool unscaled = dy_parts_of(rows) == 1;
    if (p.pad) {
      s = pad_rows(rows, h, p.h, (const bf16_t*)y, label, V, yc, st);
    } else {
      labelled_rows16_kernel<<<rows, NT, 0, st>>>(h / 8, (const uint4*)y, label, V, (uint4*)yc);
      s = launched();
    }
    for (int c0 = 0, n; c0 < V && s == BF_OK; c0 += n) {
      const int cols = n = cols_at(p, c0, V);
      LogitArgs l;
      l.label = label;
      l.lse = lse;
      l.scale = scale;
      l.col0 = c0;
      l.S_voc = V;
      l.parts = parts_of(rows, p.h);
      l.unscaled = unscaled;
      l.ldc = (int)up(cols, 8);
      l.plane = (size_t)rows * l.ldc;
      void* dz = ws + p.z;
      const bf16_t* wp = (const bf16_t*)w + (size_t)c0 * h;
      float* dwp = dw + (size_t)c0 * h;
      if (p.pad) {
        s = pad_rows(cols, h, p.h, wp, nullptr, V, ws + p.w, st);
        wp = (const bf16_t*)(ws + p.w);
        dwp = (float*)(ws + p.dw);
      }
      // (rows without a label have dz = 0 whatever their logits are)
      if (s == BF_OK) s = gemm_mfma_logits_grad(rows, cols, p.h, p.pad ? yc : y, wp, l, dz, st);
      if (s == BF_OK) s = gemm_mfma_logits_dw(rows, cols, p.h, dz, l.ldc, l.parts, l.plane, yc, dwp, p.pad ? 0 : accumulate, st);
      if (s == BF_OK && p.pad) {
        cut_rows_kernel<<<grid_for((size_t)cols * h), NT, 0, st>>>((size_t)cols * h, h, p.h, dwp, accumulate, dw + (size_t)c0 * h);
        s = launched();
      }
      if (s == BF_OK) s = gemm_mfma_logits_dy(rows, cols, p.h, (bf16_t*)dz + (unscaled ? l.parts * l.plane : 0), l.ldc, dy_parts_of(rows), l.plane, wp, planes,
                                              p.slices, c0 > 0, st);
    }
    if (s != BF_OK) return s;
    const size_t n8 = (size_t)rows * p.h / 8;
    const float factor = unscaled ? scale : 1.f;
    if (p.pad) dy_finish_kernel<true><<<grid_for(n8), NT, 0, st>>>(n8, h, p.h / 8, p.slices, (const float4*)planes, factor, (bf16_t*)dy);
    else dy_finish_kernel<false><<<grid_for(n8), NT, 0, st>>>(n8, h, p.h / 8, p.slices, (const float4*)planes, factor, (bf16_t*)dy);
    return launched();
  }
  float* yc = (float*)(ws + p.y);
  float* z = (float*)(ws + p.z);
  float* share = (float*)(ws + p.stat);
  float* dyf = (float*)dy;
  for (int c0 = 0, n; c0 < V; c0 += n) {
    const int cols = n = cols_at(p, c0, V);
    const float *wf = (const float*)w + (size_t)c0 * h, *yf = (const float*)y;
    s = product(L_NT, E_NONE, GemmArgs{rows, cols, h, yf, wf, z, nullptr, nullptr, nullptr, 0}, st);
    if (s != BF_OK) return s;
    piece_dz_kernel<<<rows, NT, 0, st>>>(cols, z, label, lse, c0, V, scale);
    if (c0 == 0) labelled_rows_kernel<<<rows, NT, 0, st>>>(h, (const float*)y, label, V, yc);
    s = launched();
    if (s != BF_OK) return s;
    s = product(L_NN, E_NONE, GemmArgs{rows, h, cols, z, wf, c0 ? share : dyf, nullptr, nullptr, nullptr, 0}, st);
    if (s != BF_OK) return s;
    if (c0) {
      add_kernel<<<grid_for((size_t)rows * h), NT, 0, st>>>((size_t)rows * h, share, dyf);
      s = launched();
      if (s != BF_OK) return s;
    }
    s = product(L_TN, E_ACCUM, GemmArgs{cols, h, rows, z, yc, dw + (size_t)c0 * h, nullptr, nullptr, nullptr, accumulate}, st);
    if (s != BF_OK) return s;
  }
  return BF_OK;
}

}  // namespace bf
