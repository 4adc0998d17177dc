// Global gradient norm over many tensors, clipping, and the Adam step on clipped gradients.
//
// norm = sqrt(sum over tensors and elements of g^2), in fp64 from the square on: no finite fp32 or bf16 gradient overflows
// it, and the sum of 1e10 terms keeps more bits than the result has.  coefficient = norm > max_norm ? max_norm / norm : 1,
// NaN where the norm is not finite.  It stays on the device: what follows reads it there, nothing waits on the host.
//
// All of it is HBM traffic (norm 4 or 2 bytes per element, scaled copy twice that, Adam 30).  A launch takes a table of tensors
// in its arguments (no copy of a table to the device, and a captured graph holds its own); the tensors' elements are dealt out in
// chunks of equal size over a grid that fills the chip, chunk c to workgroup c modulo the grid.  Sums: a thread's in the order of its
// chunks, threads and then workgroups in a fixed tree, so that a table gives the same bits every time.
#include <float.h>
#include <math.h>

#include "../../include/bf_ops.h"
#include "common.h"

namespace bf {

namespace {

constexpr int NT = 256;
constexpr int VECS = 8;                     // 16-byte accesses of a thread and chunk, all in flight at once
constexpr int MAX_WG = 2048;                // of a launch: eight to a compute unit
constexpr size_t MAX_ENTRY = (size_t)1 << 30;  // elements of a table entry; longer tensors take several

// Gradients may start at any element: 16-byte accesses that are only as aligned as their elements.
template <typename T> struct Chunk;
template <> struct Chunk<float> { typedef float V __attribute__((vector_size(16), aligned(4))); static constexpr int N = 4; };
template <> struct Chunk<bf16_t> { typedef bf16_t V __attribute__((vector_size(16), aligned(2))); static constexpr int N = 8; };

// P pointers per tensor; arguments of a kernel are limited to 4 KiB
template <int P, int CAP>
struct Table {
  const void* p[CAP][P];
  uint32_t n[CAP];
  uint32_t first[CAP + 1];  // first chunk of each entry
  int count;
};
constexpr int NORM_CAP = 220, SCALE_CAP = 150, ADAM_CAP = 75;
typedef Table<1, NORM_CAP> NormTable;
typedef Table<2, SCALE_CAP> ScaleTable;
typedef Table<5, ADAM_CAP> AdamTable;
static_assert(sizeof(NormTable) <= 3840 && sizeof(ScaleTable) <= 3840 && sizeof(AdamTable) <= 3840, "kernel arguments");

// entry of a chunk: the last one that starts at or in front of it (uniform over the workgroup)
template <typename TB>
__device__ __forceinline__ int entry_of(const TB& t, uint32_t chunk) {
  int lo = 0, hi = t.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.first[mid] <= chunk) lo = mid; else hi = mid;
  }
  return lo;
}

// 24 tensors of 4 to 16 Mi elements (0.94 GB) 159 us, 5.9 TB/s, in bf16 (0.43 GB) 80 us, 5.4; 200 of 256 to 256 Ki (22 MB) 7.5 us and the last sums 3
template <typename T>
__global__ __launch_bounds__(NT) void norm_kernel(NormTable t, double* __restrict__ part) {
  typedef typename Chunk<T>::V V;
  constexpr int N = Chunk<T>::N, CHUNK = NT * N * VECS;
  double s = 0;
  const uint32_t chunks = t.first[t.count];
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int e = entry_of(t, c);
    const T* g = (const T*)t.p[e][0];
    const uint32_t n = t.n[e], at = (c - t.first[e]) * CHUNK;
    if (at + CHUNK <= n) {
      V v[VECS];
#pragma unroll
      for (int i = 0; i < VECS; ++i) v[i] = *reinterpret_cast<const V*>(g + at + (i * NT + threadIdx.x) * N);
#pragma unroll
      for (int i = 0; i < VECS; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k) s = fma((double)(float)v[i][k], (double)(float)v[i][k], s);
    } else {
#pragma unroll 4
      for (uint32_t i = at + threadIdx.x; i < n; i += NT) s = fma((double)(float)g[i], (double)(float)g[i], s);
    }
  }
  __shared__ double red[NT / 64];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

__global__ __launch_bounds__(NT) void norm_finish_kernel(const double* __restrict__ part, int n, float max_norm, float* __restrict__ out) {
  double s = 0;
#pragma unroll 8
  for (int i = threadIdx.x; i < n; i += NT) s += part[i];
  __shared__ double red[NT / 64];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x) return;
  const double norm = sqrt(red[0] + red[1] + red[2] + red[3]);
  out[0] = (float)norm;
  // (a norm past fp32 is infinite as stored, but its coefficient is not)
  out[1] = !(norm <= DBL_MAX) ? NAN : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
}

// (those 200: 44 MB read and written in two launches of 12 us; 24 tensors of 4 to 16 Mi 333 us in fp32 and 173 in bf16, 5.2 and 5.0 TB/s)
template <typename T>
__global__ __launch_bounds__(NT) void scale_kernel(ScaleTable t, const float* __restrict__ coef) {
  typedef typename Chunk<T>::V V;
  constexpr int N = Chunk<T>::N, CHUNK = NT * N * VECS;
  const float k = coef[0];
  const uint32_t chunks = t.first[t.count];
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int e = entry_of(t, c);
    const T* g = (const T*)t.p[e][0];
    T* d = (T*)t.p[e][1];
    const uint32_t n = t.n[e], at = (c - t.first[e]) * CHUNK;
    if (at + CHUNK <= n) {
      V v[VECS];
#pragma unroll
      for (int i = 0; i < VECS; ++i) v[i] = *reinterpret_cast<const V*>(g + at + (i * NT + threadIdx.x) * N);
#pragma unroll
      for (int i = 0; i < VECS; ++i) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[i][j] = (T)((float)v[i][j] * k);
        *reinterpret_cast<V*>(d + at + (i * NT + threadIdx.x) * N) = v[i];
      }
    } else {
#pragma unroll 4
      for (uint32_t i = at + threadIdx.x; i < n; i += NT) d[i] = (T)((float)g[i] * k);
    }
  }
}

struct AdamArgs { float lr, beta1, beta2, eps, wd, c1, c2, omb1, omb2; };

// the fused Adam step (written out, so that whole chunks and their ends give the same bits)
__device__ __forceinline__ void adam_one(float& w, float& m, float& v, float g, const AdamArgs& a) {
  m = fmaf(a.omb1, g, a.beta1 * m);
  v = fmaf(a.omb2 * g, g, a.beta2 * v);
  w = fmaf(-a.lr, fmaf(a.wd, w, m * a.c1 / (sqrtf(v * a.c2) + a.eps)), w);
}

// On g * coefficient; a coefficient that is not finite leaves everything as it was
// Eight streams over HBM: the fewer places they are at, the faster.  One workgroup to a compute unit, with all its loads in flight
// at once (four streams of four vectors), and accesses that do not stay in the caches.  Norm and step of 24 tensors of 4 to 16
// Mi elements, us: 2048 workgroups with two vectors a stream 1637, without caching 1545; 512 with four 1451; 256 1386
// (256 with eight 1434; the norm alone does not change).  The step alone 1217 us, 5.8 TB/s.
constexpr int ADAM_VECS = 4;
constexpr unsigned ADAM_WG = 256;
__global__ __launch_bounds__(NT) void adam_clipped_kernel(AdamTable t, const float* __restrict__ coef, AdamArgs a) {
  typedef Chunk<float>::V V;
  typedef bf16_t V4 __attribute__((vector_size(8), aligned(2)));
  constexpr int CHUNK = NT * 4 * ADAM_VECS;
  const float k = coef[0];
  if (!(fabsf(k) <= FLT_MAX)) return;
  const uint32_t chunks = t.first[t.count];
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int e = entry_of(t, c);
    float *w = (float*)t.p[e][0], *m = (float*)t.p[e][1], *v = (float*)t.p[e][2];
    const float* g = (const float*)t.p[e][3];
    bf16_t* lp = (bf16_t*)t.p[e][4];
    const uint32_t n = t.n[e], at = (c - t.first[e]) * CHUNK;
    if (at + CHUNK <= n) {
      V ww[ADAM_VECS], mm[ADAM_VECS], vv[ADAM_VECS], gg[ADAM_VECS];
#pragma unroll
      for (int i = 0; i < ADAM_VECS; ++i) {
        const uint32_t q = at + (i * NT + threadIdx.x) * 4;
        ww[i] = __builtin_nontemporal_load(reinterpret_cast<const V*>(w + q));
        mm[i] = __builtin_nontemporal_load(reinterpret_cast<const V*>(m + q));
        vv[i] = __builtin_nontemporal_load(reinterpret_cast<const V*>(v + q));
        gg[i] = __builtin_nontemporal_load(reinterpret_cast<const V*>(g + q));
      }
#pragma unroll
      for (int i = 0; i < ADAM_VECS; ++i) {
        const uint32_t q = at + (i * NT + threadIdx.x) * 4;
        V4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float w1 = ww[i][j], m1 = mm[i][j], v1 = vv[i][j];
          adam_one(w1, m1, v1, gg[i][j] * k, a);
          ww[i][j] = w1; mm[i][j] = m1; vv[i][j] = v1;
          o[j] = (bf16_t)w1;
        }
        __builtin_nontemporal_store(ww[i], reinterpret_cast<V*>(w + q));
        __builtin_nontemporal_store(mm[i], reinterpret_cast<V*>(m + q));
        __builtin_nontemporal_store(vv[i], reinterpret_cast<V*>(v + q));
        if (lp) __builtin_nontemporal_store(o, reinterpret_cast<V4*>(lp + q));
      }
    } else {
      for (uint32_t i = at + threadIdx.x; i < n; i += NT) {
        float w1 = w[i], m1 = m[i], v1 = v[i];
        adam_one(w1, m1, v1, g[i] * k, a);
        w[i] = w1; m[i] = m1; v[i] = v1;
        if (lp) lp[i] = (bf16_t)w1;
      }
    }
  }
}

// Fills a table from tensor `at` on (`off`: elements of it already taken), as much as fits; false when nothing was left.
// size(i): elements of tensor i; ptr(i, j, o): its pointer j, o elements further on.
template <typename TB, int P, int CAP, typename SZ, typename PT>
bool fill(TB& t, uint32_t chunk, int n_tensors, int& at, size_t& off, SZ size, PT ptr) {
  t.count = 0;
  t.first[0] = 0;
  while (at < n_tensors && t.count < CAP) {
    if (off >= size(at)) { ++at; off = 0; continue; }
    const size_t left = size(at) - off, take = left < MAX_ENTRY ? left : MAX_ENTRY;
    for (int j = 0; j < P; ++j) t.p[t.count][j] = ptr(at, j, off);
    t.n[t.count] = (uint32_t)take;
    t.first[t.count + 1] = t.first[t.count] + (uint32_t)((take + chunk - 1) / chunk);  // at most CAP * MAX_ENTRY / chunk < 2^31
    ++t.count;
    off += take;
  }
  return t.count > 0;
}

bf_status launched() {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_error("clip: launch failed: %s", hipGetErrorString(e)); return BF_EDEVICE; }
  return BF_OK;
}

bool list_ok(const char* who, int n_tensors, const void* list, const size_t* n) {
  if (n_tensors < 0 || (n_tensors > 0 && (!list || !n))) { set_error("%s: bad list of tensors", who); return false; }
  return true;
}

inline unsigned grid_of(uint32_t chunks) { return chunks < MAX_WG ? chunks : MAX_WG; }

// launches of the norm: entries of a list over entries of a table
size_t norm_launches(int n_tensors, const size_t* n) {
  size_t entries = 0;
  for (int i = 0; i < n_tensors; ++i) entries += (n[i] + MAX_ENTRY - 1) / MAX_ENTRY;
  return (entries + NORM_CAP - 1) / NORM_CAP;
}

}  // namespace

size_t grad_norm_work_bytes(int n_tensors, const size_t* n) {
  if (n_tensors < 0 || (n_tensors > 0 && !n)) return 0;
  const size_t l = norm_launches(n_tensors, n);
  return (l ? l : 1) * MAX_WG * sizeof(double);
}

bf_status grad_norm(int dtype, int n_tensors, const void* const* g, const size_t* n, float max_norm, float* out, void* work, size_t work_bytes,
                    hipStream_t st) {
  if (!list_ok("bf_op_grad_norm", n_tensors, g, n)) return BF_EINVAL;
  if (!(max_norm > 0.f)) { set_error("bf_op_grad_norm: max_norm must be above 0"); return BF_EINVAL; }
  if (!out || ((uintptr_t)out & 3)) { set_error("bf_op_grad_norm: out is null or not aligned to its elements"); return BF_EINVAL; }
  if (!work || ((uintptr_t)work & 7) || work_bytes < grad_norm_work_bytes(n_tensors, n)) {
    set_error("bf_op_grad_norm: needs %zu bytes of 8-byte aligned scratch", grad_norm_work_bytes(n_tensors, n));
    return BF_EINVAL;
  }
  const size_t es = dtype == BF_BF16 ? 2 : 4;
  for (int i = 0; i < n_tensors; ++i)
    if (n[i] && (!g[i] || ((uintptr_t)g[i] & (es - 1)))) { set_error("bf_op_grad_norm: tensor %d is null or not aligned to its elements", i); return BF_EINVAL; }
  double* part = (double*)work;
  int parts = 0, at = 0;
  size_t off = 0;
  NormTable t;
  const uint32_t chunk = NT * VECS * 16 / es;
  while (fill<NormTable, 1, NORM_CAP>(t, chunk, n_tensors, at, off, [&](int i) { return n[i]; }, [&](int i, int, size_t o) { return (const char*)g[i] + o * es; })) {
    const unsigned grid = grid_of(t.first[t.count]);
    if (dtype == BF_BF16) norm_kernel<bf16_t><<<grid, NT, 0, st>>>(t, part + parts);
    else norm_kernel<float><<<grid, NT, 0, st>>>(t, part + parts);
    const bf_status s = launched();
    if (s != BF_OK) return s;
    parts += (int)grid;
  }
  norm_finish_kernel<<<1, NT, 0, st>>>(part, parts, max_norm, out);
  return launched();
}

bf_status grad_scale(int dtype, int n_tensors, const void* const* g, void* const* dst, const size_t* n, const float* coef, hipStream_t st) {
  if (!list_ok("bf_op_grad_scale", n_tensors, g, n) || !list_ok("bf_op_grad_scale", n_tensors, dst, n)) return BF_EINVAL;
  if (!coef || ((uintptr_t)coef & 3)) { set_error("bf_op_grad_scale: coef is null or not aligned to its elements"); return BF_EINVAL; }
  const size_t es = dtype == BF_BF16 ? 2 : 4;
  for (int i = 0; i < n_tensors; ++i)
    if (n[i] && (!g[i] || !dst[i] || (((uintptr_t)g[i] | (uintptr_t)dst[i]) & (es - 1)))) {
      set_error("bf_op_grad_scale: tensor %d is null or not aligned to its elements", i);
      return BF_EINVAL;
    }
  int at = 0;
  size_t off = 0;
  ScaleTable t;
  const uint32_t chunk = NT * VECS * 16 / es;
  while (fill<ScaleTable, 2, SCALE_CAP>(t, chunk, n_tensors, at, off, [&](int i) { return n[i]; },
                             [&](int i, int j, size_t o) { return (j ? (const char*)dst[i] : (const char*)g[i]) + o * es; })) {
    const unsigned grid = grid_of(t.first[t.count]);
    if (dtype == BF_BF16) scale_kernel<bf16_t><<<grid, NT, 0, st>>>(t, coef);
    else scale_kernel<float><<<grid, NT, 0, st>>>(t, coef);
    const bf_status s = launched();
    if (s != BF_OK) return s;
  }
  return BF_OK;
}

bf_status adam_clipped(int n_tensors, const bf_adam_tensor* x, const float* coef, int step, float lr, float beta1, float beta2, float eps, float wd,
                       hipStream_t st) {
  if (n_tensors < 0 || (n_tensors > 0 && !x)) { set_error("bf_op_adam_clipped: bad list of tensors"); return BF_EINVAL; }
  if (!coef || ((uintptr_t)coef & 3) || step < 1) { set_error("bf_op_adam_clipped: coef is null or not aligned to its elements, or step below 1"); return BF_EINVAL; }
  for (int i = 0; i < n_tensors; ++i) {
    if (!x[i].n) continue;
    const uintptr_t al = (uintptr_t)x[i].w | (uintptr_t)x[i].m | (uintptr_t)x[i].v | (uintptr_t)x[i].g;
    if (!x[i].w || !x[i].m || !x[i].v || !x[i].g || (al & 3) || ((uintptr_t)x[i].w_lp & 1)) {
      set_error("bf_op_adam_clipped: tensor %d has a null pointer or one not aligned to its elements", i);
      return BF_EINVAL;
    }
  }
  AdamArgs a{lr, beta1, beta2, eps, wd, (float)(1.0 / (1.0 - pow((double)beta1, (double)step))), (float)(1.0 / (1.0 - pow((double)beta2, (double)step))),
             (float)(1.0 - (double)beta1), (float)(1.0 - (double)beta2)};
  int at = 0;
  size_t off = 0;
  AdamTable t;
  while (fill<AdamTable, 5, ADAM_CAP>(
      t, NT * 4 * ADAM_VECS, n_tensors, at, off, [&](int i) { return x[i].n; },
      [&](int i, int j, size_t o) -> const void* {
        return j == 0 ? x[i].w + o : j == 1 ? x[i].m + o : j == 2 ? x[i].v + o : j == 3 ? x[i].g + o : x[i].w_lp ? (const void*)((const bf16_t*)x[i].w_lp + o) : nullptr;
      })) {
    adam_clipped_kernel<<<min(grid_of(t.first[t.count]), ADAM_WG), NT, 0, st>>>(t, coef, a);
    const bf_status s = launched();
    if (s != BF_OK) return s;
  }
  return BF_OK;
}

}  // namespace bf
