// The clipped Adam step with both moments in 8 bits, over a list of tensors.
//
// A block of 128 elements keeps 128 codes of m, 128 of v and a power-of-two scale each.  The step is taken in fp32 from what the codes stand for; the new
// moments are rounded at random: y = |moment| 2^-e lies between two codes, `step` apart, and goes up where (floor(65536 y / step) + r) mod 65536 carries, r 16
// random bits.  Rounding to nearest would freeze a mean whose change per step is under half a code (v with beta2 = 0.95 changes by 5 % at most
// on the way down, half a code of v is 1.6 to 3.1 %, of m 3.1 to 6.3 %).
// m: e4m3.  v has no sign, and the bit goes to the mantissa: codes of 4 bits of exponent and 4 of mantissa.  v is kept and not its root, so that its
// mean is the one that is unbiased; over a block it spans 5e5, its root 700.
// A v that is infinite has m's code 0xff, which stands for m = 0 and v = infinity: its element rests for good, but for the weight decay, as it does on fp32 moments, where a
// finite m is divided by it.  (v's codes have no room for it, and as the largest finite code of its neighbours' scale the next step would read it as small.)  NaN is 0x7f.
//
// HBM traffic: 18 bytes an element (w 4 + 4, g 4, codes 2 + 2, bf16 copy 2).  A block is 32 lanes of 4 elements, so that maxima meet by lane rotations.
#include <float.h>
#include <math.h>

#include "../../include/bf_ops.h"
#include "common.h"

namespace bf {

namespace {

constexpr int NT = 256, BLK = 128;
constexpr size_t MAX_ENTRY = (size_t)1 << 30;  // elements of a table entry (whole blocks); longer tensors take several

// What a launch works on, in its arguments (at most 4 KiB).  p: w, codes, scales, g, w_lp; or m, codes, scales, v
constexpr int CAP = 64;
struct Table8 {
  const void* p[CAP][5];
  uint32_t n[CAP];
  uint32_t first[CAP + 1];  // first chunk of each entry
  uint32_t key[CAP];        // of the random numbers, what element 0 of the entry adds to it included
  int count;
};
static_assert(sizeof(Table8) <= 3600, "kernel arguments");

struct AdamArgs8 { float lr, eps, wd, c1, c2, beta1, beta2, omb1, omb2; };

// xor shifts and odd multipliers (the first 32 bits of the fractions of sqrt 2 and sqrt 3): over random inputs a flipped input bit flips
// every output bit with a chance of 0.495 to 0.505
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x = (x ^ (x >> 15)) * 0x6A09E667u;
  x = (x ^ (x >> 13)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}

__device__ __forceinline__ int entry_of8(const Table8& t, uint32_t chunk) {
  int lo = 0, hi = t.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.first[mid] <= chunk) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ uint32_t max32(uint32_t x) {  // over the 32 lanes of a half wave
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x128, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x124, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x122, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x121, 0xf, 0xf, false));
  return max(x, (uint32_t)__shfl_xor((int)x, 16, 64));
}

__device__ __forceinline__ uint32_t finite_bits8(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}

// smallest e >= -127 with amax <= (1 + top / 2^23) 2^(e + EXP); 0 has -127
template <int EXP, uint32_t TOP>
__device__ __forceinline__ int exponent8(uint32_t amax) {
  return max((int)(amax >> 23) - 127 - EXP + ((amax & 0x7fffffu) > TOP ? 1 : 0), -127);
}
constexpr int EXP_M = 8, EXP_V = 14;
constexpr uint32_t TOP_M = 0x600000u, TOP_V = 0x780000u;  // 1.75, 1.9375

__device__ __forceinline__ float decode_m(uint32_t codes, int k) {
  switch (k) {  // (the byte is part of the instruction)
    case 0: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 0);
    case 1: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 1);
    case 2: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 2);
    default: return __builtin_amdgcn_cvt_f32_fp8((int)codes, 3);
  }
}
// c < 16: c / 16; else (1 + c % 16 / 16) 2^(c / 16 - 1)
__device__ __forceinline__ float decode_v(uint32_t codes, int k) {
  const uint32_t c = (codes >> (8 * k)) & 255u;
  return c < 16 ? (float)c * 0.0625f : __uint_as_float((c << 19) + ((uint32_t)(127 - 1) << 23));
}

// whether one of the four codes of m is 0xff (a byte of the complement is zero)
__device__ __forceinline__ bool any_rests(uint32_t codes) { return ((~codes - 0x01010101u) & codes & 0x80808080u) != 0; }

// the moments that a code 0xff of m stands for
__device__ __forceinline__ void resting(uint32_t codes, float (&m)[4], float (&v)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const bool r = ((codes >> (8 * k)) & 255u) == 0xffu;
    m[k] = r ? 0.f : m[k];
    v[k] = r ? __uint_as_float(0x7f800000u) : v[k];
  }
}

// New moments.  Each operation is rounded by itself, so that the codes are the same bits wherever the definition is computed like this: a moment that is
// off by one rounding lands in another code once in a million, and a small v's next code changes its step by a third.
__device__ __forceinline__ void moments8(float& m, float& v, float g, const AdamArgs8& a) {
#pragma clang fp contract(off)
  m = a.beta1 * m + a.omb1 * g;
  v = a.beta2 * v + a.omb2 * g * g;
}

// code of y >= 0 (LOW: exponent of the smallest normal code, BITS of mantissa), r: 16 random bits
template <int LOW, int BITS>
__device__ __forceinline__ uint32_t encode(float y, uint32_t r) {
  const int e = max((int)(__float_as_uint(y) >> 23) - 127, LOW);
  const uint32_t k = (uint32_t)(y * __uint_as_float((uint32_t)(127 + 16 + BITS - e) << 23));  // y / step, in 65536ths
  return (uint32_t)((e - LOW) << BITS) + ((k + r) >> 16);
}

// All loads of four runs of 4 elements are in flight at once, accesses do not stay in the caches.  230 M parameters, step / reading the moments out in bf16: 780 to 830 / 267 us, 5.0 to 5.3 and
// 5.2 TB/s (a copy reaches 4.8 to 5.6).  Of the step: with caching 40 us more; with root and quotient to the last bit 50 more; two
// runs of 4, or of 8 elements 35 more; 512 workgroups 110 more.
constexpr int VECS = 4;
constexpr int CHUNK = NT * 4 * VECS;

template <typename TG>
__global__ __launch_bounds__(NT) void adam8_kernel(Table8 t, const float* __restrict__ coef, AdamArgs8 a) {
  typedef float V4 __attribute__((vector_size(16), aligned(4)));
  typedef TG G4 __attribute__((vector_size(4 * sizeof(TG)), aligned(sizeof(TG))));
  typedef bf16_t B4 __attribute__((vector_size(8), aligned(2)));
  const float ck = coef[0];
  if (!(fabsf(ck) <= FLT_MAX)) return;
  const uint32_t chunks = t.first[t.count];
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int en = entry_of8(t, c);
    float* w = (float*)t.p[en][0];
    uint32_t* codes = (uint32_t*)t.p[en][1];
    uint8_t* scales = (uint8_t*)t.p[en][2];
    const TG* g = (const TG*)t.p[en][3];
    bf16_t* lp = (bf16_t*)t.p[en][4];
    const uint32_t n = t.n[en], at = (c - t.first[en]) * CHUNK, key = t.key[en], padded = (n + BLK - 1) / BLK * BLK;
    const bool whole = at + CHUNK <= n;
    V4 ww[VECS];
    float gg[VECS][4];
    uint32_t cm[VECS], cv[VECS];
    uint16_t sc[VECS];
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      const uint32_t q = at + (i * NT + threadIdx.x) * 4, b = q / BLK;
      if (whole) {
        ww[i] = __builtin_nontemporal_load(reinterpret_cast<const V4*>(w + q));
        const G4 x = __builtin_nontemporal_load(reinterpret_cast<const G4*>(g + q));
#pragma unroll
        for (int k = 0; k < 4; ++k) gg[i][k] = (float)x[k];
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          ww[i][k] = q + k < n ? w[q + k] : 0.f;
          gg[i][k] = q + k < n ? (float)g[q + k] : 0.f;
        }
      }
      const bool in = q < padded;
      cm[i] = in ? __builtin_nontemporal_load(codes + (size_t)b * 64 + (q % BLK) / 4) : 0u;
      cv[i] = in ? __builtin_nontemporal_load(codes + (size_t)b * 64 + 32 + (q % BLK) / 4) : 0u;
      sc[i] = in ? *reinterpret_cast<const uint16_t*>(scales + 2 * (size_t)b) : (uint16_t)0;
    }
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      const uint32_t q = at + (i * NT + threadIdx.x) * 4, b = q / BLK;
      const int em0 = (int)(sc[i] & 255u) - 127, ev0 = (int)(sc[i] >> 8) - 127;
      float m[4], v[4];
      uint32_t tm = 0, tv = 0;
      B4 o;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        m[k] = ldexpf(decode_m(cm[i], k), em0);
        v[k] = ldexpf(decode_v(cv[i], k), ev0);
      }
      if (any_rests(cm[i])) resting(cm[i], m, v);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float gk = gg[i][k] * ck;
        moments8(m[k], v[k], gk, a);
        const float wk = ww[i][k];
        // (root and reciprocal to an ulp each, 50 us less than to the last bit; they do not take numbers below 2^-126: a root counts as 2^-63 at least, of a NaN it is NaN)
        const float vc = v[k] * a.c2, root = __builtin_amdgcn_sqrtf(vc < FLT_MIN ? FLT_MIN : vc);
        ww[i][k] = fmaf(-a.lr, fmaf(a.wd, wk, m[k] * a.c1 * __builtin_amdgcn_rcpf(root + a.eps)), wk);
        o[k] = (bf16_t)(float)ww[i][k];
        const bool finite = (__float_as_uint(v[k]) & 0x7f800000u) != 0x7f800000u;
        tm = max(tm, finite ? finite_bits8(m[k]) : 0u);
        tv = max(tv, finite ? __float_as_uint(v[k]) : 0u);
      }
      const int em = exponent8<EXP_M, TOP_M>(max32(tm)), ev = exponent8<EXP_V, TOP_V>(max32(tv));
      const float um = __uint_as_float((uint32_t)(127 - em) << 23), uv = __uint_as_float((uint32_t)(127 - ev) << 23);
      uint32_t nm = 0, nv = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t h = mix32(q + k + key);
        const uint32_t bm = __float_as_uint(m[k]), bv = __float_as_uint(v[k]);
        uint32_t x = min(encode<-6, 3>(fminf(fabsf(m[k]) * um, 448.f), h & 0xffffu), 0x7eu) | ((bm >> 24) & 0x80u);
        x = (bv & 0x7f800000u) == 0x7f800000u ? 0xffu : x;
        x = (bm & 0x7f800000u) == 0x7f800000u ? 0x7fu : x;
        nm |= x << (8 * k);
        uint32_t y = min(encode<0, 4>(fminf(v[k] * uv, 31744.f), h >> 16), 255u);
        y = bv != 0 ? max(y, 1u) : 0u;
        y = (bv & 0x7f800000u) == 0x7f800000u ? 255u : y;
        nv |= y << (8 * k);
      }
      if (whole) {
        __builtin_nontemporal_store(ww[i], reinterpret_cast<V4*>(w + q));
        if (lp) __builtin_nontemporal_store(o, reinterpret_cast<B4*>(lp + q));
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (q + k < n) {
            w[q + k] = ww[i][k];
            if (lp) lp[q + k] = o[k];
          }
      }
      if (q < padded) {
        __builtin_nontemporal_store(nm, codes + (size_t)b * 64 + (q % BLK) / 4);
        __builtin_nontemporal_store(nv, codes + (size_t)b * 64 + 32 + (q % BLK) / 4);
        if ((q % BLK) == 0) *reinterpret_cast<uint16_t*>(scales + 2 * (size_t)b) = (uint16_t)((em + 127) | ((ev + 127) << 8));
      }
    }
  }
}

template <typename T>
__global__ __launch_bounds__(NT) void adam8_moments_kernel(Table8 t) {
  typedef T V4 __attribute__((vector_size(4 * sizeof(T)), aligned(sizeof(T))));
  const uint32_t chunks = t.first[t.count];
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int en = entry_of8(t, c);
    T *m = (T*)t.p[en][0], *v = (T*)t.p[en][3];
    const uint32_t* codes = (const uint32_t*)t.p[en][1];
    const uint8_t* scales = (const uint8_t*)t.p[en][2];
    const uint32_t n = t.n[en], at = (c - t.first[en]) * CHUNK;
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      const uint32_t q = at + (i * NT + threadIdx.x) * 4, b = q / BLK;
      if (q >= n) continue;
      const uint32_t cm = codes[(size_t)b * 64 + (q % BLK) / 4], cv = codes[(size_t)b * 64 + 32 + (q % BLK) / 4];
      const uint32_t sc = *reinterpret_cast<const uint16_t*>(scales + 2 * (size_t)b);
      float dm[4], dv[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        dm[k] = ldexpf(decode_m(cm, k), (int)(sc & 255u) - 127);
        dv[k] = ldexpf(decode_v(cv, k), (int)(sc >> 8) - 127);
      }
      if (any_rests(cm)) resting(cm, dm, dv);
      V4 om, ov;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        om[k] = (T)dm[k];
        ov[k] = (T)dv[k];
      }
      if (q + 4 <= n) {
        if (m) __builtin_nontemporal_store(om, reinterpret_cast<V4*>(m + q));
        if (v) __builtin_nontemporal_store(ov, reinterpret_cast<V4*>(v + q));
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (q + k < n) {
            if (m) m[q + k] = om[k];
            if (v) v[q + k] = ov[k];
          }
      }
    }
  }
}

inline size_t blocks_of(size_t n) { return (n + BLK - 1) / BLK; }

// Fills a table from tensor `at`, element `off` on; size(i), key(i), and set(i, o, p): the pointers of tensor i from element o (a multiple of 128) on
template <typename SZ, typename KY, typename ST>
bool fill8(Table8& t, int n_tensors, int& at, size_t& off, SZ size, KY key, ST set) {
  t.count = 0;
  t.first[0] = 0;
  while (at < n_tensors && t.count < CAP) {
    if (off >= size(at)) { ++at; off = 0; continue; }
    const size_t left = size(at) - off, take = left < MAX_ENTRY ? left : MAX_ENTRY;
    set(at, off, t.p[t.count]);
    t.n[t.count] = (uint32_t)take;
    t.key[t.count] = key(at) + (uint32_t)off;
    t.first[t.count + 1] = t.first[t.count] + (uint32_t)((take + CHUNK - 1) / CHUNK);  // at most 64 * 2^30 / 4096 = 2^24
    ++t.count;
    off += take;
  }
  return t.count > 0;
}

bf_status launched8(const char* who) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) { set_error("%s: launch failed: %s", who, hipGetErrorString(e)); return BF_EDEVICE; }
  return BF_OK;
}

constexpr unsigned MAX_WG = 2048;

}  // namespace

size_t adam8_state_bytes(size_t n) { return blocks_of(n) * (2 * BLK + 2); }

bf_status adam8_step(int dtype, int n_tensors, const bf_adam8_tensor* x, const float* coef, uint64_t seed, int step, double lr, double beta1, double beta2, double eps,
                     double wd, hipStream_t st) {
  if (n_tensors < 0 || (n_tensors > 0 && !x)) { set_error("bf_op_adam8: bad list of tensors"); return BF_EINVAL; }
  if (!coef || ((uintptr_t)coef & 3) || step < 1) { set_error("bf_op_adam8: coef is null or not aligned to its elements, or step below 1"); return BF_EINVAL; }
  const size_t es = dtype == BF_BF16 ? 2 : 4;
  for (int i = 0; i < n_tensors; ++i) {
    if (!x[i].n) continue;
    if (!x[i].w || !x[i].state || !x[i].g || ((uintptr_t)x[i].w & 3) || ((uintptr_t)x[i].state & 15) || ((uintptr_t)x[i].g & (es - 1)) || ((uintptr_t)x[i].w_lp & 1)) {
      set_error("bf_op_adam8: tensor %d has a null pointer, a state that is not 16-byte aligned or a tensor that is not aligned to its elements", i);
      return BF_EINVAL;
    }
  }
  AdamArgs8 a{(float)lr, (float)eps, (float)wd, (float)(1.0 / (1.0 - pow(beta1, (double)step))), (float)(1.0 / (1.0 - pow(beta2, (double)step))),
              (float)beta1, (float)beta2, (float)(1.0 - beta1), (float)(1.0 - beta2)};
  const uint32_t key = mix32(mix32(mix32((uint32_t)seed) ^ (uint32_t)(seed >> 32)) ^ (uint32_t)step);
  int at = 0;
  size_t off = 0;
  Table8 t;
  while (fill8(
      t, n_tensors, at, off, [&](int i) { return x[i].n; }, [&](int i) { return mix32(key ^ (uint32_t)i); },
      [&](int i, size_t o, const void** p) {
        p[0] = x[i].w + o;
        p[1] = (const char*)x[i].state + 2 * o;
        p[2] = (const char*)x[i].state + blocks_of(x[i].n) * 2 * BLK + o / BLK * 2;
        p[3] = (const char*)x[i].g + o * es;
        p[4] = x[i].w_lp ? (const bf16_t*)x[i].w_lp + o : nullptr;
      })) {
    const unsigned grid = t.first[t.count] < MAX_WG ? t.first[t.count] : MAX_WG;
    if (dtype == BF_BF16) adam8_kernel<bf16_t><<<grid, NT, 0, st>>>(t, coef, a);
    else adam8_kernel<float><<<grid, NT, 0, st>>>(t, coef, a);
    const bf_status s = launched8("bf_op_adam8");
    if (s != BF_OK) return s;
  }
  return BF_OK;
}

bf_status adam8_moments(int dtype, int n_tensors, const bf_adam8_moments_tensor* x, hipStream_t st) {
  if (n_tensors < 0 || (n_tensors > 0 && !x)) { set_error("bf_op_adam8_moments: bad list of tensors"); return BF_EINVAL; }
  const size_t es = dtype == BF_BF16 ? 2 : 4;
  for (int i = 0; i < n_tensors; ++i)
    if (x[i].n && (!x[i].state || ((uintptr_t)x[i].state & 15) || (((uintptr_t)x[i].m | (uintptr_t)x[i].v) & (es - 1)))) {
      set_error("bf_op_adam8_moments: tensor %d has a state that is null or not 16-byte aligned, or a tensor that is not aligned to its elements", i);
      return BF_EINVAL;
    }
  int at = 0;
  size_t off = 0;
  Table8 t;
  while (fill8(
      t, n_tensors, at, off, [&](int i) { return x[i].m || x[i].v ? x[i].n : 0; }, [](int) { return 0u; },
      [&](int i, size_t o, const void** p) {
        p[0] = x[i].m ? (const char*)x[i].m + o * es : nullptr;
        p[1] = (const char*)x[i].state + 2 * o;
        p[2] = (const char*)x[i].state + blocks_of(x[i].n) * 2 * BLK + o / BLK * 2;
        p[3] = x[i].v ? (const char*)x[i].v + o * es : nullptr;
        p[4] = nullptr;
      })) {
    const unsigned grid = t.first[t.count] < MAX_WG ? t.first[t.count] : MAX_WG;
    if (dtype == BF_BF16) adam8_moments_kernel<bf16_t><<<grid, NT, 0, st>>>(t);
    else adam8_moments_kernel<float><<<grid, NT, 0, st>>>(t);
    const bf_status s = launched8("bf_op_adam8_moments");
    if (s != BF_OK) return s;
  }
  return BF_OK;
}

}  // namespace bf
