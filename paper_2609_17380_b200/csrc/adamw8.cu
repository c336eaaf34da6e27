// AdamW over many tensors at once with moments in 8 bits (or in 32, tensor by tensor), and the moments as numbers.
//
// 256 adjacent values of a tensor share two scales, the largest |m| and the largest r = sqrt(v).  A code counts the root of a value's share of the
// scale, in 127 (m, with the sign of m) or 255 (r) parts: small values keep digits that equal steps would lose, and a code c of r is off by 2/c of v
// at most.  A root that is not zero has a code of 1 at least, so that no update divides by eps where the first moment has outlived the second.
// The update itself is det_adamw_batch's; the parameter moves by the moments before they are put into codes.
#include "common.cuh"
#include "internal.h"

namespace det {

constexpr int A8_VALUES = 256;            // values that share scales: a warp's, eight a lane
constexpr int ADAM8_JOBS = 128;           // tensors per launch
constexpr float A8_127 = 0x1.020408p-7f, A8_255 = 0x1.010102p-8f;     // 1/127, 1/255

struct Adam8Scalars { float b1, b2, omb1, omb2, eps, stepsz, isb2, decay; };
// Job j: warps first[j] .. first[j + 1] - 1 of the launch, each with 256 of its len[j] values.  s NULL: moments in 32 bits.
struct Adam8Jobs {
  int n;
  uint32_t first[ADAM8_JOBS + 1];
  const void *p[ADAM8_JOBS], *m[ADAM8_JOBS], *v[ADAM8_JOBS];
  const float* s[ADAM8_JOBS];
  float* g[ADAM8_JOBS];
  void *po[ADAM8_JOBS], *mo[ADAM8_JOBS], *vo[ADAM8_JOBS];
  float* so[ADAM8_JOBS];
  size_t len[ADAM8_JOBS];
  Adam8Scalars h[ADAM8_JOBS];
  uint8_t bf[ADAM8_JOBS];
};

__device__ __forceinline__ float a8_first(int c, float s) {
  const float t = fmul(__int2float_rn(c), A8_127);
  return fmul(s, fmul(t, fabsf(t)));
}
__device__ __forceinline__ float a8_root(int c, float s) {
  const float t = fmul(__int2float_rn(c), A8_255);
  return fmul(s, fmul(t, t));
}
// the scale of a block from its largest magnitude's bits: NaN where a value is not finite
__device__ __forceinline__ float a8_scale(uint32_t amax) { return amax >= 0x7f800000u ? __int_as_float(0x7fffffff) : __uint_as_float(amax); }
__device__ __forceinline__ float a8_inverse(float s) { return s > 0.0f ? fdiv(1.0f, s) : 0.0f; }
// a share of at most 1 (1 + 2^-23), so the code needs no clamp
__device__ __forceinline__ int a8_code(float x, float inv, float top) { return __float2int_rn(fmul(fsqrt(fmul(x, inv)), top)); }
__device__ __forceinline__ uint32_t a8_bytes(int a, int b, int c, int d) {
  return __byte_perm(__byte_perm((uint32_t)a, (uint32_t)b, 0x0040), __byte_perm((uint32_t)c, (uint32_t)d, 0x0040), 0x5410);
}

// Four adjacent values from i on, `n` of them there.
template <bool BF>
__device__ __forceinline__ void a8_load_p(const void* p, size_t i, int n, float v[4]) {
  if (n >= 4) {
    if (BF) {
      const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + i);
      v[0] = bflo(u.x); v[1] = bfhi(u.x); v[2] = bflo(u.y); v[3] = bfhi(u.y);
    } else {
      const float4 t = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
      v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = k < n ? (BF ? bf2f(static_cast<const uint16_t*>(p)[i + k]) : static_cast<const float*>(p)[i + k]) : 0.0f;
}
template <bool BF>
__device__ __forceinline__ void a8_store_p(void* p, size_t i, int n, const float v[4]) {
  if (n >= 4) {
    if (BF) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) = make_uint2(pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3]));
    else *reinterpret_cast<float4*>(static_cast<float*>(p) + i) = make_float4(v[0], v[1], v[2], v[3]);
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k < n) {
      if (BF) static_cast<uint16_t*>(p)[i + k] = f2bf(v[k]);
      else static_cast<float*>(p)[i + k] = v[k];
    }
}
__device__ __forceinline__ uint32_t a8_load_codes(const void* p, size_t i, int n) {
  if (n >= 4) return *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(p) + i);
  uint32_t u = 0;
  for (int k = 0; k < n; ++k) u |= (uint32_t)static_cast<const uint8_t*>(p)[i + k] << (8 * k);
  return u;
}
__device__ __forceinline__ void a8_store_codes(void* p, size_t i, int n, uint32_t u) {
  if (n >= 4) { *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(p) + i) = u; return; }
  for (int k = 0; k < n; ++k) static_cast<uint8_t*>(p)[i + k] = (uint8_t)(u >> (8 * k));
}
// moments of a warp's 256 values into codes
__device__ __forceinline__ void a8_put(const float (&m)[8], const float (&r)[8], int lane, size_t i0, const int (&n)[2], int8_t* m8, uint8_t* v8, float2* s) {
  uint32_t am = 0, ar = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    am = max(am, __float_as_uint(m[k]) & 0x7fffffffu);
    ar = max(ar, __float_as_uint(r[k]) & 0x7fffffffu);
  }
  am = __reduce_max_sync(0xffffffffu, am);
  ar = __reduce_max_sync(0xffffffffu, ar);
  const float sm = a8_scale(am), sr = a8_scale(ar), im = a8_inverse(sm), ir = a8_inverse(sr);
  const bool fm = am < 0x7f800000u, fr = ar < 0x7f800000u;
  if (lane == 0) *s = make_float2(sm, sr);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int a[4], b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float mv = m[4 * h + k], rv = r[4 * h + k];
      const int c = a8_code(fabsf(mv), im, 127.0f), d = a8_code(rv, ir, 255.0f);
      a[k] = fm ? (mv < 0.0f ? -c : c) : 0;
      b[k] = fr ? (rv > 0.0f ? max(d, 1) : d) : 0;
    }
    a8_store_codes(m8, i0 + 128 * h, n[h], a8_bytes(a[0], a[1], a[2], a[3]));
    a8_store_codes(v8, i0 + 128 * h, n[h], a8_bytes(b[0], b[1], b[2], b[3]));
  }
}

template <bool BF, bool EIGHT>
__device__ __forceinline__ void adam8_block(const Adam8Jobs& jobs, int j, float coef, bool clip, size_t base, int lane) {
  const Adam8Scalars h = jobs.h[j];
  const size_t len = jobs.len[j], i0 = base + lane * 4;
  int n[2];
  float p[8], g[8], m[8], r[8];
  uint32_t cm[2] = {0, 0}, cv[2] = {0, 0};
  float2 s = make_float2(0.0f, 0.0f);
  if (EIGHT) s = reinterpret_cast<const float2*>(jobs.s[j])[base / A8_VALUES];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const size_t i = i0 + 128 * q;
    n[q] = i + 4 <= len ? 4 : i < len ? (int)(len - i) : 0;
    a8_load_p<BF>(jobs.p[j], i, n[q], p + 4 * q);
    a8_load_p<false>(jobs.g[j], i, n[q], g + 4 * q);
    if (EIGHT) {
      cm[q] = a8_load_codes(jobs.m[j], i, n[q]);
      cv[q] = a8_load_codes(jobs.v[j], i, n[q]);
    } else {
      a8_load_p<false>(jobs.m[j], i, n[q], m + 4 * q);
      a8_load_p<false>(jobs.v[j], i, n[q], r + 4 * q);
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (EIGHT) {
      m[k] = a8_first((int)(int8_t)(cm[k >> 2] >> (8 * (k & 3))), s.x);
      const float w = a8_root((int)(uint8_t)(cv[k >> 2] >> (8 * (k & 3))), s.y);
      r[k] = fmul(w, w);
    }
    if (clip) g[k] = fmul(g[k], coef);
    m[k] = fadd(fmul(h.b1, m[k]), fmul(h.omb1, g[k]));
    const float v = fadd(fmul(h.b2, r[k]), fmul(h.omb2, fmul(g[k], g[k]))), root = fsqrt(v);
    p[k] = fsub(fmul(p[k], h.decay), fmul(h.stepsz, fdiv(m[k], fadd(fmul(root, h.isb2), h.eps))));
    r[k] = EIGHT ? root : v;
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const size_t i = i0 + 128 * q;
    a8_store_p<BF>(jobs.po[j], i, n[q], p + 4 * q);
    if (clip) a8_store_p<false>(jobs.g[j], i, n[q], g + 4 * q);
    if (!EIGHT) {
      a8_store_p<false>(jobs.mo[j], i, n[q], m + 4 * q);
      a8_store_p<false>(jobs.vo[j], i, n[q], r + 4 * q);
    }
  }
  if (EIGHT) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if ((k & 3) >= n[k >> 2]) m[k] = r[k] = 0.0f;                       // behind the last value
    a8_put(m, r, lane, i0, n, static_cast<int8_t*>(jobs.mo[j]), static_cast<uint8_t*>(jobs.vo[j]), reinterpret_cast<float2*>(jobs.so[j]) + base / A8_VALUES);
  }
}
__device__ __forceinline__ int a8_job(const uint32_t* first, int n, uint32_t w) {      // the last job whose first warp is <= w
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= w) lo = mid; else hi = mid - 1;
  }
  return lo;
}
__global__ void __launch_bounds__(256) k_adamw8(const __grid_constant__ Adam8Jobs jobs, const float* __restrict__ coef) {
  grid_dep();
  const uint32_t w = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (w >= jobs.first[jobs.n]) return;
  const int j = a8_job(jobs.first, jobs.n, w), lane = threadIdx.x & 31;
  const size_t base = (size_t)(w - jobs.first[j]) * A8_VALUES;
  const bool clip = coef != nullptr;
  const float c = clip ? coef[0] : 1.0f;
  if (jobs.s[j]) {
    if (jobs.bf[j]) adam8_block<true, true>(jobs, j, c, clip, base, lane);
    else adam8_block<false, true>(jobs, j, c, clip, base, lane);
  } else {
    if (jobs.bf[j]) adam8_block<true, false>(jobs, j, c, clip, base, lane);
    else adam8_block<false, false>(jobs, j, c, clip, base, lane);
  }
}

// Codes to numbers and back, many tensors at once.
struct Adam8Numbers {
  int n;
  uint32_t first[ADAM8_JOBS + 1];
  int8_t* m8[ADAM8_JOBS];
  uint8_t* v8[ADAM8_JOBS];
  float *s[ADAM8_JOBS], *m[ADAM8_JOBS], *v[ADAM8_JOBS];
  size_t len[ADAM8_JOBS];
};
template <bool PACK>
__global__ void __launch_bounds__(256) k_adamw8_numbers(const __grid_constant__ Adam8Numbers jobs) {
  grid_dep();
  const uint32_t w = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (w >= jobs.first[jobs.n]) return;
  const int j = a8_job(jobs.first, jobs.n, w), lane = threadIdx.x & 31;
  const size_t base = (size_t)(w - jobs.first[j]) * A8_VALUES, len = jobs.len[j], i0 = base + lane * 4;
  float2* s = reinterpret_cast<float2*>(jobs.s[j]) + base / A8_VALUES;
  int n[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) n[q] = i0 + 128 * q + 4 <= len ? 4 : i0 + 128 * q < len ? (int)(len - i0 - 128 * q) : 0;
  float m[8], r[8];
  if (PACK) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      a8_load_p<false>(jobs.m[j], i0 + 128 * q, n[q], m + 4 * q);
      a8_load_p<false>(jobs.v[j], i0 + 128 * q, n[q], r + 4 * q);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      m[k] = fmul(m[k], 1.0f);                                            // a subnormal number counts as zero
      r[k] = fsqrt(r[k]);
    }
    a8_put(m, r, lane, i0, n, jobs.m8[j], jobs.v8[j], s);
  } else {
    const float2 sc = *s;
    uint32_t cm[2], cv[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      cm[q] = a8_load_codes(jobs.m8[j], i0 + 128 * q, n[q]);
      cv[q] = a8_load_codes(jobs.v8[j], i0 + 128 * q, n[q]);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      m[k] = a8_first((int)(int8_t)(cm[k >> 2] >> (8 * (k & 3))), sc.x);
      const float w2 = a8_root((int)(uint8_t)(cv[k >> 2] >> (8 * (k & 3))), sc.y);
      r[k] = fmul(w2, w2);
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      a8_store_p<false>(jobs.m[j], i0 + 128 * q, n[q], m + 4 * q);
      a8_store_p<false>(jobs.v[j], i0 + 128 * q, n[q], r + 4 * q);
    }
  }
}

static double a8_ipow(double b, int e) {
  double r = 1.0;
  while (e > 0) { if (e & 1) r *= b; b *= b; e >>= 1; }
  return r;
}
static Adam8Scalars a8_scalars(const det_adamw_desc* d) {
  const double bc1 = 1.0 - a8_ipow(d->beta1, d->step), bc2 = 1.0 - a8_ipow(d->beta2, d->step);
  Adam8Scalars h;
  h.b1 = (float)d->beta1; h.b2 = (float)d->beta2;
  h.omb1 = 1.0f - h.b1; h.omb2 = 1.0f - h.b2;
  h.eps = (float)d->eps;
  h.stepsz = (float)(d->lr / bc1);
  h.isb2 = (float)(1.0 / sqrt(bc2));
  h.decay = (float)(1.0 - d->lr * d->weight_decay);
  return h;
}
static bool a8_at(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
static bool a8_moments_at(const void* m, const void* v, const void* s) {
  return s ? a8_at(m, 4) && a8_at(v, 4) && a8_at(s, 8) : a8_at(m, 16) && a8_at(v, 16);
}
// the tensors t, t + 1, ... as jobs of one launch: fill(job, tensor) for each that has values
template <class Jobs, class Fill>
static int a8_take(Jobs& jobs, int& t, int ntensors, const size_t* n, Fill fill) {
  size_t w = 0;
  jobs.n = 0;
  for (; t < ntensors && jobs.n < ADAM8_JOBS; ++t) {
    if (!n[t]) continue;
    const size_t warps = (n[t] + A8_VALUES - 1) / A8_VALUES;
    if (w + warps > 0x7fffffffull) break;                                  // its own is checked before
    jobs.first[jobs.n] = (uint32_t)w;
    jobs.len[jobs.n] = n[t];
    fill(jobs.n++, t);
    w += warps;
  }
  jobs.first[jobs.n] = (uint32_t)w;
  return (int)((w + 7) / 8);
}
}  // namespace det

using namespace det;

extern "C" size_t det_adamw8_scale_floats(size_t n) { return (n + A8_VALUES - 1) / A8_VALUES * 2; }

extern "C" int det_adamw8_batch(const det_adamw_desc* descs, const int* pdtypes, const void* const* p, float* const* g, const void* const* m,
                                const void* const* v, const float* const* s, void* const* p_out, void* const* m_out, void* const* v_out,
                                float* const* s_out, const size_t* n, int ntensors, const float* coef_dev, void* stream) {
  if (ntensors < 0 || (ntensors && (!descs || !pdtypes || !p || !g || !m || !v || !s || !p_out || !m_out || !v_out || !s_out || !n))) return DET_ERR_ARG;
  for (int t = 0; t < ntensors; ++t) {
    if (!n[t]) continue;
    if (!p[t] || !g[t] || !m[t] || !v[t] || !p_out[t] || !m_out[t] || !v_out[t] || !s[t] != !s_out[t] || descs[t].step < 1 ||
        (pdtypes[t] != DET_F32 && pdtypes[t] != DET_BF16))
      return DET_ERR_ARG;
    if (n[t] > (size_t)0x7fffffff * A8_VALUES) return DET_ERR_SHAPE;
    const size_t ap = pdtypes[t] == DET_BF16 ? 8 : 16;
    if (!a8_at(p[t], ap) || !a8_at(p_out[t], ap) || !aligned16(g[t]) || !a8_moments_at(m[t], v[t], s[t]) || !a8_moments_at(m_out[t], v_out[t], s_out[t]))
      return DET_ERR_ALIGN;
  }
  for (int t = 0; t < ntensors;) {
    Adam8Jobs jobs;
    const int ctas = a8_take(jobs, t, ntensors, n, [&](int j, int i) {
      jobs.p[j] = p[i]; jobs.g[j] = g[i]; jobs.m[j] = m[i]; jobs.v[j] = v[i]; jobs.s[j] = s[i];
      jobs.po[j] = p_out[i]; jobs.mo[j] = m_out[i]; jobs.vo[j] = v_out[i]; jobs.so[j] = s_out[i];
      jobs.h[j] = a8_scalars(&descs[i]);
      jobs.bf[j] = pdtypes[i] == DET_BF16;
    });
    if (!jobs.n) break;
    launch_after(k_adamw8, ctas, 256, 0, (cudaStream_t)stream, jobs, coef_dev);
    DET_CHECK_LAUNCH();
  }
  return DET_OK;
}

template <bool PACK>
static int a8_numbers(int8_t* const* m8, uint8_t* const* v8, float* const* s, float* const* m, float* const* v, const size_t* n, int ntensors, void* stream) {
  if (ntensors < 0 || (ntensors && (!m8 || !v8 || !s || !m || !v || !n))) return DET_ERR_ARG;
  for (int t = 0; t < ntensors; ++t) {
    if (!n[t]) continue;
    if (!m8[t] || !v8[t] || !s[t] || !m[t] || !v[t]) return DET_ERR_ARG;
    if (n[t] > (size_t)0x7fffffff * A8_VALUES) return DET_ERR_SHAPE;
    if (!a8_moments_at(m8[t], v8[t], s[t]) || !aligned16(m[t]) || !aligned16(v[t])) return DET_ERR_ALIGN;
  }
  for (int t = 0; t < ntensors;) {
    Adam8Numbers jobs;
    const int ctas = a8_take(jobs, t, ntensors, n, [&](int j, int i) { jobs.m8[j] = m8[i]; jobs.v8[j] = v8[i]; jobs.s[j] = s[i]; jobs.m[j] = m[i]; jobs.v[j] = v[i]; });
    if (!jobs.n) break;
    launch_after(k_adamw8_numbers<PACK>, ctas, 256, 0, (cudaStream_t)stream, jobs);
    DET_CHECK_LAUNCH();
  }
  return DET_OK;
}
extern "C" int det_adamw8_pack(const float* const* m, const float* const* v, int8_t* const* m8, uint8_t* const* v8, float* const* s, const size_t* n,
                               int ntensors, void* stream) {
  return a8_numbers<true>(m8, v8, s, const_cast<float* const*>(m), const_cast<float* const*>(v), n, ntensors, stream);
}
extern "C" int det_adamw8_unpack(const int8_t* const* m8, const uint8_t* const* v8, const float* const* s, float* const* m, float* const* v, const size_t* n,
                                 int ntensors, void* stream) {
  return a8_numbers<false>(const_cast<int8_t* const*>(m8), const_cast<uint8_t* const*>(v8), const_cast<float* const*>(s), m, v, n, ntensors, stream);
}
