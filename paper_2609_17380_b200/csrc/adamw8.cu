// AdamW over many tensors at once with moments in 8 bits (or in 32, tensor by tensor), and the moments as numbers.
//
// 256 adjacent values of a tensor share two scales, the largest |m| and the largest r = sqrt(v).  A code counts the root of a value's share of the
// scale, in 127 (m, with the sign of m) or 255 (r) parts: small values keep digits that equal steps would lose, and a code c of r is off by 2/c of v
// at most.  A root that is not zero has a code of 1 at least, so that no update divides by eps where the first moment has outlived the second.
// The update itself is det_adamw_batch's; the parameter moves by the moments before they are put into codes.
//
// 67 M values with bf16 parameters and the clip stored (16 bytes each) 198 us, 5.4 TB/s, bound by its 78 instructions a value (81 % of the issue slots); the
// moments as numbers 115 us, 5.8 TB/s.
#include "common.cuh"
#include "internal.h"
#include "rows.cuh"

namespace det {

constexpr int A8_VALUES = 256;            // values that share scales: a warp's, eight a lane
constexpr int ADAM8_JOBS = 128, ADAM8_FEW = 16;     // tensors per launch; a launch of few has a shorter table to hand over
constexpr float A8_127 = 0x1.020408p-7f, A8_255 = 0x1.010102p-8f;     // 1/127, 1/255

// Job j: CTAs first[j] .. first[j + 1] - 1 of the launch, each with `rounds` times 2048 of its len[j] values, 256 a warp and round.  A job belongs to whole
// CTAs, and its entries, constants at an index, are read once for all rounds.  s NULL: moments in 32 bits.
template <int CAP>
struct Adam8Jobs {
  int n, rounds;
  uint32_t first[CAP + 1];
  const void *p[CAP], *m[CAP], *v[CAP];
  const float* s[CAP];
  float* g[CAP];
  void *po[CAP], *mo[CAP], *vo[CAP];
  float* so[CAP];
  size_t len[CAP];
  AdamScalars h[CAP];
  uint8_t bf[CAP];
};

__device__ __forceinline__ float a8_first(int c, float s) {
  const float t = fmul(__int2float_rn(c), A8_127);
  return fmul(s, fmul(t, fabsf(t)));
}
__device__ __forceinline__ float a8_root(int c, float s) {
  const float t = fmul(__int2float_rn(c), A8_255);
  return fmul(s, fmul(t, t));
}
// fsqrt and fdiv; a zero, which sends a whole warp through the compiler's path for special operands, is answered beside them.  A value in fifty that is
// zero (weights that have had no gradient) is in every second warp.
__device__ __forceinline__ float a8_sqrt(float x) {
  const bool zero = x == 0.0f;
  const float r = fsqrt(zero ? 1.0f : x);                                 // of a negative v, which 32 bits may hold, a NaN
  return zero ? x : r;
}
__device__ __forceinline__ float a8_div(float a, float b) {
  const bool plain = a == 0.0f && b > 0.0f;                               // 0 / b is that zero
  const float q = fdiv(plain ? 1.0f : a, plain ? 1.0f : b);
  return plain ? a : q;
}
// the scale of a block from its largest magnitude's bits: NaN where a value is not finite
__device__ __forceinline__ float a8_scale(uint32_t amax) { return amax >= 0x7f800000u ? __int_as_float(0x7fffffff) : __uint_as_float(amax); }
__device__ __forceinline__ float a8_inverse(float s) { return s > 0.0f ? fdiv(1.0f, s) : 0.0f; }
// a share of at most 1 (1 + 2^-23), so the code needs no clamp
__device__ __forceinline__ int a8_code(float x, float inv, float top) { return __float2int_rn(fmul(a8_sqrt(fmul(x, inv)), top)); }

// Four adjacent values from i on, `n` of them there; FULL: all four, in the block of a tensor that has all its 256.
template <bool FULL, bool BF>
__device__ __forceinline__ void a8_load_p(const void* p, size_t i, int n, float v[4]) {
  if (FULL || n >= 4) {
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
template <bool FULL>
__device__ __forceinline__ void a8_store_f(void* p, size_t i, int n, const float v[4]) {
  if (FULL || n >= 4) { *reinterpret_cast<float4*>(static_cast<float*>(p) + i) = make_float4(v[0], v[1], v[2], v[3]); return; }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k < n) static_cast<float*>(p)[i + k] = v[k];
}
template <bool FULL>
__device__ __forceinline__ void a8_store_bf(void* p, size_t i, int n, uint32_t a, uint32_t b) {
  if (FULL || n >= 4) { *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) = make_uint2(a, b); return; }
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < n) static_cast<uint16_t*>(p)[i + k] = (uint16_t)((k < 2 ? a : b) >> (16 * (k & 1)));
}
template <bool FULL>
__device__ __forceinline__ uint32_t a8_load_codes(const void* p, size_t i, int n) {
  if (FULL || n >= 4) return *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(p) + i);
  uint32_t u = 0;
  for (int k = 0; k < n; ++k) u |= (uint32_t)static_cast<const uint8_t*>(p)[i + k] << (8 * k);
  return u;
}
template <bool FULL>
__device__ __forceinline__ void a8_store_codes(void* p, size_t i, int n, uint32_t u) {
  if (FULL || n >= 4) { *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(p) + i) = u; return; }
  for (int k = 0; k < n; ++k) static_cast<uint8_t*>(p)[i + k] = (uint8_t)(u >> (8 * k));
}
// Square roots and a quotient of two or three roundings for every value hold the issue slots longer than the memory takes, and a code needs none of
// them: it is the same for every t nearer to the exact one than t is to a border between codes.  So t is made from the hardware's approximation
// (sqrt.approx and rcp.approx: 2^-23 of the value at most), which can be off by `off` in all, and where a border is nearer than that, some value in
// four thousand, the exact steps are taken.
__device__ __forceinline__ float a8_sqrt_near(float x) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float a8_rcp_near(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// the code of t in the low byte; far: how far t is from it, at most
__device__ __forceinline__ uint32_t a8_rounded(float t, float& far) {
  const float k = fadd(t, 12582912.0f);
  far = fmaxf(far, fabsf(fsub(t, fsub(k, 12582912.0f))));
  return __float_as_uint(k);
}
// Off by: sqrt.approx for fsqrt 1.5 * 2^-23, the product with 127 another 2^-23: 127 * 2.5 * 2^-23 < 2^-14.  Of r: r itself 1.5 and its share 1 more, halved by
// the root, whose own 1.5, the product's 1: 255 * 3.75 * 2^-23 < 1.5 * 2^-13.
constexpr float A8_OFF_M = 0x1p-14f, A8_OFF_R = 0x1.8p-13f;
// The moments of a warp's 256 values into codes: m, v = r r in binary32 (r near by: a8_sqrt_near(v)).
template <bool FULL>
__device__ __forceinline__ void a8_put(const float (&m)[8], const float (&v)[8], const float (&near)[8], int lane, size_t i0, const int (&n)[2], int8_t* m8,
                                       uint8_t* v8, float2* s) {
  uint32_t am = 0, av = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    am = max(am, __float_as_uint(m[k]) & 0x7fffffffu);
    av = max(av, __float_as_uint(v[k]));                                  // a negative v counts as not finite, as its root is
  }
  am = __reduce_max_sync(0xffffffffu, am);
  av = __reduce_max_sync(0xffffffffu, av);
  // the largest root is the root of the largest
  const float sm = a8_scale(am), sr = av >= 0x7f800000u ? __int_as_float(0x7fffffff) : a8_sqrt(__uint_as_float(av));
  const float inv = a8_inverse(lane & 1 ? sr : sm), im = __shfl_sync(0xffffffffu, inv, 0), ir = __shfl_sync(0xffffffffu, inv, 1);   // one division for both
  const uint32_t fm = am < 0x7f800000u ? ~0u : 0u, fr = av < 0x7f800000u ? ~0u : 0u;
  if (lane == 0) *s = make_float2(sm, sr);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t a[4], b[4];
    float far_m = 0.0f, far_r = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float mv = m[4 * h + k], w = near[4 * h + k];
      const float tm = fmul(a8_sqrt_near(fmul(fabsf(mv), im)), 127.0f), tr = fmul(a8_sqrt_near(fmul(w, ir)), 255.0f);
      a[k] = a8_rounded(copysignf(tm, mv), far_m);
      b[k] = a8_rounded(fmaxf(tr, __saturatef(fmul(w, 0x1p100f))), far_r);      // at least 1 where r > 0, which is 2^-63 or more
    }
    if (far_m > 0.5f - A8_OFF_M || far_r > 0.5f - A8_OFF_R) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float mv = m[4 * h + k], vv = v[4 * h + k];
        const int c = a8_code(fabsf(mv), im, 127.0f);
        a[k] = (uint32_t)(mv < 0.0f ? -c : c);
        b[k] = (uint32_t)max(a8_code(a8_sqrt(vv), ir, 255.0f), vv > 0.0f ? 1 : 0);
      }
    }
    a8_store_codes<FULL>(m8, i0 + 128 * h, n[h], low_bytes(a[0], a[1], a[2], a[3]) & fm);
    a8_store_codes<FULL>(v8, i0 + 128 * h, n[h], low_bytes(b[0], b[1], b[2], b[3]) & fr);
  }
}

// p moved by the moments, exactly as det_adamw_step
__device__ __forceinline__ float a8_moved(const AdamScalars& h, float p, float m, float root) {
  return fsub(fmul(p, h.decay), fmul(h.stepsz, a8_div(m, fadd(fmul(root, h.isb2), h.eps))));
}
// A job's entries
struct Adam8Job {
  const void *p, *m, *v;
  const float* s;
  float* g;
  void *po, *mo, *vo;
  float* so;
  size_t len;
  AdamScalars h;
};
// a warp's 256 values from `base` on
template <bool FULL, bool BF, bool EIGHT>
__device__ __forceinline__ void adam8_block(const Adam8Job& job, float coef, bool clip, size_t base, int lane) {
  const AdamScalars& h = job.h;
  const size_t i0 = base + lane * 4;
  int n[2];
  float p[8], g[8], m[8], v[8], near[8];
  uint32_t cm[2], cv[2];
  float2 s;
  if (EIGHT) s = reinterpret_cast<const float2*>(job.s)[base / A8_VALUES];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const size_t i = i0 + 128 * q;
    n[q] = FULL || i + 4 <= job.len ? 4 : i < job.len ? (int)(job.len - i) : 0;
    a8_load_p<FULL, BF>(job.p, i, n[q], p + 4 * q);
    a8_load_p<FULL, false>(job.g, i, n[q], g + 4 * q);
    if (EIGHT) {
      cm[q] = a8_load_codes<FULL>(job.m, i, n[q]);
      cv[q] = a8_load_codes<FULL>(job.v, i, n[q]);
    } else {
      a8_load_p<FULL, false>(job.m, i, n[q], m + 4 * q);
      a8_load_p<FULL, false>(job.v, i, n[q], v + 4 * q);
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (EIGHT) {
      m[k] = a8_first((int)(int8_t)(cm[k >> 2] >> (8 * (k & 3))), s.x);
      const float w = a8_root((int)(uint8_t)(cv[k >> 2] >> (8 * (k & 3))), s.y);
      v[k] = fmul(w, w);
    }
    if (clip) g[k] = fmul(g[k], coef);
    m[k] = fadd(fmul(h.b1, m[k]), fmul(h.omb1, g[k]));
    v[k] = fadd(fmul(h.b2, v[k]), fmul(h.omb2, fmul(g[k], g[k])));
    if (EIGHT) near[k] = a8_sqrt_near(v[k]);
  }
  if (clip) {
    a8_store_f<FULL>(job.g, i0, n[0], g);
    a8_store_f<FULL>(job.g, i0 + 128, n[1], g + 4);
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    if (!EIGHT) {
      a8_store_f<FULL>(job.mo, i0 + 128 * q, n[q], m + 4 * q);
      a8_store_f<FULL>(job.vo, i0 + 128 * q, n[q], v + 4 * q);
    }
    float to[4];
    bool exact = !(BF && EIGHT);
    if (BF && EIGHT) {
      // The bf16 that the moved parameter is rounded to is nearly always that of every number near it.  With the approximations for root and quotient the
      // step is off by 6.5 * 2^-23 of itself, the difference's own rounding comes on top, and what is flushed on the way.  Where the ends of that interval
      // are rounded to two numbers, some value in eight thousand, or where eps is no small positive number, the exact steps are taken.
      exact = !(h.eps >= 0.0f && h.eps < 0x1p90f);
      uint32_t ends[2][2];
#pragma unroll
      for (int k = 0; k < 4; k += 2) {
        float lo[2], hi[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int i = 4 * q + k + e;
          const float step = fmul(h.stepsz, fmul(m[i], a8_rcp_near(fadd(fmul(near[i], h.isb2), h.eps))));
          const float x = fsub(fmul(p[i], h.decay), step), off = __fmaf_rn(fabsf(x), 0x1p-22f, __fmaf_rn(fabsf(step), 0x1p-20f, 0x1p-100f));
          to[k + e] = x;
          lo[e] = fsub(x, off);
          hi[e] = fadd(x, off);
        }
        ends[k / 2][0] = bf_pair(lo[0], lo[1]);
        ends[k / 2][1] = bf_pair(hi[0], hi[1]);
      }
      exact = exact || ends[0][0] != ends[0][1] || ends[1][0] != ends[1][1];
    }
    if (exact) {
#pragma unroll
      for (int k = 0; k < 4; ++k) to[k] = a8_moved(h, p[4 * q + k], m[4 * q + k], a8_sqrt(v[4 * q + k]));
    }
    if (BF) a8_store_bf<FULL>(job.po, i0 + 128 * q, n[q], bf_pair(to[0], to[1]), bf_pair(to[2], to[3]));
    else a8_store_f<FULL>(job.po, i0 + 128 * q, n[q], to);
  }
  if (EIGHT) {
    if (!FULL) {                                                          // the end of the tensor: nothing behind it counts
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if ((k & 3) >= n[k >> 2]) m[k] = v[k] = near[k] = 0.0f;
    }
    a8_put<FULL>(m, v, near, lane, i0, n, static_cast<int8_t*>(job.mo), static_cast<uint8_t*>(job.vo), reinterpret_cast<float2*>(job.so) + base / A8_VALUES);
  }
}
template <bool BF, bool EIGHT>
__device__ __forceinline__ void adam8_rounds(const Adam8Job& job, float coef, bool clip, size_t base, int rounds, int lane) {
#pragma unroll 1
  for (int r = 0; r < rounds && base < job.len; ++r, base += 8 * A8_VALUES) {
    if (base + A8_VALUES <= job.len) adam8_block<true, BF, EIGHT>(job, coef, clip, base, lane);
    else adam8_block<false, BF, EIGHT>(job, coef, clip, base, lane);
  }
}
__device__ __forceinline__ int a8_job(const uint32_t* first, int n) {      // the last job whose first CTA is <= this one
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= blockIdx.x) lo = mid; else hi = mid - 1;
  }
  return lo;
}
template <int CAP>
__global__ void __launch_bounds__(256) k_adamw8(const __grid_constant__ Adam8Jobs<CAP> jobs, const float* __restrict__ coef) {
  grid_dep();
  const int j = a8_job(jobs.first, jobs.n), lane = threadIdx.x & 31;
  const size_t base = ((size_t)(blockIdx.x - jobs.first[j]) * (8 * jobs.rounds) + (threadIdx.x >> 5)) * A8_VALUES;
  const Adam8Job job = {jobs.p[j], jobs.m[j], jobs.v[j], jobs.s[j], jobs.g[j], jobs.po[j], jobs.mo[j], jobs.vo[j], jobs.so[j], jobs.len[j], jobs.h[j]};
  if (base >= job.len) return;
  const bool clip = coef != nullptr;
  const float c = clip ? coef[0] : 1.0f;
  if (job.s) {
    if (jobs.bf[j]) adam8_rounds<true, true>(job, c, clip, base, jobs.rounds, lane);
    else adam8_rounds<false, true>(job, c, clip, base, jobs.rounds, lane);
  } else {
    if (jobs.bf[j]) adam8_rounds<true, false>(job, c, clip, base, jobs.rounds, lane);
    else adam8_rounds<false, false>(job, c, clip, base, jobs.rounds, lane);
  }
}

// A moment as the definition takes it: subnormals and either zero are +0.  On the bits, as the scale of a block is taken from the bits too (a product with 1
// or a sum with 0 is what a compiler may leave out).
__device__ __forceinline__ float a8_flushed(float x) { return (__float_as_uint(x) & 0x7fffffffu) < 0x00800000u ? 0.0f : x; }

// Codes to numbers and back, many tensors at once.
template <int CAP>
struct Adam8Numbers {
  int n, rounds;
  uint32_t first[CAP + 1];
  int8_t* m8[CAP];
  uint8_t* v8[CAP];
  float *s[CAP], *m[CAP], *v[CAP];
  size_t len[CAP];
};
template <bool PACK, bool FULL, int CAP>
__device__ __forceinline__ void adam8_numbers(const Adam8Numbers<CAP>& jobs, int j, size_t base, size_t len, int lane) {
  const size_t i0 = base + lane * 4;
  float2* s = reinterpret_cast<float2*>(jobs.s[j]) + base / A8_VALUES;
  int n[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) n[q] = FULL || i0 + 128 * q + 4 <= len ? 4 : i0 + 128 * q < len ? (int)(len - i0 - 128 * q) : 0;
  float m[8], v[8];
  if (PACK) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      a8_load_p<FULL, false>(jobs.m[j], i0 + 128 * q, n[q], m + 4 * q);
      a8_load_p<FULL, false>(jobs.v[j], i0 + 128 * q, n[q], v + 4 * q);
    }
    float near[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      m[k] = a8_flushed(m[k]);
      v[k] = a8_flushed(v[k]);
      near[k] = a8_sqrt_near(v[k]);
    }
    a8_put<FULL>(m, v, near, lane, i0, n, jobs.m8[j], jobs.v8[j], s);
  } else {
    const float2 sc = *s;
    uint32_t cm[2], cv[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      cm[q] = a8_load_codes<FULL>(jobs.m8[j], i0 + 128 * q, n[q]);
      cv[q] = a8_load_codes<FULL>(jobs.v8[j], i0 + 128 * q, n[q]);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      m[k] = a8_first((int)(int8_t)(cm[k >> 2] >> (8 * (k & 3))), sc.x);
      const float r = a8_root((int)(uint8_t)(cv[k >> 2] >> (8 * (k & 3))), sc.y);
      v[k] = fmul(r, r);
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      a8_store_f<FULL>(jobs.m[j], i0 + 128 * q, n[q], m + 4 * q);
      a8_store_f<FULL>(jobs.v[j], i0 + 128 * q, n[q], v + 4 * q);
    }
  }
}
template <bool PACK, int CAP>
__global__ void __launch_bounds__(256) k_adamw8_numbers(const __grid_constant__ Adam8Numbers<CAP> jobs) {
  grid_dep();
  const int j = a8_job(jobs.first, jobs.n), lane = threadIdx.x & 31;
  const size_t len = jobs.len[j];
  size_t base = ((size_t)(blockIdx.x - jobs.first[j]) * (8 * jobs.rounds) + (threadIdx.x >> 5)) * A8_VALUES;
#pragma unroll 1
  for (int round = 0; round < jobs.rounds && base < len; ++round, base += 8 * A8_VALUES) {
    if (base + A8_VALUES <= len) adam8_numbers<PACK, true>(jobs, j, base, len, lane);
    else adam8_numbers<PACK, false>(jobs, j, base, len, lane);
  }
}

static bool a8_moments_at(const void* m, const void* v, const void* s) {
  return s ? aligned_to(m, 4) && aligned_to(v, 4) && aligned_to(s, 8) : aligned_to(m, 16) && aligned_to(v, 16);
}
// the tensors t, t + 1, ... as jobs of one launch: fill(job, tensor) for each that has values
template <int CAP, class Jobs, class Fill>
static int a8_take(Jobs& jobs, int& t, int ntensors, const size_t* n, Fill fill) {
  // as many rounds a CTA, up to four, as the GPU would otherwise be filled times over: what a CTA does first (finding its job) takes as long as a round
  size_t ctas = 0, total = 0;
  const size_t places = (size_t)4 * (dev_sm_count() > 0 ? dev_sm_count() : 1);
  for (int i = t; i < ntensors; ++i) total += (n[i] + 8 * A8_VALUES - 1) / (8 * A8_VALUES);
  jobs.n = 0;
  jobs.rounds = (int)(total > 4 * places ? 4 : total > places ? (total + places - 1) / places : 1);
  const size_t per = (size_t)8 * A8_VALUES * jobs.rounds;
  for (; t < ntensors && jobs.n < CAP; ++t) {
    if (!n[t]) continue;
    const size_t each = (n[t] + per - 1) / per;
    if (ctas + each > 0x7fffffffull) break;                                // one tensor alone is within that, see the callers
    jobs.first[jobs.n] = (uint32_t)ctas;
    jobs.len[jobs.n] = n[t];
    fill(jobs.n++, t);
    ctas += each;
  }
  jobs.first[jobs.n] = (uint32_t)ctas;
  return (int)ctas;
}
template <int CAP>
static int a8_update(const det_adamw_desc* descs, const int* pdtypes, const void* const* p, float* const* g, const void* const* m, const void* const* v,
                     const float* const* s, void* const* p_out, void* const* m_out, void* const* v_out, float* const* s_out, const size_t* n, int ntensors,
                     const float* coef_dev, cudaStream_t st) {
  for (int t = 0; t < ntensors;) {
    Adam8Jobs<CAP> jobs;
    int last = -1;
    const int ctas = a8_take<CAP>(jobs, t, ntensors, n, [&](int j, int i) {
      jobs.p[j] = p[i]; jobs.m[j] = m[i]; jobs.v[j] = v[i]; jobs.s[j] = s[i]; jobs.g[j] = g[i];
      jobs.po[j] = p_out[i]; jobs.mo[j] = m_out[i]; jobs.vo[j] = v_out[i]; jobs.so[j] = s_out[i];
      const det_adamw_desc &d = descs[i], &e = descs[last < 0 ? i : last];  // tensors in a row mostly share theirs
      const bool same = last >= 0 && d.lr == e.lr && d.beta1 == e.beta1 && d.beta2 == e.beta2 && d.eps == e.eps && d.weight_decay == e.weight_decay &&
                        d.step == e.step;
      if (same) jobs.h[j] = jobs.h[j - 1];
      else jobs.h[j] = adamw_scalars(&d);
      last = i;
      jobs.bf[j] = pdtypes[i] == DET_BF16;
    });
    if (!jobs.n) break;
    launch_after(k_adamw8<CAP>, ctas, 256, 0, st, jobs, coef_dev);
    DET_CHECK_LAUNCH();
  }
  return DET_OK;
}
template <bool PACK, int CAP>
static int a8_convert(int8_t* const* m8, uint8_t* const* v8, float* const* s, float* const* m, float* const* v, const size_t* n, int ntensors, cudaStream_t st) {
  for (int t = 0; t < ntensors;) {
    Adam8Numbers<CAP> jobs;
    const int ctas = a8_take<CAP>(jobs, t, ntensors, n, [&](int j, int i) { jobs.m8[j] = m8[i]; jobs.v8[j] = v8[i]; jobs.s[j] = s[i]; jobs.m[j] = m[i]; jobs.v[j] = v[i]; });
    if (!jobs.n) break;
    launch_after(k_adamw8_numbers<PACK, CAP>, ctas, 256, 0, st, jobs);
    DET_CHECK_LAUNCH();
  }
  return DET_OK;
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
    if (!aligned_to(p[t], ap) || !aligned_to(p_out[t], ap) || !aligned16(g[t]) || !a8_moments_at(m[t], v[t], s[t]) || !a8_moments_at(m_out[t], v_out[t], s_out[t]))
      return DET_ERR_ALIGN;
  }
  const auto few = a8_update<ADAM8_FEW>, many = a8_update<ADAM8_JOBS>;
  return (ntensors <= ADAM8_FEW ? few : many)(descs, pdtypes, p, g, m, v, s, p_out, m_out, v_out, s_out, n, ntensors, coef_dev, (cudaStream_t)stream);
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
  const auto few = a8_convert<PACK, ADAM8_FEW>, many = a8_convert<PACK, ADAM8_JOBS>;
  return (ntensors <= ADAM8_FEW ? few : many)(m8, v8, s, m, v, n, ntensors, (cudaStream_t)stream);
}
extern "C" int det_adamw8_pack(const float* const* m, const float* const* v, int8_t* const* m8, uint8_t* const* v8, float* const* s, const size_t* n,
                               int ntensors, void* stream) {
  return a8_numbers<true>(m8, v8, s, const_cast<float* const*>(m), const_cast<float* const*>(v), n, ntensors, stream);
}
extern "C" int det_adamw8_unpack(const int8_t* const* m8, const uint8_t* const* v8, const float* const* s, float* const* m, float* const* v, const size_t* n,
                                 int ntensors, void* stream) {
  return a8_numbers<false>(const_cast<int8_t* const*>(m8), const_cast<uint8_t* const*>(v8), const_cast<float* const*>(s), m, v, n, ntensors, stream);
}
