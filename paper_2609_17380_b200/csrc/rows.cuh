// Eight adjacent values of a row, bf16 or f32, in registers; the 8-bit checkpoint of 32 adjacent values (four lanes of eight).
#pragma once
#include "common.cuh"

namespace det {

// two values rounded to bf16 in one instruction (one by one they go through the conversion pipe); same bits as two of f2bf
__device__ __forceinline__ uint32_t bf_pair(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// four low bytes
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// eight values rounded to bf16 and back
__device__ __forceinline__ void round8(float v[8]) {
#pragma unroll
  for (int t = 0; t < 8; t += 2) {
    const uint32_t u = bf_pair(v[t], v[t + 1]);
    v[t] = bflo(u);
    v[t + 1] = bfhi(u);
  }
}
__device__ __forceinline__ void unpack8(const uint4& u, float v[8]) {
  v[0] = bflo(u.x); v[1] = bfhi(u.x); v[2] = bflo(u.y); v[3] = bfhi(u.y);
  v[4] = bflo(u.z); v[5] = bfhi(u.z); v[6] = bflo(u.w); v[7] = bfhi(u.w);
}
// element `col` of row `row` of rows of D
__device__ __forceinline__ size_t row_at(int row, int D, int col) { return (size_t)((unsigned long long)(unsigned)row * (unsigned)D) + col; }
template <bool BF>
__device__ __forceinline__ void load8(const void* p, size_t idx, float v[8]) {
  if (BF) {
    unpack8(*reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(p) + idx), v);
  } else {
    const float4* q = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p) + idx);
    float4 a = q[0], b = q[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}
template <bool BF>
__device__ __forceinline__ void store8(void* p, size_t idx, const float v[8]) {
  if (BF) {
    uint4 u;
    u.x = bf_pair(v[0], v[1]); u.y = bf_pair(v[2], v[3]); u.z = bf_pair(v[4], v[5]); u.w = bf_pair(v[6], v[7]);
    *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(p) + idx) = u;
  } else {
    float4* q = reinterpret_cast<float4*>(reinterpret_cast<float*>(p) + idx);
    q[0] = make_float4(v[0], v[1], v[2], v[3]);
    q[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}
// The same where the row may end: n columns of it are left from the lane's first on, a multiple of 8 or none.
template <bool BF>
__device__ __forceinline__ void load8n(const void* p, size_t idx, int n, float v[8]) {
  if (n > 0) { load8<BF>(p, idx, v); return; }
#pragma unroll
  for (int t = 0; t < 8; ++t) v[t] = 0.0f;
}
// Rows of any length and address: a warp's 256 columns are read lane by lane (column lane + 32 k: 64 or 128 adjacent bytes an instruction, where eight
// adjacent values a lane touch sixteen times as many sectors) and dealt out through `room`, 256 floats of the warp's own.  `left` columns of
// the row are left from the warp's first on, `base` is that one's index.  BYTES 1: codes.
template <int BYTES>
__device__ __forceinline__ void load_any(const void* p, size_t base, int left, uint32_t raw[8]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int e = lane + 32 * k;
    raw[k] = 0u;
    if (e < left) {
      if (BYTES == 4) raw[k] = reinterpret_cast<const uint32_t*>(p)[base + e];
      else if (BYTES == 2) raw[k] = (uint32_t)reinterpret_cast<const uint16_t*>(p)[base + e] << 16;
      else raw[k] = __float_as_uint((float)reinterpret_cast<const int8_t*>(p)[base + e]);
    }
  }
}
__device__ __forceinline__ void deal_out(float* room, const uint32_t raw[8], float v[8]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < 8; ++k) room[lane + 32 * k] = __uint_as_float(raw[k]);
  __syncwarp();
  const float4 a = reinterpret_cast<const float4*>(room)[2 * lane], b = reinterpret_cast<const float4*>(room)[2 * lane + 1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  __syncwarp();
}
template <bool BF>
__device__ __forceinline__ void store_any(void* p, size_t base, int left, float* room, const float v[8]) {
  const int lane = threadIdx.x & 31;
  reinterpret_cast<float4*>(room)[2 * lane] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(room)[2 * lane + 1] = make_float4(v[4], v[5], v[6], v[7]);
  __syncwarp();
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int e = lane + 32 * k;
    if (e < left) {
      if (BF) reinterpret_cast<uint16_t*>(p)[base + e] = f2bf(room[e]);
      else reinterpret_cast<float*>(p)[base + e] = room[e];
    }
  }
  __syncwarp();
}

// ---- values on their way: asynchronous copies into a place of the thread's own, so that nothing but the thread waits for them -----------
// BYTES of eight adjacent values: 16 (bf16), 32 (f32), 8 (codes); `there` false: zeros, the address is not followed.  A CTA of T threads has
// T * BYTES bytes a row.
template <int BYTES, int T>
__device__ __forceinline__ void row_fetch(char* place, const void* src, bool there) {
  const uint32_t dst = (uint32_t)__cvta_generic_to_shared(place);
  if (BYTES == 8) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst + threadIdx.x * 8), "l"(src), "r"(there ? 8 : 0) : "memory");
  } else {
#pragma unroll
    for (int h = 0; h < BYTES / 16; ++h)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + (h * T + threadIdx.x) * 16), "l"(static_cast<const char*>(src) + h * 16),
                   "r"(there ? 16 : 0)
                   : "memory");
  }
}
__device__ __forceinline__ void fetch_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void fetch_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
template <bool BF, int T>
__device__ __forceinline__ void row_take(const char* place, float v[8]) {
  const uint4* q = reinterpret_cast<const uint4*>(place) + threadIdx.x;
  const uint4 a = q[0];
  if (BF) {
    unpack8(a, v);
  } else {
    const uint4 b = q[T];
    v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
    v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
  }
}

// ---- 8-bit checkpoints -----------------------------------------------------------------------------------
// A group is 32 adjacent values of a row.  Its step is the smallest power of two 2^E, at least 2^-126, with max|v| <= 127 * 2^E, kept as
// its binary32 exponent field E + 127 (1 .. 249); code = rne(v / 2^E) in -127 .. 127.  With a power of two every product here is exact:
// the code is the nearest one, and code * 2^E has at most 7 significant bits, so it is exact in bf16 too.  Field 255 marks a group
// that holds an infinity or a NaN: codes +-127 for the infinities and 0 for the rest, which come back as infinities and NaNs.
constexpr int A8_GROUP = 32;
// the field from the largest magnitude's bits (of the whole group): its own exponent field less 6, one more past 127/64 of its power of two
__device__ __forceinline__ uint32_t a8_field(uint32_t amax) {
  const int f = (int)(amax >> 23) - 6 + ((amax & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  return amax >= 0x7f800000u ? 255u : (uint32_t)max(f, 1);
}
__device__ __forceinline__ float a8_step(uint32_t field) { return __uint_as_float(field << 23); }
__device__ __forceinline__ float a8_inv(uint32_t field) { return __uint_as_float((254u - field) << 23); }    // of a finite group
__device__ __forceinline__ uint32_t a8_code_nonfinite(float v) {
  return fabsf(v) != __int_as_float(0x7f800000) ? 0u : (v > 0.0f ? 127u : 0x81u);
}
// codes of eight values, low byte first; |v * inv| <= 127, and adding 1.5 * 2^23 rounds it to the nearest even integer, left in the low byte (the product
// with a power of two is exact, or too small to be seen: fused or not is the same)
__device__ __forceinline__ uint2 a8_codes8(const float v[8], uint32_t field) {
  uint32_t c[8];
  if (field != 255u) {
    const float inv = a8_inv(field);
#pragma unroll
    for (int t = 0; t < 8; t += 2) {
      const float2 r = fma2(make_float2(v[t], v[t + 1]), same2(inv), same2(12582912.0f));
      c[t] = __float_as_uint(r.x);
      c[t + 1] = __float_as_uint(r.y);
    }
  } else {
#pragma unroll
    for (int t = 0; t < 8; ++t) c[t] = a8_code_nonfinite(v[t]);
  }
  uint2 o;
  o.x = low_bytes(c[0], c[1], c[2], c[3]);
  o.y = low_bytes(c[4], c[5], c[6], c[7]);
  return o;
}
// values of eight codes: a byte, its sign flipped, in the low bits of 2^23 is 2^23 + 128 + code.  In pairs, but for the SwiGLU backward pass, for which the
// compiler then keeps less in flight (8192 x 8192: 102 us, one at a time 92; its forward from the checkpoint 84 one at a time and 76 in pairs).
template <bool PAIRS = true>
__device__ __forceinline__ void a8_values8(uint2 q, float step, float v[8]) {
  const auto number = [](uint32_t codes, int byte) { return __uint_as_float(__byte_perm(codes, 0x4b000000u, 0x7540 + byte)); };
  const auto pair = [&](uint32_t codes, int byte, float* to) {
    const float2 r = mul2(fma2(make_float2(number(codes, byte), number(codes, byte + 1)), same2(1.0f), same2(-8388736.0f)), same2(step));
    to[0] = r.x;
    to[1] = r.y;
  };
  if (PAIRS) {
    q.x ^= 0x80808080u;
    q.y ^= 0x80808080u;
#pragma unroll
    for (int t = 0; t < 4; t += 2) {
      pair(q.x, t, v + t);
      pair(q.y, t, v + 4 + t);
    }
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      v[t] = fmul(fsub(number(q.x ^ 0x80808080u, t), 8388736.0f), step);
      v[4 + t] = fmul(fsub(number(q.y ^ 0x80808080u, t), 8388736.0f), step);
    }
  }
}
// the largest magnitude of eight values as bits: an order of unsigned integers, NaNs above infinity
__device__ __forceinline__ uint32_t a8_amax8(const float v[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int t = 0; t < 8; ++t) m = max(m, __float_as_uint(v[t]) & 0x7fffffffu);
  return m;
}
// over the four lanes that hold a group; all lanes of the warp take part
__device__ __forceinline__ uint32_t a8_quad_max(uint32_t m) {
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  return max(m, __shfl_xor_sync(0xffffffffu, m, 2));
}

}  // namespace det
