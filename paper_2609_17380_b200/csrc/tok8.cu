// Products of 8-bit integers with a scale for each token and each output channel, and the gated feed-forward block on them.
//
//   codes of a row v (a token's activations, a channel's weights):  a = max|v|, s = a / 127, code = rne(v (1/s)) in [-127, 127]
//   Y[m,n] = sum_k qX[m,k] qW[n,k] * (s_x[m] s_w[n])
// A scale can be taken out of a sum only where its index is not the one that is summed over.  So the backward pass puts the scale of the contracted
// index into the gradient before that is quantised, and all three products are exact integers with scales outside:
//   A[m,n] = dY[m,n] s_w[n], by token:    dX[m,k] = s_a[m] sum_n qA[m,n] qW[n,k]
//   G[m,n] = dY[m,n] s_x[m], by channel:  dW[n,k] = s_g[n] sum_m qG[m,n] qX[m,k]
// The sums are exact in int32 (contractions below 2^17), so no order of them shows and a contraction may be split over CTAs.
#include "tc05.cuh"
#include "internal.h"
#include "rows.cuh"

namespace det {

constexpr int T8_K = 128;                                // bytes (= codes) a stage along the contraction
__host__ __device__ __forceinline__ int t8_ld(int K) { return (K + 15) / 16 * 16; }   // bytes from a row of codes to the next

// ---- codes -------------------------------------------------------------------------------------------------
// The scale of a group from the largest magnitude's bits; one with an infinity or a NaN has the scale NaN and codes 0.
__device__ __forceinline__ float t8_scale(uint32_t amax) {
  return amax >= 0x7f800000u ? __int_as_float(0x7fffffff) : fdiv(__uint_as_float(amax), 127.0f);
}
__device__ __forceinline__ float t8_inverse(float s) { return s > 0.0f ? fdiv(1.0f, s) : 0.0f; }     // 0 for a scale that is 0 or NaN
// rne(v * inv) in the low byte of the result; |v * inv| is at most 127 (1 + 2^-22), so nothing has to be clamped.  dead: the group has the scale NaN.
__device__ __forceinline__ uint32_t t8_code(float v, float inv) { return __float_as_uint(fadd(fmul(v, inv), 12582912.0f)); }
__device__ __forceinline__ uint32_t t8_pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
__device__ __forceinline__ uint2 t8_codes8(const float v[8], float inv, bool dead) {
  uint32_t c[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) c[t] = t8_code(v[t], inv);
  return dead ? make_uint2(0u, 0u) : make_uint2(t8_pack4(c[0], c[1], c[2], c[3]), t8_pack4(c[4], c[5], c[6], c[7]));
}
__device__ __forceinline__ uint32_t t8_max8(const float v[8], uint32_t m) {
#pragma unroll
  for (int t = 0; t < 8; ++t) m = max(m, __float_as_uint(v[t]) & 0x7fffffffu);
  return m;
}

// Rows of a multiple of 8 columns, 16-byte aligned: WPR warps a row, up to 64 values a lane, which stay in registers.
template <int WPR>
__global__ void __launch_bounds__(256) k_t8_rows(const uint16_t* __restrict__ x, size_t ld, int M, int K, int8_t* __restrict__ q, float* __restrict__ s) {
  grid_dep();
  __shared__ uint32_t part[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = blockIdx.x * (8 / WPR) + warp / WPR, first = ((warp % WPR) * 32 + lane) * 8, ldq = t8_ld(K);
  const bool there = row < M;
  float v[8][8];
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int c = first + k * (WPR * 256);
    load8n<true>(x, (size_t)row * ld + c, there && c < K, v[k]);
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) m = t8_max8(v[k], m);
  m = __reduce_max_sync(0xffffffffu, m);
  if (WPR > 1) {
    if (lane == 0) part[warp] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WPR; ++w) m = max(m, part[warp / WPR * WPR + w]);
  }
  if (!there) return;
  const float sc = t8_scale(m), inv = t8_inverse(sc);
  const bool dead = m >= 0x7f800000u;
  if (first == 0) s[row] = sc;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int c = first + k * (WPR * 256);
    if (c < ldq) *reinterpret_cast<uint2*>(q + (size_t)row * ldq + c) = c < K ? t8_codes8(v[k], inv, dead) : make_uint2(0u, 0u);
  }
}
// Any width, stride and address: a CTA a row, which is read twice.
__global__ void __launch_bounds__(256) k_t8_rows_any(const uint16_t* __restrict__ x, size_t ld, int K, int8_t* __restrict__ q, float* __restrict__ s) {
  grid_dep();
  __shared__ uint32_t part[8];
  const int row = blockIdx.x, ldq = t8_ld(K);
  const uint16_t* p = x + (size_t)row * ld;
  uint32_t m = 0;
  for (int c = threadIdx.x; c < K; c += 256) m = max(m, ((uint32_t)p[c] << 16) & 0x7fffffffu);
  m = __reduce_max_sync(0xffffffffu, m);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) m = max(m, part[w]);
  const float sc = t8_scale(m), inv = t8_inverse(sc);
  if (threadIdx.x == 0) s[row] = sc;
  for (int c = threadIdx.x; c < ldq; c += 256)
    q[(size_t)row * ldq + c] = c < K && m < 0x7f800000u ? (int8_t)t8_code(bf2f(p[c]), inv) : (int8_t)0;
}

// Codes [R, ld(C)] -> [C, ld(R)], through shared memory, whole 128-byte lines on both sides but at the edges.  What lies behind column C of the
// input is zero; so is what is written behind column R.
__global__ void __launch_bounds__(128) k_t8_transpose(const int8_t* __restrict__ in, int R, int C, int8_t* __restrict__ out) {
  __shared__ __align__(16) uint8_t tile[128 * 128];
  const int t = threadIdx.x, c0 = blockIdx.x * 128 + grid_dep(), r0 = blockIdx.y * 128, ldi = t8_ld(C), ldo = t8_ld(R);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = i * 16 + (t >> 3), ch = (t & 7) * 16;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (r0 + r < R && c0 + ch < ldi) v = __ldg(reinterpret_cast<const uint4*>(in + (size_t)(r0 + r) * ldi + c0 + ch));
    *reinterpret_cast<uint4*>(tile + r * 128 + ch) = v;
  }
  __syncthreads();
  uint32_t w[32];
#pragma unroll
  for (int k = 0; k < 32; ++k)
    w[k] = (uint32_t)tile[(4 * k) * 128 + t] | ((uint32_t)tile[(4 * k + 1) * 128 + t] << 8) | ((uint32_t)tile[(4 * k + 2) * 128 + t] << 16) |
           ((uint32_t)tile[(4 * k + 3) * 128 + t] << 24);
  __syncthreads();                       // everybody has read its column: the tile becomes the transposed output tile
#pragma unroll
  for (int g = 0; g < 8; ++g)            // row t of it, sixteen-byte pieces XOR-swizzled by row
    *reinterpret_cast<uint4*>(tile + t * 128 + ((g ^ (t & 7)) << 4)) = make_uint4(w[4 * g], w[4 * g + 1], w[4 * g + 2], w[4 * g + 3]);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = i * 16 + (t >> 3), ch = t & 7;
    if (c0 + r < C && r0 + ch * 16 < ldo)
      *reinterpret_cast<uint4*>(out + (size_t)(c0 + r) * ldo + r0 + ch * 16) = *reinterpret_cast<const uint4*>(tile + r * 128 + ((ch ^ (r & 7)) << 4));
  }
}

// ---- operands of the backward products ---------------------------------------------------------------------
// dY [M, N] with the scales of the channels (A) and of the tokens (G).  Largest magnitudes first: a warp reads 256 columns of a row, a CTA 128 rows.
__device__ __forceinline__ void t8_load8(const uint16_t* p, size_t at, int n, bool vec, float v[8]) {
  if (vec && n >= 8) { load8<true>(p, at, v); return; }
#pragma unroll
  for (int t = 0; t < 8; ++t) v[t] = t < n ? bf2f(p[at + t]) : 0.0f;
}
constexpr int T8_GR = 128;
__global__ void __launch_bounds__(256) k_t8_grad_max(const uint16_t* __restrict__ dy, size_t ld, int M, int N, const float* __restrict__ s_x,
                                                     const float* __restrict__ s_w, uint32_t* __restrict__ rowmax, uint32_t* __restrict__ colmax, int vec) {
  grid_dep();
  __shared__ uint32_t cols[8][256];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x * 256 + lane * 8, r0 = blockIdx.y * T8_GR;
  const int left = N - c;
  float sw[8];
  uint32_t cm[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    sw[t] = t < left ? s_w[c + t] : 0.0f;
    cm[t] = 0;
  }
#pragma unroll 4
  for (int i = 0; i < T8_GR / 8; ++i) {
    const int r = r0 + i * 8 + warp;
    if (r >= M) break;
    float v[8];
    t8_load8(dy, (size_t)r * ld + c, left, vec, v);
    const float sx = s_x[r];
    uint32_t rm = 0;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      if (t >= left) break;
      rm = max(rm, __float_as_uint(fmul(v[t], sw[t])) & 0x7fffffffu);
      cm[t] = max(cm[t], __float_as_uint(fmul(v[t], sx)) & 0x7fffffffu);
    }
    rm = __reduce_max_sync(0xffffffffu, rm);
    if (lane == 0) atomicMax(rowmax + r, rm);
  }
#pragma unroll
  for (int t = 0; t < 8; ++t) cols[warp][lane * 8 + t] = cm[t];
  __syncthreads();
  const int j = blockIdx.x * 256 + threadIdx.x;
  uint32_t m = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) m = max(m, cols[w][threadIdx.x]);
  if (j < N) atomicMax(colmax + j, m);
}
// Then the codes: A as it lies, G transposed.  A thread has 8 rows of 8 columns of a tile of 128 x 128; eight codes of a column are a piece of 8 bytes
// whose place in shared memory is swizzled by the group of columns, so that the sixteen of a warp meet in no bank.
__global__ void __launch_bounds__(256) k_t8_grad_codes(const uint16_t* __restrict__ dy, size_t ld, int M, int N, const float* __restrict__ s_x,
                                                       const float* __restrict__ s_w, const uint32_t* __restrict__ rowmax,
                                                       const uint32_t* __restrict__ colmax, int8_t* __restrict__ qa, float* __restrict__ s_a,
                                                       int8_t* __restrict__ qgt, float* __restrict__ s_g, int vec) {
  grid_dep();
  __shared__ __align__(16) uint8_t tile[128 * 128];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, r0 = blockIdx.y * 128, c0 = blockIdx.x * 128, c = c0 + tx * 8;
  const int left = N - c, ldn = t8_ld(N), ldm = t8_ld(M);
  float sw[8], ig[8];
  bool dead_c[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const uint32_t m = t < left ? colmax[c + t] : 0u;
    const float sg = t8_scale(m);
    sw[t] = t < left ? s_w[c + t] : 0.0f;
    ig[t] = t8_inverse(sg);
    dead_c[t] = m >= 0x7f800000u;
    if (blockIdx.y == 0 && ty == 0 && t < left) s_g[c + t] = sg;
  }
  uint32_t piece[8][2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t g[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = r0 + ty * 8 + h * 4 + i;
      const bool there = r < M;
      float v[8];
      t8_load8(dy, (size_t)r * ld + c, there ? left : 0, vec, v);
      const uint32_t m = there ? rowmax[r] : 0u;
      const float sa = t8_scale(m), ia = t8_inverse(sa), sx = there ? s_x[r] : 0.0f;
      if (there && blockIdx.x == 0 && tx == 0) s_a[r] = sa;
      float a[8];
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        a[t] = fmul(v[t], sw[t]);
        g[i][t] = dead_c[t] || !there ? 0u : t8_code(fmul(v[t], sx), ig[t]);
      }
      if (there && c < ldn) *reinterpret_cast<uint2*>(qa + (size_t)r * ldn + c) = t8_codes8(a, ia, m >= 0x7f800000u);
    }
#pragma unroll
    for (int t = 0; t < 8; ++t) piece[t][h] = t8_pack4(g[0][t], g[1][t], g[2][t], g[3][t]);
  }
#pragma unroll
  for (int t = 0; t < 8; ++t) *reinterpret_cast<uint2*>(tile + (tx * 8 + t) * 128 + ((ty ^ tx) << 3)) = make_uint2(piece[t][0], piece[t][1]);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int col = i * 32 + (threadIdx.x >> 3), ch = threadIdx.x & 7, f = (col >> 3) & 15;
    uint4 w = *reinterpret_cast<const uint4*>(tile + col * 128 + (((2 * ch) ^ (f & 14)) << 3));
    if (f & 1) w = make_uint4(w.z, w.w, w.x, w.y);
    if (c0 + col < N && r0 + ch * 16 < ldm) *reinterpret_cast<uint4*>(qgt + (size_t)(c0 + col) * ldm + r0 + ch * 16) = w;
  }
}

// ---- products ----------------------------------------------------------------------------------------------
enum { T8_BF16 = 0, T8_F32 = 1, T8_GLU = 2 };
struct T8Out {
  void* out;             // BF16: bf16 [I, J]; F32: f32 [I, J]; GLU: h, bf16 [I, J]
  size_t ld;             // elements from a row of it to the next
  const float* rs;       // scale of every row
  const float* cs;       // scale of every column (GLU: of the gates, then of the ups), or NULL
  uint16_t* gu;          // GLU: gate and up, bf16 [I, 2 J], or NULL
  size_t ld_gu;
  int I, J, K;
  int vec, vec_gu;       // rows in whole sixteen-byte pieces
};

// A warp's 32 rows x 32 columns, a row a lane (`w`: NW sixteen-byte words of ES-byte elements), through a staging tile so that every store
// instruction writes whole row segments; rows and columns that are left, from the warp's first on.
template <int NW, int ES>
__device__ __forceinline__ void t8_store(uint8_t* stage, uint8_t* base, size_t pitch, int rows, int cols, int vec, const uint4 (&w)[NW]) {
  const int lane = threadIdx.x & 31;
  constexpr int SH = NW == 8 ? 0 : 1, RPI = 32 / NW;
  __syncwarp();
#pragma unroll
  for (int v = 0; v < NW; ++v) *reinterpret_cast<uint4*>(stage + lane * (NW * 16) + ((v ^ ((lane >> SH) & (NW - 1))) << 4)) = w[v];
  __syncwarp();
  if (vec && cols >= 32) {
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const int r = i * RPI + lane / NW, piece = lane % NW;
      const uint4 x = *reinterpret_cast<const uint4*>(stage + r * (NW * 16) + ((piece ^ ((r >> SH) & (NW - 1))) << 4));
      if (r < rows) *reinterpret_cast<uint4*>(base + r * pitch + piece * 16) = x;
    }
  } else if (lane < cols) {
    const int piece = lane * ES / 16, at = lane * ES % 16;
    for (int r = 0; r < 32 && r < rows; ++r) {
      const uint8_t* p = stage + r * (NW * 16) + ((piece ^ ((r >> SH) & (NW - 1))) << 4) + at;
      if (ES == 2) *reinterpret_cast<uint16_t*>(base + r * pitch + lane * 2) = *reinterpret_cast<const uint16_t*>(p);
      else *reinterpret_cast<uint32_t*>(base + r * pitch + lane * 4) = *reinterpret_cast<const uint32_t*>(p);
    }
  }
}
// 32 accumulators of a row, times the row's scale and the columns' (in shared memory), as bf16 pairs
__device__ __forceinline__ void t8_scaled(const uint32_t (&r)[32], float rs, const float* cs, bool by_col, uint4 (&o)[4]) {
#pragma unroll
  for (int v = 0; v < 8; ++v) {
    const float4 c = by_col ? *reinterpret_cast<const float4*>(cs + 4 * v) : make_float4(1.0f, 1.0f, 1.0f, 1.0f);
    const float2 s0 = by_col ? mul2(same2(rs), make_float2(c.x, c.y)) : same2(rs), s1 = by_col ? mul2(same2(rs), make_float2(c.z, c.w)) : same2(rs);
    const float2 a = mul2(make_float2(__int2float_rn((int)r[4 * v]), __int2float_rn((int)r[4 * v + 1])), s0);
    const float2 b = mul2(make_float2(__int2float_rn((int)r[4 * v + 2]), __int2float_rn((int)r[4 * v + 3])), s1);
    reinterpret_cast<uint32_t*>(o)[2 * v] = bf_pair(a.x, a.y);
    reinterpret_cast<uint32_t*>(o)[2 * v + 1] = bf_pair(b.x, b.y);
  }
}
__device__ __forceinline__ float t8_sigmoid(float g) { return fdiv(1.0f, fadd(1.0f, det_exp(-g))); }
__device__ __forceinline__ uint32_t t8_glu2(uint32_t g, uint32_t u) {
  const float2 sg = make_float2(t8_sigmoid(bflo(g)), t8_sigmoid(bfhi(g)));
  const float2 h = mul2(mul2(make_float2(bflo(g), bfhi(g)), sg), make_float2(bflo(u), bfhi(u)));
  return bf_pair(h.x, h.y);
}
// Columns j0 .. j0 + CW of the warp's 32 rows (row0 the first); GLU: the ups' accumulators lie UP columns behind the gates'.  stage: the
// warp's own 4 KiB in shared memory, whose upper half holds the columns' scales (bf16 rows take the lower one alone).
template <int EPI, int CW, int UP>
__device__ __forceinline__ void t8_epilogue(const T8Out& o, uint32_t taddr, int row0, int j0, uint8_t* stage) {
  float* cs = reinterpret_cast<float*>(stage + 2048);
  const int lane = threadIdx.x & 31, rows = o.I - row0;
  if (rows <= 0) return;
  const float rs = lane < rows ? o.rs[row0 + lane] : 0.0f;
#pragma unroll 1
  for (int c = 0; c < CW; c += 32) {
    const int j = j0 + c, cols = o.J - j;
    if (cols <= 0) break;
    uint32_t r[32];
    tmem_ld32(taddr + (uint32_t)c, r);
    if (EPI == T8_F32) {
      uint4 w[8];
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float2 f = mul2(make_float2(__int2float_rn((int)r[2 * v]), __int2float_rn((int)r[2 * v + 1])), same2(rs));
        reinterpret_cast<float2*>(w)[v] = f;
      }
      t8_store<8, 4>(stage, reinterpret_cast<uint8_t*>(reinterpret_cast<float*>(o.out) + row0 * o.ld + j), o.ld * 4, rows, cols, o.vec, w);
      continue;
    }
    if (o.cs) {
      __syncwarp();
      cs[lane] = lane < cols ? o.cs[j + lane] : 0.0f;
      if (EPI == T8_GLU) cs[32 + lane] = lane < cols ? o.cs[o.J + j + lane] : 0.0f;
      __syncwarp();
    }
    uint4 g[4];
    t8_scaled(r, rs, cs, o.cs != nullptr, g);
    if (EPI == T8_BF16) {
      t8_store<4, 2>(stage, reinterpret_cast<uint8_t*>(reinterpret_cast<uint16_t*>(o.out) + row0 * o.ld + j), o.ld * 2, rows, cols, o.vec, g);
      continue;
    }
    uint4 u[4];
    tmem_ld32(taddr + (uint32_t)(UP + c), r);
    t8_scaled(r, rs, cs + 32, true, u);
    if (o.gu) {
      uint8_t* p = reinterpret_cast<uint8_t*>(o.gu + row0 * o.ld_gu + j);
      t8_store<4, 2>(stage, p, o.ld_gu * 2, rows, cols, o.vec_gu, g);
      t8_store<4, 2>(stage, p + (size_t)o.J * 2, o.ld_gu * 2, rows, cols, o.vec_gu, u);
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      uint32_t* gp = reinterpret_cast<uint32_t*>(g) + v;
      *gp = t8_glu2(*gp, reinterpret_cast<const uint32_t*>(u)[v]);
    }
    t8_store<4, 2>(stage, reinterpret_cast<uint8_t*>(reinterpret_cast<uint16_t*>(o.out) + row0 * o.ld + j), o.ld * 2, rows, cols, o.vec, g);
  }
}

// Tiles of 128 x BN by one CTA, or of 256 x 256 by the two of a cluster (PAIR; each has 128 rows and stages half of the columns' operand).  The
// columns of a GLU tile are BN / 2 gates and the ups that belong to them.  Roles, ring and waits as in igemm.cu.
template <bool PAIR, int BN>
struct T8Tile {
  static constexpr int BM = PAIR ? 256 : 128, BROWS = PAIR ? BN / 2 : BN;         // BROWS: rows of the columns' operand that a CTA stages
  static constexpr int STAGE_A = 128 * T8_K, STAGE_B = BROWS * T8_K, STAGE = STAGE_A + STAGE_B;
  static constexpr int STAGES = PAIR ? 6 : (BN == 128 ? 6 : 8), EW = BN == 64 ? 4 : 8;
  static constexpr int THREADS = 64 + 32 * EW, TCOLS = 2 * BN;
  static constexpr size_t SMEM = (size_t)STAGES * STAGE + EW * 4096 + 1024;
};
template <bool PAIR, int BN, int EPI>
__global__ void __launch_bounds__(T8Tile<PAIR, BN>::THREADS, 1)
    k_t8_gemm(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ T8Out o, int* status) {
  typedef T8Tile<PAIR, BN> T;
  constexpr int STAGES = T::STAGES, EW = T::EW, BH = EPI == T8_GLU ? BN / 2 : BN;    // BH: columns of the output in a tile
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ __align__(8) uint64_t bar_full[STAGES], bar_empty[STAGES], bar_tfull[2], bar_tempty[2];
  __shared__ uint32_t tmem_base_s;
  __shared__ int abort_s;
  volatile int* abort_flag = &abort_s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0;
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(&bar_full[s], 1); mbar_init(&bar_empty[s], 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(&bar_tfull[a], 1); mbar_init(&bar_tempty[a], PAIR ? 2 * EW : EW); }
    abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmA)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmB)) : "memory");
  }
  if (warp == 1) {
    if (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"((uint32_t)T::TCOLS) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"((uint32_t)T::TCOLS) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();          // the peer's barriers are initialised before anything can signal them
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_s;
  grid_dep();

  const int tiles_i = (o.I + T::BM - 1) / T::BM, tiles_j = (o.J + BH - 1) / BH, tiles = tiles_i * tiles_j, kblocks = (o.K + T8_K - 1) / T8_K;
  const int unit = PAIR ? blockIdx.x >> 1 : blockIdx.x, units = PAIR ? gridDim.x >> 1 : gridDim.x;
  // the dimension with fewer tiles runs fastest: the CTAs of one time share its operand's tiles and the other operand streams through L2 once
  auto origin = [&](int tile, int& i0, int& j0) {
    if (tiles_j <= tiles_i) { j0 = (tile % tiles_j) * BH; i0 = (tile / tiles_j) * T::BM; }
    else { i0 = (tile % tiles_i) * T::BM; j0 = (tile / tiles_i) * BH; }
  };
  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int tile = unit; tile < tiles && ok; tile += units) {
        int i0, j0;
        origin(tile, i0, j0);
        for (int kb = 0; kb < kblocks; ++kb) {
          if (!mbar_wait(&bar_empty[stage], phase ^ 1u, abort_flag, status)) { ok = false; break; }
          uint8_t *sa = smem + stage * T::STAGE, *sb = sa + T::STAGE_A;
          if (PAIR) {
            if (rank == 0) mbar_expect_tx(&bar_full[stage], 2 * T::STAGE);       // both CTAs' tiles complete on this barrier
            tma_load_2d_pair(sa, &tmA, kb * T8_K, i0 + (int)rank * 128, &bar_full[stage]);
            tma_load_2d_pair(sb, &tmB, kb * T8_K, j0 + (int)rank * (EPI == T8_GLU ? o.J : T::BROWS), &bar_full[stage]);
          } else {
            mbar_expect_tx(&bar_full[stage], T::STAGE);
            tma_load_2d(sa, &tmA, kb * T8_K, i0, &bar_full[stage]);
            tma_load_2d(sb, &tmB, kb * T8_K, j0, &bar_full[stage]);
            if (EPI == T8_GLU) tma_load_2d(sb + T::STAGE_B / 2, &tmB, kb * T8_K, o.J + j0, &bar_full[stage]);
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      // D = S32, A = B = signed 8-bit, both K-major
      constexpr uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(T::BM >> 4) << 24);
      int stage = 0, it = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int tile = unit; tile < tiles && ok; tile += units, ++it) {
        const int acc = it & 1;
        if (!mbar_wait(&bar_tempty[acc], ((uint32_t)(it >> 1) & 1u) ^ 1u, abort_flag, status)) { ok = false; break; }
        tc_fence_after();
        const uint32_t tmem_d = tmem_base + (uint32_t)(acc * BN);
        for (int kb = 0; kb < kblocks; ++kb) {
          if (!mbar_wait(&bar_full[stage], phase, abort_flag, status)) { ok = false; break; }
          tc_fence_after();
          const uint32_t sa = smem_u32(smem + stage * T::STAGE);
          const uint64_t da = make_smem_desc(sa), db = make_smem_desc(sa + T::STAGE_A);
#pragma unroll
          for (int k4 = 0; k4 < T8_K / 32; ++k4) {
            if (PAIR) umma_i8_pair(tmem_d, da + (uint64_t)(k4 * 2), db + (uint64_t)(k4 * 2), idesc, (kb | k4) ? 1u : 0u);
            else umma_i8(tmem_d, da + (uint64_t)(k4 * 2), db + (uint64_t)(k4 * 2), idesc, (kb | k4) ? 1u : 0u);
          }
          if (PAIR) umma_commit_pair(&bar_empty[stage]);
          else umma_commit(&bar_empty[stage]);
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
        if (ok) {
          if (PAIR) umma_commit_pair(&bar_tfull[acc]);
          else umma_commit(&bar_tfull[acc]);
        }
      }
    }
  } else {
    const int q = warp & 3, part = (warp - 2) >> 2;      // TMEM lane quarter this warp may read; its share of the columns
    constexpr int CW = BH / (EW / 4);
    uint8_t* stage = smem + STAGES * T::STAGE + (warp - 2) * 4096;
    const uint32_t free0 = PAIR ? mapa_u32(smem_u32(&bar_tempty[0]), 0) : 0, free1 = PAIR ? mapa_u32(smem_u32(&bar_tempty[1]), 0) : 0;
    int it = 0;
    for (int tile = unit; tile < tiles; tile += units, ++it) {
      const int acc = it & 1;
      int i0, j0;
      origin(tile, i0, j0);
      mbar_wait(&bar_tfull[acc], (uint32_t)(it >> 1) & 1u, abort_flag, status);      // passed over when it ran out: the lanes stay together
      tc_fence_after();
      t8_epilogue<EPI, CW, BN / 2>(o, tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * BN + part * CW), i0 + (int)rank * 128 + q * 32,
                                   j0 + part * CW, stage);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (PAIR) mbar_arrive_remote(acc ? free1 : free0);
        else mbar_arrive(&bar_tempty[acc]);
      }
    }
  }

  // teardown: everyone meets here (the peer may still signal this CTA's barriers or read its tiles); after a timeout copies in flight get time to land
  __syncthreads();
  if (abort_s) {
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000ll) { }
    __syncthreads();
  }
  if (PAIR) cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)T::TCOLS) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)T::TCOLS) : "memory");
  }
}

template <bool PAIR, int BN, int EPI>
static int t8_launch(const int8_t* A, const int8_t* B, int rows_b, const T8Out& o, int* status, cudaStream_t st) {
  typedef T8Tile<PAIR, BN> T;
  constexpr int BH = EPI == T8_GLU ? BN / 2 : BN;
  static DevOnce once = {};
  if (dev_ensure_smem(once, (const void*)k_t8_gemm<PAIR, BN, EPI>, T::SMEM) != DET_OK) return DET_ERR_CUDA;
  const int sms = dev_sm_count();
  if (sms < 2) return DET_ERR_CUDA;
  CUtensorMap ta, tb;
  if (!make_map_ld(&ta, A, o.I, o.K, t8_ld(o.K), 128) || !make_map_ld(&tb, B, rows_b, o.K, t8_ld(o.K), !PAIR && EPI == T8_GLU ? BN / 2 : T::BROWS))
    return DET_ERR_CUDA;
  const long long tiles = (long long)((o.I + T::BM - 1) / T::BM) * ((o.J + BH - 1) / BH);
  const int units = PAIR ? sms / 2 : sms, grid = (int)(tiles < units ? tiles : units) * (PAIR ? 2 : 1);
  launch_after_cluster(k_t8_gemm<PAIR, BN, EPI>, grid, T::THREADS, T::SMEM, PAIR ? 2 : 1, st, ta, tb, o, status);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
// The tile by whole rounds of tiles over the SMs, each the longer of its multiply loop and its epilogue (microseconds, the figures of igemm.cu).
template <int EPI>
static int t8_product(const int8_t* A, const int8_t* B, int rows_b, const T8Out& o, int* status, cudaStream_t st) {
  const int sms = dev_sm_count();
  if (sms < 2) return DET_ERR_CUDA;
  static const struct { int bn, bi; double step, turn, epi[3]; } C[3] = {
      {256, 256, 0.365, 0.9, {4.2, 6.6, 9.0}}, {128, 128, 0.30, 0.5, {1.7, 3.8, 5.0}}, {64, 128, 0.30, 0.5, {1.7, 1.8, 4.0}}};
  int pick = 0;
  double best = 0.0;
  for (int i = 0; i < 3; ++i) {
    const int bh = EPI == T8_GLU ? C[i].bn / 2 : C[i].bn, units = i == 0 ? sms / 2 : sms;
    const double tiles = (double)((o.I + C[i].bi - 1) / C[i].bi) * ((o.J + bh - 1) / bh), rounds = (double)(long long)((tiles + units - 1) / units);
    const double loop = ((o.K + T8_K - 1) / T8_K) * C[i].step, e = C[i].epi[EPI], t = rounds * ((loop > e ? loop : e) + C[i].turn) + (loop > e ? e : loop);
    if (i == 0 || t < best) { best = t; pick = i; }
  }
  if (pick == 0) return t8_launch<true, 256, EPI>(A, B, rows_b, o, status, st);
  if (pick == 1) return t8_launch<false, 128, EPI>(A, B, rows_b, o, status, st);
  return t8_launch<false, 64, EPI>(A, B, rows_b, o, status, st);
}

static int t8_quant(const uint16_t* X, int ld, int M, int K, int8_t* q, float* s, cudaStream_t st) {
  if (K % 8 == 0 && ld % 8 == 0 && aligned16(X) && K <= 16384) {
    if (K <= 2048) launch_after(k_t8_rows<1>, (unsigned)((M + 7) / 8), 256, 0, st, X, (size_t)ld, M, K, q, s);
    else if (K <= 8192) launch_after(k_t8_rows<4>, (unsigned)((M + 1) / 2), 256, 0, st, X, (size_t)ld, M, K, q, s);
    else launch_after(k_t8_rows<8>, (unsigned)M, 256, 0, st, X, (size_t)ld, M, K, q, s);
  } else {
    launch_after(k_t8_rows_any, (unsigned)M, 256, 0, st, X, (size_t)ld, K, q, s);
  }
  DET_CHECK_LAUNCH();
  return DET_OK;
}
static bool aligned_to(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
// sizes that every call shares: contractions below 2^17 (int32), rows and columns that tensor maps and tiles can number
static int t8_sizes(long long M, long long N, long long K) {
  if (M < 0 || N <= 0 || K <= 0) return DET_ERR_ARG;
  if (M > (1 << 28) || N > (1 << 28)) return DET_ERR_SHAPE;
  return K >= (1 << 17) ? DET_ERR_RANGE : DET_OK;
}
static int t8_vec(const void* p, size_t ld, int size) { return aligned16(p) && ld * size % 16 == 0; }

// gradient operands into the workspace, then both products
struct T8Ws { size_t qa, qgt, qxt, s_a, s_g, rowmax, colmax, dgu, bytes; };
static T8Ws t8_ws(int M, int N, int K, bool glu) {
  T8Ws w;
  size_t at = 0;
  auto take = [&](size_t n) { const size_t here = at; at += align_up(n, 256); return here; };
  w.qa = take((size_t)M * t8_ld(N));
  w.qgt = take((size_t)N * t8_ld(M));
  w.qxt = take((size_t)K * t8_ld(M));
  w.s_a = take((size_t)M * 4);
  w.s_g = take((size_t)N * 4);
  w.rowmax = take((size_t)M * 4);
  w.colmax = take((size_t)N * 4);
  w.dgu = take(glu ? (size_t)M * N * 2 : 0);
  w.bytes = at;
  return w;
}
static int t8_backward(const uint16_t* dY, int ld_dy, const int8_t* qX, const float* s_x, const int8_t* qWt, const float* s_w, int M, int N, int K,
                       uint16_t* dX, int ld_dx, float* dW, const T8Ws& w, char* ws, int* status, cudaStream_t st) {
  int8_t *qa = (int8_t*)(ws + w.qa), *qgt = (int8_t*)(ws + w.qgt), *qxt = (int8_t*)(ws + w.qxt);
  float *s_a = (float*)(ws + w.s_a), *s_g = (float*)(ws + w.s_g);
  uint32_t *rowmax = (uint32_t*)(ws + w.rowmax), *colmax = (uint32_t*)(ws + w.colmax);
  if (cudaMemsetAsync(rowmax, 0, w.dgu - w.rowmax, st) != cudaSuccess) { cudaGetLastError(); return DET_ERR_CUDA; }
  const int vec = t8_vec(dY, ld_dy, 2);
  launch_after(k_t8_grad_max, dim3((N + 255) / 256, (M + T8_GR - 1) / T8_GR), 256, 0, st, dY, (size_t)ld_dy, M, N, s_x, s_w, rowmax, colmax, vec);
  launch_after(k_t8_grad_codes, dim3((N + 127) / 128, (M + 127) / 128), 256, 0, st, dY, (size_t)ld_dy, M, N, s_x, s_w, rowmax, colmax, qa, s_a, qgt, s_g, vec);
  DET_CHECK_LAUNCH();
  if (dX) {
    T8Out o = {};
    o.out = dX; o.ld = ld_dx; o.rs = s_a; o.I = M; o.J = K; o.K = N; o.vec = t8_vec(dX, ld_dx, 2);
    const int rc = t8_product<T8_BF16>(qa, qWt, K, o, status, st);
    if (rc != DET_OK) return rc;
  }
  if (dW) {
    launch_after(k_t8_transpose, dim3((K + 127) / 128, (M + 127) / 128), 128, 0, st, qX, M, K, qxt);
    T8Out o = {};
    o.out = dW; o.ld = K; o.rs = s_g; o.I = N; o.J = K; o.K = M; o.vec = t8_vec(dW, K, 4);
    const int rc = t8_product<T8_F32>(qgt, qxt, K, o, status, st);
    if (rc != DET_OK) return rc;
  }
  DET_CHECK_LAUNCH();
  return DET_OK;
}
}  // namespace det

using namespace det;

extern "C" int det_tok8_ld(int K) { return K > 0 && K < (1 << 30) ? t8_ld(K) : 0; }

extern "C" int det_tok8_quant(const det_bf16* X, int ld, int M, int K, int8_t* qX, float* s_x, void* stream) {
  if (!X || !qX || !s_x || ld < K) return DET_ERR_ARG;
  const int rc = t8_sizes(M, 1, K);
  if (rc != DET_OK) return rc;
  if (!aligned_to(X, 2) || !aligned16(qX) || !aligned_to(s_x, 4)) return DET_ERR_ALIGN;
  return M ? t8_quant(X, ld, M, K, qX, s_x, (cudaStream_t)stream) : DET_OK;
}
extern "C" int det_tok8_transpose(const int8_t* q, int M, int K, int8_t* qT, void* stream) {
  if (!q || !qT) return DET_ERR_ARG;
  const int rc = t8_sizes(M, 1, K);
  if (rc != DET_OK) return rc;
  if ((M + 127) / 128 > 65535) return DET_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(qT)) return DET_ERR_ALIGN;
  if (!M) return DET_OK;
  launch_after(k_t8_transpose, dim3((K + 127) / 128, (M + 127) / 128), 128, 0, (cudaStream_t)stream, q, M, K, qT);
  DET_CHECK_LAUNCH();
  return DET_OK;
}

static int t8_fwd_check(const void* q, const float* s_x, const int8_t* qW, const float* s_w, int M, int N, int K, const void* Y, int ld_y) {
  if (!q || !s_x || !qW || !s_w || !Y || ld_y < N) return DET_ERR_ARG;
  const int rc = t8_sizes(M, N, K);
  if (rc != DET_OK) return rc;
  if (!aligned16(q) || !aligned16(qW) || !aligned_to(s_x, 4) || !aligned_to(s_w, 4) || !aligned_to(Y, 2)) return DET_ERR_ALIGN;
  return DET_OK;
}
extern "C" int det_tok8_linear_fwd_q(const int8_t* qX, const float* s_x, const int8_t* qW, const float* s_w, int M, int N, int K, det_bf16* Y, int ld_y,
                                     void* stream, int* status_dev) {
  const int rc = t8_fwd_check(qX, s_x, qW, s_w, M, N, K, Y, ld_y);
  if (rc != DET_OK || !M) return rc;
  T8Out o = {};
  o.out = Y; o.ld = ld_y; o.rs = s_x; o.cs = s_w; o.I = M; o.J = N; o.K = K; o.vec = t8_vec(Y, ld_y, 2);
  return t8_product<T8_BF16>(qX, qW, N, o, status_dev, (cudaStream_t)stream);
}
extern "C" int det_tok8_linear_fwd(const det_bf16* X, int ld, const int8_t* qW, const float* s_w, int M, int N, int K, det_bf16* Y, int ld_y, int8_t* qX,
                                   float* s_x, void* stream, int* status_dev) {
  if (!X || ld < K) return DET_ERR_ARG;
  int rc = t8_fwd_check(qX, s_x, qW, s_w, M, N, K, Y, ld_y);
  if (rc != DET_OK) return rc;
  if (!aligned_to(X, 2)) return DET_ERR_ALIGN;
  if (!M) return DET_OK;
  rc = t8_quant(X, ld, M, K, qX, s_x, (cudaStream_t)stream);
  return rc != DET_OK ? rc : det_tok8_linear_fwd_q(qX, s_x, qW, s_w, M, N, K, Y, ld_y, stream, status_dev);
}

extern "C" size_t det_tok8_linear_bwd_ws_bytes(int M, int N, int K) { return M > 0 && N > 0 && K > 0 ? t8_ws(M, N, K, false).bytes : 0; }
static int t8_bwd_check(const void* d, const int8_t* qX, const float* s_x, const int8_t* qWt, const float* s_w, int M, int N, int K, const void* dX, int ld_dx,
                        const float* dW, const void* ws, size_t need, size_t ws_bytes) {
  if (!d || !qX || !s_x || !qWt || !s_w || (!dX && !dW) || (dX && ld_dx < K)) return DET_ERR_ARG;
  int rc = t8_sizes(M, N, K);
  if (rc != DET_OK) return rc;
  if (M >= (1 << 17) || N >= (1 << 17)) return DET_ERR_RANGE;          // contracted over as well
  if (!aligned_to(d, 2) || !aligned16(qX) || !aligned16(qWt) || !aligned_to(s_x, 4) || !aligned_to(s_w, 4) || !aligned_to(dX, 2) || !aligned_to(dW, 4))
    return DET_ERR_ALIGN;
  if (M && (!ws || !aligned_to(ws, 256) || ws_bytes < need)) return DET_ERR_WORKSPACE;
  return DET_OK;
}
static int t8_no_rows(float* dW, int N, int K, cudaStream_t st) {      // the gradient of weights that no token met
  if (dW && cudaMemsetAsync(dW, 0, (size_t)N * K * 4, st) != cudaSuccess) { cudaGetLastError(); return DET_ERR_CUDA; }
  return DET_OK;
}
extern "C" int det_tok8_linear_bwd(const det_bf16* dY, int ld_dy, const int8_t* qX, const float* s_x, const int8_t* qWt, const float* s_w, int M, int N,
                                   int K, det_bf16* dX, int ld_dx, float* dW, void* ws, size_t ws_bytes, void* stream, int* status_dev) {
  if (ld_dy < N) return DET_ERR_ARG;
  const int rc = t8_bwd_check(dY, qX, s_x, qWt, s_w, M, N, K, dX, ld_dx, dW, ws, det_tok8_linear_bwd_ws_bytes(M, N, K), ws_bytes);
  if (rc != DET_OK) return rc;
  if (!M) return t8_no_rows(dW, N, K, (cudaStream_t)stream);
  return t8_backward(dY, ld_dy, qX, s_x, qWt, s_w, M, N, K, dX, ld_dx, dW, t8_ws(M, N, K, false), (char*)ws, status_dev, (cudaStream_t)stream);
}

extern "C" int det_tok8_glu_fwd_q(const int8_t* qX, const float* s_x, const int8_t* qW, const float* s_w, int M, int F, int K, det_bf16* h, int ld_h,
                                  det_bf16* gu, int ld_gu, void* stream, int* status_dev) {
  if (F > (1 << 27)) return DET_ERR_SHAPE;
  const int rc = t8_fwd_check(qX, s_x, qW, s_w, M, F, K, h, ld_h);
  if (rc != DET_OK) return rc;
  if (gu && ld_gu < 2 * F) return DET_ERR_ARG;
  if (!aligned_to(gu, 2)) return DET_ERR_ALIGN;
  if (!M) return DET_OK;
  T8Out o = {};
  o.out = h; o.ld = ld_h; o.rs = s_x; o.cs = s_w; o.gu = gu; o.ld_gu = ld_gu; o.I = M; o.J = F; o.K = K; o.vec = t8_vec(h, ld_h, 2);
  o.vec_gu = t8_vec(gu, ld_gu, 2) && F % 8 == 0;
  return t8_product<T8_GLU>(qX, qW, 2 * F, o, status_dev, (cudaStream_t)stream);
}
extern "C" int det_tok8_glu_fwd(const det_bf16* X, int ld, const int8_t* qW, const float* s_w, int M, int F, int K, det_bf16* h, int ld_h, det_bf16* gu,
                                int ld_gu, int8_t* qX, float* s_x, void* stream, int* status_dev) {
  if (!X || ld < K) return DET_ERR_ARG;
  if (F > (1 << 27)) return DET_ERR_SHAPE;
  int rc = t8_fwd_check(qX, s_x, qW, s_w, M, F, K, h, ld_h);
  if (rc != DET_OK) return rc;
  if (gu && ld_gu < 2 * F) return DET_ERR_ARG;
  if (!aligned_to(X, 2) || !aligned_to(gu, 2)) return DET_ERR_ALIGN;
  if (!M) return DET_OK;
  rc = t8_quant(X, ld, M, K, qX, s_x, (cudaStream_t)stream);
  return rc != DET_OK ? rc : det_tok8_glu_fwd_q(qX, s_x, qW, s_w, M, F, K, h, ld_h, gu, ld_gu, stream, status_dev);
}

// dgu as det_swiglu_bwd gives it, any width and stride: a thread a value
__global__ void __launch_bounds__(256) k_t8_dgu(const uint16_t* __restrict__ dh, size_t ld_dh, const uint16_t* __restrict__ gu, size_t ld_gu, int F,
                                                uint16_t* __restrict__ dgu) {
  const int j = blockIdx.x * 256 + threadIdx.x + grid_dep();
  const size_t r = blockIdx.y;
  if (j >= F) return;
  const float d = bf2f(dh[r * ld_dh + j]), g = bf2f(gu[r * ld_gu + j]), u = bf2f(gu[r * ld_gu + F + j]), sg = t8_sigmoid(g);
  dgu[r * 2 * F + j] = f2bf(fmul(fmul(d, u), fmul(sg, fadd(1.0f, fmul(g, fsub(1.0f, sg))))));
  dgu[r * 2 * F + F + j] = f2bf(fmul(d, fmul(g, sg)));
}
extern "C" size_t det_tok8_glu_bwd_ws_bytes(int M, int F, int K) {
  return M > 0 && F > 0 && F <= (1 << 27) && K > 0 ? t8_ws(M, 2 * F, K, true).bytes : 0;
}
extern "C" int det_tok8_glu_bwd(const det_bf16* dh, int ld_dh, const det_bf16* gu, int ld_gu, const int8_t* qX, const float* s_x, const int8_t* qWt,
                                const float* s_w, int M, int F, int K, det_bf16* dX, int ld_dx, float* dW, void* ws, size_t ws_bytes, void* stream,
                                int* status_dev) {
  if (F > (1 << 27)) return DET_ERR_SHAPE;
  if (!gu || ld_dh < F || ld_gu < 2 * F) return DET_ERR_ARG;
  const int rc = t8_bwd_check(dh, qX, s_x, qWt, s_w, M, 2 * F, K, dX, ld_dx, dW, ws, det_tok8_glu_bwd_ws_bytes(M, F, K), ws_bytes);
  if (rc != DET_OK) return rc;
  if (!aligned_to(gu, 2)) return DET_ERR_ALIGN;
  if (!M) return t8_no_rows(dW, 2 * F, K, (cudaStream_t)stream);
  const T8Ws w = t8_ws(M, 2 * F, K, true);
  uint16_t* dgu = (uint16_t*)((char*)ws + w.dgu);
  for (int r = 0; r < M; r += 32768) {
    const int rows = M - r < 32768 ? M - r : 32768;
    launch_after(k_t8_dgu, dim3((F + 255) / 256, rows), 256, 0, (cudaStream_t)stream, dh + (size_t)r * ld_dh, (size_t)ld_dh, gu + (size_t)r * ld_gu,
                 (size_t)ld_gu, F, dgu + (size_t)r * 2 * F);
  }
  DET_CHECK_LAUNCH();
  return t8_backward(dgu, 2 * F, qX, s_x, qWt, s_w, M, 2 * F, K, dX, ld_dx, dW, w, (char*)ws, status_dev, (cudaStream_t)stream);
}
