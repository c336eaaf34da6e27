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
#include "sigmoid.cuh"
#include "../../include/det_test.h"

namespace det {

constexpr int T8_K = 128;                                // bytes (= codes) a stage along the contraction
constexpr size_t T8_FEW_SMEM = 64 * 1024;                // codes of few tokens in a CTA
__host__ __device__ __forceinline__ int t8_ld(int K) { return (K + 15) / 16 * 16; }   // bytes from a row of codes to the next

// ---- codes -------------------------------------------------------------------------------------------------
// The scale of a group from the largest magnitude's bits; one with an infinity or a NaN has the scale NaN and codes 0.
__device__ __forceinline__ float t8_scale(uint32_t amax) {
  return amax >= 0x7f800000u ? __int_as_float(0x7fffffff) : fdiv(__uint_as_float(amax), 127.0f);
}
__device__ __forceinline__ float t8_inverse(float s) { return s > 0.0f ? fdiv(1.0f, s) : 0.0f; }     // 0 for a scale that is 0 or NaN
// rne(v * inv) in the low byte of the result; |v * inv| is at most 127 (1 + 2^-22), so nothing has to be clamped.  dead: the group has the scale NaN.
__device__ __forceinline__ uint32_t t8_code(float v, float inv) { return __float_as_uint(fadd(fmul(v, inv), 12582912.0f)); }
__device__ __forceinline__ uint2 t8_codes8(const float v[8], float inv, bool dead) {
  uint32_t c[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) c[t] = t8_code(v[t], inv);
  return dead ? make_uint2(0u, 0u) : make_uint2(low_bytes(c[0], c[1], c[2], c[3]), low_bytes(c[4], c[5], c[6], c[7]));
}

// Rows of a multiple of 8 columns, 16-byte aligned: WPR warps a row, up to 64 values a lane, which stay in registers as they came, so that a row is read
// once.  Bound by memory: 8192 x 2048 10 us, 0.8 of the copy's rate, 8192 x 8192 37 us.
template <int WPR>
__global__ void __launch_bounds__(256) k_t8_rows(const uint16_t* __restrict__ x, size_t ld, int M, int K, int8_t* __restrict__ q, float* __restrict__ s) {
  grid_dep();
  __shared__ uint32_t part[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = blockIdx.x * (8 / WPR) + warp / WPR, first = ((warp % WPR) * 32 + lane) * 8, ldq = t8_ld(K);
  const bool there = row < M;
  uint4 v[8];
  uint32_t pair = 0;                      // the largest of the lower halves and of the upper ones
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int c = first + k * (WPR * 256);
    v[k] = there && c < K ? __ldg(reinterpret_cast<const uint4*>(x + (size_t)row * ld + c)) : make_uint4(0u, 0u, 0u, 0u);
  }
#pragma unroll
  for (int k = 0; k < 8; ++k)
    pair = __vmaxu2(pair, __vmaxu2(__vmaxu2(v[k].x & 0x7fff7fffu, v[k].y & 0x7fff7fffu), __vmaxu2(v[k].z & 0x7fff7fffu, v[k].w & 0x7fff7fffu)));
  uint32_t m = __reduce_max_sync(0xffffffffu, max(pair << 16, pair & 0xffff0000u));
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
    if (c >= ldq) break;
    float f[8];
    unpack8(v[k], f);                     // zeros behind the row's end
    *reinterpret_cast<uint2*>(q + (size_t)row * ldq + c) = t8_codes8(f, inv, dead);
  }
}
// Any width, stride and address: a CTA a row, an element a thread at a time, up to 2048 of them kept in registers (LONG: read twice); 1531 x 1003 4 us, where a
// warp a row took 6.8; 8192 x 2041 16 us and 8192 x 8191 52, where k_t8_rows takes 8 for 2048 columns and 30 for 8192.
template <bool LONG>
__global__ void __launch_bounds__(256) k_t8_rows_any(const uint16_t* __restrict__ x, size_t ld, int K, int8_t* __restrict__ q, float* __restrict__ s) {
  grid_dep();
  __shared__ uint32_t part[8];
  const int row = blockIdx.x, ldq = t8_ld(K);
  const uint16_t* p = x + (size_t)row * ld;
  uint32_t v[8], m = 0;
  if (LONG) {
#pragma unroll 8
    for (int c = threadIdx.x; c < K; c += 256) m = max(m, (uint32_t)__ldg(p + c) & 0x7fffu);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int c = threadIdx.x + k * 256;
      v[k] = c < K ? __ldg(p + c) : 0u;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) m = max(m, v[k] & 0x7fffu);
  }
  m = __reduce_max_sync(0xffffffffu, m);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) m = max(m, part[w]);
  const float sc = t8_scale(m << 16), inv = t8_inverse(sc);
  const bool dead = m >= 0x7f80u;
  if (threadIdx.x == 0) s[row] = sc;
  int8_t* to = q + (size_t)row * ldq;
  if (LONG) {
#pragma unroll 8
    for (int c = threadIdx.x; c < ldq; c += 256) to[c] = c < K && !dead ? (int8_t)t8_code(bf2f(__ldg(p + c)), inv) : (int8_t)0;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int c = threadIdx.x + k * 256;
      if (c < ldq) to[c] = dead ? (int8_t)0 : (int8_t)t8_code(__uint_as_float(v[k] << 16), inv);
    }
  }
}

// Codes [R, ld(C)] -> [C, ld(R)], through shared memory, whole 128-byte lines on both sides but at the edges.  What lies behind column C of the
// input is zero; so is what is written behind column R.
// fill: the kernel before has nothing to do with it (common.cuh).  zero: words that are set to 0 besides.
__global__ void __launch_bounds__(128) k_t8_transpose(const int8_t* __restrict__ in, int R, int C, int8_t* __restrict__ out, int fill, uint32_t* __restrict__ zero,
                                                      int nzero) {
  __shared__ __align__(16) uint8_t tile[128 * 128];
  if (fill) grid_fill_begin();
  else grid_dep();
  for (int i = (blockIdx.y * gridDim.x + blockIdx.x) * 128 + threadIdx.x; i < nzero; i += gridDim.x * gridDim.y * 128) zero[i] = 0u;
  const int t = threadIdx.x, c0 = blockIdx.x * 128, r0 = blockIdx.y * 128, ldi = t8_ld(C), ldo = t8_ld(R);
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
  if (fill) grid_fill_end();
}

// ---- operands of the backward products ---------------------------------------------------------------------
// The gradient of the product's output, [M, N], with the scales of the channels (A) and of the tokens (G).  It is dY itself, or (GLU) what the activation
// makes of dh [M, F] and the kept gu [M, 2F], N = 2F, rounded to bf16.  The pass over the largest magnitudes stores that one for the pass over the codes:
// worked out again there it would cost 2 bytes a pair less, but both passes are then bound by their instructions (8192 x 8192: 124 + 168 us).
struct T8Grad {
  const uint16_t *d, *gu;
  size_t ld, ld_gu;
  const float *s_x, *s_w;
  uint16_t* dgu;                          // GLU: the gradient, rows ld_dgu apart
  size_t ld_dgu;
  int M, N, W;                            // W: columns of d, N or N / 2
  int vec, by4;                           // rows in whole pieces of sixteen bytes; of eight
  int tile;                               // rows of a tile of the first pass, 16 to 128
};
// Four adjacent values from `at` on, n of them there; FULL: all, in one piece.
template <bool FULL>
__device__ __forceinline__ uint2 t8_load4(const uint16_t* p, size_t at, int n, int by4) {
  if (FULL || (by4 && n >= 4)) return __ldg(reinterpret_cast<const uint2*>(p + at));
  uint32_t w[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) w[t] = t < n ? p[at + t] : 0u;
  return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}
__device__ __forceinline__ float t8_at(const uint2& v, int t) { return t & 1 ? bfhi(t & 2 ? v.y : v.x) : bflo(t & 2 ? v.y : v.x); }

// Largest magnitudes first.  A tile is up to 128 rows of 256 columns (GLU: of either half); a warp has every eighth
// row, a lane eight of its columns.  Of a whole tile the rows come in by asynchronous copies, each lane's into places of its own, T8_AHEAD of them on their way, the
// next tile's first ones with this one's last.  8192 x (2 x 8192) with the activation's gradient 118 us (10 bytes a pair: 5.7 TB/s; 129 in a
// long run), by waits and instructions in turn (issue slots 54 % at 2048 rows); loads into registers four rows at a time took 150.
// The sigmoids are looked up at every size: all of the backward with the table and with the formula 82 and 91 us at 4096 x (2 x 2048) x 1024, 23.2 and
// 25.0 at 512 x (2 x 2048) x 256, 19.0 and 21.0 at 256 x (2 x 1024) x 256, alike at 64 x (2 x 256) x 256, where five launches are what it takes.
constexpr int T8_AHEAD = 4;
// eight columns' values of a row: GLU dh, gate and up, else dY
template <bool GLU>
struct T8Row { uint4 d, e, u; };
// a row's part of the maxima, and (GLU) its gradient stored
template <bool FULL, bool GLU>
__device__ __forceinline__ void t8_max_row(const T8Grad& x, int r, const T8Row<GLU>& w, float sx, int left, uint16_t* to, const float (&sw)[2][8],
                                           uint32_t (&cm)[2][8], uint32_t* __restrict__ rowmax, const float* tab) {
  constexpr int H = GLU ? 2 : 1;
  const bool there = FULL || r < x.M;
  const uint32_t d4[4] = {w.d.x, w.d.y, w.d.z, w.d.w}, e4[4] = {w.e.x, w.e.y, w.e.z, w.e.w}, u4[4] = {w.u.x, w.u.y, w.u.z, w.u.w};
  uint32_t v[2][4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (!GLU) { v[0][k] = d4[k]; continue; }
    float dg[2], du[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float d = t ? bfhi(d4[k]) : bflo(d4[k]), g = t ? bfhi(e4[k]) : bflo(e4[k]), u = t ? bfhi(u4[k]) : bflo(u4[k]), sg = sigmoid_a8<1>(g, tab);
      du[t] = fmul(d, fmul(g, sg));
      dg[t] = fmul(fmul(d, u), fmul(sg, fadd(1.0f, fmul(g, fsub(1.0f, sg)))));
    }
    v[0][k] = bf_pair(dg[0], dg[1]);
    v[1][k] = bf_pair(du[0], du[1]);
  }
  if (GLU && there) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (FULL) {
        *reinterpret_cast<uint4*>(to + h * x.W) = make_uint4(v[h][0], v[h][1], v[h][2], v[h][3]);
      } else {
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (32 * t < left) to[h * x.W + 32 * t] = (uint16_t)(v[h][t >> 1] >> (16 * (t & 1)));
      }
    }
  }
  uint32_t rm = 0;
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // no factor is negative, and a NaN's bits are the largest
      const float lo = fabsf(bflo(v[h][k])), hi = fabsf(bfhi(v[h][k]));
      rm = __vimax3_u32(rm, __float_as_uint(fmul(lo, sw[h][2 * k])), __float_as_uint(fmul(hi, sw[h][2 * k + 1])));
      cm[h][2 * k] = max(cm[h][2 * k], __float_as_uint(fmul(lo, sx)));
      cm[h][2 * k + 1] = max(cm[h][2 * k + 1], __float_as_uint(fmul(hi, sx)));
    }
  rm = __reduce_max_sync(0xffffffffu, rm);
  if ((threadIdx.x & 31) == 0 && there) atomicMax(rowmax + r, rm);
}
__device__ __forceinline__ void t8_copy16(uint32_t place, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(place), "l"(src) : "memory");
}
template <bool GLU>
struct T8MaxRoom {                        // of a CTA, in shared memory
  static constexpr int SLOT = (GLU ? 3 : 1) * 256 * 16, TABLE = GLU ? 2 * SG_TAB * 4 : 0;
  static constexpr size_t BYTES = TABLE + 8 * 256 * 4 + T8_AHEAD * SLOT;
};
__device__ __forceinline__ uint4 t8_load8_any(const uint16_t* p, int n) {
  uint32_t w[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) w[t] = 32 * t < n ? p[32 * t] : 0u;
  return make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
}
template <bool GLU>
__global__ void __launch_bounds__(256, 2) k_t8_grad_max(const __grid_constant__ T8Grad x, uint32_t* __restrict__ rowmax, uint32_t* __restrict__ colmax) {
  typedef T8MaxRoom<GLU> Room;
  constexpr int H = GLU ? 2 : 1;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  float* tab = reinterpret_cast<float*>(smem_raw);
  uint32_t* cols = reinterpret_cast<uint32_t*>(smem_raw + Room::TABLE);   // [8][256]
  const uint8_t* place = smem_raw + Room::TABLE + 8 * 256 * 4 + threadIdx.x * 16;
  const uint32_t place_u = (uint32_t)__cvta_generic_to_shared(place);
  sg_copy_table<GLU ? 1 : 0>(tab);
  grid_dep();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int across = (x.W + 255) / 256, tiles = across * ((x.M + x.tile - 1) / x.tile), rows = x.tile / 8;
  auto whole = [&](int tile) { return x.vec && tile % across * 256 + 256 <= x.W && tile / across * x.tile + x.tile <= x.M; };
  // where the next row to fetch lies, and how many of its tile's rows have been fetched
  const uint16_t *fd = nullptr, *fg = nullptr;
  auto begin = [&](int tile) {
    const size_t r = tile / across * x.tile + warp;
    const int c = tile % across * 256 + lane * 8;
    fd = x.d + r * x.ld + c;
    if (GLU) fg = x.gu + r * x.ld_gu + c;
  };
  auto fetch = [&](int slot) {
    const uint32_t to = place_u + slot * Room::SLOT;
    t8_copy16(to, fd);
    fd += 8 * x.ld;
    if (GLU) {
      t8_copy16(to + 4096, fg);
      t8_copy16(to + 8192, fg + x.W);
      fg += 8 * x.ld_gu;
    }
  };
  bool ahead = false;                                                     // the first rows are on their way
#pragma unroll 1
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    // a lane's eight columns are adjacent in a whole tile, else 32 apart, so that values that are read one by one lie side by side over the lanes
    const bool full = whole(tile);
    const int step = full ? 1 : 32, c = tile % across * 256 + (full ? lane * 8 : lane), r0 = tile / across * x.tile + warp, left = x.W - c;
    float sw[2][8];
    uint32_t cm[2][8];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        sw[h][t] = step * t < left ? fabsf(x.s_w[h * x.W + c + step * t]) : 0.0f;
        cm[h][t] = 0;
      }
    const float sx_all = lane < rows && r0 + lane * 8 < x.M ? fabsf(__ldg(x.s_x + r0 + lane * 8)) : 0.0f;     // row i's with lane i
    uint16_t* to = GLU ? x.dgu + r0 * x.ld_dgu + c : nullptr;
    if (full) {
      const int then = tile + gridDim.x;
      const bool more = then < tiles && whole(then);
      if (!ahead) {
        begin(tile);
#pragma unroll
        for (int i = 0; i < T8_AHEAD; ++i) {
          fetch(i);
          fetch_close();
        }
      }
#pragma unroll 1
      for (int i0 = 0; i0 < rows; i0 += T8_AHEAD) {
        const bool end = i0 + T8_AHEAD == rows;                           // this tile's rows are all on their way
        if (end && more) begin(then);
#pragma unroll
        for (int k = 0; k < T8_AHEAD; ++k) {
          const float sx = __shfl_sync(0xffffffffu, sx_all, i0 + k);
          fetch_wait<T8_AHEAD - 1>();
          const uint8_t* from = place + k * Room::SLOT;
          T8Row<GLU> w;
          w.d = *reinterpret_cast<const uint4*>(from);
          if (GLU) {
            w.e = *reinterpret_cast<const uint4*>(from + 4096);
            w.u = *reinterpret_cast<const uint4*>(from + 8192);
          }
          if (!end || more) fetch(k);
          fetch_close();                                                  // of nothing at the very end, so that the count stays
          t8_max_row<true, GLU>(x, r0 + (i0 + k) * 8, w, sx, left, to, sw, cm, rowmax, tab);
          if (GLU) to += 8 * x.ld_dgu;
        }
      }
      ahead = more;
    } else {
#pragma unroll 1
      for (int i = 0; i < rows; i += 2) {                                 // two rows' values, read one by one, on their way together
        T8Row<GLU> w[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const size_t r = r0 + (i + k) * 8;
          const int n = r < (size_t)x.M ? left : 0;
          w[k].d = t8_load8_any(x.d + r * x.ld + c, n);
          if (GLU) {
            w[k].e = t8_load8_any(x.gu + r * x.ld_gu + c, n);
            w[k].u = t8_load8_any(x.gu + r * x.ld_gu + x.W + c, n);
          }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          t8_max_row<false, GLU>(x, r0 + (i + k) * 8, w[k], __shfl_sync(0xffffffffu, sx_all, i + k), left, to, sw, cm, rowmax, tab);
          if (GLU) to += 8 * x.ld_dgu;
        }
      }
    }
#pragma unroll
    for (int h = 0; h < H; ++h) {
      if (tile != blockIdx.x || h) __syncthreads();                       // the columns before have been read
#pragma unroll
      for (int t = 0; t < 8; ++t) cols[warp * 256 + (full ? lane * 8 : lane) + step * t] = cm[h][t];
      __syncthreads();
      uint32_t m = 0;
#pragma unroll
      for (int w = 0; w < 8; ++w) m = max(m, cols[w * 256 + threadIdx.x]);
      const int j = tile % across * 256 + threadIdx.x;
      if (j < x.W) atomicMax(colmax + h * x.W + j, m);
    }
  }
}
// Then the codes: A as it lies, G transposed.  A tile is 128 rows of 128 columns, in two halves of 64; a thread has 8 rows of 4
// columns of each, four rows on their way together.  A CTA works out the scales and inverses of its rows and columns once, a thread each.  Eight codes of a
// column are a piece of 8 bytes, whose place in its row of the transposed tile is swizzled by the columns' four, so that a warp's pieces meet in no bank.
// 8192 x 16384 111 us (4 bytes a value: 4.8 TB/s; 121 in a long run), issue slots 61 % at 2048 rows; thread by thread the scales alone were a fifth of the instructions (484 us).
struct T8CodeRoom {
  uint8_t out[128 * 128];
  float sx[128], ia[128], sw[128], ig[128];                               // an inverse of -1: the scale is a NaN, the codes are 0
};
template <bool FULL>
__device__ __forceinline__ void t8_code_fetch(const T8Grad& x, int r0, const int (&at)[2], const int (&left)[2], uint2 (&w)[4][2]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (!FULL && r0 + k >= x.M) { w[k][0] = w[k][1] = make_uint2(0u, 0u); continue; }
#pragma unroll
    for (int h = 0; h < 2; ++h) w[k][h] = t8_load4<FULL>(x.d, (r0 + k) * x.ld + at[h], left[h], x.by4);
  }
}
// w: the first four rows, which were fetched before the scales were there
template <bool FULL>
__device__ __forceinline__ void t8_code_rows(const T8Grad& x, uint2 (&w)[4][2], int r0, int at0, const int (&at)[2], const int (&left)[2], const float (&sw)[2][4],
                                             const float (&ig)[2][4], const T8CodeRoom& room, int8_t* __restrict__ qa, uint32_t (&g)[2][2][4]) {
  const int ldn = t8_ld(x.N);
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (half) t8_code_fetch<FULL>(x, r0 + 4, at, left, w);
    const float4 sx4 = *reinterpret_cast<const float4*>(room.sx + at0 + half * 4), ia4 = *reinterpret_cast<const float4*>(room.ia + at0 + half * 4);
    const float sx[4] = {sx4.x, sx4.y, sx4.z, sx4.w}, ia[4] = {ia4.x, ia4.y, ia4.z, ia4.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int r = r0 + half * 4 + k;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t a[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float y = t8_at(w[k][h], t);
          const uint32_t code = t8_code(fmul(y, sx[k]), ig[h][t]);
          a[t] = t8_code(fmul(y, sw[h][t]), ia[k]);
          g[h][half][t] = k == 0 ? code : __byte_perm(g[h][half][t], code, k == 1 ? 0x3240 : k == 2 ? 0x3410 : 0x4210);
        }
        if (!FULL && r >= x.M) continue;
        const uint32_t q = ia[k] < 0.0f ? 0u : low_bytes(a[0], a[1], a[2], a[3]);
        int8_t* row = qa + (size_t)r * ldn;
        if (FULL || at[h] < ldn) *reinterpret_cast<uint32_t*>(row + at[h]) = q;     // behind the row's end zeros
      }
    }
  }
}
__global__ void __launch_bounds__(256, 3) k_t8_grad_codes(const __grid_constant__ T8Grad x, const uint32_t* __restrict__ rowmax,
                                                          const uint32_t* __restrict__ colmax, float* __restrict__ s_a, float* __restrict__ s_g,
                                                          int8_t* __restrict__ qa, int8_t* __restrict__ qgt) {
  grid_dep();
  __shared__ __align__(16) T8CodeRoom room;
  // eight tiles of rows under one another, then the next columns: what runs at a time reads long pieces of rows and writes long pieces of columns
  const int across = (x.N + 127) / 128, down = (x.M + 127) / 128, panel = blockIdx.x / (8 * across), in = blockIdx.x - panel * 8 * across;
  const int high = min(8, down - panel * 8), c0 = in / high * 128, r0 = (panel * 8 + in % high) * 128;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, ldm = t8_ld(x.M);
  const int at[2] = {c0 + tx * 4, c0 + tx * 4 + 64}, left[2] = {x.N - at[0], x.N - at[1]};
  const bool full = x.by4 && c0 + 128 <= x.N && r0 + 128 <= x.M;
  uint2 w[4][2];
  if (full) t8_code_fetch<true>(x, r0 + ty * 8, at, left, w);
  else t8_code_fetch<false>(x, r0 + ty * 8, at, left, w);
  {
    const int k = threadIdx.x & 127;
    const bool row = threadIdx.x < 128, there = row ? r0 + k < x.M : c0 + k < x.N;
    const uint32_t m = !there ? 0u : row ? rowmax[r0 + k] : colmax[c0 + k];
    const float factor = !there ? 0.0f : row ? x.s_x[r0 + k] : x.s_w[c0 + k], s = t8_scale(m), inv = m >= 0x7f800000u ? -1.0f : t8_inverse(s);
    (row ? room.sx : room.sw)[k] = factor;
    (row ? room.ia : room.ig)[k] = inv;
    if (there && row && c0 == 0) s_a[r0 + k] = s;
    if (there && !row && r0 == 0) s_g[c0 + k] = s;
  }
  __syncthreads();
  float sw[2][4], ig[2][4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float4 a = *reinterpret_cast<const float4*>(room.sw + h * 64 + tx * 4), b = *reinterpret_cast<const float4*>(room.ig + h * 64 + tx * 4);
    sw[h][0] = a.x; sw[h][1] = a.y; sw[h][2] = a.z; sw[h][3] = a.w;
    ig[h][0] = b.x; ig[h][1] = b.y; ig[h][2] = b.z; ig[h][3] = b.w;
  }
  uint32_t g[2][2][4];                                                    // [half of the columns][four rows][column], a byte a row
  if (full) t8_code_rows<true>(x, w, r0 + ty * 8, ty * 8, at, left, sw, ig, room, qa, g);
  else t8_code_rows<false>(x, w, r0 + ty * 8, ty * 8, at, left, sw, ig, room, qa, g);
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const bool dead = ig[h][t] < 0.0f;
      *reinterpret_cast<uint2*>(room.out + (h * 64 + tx * 4 + t) * 128 + ((ty ^ tx) << 3)) = make_uint2(dead ? 0u : g[h][0][t], dead ? 0u : g[h][1][t]);
    }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k = i * 32 + (threadIdx.x >> 3), ch = threadIdx.x & 7, f = (k >> 2) & 15;
    uint4 w = *reinterpret_cast<const uint4*>(room.out + k * 128 + (((2 * ch) ^ (f & 14)) << 3));
    if (f & 1) w = make_uint4(w.z, w.w, w.x, w.y);
    if (c0 + k < x.N && r0 + ch * 16 < ldm) *reinterpret_cast<uint4*>(qgt + (size_t)(c0 + k) * ldm + r0 + ch * 16) = w;
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
    uint8_t* to = base + lane * ES;
#pragma unroll 2
    for (int r0 = 0; r0 < 32; r0 += 8) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int r = r0 + k;
        const uint8_t* p = stage + r * (NW * 16) + ((piece ^ ((r >> SH) & (NW - 1))) << 4) + at;
        if (r < rows) {
          if (ES == 2) *reinterpret_cast<uint16_t*>(to) = *reinterpret_cast<const uint16_t*>(p);
          else *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(p);
        }
        to += pitch;
      }
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
__device__ __forceinline__ uint32_t t8_glu2(uint32_t g, uint32_t u, const float* tab) {
  const float2 sg = make_float2(sigmoid_a8<1>(bflo(g), tab), sigmoid_a8<1>(bfhi(g), tab));
  const float2 h = mul2(mul2(make_float2(bflo(g), bfhi(g)), sg), make_float2(bflo(u), bfhi(u)));
  return bf_pair(h.x, h.y);
}
// The scales that a warp needs for a tile: its rows' a lane, its columns' in steps of 32.  They are fetched while the tile before is worked on.
template <int EPI, int CW>
struct T8Scales {
  float row, col[EPI == T8_F32 ? 1 : CW / 32], up[EPI == T8_GLU ? CW / 32 : 1];
  __device__ __forceinline__ void fetch(const T8Out& o, int row0, int j0) {
    const int lane = threadIdx.x & 31;
    row = row0 + lane < o.I ? __ldg(o.rs + row0 + lane) : 0.0f;
    if (EPI == T8_F32) return;
#pragma unroll
    for (int c = 0; c < CW / 32; ++c) {
      const int j = j0 + c * 32 + lane;
      col[c] = j < o.J && o.cs ? __ldg(o.cs + j) : 0.0f;
      if (EPI == T8_GLU) up[c] = j < o.J ? __ldg(o.cs + o.J + j) : 0.0f;
    }
  }
};
// Columns j0 .. j0 + CW of the warp's 32 rows (row0 the first); GLU: the ups' accumulators lie UP columns behind the gates'.  stage: the
// warp's own staging tile in shared memory, with room for the columns' scales behind it.  read_all: called once, when the last accumulator is in registers.
template <int EPI, int CW, int UP, class F>
__device__ __forceinline__ void t8_epilogue(const T8Out& o, const T8Scales<EPI, CW>& sc, uint32_t taddr, int row0, int j0, uint8_t* stage, const float* tab,
                                            F read_all) {
  float* cs = reinterpret_cast<float*>(stage + 2048);
  const int lane = threadIdx.x & 31, rows = o.I - row0;
  if (rows <= 0 || o.J <= j0) { read_all(); return; }
#pragma unroll
  for (int c = 0; c < CW; c += 32) {
    const int j = j0 + c, cols = o.J - j;
    if (c && cols <= 0) break;
    const bool last = c + 32 == CW || cols <= 32;
    uint32_t r[32];
    if (EPI == T8_F32) {
      tmem_ld32(taddr + (uint32_t)c, r);
      if (last) read_all();
      uint4 w[8];
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float2 f = mul2(make_float2(__int2float_rn((int)r[2 * v]), __int2float_rn((int)r[2 * v + 1])), same2(sc.row));
        reinterpret_cast<float2*>(w)[v] = f;
      }
      t8_store<8, 4>(stage, reinterpret_cast<uint8_t*>(reinterpret_cast<float*>(o.out) + row0 * o.ld + j), o.ld * 4, rows, cols, o.vec, w);
      continue;
    }
    tmem_ld32_nowait(taddr + (uint32_t)c, r);
    uint32_t r2[32];
    if (EPI == T8_GLU) tmem_ld32_nowait(taddr + (uint32_t)(UP + c), r2);
    if (o.cs) {
      __syncwarp();
      cs[lane] = sc.col[c / 32];
      if (EPI == T8_GLU) cs[32 + lane] = sc.up[c / 32];
      __syncwarp();
    }
    tmem_wait_ld();
    if (last) read_all();
    uint4 g[4];
    t8_scaled(r, sc.row, cs, o.cs != nullptr, g);
    if (EPI == T8_BF16) {
      t8_store<4, 2>(stage, reinterpret_cast<uint8_t*>(reinterpret_cast<uint16_t*>(o.out) + row0 * o.ld + j), o.ld * 2, rows, cols, o.vec, g);
      continue;
    }
    uint4 u[4];
    t8_scaled(r2, sc.row, cs + 32, true, u);
    if (o.gu) {
      uint8_t* p = reinterpret_cast<uint8_t*>(o.gu + row0 * o.ld_gu + j);
      t8_store<4, 2>(stage, p, o.ld_gu * 2, rows, cols, o.vec_gu, g);
      t8_store<4, 2>(stage, p + (size_t)o.J * 2, o.ld_gu * 2, rows, cols, o.vec_gu, u);
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      uint32_t* gp = reinterpret_cast<uint32_t*>(g) + v;
      *gp = t8_glu2(*gp, reinterpret_cast<const uint32_t*>(u)[v], tab);
    }
    t8_store<4, 2>(stage, reinterpret_cast<uint8_t*>(reinterpret_cast<uint16_t*>(o.out) + row0 * o.ld + j), o.ld * 2, rows, cols, o.vec, g);
  }
}

// Tiles of 128 x BN by one CTA, or of 256 x 256 by the two of a cluster (PAIR; each has 128 rows and stages half of the columns' operand).  The
// columns of a GLU tile are BN / 2 gates and the ups that belong to them.  Roles, ring and waits as in igemm.cu.  8192 x 6144 x 2048 75 us
// (2.8 POP/s) in a short run and 86 in a long one, 8192 x 8192 x 2048 99 and 113, 8192 x 2048 x 16384 180 and 206, the gated block 8192 x (2 x 8192) x 2048 with
// three outputs 224 (2.5) and 253: a long run draws 985 W, the power limit, and the clock falls from 1965 MHz to 1500 to 1650.  In a launch of its own over 2048
// rows the tensor pipe is 65 % active, 76 % with a contraction of 16384 and 57 % in the gated block: few rounds of tiles, the last one part full.
template <bool PAIR, int BN, int EPI>
struct T8Tile {
  static constexpr int BM = PAIR ? 256 : 128, BROWS = PAIR ? BN / 2 : BN;         // BROWS: rows of the columns' operand that a CTA stages
  static constexpr int STAGE_A = 128 * T8_K, STAGE_B = BROWS * T8_K, STAGE = STAGE_A + STAGE_B;
  static constexpr int STAGES = (PAIR || BN == 128 ? 6 : 8) - (EPI == T8_F32 ? 0 : 1), EW = BN == 64 ? 4 : 8;    // one less where the sigmoids, or CTAs of the transposition beside, want the room
  static constexpr int WARP = EPI == T8_F32 ? 4096 : 2048 + 256;                    // staging tile of a warp, and the scales of its columns
  static constexpr int THREADS = 64 + 32 * EW, TCOLS = 2 * BN;
  static constexpr size_t SMEM = (size_t)STAGES * STAGE + EW * WARP + (EPI == T8_GLU ? 2 * SG_TAB * 4 : 0) + 1024;
};
// An accumulator is free again, on the barrier of the pair's leader.  What this orders is tensor memory's (tcgen05.wait::ld and the fence before it), no
// other memory: with release semantics it would wait for the tile's stores as well.
__device__ __forceinline__ void t8_arrive_leader(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
template <bool PAIR, int BN, int EPI>
__global__ void __launch_bounds__(T8Tile<PAIR, BN, EPI>::THREADS, 1)
    k_t8_gemm(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ T8Out o, int* status, int fill) {
  typedef T8Tile<PAIR, BN, EPI> T;
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
  if (fill) grid_fill_begin();           // nothing of the kernel before is needed (common.cuh)
  else grid_dep();

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
    uint8_t* stage = smem + STAGES * T::STAGE + (warp - 2) * T::WARP;
    float* tab = reinterpret_cast<float*>(smem + STAGES * T::STAGE + EW * T::WARP);
    if (EPI == T8_GLU) {                                 // while the first tile's operands are on their way
      sg_fill_table<1>(tab, threadIdx.x - 64, EW * 32);
      asm volatile("bar.sync 1, %0;" ::"n"(EW * 32) : "memory");
    }
    const uint32_t free0 = PAIR ? mapa_u32(smem_u32(&bar_tempty[0]), 0) : 0, free1 = PAIR ? mapa_u32(smem_u32(&bar_tempty[1]), 0) : 0;
    int it = 0, i0 = 0, j0 = 0;
    T8Scales<EPI, CW> next = {};
    if (unit < tiles) {
      origin(unit, i0, j0);
      next.fetch(o, i0 + (int)rank * 128 + q * 32, j0 + part * CW);
    }
    for (int tile = unit; tile < tiles; tile += units, ++it) {
      const int acc = it & 1, row0 = i0 + (int)rank * 128 + q * 32, col0 = j0 + part * CW;
      const T8Scales<EPI, CW> now = next;
      if (tile + units < tiles) {
        origin(tile + units, i0, j0);
        next.fetch(o, i0 + (int)rank * 128 + q * 32, j0 + part * CW);
      }
      mbar_wait(&bar_tfull[acc], (uint32_t)(it >> 1) & 1u, abort_flag, status);      // passed over when it ran out: the lanes stay together
      tc_fence_after();
      t8_epilogue<EPI, CW, BN / 2>(o, now, tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * BN + part * CW), row0, col0, stage, tab, [&] {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR) t8_arrive_leader(acc ? free1 : free0);
          else mbar_arrive(&bar_tempty[acc]);
        }
      });
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
  if (fill) grid_fill_end();
}

// ---- few tokens ----------------------------------------------------------------------------------------------
// Up to eight tokens: the weights are read once, a warp R channels (GLU: R / 2 gates and their ups) at a time in pieces of 16 bytes a lane, against the
// tokens' codes in shared memory.  A CTA makes the codes itself (QUANT) or fetches them: made by a launch of its own they cost more than all of this for one
// token.  Bound by memory, or by the latency of making the codes where the weights are small: 1 x 2048 x 2048 3.5 us, gates and ups of one token 2 x 8192 x 2048
// 6.2 (5.4 TB/s); with a launch for the codes and tiles of the tensor cores 15 and 22.
struct T8Few {
  const uint16_t* x;     // QUANT: the tokens, rows ld apart; their codes and scales go to q and s
  size_t ld;
  int8_t* q;
  float* s;
  const int8_t* w;
  T8Out o;
};
template <int MT, int R, bool GLU, bool QUANT>
__global__ void __launch_bounds__(256, MT <= 2 ? 4 : 2) k_t8_few(const __grid_constant__ T8Few f) {
  extern __shared__ __align__(16) uint8_t smem_raw[];                     // the tokens' codes
  __shared__ float s_x[MT];
  __shared__ uint32_t part[MT][8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, K = f.o.K, M = f.o.I, ldk = t8_ld(K), pieces = ldk / 16;
  constexpr int PITCH = QUANT ? 2 : 1;                                    // of a token's codes, in rows of codes
  constexpr int OUT = GLU ? R / 2 : R;                                    // channels of the output a warp has at a time
  constexpr int U = R >= 4 ? 2 : 4;                                       // pieces of a row on their way together
  const int J = f.o.J, tasks = (J + OUT - 1) / OUT;
  auto row = [&](int task, int r) {                                       // r-th of a task's rows of the weights
    const int j = min(task * OUT + (GLU ? r >> 1 : r), J - 1) + (GLU && (r & 1) ? J : 0);
    return reinterpret_cast<const uint4*>(f.w + (size_t)j * ldk);
  };
  auto fetch = [&](uint4 (&w)[U][R], const uint4* const (&rows)[R], int p0) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < R; ++r) w[u][r] = p0 + 32 * u < pieces ? __ldg(rows[r] + p0 + 32 * u) : make_uint4(0u, 0u, 0u, 0u);
  };
  grid_dep();
  // the first weights are on their way while the codes are made
  int task = blockIdx.x * 8 + warp;
  const uint4* rows[R];
  uint4 w[U][R];
#pragma unroll
  for (int r = 0; r < R; ++r) rows[r] = row(min(task, tasks - 1), r);
  fetch(w, rows, lane);
  if (QUANT) {
    uint32_t m[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      m[t] = 0;
      if (t < M)
        for (int c = threadIdx.x; c < K; c += 256) {
          const uint32_t u = f.x[t * f.ld + c];
          m[t] = max(m[t], u << 16 & 0x7fffffffu);
          reinterpret_cast<uint16_t*>(smem_raw)[t * ldk + c] = (uint16_t)u;   // the values for now, twice the codes' room
        }
      m[t] = __reduce_max_sync(0xffffffffu, m[t]);
      if (lane == 0) part[t][warp] = m[t];
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      m[t] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m[t] = max(m[t], part[t][i]);
      const float sc = t8_scale(m[t]), inv = t8_inverse(sc);
      if (threadIdx.x == 0) {
        s_x[t] = sc;
        if (blockIdx.x == 0 && t < M) f.s[t] = sc;
      }
      // sixteen values into a piece of codes: a token's codes lie where its values lay, so all of them are read before any is written
      const uint16_t* v = reinterpret_cast<const uint16_t*>(smem_raw) + t * ldk;
      for (int p0 = 0; p0 < pieces; p0 += 256) {
        const int p = p0 + threadIdx.x;
        uint32_t b[4] = {0, 0, 0, 0};
        if (p < pieces && m[t] < 0x7f800000u) {
#pragma unroll
          for (int k = 0; k < 16; ++k)
            if (p * 16 + k < K) b[k >> 2] |= (t8_code(bf2f(v[p * 16 + k]), inv) & 255u) << (8 * (k & 3));
        }
        __syncthreads();
        if (p < pieces) {
          const uint4 c = make_uint4(b[0], b[1], b[2], b[3]);
          *reinterpret_cast<uint4*>(smem_raw + (size_t)t * ldk * 2 + p * 16) = c;
          if (blockIdx.x == 0 && t < M) *reinterpret_cast<uint4*>(f.q + (size_t)t * ldk + p * 16) = c;
        }
      }
    }
  } else {
    for (int i = threadIdx.x; i < MT * pieces; i += 256) {
      const int t = i / pieces;
      reinterpret_cast<uint4*>(smem_raw)[i] = t < M ? reinterpret_cast<const uint4*>(f.q)[i] : make_uint4(0u, 0u, 0u, 0u);
    }
    if (threadIdx.x < MT) s_x[threadIdx.x] = threadIdx.x < M ? f.s[threadIdx.x] : 0.0f;
  }
  __syncthreads();
#pragma unroll 1
  for (bool first = true; task < tasks; task += gridDim.x * 8, first = false) {
    const int j0 = task * OUT;
    if (!first) {
#pragma unroll
      for (int r = 0; r < R; ++r) rows[r] = row(task, r);
    }
    int acc[R][MT];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int t = 0; t < MT; ++t) acc[r][t] = 0;
    for (int p0 = lane; p0 < pieces; p0 += 32 * U) {
      if (!first || p0 >= 32) fetch(w, rows, p0);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (p0 + 32 * u >= pieces) break;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const uint4 x = *reinterpret_cast<const uint4*>(smem_raw + (size_t)t * PITCH * ldk + (p0 + 32 * u) * 16);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            int a = acc[r][t];
            a = __dp4a((int)w[u][r].x, (int)x.x, a);
            a = __dp4a((int)w[u][r].y, (int)x.y, a);
            a = __dp4a((int)w[u][r].z, (int)x.z, a);
            acc[r][t] = __dp4a((int)w[u][r].w, (int)x.w, a);
          }
        }
      }
    }
    // lane k takes output k / MT of the warp's and token k % MT
    int mine = 0, up = 0;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const int sum = __reduce_add_sync(0xffffffffu, acc[r][t]);
        if (lane == (GLU ? r >> 1 : r) * MT + t) {
          if (GLU && (r & 1)) up = sum;
          else mine = sum;
        }
      }
    const int j = j0 + lane / MT, t = lane % MT;
    if (lane < OUT * MT && j < J && t < M) {
      const float sx = s_x[t];
      const uint16_t y = f2bf(fmul(__int2float_rn(mine), fmul(sx, f.o.cs[j])));
      uint16_t* out = reinterpret_cast<uint16_t*>(f.o.out) + t * f.o.ld + j;
      if (!GLU) {
        *out = y;
      } else {
        const uint16_t z = f2bf(fmul(__int2float_rn(up), fmul(sx, f.o.cs[J + j])));
        if (f.o.gu) {
          f.o.gu[t * f.o.ld_gu + j] = y;
          f.o.gu[t * f.o.ld_gu + J + j] = z;
        }
        *out = f2bf(fmul(fmul(bf2f(y), sigmoid_a8<0>(bf2f(y), nullptr)), bf2f(z)));
      }
    }
  }
}
template <int MT, int R, bool GLU, bool QUANT>
static int t8_few_launch(const T8Few& f, int sms, cudaStream_t st) {
  const size_t smem = (size_t)MT * t8_ld(f.o.K) * (QUANT ? 2 : 1);
  static DevOnce once = {};
  if (smem > 40 * 1024 && dev_ensure_smem(once, (const void*)k_t8_few<MT, R, GLU, QUANT>, T8_FEW_SMEM) != DET_OK) return DET_ERR_CUDA;
  const long long ctas = ((long long)(f.o.J + (GLU ? R / 2 : R) - 1) / (GLU ? R / 2 : R) + 7) / 8;
  const int most = (MT <= 2 ? 4 : 2) * sms;
  launch_after(k_t8_few<MT, R, GLU, QUANT>, (unsigned)(ctas < most ? ctas : most), 256, smem, st, f);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
// Four channels at a time where there are enough of them for every warp, else fewer: more warps, each with less to wait for
template <int MT, bool GLU, bool QUANT>
static int t8_few_rows(const T8Few& f, int sms, cudaStream_t st) {
  const long long rows = (long long)f.o.J * (GLU ? 2 : 1), warps = 16LL * sms;
  if (rows >= 4 * warps) return t8_few_launch<MT, 4, GLU, QUANT>(f, sms, st);
  if (GLU || rows >= 2 * warps) return t8_few_launch<MT, 2, GLU, QUANT>(f, sms, st);
  return t8_few_launch<MT, GLU ? 2 : 1, GLU, QUANT>(f, sms, st);
}
// Whether a call is for this: few tokens, whose codes fit into a CTA's share of shared memory; more than four only where the tensor cores' tiles would not
// have the SMs to themselves (8 tokens, 16384 channels of 2048: 12.6 here, 13.1 there, gates and ups 11.5 and 14.8; 2048 channels of 8192 12.0 and 8.0).
// quant: the codes are made here too.
static bool t8_few_fits(int M, int rows, int K, bool quant) {
  return (M <= (quant ? 2 : 4) || (!quant && M <= 8 && rows >= 12288)) && (size_t)(M > 4 ? 8 : M > 2 ? 4 : M) * t8_ld(K) * (quant ? 2 : 1) <= T8_FEW_SMEM;
}
template <bool GLU, bool QUANT>
static int t8_few(const T8Few& f, cudaStream_t st) {
  const int sms = dev_sm_count();
  if (sms <= 0) return DET_ERR_CUDA;
  if (f.o.I == 1) return t8_few_rows<1, GLU, QUANT>(f, sms, st);
  if (f.o.I == 2) return t8_few_rows<2, GLU, QUANT>(f, sms, st);
  if constexpr (!QUANT) return f.o.I <= 4 ? t8_few_rows<4, GLU, false>(f, sms, st) : t8_few_rows<8, GLU, false>(f, sms, st);
  return DET_ERR_SHAPE;
}

template <bool PAIR, int BN, int EPI>
static int t8_launch(const int8_t* A, const int8_t* B, int rows_b, const T8Out& o, int fill, int* status, cudaStream_t st) {
  typedef T8Tile<PAIR, BN, EPI> T;
  constexpr int BH = EPI == T8_GLU ? BN / 2 : BN;
  static DevOnce once = {};
  if (dev_ensure_smem(once, (const void*)k_t8_gemm<PAIR, BN, EPI>, T::SMEM, EPI == T8_BF16) != DET_OK) return DET_ERR_CUDA;
  const int sms = dev_sm_count();
  if (sms < 2) return DET_ERR_CUDA;
  CUtensorMap ta, tb;
  if (!make_map_ld(&ta, A, o.I, o.K, t8_ld(o.K), 128) || !make_map_ld(&tb, B, rows_b, o.K, t8_ld(o.K), !PAIR && EPI == T8_GLU ? BN / 2 : T::BROWS))
    return DET_ERR_CUDA;
  const long long tiles = (long long)((o.I + T::BM - 1) / T::BM) * ((o.J + BH - 1) / BH);
  const int units = PAIR ? sms / 2 : sms, grid = (int)(tiles < units ? tiles : units) * (PAIR ? 2 : 1);
  launch_after_cluster(k_t8_gemm<PAIR, BN, EPI>, grid, T::THREADS, T::SMEM, PAIR ? 2 : 1, st, ta, tb, o, status, fill);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
// ---- few tiles -----------------------------------------------------------------------------------------------
// Where the output has fewer tiles of 128 x 64 than the GPU has SMs and the contraction is long, the CTAs of a cluster share a tile: each sums its part of the
// contraction in its tensor memory, puts the sums where the others can read them, and takes the columns that are its own from all of them.  The sums are
// exact, so nothing shows of how many there were.  BM: rows of the tokens' operand that are staged (the tensor core takes 128, of which the others are never
// looked at).
template <int BM>
struct T8Split {
  static constexpr int STAGE_A = BM * T8_K, STAGE_B = 64 * T8_K, STAGE = STAGE_A + STAGE_B, STAGES = 6;
  static constexpr int PITCH = 68;                                        // ints from a row of sums to the next: eight rows' sixteen bytes meet in no bank
  // the tensor core reads 128 rows from where an operand begins: behind the last stage there has to be room
  static constexpr size_t SMEM = (size_t)STAGES * STAGE + (128 * T8_K - STAGE > 0 ? 128 * T8_K - STAGE : 0) + 1024;
  static_assert((size_t)BM * PITCH * 4 <= (size_t)STAGES * STAGE, "the sums lie where the stages lay");
};
__device__ __forceinline__ uint4 ld_cluster16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
// four adjacent values of a row, `left` of them in it
template <class T>
__device__ __forceinline__ void t8_put4(T* to, int left, int vec, const T (&v)[4]) {
  if (vec && left >= 4) {
    if (sizeof(T) == 2) *reinterpret_cast<uint2*>(to) = make_uint2((uint32_t)v[0] | (uint32_t)v[1] << 16, (uint32_t)v[2] | (uint32_t)v[3] << 16);
    else *reinterpret_cast<float4*>(to) = make_float4(v[0], v[1], v[2], v[3]);
    return;
  }
#pragma unroll
  for (int t = 0; t < 4; ++t)
    if (t < left) to[t] = v[t];
}
template <int BM, int EPI>
__global__ void __launch_bounds__(192) k_t8_split(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                                                  const __grid_constant__ T8Out o, int parts, int* status, int fill) {
  typedef T8Split<BM> T;
  constexpr int BH = EPI == T8_GLU ? 32 : 64;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ __align__(8) uint64_t bar_full[T::STAGES], bar_empty[T::STAGES], bar_done;
  __shared__ uint32_t tmem_base_s;
  __shared__ int abort_s;
  volatile int* abort_flag = &abort_s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();
  if (threadIdx.x == 0) {
    for (int s = 0; s < T::STAGES; ++s) { mbar_init(&bar_full[s], 1); mbar_init(&bar_empty[s], 1); }
    mbar_init(&bar_done, 1);
    abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmA)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmB)) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"(64u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_s;
  if (fill) grid_fill_begin();
  else grid_dep();

  const int tile = blockIdx.x / parts, tiles_i = (o.I + 127) / 128, i0 = tile % tiles_i * 128, j0 = tile / tiles_i * BH;
  const int kblocks = (o.K + T8_K - 1) / T8_K, kb0 = (int)((long long)kblocks * rank / parts), kb1 = (int)((long long)kblocks * (rank + 1) / parts);
  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait(&bar_empty[stage], phase ^ 1u, abort_flag, status)) break;
        uint8_t *sa = smem + stage * T::STAGE, *sb = sa + T::STAGE_A;
        mbar_expect_tx(&bar_full[stage], T::STAGE);
        tma_load_2d(sa, &tmA, kb * T8_K, i0, &bar_full[stage]);
        tma_load_2d(sb, &tmB, kb * T8_K, j0, &bar_full[stage]);
        if (EPI == T8_GLU) tma_load_2d(sb + T::STAGE_B / 2, &tmB, kb * T8_K, o.J + j0, &bar_full[stage]);
        if (++stage == T::STAGES) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(64 >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait(&bar_full[stage], phase, abort_flag, status)) { ok = false; break; }
        tc_fence_after();
        const uint32_t sa = smem_u32(smem + stage * T::STAGE);
        const uint64_t da = make_smem_desc(sa), db = make_smem_desc(sa + T::STAGE_A);
#pragma unroll
        for (int k4 = 0; k4 < T8_K / 32; ++k4) umma_i8(tmem_base, da + (uint64_t)(k4 * 2), db + (uint64_t)(k4 * 2), idesc, (kb > kb0 || k4) ? 1u : 0u);
        umma_commit(&bar_empty[stage]);
        if (++stage == T::STAGES) { stage = 0; phase ^= 1u; }
      }
      if (ok) umma_commit(&bar_done);
    }
  }
  const int q = warp & 3, row = q * 32 + lane, rows = o.I - i0 < BM ? o.I - i0 : BM;
  int* sums = reinterpret_cast<int*>(smem);
  if (warp >= 2) {
    mbar_wait(&bar_done, 0, abort_flag, status);         // passed over when it ran out; all operands have been read when it has not
    tc_fence_after();
    if (q * 32 < rows) {
#pragma unroll
      for (int c = 0; c < 64; c += 32) {
        uint32_t r[32];
        tmem_ld32(tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)c, r);
        if (row < rows) {
#pragma unroll
          for (int v = 0; v < 8; ++v) *reinterpret_cast<uint4*>(sums + row * T::PITCH + c + 4 * v) = make_uint4(r[4 * v], r[4 * v + 1], r[4 * v + 2], r[4 * v + 3]);
        }
      }
    }
    tc_fence_before();
  }
  __syncwarp();
  __syncthreads();
  if (abort_s) {                                         // copies in flight get time to land
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000ll) { }
    __syncthreads();
  }
  cluster_sync_all();
  if (warp >= 2) {
    // this CTA's columns, four of a row a thread and adjacent ones in adjacent threads; parts divides BH / 4
    const int groups = BH / 4 / parts, items = rows * groups;
    for (int i = threadIdx.x - 64; i < items; i += 128) {
      const int r = i / groups, c = (rank * groups + i % groups) * 4, j = j0 + c, left = o.J - j;
      if (left <= 0) continue;
      const uint32_t mine = smem_u32(sums + r * T::PITCH + c);
      int a[4] = {0, 0, 0, 0}, b[4] = {0, 0, 0, 0};
      for (int p = 0; p < parts; ++p) {
        const uint32_t there = mapa_u32(mine, (uint32_t)p);
        const uint4 x = ld_cluster16(there);
        a[0] += (int)x.x; a[1] += (int)x.y; a[2] += (int)x.z; a[3] += (int)x.w;
        if (EPI == T8_GLU) {
          const uint4 y = ld_cluster16(there + 32 * 4);
          b[0] += (int)y.x; b[1] += (int)y.y; b[2] += (int)y.z; b[3] += (int)y.w;
        }
      }
      const float rs = __ldg(o.rs + i0 + r);
      float f[4], h[4];
      uint16_t y[4], z[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const bool there = t < left;
        f[t] = fmul(__int2float_rn(a[t]), o.cs ? fmul(rs, there ? __ldg(o.cs + j + t) : 0.0f) : rs);
        y[t] = f2bf(f[t]);
        if (EPI != T8_GLU) continue;
        z[t] = f2bf(fmul(__int2float_rn(b[t]), fmul(rs, there ? __ldg(o.cs + o.J + j + t) : 0.0f)));
        h[t] = fmul(fmul(bf2f(y[t]), sigmoid_a8<0>(bf2f(y[t]), nullptr)), bf2f(z[t]));
      }
      if (EPI == T8_F32) {
        t8_put4(reinterpret_cast<float*>(o.out) + (i0 + r) * o.ld + j, left, o.vec, f);
      } else if (EPI == T8_BF16) {
        t8_put4(reinterpret_cast<uint16_t*>(o.out) + (i0 + r) * o.ld + j, left, o.vec, y);
      } else {
        if (o.gu) {
          uint16_t* g = o.gu + (i0 + r) * o.ld_gu + j;
          t8_put4(g, left, o.vec_gu, y);
          t8_put4(g + o.J, left, o.vec_gu, z);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) y[t] = f2bf(h[t]);
        t8_put4(reinterpret_cast<uint16_t*>(o.out) + (i0 + r) * o.ld + j, left, o.vec, y);
      }
    }
  }
  __syncwarp();
  cluster_sync_all();                                    // nobody leaves while the others read
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(64u) : "memory");
  }
  if (fill) grid_fill_end();
}
template <int BM, int EPI>
static int t8_split_launch(const int8_t* A, const int8_t* B, int rows_b, const T8Out& o, int parts, int fill, int* status, cudaStream_t st) {
  static DevOnce once = {};
  if (dev_ensure_smem(once, (const void*)k_t8_split<BM, EPI>, T8Split<BM>::SMEM) != DET_OK) return DET_ERR_CUDA;
  CUtensorMap ta, tb;
  if (!make_map_ld(&ta, A, o.I, o.K, t8_ld(o.K), BM) || !make_map_ld(&tb, B, rows_b, o.K, t8_ld(o.K), EPI == T8_GLU ? 32 : 64)) return DET_ERR_CUDA;
  const int bh = EPI == T8_GLU ? 32 : 64, tiles = ((o.I + 127) / 128) * ((o.J + bh - 1) / bh);
  launch_after_cluster(k_t8_split<BM, EPI>, tiles * parts, 192, T8Split<BM>::SMEM, parts, st, ta, tb, o, parts, status, fill);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
template <int EPI>
static int t8_split(const int8_t* A, const int8_t* B, int rows_b, const T8Out& o, int parts, int fill, int* status, cudaStream_t st) {
  if (o.I <= 32) return t8_split_launch<32, EPI>(A, B, rows_b, o, parts, fill, status, st);
  return t8_split_launch<128, EPI>(A, B, rows_b, o, parts, fill, status, st);
}

// The tile by whole rounds of tiles over the SMs, each the longer of its multiply loop and its epilogue, once the other of the two and what a launch takes
// (microseconds; steps and turns of igemm.cu).  Tiles that the CTAs of a cluster share: as many CTAs as the SMs have room for, at least two steps of the
// contraction for each; their exchange takes longer the more rows there are.  Measured with every tile and number of CTAs
// over 52 shapes, 18 of them weights' gradients: the rule takes at most 1.05 of the best time but for 24 x 2048 x 2048 (1.14: eight CTAs to a tile where four are
// best), the gated 30 x 1000 x 4000 (1.13, likewise) and the gradient 2048 x 2048 x 512 (1.10: the pair where 128 columns are best).  24 x 2048 x 8192 with 8
// CTAs to a tile 8.5, alone 21.1; 128 x 2048 x 8192 with 4 12.2, alone 21.4; 256 x 2048 x 2048 with 2 11.3, alone 7.7 (64 columns), 8.4 (128), 10.8 (pair);
// 2738 x 520 x 1003 8.5, 6.9, 8.7; 8192 x 2048 x 2048 70, 38, 29; gradients 520 x 264 x 1030 5.7, 7.2, 9.3 and 2048 x 8192 x 8192 274, 136, 97.
struct T8Plan { int pick, parts; long long ctas; };      // pick: pair, 128 or 64 columns; parts > 1: CTAs to a tile
static T8Plan t8_plan(int epi, const T8Out& o, int sms) {
  static const struct { int bn, bi; double step, turn, epi[3]; } C[3] = {
      {256, 256, 0.365, 0.9, {4.2, 6.6, 6.0}}, {128, 128, 0.30, 0.5, {1.7, 3.8, 3.0}}, {64, 128, 0.30, 0.5, {1.2, 1.5, 2.0}}};
  const int steps = (o.K + T8_K - 1) / T8_K;
  T8Plan plan = {0, 1, 0};
  double best = 0.0;
  for (int i = 0; i < 3; ++i) {
    const int bh = epi == T8_GLU ? C[i].bn / 2 : C[i].bn, units = i == 0 ? sms / 2 : sms;
    const double tiles = (double)((o.I + C[i].bi - 1) / C[i].bi) * ((o.J + bh - 1) / bh), rounds = (double)(long long)((tiles + units - 1) / units);
    const double loop = steps * C[i].step, e = C[i].epi[epi], t = 2.0 + rounds * ((loop > e ? loop : e) + C[i].turn) + (loop > e ? e : loop);
    if (i == 0 || t < best) {
      best = t;
      plan.pick = i;
      plan.ctas = (long long)(tiles < units ? tiles : units) * (i == 0 ? 2 : 1);
    }
  }
  const int bh = epi == T8_GLU ? 32 : 64, room = o.I <= 32 ? 2 * sms : sms;
  const long long tiles = (long long)((o.I + 127) / 128) * ((o.J + bh - 1) / bh);
  // clusters of eight large CTAs find their SMs in few places: half of the GPU
  int parts = 1;
  while (parts < 8 && tiles * parts * 2 <= (parts == 4 && o.I > 32 ? room / 2 : room) && steps >= parts * 4) parts *= 2;
  if (parts > 1 && 5.2 + 0.025 * (o.I < 128 ? o.I : 168) + steps * 0.27 / parts < best) {
    plan.parts = parts;
    plan.ctas = tiles * parts;
  }
  return plan;
}
template <int EPI>
static int t8_product(const T8Plan& plan, const int8_t* A, const int8_t* B, int rows_b, const T8Out& o, int fill, int* status, cudaStream_t st) {
  if (plan.parts > 1) return t8_split<EPI>(A, B, rows_b, o, plan.parts, fill, status, st);
  if (plan.pick == 0) return t8_launch<true, 256, EPI>(A, B, rows_b, o, fill, status, st);
  if (plan.pick == 1) return t8_launch<false, 128, EPI>(A, B, rows_b, o, fill, status, st);
  return t8_launch<false, 64, EPI>(A, B, rows_b, o, fill, status, st);
}
template <int EPI>
static int t8_product(const int8_t* A, const int8_t* B, int rows_b, const T8Out& o, int* status, cudaStream_t st) {
  const int sms = dev_sm_count();
  return sms < 2 ? DET_ERR_CUDA : t8_product<EPI>(t8_plan(EPI, o, sms), A, B, rows_b, o, 0, status, st);
}

static int t8_quant(const uint16_t* X, int ld, int M, int K, int8_t* q, float* s, cudaStream_t st) {
  if (K % 8 == 0 && ld % 8 == 0 && aligned16(X) && K <= 16384) {
    if (K <= 2048) launch_after(k_t8_rows<1>, (unsigned)((M + 7) / 8), 256, 0, st, X, (size_t)ld, M, K, q, s);
    else if (K <= 8192) launch_after(k_t8_rows<4>, (unsigned)((M + 1) / 2), 256, 0, st, X, (size_t)ld, M, K, q, s);
    else launch_after(k_t8_rows<8>, (unsigned)M, 256, 0, st, X, (size_t)ld, M, K, q, s);
  } else {
    launch_after(K <= 2048 ? k_t8_rows_any<false> : k_t8_rows_any<true>, (unsigned)M, 256, 0, st, X, (size_t)ld, K, q, s);
  }
  DET_CHECK_LAUNCH();
  return DET_OK;
}
// sizes that every call shares: contractions below 2^17 (int32), rows and columns that tensor maps and tiles can number
static int t8_sizes(long long M, long long N, long long K) {
  if (M < 0 || N <= 0 || K <= 0) return DET_ERR_ARG;
  if (M > (1 << 28) || N > (1 << 28)) return DET_ERR_SHAPE;
  return K >= (1 << 17) ? DET_ERR_RANGE : DET_OK;
}
static int t8_vec(const void* p, size_t ld, int size) { return aligned16(p) && ld * size % 16 == 0; }

// gradient operands into the workspace, then both products
struct T8Ws { size_t qa, qgt, qxt, s_a, s_g, rowmax, colmax, dgu, bytes; };
static size_t t8_ld_dgu(int N) { return ((size_t)N + 7) / 8 * 8; }
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
  w.dgu = take(glu ? (size_t)M * t8_ld_dgu(N) * 2 : 0);
  w.bytes = at;
  return w;
}
struct T8Operands { uint32_t *rowmax, *colmax; float *s_a, *s_g; int8_t *qa, *qgt; };
// Rows of a tile of the pass over the largest magnitudes: the most with which there are still some tiles for every place of a CTA, as it stays and walks over
// them.  Rows without a common alignment, whose loads wait one by one: with too few tiles of 32 for the SMs, 16 (all of the backward with 16 and 32, gated block: 64
// tiles of 32, 500 x 1003, 22.3 and 23.6 us; 192, 1003 x 1369, 33.9 and 33.6; 756, 2000 x 3001, 97.8 and 94.3; linear: 18.7 and 19.9, 26.6 and 25.8, 47.8 and 46.3).
static int t8_tile_rows(int M, int W, int vec, int sms) {
  const long long across = (W + 255) / 256;
  int tile = 128;
  while (tile > 32 && across * ((M + tile - 1) / tile) < 6 * sms) tile /= 2;
  return !vec && across * ((M + 31) / 32) < sms ? 16 : tile;
}
template <bool GLU>
static int t8_largest(T8Grad x, const T8Operands& o, int sms, cudaStream_t st) {
  const size_t smem = T8MaxRoom<GLU>::BYTES;
  static DevOnce once = {};
  if (smem > 48 * 1024 && dev_ensure_smem(once, (const void*)k_t8_grad_max<GLU>, smem) != DET_OK) return DET_ERR_CUDA;
  const long long across = (x.W + 255) / 256;
  x.tile = t8_tile_rows(x.M, x.W, x.vec, sms);
  const long long tiles = across * ((x.M + x.tile - 1) / x.tile), most = (GLU ? 2LL : 3LL) * sms;    // CTAs stay and walk over the tiles
  launch_after(k_t8_grad_max<GLU>, (unsigned)(tiles < most ? tiles : most), 256, smem, st, x, o.rowmax, o.colmax);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
static int t8_backward(const T8Grad& x, const int8_t* qX, const int8_t* qWt, int K, uint16_t* dX, int ld_dx, float* dW, char* ws, int* status,
                       cudaStream_t st) {
  const int M = x.M, N = x.N, sms = dev_sm_count();
  if (sms <= 0) return DET_ERR_CUDA;
  const T8Ws w = t8_ws(M, N, K, x.gu != nullptr);
  int8_t* qxt = (int8_t*)(ws + w.qxt);
  const T8Operands op = {(uint32_t*)(ws + w.rowmax), (uint32_t*)(ws + w.colmax), (float*)(ws + w.s_a), (float*)(ws + w.s_g), (int8_t*)(ws + w.qa), (int8_t*)(ws + w.qgt)};
  T8Out ox = {}, ow = {};
  ox.out = dX; ox.ld = ld_dx; ox.rs = op.s_a; ox.I = M; ox.J = K; ox.K = N; ox.vec = t8_vec(dX, ld_dx, 2);
  ow.out = dW; ow.ld = K; ow.rs = op.s_g; ow.I = N; ow.J = K; ow.K = M; ow.vec = t8_vec(dW, K, 4);
  const T8Plan px = t8_plan(T8_BF16, ox, sms), pw = t8_plan(T8_F32, ow, sms);
  const dim3 tgrid((K + 127) / 128, (M + 127) / 128);
  // Where the first product leaves SMs without a CTA the second comes in beside it, and the transposition is done first, which sets the maxima to 0 as well; else
  // it runs beside the first product, which leaves the memory idle and room on every SM for two CTAs of it (8192 x 2048 x 8192: 248 -> 229 us).
  const bool beside = dX && dW && px.ctas < sms;
  const int words = (int)((w.dgu - w.rowmax) / 4);
  if (beside) launch_after(k_t8_transpose, tgrid, 128, 0, st, qX, M, K, qxt, 0, op.rowmax, words);
  else if (cudaMemsetAsync(op.rowmax, 0, (size_t)words * 4, st) != cudaSuccess) { cudaGetLastError(); return DET_ERR_CUDA; }
  const int rc0 = x.gu ? t8_largest<true>(x, op, sms, st) : t8_largest<false>(x, op, sms, st);
  if (rc0 != DET_OK) return rc0;
  T8Grad y = x;                                                            // as the codes are made of it
  if (x.gu) { y.d = x.dgu; y.ld = x.ld_dgu; y.W = N; y.by4 = 1; }
  launch_after(k_t8_grad_codes, (unsigned)((N + 127) / 128) * ((M + 127) / 128), 256, 0, st, y, op.rowmax, op.colmax, op.s_a, op.s_g, op.qa, op.qgt);
  DET_CHECK_LAUNCH();
  int rc = DET_OK;
  if (dX) rc = t8_product<T8_BF16>(px, op.qa, qWt, K, ox, 0, status, st);
  if (dW && rc == DET_OK) {
    if (!beside) launch_after(k_t8_transpose, tgrid, 128, 0, st, qX, M, K, qxt, dX ? 1 : 0, (uint32_t*)nullptr, 0);
    rc = t8_product<T8_F32>(pw, op.qgt, qxt, K, ow, beside ? 1 : 0, status, st);
  }
  if (rc != DET_OK) return rc;
  DET_CHECK_LAUNCH();
  return DET_OK;
}
}  // namespace det

using namespace det;

extern "C" int det_test_tok8_plan(int epi, int I, int J, int K, int sms, int plan[2]) {
  if (epi < 0 || epi > 2 || I <= 0 || J <= 0 || K <= 0 || sms < 2 || !plan) return DET_ERR_ARG;
  T8Out o = {};
  o.I = I; o.J = J; o.K = K;
  const T8Plan p = t8_plan(epi, o, sms);
  plan[0] = p.pick;
  plan[1] = p.parts;
  return DET_OK;
}
extern "C" int det_test_tok8_tile_rows(int M, int W, int vec, int sms) { return M > 0 && W > 0 && sms > 0 ? t8_tile_rows(M, W, vec, sms) : DET_ERR_ARG; }

extern "C" int det_tok8_ld(int K) { return K > 0 && K < (1 << 30) ? t8_ld(K) : 0; }

extern "C" int det_tok8_quant(const det_bf16* X, int ld, int M, int K, int8_t* qX, float* s_x, void* stream) {
  if ((M && (!X || !qX || !s_x)) || ld < K) return DET_ERR_ARG;
  const int rc = t8_sizes(M, 1, K);
  if (rc != DET_OK) return rc;
  if (!aligned_to(X, 2) || !aligned16(qX) || !aligned_to(s_x, 4)) return DET_ERR_ALIGN;
  return M ? t8_quant(X, ld, M, K, qX, s_x, (cudaStream_t)stream) : DET_OK;
}
extern "C" int det_tok8_transpose(const int8_t* q, int M, int K, int8_t* qT, void* stream) {
  if (M && (!q || !qT)) return DET_ERR_ARG;
  const int rc = t8_sizes(M, 1, K);
  if (rc != DET_OK) return rc;
  if ((M + 127) / 128 > 65535) return DET_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(qT)) return DET_ERR_ALIGN;
  if (!M) return DET_OK;
  launch_after(k_t8_transpose, dim3((K + 127) / 128, (M + 127) / 128), 128, 0, (cudaStream_t)stream, q, M, K, qT, 0, (uint32_t*)nullptr, 0);
  DET_CHECK_LAUNCH();
  return DET_OK;
}

// what has a row for every token may be NULL where there are none, as an empty tensor's address is
static int t8_fwd_check(const void* q, const float* s_x, const int8_t* qW, const float* s_w, int M, int N, int K, const void* Y, int ld_y) {
  if ((M && (!q || !s_x || !Y)) || !qW || !s_w || ld_y < N) return DET_ERR_ARG;
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
  if (t8_few_fits(M, N, K, false))
    return t8_few<false, false>(T8Few{nullptr, 0, const_cast<int8_t*>(qX), const_cast<float*>(s_x), qW, o}, (cudaStream_t)stream);
  return t8_product<T8_BF16>(qX, qW, N, o, status_dev, (cudaStream_t)stream);
}
extern "C" int det_tok8_linear_fwd(const det_bf16* X, int ld, const int8_t* qW, const float* s_w, int M, int N, int K, det_bf16* Y, int ld_y, int8_t* qX,
                                   float* s_x, void* stream, int* status_dev) {
  if ((M && !X) || ld < K) return DET_ERR_ARG;
  int rc = t8_fwd_check(qX, s_x, qW, s_w, M, N, K, Y, ld_y);
  if (rc != DET_OK) return rc;
  if (!aligned_to(X, 2)) return DET_ERR_ALIGN;
  if (!M) return DET_OK;
  if (t8_few_fits(M, N, K, true)) {
    T8Out o = {};
    o.out = Y; o.ld = ld_y; o.cs = s_w; o.I = M; o.J = N; o.K = K;
    return t8_few<false, true>(T8Few{X, (size_t)ld, qX, s_x, qW, o}, (cudaStream_t)stream);
  }
  rc = t8_quant(X, ld, M, K, qX, s_x, (cudaStream_t)stream);
  return rc != DET_OK ? rc : det_tok8_linear_fwd_q(qX, s_x, qW, s_w, M, N, K, Y, ld_y, stream, status_dev);
}

extern "C" size_t det_tok8_linear_bwd_ws_bytes(int M, int N, int K) { return M > 0 && N > 0 && K > 0 ? t8_ws(M, N, K, false).bytes : 0; }
static int t8_bwd_check(const void* d, const int8_t* qX, const float* s_x, const int8_t* qWt, const float* s_w, int M, int N, int K, const void* dX, int ld_dx,
                        const float* dW, const void* ws, size_t need, size_t ws_bytes) {
  if ((M && (!d || !qX || !s_x || (!dX && !dW))) || !qWt || !s_w || (dX && ld_dx < K)) return DET_ERR_ARG;
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
  const T8Grad x = {dY, nullptr, (size_t)ld_dy, 0, s_x, s_w, nullptr, 0, M, N, N, t8_vec(dY, ld_dy, 2), aligned_to(dY, 8) && ld_dy % 4 == 0, 0};
  return t8_backward(x, qX, qWt, K, dX, ld_dx, dW, (char*)ws, status_dev, (cudaStream_t)stream);
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
  if (t8_few_fits(M, 2 * F, K, false))
    return t8_few<true, false>(T8Few{nullptr, 0, const_cast<int8_t*>(qX), const_cast<float*>(s_x), qW, o}, (cudaStream_t)stream);
  return t8_product<T8_GLU>(qX, qW, 2 * F, o, status_dev, (cudaStream_t)stream);
}
extern "C" int det_tok8_glu_fwd(const det_bf16* X, int ld, const int8_t* qW, const float* s_w, int M, int F, int K, det_bf16* h, int ld_h, det_bf16* gu,
                                int ld_gu, int8_t* qX, float* s_x, void* stream, int* status_dev) {
  if ((M && !X) || ld < K) return DET_ERR_ARG;
  if (F > (1 << 27)) return DET_ERR_SHAPE;
  int rc = t8_fwd_check(qX, s_x, qW, s_w, M, F, K, h, ld_h);
  if (rc != DET_OK) return rc;
  if (gu && ld_gu < 2 * F) return DET_ERR_ARG;
  if (!aligned_to(X, 2) || !aligned_to(gu, 2)) return DET_ERR_ALIGN;
  if (!M) return DET_OK;
  if (t8_few_fits(M, 2 * F, K, true)) {
    T8Out o = {};
    o.out = h; o.ld = ld_h; o.cs = s_w; o.gu = gu; o.ld_gu = ld_gu; o.I = M; o.J = F; o.K = K;
    return t8_few<true, true>(T8Few{X, (size_t)ld, qX, s_x, qW, o}, (cudaStream_t)stream);
  }
  rc = t8_quant(X, ld, M, K, qX, s_x, (cudaStream_t)stream);
  return rc != DET_OK ? rc : det_tok8_glu_fwd_q(qX, s_x, qW, s_w, M, F, K, h, ld_h, gu, ld_gu, stream, status_dev);
}

extern "C" size_t det_tok8_glu_bwd_ws_bytes(int M, int F, int K) {
  return M > 0 && F > 0 && F <= (1 << 27) && K > 0 ? t8_ws(M, 2 * F, K, true).bytes : 0;
}
extern "C" int det_tok8_glu_bwd(const det_bf16* dh, int ld_dh, const det_bf16* gu, int ld_gu, const int8_t* qX, const float* s_x, const int8_t* qWt,
                                const float* s_w, int M, int F, int K, det_bf16* dX, int ld_dx, float* dW, void* ws, size_t ws_bytes, void* stream,
                                int* status_dev) {
  if (F > (1 << 27)) return DET_ERR_SHAPE;
  if ((M && !gu) || ld_dh < F || ld_gu < 2 * F) return DET_ERR_ARG;
  const int rc = t8_bwd_check(dh, qX, s_x, qWt, s_w, M, 2 * F, K, dX, ld_dx, dW, ws, det_tok8_glu_bwd_ws_bytes(M, F, K), ws_bytes);
  if (rc != DET_OK) return rc;
  if (!aligned_to(gu, 2)) return DET_ERR_ALIGN;
  if (!M) return t8_no_rows(dW, 2 * F, K, (cudaStream_t)stream);
  const T8Grad x = {dh, gu, (size_t)ld_dh, (size_t)ld_gu, s_x, s_w, (uint16_t*)((char*)ws + t8_ws(M, 2 * F, K, true).dgu), t8_ld_dgu(2 * F), M, 2 * F, F, t8_vec(dh, ld_dh, 2) && t8_vec(gu, ld_gu, 2) && F % 8 == 0, 0, 0};
  return t8_backward(x, qX, qWt, K, dX, ld_dx, dW, (char*)ws, status_dev, (cudaStream_t)stream);
}
