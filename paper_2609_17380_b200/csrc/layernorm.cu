// Layer norm, forward and backward: the norm that subtracts the mean, with gain and shift.
//   forward   mean = sum(x) / D, d = x - mean, rstd = 1 / sqrt(sum(d^2) / D + eps), y = (d * rstd) * gamma + beta
//   backward  xhat = (x - mean) * rstd, w = dy * gamma, c1 = sum(w) / D, c2 = sum(w * xhat) / D,
//             dx = rstd * ((w - c1) - xhat * c2), dgamma = sum over rows of dy * xhat, dbeta = sum over rows of dy
// Every sum is the fixed tree; the variance comes from the differences to the mean, so a mean far from zero costs no digits.  What bounds
// them is memory: a row is read once and stays in registers between the two sums of the forward pass and between sums and output
// of the backward one.
#include <type_traits>

#include <algorithm>

#include "../../include/det_test.h"
#include "common.cuh"
#include "internal.h"
#include "rows.cuh"

namespace det {

// A row is held by WPR warps, a leaf of 256 columns each, eight adjacent columns a lane.  WPR < 8: a CTA of eight warps has 8 / WPR such groups,
// with rows of their own; WPR >= 8: the CTA is one group.  ROWS rows of a group are worked on at a time (backward one where 32 warps hold a row: there
// are 64 registers a thread).
template <int WPR, bool BF, bool VEC>
struct LnShape {
  static constexpr int GROUPS = WPR < 8 ? 8 / WPR : 1, THREADS = 32 * WPR * GROUPS, ROWS = BF && VEC && WPR <= 8 ? 4 : 2, AHEAD = ROWS == 4 ? 2 : 3;
  static constexpr bool AHEAD_ROWS = BF && VEC;          // binary32 rows: a CTA for every two rows and loads in place (25.5 us for 8192 x 2048, 36 ahead)
  static constexpr int CTAS = WPR == 32 ? 1 : (WPR == 16 ? 2 : (ROWS == 4 ? 3 : 4));
};
// The rows that a CTA of the forward pass works on: GROUPS * ROWS of them from `base` on, then, with rows on their way ahead, those `stride` behind.  That
// stays below LN_ROWS and a few thousand.  Without, there is a CTA for every such piece: the next would be `rows` behind, past 2^31 where there are more than 2^30.
template <class S>
struct LnWalk {
  static constexpr int PIECE = S::GROUPS * S::ROWS;
  int base, stride;
  __host__ __device__ __forceinline__ LnWalk(unsigned cta, unsigned ctas) : base((int)cta * PIECE), stride(S::AHEAD_ROWS ? (int)ctas * PIECE : 0) {}
  __host__ __device__ __forceinline__ void next(int rows) { base = S::AHEAD_ROWS ? base + stride : rows; }
};
enum { LN_F32 = 0, LN_BF16 = 1, LN_ACT8 = 2 };   // what x is backward: as dy, or the 8-bit checkpoint (dy bf16)
template <int WPR, int KIND, bool VEC>
struct LnBwd {
  static constexpr int GROUPS = WPR < 8 ? 8 / WPR : 1, THREADS = 32 * WPR * GROUPS, ROWS = WPR == 32 ? 1 : (WPR == 16 || KIND == LN_F32 || !VEC ? 2 : 4);
  static constexpr bool AHEAD_ROWS = VEC && (KIND != LN_F32 || WPR > 8);  // f32: loads in place with a third CTA do better than 128 KiB on their way
  static constexpr int CTAS = WPR > 8 ? 1 : (AHEAD_ROWS || !VEC ? 2 : 3), LEVELS = WPR <= 8 && ROWS == 4 ? 1 : (KIND == LN_F32 && WPR == 32 ? 1 : 2);
};

// The tree over N nodes of which the first `have` exist (at least one); all of them in the usual case, without a test.
template <int N>
__device__ __forceinline__ float node_tree(float (&v)[N], int have) {
  if (have >= N) {
#pragma unroll
    for (int w = 1; w < N; w <<= 1)
#pragma unroll
      for (int j = 0; j < N; j += 2 * w) v[j] = fadd(v[j], v[j + w]);
  } else {
#pragma unroll
    for (int w = 1; w < N; w <<= 1)
#pragma unroll
      for (int j = 0; j < N; j += 2 * w) v[j] = j + w < have ? fadd(v[j], v[j + w]) : v[j];
  }
  return v[0];
}
// The sum of one row is that row, carried up without an addition: flushed like every value that enters or leaves an operation.
__device__ __forceinline__ float ln_flush(float r) { return (__float_as_uint(r) & 0x7f800000u) ? r : __uint_as_float(__float_as_uint(r) & 0x80000000u); }
// Two neighbours of a lane's columns in packed arithmetic, no product fused with a sum (8192 x 2048 backward with the residual stream 37.7 -> 36.3 us, 15.9 -> 13.5 million instructions).
__device__ __forceinline__ float2 two(const float* v) { return make_float2(v[0], v[1]); }
__device__ __forceinline__ void two(float* v, float2 x) { v[0] = x.x; v[1] = x.y; }
template <int N>
__device__ __forceinline__ float2 node_tree2(float2 (&v)[N], int have, float2 one) {
  if (have >= N) {
#pragma unroll
    for (int w = 1; w < N; w <<= 1)
#pragma unroll
      for (int j = 0; j < N; j += 2 * w) v[j] = add2(v[j], v[j + w], one);
  } else {
#pragma unroll
    for (int w = 1; w < N; w <<= 1)
#pragma unroll
      for (int j = 0; j < N; j += 2 * w)
        if (j + w < have) v[j] = add2(v[j], v[j + w], one);
  }
  return v[0];
}
// The row's tree over its WPR leaf sums (in shared memory, one barrier back); a leaf beyond D does not exist.  (The tests for existence in 64 bits and
// in every place cost as many instructions as the rest of the kernels.)
template <int WPR>
__device__ __forceinline__ float row_tree(const float* leaf, int leaves) {
  if (WPR <= 8) {
    float L[WPR];
    if (WPR >= 4) {
#pragma unroll
      for (int j = 0; j < WPR / 4; ++j) {
        const float4 q = reinterpret_cast<const float4*>(leaf)[j];
        L[4 * j] = q.x; L[4 * j + 1] = q.y; L[4 * j + 2] = q.z; L[4 * j + 3] = q.w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < WPR; ++j) L[j] = leaf[j];
    }
    return node_tree<WPR>(L, leaves);
  }
  const int lane = threadIdx.x & 31;
  float v = leaf[lane % WPR];
#pragma unroll
  for (int w = 1; w < WPR; w <<= 1) {
    const float o = __shfl_xor_sync(0xffffffffu, v, w);
    const int right = ((lane % WPR) | w) & ~(w - 1);
    v = right < leaves ? fadd(v, o) : ((lane & w) ? o : v);
  }
  return v;
}
// The trees of N rows (or of two sums of rows) at `leaf`, N a power of two, dealt out over the lanes: lane l has row l mod N.  Every thread needs all of
// them, and each is a dozen instructions, the root and the division behind the second one forty more.
template <int N, int WPR>
__device__ __forceinline__ float dealt_tree(const float* leaf, int leaves) {
  if (WPR <= 8) return row_tree<WPR>(leaf + (threadIdx.x % N) * WPR, leaves);
  float r = 0.0f;                                        // wide rows: the lanes share each tree
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float v = row_tree<WPR>(leaf + j * WPR, leaves);
    if (threadIdx.x % N == j) r = v;
  }
  return r;
}
// The leaves of N sums (a power of two; each lane has its eight terms' sums in v), sum j's to out[j * WPR].  Each step of the butterfly over the lanes
// hands half of the sums to the neighbour while there are several, so that eight sums take 9 exchanges instead of 40; the tree of each is the same.
template <int N, int WPR>
__device__ __forceinline__ void leaf_sums(const float (&v)[N], float* out, int warp, int D, bool full) {
  const int lane = threadIdx.x & 31;
  if (full) {
    float s[N];
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] = v[j];
    int sum = 0;
#pragma unroll
    for (int w = 1, left = N; w < 32; w <<= 1) {
      if (left > 1) {
        left /= 2;
        const bool up = lane & w;
        sum += up ? left : 0;
#pragma unroll
        for (int j = 0; j < N / 2; ++j)
          if (j < left) {
            const float away = up ? s[j] : s[j + left];
            s[j] = fadd(up ? s[j + left] : s[j], __shfl_xor_sync(0xffffffffu, away, w));
          }
      } else {
        s[0] = fadd(s[0], __shfl_xor_sync(0xffffffffu, s[0], w));
      }
    }
    if (lane < N) out[sum * WPR + warp] = s[0];
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float r = warp_tree(v[j], (long long)warp * 256, 8, D);
      if (lane == 0) out[j * WPR + warp] = r;
    }
  }
}
// the sum of a lane's eight terms
template <bool VEC>
__device__ __forceinline__ float lane_sum(const float v[8], int e0, int D) { return VEC || e0 + 8 <= D ? tree8_full(v) : tree8(v, e0, D); }

// of two sets of terms
template <bool VEC>
__device__ __forceinline__ float2 lane_sums(const float a[8], const float b[8], int e0, int D, float2 one) {
  if (!VEC && e0 + 8 > D) return make_float2(tree8(a, e0, D), tree8(b, e0, D));
  float2 s[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) s[j] = make_float2(fadd(a[2 * j], a[2 * j + 1]), fadd(b[2 * j], b[2 * j + 1]));
  return add2(add2(s[0], s[1], one), add2(s[2], s[3], one), one);
}

// Rows are walked over by as many CTAs as the GPU holds; what the next passes need is on its way (AHEAD passes, each thread its own
// columns) while one is worked on: with a CTA for every few rows the loads of 8192 x 2048 stood still at the barriers (21 us, 32 with the residual
// stream).
template <bool BF, int WPR, bool VEC, bool RES>
__global__ void __launch_bounds__(LnShape<WPR, BF, VEC>::THREADS, LnShape<WPR, BF, VEC>::CTAS)
    k_ln_fwd(const void* __restrict__ x, const void* __restrict__ res, const void* __restrict__ gamma, const void* __restrict__ beta,
             int rows, int D, float eps, float invD, void* __restrict__ sum, void* __restrict__ y, float* __restrict__ mean,
             float* __restrict__ rstd, const float* __restrict__ s_q, int8_t* __restrict__ qy, int8_t* __restrict__ q8,
             uint8_t* __restrict__ e8) {
  grid_dep();
  using S = LnShape<WPR, BF, VEC>;
  constexpr int R = S::ROWS, T = S::THREADS, EL = BF ? 2 : 4, BYTES = T * 8 * EL * (RES ? 2 : 1);      // BYTES: a row on its way
  static_assert(S::AHEAD_ROWS || !VEC || !RES, "the residual stream is bf16");
  extern __shared__ __align__(16) char smem[];
  __shared__ __align__(16) float leaf_s[S::GROUPS][2][R][WPR];
  float* room = reinterpret_cast<float*>(smem) + (threadIdx.x >> 5) * 256;            // VEC false: of the warp
  const int grp = (threadIdx.x >> 5) / WPR, warp = (threadIdx.x >> 5) % WPR, lane = threadIdx.x & 31;
  const int e0 = warp * 256 + lane * 8, n = D - e0;
  const bool full = D - warp * 256 >= 256 || D <= warp * 256;     // the warp's leaf is whole, or there is none
  const int leaves = (D + 255) >> 8;
  const float2 one = same2(c_one);
  LnWalk<S> walk(blockIdx.x, gridDim.x);
  auto fetch = [&](int first, int slot) {
    if (S::AHEAD_ROWS) {
      if (first < rows) {
        char* place = smem + slot * R * BYTES;
        size_t at = row_at(first, D, e0) * EL;
#pragma unroll
        for (int a = 0; a < R; ++a, place += BYTES, at += (size_t)D * EL) {
          const bool there = first + a < rows && n > 0;
          row_fetch<8 * EL, T>(place, static_cast<const char*>(x) + at, there);
          if (RES) row_fetch<8 * EL, T>(place + T * 8 * EL, static_cast<const char*>(res) + at, there);
        }
      }
      fetch_close();
    }
  };
  int first = walk.base + grp * R;
#pragma unroll
  for (int k = 0; k < S::AHEAD - 1; ++k) fetch(first + k * walk.stride, k);
  float g[8], b[8];
  const int w0 = warp * 256, left = D - w0;              // the warp's first column, how many are left from there
  auto take = [&](const void* p, float v[8]) {
    if (VEC) {
      load8n<BF>(p, e0, n, v);
    } else {
      uint32_t raw[8];
      load_any<EL>(p, w0, left, raw);
      deal_out(room, raw, v);
    }
  };
  if (gamma) take(gamma, g);
  if (beta) take(beta, b);
  const float inv_q = (BF && VEC && qy) ? fdiv(1.0f, s_q[0]) : 0.0f;
  // all groups of the CTA make the same passes
  for (int slot = 0; walk.base < rows; walk.next(rows), first += walk.stride) {
    float v[R][8];
    if (S::AHEAD_ROWS) {
      const int next = slot == 0 ? S::AHEAD - 1 : slot - 1;
      fetch(first + (S::AHEAD - 1) * walk.stride, next);
      fetch_wait<S::AHEAD - 1>();
    }
    const char* place = smem + slot * R * BYTES;
    slot = slot + 1 == S::AHEAD ? 0 : slot + 1;
    float part[R];
    uint32_t raw[R][8], raw_res[R][8];
    if (!VEC) {
#pragma unroll
      for (int a = 0; a < R; ++a) {
        load_any<EL>(x, row_at(first + a, D, w0), first + a < rows ? left : 0, raw[a]);
        if (RES) load_any<EL>(res, row_at(first + a, D, w0), first + a < rows ? left : 0, raw_res[a]);
      }
    } else if (!S::AHEAD_ROWS) {
#pragma unroll
      for (int a = 0; a < R; ++a) load8n<BF>(x, row_at(first + a, D, e0), first + a < rows ? n : 0, v[a]);
    }
#pragma unroll
    for (int a = 0; a < R; ++a) {
      const int m = first + a < rows ? n : 0;
      const size_t at = row_at(first + a, D, e0);
      if (S::AHEAD_ROWS) row_take<BF, T>(place + a * BYTES, v[a]);
      else if (!VEC) deal_out(room, raw[a], v[a]);
      if (RES) {   // the residual sum in front of the norm: rounded and stored, and the rounded one is what is normalised
        float c[8];
        if (S::AHEAD_ROWS) row_take<BF, T>(place + a * BYTES + T * 8 * EL, c);
        else deal_out(room, raw_res[a], c);
#pragma unroll
        for (int t = 0; t < 8; t += 2) two(v[a] + t, add2(two(v[a] + t), two(c + t), one));
        if (!VEC) store_any<BF>(sum, row_at(first + a, D, w0), first + a < rows ? left : 0, room, v[a]);
        else if (m > 0) store8<BF>(sum, at, v[a]);
        if (BF) {
          round8(v[a]);
        }
      }
      if (BF && VEC && q8) {   // the checkpoint of what is normalised
        const uint32_t field = a8_field(a8_quad_max(a8_amax8(v[a])));
        if (m > 0) {
          *reinterpret_cast<uint2*>(q8 + at) = a8_codes8(v[a], field);
          if ((lane & 3) == 0) e8[(size_t)(first + a) * ((D + A8_GROUP - 1) / A8_GROUP) + e0 / A8_GROUP] = (uint8_t)field;
        }
      }
      part[a] = lane_sum<VEC>(v[a], e0, D);
    }
    leaf_sums<R, WPR>(part, leaf_s[grp][0][0], warp, D, full);
    __syncthreads();
    const float mu_mine = fmul(dealt_tree<R, WPR>(leaf_s[grp][0][0], leaves), invD);
#pragma unroll
    for (int a = 0; a < R; ++a) {
      const float mu = __shfl_sync(0xffffffffu, mu_mine, a);
      float sq[8];
#pragma unroll
      for (int t = 0; t < 8; t += 2) {
        const float2 d = fma2(same2(mu), same2(-1.0f), two(v[a] + t));
        two(v[a] + t, d);
        two(sq + t, mul2(d, d));
      }
      part[a] = lane_sum<VEC>(sq, e0, D);
    }
    leaf_sums<R, WPR>(part, leaf_s[grp][1][0], warp, D, full);
    __syncthreads();
    const float rs_mine = fdiv(1.0f, fsqrt(fadd(fmul(dealt_tree<R, WPR>(leaf_s[grp][1][0], leaves), invD), eps)));
    if (warp == 0 && lane < R && first + lane < rows) {
      mean[first + lane] = mu_mine;
      rstd[first + lane] = rs_mine;
    }
#pragma unroll
    for (int a = 0; a < R; ++a) {
      const float rs = __shfl_sync(0xffffffffu, rs_mine, a);
      if (first + a >= rows) continue;
      float o[8];
#pragma unroll
      for (int t = 0; t < 8; t += 2) two(o + t, mul2(two(v[a] + t), same2(rs)));
      if (gamma) {
#pragma unroll
        for (int t = 0; t < 8; t += 2) two(o + t, mul2(two(o + t), two(g + t)));
      }
      if (beta) {
#pragma unroll
        for (int t = 0; t < 8; t += 2) two(o + t, add2(two(o + t), two(b + t), one));
      }
      const size_t at = row_at(first + a, D, e0);
      if (!VEC) store_any<BF>(y, row_at(first + a, D, w0), left, room, o);
      else if (n > 0) store8<BF>(y, at, o);
      if (BF && VEC && qy && n > 0) {   // the next linear's quantiser, applied to the bf16 values just stored
        round8(o);
        *reinterpret_cast<uint2*>(qy + at) = quant8(o, inv_q);
      }
    }
  }
}

// Backward.  Each group of warps takes `passes` x ROWS adjacent rows (passes a power of two), ROWS at a time; a lane sees the same eight columns of
// all of them, so the trees of dgamma and dbeta over the group's rows run in its own registers, the nodes of finished passes waiting
// in shared memory as the digits of a binary counter do.  The node of a block goes to out_g, out_b [block][D], for k_ln_cols; with one block they are dgamma and dbeta.
// What is fetched ahead of a pass: dy, x (or its codes) and the bypassing gradient of its rows, AHEAD passes of them.  As many CTAs as the GPU holds walk
// over the blocks of rows, so the loads go on across the blocks.
template <int KIND, int WPR, bool VEC>
struct LnFetch {
  static constexpr int AHEAD = WPR == 16 && KIND != LN_F32 ? 3 : 2;
  static constexpr int DY = KIND == LN_F32 ? 32 : 16, X = KIND == LN_F32 ? 32 : (KIND == LN_BF16 ? 16 : 8);
  static constexpr int T = LnBwd<WPR, KIND, VEC>::THREADS, R = LnBwd<WPR, KIND, VEC>::ROWS;
  static constexpr int ROW = T * (DY + X), ROW_RES = ROW + T * DY;                 // bytes of a row
};
template <int KIND, int WPR, bool VEC, bool RES>
__global__ void __launch_bounds__(LnBwd<WPR, KIND, VEC>::THREADS, LnBwd<WPR, KIND, VEC>::CTAS)
    k_ln_bwd(const void* __restrict__ dy, const void* __restrict__ x, const uint8_t* __restrict__ e8, const void* __restrict__ gamma,
             const float* __restrict__ mean, const float* __restrict__ rstd, int rows, int D, float invD, int nb, int passes, const void* res,
             void* dx, float* __restrict__ out_g, float* __restrict__ out_b, float4* __restrict__ upper, int upper_levels) {
  grid_dep();
  constexpr bool BF = KIND != LN_F32, STAGED = LnBwd<WPR, KIND, VEC>::AHEAD_ROWS;
  using S = LnBwd<WPR, KIND, VEC>;
  using Fx = LnFetch<KIND, WPR, VEC>;
  constexpr int R = S::ROWS, T = S::THREADS, BYTES = RES ? Fx::ROW_RES : Fx::ROW, AHEAD = Fx::AHEAD;
  extern __shared__ __align__(16) char smem[];            // the rows on their way, then the waiting nodes [levels][4][T]
  float4* waiting = reinterpret_cast<float4*>(smem + (STAGED ? AHEAD * R * BYTES : 0));
  __shared__ __align__(16) float rooms[VEC ? 1 : T / 32][VEC ? 4 : 256];
  float* room = rooms[VEC ? 0 : threadIdx.x >> 5];
  __shared__ __align__(16) float leaf_s[2][S::GROUPS][R][2][WPR];
  const int grp = (threadIdx.x >> 5) / WPR, warp = (threadIdx.x >> 5) % WPR, lane = threadIdx.x & 31;
  const int e0 = warp * 256 + lane * 8, n = D - e0;
  const bool full = D - warp * 256 >= 256 || D <= warp * 256;     // the warp's leaf is whole, or there is none
  const int leaves = (D + 255) >> 8;
  const float2 one = same2(c_one), minus = same2(-c_one);
  const bool cols = out_g || out_b;
  const int groups8 = (D + A8_GROUP - 1) / A8_GROUP;
  const int block = S::GROUPS * R * passes, stride = gridDim.x * block, mine = grp * R * passes;   // rows: of a block, to this CTA's next one, of the groups before
  // the row's statistics and, of a checkpoint, the step travel in registers, a pass ahead
  float mu_next[R], rs_next[R];
  uint32_t step_next[R];                                  // the field: a step worked out here would wait for the load
  struct { int base, p, slot; } ahead = {(int)blockIdx.x * block, 0, 0};        // the pass to fetch next
  auto fetch = [&]() {
    if (STAGED) {
      if (ahead.base < rows) {
        char* place = smem + ahead.slot * R * BYTES;
        const int row = ahead.base + mine + ahead.p * R;
        size_t at = row_at(row, D, e0);
#pragma unroll
        for (int a = 0; a < R; ++a, place += BYTES, at += D) {
          const bool there = row + a < rows && n > 0;
          row_fetch<Fx::DY, T>(place, static_cast<const char*>(dy) + at * (BF ? 2 : 4), there);
          row_fetch<Fx::X, T>(place + T * Fx::DY, static_cast<const char*>(x) + at * (KIND == LN_ACT8 ? 1 : (BF ? 2 : 4)), there);
          if (RES) row_fetch<Fx::DY, T>(place + T * (Fx::DY + Fx::X), static_cast<const char*>(res) + at * (BF ? 2 : 4), there);
        }
      }
      fetch_close();
      ahead.slot = ahead.slot + 1 == AHEAD ? 0 : ahead.slot + 1;
      if (++ahead.p == passes) { ahead.p = 0; ahead.base += stride; }
    }
  };
  auto statistics = [&](int first) {
#pragma unroll
    for (int a = 0; a < R; ++a) {
      const int row = first + a;
      const bool there = row < rows;
      mu_next[a] = there ? mean[row] : 0.0f;
      rs_next[a] = there ? rstd[row] : 0.0f;
      if (KIND == LN_ACT8 && VEC) step_next[a] = there && n > 0 ? e8[(size_t)row * groups8 + e0 / A8_GROUP] : 0u;
    }
  };
#pragma unroll
  for (int k = 0; k < AHEAD - 1; ++k) fetch();
  statistics(blockIdx.x * block + mine);
  float g[8];
  const int w0 = warp * 256, left = D - w0;              // the warp's first column, how many are left from there
  if (gamma) {
    if (VEC) {
      load8n<BF>(gamma, e0, n, g);
    } else {
      uint32_t raw[8];
      load_any<BF ? 2 : 4>(gamma, w0, left, raw);
      deal_out(room, raw, g);
    }
  }
  float node[16];                                         // of this group's rows so far: 8 columns of dgamma, 8 of dbeta
  int slot = 0;
  bool odd = false;                                       // which half of leaf_s the pass uses
#pragma unroll 1
  for (int blk = blockIdx.x; blk < nb; blk += gridDim.x) {
  const int r0 = blk * block + mine;
#pragma unroll 1
  for (int p = 0; p < passes; ++p) {
    const int first = r0 + p * R;
    float w[R][8], xh[R][8], rs[R], mu[R], step[R];
#pragma unroll
    for (int a = 0; a < R; ++a) { mu[a] = mu_next[a]; rs[a] = rs_next[a]; step[a] = KIND == LN_ACT8 && VEC ? a8_step(step_next[a]) : 0.0f; }
    fetch();
    statistics(p + 1 < passes ? first + R : r0 + stride);
    if (STAGED) fetch_wait<AHEAD - 1>();
    const char* place = smem + slot * R * BYTES;
    slot = slot + 1 == AHEAD ? 0 : slot + 1;
    if (!VEC) {   // all loads first, then dealt out
      uint32_t raw_dy[R][8], raw_x[R][8];
#pragma unroll
      for (int a = 0; a < R; ++a) {
        const int l = first + a < rows ? left : 0;
        load_any<BF ? 2 : 4>(dy, row_at(first + a, D, w0), l, raw_dy[a]);
        load_any<KIND == LN_F32 ? 4 : (KIND == LN_BF16 ? 2 : 1)>(x, row_at(first + a, D, w0), l, raw_x[a]);
        if (KIND == LN_ACT8) {   // the columns lane + 32 k are of one group for each k
#pragma unroll
          for (int t = 0; t < 8; ++t)
            raw_x[a][t] = __float_as_uint(fmul(__uint_as_float(raw_x[a][t]), l > 32 * t ? a8_step(e8[(size_t)(first + a) * groups8 + warp * 8 + t]) : 0.0f));
        }
      }
#pragma unroll
      for (int a = 0; a < R; ++a) {
        deal_out(room, raw_dy[a], w[a]);
        deal_out(room, raw_x[a], xh[a]);
      }
    }
#pragma unroll
    for (int a = 0; a < R; ++a) {
      const int row = first + a, m = row < rows ? n : 0;
      if (STAGED) row_take<BF, T>(place + a * BYTES, w[a]);
      else if (VEC) load8n<BF>(dy, row_at(row, D, e0), m, w[a]);
      if (STAGED && KIND == LN_ACT8) a8_values8(reinterpret_cast<const uint2*>(place + a * BYTES + T * Fx::DY)[threadIdx.x], step[a], xh[a]);
      else if (STAGED) row_take<BF, T>(place + a * BYTES + T * Fx::DY, xh[a]);
      else if (VEC) load8n<BF>(x, row_at(row, D, e0), m, xh[a]);
#pragma unroll
      for (int t = 0; t < 8; t += 2) two(xh[a] + t, mul2(fma2(same2(mu[a]), same2(-1.0f), two(xh[a] + t)), same2(rs[a])));
    }
    if (cols) {   // rows in pairs, pairs in pairs; a right node exists iff its first row does, else the left one is carried up unchanged
#pragma unroll
      for (int t = 0; t < 8; t += 2) {
        float2 c[R], d[R];
#pragma unroll
        for (int a = 0; a < R; ++a) { d[a] = two(w[a] + t); c[a] = mul2(d[a], two(xh[a] + t)); }
        two(node + t, node_tree2<R>(c, rows - first, one));
        two(node + 8 + t, node_tree2<R>(d, rows - first, one));
      }
      // the lowest levels in shared memory, the others, which are met rarely, in the CTA's place in the workspace
      float4* far = upper + (size_t)blockIdx.x * upper_levels * 4 * T + threadIdx.x;
      const auto join = [&](const float4* l, bool have) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float4 q = l[t * T];
          const float2 a = make_float2(q.x, q.y), b = make_float2(q.z, q.w);
          two(node + 4 * t, have ? add2(a, two(node + 4 * t), one) : a);
          two(node + 4 * t + 2, have ? add2(b, two(node + 4 * t + 2), one) : b);
        }
      };
      const auto wait = [&](float4* l) {
#pragma unroll
        for (int t = 0; t < 4; ++t) l[t * T] = make_float4(node[4 * t], node[4 * t + 1], node[4 * t + 2], node[4 * t + 3]);
      };
      int level = 0;
      for (; (p >> level) & 1; ++level) {
        const bool have = r0 + ((p >> level) << level) * R < rows;
        if (level < S::LEVELS) join(waiting + level * 4 * T + threadIdx.x, have);
        else join(far + (level - S::LEVELS) * 4 * T, have);
      }
      if (p + 1 < passes) {
        if (level < S::LEVELS) wait(waiting + level * 4 * T + threadIdx.x);
        else wait(far + (level - S::LEVELS) * 4 * T);
      }
    }
    if (gamma) {
#pragma unroll
      for (int a = 0; a < R; ++a)
#pragma unroll
        for (int t = 0; t < 8; t += 2) two(w[a] + t, mul2(two(w[a] + t), two(g + t)));
    }
    float (*leaf)[2][WPR] = leaf_s[odd][grp];
    odd = !odd;
    float part[2 * R];
#pragma unroll
    for (int a = 0; a < R; ++a) {
      float pr[8];
#pragma unroll
      for (int t = 0; t < 8; t += 2) two(pr + t, mul2(two(w[a] + t), two(xh[a] + t)));
      two(part + 2 * a, lane_sums<VEC>(w[a], pr, e0, D, one));
    }
    leaf_sums<2 * R, WPR>(part, leaf[0][0], warp, D, full);
    __syncthreads();
    const float c_mine = fmul(dealt_tree<2 * R, WPR>(leaf[0][0], leaves), invD);
#pragma unroll
    for (int a = 0; a < R; ++a) {
      const float c1 = __shfl_sync(0xffffffffu, c_mine, 2 * a), c2 = __shfl_sync(0xffffffffu, c_mine, 2 * a + 1);
      const int m = first + a < rows ? n : 0;
      const size_t at = row_at(first + a, D, e0);
      float o[8];
#pragma unroll
      for (int t = 0; t < 8; t += 2)
        two(o + t, mul2(same2(rs[a]), fma2(mul2(two(xh[a] + t), same2(c2)), minus, add2(two(w[a] + t), same2(-c1), one))));
      if (RES) {   // the gradient that bypasses the norm (res may be dx)
        float b[8];
        if (STAGED) {
          row_take<BF, T>(place + a * BYTES + T * (Fx::DY + Fx::X), b);
        } else {
          uint32_t raw[8];
          load_any<BF ? 2 : 4>(res, row_at(first + a, D, w0), first + a < rows ? left : 0, raw);
          deal_out(room, raw, b);
        }
#pragma unroll
        for (int t = 0; t < 8; t += 2) two(o + t, add2(two(o + t), two(b + t), one));
      }
      if (!VEC) store_any<BF>(dx, row_at(first + a, D, w0), first + a < rows ? left : 0, room, o);
      else if (m > 0) store8<BF>(dx, at, o);
    }
  }
  if (!cols) continue;
  if (S::GROUPS > 1) {   // the tree over the groups' nodes
    __syncthreads();
    float* meet = reinterpret_cast<float*>(waiting) + threadIdx.x;
#pragma unroll
    for (int t = 0; t < 16; ++t) meet[t * T] = node[t];
    __syncthreads();
    if (grp == 0) {
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        float c[S::GROUPS];
#pragma unroll
        for (int k = 0; k < S::GROUPS; ++k) c[k] = meet[t * T + k * WPR * 32];
        node[t] = node_tree<S::GROUPS>(c, (rows - r0 + R * passes - 1) / (R * passes));
      }
    }
    __syncthreads();
  }
  if (grp == 0) {
#pragma unroll
    for (int t = 0; t < 16; ++t) node[t] = ln_flush(node[t]);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      float* dst = w ? out_b : out_g;
      if (!dst) continue;
      dst += (size_t)blk * D + e0;
      if (!VEC) store_any<false>(dst - lane * 8, 0, left, room, node + 8 * w);
      else if (n > 0) store8<false>(dst, 0, node + 8 * w);
    }
  }
  }
}

// The trees over the nb row blocks of every column of dgamma (y = 0) and dbeta (y = 1): a CTA has 32 columns, a warp 32 of 1024 adjacent nodes at a time
// (independent loads), the first warp the tree over the warps' nodes; nodes of finished thousands wait as the digits of a binary counter do.
__global__ void __launch_bounds__(1024) k_ln_cols(const float* __restrict__ partial, int nb, int D, float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float nodes[32][33];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = blockIdx.x * 32 + lane;
  float* out = blockIdx.y ? dbeta : dgamma;
  grid_dep();
  if (!out) return;
  partial += (size_t)blockIdx.y * nb * D;
  float waiting[22], r = 0.0f;
  const int thousands = (nb + 1023) / 1024;
  for (int c = 0; c < thousands; ++c) {
    const int first = c * 1024 + warp * 32, have = nb - first;
    if (have > 0 && col < D) {
      float s[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) s[i] = i < have ? partial[(size_t)(first + i) * D + col] : 0.0f;
      nodes[warp][lane] = node_tree<32>(s, have);
    }
    __syncthreads();
    if (warp == 0) {
      float s[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) s[i] = nodes[i][lane];
      r = node_tree<32>(s, (nb - c * 1024 + 31) / 32);
      int level = 0;
      for (; (c >> level) & 1; ++level) r = fadd(waiting[level], r);
      waiting[level] = r;
    }
    __syncthreads();
  }
  if (warp || col >= D) return;
  // what waits beside the last thousand's node, from the lowest level up: the nodes to their left
  int level = 0;
  while (((thousands - 1) >> level) & 1) ++level;
  for (++level; (thousands >> level) != 0; ++level)
    if ((thousands >> level) & 1) r = fadd(waiting[level], r);
  out[col] = r;
}

// ---- host side -------------------------------------------------------------------------------------------
template <class F>
static void with_wpr(int D, F f) {
  if (D <= 256) f(std::integral_constant<int, 1>());
  else if (D <= 512) f(std::integral_constant<int, 2>());
  else if (D <= 1024) f(std::integral_constant<int, 4>());
  else if (D <= 2048) f(std::integral_constant<int, 8>());
  else if (D <= 4096) f(std::integral_constant<int, 16>());
  else f(std::integral_constant<int, 32>());
}
template <class F>
static void with_bool(bool b, F f) { if (b) f(std::true_type()); else f(std::false_type()); }

// CTAs of the forward pass: with rows on their way ahead all that are on a GPU of `sms` SMs at once, else one for every piece of rows
template <class S>
static unsigned ln_ctas(int rows, int sms) {
  const long long pieces = ((long long)rows + LnWalk<S>::PIECE - 1) / LnWalk<S>::PIECE, most = (long long)S::CTAS * std::max(sms, 1);
  return (unsigned)(S::AHEAD_ROWS ? std::min(pieces, most) : pieces);
}
static int ln_fwd(bool bf, const void* x, const void* res, const void* gamma, const void* beta, int rows, int D, float eps, void* sum,
                  void* y, float* mean, float* rstd, const float* s_q, int8_t* qy, int8_t* q8, uint8_t* e8, cudaStream_t st) {
  int rc = DET_OK;
  with_wpr(D, [&](auto wpr) {
    with_bool(bf, [&](auto is_bf) {
      with_bool(D % 8 == 0, [&](auto is_vec) {
        with_bool(res != nullptr, [&](auto is_res) {
          constexpr int W = decltype(wpr)::value;
          constexpr bool BF = decltype(is_bf)::value, VEC = decltype(is_vec)::value, RES = decltype(is_res)::value;
          if constexpr (BF || !RES) {
            using S = LnShape<W, BF, VEC>;
            const size_t smem = S::AHEAD_ROWS ? (size_t)S::AHEAD * S::ROWS * S::THREADS * 8 * (BF ? 2 : 4) * (RES ? 2 : 1) : (VEC ? 0 : (size_t)S::THREADS * 32);
            auto kern = k_ln_fwd<BF, W, VEC, RES>;
            static DevOnce once;
            if (smem > 40 * 1024) rc = dev_ensure_smem(once, (const void*)kern, smem);
            if (rc != DET_OK) return;
            launch_after(kern, dim3(ln_ctas<S>(rows, dev_sm_count())), S::THREADS, smem, st, x, res, gamma, beta, rows, D, eps, (float)(1.0 / (double)D), sum, y, mean,
                         rstd, s_q, qy, q8, e8);
          }
        });
      });
    });
  });
  if (rc != DET_OK) return rc;
  DET_CHECK_LAUNCH();
  return DET_OK;
}

// Rows of a block of the backward pass, whose nodes go to memory for the second kernel: more of them while the CTA with the most has not much more to do (all
// that are on the GPU at once share the blocks).  Fewer nodes are less to write and to read: 8192 x 2048 with blocks of 8 and 32 rows 36.5
// and 34.0 us, 8192 x 4096 with 2 and 16 passes 82 and 68; but 12000 x 2048 with 4 passes 49 and with 8, where the busiest CTA has half as much again, 59.
constexpr int LN_PASSES = 16, LN_SLACK = 5;                // passes of a block at most; of the busiest CTA, to those with blocks of one, times 4
struct LnBlock {
  int passes, rows, levels, upper, ctas;                 // passes of a block, its rows; levels of waiting nodes, how many in the workspace; CTAs at once
  size_t level;                                          // bytes of a CTA's waiting nodes of a level
  int blocks(int n) const { return (int)(((long long)n + rows - 1) / rows); }
  int grid(int n) const { return std::min(blocks(n), ctas); }
};
template <int KIND>
static LnBlock ln_block(int rows, int D) {
  LnBlock r{};
  int per = 0, own = 0;
  with_wpr(D, [&](auto wpr) {
    with_bool(D % 8 == 0, [&](auto is_vec) {
      using S = LnBwd<decltype(wpr)::value, KIND, decltype(is_vec)::value>;
      per = S::GROUPS * S::ROWS;
      own = S::LEVELS;
      r.ctas = S::CTAS * 148;
      r.level = (size_t)16 * S::THREADS * sizeof(float);
    });
  });
  const auto most = [&](int passes) {                    // passes of the CTA with the most
    const long long blocks = ((long long)rows + (long long)passes * per - 1) / ((long long)passes * per);
    return (blocks + r.ctas - 1) / r.ctas * passes;
  };
  r.passes = 1;
  for (int p = 2; p <= LN_PASSES; p *= 2)
    if (4 * most(p) <= LN_SLACK * most(1)) {
      r.passes = p;
      ++r.levels;
    } else {
      break;
    }
  r.rows = r.passes * per;
  r.upper = std::max(0, r.levels - own);
  return r;
}
static size_t ln_nodes(int nb, int D) { return ((size_t)2 * nb * D * sizeof(float) + 15) / 16 * 16; }
template <int KIND>
static int ln_bwd(const void* dy, const void* x, const uint8_t* e8, const void* gamma, const float* mean, const float* rstd, int rows, int D,
                  const void* res, void* dx, float* dgamma, float* dbeta, void* ws, cudaStream_t st) {
  const bool cols = dgamma || dbeta;
  const LnBlock block = ln_block<KIND>(rows, D);
  const int nb = block.blocks(rows);
  const bool direct = nb == 1 && (D % 8 != 0 || (aligned16(dgamma) && aligned16(dbeta)));     // few rows: no second launch
  float* partial = (float*)ws;
  float *out_g = direct ? dgamma : cols ? partial : nullptr, *out_b = direct ? dbeta : cols ? partial + (size_t)nb * D : nullptr;
  float4* upper = cols ? (float4*)((char*)ws + ln_nodes(nb, D)) : nullptr;
  int rc = DET_OK;
  with_wpr(D, [&](auto wpr) {
    with_bool(D % 8 == 0, [&](auto is_vec) {
      with_bool(res != nullptr, [&](auto is_res) {
        constexpr int W = decltype(wpr)::value;
        constexpr bool VEC = decltype(is_vec)::value, RES = decltype(is_res)::value;
        if constexpr (!(RES && KIND == LN_F32)) {
          using S = LnBwd<W, KIND, VEC>;
          const int levels = std::max(std::min(block.levels, (int)S::LEVELS), S::GROUPS > 1 ? 1 : 0);      // in shared memory; the groups meet in the first
          const size_t ahead = S::AHEAD_ROWS ? (size_t)LnFetch<KIND, W, VEC>::AHEAD * S::ROWS * (RES ? LnFetch<KIND, W, VEC>::ROW_RES : LnFetch<KIND, W, VEC>::ROW) : 0;
          auto kern = k_ln_bwd<KIND, W, VEC, RES>;
          static DevOnce once;
          rc = dev_ensure_smem(once, (const void*)kern, ahead + S::LEVELS * block.level);
          if (rc != DET_OK) return;
          launch_after(kern, dim3((unsigned)block.grid(rows)), S::THREADS, ahead + (cols ? levels * block.level : 0), st, dy, x, e8, gamma, mean, rstd, rows, D,
                       (float)(1.0 / (double)D), nb, block.passes, res, dx, out_g, out_b, upper, block.upper);
        }
      });
    });
  });
  if (rc != DET_OK) return rc;
  if (cols && !direct)
    launch_after(k_ln_cols, dim3((D + 31) / 32, 2), 1024, 0, st, (const float*)partial, nb, D, dgamma, dbeta);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
constexpr int LN_ROWS = 2000000000;         // so that the rows of the last CTA have numbers too
static bool elem_aligned(const void* p, int D, size_t elem) { return (uintptr_t)p % (D % 8 == 0 ? 16 : elem) == 0; }

}  // namespace det

using namespace det;

extern "C" int det_layernorm_fwd(int io, const void* x, const void* gamma, const void* beta, int rows, int D, float eps, void* y, float* mean,
                                 float* rstd, void* stream) {
  if (!x || !y || !mean || !rstd || rows < 0 || D <= 0 || (io != DET_F32 && io != DET_BF16)) return DET_ERR_ARG;
  if (D > 8192 || rows > LN_ROWS) return DET_ERR_SHAPE;
  const size_t el = io == DET_BF16 ? 2 : 4;
  if (!elem_aligned(x, D, el) || !elem_aligned(y, D, el) || !elem_aligned(gamma, D, el) || !elem_aligned(beta, D, el)) return DET_ERR_ALIGN;
  if (rows == 0) return DET_OK;
  return ln_fwd(io == DET_BF16, x, nullptr, gamma, beta, rows, D, eps, nullptr, y, mean, rstd, nullptr, nullptr, nullptr, nullptr, (cudaStream_t)stream);
}

extern "C" int det_test_layernorm_walk(int io, int rows, int D, int sms, long long seen[4]) {
  if (rows <= 0 || rows > LN_ROWS || D <= 0 || D > 8192 || sms <= 0 || !seen || (io != DET_F32 && io != DET_BF16)) return DET_ERR_ARG;
  with_wpr(D, [&](auto wpr) {
    with_bool(io == DET_BF16, [&](auto is_bf) {
      with_bool(D % 8 == 0, [&](auto is_vec) {
        using S = LnShape<decltype(wpr)::value, decltype(is_bf)::value, decltype(is_vec)::value>;
        const unsigned ctas = ln_ctas<S>(rows, sms);
        seen[0] = seen[1] = 0;
        seen[2] = rows;
        seen[3] = -1;
        for (unsigned cta = 0; cta < ctas; ++cta) {
          long long passes = 0;
          for (LnWalk<S> w(cta, ctas); w.base < rows; w.next(rows), ++passes) {
            seen[2] = std::min<long long>(seen[2], w.base);
            seen[3] = std::max<long long>(seen[3], w.base);
          }
          seen[0] += passes;
          seen[1] = std::max(seen[1], passes);
        }
      });
    });
  });
  return DET_OK;
}

extern "C" int det_residual_layernorm_fwd(const det_bf16* a, const det_bf16* b, const det_bf16* gamma, const det_bf16* beta, int rows, int D,
                                          float eps, det_bf16* sum, det_bf16* y, float* mean, float* rstd, const float* s_q, int8_t* qy,
                                          int8_t* q8, uint8_t* e8, void* stream) {
  if (!a || (b && !sum) || !y || !mean || !rstd || (qy && !s_q) || (!q8 != !e8) || rows < 0 || D <= 0) return DET_ERR_ARG;
  if (D > 8192 || rows > LN_ROWS || (D % 8 && (qy || q8))) return DET_ERR_SHAPE;
  if (!elem_aligned(a, D, 2) || !elem_aligned(b, D, 2) || !elem_aligned(gamma, D, 2) || !elem_aligned(beta, D, 2) ||
      (b && !elem_aligned(sum, D, 2)) || !elem_aligned(y, D, 2) || (((uintptr_t)qy | (uintptr_t)q8) & 7u))
    return DET_ERR_ALIGN;
  if (rows == 0) return DET_OK;
  return ln_fwd(true, a, b, gamma, beta, rows, D, eps, sum, y, mean, rstd, s_q, qy, q8, e8, (cudaStream_t)stream);
}

extern "C" size_t det_layernorm_bwd_ws_bytes(int rows, int D) {
  if (rows <= 0 || D <= 0 || D > 8192) return 256;
  size_t most = 0;
  for (const LnBlock& b : {ln_block<LN_F32>(rows, D), ln_block<LN_BF16>(rows, D), ln_block<LN_ACT8>(rows, D)})
    most = std::max(most, ln_nodes(b.blocks(rows), D) + b.level * b.upper * b.grid(rows));
  return align_up(most, 256);
}

// what the three backward calls have in common: checks, nothing to do, launch
template <int KIND>
static int ln_bwd_entry(const void* dy, const void* x, const uint8_t* e8, const void* gamma, const float* mean, const float* rstd, int rows, int D,
                        const void* res, void* dx, float* dgamma, float* dbeta, void* ws, size_t ws_bytes, cudaStream_t st) {
  if (!dy || !x || !mean || !rstd || !dx || rows < 0 || D <= 0) return DET_ERR_ARG;
  if (D > 8192 || rows > LN_ROWS) return DET_ERR_SHAPE;
  const size_t el = KIND == LN_F32 ? 4 : 2;
  if (!elem_aligned(dy, D, el) || !elem_aligned(dx, D, el) || !elem_aligned(gamma, D, el) || !elem_aligned(res, D, el)) return DET_ERR_ALIGN;
  if (KIND == LN_ACT8 ? (D % 8 == 0 && ((uintptr_t)x & 7u)) : !elem_aligned(x, D, el)) return DET_ERR_ALIGN;
  if ((dgamma || dbeta) && rows > 0 && (!ws || !aligned16(ws) || ws_bytes < det_layernorm_bwd_ws_bytes(rows, D))) return DET_ERR_WORKSPACE;
  if (rows == 0) {
    if (dgamma && cudaMemsetAsync(dgamma, 0, (size_t)D * sizeof(float), st) != cudaSuccess) return DET_ERR_CUDA;
    if (dbeta && cudaMemsetAsync(dbeta, 0, (size_t)D * sizeof(float), st) != cudaSuccess) return DET_ERR_CUDA;
    return DET_OK;
  }
  return ln_bwd<KIND>(dy, x, e8, gamma, mean, rstd, rows, D, res, dx, dgamma, dbeta, ws, st);
}

extern "C" int det_layernorm_bwd(int io, const void* dy, const void* x, const void* gamma, const float* mean, const float* rstd, int rows,
                                 int D, void* dx, float* dgamma, float* dbeta, void* ws, size_t ws_bytes, void* stream) {
  if (io == DET_BF16)
    return ln_bwd_entry<LN_BF16>(dy, x, nullptr, gamma, mean, rstd, rows, D, nullptr, dx, dgamma, dbeta, ws, ws_bytes, (cudaStream_t)stream);
  if (io != DET_F32) return DET_ERR_ARG;
  return ln_bwd_entry<LN_F32>(dy, x, nullptr, gamma, mean, rstd, rows, D, nullptr, dx, dgamma, dbeta, ws, ws_bytes, (cudaStream_t)stream);
}

extern "C" int det_layernorm_bwd_residual(const det_bf16* dy, const det_bf16* x, const det_bf16* gamma, const float* mean, const float* rstd,
                                          int rows, int D, const det_bf16* res, det_bf16* dx, float* dgamma, float* dbeta, void* ws,
                                          size_t ws_bytes, void* stream) {
  if (!res) return DET_ERR_ARG;
  return ln_bwd_entry<LN_BF16>(dy, x, nullptr, gamma, mean, rstd, rows, D, res, dx, dgamma, dbeta, ws, ws_bytes, (cudaStream_t)stream);
}

extern "C" int det_layernorm_bwd_act8(const det_bf16* dy, const int8_t* q8, const uint8_t* e8, const det_bf16* gamma, const float* mean,
                                      const float* rstd, int rows, int D, const det_bf16* res, det_bf16* dx, float* dgamma, float* dbeta,
                                      void* ws, size_t ws_bytes, void* stream) {
  if (!e8) return DET_ERR_ARG;
  return ln_bwd_entry<LN_ACT8>(dy, q8, e8, gamma, mean, rstd, rows, D, res, dx, dgamma, dbeta, ws, ws_bytes, (cudaStream_t)stream);
}
