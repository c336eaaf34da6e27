// Activations kept in 8 bits between the forward and the backward pass: storing and restoring them, and SwiGLU from and to them.
// The format (rows.cuh) has a power-of-two step for every 32 adjacent values of a row, so nothing here rounds but the code itself.
// All of it is bound by memory: every value is read and written once, eight a thread.
#include "common.cuh"
#include "internal.h"
#include "rows.cuh"

namespace det {

// i / d for i below 2^31 by a multiplication
struct Divider {
  uint32_t d, m;
  int s;
  explicit Divider(uint32_t n) : d(n), s(0) {
    while ((1ull << s) < n) ++s;
    m = (uint32_t)((((1ull << s) - n) << 32) / n) + 1;
  }
  __device__ __forceinline__ uint32_t operator()(uint32_t i) const { return (__umulhi(i, m) + i) >> s; }
};

// Rows of a multiple of 8 columns, 16-byte aligned: a lane has eight adjacent values, four lanes a group; A8_EACH such pieces a thread, 256 apart, their
// loads ahead of the rest.
constexpr int A8_EACH = 4;
template <bool BF>
__global__ void __launch_bounds__(256) k_a8_pack(const void* __restrict__ x, size_t ld, Divider lanes, uint32_t pieces, int D, int8_t* __restrict__ q,
                                                 uint8_t* __restrict__ e) {
  grid_dep();
  // lanes: pieces of a row, the last group's whole four included
  const uint32_t first = blockIdx.x * (256 * A8_EACH) + threadIdx.x;
  float v[A8_EACH][8];
  uint32_t r[A8_EACH], c[A8_EACH];
  bool have[A8_EACH];
#pragma unroll
  for (int k = 0; k < A8_EACH; ++k) {
    const uint32_t i = first + 256 * k;
    r[k] = lanes(i);
    c[k] = (i - r[k] * lanes.d) * 8;
    have[k] = i < pieces && c[k] < (uint32_t)D;
    load8n<BF>(x, (size_t)r[k] * ld + c[k], have[k], v[k]);
  }
#pragma unroll
  for (int k = 0; k < A8_EACH; ++k) {
    const uint32_t field = a8_field(a8_quad_max(a8_amax8(v[k])));
    if (!have[k]) continue;
    *reinterpret_cast<uint2*>(q + (size_t)r[k] * D + c[k]) = a8_codes8(v[k], field);
    if ((threadIdx.x & 3) == 0) e[(first + 256 * k) / 4] = (uint8_t)field;
  }
}
template <bool BF>
__global__ void __launch_bounds__(256) k_a8_unpack(const int8_t* __restrict__ q, const uint8_t* __restrict__ e, Divider lanes, uint32_t pieces, int D,
                                                   void* __restrict__ y, size_t ld) {
  grid_dep();
  const uint32_t first = blockIdx.x * (256 * A8_EACH) + threadIdx.x;
  uint2 codes[A8_EACH];
  uint32_t r[A8_EACH], c[A8_EACH], field[A8_EACH];
  bool have[A8_EACH];
#pragma unroll
  for (int k = 0; k < A8_EACH; ++k) {
    const uint32_t i = first + 256 * k;
    r[k] = lanes(i);
    c[k] = (i - r[k] * lanes.d) * 8;
    have[k] = i < pieces && c[k] < (uint32_t)D;
    if (!have[k]) continue;
    codes[k] = *reinterpret_cast<const uint2*>(q + (size_t)r[k] * D + c[k]);
    field[k] = e[i / 4];
  }
#pragma unroll
  for (int k = 0; k < A8_EACH; ++k) {
    if (!have[k]) continue;
    float v[8];
    a8_values8(codes[k], a8_step(field[k]), v);
    store8<BF>(y, (size_t)r[k] * ld + c[k], v);
  }
}
// Any width, stride and address: a lane per value, a warp per group, A8_GROUPS of them one after the other with their loads ahead of the rest.
constexpr int A8_GROUPS = 8;
template <bool BF>
__global__ void __launch_bounds__(256) k_a8_pack_any(const void* __restrict__ x, size_t ld, Divider ng, uint32_t groups, int D, int8_t* __restrict__ q,
                                                     uint8_t* __restrict__ e) {
  grid_dep();
  const uint32_t first = (blockIdx.x * 8 + (threadIdx.x >> 5)) * A8_GROUPS;
  const int lane = threadIdx.x & 31;
  float v[A8_GROUPS];
  size_t at[A8_GROUPS];
  bool have[A8_GROUPS];
#pragma unroll
  for (int k = 0; k < A8_GROUPS; ++k) {
    const uint32_t r = ng(first + k), c = (first + k - r * ng.d) * A8_GROUP + lane;
    have[k] = first + k < groups && c < (uint32_t)D;
    at[k] = (size_t)r * D + c;
    const size_t from = (size_t)r * ld + c;
    v[k] = have[k] ? (BF ? bf2f(reinterpret_cast<const uint16_t*>(x)[from]) : reinterpret_cast<const float*>(x)[from]) : 0.0f;
  }
  uint32_t mine = 0;                                     // lane k keeps the field of group k
#pragma unroll
  for (int k = 0; k < A8_GROUPS; ++k) {
    const uint32_t field = a8_field(__reduce_max_sync(0xffffffffu, __float_as_uint(v[k]) & 0x7fffffffu));
    if (have[k]) q[at[k]] = (int8_t)(field != 255u ? __float_as_uint(fadd(fmul(v[k], a8_inv(field)), 12582912.0f)) : a8_code_nonfinite(v[k]));
    if (lane == k) mine = field;
  }
  if (lane < A8_GROUPS && first + lane < groups) e[first + lane] = (uint8_t)mine;
}
template <bool BF>
__global__ void __launch_bounds__(256) k_a8_unpack_any(const int8_t* __restrict__ q, const uint8_t* __restrict__ e, Divider ng, uint32_t groups, int D,
                                                       void* __restrict__ y, size_t ld) {
  grid_dep();
  const uint32_t first = (blockIdx.x * 8 + (threadIdx.x >> 5)) * A8_GROUPS;
  const int lane = threadIdx.x & 31;
  float v[A8_GROUPS];
  size_t to[A8_GROUPS];
  bool have[A8_GROUPS];
  const uint32_t mine = lane < A8_GROUPS && first + lane < groups ? e[first + lane] : 0u;
#pragma unroll
  for (int k = 0; k < A8_GROUPS; ++k) {
    const uint32_t r = ng(first + k), c = (first + k - r * ng.d) * A8_GROUP + lane;
    have[k] = first + k < groups && c < (uint32_t)D;
    to[k] = (size_t)r * ld + c;
    v[k] = have[k] ? (float)q[(size_t)r * D + c] : 0.0f;
  }
#pragma unroll
  for (int k = 0; k < A8_GROUPS; ++k) {
    const float step = a8_step(__shfl_sync(0xffffffffu, mine, k));
    if (!have[k]) continue;
    if (BF) reinterpret_cast<uint16_t*>(y)[to[k]] = f2bf(fmul(v[k], step));
    else reinterpret_cast<float*>(y)[to[k]] = fmul(v[k], step);
  }
}

// ---- SwiGLU: gu [rows, 2F] = (gate | up), F a multiple of 32, so no group holds both -----------------------
// The gate is a bf16 either way, so its sigmoid has few values: 33 exponents of magnitude (below 2^-26 it is 1/2, from 128 on 1 or 0) of 128 fractions and two
// signs.  They are evaluated by the compiler, with the steps of the formula, and looked up in shared memory: with an exponential and a division for every
// value the three kernels took 160, 133 and 152 us for 8192 x 8192, bound by the arithmetic; now 92, 76 and 92 (each over and over; the three in turn on the same tensors 284), where the
// bytes alone would take 83, 42 and 83 at the measured copy's rate.
constexpr int SG_LOW = 0x3280, SG_TOP = 0x4300, SG_TAB = (SG_TOP - SG_LOW + 1 + 255) / 256 * 256;
struct __align__(16) SgTable { float v[2 * SG_TAB]; };     // of positive gates, of negative ones
constexpr float sg_at(int bits, bool negative) {
  float x = 1.0f + (bits & 127) / 128.0f;
  for (int e = bits >> 7; e > 127; --e) x *= 2.0f;
  for (int e = bits >> 7; e < 127; ++e) x *= 0.5f;
  if (!negative) x = -x;
  if (x > 0x1.62e42ep+6f) return 0.0f;                     // x: -gate
  const float d = 1.0f + det_exp_at(x), q = 1.0f / d;
  return q < 0x1p-126f ? 0.0f : q;
}
// Where entry i lies: a code below 64 has fractions that end in zeros, and in order of the magnitude they would meet in a few banks of shared memory.
constexpr int sg_place(int i) { return i ^ ((i >> 3) & 31); }
constexpr SgTable sg_make_table() {
  SgTable t{};
  for (int i = 0; i < SG_TAB; ++i) {
    t.v[sg_place(i)] = sg_at(SG_LOW + i, false);
    t.v[SG_TAB + sg_place(i)] = sg_at(SG_LOW + i, true);
  }
  return t;
}
__device__ constexpr SgTable sg_table_image = sg_make_table();

// the sigmoid of a gate; by table a NaN has that of an infinity, and what it is multiplied with, the gate itself, is the NaN
// (TAB 0: by the formula, 1: by table in order, for gates with any fractions, 2: by table in its places)
template <int TAB>
__device__ __forceinline__ float sigmoid_a8(float g, const float* tab) {
  if (!TAB) return fdiv(1.0f, fadd(1.0f, det_exp(-g)));
  const uint32_t u = __float_as_uint(g);
  int i = __vimin_s32_relu((int)((u >> 14) & 0x1fffcu) - 4 * SG_LOW, 4 * (SG_TOP - SG_LOW));           // in bytes
  if (TAB == 2) i ^= (i >> 3) & 0x7c;
  return *reinterpret_cast<const float*>(reinterpret_cast<const char*>(tab) + i + (int)(u >> 31) * (4 * SG_TAB));
}
template <int TAB>
__device__ __forceinline__ void sg_copy_table(float* tab) {
  if (!TAB) return;
  for (int i = threadIdx.x; i < 2 * SG_TAB / 4; i += 256) {
    const float4 v = reinterpret_cast<const float4*>(sg_table_image.v)[i];
    if (TAB == 2) {
      reinterpret_cast<float4*>(tab)[i] = v;
    } else {   // SG_TAB is a multiple of 256, so a place is undone in either half alike
      const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        int at = 4 * i + k;
        at ^= (at >> 3) & 28;                            // undoes the upper three of the five bits, which the lower two came from
        at ^= (at >> 3) & 3;
        tab[at] = w[k];
      }
    }
  }
  __syncthreads();
}
// Eight adjacent gates and their ups on their way: of gu, or codes and fields of the checkpoint; dh beside them in the backward pass.
struct SgRaw {
  uint4 g, u, d;
  uint32_t fg, fu;
};
// FROM: gate and up come from the checkpoint (gu absent), else they come from gu and the checkpoint is written.  A thread has eight adjacent gates and
// their ups at a time, the next ones on their way; `pieces` of them are walked over by CTAs that stay (TAB) or there is a thread for each.
template <bool FROM, int TAB>
__global__ void __launch_bounds__(256, 4) k_swiglu_fwd_a8(const uint16_t* __restrict__ gu, int8_t* q, uint8_t* e, Divider lanes, uint32_t pieces, int F,
                                                          uint16_t* __restrict__ h, const float* __restrict__ s_q, int8_t* __restrict__ qh) {
  __shared__ __align__(16) float tab[TAB ? 2 * SG_TAB : 4];
  sg_copy_table<TAB>(tab);
  grid_dep();
  const float inv_q = qh ? fdiv(1.0f, s_q[0]) : 0.0f;
  const uint32_t step = gridDim.x * 256;
  auto fetch = [&](uint32_t i) {
    SgRaw w = {};
    if (i >= pieces) return w;
    const uint32_t r = lanes(i), c = (i - r * lanes.d) * 8;
    const size_t at = (size_t)r * 2 * F + c;
    if (FROM) {
      const uint2 a = *reinterpret_cast<const uint2*>(q + at), b = *reinterpret_cast<const uint2*>(q + at + F);
      w.g.x = a.x; w.g.y = a.y; w.u.x = b.x; w.u.y = b.y;
      w.fg = e[at / A8_GROUP];
      w.fu = e[(at + F) / A8_GROUP];
    } else {
      w.g = *reinterpret_cast<const uint4*>(gu + at);
      w.u = *reinterpret_cast<const uint4*>(gu + at + F);
    }
    return w;
  };
  SgRaw next = fetch(blockIdx.x * 256 + threadIdx.x);
  for (uint32_t base = blockIdx.x * 256; base < pieces; base += step) {
    const uint32_t i = base + threadIdx.x;
    const SgRaw now = next;
    if (TAB) next = fetch(i + step);
    const bool have = i < pieces;
    const uint32_t r = have ? lanes(i) : 0, c = have ? (i - r * lanes.d) * 8 : 0;
    float g[8], u[8], o[8];
    if (FROM) {
      if (!have) continue;
      a8_values8(make_uint2(now.g.x, now.g.y), a8_step(now.fg), g);
      a8_values8(make_uint2(now.u.x, now.u.y), a8_step(now.fu), u);
    } else {
      const size_t at = (size_t)r * 2 * F + c;
      unpack8(now.g, g);
      unpack8(now.u, u);
      const uint32_t fg = a8_field(a8_quad_max(a8_amax8(g))), fu = a8_field(a8_quad_max(a8_amax8(u)));
      if (!have) continue;
      *reinterpret_cast<uint2*>(q + at) = a8_codes8(g, fg);
      *reinterpret_cast<uint2*>(q + at + F) = a8_codes8(u, fu);
      if ((i & 3) == 0) {
        e[at / A8_GROUP] = (uint8_t)fg;
        e[(at + F) / A8_GROUP] = (uint8_t)fu;
      }
    }
#pragma unroll
    for (int t = 0; t < 8; t += 2) {
      const float2 sg = make_float2(sigmoid_a8<TAB>(g[t], tab), sigmoid_a8<TAB>(g[t + 1], tab));
      const float2 r = mul2(mul2(make_float2(g[t], g[t + 1]), sg), make_float2(u[t], u[t + 1]));
      o[t] = r.x;
      o[t + 1] = r.y;
    }
    store8<true>(h, (size_t)r * F + c, o);
    if (qh) {   // the next linear's quantiser, applied to the bf16 values just stored
      round8(o);
      *reinterpret_cast<uint2*>(qh + (size_t)r * F + c) = quant8(o, inv_q);
    }
  }
}
template <int TAB>
__global__ void __launch_bounds__(256, 4) k_swiglu_bwd_a8(const uint16_t* __restrict__ dh, const int8_t* __restrict__ q, const uint8_t* __restrict__ e,
                                                          Divider lanes, uint32_t pieces, int F, uint16_t* __restrict__ dgu) {
  __shared__ __align__(16) float tab[TAB ? 2 * SG_TAB : 4];
  sg_copy_table<TAB>(tab);
  grid_dep();
  const uint32_t step = gridDim.x * 256;
  auto fetch = [&](uint32_t i) {
    SgRaw w = {};
    if (i >= pieces) return w;
    const uint32_t r = lanes(i), c = (i - r * lanes.d) * 8;
    const size_t at = (size_t)r * 2 * F + c;
    const uint2 a = *reinterpret_cast<const uint2*>(q + at), b = *reinterpret_cast<const uint2*>(q + at + F);
    w.g.x = a.x; w.g.y = a.y; w.u.x = b.x; w.u.y = b.y;
    w.fg = e[at / A8_GROUP];
    w.fu = e[(at + F) / A8_GROUP];
    w.d = *reinterpret_cast<const uint4*>(dh + (size_t)r * F + c);
    return w;
  };
  uint32_t i = blockIdx.x * 256 + threadIdx.x;
  SgRaw next = fetch(i);
  for (; i < pieces; i += step) {
    const SgRaw now = next;
    if (TAB) next = fetch(i + step);
    const uint32_t r = lanes(i), c = (i - r * lanes.d) * 8;
    const size_t at = (size_t)r * 2 * F + c;
    float g[8], u[8], d[8], dg[8], du[8];
    a8_values8<false>(make_uint2(now.g.x, now.g.y), a8_step(now.fg), g);
    a8_values8<false>(make_uint2(now.u.x, now.u.y), a8_step(now.fu), u);
    unpack8(now.d, d);
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const float sg = sigmoid_a8<TAB>(g[t], tab);
      du[t] = fmul(d[t], fmul(g[t], sg));
      dg[t] = fmul(fmul(d[t], u[t]), fmul(sg, fadd(1.0f, fmul(g[t], fsub(1.0f, sg)))));
    }
    store8<true>(dgu, at, dg);
    store8<true>(dgu, at + F, du);
  }
}

static unsigned blocks_for(size_t n, size_t each) { return (unsigned)((n + each - 1) / each); }
// SwiGLU: by table where every one of the CTAs that the GPU holds, four on an SM, has several pieces a thread (the table is 34 KiB to each)
constexpr int SG_CTAS = 4;
static bool sg_by_table(size_t pieces) { return pieces >= (size_t)SG_CTAS * dev_sm_count() * 256 * 2; }

}  // namespace det

using namespace det;

extern "C" size_t det_act8_exp_bytes(int rows, int D) {
  return rows > 0 && D > 0 ? (size_t)rows * (((size_t)D + A8_GROUP - 1) / A8_GROUP) : 0;
}

static int a8_check(int io, const void* x, int ld, int rows, int D, const void* q, const void* e) {
  if (!x || !q || !e || rows < 0 || D <= 0 || ld < D || (io != DET_F32 && io != DET_BF16)) return DET_ERR_ARG;
  if ((size_t)rows * (((size_t)D + 31) / 32) >= ((size_t)1 << 28)) return DET_ERR_SHAPE;      // four pieces a group, numbered in 31 bits
  if ((uintptr_t)x % (io == DET_BF16 ? 2 : 4)) return DET_ERR_ALIGN;
  return DET_OK;
}
static bool a8_vec(int io, const void* x, int ld, int D, const void* q) {
  return D % 8 == 0 && ld % (io == DET_BF16 ? 8 : 4) == 0 && aligned16(x) && ((uintptr_t)q & 7u) == 0;
}

extern "C" int det_act8_pack(int io, const void* x, int ld, int rows, int D, int8_t* q8, uint8_t* e8, void* stream) {
  const int rc = a8_check(io, x, ld, rows, D, q8, e8);
  if (rc != DET_OK || rows == 0) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  const uint32_t groups = (uint32_t)det_act8_exp_bytes(rows, D), ng = groups / rows;
  if (a8_vec(io, x, ld, D, q8))
    launch_after(io == DET_BF16 ? k_a8_pack<true> : k_a8_pack<false>, blocks_for(groups * 4, 256 * A8_EACH), 256, 0, st, x, (size_t)ld, Divider(ng * 4),
                 groups * 4, D, q8, e8);
  else
    launch_after(io == DET_BF16 ? k_a8_pack_any<true> : k_a8_pack_any<false>, blocks_for(groups, 8 * A8_GROUPS), 256, 0, st, x, (size_t)ld, Divider(ng),
                 groups, D, q8, e8);
  DET_CHECK_LAUNCH();
  return DET_OK;
}

extern "C" int det_act8_unpack(int io, const int8_t* q8, const uint8_t* e8, int rows, int D, void* y, int ld, void* stream) {
  const int rc = a8_check(io, y, ld, rows, D, q8, e8);
  if (rc != DET_OK || rows == 0) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  const uint32_t groups = (uint32_t)det_act8_exp_bytes(rows, D), ng = groups / rows;
  if (a8_vec(io, y, ld, D, q8))
    launch_after(io == DET_BF16 ? k_a8_unpack<true> : k_a8_unpack<false>, blocks_for(groups * 4, 256 * A8_EACH), 256, 0, st, q8, e8, Divider(ng * 4),
                 groups * 4, D, y, (size_t)ld);
  else
    launch_after(io == DET_BF16 ? k_a8_unpack_any<true> : k_a8_unpack_any<false>, blocks_for(groups, 8 * A8_GROUPS), 256, 0, st, q8, e8, Divider(ng), groups,
                 D, y, (size_t)ld);
  DET_CHECK_LAUNCH();
  return DET_OK;
}

static int swiglu_a8_check(const void* a, const void* b, const int8_t* q8, const uint8_t* e8, int rows, int F) {
  if (!a || !b || !q8 || !e8 || rows < 0 || F <= 0) return DET_ERR_ARG;
  if (F % 32 || F > (1 << 29) || (size_t)rows * (F / 8) >= ((size_t)1 << 30)) return DET_ERR_SHAPE;
  if (!aligned16(a) || !aligned16(b) || ((uintptr_t)q8 & 7u)) return DET_ERR_ALIGN;
  return DET_OK;
}
template <bool FROM>
static void swiglu_a8_fwd(const det_bf16* gu, int8_t* q8, uint8_t* e8, int rows, int F, det_bf16* h, const float* s_q, int8_t* qh, cudaStream_t st) {
  const uint32_t pieces = (uint32_t)rows * (F / 8);
  const bool tab = sg_by_table(pieces);
  launch_after(tab ? k_swiglu_fwd_a8<FROM, FROM ? 2 : 1> : k_swiglu_fwd_a8<FROM, 0>, tab ? SG_CTAS * dev_sm_count() : blocks_for(pieces, 256), 256, 0, st, gu, q8,
               e8, Divider(F / 8), pieces, F, h, s_q, qh);
}
extern "C" int det_swiglu_fwd_act8(const det_bf16* gu, int rows, int F, det_bf16* h, int8_t* q8, uint8_t* e8, const float* s_q, int8_t* qh,
                                   void* stream) {
  const int rc = swiglu_a8_check(gu, h, q8, e8, rows, F);
  if (rc != DET_OK) return rc;
  if (qh && !s_q) return DET_ERR_ARG;
  if ((uintptr_t)qh & 7u) return DET_ERR_ALIGN;
  if (rows == 0) return DET_OK;
  swiglu_a8_fwd<false>(gu, q8, e8, rows, F, h, s_q, qh, (cudaStream_t)stream);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
extern "C" int det_swiglu_act8(const int8_t* q8, const uint8_t* e8, int rows, int F, det_bf16* h, const float* s_q, int8_t* qh, void* stream) {
  const int rc = swiglu_a8_check(h, h, q8, e8, rows, F);
  if (rc != DET_OK) return rc;
  if (qh && !s_q) return DET_ERR_ARG;
  if ((uintptr_t)qh & 7u) return DET_ERR_ALIGN;
  if (rows == 0) return DET_OK;
  swiglu_a8_fwd<true>(nullptr, const_cast<int8_t*>(q8), const_cast<uint8_t*>(e8), rows, F, h, s_q, qh, (cudaStream_t)stream);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
extern "C" int det_swiglu_bwd_act8(const det_bf16* dh, const int8_t* q8, const uint8_t* e8, int rows, int F, det_bf16* dgu, void* stream) {
  const int rc = swiglu_a8_check(dh, dgu, q8, e8, rows, F);
  if (rc != DET_OK || rows == 0) return rc;
  const uint32_t pieces = (uint32_t)rows * (F / 8);
  const bool tab = sg_by_table(pieces);
  launch_after(tab ? k_swiglu_bwd_a8<2> : k_swiglu_bwd_a8<0>, tab ? SG_CTAS * dev_sm_count() : blocks_for(pieces, 256), 256, 0, (cudaStream_t)stream, dh,
               q8, e8, Divider(F / 8), pieces, F, dgu);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
