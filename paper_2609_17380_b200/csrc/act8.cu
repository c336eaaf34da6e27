// Activations kept in 8 bits between the forward and the backward pass: storing and restoring them, and SwiGLU from and to them.
// The format (rows.cuh) has a power-of-two step for every 32 adjacent values of a row, so nothing here rounds but the code itself.
// All of it is bound by memory: every value is read and written once, eight a thread.
#include "common.cuh"
#include "internal.h"
#include "rows.cuh"

namespace det {

// Rows of a multiple of 8 columns, 16-byte aligned: a lane has eight adjacent values, four lanes a group.
template <bool BF>
__global__ void __launch_bounds__(256) k_a8_pack(const void* __restrict__ x, size_t ld, int rows, int D, int8_t* __restrict__ q,
                                                 uint8_t* __restrict__ e) {
  grid_dep();
  const size_t lanes = (size_t)((D + A8_GROUP - 1) / A8_GROUP) * 4;          // per row, the last group's whole four included
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  const size_t r = i / lanes, c = (i % lanes) * 8;
  const bool have = r < (size_t)rows && c < (size_t)D;
  float v[8];
  load8n<BF>(x, r * ld + c, have, v);
  const uint32_t field = a8_field(a8_quad_max(a8_amax8(v)));
  if (!have) return;
  *reinterpret_cast<uint2*>(q + r * D + c) = a8_codes8(v, field);
  if ((i & 3) == 0) e[i / 4] = (uint8_t)field;
}
template <bool BF>
__global__ void __launch_bounds__(256) k_a8_unpack(const int8_t* __restrict__ q, const uint8_t* __restrict__ e, int rows, int D,
                                                   void* __restrict__ y, size_t ld) {
  grid_dep();
  const size_t lanes = (size_t)D / 8;
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  const size_t r = i / lanes, c = (i % lanes) * 8;
  if (r >= (size_t)rows) return;
  float v[8];
  a8_values8(*reinterpret_cast<const uint2*>(q + r * D + c), a8_step(e[r * ((D + A8_GROUP - 1) / A8_GROUP) + c / A8_GROUP]), v);
  store8<BF>(y, r * ld + c, v);
}
// Any width, stride and address: a warp per group, a lane per value.
template <bool BF>
__global__ void __launch_bounds__(256) k_a8_pack_any(const void* __restrict__ x, size_t ld, int rows, int D, int8_t* __restrict__ q,
                                                     uint8_t* __restrict__ e) {
  grid_dep();
  const size_t ng = (D + A8_GROUP - 1) / A8_GROUP, w = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  const size_t r = w / ng, c = (w % ng) * A8_GROUP + lane;
  if (r >= (size_t)rows) return;
  const bool have = c < (size_t)D;
  const float v = have ? (BF ? bf2f(reinterpret_cast<const uint16_t*>(x)[r * ld + c]) : reinterpret_cast<const float*>(x)[r * ld + c]) : 0.0f;
  const uint32_t field = a8_field(__reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7fffffffu));
  if (have) q[r * D + c] = (int8_t)(field != 255u ? __float_as_uint(fadd(fmul(v, a8_inv(field)), 12582912.0f)) : a8_code_nonfinite(v));
  if (lane == 0) e[w] = (uint8_t)field;
}
template <bool BF>
__global__ void __launch_bounds__(256) k_a8_unpack_any(const int8_t* __restrict__ q, const uint8_t* __restrict__ e, int rows, int D,
                                                       void* __restrict__ y, size_t ld) {
  grid_dep();
  const size_t ng = (D + A8_GROUP - 1) / A8_GROUP, w = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const size_t r = w / ng, c = (w % ng) * A8_GROUP + (threadIdx.x & 31);
  if (r >= (size_t)rows || c >= (size_t)D) return;
  const float v = fmul((float)q[r * D + c], a8_step(e[w]));
  if (BF) reinterpret_cast<uint16_t*>(y)[r * ld + c] = f2bf(v);
  else reinterpret_cast<float*>(y)[r * ld + c] = v;
}

// ---- SwiGLU: gu [rows, 2F] = (gate | up), F a multiple of 32, so no group holds both -----------------------
__device__ __forceinline__ float sigmoid_a8(float g) { return fdiv(1.0f, fadd(1.0f, det_exp(-g))); }

// FROM: gate and up come from the checkpoint (gu absent), else they come from gu and the checkpoint is written
template <bool FROM>
__global__ void __launch_bounds__(256) k_swiglu_fwd_a8(const uint16_t* __restrict__ gu, int8_t* q, uint8_t* e, int rows, int F,
                                                       uint16_t* __restrict__ h, const float* __restrict__ s_q, int8_t* __restrict__ qh) {
  grid_dep();
  const size_t lanes = (size_t)F / 8, i = (size_t)blockIdx.x * 256 + threadIdx.x;
  const bool have = i < lanes * rows;
  const size_t r = have ? i / lanes : 0, c = have ? (i % lanes) * 8 : 0, at = r * 2 * F + c;
  float g[8], u[8], o[8];
  if (FROM) {
    if (!have) return;
    a8_values8(*reinterpret_cast<const uint2*>(q + at), a8_step(e[at / A8_GROUP]), g);
    a8_values8(*reinterpret_cast<const uint2*>(q + at + F), a8_step(e[(at + F) / A8_GROUP]), u);
  } else {
    load8n<true>(gu, at, have, g);
    load8n<true>(gu, at + F, have, u);
    const uint32_t fg = a8_field(a8_quad_max(a8_amax8(g))), fu = a8_field(a8_quad_max(a8_amax8(u)));
    if (!have) return;
    *reinterpret_cast<uint2*>(q + at) = a8_codes8(g, fg);
    *reinterpret_cast<uint2*>(q + at + F) = a8_codes8(u, fu);
    if ((i & 3) == 0) {
      e[at / A8_GROUP] = (uint8_t)fg;
      e[(at + F) / A8_GROUP] = (uint8_t)fu;
    }
  }
#pragma unroll
  for (int t = 0; t < 8; ++t) o[t] = fmul(fmul(g[t], sigmoid_a8(g[t])), u[t]);
  store8<true>(h, r * F + c, o);
  if (qh) {   // the next linear's quantiser, applied to the bf16 values just stored
    const float inv_q = fdiv(1.0f, s_q[0]);
#pragma unroll
    for (int t = 0; t < 8; ++t) o[t] = bf2f(f2bf(o[t]));
    *reinterpret_cast<uint2*>(qh + r * F + c) = quant8(o, inv_q);
  }
}
__global__ void __launch_bounds__(256) k_swiglu_bwd_a8(const uint16_t* __restrict__ dh, const int8_t* __restrict__ q,
                                                       const uint8_t* __restrict__ e, int rows, int F, uint16_t* __restrict__ dgu) {
  grid_dep();
  const size_t lanes = (size_t)F / 8, i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= lanes * rows) return;
  const size_t r = i / lanes, c = (i % lanes) * 8, at = r * 2 * F + c;
  float g[8], u[8], d[8], dg[8], du[8];
  a8_values8(*reinterpret_cast<const uint2*>(q + at), a8_step(e[at / A8_GROUP]), g);
  a8_values8(*reinterpret_cast<const uint2*>(q + at + F), a8_step(e[(at + F) / A8_GROUP]), u);
  load8<true>(dh, r * F + c, d);
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const float sg = sigmoid_a8(g[t]);
    du[t] = fmul(d[t], fmul(g[t], sg));
    dg[t] = fmul(fmul(d[t], u[t]), fmul(sg, fadd(1.0f, fmul(g[t], fsub(1.0f, sg)))));
  }
  store8<true>(dgu, at, dg);
  store8<true>(dgu, at + F, du);
}

static unsigned blocks_for(size_t threads) { return (unsigned)((threads + 255) / 256); }

}  // namespace det

using namespace det;

extern "C" size_t det_act8_exp_bytes(int rows, int D) {
  return rows > 0 && D > 0 ? (size_t)rows * (((size_t)D + A8_GROUP - 1) / A8_GROUP) : 0;
}

static int a8_check(int io, const void* x, int ld, int rows, int D, const void* q, const void* e) {
  if (!x || !q || !e || rows < 0 || D <= 0 || ld < D || (io != DET_F32 && io != DET_BF16)) return DET_ERR_ARG;
  if ((size_t)rows * (((size_t)D + 31) / 32) > ((size_t)1 << 33)) return DET_ERR_SHAPE;      // blocks of 8 warps in a grid
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
  const size_t groups = det_act8_exp_bytes(rows, D);
  if (a8_vec(io, x, ld, D, q8))
    launch_after(io == DET_BF16 ? k_a8_pack<true> : k_a8_pack<false>, blocks_for(groups * 4), 256, 0, st, x, (size_t)ld, rows, D, q8, e8);
  else
    launch_after(io == DET_BF16 ? k_a8_pack_any<true> : k_a8_pack_any<false>, blocks_for(groups * 32), 256, 0, st, x, (size_t)ld, rows, D, q8, e8);
  DET_CHECK_LAUNCH();
  return DET_OK;
}

extern "C" int det_act8_unpack(int io, const int8_t* q8, const uint8_t* e8, int rows, int D, void* y, int ld, void* stream) {
  const int rc = a8_check(io, y, ld, rows, D, q8, e8);
  if (rc != DET_OK || rows == 0) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  if (a8_vec(io, y, ld, D, q8))
    launch_after(io == DET_BF16 ? k_a8_unpack<true> : k_a8_unpack<false>, blocks_for((size_t)rows * (D / 8)), 256, 0, st, q8, e8, rows, D, y, (size_t)ld);
  else
    launch_after(io == DET_BF16 ? k_a8_unpack_any<true> : k_a8_unpack_any<false>, blocks_for(det_act8_exp_bytes(rows, D) * 32), 256, 0, st, q8, e8, rows, D, y, (size_t)ld);
  DET_CHECK_LAUNCH();
  return DET_OK;
}

static int swiglu_a8_check(const void* a, const void* b, const int8_t* q8, const uint8_t* e8, int rows, int F) {
  if (!a || !b || !q8 || !e8 || rows < 0 || F <= 0) return DET_ERR_ARG;
  if (F % 32 || F > (1 << 29) || (size_t)rows * (F / 8) > ((size_t)1 << 38)) return DET_ERR_SHAPE;
  if (!aligned16(a) || !aligned16(b) || ((uintptr_t)q8 & 7u)) return DET_ERR_ALIGN;
  return DET_OK;
}
extern "C" int det_swiglu_fwd_act8(const det_bf16* gu, int rows, int F, det_bf16* h, int8_t* q8, uint8_t* e8, const float* s_q, int8_t* qh,
                                   void* stream) {
  const int rc = swiglu_a8_check(gu, h, q8, e8, rows, F);
  if (rc != DET_OK) return rc;
  if (qh && !s_q) return DET_ERR_ARG;
  if ((uintptr_t)qh & 7u) return DET_ERR_ALIGN;
  if (rows == 0) return DET_OK;
  launch_after(k_swiglu_fwd_a8<false>, blocks_for((size_t)rows * (F / 8)), 256, 0, (cudaStream_t)stream, gu, q8, e8, rows, F, h, s_q, qh);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
extern "C" int det_swiglu_act8(const int8_t* q8, const uint8_t* e8, int rows, int F, det_bf16* h, const float* s_q, int8_t* qh, void* stream) {
  const int rc = swiglu_a8_check(h, h, q8, e8, rows, F);
  if (rc != DET_OK) return rc;
  if (qh && !s_q) return DET_ERR_ARG;
  if ((uintptr_t)qh & 7u) return DET_ERR_ALIGN;
  if (rows == 0) return DET_OK;
  launch_after(k_swiglu_fwd_a8<true>, blocks_for((size_t)rows * (F / 8)), 256, 0, (cudaStream_t)stream, nullptr, const_cast<int8_t*>(q8),
               const_cast<uint8_t*>(e8), rows, F, h, s_q, qh);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
extern "C" int det_swiglu_bwd_act8(const det_bf16* dh, const int8_t* q8, const uint8_t* e8, int rows, int F, det_bf16* dgu, void* stream) {
  const int rc = swiglu_a8_check(dh, dgu, q8, e8, rows, F);
  if (rc != DET_OK || rows == 0) return rc;
  launch_after(k_swiglu_bwd_a8, blocks_for((size_t)rows * (F / 8)), 256, 0, (cudaStream_t)stream, dh, q8, e8, rows, F, dgu);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
