// The sigmoid of a bf16 gate by table.
// A bf16 has few values whose sigmoid matters: 33 exponents of magnitude (below 2^-26 it is 1/2, from 128 on 1 or 0) of 128 fractions and two
// signs.  They are evaluated by the compiler, with the steps of the formula (1 / (1 + det_exp(-g))), and looked up in shared memory.
#pragma once
#include "common.cuh"

namespace det {

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
// the table into shared memory by the threads `at` of `threads`
template <int TAB>
__device__ __forceinline__ void sg_fill_table(float* tab, int at, int threads) {
  for (int i = at; i < 2 * SG_TAB / 4; i += threads) {
    const float4 v = reinterpret_cast<const float4*>(sg_table_image.v)[i];
    if (TAB == 2) {
      reinterpret_cast<float4*>(tab)[i] = v;
    } else {   // SG_TAB is a multiple of 256, so a place is undone in either half alike
      const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        int to = 4 * i + k;
        to ^= (to >> 3) & 28;                            // undoes the upper three of the five bits, which the lower two came from
        to ^= (to >> 3) & 3;
        tab[to] = w[k];
      }
    }
  }
}
// by all 256 threads of a CTA
template <int TAB>
__device__ __forceinline__ void sg_copy_table(float* tab) {
  if (!TAB) return;
  sg_fill_table<TAB>(tab, threadIdx.x, 256);
  __syncthreads();
}
}  // namespace det
