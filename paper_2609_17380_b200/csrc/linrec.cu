// Gated linear recurrence over the rows of a sequence, per channel, forward and backward:
//   f = 1 / (1 + exp(-g)), z = 1 - f,   h_t = f_t h_{t-1} + z_t v_t   (a row with a cut starts from 0 instead of h_{t-1})
//   dh_t = dy_t + f_{t+1} dh_{t+1},  dv = dh z,  dg = dh (h_{t-1} - v) f z
// f and z come from one exponential: with e = exp(-|g|) the smaller of them is m = e / (1 + e) and the larger 1 - m, so neither
// loses digits where the gate saturates.
//
// Order of the sums.  A span of rows is the map s -> A s + H.  A sequence is cut into blocks of 64 rows, a block into chunks of 8.  Chunk maps are
// composed row by row from the identity; the maps of the chunks before a chunk, from the block's start on, one after the other; the state at
// a block's start is the block map applied to the state at the start of the block before; the state at a chunk's start is the map of the
// chunks before it applied to that; inside a chunk the recurrence is walked row by row.  A map with A = 0 lets nothing in, not even
// a NaN.  The backward pass is the same from the last row to the first.  None of it depends on how blocks are dealt out.
//
// A warp walks a chunk of 64 channels (two a lane), a CTA of eight warps a block; the CTAs of a cluster take adjacent blocks, hand each other their
// block maps through distributed shared memory, one cluster barrier per round, and every CTA applies the maps of the blocks before its own.
// So every value is read once and written once however long a sequence is and however few there are, with no workspace.
#include "common.cuh"
#include "internal.h"

namespace det {

constexpr int LR_CHUNK = 8, LR_WARPS = 8, LR_BLOCK = LR_CHUNK * LR_WARPS, LR_MAXC = 8, LR_CH = 64;

// The gate of a bf16 has few arguments: the magnitudes from 2^-26 (e rounds to 1 below it) to 128 (e flushes to 0 long before), 33 exponents of
// 128 fractions.  A CTA with many rows evaluates them all once into shared memory: a lookup instead of an exponential and a
// division for every value.
constexpr uint32_t LR_LOW = 0x3280u, LR_TOP = 0x4300u;
constexpr int LR_TAB = LR_TOP - LR_LOW + 1;

__device__ __forceinline__ float lr_minor(float g) {
  const float e = det_exp_le0(-fabsf(g));
  return fdiv(e, fadd(1.0f, e));
}
__device__ __forceinline__ void lr_gate(float m, uint32_t negative, float& f, float& z) {
  const float M = fsub(1.0f, m);
  f = negative ? m : M;
  z = negative ? M : m;
}
// gates of the two channels in one word
template <bool TAB>
__device__ __forceinline__ void lr_gate2(uint32_t w, const float* tab, float f[2], float z[2]) {
  float m0, m1;
  if (TAB) {
    m0 = tab[min(max(w & 0x7fffu, LR_LOW), LR_TOP) - LR_LOW];
    m1 = tab[min(max((w >> 16) & 0x7fffu, LR_LOW), LR_TOP) - LR_LOW];
    if ((w & 0x7fffu) > 0x7f80u) m0 = __int_as_float(0x7fffffff);
    if (((w >> 16) & 0x7fffu) > 0x7f80u) m1 = __int_as_float(0x7fffffff);
  } else {
    m0 = lr_minor(bflo(w));
    m1 = lr_minor(bfhi(w));
  }
  lr_gate(m0, w & 0x8000u, f[0], z[0]);
  lr_gate(m1, w & 0x80000000u, f[1], z[1]);
}
struct LrMap { float2 a, h; };                           // s -> a s + h for two channels
__device__ __forceinline__ float lr_apply1(float a, float h, float s) { return a == 0.0f ? h : fadd(fmul(a, s), h); }
__device__ __forceinline__ float2 lr_apply(const LrMap& m, float2 s) { return make_float2(lr_apply1(m.a.x, m.h.x, s.x), lr_apply1(m.a.y, m.h.y, s.y)); }
// the map `first`, then `then`
__device__ __forceinline__ LrMap lr_compose(const LrMap& first, const LrMap& then) {
  LrMap r;
  r.h = lr_apply(then, first.h);
  r.a = make_float2(then.a.x == 0.0f ? 0.0f : fmul(first.a.x, then.a.x), then.a.y == 0.0f ? 0.0f : fmul(first.a.y, then.a.y));
  return r;
}
__device__ __forceinline__ float4 lr_pack(const LrMap& m) { return make_float4(m.a.x, m.a.y, m.h.x, m.h.y); }
__device__ __forceinline__ LrMap lr_unpack(float4 v) { return LrMap{make_float2(v.x, v.y), make_float2(v.z, v.w)}; }

struct LrShared {
  float4 chunk[LR_WARPS][32];                            // the CTA's chunk maps of this round
  float4 block[2][LR_MAXC][32];                          // block maps of the cluster, by rank; two rounds
  float tab[LR_TAB];
};
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void store_in_cluster(const void* local, int rank, float4 v) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(local)), "r"(rank));
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(a), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void lr_table(LrShared& sh) {
  for (int i = threadIdx.x; i < LR_TAB; i += LR_WARPS * 32) sh.tab[i] = lr_minor(__uint_as_float((LR_LOW + i) << 16));
  __syncthreads();
}

struct LrArgs {
  const uint16_t *g, *v, *dy;
  const uint8_t* flags;
  const float *first, *states;                           // state before the first row, or gradient of the state behind the last one
  uint16_t *y, *dg, *dv;
  float *last, *save;                                    // what comes out at the other end; states at the starts of the blocks
  size_t ld, ld_y, ld_d;
  int S, D, strips, nb, cl;                              // cl: CTAs of a cluster
};

// What the threads of a warp need to know of their chunk
struct LrPlace {
  int b, c0, rank, warp, lane;                           // sequence, first channel of the lane, rank in the cluster
  bool have;                                             // the lane's channels exist
};
__device__ __forceinline__ LrPlace lr_place(const LrArgs& p) {
  LrPlace r;
  r.rank = blockIdx.x % p.cl;
  const int q = blockIdx.x / p.cl;
  r.b = q / p.strips;
  r.warp = threadIdx.x >> 5;
  r.lane = threadIdx.x & 31;
  r.c0 = (q % p.strips) * LR_CH + 2 * r.lane;
  r.have = r.c0 < p.D;
  return r;
}
// bit i: row i of the chunk that starts at row t0 has a cut
template <bool FLAGS>
__device__ __forceinline__ uint32_t lr_cuts(const LrArgs& p, const LrPlace& at, int t0) {
  if (!FLAGS) return 0;
  const int t = t0 + at.lane;
  return __ballot_sync(0xffffffffu, at.lane < LR_CHUNK && t < p.S && p.flags[(size_t)at.b * p.S + t] != 0);
}
__device__ __forceinline__ void lr_load(const uint16_t* x, size_t ld, const LrArgs& p, const LrPlace& at, int t0, uint32_t w[LR_CHUNK]) {
  const uint16_t* q = x + ((size_t)at.b * p.S + t0) * ld + at.c0;
#pragma unroll
  for (int i = 0; i < LR_CHUNK; ++i) w[i] = at.have && t0 + i < p.S ? __ldg(reinterpret_cast<const uint32_t*>(q + i * ld)) : 0u;
}
// The round's hand-over: this warp's chunk map in, the map of the chunks before it out; `s`, the state at the start of the round, becomes
// the one at the start of the next round, and the state at the start of this CTA's block is returned.  `chunks` of the block exist, `blocks`
// of the round; chunk `k` of the order is walked by this warp.
__device__ __forceinline__ float2 lr_hand_over(LrShared& sh, const LrArgs& p, const LrPlace& at, int round, int k, int chunks, int blocks,
                                               const LrMap& mine, LrMap& before, float2& s) {
  sh.chunk[k][at.lane] = lr_pack(mine);
  __syncthreads();
  if (k > 0 && chunks > 0) {
    before = lr_unpack(sh.chunk[0][at.lane]);
    for (int i = 1; i < min(k, chunks); ++i) before = lr_compose(before, lr_unpack(sh.chunk[i][at.lane]));
    if (k == LR_WARPS - 1) {
      const float4 whole = lr_pack(chunks == LR_WARPS ? lr_compose(before, mine) : before);
      if (p.cl == 1) sh.block[round & 1][0][at.lane] = whole;
      else
        for (int r = 0; r < p.cl; ++r) store_in_cluster(&sh.block[round & 1][at.rank][at.lane], r, whole);
    }
  }
  if (p.cl == 1) {
    __syncthreads();
  } else {
    cluster_arrive();
    cluster_wait();
  }
  float2 start = s;
  for (int r = 0; r < blocks; ++r) {
    s = lr_apply(lr_unpack(sh.block[round & 1][r][at.lane]), s);
    if (r + 1 == at.rank) start = s;
  }
  return start;
}

template <bool TAB, bool FLAGS>
__global__ void __launch_bounds__(LR_WARPS * 32, 3) k_linrec_fwd(const __grid_constant__ LrArgs p) {
  __shared__ LrShared sh;
  const LrPlace at = lr_place(p);
  if (p.cl > 1) cluster_arrive();                        // every CTA has started before another one writes to its shared memory
  if (TAB) lr_table(sh);
  grid_dep();
  uint32_t wg[LR_CHUNK], wv[LR_CHUNK];
  int t0 = (at.rank * LR_WARPS + at.warp) * LR_CHUNK;
  lr_load(p.g, p.ld, p, at, t0, wg);
  lr_load(p.v, p.ld, p, at, t0, wv);
  float2 s = make_float2(0.0f, 0.0f);
  if (p.first && at.have) s = *reinterpret_cast<const float2*>(p.first + (size_t)at.b * p.D + at.c0);
  __syncwarp();
  if (p.cl > 1) cluster_wait();
  const int rounds = (p.nb + p.cl - 1) / p.cl;
  for (int k = 0; k < rounds; ++k, t0 += p.cl * LR_BLOCK) {
    const int blk = k * p.cl + at.rank, b0 = blk * LR_BLOCK;
    const int chunks = max(0, min(LR_WARPS, (p.S - b0 + LR_CHUNK - 1) / LR_CHUNK)), n = p.S - t0;     // n rows of the chunk exist
    const uint32_t cuts = lr_cuts<FLAGS>(p, at, t0);
    float f[LR_CHUNK][2], u[LR_CHUNK][2];
    LrMap mine;
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) {
      float z[2];
      lr_gate2<TAB>(wg[i], sh.tab, f[i], z);
      u[i][0] = fmul(z[0], bflo(wv[i]));
      u[i][1] = fmul(z[1], bfhi(wv[i]));
      const bool cut = FLAGS && (cuts >> i) & 1;
      if (i == 0) {
        mine.a = cut ? make_float2(0.0f, 0.0f) : make_float2(f[0][0], f[0][1]);
        mine.h = make_float2(u[0][0], u[0][1]);
      } else if (i < n) {
        mine.a = cut ? make_float2(0.0f, 0.0f) : make_float2(fmul(mine.a.x, f[i][0]), fmul(mine.a.y, f[i][1]));
        mine.h = cut ? make_float2(u[i][0], u[i][1]) : make_float2(fadd(fmul(f[i][0], mine.h.x), u[i][0]), fadd(fmul(f[i][1], mine.h.y), u[i][1]));
      }
    }
    const int tn = t0 + p.cl * LR_BLOCK;                 // the loads of the next round are under way while this one is handed over
    lr_load(p.g, p.ld, p, at, tn, wg);
    lr_load(p.v, p.ld, p, at, tn, wv);
    LrMap before = mine;
    const float2 start = lr_hand_over(sh, p, at, k, at.warp, chunks, min(p.cl, p.nb - k * p.cl), mine, before, s);
    if (p.save && at.warp == 0 && n > 0 && at.have) *reinterpret_cast<float2*>(p.save + ((size_t)at.b * p.nb + blk) * p.D + at.c0) = start;
    float2 h = at.warp ? lr_apply(before, start) : start;
    uint16_t* out = p.y + ((size_t)at.b * p.S + t0) * p.ld_y + at.c0;
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) {
      const bool cut = FLAGS && (cuts >> i) & 1;
      h = cut ? make_float2(u[i][0], u[i][1]) : make_float2(fadd(fmul(f[i][0], h.x), u[i][0]), fadd(fmul(f[i][1], h.y), u[i][1]));
      if (i < n && at.have) *reinterpret_cast<uint32_t*>(out + i * p.ld_y) = pack_bf2(h.x, h.y);
    }
    __syncwarp();
  }
  if (p.last && at.have && at.rank == 0 && at.warp == 0) *reinterpret_cast<float2*>(p.last + (size_t)at.b * p.D + at.c0) = s;
}

template <bool TAB, bool FLAGS>
__global__ void __launch_bounds__(LR_WARPS * 32, 2) k_linrec_bwd(const __grid_constant__ LrArgs p) {
  __shared__ LrShared sh;
  __shared__ float4 ahead[LR_WARPS][32];                 // the chunk maps of the forward recurrence
  const LrPlace at = lr_place(p);
  if (p.cl > 1) cluster_arrive();
  if (TAB) lr_table(sh);
  grid_dep();
  uint32_t wg[LR_CHUNK] = {}, wv[LR_CHUNK] = {}, wd[LR_CHUNK] = {};
  float2 s = make_float2(0.0f, 0.0f);
  if (p.first && at.have) s = *reinterpret_cast<const float2*>(p.first + (size_t)at.b * p.D + at.c0);
  __syncwarp();
  if (p.cl > 1) cluster_wait();
  const int rounds = (p.nb + p.cl - 1) / p.cl;
  for (int k = 0; k < rounds; ++k) {
    const int blk = p.nb - 1 - (k * p.cl + at.rank), b0 = blk * LR_BLOCK;         // from the last block to the first; below 0: none
    const int chunks = blk < 0 ? 0 : min(LR_WARPS, (p.S - b0 + LR_CHUNK - 1) / LR_CHUNK);
    const int t0 = b0 + at.warp * LR_CHUNK, n = blk < 0 ? 0 : p.S - t0;
    uint32_t cuts = 0;
    float2 state = make_float2(0.0f, 0.0f);
    if (blk >= 0) {
      lr_load(p.g, p.ld, p, at, t0, wg);
      lr_load(p.v, p.ld, p, at, t0, wv);
      lr_load(p.dy, p.ld_y, p, at, t0, wd);
      if (at.have) state = *reinterpret_cast<const float2*>(p.states + ((size_t)at.b * p.nb + blk) * p.D + at.c0);
      __syncwarp();
      cuts = lr_cuts<FLAGS>(p, at, t0);
    }
    float f[LR_CHUNK][2], z[LR_CHUNK][2];
    LrMap mine, fore;                                    // of the gradient, of the state
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) {
      lr_gate2<TAB>(wg[i], sh.tab, f[i], z[i]);
      const bool cut = FLAGS && (cuts >> i) & 1;
      const float2 u = make_float2(fmul(z[i][0], bflo(wv[i])), fmul(z[i][1], bfhi(wv[i])));
      if (i == 0) {
        fore.a = cut ? make_float2(0.0f, 0.0f) : make_float2(f[0][0], f[0][1]);
        fore.h = u;
      } else if (i < n) {
        fore.a = cut ? make_float2(0.0f, 0.0f) : make_float2(fmul(fore.a.x, f[i][0]), fmul(fore.a.y, f[i][1]));
        fore.h = cut ? u : make_float2(fadd(fmul(f[i][0], fore.h.x), u.x), fadd(fmul(f[i][1], fore.h.y), u.y));
      }
    }
    bool any = false;
    mine.a = mine.h = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = LR_CHUNK - 1; i >= 0; --i) {
      if (i >= n) continue;
      const bool cut = FLAGS && (cuts >> i) & 1;
      const float2 d = make_float2(bflo(wd[i]), bfhi(wd[i]));
      if (!any) {
        mine.a = make_float2(f[i][0], f[i][1]);
        mine.h = make_float2(fmul(f[i][0], d.x), fmul(f[i][1], d.y));
      } else {
        mine.a = make_float2(fmul(f[i][0], mine.a.x), fmul(f[i][1], mine.a.y));
        mine.h = make_float2(fmul(f[i][0], fadd(d.x, mine.h.x)), fmul(f[i][1], fadd(d.y, mine.h.y)));
      }
      if (cut) mine.a = mine.h = make_float2(0.0f, 0.0f);
      any = true;
    }
    ahead[at.warp][at.lane] = lr_pack(fore);
    LrMap behind = mine;
    // the order of the backward pass: chunk 0 is the block's last one that exists; warps beyond the end stay behind it
    const int order = at.warp < chunks ? chunks - 1 - at.warp : at.warp;
    const float2 start = lr_hand_over(sh, p, at, k, order, chunks, min(p.cl, p.nb - k * p.cl), mine, behind, s);
    if (n > 0 && at.have) {
      float2 h = state;
      if (at.warp) {
        LrMap before = lr_unpack(ahead[0][at.lane]);
        for (int i = 1; i < at.warp; ++i) before = lr_compose(before, lr_unpack(ahead[i][at.lane]));
        h = lr_apply(before, state);
      }
      float2 prev[LR_CHUNK];
#pragma unroll
      for (int i = 0; i < LR_CHUNK; ++i) {
        const bool cut = FLAGS && (cuts >> i) & 1;
        prev[i] = cut ? make_float2(0.0f, 0.0f) : h;
        const float2 u = make_float2(fmul(z[i][0], bflo(wv[i])), fmul(z[i][1], bfhi(wv[i])));
        h = cut ? u : make_float2(fadd(fmul(f[i][0], h.x), u.x), fadd(fmul(f[i][1], h.y), u.y));
      }
      float2 c = order ? lr_apply(behind, start) : start;
      const size_t o = ((size_t)at.b * p.S + t0) * p.ld_d + at.c0;
#pragma unroll
      for (int i = LR_CHUNK - 1; i >= 0; --i) {
        if (i >= n) continue;
        const bool cut = FLAGS && (cuts >> i) & 1;
        const float2 d = make_float2(fadd(bflo(wd[i]), c.x), fadd(bfhi(wd[i]), c.y));
        c = cut ? make_float2(0.0f, 0.0f) : make_float2(fmul(f[i][0], d.x), fmul(f[i][1], d.y));
        *reinterpret_cast<uint32_t*>(p.dv + o + i * p.ld_d) = pack_bf2(fmul(d.x, z[i][0]), fmul(d.y, z[i][1]));
        *reinterpret_cast<uint32_t*>(p.dg + o + i * p.ld_d) =
            pack_bf2(fmul(fmul(d.x, fsub(prev[i].x, bflo(wv[i]))), fmul(f[i][0], z[i][0])),
                     fmul(fmul(d.y, fsub(prev[i].y, bfhi(wv[i]))), fmul(f[i][1], z[i][1])));
      }
    }
    __syncthreads();                                     // `ahead` is read by then
  }
  if (p.last && at.have && at.rank == 0 && at.warp == 0) *reinterpret_cast<float2*>(p.last + (size_t)at.b * p.D + at.c0) = s;
}

// CTAs of a cluster: enough for the GPU to be covered `waves` times by the strips and sequences there are, no more than there are blocks
static int lr_cluster(int chains, int nb, int waves) {
  int cl = 1;
  while (cl < LR_MAXC && 2 * cl <= nb && (long long)chains * 2 * cl <= (long long)waves * dev_sm_count()) cl *= 2;
  return cl;
}
static int lr_launch(void (*kern)(const LrArgs), const LrArgs& p, long long ctas, cudaStream_t st) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.cl;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(LR_WARPS * 32);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = p.cl > 1 ? 2 : 1;
  note_launch();
  cudaLaunchKernelEx(&cfg, kern, p);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
static int lr_check(const void* a, const void* b, int ld, int B, int S, int D) {
  if (!a || !b || B < 0 || S < 0 || D <= 0 || ld < D) return DET_ERR_ARG;
  if (D % 2 || ld % 2 || S > (1 << 30)) return DET_ERR_SHAPE;
  if ((long long)B * ((D + LR_CH - 1) / LR_CH) > (1 << 27)) return DET_ERR_SHAPE;
  if (((uintptr_t)a | (uintptr_t)b) & 3u) return DET_ERR_ALIGN;
  return DET_OK;
}
// the state passes through where there are no rows
static int lr_empty(const float* in, float* out, size_t n, cudaStream_t st) {
  if (!out || out == in || n == 0) return DET_OK;
  const cudaError_t rc = in ? cudaMemcpyAsync(out, in, n * sizeof(float), cudaMemcpyDeviceToDevice, st) : cudaMemsetAsync(out, 0, n * sizeof(float), st);
  return rc == cudaSuccess ? DET_OK : DET_ERR_CUDA;
}

}  // namespace det

using namespace det;

extern "C" size_t det_linrec_state_floats(int B, int S, int D) {
  return B > 0 && S > 0 && D > 0 ? (size_t)B * (((size_t)S + LR_BLOCK - 1) / LR_BLOCK) * (size_t)D : 0;
}

extern "C" int det_linrec_fwd(const det_bf16* g, const det_bf16* v, int ld, int B, int S, int D, det_bf16* y, int ld_y, const uint8_t* flags,
                              const float* h0, float* hT, float* states, void* stream) {
  const int rc = lr_check(g, v, ld, B, S, D);
  if (rc != DET_OK) return rc;
  if (!y || ld_y < D) return DET_ERR_ARG;
  if (ld_y % 2) return DET_ERR_SHAPE;
  if (((uintptr_t)y & 3u) || (((uintptr_t)h0 | (uintptr_t)hT | (uintptr_t)states) & 7u)) return DET_ERR_ALIGN;
  cudaStream_t st = (cudaStream_t)stream;
  if (B == 0 || S == 0) return lr_empty(h0, hT, (size_t)B * D, st);
  LrArgs p = {};
  p.g = g; p.v = v; p.flags = flags; p.first = h0; p.y = y; p.last = hT; p.save = states;
  p.ld = ld; p.ld_y = ld_y; p.S = S; p.D = D;
  p.strips = (D + LR_CH - 1) / LR_CH;
  p.nb = (S + LR_BLOCK - 1) / LR_BLOCK;
  p.cl = lr_cluster(B * p.strips, p.nb, 3);
  const bool tab = p.nb / p.cl >= 4;
  auto kern = tab ? (flags ? k_linrec_fwd<true, true> : k_linrec_fwd<true, false>) : (flags ? k_linrec_fwd<false, true> : k_linrec_fwd<false, false>);
  return lr_launch(kern, p, (long long)B * p.strips * p.cl, st);
}

extern "C" int det_linrec_bwd(const det_bf16* dy, int ld_y, const det_bf16* g, const det_bf16* v, int ld, int B, int S, int D,
                              const float* states, det_bf16* dg, det_bf16* dv, int ld_d, const uint8_t* flags, const float* dhT, float* dh0,
                              void* stream) {
  const int rc = lr_check(g, v, ld, B, S, D);
  if (rc != DET_OK) return rc;
  if (!dy || ld_y < D || !dg || !dv || ld_d < D || (!states && B > 0 && S > 0)) return DET_ERR_ARG;
  if (ld_y % 2 || ld_d % 2) return DET_ERR_SHAPE;
  if ((((uintptr_t)dy | (uintptr_t)dg | (uintptr_t)dv) & 3u) || (((uintptr_t)dhT | (uintptr_t)dh0 | (uintptr_t)states) & 7u)) return DET_ERR_ALIGN;
  cudaStream_t st = (cudaStream_t)stream;
  if (B == 0 || S == 0) return lr_empty(dhT, dh0, (size_t)B * D, st);
  LrArgs p = {};
  p.g = g; p.v = v; p.dy = dy; p.flags = flags; p.first = dhT; p.states = states; p.dg = dg; p.dv = dv; p.last = dh0;
  p.ld = ld; p.ld_y = ld_y; p.ld_d = ld_d; p.S = S; p.D = D;
  p.strips = (D + LR_CH - 1) / LR_CH;
  p.nb = (S + LR_BLOCK - 1) / LR_BLOCK;
  p.cl = lr_cluster(B * p.strips, p.nb, 2);
  const bool tab = p.nb / p.cl >= 4;
  auto kern = tab ? (flags ? k_linrec_bwd<true, true> : k_linrec_bwd<true, false>) : (flags ? k_linrec_bwd<false, true> : k_linrec_bwd<false, false>);
  return lr_launch(kern, p, (long long)B * p.strips * p.cl, st);
}
