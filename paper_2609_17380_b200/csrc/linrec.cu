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
// A chunk is walked by a half or a whole warp, two channels a lane, so a CTA of eight warps has a strip of 64 channels and one block, or 32 channels
// and two blocks, a round.  The CTAs of a cluster take adjacent blocks, hand each other their block maps through distributed shared memory, one
// cluster barrier per round, and every CTA applies the maps of the blocks before its own.  So every value is read once and written
// once however long a sequence is and however few there are, with no workspace.  The raw values of the next round come in by asynchronous copies,
// each thread its own, while this round is handed over.
#include "common.cuh"
#include "internal.h"

namespace det {

constexpr int LR_CHUNK = 8, LR_CHUNKS = 8, LR_BLOCK = LR_CHUNK * LR_CHUNKS, LR_T = 256, LR_MAXC = 16;

// The gate of a bf16 has few arguments: the magnitudes from 2^-26 (e rounds to 1 below it) to 128 (e flushes to 0 long before), 33 exponents of
// 128 fractions.  A CTA with many rows evaluates them all once into shared memory: a lookup instead of an exponential and a
// division for every value.
constexpr int LR_LOW = 0x3280, LR_TOP = 0x4300, LR_TAB = LR_TOP - LR_LOW + 1;

__device__ __forceinline__ float lr_minor(float g) {
  const float e = det_exp_le0(-fabsf(g));
  return fdiv(e, fadd(1.0f, e));
}
__device__ __forceinline__ void lr_gate(float m, bool negative, float& f, float& z) {
  const float M = fsub(1.0f, m);
  f = negative ? m : M;
  z = negative ? M : m;
}
// gates of the two channels in one word; a NaN is looked up as an infinity: lr_gates puts it right
template <bool TAB>
__device__ __forceinline__ void lr_gate2(uint32_t w, const float* tab, float f[2], float z[2]) {
  const char* t = reinterpret_cast<const char*>(tab);
  const float m0 = TAB ? *reinterpret_cast<const float*>(t + __vimin_s32_relu((int)((w << 2) & 0x1fffcu) - 4 * LR_LOW, 4 * (LR_TAB - 1))) : lr_minor(bflo(w));
  const float m1 = TAB ? *reinterpret_cast<const float*>(t + __vimin_s32_relu((int)((w >> 14) & 0x1fffcu) - 4 * LR_LOW, 4 * (LR_TAB - 1))) : lr_minor(bfhi(w));
  lr_gate(m0, w & 0x8000u, f[0], z[0]);
  lr_gate(m1, (int)w < 0, f[1], z[1]);
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
__device__ __forceinline__ float2 lr_step(const float f[2], const float2 u, float2 h, bool cut) {
  return cut ? u : make_float2(fadd(fmul(f[0], h.x), u.x), fadd(fmul(f[1], h.y), u.y));
}
// row i of a map that has come to `m` (i == 0: the map of the row alone); rows from the n-th on do not exist
__device__ __forceinline__ void lr_extend(LrMap& m, int i, int n, const float f[2], const float2 u, bool cut) {
  if (i >= n && i > 0) return;
  const float2 a = i ? make_float2(fmul(m.a.x, f[0]), fmul(m.a.y, f[1])) : make_float2(f[0], f[1]);
  m.h = i ? lr_step(f, u, m.h, cut) : u;
  m.a = cut ? make_float2(0.0f, 0.0f) : a;
}

// NS: tensors that come in by asynchronous copies
template <int NS>
struct LrShared {
  uint32_t raw[2][NS][LR_CHUNK][LR_T];                   // two rounds
  float4 chunk[LR_T];                                    // [chunk of the CTA][lane of it]: the chunk maps of this round
  float4 block[2][LR_MAXC * 32];                         // [block of the round][lane]: block maps of the cluster; two rounds
  float4 ahead[NS == 3 ? LR_T : 1];                      // backward: the chunk maps of the recurrence itself
  float tab[LR_TAB];
};
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void store_in_cluster(const void* local, int rank, float4 v) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(local)), "r"(rank));
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(a), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
// four bytes, or zero where there is nothing
__device__ __forceinline__ void copy4(uint32_t* dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copies_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

template <int NS>
__device__ __forceinline__ void lr_table(LrShared<NS>& sh) {
  for (int i = threadIdx.x; i < LR_TAB; i += LR_T) sh.tab[i] = lr_minor(__uint_as_float((uint32_t)(LR_LOW + i) << 16));
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

// Where a thread is.  CH channels a CTA: CH / 2 lanes a chunk, BLOCKS blocks a round.
template <int CH>
struct LrPlace {
  static constexpr int LANES = CH / 2, BLOCKS = 64 / CH;
  int b, c0, rank, blk, k, lane;                         // sequence, first channel; block of the CTA's, chunk of the block, lane of the chunk
  bool have;                                             // the lane's channels exist
  __device__ __forceinline__ LrPlace(const LrArgs& p) {
    rank = blockIdx.x % p.cl;
    const int q = blockIdx.x / p.cl;
    b = q / p.strips;
    lane = threadIdx.x % LANES;
    const int chunk = threadIdx.x / LANES;
    blk = chunk / LR_CHUNKS;
    k = chunk % LR_CHUNKS;
    c0 = (q % p.strips) * CH + 2 * lane;
    have = c0 < p.D;
  }
};
// this thread's rows of a tensor on their way: `there` of them (0: none, its address is not followed)
__device__ __forceinline__ void lr_fetch(uint32_t (*raw)[LR_T], const uint16_t* x, size_t ld, size_t row, int c0, int there) {
  const uint16_t* q = there > 0 ? x + row * ld + c0 : x;
#pragma unroll
  for (int i = 0; i < LR_CHUNK; ++i) copy4(&raw[i][threadIdx.x], i < there ? q + i * ld : x, i < there);
}
// the flag of row (lane of the chunk) of a chunk of n rows, and from the flags of the warp the cuts of this thread's chunk
template <int CH, bool FLAGS>
__device__ __forceinline__ bool lr_flag(const LrArgs& p, const LrPlace<CH>& at, int t0, int n) {
  return FLAGS && at.lane < min(n, LR_CHUNK) && p.flags[(size_t)at.b * p.S + t0 + at.lane] != 0;
}
template <int CH, bool FLAGS>
__device__ __forceinline__ uint32_t lr_cuts(bool flag) {
  if (!FLAGS) return 0;
  return __ballot_sync(0xffffffffu, flag) >> ((threadIdx.x & 31) & ~(CH / 2 - 1));
}
// The gates of a chunk.  By table a NaN gate comes out as one of an infinity: it makes its gate a NaN here.
template <bool TAB>
__device__ __forceinline__ void lr_gates(const uint32_t w[LR_CHUNK], const float* tab, float f[LR_CHUNK][2], float z[LR_CHUNK][2]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < LR_CHUNK; ++i) {
    lr_gate2<TAB>(w[i], tab, f[i], z[i]);
    if (TAB) top = __vmaxu2(top, w[i] & 0x7fff7fffu);
  }
  if (TAB && ((top & 0xffffu) > 0x7f80u || (top >> 16) > 0x7f80u)) {
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) {
      if ((w[i] & 0x7fffu) > 0x7f80u) f[i][0] = z[i][0] = __int_as_float(0x7fffffff);
      if (((w[i] >> 16) & 0x7fffu) > 0x7f80u) f[i][1] = z[i][1] = __int_as_float(0x7fffffff);
    }
  }
}
// the maps of the chunks of a block before chunk k, one after the other; k > 0, at most `chunks` exist
template <int LANES>
__device__ __forceinline__ LrMap lr_before(const float4* chunk, int k, int chunks) {
  LrMap m = lr_unpack(chunk[0]);
#pragma unroll
  for (int i = 1; i < LR_CHUNKS - 1; ++i) {
    const LrMap next = lr_unpack(chunk[i * LANES]);
    if (i < min(k, chunks)) m = lr_compose(m, next);
  }
  return m;
}
// The round's hand-over: this thread's chunk map in, the map of the chunks of its block before it out; `s`, the state at the start of the
// round, becomes the one at the start of the next round, and the state at the start of this thread's block is returned.  `chunks` of the
// block exist, `blocks` of the round; k is the chunk's place in the block in the order of the pass.
template <int CH, int NS>
__device__ __forceinline__ float2 lr_hand_over(LrShared<NS>& sh, const LrArgs& p, const LrPlace<CH>& at, int round, int k, int chunks, int blocks,
                                               const LrMap& mine, LrMap& before, float2& s) {
  constexpr int LANES = LrPlace<CH>::LANES, BLOCKS = LrPlace<CH>::BLOCKS;
  float4* chunk = sh.chunk + at.blk * LR_CHUNKS * LANES + at.lane;
  chunk[k * LANES] = lr_pack(mine);
  __syncthreads();
  float4* slots = sh.block[round & 1];
  before = mine;
  if (k > 0 && chunks > 0) before = lr_before<LANES>(chunk, k, chunks);
  if (k == LR_CHUNKS - 1 && chunks > 0) {
    const float4 whole = lr_pack(chunks == LR_CHUNKS ? lr_compose(before, mine) : before);
    float4* slot = slots + (at.rank * BLOCKS + at.blk) * LANES + at.lane;
    if (p.cl == 1) *slot = whole;
    else
      for (int r = 0; r < p.cl; ++r) store_in_cluster(slot, r, whole);
  }
  if (p.cl == 1) {
    __syncthreads();
  } else {
    // the barrier itself orders nothing: a release by every thread would wait for its stores of the round before
    if (__any_sync(0xffffffffu, k == LR_CHUNKS - 1)) asm volatile("fence.acq_rel.cluster;" ::: "memory");
    cluster_arrive();
    cluster_wait();
  }
  float2 start = s;
  const int own = at.rank * BLOCKS + at.blk;
#pragma unroll 4
  for (int r = 0; r < blocks; ++r) {
    if (r == own) start = s;
    s = lr_apply(lr_unpack(slots[r * LANES + at.lane]), s);
  }
  return start;
}

template <int CH, bool TAB, bool FLAGS>
__global__ void __launch_bounds__(LR_T, 3) k_linrec_fwd(const __grid_constant__ LrArgs p) {
  extern __shared__ __align__(16) char smem[];
  LrShared<2>& sh = *reinterpret_cast<LrShared<2>*>(smem);
  const LrPlace<CH> at(p);
  constexpr int BLOCKS = LrPlace<CH>::BLOCKS;
  if (p.cl > 1) cluster_arrive();                        // every CTA has started before another one writes to its shared memory
  if (TAB) lr_table(sh);
  grid_dep();
  const int per = p.cl * BLOCKS, rounds = (p.nb + per - 1) / per, step = per * LR_BLOCK;
  int t0 = ((at.rank * BLOCKS + at.blk) * LR_CHUNKS + at.k) * LR_CHUNK;
  bool flag = false;
  auto fetch = [&](int round, int t) {
    const int n = at.have ? p.S - t : 0;
    const size_t row = (size_t)at.b * p.S + t;
    lr_fetch(sh.raw[round & 1][0], p.g, p.ld, row, at.c0, n);
    lr_fetch(sh.raw[round & 1][1], p.v, p.ld, row, at.c0, n);
    copies_close();
    flag = lr_flag<CH, FLAGS>(p, at, t, p.S - t);
  };
  fetch(0, t0);
  float2 s = make_float2(0.0f, 0.0f);
  if (p.first && at.have) s = *reinterpret_cast<const float2*>(p.first + (size_t)at.b * p.D + at.c0);
  __syncwarp();
  if (p.cl > 1) cluster_wait();
  for (int k = 0; k < rounds; ++k, t0 += step) {
    const int blk = k * per + at.rank * BLOCKS + at.blk, n = p.S - t0;                 // n rows of the chunk exist
    const int chunks = max(0, min(LR_CHUNKS, (p.S - blk * LR_BLOCK + LR_CHUNK - 1) / LR_CHUNK));
    const uint32_t cuts = lr_cuts<CH, FLAGS>(flag);
    if (k + 1 < rounds) fetch(k + 1, t0 + step);
    else copies_close();
    copies_wait<1>();
    uint32_t wg[LR_CHUNK];
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) wg[i] = sh.raw[k & 1][0][i][threadIdx.x];
    float f[LR_CHUNK][2], u[LR_CHUNK][2];
    lr_gates<TAB>(wg, sh.tab, f, u);
    LrMap mine;
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) {
      const uint32_t w = sh.raw[k & 1][1][i][threadIdx.x];
      u[i][0] = fmul(u[i][0], bflo(w));
      u[i][1] = fmul(u[i][1], bfhi(w));
      lr_extend(mine, i, n, f[i], make_float2(u[i][0], u[i][1]), (cuts >> i) & 1);
    }
    LrMap before;
    const float2 start = lr_hand_over(sh, p, at, k, at.k, chunks, min(per, p.nb - k * per), mine, before, s);
    if (p.save && at.k == 0 && n > 0 && at.have) *reinterpret_cast<float2*>(p.save + ((size_t)at.b * p.nb + blk) * p.D + at.c0) = start;
    float2 h = at.k ? lr_apply(before, start) : start;
    uint16_t* out = p.y + ((size_t)at.b * p.S + t0) * p.ld_y + at.c0;
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) {
      h = lr_step(f[i], make_float2(u[i][0], u[i][1]), h, (cuts >> i) & 1);
      if (i < n && at.have) *reinterpret_cast<uint32_t*>(out + i * p.ld_y) = pack_bf2(h.x, h.y);
    }
    __syncwarp();
  }
  if (p.last && at.have && threadIdx.x < CH / 2 && at.rank == 0) *reinterpret_cast<float2*>(p.last + (size_t)at.b * p.D + at.c0) = s;
}

template <int CH, bool TAB, bool FLAGS>
__global__ void __launch_bounds__(LR_T, 2) k_linrec_bwd(const __grid_constant__ LrArgs p) {
  extern __shared__ __align__(16) char smem[];
  LrShared<3>& sh = *reinterpret_cast<LrShared<3>*>(smem);
  const LrPlace<CH> at(p);
  constexpr int LANES = LrPlace<CH>::LANES, BLOCKS = LrPlace<CH>::BLOCKS;
  if (p.cl > 1) cluster_arrive();
  if (TAB) lr_table(sh);
  grid_dep();
  const int per = p.cl * BLOCKS, rounds = (p.nb + per - 1) / per;
  bool flag = false;
  float2 state_next = make_float2(0.0f, 0.0f);
  auto fetch = [&](int round, int blk) {                 // blk below 0: there is none
    const int t = blk * LR_BLOCK + at.k * LR_CHUNK, n = blk >= 0 && at.have ? p.S - t : 0;
    const size_t row = blk >= 0 ? (size_t)at.b * p.S + t : 0;
    lr_fetch(sh.raw[round & 1][0], p.g, p.ld, row, at.c0, n);
    lr_fetch(sh.raw[round & 1][1], p.v, p.ld, row, at.c0, n);
    lr_fetch(sh.raw[round & 1][2], p.dy, p.ld_y, row, at.c0, n);
    copies_close();
    flag = lr_flag<CH, FLAGS>(p, at, t, blk >= 0 ? p.S - t : 0);
    if (blk >= 0 && at.have) state_next = *reinterpret_cast<const float2*>(p.states + ((size_t)at.b * p.nb + blk) * p.D + at.c0);
  };
  int blk = p.nb - 1 - (at.rank * BLOCKS + at.blk);       // from the last block to the first
  fetch(0, blk);
  float2 s = make_float2(0.0f, 0.0f);
  if (p.first && at.have) s = *reinterpret_cast<const float2*>(p.first + (size_t)at.b * p.D + at.c0);
  __syncwarp();
  if (p.cl > 1) cluster_wait();
  for (int r = 0; r < rounds; ++r, blk -= per) {
    const int chunks = blk < 0 ? 0 : min(LR_CHUNKS, (p.S - blk * LR_BLOCK + LR_CHUNK - 1) / LR_CHUNK);
    const int t0 = blk * LR_BLOCK + at.k * LR_CHUNK, n = blk < 0 ? 0 : p.S - t0;
    const uint32_t cuts = lr_cuts<CH, FLAGS>(flag);
    const float2 state = state_next;
    if (r + 1 < rounds) fetch(r + 1, blk - per);
    else copies_close();
    copies_wait<1>();
    const uint32_t (*raw)[LR_CHUNK][LR_T] = sh.raw[r & 1];
    uint32_t wg[LR_CHUNK];
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) wg[i] = raw[0][i][threadIdx.x];
    float f[LR_CHUNK][2], z[LR_CHUNK][2];
    lr_gates<TAB>(wg, sh.tab, f, z);
    LrMap mine, fore;                                    // of the gradient, of the state
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) {
      const uint32_t w = raw[1][i][threadIdx.x];
      lr_extend(fore, i, n, f[i], make_float2(fmul(z[i][0], bflo(w)), fmul(z[i][1], bfhi(w))), (cuts >> i) & 1);
    }
    bool any = false;
    mine.a = mine.h = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = LR_CHUNK - 1; i >= 0; --i) {
      if (i >= n) continue;
      const uint32_t w = raw[2][i][threadIdx.x];
      const float2 d = make_float2(bflo(w), bfhi(w));
      mine.h = any ? make_float2(fmul(f[i][0], fadd(d.x, mine.h.x)), fmul(f[i][1], fadd(d.y, mine.h.y))) : make_float2(fmul(f[i][0], d.x), fmul(f[i][1], d.y));
      mine.a = any ? make_float2(fmul(f[i][0], mine.a.x), fmul(f[i][1], mine.a.y)) : make_float2(f[i][0], f[i][1]);
      if ((cuts >> i) & 1) mine.a = mine.h = make_float2(0.0f, 0.0f);
      any = true;
    }
    sh.ahead[threadIdx.x] = lr_pack(fore);
    // the order of the backward pass: chunk 0 is the block's last one that exists; those beyond the end stay behind it
    const int order = at.k < chunks ? chunks - 1 - at.k : at.k;
    LrMap behind;
    const float2 start = lr_hand_over(sh, p, at, r, order, chunks, min(per, p.nb - r * per), mine, behind, s);
    if (n > 0 && at.have) {
      float2 h = state;
      if (at.k) h = lr_apply(lr_before<LANES>(sh.ahead + at.blk * LR_CHUNKS * LANES + at.lane, at.k, LR_CHUNKS), state);
      float2 prev[LR_CHUNK];
#pragma unroll
      for (int i = 0; i < LR_CHUNK; ++i) {
        const uint32_t w = raw[1][i][threadIdx.x];
        const bool cut = (cuts >> i) & 1;
        prev[i] = cut ? make_float2(0.0f, 0.0f) : h;
        h = lr_step(f[i], make_float2(fmul(z[i][0], bflo(w)), fmul(z[i][1], bfhi(w))), h, cut);
        prev[i] = make_float2(fsub(prev[i].x, bflo(w)), fsub(prev[i].y, bfhi(w)));
      }
      float2 c = order ? lr_apply(behind, start) : start;
      const size_t o = ((size_t)at.b * p.S + t0) * p.ld_d + at.c0;
#pragma unroll
      for (int i = LR_CHUNK - 1; i >= 0; --i) {
        if (i >= n) continue;
        const uint32_t w = raw[2][i][threadIdx.x];
        const float2 d = make_float2(fadd(bflo(w), c.x), fadd(bfhi(w), c.y));
        c = (cuts >> i) & 1 ? make_float2(0.0f, 0.0f) : make_float2(fmul(f[i][0], d.x), fmul(f[i][1], d.y));
        *reinterpret_cast<uint32_t*>(p.dv + o + i * p.ld_d) = pack_bf2(fmul(d.x, z[i][0]), fmul(d.y, z[i][1]));
        *reinterpret_cast<uint32_t*>(p.dg + o + i * p.ld_d) =
            pack_bf2(fmul(fmul(d.x, prev[i].x), fmul(f[i][0], z[i][0])), fmul(fmul(d.y, prev[i].y), fmul(f[i][1], z[i][1])));
      }
    }
    __syncthreads();                                     // `ahead` is read by then
  }
  if (p.last && at.have && threadIdx.x < CH / 2 && at.rank == 0) *reinterpret_cast<float2*>(p.last + (size_t)at.b * p.D + at.c0) = s;
}

// Sequences of one chunk (a token at a time among them): a thread walks two channels alone, with nothing to hand over.
template <bool BWD>
__global__ void __launch_bounds__(128) k_linrec_chunk(const __grid_constant__ LrArgs p, size_t threads) {
  grid_dep();
  const size_t i = (size_t)blockIdx.x * 128 + threadIdx.x;
  if (i >= threads) return;
  const int b = (int)(i / (p.D / 2)), c0 = 2 * (int)(i % (p.D / 2)), n = p.S;
  const size_t row = (size_t)b * p.S, at = (size_t)b * p.D + c0;
  uint32_t wg[LR_CHUNK], wv[LR_CHUNK], wd[LR_CHUNK], cuts = 0;
#pragma unroll
  for (int t = 0; t < LR_CHUNK; ++t) {
    const bool there = t < n;
    wg[t] = there ? __ldg(reinterpret_cast<const uint32_t*>(p.g + (row + t) * p.ld + c0)) : 0u;
    wv[t] = there ? __ldg(reinterpret_cast<const uint32_t*>(p.v + (row + t) * p.ld + c0)) : 0u;
    wd[t] = BWD && there ? __ldg(reinterpret_cast<const uint32_t*>(p.dy + (row + t) * p.ld_y + c0)) : 0u;
    if (p.flags && there && p.flags[row + t]) cuts |= 1u << t;
  }
  float2 s = p.first ? *reinterpret_cast<const float2*>(p.first + at) : make_float2(0.0f, 0.0f);
  float2 h = BWD ? *reinterpret_cast<const float2*>(p.states + at) : s;
  if (p.save) *reinterpret_cast<float2*>(p.save + at) = s;
  float f[LR_CHUNK][2], z[LR_CHUNK][2];
  float2 prev[LR_CHUNK];
  LrMap m;
  m.a = m.h = make_float2(0.0f, 0.0f);
#pragma unroll
  for (int t = 0; t < LR_CHUNK; ++t) {
    if (t >= n) continue;
    lr_gate2<false>(wg[t], nullptr, f[t], z[t]);
    const bool cut = (cuts >> t) & 1;
    const float2 v = make_float2(bflo(wv[t]), bfhi(wv[t])), u = make_float2(fmul(z[t][0], v.x), fmul(z[t][1], v.y));
    if (!BWD) lr_extend(m, t, n, f[t], u, cut);
    prev[t] = cut ? make_float2(fsub(0.0f, v.x), fsub(0.0f, v.y)) : make_float2(fsub(h.x, v.x), fsub(h.y, v.y));
    h = lr_step(f[t], u, h, cut);
    if (!BWD) *reinterpret_cast<uint32_t*>(p.y + (row + t) * p.ld_y + c0) = pack_bf2(h.x, h.y);
  }
  if (BWD) {
    float2 c = s;
#pragma unroll
    for (int t = LR_CHUNK - 1; t >= 0; --t) {
      if (t >= n) continue;
      const bool cut = (cuts >> t) & 1;
      const float2 dy = make_float2(bflo(wd[t]), bfhi(wd[t])), d = make_float2(fadd(dy.x, c.x), fadd(dy.y, c.y));
      c = cut ? make_float2(0.0f, 0.0f) : make_float2(fmul(f[t][0], d.x), fmul(f[t][1], d.y));
      m.h = t + 1 < n ? make_float2(fmul(f[t][0], fadd(dy.x, m.h.x)), fmul(f[t][1], fadd(dy.y, m.h.y))) : make_float2(fmul(f[t][0], dy.x), fmul(f[t][1], dy.y));
      m.a = t + 1 < n ? make_float2(fmul(f[t][0], m.a.x), fmul(f[t][1], m.a.y)) : make_float2(f[t][0], f[t][1]);
      if (cut) m.a = m.h = make_float2(0.0f, 0.0f);
      *reinterpret_cast<uint32_t*>(p.dv + (row + t) * p.ld_d + c0) = pack_bf2(fmul(d.x, z[t][0]), fmul(d.y, z[t][1]));
      *reinterpret_cast<uint32_t*>(p.dg + (row + t) * p.ld_d + c0) =
          pack_bf2(fmul(fmul(d.x, prev[t].x), fmul(f[t][0], z[t][0])), fmul(fmul(d.y, prev[t].y), fmul(f[t][1], z[t][1])));
    }
  }
  if (p.last) *reinterpret_cast<float2*>(p.last + at) = lr_apply(m, s);
}

// The strip and the cluster: narrower strips and larger clusters until CTAs cover the GPU `waves` times, no more CTAs than there are blocks.
struct LrPlan { int ch, cl; };
static LrPlan lr_plan(int B, int D, int nb, int waves) {
  const long long room = (long long)waves * dev_sm_count();
  LrPlan q = {64, 1};
  auto chains = [&](int ch) { return (long long)B * ((D + ch - 1) / ch); };
  if (nb > 1 && chains(32) <= room) q.ch = 32;
  while (q.cl < LR_MAXC && 2 * q.cl * (64 / q.ch) <= nb && chains(q.ch) * 2 * q.cl <= room) q.cl *= 2;
  return q;
}
template <int NS>
static int lr_launch(void (*kern)(const LrArgs), LrArgs& p, LrPlan q, int B, DevOnce& once, cudaStream_t st) {
  p.cl = q.cl;
  p.strips = (p.D + q.ch - 1) / q.ch;
  int rc = dev_ensure_smem(once, (const void*)kern, sizeof(LrShared<NS>));
  if (rc != DET_OK) return rc;
  if (q.cl > 8 && cudaFuncSetAttribute((const void*)kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return DET_ERR_CUDA;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.cl;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((long long)B * p.strips * p.cl));
  cfg.blockDim = dim3(LR_T);
  cfg.dynamicSmemBytes = sizeof(LrShared<NS>);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = p.cl > 1 ? 2 : 1;
  note_launch();
  cudaLaunchKernelEx(&cfg, kern, p);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
template <int CH, bool TAB, bool FLAGS>
static int lr_run(bool bwd, LrArgs& p, LrPlan q, int B, cudaStream_t st) {
  static DevOnce fwd_once, bwd_once;
  return bwd ? lr_launch<3>(k_linrec_bwd<CH, TAB, FLAGS>, p, q, B, bwd_once, st) : lr_launch<2>(k_linrec_fwd<CH, TAB, FLAGS>, p, q, B, fwd_once, st);
}
static int lr_any(bool bwd, LrArgs& p, int B, cudaStream_t st) {
  p.nb = (p.S + LR_BLOCK - 1) / LR_BLOCK;
  if (p.S <= LR_CHUNK) {
    const size_t threads = (size_t)B * (p.D / 2);
    launch_after(bwd ? k_linrec_chunk<true> : k_linrec_chunk<false>, dim3((unsigned)((threads + 127) / 128)), 128, 0, st, p, threads);
    DET_CHECK_LAUNCH();
    return DET_OK;
  }
  const LrPlan q = lr_plan(B, p.D, p.nb, bwd ? 2 : 3);
  const bool tab = p.nb * 64 / q.ch / q.cl >= 4;
  if (q.ch == 64)
    return tab ? (p.flags ? lr_run<64, true, true>(bwd, p, q, B, st) : lr_run<64, true, false>(bwd, p, q, B, st))
               : (p.flags ? lr_run<64, false, true>(bwd, p, q, B, st) : lr_run<64, false, false>(bwd, p, q, B, st));
  return tab ? (p.flags ? lr_run<32, true, true>(bwd, p, q, B, st) : lr_run<32, true, false>(bwd, p, q, B, st))
             : (p.flags ? lr_run<32, false, true>(bwd, p, q, B, st) : lr_run<32, false, false>(bwd, p, q, B, st));
}
static int lr_check(const void* a, const void* b, int ld, int B, int S, int D) {
  if (!a || !b || B < 0 || S < 0 || D <= 0 || ld < D) return DET_ERR_ARG;
  if (D % 2 || ld % 2 || S > (1 << 30)) return DET_ERR_SHAPE;
  if ((long long)B * ((D + 31) / 32) > (1 << 26)) return DET_ERR_SHAPE;
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
  return lr_any(false, p, B, st);
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
  return lr_any(true, p, B, st);
}
