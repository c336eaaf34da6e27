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
// and two blocks, a round.  One warp composes the chunk maps of a round.  The CTAs of a cluster take adjacent blocks and hand each other their
// block maps through distributed shared memory, by stores that complete a transaction barrier of the receiver (a fence and a cluster barrier a round
// took 1300 cycles of 4800); every CTA applies the maps of the blocks before its own.
// So every value is read once and written once however long a sequence is and however few there are, with no workspace.  The raw
// values of the next round come in by asynchronous copies while this one is worked on.
#include "common.cuh"
#include "internal.h"
#include "tc05.cuh"

namespace det {

constexpr int LR_CHUNK = 8, LR_CHUNKS = 8, LR_BLOCK = LR_CHUNK * LR_CHUNKS, LR_T = 256, LR_MAXC = 16;

__device__ __forceinline__ float lr_minor(float g) {
  const float e = det_exp_le0(-fabsf(g));
  return fdiv(e, fadd(1.0f, e));
}
// The gate of a bf16 has few arguments: the magnitudes from 2^-26 (e rounds to 1 below it) to 128 (e flushes to 0 long before), 33 exponents of
// 128 fractions.  Their values of lr_minor, evaluated by the compiler with the same steps, are part of the library; a CTA copies them into shared
// memory: a lookup instead of an exponential and a division for every value (some 30 of 50 instructions).
constexpr int LR_LOW = 0x3280, LR_TOP = 0x4300, LR_TAB = (LR_TOP - LR_LOW + 1 + 3) / 4 * 4;
struct __align__(16) LrTable { float m[LR_TAB]; };
constexpr float lr_minor_at(int bits) {
  float x = -(1.0f + (bits & 127) / 128.0f);
  for (int e = bits >> 7; e > 127; --e) x *= 2.0f;
  for (int e = bits >> 7; e < 127; ++e) x *= 0.5f;
  if (x < -0x1.5d58a0p+6f) return 0.0f;
  float t = x * 0x1.715476p+0f;
  t = t + 12582912.0f;
  const float kf = t - 12582912.0f;
  t = kf * 0x1.62e400p-1f;
  float r = x - t;
  t = kf * 0x1.7f7d1cp-20f;
  r = r - t;
  const float c[7] = {0x1.6c16c2p-10f, 0x1.111112p-7f, 0x1.555556p-5f, 0x1.555556p-3f, 0.5f, 1.0f, 1.0f};
  float q = 0x1.a01a02p-13f;
  for (int i = 0; i < 7; ++i) {
    t = q * r;
    q = t + c[i];
  }
  for (int k = (int)kf; k < 0; ++k) q *= 0.5f;
  const float d = 1.0f + q;
  return q / d;
}
constexpr LrTable lr_make_table() {
  LrTable t{};
  for (int i = 0; i < LR_TAB; ++i) t.m[i] = lr_minor_at(LR_LOW + i);
  return t;
}
__device__ constexpr LrTable lr_table_image = lr_make_table();

__device__ __forceinline__ void lr_gate(float m, bool negative, float& f, float& z) {
  const float M = fsub(1.0f, m);
  f = negative ? m : M;
  z = negative ? M : m;
}
// gates of the two channels in one word; by table a NaN is looked up as an infinity: lr_gates puts it right
template <bool TAB>
__device__ __forceinline__ void lr_gate2(uint32_t w, const float* tab, float f[2], float z[2]) {
  const char* t = reinterpret_cast<const char*>(tab);
  constexpr int last = 4 * (LR_TOP - LR_LOW);
  const float m0 = TAB ? *reinterpret_cast<const float*>(t + __vimin_s32_relu((int)((w << 2) & 0x1fffcu) - 4 * LR_LOW, last)) : lr_minor(bflo(w));
  const float m1 = TAB ? *reinterpret_cast<const float*>(t + __vimin_s32_relu((int)((w >> 14) & 0x1fffcu) - 4 * LR_LOW, last)) : lr_minor(bfhi(w));
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

// CH channels a CTA: LANES lanes a chunk, BLOCKS blocks a round.
template <int CH>
struct LrDim {
  static constexpr int LANES = CH / 2, BLOCKS = 64 / CH, PAD = CH == 64 ? 0 : 16;     // PAD: so that the two halves of a warp read different banks
  static constexpr int STRIDE = LR_CHUNK * LANES + PAD, RAW = BLOCKS * LR_CHUNKS * STRIDE;
};
// NS: tensors that come in by asynchronous copies.  The block maps of the cluster, two rounds of them, lie behind this.
template <int CH, int NS>
struct __align__(16) LrShared {
  uint32_t raw[NS == 3 ? 2 : 1][NS][LrDim<CH>::RAW];     // backward two rounds; [chunk of the CTA][row][lane]
  float tab[LR_TAB];
  float4 chunk[LR_T];                                    // [block of the CTA][chunk][lane]: the chunk maps of this round, then the maps of those before
  float4 ahead[NS == 3 ? LR_T : 1];                      // backward: the same of the recurrence itself
  float2 start[32];                                      // [block of the CTA][lane]: what comes into the blocks
  float2 state[NS == 3 ? 32 : 1];                        // backward: the states in front of the blocks
  unsigned long long arrived[2];                         // transaction barriers of the block maps, two rounds
  int gone;                                              // a wait ran out
  __device__ __forceinline__ float4* slots(int round, int cl) { return reinterpret_cast<float4*>(this + 1) + (round & 1) * 32 * cl; }
  static size_t bytes(int cl) { return sizeof(LrShared) + (size_t)2 * cl * 32 * sizeof(float4); }
};
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// a float4 into the place of `local` in the CTA `rank` of the cluster, counted by its barrier in the place of `bar`
__device__ __forceinline__ void store_in_cluster(const void* local, const void* bar, int rank, float4 v) {
  uint32_t a, b;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(local)), "r"(rank));
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(b) : "r"(smem_u32(bar)), "r"(rank));
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(a), "f"(v.x), "f"(v.y),
               "f"(v.z), "f"(v.w), "r"(b)
               : "memory");
}
// 16 or 4 bytes, zeros where there is nothing (the address is not followed then)
template <int WORDS>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool there) {
  if (WORDS == 4) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copies_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

struct LrArgs {
  const uint16_t *g, *v, *dy;
  const uint8_t* flags;
  const float *first, *states;                           // state before the first row, or gradient of the state behind the last one
  uint16_t *y, *dg, *dv;
  float *last, *save;                                    // what comes out at the other end; states at the starts of the blocks
  size_t ld, ld_y, ld_d;
  int S, D, strips, nb, cl;                              // cl: CTAs of a cluster
  int* status;
};

// Where a thread is
template <int CH>
struct LrPlace {
  int b, c0, rank, blk, k, lane;                         // sequence, first channel of the strip; block of the CTA's, chunk of the block, lane of the chunk
  bool have;                                             // the lane's channels exist
  __device__ __forceinline__ LrPlace(const LrArgs& p) {
    rank = blockIdx.x % p.cl;
    const int q = blockIdx.x / p.cl;
    b = q / p.strips;
    lane = threadIdx.x % LrDim<CH>::LANES;
    const int chunk = threadIdx.x / LrDim<CH>::LANES;
    blk = chunk / LR_CHUNKS;
    k = chunk % LR_CHUNKS;
    c0 = (q % p.strips) * CH;
    have = c0 + 2 * lane < p.D;
  }
};
// The rows of the CTA's blocks of one tensor on their way, in pieces of WORDS words: block j starts at row first + j * step (64 or -64), rows
// outside the sequence and channels outside the tensor are zeros.
template <int CH, int WORDS>
__device__ __forceinline__ void lr_fetch(uint32_t* raw, const uint16_t* x, size_t ld, const LrArgs& p, const LrPlace<CH>& at, int first, int step) {
  constexpr int LANES = LrDim<CH>::LANES, PER = LANES / WORDS, COUNT = LrDim<CH>::BLOCKS * LR_BLOCK * PER / LR_T;
  const uint32_t dst = (uint32_t)__cvta_generic_to_shared(raw);
  const int word = (threadIdx.x % PER) * WORDS, r0 = threadIdx.x / PER;
  const bool have = at.c0 + 2 * word < p.D;
  const uint16_t* base = x + (size_t)at.b * p.S * ld + at.c0 + 2 * word;
#pragma unroll
  for (int j = 0; j < COUNT; ++j) {
    const int row = r0 + j * (LR_T / PER), t = first + (row / LR_BLOCK) * step + row % LR_BLOCK;
    const bool there = have && (unsigned)t < (unsigned)p.S;
    copy_async<WORDS>(dst + 4 * ((row / LR_CHUNK) * LrDim<CH>::STRIDE + (row % LR_CHUNK) * LANES + word), there ? base + (size_t)t * ld : x, there);
  }
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
// The gates of a chunk.  A NaN gate comes out of the table as one of an infinity: it makes its gate a NaN here.
__device__ __forceinline__ void lr_gates(const uint32_t* raw, int lanes, const float* tab, float f[LR_CHUNK][2], float z[LR_CHUNK][2]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < LR_CHUNK; ++i) {
    const uint32_t w = raw[i * lanes];
    lr_gate2<true>(w, tab, f[i], z[i]);
    top = __vmaxu2(top, w & 0x7fff7fffu);
  }
  if ((top & 0xffffu) > 0x7f80u || (top >> 16) > 0x7f80u) {
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) {
      const uint32_t w = raw[i * lanes];
      if ((w & 0x7fffu) > 0x7f80u) f[i][0] = z[i][0] = __int_as_float(0x7fffffff);
      if (((w >> 16) & 0x7fffu) > 0x7f80u) f[i][1] = z[i][1] = __int_as_float(0x7fffffff);
    }
  }
}
// The maps of the `chunks` chunks of a block, one after the other, by one thread: the map of those before chunk k takes chunk k's place, the map
// of all comes back.
template <int LANES>
__device__ __forceinline__ LrMap lr_scan(float4* chunk, int chunks) {
  LrMap m = lr_unpack(chunk[0]);
  if (chunks == LR_CHUNKS) {
    float4 next[LR_CHUNKS];
#pragma unroll
    for (int i = 1; i < LR_CHUNKS; ++i) next[i] = chunk[i * LANES];
#pragma unroll
    for (int i = 1; i < LR_CHUNKS; ++i) {
      chunk[i * LANES] = lr_pack(m);
      m = lr_compose(m, lr_unpack(next[i]));
    }
  } else {
#pragma unroll 1
    for (int i = 1; i < chunks; ++i) {
      const LrMap here = lr_unpack(chunk[i * LANES]);
      chunk[i * LANES] = lr_pack(m);
      m = lr_compose(m, here);
    }
  }
  return m;
}
// The round's hand-over, by the first warp, a thread per block of the CTA and lane: block maps to the CTAs of the cluster, what comes into each block
// of this CTA back.  `s`, what comes into the round, becomes what comes into the next one.  `chunks` of the thread's block exist, in the places from
// `first` on; `blocks` of the round.
// The maps of two rounds have places of their own: a CTA sends those of round r + 2 when it has all of round r + 1, this CTA's among them, which this CTA
// sent after it had read round r's.
template <int CH, int NS>
__device__ __forceinline__ float2 lr_hand_over(LrShared<CH, NS>& sh, const LrArgs& p, const LrPlace<CH>& at, int round, int first, int chunks, int blocks,
                                               float2& s) {
  constexpr int LANES = LrDim<CH>::LANES, BLOCKS = LrDim<CH>::BLOCKS, BATCH = 8;
  const int blk = threadIdx.x / LANES, own = at.rank * BLOCKS + blk;
  float4* slots = sh.slots(round, p.cl);
  uint64_t* bar = reinterpret_cast<uint64_t*>(&sh.arrived[round & 1]);
  if (p.cl > 1 && threadIdx.x == 0) mbar_expect_tx(bar, p.cl * 32 * sizeof(float4));
  const float4 whole = lr_pack(lr_scan<LANES>(sh.chunk + (blk * LR_CHUNKS + first) * LANES + at.lane, chunks));
  if (p.cl == 1) {
    slots[own * LANES + at.lane] = whole;
    __syncwarp();
  } else {
#pragma unroll 4
    for (int r = 0; r < p.cl; ++r) store_in_cluster(&slots[own * LANES + at.lane], bar, r, whole);
    mbar_wait_warp(bar, (round >> 1) & 1, &sh.gone, p.status);
  }
  float2 start = s;
  if (p.cl == 1) {
    for (int r = 0; r < blocks; ++r) {
      if (r == own) start = s;
      s = lr_apply(lr_unpack(slots[r * LANES + at.lane]), s);
    }
    return start;
  }
  for (int r0 = 0; r0 < blocks; r0 += BATCH) {
    float4 m[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) m[i] = slots[min(r0 + i, blocks - 1) * LANES + at.lane];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      if (r0 + i == own) start = s;
      if (r0 + i < blocks) s = lr_apply(lr_unpack(m[i]), s);
    }
  }
  return start;
}
// before the first round: the barriers, known to the cluster before anyone sends
template <int CH, int NS>
__device__ __forceinline__ void lr_open(LrShared<CH, NS>& sh, const LrArgs& p) {
  if (threadIdx.x == 0) {
    sh.gone = 0;
    mbar_init(reinterpret_cast<uint64_t*>(&sh.arrived[0]), 1);
    mbar_init(reinterpret_cast<uint64_t*>(&sh.arrived[1]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (p.cl > 1) cluster_arrive();
}
// no CTA leaves while another one may still send to it (after a wait that ran out)
__device__ __forceinline__ void lr_close(const LrArgs& p) {
  if (p.cl == 1) return;
  cluster_arrive();
  cluster_wait();
}
template <int CH, int NS>
__device__ __forceinline__ void lr_copy_table(LrShared<CH, NS>& sh) {
  const uint32_t dst = (uint32_t)__cvta_generic_to_shared(sh.tab);
  for (int i = threadIdx.x; i < LR_TAB / 4; i += LR_T) copy_async<4>(dst + 16 * i, lr_table_image.m + 4 * i, true);
}

template <int CH, int WORDS, bool FLAGS>
__global__ void __launch_bounds__(LR_T, 4) k_linrec_fwd(const __grid_constant__ LrArgs p) {
  extern __shared__ __align__(16) char smem[];
  LrShared<CH, 2>& sh = *reinterpret_cast<LrShared<CH, 2>*>(smem);
  const LrPlace<CH> at(p);
  constexpr int LANES = LrDim<CH>::LANES, BLOCKS = LrDim<CH>::BLOCKS;
  lr_open(sh, p);
  lr_copy_table(sh);
  grid_dep();
  const int per = p.cl * BLOCKS, rounds = (p.nb + per - 1) / per, step = per * LR_BLOCK;
  int b0 = at.rank * BLOCKS * LR_BLOCK;                  // the CTA's first row of the round
  const int ch = at.c0 + 2 * at.lane;
  const bool lead = threadIdx.x < 32;
  bool flag = false;
  auto fetch = [&](int row) {
    lr_fetch<CH, WORDS>(sh.raw[0][0], p.g, p.ld, p, at, row, LR_BLOCK);
    lr_fetch<CH, WORDS>(sh.raw[0][1], p.v, p.ld, p, at, row, LR_BLOCK);
    const int t = row + (at.blk * LR_CHUNKS + at.k) * LR_CHUNK;
    flag = lr_flag<CH, FLAGS>(p, at, t, p.S - t);
  };
  fetch(b0);
  float2 s = make_float2(0.0f, 0.0f);
  if (lead && p.first && at.have) s = *reinterpret_cast<const float2*>(p.first + (size_t)at.b * p.D + ch);
  copies_done();
  __syncthreads();
  if (p.cl > 1) cluster_wait();
  for (int k = 0; k < rounds; ++k, b0 += step) {
    const int t0 = b0 + (at.blk * LR_CHUNKS + at.k) * LR_CHUNK, n = p.S - t0;          // n rows of the chunk exist
    const uint32_t cuts = lr_cuts<CH, FLAGS>(flag);
    const uint32_t* raw = sh.raw[0][0] + (at.blk * LR_CHUNKS + at.k) * LrDim<CH>::STRIDE + at.lane;
    float f[LR_CHUNK][2], u[LR_CHUNK][2];
    lr_gates(raw, LANES, sh.tab, f, u);
    raw += LrDim<CH>::RAW;
    LrMap mine;
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) {
      const uint32_t w = raw[i * LANES];
      u[i][0] = fmul(u[i][0], bflo(w));
      u[i][1] = fmul(u[i][1], bfhi(w));
      lr_extend(mine, i, n, f[i], make_float2(u[i][0], u[i][1]), (cuts >> i) & 1);
    }
    sh.chunk[threadIdx.x] = lr_pack(mine);               // [block][chunk][lane] is the thread's number
    __syncthreads();
    if (k + 1 < rounds) fetch(b0 + step);                // the raw values of this round are read
    if (lead) {
      const int row = b0 + (threadIdx.x / LANES) * LR_BLOCK, blk = row / LR_BLOCK;
      const int chunks = max(0, min(LR_CHUNKS, (p.S - row + LR_CHUNK - 1) / LR_CHUNK));
      const float2 start = lr_hand_over(sh, p, at, k, 0, chunks, min(per, p.nb - k * per), s);
      sh.start[threadIdx.x] = start;
      if (p.save && chunks > 0 && at.have) *reinterpret_cast<float2*>(p.save + ((size_t)at.b * p.nb + blk) * p.D + ch) = start;
    }
    copies_done();
    __syncthreads();
    if (sh.gone) break;
    float2 h = sh.start[at.blk * LANES + at.lane];
    if (at.k) h = lr_apply(lr_unpack(sh.chunk[threadIdx.x]), h);
    uint16_t* out = p.y + ((size_t)at.b * p.S + t0) * p.ld_y + ch;
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) {
      h = lr_step(f[i], make_float2(u[i][0], u[i][1]), h, (cuts >> i) & 1);
      if (i < n && at.have) *reinterpret_cast<uint32_t*>(out) = pack_bf2(h.x, h.y);
      out += p.ld_y;
    }
    __syncwarp();
  }
  copies_done();
  lr_close(p);
  if (p.last && at.have && threadIdx.x < LANES && at.rank == 0) *reinterpret_cast<float2*>(p.last + (size_t)at.b * p.D + ch) = s;
}

template <int CH, int WORDS, bool FLAGS>
__global__ void __launch_bounds__(LR_T, 2) k_linrec_bwd(const __grid_constant__ LrArgs p) {
  extern __shared__ __align__(16) char smem[];
  LrShared<CH, 3>& sh = *reinterpret_cast<LrShared<CH, 3>*>(smem);
  const LrPlace<CH> at(p);
  constexpr int LANES = LrDim<CH>::LANES, BLOCKS = LrDim<CH>::BLOCKS;
  lr_open(sh, p);
  lr_copy_table(sh);
  grid_dep();
  const int per = p.cl * BLOCKS, rounds = (p.nb + per - 1) / per;
  const int ch = at.c0 + 2 * at.lane, warp = threadIdx.x >> 5, own = (threadIdx.x & 31) / LANES;
  int top = p.nb - 1 - at.rank * BLOCKS;                 // the CTA's blocks of the round are top, top - 1; below 0: none
  bool flag = false;
  float2 state = make_float2(0.0f, 0.0f);
  auto fetch = [&](int round, int first) {
    const int row = first * LR_BLOCK;
    lr_fetch<CH, WORDS>(sh.raw[round & 1][0], p.g, p.ld, p, at, row, -LR_BLOCK);
    lr_fetch<CH, WORDS>(sh.raw[round & 1][1], p.v, p.ld, p, at, row, -LR_BLOCK);
    lr_fetch<CH, WORDS>(sh.raw[round & 1][2], p.dy, p.ld_y, p, at, row, -LR_BLOCK);
    const int t = (first - at.blk) * LR_BLOCK + at.k * LR_CHUNK;
    flag = lr_flag<CH, FLAGS>(p, at, t, first - at.blk < 0 ? 0 : p.S - t);
    if (warp == 1 && first - own >= 0 && at.have) state = *reinterpret_cast<const float2*>(p.states + ((size_t)at.b * p.nb + first - own) * p.D + ch);
  };
  fetch(0, top);
  float2 s = make_float2(0.0f, 0.0f);
  if (warp == 0 && p.first && at.have) s = *reinterpret_cast<const float2*>(p.first + (size_t)at.b * p.D + ch);
  copies_done();
  __syncthreads();
  if (p.cl > 1) cluster_wait();
  for (int r = 0; r < rounds; ++r, top -= per) {
    const int blk = top - at.blk, t0 = blk * LR_BLOCK + at.k * LR_CHUNK, n = blk < 0 ? 0 : p.S - t0;
    const int chunks = blk < 0 ? 0 : min(LR_CHUNKS, (p.S - blk * LR_BLOCK + LR_CHUNK - 1) / LR_CHUNK);
    const uint32_t cuts = lr_cuts<CH, FLAGS>(flag);
    const float2 front = state;
    if (r + 1 < rounds) fetch(r + 1, top - per);
    const uint32_t* raw = sh.raw[r & 1][0] + (at.blk * LR_CHUNKS + at.k) * LrDim<CH>::STRIDE + at.lane;
    float f[LR_CHUNK][2], z[LR_CHUNK][2];
    uint32_t wv[LR_CHUNK], wd[LR_CHUNK];
    lr_gates(raw, LANES, sh.tab, f, z);
    LrMap mine, fore;                                    // of the gradient, of the state
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) {
      wv[i] = raw[LrDim<CH>::RAW + i * LANES];
      wd[i] = raw[2 * LrDim<CH>::RAW + i * LANES];
      lr_extend(fore, i, n, f[i], make_float2(fmul(z[i][0], bflo(wv[i])), fmul(z[i][1], bfhi(wv[i]))), (cuts >> i) & 1);
    }
    bool any = false;
    mine.a = mine.h = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = LR_CHUNK - 1; i >= 0; --i) {
      if (i >= n) continue;
      const float2 d = make_float2(bflo(wd[i]), bfhi(wd[i]));
      mine.h = any ? make_float2(fmul(f[i][0], fadd(d.x, mine.h.x)), fmul(f[i][1], fadd(d.y, mine.h.y))) : make_float2(fmul(f[i][0], d.x), fmul(f[i][1], d.y));
      mine.a = any ? make_float2(fmul(f[i][0], mine.a.x), fmul(f[i][1], mine.a.y)) : make_float2(f[i][0], f[i][1]);
      if ((cuts >> i) & 1) mine.a = mine.h = make_float2(0.0f, 0.0f);
      any = true;
    }
    // in the order of the backward pass: the block's last chunk, which may not exist, has the first place
    float4* place = sh.chunk + (at.blk * LR_CHUNKS + LR_CHUNKS - 1 - at.k) * LANES + at.lane;
    *place = lr_pack(mine);
    sh.ahead[threadIdx.x] = lr_pack(fore);
    __syncthreads();
    if (warp == 0) {
      const int b = top - own, have = b < 0 ? 0 : min(LR_CHUNKS, (p.S - b * LR_BLOCK + LR_CHUNK - 1) / LR_CHUNK);
      sh.start[threadIdx.x] = lr_hand_over(sh, p, at, r, have ? LR_CHUNKS - have : 0, have, min(per, p.nb - r * per), s);
    } else if (warp == 1) {
      lr_scan<LANES>(sh.ahead + own * LR_CHUNKS * LANES + at.lane, LR_CHUNKS);
      sh.state[threadIdx.x & 31] = front;
    }
    copies_done();
    __syncthreads();
    if (sh.gone) break;
    float2 h = sh.state[at.blk * LANES + at.lane], c = sh.start[at.blk * LANES + at.lane];
    if (at.k) h = lr_apply(lr_unpack(sh.ahead[threadIdx.x]), h);
    if (at.k + 1 < chunks) c = lr_apply(lr_unpack(*place), c);
    float2 diff[LR_CHUNK];                               // h_{t-1} - v
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) {
      const bool cut = (cuts >> i) & 1;
      const float2 v = make_float2(bflo(wv[i]), bfhi(wv[i]));
      diff[i] = cut ? make_float2(fsub(0.0f, v.x), fsub(0.0f, v.y)) : make_float2(fsub(h.x, v.x), fsub(h.y, v.y));
      h = lr_step(f[i], make_float2(fmul(z[i][0], v.x), fmul(z[i][1], v.y)), h, cut);
    }
    const size_t o = ((size_t)at.b * p.S + t0 + LR_CHUNK - 1) * p.ld_d + ch;           // only followed where the row exists
    uint16_t *dv = p.dv + o, *dg = p.dg + o;
#pragma unroll
    for (int i = LR_CHUNK - 1; i >= 0; --i, dv -= p.ld_d, dg -= p.ld_d) {
      if (i >= n) continue;
      const float2 d = make_float2(fadd(bflo(wd[i]), c.x), fadd(bfhi(wd[i]), c.y));
      c = (cuts >> i) & 1 ? make_float2(0.0f, 0.0f) : make_float2(fmul(f[i][0], d.x), fmul(f[i][1], d.y));
      if (!at.have) continue;
      *reinterpret_cast<uint32_t*>(dv) = pack_bf2(fmul(d.x, z[i][0]), fmul(d.y, z[i][1]));
      *reinterpret_cast<uint32_t*>(dg) =
          pack_bf2(fmul(fmul(d.x, diff[i].x), fmul(f[i][0], z[i][0])), fmul(fmul(d.y, diff[i].y), fmul(f[i][1], z[i][1])));
    }
    __syncwarp();
  }
  copies_done();
  lr_close(p);
  if (p.last && at.have && threadIdx.x < LANES && at.rank == 0) *reinterpret_cast<float2*>(p.last + (size_t)at.b * p.D + ch) = s;
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

// The strip and the cluster: narrow strips, then larger clusters, while their CTAs are all on the GPU at once (`per_sm` of them on an SM), no more CTAs
// than there are blocks.  Clusters do not fill the GPU: of 444 CTAs, three on an SM, 416 fit in clusters of 4, 384 in clusters of 8, 336 in
// clusters of 16, and a round of 65536 x 512 that needed 256 of 224 took twice as long.
struct LrPlan { int ch, cl; };
static LrPlan lr_plan(int B, int D, int nb, int per_sm) {
  const long long slots = (long long)per_sm * dev_sm_count();
  LrPlan q = {64, 1};
  auto chains = [&](int ch) { return (long long)B * ((D + ch - 1) / ch); };
  if (nb > 1 && chains(32) <= slots) q.ch = 32;
  while (q.cl < LR_MAXC && 2 * q.cl * (64 / q.ch) <= nb && chains(q.ch) * 2 * q.cl <= (q.cl == 8 ? slots * 3 / 4 : (q.cl > 1 ? slots * 6 / 7 : slots))) q.cl *= 2;
  return q;
}
static int lr_launch(void (*kern)(const LrArgs), const LrArgs& p, int B, size_t smem, size_t most, DevOnce& once, cudaStream_t st) {
  int rc = dev_ensure_smem(once, (const void*)kern, most);
  if (rc != DET_OK) return rc;
  if (p.cl > 8 && cudaFuncSetAttribute((const void*)kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
    cudaGetLastError();
    return DET_ERR_CUDA;
  }
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.cl;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((long long)B * p.strips * p.cl));
  cfg.blockDim = dim3(LR_T);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = p.cl > 1 ? 2 : 1;
  note_launch();
  cudaLaunchKernelEx(&cfg, kern, p);
  DET_CHECK_LAUNCH();
  return DET_OK;
}
template <int CH, int WORDS, bool FLAGS>
static int lr_run(bool bwd, const LrArgs& p, int B, cudaStream_t st) {
  static DevOnce fwd_once, bwd_once;
  using Sf = LrShared<CH, 2>;
  using Sb = LrShared<CH, 3>;
  return bwd ? lr_launch(k_linrec_bwd<CH, WORDS, FLAGS>, p, B, Sb::bytes(p.cl), Sb::bytes(LR_MAXC), bwd_once, st)
             : lr_launch(k_linrec_fwd<CH, WORDS, FLAGS>, p, B, Sf::bytes(p.cl), Sf::bytes(LR_MAXC), fwd_once, st);
}
template <int CH>
static int lr_pick(bool bwd, const LrArgs& p, int B, bool wide, cudaStream_t st) {
  return wide ? (p.flags ? lr_run<CH, 4, true>(bwd, p, B, st) : lr_run<CH, 4, false>(bwd, p, B, st))
              : (p.flags ? lr_run<CH, 1, true>(bwd, p, B, st) : lr_run<CH, 1, false>(bwd, p, B, st));
}
static int lr_any(bool bwd, LrArgs& p, int B, cudaStream_t st) {
  p.nb = (p.S + LR_BLOCK - 1) / LR_BLOCK;
  if (p.S <= LR_CHUNK) {
    const size_t threads = (size_t)B * (p.D / 2);
    launch_after(bwd ? k_linrec_chunk<true> : k_linrec_chunk<false>, dim3((unsigned)((threads + 127) / 128)), 128, 0, st, p, threads);
    DET_CHECK_LAUNCH();
    return DET_OK;
  }
  const LrPlan q = lr_plan(B, p.D, p.nb, bwd ? 2 : 4);
  p.cl = q.cl;
  p.strips = (p.D + q.ch - 1) / q.ch;
  // whole pieces of 16 bytes where the tensors allow it
  const bool wide = p.D % 8 == 0 && p.ld % 8 == 0 && aligned16(p.g) && aligned16(p.v) && (!bwd || (p.ld_y % 8 == 0 && aligned16(p.dy)));
  return q.ch == 64 ? lr_pick<64>(bwd, p, B, wide, st) : lr_pick<32>(bwd, p, B, wide, st);
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
                              const float* h0, float* hT, float* states, void* stream, int* status_dev) {
  const int rc = lr_check(g, v, ld, B, S, D);
  if (rc != DET_OK) return rc;
  if (!y || ld_y < D) return DET_ERR_ARG;
  if (ld_y % 2) return DET_ERR_SHAPE;
  if (((uintptr_t)y & 3u) || (((uintptr_t)h0 | (uintptr_t)hT | (uintptr_t)states) & 7u)) return DET_ERR_ALIGN;
  cudaStream_t st = (cudaStream_t)stream;
  if (B == 0 || S == 0) return lr_empty(h0, hT, (size_t)B * D, st);
  LrArgs p = {};
  p.g = g; p.v = v; p.flags = flags; p.first = h0; p.y = y; p.last = hT; p.save = states; p.status = status_dev;
  p.ld = ld; p.ld_y = ld_y; p.S = S; p.D = D;
  return lr_any(false, p, B, st);
}

extern "C" int det_linrec_bwd(const det_bf16* dy, int ld_y, const det_bf16* g, const det_bf16* v, int ld, int B, int S, int D,
                              const float* states, det_bf16* dg, det_bf16* dv, int ld_d, const uint8_t* flags, const float* dhT, float* dh0,
                              void* stream, int* status_dev) {
  const int rc = lr_check(g, v, ld, B, S, D);
  if (rc != DET_OK) return rc;
  if (!dy || ld_y < D || !dg || !dv || ld_d < D || (!states && B > 0 && S > 0)) return DET_ERR_ARG;
  if (ld_y % 2 || ld_d % 2) return DET_ERR_SHAPE;
  if ((((uintptr_t)dy | (uintptr_t)dg | (uintptr_t)dv) & 3u) || (((uintptr_t)dhT | (uintptr_t)dh0 | (uintptr_t)states) & 7u)) return DET_ERR_ALIGN;
  cudaStream_t st = (cudaStream_t)stream;
  if (B == 0 || S == 0) return lr_empty(dhT, dh0, (size_t)B * D, st);
  LrArgs p = {};
  p.g = g; p.v = v; p.dy = dy; p.flags = flags; p.first = dhT; p.states = states; p.dg = dg; p.dv = dv; p.last = dh0; p.status = status_dev;
  p.ld = ld; p.ld_y = ld_y; p.ld_d = ld_d; p.S = S; p.D = D;
  return lr_any(true, p, B, st);
}
