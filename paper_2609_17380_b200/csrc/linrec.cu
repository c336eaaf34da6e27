// Gated linear recurrence over the rows of a sequence, per channel, forward and backward:
//   f = 1 / (1 + exp(-g)), z = 1 - f,   h_t = f_t h_{t-1} + z_t v_t   (a row with a cut starts from 0 instead of h_{t-1})
//   dh_t = dy_t + f_{t+1} dh_{t+1},  dv = dh z,  dg = dh (h_{t-1} - v) f z
// f and z come from one exponential: with e = exp(-|g|) the smaller of them is m = e / (1 + e) and the larger 1 - m, so neither
// loses digits where the gate saturates.
//
// Order of the sums.  Some rows are the map s -> A s + H.  A sequence is cut into chunks of 8 rows, from its first row on; blocks of 2 chunks, groups of
// 4 blocks and spans of 2 groups are counted from its first chunk on (backward from its last).  A chunk's map is composed row by row, a block's of its chunks, a group's of its blocks one after
// the other, a span's of its groups.  What comes into a span or a group is the map of the one before, in its span, applied to what came into that; what comes
// into a block or a chunk is the map of all those before it, in its group or block, applied to what comes into that; inside a chunk the recurrence is
// walked row by row.  Gates are never below +0.  A row with a cut has A = -0, a sign that every product keeps: such a map lets nothing in, not even a NaN.  A
// product of gates that underflowed is +0, and what is not finite goes on through it as it does through the rows one by one.
//
// A warp has a block of 32 channels: sixteen lanes a chunk, two channels a lane, so that a row's piece is 64 bytes (of 32 bytes the L1 cache was 64 % busy
// with finding lines); the maps of its two chunks meet in a shuffle.  Eight warps have the blocks of a span, and every warp composes the block maps again
// from shared memory, a group in each half.
// Where there are few strips the CTAs of a cluster take adjacent spans: they send each other the span maps, by stores that complete a transaction
// barrier of the receiver, and one warp of each applies them in turn.  So every value is read once and written once however long a sequence is and however
// few there are, with no workspace.  A warp's raw values of the next round come in by asynchronous copies as soon as those of this round are in registers
// (in a cluster, as soon as its maps are sent).
#include <algorithm>
#include <mutex>
#include <type_traits>

#include "common.cuh"
#include "internal.h"
#include "rows.cuh"
#include "tc05.cuh"

namespace det {

constexpr int LR_CHUNK = 8, LR_BLOCK = 2, LR_GROUP = 4, LR_WARPS = 8, LR_T = 32 * LR_WARPS, LR_CH = 32, LR_MAXC = 16;
constexpr int LR_ROWS = LR_WARPS * LR_BLOCK * LR_CHUNK;   // of a span

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
  const float q = det_exp_at(x), d = 1.0f + q;
  return q / d;
}
constexpr LrTable lr_make_table() {
  LrTable t{};
  for (int i = 0; i < LR_TAB; ++i) t.m[i] = lr_minor_at(LR_LOW + i);
  return t;
}
__device__ constexpr LrTable lr_table_image = lr_make_table();

// gates of the two channels in one word; by table a NaN is looked up as an infinity: lr_gates puts it right
template <bool TAB>
__device__ __forceinline__ void lr_gate2(uint32_t w, const float* tab, float2& f, float2& z) {
  const char* t = reinterpret_cast<const char*>(tab);
  constexpr int last = 4 * (LR_TOP - LR_LOW);
  const float m0 = TAB ? *reinterpret_cast<const float*>(t + __vimin_s32_relu((int)(w & 0x7fffu) * 4 - 4 * LR_LOW, last)) : lr_minor(bflo(w));
  const float m1 = TAB ? *reinterpret_cast<const float*>(t + __vimin_s32_relu((int)((w >> 14) & 0x1fffcu) - 4 * LR_LOW, last)) : lr_minor(bfhi(w));
  const float2 M = fma2(make_float2(m0, m1), same2(-1.0f), same2(1.0f));             // 1 - m, rounded once either way
  const bool n0 = w & 0x8000u, n1 = (int)w < 0;
  f = make_float2(n0 ? m0 : M.x, n1 ? m1 : M.y);
  z = make_float2(n0 ? M.x : m0, n1 ? M.y : m1);
}
struct LrMap { float2 a, h; };                           // s -> a s + h for two channels
// Pairs of channels in packed arithmetic, no product fused with a sum: `one` is the factor 1 that add2 needs.
__device__ __forceinline__ float2 lr_axpy(float2 a, float2 s, float2 h, float2 one) { return add2(mul2(a, s), h, one); }
__device__ __forceinline__ float2 lr_sub(float2 a, float2 b) { return fma2(b, same2(-1.0f), a); }
// a map with a cut among its rows
__device__ __forceinline__ bool lr_closed(float a) { return __float_as_uint(a) == 0x80000000u; }
__device__ __forceinline__ float2 lr_apply(const LrMap& m, float2 s, float2 one) {
  const float2 r = lr_axpy(m.a, s, m.h, one);
  return make_float2(lr_closed(m.a.x) ? m.h.x : r.x, lr_closed(m.a.y) ? m.h.y : r.y);
}
// the map `first`, then `then`
__device__ __forceinline__ LrMap lr_compose(const LrMap& first, const LrMap& then, float2 one) {
  const float2 a = mul2(first.a, then.a), h = lr_axpy(then.a, first.h, then.h, one);
  const bool x = lr_closed(then.a.x), y = lr_closed(then.a.y);
  return LrMap{make_float2(x ? -0.0f : a.x, y ? -0.0f : a.y), make_float2(x ? then.h.x : h.x, y ? then.h.y : h.y)};
}
__device__ __forceinline__ float4 lr_pack(const LrMap& m) { return make_float4(m.a.x, m.a.y, m.h.x, m.h.y); }
__device__ __forceinline__ LrMap lr_unpack(float4 v) { return LrMap{make_float2(v.x, v.y), make_float2(v.z, v.w)}; }
__device__ __forceinline__ float2 lr_step(float2 f, float2 u, float2 h, bool cut, float2 one) {
  const float2 r = lr_axpy(f, h, u, one);
  return cut ? u : r;
}
// one more row of a chunk's map (first: the map of the row alone)
__device__ __forceinline__ void lr_extend(LrMap& m, bool first, float2 f, float2 u, bool cut, float2 one) {
  m.h = first ? u : lr_step(f, u, m.h, cut, one);
  m.a = first ? f : mul2(m.a, f);
  if (cut) m.a = same2(-0.0f);
}
// the same from the last row to the first, of the gradient
__device__ __forceinline__ void lr_extend_back(LrMap& m, bool first, float2 f, float2 d, bool cut, float2 one) {
  m.h = mul2(f, first ? d : add2(m.h, d, one));
  m.a = first ? f : mul2(m.a, f);
  if (cut) {
    m.a = same2(-0.0f);
    m.h = same2(0.0f);
  }
}
// dg of a row: (dh (h_{t-1} - v)) (f z)
__device__ __forceinline__ uint32_t lr_dg(float2 d, float2 diff, float2 f, float2 z) {
  const float2 r = mul2(mul2(d, diff), mul2(f, z));
  return bf_pair(r.x, r.y);
}

// NS: tensors that come in by asynchronous copies.  A chunk's raw values take 16 words more than they have, so that the two chunks of a warp read
// different banks.
constexpr int LR_RAW = LR_CHUNK * 16 + 16;
template <int NS, bool JOINED>
struct __align__(16) LrShared {
  uint32_t raw[LR_WARPS][NS][LR_BLOCK][LR_RAW];  // of each warp: [tensor][chunk][row, lane of 16]
  float tab[LR_TAB];
  float4 block[2][LR_WARPS][16];                         // the block maps of this round; two rounds
  float4 span[2][JOINED ? LR_MAXC : 1][16];             // the span maps of the cluster; two rounds
  float2 start[LR_MAXC + 1][16];                         // what comes into the spans of the cluster, and into the next round
  unsigned long long arrived[2];                         // transaction barriers of the span maps, two rounds
  int gone;                                              // a wait ran out
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
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

struct LrArgs {
  const uint16_t *g, *v, *dy;
  const uint8_t* flags;
  const float *first, *states;                           // what comes into the first chunk; backward: the states in front of the chunks
  uint16_t *y, *dg, *dv;
  float *last, *save;                                    // what comes out of the last chunk; forward: the states for the backward pass
  size_t ld, ld_y, ld_d;
  int S, D, n, cl;                                       // n chunks, cl CTAs of a cluster
  int strips, items, step, rounds;                       // strips of a row and of all sequences (items); from a CTA's item to its next, rounds of one
  int* status;
};

// Where a thread is: rank in its cluster, warp (of the span, in the order of the pass), chunk o of its block, lane of 16.
template <bool JOINED>
struct LrPlace {
  int rank, warp, o, lane;
  __device__ __forceinline__ LrPlace(const LrArgs& p) {
    rank = JOINED ? blockIdx.x % p.cl : 0;
    warp = threadIdx.x >> 5;
    o = (threadIdx.x >> 4) & 1;
    lane = threadIdx.x & 15;
  }
};
// What a CTA does in a round: the span `span` (in the order of the pass) of sequence b and the 32 channels from ch0 on.  Round k of an item (a sequence's
// strip); only a lone CTA has more than one item.
template <bool BACK, bool JOINED>
struct LrRound {
  int item, k, b, ch0, span;
  __device__ __forceinline__ LrRound(const LrArgs& p, const LrPlace<JOINED>& at) : item(JOINED ? blockIdx.x / p.cl : blockIdx.x), k(0) { begin(p, at); }
  __device__ __forceinline__ void begin(const LrArgs& p, const LrPlace<JOINED>& at) {
    b = item / p.strips;
    ch0 = (item - b * p.strips) * LR_CH;
    span = at.rank;
  }
  __device__ __forceinline__ bool more(const LrArgs& p) const { return item < p.items; }
  __device__ __forceinline__ bool last(const LrArgs& p) const { return k + 1 == p.rounds; }
  __device__ __forceinline__ void next(const LrArgs& p, const LrPlace<JOINED>& at) {
    ++k;
    span += JOINED ? p.cl : 1;
    if (k < p.rounds) return;
    k = 0;
    item += p.step;
    begin(p, at);
  }
  // the first row of a warp's chunk; below 0 or from S on there is none
  __device__ __forceinline__ int row(const LrArgs& p, int warp, int o) const {
    const int chunk = (span * LR_WARPS + warp) * LR_BLOCK + o;
    return (BACK ? p.n - 1 - chunk : chunk) * LR_CHUNK;
  }
  // all rows and all channels exist
  __device__ __forceinline__ bool full(const LrArgs& p) const {
    return ch0 + LR_CH <= p.D && (span + 1) * LR_ROWS <= (BACK ? p.n * LR_CHUNK : p.S) && (!BACK || span > 0 || p.S % LR_CHUNK == 0);
  }
  __device__ __forceinline__ size_t state(const LrArgs& p, const LrPlace<JOINED>& at) const { return (size_t)b * p.D + ch0 + 2 * at.lane; }
};

// A thread's place in a tensor of the rows, in pieces of WORDS words: where it reads or writes for the first chunk of its warp's block (WORDS 0: of its own
// chunk, its own channels).  Kept from round to round: worked out anew for every row the addresses were a tenth of the instructions.
template <int WORDS>
struct LrCursor {
  static constexpr int PER = WORDS ? 16 / WORDS : 16, ROWS = 32 / PER;                // pieces of a row, rows of an instruction
  const uint16_t* at;
  template <bool BACK, bool JOINED>
  __device__ __forceinline__ void begin(const uint16_t* x, size_t ld, const LrArgs& p, const LrPlace<JOINED>& w, const LrRound<BACK, JOINED>& r) {
    const int l = threadIdx.x & 31, row = WORDS ? l / PER : 0;
    at = x + ((long long)r.b * p.S + r.row(p, w.warp, WORDS ? 0 : w.o) + row) * (long long)ld + r.ch0 + (WORDS ? 2 * (l % PER * WORDS) : 2 * w.lane);
  }
  template <bool BACK>
  __device__ __forceinline__ void next(size_t ld, const LrArgs& p) {
    const long long d = (long long)p.cl * LR_ROWS * (long long)ld;
    at += BACK ? -d : d;
  }
};
// The rows of a warp's block of one tensor on their way.  The address is only followed where the row exists.
template <bool FULL, int WORDS, bool BACK, bool JOINED>
__device__ __forceinline__ void lr_fetch(uint32_t (*raw)[LR_RAW], const LrCursor<WORDS>& c, const uint16_t* x, size_t ld, const LrArgs& p, const LrPlace<JOINED>& at,
                                         const LrRound<BACK, JOINED>& r) {
  constexpr int PER = LrCursor<WORDS>::PER, ROWS = LrCursor<WORDS>::ROWS;
  const int l = threadIdx.x & 31, word = l % PER * WORDS, row = l / PER;
  const bool have = FULL || r.ch0 + 2 * word < p.D;
  const uint32_t dst = smem_u32(raw) + 4 * (row * 16 + word);
  const int t0 = r.row(p, at.warp, 0) + row;
#pragma unroll
  for (int j = 0; j < LR_BLOCK * LR_CHUNK / ROWS; ++j) {
    // chunk 1 lies behind chunk 0 forward and before it backward
    const int o = j * ROWS / LR_CHUNK, i = j * ROWS % LR_CHUNK, off = (BACK ? -o : o) * LR_CHUNK + i;
    const bool there = FULL || (have && (unsigned)(t0 + off) < (unsigned)p.S);
    copy_async<WORDS>(dst + 4 * (o * LR_RAW + i * 16), there ? c.at + off * (long long)ld : x, there);
  }
}
// the flag of the row `lane` of a chunk of n rows from t on
template <bool FLAGS>
__device__ __forceinline__ uint32_t lr_flag(const LrArgs& p, int b, int lane, int t, int n) {
  return FLAGS && lane < min(n, LR_CHUNK) ? p.flags[(size_t)b * p.S + t + lane] : 0u;
}
// work(std::true_type) with cuts of a warp's rows, work(std::false_type) without: rows without a cut need no selection, and cuts are few (65536 rows of 512
// channels with a cut every 700: 121 -> 110 us forward, 164 -> 159 backward)
template <bool FLAGS, typename W>
__device__ __forceinline__ void lr_with_cuts(uint32_t cuts, W&& work) {
  if (FLAGS && cuts) work(std::true_type{});
  else work(std::false_type{});
}
// The gates of a chunk.  A NaN comes out of the table as an infinity's gate and is put right here.  Whether there is one (or an infinity) shows the sum
// of all words times zero.
__device__ __forceinline__ void lr_gates(const uint32_t* raw, const float* tab, float2 f[LR_CHUNK], float2 z[LR_CHUNK]) {
  __nv_bfloat162 odd = __float2bfloat162_rn(0.0f);
#pragma unroll
  for (int i = 0; i < LR_CHUNK; ++i) {
    const uint32_t w = raw[i * 16];
    lr_gate2<true>(w, tab, f[i], z[i]);
    odd = __hfma2(reinterpret_cast<const __nv_bfloat162&>(w), __float2bfloat162_rn(0.0f), odd);
  }
  if (reinterpret_cast<uint32_t&>(odd) & 0x7fff7fffu) {
#pragma unroll
    for (int i = 0; i < LR_CHUNK; ++i) {
      const uint32_t w = raw[i * 16];
      if ((w & 0x7fffu) > 0x7f80u) f[i].x = z[i].x = __int_as_float(0x7fffffff);
      if (((w >> 16) & 0x7fffu) > 0x7f80u) f[i].y = z[i].y = __int_as_float(0x7fffffff);
    }
  }
}
__device__ __forceinline__ LrMap lr_from(const LrMap& m, int lane) {
  return LrMap{make_float2(__shfl_sync(0xffffffffu, m.a.x, lane), __shfl_sync(0xffffffffu, m.a.y, lane)),
               make_float2(__shfl_sync(0xffffffffu, m.h.x, lane), __shfl_sync(0xffffffffu, m.h.y, lane))};
}
// The hand-over of a round: the map of this thread's chunk in, what comes into the chunk out; `s`, what comes into the round, becomes what comes into
// the next one.  `turn` counts the rounds of the CTA; `meanwhile` is done while the maps of the others are on their way.
// The maps of two rounds have places of their own: a warp writes its block's map of round r + 2 behind a barrier of round r + 1, which all warps pass
// when they have read round r's; a CTA sends its span's map of round r + 2 when it has all of round r + 1, that of the receiver among them, which was
// sent behind the barrier that the receiver's reader of round r has passed too.
template <bool FULL, bool BACK, int NS, bool JOINED, typename M>
__device__ __forceinline__ float2 lr_hand_over(LrShared<NS, JOINED>& sh, const LrArgs& p, const LrPlace<JOINED>& at, const LrRound<BACK, JOINED>& r, int turn,
                                               const LrMap& mine, float2& s, float2 one, M&& meanwhile) {
  const int chunks = p.n - r.span * LR_WARPS * LR_BLOCK, blocks = (chunks + 1) / LR_BLOCK;               // from the CTA's first ones on
  const LrMap other = lr_from(mine, threadIdx.x ^ 16), both = lr_compose(other, mine, one);              // `both`: in the lanes of chunk 1
  const bool two = FULL || chunks > at.warp * LR_BLOCK + 1;
  float4(*const maps)[16] = sh.block[turn & 1];
  uint64_t* bar = reinterpret_cast<uint64_t*>(&sh.arrived[turn & 1]);
  if (at.o == (two ? 1 : 0)) maps[at.warp][at.lane] = lr_pack(two ? both : mine);
  if (JOINED && threadIdx.x == 0) mbar_expect_tx(bar, p.cl * 16 * sizeof(float4));
  __syncthreads();
  // a group in each half of the warp
  LrMap group = lr_unpack(maps[at.o * LR_GROUP][at.lane]), before = group;
#pragma unroll
  for (int i = 1; i < LR_GROUP; ++i) {
    const LrMap m = lr_unpack(maps[at.o * LR_GROUP + i][at.lane]);
    if (i == (at.warp & 3)) before = group;
    if (FULL || at.o * LR_GROUP + i < blocks) group = lr_compose(group, m, one);
  }
  const int half = at.warp / LR_GROUP;
  const LrMap g0 = lr_from(group, at.lane), g1 = lr_from(group, 16 + at.lane);
  LrMap span = g0;
  if (FULL || blocks > LR_GROUP) span = lr_compose(g0, g1, one);
  float2 start = s;
  if (!JOINED) {
    s = lr_apply(span, s, one);
  } else {
    float4(*const place)[16] = sh.span[turn & 1];
    const int to = at.warp + LR_WARPS * at.o;
    if (to < p.cl) store_in_cluster(&place[at.rank][at.lane], bar, to, lr_pack(span));
    meanwhile();
    if (at.warp == 0) {   // a lane a channel: the packed instructions take longer one after the other (1 x 65536 x 64 58.7 -> 55.9 us)
      constexpr int BATCH = 4;
      const int l = threadIdx.x & 31;
      mbar_wait_warp(bar, (turn >> 1) & 1, &sh.gone, p.status);
      const int spans = min(p.cl, (p.n + LR_WARPS * LR_BLOCK - 1) / (LR_WARPS * LR_BLOCK) - (r.span - at.rank));
      const float* maps = reinterpret_cast<const float*>(place) + l / 2 * 4 + l % 2;
      float* in = reinterpret_cast<float*>(sh.start) + l;
      float c = in[LR_MAXC * LR_CH];
      int i = 0;
      for (; i + BATCH <= spans; i += BATCH) {
        float m[BATCH][2];
#pragma unroll
        for (int j = 0; j < BATCH; ++j) m[j][0] = maps[(i + j) * 64], m[j][1] = maps[(i + j) * 64 + 2];
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
          in[(i + j) * LR_CH] = c;
          c = lr_closed(m[j][0]) ? m[j][1] : fadd(fmul(m[j][0], c), m[j][1]);
        }
      }
      for (; i < spans; ++i) {
        in[i * LR_CH] = c;
        c = lr_closed(maps[i * 64]) ? maps[i * 64 + 2] : fadd(fmul(maps[i * 64], c), maps[i * 64 + 2]);
      }
      in[LR_MAXC * LR_CH] = c;
    }
    __syncthreads();
    start = sh.start[at.rank][at.lane];
    s = sh.start[LR_MAXC][at.lane];
  }
  before = lr_from(before, half * 16 + at.lane);
  if (half) start = lr_apply(g0, start, one);
  if (at.warp & 3) start = lr_apply(before, start, one);
  const float2 second = lr_apply(other, start, one);
  return at.o ? second : start;
}
// before the first round: the barriers, known to the cluster before anyone sends, and the table on its way
template <int NS, bool JOINED>
__device__ __forceinline__ void lr_open(LrShared<NS, JOINED>& sh, const LrArgs& p) {
  if (JOINED) {
    if (threadIdx.x == 0) {
      sh.gone = 0;
      mbar_init(reinterpret_cast<uint64_t*>(&sh.arrived[0]), 1);
      mbar_init(reinterpret_cast<uint64_t*>(&sh.arrived[1]), 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    cluster_arrive();
  }
  const uint32_t dst = smem_u32(sh.tab);
  for (int i = threadIdx.x; i < LR_TAB / 4; i += LR_T) copy_async<4>(dst + 16 * i, lr_table_image.m + 4 * i, true);
}
// no CTA leaves while another one may still send to it (after a wait that ran out)
__device__ __forceinline__ void lr_close() {
  cluster_arrive();
  cluster_wait();
}

// Measured on a B200 (its copy moves 6.53 TB/s), calls one behind the other on inputs that change: 4 x 2048 x 2048 29 us forward and 41 backward, where
// the bytes alone would take 15 and 26; 8 x 4096 x 2048 106 and 152 of 62 and 103 (with the L2 cache flushed in front of every call 113 and 158); 3 x 1999 x
// 1502, pieces of 4 bytes, 24 and 35 of 8 and 14; 1 x 65536 x 512 with cuts 93 and 132 of 31 and 51.  The lone CTAs of the first two are bound by what a round
// waits for, lookups and the hand-over's barrier with 16 warps on an SM (issue slots 54 %, L1 60 %, no arithmetic pipe above 50 %, some 500 instructions a
// round of 8 rows a warp forward), on 256 of 296 places; the last by the steps that a round of a cluster has to wait for one after the other.
template <int WORDS, bool FLAGS, bool JOINED>
__global__ void __launch_bounds__(LR_T, 2) k_linrec_fwd(const __grid_constant__ LrArgs p) {
  extern __shared__ __align__(16) char smem[];
  LrShared<2, JOINED>& sh = *reinterpret_cast<LrShared<2, JOINED>*>(smem);
  const LrPlace<JOINED> at(p);
  const float2 one = same2(c_one);
  lr_open(sh, p);
  grid_dep();
  uint32_t(*raw)[LR_BLOCK][LR_RAW] = sh.raw[at.warp];
  LrRound<false, JOINED> r(p, at), ahead = r;
  uint32_t flag = 0;                                     // compared in the round that uses it: a comparison here waits for the load
  float2 s = make_float2(0.0f, 0.0f), first = s;
  LrCursor<WORDS> cg, cv;
  LrCursor<0> cy;
  auto fetch = [&] {
    const LrRound<false, JOINED>& r = ahead;                       // of the round that is fetched
    if (r.k == 0) {
      cg.begin(p.g, p.ld, p, at, r);
      cv.begin(p.v, p.ld, p, at, r);
    } else {
      cg.template next<false>(p.ld, p);
      cv.template next<false>(p.ld, p);
    }
    if (r.full(p)) {
      lr_fetch<true>(raw[0], cg, p.g, p.ld, p, at, r);
      lr_fetch<true>(raw[1], cv, p.v, p.ld, p, at, r);
    } else {
      lr_fetch<false>(raw[0], cg, p.g, p.ld, p, at, r);
      lr_fetch<false>(raw[1], cv, p.v, p.ld, p, at, r);
    }
    const int t = r.row(p, at.warp, at.o);
    flag = lr_flag<FLAGS>(p, r.b, at.lane, t, p.S - t);
    if (p.first && ahead.k == 0 && r.ch0 + 2 * at.lane < p.D) first = *reinterpret_cast<const float2*>(p.first + r.state(p, at));
    ahead.next(p, at);
  };
  fetch();
  copies_done();
  __syncthreads();                                       // the table
  if (JOINED) cluster_wait();
  int turn = 0;
  for (; r.more(p); r.next(p, at), ++turn) {
    const int t0 = r.row(p, at.warp, at.o);
    if (r.k == 0) {
      s = first;
      if (JOINED && threadIdx.x < 16) sh.start[LR_MAXC][at.lane] = s;                 // read behind the barrier of the hand-over
      cy.begin(p.y, p.ld_y, p, at, r);
    }
    auto round = [&](auto whole) {
      constexpr bool FULL = decltype(whole)::value;
      const int n = FULL ? LR_CHUNK : p.S - t0;          // n rows of the chunk exist
      const bool have = FULL || r.ch0 + 2 * at.lane < p.D;
      const uint32_t all = FLAGS ? __ballot_sync(0xffffffffu, flag != 0) : 0u, cuts = (all >> (threadIdx.x & 16)) & 0xffu;
      const uint32_t* q = raw[0][at.o] + at.lane;
      float2 f[LR_CHUNK], u[LR_CHUNK];
      lr_gates(q, sh.tab, f, u);
      LrMap mine;
      lr_with_cuts<FLAGS>(all, [&](auto some) {
#pragma unroll
        for (int i = 0; i < LR_CHUNK; ++i) {
          const uint32_t w = q[LR_BLOCK * LR_RAW + i * 16];
          u[i] = mul2(u[i], make_float2(bflo(w), bfhi(w)));
          if (i == 0 || i < n) lr_extend(mine, i == 0, f[i], u[i], decltype(some)::value && ((cuts >> i) & 1), one);
        }
      });
      __syncwarp();
      const auto next_round = [&] { if (ahead.more(p)) fetch(); };
      if (!JOINED) next_round();
      float2 h = lr_hand_over<FULL>(sh, p, at, r, turn, mine, s, one, next_round);
      if (p.save && n > 0 && have) *reinterpret_cast<float2*>(p.save + r.state(p, at) + ((size_t)r.b * (p.n - 1) + t0 / LR_CHUNK) * p.D) = h;
      uint16_t* out = const_cast<uint16_t*>(cy.at);
      lr_with_cuts<FLAGS>(all, [&](auto some) {
#pragma unroll
        for (int i = 0; i < LR_CHUNK; ++i) {
          h = lr_step(f[i], u[i], h, decltype(some)::value && ((cuts >> i) & 1), one);
          if (i < n && have) *reinterpret_cast<uint32_t*>(out) = bf_pair(h.x, h.y);
          out += p.ld_y;
        }
      });
    };
    if (r.full(p)) round(std::true_type{});
    else round(std::false_type{});
    cy.template next<false>(p.ld_y, p);
    if (p.last && r.last(p) && threadIdx.x < 16 && at.rank == 0 && r.ch0 + 2 * at.lane < p.D) *reinterpret_cast<float2*>(p.last + r.state(p, at)) = s;
    copies_done();
    __syncwarp();
    if (JOINED && *static_cast<volatile int*>(&sh.gone)) break;                    // set before the round's second barrier: all see the same
  }
  if (JOINED) lr_close();
}

template <int WORDS, bool FLAGS, bool JOINED>
__global__ void __launch_bounds__(LR_T, 2) k_linrec_bwd(const __grid_constant__ LrArgs p) {
  extern __shared__ __align__(16) char smem[];
  LrShared<3, JOINED>& sh = *reinterpret_cast<LrShared<3, JOINED>*>(smem);
  const LrPlace<JOINED> at(p);
  const float2 one = same2(c_one);
  lr_open(sh, p);
  grid_dep();
  uint32_t(*raw)[LR_BLOCK][LR_RAW] = sh.raw[at.warp];
  LrRound<true, JOINED> r(p, at), ahead = r;
  uint32_t flag = 0;                                     // compared in the round that uses it: a comparison here waits for the load
  float2 s = make_float2(0.0f, 0.0f), first = s, next = s;                            // next: the state in front of the thread's chunk
  LrCursor<WORDS> cg, cv, cdy;
  LrCursor<0> odv, odg;
  auto fetch = [&] {
    const LrRound<true, JOINED>& r = ahead;                       // of the round that is fetched
    if (r.k == 0) {
      cg.begin(p.g, p.ld, p, at, r);
      cv.begin(p.v, p.ld, p, at, r);
      cdy.begin(p.dy, p.ld_y, p, at, r);
    } else {
      cg.template next<true>(p.ld, p);
      cv.template next<true>(p.ld, p);
      cdy.template next<true>(p.ld_y, p);
    }
    if (r.full(p)) {
      lr_fetch<true>(raw[0], cg, p.g, p.ld, p, at, r);
      lr_fetch<true>(raw[1], cv, p.v, p.ld, p, at, r);
      lr_fetch<true>(raw[2], cdy, p.dy, p.ld_y, p, at, r);
    } else {
      lr_fetch<false>(raw[0], cg, p.g, p.ld, p, at, r);
      lr_fetch<false>(raw[1], cv, p.v, p.ld, p, at, r);
      lr_fetch<false>(raw[2], cdy, p.dy, p.ld_y, p, at, r);
    }
    const int t = r.row(p, at.warp, at.o);
    const bool have = r.ch0 + 2 * at.lane < p.D;
    flag = lr_flag<FLAGS>(p, r.b, at.lane, t, t < 0 ? 0 : p.S - t);
    if (t >= 0 && have) next = *reinterpret_cast<const float2*>(p.states + r.state(p, at) + ((size_t)r.b * (p.n - 1) + t / LR_CHUNK) * p.D);
    if (p.first && ahead.k == 0 && have) first = *reinterpret_cast<const float2*>(p.first + r.state(p, at));
    ahead.next(p, at);
  };
  fetch();
  copies_done();
  __syncthreads();                                       // the table
  if (JOINED) cluster_wait();
  int turn = 0;
  for (; r.more(p); r.next(p, at), ++turn) {
    const int t0 = r.row(p, at.warp, at.o);
    if (r.k == 0) {
      s = first;
      if (JOINED && threadIdx.x < 16) sh.start[LR_MAXC][at.lane] = s;                 // read behind the barrier of the hand-over
      odv.begin(p.dv, p.ld_d, p, at, r);
      odg.begin(p.dg, p.ld_d, p, at, r);
    }
    auto round = [&](auto whole) {
      constexpr bool FULL = decltype(whole)::value;
      const int n = FULL ? LR_CHUNK : t0 < 0 ? 0 : p.S - t0;                          // n rows of the chunk exist
      const bool have = FULL || r.ch0 + 2 * at.lane < p.D;
      const uint32_t all = FLAGS ? __ballot_sync(0xffffffffu, flag != 0) : 0u, cuts = (all >> (threadIdx.x & 16)) & 0xffu;
      float2 h = next;
      const uint32_t* q = raw[0][at.o] + at.lane;
      float2 f[LR_CHUNK], z[LR_CHUNK];
      uint32_t wv[LR_CHUNK], wd[LR_CHUNK];
      lr_gates(q, sh.tab, f, z);
#pragma unroll
      for (int i = 0; i < LR_CHUNK; ++i) {
        wv[i] = q[LR_BLOCK * LR_RAW + i * 16];
        wd[i] = q[2 * LR_BLOCK * LR_RAW + i * 16];
      }
      __syncwarp();
      const auto next_round = [&] { if (ahead.more(p)) fetch(); };
      if (!JOINED) next_round();
      LrMap mine;
      mine.a = mine.h = same2(0.0f);
      lr_with_cuts<FLAGS>(all, [&](auto some) {
#pragma unroll
        for (int i = LR_CHUNK - 1; i >= 0; --i)
          if (i < n) lr_extend_back(mine, i == (FULL ? LR_CHUNK : min(n, LR_CHUNK)) - 1, f[i], make_float2(bflo(wd[i]), bfhi(wd[i])), decltype(some)::value && ((cuts >> i) & 1), one);
      });
      float2 c = lr_hand_over<FULL>(sh, p, at, r, turn, mine, s, one, next_round);
      uint16_t *dv = const_cast<uint16_t*>(odv.at) + (LR_CHUNK - 1) * p.ld_d, *dg = const_cast<uint16_t*>(odg.at) + (LR_CHUNK - 1) * p.ld_d;
      lr_with_cuts<FLAGS>(all, [&](auto some) {
        float2 diff[LR_CHUNK];                             // h_{t-1} - v
#pragma unroll
        for (int i = 0; i < LR_CHUNK; ++i) {
          const bool cut = decltype(some)::value && ((cuts >> i) & 1);
          const float2 v = make_float2(bflo(wv[i]), bfhi(wv[i]));
          diff[i] = lr_sub(cut ? same2(0.0f) : h, v);
          h = lr_step(f[i], mul2(z[i], v), h, cut, one);
        }
#pragma unroll
        for (int i = LR_CHUNK - 1; i >= 0; --i, dv -= p.ld_d, dg -= p.ld_d) {
          if (i >= n) continue;
          const float2 d = add2(c, make_float2(bflo(wd[i]), bfhi(wd[i])), one), w = mul2(d, z[i]);
          c = mul2(f[i], d);
          if (decltype(some)::value && ((cuts >> i) & 1)) c = same2(0.0f);
          if (!have) continue;
          *reinterpret_cast<uint32_t*>(dv) = bf_pair(w.x, w.y);
          *reinterpret_cast<uint32_t*>(dg) = lr_dg(d, diff[i], f[i], z[i]);
        }
      });
    };
    if (r.full(p)) round(std::true_type{});
    else round(std::false_type{});
    odv.template next<true>(p.ld_d, p);
    odg.template next<true>(p.ld_d, p);
    if (p.last && r.last(p) && threadIdx.x < 16 && at.rank == 0 && r.ch0 + 2 * at.lane < p.D) *reinterpret_cast<float2*>(p.last + r.state(p, at)) = s;
    copies_done();
    __syncwarp();
    if (JOINED && *static_cast<volatile int*>(&sh.gone)) break;                    // set before the round's second barrier: all see the same
  }
  if (JOINED) lr_close();
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
  const float2 one = same2(c_one);
  float2 f[LR_CHUNK], z[LR_CHUNK], diff[LR_CHUNK];
  LrMap m;
  m.a = m.h = same2(0.0f);
#pragma unroll
  for (int t = 0; t < LR_CHUNK; ++t) {
    if (t >= n) continue;
    lr_gate2<false>(wg[t], nullptr, f[t], z[t]);
    const bool cut = (cuts >> t) & 1;
    const float2 v = make_float2(bflo(wv[t]), bfhi(wv[t])), u = mul2(z[t], v);
    if (!BWD) lr_extend(m, t == 0, f[t], u, cut, one);
    diff[t] = lr_sub(cut ? same2(0.0f) : h, v);
    h = lr_step(f[t], u, h, cut, one);
    if (!BWD) *reinterpret_cast<uint32_t*>(p.y + (row + t) * p.ld_y + c0) = bf_pair(h.x, h.y);
  }
  if (BWD) {
    float2 c = s;
#pragma unroll
    for (int t = LR_CHUNK - 1; t >= 0; --t) {
      if (t >= n) continue;
      const bool cut = (cuts >> t) & 1;
      const float2 dy = make_float2(bflo(wd[t]), bfhi(wd[t])), d = add2(c, dy, one), w = mul2(d, z[t]);
      c = cut ? same2(0.0f) : mul2(f[t], d);
      lr_extend_back(m, t == n - 1, f[t], dy, cut, one);
      *reinterpret_cast<uint32_t*>(p.dv + (row + t) * p.ld_d + c0) = bf_pair(w.x, w.y);
      *reinterpret_cast<uint32_t*>(p.dg + (row + t) * p.ld_d + c0) = lr_dg(d, diff[t], f[t], z[t]);
    }
  }
  if (p.last) *reinterpret_cast<float2*>(p.last + at) = lr_apply(m, s, one);
}

// How a call is dealt out.  More CTAs of a cluster, of any number, while two on an SM have room for all of them.  A cluster needs its CTAs on one part of the
// GPU, and they do not pack: of 296 CTAs, two on an SM, 264 fit in clusters of 4, 240 of 8 and 224 of 16, and a pass that needed 256 where 224 fit took
// twice as long; so the runtime is asked once per device and kernel what fits.
// Where there are strips enough, lone CTAs go through several, about as many as the others.  The CTAs of a grid are not spread evenly: 256 of them ran in
// 42 us where three fitted on an SM and in 31 where two did (4 x 2048 x 2048 forward).  So no more are let on an SM than are needed, by the shared memory
// that is asked for.
using LrKernel = void (*)(const LrArgs);
constexpr int LR_MAXR = 2;                               // lone CTAs on an SM (three, with 80 registers a thread, took 30.2 us where two take 29.0)
struct LrFits {
  std::mutex lock;
  bool known[MAX_DEVICES] = {};
  struct {
    int lone[LR_MAXR], joined[LR_MAXC - 1];              // CTAs at once on the GPU: lone, 1 .. on an SM; in clusters of 2 ..
  } dev[MAX_DEVICES] = {};
};
struct LrLaunch {
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = {};
  LrLaunch(unsigned grid, int cl, size_t smem, cudaStream_t st) {
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cl;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(LR_T);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
  }
};
// shared memory of a CTA of which r fit on an SM and r + 1 do not (an SM has 228 KB; each CTA takes 1 KB more than it asks for)
static size_t lr_smem(size_t need, int r) {
  const size_t least = (size_t)228 * 1024 / (r + 1);
  return need > least ? need : least;
}
struct LrVariant {
  LrKernel kern;
  size_t smem;
};
// the CTAs that run at once, 0 if they do not run at all
static int lr_at_once(const LrVariant& v, size_t smem, int cl) {
  LrLaunch l((unsigned)cl, cl, smem, nullptr);
  int clusters = 0;
  if (cudaOccupancyMaxActiveClusters(&clusters, v.kern, &l.cfg) == cudaSuccess) return clusters * cl;
  cudaGetLastError();
  return 0;
}
template <bool BACK, int WORDS, bool FLAGS>
static int lr_run(LrArgs& p, int B, cudaStream_t st) {
  static LrFits fits;
  constexpr int NS = BACK ? 3 : 2;
  LrVariant lone{nullptr, sizeof(LrShared<NS, false>)}, joined{nullptr, sizeof(LrShared<NS, true>)};
  if constexpr (BACK) lone.kern = k_linrec_bwd<WORDS, FLAGS, false>, joined.kern = k_linrec_bwd<WORDS, FLAGS, true>;
  else lone.kern = k_linrec_fwd<WORDS, FLAGS, false>, joined.kern = k_linrec_fwd<WORDS, FLAGS, true>;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return DET_ERR_CUDA;
  auto& fit = fits.dev[dev];
  {
    std::lock_guard<std::mutex> hold(fits.lock);
    if (!fits.known[dev]) {
      const auto allow = [](const LrVariant& v, size_t smem) {
        return cudaFuncSetAttribute((const void*)v.kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) == cudaSuccess;
      };
      if (!allow(lone, lr_smem(lone.smem, 1)) || !allow(joined, lr_smem(joined.smem, 2)) ||
          cudaFuncSetAttribute((const void*)joined.kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
        cudaGetLastError();
        return DET_ERR_CUDA;
      }
      for (int r = 1; r <= LR_MAXR; ++r) fit.lone[r - 1] = lr_at_once(lone, lr_smem(lone.smem, r), 1);
      for (int cl = 2; cl <= LR_MAXC; ++cl) fit.joined[cl - 2] = lr_at_once(joined, lr_smem(joined.smem, 2), cl);
      fits.known[dev] = true;
    }
  }
  p.strips = (p.D + LR_CH - 1) / LR_CH;
  p.items = B * p.strips;
  const int spans = (p.S + LR_ROWS - 1) / LR_ROWS;
  p.cl = 1;
  for (int cl = 2; cl <= LR_MAXC && cl <= spans; ++cl)
    if ((long long)p.items * cl <= fit.joined[cl - 2]) p.cl = cl;
  p.rounds = (spans + p.cl - 1) / p.cl;
  p.cl = (spans + p.rounds - 1) / p.rounds;              // as many as have work in every round
  p.step = p.items;
  if (p.cl > 1) {
    LrLaunch l((unsigned)(p.items * p.cl), p.cl, lr_smem(joined.smem, 2), st);
    note_launch();
    cudaLaunchKernelEx(&l.cfg, joined.kern, p);
  } else {
    const int most = *std::max_element(fit.lone, fit.lone + LR_MAXR);
    if (most <= 0) return DET_ERR_CUDA;
    const int passes = (p.items + most - 1) / most;
    p.step = (p.items + passes - 1) / passes;
    int r = 0;
    while (r < LR_MAXR - 1 && p.step > fit.lone[r]) ++r;
    LrLaunch l((unsigned)p.step, 1, lr_smem(lone.smem, r + 1), st);
    note_launch();
    cudaLaunchKernelEx(&l.cfg, lone.kern, p);
  }
  DET_CHECK_LAUNCH();
  return DET_OK;
}
static int lr_any(bool back, LrArgs& p, int B, cudaStream_t st) {
  p.n = (p.S + LR_CHUNK - 1) / LR_CHUNK;
  if (p.S <= LR_CHUNK) {
    const size_t threads = (size_t)B * (p.D / 2);
    launch_after(back ? k_linrec_chunk<true> : k_linrec_chunk<false>, dim3((unsigned)((threads + 127) / 128)), 128, 0, st, p, threads);
    DET_CHECK_LAUNCH();
    return DET_OK;
  }
  // whole pieces of 16 bytes where the tensors allow it
  const bool wide = p.D % 8 == 0 && p.ld % 8 == 0 && aligned16(p.g) && aligned16(p.v) && (!back || (p.ld_y % 8 == 0 && aligned16(p.dy)));
  if (back) return wide ? (p.flags ? lr_run<true, 4, true>(p, B, st) : lr_run<true, 4, false>(p, B, st))
                        : (p.flags ? lr_run<true, 1, true>(p, B, st) : lr_run<true, 1, false>(p, B, st));
  return wide ? (p.flags ? lr_run<false, 4, true>(p, B, st) : lr_run<false, 4, false>(p, B, st))
              : (p.flags ? lr_run<false, 1, true>(p, B, st) : lr_run<false, 1, false>(p, B, st));
}
static int lr_check(const void* a, const void* b, int ld, int B, int S, int D) {
  if (!a || !b || B < 0 || S < 0 || D <= 0 || ld < D) return DET_ERR_ARG;
  if (D % 2 || ld % 2 || S > (1 << 30)) return DET_ERR_SHAPE;
  if ((long long)B * ((D + LR_CH - 1) / LR_CH) > (1 << 26)) return DET_ERR_SHAPE;
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
  return B > 0 && S > 0 && D > 0 ? (size_t)B * (((size_t)S + LR_CHUNK - 1) / LR_CHUNK) * (size_t)D : 0;
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
