// dc_attend_kernel.cuh -- the attention kernel of prompts and drafted trees on the
// tensor cores; instantiated in dc_prompt.cu and dc_tree.cu.
//
// One persistent CTA per SM takes work items in turn: two tiles of 128 query rows (A and
// B) of one KV head over a run of key tiles of 128 tokens. Warp roles (384 threads):
//   warps 0-3, 4-7  softmax warpgroups of tiles A and B, one query row (TMEM lane) a thread;
//   warp 8          producer: publishes the items to the other warps, loads the query tiles,
//                   then K and V tiles in the order in which the products take them, by TMA
//                   through one ring of stages;
//   warp 9          MMA issuer (one lane):
//                     S_X  = Q_X K^T     [128 rows x 128 keys]   from shared memory
//                     O_X += P_X V       [128 rows x D]          P_X from TMEM
//   warps 10, 11    look over the values of key tiles that are masked in part.
// TMEM columns: S_A [0, 128), S_B [128, 256), O_A [256, 256 + D), O_B [384, 384 + D). A
// warpgroup reads its S (the whole row in registers), writes the weights P over its
// first 64 columns in the inputs' type, and the second product reads them there. The
// issuer sends S_X of the next key tile right behind O_X of this one, so that one
// warpgroup's softmax runs under the other's products. P goes in two halves, each with its
// own barrier: the product with the first half's values starts while the second is computed.
//
// P is rounded to the inputs' type because the tensor cores take both operands of a product in one type: half a unit in
// the last place of each weight, of the order of the result's own rounding (relative error against 64 bits 2.3e-3 in bf16
// where sums in 32 bits alone have 1.7e-3). l sums the weights unrounded: the roundings have no bias, so that l is
// the better sum of either.
//
// Running softmax: m is a row's reference, not always its maximum: it follows the maximum
// only where that is more than 2^24 above it in weights (fp16: 2^15.75), so that O is seldom rescaled
// (P stays below that, which loses nothing in floating point; l and O are in 32 bits, and O is
// finite while a row's values are below 2^104 over its length). With 2^8 a prompt of 4096
// tokens whose scores have a deviation of 2 / 3 took 96 / 102 us instead of 91. The
// completion of S_X also says that O_X is at rest, since the products of one issuer complete
// in order: the warpgroup rescales O itself, with no further barrier.
//
// Items of one tile of queries (single tokens, small trees, short sequences) give their key
// tiles to A and B in turn, both on the same queries, and join the two results at the end:
// the pipeline is the same. Small trees over many short rows take two rows at a time instead, A one
// and B the other, with nothing to join.
//
// A masked key has weight 0, but 0 times a value that is not finite is NaN: warps 10 and 11 look
// over the values that some row of the tile must not see, in shared memory, before their stage
// is released, and a tile of rows that meets such a value is recomputed by attend_row, which
// reads only what a row sees.
//
// What bounds it: a step of both halves needs 2048 cycles of products at D 128 and takes about 2650
// (2390 without any softmax): the tensor pipe and the hand-over between the halves. One sequence
// of 32768 tokens, 32 query heads on 8 KV heads: 5.4 ms, 1.63 PFLOP/s; 4096 tokens: 91 us; trees of 16
// nodes over 2048 rows of 8192 tokens read the cache at 7.2 TB/s (1.18 ms). At D 64 a step has 1024
// cycles of products and takes 2650 all the same: there the softmax of two warps per scheduler bounds it (4096
// tokens, 64 heads: 149 us; without exponentials 120, without maxima 139. A quarter of the
// exponentials as polynomials: 162. A third S in TMEM, so that no warp waits for one: 148-154).
//
// Results go through shared memory, 128 bytes of each of a warp's 32 rows at a time, so that they
// leave together (a thread writing its own row cost 5000 to 7000 cycles an item).
//
// Barriers: every wait is bounded, and the roles meet at mbarriers only. A wait that gives up
// sets *abort; every warp then leaves its loop, the producer and the issuer wait for what they
// have in flight, and the status word says so.
#pragma once

#include <cuda.h>

#include "dc_attend.cuh"
#include "dc_device.h"
#include "dc_sm100.cuh"

namespace dc {
using namespace sm100;

namespace {

constexpr int kAttThreads = 384;
// Registers: 168 a thread at launch, then shared out by warpgroups (the sum stays: 216 +
// 216 + 72 = 3 x 168). A softmax thread holds its whole row of S.
constexpr int kAttRegsRow = 216, kAttRegsIssue = 72;
constexpr int kAttCols = 512;
constexpr int kItemRing = 4;  // items published ahead

template <int D>
struct AttSmem {
  static constexpr int TILE = 128 * D * 2;
  static constexpr int STAGES = D == 128 ? 4 : 8;
  static constexpr int Q = 0;  // two query tiles
  static constexpr int RING = 2 * TILE;
  static constexpr int OUT = RING + STAGES * TILE;  // 4 KB a softmax warp
  static constexpr int MISC = OUT + 8 * 4096;       // barriers
  static constexpr int ITEM = MISC + 512;           // Published [4]
  static constexpr int FLAG = ITEM + kItemRing * 96;  // int [4][2]: what warps 10 and 11 found
  static constexpr int XCH = MISC + 1024;           // float2 [2][128]: m, l of both tiles
  static constexpr int BYTES = XCH + 2048;
  static_assert(BYTES <= 232448, "more shared memory than a CTA may have");
};

__device__ __forceinline__ AttnItem load_item(const AttnArgs& a, int i) {
  const int4* p = reinterpret_cast<const int4*>(a.items + i);
  const int4 x = __ldg(p), y = __ldg(p + 1), z = __ldg(p + 2), w = __ldg(p + 3);
  return AttnItem{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w, w.x, w.y, w.z, w.w};
}

// Trees: the key tiles of all rows, a.tiles each (the cached tokens', then the drafted ones'; rows may
// have fewer), in one line of a.line places for every pair of query tiles, the lines one behind the
// other. Every line has a.ctas CTAs, which take equal parts of it: those that read a row's keys for
// its pairs do so at the same time, the first from HBM and the others from L2 (8 heads, 64 nodes over
// 128 rows of 4097 tokens: 297 MB read, 114 us; with all lines cut as one, so that those CTAs are up
// to half a row apart, 507 MB and 119 us).
__host__ __device__ inline int tree_from(const AttnArgs& a, int b) {
  const int p = b / a.ctas, i = b - p * a.ctas;
  return p * a.line + i * a.per + (i < a.extra ? i : a.extra);
}

// The CTA that takes place `at`.
__device__ __forceinline__ int tree_cta(const AttnArgs& a, int at) {
  const int p = at / a.line, big = a.extra * (a.per + 1);
  at -= p * a.line;
  return p * a.ctas + (at < big ? at / (a.per + 1) : a.extra + (at - big) / a.per);
}

// The item that starts at place `at` of that line, as far as it goes before `end`.
__device__ __forceinline__ AttnItem tree_item(const AttnArgs& a, int b, int at, int end) {
  const int tpt = kAttRows / a.G, i = at / a.tiles, j0 = at - i * a.tiles;
  const int j1 = min(a.tiles, j0 + end - at);
  AttnItem it;
  it.y = a.two ? 2 * i : i % a.rows;
  it.lb = it.y / a.kvh;
  it.h = it.y % a.kvh;
  it.t0 = a.two ? 0 : i / a.rows * 2 * tpt;
  it.tend = a.nodes;
  it.k0 = 0;
  it.klen = a.rowlen ? __ldg(a.rowlen + it.y) : a.n;
  it.off = kSeesAll;
  const int own = (it.klen + kAttTok - 1) / kAttTok + 1;
  it.j0 = a.two ? 0 : min(j0, own);
  it.j1 = a.two ? own : min(j1, own);
  // a CTA has at most two parts of items: the end of one, then the start of another
  it.slot = j0 == 0 && j1 == a.tiles ? -1 : 2 * b + (j0 == 0 ? 1 : 0);
  it.alt = a.two && it.y + 1 < a.rows ? 2 : it.tend - it.t0 <= tpt;
  it.eA = it.eB = it.j1;
  it.lowA = it.lowB = it.klen;
  return it;
}

// An item's steps: key tile of step i, and which of A (1) and B (2) take it: one each in turn, or
// both from their first step on.
template <bool TREE>
struct Steps {
  int n, j0, j1, alt, look, skipA, skipB, lowA, lowB, draft;
  __device__ __forceinline__ Steps(const AttnItem& it)
      : n((it.j1 - it.j0) << (it.alt == 2)), j0(it.j0), j1(it.j1), alt(it.alt), look(it.alt ? 2 : 1), skipA(max(0, it.j1 - it.eA)),
        skipB(max(0, it.j1 - it.eB)), lowA(it.lowA), lowB(it.lowB),
        draft(TREE ? (it.klen + kAttTok - 1) / kAttTok : -1) {}
  // the tiles that may be masked come first in prompts, last in trees
  __device__ __forceinline__ int tile(int i) const { return TREE ? j0 + (i >> (alt == 2)) : j1 - 1 - i; }
  // whether some row of tile A (x = 0) or B must not see some key of step i's tile
  __device__ __forceinline__ bool masked(int i, int x) const {
    const int j = tile(i);
    return (TREE && j == draft) || (j + 1) * kAttTok > (x ? lowB : lowA);
  }
  // which of those that take the step
  __device__ __forceinline__ int masked(int i) const {
    const int w = alt ? 1 << (i & 1) : (i >= skipA ? 1 : 0) | (i >= skipB ? 2 : 0);
    return (w & 1 && masked(i, 0) ? 1 : 0) | (w & 2 && masked(i, 1) ? 2 : 0);
  }
  // load p of the item's 2 n: V or K of which step. K0 V0 K1 V1 ..., or, where A and B take steps in
  // turn, K0 K1 V0 K2 V1 K3 ...: as the products take them
  __device__ __forceinline__ int load(int p, bool& v) const {
    if (!alt) {
      v = p & 1;
      return p >> 1;
    }
    const bool last = p == 2 * n - 1;
    v = last || (p >= 2 && !(p & 1));
    return last ? n - 1 : v ? (p - 2) >> 1 : p < 2 ? p : (p + 1) >> 1;
  }
  // steps of A (x = 0) or B
  __device__ __forceinline__ int count(int x) const { return alt ? (n + 1 - x) / 2 : max(0, n - (x ? skipB : skipA)); }
};

// Waits as mbar_wait does, in few instructions: what gave up is kept in *abort and recorded at the
// end. Items of few steps run through most of the kernel's code (100 KB of it), so that its size
// counts: with mbar_wait's record at each of the twenty waits, one copy of each warp's loads and one
// of the result's reads (129 -> 105 KB), trees of 8 nodes over 4096 rows of 410 tokens went from
// 285 to 197 us, a prompt of 4096 from 93.5 to 91.2 us.
__device__ __forceinline__ bool att_wait(uint64_t* bar, uint32_t parity, volatile int* abort, int site, uint64_t limit_ns) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = globaltimer_ns();
#pragma unroll 1
  for (;;) {
    if (mbar_try_wait(bar, parity)) return true;
    if (*abort) return false;
    if (globaltimer_ns() - t0 > limit_ns) {
      *abort = site;
      return false;
    }
  }
}

// What the producer tells the other warps of an item.
struct Published {
  AttnItem it;
  int4 of[2];  // A's and B's: first query token, first step, number of steps, lowA or lowB
};
static_assert(sizeof(Published) == 96, "AttSmem::ITEM");

template <class T>
struct Mma;
template <>
struct Mma<TypeBf16> {
  static constexpr float kAbove = 24.f, kRoom = 0.f;
  static constexpr uint32_t id(int N, int b_mn) { return idesc_bf16(128, N, 0, b_mn); }
  // a zero, or NaN where any of the values is not finite
  static __device__ __forceinline__ uint32_t look(uint32_t x, uint32_t acc) {
    __nv_bfloat162 r = __hfma2(*reinterpret_cast<__nv_bfloat162*>(&x), __float2bfloat162_rn(0.f),
                               *reinterpret_cast<__nv_bfloat162*>(&acc));
    return *reinterpret_cast<uint32_t*>(&r);
  }
};
template <>
struct Mma<TypeHalf> {
  // 2^16 is past the type's range. A weight below 2^-14 loses bits, one below 2^-25 is lost. So a new reference lies 2^5
  // below the maximum: the n smaller weights of a row are off by n 2^-30 of the largest at most, a quarter of the type's
  // rounding for 131072 keys (by n 2^-25 with the maximum itself: 1048575 keys of weight 2^-25.2 beside one of 1 were all
  // lost, 2.6% of the result). It leaves 2^10.75 to rise before the next one: a prompt of 4096 tokens takes 94 us as
  // before with scores of deviation 1, 101 instead of 95 with 3; 2^7 below: 103.
  static constexpr float kAbove = 15.75f, kRoom = 5.f;
  static constexpr uint32_t id(int N, int b_mn) { return idesc_f16(128, N, 0, b_mn); }
  static __device__ __forceinline__ uint32_t look(uint32_t x, uint32_t acc) {
    __half2 r = __hfma2(*reinterpret_cast<__half2*>(&x), __float2half2_rn(0.f), *reinterpret_cast<__half2*>(&acc));
    return *reinterpret_cast<uint32_t*>(&r);
  }
};

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// Pairs of 32-bit values.
__device__ __forceinline__ uint64_t pair2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpair2(uint64_t x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// Reciprocal to 1 unit in the last place; of 0: infinity.
__device__ __forceinline__ float rcp(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// A place in the ring of stages, and how often the ring has come round (the phase).
template <int ST>
struct Place {
  uint32_t s = 0, phase = 0;
  __device__ __forceinline__ void operator++() {
    if (++s == ST) s = 0, phase ^= 1u;
  }
};

// Where one row's result goes: o / l and lse, or, of a part of the keys, o, m and l.
struct RowOut {
  uint8_t* out;    // the row's output, or its place in the partial results
  float* lse;      // or null
  float2* part_ml; // or null: all keys
  bool sees;       // false: o = 0, lse = -infinity
  __device__ __forceinline__ void stats(const AttnArgs& a, float m, float l) const {
    if (part_ml) *part_ml = sees ? make_float2(m, l) : make_float2(-INFINITY, -1.f);
    else if (lse) *lse = sees ? fmaf(m, a.scale, logf(l)) : -INFINITY;
  }
};

// A warp's 32 rows of 8 16-byte chunks from its buffer (row r's chunk e at r * 8 + (e ^ (r % 8))) to
// global memory: lane writes chunk lane % 8 of rows 4 i + lane / 8, to[i] + at, where on.
__device__ __forceinline__ void flush_rows(const uint4* buf, uint8_t* const (&to)[8], uint32_t on, int at) {
  const int lane = threadIdx.x & 31, e = lane & 7;
  __syncwarp();
  uint4 v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = i * 4 + lane / 8;
    v[i] = buf[r * 8 + (e ^ (r & 7))];
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (on >> (i * 4 + lane / 8) & 1u) *reinterpret_cast<uint4*>(to[i] + at) = v[i];
}

// LONG: some item has more keys than kAttLongKeys, and the waits take AttnArgs::wait_ns (which as an operand of every
// wait costs 1 to 2% of any prompt: 5340 us instead of 5250 for 32768 tokens).
template <class T, int D, bool TREE, bool LONG>
__global__ void __launch_bounds__(kAttThreads, 1)
    attend_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                  const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmKD,
                  const __grid_constant__ CUtensorMap tmVD, const AttnArgs a) {
  using L = AttSmem<D>;
  constexpr int ST = L::STAGES;
  extern __shared__ __align__(1024) uint8_t smem[];
  // (swizzled tiles need 1024-byte alignment, which the base of dynamic shared memory has
  // where a kernel has no static shared memory)
  if (smem_u32(smem) & 1023u) {
    if (threadIdx.x == 0) atomicOr(a.status, kStatusBadShape);
    return;
  }
  uint64_t* bar = reinterpret_cast<uint64_t*>(smem + L::MISC);
  uint64_t *b_full = bar, *b_empty = bar + 8, *b_qfull = bar + 16, *b_qempty = bar + 17, *b_s = bar + 18,
           *b_p = bar + 20 /* [X][half] */, *b_o = bar + 24, *b_drain = bar + 26, *b_item = bar + 27, *b_free = bar + 31,
           *b_look = bar + 35, *b_x = bar + 39;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::MISC + 400);
  volatile int* abort = reinterpret_cast<int*>(smem + L::MISC + 404);
  Published* ring = reinterpret_cast<Published*>(smem + L::ITEM);
  volatile int* flags = reinterpret_cast<int*>(smem + L::FLAG);
  float2* xch = reinterpret_cast<float2*>(smem + L::XCH);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < ST; ++s) {
      mbar_init(&b_full[s], 1);
      mbar_init(&b_empty[s], 3);  // the issuer's commit, warps 10 and 11
    }
    mbar_init(b_qfull, 1);
    mbar_init(b_qempty, 1);
    for (int x = 0; x < 2; ++x) {
      mbar_init(&b_s[x], 1);
      mbar_init(&b_p[2 * x], 4);
      mbar_init(&b_p[2 * x + 1], 4);
      mbar_init(&b_o[x], 1);
      mbar_init(&b_x[x], 8);
    }
    for (int e = 0; e < kItemRing; ++e) {
      mbar_init(&b_item[e], 1);
      mbar_init(&b_free[e], 11);  // softmax warps, issuer, warps 10 and 11
      mbar_init(&b_look[e], 2);
    }
    mbar_init(b_drain, 1);
    *abort = 0;
    fence_mbar_init();
  }
  if (warp == 9) {
    tmem_alloc(tmem_slot, kAttCols);
    tmem_relinquish();
  }
  if (warp == 8 && lane == 0) {
    prefetch_tmap(&tmQ);
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
    if (TREE) {
      prefetch_tmap(&tmKD);
      prefetch_tmap(&tmVD);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_dep_wait();    // all inputs, and the outputs' and partial results' last readers
  grid_dep_launch();  // the partial results' merge, if any, may get ready
  const int tpt = kAttRows / a.G;

  auto wait = [&](uint64_t* b, uint32_t parity, int site) { return att_wait(b, parity, abort, site, LONG ? a.wait_ns : kAttWaitNs); };
  // Waits for published item number k; false: no more, or the wait gave up.
  auto ready = [&](int k, int site) {
    const int e = k % kItemRing;
    return wait(&b_item[e], (k / kItemRing) & 1, site) && ring[e].it.y >= 0;
  };

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kAttRegsIssue));
    if (warp == 8) {
      // ---------------------------------------------------------- producer
      if (elect_one()) {
        const uint64_t pol = TREE && a.pairs == 1 ? l2_evict_first_policy() : l2_evict_normal_policy();
        const uint32_t qbytes = (uint32_t)(tpt * a.G) * (uint32_t)D * 2u;
        int g = 0, sent = 0;
        int at = 0, end = 0;
        if (TREE) {
          at = tree_from(a, blockIdx.x);
          end = tree_from(a, blockIdx.x + 1);
        } else {
          at = __ldg(a.first + blockIdx.x);
          end = __ldg(a.first + blockIdx.x + 1);
        }
        AttnItem next{};
        auto fetch = [&] {
          if (at >= end) {
            next.y = -1;
          } else if (TREE) {
            next = tree_item(a, blockIdx.x, at, end);
            at = (at / a.tiles + 1) * a.tiles;
          } else {
            next = load_item(a, at);
            ++at;
          }
        };
        fetch();
        for (int k = 0; !*abort; ++k) {
          const AttnItem it = next;
          const int e = k % kItemRing;
          if (!wait(&b_free[e], ((k / kItemRing) & 1) ^ 1, 200)) break;
          int4* p = reinterpret_cast<int4*>(ring + e);
          p[0] = make_int4(it.y, it.h, it.lb, it.t0);
          p[1] = make_int4(it.tend, it.k0, it.klen, it.off);
          p[2] = make_int4(it.j0, it.j1, it.slot, it.alt);
          p[3] = make_int4(it.eA, it.eB, it.lowA, it.lowB);
          const Steps<TREE> st(it);
          p[4] = make_int4(it.t0, st.alt ? 0 : st.skipA, st.count(0), it.lowA);
          p[5] = make_int4(st.alt ? it.t0 : it.t0 + tpt, st.alt ? st.alt & 1 : st.skipB, st.count(1), it.lowB);
          mbar_arrive(&b_item[e]);
          if (it.y < 0) break;
          fetch();
          if (st.n == 0) continue;
          if (!wait(b_qempty, (sent & 1) ^ 1, 201)) break;
          const bool two = TREE && st.alt == 2;
          mbar_expect_tx(b_qfull, st.alt == 1 ? qbytes : 2 * qbytes);
          for (int x = 0; x < (st.alt == 1 ? 1 : 2); ++x)
            for (int c = 0; c < D / 64; ++c)
              tma_load_5d(smem + L::Q + x * L::TILE + c * 16384, &tmQ, c * 64, 0, two ? (it.y + x) % a.kvh : it.h,
                          two ? 0 : it.t0 + x * tpt, two ? (it.y + x) / a.kvh : it.lb, b_qfull);
          ++sent;
#pragma unroll 1
          for (int p2 = 0; p2 < 2 * st.n; ++p2) {
            bool v;
            const int i = st.load(p2, v), j = st.tile(i), s = g % ST;
            if (!wait(&b_empty[s], ((g / ST) & 1) ^ 1, 202)) break;
            mbar_expect_tx(&b_full[s], L::TILE);
            const bool d = TREE && j == st.draft;
            const CUtensorMap* tm = d ? (v ? &tmVD : &tmKD) : v ? &tmV : &tmK;
#pragma unroll
            for (int c = 0; c < D / 64; ++c)
              tma_load_3d(smem + L::RING + s * L::TILE + c * 16384, tm, c * 64, it.y + (two ? i & 1 : 0), d ? 0 : it.k0 + j * kAttTok,
                          &b_full[s], pol);
            ++g;
          }
        }
        // every issued load must land before the CTA may exit
        for (int t = g - ST < 0 ? 0 : g - ST; t < g; ++t) mbar_wait_drain(&b_full[t % ST], (t / ST) & 1);
        if (sent) mbar_wait_drain(b_qfull, (sent - 1) & 1);
      }
      __syncwarp();
    } else if (warp == 9) {
      // ---------------------------------------------------------- MMA issuer
      if (elect_one()) {
        const uint32_t q_lo = sdesc_lo(smem_u32(smem + L::Q), 16), k_lo = sdesc_lo(smem_u32(smem + L::RING), 16),
                       v_lo = sdesc_lo(smem_u32(smem + L::RING), 16384);
        constexpr uint32_t hi = sdesc_hi(1024, 2);
        constexpr uint32_t id_s = Mma<T>::id(128, 0), id_o = Mma<T>::id(D, 1);
        Place<ST> g;
        uint32_t items = 0, np[2] = {0, 0};  // query tiles and P tiles taken, modulo 2
        bool ok = true;
        for (int k = 0; ok && ready(k, 203); ++k) {
          const Steps<TREE> st(ring[k % kItemRing].it);
          if (st.n == 0) {
            mbar_arrive(&b_free[k % kItemRing]);
            continue;
          }
          ok = wait(b_qfull, items, 204);
          if (!ok) break;
          items ^= 1u;
          auto full = [&](const Place<ST>& p) { return wait(&b_full[p.s], p.phase, 205); };
          auto s_mma = [&](int x, uint32_t qlo, uint32_t stage) {
            const uint32_t klo = k_lo + stage * (L::TILE >> 4);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
              const uint32_t off = ((uint32_t)(ks >> 2) * 16384u + (uint32_t)(ks & 3) * 32u) >> 4;
              mma_bf16_lo(tmem + x * 128, qlo + off, hi, klo + off, hi, id_s, ks > 0);
            }
            mma_commit(&b_s[x]);
          };
          auto o_mma = [&](int x, uint32_t stage, uint32_t fresh) {
            const uint32_t vlo = v_lo + stage * (L::TILE >> 4);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if (!wait(&b_p[2 * x + h], np[x], 206)) return false;
              tc_fence_after();
#pragma unroll
              for (int ks = 4 * h; ks < 4 * h + 4; ++ks)
                mma_f16_ts_lo(tmem + 256 + x * 128, tmem + x * 128 + ks * 8, vlo + ks * (2048u >> 4), hi, id_o,
                              ks > 0 ? 1u : fresh ^ 1u);
            }
            np[x] ^= 1u;
            return true;
          };
          const int n = st.n;
          if (st.alt) {
            // A: steps 0, 2, ..., B: 1, 3, ...; S of a step goes out behind O of the one two before
            const uint32_t q1 = st.alt == 2 ? q_lo + (L::TILE >> 4) : q_lo;
            for (int i = 0; i < 2 && i < n; ++i) {
              ok = ok && full(g);
              if (!ok) break;
              tc_fence_after();
              if (i == 0) s_mma(0, q_lo, g.s);
              else s_mma(1, q1, g.s);
              mma_commit(&b_empty[g.s]);
              ++g;
            }
            if (!ok) break;
            if (n <= 2) mma_commit(b_qempty);
            auto step = [&](int x, int i) {
              if (!full(g) || !o_mma(x, g.s, i < 2)) return false;
              mma_commit(&b_empty[g.s]);
              if (i >= n - 2) mma_commit(&b_o[x]);
              ++g;
              if (i + 2 < n) {
                if (!full(g)) return false;
                tc_fence_after();
                s_mma(x, x ? q1 : q_lo, g.s);
                mma_commit(&b_empty[g.s]);
                ++g;
                if (i + 3 == n) mma_commit(b_qempty);
              }
              return true;
            };
            for (int i = 0; i < n && ok; i += 2) {
              ok = step(0, i);
              if (ok && i + 1 < n) ok = step(1, i + 1);
            }
          } else {
            const uint32_t qb = q_lo + (L::TILE >> 4);
            ok = full(g);
            if (!ok) break;
            tc_fence_after();
            if (st.skipA == 0) s_mma(0, q_lo, g.s);
            if (st.skipB == 0) s_mma(1, qb, g.s);
            mma_commit(&b_empty[g.s]);
            if (n == 1) mma_commit(b_qempty);
            ++g;
            for (int i = 0; i < n; ++i) {
              const Place<ST> gv = g;
              ++g;
              const bool more = i + 1 < n;
              ok = full(gv) && (!more || full(g));
              if (!ok) break;
              if (i >= st.skipA) {
                ok = o_mma(0, gv.s, i == st.skipA);
                if (!ok) break;
                if (!more) mma_commit(&b_o[0]);
              }
              if (more && i + 1 >= st.skipA) s_mma(0, q_lo, g.s);
              if (i >= st.skipB) {
                ok = o_mma(1, gv.s, i == st.skipB);
                if (!ok) break;
                if (!more) mma_commit(&b_o[1]);
              }
              if (more && i + 1 >= st.skipB) s_mma(1, qb, g.s);
              mma_commit(&b_empty[gv.s]);
              if (more) {
                mma_commit(&b_empty[g.s]);
                if (i + 2 == n) mma_commit(b_qempty);
                ++g;
              }
            }
          }
          if (ok) mbar_arrive(&b_free[k % kItemRing]);
        }
        // all issued MMAs complete before TMEM is released
        mma_commit(b_drain);
        mbar_wait_drain(b_drain, 0);
      }
      __syncwarp();
    } else {
      // ---------------------------------------------------------- values of partly masked tiles
      // (These warps wait for and release every load, so that a stage's phase cannot pass them by,
      // nor they it: a wait for a parity is sound only one phase away.)
      Place<ST> g;
      for (int k = 0; __all_sync(0xffffffffu, ready(k, 207)); ++k) {
        const Steps<TREE> st(ring[k % kItemRing].it);
        int found = 0;
        bool ok = true;
#pragma unroll 1
        for (int p2 = 0; p2 < 2 * st.n; ++p2) {
          ok = __all_sync(0xffffffffu, wait(&b_full[g.s], g.phase, 208));
          if (!ok) break;
          bool v;
          const int i = st.load(p2, v), mk = v ? st.masked(i) : 0;
          if (mk) {
            // the keys that some row must not see
            const int j = st.tile(i);
            int lo = max(0, min(mk & 1 ? st.lowA : kSeesAll, mk & 2 ? st.lowB : kSeesAll) - j * kAttTok), hi = kAttTok;
            if (TREE && j == st.draft) lo = 0, hi = a.nodes;
            uint32_t acc[4] = {};
#pragma unroll 1
            for (int c = 0; c < D / 64; ++c) {
              const uint4* vt = reinterpret_cast<const uint4*>(smem + L::RING + g.s * L::TILE + c * 16384);
#pragma unroll 4
              for (int e = lo * 8 + (warp - 10) * 32 + lane; e < hi * 8; e += 64) {
                const uint4 w = vt[e];
                acc[0] = Mma<T>::look(w.x, acc[0]);
                acc[1] = Mma<T>::look(w.y, acc[1]);
                acc[2] = Mma<T>::look(w.z, acc[2]);
                acc[3] = Mma<T>::look(w.w, acc[3]);
              }
            }
            if (__any_sync(0xffffffffu, ((acc[0] | acc[1] | acc[2] | acc[3]) & 0x7fff7fffu) != 0u)) found |= mk;
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&b_empty[g.s]);
          ++g;
        }
        if (!ok) break;
        if (lane == 0) {
          flags[2 * (k % kItemRing) + warp - 10] = found;
          mbar_arrive(&b_look[k % kItemRing]);
          mbar_arrive(&b_free[k % kItemRing]);
        }
        __syncwarp();
      }
    }
  } else {
    // ------------------------------------------------------------ softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kAttRegsRow));
    const int X = warp >> 2;
    const int row = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lanes + X * 128, t_o = tmem + lanes + 256 + X * 128;
    uint4* const buf = reinterpret_cast<uint4*>(smem + L::OUT + warp * 4096);
    const float c = a.c, grow = Mma<T>::kAbove / c;
    // (finite, so that a scale near the smallest there is leaves m finite)
    const float room = Mma<T>::kRoom > 0.f ? fminf(Mma<T>::kRoom / c, 1e38f) : 0.f;
    const int row_t = row / a.G, row_g = row % a.G;
    uint32_t ns = 0, no = 0, oo = 0, nx = 0;  // S tiles, results (oo: the other's) and exchanges so far, modulo 2
    for (int k = 0; __all_sync(0xffffffffu, ready(k, 209)); ++k) {
      const AttnItem& it = ring[k % kItemRing].it;  // (not kept in registers through the steps)
      const int4 of = ring[k % kItemRing].of[X];
      const int alt = it.alt == 1, steps = of.z, low = of.w, klen = it.klen;
      const bool two = TREE && it.alt == 2;
      const int y = two ? it.y + X : it.y, lb = two ? y / a.kvh : it.lb;
      const int draft = TREE ? (klen + kAttTok - 1) / kAttTok : -1;
      const int t = of.x + row_t;
      const bool valid = row < tpt * a.G && t < it.tend;
      const bool busy = __any_sync(0xffffffffu, valid);  // warps whose rows hold nothing skip the arithmetic
      const int lim = valid ? att_limit(it, t) : 0;
      const bool drafts = TREE && it.j0 <= draft && draft < it.j1;
      uint32_t nodes[4] = {};
      bool sees = TREE || lim > 0;
      if (drafts && valid) sees = tree_mask(a.parents + (long long)(lb % a.batch) * a.nodes, t, nodes);

      float m = -INFINITY, l = 0.f;
      int j = TREE ? it.j0 + of.y : it.j1 - 1 - of.y;
      const int jstep = TREE ? alt + 1 : -1 - alt;
#pragma unroll 1
      for (int i = 0; i < steps; ++i, j += jstep) {
        wait(&b_s[X], ns, 210 + X);
        ns ^= 1u;
        if (busy) {
          tc_fence_after();
          float s[4][32];
#pragma unroll
          for (int q = 0; q < 4; ++q) tmem_ld32(t_s + q * 32, s[q]);
          tmem_ld_wait();
          bool live = true;  // whether any row of the warp sees any of the second 64 keys
          if ((TREE && j == draft) || (j + 1) * kAttTok > low) {
            if (TREE && j == draft) {
              live = __any_sync(0xffffffffu, (nodes[2] | nodes[3]) != 0u);
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const uint32_t w = nodes[q];
                if (q < 2 || live) {
#pragma unroll
                  for (int e = 0; e < 32; ++e) s[q][e] = (w >> e & 1u) ? s[q][e] : -INFINITY;
                }
              }
            } else {
              // (quarters that every row of the warp sees stay as they are)
              const int cnt = lim - j * kAttTok;
              live = __any_sync(0xffffffffu, cnt > 64);
#pragma unroll
              for (int q = 0; q < 4; ++q)
                if ((q < 2 || live) && __any_sync(0xffffffffu, cnt < q * 32 + 32)) {
#pragma unroll
                  for (int e = 0; e < 32; ++e) s[q][e] = q * 32 + e < cnt ? s[q][e] : -INFINITY;
                }
            }
          }
          auto top = [&](int q) {
            float x = fmaxf(s[q][0], s[q][1]), y = fmaxf(s[q][2], s[q][3]);
#pragma unroll
            for (int e = 4; e < 32; e += 4) {
              x = max3(x, s[q][e], s[q][e + 1]);
              y = max3(y, s[q][e + 2], s[q][e + 3]);
            }
            return fmaxf(x, y);
          };
          float mx = fmaxf(top(0), top(1));
          if (live) mx = max3(mx, top(2), top(3));
          const bool up = mx > m + grow;
          if (i == 0) {
            m = mx - room;
          } else if (__any_sync(0xffffffffu, up)) {
            const float f = up ? ex2((m - (mx - room)) * c) : 1.f;
            if (up) {
              m = mx - room;
              l *= f;
            }
#pragma unroll 1
            for (int q = 0; q < D / 32; ++q) {
              float o[32];
              tmem_ld32(t_o + q * 32, o);
              tmem_ld_wait();
              uint32_t r[32];
#pragma unroll
              for (int e = 0; e < 32; ++e) r[e] = __float_as_uint(o[e] * f);
              tmem_st32(t_o + q * 32, r);
            }
          }
          const float mc = m == -INFINITY ? 0.f : m * c;
          const uint64_t c2 = pair2(c, c), mc2 = pair2(-mc, -mc);
          uint64_t sum[2] = {0, 0};  // pairs of 0.f
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (h == 0 || live) {
#pragma unroll
              for (int q = 2 * h; q < 2 * h + 2; ++q) {
                uint32_t r[16];
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                  const float2 x = unpair2(fma2(pair2(s[q][e], s[q][e + 1]), c2, mc2));
                  const float p0 = ex2(x.x), p1 = ex2(x.y);
                  sum[e / 2 & 1] = add2(sum[e / 2 & 1], pair2(p0, p1));
                  r[e / 2] = T::pack(p0, p1);
                }
                tmem_st16(t_s + q * 16, r);
              }
            } else {
              const uint32_t zero[32] = {};
              tmem_st32(t_s + 32, zero);
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&b_p[2 * X + h]);
          }
          const float2 z = unpair2(add2(sum[0], sum[1]));
          l += z.x + z.y;
        } else if (lane == 0) {
          mbar_arrive(&b_p[2 * X]);
          mbar_arrive(&b_p[2 * X + 1]);
        }
      }

      // ---------------------------------------------------------- the item's result
      // (all that does not need O goes before the wait for it)
      wait(&b_look[k % kItemRing], (k / kItemRing) & 1, 214);
      const int found = flags[2 * (k % kItemRing)] | flags[2 * (k % kItemRing) + 1];
      const bool bad = alt ? found != 0 : (found >> X & 1) != 0;
      // of two results over the same rows, each warpgroup joins half the dims
      float f = 1.f, fy = 0.f;
      int other = 0;
      if (alt) {
        xch[X * 128 + row] = make_float2(m, l);
        __syncwarp();
        if (lane == 0) mbar_arrive(&b_x[0]);
        wait(&b_x[0], nx, 215);
        const float2 y = xch[(X ^ 1) * 128 + row];
        const float mm = fmaxf(m, y.x);
        other = ring[k % kItemRing].of[X ^ 1].z;
        f = m == -INFINITY ? 0.f : ex2((m - mm) * c);
        fy = y.x == -INFINITY ? 0.f : ex2((y.x - mm) * c);
        l = l * f + y.y * fy;
        m = mm;
      }
      const int slot = it.slot;
      auto place = [&](int tok, int hd, int r) {
        RowOut x;
        x.lse = a.lse ? a.lse + (long long)tok * a.kvh * a.G + hd : nullptr;
        if (slot >= 0) {
          x.out = reinterpret_cast<uint8_t*>(a.part + ((long long)slot * a.prows + r) * D);
          x.part_ml = a.part_ml + ((long long)slot * a.prows + r);
        } else {
          x.out = reinterpret_cast<uint8_t*>(a.out + lb * a.o_lb + (long long)tok * a.o_t + hd * a.o_h);
          x.part_ml = nullptr;
        }
        return x;
      };
      // (debug builds: whether the row's place lies within the output or the partial results)
      auto fits = [&](int tok, int hd, int r) {
        return slot >= 0 ? DC_INB(a, (long long)slot * a.prows + r, a.part_rows, 320)
                         : DC_INB(a, lb * a.o_lb + (long long)tok * a.o_t + hd * a.o_h + D - 1, a.out_len, 321);
      };
      const int head = (two ? y % a.kvh : it.h) * a.G + row_g, prow = (alt ? 0 : X * 128) + row;
      RowOut ro = place(t, head, prow);
      ro.sees = sees;
      const bool writes = valid && fits(t, head, prow);
      // where this lane's share of the rows goes
      uint8_t* to[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        to[i] = reinterpret_cast<uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(ro.out),
                                                       i * 4 + lane / 8)) + (lane & 7) * 16;
      const uint32_t on = __ballot_sync(0xffffffffu, writes);
      if (!bad && writes && (!alt || X == 0)) ro.stats(a, m, l);
      {
        const float inv = slot >= 0 ? 1.f : sees ? rcp(l) : 0.f;
        f *= inv;
        fy *= inv;
      }
      if (steps) {
        wait(&b_o[X], no, 212 + X);
        no ^= 1u;
      }
      // (the other's products: it has passed its earlier results, as its part of the exchange says)
      if (other) wait(&b_o[X ^ 1], oo, 213);
      oo ^= ring[k % kItemRing].of[X ^ 1].z ? 1u : 0u;
      tc_fence_after();
      if (bad) {
        // a value that is not finite in a tile that is masked in part: this tile's rows anew
        // (of two results over the same rows, by the first warpgroup)
        if (!(alt && X == 1)) {
          for (int rr = 0; rr < 32; ++rr) {
            if (!__shfl_sync(0xffffffffu, (int)writes, rr)) continue;
            const int tok = __shfl_sync(0xffffffffu, t, rr), hd = __shfl_sync(0xffffffffu, head, rr);
            const int see = __shfl_sync(0xffffffffu, lim, rr);
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = __shfl_sync(0xffffffffu, nodes[q], rr);
            RowOut x = place(tok, hd, __shfl_sync(0xffffffffu, prow, rr));
            x.sees = __shfl_sync(0xffffffffu, (int)sees, rr);
            const int from = it.j0 * kAttTok, to = x.sees ? min(see, it.j1 * kAttTok) : from;
            float o[D / 32], mm, ll;
            const long long dr = (long long)y * a.nodes * D;
            attend_row<T, D>(a, a.q + lb * a.q_lb + (long long)tok * a.q_t + hd * a.q_h,
                             a.k + it.k0 * a.k_t + y * a.k_y, a.v + it.k0 * a.v_t + y * a.v_y, a.kd + dr, a.vd + dr,
                             from, to, drafts && x.sees ? w : nullptr, mm, ll, o);
            if (lane == 0) x.stats(a, mm, ll);
            const float inv = x.sees ? 1.f / ll : 0.f;
#pragma unroll
            for (int e = 0; e < D / 64; ++e) {
              if (x.part_ml) reinterpret_cast<float2*>(x.out)[lane * (D / 64) + e] = make_float2(o[2 * e], o[2 * e + 1]);
              else reinterpret_cast<uint32_t*>(x.out)[lane * (D / 64) + e] = T::pack(o[2 * e] * inv, o[2 * e + 1] * inv);
            }
          }
        }
      } else if (busy) {
        const int d0 = alt ? X * (D / 2) : 0, d1 = alt ? d0 + D / 2 : D;
        // (an unused node's O holds what its query made of the cached tokens: NaN, of a query that is)
        const bool blank = TREE && __any_sync(0xffffffffu, !sees);
        // 32 dims of this row's result
        auto dims = [&](int d, float (&o)[32]) {
          if (steps) {
            tmem_ld32(t_o + d, o);
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0.f;
          }
          if (other) {
            float z[32];
            tmem_ld32(tmem + lanes + 256 + (X ^ 1) * 128 + d, z);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = fmaf(z[e], fy, o[e] * f);
          } else {
            tmem_ld_wait();
            const uint64_t f2 = pair2(f, f);
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              const float2 x = unpair2(mul2(pair2(o[e], o[e + 1]), f2));
              o[e] = x.x;
              o[e + 1] = x.y;
            }
          }
          if (blank) {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = sees ? o[e] : 0.f;
          }
        };
        // 128 bytes of each row at a time: 64 dims, or 32 of a partial result (or 32 that are all there
        // are: each row's second half is then written by no lane)
        const uint32_t both = slot < 0 && d1 - d0 < 64 && (lane & 4) ? 0u : on;
#pragma unroll 1
        for (int d = d0; d < d1; d += 32) {
          float o[32];
          dims(d, o);
          if (slot >= 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              buf[lane * 8 + (e ^ (lane & 7))] = make_uint4(__float_as_uint(o[4 * e]), __float_as_uint(o[4 * e + 1]),
                                                            __float_as_uint(o[4 * e + 2]), __float_as_uint(o[4 * e + 3]));
          } else {
            const int h = (d - d0) >> 3 & 4;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              buf[lane * 8 + ((h + e) ^ (lane & 7))] =
                  make_uint4(T::pack(o[8 * e], o[8 * e + 1]), T::pack(o[8 * e + 2], o[8 * e + 3]),
                             T::pack(o[8 * e + 4], o[8 * e + 5]), T::pack(o[8 * e + 6], o[8 * e + 7]));
            if (!h && d + 32 < d1) continue;
          }
          flush_rows(buf, to, both, slot >= 0 ? d * 4 : (d & ~63) * 2 + (d1 - d0 < 64 ? d0 % 64 * 2 : 0));
        }
      }
      tc_fence_before();
      __syncwarp();
      if (alt) {
        // the other warpgroup has read this one's O and statistics before they are written again
        if (lane == 0) mbar_arrive(&b_x[1]);
        wait(&b_x[1], nx, 216);
        nx ^= 1u;
      }
      if (lane == 0) mbar_arrive(&b_free[k % kItemRing]);
    }
  }
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, kAttCols);
  }
  if (threadIdx.x == 0 && *abort) {
    record_timeout(a.dbg, (unsigned)*abort, 0u, 0u);
    atomicOr(a.status, kStatusTimeout);
  }
}

// Joins the partial results of the parts of one item, in order: block x an item, y 32 of its rows, a
// warp four of them at once: lane 8 i + s takes m and l of row i's part s (8 parts at a time), then
// the parts' O come with all loads in flight. Prompts:
// `merges` lists each item's first part and their number; trees: merge i belongs to the boundary
// between CTAs i and i + 1, if that is the first one within its item.
template <class T, int D, bool TREE>
__global__ void __launch_bounds__(256) merge_kernel(const AttnArgs a) {
  constexpr int E = D / 32, W = 4;
  const int lane = threadIdx.x & 31, tpt = kAttRows / a.G, gi = blockIdx.x;
  AttnItem it;
  int parts, slot;  // the first part's; the others': the next ones (prompts), or every second from 2 (gi + 1)
  if constexpr (TREE) {
    const int cut = tree_from(a, gi + 1), i0 = cut / a.tiles * a.tiles;
    if (cut == i0 || tree_from(a, gi) > i0) return;
    it = tree_item(a, gi, i0, i0 + a.tiles);
    parts = tree_cta(a, i0 + a.tiles - 1) - gi + 1;
    slot = 2 * gi + 1;
  } else {
    const int2 mg = __ldg(a.merges + gi);
    it = load_item(a, mg.x);
    parts = mg.y;
    slot = it.slot;
  }
  const int r0 = blockIdx.y * 32 + threadIdx.x / 32 * W;
  bool valid[W];
  int tok[W], head[W];
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const int r = r0 + i, rr = r % 128;  // rows of tile A, then of tile B
    tok[i] = it.t0 + r / 128 * tpt + rr / a.G;
    head[i] = it.h * a.G + rr % a.G;
    valid[i] = r < a.prows && rr < tpt * a.G && tok[i] < it.tend &&
               DC_INB(a, it.lb * a.o_lb + (long long)tok[i] * a.o_t + head[i] * a.o_h + D - 1, a.out_len, 322) &&
               DC_INB(a, (long long)slot * a.prows + r, a.part_rows, 323);
  }
  grid_dep_wait();
  auto place = [&](int s) { return (long long)(TREE && s ? 2 * (gi + s) : slot + s) * a.prows + r0; };
  // this lane's row and part
  const int li = lane / 8, ls = lane % 8;
  bool lv = false;
#pragma unroll
  for (int i = 0; i < W; ++i) lv = lv || (i == li && valid[i]);
  auto load = [&](int s) { return lv && s < parts ? a.part_ml[place(s) + li] : make_float2(-INFINITY, 0.f); };
  const float2 v0 = load(ls);  // (8 parts or fewer: read once)
  float mm = v0.x;
  bool unseen = v0.y < 0.f;
  for (int s = 8; s < parts; s += 8) {
    const float2 v = load(s + ls);
    mm = fmaxf(mm, v.x);
    unseen = unseen || v.y < 0.f;
  }
#pragma unroll
  for (int x = 1; x < 8; x *= 2) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, x));
  const uint32_t blind = __ballot_sync(0xffffffffu, unseen);
  float ll = 0.f, o[W][E] = {};
  for (int s0 = 0; s0 < parts; s0 += 8) {
    const float2 v = s0 ? load(s0 + ls) : v0;
    // (a part of which the row sees nothing has no say, whatever it holds: factor -1)
    const bool none = v.x == -INFINITY && !(v.y != v.y);
    const float f = none ? -1.f : v.x == -INFINITY ? 1.f : ex2((v.x - mm) * a.c);
    if (!none) ll = fmaf(f, v.y, ll);
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      if (s0 + s >= parts) break;
      const float* part = a.part + place(s0 + s) * D + lane * E;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float fi = __shfl_sync(0xffffffffu, f, i * 8 + s);
        if (!valid[i]) continue;
        float x[E];
        if constexpr (E == 4) {
          const float4 y = *reinterpret_cast<const float4*>(part + (long long)i * D);
          x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w;
        } else {
          const float2 y = *reinterpret_cast<const float2*>(part + (long long)i * D);
          x[0] = y.x; x[1] = y.y;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) o[i][e] = fi == -1.f ? o[i][e] : fmaf(fi, x[e], o[i][e]);
      }
    }
  }
#pragma unroll
  for (int x = 1; x < 8; x *= 2) ll += __shfl_xor_sync(0xffffffffu, ll, x);
  float m[W], l[W];
  bool sees[W];
#pragma unroll
  for (int i = 0; i < W; ++i) {
    m[i] = __shfl_sync(0xffffffffu, mm, i * 8);
    l[i] = __shfl_sync(0xffffffffu, ll, i * 8);
    sees[i] = (blind >> (i * 8) & 0xffu) == 0u;
  }
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if (!valid[i]) continue;
    const float inv = sees[i] ? rcp(l[i]) : 0.f;
    uint32_t* to = reinterpret_cast<uint32_t*>(a.out + it.lb * a.o_lb + (long long)tok[i] * a.o_t + head[i] * a.o_h) + lane * (E / 2);
    uint32_t w[E / 2];
#pragma unroll
    for (int e = 0; e < E; e += 2) w[e / 2] = sees[i] ? T::pack(o[i][e] * inv, o[i][e + 1] * inv) : 0u;
    if constexpr (E == 4) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
    else *to = w[0];
    if (a.lse && lane == 0) a.lse[(long long)tok[i] * a.kvh * a.G + head[i]] = sees[i] ? fmaf(m[i], a.scale, logf(l[i])) : -INFINITY;
  }
}

// Tensor maps of one call (tmKD, tmVD: trees).
struct AttMaps {
  CUtensorMap q, k, v, kd, vd;
};

template <class T, int D, bool TREE, bool LONG>
cudaError_t launch_attend_kernel(const AttMaps& m, const AttnArgs& a, int grid, cudaStream_t s) {
  static SmemLimit limit;
  if (cudaError_t e = limit.raise(attend_kernel<T, D, TREE, LONG>, AttSmem<D>::BYTES); e != cudaSuccess) return e;
  // (its set-up may run under the end of the kernel before it)
  return launch_pdl(attend_kernel<T, D, TREE, LONG>, dim3(grid), dim3(kAttThreads), AttSmem<D>::BYTES, s, m.q, m.k, m.v, m.kd,
                    m.vd, a);
}

template <class T, int D, bool TREE>
cudaError_t launch_attend(const AttMaps& m, const AttnArgs& a, int grid, cudaStream_t s) {
  const bool is_long = a.wait_ns > att_wait_ns(kAttLongKeys);
  if (cudaError_t e = is_long ? launch_attend_kernel<T, D, TREE, true>(m, a, grid, s)
                              : launch_attend_kernel<T, D, TREE, false>(m, a, grid, s);
      e != cudaSuccess)
    return e;
  if (a.n_merges == 0) return cudaSuccess;
  return launch_pdl(merge_kernel<T, D, TREE>, dim3((unsigned)a.n_merges, (unsigned)((a.prows + 31) / 32)), dim3(256), 0, s, a);
}

}  // namespace
}  // namespace dc
