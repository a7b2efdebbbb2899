// dc_attend_kernel.cuh -- the attention kernel of prompts and drafted trees on the
// tensor cores; instantiated in dc_prompt.cu and dc_tree.cu.
//
// One persistent CTA per SM takes work items in turn: two tiles of 128 query rows (A and
// B) of one KV head over a run of key tiles of 128 tokens. Warp roles (384 threads):
//   warps 0-3, 4-7  softmax warpgroups of tiles A and B, one query row (TMEM lane) a thread;
//   warp 8          producer: query tiles, then K and V tiles in the order in which the
//                   products take them, by TMA through one ring of stages;
//   warp 9          MMA issuer (one lane):
//                     S_X  = Q_X K^T     [128 rows x 128 keys]   from shared memory
//                     O_X += P_X V       [128 rows x D]          P_X from TMEM
//   warps 10, 11    idle (the third warpgroup gives up registers as a whole)
// TMEM columns: S_A [0, 128), S_B [128, 256), O_A [256, 256 + D), O_B [384, 384 + D). A
// warpgroup reads its S (the whole row in registers), writes the weights P over its
// first 64 columns in the inputs' type, and the second product reads them there. The
// issuer sends S_X of the next key tile right behind O_X of this one, so that one
// warpgroup's softmax runs under the other's products.
//
// Running softmax: m is a row's reference, not always its maximum: it follows the maximum
// only where that is more than 2^8 above it in weights, so that O is seldom rescaled (P
// stays below 2^8, which loses nothing in floating point; l and O are in 32 bits). The
// completion of S_X also says that O_X is at rest, since the products of one issuer complete
// in order: the warpgroup rescales O itself, with no further barrier.
//
// Items of one tile of queries (single tokens, small trees, short sequences) give their key
// tiles to A and B in turn, both on the same queries, and join the two results at the end:
// the pipeline is the same.
//
// A masked key has weight 0, but 0 times a value that is not finite is NaN: the values of key
// tiles that are masked in part are looked over in shared memory, and a tile of rows that
// meets such a value is recomputed by attend_row, which reads only what a row sees.
//
// Barriers: every wait is bounded. A wait that gives up sets *abort; the softmax
// warps then go on without waiting (their loops and named barriers match all the same), the
// producer and the issuer stop, wait for what they have in flight, and the status word
// says so.
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

template <int D>
struct AttSmem {
  static constexpr int TILE = 128 * D * 2;
  static constexpr int STAGES = D == 128 ? 5 : 8;
  static constexpr int Q = 0;  // two query tiles
  static constexpr int RING = 2 * TILE;
  static constexpr int MISC = RING + STAGES * TILE;
  static constexpr int XCH = MISC + 512;  // float2 [2][128]: m, l of both tiles
  static constexpr int BYTES = XCH + 2048;
  static_assert(BYTES <= 232448, "more shared memory than a CTA may have");
};

__device__ __forceinline__ AttnItem load_item(const AttnArgs& a, int i) {
  const int4* p = reinterpret_cast<const int4*>(a.items + i);
  const int4 x = __ldg(p), y = __ldg(p + 1), z = __ldg(p + 2);
  return AttnItem{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
}

// Work item i of a tree call: row, pair of query tiles, and share of its key tiles (the
// cached tokens', then the drafted ones').
__device__ __forceinline__ AttnItem tree_item(const AttnArgs& a, int i) {
  const int tpt = kAttRows / a.G, sp = i % a.nsplit, rest = i / a.nsplit;
  AttnItem it;
  it.y = rest / a.pairs;
  it.lb = it.y / a.kvh;
  it.h = it.y % a.kvh;
  it.t0 = rest % a.pairs * 2 * tpt;
  it.tend = a.nodes;
  it.k0 = 0;
  it.klen = a.rowlen ? __ldg(a.rowlen + it.y) : a.n;
  it.off = kSeesAll;
  const int tiles = (it.klen + kAttTok - 1) / kAttTok + 1;
  it.j0 = (int)((long long)tiles * sp / a.nsplit);
  it.j1 = (int)((long long)tiles * (sp + 1) / a.nsplit);
  it.slot = a.nsplit > 1 ? i : -1;
  it.alt = it.tend - it.t0 <= tpt;
  return it;
}

// An item's steps: key tile of step i, and which of A (1) and B (2) take it.
template <bool TREE>
struct Steps {
  int n, j0, j1, eA, eB, alt, look;
  __device__ __forceinline__ Steps(const AttnArgs& a, const AttnItem& it) {
    j0 = it.j0;
    j1 = it.j1;
    n = j1 - j0;
    alt = it.alt;
    look = alt ? 2 : 1;
    eA = eB = j1;
    if (!TREE && !alt) {
      const int tpt = kAttRows / a.G;
      eA = (att_limit(it, it.t0 + tpt - 1) + kAttTok - 1) / kAttTok;
      eB = (att_limit(it, min(it.tend, it.t0 + 2 * tpt) - 1) + kAttTok - 1) / kAttTok;
    }
  }
  // the tiles that may be masked come first in prompts, last in trees
  __device__ __forceinline__ int tile(int i) const { return TREE ? j0 + i : j1 - 1 - i; }
  __device__ __forceinline__ int who(int i) const {
    if (i >= n) return 0;
    if (alt) return 1 << (i & 1);
    if (TREE) return 3;
    const int j = tile(i);
    return (j < eA ? 1 : 0) | (j < eB ? 2 : 0);
  }
  // steps of A (x = 0) or B
  __device__ __forceinline__ int count(int x) const {
    return alt ? (n + 1 - x) / 2 : max(0, min(x ? eB : eA, j1) - j0);
  }
  // where V of step i comes in the item's loads: K of the first `look` steps, then V of
  // each step and K of the step `look` later
  __device__ __forceinline__ int v_at(int i) const { return i + min(n, look + i); }
};

__device__ __forceinline__ uint32_t below(int count, int word) {
  const int c = count - 32 * word;
  return c >= 32 ? 0xffffffffu : c <= 0 ? 0u : (1u << c) - 1u;
}

template <class T>
struct Mma;
template <>
struct Mma<TypeBf16> {
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
  static constexpr uint32_t id(int N, int b_mn) { return idesc_f16(128, N, 0, b_mn); }
  static __device__ __forceinline__ uint32_t look(uint32_t x, uint32_t acc) {
    __half2 r = __hfma2(*reinterpret_cast<__half2*>(&x), __float2half2_rn(0.f), *reinterpret_cast<__half2*>(&acc));
    return *reinterpret_cast<uint32_t*>(&r);
  }
};

// One row's result: o / l and lse, or, of a part of the keys, o, m and l.
template <class T, int D>
struct RowOut {
  uint32_t* out;   // the row's output, as 32-bit words
  float* lse;      // or null
  float* part;     // the row's place in the partial results, or null
  float2* part_ml;
  bool sees;       // false: o = 0, lse = -infinity
  __device__ __forceinline__ void stats(const AttnArgs& a, float m, float l) const {
    if (part) *part_ml = sees ? make_float2(m, l) : make_float2(-INFINITY, -1.f);
    else if (lse) *lse = sees ? fmaf(m, a.scale, logf(l)) : -INFINITY;
  }
};

template <class T, int D, bool TREE>
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
  uint64_t *b_full = bar, *b_empty = bar + ST, *b_qfull = bar + 2 * ST, *b_qempty = b_qfull + 1, *b_s = b_qfull + 2,
           *b_p = b_qfull + 4, *b_o = b_qfull + 6, *b_drain = b_qfull + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::MISC + 400);
  volatile int* abort = reinterpret_cast<int*>(smem + L::MISC + 404);
  float2* xch = reinterpret_cast<float2*>(smem + L::XCH);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < ST; ++s) {
      mbar_init(&b_full[s], 1);
      mbar_init(&b_empty[s], 1);
    }
    mbar_init(b_qfull, 1);
    mbar_init(b_qempty, 1);
    for (int x = 0; x < 2; ++x) {
      mbar_init(&b_s[x], 1);
      mbar_init(&b_p[x], 4);
      mbar_init(&b_o[x], 1);
    }
    mbar_init(b_drain, 1);
    *abort = 0;
    fence_mbar_init();
  }
  if (warp == 9) {
    tmem_alloc(tmem_slot, kAttCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  int i0, i1, istep;
  if (TREE) {
    i0 = blockIdx.x;
    i1 = a.n_items;
    istep = gridDim.x;
  } else {
    i0 = __ldg(a.first + blockIdx.x);
    i1 = __ldg(a.first + blockIdx.x + 1);
    istep = 1;
  }
  grid_dep_launch();  // the partial results' merge, if any, may get ready
  auto item = [&](int i) { return TREE ? tree_item(a, i) : load_item(a, i); };
  const int tpt = kAttRows / a.G;

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kAttRegsIssue));
    if (warp == 8) {
    // ------------------------------------------------------------ producer
    if (elect_one()) {
      const uint64_t pol = TREE ? l2_evict_first_policy() : l2_evict_normal_policy();
      const uint32_t qbytes = (uint32_t)(tpt * a.G) * (uint32_t)D * 2u;
      int g = 0, items = 0, q_sent = 0;
      for (int ii = i0; ii < i1 && !*abort; ii += istep) {
        const AttnItem it = item(ii);
        const Steps<TREE> st(a, it);
        if (st.n == 0) continue;
        if (!mbar_wait(b_qempty, (items & 1) ^ 1, abort, a.dbg, 201u, (unsigned)ii)) break;
        mbar_expect_tx(b_qfull, st.alt ? qbytes : 2 * qbytes);
        for (int x = 0; x < (st.alt ? 1 : 2); ++x)
          for (int c = 0; c < D / 64; ++c)
            tma_load_5d(smem + L::Q + x * L::TILE + c * 16384, &tmQ, c * 64, 0, it.h, it.t0 + x * tpt, it.lb, b_qfull);
        q_sent = ++items;
        const int draft = TREE ? (it.klen + kAttTok - 1) / kAttTok : -1;
        auto load = [&](int j, bool v) {
          const int s = g % ST;
          if (!mbar_wait(&b_empty[s], ((g / ST) & 1) ^ 1, abort, a.dbg, 202u, (unsigned)g)) return;
          mbar_expect_tx(&b_full[s], L::TILE);
          const bool d = TREE && j == draft;
          const CUtensorMap* tm = d ? (v ? &tmVD : &tmKD) : v ? &tmV : &tmK;
          for (int c = 0; c < D / 64; ++c)
            tma_load_3d(smem + L::RING + s * L::TILE + c * 16384, tm, c * 64, it.y, d ? 0 : it.k0 + j * kAttTok,
                        &b_full[s], pol);
          ++g;
        };
        for (int i = 0; i < st.look && i < st.n; ++i) load(st.tile(i), false);
        for (int i = 0; i < st.n && !*abort; ++i) {
          load(st.tile(i), true);
          if (i + st.look < st.n) load(st.tile(i + st.look), false);
        }
      }
      // every issued load must land before the CTA may exit
      for (int t = g - ST < 0 ? 0 : g - ST; t < g; ++t) mbar_wait_drain(&b_full[t % ST], (t / ST) & 1);
      if (q_sent) mbar_wait_drain(b_qfull, (q_sent - 1) & 1);
    }
    __syncwarp();
  } else if (warp == 9) {
    // ------------------------------------------------------------ MMA issuer
    if (elect_one()) {
      const uint32_t q_lo = sdesc_lo(smem_u32(smem + L::Q), 16), k_lo = sdesc_lo(smem_u32(smem + L::RING), 16),
                     v_lo = sdesc_lo(smem_u32(smem + L::RING), 16384);
      constexpr uint32_t hi = sdesc_hi(1024, 2);
      constexpr uint32_t id_s = Mma<T>::id(128, 0), id_o = Mma<T>::id(D, 1);
      int g = 0, items = 0;
      unsigned np0 = 0, np1 = 0;  // P tiles taken of A and B
      for (int ii = i0; ii < i1 && !*abort; ii += istep) {
        const AttnItem it = item(ii);
        const Steps<TREE> st(a, it);
        if (st.n == 0) continue;
        if (!mbar_wait(b_qfull, items & 1, abort, a.dbg, 203u, (unsigned)ii)) break;
        ++items;
        int gk = g;  // this item's next load among all loads
        auto full = [&](int at) { return mbar_wait(&b_full[at % ST], (at / ST) & 1, abort, a.dbg, 204u, (unsigned)at); };
        auto s_mma = [&](int x, int at) {
          const uint32_t klo = k_lo + (uint32_t)(at % ST) * (L::TILE >> 4);
          const uint32_t qlo = q_lo + (st.alt ? 0u : (uint32_t)x * (L::TILE >> 4));
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint32_t off = ((uint32_t)(ks >> 2) * 16384u + (uint32_t)(ks & 3) * 32u) >> 4;
            mma_bf16_lo(tmem + x * 128, qlo + off, hi, klo + off, hi, id_s, ks > 0);
          }
          mma_commit(&b_s[x]);
        };
        bool ok = true;
        for (int i = 0; i < st.look && i < st.n && ok; ++i) {
          ok = full(gk);
          if (!ok) break;
          tc_fence_after();
          const int w = st.who(i);
          if (w & 1) s_mma(0, gk);
          if (w & 2) s_mma(1, gk);
          mma_commit(&b_empty[gk % ST]);
          ++gk;
        }
        if (st.look >= st.n) mma_commit(b_qempty);
        int left0 = st.count(0), left1 = st.count(1);  // steps to come
        bool fresh0 = true, fresh1 = true;
        for (int i = 0; i < st.n && ok; ++i) {
          const int w = st.who(i), w2 = st.who(i + st.look), vat = gk, kat = gk + 1;
          ok = full(vat);
          if (!ok) break;
          bool have_k = false;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (w >> x & 1) {
              unsigned& np = x ? np1 : np0;
              ok = mbar_wait(&b_p[x], np & 1, abort, a.dbg, 205u, (unsigned)ii);
              if (!ok) break;
              ++np;
              tc_fence_after();
              bool& fresh = x ? fresh1 : fresh0;
              const uint32_t vlo = v_lo + (uint32_t)(vat % ST) * (L::TILE >> 4);
#pragma unroll
              for (int ks = 0; ks < kAttTok / 16; ++ks)
                mma_f16_ts_lo(tmem + 256 + x * 128, tmem + x * 128 + ks * 8, vlo + ks * (2048u >> 4), hi, id_o,
                              (!fresh || ks > 0) ? 1u : 0u);
              fresh = false;
              if (--(x ? left1 : left0) == 0) mma_commit(&b_o[x]);
            }
            if (w2 >> x & 1) {
              if (!have_k) {
                ok = full(kat);
                if (!ok) break;
                have_k = true;
              }
              tc_fence_after();
              s_mma(x, kat);
            }
          }
          if (!ok) break;
          mma_commit(&b_empty[vat % ST]);
          ++gk;
          if (i + st.look < st.n) {
            mma_commit(&b_empty[kat % ST]);
            ++gk;
            if (i + st.look == st.n - 1) mma_commit(b_qempty);
          }
        }
        if (!ok) break;
        g = gk;
      }
      // all issued MMAs complete before TMEM is released
      mma_commit(b_drain);
      mbar_wait_drain(b_drain, 0);
    }
    __syncwarp();
    }
  } else {
    // ------------------------------------------------------------ softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kAttRegsRow));
    const int X = warp >> 2;
    const int row = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lanes + X * 128, t_o = tmem + lanes + 256 + X * 128;
    const float c = a.c, grow = 8.f / c;
    const int row_t = row / a.G, row_g = row % a.G;
    unsigned ns = 0, no = 0;  // S tiles and results taken
    int g0 = 0;               // loads of the items before
    for (int ii = i0; ii < i1; ii += istep) {
      const AttnItem it = item(ii);
      const Steps<TREE> st(a, it);
      const int tx = it.t0 + (st.alt ? 0 : X * tpt);  // this tile's first token
      const int t = tx + row_t;
      const bool valid = row < tpt * a.G && t < it.tend;
      const bool busy = __any_sync(0xffffffffu, valid);  // warps whose rows hold nothing skip the arithmetic
      const int draft = TREE ? (it.klen + kAttTok - 1) / kAttTok : -1;
      const int lim = valid ? att_limit(it, t) : 0;
      const int lim0 = TREE ? it.klen : att_limit(it, tx);  // the tile's first row's
      uint32_t nodes[4] = {};
      bool sees = lim > 0;
      if (TREE && valid && it.j1 > draft)
        sees = tree_mask(a.parents + (long long)(it.lb % a.batch) * a.nodes, t, nodes);

      float m = -INFINITY, l = 0.f;
      uint32_t look = 0;
      int mine = 0;  // steps of this tile so far
      for (int i = 0; i < st.n; ++i) {
        if (!(st.who(i) >> X & 1)) continue;
        const int j = st.tile(i);
        mbar_wait(&b_s[X], ns & 1, abort, a.dbg, 206u + X, (unsigned)ii);
        ++ns;
        tc_fence_after();
        const bool masked = TREE ? (j == draft || (j + 1) * kAttTok > it.klen) : (j + 1) * kAttTok > lim0;
        if (busy) {
          float s[4][32];
#pragma unroll
          for (int q = 0; q < 4; ++q) tmem_ld32(t_s + q * 32, s[q]);
          tmem_ld_wait();
          if (masked) {
            const int cnt = lim - j * kAttTok;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const uint32_t w = TREE && j == draft ? nodes[q] : below(cnt, q);
#pragma unroll
              for (int e = 0; e < 32; ++e) s[q][e] = (w >> e & 1u) ? s[q][e] : -INFINITY;
            }
          }
          float mt[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            mt[q] = s[q][0];
#pragma unroll
            for (int e = 1; e < 32; ++e) mt[q] = fmaxf(mt[q], s[q][e]);
          }
          const float mx = fmaxf(fmaxf(mt[0], mt[1]), fmaxf(mt[2], mt[3]));
          const bool up = mx > m + grow;
          if (mine == 0) {
            m = mx;
          } else if (__any_sync(0xffffffffu, up)) {
            const float f = up ? ex2((m - mx) * c) : 1.f;
            if (up) {
              m = mx;
              l *= f;
            }
#pragma unroll
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
          float lq[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t r[16];
            float l0 = 0.f, l1 = 0.f;
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              const float p0 = ex2(fmaf(s[q][e], c, -mc)), p1 = ex2(fmaf(s[q][e + 1], c, -mc));
              l0 += p0;
              l1 += p1;
              r[e / 2] = T::pack(p0, p1);
            }
            lq[q] = l0 + l1;
            tmem_st16(t_s + q * 16, r);
          }
          l += (lq[0] + lq[1]) + (lq[2] + lq[3]);
          tmem_st_wait();
        }
        if (masked) {
          const int at = g0 + st.v_at(i);
          mbar_wait(&b_full[at % ST], (at / ST) & 1, abort, a.dbg, 208u + X, (unsigned)ii);
          const uint4* vt = reinterpret_cast<const uint4*>(smem + L::RING + (at % ST) * L::TILE) + row;
#pragma unroll 4
          for (int e = 0; e < L::TILE / 2048; ++e) {
            const uint4 w = vt[e * 128];
            look = Mma<T>::look(w.x, look);
            look = Mma<T>::look(w.y, look);
            look = Mma<T>::look(w.z, look);
            look = Mma<T>::look(w.w, look);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&b_p[X]);
        ++mine;
      }
      g0 += 2 * st.n;

      // ---------------------------------------------------------- the item's result
      bool bad = (look & 0x7fff7fffu) != 0u;
      if (mine) {
        mbar_wait(&b_o[X], no & 1, abort, a.dbg, 210u + X, (unsigned)ii);
        ++no;
        tc_fence_after();
      }
      if (st.alt) {
        if (mine == 0) m = -INFINITY, l = 0.f;
        xch[X * 128 + row] = make_float2(m, l);
        bad = named_bar_or(3, 256, bad);
      } else {
        bad = named_bar_or(1 + X, 128, bad);
      }
      RowOut<T, D> ro;
      const int head = it.h * a.G + row_g;
      auto place = [&](int tok, int hd, int r) {
        RowOut<T, D> x;
        x.out = reinterpret_cast<uint32_t*>(a.out + it.lb * a.o_lb + (long long)tok * a.o_t + hd * a.o_h);
        x.lse = a.lse ? a.lse + (long long)tok * a.kvh * a.G + hd : nullptr;
        x.part = it.slot >= 0 ? a.part + ((long long)it.slot * a.prows + r) * D : nullptr;
        x.part_ml = it.slot >= 0 ? a.part_ml + ((long long)it.slot * a.prows + r) : nullptr;
        return x;
      };
      const int prow = (st.alt ? 0 : X * 128) + row;
      ro = place(t, head, prow);
      ro.sees = TREE && it.j1 <= draft ? true : sees;
      if (bad) {
        // a value that is not finite in a tile that is masked in part: this tile's rows anew
        // (of two results over the same rows, by the first warpgroup)
        if (!(st.alt && X == 1)) {
          for (int rr = 0; rr < 32; ++rr) {
            if (!__shfl_sync(0xffffffffu, (int)valid, rr)) continue;
            const int tok = __shfl_sync(0xffffffffu, t, rr), hd = __shfl_sync(0xffffffffu, head, rr);
            const int see = __shfl_sync(0xffffffffu, lim, rr);
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = __shfl_sync(0xffffffffu, nodes[q], rr);
            const int from = it.j0 * kAttTok, to = min(see, it.j1 * kAttTok);
            RowOut<T, D> x = place(tok, hd, __shfl_sync(0xffffffffu, prow, rr));
            x.sees = __shfl_sync(0xffffffffu, (int)ro.sees, rr);
            float o[D / 32], mm, ll;
            const long long dr = (long long)it.y * a.nodes * D;
            attend_row<T, D>(a, a.q + it.lb * a.q_lb + (long long)tok * a.q_t + hd * a.q_h,
                             a.k + it.k0 * a.k_t + it.y * a.k_y, a.v + it.k0 * a.v_t + it.y * a.v_y, a.kd + dr, a.vd + dr,
                             from, x.sees ? to : from, TREE && it.j1 > draft && x.sees ? w : nullptr, mm, ll, o);
            if (lane == 0) x.stats(a, mm, ll);
            const float inv = x.sees ? 1.f / ll : 0.f;
#pragma unroll
            for (int e = 0; e < D / 64; ++e) {
              if (x.part) reinterpret_cast<float2*>(x.part)[lane * (D / 64) + e] = make_float2(o[2 * e], o[2 * e + 1]);
              else x.out[lane * (D / 64) + e] = T::pack(o[2 * e] * inv, o[2 * e + 1] * inv);
            }
          }
        }
      } else if (busy) {
        // of two results over the same rows, each warpgroup joins half the dims
        float f = 1.f, fy = 0.f;
        bool other = false;
        if (st.alt) {
          const float2 y = xch[(X ^ 1) * 128 + row];
          const float mm = fmaxf(m, y.x);
          other = st.count(X ^ 1) > 0;
          f = m == -INFINITY ? 0.f : ex2((m - mm) * c);
          fy = y.x == -INFINITY ? 0.f : ex2((y.x - mm) * c);
          l = l * f + y.y * fy;
          m = mm;
        }
        const float inv = ro.part ? 1.f : ro.sees ? 1.f / l : 0.f;
        const int d0 = st.alt ? X * (D / 2) : 0, d1 = st.alt ? d0 + D / 2 : D;
        if (valid && (!st.alt || X == 0)) ro.stats(a, m, l);
        for (int d = d0; d < d1; d += 32) {
          float o[32];
          if (mine) {
            tmem_ld32(t_o + d, o);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0.f;
          }
          if (st.alt) {
            float z[32];
            if (other) {
              tmem_ld32(tmem + lanes + 256 + (X ^ 1) * 128 + d, z);
              tmem_ld_wait();
            } else {
#pragma unroll
              for (int e = 0; e < 32; ++e) z[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = fmaf(z[e], fy, o[e] * f);
          }
          if (!ro.sees) {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0.f;
          }
          if (valid) {
            if (ro.part) {
#pragma unroll
              for (int e = 0; e < 32; e += 4)
                *reinterpret_cast<float4*>(ro.part + d + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
            } else {
#pragma unroll
              for (int e = 0; e < 32; e += 8)
                *reinterpret_cast<uint4*>(ro.out + (d + e) / 2) =
                    make_uint4(T::pack(o[e] * inv, o[e + 1] * inv), T::pack(o[e + 2] * inv, o[e + 3] * inv),
                               T::pack(o[e + 4] * inv, o[e + 5] * inv), T::pack(o[e + 6] * inv, o[e + 7] * inv));
            }
          }
        }
      }
      tc_fence_before();
      // the other warpgroup has read this one's O and statistics before they are written again
      if (st.alt) named_bar(3, 256);
    }
  }
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, kAttCols);
  }
  if (threadIdx.x == 0 && *abort) atomicOr(a.status, kStatusTimeout);
}

// Joins the partial results of work items that share their query rows, in order: a warp per
// row. Prompts: `merges` lists each group's first item and its parts; trees: nsplit
// consecutive items each.
template <class T, int D, bool TREE>
__global__ void __launch_bounds__(256) merge_kernel(const AttnArgs a) {
  grid_dep_wait();
  const int lane = threadIdx.x & 31, tpt = kAttRows / a.G;
  for (long long u = (long long)blockIdx.x * 8 + threadIdx.x / 32; u < (long long)a.n_merges * a.prows;
       u += (long long)gridDim.x * 8) {
    const int gi = (int)(u / a.prows), r = (int)(u % a.prows);
    AttnItem it;
    int parts;
    if constexpr (TREE) {
      it = tree_item(a, gi * a.nsplit);
      parts = a.nsplit;
    } else {
      const int2 mg = __ldg(a.merges + gi);
      it = load_item(a, mg.x);
      parts = mg.y;
    }
    // rows of tile A, then of tile B
    const int x = r / 128, rr = r % 128, t = it.t0 + x * tpt + rr / a.G;
    if (rr >= tpt * a.G || t >= it.tend) continue;
    const float2* ml = a.part_ml + (long long)it.slot * a.prows + r;
    const float* part = a.part + ((long long)it.slot * a.prows + r) * D;
    float m = -INFINITY, l = 0.f;
    bool sees = true;
    for (int s = 0; s < parts; ++s) {
      const float2 v = ml[(long long)s * a.prows];
      m = fmaxf(m, v.x);
      sees = sees && !(v.y < 0.f);
    }
    float o[D / 32] = {};
    for (int s = 0; s < parts && sees; ++s) {
      const float2 v = ml[(long long)s * a.prows];
      if (v.x == -INFINITY && v.y == 0.f) continue;
      const float f = v.x == -INFINITY ? 1.f : ex2((v.x - m) * a.c);
      l = fmaf(f, v.y, l);
      const float* p = part + (long long)s * a.prows * D + lane * (D / 32);
#pragma unroll
      for (int e = 0; e < D / 32; ++e) o[e] = fmaf(f, p[e], o[e]);
    }
    const float inv = sees ? 1.f / l : 0.f;
    const int head = it.h * a.G + rr % a.G;
    uint32_t* to = reinterpret_cast<uint32_t*>(a.out + it.lb * a.o_lb + (long long)t * a.o_t + head * a.o_h) + lane * (D / 64);
#pragma unroll
    for (int e = 0; e < D / 64; ++e) to[e] = T::pack(o[2 * e] * inv, o[2 * e + 1] * inv);
    if (a.lse && lane == 0) a.lse[(long long)t * a.kvh * a.G + head] = sees ? fmaf(m, a.scale, logf(l)) : -INFINITY;
  }
}

// Tensor maps of one call (tmKD, tmVD: trees).
struct AttMaps {
  CUtensorMap q, k, v, kd, vd;
};

template <class T, int D, bool TREE>
cudaError_t launch_attend(const AttMaps& m, const AttnArgs& a, int grid, int num_sms, cudaStream_t s) {
  static SmemLimit limit;
  if (cudaError_t e = limit.raise(attend_kernel<T, D, TREE>, AttSmem<D>::BYTES); e != cudaSuccess) return e;
  attend_kernel<T, D, TREE><<<grid, kAttThreads, AttSmem<D>::BYTES, s>>>(m.q, m.k, m.v, m.kd, m.vd, a);
  if (cudaError_t e = cudaGetLastError(); e != cudaSuccess) return e;
  if (a.n_merges == 0) return cudaSuccess;
  const long long blocks = ((long long)a.n_merges * a.prows + 7) / 8;
  return launch_pdl(merge_kernel<T, D, TREE>, dim3((unsigned)(blocks < 8ll * num_sms ? blocks : 8ll * num_sms)), dim3(256),
                    0, s, a);
}

}  // namespace
}  // namespace dc
