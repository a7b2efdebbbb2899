// dc_paged_attend.cu -- attention of one token of each sequence over a paged cache
// (dc_paged_attend).
//
// The query rows of a KV head's G query heads read its keys and values once:
//   o = sum_j p_j v_j / l,  p_j = 2^(c q . k_j - m),  l = sum_j p_j,  c = scale log2(e)
// A unit of work is a sequence's tokens and one KV head (behind a prefix that it shares, the tokens of its own), in
// tiles of 64 tokens. The tiles of all units lie in one line, with kPagStart places before each unit's for its start
// and end, and the CTAs, one an SM, cut the line into equal parts: a ragged batch needs no plan, since every
// CTA counts the line from the lengths on the device. Units that are cut, or that have a prefix, leave partial results,
// which paged_merge_kernel joins in a fixed order.
//
// A CTA: the last two warps load K, and queries and V (TMA, one box a page or half a page, a tile's in a ring of stages); teams
// of four warps take the tiles in turn, a warp 16 tokens of its team's tile, and keep a running softmax of their own:
//   S^T = K Q^T  [16 tokens x 8 rows], O^T += V^T P^T  [16 dims x 8 rows]
// on mma.sync m16n8k16: with 8 rows of queries to a KV head a 128-row tcgen05 tile would be nearly empty,
// and the tokens' side fills the 16 rows of this one. S^T leaves the first product in the layout that movmatrix
// turns into the second one's operand. The warps' results are joined in shared memory at a unit's end. Two teams where
// the registers last: a tile is a chain of some 700 cycles, in which HBM sends one of 64 dims (64 sequences of 1000 to 3331
// tokens, 4 KV heads of 64 dims, 8 query heads each: 38.4 us with one team, 30.4 with two, 31.7 with four; of 128 dims 79.4
// and 78.3 for the 130224 tokens below).
//
// What bounds it: HBM, behind some 9 us of latencies. 8 sequences of 32768 to 1 tokens, 8 KV heads of 128 dims: 524 MB in 79-80 us,
// 6.5-6.6 TB/s; on the way to that 7.1 TB/s between the first tile, 4 us after the start (lengths, line, page number, first
// boxes, each waits for the one before), and the last, then 1 us for a unit's end and 2.5 for the merge. (A CTA that
// happened to have many short units came 10 us behind the others before the units' starts counted in the line: 90 us.)
//
// Both operands of a product have one type, so P enters the second one rounded to the cache's. For up to 8 rows it does in
// two parts, the leading bits of each weight and the rest, rounded (16 bits of bf16 weights, 22 of fp16 ones): the results are off
// by their own rounding alone (8 sequences of 16384 tokens against 64 bits, 8 KV heads of 128 dims, bf16: 1.64e-3, with one
// part 2.15e-3), and HBM hides the second product (86.4 us, 86.1 with one part; 84.6 and 84.1 with 4 heads; single tokens of
// few pages 0.1 to 0.2 us more). More rows do not hide it: 16 of them 53.0 us instead of 51.9 (64 dims: 37.6, 34.7), 32 68.0
// instead of 58.4 (47.3, 42.4); their weights have one part, off by half a unit in the last place each, of the order of the result's
// rounding. l sums the weights unrounded. In fp16 the weights are up to 2^14 instead of 1, so that those above 2^-28 of the
// largest keep all their bits (taken back where the warps' results are joined).
#include <algorithm>

#include "dc_device.h"
#include "dc_paged.h"
#include "dc_rotate.cuh"
#include "dc_sm100.cuh"

namespace dc {
using namespace sm100;

namespace {

constexpr int kPagTok = 64;                  // tokens of a tile
constexpr int kPagTeam = 4;                  // warps of a team
constexpr int kPagMinTiles = 4;              // of a CTA, where there are more SMs than work
constexpr int kPagStart = 2;                 // what a unit's start and end take, in tiles

template <class T>
struct Frag;
template <>
struct Frag<Bf16> {
  static constexpr float kRoom = 0.f;
  using Type = TypeBf16;
  static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
template <>
struct Frag<Half> {
  static constexpr float kRoom = 14.f;
  using Type = TypeHalf;
  static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
template <int THREADS>
__device__ __forceinline__ void consumers_sync() {
  asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
}

// NT: blocks of 8 query rows of a unit.
template <int D, int NT>
struct PagSmem {
  static constexpr int RB = 8 * NT;
  static constexpr int TEAMS = NT == 4 ? 1 : 2, WARPS = kPagTeam * TEAMS, THREADS = 32 * (WARPS + 2);
  static constexpr bool TWO = NT == 1;          // P in two parts
  static constexpr int HALF = kPagTok * D * 2;  // a tile's K, or V
  static constexpr int STAGE = 2 * HALF;
  static constexpr int ST = D == 128 ? (NT == 4 ? 3 : 4) : (NT == 4 ? 6 : 8);  // (a stage belongs to one team)
  static constexpr int QROW = D * 2 + 16;  // (so that 8 rows lie in different banks)
  static constexpr int RED_ROW = D + 4;    // floats
  static constexpr int Q = ST * STAGE;
  static constexpr int RED = Q + 2 * RB * QROW;
  static constexpr int ML = RED + WARPS * RB * RED_ROW * 4;
  static constexpr int MISC = ML + WARPS * RB * 8;  // barriers, then the stages' valid counts
  static constexpr int VALID = MISC + 256;              // int [ST][4]
  static constexpr int SCAN = VALID + ST * 16;          // int [20], abort flag
  static constexpr int LINE = SCAN + 96;                // int [sequences + 1]
};
constexpr int kPagSeqs = 4096;  // sequences of a call, at most

// The tokens of sequence s that its own units cover are n ones from `from` on, up to len (0: it sees nothing).
struct SeqRun {
  int from, n, len;
};
// BEHIND: from L2, as said where the kernel begins.
template <bool BEHIND>
__device__ __forceinline__ int from_table(const int* p) { return BEHIND ? __ldcg(p) : __ldg(p); }
template <bool BEHIND>
__device__ __forceinline__ SeqRun seq_run(const PagedAttn& a, int s) {
  SeqRun r;
  const long long room = (long long)a.W << a.c.log;
  r.len = (int)min((long long)max(0, from_table<BEHIND>(a.lens + s)), room);
  r.from = s < a.sh.seqs ? __ldg(a.sh.prefix + s) : 0;
  r.n = r.len < r.from ? 0 : r.len - r.from;
  if (r.len < r.from) r.len = 0;
  return r;
}
// Tokens that the unit's tiles count: with a selection whole pages, as many as are read.
__device__ __forceinline__ int run_tokens(const PagedAttn& a, const SeqRun& r) {
  if (!a.selected) return r.n;
  return min(a.count, (int)(((unsigned)r.len + a.c.page - 1) >> a.c.log)) << a.c.log;  // (lengths may end at 2^31 - 1)
}

// The line's division: CTA b takes places [from(b), from(b + 1)); cta(x): who has place x.
struct PagCut {
  int per, extra;
  __device__ __forceinline__ PagCut(int total, int ctas) : per(total / ctas), extra(total - per * ctas) {}
  __device__ __forceinline__ int from(int b) const { return b * per + min(b, extra); }
  __device__ __forceinline__ int cta(int x) const {
    const int big = extra * (per + 1);
    return x < big ? x / (per + 1) : extra + (x - big) / per;
  }
};

// BEHIND: launched behind the prefixes' kernel.
template <class T, int D, int NT, bool BEHIND>
__global__ void __launch_bounds__(PagSmem<D, NT>::THREADS, 1)
    paged_attend_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                        const __grid_constant__ PagedAttn a) {
  using L = PagSmem<D, NT>;
  constexpr int RB = L::RB, ST = L::ST, TEAMS = L::TEAMS, WARPS = L::WARPS, THREADS = L::THREADS;
  extern __shared__ __align__(1024) uint8_t smem[];
  if (smem_u32(smem) & 1023u) {
    if (threadIdx.x == 0) atomicOr(a.c.status, kStatusBadShape);
    return;
  }
  uint64_t* bar = reinterpret_cast<uint64_t*>(smem + L::MISC);
  uint64_t *b_full = bar, *b_empty = bar + ST, *b_qfull = bar + 2 * ST, *b_qempty = bar + 2 * ST + 2;
  int* valid = reinterpret_cast<int*>(smem + L::VALID);
  int* scan = reinterpret_cast<int*>(smem + L::SCAN);
  volatile int* abort = scan + 20;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int* line = reinterpret_cast<int*>(smem + L::LINE);
  if (threadIdx.x == 0) {
    for (int s = 0; s < ST; ++s) {
      mbar_init(&b_full[s], 2);  // both producers
      mbar_init(&b_empty[s], kPagTeam);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(&b_qfull[x], 1);
      mbar_init(&b_qempty[x], WARPS);
    }
    *abort = 0;
    fence_mbar_init();
  }
  if (warp >= WARPS && lane == 0) prefetch_tmap(warp > WARPS ? &tmV : &tmK);
  // (Behind the prefixes' kernel, which is not needed until its results are joined, this one starts beside it and waits for it
  // at the end. What came before that kernel is complete: each of its blocks waits before it lets this one start. This one's
  // own wait, which would also say so to its L1 caches, comes too late: lengths and page numbers are read from L2, where
  // TMA reads the rest.)
  if (!BEHIND) grid_dep_wait();
  grid_dep_launch();
  if (warp >= WARPS && lane == 0) fence_proxy_async_global();  // (the producer's: what threads of earlier kernels wrote)

  // ---- the line: every sequence's first place
  constexpr int START = kPagStart;
  const int kvh = a.c.kvh, units = a.blocks * kvh;
  {
    auto places = [&](int s) {
      if (s >= a.S) return 0;
      if (blockIdx.x == 0 && from_table<BEHIND>(a.lens + s) > ((long long)a.W << a.c.log)) atomicOr(a.c.status, kStatusBadPage);
      return units * (START + max(1, (int)(((unsigned)run_tokens(a, seq_run<BEHIND>(a, s)) + kPagTok - 1) / kPagTok)));
    };
    int base = 0;
    for (int s0 = 0; s0 < a.S; s0 += THREADS) {
      const int s = s0 + threadIdx.x;
      int x = places(s);
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      if (lane == 31) scan[warp] = x;
      __syncthreads();
      int before = base;
      for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) before += scan[w];
        base += scan[w];
      }
      if (s < a.S) line[s + 1] = before + x;
      __syncthreads();
    }
    if (threadIdx.x == 0) line[0] = 0;
    __syncthreads();
  }
  const int total = line[a.S];
  const int ctas = min((int)gridDim.x, max(1, a.whole ? total / (START + 1) : (total + kPagMinTiles - 1) / kPagMinTiles));
  if (blockIdx.x == 0 && !a.whole) {
    for (int s = threadIdx.x; s <= a.S; s += THREADS)
      if (DC_INB(a.c, s, a.S + 2, 414)) a.line[s] = line[s];
    if (threadIdx.x == 0) a.line[a.S + 1] = ctas;
  }
  if ((int)blockIdx.x >= ctas) {
    if (BEHIND) grid_dep_wait();
    return;
  }
  const PagCut cut(total, ctas);
  // The sequence that has place x, the last one whose first place is not behind it.
  auto seq_at = [&](int x) {
    int s = 0;
    for (int n = a.S; n > 1;) {
      const int m = n / 2;
      if (line[s + m] <= x) s += m, n -= m;
      else n = m;
    }
    return s;
  };
  // Where CTA b's part begins: of whole units, with the first that begins there.
  auto part_of = [&](int b) {
    const int x = cut.from(b);
    if (!a.whole || x == total) return x;
    const int s = seq_at(x), len = (line[s + 1] - line[s]) / units, off = x - line[s];
    return line[s] + (off + len - 1) / len * len;
  };
  const int from = part_of(blockIdx.x), to = part_of(blockIdx.x + 1);
  auto wait = [&](uint64_t* b, uint32_t parity, unsigned site) { return mbar_wait(b, parity, abort, a.c.dbg, site); };

  if (warp >= WARPS) {
    // ------------------------------------------------------------ producers: of keys; of queries and values
    const bool of_v = warp > WARPS;
    // 32 boxes at a time (a box is a page, or half of one of 128 tokens): lane i finds the unit of place i / nb and
    // looks up the page of its box i % nb, whatever units the places belong to; then the places' tiles in turn.
    const uint64_t pol = l2_evict_first_policy();
    const int PB = min(a.c.page, kPagTok), log_b = min(a.c.log, 6), nb = kPagTok >> log_b;  // boxes of a tile
    const int log_p = a.c.log - log_b, in_page = (1 << log_p) - 1;                        // boxes of a page: 1 or 2
    const int log_n = 6 - log_b;
    int g = 0, nu = 0;
    bool ok = true;
    for (int p0 = from; p0 < to && ok; p0 += 32 >> log_n) {
      const int p = p0 + (lane >> log_n);
      int y = 0, n = 0, s = 0, unit = 0, h = 0, t = -1;  // of this lane's box: place in the pool, tokens; its tile (below 0: none)
      if (p < to) {
        s = seq_at(p);
        const int len = (line[s + 1] - line[s]) / units, off = p - line[s];
        unit = off / len;
        t = off - unit * len - START;
        h = a.blocks == 1 ? unit : unit % kvh;
        if (t >= 0) {
          const SeqRun run = seq_run<BEHIND>(a, s);
          const int* sel = a.selected ? a.selected + (long long)(s * kvh + h) * a.count : nullptr;
          int x = (t << log_n) + (lane & (nb - 1));  // the box's place in the selection, then in the sequence
          bool there = true;
          if (sel) {
            there = x < run_tokens(a, run) >> log_b;
            if (there) {
              const int e = __ldg(sel + (x >> log_p));
              there = e >= 0 && e < a.W;
              x = (e << log_p) + (x & in_page);
            }
          } else {
            x += run.from >> log_b;
          }
          const long long tok = (long long)x << log_b;
          if (there && tok < run.len) {
            const int page = from_table<BEHIND>(a.tables + (long long)s * a.W + (x >> log_p));
            if (page < 0 || page >= a.c.pages) {
              atomicOr(a.c.status, kStatusBadPage);
            } else {
              n = (int)min((long long)PB, run.len - tok);
              y = ((page * kvh + h) << a.c.log) + (x & in_page) * PB;
              if (!DC_INB(a.c, y + PB - 1, (long long)a.c.pages * kvh * a.c.page, 415)) n = 0;
            }
          }
        }
      }
      for (int i = 0; i < 32 && p0 + (i >> log_n) < to; i += nb) {
        const int ti = __shfl_sync(0xffffffffu, t, i);
        if (ti < 0) continue;
        if (of_v && (ti == 0 || (p0 == from && i == 0))) {
          // a unit's first tile here: its queries
          const int us = __shfl_sync(0xffffffffu, s, i), uh = __shfl_sync(0xffffffffu, h, i);
          const int r0 = a.blocks == 1 ? 0 : __shfl_sync(0xffffffffu, unit, i) / kvh * RB, nr = min(RB, a.c.G - r0);
          ok = __all_sync(0xffffffffu, wait(&b_qempty[nu & 1], ((nu >> 1) & 1) ^ 1, 501));
          if (!ok) break;
          if (lane == 0) mbar_expect_tx(&b_qfull[nu & 1], (uint32_t)nr * D * 2);
          __syncwarp();
          if (lane < nr)
            bulk_load(smem + L::Q + ((nu & 1) * RB + lane) * L::QROW, a.q + us * a.q_s + (uh * a.c.G + r0 + lane) * a.q_h,
                      D * 2, &b_qfull[nu & 1]);
          ++nu;
        }
        const int st = g % ST;
        ok = __all_sync(0xffffffffu, wait(&b_empty[st], ((g / ST) & 1) ^ 1, 502));
        if (!ok) break;
        const bool mine = lane >= i && lane < i + nb;
        const int loads = __popc(__ballot_sync(0xffffffffu, mine && n > 0));
        if (mine && !of_v) valid[st * 4 + lane - i] = n;
        __syncwarp();
        if (lane == 0) {
          if (loads) mbar_expect_tx(&b_full[st], (uint32_t)loads * PB * D * 2);
          else mbar_arrive(&b_full[st]);
        }
        __syncwarp();
        if (mine && n > 0)
          tma_load_4d(smem + st * L::STAGE + (of_v ? L::HALF : 0) + (lane - i) * PB * D * 2, of_v ? &tmV : &tmK, 0, y, 0, a.layer,
                      &b_full[st], pol);
        ++g;
      }
    }
    // every issued load must land before the CTA may exit (a stage's phase ends with the other producer's too; without that,
    // after a wait that gave up, this one runs out of time)
    if (lane == 0) {
      for (int t = g - ST < 0 ? 0 : g - ST; t < g; ++t) mbar_wait_drain(&b_full[t % ST], (t / ST) & 1);
      for (int t = nu - 2 < 0 ? 0 : nu - 2; t < nu; ++t) mbar_wait_drain(&b_qfull[t & 1], (t >> 1) & 1);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax
    const int PB = min(a.c.page, kPagTok), team = warp / kPagTeam, tok0 = warp % kPagTeam * 16, sub = tok0 / PB, rr0 = tok0 % PB;
    const uint32_t ring = smem_u32(smem);
    // this lane's rows of the ldmatrix operands: K (tokens by dims), V (dims by tokens, transposed on the way)
    const int kr = rr0 + (lane & 15), vr = rr0 + (lane & 7) + (lane >> 4) * 8;
    const uint32_t box = (uint32_t)(sub * PB * D * 2);
    const uint32_t k_at = box + kr * 128, v_at = L::HALF + box + vr * 128;
    const uint32_t k_c = lane >> 4, v_c = (lane >> 3) & 1;
    auto chunk = [&](uint32_t at, int r, uint32_t ch) { return at + (ch >> 3) * (PB * 128) + (((ch & 7) ^ (r & 7)) << 4); };
    float* red = reinterpret_cast<float*>(smem + L::RED);
    float2* red_ml = reinterpret_cast<float2*>(smem + L::ML);
    const float c2 = a.c2;
    int g = 0, nu = 0;
    int s = from < to ? seq_at(from) : 0;
    for (int place = from; place < to;) {
      while (line[s + 1] <= place) ++s;
      const int len = (line[s + 1] - line[s]) / units, off = place - line[s], unit = off / len, at = off - unit * len;
      const int end = min(len, at + to - place), tiles = len - START;
      const int j0 = max(0, at - START), j1 = max(0, end - START);
      place += end - at;
      if (j0 >= j1) continue;  // (a start without a tile)
      const int block = a.blocks == 1 ? 0 : unit / kvh, h = unit - block * kvh, r0 = block * RB, nr = min(RB, a.c.G - r0);
      // queries: the second operand of S^T = K Q^T
      uint32_t qf[D / 16][NT][2];
      // (a wait that gave up: the walk goes on to its end without waiting, so that the warps meet at their barrier)
      bool ok = __all_sync(0xffffffffu, wait(&b_qfull[nu & 1], (nu >> 1) & 1, 503));
      {
        const uint8_t* qs = smem + L::Q + (nu & 1) * RB * L::QROW;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const uint32_t* p = reinterpret_cast<const uint32_t*>(qs + (t * 8 + lane / 4) * L::QROW) + ks * 8 + lane % 4;
            qf[ks][t][0] = p[0];
            qf[ks][t][1] = p[4];
          }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&b_qempty[nu & 1]);
      ++nu;
      float o[D / 16][NT][4], m[NT][2], l[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        m[t][0] = m[t][1] = -INFINITY;
        l[t][0] = l[t][1] = 0.f;
#pragma unroll
        for (int e = 0; e < D / 16; ++e) o[e][t][0] = o[e][t][1] = o[e][t][2] = o[e][t][3] = 0.f;
      }
#pragma unroll 1
      for (int j = j0; j < j1; ++j, ++g) {
        if (TEAMS > 1 && g % TEAMS != team) continue;
        const int st = g % ST;
        ok = ok && __all_sync(0xffffffffu, wait(&b_full[st], (g / ST) & 1, 504));
        if (!ok) continue;
        const int n = valid[st * 4 + sub] - rr0;  // tokens of this warp's 16
        if (n > 0) {
          const uint32_t base = ring + st * L::STAGE;
          if (n < 16) {
            // values behind the last token: 0 times what is there must be 0
            const int ch = D / 8;
            for (int i = lane; i < (16 - n) * ch; i += 32) {
              const int r = rr0 + n + i / ch;
              *reinterpret_cast<uint4*>(smem + st * L::STAGE + L::HALF + box + i % ch / 8 * (PB * 128) + r * 128 + i % 8 * 16) =
                  make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async();
            __syncwarp();
          }
          float z[NT][4] = {};
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            uint32_t f[4];
            ldmatrix4(f, chunk(base + k_at, kr, 2 * ks + k_c));
#pragma unroll
            for (int t = 0; t < NT; ++t)
              if (NT == 1 || t * 8 < nr) Frag<T>::mma(z[t], f, qf[ks][t][0], qf[ks][t][1]);
          }
          if (n < 16) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              if (lane / 4 >= n) z[t][0] = z[t][1] = -INFINITY;
              if (lane / 4 + 8 >= n) z[t][2] = z[t][3] = -INFINITY;
            }
          }
          float mx[NT][2];
          bool up = false;
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            mx[t][0] = mx[t][1] = -INFINITY;
            if (NT == 1 || t * 8 < nr) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                float x = fmaxf(z[t][e], z[t][e + 2]);
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                mx[t][e] = x;
                up = up || x > m[t][e];
              }
            }
          }
          if (__any_sync(0xffffffffu, up)) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              float f[2];
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float x = fmaxf(m[t][e], mx[t][e]);
                f[e] = x == m[t][e] ? 1.f : ex2((m[t][e] - x) * c2);
                m[t][e] = x;
                l[t][e] *= f[e];
              }
#pragma unroll
              for (int e = 0; e < D / 16; ++e) {
                o[e][t][0] *= f[0];
                o[e][t][1] *= f[1];
                o[e][t][2] *= f[0];
                o[e][t][3] *= f[1];
              }
            }
          }
          uint32_t p[NT][2], rest[NT][2];
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            // (the difference first: the rounding of m c alone is a factor of any size where scores are far from 0)
            constexpr float up2 = Frag<T>::kRoom;
            const float m0 = m[t][0] == -INFINITY ? 0.f : m[t][0], m1 = m[t][1] == -INFINITY ? 0.f : m[t][1];
            const float p0 = ex2(fmaf(z[t][0] - m0, c2, up2)), p1 = ex2(fmaf(z[t][1] - m1, c2, up2));
            const float p2 = ex2(fmaf(z[t][2] - m0, c2, up2)), p3 = ex2(fmaf(z[t][3] - m1, c2, up2));
            l[t][0] += p0 + p2;
            l[t][1] += p1 + p3;
            if constexpr (L::TWO) {
              uint32_t h0, h1, r0, r1;
              Frag<T>::Type::parts(p0, p1, h0, r0);
              Frag<T>::Type::parts(p2, p3, h1, r1);
              p[t][0] = transpose8(h0);
              p[t][1] = transpose8(h1);
              rest[t][0] = transpose8(r0);
              rest[t][1] = transpose8(r1);
            } else {
              p[t][0] = transpose8(T::pack(p0, p1));
              p[t][1] = transpose8(T::pack(p2, p3));
            }
          }
#pragma unroll
          for (int e = 0; e < D / 16; ++e) {
            uint32_t f[4];
            ldmatrix4_trans(f, chunk(base + v_at, vr, 2 * e + v_c));
#pragma unroll
            for (int t = 0; t < NT; ++t)
              if (NT == 1 || t * 8 < nr) {
                Frag<T>::mma(o[e][t], f, p[t][0], p[t][1]);
                if constexpr (L::TWO) Frag<T>::mma(o[e][t], f, rest[t][0], rest[t][1]);
              }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&b_empty[st]);
      }
      // ---- the unit's result: the four warps' joined
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float x = l[t][e];
          x += __shfl_xor_sync(0xffffffffu, x, 4);
          x += __shfl_xor_sync(0xffffffffu, x, 8);
          x += __shfl_xor_sync(0xffffffffu, x, 16);
          const int r = t * 8 + lane % 4 * 2 + e;
          if (lane < 4) red_ml[warp * RB + r] = make_float2(m[t][e], x);
#pragma unroll
          for (int d = 0; d < D / 16; ++d) {
            float* to_d = red + (warp * RB + r) * L::RED_ROW + d * 16 + lane / 4;
            to_d[0] = o[d][t][e];
            to_d[8] = o[d][t][e + 2];
          }
        }
      }
      consumers_sync<32 * WARPS>();
      const bool joined = s < a.sh.seqs;
      long long slot = -1;
      if (j0 > 0 || j1 < tiles) slot = 2ll * blockIdx.x + (j0 == 0 ? 1 : 0);
      else if (joined) slot = 2ll * a.grid + (long long)s * units + unit;
      constexpr int E = D / 32;
      for (int r = warp; r < nr; r += WARPS) {
        float2 ml[WARPS];
        float mm = -INFINITY;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
          ml[w] = red_ml[w * RB + r];
          mm = fmaxf(mm, ml[w].x);
        }
        float sum = 0.f, x[E] = {};
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
          // (scores of NaN alone leave a reference of -infinity and a sum of NaN)
          if (ml[w].x == -INFINITY && ml[w].y == 0.f) continue;
          const float f = ml[w].x == -INFINITY ? 1.f : ex2(fmaf(ml[w].x - mm, c2, -Frag<T>::kRoom));
          sum = fmaf(f, ml[w].y, sum);
          const float* from_w = red + (w * RB + r) * L::RED_ROW + lane * E;
#pragma unroll
          for (int e = 0; e < E; ++e) x[e] = fmaf(f, from_w[e], x[e]);
        }
        if (slot >= 0) {
          const long long at = slot * RB + r;
          if (DC_INB(a.c, at, a.slots * RB, 410)) {
            float* to_p = a.part + at * D + lane * E;
            if constexpr (E == 4) *reinterpret_cast<float4*>(to_p) = make_float4(x[0], x[1], x[2], x[3]);
            else *reinterpret_cast<float2*>(to_p) = make_float2(x[0], x[1]);
            if (lane == 0) a.part_ml[at] = make_float2(mm, sum);
          }
        } else {
          const long long row = (long long)s * a.c.qh + h * a.c.G + r0 + r;
          if (!DC_INB(a.c, row, (long long)a.S * a.c.qh, 413)) continue;
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          uint32_t y[E / 2];
#pragma unroll
          for (int e = 0; e < E; e += 2) y[e / 2] = sum == 0.f ? 0u : T::pack(x[e] * inv, x[e + 1] * inv);
          uint32_t* to_o = reinterpret_cast<uint32_t*>(a.out + row * D) + lane * (E / 2);
          if constexpr (E == 4) *reinterpret_cast<uint2*>(to_o) = make_uint2(y[0], y[1]);
          else *to_o = y[0];
          if (a.lse && lane == 0) a.lse[row] = sum == 0.f ? -INFINITY : fmaf(mm, a.scale, logf(sum));
        }
      }
      consumers_sync<32 * WARPS>();
    }
  }
  __syncthreads();
  if (threadIdx.x == 0 && *abort) atomicOr(a.c.status, kStatusTimeout);
  if (BEHIND) grid_dep_wait();
}

// Joins the parts of one query row, a block each: those of its sequence's own tokens, then those of the prefix that it
// shares. Lane i of every warp takes the statistics of part i, 32 at a time; the parts' sums are shared out to the
// four warps, whose loads are all in flight at once, and added up in a fixed order.
// (Before its wait only what the host uploaded may be read.)
constexpr int kMergeWarps = 4;
template <class T, int D>
__global__ void __launch_bounds__(32 * kMergeWarps) paged_merge_kernel(const __grid_constant__ PagedAttn a) {
  constexpr int E = D / 32, START = kPagStart;
  __shared__ float shared[kMergeWarps - 1][D];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, row = blockIdx.x;
  const int s = row / a.c.qh, hq = row - s * a.c.qh, h = hq / a.c.G, r = hq - h * a.c.G;
  const int RB = a.rows, units = a.blocks * a.c.kvh, block = a.blocks == 1 ? 0 : r / RB, unit = block * a.c.kvh + h, rr = r - block * RB;
  // parts of the prefix: n2 of them, prows rows apart
  const bool joined = s < a.sh.seqs;
  int n2 = 0, least = 0;
  long long pre = 0;
  if (joined) {
    const int g = __ldg(a.sh.group + s), tokens = __ldg(a.sh.prefix + s), tpt = kAttRows / a.c.G;
    const int i = s - __ldg(a.sh.first + g), pair = i / (2 * tpt), in = i - pair * 2 * tpt;
    if (tokens > 0) {
      const int2 run = __ldg(a.sh.runs + __ldg(a.sh.unit + g) + pair * a.c.kvh + h);
      n2 = run.y;
      pre = (long long)run.x * a.sh.prows + (in >= tpt ? kAttRows : 0) + (in >= tpt ? in - tpt : in) * a.c.G + r;
    }
    least = max(1, tokens);
  }
  grid_dep_wait();
  const int len = joined ? a.lens[s] : 0;  // (looked at at the end: before the parts' loads it takes 2.7 us of 64 sequences' merge)
  // parts of its own tokens: n1; the first one's row, the second one's, the others 2 RB apart
  const int total = a.line[a.S], ctas = a.line[a.S + 1], at = a.line[s], ul = (a.line[s + 1] - at) / units, x0 = at + unit * ul;
  const PagCut cut(total, ctas);
  const int b0 = cut.cta(x0 + START), n1 = cut.cta(x0 + ul - 1) - b0 + 1;
  if (!joined && n1 == 1) return;  // (the result is there already)
  const int first = (n1 == 1 ? 2 * a.grid + s * units + unit : 2 * b0 + 1) * RB + rr, second = (2 * b0 + 2) * RB + rr;
  float mm = -INFINITY, sum = 0.f, x[E] = {};
  // (a reference is a score; the prefix's statistics hold a sum of -1 where a row saw nothing)
  auto load = [&](int i) {
    if (i < n1) {
      const int p = i == 0 ? first : second + (i - 1) * 2 * RB;
      return DC_INB(a.c, p, a.slots * RB, 411) ? a.part_ml[p] : make_float2(-INFINITY, 0.f);
    }
    const long long p = pre + (long long)(i - n1) * a.sh.prows;
    if (i >= n1 + n2 || !DC_INB(a.c, p, (long long)a.sh.places * a.sh.prows, 412)) return make_float2(-INFINITY, 0.f);
    const float2 v = a.pre_ml[p];
    return v.y < 0.f ? make_float2(-INFINITY, 0.f) : v;
  };
  auto sums = [&](int i) {
    const float* p = i < n1 ? a.part + (long long)(i == 0 ? first : second + (i - 1) * 2 * RB) * D
                            : a.pre + (pre + (long long)(i - n1) * a.sh.prows) * D;
    return p + lane * E;
  };
  const int parts = n1 + n2;
  const float2 v0 = load(lane);  // (32 parts or fewer: read once)
  mm = v0.x;
  for (int i = 32; i < parts; i += 32) mm = fmaxf(mm, load(i + lane).x);
#pragma unroll
  for (int x = 1; x < 32; x *= 2) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, x));
  for (int i0 = 0; i0 < parts; i0 += 32) {
    const float2 v = i0 ? load(i0 + lane) : v0;
    // (scores of NaN alone leave a reference of -infinity and a sum of NaN)
    const float f = v.x == -INFINITY ? (v.y != v.y ? 1.f : 0.f) : ex2((v.x - mm) * a.c2);
    if (i0 + lane < parts) sum = fmaf(f, v.y, sum);
    const int n = min(32, parts - i0);
#pragma unroll
    for (int k = 0; k < 32 / kMergeWarps; ++k) {
      const int i = k * kMergeWarps + warp;
      const float fi = __shfl_sync(0xffffffffu, f, i);
      if (i >= n) continue;
      const float* p = sums(i0 + i);
      if constexpr (E == 4) {
        const float4 z = *reinterpret_cast<const float4*>(p);
        x[0] = fmaf(fi, z.x, x[0]);
        x[1] = fmaf(fi, z.y, x[1]);
        x[2] = fmaf(fi, z.z, x[2]);
        x[3] = fmaf(fi, z.w, x[3]);
      } else {
        const float2 z = *reinterpret_cast<const float2*>(p);
        x[0] = fmaf(fi, z.x, x[0]);
        x[1] = fmaf(fi, z.y, x[1]);
      }
    }
  }
  if (warp > 0) {
#pragma unroll
    for (int e = 0; e < E; ++e) shared[warp - 1][lane * E + e] = x[e];
  }
  __syncthreads();
  if (warp > 0) return;
#pragma unroll
  for (int w = 0; w < kMergeWarps - 1; ++w)
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] += shared[w][lane * E + e];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (joined && len < least) sum = 0.f;  // a sequence that is shorter than its prefix, or not in use, sees nothing
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  uint32_t y[E / 2];
#pragma unroll
  for (int e = 0; e < E; e += 2) y[e / 2] = sum == 0.f ? 0u : T::pack(x[e] * inv, x[e + 1] * inv);
  if (!DC_INB(a.c, row, (long long)a.S * a.c.qh, 416)) return;
  uint32_t* to = reinterpret_cast<uint32_t*>(a.out + (long long)row * D) + lane * (E / 2);
  if constexpr (E == 4) *reinterpret_cast<uint2*>(to) = make_uint2(y[0], y[1]);
  else *to = y[0];
  if (a.lse && lane == 0) a.lse[row] = sum == 0.f ? -INFINITY : fmaf(mm, a.scale, logf(sum));
}

template <class T, int D, int NT, bool BEHIND>
cudaError_t launch(const PagedAttn& a, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t s) {
  static SmemLimit limit;
  if (cudaError_t e = limit.raise(paged_attend_kernel<T, D, NT, BEHIND>, PagSmem<D, NT>::LINE + (kPagSeqs + 1) * 4); e != cudaSuccess)
    return e;
  const size_t bytes = PagSmem<D, NT>::LINE + (size_t)(a.S + 1) * 4;
  if (cudaError_t e = launch_pdl(paged_attend_kernel<T, D, NT, BEHIND>, dim3(a.grid), dim3(PagSmem<D, NT>::THREADS), bytes, s, k, v, a); e != cudaSuccess)
    return e;
  if (a.whole) return cudaSuccess;
  const int rows = a.S * a.c.qh;  // (4096 * 1024 * 128 at most)
  return launch_pdl(paged_merge_kernel<T, D>, dim3((unsigned)rows), dim3(32 * kMergeWarps), 0, s, a);
}

template <class T, int D, bool BEHIND>
cudaError_t launch_rows(const PagedAttn& a, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t s) {
  if (a.rows == 8) return launch<T, D, 1, BEHIND>(a, k, v, s);
  if (a.rows == 16) return launch<T, D, 2, BEHIND>(a, k, v, s);
  return launch<T, D, 4, BEHIND>(a, k, v, s);
}
template <class T, int D>
cudaError_t launch_any(const PagedAttn& a, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t s) {
  return a.sh.grid > 0 ? launch_rows<T, D, true>(a, k, v, s) : launch_rows<T, D, false>(a, k, v, s);
}

static_assert(PagSmem<128, 1>::LINE + (kPagSeqs + 1) * 4 <= 232448 && PagSmem<128, 2>::LINE + (kPagSeqs + 1) * 4 <= 232448 &&
                  PagSmem<128, 4>::LINE + (kPagSeqs + 1) * 4 <= 232448 && PagSmem<64, 4>::LINE + (kPagSeqs + 1) * 4 <= 232448 &&
                  PagSmem<64, 2>::LINE + (kPagSeqs + 1) * 4 <= 232448,
              "more shared memory than a CTA may have");
static_assert(PagSmem<64, 1>::ST * 2 + 4 <= 32 && PagSmem<64, 1>::WARPS + 2 <= 20, "barriers, scan");
static_assert(PagSmem<128, 1>::ST % 2 == 0 && PagSmem<64, 1>::ST % 2 == 0 && PagSmem<128, 2>::ST % 2 == 0 && PagSmem<64, 2>::ST % 2 == 0,
              "a stage belongs to one team");

}  // namespace

long long paged_tiles(const PagedAttn& a) {
  const long long pages = a.count ? std::min(a.count, a.W) : a.W;
  return std::max(1ll, (pages * a.c.page + kPagTok - 1) / kPagTok);
}

size_t paged_workspace(PagedAttn* a, int D, int num_sms, char* base) {
  a->rows = a->c.G > 16 ? 32 : a->c.G > 8 ? 16 : 8;
  a->grid = num_sms;
  a->blocks = (a->c.G + a->rows - 1) / a->rows;
  // Units stay whole, with no second kernel (2 us on the host, 2.5 to 4 on the device) and no workspace, where the SMs that
  // then have less to do than others would have saved at most eight tiles' time (0.45 us each). us, whole and cut: 256 units
  // of 10 tiles of 128 dims 15.2, 18.3; 96 of 10 of 64 dims 11.3, 12.8; 6 of 16 of 64 dims 12.5, 8.7; 32 of 32 of 128 dims 17.9,
  // 11.2. (At most 32 tiles: the tables' width bounds lengths that may be uneven.)
  const long long tiles = paged_tiles(*a), units = (long long)a->S * a->blocks * a->c.kvh;
  const long long idle = (units + num_sms - 1) / num_sms * num_sms - units;
  a->whole = a->sh.groups == 0 && tiles <= 32 && idle * tiles <= 8ll * num_sms;
  if (a->whole) return 0;
  size_t end = 0;
  auto take = [&](size_t bytes) {
    const size_t at = (end + 15) / 16 * 16;
    end = at + bytes;
    return base + at;
  };
  a->slots = 2ll * a->grid + (a->sh.groups ? (long long)a->S * a->blocks * a->c.kvh : 0);
  const size_t rows = (size_t)a->slots * a->rows, pre = (size_t)a->sh.places * a->sh.prows;
  a->part = reinterpret_cast<float*>(take(rows * D * 4));
  a->part_ml = reinterpret_cast<float2*>(take(rows * 8));
  a->line = reinterpret_cast<int*>(take((size_t)(a->S + 2) * 4));
  a->pre = reinterpret_cast<float*>(take(pre * D * 4));
  a->pre_ml = reinterpret_cast<float2*>(take(pre * 8));
  return end;
}

cudaError_t launch_paged_attend(const PagedAttn& a, int D, int dtype, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t s) {
  if (dtype == DC_BF16) return D == 128 ? launch_any<Bf16, 128>(a, k, v, s) : launch_any<Bf16, 64>(a, k, v, s);
  return D == 128 ? launch_any<Half, 128>(a, k, v, s) : launch_any<Half, 64>(a, k, v, s);
}

}  // namespace dc
