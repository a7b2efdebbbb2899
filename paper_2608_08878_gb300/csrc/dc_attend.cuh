// dc_attend.cuh -- softmax attention of blocks of queries over keys in up to two
// places (a prompt's packed keys; a cache row's slots and then the drafted tokens):
// what dc_prompt.cu and dc_tree.cu share.
//
// A query row is one (token, query head); the rows of a KV head's G query heads are
// stacked, row = token * G + head, so that they read its keys and values once.
//   o = sum_j p_j v_j / l,  p_j = exp(scale (q . k_j) - m),  l = sum_j p_j
// over the keys j that the row sees. A row that sees none has o = 0, lse = -infinity.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dc_common.cuh"

namespace dc {

constexpr int kAttTok = 128;    // keys of a tile
constexpr int kAttRows = 128;   // query rows of a tile: 128 / G tokens
constexpr int kMaxNodes = 128;  // drafted tokens of a tree: one tile of keys

// Tensors of 16-bit elements; strides in elements.
struct AttnArgs {
  const uint16_t* q;
  long long q_t, q_h, q_lb;  // token, head, (layer, sequence) block
  const uint16_t *k, *v;     // first key place
  long long k_t, k_y, v_t, v_y;
  const uint16_t *kd, *vd;   // drafted keys [y][nodes][D]
  uint16_t* out;
  long long o_t, o_h, o_lb;
  float* lse;                // [token][head], or null (prompts)
  int G, kvh;
  float scale, c;            // c = scale * log2(e)
  // prompts: the plan's items
  const struct AttnItem* items;
  const int* first;          // CTA b takes items [first[b], first[b + 1])
  const int2* merges;        // work split over keys: each group's first item and its parts
  int n_items, n_merges;
  // partial results: fp32 [slot][prows][D], and each row's m and l
  float* part;
  float2* part_ml;
  int prows;
  long long out_len, part_rows;  // debug builds: elements of out, rows of part
  // trees
  int n, nodes, batch, rows, pairs, tiles, grid, line, ctas, per, extra;
  int two;  // whether items are two rows of one query tile each
  const int* rowlen;         // each row's length, or null (n)
  const int* parents;        // [batch][nodes]
  // pages: tables of their numbers [..][width], the pool's pages and their tokens, the layer, the status bit of a bad number
  const int* tables;
  int width, pages, page, layer;
  unsigned bad_page;
  unsigned long long wait_ns;  // att_wait_ns of the longest item
  unsigned* status;
  unsigned* dbg;
};

// How long a wait of the attention kernel may take before it gives up: kAttWaitNs, and where an item has more than
// kAttLongKeys keys what the other roles stand still while attend_row goes over it (a warp's 32 rows, the keys twice each:
// 18 us a key measured, 0.73 s for 40000; five times that).
#ifdef DC_DEBUG_BOUNDS
constexpr unsigned long long kAttWaitNs = 500000000ull;  // (so that a test can tell the two apart)
constexpr long long kAttLongKeys = 8192;
#else
constexpr unsigned long long kAttWaitNs = 10000000000ull;
constexpr long long kAttLongKeys = 262144;
#endif
inline unsigned long long att_wait_ns(long long keys) { return kAttWaitNs + 90000ull * (unsigned long long)keys; }

// Two tiles of query rows (A, then B) of one KV head and the keys they see.
struct AttnItem {
  int y, h, lb;   // key row coordinate; KV head and (layer, sequence) of the queries
  int t0, tend;   // A's first query token; the end of its sequence's tokens
  int k0, klen;   // the sequence's first key token (pages: its table's row) and its key count
  int off;        // query token t sees keys [0, min(klen, t + off)); kSeesAll: all
  int j0, j1;     // key tiles
  int slot;       // where a part of the keys leaves its partial result; -1: all keys
  int alt;        // 1: one tile of query rows only; 2 (trees): one tile of row y and one of row y + 1
  int eA, eB;     // key tiles that A's and B's rows see: below these
  int lowA, lowB; // what A's and B's first row sees, the least of their rows
};
constexpr int kSeesAll = 1 << 30;

// (t and off stay below 2^29, so the sum fits)
__host__ __device__ inline int att_limit(const AttnItem& it, int t) {
  const int x = t + it.off;
  return x < 0 ? 0 : x < it.klen ? x : it.klen;
}

// parts: weights (not below 0) in two numbers each, first their leading bits, towards 0, then what is left, rounded. That is never
// 0, so that infinity times the two is infinity: it is 2^-23 of the weight too large (bf16), or has its last bit set (fp16, 2^-24 at
// least: where weights are up to 2^14, n of them that are lost count as n 2^-38 of the largest). A clamp to the least
// number instead of these took 2 us of 80 of single tokens' attention.
struct TypeBf16 {
  static __device__ __forceinline__ void parts(float a, float b, uint32_t& first, uint32_t& rest) {
    constexpr float one = 1.f + 0x1p-23f;
    const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
    first = __byte_perm(x, y, 0x7632);
    rest = pack(fmaf(a, one, -__uint_as_float(x & 0xffff0000u)), fmaf(b, one, -__uint_as_float(y & 0xffff0000u)));
  }
  static __device__ __forceinline__ float2 two(uint32_t u) { return make_float2(bf16lo(u), bf16hi(u)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
  }
};
struct TypeHalf {
  static __device__ __forceinline__ void parts(float a, float b, uint32_t& first, uint32_t& rest) {
    const float x = __uint_as_float(__float_as_uint(a) & 0xffffe000u), y = __uint_as_float(__float_as_uint(b) & 0xffffe000u);
    first = pack(x, y);
    rest = pack(a - x, b - y) | 0x00010001u;
  }
  static __device__ __forceinline__ float2 two(uint32_t u) { return __half22float2(*reinterpret_cast<__half2*>(&u)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
  }
};

// The drafted tokens that node i sees (itself and its ancestors), 128 bits; false for
// an unused node. Parents come before their children, so the walk goes down and ends.
__device__ __forceinline__ bool tree_mask(const int* parents, int i, uint32_t (&w)[4]) {
  w[0] = w[1] = w[2] = w[3] = 0u;
  for (int x = i;;) {
    const uint32_t b = 1u << (x & 31);
    if (x < 32) w[0] |= b;
    else if (x < 64) w[1] |= b;
    else if (x < 96) w[2] |= b;
    else w[3] |= b;
    const int up = parents[x];
    if (up == -1) return true;
    if (up < -1 || up >= x) return false;
    x = up;
  }
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// One query row by one warp on plain arithmetic, D / 32 dims a lane: o (not divided by
// l), m (in units of 1 / c: raw q . k) and l over keys [j0, j1) of the first place below
// lim and the drafted ones of mask w. Only keys that the row sees are read.
template <class T, int D>
__device__ __noinline__ void attend_row(const AttnArgs& a, const uint16_t* q, const uint16_t* k, const uint16_t* v,
                                        const uint16_t* kd, const uint16_t* vd, int j0, int j1, const uint32_t* w,
                                        float& m, float& l, float (&o)[D / 32]) {
  constexpr int E = D / 64;  // 32-bit words a lane
  const int lane = threadIdx.x & 31;
  float x[D / 32];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float2 f = T::two(reinterpret_cast<const uint32_t*>(q)[lane * E + e]);
    x[2 * e] = f.x;
    x[2 * e + 1] = f.y;
  }
  auto dot = [&](const uint16_t* key) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float2 f = T::two(reinterpret_cast<const uint32_t*>(key)[lane * E + e]);
      s = fmaf(x[2 * e], f.x, fmaf(x[2 * e + 1], f.y, s));
    }
    return warp_sum(s);
  };
  m = -INFINITY;
  l = 0.f;
#pragma unroll
  for (int e = 0; e < D / 32; ++e) o[e] = 0.f;
  // the largest score, then the sums
  auto best = [&](const uint16_t* kj) { m = fmaxf(m, dot(kj)); };
#pragma unroll 4
  for (int j = j0; j < j1; ++j) best(k + j * a.k_t);
  if (w)
    for (int j = 0; j < a.nodes; ++j)
      if (w[j >> 5] >> (j & 31) & 1u) best(kd + (long long)j * D);
  {
    const float ref = m == -INFINITY ? 0.f : m;
    auto key = [&](const uint16_t* kj, const uint16_t* vj) {
      const float p = exp2f((dot(kj) - ref) * a.c);
      l += p;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float2 f = T::two(reinterpret_cast<const uint32_t*>(vj)[lane * E + e]);
        o[2 * e] = fmaf(p, f.x, o[2 * e]);
        o[2 * e + 1] = fmaf(p, f.y, o[2 * e + 1]);
      }
    };
#pragma unroll 4
    for (int j = j0; j < j1; ++j) key(k + j * a.k_t, v + j * a.v_t);
    if (w)
      for (int j = 0; j < a.nodes; ++j)
        if (w[j >> 5] >> (j & 31) & 1u) key(kd + (long long)j * D, vd + (long long)j * D);
  }
}

}  // namespace dc
