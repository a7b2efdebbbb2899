// dc_paged_select.cu -- the pages whose keys can have the largest scores with a query
// (dc_paged_select).
//
// A page's keys lie within [lo_i, hi_i] in dim i, so no score q . k of theirs is above
//   z = sum_i max(q_i, 0) hi_i + min(q_i, 0) lo_i.
// Its products are exact in 32 bits (16-bit factors), and of each two one is 0, so that fused multiply-adds round as
// the additions of the q_i hi_i or q_i lo_i alone would; their sum goes by neighbouring pairs, the eight dims of a lane
// first, then lanes 1, 2, 4 and 8 apart, and has the same bits however the pages are divided. (Choosing hi or lo by the
// sign first took 35 instructions a head and page of a lane instead of 11.)
//
// A cluster of CTAs takes a (sequence, KV head): each scores a share of its pages, D / 8 lanes a page, several pages'
// bounds on their way at once, and leaves them with the first CTA as 32-bit keys in the order of the numbers (the
// largest over the query heads). That CTA selects: a histogram of 2048 equal bins over the keys' range, the keys of the
// bin that holds the last one kept ranked by comparing each with all (many equal scores take a radix select), and
// the kept places written in order by ballots. Bound by the latency of these steps.
#include <algorithm>

#include "dc_device.h"
#include "dc_paged.h"
#include "dc_rotate.cuh"
#include "dc_select.cuh"
#include "dc_sm100.cuh"

namespace dc {
namespace {

constexpr int kSelThreads = 512, kSelWarps = kSelThreads / kWarp;
constexpr int kSelRounds = 4;    // pages of a warp at once: rounds of 32 / (D / 8)
constexpr int kSelKeys = 8192;   // keys that the selecting CTA keeps in shared memory; more lie in the workspace
constexpr int kSelBins = 2048;
constexpr int kSelList = 512;    // keys of the last bin that are ranked directly
constexpr uint32_t kKeyNan = 0xfffffffeu, kKeyLow = 0x007fffffu;  // the last: -infinity's

__device__ __forceinline__ uint32_t page_key(float z) { return z != z ? kKeyNan : score_key(z); }
// The larger of two, NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

struct SelectView {
  PagedView c;
  const uint16_t* q;
  long long q_s, q_h;
  const int *lens, *tables;
  int S, W, count, first, last;
  uint32_t* keys;  // [S][kvh][W]
  int* out;
  // the pages of sequence s
  __device__ __forceinline__ int pages_of(int s) const {
    const long long n = __ldg(lens + s);
    return n < 1 ? 0 : (int)min((long long)W, (n + c.page - 1) >> c.log);
  }
};

// A lane's eight dims of a page's bounds, or of the positive or negative part of a query, in 32 bits: dims 0 and 2, 1 and
// 3, 4 and 6, 5 and 7 in pairs.
struct Eight {
  F2 v[4];
};
template <class T>
__device__ __forceinline__ void eight(uint4 u, float2 (&f)[4]) {
  f[0] = T::two(u.x);
  f[1] = T::two(u.y);
  f[2] = T::two(u.z);
  f[3] = T::two(u.w);
}
__device__ __forceinline__ Eight pairs_of(const float2 (&f)[4]) {
  return Eight{{f2(f[0].x, f[1].x), f2(f[0].y, f[1].y), f2(f[2].x, f[3].x), f2(f[2].y, f[3].y)}};
}

// Two query heads (behind the last: it once more).
template <class T>
struct TwoQueries {
  Eight pos[2], neg[2];
  __device__ __forceinline__ TwoQueries(const SelectView& a, int s, int h, int g0, int l) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int head = h * a.c.G + min(g0 + g, a.c.G - 1);
      float2 f[4], p[4], n[4];
      eight<T>(__ldg(reinterpret_cast<const uint4*>(a.q + s * a.q_s + head * a.q_h) + l), f);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[e] = make_float2(max_nan(f[e].x, 0.f), max_nan(f[e].y, 0.f));
        n[e] = make_float2(-max_nan(-f[e].x, 0.f), -max_nan(-f[e].y, 0.f));
      }
      pos[g] = pairs_of(p);
      neg[g] = pairs_of(n);
    }
  }
  // A page's two scores: even lanes get the first one's.
  template <int LP>
  __device__ __forceinline__ float score(const Eight& hi, const Eight& lo) const {
    float y[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      // dims 0 + 1 and 2 + 3, then 4 + 5 and 6 + 7
      const float2 z0 = f2_out(fma2(pos[g].v[1], hi.v[1], fma2(neg[g].v[1], lo.v[1], fma2(pos[g].v[0], hi.v[0], neg[g].v[0] * lo.v[0]))));
      const float2 z1 = f2_out(fma2(pos[g].v[3], hi.v[3], fma2(neg[g].v[3], lo.v[3], fma2(pos[g].v[2], hi.v[2], neg[g].v[2] * lo.v[2]))));
      y[g] = __fadd_rn(__fadd_rn(z0.x, z0.y), __fadd_rn(z1.x, z1.y));
    }
    const bool odd = threadIdx.x & 1;
    float z = __fadd_rn(odd ? y[1] : y[0], __shfl_xor_sync(0xffffffffu, odd ? y[0] : y[1], 1));
#pragma unroll
    for (int o = 2; o < LP; o <<= 1) z = __fadd_rn(z, __shfl_xor_sync(0xffffffffu, z, o));
    return z;
  }
};

// The keys of pages [j0, j1) of a sequence and KV head, by a CTA: put(j, key). Bound by its instructions (some
// 160 a warp for two pages of 128 dims and four heads; 18 ns a page of a CTA) and their latency: four rounds side by side.
template <class T, int D, class Put>
__device__ __forceinline__ void score_pages(const SelectView& a, int s, int h, int j0, int j1, Put put) {
  constexpr int LP = D / 8, PW = kWarp / LP, STEP = kSelWarps * kSelRounds * PW;  // lanes a page; pages a round, of a CTA
  const int lane = threadIdx.x & 31, warp = threadIdx.x / kWarp, l = lane % LP;
  const int* table = a.tables + (long long)s * a.W;
  int page[kSelRounds];
  auto look = [&](int first) {
#pragma unroll
    for (int i = 0; i < kSelRounds; ++i) page[i] = first + i * PW < j1 ? __ldg(table + first + i * PW) : 0;
  };
  int first = j0 + warp * kSelRounds * PW + lane / LP;
  look(first);
  for (; first - lane / LP < j1; first += STEP) {
    uint4 hi[kSelRounds], lo[kSelRounds];
    uint32_t bad = 0u;
#pragma unroll
    for (int i = 0; i < kSelRounds; ++i) {
      bool fine = (unsigned)page[i] < (unsigned)a.c.pages;
      if (!fine) bad |= 1u << i;
      fine = fine && DC_INB(a.c, ((long long)page[i] * a.c.kvh + h) * 2 * LP + LP + l, (long long)a.c.pages * a.c.kvh * 2 * LP, 420);
      // (below 2^32: a layer has fewer than 2^27 heads of pages)
      const uint4* b = reinterpret_cast<const uint4*>(a.c.bounds) + (unsigned)((fine ? page[i] : 0) * a.c.kvh + h) * (unsigned)(2 * LP);
      hi[i] = __ldg(b + l);
      lo[i] = __ldg(b + LP + l);
    }
    look(first + STEP);
    float best[kSelRounds];
#pragma unroll
    for (int i = 0; i < kSelRounds; ++i) best[i] = -INFINITY;
#pragma unroll 1
    for (int g0 = 0; g0 < a.c.G; g0 += 2) {
      const TwoQueries<T> q(a, s, h, g0, l);
#pragma unroll
      for (int i = 0; i < kSelRounds; ++i) {
        float2 f[4], g[4];
        eight<T>(hi[i], f);
        eight<T>(lo[i], g);
        best[i] = max_nan(best[i], q.template score<LP>(pairs_of(f), pairs_of(g)));
      }
    }
#pragma unroll
    for (int i = 0; i < kSelRounds; ++i) {
      best[i] = max_nan(best[i], __shfl_xor_sync(0xffffffffu, best[i], 1));
      const int j = first + i * PW;
      if (l == 0 && j < j1) {
        const bool wrong = bad >> i & 1u;
        if (wrong) atomicOr(a.c.status, kStatusBadPage);
        put(j, wrong ? kKeyLow : page_key(best[i]));
      }
    }
  }
}

// Which of n keys are the `need` largest (1 <= need < n), the lower place first where they are equal: those above
// *least, and those equal to it up to place *cut. By a CTA.
struct TopScratch {
  int hist[kSelBins];
  int list[kSelList];
  int sh[4], wsum[kSelWarps], slots[kSelWarps];
  unsigned long long best[kSelWarps];
};
template <class Key>
__device__ __forceinline__ void top_keys(int n, int need, Key key, TopScratch& m, uint32_t* least, int* cut) {
  const int tid = threadIdx.x, lane = tid % kWarp, warp = tid / kWarp;
  auto sync = [] { __syncthreads(); };
  for (int b = tid; b < kSelBins; b += kSelThreads) m.hist[b] = 0;
  if (tid == 0) m.sh[2] = 0;
  uint32_t kmin = 0xffffffffu, kmax = 0u;
#pragma unroll 4
  for (int i = tid; i < n; i += kSelThreads) {
    kmin = min(kmin, key(i));
    kmax = max(kmax, key(i));
  }
  kmin = __reduce_min_sync(0xffffffffu, kmin);
  kmax = __reduce_max_sync(0xffffffffu, kmax);
  if (lane == 0) m.best[warp] = ((unsigned long long)kmax << 32) | kmin;
  __syncthreads();
  kmin = __reduce_min_sync(0xffffffffu, lane < kSelWarps ? (uint32_t)m.best[lane] : 0xffffffffu);
  kmax = __reduce_max_sync(0xffffffffu, lane < kSelWarps ? (uint32_t)(m.best[lane] >> 32) : 0u);
  const int bits = kmax > kmin ? 32 - __clz(kmax - kmin) : 0, shift = bits > 11 ? bits - 11 : 0;
  auto bin = [&](uint32_t k) { return (k - kmin) >> shift; };  // < kSelBins
#pragma unroll 4
  for (int i = tid; i < n; i += kSelThreads) atomicAdd(&m.hist[bin(key(i))], 1);
  __syncthreads();
  // thread t holds bins kSelBins - 1 - 4 t - (0..3), so that an exclusive scan over the threads counts the keys above
  int c[4], four = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    c[q] = m.hist[kSelBins - 1 - 4 * tid - q];
    four += c[q];
  }
  int all;
  int before = team_exclusive_scan<kSelThreads>(four, tid, m.wsum, &all, sync);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (before < need && need <= before + c[q]) {
      m.sh[0] = kSelBins - 1 - 4 * tid - q;
      m.sh[1] = before;
    }
    before += c[q];
  }
  __syncthreads();
  const uint32_t last = (uint32_t)m.sh[0];
  const int above = m.sh[1], members = m.hist[last];
  if (members <= kSelList) {
#pragma unroll 4
    for (int i = tid; i < n; i += kSelThreads)
      if (bin(key(i)) == last) m.list[atomicAdd(&m.sh[2], 1)] = i;
    __syncthreads();
    if (tid < members) {
      const int mine = m.list[tid];
      const uint32_t k = key(mine);
      int rank = 0;
      for (int o = 0; o < members; ++o) {
        const int other = m.list[o];
        const uint32_t ko = key(other);
        rank += ko > k || (ko == k && other < mine);
      }
      if (rank == need - above - 1) {
        m.sh[0] = (int)k;
        m.sh[3] = mine;
      }
    }
    __syncthreads();
    *least = (uint32_t)m.sh[0];
    *cut = m.sh[3];
    return;
  }
  __syncthreads();
  const SelectScratch scr{m.hist, m.sh, m.wsum, m.best, m.slots};
  int gt = 0;
  const uint32_t t = team_radix_select_wide<kSelThreads>(n, need, key, [](int) { return true; }, tid, scr, &gt, sync);
  // the (need - gt)-th lowest place among the equal ones
  auto tied = [&](int i) { return key(i) == t; };
  auto place = [](int i) { return ~(uint32_t)i; };
  int gt2 = 0;
  *cut = (int)~team_radix_select_wide<kSelThreads>(n, need - gt, place, tied, tid, scr, &gt2, sync);
  *least = t;
}

template <class T, int D>
__global__ void __launch_bounds__(kSelThreads, 1) page_select_kernel(const SelectView a, int ctas) {
  __shared__ uint32_t near[kSelKeys];
  __shared__ TopScratch scratch;
  const long long row = blockIdx.x / ctas;
  const int rank = (int)(blockIdx.x - row * ctas);
  const int s = (int)(row / a.c.kvh), h = (int)(row - (long long)s * a.c.kvh), tid = threadIdx.x, lane = tid % kWarp,
            warp = tid / kWarp;
  // (a CTA of the cluster may write to the first one's shared memory once that one runs)
  if (ctas > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  grid_dep_wait();
  grid_dep_launch();
  const int pages = a.pages_of(s);
  int* out = a.out + row * a.count;
  [[maybe_unused]] const int* end = a.out + (long long)a.S * a.c.kvh * a.count;  // (debug builds: what every write is checked against)
  if (ctas > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  if (pages <= a.count) {  // (the whole cluster)
    if (rank == 0)
      for (int i = tid; i < a.count; i += kSelThreads)
        if (DC_INB(a.c, out + i - a.out, end - a.out, 423)) out[i] = i < pages ? i : -1;
    return;
  }
  // n pages between those that are kept in any case, `need` of them
  const int n = pages - a.first - a.last, need = a.count - a.first - a.last;
  const bool all_near = n <= kSelKeys;
  uint32_t* far = a.keys + row * a.W;
  if (need > 0) {
    const int j0 = a.first + (int)((long long)n * rank / ctas), j1 = a.first + (int)((long long)n * (rank + 1) / ctas);
    score_pages<T, D>(a, s, h, j0, j1, [&](int j, uint32_t key) {
      if (!DC_INB(a.c, j - a.first, min(n, all_near ? kSelKeys : a.W), 421)) return;
      if (!all_near) {
        if (DC_INB(a.c, row * a.W + j - a.first, (long long)a.S * a.c.kvh * a.W, 422)) far[j - a.first] = key;
      } else if (rank == 0) near[j - a.first] = key;
      else sm100::st_cluster(sm100::cluster_addr(near + (j - a.first), 0), key);
    });
  }
  if (ctas > 1) {
    sm100::cluster_sync();
    if (rank > 0) return;
  } else {
    __syncthreads();
  }
  for (int i = tid; i < a.first + a.last; i += kSelThreads) {
    int* to = out + (i < a.first ? i : i + need);
    if (DC_INB(a.c, to - a.out, end - a.out, 424)) *to = i < a.first ? i : i + n;
  }
  if (need == 0) return;
  auto key = [&](int i) { return all_near ? near[i] : far[i]; };
  uint32_t least;
  int cut;
  top_keys(n, need, key, scratch, &least, &cut);
  // each warp takes a run of 32 places: its kept ones counted, the counts summed over the warps before, the places written
  auto kept = [&](int i) {
    if (i >= n) return false;
    const uint32_t k = key(i);
    return k > least || (k == least && i <= cut);
  };
  const int groups = (n + kWarp - 1) / kWarp;
  const int g0 = (int)((long long)groups * warp / kSelWarps), g1 = (int)((long long)groups * (warp + 1) / kSelWarps);
  int count = 0;
#pragma unroll 4
  for (int g = g0; g < g1; ++g) count += __popc(__ballot_sync(0xffffffffu, kept(g * kWarp + lane)));
  if (lane == 0) scratch.slots[warp] = count;
  __syncthreads();
  int at = (int)__reduce_add_sync(0xffffffffu, lane < warp ? (unsigned)scratch.slots[lane] : 0u);
  out += a.first;
#pragma unroll 4
  for (int g = g0; g < g1; ++g) {
    const int i = g * kWarp + lane;
    const bool f = kept(i);
    const unsigned mk = __ballot_sync(0xffffffffu, f);
    const int to = at + __popc(mk & ((1u << lane) - 1u));
    if (f && to < need && DC_INB(a.c, out + to - a.out, end - a.out, 425)) out[to] = a.first + i;
    at += __popc(mk);
  }
}

// Clusters of this many CTAs that the device holds at once; 0 if it has none of them.
template <class T, int D>
int clusters_of(int ctas) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kSelThreads);
  cudaLaunchAttribute la[1];
  la[0].id = cudaLaunchAttributeClusterDimension;
  la[0].val.clusterDim.x = (unsigned)ctas;
  la[0].val.clusterDim.y = la[0].val.clusterDim.z = 1;
  cfg.attrs = la;
  cfg.numAttrs = 1;
  int n = 0;
  cudaError_t e = cudaFuncSetAttribute(page_select_kernel<T, D>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&n, page_select_kernel<T, D>, &cfg);
  if (e != cudaSuccess) cudaGetLastError();
  return e == cudaSuccess ? n : 0;
}

template <class T, int D>
cudaError_t launch_select(const SelectView& v, int num_sms, cudaStream_t s) {
  const long long rows = (long long)v.S * v.c.kvh;
  // CTAs of a row: one for 64 pages, as long as every one of them has an SM; above 8 of them 16 or 12, where the device holds
  // that many clusters at once (us with 8 and with more, bounds in L2 and not: 8 rows of 2048 pages of 64 and 4 query heads, 12:
  // 11.5, 10.9 and 14.5, 14.4; of 8192 30.0, 24.7 and 36.0, 30.2; 4 rows of 2048 and 8 query heads, 16: 14.5, 11.0 and 17.8, 14.1.
  // 16 for 8 rows, in two turns: 12.7 instead of 10.9).
  int ctas = 1;
  while (v.W > v.count && ctas < 8 && ctas * 64 < v.W && rows * ctas * 2 <= num_sms) ctas *= 2;
  if (ctas == 8 && v.W > 8 * 64 && rows * 12 <= num_sms) {
    static PerDevice<int> of16, of12;
    if (rows <= of16.get([] { return clusters_of<T, D>(16); })) ctas = 16;
    else if (rows <= of12.get([] { return clusters_of<T, D>(12); })) ctas = 12;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * ctas));
  cfg.blockDim = dim3(kSelThreads);
  cfg.stream = s;
  cudaLaunchAttribute la[2];
  la[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  la[0].val.programmaticStreamSerializationAllowed = 1;
  la[1].id = cudaLaunchAttributeClusterDimension;
  la[1].val.clusterDim.x = (unsigned)ctas;
  la[1].val.clusterDim.y = la[1].val.clusterDim.z = 1;
  cfg.attrs = la;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, page_select_kernel<T, D>, v, ctas);
}

}  // namespace

cudaError_t launch_paged_select(const PagedView& c, int D, int dtype, const dc_paged_select_args& x, int num_sms,
                                cudaStream_t s) {
  SelectView v{};
  v.c = c;
  v.q = static_cast<const uint16_t*>(x.q);
  v.q_s = x.q_seq_stride;
  v.q_h = x.q_head_stride;
  v.lens = x.lens;
  v.tables = x.tables;
  v.S = x.seqs;
  v.W = x.table_width;
  v.count = x.count;
  v.first = x.keep_first;
  v.last = x.keep_last;
  v.keys = static_cast<uint32_t*>(x.workspace);
  v.out = x.out;
  if (dtype == DC_BF16) return D == 128 ? launch_select<Bf16, 128>(v, num_sms, s) : launch_select<Bf16, 64>(v, num_sms, s);
  return D == 128 ? launch_select<Half, 128>(v, num_sms, s) : launch_select<Half, 64>(v, num_sms, s);
}

}  // namespace dc
