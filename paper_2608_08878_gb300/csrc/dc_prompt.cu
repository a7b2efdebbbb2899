// dc_prompt.cu -- attention of packed prompts (dc_prompt_plan_create,
// dc_prompt_attend): the plan's work items and the C ABI.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdio>
#include <functional>
#include <memory>
#include <new>
#include <queue>
#include <string>
#include <vector>

#include "../../include/distillcache.h"
#include "dc_attend_kernel.cuh"
#include "dc_prompt.h"

namespace dc {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

bool att_map(CUtensorMap* m, bool bf16, const void* base, int rank, const long long* dims, const long long* strides,
             const int* box) {
  static const EncodeTiledFn encode = [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q);
    return e == cudaSuccess && q == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeTiledFn>(fn) : nullptr;
  }();
  if (!encode) return false;
  cuuint64_t d[5], st[4];
  cuuint32_t b[5], one[5];
  for (int i = 0; i < rank; ++i) {
    d[i] = (cuuint64_t)dims[i];
    b[i] = (cuuint32_t)box[i];
    one[i] = 1;
    if (i) st[i - 1] = dims[i] > 1 ? (cuuint64_t)strides[i - 1] * 2 : 16;
  }
  return encode(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank,
                const_cast<void*>(base), d, st, b, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool att_map_q(CUtensorMap* m, bool bf16, const AttnArgs& a, int D, long long tokens, long long lbs) {
  const long long dims[5] = {D, a.G, a.kvh, tokens, lbs}, strides[4] = {a.q_h, a.G * a.q_h, a.q_t, a.q_lb};
  const int box[5] = {64, a.G, 1, kAttRows / a.G, 1};
  return att_map(m, bf16, a.q, 5, dims, strides, box);
}

bool att_map_kv(CUtensorMap* m, bool bf16, const void* base, int D, long long ys, long long y_stride, long long tokens,
                long long t_stride) {
  const long long dims[3] = {D, ys, tokens}, strides[2] = {y_stride, t_stride};
  const int box[3] = {64, 1, kAttTok};
  return att_map(m, bf16, base, 3, dims, strides, box);
}

namespace {

thread_local std::string g_prompt_error;

dc_status prompt_fail(dc_status s, const std::string& msg) {
  g_prompt_error = msg;
  return s;
}

dc_status prompt_cuda(cudaError_t e, const char* what) {
  return prompt_fail(e == cudaErrorMemoryAllocation ? DC_ERR_OOM : DC_ERR_CUDA,
                     std::string(what) + ": " + cudaGetErrorString(e));
}

constexpr unsigned kPlanMagic = 0x44435050u;  // "DCPP"

// While one lives, this thread's allocations, frees and waits are no part of a stream capture that is under way here or in
// another thread: under the default mode each of them is refused, and the capture lost.
class OutsideCapture {
 public:
  OutsideCapture() { cudaThreadExchangeStreamCaptureMode(&mode_); }
  ~OutsideCapture() { cudaThreadExchangeStreamCaptureMode(&mode_); }
  OutsideCapture(const OutsideCapture&) = delete;
  OutsideCapture& operator=(const OutsideCapture&) = delete;

 private:
  cudaStreamCaptureMode mode_ = cudaStreamCaptureModeRelaxed;
};

// Copies to the device and waits until it is there, whatever stream the next call is on. (cudaMemcpy may return once
// pageable memory is staged, and orders the rest on the legacy stream only, which a non-blocking stream does not wait
// for; and it waits for all that the legacy stream is busy with. A stream of its own does neither. It is kept, one a
// device: making one took 18 us of a small plan's 39.)
cudaError_t upload_now(void* dst, const void* src, size_t bytes) {
  static std::atomic<cudaStream_t> kept[kDevices];
  const int dev = device_slot();
  cudaStream_t s = dev >= 0 ? kept[dev].load(std::memory_order_acquire) : nullptr;
  bool drop = false;
  if (!s) {
    cudaError_t e = cudaStreamCreateWithFlags(&s, cudaStreamNonBlocking);
    if (e != cudaSuccess) return e;
    cudaStream_t none = nullptr;
    drop = dev < 0 || !kept[dev].compare_exchange_strong(none, s);
  }
  const cudaError_t e = cudaMemcpyAsync(dst, src, bytes, cudaMemcpyHostToDevice, s), done = cudaStreamSynchronize(s);
  if (drop) cudaStreamDestroy(s);
  return e != cudaSuccess ? e : done;
}

}  // namespace
}  // namespace dc

struct dc_prompt_plan {
  unsigned magic = dc::kPlanMagic;
  int device = 0;
  int q_heads = 0, kv_heads = 0, head_dim = 0;
  long long q_tokens = 0, k_tokens = 0;
  int n_items = 0, n_merges = 0, n_slots = 0, prows = 0, grid = 0, num_sms = 0;
  int item_tiles = 0;  // key tiles of the longest item
  // device: one allocation, the status words first
  unsigned* status = nullptr;     // [0] status, [8..15] the first failure
  dc::AttnItem* items = nullptr;
  int* first = nullptr;
  int2* merges = nullptr;
  size_t workspace() const { return (size_t)n_slots * prows * (head_dim + 2) * sizeof(float); }
};

namespace dc {
namespace {

// Times in us that divide the work (measured with heads of 128 dims): a key tile of an item
// with two tiles of query rows, or with one; an item's start and end; the second kernel and the
// bytes of partial results that it takes in a us.
constexpr double kStepUs = 1.4, kAltStepUs = 1.0, kItemUs = 3.5, kMergeUs = 4.0, kMergeBytes = 5e6;

double step_cost(const AttnItem& it) { return it.alt ? kAltStepUs : kStepUs; }
double item_cost(const AttnItem& it) { return (it.j1 - it.j0) * step_cost(it) + kItemUs; }

// Items (of one part each) or parts, those of CTA b at [first[b], first[b + 1]).
struct Division {
  std::vector<AttnItem> items;
  std::vector<int> first;
  std::vector<int2> merges;  // an item's first part and its parts
  int slots = 0, prows = 0;
  double us = 0;
};

// Whole items, the longest first, each to the CTA with the least to do.
Division divide_whole(const std::vector<AttnItem>& items, int num_sms) {
  Division d;
  std::vector<int> order(items.size());
  for (size_t i = 0; i < order.size(); ++i) order[i] = (int)i;
  std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return item_cost(items[a]) > item_cost(items[b]); });
  const int grid = (int)std::min<size_t>(items.size(), (size_t)num_sms);
  std::vector<std::vector<int>> of(grid);
  using Load = std::pair<double, int>;
  std::priority_queue<Load, std::vector<Load>, std::greater<Load>> least;
  for (int b = 0; b < grid; ++b) least.push({0.0, b});
  for (int i : order) {
    Load x = least.top();
    least.pop();
    of[x.second].push_back(i);
    x.first += item_cost(items[i]);
    d.us = std::max(d.us, x.first);
    least.push(x);
  }
  for (int b = 0; b < grid; ++b) {
    d.first.push_back((int)d.items.size());
    for (int i : of[b]) d.items.push_back(items[i]);
  }
  d.first.push_back((int)d.items.size());
  return d;
}

// All key tiles in one line, cut into `grid` parts of equal time. A part of an item has 2 key
// tiles at least.
Division divide_cut(const std::vector<AttnItem>& items, int grid, int G, int D) {
  Division d;
  double total = grid * kItemUs;  // (each cut starts an item once more)
  for (const AttnItem& it : items) total += item_cost(it);
  // (what a CTA leaves of its share goes to the next one)
  double load = 0, share = total / grid;
  d.first.push_back(0);
  auto next = [&] {
    d.us = std::max(d.us, load);
    share += total / grid - load;
    load = 0;
    d.first.push_back((int)d.items.size());
  };
  double partial = 0;
  for (const AttnItem& it : items) {
    int at = it.j0, parts = 0;
    const int index = (int)d.items.size();
    for (;;) {
      AttnItem x = it;
      x.j0 = at;
      const bool last = (int)d.first.size() == grid;  // the last CTA takes what is left
      if (!last && load + item_cost(x) > share + kItemUs / 2) {
        const int fit = (int)((share - load - kItemUs) / step_cost(it));
        if (fit < 2 && load > 0) {
          next();
          continue;
        }
        if (std::max(fit, 2) < x.j1 - x.j0 - 1) x.j1 = x.j0 + std::max(fit, 2);
      }
      at = x.j1;
      if (parts || at < it.j1) x.slot = d.slots++;
      ++parts;
      load += item_cost(x);
      d.items.push_back(x);
      if (at >= it.j1) break;
      next();
    }
    if (parts > 1) {
      const int rows = it.alt ? (it.tend - it.t0) * G : 256;
      d.prows = std::max(d.prows, rows);
      partial += (double)parts * rows * D * 8;
      d.merges.push_back(make_int2(index, parts));
    }
  }
  next();
  if (!d.merges.empty()) d.us += kMergeUs + partial / kMergeBytes;
  return d;
}

Division plan_items(const int* q_lens, const int* k_lens, int n, int kvh, int G, int D, bool causal, int num_sms) {
  const int tpt = kAttRows / G;
  std::vector<AttnItem> items;
  long long q0 = 0, k0 = 0;
  long long tiles = 0;
  for (int s = 0; s < n; ++s) {
    const int ql = q_lens[s], kl = k_lens[s];
    for (int t = 0; t < ql; t += 2 * tpt)
      for (int h = 0; h < kvh; ++h) {
        AttnItem it{};
        it.y = it.h = h;
        it.t0 = (int)q0 + t;
        it.tend = (int)(q0 + ql);
        it.k0 = (int)k0;
        it.klen = kl;
        it.off = causal ? (int)(kl - ql + 1 - q0) : kSeesAll;
        it.j1 = (att_limit(it, std::min(it.tend, it.t0 + 2 * tpt) - 1) + kAttTok - 1) / kAttTok;
        it.slot = -1;
        it.alt = it.tend - it.t0 <= tpt;
        it.lowA = att_limit(it, it.t0);
        it.lowB = it.alt ? it.lowA : att_limit(it, it.t0 + tpt);
        it.eA = it.alt ? it.j1 : (att_limit(it, it.t0 + tpt - 1) + kAttTok - 1) / kAttTok;
        it.eB = it.j1;
        items.push_back(it);
        tiles += it.j1;
      }
    q0 += ql;
    k0 += kl;
  }
  Division best = divide_whole(items, num_sms);
  // Work cut evenly where that is quicker, merge included: on all SMs, or, of little work, on fewer
  // with more tiles each.
  for (int least = 2; least <= 8 && !items.empty(); least *= 2) {
    const int grid = (int)std::min<long long>(num_sms, tiles / least);
    if (grid < 2) break;
    Division cut = divide_cut(items, grid, G, D);
    if (cut.us < best.us) best = std::move(cut);
    if (grid < num_sms) continue;
    break;
  }
  return best;
}

}  // namespace
}  // namespace dc

using dc::prompt_cuda;
using dc::prompt_fail;

extern "C" {

const char* dc_prompt_last_error(void) { return dc::g_prompt_error.c_str(); }

dc_status dc_prompt_plan_create(const int* q_lens, const int* k_lens, int n, int q_heads, int kv_heads, int head_dim,
                                int causal, dc_prompt_plan** out) try {
  if (!out) return prompt_fail(DC_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (!q_lens || n < 1) return prompt_fail(DC_ERR_INVALID_ARG, "need the lengths of at least one sequence");
  if (!k_lens) k_lens = q_lens;
  if (head_dim != 64 && head_dim != 128) return prompt_fail(DC_ERR_INVALID_ARG, "head_dim must be 64 or 128");
  if (kv_heads < 1 || kv_heads > 65535 || q_heads < kv_heads || q_heads % kv_heads || q_heads / kv_heads > dc::kAttRows)
    return prompt_fail(DC_ERR_INVALID_ARG, "q_heads must be kv_heads times 1 to 128");
  long long qt = 0, kt = 0;
  for (int s = 0; s < n; ++s) {
    if (q_lens[s] < 0 || k_lens[s] < 0) return prompt_fail(DC_ERR_INVALID_ARG, "lengths must be >= 0");
    qt += q_lens[s];
    kt += k_lens[s];
  }
  if (qt > (1 << 29) || kt > (1 << 29)) return prompt_fail(DC_ERR_INVALID_ARG, "at most 2^29 packed tokens");
  // (64 bytes an item, and their numbers are ints)
  long long count = 0;
  const int item_tokens = 2 * (dc::kAttRows / (q_heads / kv_heads));
  for (int s = 0; s < n; ++s) count += ((long long)q_lens[s] + item_tokens - 1) / item_tokens * kv_heads;
  if (count > (1 << 29)) return prompt_fail(DC_ERR_INVALID_ARG, "too much work: at most 2^29 items of 256 query rows");
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return prompt_cuda(e, "cudaGetDevice");
  const dc::Division v = dc::plan_items(q_lens, k_lens, n, kv_heads, q_heads / kv_heads, head_dim, causal != 0, sms);
  // one block on the device: status words, items, each CTA's first item, merges
  auto up = [](size_t x) { return (x + 15) / 16 * 16; };
  const size_t at_items = 64, at_first = up(at_items + v.items.size() * sizeof(dc::AttnItem)),
               at_merges = up(at_first + v.first.size() * sizeof(int)), bytes = up(at_merges + v.merges.size() * sizeof(int2));
  std::vector<char> host(bytes, 0);
  std::copy_n((const char*)v.items.data(), v.items.size() * sizeof(dc::AttnItem), host.data() + at_items);
  std::copy_n((const char*)v.first.data(), v.first.size() * sizeof(int), host.data() + at_first);
  std::copy_n((const char*)v.merges.data(), v.merges.size() * sizeof(int2), host.data() + at_merges);
  auto p = std::make_unique<dc_prompt_plan>();
  const dc::OutsideCapture outside;
  char* block = nullptr;
  e = cudaMalloc(&block, bytes);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return prompt_cuda(e, "plan allocation");
  }
  e = dc::upload_now(block, host.data(), bytes);
  if (e != cudaSuccess) {
    cudaFree(block);
    return prompt_cuda(e, "plan upload");
  }
  p->device = dev;
  p->num_sms = sms;
  p->q_heads = q_heads;
  p->kv_heads = kv_heads;
  p->head_dim = head_dim;
  p->q_tokens = qt;
  p->k_tokens = kt;
  p->n_items = (int)v.items.size();
  p->n_merges = (int)v.merges.size();
  p->n_slots = v.slots;
  p->prows = v.prows;
  p->grid = (int)v.first.size() - 1;
  for (const dc::AttnItem& it : v.items) p->item_tiles = std::max(p->item_tiles, it.j1 - it.j0);
  p->status = (unsigned*)block;
  p->items = (dc::AttnItem*)(block + at_items);
  p->first = (int*)(block + at_first);
  p->merges = (int2*)(block + at_merges);
  *out = p.release();
  return DC_OK;
} catch (const std::bad_alloc&) {
  return prompt_fail(DC_ERR_OOM, "host allocation failed");
}

dc_status dc_prompt_plan_destroy(dc_prompt_plan* p) {
  if (!p) return DC_OK;
  if (p->magic != dc::kPlanMagic) return DC_ERR_INVALID_ARG;
  {
    const dc::OutsideCapture outside;
    cudaFree(p->status);
  }
  p->magic = 0;
  delete p;
  return DC_OK;
}

dc_status dc_prompt_attend(const dc_prompt_plan* p, const dc_prompt_args* args, void* stream) {
  if (!p || p->magic != dc::kPlanMagic) return prompt_fail(DC_ERR_INVALID_ARG, "not a plan");
  if (!args) return prompt_fail(DC_ERR_INVALID_ARG, "args is NULL");
  const dc_prompt_args& x = *args;
  if (x.dtype != DC_BF16 && x.dtype != DC_FP16) return prompt_fail(DC_ERR_INVALID_ARG, "dtype must be DC_BF16 or DC_FP16");
  if (!(x.scale > 0.f) || !std::isfinite(x.scale)) return prompt_fail(DC_ERR_INVALID_ARG, "scale must be positive and finite");
  if (p->n_items == 0) return DC_OK;
  if (!x.q || !x.out || (p->k_tokens && (!x.k || !x.v))) return prompt_fail(DC_ERR_INVALID_ARG, "NULL pointer");
  const uintptr_t at = (uintptr_t)x.q | (uintptr_t)x.out | (p->k_tokens ? (uintptr_t)x.k | (uintptr_t)x.v : 0);
  const long long strides[] = {x.q_token_stride, x.q_head_stride, x.k_token_stride, x.k_head_stride, x.v_token_stride, x.v_head_stride};
  const long long counts[] = {p->q_tokens, p->q_heads, p->k_tokens, p->kv_heads, p->k_tokens, p->kv_heads};
  for (int i = 0; i < 6; ++i)  // (the stride of a dimension of one says nothing)
    if (counts[i] > 1 && (strides[i] < 8 || strides[i] % 8 || strides[i] >= (1ll << 38)))
      return prompt_fail(DC_ERR_INVALID_ARG, "strides must be multiples of 8 in [8, 2^38)");
  if (x.workspace_bytes < p->workspace() || (p->workspace() && (!x.workspace || (uintptr_t)x.workspace & 15)))
    return prompt_fail(DC_ERR_INVALID_ARG, "the workspace must hold dc_prompt_workspace bytes, 16-byte aligned");
  if (at & 15) return prompt_fail(DC_ERR_INVALID_ARG, "q, k, v and out must be 16-byte aligned");
  if ((uintptr_t)x.lse & 3) return prompt_fail(DC_ERR_INVALID_ARG, "lse must be 4-byte aligned");
  int dev = -1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return prompt_cuda(e, "cudaGetDevice");
  if (dev != p->device) return prompt_fail(DC_ERR_INVALID_ARG, "the plan belongs to another device");
  dc::AttnArgs a{};
  a.q = (const uint16_t*)x.q;
  a.q_t = x.q_token_stride;
  a.q_h = x.q_head_stride;
  a.k = (const uint16_t*)x.k;
  a.v = (const uint16_t*)x.v;
  a.k_t = x.k_token_stride;
  a.k_y = x.k_head_stride;
  a.v_t = x.v_token_stride;
  a.v_y = x.v_head_stride;
  a.out = (uint16_t*)x.out;
  a.o_t = (long long)p->q_heads * p->head_dim;
  a.o_h = p->head_dim;
  a.lse = x.lse;
  a.G = p->q_heads / p->kv_heads;
  a.kvh = p->kv_heads;
  a.scale = x.scale;
  a.c = (float)(1.4426950408889634 * x.scale);
  a.items = p->items;
  a.first = p->first;
  a.merges = p->merges;
  a.n_items = p->n_items;
  a.n_merges = p->n_merges;
  a.prows = p->prows;
  a.part = (float*)x.workspace;
  a.part_rows = (long long)p->n_slots * p->prows;
  a.out_len = p->q_tokens * a.o_t;
  a.part_ml = (float2*)((float*)x.workspace + (size_t)p->n_slots * p->prows * p->head_dim);
  a.wait_ns = dc::att_wait_ns((long long)p->item_tiles * dc::kAttTok);
  a.status = p->status;
  a.dbg = p->status + 8;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool bf = x.dtype == DC_BF16;
  const int D = p->head_dim;
  dc::AttMaps m;
  // (no keys at all: every row's result is 0, and the maps of keys are not used)
  const bool none = p->k_tokens == 0;
  if (!dc::att_map_q(&m.q, bf, a, D, p->q_tokens, 1) ||
      !dc::att_map_kv(&m.k, bf, none ? x.q : x.k, D, p->kv_heads, none ? D : a.k_y, none ? 1 : p->k_tokens, none ? D : a.k_t) ||
      !dc::att_map_kv(&m.v, bf, none ? x.q : x.v, D, p->kv_heads, none ? D : a.v_y, none ? 1 : p->k_tokens, none ? D : a.v_t))
    return prompt_fail(DC_ERR_INVALID_ARG, "cuTensorMapEncodeTiled rejected the layout of q, k or v");
  m.kd = m.k;
  m.vd = m.v;
  if (D == 128)
    e = bf ? dc::launch_attend<dc::TypeBf16, 128, false>(m, a, p->grid, s)
           : dc::launch_attend<dc::TypeHalf, 128, false>(m, a, p->grid, s);
  else
    e = bf ? dc::launch_attend<dc::TypeBf16, 64, false>(m, a, p->grid, s)
           : dc::launch_attend<dc::TypeHalf, 64, false>(m, a, p->grid, s);
  if (e != cudaSuccess) return prompt_cuda(e, "launch");
  return DC_OK;
}

dc_status dc_prompt_workspace(const dc_prompt_plan* p, size_t* bytes) {
  if (!p || p->magic != dc::kPlanMagic || !bytes) return prompt_fail(DC_ERR_INVALID_ARG, "not a plan");
  *bytes = p->workspace();
  return DC_OK;
}

dc_status dc_prompt_check(const dc_prompt_plan* p, void* stream) {
  if (!p || p->magic != dc::kPlanMagic) return prompt_fail(DC_ERR_INVALID_ARG, "not a plan");
  cudaError_t e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
  unsigned st[16] = {};
  if (e == cudaSuccess) e = cudaMemcpy(st, p->status, sizeof st, cudaMemcpyDeviceToHost);
  if (e != cudaSuccess) return prompt_cuda(e, "check");
  if (st[0]) {
    char buf[160];
    std::snprintf(buf, sizeof buf, "kernel status word 0x%x (first wait timeout: site %u block %u parity %u info 0x%x)", st[0],
                  st[9], st[10], st[11], st[12]);
    return prompt_fail(DC_ERR_DEVICE, buf);
  }
  return DC_OK;
}

}  // extern "C"
