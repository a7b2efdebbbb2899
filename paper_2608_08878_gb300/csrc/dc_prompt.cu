// dc_prompt.cu -- attention of packed prompts (dc_prompt_plan_create,
// dc_prompt_attend): the plan's work items and the C ABI.
#include <algorithm>
#include <cmath>
#include <new>
#include <string>
#include <vector>

#include "../../include/distillcache.h"
#include "dc_prompt.h"

namespace dc {
namespace {

// A block per item, a warp per query row.
template <class T, int D>
__global__ void __launch_bounds__(256) prompt_rows_kernel(AttnArgs a) {
  const AttnItem it = a.items[blockIdx.x];
  const int lane = threadIdx.x & 31, tpt = kAttRows / a.G;
  const int t1 = min(it.tend, it.t0 + (it.alt ? 1 : 2) * tpt);
  for (int r = threadIdx.x / 32; r < (t1 - it.t0) * a.G; r += 8) {
    const int t = it.t0 + r / a.G, head = it.h * a.G + r % a.G, lim = att_limit(it, t);
    float m, l, o[D / 32];
    attend_row<T, D>(a, a.q + t * a.q_t + head * a.q_h, a.k + it.k0 * a.k_t + it.y * a.k_y,
                     a.v + it.k0 * a.v_t + it.y * a.v_y, nullptr, nullptr, 0, lim, nullptr, m, l, o);
    const float inv = lim > 0 ? 1.f / l : 0.f;
    uint32_t* to = reinterpret_cast<uint32_t*>(a.out + t * a.o_t + head * a.o_h) + lane * (D / 64);
#pragma unroll
    for (int e = 0; e < D / 64; ++e) to[e] = T::pack(o[2 * e] * inv, o[2 * e + 1] * inv);
    if (a.lse && lane == 0) a.lse[(long long)t * a.kvh * a.G + head] = lim > 0 ? fmaf(m, a.scale, logf(l)) : -INFINITY;
  }
}

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

}  // namespace
}  // namespace dc

struct dc_prompt_plan {
  unsigned magic = dc::kPlanMagic;
  int device = 0;
  int q_heads = 0, kv_heads = 0, head_dim = 0;
  long long q_tokens = 0, k_tokens = 0;
  int n_items = 0;
  dc::AttnItem* items = nullptr;  // device
};

namespace dc {
namespace {

std::vector<AttnItem> plan_items(const int* q_lens, const int* k_lens, int n, int kvh, int G, bool causal) {
  const int tpt = kAttRows / G;
  std::vector<AttnItem> items;
  long long q0 = 0, k0 = 0;
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
        it.off = causal ? kl - ql + 1 - (int)q0 : kSeesAll;
        const int last = std::min(it.tend, it.t0 + 2 * tpt) - 1;
        it.j0 = 0;
        it.j1 = (att_limit(it, last) + kAttTok - 1) / kAttTok;
        it.slot = -1;
        it.alt = it.tend - it.t0 <= tpt;
        items.push_back(it);
      }
    q0 += ql;
    k0 += kl;
  }
  // the longest first
  std::stable_sort(items.begin(), items.end(), [](const AttnItem& a, const AttnItem& b) { return a.j1 - a.j0 > b.j1 - b.j0; });
  return items;
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
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return prompt_cuda(e, "cudaGetDevice");
  const auto items = dc::plan_items(q_lens, k_lens, n, kv_heads, q_heads / kv_heads, causal != 0);
  dc::AttnItem* d = nullptr;
  if (!items.empty()) {
    e = cudaMalloc(&d, items.size() * sizeof(dc::AttnItem));
    if (e != cudaSuccess) {
      cudaGetLastError();
      return prompt_cuda(e, "plan allocation");
    }
    e = cudaMemcpy(d, items.data(), items.size() * sizeof(dc::AttnItem), cudaMemcpyHostToDevice);
    if (e != cudaSuccess) {
      cudaFree(d);
      return prompt_cuda(e, "plan upload");
    }
  }
  dc_prompt_plan* p = new dc_prompt_plan();
  p->device = dev;
  p->q_heads = q_heads;
  p->kv_heads = kv_heads;
  p->head_dim = head_dim;
  p->q_tokens = qt;
  p->k_tokens = kt;
  p->n_items = (int)items.size();
  p->items = d;
  *out = p;
  return DC_OK;
} catch (const std::bad_alloc&) {
  return prompt_fail(DC_ERR_OOM, "host allocation failed");
}

dc_status dc_prompt_plan_destroy(dc_prompt_plan* p) {
  if (!p) return DC_OK;
  if (p->magic != dc::kPlanMagic) return DC_ERR_INVALID_ARG;
  cudaFree(p->items);
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
  for (long long st : strides)
    if (st < 0 || st % 8 || st >= (1ll << 38)) return prompt_fail(DC_ERR_INVALID_ARG, "strides must be multiples of 8 in [0, 2^38)");
  if (at & 15) return prompt_fail(DC_ERR_INVALID_ARG, "q, k, v and out must be 16-byte aligned");
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
  a.n_items = p->n_items;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool bf = x.dtype == DC_BF16;
  if (p->head_dim == 128) {
    if (bf) dc::prompt_rows_kernel<dc::TypeBf16, 128><<<p->n_items, 256, 0, s>>>(a);
    else dc::prompt_rows_kernel<dc::TypeHalf, 128><<<p->n_items, 256, 0, s>>>(a);
  } else {
    if (bf) dc::prompt_rows_kernel<dc::TypeBf16, 64><<<p->n_items, 256, 0, s>>>(a);
    else dc::prompt_rows_kernel<dc::TypeHalf, 64><<<p->n_items, 256, 0, s>>>(a);
  }
  e = cudaGetLastError();
  if (e != cudaSuccess) return prompt_cuda(e, "launch");
  return DC_OK;
}

}  // extern "C"
