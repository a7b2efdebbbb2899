// dc_paged.cu -- the C ABI of the paged cache: handles, argument checks, tensor maps.
#include <algorithm>
#include <cstdio>
#include <memory>
#include <new>
#include <string>
#include <vector>

#include "../../include/distillcache.h"
#include "dc_device.h"
#include "dc_outside.h"
#include "dc_paged.h"
#include "dc_prompt.h"

namespace dc {
namespace {

thread_local std::string g_paged_error;

dc_status paged_fail(dc_status s, const std::string& msg) {
  g_paged_error = msg;
  return s;
}

dc_status paged_cuda(cudaError_t e, const char* what) {
  cudaGetLastError();
  return paged_fail(e == cudaErrorMemoryAllocation ? DC_ERR_OOM : DC_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

constexpr unsigned kPagedMagic = 0x44435047u, kSharedMagic = 0x44435053u;
constexpr int kMostSeqs = 4096;

bool bad_stride(long long n) { return n < 0 || n % 8 || n >= (1ll << 38); }

}  // namespace
}  // namespace dc

struct dc_paged {
  unsigned magic = dc::kPagedMagic;
  int device = 0, num_sms = 0, layers = 0, D = 0, dtype = 0;
  dc::PagedView view{};  // layer 0
  CUtensorMap k{}, v{};    // boxes of one page's tokens, 64 at most, all dims
  CUtensorMap k1{}, v1{};  // boxes of a whole page, 64 dims
  unsigned* status = nullptr;  // [0] status, [8..15] the first failure
  long long layer_elems() const { return view.pages_end(D); }
  dc::PagedView layer(int i) const {
    dc::PagedView x = view;
    x.k += i * layer_elems();
    x.v += i * layer_elems();
    x.bounds += (long long)i * view.pages * view.kvh * 2 * D;
    return x;
  }
};

struct dc_paged_shared {
  unsigned magic = dc::kSharedMagic;
  int device = 0, G = 0, kvh = 0, page = 0, most = 0;  // most: the longest prefix's tokens
  dc::SharedView view{};
  char* block = nullptr;
};

using dc::paged_cuda;
using dc::paged_fail;

extern "C" {

const char* dc_paged_last_error(void) { return dc::g_paged_error.c_str(); }

dc_status dc_paged_create(const dc_paged_config* cfg, dc_paged** out) try {
  if (!out) return paged_fail(DC_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (!cfg) return paged_fail(DC_ERR_INVALID_ARG, "cfg is NULL");
  const dc_paged_config& c = *cfg;
  if (c.layers < 1 || c.pages < 1) return paged_fail(DC_ERR_INVALID_ARG, "layers and pages must be >= 1");
  if (c.page_size != 16 && c.page_size != 32 && c.page_size != 64 && c.page_size != 128)
    return paged_fail(DC_ERR_INVALID_ARG, "page_size must be 16, 32, 64 or 128");
  if (c.head_dim != 64 && c.head_dim != 128) return paged_fail(DC_ERR_INVALID_ARG, "head_dim must be 64 or 128");
  if (c.kv_heads < 1 || c.kv_heads > 1024 || c.q_heads < c.kv_heads || c.q_heads % c.kv_heads || c.q_heads / c.kv_heads > 128)
    return paged_fail(DC_ERR_INVALID_ARG, "q_heads must be kv_heads (at most 1024) times 1 to 128");
  if (c.dtype != DC_BF16 && c.dtype != DC_FP16) return paged_fail(DC_ERR_INVALID_ARG, "dtype must be DC_BF16 or DC_FP16");
  const long long rows = (long long)c.pages * c.kv_heads * c.page_size;
  if (rows >= (1ll << 31)) return paged_fail(DC_ERR_INVALID_ARG, "pages * kv_heads * page_size must stay below 2^31");
  if (!c.k || !c.v || !c.bounds) return paged_fail(DC_ERR_INVALID_ARG, "NULL pointer");
  if (((uintptr_t)c.k | (uintptr_t)c.v | (uintptr_t)c.bounds) & 15)
    return paged_fail(DC_ERR_INVALID_ARG, "k, v and bounds must be 16-byte aligned");
  auto h = std::make_unique<dc_paged>();
  cudaError_t e = cudaGetDevice(&h->device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->num_sms, cudaDevAttrMultiProcessorCount, h->device);
  if (e != cudaSuccess) return paged_cuda(e, "cudaGetDevice");
  h->layers = c.layers;
  h->D = c.head_dim;
  h->dtype = c.dtype;
  dc::PagedView& p = h->view;
  p.k = static_cast<uint16_t*>(c.k);
  p.v = static_cast<uint16_t*>(c.v);
  p.bounds = static_cast<uint16_t*>(c.bounds);
  p.pages = c.pages;
  p.page = c.page_size;
  p.log = c.page_size == 16 ? 4 : c.page_size == 32 ? 5 : c.page_size == 64 ? 6 : 7;
  p.kvh = c.kv_heads;
  p.qh = c.q_heads;
  p.G = c.q_heads / c.kv_heads;
  // [layer][half of the dims][token of a head in a page][64 dims]
  const int D = c.head_dim, box_rows = c.page_size < 64 ? c.page_size : 64;
  const long long dims[4] = {64, rows, D / 64, c.layers}, strides[3] = {D, 64, rows * D};
  const int box[4] = {64, box_rows, D / 64, 1}, page[4] = {64, c.page_size, 1, 1};
  const bool bf = c.dtype == DC_BF16;
  if (!dc::att_map(&h->k, bf, c.k, 4, dims, strides, box) || !dc::att_map(&h->v, bf, c.v, 4, dims, strides, box) ||
      !dc::att_map(&h->k1, bf, c.k, 4, dims, strides, page) || !dc::att_map(&h->v1, bf, c.v, 4, dims, strides, page))
    return paged_fail(DC_ERR_INVALID_ARG, "cuTensorMapEncodeTiled rejected the layout");
  const dc::OutsideCapture outside;
  e = cudaMalloc(&h->status, 64);
  if (e != cudaSuccess) return paged_cuda(e, "allocation");
  const unsigned zero[16] = {};
  e = dc::upload_now(h->status, zero, sizeof zero);
  if (e != cudaSuccess) {
    cudaFree(h->status);
    return paged_cuda(e, "upload");
  }
  p.status = h->status;
  p.dbg = h->status + 8;
  *out = h.release();
  return DC_OK;
} catch (const std::bad_alloc&) {
  return paged_fail(DC_ERR_OOM, "host allocation failed");
}

dc_status dc_paged_destroy(dc_paged* h) {
  if (!h) return DC_OK;
  if (h->magic != dc::kPagedMagic) return DC_ERR_INVALID_ARG;
  {
    const dc::OutsideCapture outside;
    cudaFree(h->status);
  }
  h->magic = 0;
  delete h;
  return DC_OK;
}

dc_status dc_paged_check(dc_paged* h, void* stream) {
  if (!h || h->magic != dc::kPagedMagic) return paged_fail(DC_ERR_INVALID_ARG, "not a paged cache");
  unsigned st[16] = {};
  bool captures = false;
  const cudaError_t e = dc::fetch_status(static_cast<cudaStream_t>(stream), h->status, st, &captures);
  if (captures) return paged_fail(DC_ERR_INVALID_ARG, "the stream is capturing: its calls have not run yet");
  if (e != cudaSuccess) return paged_cuda(e, "check");
  if (st[0]) {
    char buf[256];
    std::snprintf(buf, sizeof buf, "kernel status word 0x%x:%s%s%s%s", st[0],
                  st[0] & dc::kStatusBadPage ? " a page number outside the pool or a position behind a table;" : "",
                  st[0] & dc::kStatusBadStart ? " starts out of order;" : "",
                  st[0] & dc::kStatusTimeout ? " a wait that ran out of time;" : "",
                  st[0] & (dc::kStatusBadShape | dc::kStatusBounds) ? " an internal check;" : "");
    return paged_fail(DC_ERR_DEVICE, buf);
  }
  return DC_OK;
}

// What every call checks first.
static dc_status paged_begin(const dc_paged* h, int layer, int seqs, int width) {
  if (layer < 0 || layer >= h->layers) return paged_fail(DC_ERR_INVALID_ARG, "layer out of range");
  if (seqs < 0 || seqs > dc::kMostSeqs) return paged_fail(DC_ERR_INVALID_ARG, "at most 4096 sequences");
  if (width < 0 || width > (1 << 24)) return paged_fail(DC_ERR_INVALID_ARG, "table_width must lie in [0, 2^24]");
  return DC_OK;
}
static dc_status paged_device(const dc_paged* h) {
  int dev = -1;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return paged_cuda(e, "cudaGetDevice");
  if (dev != h->device) return paged_fail(DC_ERR_INVALID_ARG, "the cache belongs to another device");
  return DC_OK;
}

dc_status dc_paged_append(dc_paged* h, const dc_paged_append_args* args, void* stream) {
  if (!h || h->magic != dc::kPagedMagic) return paged_fail(DC_ERR_INVALID_ARG, "not a paged cache");
  if (!args) return paged_fail(DC_ERR_INVALID_ARG, "args is NULL");
  const dc_paged_append_args& a = *args;
  if (dc_status st = paged_begin(h, a.layer, a.seqs, a.table_width); st != DC_OK) return st;
  if (a.tokens < 0 || a.tokens > (1ll << 30)) return paged_fail(DC_ERR_INVALID_ARG, "bad token count");
  if (a.rotary_dim < 0 || a.rotary_dim > h->D || a.rotary_dim % 16)
    return paged_fail(DC_ERR_INVALID_ARG, "rotary_dim must be 0 or a multiple of 16 up to head_dim");
  if (a.norm && !(a.eps >= 0.f)) return paged_fail(DC_ERR_INVALID_ARG, "eps must be >= 0");
  if (a.tokens == 0) return DC_OK;
  if (a.seqs == 0) return paged_fail(DC_ERR_INVALID_ARG, "tokens of no sequence");
  if (!a.starts && a.tokens % a.seqs) return paged_fail(DC_ERR_INVALID_ARG, "without starts every sequence has equally many tokens");
  if (!a.lens || !a.tables || !a.k || !a.v || (a.rotary_dim && !a.inv_freq) || (a.q && !a.q_out))
    return paged_fail(DC_ERR_INVALID_ARG, "NULL pointer");
  if (((uintptr_t)a.q | (a.q ? (uintptr_t)a.q_out : 0) | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.k_out) & 15)
    return paged_fail(DC_ERR_INVALID_ARG, "q, k, v and their outputs must be 16-byte aligned");
  if (((uintptr_t)a.starts | (uintptr_t)a.lens | (uintptr_t)a.tables | (uintptr_t)a.inv_freq | (uintptr_t)a.q_weight |
       (uintptr_t)a.k_weight) & 3)
    return paged_fail(DC_ERR_INVALID_ARG, "starts, lens, tables, inv_freq and weights must be 4-byte aligned");
  using dc::bad_stride;
  if (bad_stride(a.k_token_stride) || bad_stride(a.k_head_stride) || bad_stride(a.v_token_stride) || bad_stride(a.v_head_stride) ||
      (a.q && (bad_stride(a.q_token_stride) || bad_stride(a.q_head_stride) || bad_stride(a.q_out_token_stride) ||
               bad_stride(a.q_out_head_stride))) ||
      (a.k_out && (bad_stride(a.k_out_token_stride) || bad_stride(a.k_out_head_stride))))
    return paged_fail(DC_ERR_INVALID_ARG, "strides must be multiples of 8 in [0, 2^38)");
  if (dc_status st = paged_device(h); st != DC_OK) return st;
  const cudaError_t e =
      dc::launch_paged_append(h->layer(a.layer), h->D, h->dtype, a, h->num_sms, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? DC_OK : paged_cuda(e, "launch");
}

dc_status dc_paged_shared_create(dc_paged* h, const int* sizes, const int* tokens, int n, dc_paged_shared** out) try {
  if (!out) return paged_fail(DC_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (!h || h->magic != dc::kPagedMagic) return paged_fail(DC_ERR_INVALID_ARG, "not a paged cache");
  if (!sizes || !tokens || n < 1 || n > dc::kMostSeqs) return paged_fail(DC_ERR_INVALID_ARG, "need 1 to 4096 groups");
  long long seqs = 0;
  for (int g = 0; g < n; ++g) {
    if (sizes[g] < 1) return paged_fail(DC_ERR_INVALID_ARG, "a group has at least one sequence");
    if (tokens[g] < 0 || tokens[g] % h->view.page || tokens[g] > (1 << 30))
      return paged_fail(DC_ERR_INVALID_ARG, "shared tokens must be whole pages, at most 2^30 tokens");
    seqs += sizes[g];
  }
  if (seqs > dc::kMostSeqs) return paged_fail(DC_ERR_INVALID_ARG, "at most 4096 sequences");
  if (dc_status st = paged_device(h); st != DC_OK) return st;
  // (64 bytes a unit; a piece is a unit's, or one of a CTA's first and last)
  const int block = 2 * (dc::kAttRows / h->view.G);
  long long units = 0;
  for (int g = 0; g < n; ++g) units += ((long long)sizes[g] + block - 1) / block * h->view.kvh;
  if (units > (1 << 24)) return paged_fail(DC_ERR_INVALID_ARG, "too much work: at most 2^24 units of 256 query rows");
  const dc::PrefixPlan v = dc::plan_prefixes(sizes, tokens, n, h->view.kvh, h->view.G, h->num_sms);
  std::vector<int> first(1, 0), group, prefix;
  for (int g = 0; g < n; ++g) {
    group.insert(group.end(), (size_t)sizes[g], g);
    prefix.insert(prefix.end(), (size_t)sizes[g], tokens[g]);
    first.push_back((int)group.size());
  }
  auto p = std::make_unique<dc_paged_shared>();
  // one block on the device
  std::vector<char> host;
  auto put = [&](const void* x, size_t bytes) {
    const size_t at = (host.size() + 15) / 16 * 16;
    host.resize(at + bytes);
    if (bytes) std::copy_n((const char*)x, bytes, host.data() + at);
    return at;
  };
  const size_t at_items = put(v.items.data(), v.items.size() * sizeof(dc::AttnItem)), at_cta = put(v.cta.data(), v.cta.size() * 4),
               at_runs = put(v.runs.data(), v.runs.size() * sizeof(int2)), at_unit = put(v.unit.data(), v.unit.size() * 4),
               at_group = put(group.data(), group.size() * 4), at_prefix = put(prefix.data(), prefix.size() * 4),
               at_first = put(first.data(), first.size() * 4);
  p->device = h->device;
  p->G = h->view.G;
  p->kvh = h->view.kvh;
  p->page = h->view.page;
  p->most = *std::max_element(tokens, tokens + n);
  const dc::OutsideCapture outside;
  cudaError_t e = cudaMalloc(&p->block, host.size());
  if (e != cudaSuccess) return paged_cuda(e, "allocation");
  e = dc::upload_now(p->block, host.data(), host.size());
  if (e != cudaSuccess) {
    cudaFree(p->block);
    return paged_cuda(e, "upload");
  }
  dc::SharedView& w = p->view;
  w.groups = n;
  w.seqs = (int)group.size();
  w.group = (const int*)(p->block + at_group);
  w.prefix = (const int*)(p->block + at_prefix);
  w.first = (const int*)(p->block + at_first);
  w.unit = (const int*)(p->block + at_unit);
  w.runs = (const int2*)(p->block + at_runs);
  w.items = (const dc::AttnItem*)(p->block + at_items);
  w.cta = (const int*)(p->block + at_cta);
  w.grid = v.items.empty() ? 0 : (int)v.cta.size() - 1;
  w.places = v.places;
  w.prows = v.prows;
  w.item_tiles = v.item_tiles;
  *out = p.release();
  return DC_OK;
} catch (const std::bad_alloc&) {
  return paged_fail(DC_ERR_OOM, "host allocation failed");
}

dc_status dc_paged_shared_destroy(dc_paged_shared* g) {
  if (!g) return DC_OK;
  if (g->magic != dc::kSharedMagic) return DC_ERR_INVALID_ARG;
  {
    const dc::OutsideCapture outside;
    cudaFree(g->block);
  }
  g->magic = 0;
  delete g;
  return DC_OK;
}

static void paged_attn(const dc_paged* h, int layer, int seqs, int width, int count, const dc_paged_shared* shared,
                       dc::PagedAttn* a) {
  a->c = h->layer(layer);
  a->layer = layer;
  a->S = seqs;
  a->W = width;
  a->count = count;
  if (shared) a->sh = shared->view;
}

static dc_status paged_shared_fits(const dc_paged* h, const dc_paged_shared* g, int seqs) {
  if (!g) return DC_OK;
  if (g->magic != dc::kSharedMagic) return paged_fail(DC_ERR_INVALID_ARG, "not shared prefixes");
  if (g->device != h->device || g->G != h->view.G || g->kvh != h->view.kvh || g->page != h->view.page)
    return paged_fail(DC_ERR_INVALID_ARG, "the shared prefixes belong to a cache of another shape or device");
  if (g->view.seqs > seqs) return paged_fail(DC_ERR_INVALID_ARG, "the shared prefixes have more sequences than the call");
  return DC_OK;
}

dc_status dc_paged_attend_workspace(dc_paged* h, int seqs, int width, int count, const dc_paged_shared* shared, size_t* bytes) {
  if (!h || h->magic != dc::kPagedMagic) return paged_fail(DC_ERR_INVALID_ARG, "not a paged cache");
  if (!bytes) return paged_fail(DC_ERR_INVALID_ARG, "bytes is NULL");
  if (dc_status st = paged_begin(h, 0, seqs, width); st != DC_OK) return st;
  if (count < 0 || count > 65536) return paged_fail(DC_ERR_INVALID_ARG, "count must be 0 to 65536");
  if (dc_status st = paged_shared_fits(h, shared, seqs); st != DC_OK) return st;
  dc::PagedAttn a{};
  paged_attn(h, 0, seqs, width, count, shared, &a);
  *bytes = dc::paged_workspace(&a, h->D, h->num_sms, nullptr);
  return DC_OK;
}

dc_status dc_paged_attend(dc_paged* h, const dc_paged_attend_args* args, void* stream) {
  if (!h || h->magic != dc::kPagedMagic) return paged_fail(DC_ERR_INVALID_ARG, "not a paged cache");
  if (!args) return paged_fail(DC_ERR_INVALID_ARG, "args is NULL");
  const dc_paged_attend_args& x = *args;
  if (dc_status st = paged_begin(h, x.layer, x.seqs, x.table_width); st != DC_OK) return st;
  if (!(x.scale > 0.f) || !(x.scale <= 1e30f)) return paged_fail(DC_ERR_INVALID_ARG, "scale must lie in (0, 1e30]");
  if (x.selected ? x.count < 1 || x.count > 65536 : x.count != 0)
    return paged_fail(DC_ERR_INVALID_ARG, "count must be 1 to 65536 with a selection, 0 without");
  if (x.selected && x.shared) return paged_fail(DC_ERR_INVALID_ARG, "a selection and shared prefixes do not go together");
  if (dc_status st = paged_shared_fits(h, x.shared, x.seqs); st != DC_OK) return st;
  if (x.seqs == 0) return DC_OK;
  if (!x.q || !x.out || !x.lens || (x.table_width && !x.tables)) return paged_fail(DC_ERR_INVALID_ARG, "NULL pointer");
  if (((uintptr_t)x.q | (uintptr_t)x.out) & 15) return paged_fail(DC_ERR_INVALID_ARG, "q and out must be 16-byte aligned");
  if (((uintptr_t)x.lens | (uintptr_t)x.tables | (uintptr_t)x.selected | (uintptr_t)x.lse) & 3)
    return paged_fail(DC_ERR_INVALID_ARG, "lens, tables, selected and lse must be 4-byte aligned");
  if (dc::bad_stride(x.q_seq_stride) || dc::bad_stride(x.q_head_stride))
    return paged_fail(DC_ERR_INVALID_ARG, "strides must be multiples of 8 in [0, 2^38)");
  dc::PagedAttn a{};
  paged_attn(h, x.layer, x.seqs, x.table_width, x.count, x.shared, &a);
  const size_t need = dc::paged_workspace(&a, h->D, h->num_sms, static_cast<char*>(x.workspace));
  if (x.workspace_bytes < need || (need && (!x.workspace || (uintptr_t)x.workspace & 15)))
    return paged_fail(DC_ERR_INVALID_ARG, "the workspace must hold dc_paged_attend_workspace bytes, 16-byte aligned");
  // (places of the line are ints)
  if ((long long)x.seqs * a.blocks * h->view.kvh * (dc::paged_tiles(a) + 8) >= (1ll << 31))
    return paged_fail(DC_ERR_INVALID_ARG, "too much work: 2^31 tiles of 64 tokens or more");
  if (a.slots * a.rows >= (1ll << 31)) return paged_fail(DC_ERR_INVALID_ARG, "too many rows of partial results");
  if (dc_status st = paged_device(h); st != DC_OK) return st;
  a.q = static_cast<const uint16_t*>(x.q);
  a.q_s = x.q_seq_stride;
  a.q_h = x.q_head_stride;
  a.lens = x.lens;
  a.tables = x.tables;
  a.selected = x.selected;
  a.scale = x.scale;
  a.c2 = (float)(1.4426950408889634 * x.scale);
  a.out = static_cast<uint16_t*>(x.out);
  a.lse = x.lse;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (a.sh.grid) {
    // (the prefixes' kernel reads a group's table row as far as the prefix goes)
    if ((long long)x.table_width * h->view.page < x.shared->most)
      return paged_fail(DC_ERR_INVALID_ARG, "a shared prefix is longer than the tables are wide");
    const char* why = nullptr;
    e = dc::launch_prefixes(a, h->D, h->dtype, h->k1, h->v1, s, &why);
    if (why) return paged_fail(DC_ERR_INVALID_ARG, why);
  }
  if (e == cudaSuccess) e = dc::launch_paged_attend(a, h->D, h->dtype, h->k, h->v, s);
  return e == cudaSuccess ? DC_OK : paged_cuda(e, "launch");
}

dc_status dc_paged_select(dc_paged* h, const dc_paged_select_args* args, void* stream) {
  if (!h || h->magic != dc::kPagedMagic) return paged_fail(DC_ERR_INVALID_ARG, "not a paged cache");
  if (!args) return paged_fail(DC_ERR_INVALID_ARG, "args is NULL");
  const dc_paged_select_args& x = *args;
  if (dc_status st = paged_begin(h, x.layer, x.seqs, x.table_width); st != DC_OK) return st;
  if (x.count < 1 || x.count > 65536) return paged_fail(DC_ERR_INVALID_ARG, "count must be 1 to 65536");
  if (x.keep_first < 0 || x.keep_last < 0 || (long long)x.keep_first + x.keep_last > x.count)
    return paged_fail(DC_ERR_INVALID_ARG, "keep_first and keep_last must be >= 0 and at most count together");
  if (x.seqs == 0) return DC_OK;
  if (!x.q || !x.out || !x.lens || (x.table_width && !x.tables)) return paged_fail(DC_ERR_INVALID_ARG, "NULL pointer");
  if ((uintptr_t)x.q & 15) return paged_fail(DC_ERR_INVALID_ARG, "q must be 16-byte aligned");
  if (((uintptr_t)x.lens | (uintptr_t)x.tables | (uintptr_t)x.out) & 3)
    return paged_fail(DC_ERR_INVALID_ARG, "lens, tables and out must be 4-byte aligned");
  if (dc::bad_stride(x.q_seq_stride) || dc::bad_stride(x.q_head_stride))
    return paged_fail(DC_ERR_INVALID_ARG, "strides must be multiples of 8 in [0, 2^38)");
  const size_t need = 4ull * x.seqs * h->view.kvh * x.table_width;
  if (x.workspace_bytes < need || (need && (!x.workspace || (uintptr_t)x.workspace & 15)))
    return paged_fail(DC_ERR_INVALID_ARG, "the workspace must hold 4 * seqs * kv_heads * table_width bytes, 16-byte aligned");
  if (dc_status st = paged_device(h); st != DC_OK) return st;
  const cudaError_t e = dc::launch_paged_select(h->layer(x.layer), h->D, h->dtype, x, h->num_sms, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? DC_OK : paged_cuda(e, "launch");
}

}  // extern "C"
