// dc_paged.h -- what the parts of the paged cache share: the layout of a layer, and
// the launchers behind dc_paged_*.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <vector>

#include "../../include/distillcache.h"
#include "dc_attend.cuh"
#include "dc_common.cuh"

namespace dc {

constexpr unsigned kStatusBadPage = 8u;   // a page number or position outside the cache
constexpr unsigned kStatusBadStart = 16u;  // starts out of order

// One layer. Element (page, head, slot, dim) of K and V is at ((page * kvh + head) * page_size + slot) * D + dim.
struct PagedView {
  uint16_t *k, *v, *bounds;
  int pages, page, log;  // pages of the pool; tokens of a page, and its logarithm
  int kvh, qh, G;
  unsigned* status;
  unsigned* dbg;
  __host__ __device__ long long pages_end(int D) const { return (long long)pages * kvh * page * D; }
};

// The shared prefixes of a batch. Attention over them is planned on the host: units (group, block of its sequences, KV
// head) of query rows, cut into pieces (AttnItem) of equal time for the CTAs, each with a place for its result.
struct SharedView {
  int groups, seqs;     // seqs: of all groups
  const int *group, *prefix;  // [seqs]: its group, the tokens that it shares
  const int* first;     // [groups + 1]: a group's first sequence
  const int* unit;      // [groups]: a group's first unit
  const int2* runs;     // [units]: first place of a unit's results, and how many
  const struct AttnItem* items;
  const int* cta;       // CTA b takes items [cta[b], cta[b + 1])
  int grid, places, prows, item_tiles;  // prows: rows of a place
};

// Attention of one token a sequence over its own tokens: a unit of work is up to `rows` of a KV head's query heads.
struct PagedAttn {
  PagedView c;
  SharedView sh;
  const uint16_t* q;
  long long q_s, q_h;
  const int *lens, *tables, *selected;
  int layer, S, W, count;
  float scale, c2;  // c2 = scale * log2(e)
  uint16_t* out;
  float* lse;
  float* part;      // [2 grid][rows][D], with shared prefixes then [S kvh blocks][rows][D]: sums of weighted values
  float2* part_ml;  // likewise: the weights' reference, a score, and their sum
  int* line;        // each sequence's first place, all places, the CTAs that took them
  float* pre;       // [places][prows][D]: of the prefixes
  float2* pre_ml;   // likewise
  int rows, grid;
  int blocks;       // units of a sequence and KV head: its query heads in blocks of `rows`
  int whole;        // whether no unit is cut
  long long slots;
};

cudaError_t launch_paged_append(const PagedView& c, int D, int dtype, const dc_paged_append_args& a, int num_sms, cudaStream_t s);
// The tiles of a sequence's unit, at most (by the table's width or the selection).
long long paged_tiles(const PagedAttn& a);
// Bytes of a call's workspace; sets rows, grid, blocks, whole and slots, and the pointers into it.
size_t paged_workspace(PagedAttn* a, int D, int num_sms, char* base);
cudaError_t launch_paged_attend(const PagedAttn& a, int D, int dtype, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t s);

// The plan of attention over shared prefixes; throws bad_alloc.
struct PrefixPlan {
  std::vector<AttnItem> items;
  std::vector<int> cta, unit;
  std::vector<int2> runs;
  int places = 0, prows = 0, item_tiles = 0;
};
PrefixPlan plan_prefixes(const int* sizes, const int* tokens, int n, int kvh, int G, int num_sms);
// k, v: maps of boxes of one page (att_map), 64 dims wide.
cudaError_t launch_prefixes(const PagedAttn& a, int D, int dtype, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t s,
                            const char** why);
cudaError_t launch_paged_select(const PagedView& c, int D, int dtype, const dc_paged_select_args& a, int num_sms, cudaStream_t s);

}  // namespace dc
