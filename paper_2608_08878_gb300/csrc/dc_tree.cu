// dc_tree.cu -- attention of drafted trees over the rows of a cache (dc_tree_attend).
#include <algorithm>

#include "dc_attend_kernel.cuh"
#include "dc_prompt.h"

namespace dc {

long long tree_plan(AttnArgs* a, int D, int num_sms) {
  const int tpt = kAttRows / a->G;
  a->pairs = (a->nodes + 2 * tpt - 1) / (2 * tpt);
  a->prows = a->nodes <= tpt ? a->nodes * a->G : 256;
  a->n_items = a->rows * a->pairs;
  a->tiles = (a->n + kAttTok - 1) / kAttTok + 1;
  const long long total = (long long)a->n_items * a->tiles;  // (8 million at most in this GPU's memory)
  if (total >= 1ll << 30) return -1;
  // CTAs: every SM an equal share of a line's key tiles, but at least 2 tiles; or, of few items,
  // one each, where the items are so short that parts would not pay for the merge (about 6 tiles).
  a->line = a->rows * a->tiles;
  a->ctas = std::min(num_sms / a->pairs, std::max(1, a->line / 2));
  if (a->n_items <= num_sms && (a->tiles <= 8 || a->n_items == num_sms)) a->ctas = a->rows;
  // More rows than SMs, short ones of one query tile: two whole rows an item, so that nothing is joined and
  // each half has its own chain of steps. Trees of 8 nodes, one row an item -> two, us: 256 rows x 410 tokens
  // of 128 dims 28 -> 16, 4096 x 410 206 -> 185, 4096 x 640 232 -> 235, 4096 x 1000 331 -> 342; of 64 dims 4096 x 410
  // 193 -> 133, 4096 x 1000 248 -> 208. Long rows read at the same rate either way, and parts of equal size
  // balance better than whole rows.
  a->two = a->rows > num_sms && a->nodes <= tpt && !a->rowlen && a->tiles * D <= 640;
  int longest = a->tiles;  // key tiles of an item
  if (a->two) {
    a->tiles = 1;  // (a place is an item)
    a->line = (a->rows + 1) / 2;
    a->ctas = std::min(num_sms, a->line);
  }
  a->per = a->line / a->ctas;
  a->extra = a->line % a->ctas;
  if (!a->two) longest = std::min(longest, a->per + (a->extra ? 1 : 0));
  a->wait_ns = att_wait_ns((long long)longest * kAttTok);
  const int grid = a->grid = a->ctas * a->pairs;
  bool cut = false;
  for (int b = 1; b < grid && !cut; ++b) cut = tree_from(*a, b) % a->tiles != 0;
  a->n_merges = cut ? grid - 1 : 0;
  return cut ? 2ll * grid : 0;
}

cudaError_t launch_tree(const AttnArgs& a, int D, cudaStream_t s, const char** why) {
  AttMaps m;
  const long long tokens = std::max(1, a.n);  // (slots beyond are not read: their places are filled with zeros)
  const bool ok = att_map_q(&m.q, true, a, D, a.nodes, a.rows / a.kvh) &&
                  att_map_kv(&m.k, true, a.k, D, a.rows, a.k_y, tokens, a.k_t) &&
                  att_map_kv(&m.v, true, a.v, D, a.rows, a.v_y, tokens, a.v_t) &&
                  att_map_kv(&m.kd, true, a.kd, D, a.rows, (long long)a.nodes * D, a.nodes, D) &&
                  att_map_kv(&m.vd, true, a.vd, D, a.rows, (long long)a.nodes * D, a.nodes, D);
  if (!ok) {
    *why = "cuTensorMapEncodeTiled rejected the layout";
    return cudaErrorInvalidValue;
  }
  return D == 128 ? launch_attend<TypeBf16, 128, true>(m, a, a.grid, s)
                  : launch_attend<TypeBf16, 64, true>(m, a, a.grid, s);
}

}  // namespace dc
