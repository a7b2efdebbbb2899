// dc_tree.cu -- attention of drafted trees over the rows of a cache (dc_tree_attend).
#include <algorithm>

#include "dc_attend_kernel.cuh"
#include "dc_prompt.h"

namespace dc {

long long tree_plan(AttnArgs* a, int D, int num_sms) {
  const int tpt = kAttRows / a->G;
  a->pairs = (a->nodes + 2 * tpt - 1) / (2 * tpt);
  a->prows = a->nodes <= tpt ? a->nodes * a->G : 256;
  const long long items = (long long)a->rows * a->pairs;
  const int tiles = (a->n + kAttTok - 1) / kAttTok + 1;
  // Parts of a row: as few as fill the SMs evenly. In units of a key tile's two products: a
  // part costs its tiles (twice with two tiles of queries) and 5 for its start and end, and the
  // merge of parts 5 more.
  const double unit = a->nodes <= tpt ? 1.0 : 2.0;
  double best = 0;
  a->nsplit = 1;
  for (int ns = 1; ns <= std::min(tiles, 64); ++ns) {
    const double rounds = (double)((items * ns + num_sms - 1) / num_sms);
    const double cost = rounds * ((tiles + ns - 1) / ns * unit + 5.0) + (ns > 1 ? 5.0 : 0.0);
    if (ns == 1 || cost < best) best = cost, a->nsplit = ns;
  }
  a->n_items = (int)(items * a->nsplit);
  a->n_merges = a->nsplit > 1 ? (int)items : 0;
  return a->nsplit > 1 ? items * a->nsplit : 0;
}

cudaError_t launch_tree(const AttnArgs& a, int D, long long tokens, int num_sms, cudaStream_t s, const char** why) {
  AttMaps m;
  const bool ok = att_map_q(&m.q, true, a, D, a.nodes, a.rows / a.kvh) &&
                  att_map_kv(&m.k, true, a.k, D, a.rows, a.k_y, tokens, a.k_t) &&
                  att_map_kv(&m.v, true, a.v, D, a.rows, a.v_y, tokens, a.v_t) &&
                  att_map_kv(&m.kd, true, a.kd, D, a.rows, (long long)a.nodes * D, a.nodes, D) &&
                  att_map_kv(&m.vd, true, a.vd, D, a.rows, (long long)a.nodes * D, a.nodes, D);
  if (!ok) {
    *why = "cuTensorMapEncodeTiled rejected the layout";
    return cudaErrorInvalidValue;
  }
  const int grid = std::min(a.n_items, num_sms);
  return D == 128 ? launch_attend<TypeBf16, 128, true>(m, a, grid, num_sms, s)
                  : launch_attend<TypeBf16, 64, true>(m, a, grid, num_sms, s);
}

}  // namespace dc
