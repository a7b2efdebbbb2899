// dc_tree.cu -- attention of drafted trees over the rows of a cache (dc_tree_attend).
#include "dc_prompt.h"

namespace dc {
namespace {

// A warp per query row.
template <int D>
__global__ void __launch_bounds__(256) tree_rows_kernel(AttnArgs a) {
  const int lane = threadIdx.x & 31, per = a.nodes * a.G;
  for (long long u = (long long)blockIdx.x * 8 + threadIdx.x / 32; u < (long long)a.rows * per; u += (long long)gridDim.x * 8) {
    const int y = (int)(u / per), i = (int)(u % per) / a.G, g = (int)(u % a.G);
    const int lb = y / a.kvh, head = (y % a.kvh) * a.G + g;
    uint32_t w[4];
    const bool used = tree_mask(a.parents + (long long)(lb % a.batch) * a.nodes, i, w);
    float m, l = 1.f, o[D / 32] = {};
    if (used)
      attend_row<TypeBf16, D>(a, a.q + lb * a.q_lb + i * a.q_t + head * a.q_h, a.k + y * a.k_y, a.v + y * a.v_y,
                              a.kd + (long long)y * a.nodes * D, a.vd + (long long)y * a.nodes * D, 0,
                              a.rowlen ? a.rowlen[y] : a.n, w, m, l, o);
    uint32_t* to = reinterpret_cast<uint32_t*>(a.out + lb * a.o_lb + i * a.o_t + head * a.o_h) + lane * (D / 64);
#pragma unroll
    for (int e = 0; e < D / 64; ++e) to[e] = TypeBf16::pack(o[2 * e] / l, o[2 * e + 1] / l);
  }
}

}  // namespace

cudaError_t launch_tree(const AttnArgs& a, int D, int num_sms, cudaStream_t s) {
  if (D == 128) tree_rows_kernel<128><<<num_sms * 8, 256, 0, s>>>(a);
  else tree_rows_kernel<64><<<num_sms * 8, 256, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace dc
