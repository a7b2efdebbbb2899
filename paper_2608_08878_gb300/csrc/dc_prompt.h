// dc_prompt.h -- launchers of the attention kernels of prompts and drafted trees.
#pragma once

#include <cuda_runtime.h>

#include "dc_attend.cuh"

namespace dc {

// Attention of drafted trees over the rows of a cache (AttnArgs' tree fields); D 64 or 128.
cudaError_t launch_tree(const AttnArgs& a, int D, int num_sms, cudaStream_t s);

}  // namespace dc
