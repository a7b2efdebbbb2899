// dc_prompt.h -- launchers and tensor maps of the attention kernels of prompts and
// drafted trees.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include "dc_attend.cuh"

namespace dc {

// A map of 16-bit elements with 128-byte swizzle, box 64 dims wide: `dims` sizes (the
// first is the head's dims) and `strides` in elements from the second dimension on. False where
// the driver rejects it. A stride of a dimension of one says nothing and may be anything.
bool att_map(CUtensorMap* m, bool bf16, const void* base, int rank, const long long* dims, const long long* strides,
             const int* box);
// Queries: [lb][token][kvh * G heads][D], boxes of 128 / G tokens of one KV head.
bool att_map_q(CUtensorMap* m, bool bf16, const AttnArgs& a, int D, long long tokens, long long lbs);
// Keys or values: [y][token][D], boxes of 128 tokens.
bool att_map_kv(CUtensorMap* m, bool bf16, const void* base, int D, long long ys, long long y_stride, long long tokens,
                long long t_stride);

// Attention of drafted trees over the rows of a cache (AttnArgs' tree fields), D 64 or
// 128. tree_plan sets how the work is divided, and returns the partial results' slots (-1: too
// much work to count); launch_tree needs a.part and a.part_ml for them. *why on a map that the
// driver rejects.
long long tree_plan(AttnArgs* a, int D, int num_sms);
cudaError_t launch_tree(const AttnArgs& a, int D, cudaStream_t s, const char** why);

}  // namespace dc
