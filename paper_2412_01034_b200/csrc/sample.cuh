// The choice of the next token (sample.cu).
#pragma once

#include "layer_common.cuh"

namespace qil {

qil_status launch_sample(const void* logits, qil_dtype type, long long ld, const float* u, const float* temperature, const int* top_k,
                         const float* top_p, const float* min_p, int* out, int B, int V, cudaStream_t st);

}  // namespace qil
