// What the two attention kernels over the paged cache share: the packing of query rows, the visible end of a row, the
// workspace.
#pragma once

#include "layer_common.cuh"

namespace qil {

// Query heads that share a key head are packed into the rows of one tile: row r of a request and key head h is new token
// r / G, query head h G + r % G.  Requests of at most kFewRows rows (single tokens, short drafts) run on the kernel that
// splits the cache over the GPU, the others on the tensor-memory kernel.
constexpr int kFewRows = 16, kTileRows = 128, kMostTogether = 8;

struct AttnParams {
    const __nv_bfloat16 *q, *k, *v;
    __nv_bfloat16* out;
    PagedCache c;
    int G;               // query heads of a key head
    float scale_log2;    // scale * log2(e)
    int page_shift;      // log2 of the page size
    int chunk;           // few rows: cached tokens of one block
    int slots;           // few rows: blocks per request and key head at most
    int together;        // few rows: the blocks of a request and key head are one cluster
    int few_rows;        // few rows: rows of a part in the workspace
    int splits;          // many rows: parts of the cache
    int tile_tokens;     // many rows: new tokens of a row tile, kTileRows / G
    int* status;
    int* counters;       // [num_seqs][num_kv_heads] parts written so far, zero between launches
    float *few_parts, *many_parts;
    int both;            // both kernels are launched, many rows first
};

// cached tokens that the table can name
__device__ __forceinline__ int cache_end(const PagedCache& c, int kv_len) { return min(max(kv_len, 0), c.max_pages * c.page_size); }

__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// one of eight bf16 is infinite or NaN
__device__ __forceinline__ bool any_not_finite(uint4 v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    bool any = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) any |= (w[e] & 0x7F800000u) == 0x7F800000u || (w[e] & 0x7F80u) == 0x7F80u;
    return any;
}

qil_status launch_attn_few(const AttnParams& p, cudaStream_t st);
qil_status launch_attn_many(const AttnParams& p, cudaStream_t st);
qil_status launch_attn_many_join(const AttnParams& p, cudaStream_t st);

}  // namespace qil
