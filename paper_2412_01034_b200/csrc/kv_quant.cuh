// The quantised paged cache as the kernels receive it: codes [num_pages][num_kv_heads][page_size][head_dim] of 8 or 4 bits
// (4 bits: code d of a head in 32-bit word d / 8, bits 4 (d % 8)), scales [num_pages][num_kv_heads][page_size] bf16 (4 bits:
// pairs of scale and zero point).
#pragma once

#include "layer_common.cuh"

namespace qil {

struct QuantCache {
    void *k, *v;
    __nv_bfloat16 *ks, *vs;
    int bits;
};

qil_status launch_rope_append_q(const void* qkv, const float* cos_sin, void* q_out, const QuantCache& kvq, const PagedCache& c, int max_pos,
                                cudaStream_t st);
qil_status launch_kv_read_q(const QuantCache& kvq, const PagedCache& c, void* k_out, void* v_out, cudaStream_t st);
size_t attn_paged_q_workspace(int total_q, int num_seqs, int num_heads, int num_kv_heads, int head_dim, int bits, int max_q_len, int max_kv_len);
qil_status launch_attn_paged_q(const void* q, const QuantCache& kvq, void* out, const PagedCache& c, int max_q_len, int max_kv_len, float scale,
                               void* ws, cudaStream_t st);

}  // namespace qil
