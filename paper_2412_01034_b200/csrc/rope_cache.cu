// Rotary position embedding of the queries and keys of new tokens, and the append of their keys and values to a paged
// cache (the writer of the cache that the attention of attn_paged.cu reads).
//   qkv [T][(H + 2 Hk) D] bf16, the output of one fused projection: H query heads, Hk key heads, Hk value heads
//   token t of request b has cache position p = kv_len[b] - q_len[b] + (t - cu_q[b])
//   (a, b) = (x[i], x[i + D/2]) -> (a cos - b sin, b cos + a sin) with the table's row p, for query and key heads
//   caches [num_pages][Hk][page_size][D]; position p sits in page block_table[b][p / page_size], slot p % page_size
// One pass, memory bound.  A thread turns 8 pairs (two 16-byte loads and stores) or copies 8 values.  The angles come from a
// table: a sine of position * frequency formed in fp32 would be off by up to position * 2^-24 radians.
#include "layer_common.cuh"

namespace qil {

namespace {

__global__ void __launch_bounds__(256) rope_append_kernel(const __nv_bfloat16* __restrict__ qkv, const float* __restrict__ cos_sin,
                                                          __nv_bfloat16* __restrict__ q_out, __nv_bfloat16* __restrict__ k_cache,
                                                          __nv_bfloat16* __restrict__ v_cache, PagedCache c, int max_pos, int pieces) {
    const int t = blockIdx.x;
    const int seq = request_of_row(c.cu_q, c.num_seqs, t);
    int pos = -1;
    if (seq < c.num_seqs) {
        int lo, hi;
        request_rows(c.cu_q, seq, c.total_q, lo, hi);
        pos = __ldg(c.kv_len + seq) - (hi - lo) + (t - lo);
    }
    const int D = c.head_dim, half = D / 2, H = c.num_heads, Hk = c.num_kv_heads;
    const bool known = pos >= 0 && pos < max_pos;
    const int page_at = known ? pos / c.page_size : 0, slot = known ? pos - page_at * c.page_size : 0;
    int page = -1;
    if (known && page_at < c.max_pages) page = __ldg(c.block_table + (size_t)seq * c.max_pages + page_at);
    const bool store = page >= 0 && page < c.num_pages;
    const __nv_bfloat16* src = qkv + (size_t)t * (H + 2 * Hk) * D;
    const int turned = (H + Hk) * (half / 8);   // pieces of 8 pairs, then pieces of 16 values
    for (int i = blockIdx.y * blockDim.x + threadIdx.x; i < pieces; i += gridDim.y * blockDim.x) {
        if (i < turned) {
            const int head = i / (half / 8), o = (i - head * (half / 8)) * 8;
            float a[8], b[8], u[8], v[8];
            unpack8(*reinterpret_cast<const uint4*>(src + head * D + o), a);
            unpack8(*reinterpret_cast<const uint4*>(src + head * D + o + half), b);
            if (known) {
                const float* cs = cos_sin + (size_t)pos * D + o;
#pragma unroll
                for (int j = 0; j < 8; j += 4) {
                    const float4 co = __ldg(reinterpret_cast<const float4*>(cs + j)), si = __ldg(reinterpret_cast<const float4*>(cs + half + j));
                    const float cv[4] = {co.x, co.y, co.z, co.w}, sv[4] = {si.x, si.y, si.z, si.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        u[j + e] = a[j + e] * cv[e] - b[j + e] * sv[e];
                        v[j + e] = b[j + e] * cv[e] + a[j + e] * sv[e];
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] = v[j] = 0.f;
            }
            __nv_bfloat16* dst = nullptr;
            if (head < H) dst = q_out + ((size_t)t * H + head) * D;
            else if (store) dst = k_cache + (((size_t)page * Hk + head - H) * c.page_size + slot) * D;
            if (dst) {
                *reinterpret_cast<uint4*>(dst + o) = pack8(u);
                *reinterpret_cast<uint4*>(dst + o + half) = pack8(v);
            }
        } else if (store) {
            const int e = (i - turned) * 16, head = e / D, o = e - head * D;
            const uint4* from = reinterpret_cast<const uint4*>(src + (H + Hk) * D + e);
            uint4* to = reinterpret_cast<uint4*>(v_cache + (((size_t)page * Hk + head) * c.page_size + slot) * D + o);
            to[0] = from[0];
            to[1] = from[1];
        }
    }
}

}  // namespace

qil_status launch_rope_append(const void* qkv, const float* cos_sin, void* q_out, void* k_cache, void* v_cache, const PagedCache& c,
                              int max_pos, cudaStream_t st) {
    const int pieces = (c.num_heads + 2 * c.num_kv_heads) * (c.head_dim / 16);
    const unsigned per_token = (unsigned)((pieces + 255) / 256);
    rope_append_kernel<<<dim3((unsigned)c.total_q, per_token), 256, 0, st>>>(
        reinterpret_cast<const __nv_bfloat16*>(qkv), cos_sin, reinterpret_cast<__nv_bfloat16*>(q_out), reinterpret_cast<__nv_bfloat16*>(k_cache),
        reinterpret_cast<__nv_bfloat16*>(v_cache), c, max_pos, pieces);
    return launch_status();
}

}  // namespace qil
