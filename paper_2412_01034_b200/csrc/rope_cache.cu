// Rotary position embedding of the queries and keys of new tokens, and the append of their keys and values to a paged
// cache (the writer of the cache that the attention of attn_paged.cu reads).
//   qkv [T][(H + 2 Hk) D] bf16, the output of one fused projection: H query heads, Hk key heads, Hk value heads
//   token t of request b has cache position p = kv_len[b] - q_len[b] + (t - cu_q[b])
//   (a, b) = (x[i], x[i + D/2]) -> (a cos - b sin, b cos + a sin) with the table's row p, for query and key heads
//   caches [num_pages][Hk][page_size][D]; position p sits in page block_table[b][p / page_size], slot p % page_size
// One pass, memory bound.  A thread turns 8 pairs (two 16-byte loads and stores) or copies 16 values; what it reads is asked
// for before the request, its page and its angles are looked up (4200 tokens of 32 + 32 + 32 heads: 45.3 us = 6.0 TB/s, 91 %
// of the copy rate; with the look-up first 51 us; 32 single tokens 3.6 us).  The angles come from a table: a sine of position *
// frequency formed in fp32 would be off by up to position * 2^-24 radians.
#include "layer_common.cuh"

namespace qil {

namespace {

constexpr int kThreads = 256;

template <int kDim>
__global__ void __launch_bounds__(kThreads) rope_append_kernel(const __nv_bfloat16* __restrict__ qkv, const float* __restrict__ cos_sin,
                                                               __nv_bfloat16* __restrict__ q_out, __nv_bfloat16* __restrict__ k_cache,
                                                               __nv_bfloat16* __restrict__ v_cache, PagedCache c, int max_pos, int pieces) {
    constexpr int kHalf = kDim / 2, kPer = kHalf / 8;   // pieces of 8 pairs per head, and as many of 16 values
    const int t = blockIdx.x, H = c.num_heads, Hk = c.num_kv_heads;
    wait_for_earlier_kernels();
    const int i = blockIdx.y * kThreads + threadIdx.x, piece = min(i, pieces - 1), head = piece / kPer, o = (piece % kPer) * 8;
    const bool turn = head < H + Hk;
    const __nv_bfloat16* src = qkv + ((size_t)t * (H + 2 * Hk) + head) * kDim + (turn ? o : 2 * o);
    const uint4 first = *reinterpret_cast<const uint4*>(src), second = *reinterpret_cast<const uint4*>(src + (turn ? kHalf : 8));
    int seq = 0, lo = 0, hi = 0, kv = 0;
    const bool held = request_at_row(c.cu_q, c.kv_len, c.num_seqs, c.total_q, t, seq, lo, hi, kv);
    const int pos = kv - (hi - lo) + (t - lo);
    const bool known = held && t >= lo && pos >= 0 && pos < max_pos;
    if (i >= pieces) return;
    __nv_bfloat16* dst = nullptr;
    if (head < H) {
        dst = q_out + ((size_t)t * H + head) * kDim;
    } else if (known) {
        const int page_at = pos / c.page_size, slot = pos - page_at * c.page_size;
        const int page = page_at < c.max_pages ? __ldg(c.block_table + (size_t)seq * c.max_pages + page_at) : -1;
        if (page >= 0 && page < c.num_pages)
            dst = (turn ? k_cache : v_cache) + (((size_t)page * Hk + (head - H - (turn ? 0 : Hk))) * c.page_size + slot) * kDim;
    }
    if (!dst) return;
    if (!turn) {
        *reinterpret_cast<uint4*>(dst + 2 * o) = first;
        *reinterpret_cast<uint4*>(dst + 2 * o + 8) = second;
        return;
    }
    float a[8], b[8], u[8], v[8];
    unpack8(first, a);
    unpack8(second, b);
    const float4* cs = reinterpret_cast<const float4*>(cos_sin + (size_t)(known ? pos : 0) * kDim + o);
    const float4 co[2] = {__ldg(cs), __ldg(cs + 1)}, si[2] = {__ldg(cs + kHalf / 4), __ldg(cs + kHalf / 4 + 1)};
    const float cv[8] = {co[0].x, co[0].y, co[0].z, co[0].w, co[1].x, co[1].y, co[1].z, co[1].w};
    const float sv[8] = {si[0].x, si[0].y, si[0].z, si[0].w, si[1].x, si[1].y, si[1].z, si[1].w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        u[e] = known ? a[e] * cv[e] - b[e] * sv[e] : 0.f;
        v[e] = known ? b[e] * cv[e] + a[e] * sv[e] : 0.f;
    }
    *reinterpret_cast<uint4*>(dst + o) = pack8(u);
    *reinterpret_cast<uint4*>(dst + o + kHalf) = pack8(v);
}

}  // namespace

qil_status launch_rope_append(const void* qkv, const float* cos_sin, void* q_out, void* k_cache, void* v_cache, const PagedCache& c,
                              int max_pos, cudaStream_t st) {
    const int pieces = (c.num_heads + 2 * c.num_kv_heads) * (c.head_dim / 16);
    const dim3 grid((unsigned)c.total_q, (unsigned)((pieces + kThreads - 1) / kThreads));
    auto go = [&](auto kernel) {
        return launch_early(kernel, grid, kThreads, 0, st, reinterpret_cast<const __nv_bfloat16*>(qkv), cos_sin,
                            reinterpret_cast<__nv_bfloat16*>(q_out), reinterpret_cast<__nv_bfloat16*>(k_cache),
                            reinterpret_cast<__nv_bfloat16*>(v_cache), c, max_pos, pieces);
    };
    return c.head_dim == 128 ? go(rope_append_kernel<128>) : go(rope_append_kernel<64>);
}

}  // namespace qil
