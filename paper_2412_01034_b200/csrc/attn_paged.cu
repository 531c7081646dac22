// Attention of the new tokens of many requests over a paged cache, causal, grouped heads.
//   request b: q_len new tokens (rows cu_q[b] ... cu_q[b+1] of q), kv_len cached tokens with the new ones among them
//   new token i of a request has position p = kv_len - q_len + i and sees the cached tokens j <= p
//   o = sum_j softmax_j(scale q . k_j) v_j;  a token that sees nothing (p < 0) gets zeros
#include "layer_common.cuh"

namespace qil {

namespace {

// One warp per (token, head): the cached tokens one after another, lanes over the head's dimension.
template <int kDim>
__global__ void __launch_bounds__(128) attn_rows_kernel(const __nv_bfloat16* __restrict__ q, const __nv_bfloat16* __restrict__ k_cache,
                                                        const __nv_bfloat16* __restrict__ v_cache, __nv_bfloat16* __restrict__ out,
                                                        PagedCache c, float scale_log2) {
    constexpr int kPer = kDim / 32;
    const int lane = threadIdx.x & 31;
    const long long item = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (item >= (long long)c.total_q * c.num_heads) return;
    const int t = (int)(item / c.num_heads), head = (int)(item % c.num_heads), kvh = head / (c.num_heads / c.num_kv_heads);
    const int seq = request_of_row(c.cu_q, c.num_seqs, t);
    int pos = -1;
    if (seq < c.num_seqs) {
        int lo, hi;
        request_rows(c.cu_q, seq, c.total_q, lo, hi);
        const int kv = min(max(__ldg(c.kv_len + seq), 0), c.max_pages * c.page_size);
        pos = kv - (hi - lo) + (t - lo);
    }
    float qv[kPer], o[kPer], m = -INFINITY, l = 0.f;
    for (int i = 0; i < kPer; ++i) {
        qv[i] = __bfloat162float(q[item * kDim + lane * kPer + i]) * scale_log2;
        o[i] = 0.f;
    }
    for (int j = 0; j <= pos; ++j) {
        const int page = __ldg(c.block_table + (size_t)seq * c.max_pages + j / c.page_size);
        if (page < 0 || page >= c.num_pages) continue;
        const size_t at = (((size_t)page * c.num_kv_heads + kvh) * c.page_size + j % c.page_size) * kDim + lane * kPer;
        float s = 0.f;
        for (int i = 0; i < kPer; ++i) s = fmaf(qv[i], __bfloat162float(k_cache[at + i]), s);
        s = warp_sum(s);
        const float top = fmaxf(m, s), keep = exp2f(m - top), p = exp2f(s - top);
        m = top;
        l = l * keep + p;
        for (int i = 0; i < kPer; ++i) o[i] = fmaf(p, __bfloat162float(v_cache[at + i]), o[i] * keep);
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    for (int i = 0; i < kPer; ++i) out[item * kDim + lane * kPer + i] = __float2bfloat16_rn(o[i] * inv);
}

}  // namespace

size_t attn_paged_workspace(int total_q, int num_seqs, int num_heads, int num_kv_heads, int head_dim, int max_q_len, int max_kv_len) {
    return 16;
}

qil_status launch_attn_paged(const void* q, const void* k_cache, const void* v_cache, void* out, const PagedCache& c, int max_q_len,
                             int max_kv_len, float scale, void* ws, cudaStream_t st) {
    const long long items = (long long)c.total_q * c.num_heads;
    const float s2 = scale * 1.4426950408889634f;
    auto go = [&](auto kernel) {
        kernel<<<(unsigned)((items + 3) / 4), 128, 0, st>>>(
            reinterpret_cast<const __nv_bfloat16*>(q), reinterpret_cast<const __nv_bfloat16*>(k_cache),
            reinterpret_cast<const __nv_bfloat16*>(v_cache), reinterpret_cast<__nv_bfloat16*>(out), c, s2);
    };
    if (c.head_dim == 128) go(attn_rows_kernel<128>);
    else go(attn_rows_kernel<64>);
    return launch_status();
}

}  // namespace qil
