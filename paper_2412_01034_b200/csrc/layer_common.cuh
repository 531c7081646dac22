// Device helpers shared by the operators between the linears of a decoder layer (norm, rotary cache writer, attention,
// adapters of many requests).
#pragma once

#include <atomic>

#include "qil_common.cuh"

namespace qil {

__device__ __forceinline__ void unpack8(const uint4 v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}

// Rows [lo, hi) of request b in packed tensors of `total` rows.  The starts are read as they are but never used beyond the
// tensor, so that a wrong array cannot make a kernel leave its buffers.
__device__ __forceinline__ void request_rows(const int* __restrict__ cu, int b, int total, int& lo, int& hi) {
    lo = min(max(__ldg(cu + b), 0), total);
    hi = min(max(__ldg(cu + b + 1), lo), total);
}

// The request that holds packed row t: the number of requests that end at or before it.  All 32 lanes of a warp take part.
__device__ __forceinline__ int request_of_row(const int* __restrict__ cu, int num_seqs, int t) {
    const int lane = threadIdx.x & 31;
    int b = 0;
    for (int base = 0; base < num_seqs; base += 32) {
        const bool before = base + lane < num_seqs && __ldg(cu + base + lane + 1) <= t;
        const unsigned m = __ballot_sync(0xffffffffu, before);
        b += __popc(m);
        if (m != 0xffffffffu) break;
    }
    return b;
}

// The same with what a kernel needs next, in one trip to memory: the request's rows [lo, hi) and its number of cached
// tokens.  False when no request holds the row.
__device__ __forceinline__ bool request_at_row(const int* __restrict__ cu, const int* __restrict__ kv_len, int num_seqs, int total, int t,
                                               int& seq, int& lo, int& hi, int& kv) {
    const int lane = threadIdx.x & 31;
    for (int base = 0; base < num_seqs; base += 32) {
        const int b = min(base + lane, num_seqs - 1);
        const int start = __ldg(cu + b), end = __ldg(cu + b + 1), len = __ldg(kv_len + b);
        const unsigned past = __ballot_sync(0xffffffffu, base + lane < num_seqs && end > t);
        if (past) {
            const int who = __ffs(past) - 1;
            seq = base + who;
            lo = min(max(__shfl_sync(0xffffffffu, start, who), 0), total);
            hi = min(max(__shfl_sync(0xffffffffu, end, who), lo), total);
            kv = __shfl_sync(0xffffffffu, len, who);
            return true;
        }
    }
    return false;
}

// Packed rows are cut into tiles of `rows`, each request on its own (its last tile may be short): the request and the
// first row of tile t, or false when there are fewer tiles.  All 32 lanes of a warp take part and get the same answer.
__device__ __forceinline__ bool find_tile(const int* __restrict__ cu, int num_seqs, int total, int rows, int t, int& seq, int& row0, int& row1) {
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int base = 0; base < num_seqs; base += 32) {
        int lo = 0, hi = 0;
        if (base + lane < num_seqs) request_rows(cu, base + lane, total, lo, hi);
        const int n = (hi - lo + rows - 1) / rows;
        int incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += up;
        }
        const unsigned past = __ballot_sync(0xffffffffu, before + incl > t);
        if (past) {
            const int who = __ffs(past) - 1;
            const int first = before + __shfl_sync(0xffffffffu, incl - n, who);
            const int s_lo = __shfl_sync(0xffffffffu, lo, who), s_hi = __shfl_sync(0xffffffffu, hi, who);
            seq = base + who;
            row0 = s_lo + (t - first) * rows;
            row1 = min(row0 + rows, s_hi);
            return true;
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
    }
    return false;
}

// D[16 x 8] += A[16 x 16] B[16 x 8], bf16 operands, fp32 accumulators
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Lets a kernel use `bytes` of shared memory, once per device (`done` belongs to the kernel).
template <class Kernel>
inline bool allow_smem(Kernel kernel, int bytes, std::atomic<unsigned long long>& done) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return false;
    }
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;
    if (bit && (done.load(std::memory_order_relaxed) & bit)) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
        (void)cudaGetLastError();
        return false;
    }
    done.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

// Every kernel of the layer operators is launched early: it is ready when the kernel before it in the stream ends, which
// takes the gap between two short kernels (2.5 us) out of a chain of them.  A block's first act is to wait until everything
// before is complete and visible.  Inside an operator a first kernel may let the second one's blocks come up beside it once
// its own have done that wait, so that the second only has to wait for the first.  (Between operators that gained nothing:
// blocks that wait take the place of blocks that work.)
__device__ __forceinline__ void wait_for_earlier_kernels() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_kernel_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// An early launch, as described above; in clusters of `cluster` blocks along x.
template <class Kernel, class... Args>
inline qil_status launch_early_clusters(Kernel kernel, unsigned cluster, dim3 grid, int threads, size_t smem, cudaStream_t st, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess) return QIL_OK;
    (void)cudaGetLastError();
    return QIL_ERR_CUDA;
}

template <class Kernel, class... Args>
inline qil_status launch_early(Kernel kernel, dim3 grid, int threads, size_t smem, cudaStream_t st, Args... args) {
    return launch_early_clusters(kernel, 1u, grid, threads, smem, st, args...);
}

// Internal launchers.
bool rmsnorm_supported(int K);
qil_status launch_rmsnorm(const void* x, const void* residual, const void* weight, void* residual_out, void* y, int8_t* qy,
                          float* scales, int M, int K, float eps, cudaStream_t st);

struct PagedCache {   // the paged key / value cache and the requests that use it, as the entry points receive them
    const int *cu_q, *kv_len, *block_table;
    int total_q, num_seqs, num_heads, num_kv_heads, head_dim, page_size, num_pages, max_pages;
};
qil_status launch_rope_append(const void* qkv, const float* cos_sin, void* q_out, void* k_cache, void* v_cache, const PagedCache& c,
                              int max_pos, cudaStream_t st);
size_t attn_paged_workspace(int total_q, int num_seqs, int num_heads, int num_kv_heads, int head_dim, int max_q_len, int max_kv_len);
qil_status launch_attn_paged(const void* q, const void* k_cache, const void* v_cache, void* out, const PagedCache& c, int max_q_len,
                             int max_kv_len, float scale, void* ws, cudaStream_t st);

size_t lora_batch_workspace(int M, int num_seqs, int rank);
qil_status launch_lora_batch_add(const void* x, const void* a, const void* b, const void* y, void* out, const int* cu_q, const int* adapter,
                                 const float* scales, int M, int N, int K, int rank, int num_seqs, int num_adapters, long long ldx,
                                 long long ldy, long long ldo, void* ws, cudaStream_t st);

}  // namespace qil
