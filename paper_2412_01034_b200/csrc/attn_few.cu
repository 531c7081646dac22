// Attention over the paged cache for requests with few query rows (new tokens x heads of a group <= 16): single tokens and
// short drafts.  Memory bound: every cached key and value of a request is read once per key head, 4 D bytes a token, and
// the query rows are one 16-row operand.
// Measured: 32 requests of up to 4099 tokens, 32 key heads of 128 (1.38 GB): 213 us from memory = 6.45 TB/s, 98 % of the copy
// rate.  48 requests of up to 300 tokens: 32 us against 23 at the copy rate; one token over 287: 5.1 us: there a block's way
// to its first tile (lengths, page, keys: three trips to memory) is what counts.
//
// A block takes `chunk` cached tokens of one request and key head; its four warps take tiles of 16 tokens in turn and are
// independent of one another: each has its own ring of tiles in shared memory (cp.async, 16-byte pieces, the pieces of a
// row permuted by row % 8 so that ldmatrix reads every bank once), its own running maximum and sum, and its own
// accumulators, so that the loop has no block-wide barrier.  S = Q K^T and O += P V run on mma.sync 16 x 8 x 16: the
// tensor pipe is idle most of the time here and the multiply-adds of up to 16 rows cost the same as those of one.
// A page holds a multiple of 16 tokens, so a tile lies in one page.  Tokens behind the last one arrive as zeros (cp.async
// with a source size of zero), so that whatever the page holds there never meets a weight of zero.
// Of several new tokens the earlier ones must not see the later ones' values: tiles that hold such values are looked through,
// and those with an infinity or a NaN are added token by token.
// The warps' results are joined in shared memory.  Where a request has several blocks, up to eight of them in a launch of
// one round are a cluster and join their results through one another's shared memory, each a share of the outputs;
// otherwise each writes its part (fp32, with maximum and sum) to the workspace, and the block that counts itself in last
// adds the parts.  Either way in the order of the blocks.
#include "attn_paged.cuh"

namespace qil {

namespace {

constexpr int kWarps = 4, kTile = 16;

template <int kDim>
struct FewShape {
    static constexpr int kTileBytes = kTile * kDim * 2;
    static constexpr int kStages = 3 * (128 / kDim);   // 96 KB a block, two blocks an SM
    static constexpr int kWarpBytes = kStages * 2 * kTileBytes;
    static constexpr int kSmem = kWarps * kWarpBytes;
    static_assert((kWarps + 1) * kTile * kDim * 4 <= kSmem, "the warps' results and the block's fit where the rings were");
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float2 lds_pair(uint32_t addr) {   // two bf16
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// a value at this address of another block's shared memory
__device__ __forceinline__ float ld_block(uint32_t addr, int block) {
    uint32_t there;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(block));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(there) : "memory");
    return v;
}
__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
    return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
}
__device__ __forceinline__ float quad_sum(float v) {
    v += __shfl_xor_sync(0xffffffffu, v, 1);
    return v + __shfl_xor_sync(0xffffffffu, v, 2);
}

// kTogether: the blocks of a request and key head are one cluster.
template <int kDim, bool kTogether>
__global__ void __launch_bounds__(32 * kWarps) attn_few_kernel(const AttnParams p) {
    using Shape = FewShape<kDim>;
    constexpr int kStages = Shape::kStages, kTileBytes = Shape::kTileBytes, kPieces = kDim / 8;   // 16-byte pieces of a row
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ float s_m[kWarps][16], s_l[kWarps][16];
    __shared__ float s_scale[2][16];
    __shared__ int s_last;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    const int split = blockIdx.x, kvh = blockIdx.y, seq = blockIdx.z, G = p.G, H = p.c.num_heads;
    // Behind the kernel for many rows, whose blocks have all seen the end of what came before, nothing is waited for: the two
    // run side by side.  But what comes after this launch may need both, so one more block lasts until that kernel ends.
    if (!p.both) wait_for_earlier_kernels();
    if (seq == p.c.num_seqs) {
        if (split == 0 && kvh == 0) wait_for_earlier_kernels();
        return;
    }
    const int begin = split * p.chunk;
    const int* table = p.c.block_table + (size_t)seq * p.c.max_pages;
    // (the first tile's page and the length are on the way with the starts, not after them)
    const int kv = __ldg(p.c.kv_len + seq);
    int page = __ldg(table + min((begin + (int)(threadIdx.x >> 5) * kTile) >> p.page_shift, p.c.max_pages - 1));
    int row0, row1;
    request_rows(p.c.cu_q, seq, p.c.total_q, row0, row1);
    const int q_len = row1 - row0;
    if (q_len <= 0 || q_len * (long long)G > kFewRows) return;
    const int rows = q_len * G, end = cache_end(p.c, kv), first_pos = kv - q_len;
    // A part in the workspace has room for the rows of max_q_len tokens: a request with more of them (the bound was wrong) is
    // left out, it would write over its neighbours' parts and past the workspace.
    if (!kTogether && p.slots > 1 && rows > p.few_rows) return;
    const int parts = max(1, min((end + p.chunk - 1) / p.chunk, p.slots));
    const bool idle = split >= parts;   // (more blocks than the request's tokens need)
    if (idle && !kTogether) return;
    const int stop = idle ? begin : split + 1 == parts ? end : min(begin + p.chunk, end);
    const int tiles = (stop - begin + kTile - 1) / kTile;

    // visible tokens of this lane's two rows
    int see[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) see[h] = g + 8 * h < rows ? min(first_pos + (g + 8 * h) / G + 1, end) : 0;
    const int all_see = min(first_pos + 1, end);   // every row sees what the first new token sees

    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * Shape::kWarpBytes;
    auto page_of = [&](int i) -> int {   // page of tile i (of the last tile where there is none)
        return __ldg(table + (min(begin + i * kTile, stop - 1) >> p.page_shift));
    };
    auto fetch = [&](int i, int stage, int page) {
        const int tok = begin + i * kTile;
        const bool there = page >= 0 && page < p.c.num_pages;
        const size_t at = there ? (((size_t)page * p.c.num_kv_heads + kvh) * p.c.page_size + (tok & (p.c.page_size - 1))) * kDim : 0;
        const uint32_t dst = ring + stage * 2 * kTileBytes;
#pragma unroll
        for (int j = 0; j < kTile * kPieces / 32; ++j) {
            const int piece = j * 32 + lane, r = piece / kPieces, o = piece % kPieces;
            const uint32_t to = dst + r * (kDim * 2) + ((o & ~7) | ((o ^ r) & 7)) * 16;
            const uint32_t bytes = there && tok + r < stop ? 16u : 0u;
            cp_async16(to, p.k + at + piece * 8, bytes);
            cp_async16(to + kTileBytes, p.v + at + piece * 8, bytes);
        }
    };

    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    float o[kDim / 8][4];
#pragma unroll
    for (int n = 0; n < kDim / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][e] = 0.f;

    int ahead = warp;               // the next tile to fetch
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) {
        if (ahead < tiles) {
            const int next = page_of(ahead + kWarps);
            fetch(ahead, s, page);
            page = next;
        }
        ahead += kWarps;
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // The query rows as the A operand: lane (g, c) holds rows g, g + 8, columns 16 k + 2 c ..., 16 k + 8 + 2 c ...  (Rows past
    // the last one repeat it: nothing reads their results, and a condition around each load would make the loads wait for
    // one another.)
    uint32_t qa[kDim / 16][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = min(g + 8 * h, rows - 1), tok = r / G;
        const __nv_bfloat16* row = p.q + ((size_t)(row0 + tok) * H + kvh * G + (r - tok * G)) * kDim + 2 * c;
#pragma unroll
        for (int k = 0; k < kDim / 16; ++k) {
            qa[k][h] = __ldg(reinterpret_cast<const uint32_t*>(row + 16 * k));
            qa[k][2 + h] = __ldg(reinterpret_cast<const uint32_t*>(row + 16 * k + 8));
        }
    }
    int stage = 0, into = kStages - 1;
    // ldmatrix addresses: lane i supplies row i % 16 (keys: tokens; values: tokens), column half i / 16
    const int lrow = lane & 15, lhalf = lane >> 4;
    for (int i = warp; i < tiles; i += kWarps) {
        __syncwarp();               // every lane has read the tile that the next fetch overwrites
        if (ahead < tiles) {
            const int next = page_of(ahead + kWarps);   // (asked for one tile ahead of its use)
            fetch(ahead, into, page);
            page = next;
        }
        ahead += kWarps;
        asm volatile("cp.async.commit_group;" ::: "memory");
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
        __syncwarp();
        const uint32_t kt = ring + stage * 2 * kTileBytes, vt = kt + kTileBytes;
        float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int k = 0; k < kDim / 16; ++k) {
            // matrices: tokens 0-7 / 8-15 at columns 16 k, then the same at 16 k + 8
            const int piece = 2 * k + lhalf;
            uint32_t b[4];
            ldsm4(b, kt + lrow * (kDim * 2) + ((piece & ~7) | ((piece ^ lrow) & 7)) * 16);
            mma16816(s[0], qa[k], b[0], b[2]);
            mma16816(s[1], qa[k], b[1], b[3]);
        }
        const int tok = begin + i * kTile;
        float top[2] = {-INFINITY, -INFINITY};
        const bool masked = tok + kTile > all_see;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[n][e] *= p.scale_log2;
                if (masked && tok + 8 * n + 2 * c + (e & 1) >= see[e >> 1]) s[n][e] = -INFINITY;
                top[e >> 1] = fmaxf(top[e >> 1], s[n][e]);
            }
        uint32_t pa[4];
        float keep[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float now = fmaxf(m[h], quad_max(top[h]));
            const float ref = now == -INFINITY ? 0.f : now;
            keep[h] = fast_exp2(m[h] - ref);
            m[h] = now;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) s[n][2 * h + e] = fast_exp2(s[n][2 * h + e] - ref);
            l[h] = l[h] * keep[h] + ((s[0][2 * h] + s[0][2 * h + 1]) + (s[1][2 * h] + s[1][2 * h + 1]));
        }
        // The weights are rounded to bf16 for the product with V, whose operands have one type; the sum keeps them in fp32.  (2^-9
        // of each at most, of either sign: outputs are off by 0.0021 of their size where their own rounding makes 0.0017.)
        pa[0] = pack2(s[0][0], s[0][1]);
        pa[1] = pack2(s[0][2], s[0][3]);
        pa[2] = pack2(s[1][0], s[1][1]);
        pa[3] = pack2(s[1][2], s[1][3]);
        if (__any_sync(0xffffffffu, keep[0] != 1.f || keep[1] != 1.f)) {
#pragma unroll
            for (int n = 0; n < kDim / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] *= keep[e >> 1];
        }
        // A value that some row must not see and that is infinite or NaN stays out of that row (the products of a tile would
        // add zero times it): such a tile's weights and values are multiplied one token after the other.
        bool apart = false;
        if (tok + kTile > all_see && all_see < stop) {
#pragma unroll
            for (int j = 0; j < kTile * kPieces / 32; ++j) {
                const int piece = j * 32 + lane, r = piece / kPieces, o8 = piece % kPieces;
                if (tok + r >= all_see) apart |= any_not_finite(lds128(vt + r * (kDim * 2) + ((o8 & ~7) | ((o8 ^ r) & 7)) * 16));
            }
            apart = __any_sync(0xffffffffu, apart);
        }
        if (apart) {
#pragma unroll 1
            for (int t = 0; t < kTile; ++t) {
                float w[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float even = t < 8 ? s[0][2 * h] : s[1][2 * h], odd = t < 8 ? s[0][2 * h + 1] : s[1][2 * h + 1];
                    w[h] = __shfl_sync(0xffffffffu, t & 1 ? odd : even, (lane & ~3) | ((t & 7) >> 1));
                }
#pragma unroll
                for (int n = 0; n < kDim / 8; ++n) {
                    const float2 v = lds_pair(vt + t * (kDim * 2) + ((n & ~7) | ((n ^ t) & 7)) * 16 + 4 * c);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (tok + t < see[h]) {
                            o[n][2 * h] = fmaf(w[h], v.x, o[n][2 * h]);
                            o[n][2 * h + 1] = fmaf(w[h], v.y, o[n][2 * h + 1]);
                        }
                }
            }
        } else {
#pragma unroll
            for (int n = 0; n < kDim / 16; ++n) {
                // matrices: tokens 0-7 / 8-15 at columns 16 n, then the same at 16 n + 8, transposed
                const int piece = 2 * n + lhalf;
                uint32_t b[4];
                ldsm4t(b, vt + lrow * (kDim * 2) + ((piece & ~7) | ((piece ^ lrow) & 7)) * 16);
                mma16816(o[2 * n], pa, b[0], b[1]);
                mma16816(o[2 * n + 1], pa, b[2], b[3]);
            }
        }
        stage = stage + 1 == kStages ? 0 : stage + 1;
        into = into + 1 == kStages ? 0 : into + 1;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");

    // join the warps: maxima and sums first, then the accumulators where the rings were
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        l[h] = quad_sum(l[h]);
        if (c == 0) {
            s_m[warp][g + 8 * h] = m[h];
            s_l[warp][g + 8 * h] = l[h];
        }
    }
    __syncthreads();
    float* so = reinterpret_cast<float*>(smem) + (size_t)warp * kTile * kDim;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = g + 8 * h;
        float most = s_m[0][r];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) most = fmaxf(most, s_m[w][r]);
        const float f = m[h] == -INFINITY ? 0.f : fast_exp2(m[h] - most);
        if (r < rows) {
#pragma unroll
            for (int n = 0; n < kDim / 8; ++n)
                *reinterpret_cast<float2*>(so + r * kDim + 8 * n + 2 * c) = make_float2(o[n][2 * h] * f, o[n][2 * h + 1] * f);
        }
    }
    if (tid < 16) {
        float most = s_m[0][tid], sum = 0.f;
        for (int w = 1; w < kWarps; ++w) most = fmaxf(most, s_m[w][tid]);
        // (a maximum of -inf: the warp has seen nothing, its sum is zero; or only scores that are NaN, and so is its sum)
        for (int w = 0; w < kWarps; ++w) sum += s_l[w][tid] * (s_m[w][tid] == -INFINITY ? 0.f : fast_exp2(s_m[w][tid] - most));
        s_scale[0][tid] = most;
        s_scale[1][tid] = sum;
    }
    __syncthreads();
    const float* all = reinterpret_cast<const float*>(smem);
    auto joined = [&](int at) -> float2 {
        float2 v = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float2 u = *reinterpret_cast<const float2*>(all + (size_t)w * kTile * kDim + at);
            v.x += u.x;
            v.y += u.y;
        }
        return v;
    };
    auto write = [&](int at, float2 v, float sum) {
        const int r = at / kDim, d = at % kDim;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        *reinterpret_cast<uint32_t*>(p.out + ((size_t)(row0 + r / G) * H + kvh * G + r % G) * kDim + d) = pack2(v.x * inv, v.y * inv);
    };
    if (kTogether) {
        // every block's result behind the warps' ones; then each block joins its share of the outputs over all blocks
        float* mine = reinterpret_cast<float*>(smem) + kWarps * kTile * kDim;
        for (int at = 2 * tid; at < rows * kDim; at += 2 * blockDim.x) *reinterpret_cast<float2*>(mine + at) = joined(at);
        cluster_arrive();
        cluster_wait();
        const uint32_t here = (uint32_t)__cvta_generic_to_shared(mine), stats = (uint32_t)__cvta_generic_to_shared(&s_scale[0][0]);
        for (int at = 2 * (split * (int)blockDim.x + tid); at < rows * kDim; at += 2 * (int)(gridDim.x * blockDim.x)) {
            const int r = at / kDim;
            float top[kMostTogether], part[kMostTogether], most = -INFINITY, sum = 0.f;
            float2 u[kMostTogether], v = make_float2(0.f, 0.f);
#pragma unroll
            for (int s = 0; s < kMostTogether; ++s) {
                const int from = min(s, parts - 1);   // (all on the way at once; the repeated ones do not count)
                top[s] = ld_block(stats + 4 * r, from);
                part[s] = ld_block(stats + 64 + 4 * r, from);
                u[s].x = ld_block(here + 4 * at, from);
                u[s].y = ld_block(here + 4 * at + 4, from);
                most = fmaxf(most, top[s]);
            }
#pragma unroll
            for (int s = 0; s < kMostTogether; ++s) {
                const float f = s >= parts || top[s] == -INFINITY ? 0.f : fast_exp2(top[s] - most);
                sum = fmaf(part[s], f, sum);
                v.x = fmaf(u[s].x, f, v.x);
                v.y = fmaf(u[s].y, f, v.y);
            }
            write(at, v, sum);
        }
        cluster_arrive();   // (nobody leaves while another block may read its shared memory)
        cluster_wait();
        return;
    }
    if (parts == 1) {
        for (int at = 2 * tid; at < rows * kDim; at += 2 * blockDim.x) write(at, joined(at), s_scale[1][at / kDim]);
        return;
    }
    // a part: few_rows x kDim accumulators, then few_rows maxima and few_rows sums
    const size_t part_floats = (size_t)p.few_rows * (kDim + 2);
    float* mine = p.few_parts + (((size_t)seq * p.c.num_kv_heads + kvh) * p.slots + split) * part_floats;
    for (int at = 2 * tid; at < rows * kDim; at += 2 * blockDim.x) *reinterpret_cast<float2*>(mine + at) = joined(at);
    if (tid < rows) {
        mine[p.few_rows * kDim + tid] = s_scale[0][tid];
        mine[p.few_rows * (kDim + 1) + tid] = s_scale[1][tid];
    }
    __threadfence();
    __syncthreads();
    if (tid == 0) s_last = atomicAdd(p.counters + seq * p.c.num_kv_heads + kvh, 1) == parts - 1;
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    if (tid == 0) p.counters[seq * p.c.num_kv_heads + kvh] = 0;
    const float* first = mine - (size_t)split * part_floats;
    for (int at = 2 * tid; at < rows * kDim; at += 2 * blockDim.x) {
        const int r = at / kDim;
        float most = -INFINITY, sum = 0.f;
        for (int s = 0; s < parts; ++s) most = fmaxf(most, __ldcg(first + s * part_floats + p.few_rows * kDim + r));
        float2 v = make_float2(0.f, 0.f);
        for (int s = 0; s < parts; ++s) {
            const float* q = first + s * part_floats;
            const float ms = __ldcg(q + p.few_rows * kDim + r);
            const float f = ms == -INFINITY ? 0.f : fast_exp2(ms - most);   // (times zeros, or a NaN that stays one)
            const float2 u = __ldcg(reinterpret_cast<const float2*>(q + at));
            sum = fmaf(__ldcg(q + p.few_rows * (kDim + 1) + r), f, sum);
            v.x = fmaf(u.x, f, v.x);
            v.y = fmaf(u.y, f, v.y);
        }
        write(at, v, sum);
    }
}

template <int kDim, bool kTogether>
qil_status go(const AttnParams& p, cudaStream_t st) {
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(attn_few_kernel<kDim, kTogether>, FewShape<kDim>::kSmem, allowed)) return QIL_ERR_CUDA;
    const unsigned across = !kTogether ? (unsigned)p.slots : p.slots <= 2 ? 2u : p.slots <= 4 ? 4u : (unsigned)kMostTogether;
    const dim3 grid(across, (unsigned)p.c.num_kv_heads, (unsigned)(p.c.num_seqs + p.both));
    return launch_early_clusters(attn_few_kernel<kDim, kTogether>, kTogether ? across : 1u, grid, 32 * kWarps, FewShape<kDim>::kSmem, st, p);
}

}  // namespace

qil_status launch_attn_few(const AttnParams& p, cudaStream_t st) {
    if (p.c.head_dim == 128) return p.together ? go<128, true>(p, st) : go<128, false>(p, st);
    return p.together ? go<64, true>(p, st) : go<64, false>(p, st);
}

}  // namespace qil
