// Low-rank adapters of many requests beside one shared projection (the side path of lora_side.cu for a batch in which every
// request brings its own adapter, or none):
//   out[m] = bf16( y[m] + scales[a] * (x[m] A_a^T) B_a^T ),  a = adapter of the request that row m belongs to
//   A [n][r][K] bf16    B [n][N][r] bf16    rows of request b: cu_q[b] ... cu_q[b+1]
// Memory bound in both regimes: at decode length the adapters' matrices are what is read, in prompts x and y.  Two kernels:
//   1. t[slice][m][j] = x . A^T over a slice of K, fp32 in the workspace,
//   2. out = y + scale t B^T, one pass over y.
// Rows are cut into tiles per request, so that a tile has one adapter.  The products run on mma.sync (16 x 8 x 16): with a
// rank of 8 to 64 against two streams of K or N elements per row, a multiply costs nothing next to its operands' bytes.
// A lane fetches its own operands in 16-byte pieces and no other lane reads them, so that nothing is rearranged (single tokens:
// into registers; prompts: through a ring of the lane's own pieces in shared memory, which holds more in flight).  The order
// of a contraction's terms is free: lane c of four takes 8 neighbouring elements and both operands use the same order; and
// the columns of a group of four 16 x 8 results are dealt out so that a lane ends up with 8 neighbouring outputs.
// Measured: 32 single tokens, 12 adapters of rank 16, 4096 x 4096: 6.0 us (7.5 cold), a chain of five trips to memory (request, adapter,
// operands, the cluster's parts, outputs).  4000 rows in nine prompts, rank 32, 4096 -> 11008: 12 + 33 us, against 34 us for
// x, y and the output at the copy rate; of the second kernel's traffic a third is B, re-read from L2 for every 64 rows.
// t is split into two bf16 terms (hi + lo) before it is multiplied: it keeps 16 significant bits.
#include "layer_common.cuh"

namespace qil {

namespace {

constexpr int kDownWarps = 4, kUpWarps = 8, kMaxSlices = 32, kFusedWarps = 8, kCluster = 8;
// Depth of the rings, and blocks of the second kernel per SM: by shared memory two blocks of either kernel fit an SM (4000
// rows, rank 32, 4096 -> 11008: 45 us in all; a stage more of either ring takes a block away: 52 to 70 us; blocks of half the
// size and twice as many: 47 us, shorter shares of the outputs per block: 50 to 57 us).
constexpr int kDownStages = 3, kUpStages = 2, kUpBlocks = 2;

struct LoraParams {
    const __nv_bfloat16 *x, *a, *b, *y;
    __nv_bfloat16* out;
    float* t;   // [slices][M][rank]
    const int *cu, *adapter;
    const float* scales;
    int M, N, K, rank, num_seqs, num_adapters, slices, slice_blocks;   // a slice is slice_blocks blocks of 32 columns of K
    long long ldx, ldy, ldo;
};

template <int kBytes>
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src) {
    if (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(kBytes) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

// Two values as sums of two bf16 terms each.  What is finite stays so (a value beyond bf16's largest has that as its first
// term), and an infinity has no second term: inf - inf would make the product NaN.
__device__ __forceinline__ void split2(float2 v, uint32_t& hi, uint32_t& lo) {
    constexpr float kMost = 3.3895313892515355e38f;   // (2 - 2^-7) 2^127
    const auto first = [](float x) { return fabsf(x) > kMost && fabsf(x) < INFINITY ? copysignf(kMost, x) : x; };
    const auto rest = [](float x, float h) { return fabsf(x) == INFINITY ? 0.f : x - h; };
    hi = pack2(first(v.x), first(v.y));
    lo = pack2(rest(v.x, __uint_as_float(hi << 16)), rest(v.y, __uint_as_float(hi & 0xFFFF0000u)));
}

// kMT: row tiles of 16 per block; kNR: column tiles of 8 of the rank (the rank padded up to 8, 16, 32 or 64)
template <int kMT, int kNR>
__global__ void __launch_bounds__(32 * kDownWarps) lora_batch_down_kernel(const LoraParams p) {
    __shared__ float part[kDownWarps - 1][kMT * kNR * 4 * 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    wait_for_earlier_kernels();
    let_next_kernel_start();   // (the second kernel reads what came before this one ahead of its own wait)
    int seq, row0, row1;
    if (!find_tile(p.cu, p.num_seqs, p.M, 16 * kMT, blockIdx.x, seq, row0, row1)) return;
    const int ad = __ldg(p.adapter + seq);
    if (ad < 0 || ad >= p.num_adapters) return;
    const __nv_bfloat16* a = p.a + (size_t)ad * p.rank * p.K;
    float acc[kMT][kNR][4];
#pragma unroll
    for (int m = 0; m < kMT; ++m)
#pragma unroll
        for (int n = 0; n < kNR; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[m][n][e] = 0.f;
    // Rows past the tile's last and rank rows past the last repeat the last one: nobody reads their results.
    const __nv_bfloat16 *xr[kMT][2], *ar[kNR];
#pragma unroll
    for (int m = 0; m < kMT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) xr[m][h] = p.x + min(row0 + 16 * m + 8 * h + g, row1 - 1) * p.ldx;
#pragma unroll
    for (int n = 0; n < kNR; ++n) ar[n] = a + (size_t)min(8 * n + g, p.rank - 1) * p.K;
    const int first = blockIdx.y * p.slice_blocks, last = min(first + p.slice_blocks, (p.K + 31) / 32);
    // The lane's own 16-byte pieces of the next blocks of K go through a ring in shared memory instead of registers: two
    // blocks are in flight beside the one at work.
    extern __shared__ __align__(16) unsigned char ring[];
    constexpr int kPieces = 2 * kMT + kNR, kStageBytes = kPieces * 512;
    const uint32_t slot = (uint32_t)__cvta_generic_to_shared(ring) + warp * (kDownStages * kStageBytes) + lane * 16;
    auto fetch = [&](int kb, int stage) {
        const int at = min(kb * 32 + c * 8, p.K - 8);   // this lane's 8 columns (K is a multiple of 8: all or none of them exist)
        const uint32_t to = slot + stage * kStageBytes;
#pragma unroll
        for (int m = 0; m < kMT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) cp_async<16>(to + (2 * m + h) * 512, xr[m][h] + at);
#pragma unroll
        for (int n = 0; n < kNR; ++n) cp_async<16>(to + (2 * kMT + n) * 512, ar[n] + at);
    };
    int ahead = first + warp, into = 0, stage = 0;
#pragma unroll
    for (int s = 0; s < kDownStages - 1; ++s, ahead += kDownWarps, ++into) {
        if (ahead < last) fetch(ahead, into);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
#pragma unroll 1
    for (int kb = first + warp; kb < last; kb += kDownWarps) {
        if (ahead < last) fetch(ahead, into);
        asm volatile("cp.async.commit_group;" ::: "memory");
        asm volatile("cp.async.wait_group %0;" ::"n"(kDownStages - 1) : "memory");
        ahead += kDownWarps;
        into = into + 1 == kDownStages ? 0 : into + 1;
        uint4 xv[kMT][2], av[kNR];
#pragma unroll
        for (int m = 0; m < kMT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) xv[m][h] = lds16(slot + stage * kStageBytes + (2 * m + h) * 512);
#pragma unroll
        for (int n = 0; n < kNR; ++n) av[n] = lds16(slot + stage * kStageBytes + (2 * kMT + n) * 512);
        stage = stage + 1 == kDownStages ? 0 : stage + 1;
        // (repeated columns of A are finite or their row's result is not anyway: zeros of x are enough)
        const uint32_t in = kb * 32 + c * 8 < p.K ? 0xFFFFFFFFu : 0u;
#pragma unroll
        for (int m = 0; m < kMT; ++m) {
            const uint32_t a0[4] = {xv[m][0].x & in, xv[m][1].x & in, xv[m][0].y & in, xv[m][1].y & in};
            const uint32_t a1[4] = {xv[m][0].z & in, xv[m][1].z & in, xv[m][0].w & in, xv[m][1].w & in};
#pragma unroll
            for (int n = 0; n < kNR; ++n) {
                mma16816(acc[m][n], a0, av[n].x, av[n].y);
                mma16816(acc[m][n], a1, av[n].z, av[n].w);
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    // the warps' parts, added in warp order
    if (warp > 0) {
#pragma unroll
        for (int m = 0; m < kMT; ++m)
#pragma unroll
            for (int n = 0; n < kNR; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) part[warp - 1][((m * kNR + n) * 4 + e) * 32 + lane] = acc[m][n][e];
    }
    __syncthreads();
    if (warp > 0) return;
    float* t = p.t + (size_t)blockIdx.y * p.M * p.rank;
#pragma unroll
    for (int m = 0; m < kMT; ++m)
#pragma unroll
        for (int n = 0; n < kNR; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int w = 0; w < kDownWarps - 1; ++w) acc[m][n][e] += part[w][((m * kNR + n) * 4 + e) * 32 + lane];
            const int j = 8 * n + 2 * c;
            if (j < p.rank) {
                const int row = row0 + 16 * m + g;
                if (row < row1) *reinterpret_cast<float2*>(t + (size_t)row * p.rank + j) = make_float2(acc[m][n][0], acc[m][n][1]);
                if (row + 8 < row1) *reinterpret_cast<float2*>(t + (size_t)(row + 8) * p.rank + j) = make_float2(acc[m][n][2], acc[m][n][3]);
            }
        }
}

// A warp takes groups of 32 outputs in turn, with the next groups' y and B on the way while it works: a block's way to its
// first product (the request, its adapter, t) is several trips to memory long and is paid once.
template <int kMT, int kNR>
__global__ void __launch_bounds__(32 * kUpWarps, kUpBlocks) lora_batch_up_kernel(const LoraParams p) {
    constexpr int kRank = 8 * kNR, kW = kRank / 4, kSteps = kRank <= 16 ? 1 : kRank / 16;   // kW: rank elements of a lane
    constexpr int kBQ = kW == 16 ? 2 : 1;
    // t as the A operand of the products, in the order of the lanes' registers: [row tile][step][hi, lo][lane][4 words]
    __shared__ __align__(16) uint32_t frag[kMT * kSteps * 2 * 32 * 4];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    int seq, row0, row1;
    // Blocks without work leave at once, all but one: what comes after this launch waits for it alone, so it has to last until
    // the first kernel ends even if no request has an adapter.
    const bool found = find_tile(p.cu, p.num_seqs, p.M, 16 * kMT, blockIdx.x, seq, row0, row1);
    const int ad = found ? __ldg(p.adapter + seq) : -1;
    const bool none = ad < 0 || ad >= p.num_adapters;
    if (!found || (none && p.out == p.y)) {
        if (blockIdx.x == 0 && blockIdx.y == 0) wait_for_earlier_kernels();
        return;
    }
    const __nv_bfloat16* b = p.b + (size_t)(none ? 0 : ad) * p.N * p.rank;
    // Rows past the tile's last, columns past N and rank elements past the rank repeat others: the first two are not
    // written, the last meet zeros of t.  (Conditions around the loads would make them wait for one another.)
    // The lane's own pieces of y and B of the next groups go through a ring in shared memory, as in the first kernel.
    extern __shared__ __align__(16) unsigned char ring[];
    constexpr int kPieces = 2 * kMT + 4 * kBQ, kStageBytes = kPieces * 512;
    const uint32_t slot = (uint32_t)__cvta_generic_to_shared(ring) + warp * (kUpStages * kStageBytes) + lane * 16;
    auto fetch = [&](int n0, int stage) {
        const uint32_t to = slot + stage * kStageBytes;
#pragma unroll
        for (int m = 0; m < kMT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                cp_async<16>(to + (2 * m + h) * 512, p.y + min(row0 + 16 * m + 8 * h + g, row1 - 1) * p.ldy + min(n0 + 8 * c, p.N - 8));
        // B rows of the 32 columns: column (2c, 2c + 1) of result tile i is output n0 + 8 c + 2 i, + 1
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat16* row = b + (size_t)min(n0 + 8 * (g >> 1) + 2 * i + (g & 1), p.N - 1) * p.rank;
#pragma unroll
            for (int h = 0; h < kBQ; ++h)
                cp_async<(kW < 8 ? 2 * kW : 16)>(to + (2 * kMT + i * kBQ + h) * 512, row + min(kW * c + 8 * h, p.rank - (kW < 8 ? kW : 8)));
        }
    };
    int n0 = (blockIdx.y * kUpWarps + warp) * 32;
    const int stride = gridDim.y * kUpWarps * 32;
    int ahead = n0, into = 0, stage = 0;
#pragma unroll
    for (int s = 0; s < kUpStages - 1; ++s, ahead += stride, ++into) {
        if (ahead < p.N) fetch(ahead, into);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    const float scale = __ldg(p.scales + (none ? 0 : ad));
    wait_for_earlier_kernels();   // t is written by the first kernel, which may still be running
    if (!none) {
        for (int i = threadIdx.x; i < kMT * 16 * (kRank / 2); i += blockDim.x) {
            const int m = i / (kRank / 2), j = 2 * (i % (kRank / 2));
            const float* t = p.t + (size_t)min(row0 + m, row1 - 1) * p.rank + min(j, p.rank - 2);
            float2 v = make_float2(0.f, 0.f);
#pragma unroll 4
            for (int s = 0; s < p.slices; ++s) {
                const float2 u = __ldcg(reinterpret_cast<const float2*>(t + (size_t)s * p.M * p.rank));
                v.x += u.x;
                v.y += u.y;
            }
            v.x = j < p.rank ? v.x * scale : 0.f;
            v.y = j < p.rank ? v.y * scale : 0.f;
            uint32_t hi, lo;
            split2(v, hi, lo);
            const int at = j % kW, step = at >> 2, reg = ((m & 15) >> 3) + 2 * ((at & 3) >> 1);
            uint32_t* f = frag + ((((m >> 4) * kSteps + step) * 2) * 32 + (m & 7) * 4 + j / kW) * 4 + reg;
            f[0] = hi;
            f[32 * 4] = lo;
        }
    }
    __syncthreads();
#pragma unroll 1
    for (; n0 < p.N; n0 += stride) {
        if (ahead < p.N) fetch(ahead, into);
        asm volatile("cp.async.commit_group;" ::: "memory");
        asm volatile("cp.async.wait_group %0;" ::"n"(kUpStages - 1) : "memory");
        ahead += stride;
        into = into + 1 == kUpStages ? 0 : into + 1;
        const uint32_t from = slot + stage * kStageBytes;
        stage = stage + 1 == kUpStages ? 0 : stage + 1;
        uint4 bn[4][kBQ];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < kBQ; ++h) bn[i][h] = lds16(from + (2 * kMT + i * kBQ + h) * 512);
        const int n = n0 + 8 * c;      // this lane's 8 outputs (N is a multiple of 8: all or none of them exist)
#pragma unroll
        for (int m = 0; m < kMT; ++m) {
            float acc[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][e] = 0.f;
            if (!none) {
#pragma unroll
                for (int s = 0; s < kSteps; ++s)
#pragma unroll
                    for (int part = 0; part < 2; ++part) {
                        const uint4 v = *reinterpret_cast<const uint4*>(frag + ((((m * kSteps + s) * 2) + part) * 32 + lane) * 4);
                        const uint32_t a[4] = {v.x, v.y, kW == 2 ? 0u : v.z, kW == 2 ? 0u : v.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint4 q = bn[i][kW == 16 ? s >> 1 : 0];
                            if (s & 1) mma16816(acc[i], a, q.z, q.w);
                            else mma16816(acc[i], a, q.x, kW == 2 ? 0u : q.y);
                        }
                    }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = row0 + 16 * m + 8 * h + g;
                if (row < row1 && n < p.N) {
                    float o[8];
                    unpack8(lds16(from + (2 * m + h) * 512), o);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        o[2 * i] += acc[i][2 * h];
                        o[2 * i + 1] += acc[i][2 * h + 1];
                    }
                    *reinterpret_cast<uint4*>(p.out + row * p.ldo + n) = pack8(o);
                }
            }
        }
    }
}

// Both products in one kernel, for tiles of 16 rows: a cluster of kCluster blocks takes a tile.  Each block multiplies by its
// slice of K, the blocks add their parts through one another's shared memory, and each goes on to its share of the
// outputs, whose y and B are on their way from the beginning: one launch, and t never goes to memory.
template <int kNR>
__global__ void __launch_bounds__(32 * kFusedWarps) __cluster_dims__(kCluster, 1, 1) lora_batch_fused_kernel(const LoraParams p) {
    constexpr int kRank = 8 * kNR, kW = kRank / 4, kSteps = kRank <= 16 ? 1 : kRank / 16, kBQ = kW == 16 ? 2 : 1;
    __shared__ float part[kFusedWarps][16 * kRank];   // [warp][row][rank]; the block's part ends up in the first
    __shared__ __align__(16) uint32_t frag[kSteps * 2 * 32 * 4];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int tile = blockIdx.x / kCluster, mine = blockIdx.x % kCluster;
    wait_for_earlier_kernels();
    int seq, row0, row1;
    if (!find_tile(p.cu, p.num_seqs, p.M, 16, tile, seq, row0, row1)) return;   // (the whole cluster)
    const int ad = __ldg(p.adapter + seq);
    const bool none = ad < 0 || ad >= p.num_adapters;
    if (none && p.out == p.y) return;
    const int use = none ? 0 : ad;
    const __nv_bfloat16 *a = p.a + (size_t)use * p.rank * p.K, *b = p.b + (size_t)use * p.N * p.rank;
    const __nv_bfloat16* xr[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) xr[h] = p.x + min(row0 + 8 * h + g, row1 - 1) * p.ldx;
    // (rows, columns and rank elements that do not exist repeat others, as in the kernels above)
    uint4 yv[2], bq[4][kBQ];
    auto load = [&](int n0) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            yv[h] = *reinterpret_cast<const uint4*>(p.y + min(row0 + 8 * h + g, row1 - 1) * p.ldy + min(n0 + 8 * c, p.N - 8));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat16* row = b + (size_t)min(n0 + 8 * (g >> 1) + 2 * i + (g & 1), p.N - 1) * p.rank;
#pragma unroll
            for (int h = 0; h < kBQ; ++h) {
                const __nv_bfloat16* from = row + min(kW * c + 8 * h, p.rank - (kW < 8 ? kW : 8));
                if (kW == 2) bq[i][h] = make_uint4(__ldg(reinterpret_cast<const uint32_t*>(from)), 0u, 0u, 0u);
                else if (kW == 4) {
                    const uint2 v = __ldg(reinterpret_cast<const uint2*>(from));
                    bq[i][h] = make_uint4(v.x, v.y, 0u, 0u);
                } else bq[i][h] = __ldg(reinterpret_cast<const uint4*>(from));
            }
        }
    };
    const int groups = (p.N + 31) / 32, g0 = (int)((long long)groups * mine / kCluster), g1 = (int)((long long)groups * (mine + 1) / kCluster);
    load(min(g0 + warp, groups - 1) * 32);
    const float scale = __ldg(p.scales + use);
    float acc[kNR][4];
#pragma unroll
    for (int n = 0; n < kNR; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[n][e] = 0.f;
    if (!none) {
        const int blocks = (p.K + 31) / 32, last = (int)((long long)blocks * (mine + 1) / kCluster);
#pragma unroll 2
        for (int kb = (int)((long long)blocks * mine / kCluster) + warp; kb < last; kb += kFusedWarps) {
            const int k = kb * 32 + c * 8, at = min(k, p.K - 8);
            uint4 xv[2], av[kNR];
#pragma unroll
            for (int h = 0; h < 2; ++h) xv[h] = __ldg(reinterpret_cast<const uint4*>(xr[h] + at));
#pragma unroll
            for (int n = 0; n < kNR; ++n) av[n] = __ldg(reinterpret_cast<const uint4*>(a + (size_t)min(8 * n + g, p.rank - 1) * p.K + at));
            const uint32_t in = k < p.K ? 0xFFFFFFFFu : 0u;   // (A's repeated columns are finite or their row's result is not: zeros of x do)
            const uint32_t a0[4] = {xv[0].x & in, xv[1].x & in, xv[0].y & in, xv[1].y & in};
            const uint32_t a1[4] = {xv[0].z & in, xv[1].z & in, xv[0].w & in, xv[1].w & in};
#pragma unroll
            for (int n = 0; n < kNR; ++n) {
                mma16816(acc[n], a0, av[n].x, av[n].y);
                mma16816(acc[n], a1, av[n].z, av[n].w);
            }
        }
    }
#pragma unroll
    for (int n = 0; n < kNR; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            *reinterpret_cast<float2*>(&part[warp][(g + 8 * h) * kRank + 8 * n + 2 * c]) = make_float2(acc[n][2 * h], acc[n][2 * h + 1]);
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * kRank; i += blockDim.x) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kFusedWarps; ++w) v += part[w][i];
        part[0][i] = v;
    }
    const uint32_t here = (uint32_t)__cvta_generic_to_shared(&part[0][0]);
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    for (int i = threadIdx.x; i < 16 * (kRank / 2); i += blockDim.x) {
        const int m = i / (kRank / 2), j = 2 * (i % (kRank / 2));
        float2 v = make_float2(0.f, 0.f);
#pragma unroll
        for (int r = 0; r < kCluster; ++r) {
            uint32_t there;
            float2 u;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here + (uint32_t)(m * kRank + j) * 4u), "r"(r));
            asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(u.x), "=f"(u.y) : "r"(there) : "memory");
            v.x += u.x;
            v.y += u.y;
        }
        v.x = j < p.rank ? v.x * scale : 0.f;
        v.y = j < p.rank ? v.y * scale : 0.f;
        uint32_t hi, lo;
        split2(v, hi, lo);
        const int at = j % kW, step = at >> 2, reg = (m >> 3) + 2 * ((at & 3) >> 1);
        uint32_t* f = frag + (step * 2 * 32 + (m & 7) * 4 + j / kW) * 4 + reg;
        f[0] = hi;
        f[32 * 4] = lo;
    }
    __syncthreads();
    // (the others may still read this block's part: it stays until all have)
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    for (int n = g0 + warp; n < g1; n += kFusedWarps) {
        uint4 yn[2] = {yv[0], yv[1]}, bn[4][kBQ];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < kBQ; ++h) bn[i][h] = bq[i][h];
        if (n + kFusedWarps < g1) load((n + kFusedWarps) * 32);
        float o4[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o4[i][e] = 0.f;
        if (!none) {
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint4 v = *reinterpret_cast<const uint4*>(frag + ((s * 2 + half) * 32 + lane) * 4);
                    const uint32_t f[4] = {v.x, v.y, kW == 2 ? 0u : v.z, kW == 2 ? 0u : v.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint4 q = bn[i][kW == 16 ? s >> 1 : 0];
                        if (s & 1) mma16816(o4[i], f, q.z, q.w);
                        else mma16816(o4[i], f, q.x, kW == 2 ? 0u : q.y);
                    }
                }
        }
        const int col = n * 32 + 8 * c;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = row0 + 8 * h + g;
            if (row < row1 && col < p.N) {
                float o[8];
                unpack8(yn[h], o);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    o[2 * i] += o4[i][2 * h];
                    o[2 * i + 1] += o4[i][2 * h + 1];
                }
                *reinterpret_cast<uint4*>(p.out + row * p.ldo + col) = pack8(o);
            }
        }
    }
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Row tiles of 16 per block.  A tile wastes what its request does not fill, so a batch of single tokens takes tiles of 16
// (the fused kernel); prompts take 64 rows (32 at rank 64, for the accumulators' registers): the adapter is read once per tile.
int lora_row_tiles(int M, int num_seqs, int rank) {
    if (M <= 16LL * num_seqs) return 1;
    return rank > 32 ? 2 : 4;
}
int lora_max_tiles(int M, int num_seqs, int rank) { return M / (16 * lora_row_tiles(M, num_seqs, rank)) + num_seqs; }

// Slices of K for the first kernel: one round of two blocks per SM (a second round costs more than longer slices do), at
// least 256 columns each.
int lora_batch_slices(int M, int num_seqs, int rank, int K) {
    const int tiles = lora_max_tiles(M, num_seqs, rank);
    int s = 2 * num_sms() / tiles;
    s = s < K / 256 ? s : K / 256;
    s = s < kMaxSlices ? s : kMaxSlices;
    return s < 1 ? 1 : s;
}

template <int kMT, int kNR>
qil_status launch_two(const LoraParams& p, dim3 down, dim3 up, cudaStream_t st) {
    constexpr int kDown = kDownWarps * kDownStages * (2 * kMT + kNR) * 512, kUp = kUpWarps * kUpStages * (2 * kMT + 4 * (kNR == 8 ? 2 : 1)) * 512;
    static std::atomic<unsigned long long> down_allowed{0}, up_allowed{0};
    if (!allow_smem(lora_batch_down_kernel<kMT, kNR>, kDown, down_allowed) || !allow_smem(lora_batch_up_kernel<kMT, kNR>, kUp, up_allowed))
        return QIL_ERR_CUDA;
    const qil_status s = launch_early(lora_batch_down_kernel<kMT, kNR>, down, 32 * kDownWarps, kDown, st, p);
    return s != QIL_OK ? s : launch_early(lora_batch_up_kernel<kMT, kNR>, up, 32 * kUpWarps, kUp, st, p);
}

}  // namespace

size_t lora_batch_workspace(int M, int num_seqs, int rank) {
    if (lora_row_tiles(M, num_seqs, rank) == 1) return 16;   // (t stays on the chip)
    return (size_t)lora_batch_slices(M, num_seqs, rank, 1 << 30) * M * rank * sizeof(float);
}

qil_status launch_lora_batch_add(const void* x, const void* a, const void* b, const void* y, void* out, const int* cu_q, const int* adapter,
                                 const float* scales, int M, int N, int K, int rank, int num_seqs, int num_adapters, long long ldx,
                                 long long ldy, long long ldo, void* ws, cudaStream_t st) {
    LoraParams p;
    p.x = reinterpret_cast<const __nv_bfloat16*>(x);
    p.a = reinterpret_cast<const __nv_bfloat16*>(a);
    p.b = reinterpret_cast<const __nv_bfloat16*>(b);
    p.y = reinterpret_cast<const __nv_bfloat16*>(y);
    p.out = reinterpret_cast<__nv_bfloat16*>(out);
    p.t = reinterpret_cast<float*>(ws);
    p.cu = cu_q; p.adapter = adapter; p.scales = scales;
    p.M = M; p.N = N; p.K = K; p.rank = rank; p.num_seqs = num_seqs; p.num_adapters = num_adapters;
    p.ldx = ldx; p.ldy = ldy; p.ldo = ldo;
    const unsigned tiles = (unsigned)lora_max_tiles(M, num_seqs, rank);
    if (lora_row_tiles(M, num_seqs, rank) == 1) {
        auto go = [&](auto kernel) { return launch_early(kernel, dim3(tiles * kCluster), 32 * kFusedWarps, 0, st, p); };
        if (rank <= 8) return go(lora_batch_fused_kernel<1>);
        if (rank <= 16) return go(lora_batch_fused_kernel<2>);
        return rank <= 32 ? go(lora_batch_fused_kernel<4>) : go(lora_batch_fused_kernel<8>);
    }
    const int blocks = (K + 31) / 32;
    p.slices = lora_batch_slices(M, num_seqs, rank, K);
    p.slice_blocks = (blocks + p.slices - 1) / p.slices;
    p.slices = (blocks + p.slice_blocks - 1) / p.slice_blocks;
    // second kernel: one round of blocks, or all the columns there are
    const unsigned groups = (unsigned)((N + 32 * kUpWarps - 1) / (32 * kUpWarps));
    unsigned across = (unsigned)(kUpBlocks * num_sms()) / tiles;
    if (across < 1) across = 1;
    if (across > groups) across = groups;
    const dim3 down(tiles, (unsigned)p.slices), up(tiles, across);
    if (rank <= 8) return launch_two<4, 1>(p, down, up, st);
    if (rank <= 16) return launch_two<4, 2>(p, down, up, st);
    if (rank <= 32) return launch_two<4, 4>(p, down, up, st);
    return launch_two<2, 8>(p, down, up, st);
}

}  // namespace qil
