// Attention over the quantised paged cache for requests with few query rows (new tokens x heads of a group <= 16): single
// tokens and short drafts.  Memory bound: every cached code is read once per key head.
//
// As in attn_few.cu a block takes `chunk` cached tokens of one request and key head, its four warps take tiles of 16 tokens in
// turn, each with its own ring in shared memory, and blocks of a request are joined in a cluster or through the workspace.
// What differs is what a tile costs apart from its bytes, a half or a quarter of those of bf16:
//   S^T = K Q^T and O^T += V^T P^T: the cache is the 16-row operand of mma.sync 16 x 8 x 16 and the query rows are the 8
//   columns, so that up to 8 rows take half the products and accumulators of a tile of 16 rows.
//   Codes become bf16 in registers by a few logic operations, exactly: whole numbers of at most 8 bits.  The operands' columns
//   may be in any order as long as both sides agree, so a lane's codes are 16 bytes or less in one piece, and the words come
//   apart in the order that needs the fewest operations (nibbles 0 and 4 of a word are one mask away from a pair).
//   A key's scale multiplies its scores, a value's scale its weight.  Zero points: S = s (q . (128 + c) - (128 + z) sum q) for
//   keys; for values, whose sums cancel, 128 + z is taken off every code.
//   The running reference of a row is only raised by scores more than 2^8 above it, which a vote finds; maxima are reduced
//   over the lanes in those tiles alone, sums once at the end.
// A weight times its value's scale is rounded to bf16 for the product (2^-9 of each at most, of either sign).
// Codes are finite whatever they are, so nothing behind a request's last token can reach a result: its weight is replaced by
// zero after its scale has been applied.
#include "attn_paged_q.cuh"

namespace qil {

namespace {

constexpr int kWarps = 4, kTile = 16;

template <int kDim, int kBits>
struct FewQ {
    static constexpr int kRowBytes = kDim * kBits / 8;               // 128, 64, 64, 32
    static constexpr int kTileBytes = kTile * kRowBytes;
    static constexpr int kParBytes = kTile * (kBits == 8 ? 2 : 4);   // of one side
    static constexpr int kStageBytes = 2 * kTileBytes + 2 * kParBytes;
    static constexpr int kStages = 13056 / kStageBytes;              // 51 KB a block, four blocks an SM
    static constexpr int kWarpBytes = kStages * kStageBytes;
    static constexpr int kSteps = kDim / 16;
    static_assert(kStages >= 2, "a tile ahead");
};

// Where 16-byte piece `piece` of row `row` of a tile lies.  Rows of 128 bytes: the eight lanes of a load that read four
// pieces of two rows (keys) or two pieces of every second row (values) meet all banks; shorter rows share 128-byte lines.
template <int kRowBytes>
__device__ __forceinline__ uint32_t place(int row, int piece) {
    if (kRowBytes == 128) return row * 128 + ((piece ^ (row & 6) ^ ((row & 1) << 2)) & 7) * 16;
    if (kRowBytes == 64) return (row >> 1) * 128 + ((((row & 1) * 4 + piece) ^ (row & 6)) & 7) * 16;
    return (row >> 2) * 128 + (((row & 3) * 2 + piece) ^ ((row >> 1) & 2)) * 16;
}

__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
    return d;
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t addr) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}
// kWords words at byte offset `at` (a multiple of their size) of a row of a tile
template <int kRowBytes, int kWords>
__device__ __forceinline__ void load_words(uint32_t tile, int row, int at, uint32_t (&w)[kWords]) {
    const uint32_t addr = tile + place<kRowBytes>(row, at >> 4) + (at & 15);
    if constexpr (kWords == 4) {
        const uint4 v = lds128(addr);
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else if constexpr (kWords == 2) {
        const uint2 v = lds64(addr);
        w[0] = v.x, w[1] = v.y;
    } else {
        w[0] = lds32(addr);
    }
}
// sum or maximum over the lanes that hold the same query rows
template <class F>
__device__ __forceinline__ float over_tokens(float v, F f) {
    v = f(v, __shfl_xor_sync(0xffffffffu, v, 4));
    v = f(v, __shfl_xor_sync(0xffffffffu, v, 8));
    return f(v, __shfl_xor_sync(0xffffffffu, v, 16));
}

// kCols: columns of 8 query rows.  kTogether: the blocks of a request and key head are one cluster.
template <int kDim, int kBits, int kCols, bool kTogether>
__global__ void __launch_bounds__(32 * kWarps, kCols == 1 ? 4 : 3) attn_few_q_kernel(const AttnQuantParams pq) {
    using Shape = FewQ<kDim, kBits>;
    constexpr int kStages = Shape::kStages, kRowBytes = Shape::kRowBytes, kTileBytes = Shape::kTileBytes, kSteps = Shape::kSteps;
    constexpr int kRows = 8 * kCols, kKeyWords = kRowBytes >= 64 ? 4 : 2, kKeyLoads = kRowBytes == 128 ? 2 : 1, kValWords = kRowBytes / 32;
    const AttnParams& p = pq.a;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows];
    __shared__ float s_scale[2][kRows];
    __shared__ int s_last;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    const int split = blockIdx.x, kvh = blockIdx.y, seq = blockIdx.z, G = p.G, H = p.c.num_heads;
    // (beside the kernel for many rows, as in attn_few.cu)
    if (!p.both) wait_for_earlier_kernels();
    if (seq == p.c.num_seqs) {
        if (split == 0 && kvh == 0) wait_for_earlier_kernels();
        return;
    }
    const int begin = split * p.chunk;
    const int* table = p.c.block_table + (size_t)seq * p.c.max_pages;
    const int kv = __ldg(p.c.kv_len + seq);
    int page = __ldg(table + min((begin + warp * kTile) >> p.page_shift, p.c.max_pages - 1));
    int row0, row1;
    request_rows(p.c.cu_q, seq, p.c.total_q, row0, row1);
    const int q_len = row1 - row0;
    if (q_len <= 0 || q_len * (long long)G > kFewRows) return;
    const int rows = q_len * G, end = cache_end(p.c, kv), first_pos = kv - q_len;
    // a request with more rows than the bound says is left out
    if (rows > kRows || (!kTogether && p.slots > 1 && rows > p.few_rows)) return;
    const int parts = max(1, min((end + p.chunk - 1) / p.chunk, p.slots));
    const bool idle = split >= parts;
    if (idle && !kTogether) return;
    const int stop = idle ? begin : split + 1 == parts ? end : min(begin + p.chunk, end);
    const int tiles = (stop - begin + kTile - 1) / kTile;

    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * Shape::kWarpBytes;
    auto page_of = [&](int i) -> int { return __ldg(table + (min(begin + i * kTile, stop - 1) >> p.page_shift)); };
    auto fetch = [&](int i, int stage, int page) {
        const int tok = begin + i * kTile;
        const uint32_t bytes = page >= 0 && page < p.c.num_pages ? 16u : 0u;   // (a page that does not exist: zeros)
        const size_t at = bytes ? ((size_t)page * p.c.num_kv_heads + kvh) * p.c.page_size + (tok & (p.c.page_size - 1)) : 0;   // a row of the cache
        const uint32_t dst = ring + stage * Shape::kStageBytes;
        const char *k = static_cast<const char*>(pq.kv.k) + at * kRowBytes, *v = static_cast<const char*>(pq.kv.v) + at * kRowBytes;
#pragma unroll
        for (int j = 0; j < kRowBytes / 32; ++j) {
            const int piece = j * 32 + lane;
            const uint32_t to = dst + place<kRowBytes>(piece / (kRowBytes / 16), piece % (kRowBytes / 16));
            cp_async16(to, k + piece * 16, bytes);
            cp_async16(to + kTileBytes, v + piece * 16, bytes);
        }
        constexpr int kPieces = Shape::kParBytes / 16;
        if (lane < 2 * kPieces) {
            const char* par = reinterpret_cast<const char*>(lane < kPieces ? pq.kv.ks : pq.kv.vs) + at * (Shape::kParBytes / kTile);
            cp_async16(dst + 2 * kTileBytes + lane * 16, par + (lane % kPieces) * 16, bytes);
        }
    };

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

    // visible tokens of this lane's query rows 8 n + 2 c, 8 n + 2 c + 1
    int see[kCols][2];
#pragma unroll
    for (int n = 0; n < kCols; ++n)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = 8 * n + 2 * c + j;
            see[n][j] = r < rows ? min(first_pos + r / G + 1, end) : 0;
        }
    const int all_see = min(first_pos + 1, end);   // every row sees what the first new token sees

    // The query rows as the B operand: lane (g, c) holds row 8 n + g in the order in which the codes of lane c come apart.
    uint32_t qb[kCols][kSteps][2];
    float total[kCols][2];   // 4 bits: sums of the elements of rows 8 n + 2 c, 8 n + 2 c + 1
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
        const int r = min(8 * n + g, rows - 1), tok = r / G;
        const __nv_bfloat16* row = p.q + ((size_t)(row0 + tok) * H + kvh * G + (r - tok * G)) * kDim;
        float sum = 0.f;
#pragma unroll
        for (int s = 0; s < kSteps; s += 2) {   // eight elements
            const int d = kBits == 4 ? c * (kDim / 4) + 8 * (s / 2) : (s >> 2) * 64 + 16 * c + 4 * (s & 3);
            const uint4 x = __ldg(reinterpret_cast<const uint4*>(row + d));
            if (kBits == 4) {   // elements (0, 4), (1, 5); (2, 6), (3, 7)
                qb[n][s][0] = __byte_perm(x.x, x.z, 0x5410);
                qb[n][s][1] = __byte_perm(x.x, x.z, 0x7632);
                qb[n][s + 1][0] = __byte_perm(x.y, x.w, 0x5410);
                qb[n][s + 1][1] = __byte_perm(x.y, x.w, 0x7632);
                float f[8];
                unpack8(x, f);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += f[e];
            } else {            // elements (0, 2), (1, 3) of each word of codes
                qb[n][s][0] = __byte_perm(x.x, x.y, 0x5410);
                qb[n][s][1] = __byte_perm(x.x, x.y, 0x7632);
                qb[n][s + 1][0] = __byte_perm(x.z, x.w, 0x5410);
                qb[n][s + 1][1] = __byte_perm(x.z, x.w, 0x7632);
            }
        }
        if (kBits == 4) {
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            total[n][0] = __shfl_sync(0xffffffffu, sum, 8 * c);
            total[n][1] = __shfl_sync(0xffffffffu, sum, 8 * c + 4);
        }
    }

    float m[kCols][2], l[kCols][2], o[kCols][kSteps][4];
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
#pragma unroll
        for (int j = 0; j < 2; ++j) m[n][j] = -INFINITY, l[n][j] = 0.f;
#pragma unroll
        for (int t = 0; t < kSteps; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][t][e] = 0.f;
    }

    int stage = 0, into = kStages - 1;
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
        const uint32_t kt = ring + stage * Shape::kStageBytes, vt = kt + kTileBytes, kp = kt + 2 * kTileBytes, vp = kp + Shape::kParBytes;

        // ---- scores of tokens g and g + 8 for rows 2 c, 2 c + 1
        float s[kCols][4];
#pragma unroll
        for (int n = 0; n < kCols; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
#pragma unroll
        for (int h = 0; h < kKeyLoads; ++h) {
            uint32_t w[2][kKeyWords];
            load_words<kRowBytes>(kt, g, h * 64 + c * (4 * kKeyWords), w[0]);
            load_words<kRowBytes>(kt, g + 8, h * 64 + c * (4 * kKeyWords), w[1]);
#pragma unroll
            for (int x = 0; x < kKeyWords; ++x) {
                if constexpr (kBits == 8) {
                    const uint32_t a[4] = {bytes02(w[0][x]), bytes02(w[1][x]), bytes02(w[0][x] >> 8), bytes02(w[1][x] >> 8)};
#pragma unroll
                    for (int n = 0; n < kCols; ++n) mma16816(s[n], a, qb[n][kKeyWords * h + x][0], qb[n][kKeyWords * h + x][1]);
                } else {
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const uint32_t a[4] = {plus128<0x000F000Fu>(w[0][x] >> (8 * y)), plus128<0x000F000Fu>(w[1][x] >> (8 * y)),
                                               plus128<0x000F000Fu>(w[0][x] >> (8 * y + 4)), plus128<0x000F000Fu>(w[1][x] >> (8 * y + 4))};
#pragma unroll
                        for (int n = 0; n < kCols; ++n) mma16816(s[n], a, qb[n][2 * x + y][0], qb[n][2 * x + y][1]);
                    }
                }
            }
        }
        float v_scale[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = g + 8 * h;
            if constexpr (kBits == 8) {
                const float k_scale = __uint_as_float(lds16(kp + 2 * at) << 16) * p.scale_log2;
                v_scale[h] = __uint_as_float(lds16(vp + 2 * at) << 16);
#pragma unroll
                for (int n = 0; n < kCols; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) s[n][2 * h + j] *= k_scale;
            } else {
                const uint32_t k_par = lds32(kp + 4 * at);
                const float k_scale = __uint_as_float(k_par << 16) * p.scale_log2, zero = -128.f - __uint_as_float(k_par & 0xFFFF0000u);
                v_scale[h] = __uint_as_float(lds32(vp + 4 * at) << 16);
#pragma unroll
                for (int n = 0; n < kCols; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) s[n][2 * h + j] = fmaf(zero, total[n][j], s[n][2 * h + j]) * k_scale;
            }
        }

        // ---- weights
        const int tok = begin + i * kTile;
        const bool masked = tok + kTile > all_see;
        if (masked) {
#pragma unroll
            for (int n = 0; n < kCols; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (tok + g + 8 * (e >> 1) >= see[n][e & 1]) s[n][e] = -INFINITY;
        }
        bool raise = false;
#pragma unroll
        for (int n = 0; n < kCols; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) raise |= fmaxf(s[n][j], s[n][2 + j]) > m[n][j] + 8.f;
        if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
            for (int n = 0; n < kCols; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float now = fmaxf(m[n][j], over_tokens(fmaxf(s[n][j], s[n][2 + j]), [](float a, float b) { return fmaxf(a, b); }));
                    const float keep = now == m[n][j] ? 1.f : fast_exp2(m[n][j] - now);
                    m[n][j] = now;
                    l[n][j] *= keep;
#pragma unroll
                    for (int t = 0; t < kSteps; ++t) {
                        o[n][t][j] *= keep;
                        o[n][t][2 + j] *= keep;
                    }
                }
        }
        uint32_t pb[kCols][2];
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
            float w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float ref = m[n][e & 1] == -INFINITY ? 0.f : m[n][e & 1];
                const float x = fast_exp2(s[n][e] - ref);
                l[n][e & 1] += x;
                w[e] = x * v_scale[e >> 1];
            }
            if (masked) {   // (a scale behind the last token may be anything)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (tok + g + 8 * (e >> 1) >= see[n][e & 1]) w[e] = 0.f;
            }
            pb[n][0] = transpose8(pack2(w[0], w[1]));
            pb[n][1] = transpose8(pack2(w[2], w[3]));
        }

        // ---- weighted values: lane g holds elements g D / 8 ... of the tile's tokens 2 c, 2 c + 1, 2 c + 8, 2 c + 9
        uint32_t w[4][kValWords];
#pragma unroll
        for (int x = 0; x < 4; ++x) load_words<kRowBytes>(vt, 2 * c + (x & 1) + 8 * (x >> 1), g * (4 * kValWords), w[x]);
        if constexpr (kBits == 8) {
#pragma unroll
            for (int x = 0; x < kValWords; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {   // elements 4 x + 2 y, 4 x + 2 y + 1: bytes 0 and 1 of a word of both tokens
                    const uint32_t lo = __byte_perm(w[0][x], w[1][x], y ? 0x7632 : 0x5410), hi = __byte_perm(w[2][x], w[3][x], y ? 0x7632 : 0x5410);
                    const uint32_t a[4] = {bytes02(lo), bytes02(lo >> 8), bytes02(hi), bytes02(hi >> 8)};
#pragma unroll
                    for (int n = 0; n < kCols; ++n) mma16816(o[n][2 * x + y], a, pb[n][0], pb[n][1]);
                }
        } else {
            uint32_t zero[2];   // 128 + zero points of tokens 2 c, 2 c + 1 and 2 c + 8, 2 c + 9
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint2 par = lds64(vp + 4 * (2 * c + 8 * h));
                uint32_t z = __byte_perm(par.x, par.y, 0x7632);
                // (behind the last token it may be anything, and the weight of zero must not meet a NaN)
                asm("min.bf16x2 %0, %0, %1;" : "+r"(z) : "r"(0x41704170u));
                asm("max.bf16x2 %0, %0, %1;" : "+r"(z) : "r"(0u));
                asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(zero[h]) : "r"(z), "r"(0x43004300u));
            }
#pragma unroll
            for (int x = 0; x < kValWords; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {   // half a word of both tokens: elements 8 x + 4 y ...
                    const uint32_t lo = __byte_perm(w[0][x], w[1][x], y ? 0x7632 : 0x5410), hi = __byte_perm(w[2][x], w[3][x], y ? 0x7632 : 0x5410);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t a[4] = {bf2_sub(plus128<0x000F000Fu>(lo >> (8 * e)), zero[0]), bf2_sub(plus128<0x000F000Fu>(lo >> (8 * e + 4)), zero[0]),
                                               bf2_sub(plus128<0x000F000Fu>(hi >> (8 * e)), zero[1]), bf2_sub(plus128<0x000F000Fu>(hi >> (8 * e + 4)), zero[1])};
#pragma unroll
                        for (int n = 0; n < kCols; ++n) mma16816(o[n][4 * x + 2 * y + e], a, pb[n][0], pb[n][1]);
                    }
                }
        }
        stage = stage + 1 == kStages ? 0 : stage + 1;
        into = into + 1 == kStages ? 0 : into + 1;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");

    // join the warps: references and sums first, then the accumulators where the rings were
#pragma unroll
    for (int n = 0; n < kCols; ++n)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            l[n][j] = over_tokens(l[n][j], [](float a, float b) { return a + b; });
            if (g == 0) {
                s_m[warp][8 * n + 2 * c + j] = m[n][j];
                s_l[warp][8 * n + 2 * c + j] = l[n][j];
            }
        }
    __syncthreads();
    float* so = reinterpret_cast<float*>(smem) + (size_t)warp * kRows * kDim;
#pragma unroll
    for (int n = 0; n < kCols; ++n)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = 8 * n + 2 * c + j;
            float most = s_m[0][r];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) most = fmaxf(most, s_m[w][r]);
            const float f = m[n][j] == -INFINITY ? 0.f : fast_exp2(m[n][j] - most);
            if (r < rows) {   // elements g D / 8 + 2 t, 2 t + 1
#pragma unroll
                for (int t = 0; t < kSteps; t += 2)
                    *reinterpret_cast<float4*>(so + r * kDim + g * (kDim / 8) + 2 * t) =
                        make_float4(o[n][t][j] * f, o[n][t][2 + j] * f, o[n][t + 1][j] * f, o[n][t + 1][2 + j] * f);
            }
        }
    if (tid < kRows) {
        float most = s_m[0][tid], sum = 0.f;
        for (int w = 1; w < kWarps; ++w) most = fmaxf(most, s_m[w][tid]);
        // (a reference of -inf: the warp has seen nothing, its sum is zero; or only scores that are NaN, and so is its sum)
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
            const float2 u = *reinterpret_cast<const float2*>(all + (size_t)w * kRows * kDim + at);
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
        float* mine = reinterpret_cast<float*>(smem) + kWarps * kRows * kDim;
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
                part[s] = ld_block(stats + 4 * (kRows + r), from);
                u[s].x = ld_block(here + 4 * at, from);
                u[s].y = ld_block(here + 4 * at + 4, from);
                most = fmaxf(most, top[s]);
            }
#pragma unroll
            for (int s = 0; s < kMostTogether; ++s) {
                const float f = s >= parts || top[s] == -INFINITY ? 0.f : fast_exp2(top[s] - most);
                if (s < parts) {
                    sum = fmaf(part[s], f, sum);
                    v.x = fmaf(u[s].x, f, v.x);
                    v.y = fmaf(u[s].y, f, v.y);
                }
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
    // a part: few_rows x kDim accumulators, then few_rows references and few_rows sums
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

template <int kDim, int kBits, int kCols, bool kTogether>
qil_status go(const AttnQuantParams& p, cudaStream_t st) {
    constexpr int kJoin = (kWarps + 1) * 8 * kCols * kDim * 4, kRing = kWarps * FewQ<kDim, kBits>::kWarpBytes, kSmem = kJoin > kRing ? kJoin : kRing;
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(attn_few_q_kernel<kDim, kBits, kCols, kTogether>, kSmem, allowed)) return QIL_ERR_CUDA;
    const int slots = p.a.slots;
    const unsigned across = !kTogether ? (unsigned)slots : slots <= 2 ? 2u : slots <= 4 ? 4u : (unsigned)kMostTogether;
    const dim3 grid(across, (unsigned)p.a.c.num_kv_heads, (unsigned)(p.a.c.num_seqs + p.a.both));
    return launch_early_clusters(attn_few_q_kernel<kDim, kBits, kCols, kTogether>, kTogether ? across : 1u, grid, 32 * kWarps, kSmem, st, p);
}

template <int kDim, int kBits>
qil_status go(const AttnQuantParams& p, cudaStream_t st) {
    if (p.a.few_rows <= 8) return p.a.together ? go<kDim, kBits, 1, true>(p, st) : go<kDim, kBits, 1, false>(p, st);
    return p.a.together ? go<kDim, kBits, 2, true>(p, st) : go<kDim, kBits, 2, false>(p, st);
}

}  // namespace

qil_status launch_attn_few_q(const AttnQuantParams& p, cudaStream_t st) {
    if (p.a.c.head_dim == 128) return p.kv.bits == 8 ? go<128, 8>(p, st) : go<128, 4>(p, st);
    return p.kv.bits == 8 ? go<64, 8>(p, st) : go<64, 4>(p, st);
}

}  // namespace qil
