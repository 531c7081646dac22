// Attention over the quantised paged cache for requests with few query rows (new tokens x heads of a group <= 16): single
// tokens and short drafts.  Memory bound: every cached code is read once per key head.
//
// As in attn_few.cu a block takes `chunk` cached tokens of one request and key head, its four warps take tiles of 16 tokens in
// turn, each with its own ring in shared memory, and blocks of a request are joined in a cluster or through the workspace.
// What differs is what a tile costs apart from its bytes, a half or a quarter of those of bf16:
//   S^T = K Q^T and O^T += V^T P^T: the cache is the 16-row operand of mma.sync and the query rows are the 8 columns, so that up
//   to 8 rows take half the products and accumulators of a tile of 16 rows.
//   The integer pipe (masks, shifts, byte selects) is what a tile of codes would be bound by, so keys meet the queries as they
//   are, in whole numbers: a query row is t (256 h + l) with h and l of 8 bits (off by 2^-16 of the row's largest element at
//   most), its scores are exact int32 sums, 256 (k . h) + k . l less the zero point times the row's sum.
//   Values become bf16 in registers by a few logic operations, exactly.  The operands' columns may be in any order as long as
//   both sides agree, so a lane's codes are 16 bytes or less in one piece, and the words come apart in the order that needs the
//   fewest operations.
//   A key's scale multiplies its scores, a value's scale its weight.
//   The running reference of a row is only raised by scores more than 2^8 above it, which a vote finds; maxima are reduced
//   over the lanes in those tiles alone, sums once at the end.
//   Tiles of 64 bytes a token or less come two to a turn, which halves what a turn costs besides its codes.
// A weight times its value's scale is rounded to bf16 for the product (by 2^-8 of it at most, of either sign): outputs are off by
// 0.0023 of their size, 0.0017 of which are their own rounding.
// Codes are finite whatever they are, so nothing behind a request's last token can reach a result: its weight is replaced by
// zero after its scale has been applied.
//
// Measured (one B200): 8 bits, 32 requests of up to 4099 tokens, 32 key heads of 128 (0.70 GB): 117 to 132 us, 81 to 91 % of the
// copy rate.  4 bits, 48 requests of up to 9001 tokens, 8 key heads (0.28 GB): 79 to 81 us, 54 %: 360 warp instructions a tile of 16
// tokens, 167 of them on the integer pipe, which would take 41 us alone; the rest is latency and blocks of unequal length (the
// SMs are busy for 81 % of the time on average).  Tried and slower: blocks of 1, 2 and 8 warps (171, 95, 85 us), blocks of 768, 512 or
// 384 tokens (83, 92, 101 us: a block's start and join cost 5 us), shifts as multiplications (100 us).  Batches of middling size
// wait for the chain of a turn, about 1400 cycles where an SM holds few warps: 24 requests of up to 2000 tokens, 8 key heads, 4 bits
// 17.5 us (4.6 at the copy rate).
#include "attn_paged_q.cuh"

namespace qil {

namespace {

constexpr int kWarps = 4, kTile = 16;

template <int kDim, int kBits>
struct FewQ {
    static constexpr int kRowBytes = kDim * kBits / 8;               // 128, 64, 64, 32
    static constexpr int kTileBytes = kTile * kRowBytes;
    static constexpr int kParBytes = kTile * (kBits == 8 ? 2 : 4);   // of one side
    static constexpr int kSub = kRowBytes <= 64 ? 2 : 1;             // tiles of one turn of the loop
    static constexpr int kSubBytes = 2 * kTileBytes + 2 * kParBytes;
    static constexpr int kStageBytes = kSub * kSubBytes;
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

// D[16 x 8] += A[16 x 32] B[32 x 8], signed bytes, int32 accumulators
__device__ __forceinline__ void mma16832(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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

// A block of a request, from its rows and the pages of its warps' first tiles on.  kCols: columns of 8 query rows.  kTogether: the
// blocks of a request and key head are one cluster.
template <int kDim, int kBits, int kCols, bool kTogether>
__device__ __forceinline__ void attend(const AttnQuantParams& pq, unsigned char* smem, int (&page)[FewQ<kDim, kBits>::kSub], int kv, int row0, int q_len) {
    using Shape = FewQ<kDim, kBits>;
    constexpr int kSub = Shape::kSub, kTurn = kSub * kTile;   // tokens of a turn
    constexpr int kStages = Shape::kStages, kRowBytes = Shape::kRowBytes, kTileBytes = Shape::kTileBytes, kSteps = Shape::kSteps;
    constexpr int kRows = 8 * kCols, kKeyWords = kRowBytes >= 64 ? 4 : 2, kKeyLoads = kRowBytes == 128 ? 2 : 1, kValWords = kRowBytes / 32;
    const AttnParams& p = pq.a;
    __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows];
    __shared__ float s_scale[2][kRows];
    __shared__ int s_last;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    const int split = blockIdx.x, kvh = blockIdx.y, seq = blockIdx.z, G = p.G, H = p.c.num_heads;
    const int begin = split * p.chunk;
    const int* table = p.c.block_table + (size_t)seq * p.c.max_pages;
    const int rows = q_len * G, end = cache_end(p.c, kv), first_pos = kv - q_len;
    const int parts = max(1, min((end + p.chunk - 1) / p.chunk, p.slots));
    const bool idle = split >= parts;
    if (idle && !kTogether) return;
    const int stop = idle ? begin : split + 1 == parts ? end : min(begin + p.chunk, end);
    const int turns = (stop - begin + kTurn - 1) / kTurn;

    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * Shape::kWarpBytes;
    auto pages_of = [&](int i, int (&to)[kSub]) {   // of the tiles of turn i (of the last token where there are none)
#pragma unroll
        for (int u = 0; u < kSub; ++u) to[u] = __ldg(table + (min(begin + i * kTurn + u * kTile, stop - 1) >> p.page_shift));
    };
    auto fetch = [&](int i, int stage, const int (&page)[kSub]) {
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
            const int tok = begin + i * kTurn + u * kTile;
            const uint32_t bytes = page[u] >= 0 && page[u] < p.c.num_pages ? 16u : 0u;   // (a page that does not exist: zeros)
            const size_t at = bytes ? ((size_t)page[u] * p.c.num_kv_heads + kvh) * p.c.page_size + (tok & (p.c.page_size - 1)) : 0;   // a row of the cache
            const uint32_t dst = ring + stage * Shape::kStageBytes + u * Shape::kSubBytes;
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
        }
    };
    int ahead = warp;               // the next turn to fetch
    auto fetch_ahead = [&](int stage) {
        if (ahead < turns) {
            int next[kSub];
            pages_of(ahead + kWarps, next);   // (asked for one turn ahead of its use)
            fetch(ahead, stage, page);
#pragma unroll
            for (int u = 0; u < kSub; ++u) page[u] = next[u];
        }
        ahead += kWarps;
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) fetch_ahead(s);

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
    constexpr int kKSteps = kDim / 32;
    uint32_t qh[kCols][kKSteps][2], ql[kCols][kKSteps][2];
    float unit[kCols][2];   // t of rows 8 n + 2 c, 8 n + 2 c + 1, times the scale of the scores
    int total[kCols][2];    // 4 bits: sums of their whole numbers
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
        const int r = min(8 * n + g, rows - 1), tok = r / G;
        const __nv_bfloat16* row = p.q + ((size_t)(row0 + tok) * H + kvh * G + (r - tok * G)) * kDim;
        uint4 x[kKSteps];   // elements of this lane, eight to a step
        float most = 0.f, nan = 0.f;   // (nan: zero, or a NaN where an element is not finite)
#pragma unroll
        for (int k = 0; k < kKSteps; ++k)
            x[k] = __ldg(reinterpret_cast<const uint4*>(row + (kBits == 4 ? c * (kDim / 4) + 8 * k : (k >> 1) * 64 + 16 * c + 8 * (k & 1))));
#pragma unroll
        for (int k = 0; k < kKSteps; ++k) {
            float f[8];
            unpack8(x[k], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                most = fmaxf(most, fabsf(f[e]));
                nan = fmaf(f[e], 0.f, nan);
            }
        }
        most = nan == 0.f ? most : INFINITY;
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        // (a row of numbers near fp32's smallest counts as zeros; one with an element that is none has no scores)
        const bool whole = most > 1e-30f && most < INFINITY;
        const float up = whole ? 32512.f / most : 0.f;   // (once a row; the fast division gives zero above 2^126)
        float t = whole ? most * (1.f / 32512.f) : most < INFINITY ? 0.f : INFINITY - INFINITY;
        if (!whole) {   // (0 times an element that is no number)
#pragma unroll
            for (int k = 0; k < kKSteps; ++k) x[k] = make_uint4(0u, 0u, 0u, 0u);
        }
        // v = rint(f up) as the low bits of 1.5 2^23 + v: its lowest byte is l, and the next one of v + 128 is h
        uint32_t bits = 0u;
#pragma unroll
        for (int k = 0; k < kKSteps; ++k) {
            float f[8];
            uint32_t lo[8], hi[8];
            unpack8(x[k], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = fmaf(f[e], up, 12582912.f);
                lo[e] = __float_as_uint(v);
                hi[e] = __float_as_uint(v + 128.f);
                bits += lo[e];
            }
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                // 4 bits: elements 0, 2, 4, 6 of a word of codes, then the others; 8 bits: those of one word, then of the next
                const int a = kBits == 4 ? w : 4 * w, b = kBits == 4 ? 2 : 1;
                ql[n][k][w] = __byte_perm(__byte_perm(lo[a], lo[a + b], 0x0040), __byte_perm(lo[a + 2 * b], lo[a + 3 * b], 0x0040), 0x5410);
                qh[n][k][w] = __byte_perm(__byte_perm(hi[a], hi[a + b], 0x0051), __byte_perm(hi[a + 2 * b], hi[a + 3 * b], 0x0051), 0x5410);
            }
        }
        int sum = (int)(bits - (uint32_t)(kKSteps * 8) * 0x4B400000u);
        t *= p.scale_log2;
        unit[n][0] = __shfl_sync(0xffffffffu, t, 8 * c);
        unit[n][1] = __shfl_sync(0xffffffffu, t, 8 * c + 4);
        if (kBits == 4) {
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            total[n][0] = __shfl_sync(0xffffffffu, sum, 8 * c);
            total[n][1] = __shfl_sync(0xffffffffu, sum, 8 * c + 4);
        }
    }

    float m[kCols][2], ref[kCols][2], l[kCols][2], o[kCols][kSteps][4];   // (ref: m, or zero before anything is seen)
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
#pragma unroll
        for (int j = 0; j < 2; ++j) m[n][j] = -INFINITY, ref[n][j] = l[n][j] = 0.f;
#pragma unroll
        for (int t = 0; t < kSteps; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][t][e] = 0.f;
    }

    int stage = 0, into = kStages - 1;
    for (int i = warp; i < turns; i += kWarps) {
        __syncwarp();               // every lane has read what the next fetch overwrites
        fetch_ahead(into);
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
        __syncwarp();
        const uint32_t turn = ring + stage * Shape::kStageBytes;

        // ---- scores of tokens g and g + 8 of each tile for rows 2 c, 2 c + 1
        float s[kSub][kCols][4], v_scale[kSub][2];
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
            const uint32_t kt = turn + u * Shape::kSubBytes, kp = kt + 2 * kTileBytes, vp = kp + Shape::kParBytes;
            uint32_t ka[kKSteps][4];
#pragma unroll
            for (int h = 0; h < kKeyLoads; ++h) {
                uint32_t w[2][kKeyWords];
                load_words<kRowBytes>(kt, g, h * 64 + c * (4 * kKeyWords), w[0]);
                load_words<kRowBytes>(kt, g + 8, h * 64 + c * (4 * kKeyWords), w[1]);
#pragma unroll
                for (int x = 0; x < kKeyWords; ++x) {
                    if constexpr (kBits == 8) {
                        ka[(kKeyWords * h + x) >> 1][2 * (x & 1)] = w[0][x];
                        ka[(kKeyWords * h + x) >> 1][2 * (x & 1) + 1] = w[1][x];
                    } else {
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            ka[x][y] = w[y][x] & 0x0F0F0F0Fu;
                            ka[x][2 + y] = (w[y][x] >> 4) & 0x0F0F0F0Fu;
                        }
                    }
                }
            }
            int acc[kCols][2][4];
#pragma unroll
            for (int n = 0; n < kCols; ++n) {
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[n][0][e] = acc[n][1][e] = 0;
#pragma unroll
                for (int k = 0; k < kKSteps; ++k) {
                    mma16832(acc[n][0], ka[k], qh[n][k][0], qh[n][k][1]);
                    mma16832(acc[n][1], ka[k], ql[n][k][0], ql[n][k][1]);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = g + 8 * h;
                float k_scale;
                int zero = 0;
                if constexpr (kBits == 8) {
                    k_scale = __uint_as_float(lds16(kp + 2 * at) << 16);
                    v_scale[u][h] = __uint_as_float(lds16(vp + 2 * at) << 16);
                } else {
                    const uint32_t k_par = lds32(kp + 4 * at);
                    k_scale = __uint_as_float(k_par << 16);
                    zero = __float2int_rn(__uint_as_float(k_par & 0xFFFF0000u));
                    v_scale[u][h] = __uint_as_float(lds32(vp + 4 * at) << 16);
                }
#pragma unroll
                for (int n = 0; n < kCols; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int whole = acc[n][0][2 * h + j] * 256 + acc[n][1][2 * h + j];
                        s[u][n][2 * h + j] = (float)(kBits == 8 ? whole : whole - zero * total[n][j]) * (k_scale * unit[n][j]);
                    }
            }
        }

        // ---- weights
        const int tok = begin + i * kTurn;
        const bool masked = tok + kTurn > all_see;
        const auto hidden = [&](int u, int n, int e) { return tok + kTile * u + g + 8 * (e >> 1) >= see[n][e & 1]; };
        if (masked) {
#pragma unroll
            for (int u = 0; u < kSub; ++u)
#pragma unroll
                for (int n = 0; n < kCols; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (hidden(u, n, e)) s[u][n][e] = -INFINITY;
        }
        float top[kCols][2];
        bool raise = false;
#pragma unroll
        for (int n = 0; n < kCols; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                top[n][j] = fmaxf(s[0][n][j], s[0][n][2 + j]);
#pragma unroll
                for (int u = 1; u < kSub; ++u) top[n][j] = fmaxf(top[n][j], fmaxf(s[u][n][j], s[u][n][2 + j]));
                raise |= top[n][j] > m[n][j] + 8.f;
            }
        if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
            for (int n = 0; n < kCols; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float now = fmaxf(m[n][j], over_tokens(top[n][j], [](float a, float b) { return fmaxf(a, b); }));
                    const float keep = now == m[n][j] ? 1.f : fast_exp2(m[n][j] - now);
                    m[n][j] = now;
                    ref[n][j] = now == -INFINITY ? 0.f : now;
                    l[n][j] *= keep;
#pragma unroll
                    for (int t = 0; t < kSteps; ++t) {
                        o[n][t][j] *= keep;
                        o[n][t][2 + j] *= keep;
                    }
                }
        }
        uint32_t pb[kSub][kCols][2];
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int n = 0; n < kCols; ++n) {
                float w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = fast_exp2(s[u][n][e] - ref[n][e & 1]);
                    l[n][e & 1] += x;
                    w[e] = x * v_scale[u][e >> 1];
                }
                if (masked) {   // (a scale behind the last token may be anything)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (hidden(u, n, e)) w[e] = 0.f;
                }
                pb[u][n][0] = transpose8(pack2(w[0], w[1]));
                pb[u][n][1] = transpose8(pack2(w[2], w[3]));
            }

        // ---- weighted values: lane g holds elements g D / 8 ... of a tile's tokens 2 c, 2 c + 1, 2 c + 8, 2 c + 9
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
            const uint32_t vt = turn + u * Shape::kSubBytes + kTileBytes, vp = vt + kTileBytes + Shape::kParBytes;
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
                        for (int n = 0; n < kCols; ++n) mma16816(o[n][2 * x + y], a, pb[u][n][0], pb[u][n][1]);
                    }
            } else {
                uint32_t zero[2];   // 128 + zero points of tokens 2 c, 2 c + 1 and 2 c + 8, 2 c + 9
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint2 par = lds64(vp + 4 * (2 * c + 8 * h));
                    uint32_t z = __byte_perm(par.x, par.y, 0x7632);
                    if (masked) {   // (behind the last token it may be anything, and the weight of zero must not meet a NaN)
                        asm("min.bf16x2 %0, %0, %1;" : "+r"(z) : "r"(0x41704170u));
                        asm("max.bf16x2 %0, %0, %1;" : "+r"(z) : "r"(0u));
                    }
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
                            for (int n = 0; n < kCols; ++n) mma16816(o[n][4 * x + 2 * y + e], a, pb[u][n][0], pb[u][n][1]);
                        }
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

// kMostCols: columns of the request with the most rows.  In a kernel of two columns a block takes one where its request has no
// more than eight rows (single tokens beside prompts, grouped heads).
template <int kDim, int kBits, int kMostCols, bool kTogether>
__global__ void __launch_bounds__(32 * kWarps, kMostCols == 1 ? 4 : 3) attn_few_q_kernel(const AttnQuantParams pq) {
    constexpr int kSub = FewQ<kDim, kBits>::kSub;
    const AttnParams& p = pq.a;
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = threadIdx.x >> 5, split = blockIdx.x, kvh = blockIdx.y, seq = blockIdx.z;
    // (beside the kernel for many rows, as in attn_few.cu)
    if (!p.both) wait_for_earlier_kernels();
    if (seq == p.c.num_seqs) {
        if (split == 0 && kvh == 0) wait_for_earlier_kernels();
        return;
    }
    const int begin = split * p.chunk;
    const int* table = p.c.block_table + (size_t)seq * p.c.max_pages;
    const int kv = __ldg(p.c.kv_len + seq);
    int page[kSub];
#pragma unroll
    for (int u = 0; u < kSub; ++u) page[u] = __ldg(table + min((begin + (warp * kSub + u) * kTile) >> p.page_shift, p.c.max_pages - 1));
    int row0, row1;
    request_rows(p.c.cu_q, seq, p.c.total_q, row0, row1);
    const int q_len = row1 - row0;
    if (q_len <= 0 || q_len * (long long)p.G > kFewRows) return;
    // a request with more rows than the bound says is left out
    const int rows = q_len * p.G;
    if (rows > 8 * kMostCols || (!kTogether && p.slots > 1 && rows > p.few_rows)) return;
    if (kMostCols == 1 || rows <= 8) attend<kDim, kBits, 1, kTogether>(pq, smem, page, kv, row0, q_len);
    else attend<kDim, kBits, kMostCols, kTogether>(pq, smem, page, kv, row0, q_len);
}

template <int kDim, int kBits, int kCols, bool kTogether>
qil_status go(const AttnQuantParams& p, cudaStream_t st) {
    constexpr int kJoin = (kWarps + 1) * 8 * kCols * kDim * 4, kRing = kWarps * FewQ<kDim, kBits>::kWarpBytes, kSmem = kJoin > kRing ? kJoin : kRing;
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(attn_few_q_kernel<kDim, kBits, kCols, kTogether>, kSmem, allowed)) return QIL_ERR_CUDA;
    // (a cluster of as many blocks as have work, 2 to 8: one more would hold its place until the others are done)
    const unsigned across = (unsigned)p.a.slots;
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
