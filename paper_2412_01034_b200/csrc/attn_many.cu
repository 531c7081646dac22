// Attention over the paged cache for requests with many query rows (prompts, chunks of a prompt): tcgen05.mma with the
// scores, the weights and the output accumulators in tensor memory.
//
// A block takes up to 256 query rows of one request and key head as two tiles of 128 rows (whole tokens: 128 / G of them,
// so that one bulk tensor copy fetches a tile's queries for any group size), and walks the cache in tiles of
// 128 tokens.  Per tile of tokens and tile i of rows:
//   S_i = Q_i K^T      128 x 128 x D, both operands in shared memory, fp32 in tensor memory
//   P_i = exp2(S_i c - m)   by the 128 threads of group i, one row each: tcgen05.ld, running maximum and sum in registers,
//                           weights rounded to bf16 and stored with tcgen05.st over S_i's own columns
//   O_i += P_i V       A from tensor memory, V as it lies in the cache ([token][D]: the N-major operand)
// The two tiles take turns: while a group turns S_0 into P_0 the tensor pipe multiplies for tile 1.  Tensor memory is full
// at D = 128 (two S of 128 columns, two O of 128).
// The maximum that the weights refer to is only raised when a row's score exceeds it by more than 2^8; the sums stay
// far from fp32's limits and bf16 rounds relatively, so nothing is lost, and O_i is rescaled (by the group itself, between
// products) a few times instead of once per tile.
// The weights are bf16 because V is (a product's operands have one type); a second term for their lower bits would add half
// of the products' time to a kernel that waits for them.  Outputs are off by 0.0019 to 0.0023 of their size, 0.0017 of which
// are their own rounding.
// One warp copies pages with bulk tensor copies (128-byte swizzle), one thread issues the products, one warp clears what
// lies behind a request's last token in its last tile of V (a weight of zero times NaN would be NaN).
// A row of a new token that comes before one whose value is infinite or NaN meets that value all the same: rows whose results
// are not finite are looked at once more at the end, and summed again where that was the reason (no time where there are none:
// 24.5 us for four 280-token prompts with the look and without).
// Every wait is bounded; when one runs out QIL_ERR_TIMEOUT is recorded and the block ends.
//
// Measured, 4096 new tokens over 8192, 32 heads of 128 (412 GFLOP): 368 us (1120 TFLOP/s) until the power cap sets in, 396 to
// 430 us (960 to 1040 TFLOP/s at 1.65 GHz, 1000 W) sustained.  A step (128 tokens, both row tiles) takes 2830 cycles; the
// products alone would take 2048 (32 of 128 x 128 x 16, 64 cycles each), and the exponentials of both tiles 2048 on the
// special-function units as well.  Per tile: 1660 cycles from S to P, 1130 waiting (half of the product, S, and their
// latencies; the issuing thread needs 64 cycles a product, as long as the pipe does).  Tried and slower: part of the
// exponentials as a polynomial on the multiply-add pipe (454 to 543 us: more instructions, and the power cap), polling
// instead of suspended waits, blocks that stay and take tiles from a counter (no change: the start of a block, 7600 cycles,
// is the copies of all blocks starting at once).
//
// A cache of 8 or 4-bit codes (kBits): the same products in fp16, which holds what 8 or 4 bits and a scale of 8 give to 2^-11
// where bf16 would give 2^-8 (0.0034 of an output's size instead of 0.0017 with scores of ordinary size; a key's rounding grows with
// the scores, and with queries 30 times as large it is 0.0023), at the same rate.  So that fp16's range holds them
// the values are divided by a power of two of the largest scale that the block's tokens have, and a query row by one of its
// largest element; the products' results are multiplied back with the scores' factor and at the end.
//   A fourth group of 128 threads decodes: thread t takes token t of a tile, a key's codes to a tile of K and a value's to one of
//   V, in the layout that the copies would have written, two tiles of each ahead of the products.  It reads 128-byte rows from a
//   ring that bulk copies fill, shorter ones straight from memory into registers one step ahead (a row is at most one line, so
//   nothing is read twice; staging them costs 8 % more).  Its registers come from the producing warps (setmaxnreg).
//   Codes mean finite values: nothing is cleared behind the last token, and a NaN scale there is replaced.
// Measured, 4096 new tokens over 8192, 32 heads of 128: 8 bits 474 to 536 us (770 to 870 TFLOP/s), 4 bits 512 to 560, against 365
// to 410 for bf16 pages in the same minutes.  Every block decodes all tiles of its key head that its rows see, so that 16 blocks
// decode the same ones here.  The products' thread is the longest path of a step, 3600 of 4300 cycles: the decoded tiles' stores
// meet the products' reads of shared memory.  Tried and slower: 128-byte rows without the ring (730 us).  At 128 registers a
// thread at launch the instances spill 16 bytes (8 bits, D = 128) to 102 (8 bits, D = 64); those for bf16 pages 32.
#include <cuda.h>

#include <mutex>

#include "attn_paged_q.cuh"

namespace qil {

namespace {

constexpr int kRows = kTileRows, kTok = 128;
constexpr unsigned long long kWaitLimitNs = 2000000000ull;
constexpr float kMostSum = 16384.f;   // 64 weights of 2^kRaise
constexpr float kRaise = 8.f;   // log2 by which a score may exceed the reference maximum

template <int kDim, int kBits>
struct ManyShape {
    static constexpr int kHalves = kDim / 64;                 // 64 columns (128 bytes) per swizzled half
    static constexpr int kTileBytes = kTok * kDim * 2;        // Q_i, K and V tiles: 128 rows each
    static constexpr int kHalfBytes = kTok * 128;
    static constexpr int kStages = kDim == 128 ? 2 : 4;
    static constexpr int kRowBytes = kBits == 16 ? 0 : kDim * kBits / 8;   // of codes
    // Rows of 128 bytes of codes come through shared memory, a tile of keys and one of values at a time; shorter ones straight into
    // the registers of the warps that decode them (4096 tokens over 8192, 32 heads of 128: 8 bits 490 us staged, 730 direct, where
    // two tiles would take 64 registers a thread; 4 bits 542 staged, 515 direct).
    static constexpr bool kStaged = kRowBytes == 128;
    static constexpr int kBars = 2 * kTileBytes + 2 * kStages * kTileBytes + (kStaged ? 2 * kTok * kRowBytes : 0);
    static constexpr int kSmem = kBars + 1024 + (kBits == 16 ? 256 : 512);
    static constexpr uint32_t kO = 256;                       // tensor memory: S_0, S_1 at 0, 128; O_0, O_1 behind them
    static_assert(kO + 2 * kDim <= 512, "tensor memory");
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// The thread may be suspended while it waits, up to a limit of the hardware's.
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded wait: false when the limit ran out.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity) {
    if (mbar_try(bar, parity)) return true;
    unsigned long long t0 = 0, t;
#pragma unroll 1
    for (uint32_t i = 0;; ++i) {
        if (mbar_try(bar, parity)) return true;
        if ((i & 15u) == 0u) {
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
            if (i == 0u) t0 = t;
            else if (t - t0 > kWaitLimitNs) return false;
        }
    }
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// D[128 x N] (+)= A B: A in shared memory (descriptor) or in tensor memory, B in shared memory.  Descriptors come as halves.
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 ad, bd;\n\tsetp.ne.b32 p, %6, 0;\n\tmov.b64 ad, {%1, %2};\n\tmov.b64 bd, {%3, %4};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], ad, bd, %5, p;\n\t}"
        ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 bd;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 bd, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], bd, %4, p;\n\t}"
        ::"r"(d), "r"(a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(acc) : "memory");
}

#define QIL_R8(v, o) "=r"(v[o]), "=r"(v[o + 1]), "=r"(v[o + 2]), "=r"(v[o + 3]), "=r"(v[o + 4]), "=r"(v[o + 5]), "=r"(v[o + 6]), "=r"(v[o + 7])
#define QIL_I8(v, o) "r"(v[o]), "r"(v[o + 1]), "r"(v[o + 2]), "r"(v[o + 3]), "r"(v[o + 4]), "r"(v[o + 5]), "r"(v[o + 6]), "r"(v[o + 7])
// 32 consecutive 32-bit columns of this thread's lane of tensor memory (no wait)
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
        "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : QIL_R8(v, 0), QIL_R8(v, 8), QIL_R8(v, 16), QIL_R8(v, 24) : "r"(taddr));
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
        "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        ::"r"(taddr), QIL_I8(v, 0), QIL_I8(v, 8), QIL_I8(v, 16), QIL_I8(v, 24) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : QIL_R8(v, 0), QIL_R8(v, 8) : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(taddr), QIL_I8(v, 0), QIL_I8(v, 8) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
template <int n>
__device__ __forceinline__ void pin(uint32_t (&v)[n]) {   // the values exist only after the wait before this
#pragma unroll
    for (int j = 0; j < n; ++j) asm volatile("" : "+r"(v[j]));
}

// Two fp32 values in a register pair: the packed forms of add and multiply-add issue once for both.
__device__ __forceinline__ unsigned long long f2(float a, float b) {
    unsigned long long v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ void f2_split(unsigned long long v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ unsigned long long f2_fma(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ unsigned long long f2_add(unsigned long long a, unsigned long long b) {
    unsigned long long d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// Pairs of row tiles (of `tokens` new tokens each) over the requests with more than kFewRows rows; the later (longer) tiles
// of a request come first.
__device__ __forceinline__ bool find_pair(const PagedCache& c, int G, int tokens, int t, int& seq, int& lo, int& hi, int& pair) {
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int base = 0; base < c.num_seqs; base += 32) {
        int a = 0, b = 0;
        if (base + lane < c.num_seqs) request_rows(c.cu_q, base + lane, c.total_q, a, b);
        const int n = (b - a) * G > kFewRows ? (b - a + 2 * tokens - 1) / (2 * tokens) : 0;
        int incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += up;
        }
        const unsigned past = __ballot_sync(0xffffffffu, before + incl > t);
        if (past) {
            const int who = __ffs(past) - 1;
            const int last = before + __shfl_sync(0xffffffffu, incl, who) - 1;
            seq = base + who;
            lo = __shfl_sync(0xffffffffu, a, who);
            hi = __shfl_sync(0xffffffffu, b, who);
            pair = last - t;
            return true;
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
    }
    return false;
}

// Codes as fp16 values, one rounding each: eight of them (16 bytes of the result).  1024 + n is 0x6400 | n for n < 1024.
__device__ __forceinline__ uint32_t h2_sub(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t h2_mul(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t h2_fma(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
template <uint32_t mask>
__device__ __forceinline__ uint32_t plus1024(uint32_t x) {   // (x & mask) | 0x64006400
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(x), "n"(mask), "n"(0x64006400u));
    return d;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ uint4 values_of_bytes(uint32_t a, uint32_t b, uint32_t scale2) {
    const auto pair = [&](uint32_t w, uint32_t pick) {   // 1024 + 128 + code, less 1152
        return h2_mul(h2_sub(__byte_perm(w ^ 0x80808080u, 0x64646464u, pick), 0x64806480u), scale2);
    };
    return make_uint4(pair(a, 0x4140), pair(a, 0x4342), pair(b, 0x4140), pair(b, 0x4342));
}
// zero2: 1024 + zero point, twice; zero16: -(64 + zero point), twice
__device__ __forceinline__ uint4 values_of_nibbles(uint32_t w, uint32_t zero2, uint32_t zero16, uint32_t scale2) {
    uint32_t x[4];   // elements (e, e + 4)
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
        x[e] = h2_mul(h2_sub(plus1024<0x000F000Fu>(w >> (4 * e)), zero2), scale2);
        x[e + 1] = h2_mul(h2_fma(plus1024<0x00F000F0u>(w >> (4 * e)), 0x2C002C00u, zero16), scale2);   // (1024 + 16 code) / 16
    }
    return make_uint4(__byte_perm(x[0], x[1], 0x5410), __byte_perm(x[2], x[3], 0x5410), __byte_perm(x[0], x[1], 0x7632), __byte_perm(x[2], x[3], 0x7632));
}
// the weights of two tokens in the operands' type
template <int kBits>
__device__ __forceinline__ uint32_t pack_weights(float lo, float hi) { return kBits == 16 ? pack2(lo, hi) : pack_half2(lo, hi); }

// Threads: warp 0 copies, warp 1 issues the products, warp 2 clears (warp 3 idles); with a quantised cache four more warps
// decode it into the operands' tiles; then the two softmax groups.
template <int kBits>
constexpr int kThreadsOf = kBits == 16 ? 384 : 512;

template <int kDim, int kBits>
__global__ void __launch_bounds__(kThreadsOf<kBits>, 1) attn_many_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                                                                         const __grid_constant__ CUtensorMap map_v, const AttnParams p, const QuantCache kvq) {
    using Shape = ManyShape<kDim, kBits>;
    constexpr int kGroups = kBits == 16 ? 4 : 8;   // the first warp of the softmax groups
    // registers of a thread of the four warps at the front, of those that decode, of the softmax groups (512 with four groups)
    constexpr int kFrontRegs = kBits == 16 ? 80 : Shape::kStaged ? 40 : 48, kDecodeRegs = Shape::kStaged ? 104 : 112,
                  kSoftmaxRegs = kBits == 16 ? 208 : Shape::kStaged ? 184 : 176;
    static_assert(kBits == 16 || kFrontRegs + kDecodeRegs + 2 * kSoftmaxRegs <= 512, "no more than the block was launched with");
    constexpr int kStages = Shape::kStages, kTileBytes = Shape::kTileBytes, kHalfBytes = Shape::kHalfBytes, kHalves = Shape::kHalves;
    extern __shared__ unsigned char smem_raw[];
    wait_for_earlier_kernels();
    if (p.both) let_next_kernel_start();   // (the kernel for few rows fills the SMs that this one leaves)
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = p.G, H = p.c.num_heads, kvh = blockIdx.x % p.c.num_kv_heads;
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t sq = smem_u32(smem), sk = sq + 2 * kTileBytes, sv = sk + kStages * kTileBytes;
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + Shape::kBars);
    const uint32_t q_full = smem_u32(bars), s_full = q_full + 16, p_full = q_full + 32, o_done = q_full + 64, v_raw = q_full + 80,
                   drain = q_full + 88, k_full = q_full + 96, v_full = k_full + 8 * kStages, k_free = v_full + 8 * kStages, q_ready = k_free + 8 * kStages + 8, e_full = q_ready + 16, raw_full = e_full + 8,
                   raw_free = raw_full + 16;   // (before q_ready: where tensor memory is)
    int* exponents = reinterpret_cast<int*>(bars + 48);   // (a quantised cache; behind the barriers)
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 12 + 3 * kStages);
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(q_full + 8 * i, 1);       // the copy of Q_i
            mbar_init(s_full + 8 * i, 1);       // commit after S_i
            mbar_init(p_full + 16 * i, 4);      // the group's warps: weights of the first 64 tokens
            mbar_init(p_full + 16 * i + 8, 4);  // and of the others
            mbar_init(o_done + 8 * i, 1);       // commit after the last product of tile i
        }
        mbar_init(v_raw, 1);                    // the copy of a V tile whose last tokens are still to be cleared
        mbar_init(drain, 1);
        for (int i = 0; i < 2 && kBits != 16; ++i) {
            mbar_init(q_ready + 8 * i, 4);      // the group's warps: Q_i in fp16
            mbar_init(raw_full + 8 * i, 1);     // the copy of a tile of codes
            mbar_init(raw_free + 8 * i, 4);     // the decoding warps
        }
        if (kBits != 16) mbar_init(e_full, 4);  // the decoding warps: exponents of keys and values
        for (int s = 0; s < kStages; ++s) {
            mbar_init(k_full + 8 * s, kBits == 16 ? 1 : 4);   // a copy, or the decoding warps
            mbar_init(v_full + 8 * s, kBits == 16 ? 1 : 4);
            mbar_init(k_free + 8 * s, 1);       // commit after the last S of a K tile
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
    }
    int seq = 0, q_lo = 0, q_hi = 0, pair = 0;
    const bool found = find_pair(p.c, G, p.tile_tokens, blockIdx.x / p.c.num_kv_heads, seq, q_lo, q_hi, pair);
    // row r of tile i is new token (2 pair + i) tile_tokens + r / G, query head kvh G + r % G; `tokens` of them are the request's
    const int token0 = pair * 2 * p.tile_tokens;
    const int tokens[2] = {min(p.tile_tokens, q_hi - q_lo - token0), min(p.tile_tokens, q_hi - q_lo - token0 - p.tile_tokens)};
    const int kv = __ldg(p.c.kv_len + seq), end = cache_end(p.c, kv), first_pos = kv - (q_hi - q_lo);
    // cached tokens that a new token sees; tiles of them that row tile i needs, cut to this block's part of the cache
    auto visible = [&](int token) { return max(0, min(first_pos + token + 1, end)); };
    int need[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) need[i] = tokens[i] > 0 ? (visible(token0 + i * p.tile_tokens + tokens[i] - 1) + kTok - 1) / kTok : 0;
    const int all = max(need[0], need[1]);
    const int j0 = (int)((long long)all * blockIdx.z / p.splits), j1 = (int)((long long)all * (blockIdx.z + 1) / p.splits);
    const int n0 = max(0, min(need[0], j1) - j0), n1 = max(0, min(need[1], j1) - j0), n = max(n0, n1);   // (n0 <= n1, or n1 = 0)
    const int lead = n1 > 0 ? 1 : 0;              // the row tile that uses every K and V tile, and last
    const int tail = end % kTok != 0 ? end / kTok - j0 : -1;   // the tile of V whose last tokens do not exist


    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool ok = true;
    if (!found) {   // (the grid is sized for the most tiles that the requests could have)
        if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
        return;
    }

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFrontRegs));
        if (warp == 0) {
            // ---------------- copies: lane = (page of the tile, half of the head's columns) ----------------
            const int page_rows = p.c.page_size, per_tile = kTok / page_rows;
            const int* table = p.c.block_table + (size_t)seq * p.c.max_pages;
            const int my_page = kBits == 16 ? lane / kHalves : lane, my_half = kBits == 16 ? lane % kHalves : 0;
            const uint32_t my_dst = (uint32_t)(my_half * kHalfBytes + my_page * page_rows * 128);
            [[maybe_unused]] auto copy = [&](const CUtensorMap* map, uint32_t dst, uint32_t bar, int tok0, int row) {
                const int pages = min(per_tile, (end - tok0 + page_rows - 1) / page_rows);   // pages that hold cached tokens
                if (lane == 0) mbar_expect_tx(bar, (uint32_t)(pages * page_rows * kDim * 2));
                __syncwarp();
                if (lane < pages * kHalves) tma_load_2d(dst + my_dst, map, my_half * 64, row, bar);
            };
            auto first_row = [&](int tok0) {   // the cache row where this lane's page begins (a page that does not exist: no row, zeros)
                if (my_page >= per_tile || tok0 + my_page * page_rows >= end) return -1;
                const int page = __ldg(table + tok0 / page_rows + my_page);
                return page < 0 || page >= p.c.num_pages ? -page_rows : (page * p.c.num_kv_heads + kvh) * page_rows;
            };
            [[maybe_unused]] int row = (kBits == 16 || Shape::kStaged) && n > 0 ? first_row(j0 * kTok) : 0;
            if (lane < 2 && (lane ? n1 : n0) > 0) {   // Q_lane: the heads of the group by tile_tokens tokens, rows in that order
                mbar_expect_tx(q_full + 8 * lane, (uint32_t)(p.tile_tokens * G * kDim * 2));
#pragma unroll
                for (int h = 0; h < kHalves; ++h)
                    tma_load_3d(sq + lane * kTileBytes + h * kHalfBytes, &map_q, h * 64, kvh * G, q_lo + token0 + lane * p.tile_tokens,
                                q_full + 8 * lane);
            }
            if constexpr (Shape::kStaged) {
                // codes, one tile of keys and one of values at a time: they leave as soon as they are decoded
                const uint32_t raw = sv + kStages * kTileBytes;
                int sent = 0;
                for (int j = 0; j < n; ++j) {
                    const int tok0 = (j0 + j) * kTok, pages = min(per_tile, (end - tok0 + page_rows - 1) / page_rows);
                    const int next = j + 1 < n ? first_row(tok0 + kTok) : 0;
#pragma unroll
                    for (int side = 0; side < 2; ++side) {
                        if (j > 0) ok = mbar_wait(raw_free + 8 * side, (j - 1) & 1);
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) break;
                        if (lane == 0) mbar_expect_tx(raw_full + 8 * side, (uint32_t)(pages * page_rows * Shape::kRowBytes));
                        __syncwarp();
                        if (lane < pages)
                            tma_load_2d(raw + side * (kTok * Shape::kRowBytes) + lane * page_rows * Shape::kRowBytes, side ? &map_v : &map_k, 0, row,
                                        raw_full + 8 * side);
                        ++sent;
                    }
                    if (!ok) break;
                    row = next;
                }
                for (int i = 0; i < 2; ++i)
                    if ((i ? n1 : n0) > 0) (void)mbar_wait(q_full + 8 * i, 0);
                if (sent > 0) (void)mbar_wait(raw_full, ((sent - 1) / 2) & 1);
                if (sent > 1) (void)mbar_wait(raw_full + 8, (sent / 2 - 1) & 1);
            } else if constexpr (kBits != 16) {   // (the decoding warps fetch the codes)
                for (int i = 0; i < 2; ++i)
                    if ((i ? n1 : n0) > 0) (void)mbar_wait(q_full + 8 * i, 0);
            } else {
                int k_sent = 0, v_sent = 0;
                for (int j = 0; j < n; ++j) {
                    const int s = j % kStages, tok0 = (j0 + j) * kTok;
                    const int next = j + 1 < n ? first_row(tok0 + kTok) : 0;
                    // The lead's S(i) complete: K(i) is free, and V(i - 1), whose last product was issued before that S.  (The
                    // barrier of a stage cannot get a second phase ahead of this warp: that would take a K tile not copied yet.)
                    const int i = j - kStages;
                    if (i >= 0) ok = mbar_wait(k_free + 8 * s, (i / kStages) & 1);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    copy(&map_k, sk + s * kTileBytes, k_full + 8 * s, tok0, row);
                    k_sent = j + 1;
                    if (i >= 0) ok = mbar_wait(k_free + 8 * ((i + 1) % kStages), ((i + 1) / kStages) & 1);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    copy(&map_v, sv + s * kTileBytes, j == tail ? v_raw : v_full + 8 * s, tok0, row);
                    v_sent = j + 1;
                    row = next;
                }
                // no copy may still be in flight when the block retires (after a time-out elsewhere either)
                for (int i = 0; i < 2; ++i)
                    if ((i ? n1 : n0) > 0) (void)mbar_wait(q_full + 8 * i, 0);
                for (int j = max(0, k_sent - kStages); j < k_sent; ++j) (void)mbar_wait(k_full + 8 * (j % kStages), (j / kStages) & 1);
                for (int j = max(0, v_sent - kStages); j < v_sent; ++j)
                    (void)(j == tail ? mbar_wait(v_raw, 0) : mbar_wait(v_full + 8 * (j % kStages), (j / kStages) & 1));
            }
        } else if (warp == 1) {
            // ---------------- products ----------------
            if (lane == 0 && n > 0) {
                // bf16 (fp16) operands, fp32 accumulators; S: N = 128 tokens, both operands K-major; O: N = kDim, V is N-major
                constexpr uint32_t kBase = (1u << 4) | (kBits == 16 ? (1u << 7) | (1u << 10) : 0u) | ((uint32_t)(kRows >> 4) << 24);
                constexpr uint32_t kDescS = kBase | ((uint32_t)(kTok >> 3) << 17);
                constexpr uint32_t kDescO = kBase | (1u << 16) | ((uint32_t)(kDim >> 3) << 17);
                // 128-byte swizzle, version 1, 8 rows are 1024 bytes; V: the 64-column halves are kHalfBytes apart
                constexpr uint32_t kHi = (1024u >> 4) | (1u << 14) | (2u << 29);
                const uint32_t q_d = ((sq >> 4) & 0x3FFFu) | (1u << 16), k_d = ((sk >> 4) & 0x3FFFu) | (1u << 16);
                const uint32_t v_d = ((sv >> 4) & 0x3FFFu) | ((uint32_t)(kHalfBytes >> 4) << 16);
                auto scores = [&](int i, int s) {
                    const uint32_t a = q_d + (uint32_t)i * (kTileBytes >> 4), b = k_d + (uint32_t)s * (kTileBytes >> 4);
#pragma unroll
                    for (int k = 0; k < kDim / 16; ++k) {
                        const uint32_t at = (uint32_t)(k / 4) * (kHalfBytes >> 4) + 2 * (k % 4);
                        mma_ss(tmem + 128 * i, a + at, kHi, b + at, kHi, kDescS, k > 0);
                    }
                    tc_commit(s_full + 8 * i);
                    if (i == lead) tc_commit(k_free + 8 * s);
                };
                ok = mbar_wait(k_full, 0);
                for (int i = 0; i < 2 && ok; ++i) {
                    if ((i ? n1 : n0) == 0) continue;
                    ok = mbar_wait((kBits == 16 ? q_full : q_ready) + 8 * i, 0);
                    tc_fence_after();
                    if (ok) scores(i, 0);
                }
                for (int j = 0; j < n && ok; ++j) {
                    const int s = j % kStages, s1 = (j + 1) % kStages;
                    bool v_there = false, k_there = false;
                    for (int i = 0; i < 2 && ok; ++i) {
                        const int mine = i ? n1 : n0;
                        if (j >= mine) continue;
                        if (!v_there) {
                            ok = mbar_wait(v_full + 8 * s, (j / kStages) & 1);
                            v_there = true;
                        }
                        const uint32_t b = v_d + (uint32_t)s * (kTileBytes >> 4), o = tmem + Shape::kO + (uint32_t)(i * kDim);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            ok = ok && mbar_wait(p_full + 16 * i + 8 * h, j & 1);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll
                            for (int k = 4 * h; k < 4 * h + 4; ++k)   // 16 tokens: 8 columns of P, 2048 bytes of V
                                mma_ts(o, tmem + 128 * i + 8 * k, b + 128 * k, kHi, kDescO, j > 0 || k > 0);
                        }
                        if (!ok) break;
                        if (j + 1 == mine) {
                            tc_commit(o_done + 8 * i);
                            continue;
                        }
                        if (!k_there) {
                            ok = mbar_wait(k_full + 8 * s1, ((j + 1) / kStages) & 1);
                            k_there = true;
                            if (!ok) break;
                            tc_fence_after();
                        }
                        scores(i, s1);
                    }
                }
                // all products are complete before tensor memory is released
                tc_commit(drain);
                if (!mbar_wait(drain, 0)) ok = false;
            }
        } else if (kBits == 16 && warp == 2 && tail >= 0 && tail < n) {
            // ---------------- the last tile of V: tokens that do not exist become zeros ----------------
            const int s = tail % kStages;
            ok = mbar_wait(v_raw, 0);
            if (ok) {
                const int first = end % kTok, count = (kTok - first) * 8;
                for (int h = 0; h < kHalves; ++h)
                    for (int at = lane; at < count; at += 32)   // (whole rows: the swizzle stays inside a row)
                        *reinterpret_cast<uint4*>(smem + 2 * kTileBytes + (kStages + s) * kTileBytes + h * kHalfBytes + first * 128 + at * 16) =
                            make_uint4(0u, 0u, 0u, 0u);
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(v_full + 8 * s);
            }
        }
    } else if (warp < kGroups) {
        // ---------------- codes to fp16 operand tiles ----------------
        // The values of a token's codes are written in the operands' swizzle; the codes of the next tile are on the way meanwhile.
        if constexpr (kBits != 16) {
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kDecodeRegs));
            constexpr int kRowBytes = Shape::kRowBytes;
            const int* table = p.c.block_table + (size_t)seq * p.c.max_pages;
            // the row of the cache where a token lies, or -1 (loads without conditions do not wait for one another)
            const int last_tok = max(0, min(end, (j0 + n) * kTok) - 1);
            auto row_at = [&](int tok) {
                const int held = min(tok, last_tok), page = __ldg(table + (held >> p.page_shift));
                const bool there = tok == held && page >= 0 && page < p.c.num_pages;
                return there ? (page * p.c.num_kv_heads + kvh) * p.c.page_size + (held & (p.c.page_size - 1)) : -1;
            };
            auto parameter = [&](const __nv_bfloat16* scales, int row) -> uint32_t {   // scale, zero point above it
                const int at = max(row, 0);
                const uint32_t par = kBits == 8 ? (uint32_t)__ldg(reinterpret_cast<const unsigned short*>(scales) + at)
                                                : __ldg(reinterpret_cast<const uint32_t*>(scales) + at);
                return row < 0 ? 0u : par;   // (zeros, whatever lies in the place of the codes)
            };
            auto publish = [&](uint32_t full) {   // this warp's tokens are in shared memory, for the tensor cores to read
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(full);
            };
            unsigned char *k_tiles = smem + 2 * kTileBytes, *v_tiles = k_tiles + kStages * kTileBytes;
            auto row_of = [&](int j) { return row_at((j0 + j) * kTok + (tid & 127)); };   // this thread's token of tile j
            int row = row_of(0), next = row_of(1);
            uint32_t kp = parameter(kvq.ks, row), vp = parameter(kvq.vs, row);
            // The largest scales of the block's tokens put the values into fp16's range: 16 bytes of them at a time.
            uint32_t most_k = 0u, most_v = 0u;
            constexpr int kUnit = kBits == 8 ? 8 : 4;   // tokens
            const int tok0 = j0 * kTok, units = n > 0 ? (last_tok - tok0) / kUnit + 1 : 0;
#pragma unroll 1
            for (int base = tid & 127; base < units; base += 4 * 128) {
                int at[4], tok[4];
                uint4 a[4], b[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    tok[x] = tok0 + (base + 128 * x) * kUnit;
                    at[x] = row_at(min(tok[x], last_tok - (last_tok - tok0) % kUnit));
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    a[x] = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(kvq.ks) + (size_t)max(at[x], 0) * (16 / kUnit)));
                    b[x] = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(kvq.vs) + (size_t)max(at[x], 0) * (16 / kUnit)));
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const uint32_t wa[4] = {a[x].x, a[x].y, a[x].z, a[x].w}, wb[4] = {b[x].x, b[x].y, b[x].z, b[x].w};
                    const auto take = [&](uint32_t& most, uint32_t bits, bool there) {   // (scales that are no numbers do not count)
                        bits &= 0x7FFFu;
                        most = max(most, there && bits < 0x7F80u ? bits : 0u);
                    };
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool there = at[x] >= 0 && tok[x] + e * (kUnit / 4) <= last_tok;
                        take(most_k, wa[e], there);
                        take(most_v, wb[e], there);
                        if (kBits == 8) {
                            const bool second = at[x] >= 0 && tok[x] + 2 * e + 1 <= last_tok;
                            take(most_k, wa[e] >> 16, second);
                            take(most_v, wb[e] >> 16, second);
                        }
                    }
                }
            }
            most_k = __reduce_max_sync(0xffffffffu, most_k);
            most_v = __reduce_max_sync(0xffffffffu, most_v);
            if (lane == 0) {
                exponents[2 * (warp - 3)] = (int)most_k;   // (behind the results' places)
                exponents[2 * (warp - 3) + 1] = (int)most_v;
            }
            asm volatile("bar.sync 1, 128;" ::: "memory");
#pragma unroll
            for (int x = 1; x <= 4; ++x) {
                most_k = max(most_k, (uint32_t)exponents[2 * x]);
                most_v = max(most_v, (uint32_t)exponents[2 * x + 1]);
            }
            const auto exponent_of = [](uint32_t bits) { return bits ? (int)(bits >> 7) - 127 - 8 : 0; };   // scales below 2^9: 127 of them stay below 65504
            const int k_exponent = exponent_of(most_k), v_exponent = exponent_of(most_v);
            if (warp == 4 && lane == 0) {
                exponents[0] = k_exponent;
                exponents[1] = v_exponent;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(e_full);
            // The parameters of this thread's token of the next tile that it decodes, and on to the one after.  A head whose scale is
            // NaN reads as NaN.  A value like that makes its token's key one: the rows that see the token are NaN by their scores, and
            // no weight of zero meets the value.
            auto parameters = [&](int j, uint32_t& k_par, uint32_t& v_par) {
                const bool nan = (vp & 0x7FFFu) >= 0x7F80u;
                k_par = nan ? kp | 0x7FC0u : kp;
                v_par = nan ? 0u : vp;
                kp = parameter(kvq.ks, next);
                vp = parameter(kvq.vs, next);
                row = next;
                next = row_of(j + 2);
            };
            // (which tiles are free when: as for the copies of a bf16 cache)
            auto k_there = [&](int j) { return j < kStages || mbar_wait(k_free + 8 * (j % kStages), (j / kStages - 1) & 1); };
            auto v_there = [&](int j) { return j < kStages || mbar_wait(k_free + 8 * ((j + 1) % kStages), ((j + 1 - kStages) / kStages) & 1); };
            if constexpr (Shape::kStaged) {
                // a token a thread; eight threads that read or write the same piece of eight tokens meet all banks
                const int r = tid & 127;
                unsigned char *raw_k = v_tiles + kStages * kTileBytes, *raw_v = raw_k + kTok * kRowBytes;
                auto decode = [&](const unsigned char* raw, uint32_t par, int exponent, unsigned char* tile) {
                    const float scale = ldexpf(__uint_as_float(par << 16), -exponent);
                    const uint32_t scale2 = pack_half2(scale, scale);
#pragma unroll
                    for (int x = 0; x < kRowBytes / 16; ++x) {
                        const uint4 w = *reinterpret_cast<const uint4*>(raw + r * kRowBytes + ((x ^ r) & 7) * 16);
                        const uint4 f[2] = {values_of_bytes(w.x, w.y, scale2), values_of_bytes(w.z, w.w, scale2)};
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int at = 2 * x + e;
                            *reinterpret_cast<uint4*>(tile + (at >> 3) * kHalfBytes + r * 128 + ((at ^ r) & 7) * 16) = f[e];
                        }
                    }
                };
                for (int j = 0; j < n; ++j) {
                    const int s = j % kStages;
                    uint32_t k_par, v_par;
                    parameters(j, k_par, v_par);
                    ok = mbar_wait(raw_full, j & 1) && k_there(j);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    decode(raw_k, k_par, k_exponent, k_tiles + s * kTileBytes);
                    publish(k_full + 8 * s);
                    if (lane == 0) mbar_arrive(raw_free);
                    ok = mbar_wait(raw_full + 8, j & 1) && v_there(j);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    decode(raw_v, v_par, v_exponent, v_tiles + s * kTileBytes);
                    publish(v_full + 8 * s);
                    if (lane == 0) mbar_arrive(raw_free + 8);
                }
            } else {
                // 32 bytes of codes a lane and turn; lanes of the second half of a row take their two pieces in the other order, so that
                // eight lanes meet all banks
                constexpr int kAcross = kRowBytes / 32, kDown = 32 / kAcross, kTurns = 32 / kDown;
                constexpr int kOut = kBits == 8 ? 2 : 4;   // 16-byte pieces of values of 16 bytes of codes
                const int across = lane % kAcross, down = lane / kAcross, first = 32 * (warp - 4);
                const int other = kDim == 128 ? across : 0;   // which of its two pieces comes first
                auto load = [&](uint4 (&w)[kTurns][2], const void* codes, int row) {
    #pragma unroll
                    for (int x = 0; x < kTurns; ++x) {
                        const int from = max(__shfl_sync(0xffffffffu, row, x * kDown + down), 0);
                        const uint4* at = reinterpret_cast<const uint4*>(static_cast<const char*>(codes) + (size_t)from * kRowBytes) + 2 * across;
                        w[x][0] = __ldg(at + other);
                        w[x][1] = __ldg(at + (other ^ 1));
                    }
                };
                auto decode = [&](const uint4 (&w)[kTurns][2], uint32_t par, int exponent, unsigned char* tile) {
                    // (of this lane's token; the lanes that decode it fetch them)
                    const float scale = ldexpf(__uint_as_float(par << 16), -exponent), zero = __uint_as_float(par & 0xFFFF0000u);
                    const uint32_t mine = pack_half2(scale, zero);
    #pragma unroll
                    for (int x = 0; x < kTurns; ++x) {
                        const uint32_t both = __shfl_sync(0xffffffffu, mine, x * kDown + down), scale2 = __byte_perm(both, both, 0x1010);
                        uint32_t zero2 = 0u, zero16 = 0u;   // 1024 + zero point, -(64 + zero point)
                        if (kBits == 4) {
                            const uint32_t z = __byte_perm(both, both, 0x3232);
                            zero2 = h2_fma(z, 0x3C003C00u, 0x64006400u);
                            zero16 = h2_fma(z, 0xBC00BC00u, 0xD400D400u);
                        }
                        const int r = first + x * kDown + down;
    #pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const uint4 c = w[x][y];
                            uint4 f[kOut];
                            if (kBits == 8) {
                                f[0] = values_of_bytes(c.x, c.y, scale2);
                                f[1] = values_of_bytes(c.z, c.w, scale2);
                            } else {
                                f[0] = values_of_nibbles(c.x, zero2, zero16, scale2);
                                f[1] = values_of_nibbles(c.y, zero2, zero16, scale2);
                                f[kOut - 2] = values_of_nibbles(c.z, zero2, zero16, scale2);
                                f[kOut - 1] = values_of_nibbles(c.w, zero2, zero16, scale2);
                            }
                            const int at = (2 * across + (y ^ other)) * kOut;   // the first piece of the row's values
                            unsigned char* to = tile + (at >> 3) * kHalfBytes + r * 128;
    #pragma unroll
                            for (int e = 0; e < kOut; ++e) *reinterpret_cast<uint4*>(to + (((at + e) ^ r) & 7) * 16) = f[e];
                        }
                    }
                };
                uint4 kw[kTurns][2], vw[kTurns][2];
                if (n > 0) {
                    load(kw, kvq.k, row);
                    load(vw, kvq.v, row);
                }
                for (int j = 0; j < n; ++j) {
                    const int s = j % kStages;
                    uint32_t k_par, v_par;
                    parameters(j, k_par, v_par);
                    ok = __all_sync(0xffffffffu, k_there(j));
                    if (!ok) break;
                    decode(kw, k_par, k_exponent, k_tiles + s * kTileBytes);
                    publish(k_full + 8 * s);
                    if (j + 1 < n) load(kw, kvq.k, row);
                    ok = __all_sync(0xffffffffu, v_there(j));
                    if (!ok) break;
                    decode(vw, v_par, v_exponent, v_tiles + s * kTileBytes);
                    publish(v_full + 8 * s);
                    if (j + 1 < n) load(vw, kvq.v, row);
                }
            }
        }
    } else {
        // ---------------- softmax of row tile i: one row per thread ----------------
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        const int i = (warp - kGroups) >> 2, r = tid & 127, token = r / G;
        const int my_tokens = i ? tokens[1] : tokens[0];
        const bool live = token < my_tokens;   // (the other rows hold anything; they take no part in the votes below)
        const int mine = i ? n1 : n0;
        const int see = live ? visible(token0 + i * p.tile_tokens + token) - j0 * kTok : 0x40000000;   // (rows that are no token's never mask)
        float scale = p.scale_log2 == 0.f ? 1.f : fabsf(p.scale_log2), value_scale = 1.f;   // of scores and of results
        const uint32_t lane_base = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
        const uint32_t s_at = lane_base + 128 * i, o_at = lane_base + Shape::kO + (uint32_t)(i * kDim);
        auto publish = [&](int half) {   // this warp's rows of half of P are in tensor memory
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full + 16 * i + 8 * half);
        };
        if constexpr (kBits != 16) {
            // This thread's query in fp16, divided by the power of two of its largest element (8 bits fit 11; what is 2^-24 of the
            // largest or less is lost).
            if (mine > 0) {
                ok = mbar_wait(q_full + 8 * i, 0);
                ok = __all_sync(0xffffffffu, ok);
            }
            if (mine > 0 && ok) {
                unsigned char* tile = smem + i * kTileBytes + r * 128;
                uint32_t most = 0u;
#pragma unroll
                for (int x = 0; x < kDim / 8; ++x) {
                    const uint4 v = *reinterpret_cast<const uint4*>(tile + (x >> 3) * kHalfBytes + ((x ^ r) & 7) * 16);
                    most = __vmaxu2(most, __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu)));
                }
                most = max(most & 0xFFFFu, most >> 16);
                const int q_exponent = most >= 0x7F80u || most < 0x80u ? 0 : (int)(most >> 7) - 127;
                const float down = ldexpf(1.f, -q_exponent);
#pragma unroll
                for (int x = 0; x < kDim / 8; ++x) {
                    uint4* at = reinterpret_cast<uint4*>(tile + (x >> 3) * kHalfBytes + ((x ^ r) & 7) * 16);
                    float f[8];
                    unpack8(*at, f);
                    *at = make_uint4(pack_half2(f[0] * down, f[1] * down), pack_half2(f[2] * down, f[3] * down), pack_half2(f[4] * down, f[5] * down),
                                     pack_half2(f[6] * down, f[7] * down));
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(q_ready + 8 * i);
                ok = mbar_wait(e_full, 0);
                // (at least the smallest normal number: scores that small are all alike, and -inf times zero would be NaN)
                if (p.scale_log2 != 0.f) scale = fmaxf(ldexpf(scale, exponents[0] + q_exponent), 1.17549435e-38f);
                value_scale = ldexpf(1.f, exponents[1]);
            }
        }
        float ref = -INFINITY, sum = 0.f;
        for (int j = 0; j < mine && ok; ++j) {
            ok = mbar_wait(s_full + 8 * i, j & 1);
            if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
            tc_fence_after();
            uint32_t s[kTok];
#pragma unroll
            for (int c = 0; c < kTok; c += 32) tmem_ld32(s_at + c, s + c);
            tmem_ld_wait();
            pin(s);
            if (p.scale_log2 <= 0.f) {   // the sign of a negative scale; scores of a scale of zero
                const uint32_t keep = p.scale_log2 < 0.f ? 0xFFFFFFFFu : 0u, flip = keep & 0x80000000u;
#pragma unroll
                for (int c = 0; c < kTok; ++c) s[c] = (s[c] & keep) ^ flip;
            }
            const int left = see - j * kTok;   // visible tokens from the tile's first
            const bool edge = __any_sync(0xffffffffu, left < kTok);
            bool done = false;
            if (j > 0 && !edge) {
                // Weights against the present reference before the tile's maximum is known: it hardly ever exceeds the reference
                // by more than the limit, and the exponentials need not wait for it.  The first 64 tokens' product starts while
                // the other weights are computed, so for those the maximum is found beforehand; the first ones' sum says
                // itself whether one of them was too large (a maximum of them as well cost 2 % of the time).
                const unsigned long long scale2 = f2(scale, scale), base2 = f2(-ref, -ref);
                unsigned long long acc[2] = {0ull, 0ull};
                float top[2] = {-INFINITY, -INFINITY};
                auto weights = [&](int c, bool find) {
                    uint32_t w[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const unsigned long long x = f2_fma(f2(__uint_as_float(s[c + 2 * e]), __uint_as_float(s[c + 2 * e + 1])), scale2, base2);
                        float a, b;
                        f2_split(x, a, b);
                        a = fast_exp2(a);
                        b = fast_exp2(b);
                        if (find) top[e & 1] = max3(top[e & 1], __uint_as_float(s[64 + 2 * e]), __uint_as_float(s[64 + 2 * e + 1]));
                        acc[e & 1] = f2_add(acc[e & 1], f2(a, b));
                        w[e] = pack_weights<kBits>(a, b);
                    }
                    tmem_st32(s_at + c / 2, w);
                };
                weights(0, true);
                float a, b;
                f2_split(f2_add(acc[0], acc[1]), a, b);
                done = !__any_sync(0xffffffffu, live && !(a + b <= kMostSum && fmaxf(top[0], top[1]) * scale <= ref + kRaise));
                if (done) {
                    publish(0);
                    weights(64, false);
                    publish(1);
                    f2_split(f2_add(acc[0], acc[1]), a, b);
                    sum += a + b;
                }
            }
            if (!done) {
                if (edge) {
#pragma unroll
                    for (int c = 0; c < kTok; ++c)
                        if (c >= left) s[c] = 0xFF800000u;   // -inf
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < kTok; c += 2) top[(c >> 1) & 3] = max3(top[(c >> 1) & 3], __uint_as_float(s[c]), __uint_as_float(s[c + 1]));
                const float most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * scale;
                const bool raise = live && most > ref + kRaise;   // (also the first visible score: ref is -inf before it)
                if (__any_sync(0xffffffffu, raise)) {
                    const float to = raise ? most : ref;
                    const float keep = raise ? fast_exp2(ref - to) : 1.f;
                    ref = to;
                    sum *= keep;
                    if (j > 0) {   // (S_i(j) is there, so the product before it is complete)
#pragma unroll 1
                        for (int c = 0; c < kDim; c += 16) {
                            uint32_t o[16];
                            tmem_ld16(o_at + c, o);
                            tmem_ld_wait();
                            pin(o);
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
                            tmem_st16(o_at + c, o);
                        }
                    }
                }
                const float base = ref == -INFINITY ? 0.f : -ref;
                const unsigned long long scale2 = f2(scale, scale), base2 = f2(base, base);
                unsigned long long acc[2] = {0ull, 0ull};
#pragma unroll
                for (int c = 0; c < kTok; c += 64) {
                    uint32_t w[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        float a, b;
                        f2_split(f2_fma(f2(__uint_as_float(s[c + 2 * e]), __uint_as_float(s[c + 2 * e + 1])), scale2, base2), a, b);
                        a = fast_exp2(a);
                        b = fast_exp2(b);
                        acc[e & 1] = f2_add(acc[e & 1], f2(a, b));
                        w[e] = pack_weights<kBits>(a, b);
                    }
                    tmem_st32(s_at + c / 2, w);
                    publish(c / 64);
                }
                float a, b;
                f2_split(f2_add(acc[0], acc[1]), a, b);
                sum += a + b;
            }
        }
        // the rows' results
        if (mine > 0 && ok) ok = mbar_wait(o_done + 8 * i, 0);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
        if (ok) {
            // A thread holds a row, a row's results belong side by side: each warp turns its 32 rows around in its part of the
            // group's query tile (8 KB a time, pieces permuted by the row; the tile has been read, the last S is long there)
            // and writes 16 bytes a lane, whole rows at once.
            const bool whole = p.splits == 1;
            const float inv = 1.f / sum;   // (value_scale, a power of two, is applied apart: over a sum it may be too small a number)
            const size_t items = (size_t)p.c.total_q * H;
            const int item = live ? (q_lo + token0 + i * p.tile_tokens + token) * H + kvh * G + (r - token * G) : 0;   // this thread's (token, head)
            unsigned char* turn = smem + i * kTileBytes + (warp & 3) * (32 * kDim * 2);
            const int w_rows = my_tokens * G - 32 * (warp & 3);   // rows from the warp's first
            if (!whole && live)
                *reinterpret_cast<float2*>(p.many_parts + (size_t)p.splits * items * kDim + 2 * ((size_t)blockIdx.z * items + item)) =
                    make_float2(ref, sum);
            constexpr int kUnit = kDim * 2 / 16;   // 16-byte pieces of a row and turn: kDim bf16 or kDim / 2 fp32
            const int turns = whole ? 1 : 2, cols = kDim / turns;
            unsigned long long strange[2] = {0ull, 0ull};   // a NaN in it if a result of the row is not finite
            // (rows that saw nothing in this part of the cache have a sum of zero, by which the join leaves them out)
            for (int h = 0; h < turns && w_rows > 0; ++h) {
#pragma unroll 1
                for (int c = 0; c < cols; c += 16) {
                    uint32_t o[16];
                    if (mine > 0) {
                        tmem_ld16(o_at + h * cols + c, o);
                        tmem_ld_wait();
                        pin(o);
                    }
#pragma unroll
                    for (int e = 0; e < 16; e += 2)
                        strange[(e >> 1) & 1] = f2_fma(f2(__uint_as_float(o[e]), __uint_as_float(o[e + 1])), 0ull, strange[(e >> 1) & 1]);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        if (mine == 0 || sum == 0.f) o[e] = 0u;
                        if (kBits != 16 && !whole) o[e] = __float_as_uint(__uint_as_float(o[e]) * value_scale);
                    }
                    if (whole) {
#pragma unroll
                        for (int e = 0; e < 16; e += 8) {
                            float f[8];
#pragma unroll
                            for (int x = 0; x < 8; ++x) f[x] = sum == 0.f ? 0.f : __uint_as_float(o[e + x]) * inv * value_scale;
                            const int at = (c + e) / 8;
                            *reinterpret_cast<uint4*>(turn + lane * (kUnit * 16) + ((at & ~7) | ((at ^ lane) & 7)) * 16) = pack8(f);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; e += 4) {
                            const int at = (c + e) / 4;
                            *reinterpret_cast<uint4*>(turn + lane * (kUnit * 16) + ((at & ~7) | ((at ^ lane) & 7)) * 16) =
                                make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                        }
                    }
                }
                __syncwarp();
#pragma unroll 4
                for (int x = 0; x < kUnit; ++x) {
                    const int rr = (x * 32 + lane) / kUnit, at = lane % kUnit;
                    const uint4 v = *reinterpret_cast<const uint4*>(turn + rr * (kUnit * 16) + ((at & ~7) | ((at ^ rr) & 7)) * 16);
                    const size_t to = (size_t)__shfl_sync(0xffffffffu, item, rr);
                    if (rr >= w_rows) continue;
                    if (whole) *reinterpret_cast<uint4*>(p.out + to * kDim + 8 * at) = v;
                    else *reinterpret_cast<uint4*>(p.many_parts + ((size_t)blockIdx.z * items + to) * kDim + h * cols + 4 * at) = v;
                }
                __syncwarp();
            }
            // A cached value that is infinite or NaN and belongs to a later token than a row's own has met the row's weight of
            // zero.  Such rows (their weights and sums are right) are summed again over what they see, a warp to a row.
            float odd[2];
            f2_split(f2_add(strange[0], strange[1]), odd[0], odd[1]);
            const int shown = mine > 0 && live ? min(see, mine * kTok) : 0;   // tokens that the row sees, from the part's first
            // (Codes are finite: with a quantised cache there are none.)
            unsigned again = kBits != 16 ? 0u : __ballot_sync(0xffffffffu, shown > 0 && odd[0] + odd[1] != 0.f && sum < INFINITY && sum != 0.f);
            while (again) {
                const int rr = __ffs(again) - 1;
                again &= again - 1;
                const int count = __shfl_sync(0xffffffffu, shown, rr), to = __shfl_sync(0xffffffffu, item, rr);
                const float row_ref = __shfl_sync(0xffffffffu, ref, rr), row_inv = __shfl_sync(0xffffffffu, inv, rr);
                constexpr int kPer = kDim / 32;   // columns of a lane
                const int* table = p.c.block_table + (size_t)seq * p.c.max_pages;
                auto place = [&](int tok, bool& there) {   // of this lane's columns of a cached token
                    const int page = __ldg(table + (tok >> p.page_shift));
                    there = page >= 0 && page < p.c.num_pages;
                    return there ? (((size_t)page * p.c.num_kv_heads + kvh) * p.c.page_size + (tok & (p.c.page_size - 1))) * kDim + lane * kPer
                                 : (size_t)0;
                };
                auto columns = [&](const __nv_bfloat16* from, float (&f)[kPer]) {
#pragma unroll
                    for (int e = 0; e < kPer; e += 2) {
                        const uint32_t x = *reinterpret_cast<const uint32_t*>(from + e);
                        f[e] = __uint_as_float(x << 16);
                        f[e + 1] = __uint_as_float(x & 0xFFFF0000u);
                    }
                };
                const int from = j0 * kTok, upto = min(end, from + mine * kTok);
                bool met = false;
                for (int tok = from + count; tok < upto && !met; ++tok) {
                    bool there;
                    float v[kPer], zero = 0.f;
                    columns(p.v + place(tok, there), v);
#pragma unroll
                    for (int e = 0; e < kPer; ++e) zero = fmaf(v[e], 0.f, zero);
                    met = __any_sync(0xffffffffu, there && zero != zero);
                }
                if (!met) continue;   // (what the row itself sees is not finite)
                float q[kPer], sums[kPer];
                columns(p.q + (size_t)to * kDim + lane * kPer, q);
#pragma unroll
                for (int e = 0; e < kPer; ++e) sums[e] = 0.f;
                for (int tok = from; tok < from + count; ++tok) {
                    bool there;
                    const size_t at = place(tok, there);
                    if (!there) continue;   // (zeros)
                    float k[kPer], v[kPer], dot = 0.f;
                    columns(p.k + at, k);
                    columns(p.v + at, v);
#pragma unroll
                    for (int e = 0; e < kPer; ++e) dot = fmaf(q[e], k[e], dot);
#pragma unroll
                    for (int x = 16; x > 0; x >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, x);
                    const float w = fast_exp2(p.scale_log2 == 0.f ? -row_ref : fmaf(dot, p.scale_log2, -row_ref));
#pragma unroll
                    for (int e = 0; e < kPer; ++e) sums[e] = fmaf(w, v[e], sums[e]);
                }
#pragma unroll
                for (int e = 0; e < kPer; e += 2) {
                    if (whole) *reinterpret_cast<uint32_t*>(p.out + (size_t)to * kDim + lane * kPer + e) = pack2(sums[e] * row_inv, sums[e + 1] * row_inv);
                    else *reinterpret_cast<float2*>(p.many_parts + ((size_t)blockIdx.z * items + to) * kDim + lane * kPer + e) =
                             make_float2(sums[e], sums[e + 1]);
                }
            }
        }
    }
    if (!ok && p.status) atomicOr(p.status, (int)QIL_ERR_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
}

// Adds the parts of the cache in their order: one warp per (token, head).
template <int kDim>
__global__ void __launch_bounds__(128) attn_many_join_kernel(const AttnParams p) {
    constexpr int kPer = kDim / 32;
    const size_t items = (size_t)p.c.total_q * p.c.num_heads, at = (size_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    wait_for_earlier_kernels();   // the parts
    if (at >= items) return;
    const int lane = threadIdx.x & 31, t = (int)(at / p.c.num_heads);
    const int seq = request_of_row(p.c.cu_q, p.c.num_seqs, t);
    if (seq >= p.c.num_seqs) return;
    int lo, hi;
    request_rows(p.c.cu_q, seq, p.c.total_q, lo, hi);
    if ((hi - lo) * p.G <= kFewRows) return;
    const float2* stats = reinterpret_cast<const float2*>(p.many_parts + (size_t)p.splits * items * kDim);
    float most = -INFINITY, sum = 0.f, o[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) o[e] = 0.f;
    for (int s = 0; s < p.splits; ++s) most = fmaxf(most, stats[s * items + at].x);
    for (int s = 0; s < p.splits; ++s) {
        const float2 st = stats[s * items + at];
        if (st.y == 0.f) continue;
        const float f = fast_exp2(st.x - most);
        const float* part = p.many_parts + (s * items + at) * kDim + lane * kPer;
        sum = fmaf(st.y, f, sum);
#pragma unroll
        for (int e = 0; e < kPer; e += 2) {
            const float2 v = *reinterpret_cast<const float2*>(part + e);
            o[e] = fmaf(v.x, f, o[e]);
            o[e + 1] = fmaf(v.y, f, o[e + 1]);
        }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int e = 0; e < kPer; e += 2) *reinterpret_cast<uint32_t*>(p.out + at * kDim + lane * kPer + e) = pack2(o[e] * inv, o[e + 1] * inv);
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn() {
    static std::mutex mu;
    static EncodeFn fn = nullptr;
    std::lock_guard<std::mutex> lock(mu);
    if (!fn) {
        void* ptr = nullptr;
        cudaDriverEntryPointQueryResult res;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &res) != cudaSuccess ||
            res != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            return nullptr;
        }
        fn = reinterpret_cast<EncodeFn>(ptr);
    }
    return fn;
}

// The cache as a matrix of head rows: [num_pages * num_kv_heads * page_size][D]; a copy takes 64 columns of a page.
bool encode_cache(CUtensorMap* map, const void* cache, const PagedCache& c) {
    const EncodeFn enc = encode_fn();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.num_pages * c.num_kv_heads * c.page_size};
    const cuuint64_t strides[1] = {(cuuint64_t)c.head_dim * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)c.page_size}, estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(cache), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same of codes in rows of 128 bytes; a copy takes a page.
bool encode_codes(CUtensorMap* map, const void* codes, const PagedCache& c) {
    const EncodeFn enc = encode_fn();
    if (!enc) return false;
    const cuuint64_t bytes = 128;
    const cuuint64_t dims[2] = {bytes, (cuuint64_t)c.num_pages * c.num_kv_heads * c.page_size}, strides[1] = {bytes};
    const cuuint32_t box[2] = {(cuuint32_t)bytes, (cuuint32_t)c.page_size}, estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(codes), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The queries as [total_q][H][D]; a copy takes 64 columns of the G heads of a group for tile_tokens tokens.
bool encode_queries(CUtensorMap* map, const AttnParams& p) {
    const EncodeFn enc = encode_fn();
    if (!enc) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)p.c.head_dim, (cuuint64_t)p.c.num_heads, (cuuint64_t)p.c.total_q};
    const cuuint64_t strides[2] = {(cuuint64_t)p.c.head_dim * 2, (cuuint64_t)p.c.num_heads * p.c.head_dim * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)p.G, (cuuint32_t)p.tile_tokens}, estr[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<__nv_bfloat16*>(p.q), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kDim, int kBits>
qil_status go(const AttnParams& p, const QuantCache& kvq, cudaStream_t st) {
    CUtensorMap mq, mk, mv;
    if (!encode_queries(&mq, p)) return QIL_ERR_CUDA;
    mk = mv = mq;   // (codes that come without a copy)
    if (kBits == 16 && (!encode_cache(&mk, p.k, p.c) || !encode_cache(&mv, p.v, p.c))) return QIL_ERR_CUDA;
    if (ManyShape<kDim, kBits>::kStaged && (!encode_codes(&mk, kvq.k, p.c) || !encode_codes(&mv, kvq.v, p.c))) return QIL_ERR_CUDA;
    constexpr int kSmem = ManyShape<kDim, kBits>::kSmem;
    static_assert(kSmem <= 232448, "shared memory per block");
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(attn_many_kernel<kDim, kBits>, kSmem, allowed)) return QIL_ERR_CUDA;
    // (heads first, so that the long tiles of all heads start before the short ones of any)
    const dim3 grid((unsigned)((long long)p.c.num_kv_heads * (p.c.total_q / (2 * p.tile_tokens) + p.c.num_seqs)), 1u, (unsigned)p.splits);
    return launch_early(attn_many_kernel<kDim, kBits>, grid, kThreadsOf<kBits>, kSmem, st, mq, mk, mv, p, kvq);
}

}  // namespace

qil_status launch_attn_many(const AttnParams& p, cudaStream_t st) {
    return p.c.head_dim == 128 ? go<128, 16>(p, QuantCache{}, st) : go<64, 16>(p, QuantCache{}, st);
}
qil_status launch_attn_many_q(const AttnQuantParams& p, cudaStream_t st) {
    if (p.a.c.head_dim == 128) return p.kv.bits == 8 ? go<128, 8>(p.a, p.kv, st) : go<128, 4>(p.a, p.kv, st);
    return p.kv.bits == 8 ? go<64, 8>(p.a, p.kv, st) : go<64, 4>(p.a, p.kv, st);
}

qil_status launch_attn_many_join(const AttnParams& p, cudaStream_t st) {
    const long long items = (long long)p.c.total_q * p.c.num_heads;
    const dim3 grid((unsigned)((items + 3) / 4));
    return p.c.head_dim == 128 ? launch_early(attn_many_join_kernel<128>, grid, 128, 0, st, p)
                               : launch_early(attn_many_join_kernel<64>, grid, 128, 0, st, p);
}

}  // namespace qil
