// The next token of every row of logits: temperature, top-k, top-p, min-p, and one given uniform number per row.
//   x_i the logits (a NaN counts as -inf), w_i = exp((x_i - max) / T) in 64 bits, held as the whole number rint(2^42 w_i)
//   order: x descending, equal ones by index; kept are the first k, of those the ones before which less than p of their total
//   lies, and of those the ones with w >= min_p; the first is always kept
//   token: the first index, in the order of the vocabulary, at which the running sum of kept weights exceeds u times their total
// Whole numbers make every sum the same in whatever order it is formed, so the token is a function of its row alone.  A weight
// below 2^-43 of the largest counts as zero.
//
// A row is a cluster of up to eight blocks, each with its part of the logits in shared memory, read from global memory once.
// Nothing is sorted as a whole: a histogram over the values (1024 equal steps between the largest and the smallest that
// counts) gives the step in which the k-th value, or the p-th part of the weight, lies; what lies in it and above, mostly a
// few dozen values, is gathered in one block and finished there by sorting.  Where more than 1024 values remain the step alone
// is gathered (or cut again), which gives the last kept value, and a pass over the row sums and selects.
// Latency bound: every step of a row is a trip between its blocks (about 0.6 us), and the last pass over a row that does not end
// in the list has one warp that looks for the token in its share again.  Measured: one row of 32 000 (bf16, top-k and top-p) 12 to
// 13 us, 64 such rows 21 us; 64 rows of 128 003 (fp32, two rounds of blocks) greedy 14 to 16 us, top-k and top-p 58 to 60 us,
// settings of every kind 94 to 114 us, by the settings.
#include <cuda_fp16.h>

#include <type_traits>

#include "sample.cuh"

namespace qil {

namespace {

typedef unsigned long long u64;

constexpr int kMostThreads = 512, kBuckets = 1024, kCap = 1024, kMostBlocks = 8;
constexpr double kOne = 4398046511104.0;   // 2^42
constexpr double kDeepest = 29.81;         // beyond 43 log(2) = 29.8053, below which a weight rounds to zero (this far 2^y still has y > -43.5)
constexpr int kRanked = 512;               // lists of up to so many are put in order by counting
static_assert(QIL_SAMPLE_MAX_VOCAB <= 1 << 18, "an index has 18 bits beside a weight's 43");

// Shared memory, in bytes from its start; every access names the state space.  What a block tells the others lies in its own
// memory and is read by them: blocks only load from one another.
constexpr unsigned kList = 0, kHeld = kList + 8 * kCap;                 // u64: candidates; kept ones
constexpr unsigned kCounts = kHeld + 8 * kCap;                          // u32: values in the steps of the histogram
constexpr unsigned kWeights = kCounts + 4 * kBuckets;                   // u32 x 3: sums of 15, 14 and 14 bits of their weights
constexpr unsigned kWarpA = kWeights + 12 * kBuckets, kWarpB = kWarpA + kMostThreads / 4;   // u64: sums of the warps
constexpr unsigned kSlots = kWarpB + kMostThreads / 4;                        // u64 [2][2]: sums of the block, in turn
constexpr unsigned kTotal = kSlots + 32;                                // u64 [2]
constexpr unsigned kHit = kTotal + 16;                                  // [2] a step: u64 before, u64 weight before, u32 n, bucket, found
constexpr unsigned kListed = kHit + 64, kLast = kListed + 4, kLastIndex = kLast + 4;
constexpr unsigned kLogits = kListed + 16;                              // fp32
static_assert(QIL_SAMPLE_MAX_VOCAB / kMostBlocks <= 1 << 15, "a block's sums of 15 bits fit 32");

__device__ __forceinline__ u64 lds64(unsigned addr) {
    u64 v;
    asm volatile("ld.shared.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ unsigned lds32(unsigned addr) {
    unsigned v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void sts64(unsigned addr, u64 v) { asm volatile("st.shared.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory"); }
__device__ __forceinline__ void sts32(unsigned addr, unsigned v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void add_shared(unsigned addr, unsigned v) { asm volatile("red.shared.add.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ unsigned take_shared(unsigned addr) {
    unsigned old;
    asm volatile("atom.shared.add.u32 %0, [%1], 1;" : "=r"(old) : "r"(addr) : "memory");
    return old;
}

__device__ __forceinline__ unsigned ordered(float x) {
    const unsigned u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(unsigned o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }

// A variable of another block of the row (kBlocks: the row is a cluster).
template <bool kBlocks>
__device__ __forceinline__ u64 load64(unsigned addr, unsigned block) {
    if (!kBlocks) return lds64(addr);
    u64 v;
    asm volatile("{\n\t.reg .u32 there;\n\tmapa.shared::cluster.u32 there, %1, %2;\n\tld.shared::cluster.u64 %0, [there];\n\t}" : "=l"(v) : "r"(addr), "r"(block) : "memory");
    return v;
}
template <bool kBlocks>
__device__ __forceinline__ unsigned load32(unsigned addr, unsigned block) {
    if (!kBlocks) return lds32(addr);
    unsigned v;
    asm volatile("{\n\t.reg .u32 there;\n\tmapa.shared::cluster.u32 there, %1, %2;\n\tld.shared::cluster.u32 %0, [there];\n\t}" : "=r"(v) : "r"(addr), "r"(block) : "memory");
    return v;
}
template <bool kBlocks>
__device__ __forceinline__ void row_sync() {
    __syncthreads();
    if (kBlocks) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}

template <class F>
__device__ __forceinline__ u64 warp_reduce(u64 v, F f) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ u64 warp_scan(u64 v) {   // sums up to and with this lane
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 up = __shfl_up_sync(0xffffffffu, v, o);
        if ((int)(threadIdx.x & 31) >= o) v += up;
    }
    return v;
}
struct Add { __device__ u64 operator()(u64 a, u64 b) const { return a + b; } };
struct Max { __device__ u64 operator()(u64 a, u64 b) const { return a > b ? a : b; } };

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float widen(__half x) { return __half2float(x); }

// What a block of so many threads does.
template <int kThreads>
struct Sampler {

static constexpr int kWarps = kThreads / 32, kEach = kCap / kThreads;   // candidates of a thread

// A row's part in this block.  What the blocks of a row do together is called by all threads of all of them.
struct Row {
    unsigned mem;        // this block's shared memory
    int n, first;        // logits first ... first + n - 1
    unsigned blocks, mine;
    int turn, hits;      // which of the two places comes next
    double top, rate;    // the largest logit; log2(e) / temperature
    float low;           // logits below it weigh nothing
    float last;          // kept are x > last, and x == last up to index last_index
    int last_index;
    double least;        // min_p 2^42

    __device__ __forceinline__ float x(int i) const { return __uint_as_float(lds32(mem + kLogits + 4 * i)); }
    __device__ __forceinline__ bool kept(float v, int i) const { return v >= low && (v > last || (v == last && first + i <= last_index)); }
    // rint(2^42 exp((v - top) / temperature)) for v >= low: 2^f by its Taylor series, |f| <= 1/2 (off by 2^-47), times a power of two
    __device__ __forceinline__ u64 weight(float v) const {
        const double y = ((double)v - top) * rate, shifted = y + 6755399441055744.0, f = y - (shifted - 6755399441055744.0);   // (+ 1.5 2^52: rounds)
        double s = 1.0 / 39916800;
        const double z = f * 0.6931471805599453;
        s = fma(s, z, 1.0 / 3628800);
        s = fma(s, z, 1.0 / 362880);
        s = fma(s, z, 1.0 / 40320);
        s = fma(s, z, 1.0 / 5040);
        s = fma(s, z, 1.0 / 720);
        s = fma(s, z, 1.0 / 120);
        s = fma(s, z, 1.0 / 24);
        s = fma(s, z, 1.0 / 6);
        s = fma(s, z, 0.5);
        s = fma(s, z, 1.0);
        s = fma(s, z, 1.0);
        const int n = __double2loint(shifted);   // -43 ... 0
        return (u64)__double2ll_rn(s * __hiloint2double((1023 + 42 + n) << 20, 0));
    }
};

__device__ static __forceinline__ int warp_id() { return threadIdx.x >> 5; }
__device__ static __forceinline__ int lane_id() { return threadIdx.x & 31; }

// The largest of all threads' values, of two at once, over the blocks of a row.
template <bool kBlocks>
__device__ static __forceinline__ void largest(Row& r, u64& a, u64& b) {
    a = warp_reduce(a, Max());
    b = warp_reduce(b, Max());
    if (lane_id() == 0) {
        sts64(r.mem + kWarpA + 8 * warp_id(), a);
        sts64(r.mem + kWarpB + 8 * warp_id(), b);
    }
    __syncthreads();
    a = b = 0;
    for (int k = 0; k < kWarps; ++k) {
        a = Max()(a, lds64(r.mem + kWarpA + 8 * k));
        b = Max()(b, lds64(r.mem + kWarpB + 8 * k));
    }
    const unsigned slot = r.mem + kSlots + 16 * r.turn;
    if (threadIdx.x == 0) {
        sts64(slot, a);
        sts64(slot + 8, b);
    }
    row_sync<kBlocks>();
    if (kBlocks) {   // (a lane a block: one trip)
        a = load64<kBlocks>(slot, min((unsigned)lane_id(), r.blocks - 1));
        b = load64<kBlocks>(slot + 8, min((unsigned)lane_id(), r.blocks - 1));
        a = warp_reduce(a, Max());
        b = warp_reduce(b, Max());
    }
    r.turn ^= 1;
}

// The sums over the blocks before this one, and over all of them, of a value at `slot` (all threads get both).
template <bool kBlocks>
__device__ static __forceinline__ void over_blocks(const Row& r, unsigned slot, u64& before, u64& all) {
    const unsigned lane = lane_id();
    const u64 v = load64<kBlocks>(slot, min(lane, r.blocks - 1)), to = warp_scan(lane < r.blocks ? v : 0ull);
    all = __shfl_sync(0xffffffffu, to, 31);
    before = __shfl_sync(0xffffffffu, to - v, r.mine);
}

struct Hit {
    bool found;
    u64 n_before, w_before, total;   // of the values above the step; of all (weights, where they are asked for)
    unsigned n;                      // values in the step
    int bucket;
};

// The steps of [lo, hi], lo < hi: equal ones, counted from the top.  In fp32 where its range allows; either way a larger value
// is never in a later step, hi in the first and lo in the last.
struct Steps {
    float top, per_unit;
    double wide_top, wide_per_unit;
    bool wide;
    __device__ __forceinline__ Steps(double lo, double hi) {
        const double range = hi - lo;
        wide = !(range > 1e-30 && range < 1e38 && fabs(hi) < 1e38);
        top = (float)hi;
        per_unit = wide ? 0.f : (float)((double)kBuckets / range);
        wide_top = hi;
        wide_per_unit = (double)kBuckets / range;
    }
    __device__ __forceinline__ int of(float x) const {
        if (wide) {
            const double b = (wide_top - (double)x) * wide_per_unit;
            return b < (double)(kBuckets - 1) ? (int)b : kBuckets - 1;
        }
        return min((int)((top - x) * per_unit), kBuckets - 1);
    }
};

// The step of [lo, hi] in which the goal lies: the first before whose end `goal` of the kept values' number (or weight) lies.
// n0 and w0 lie above hi.
template <bool kBlocks, bool kWeigh>
__device__ static __forceinline__ Hit find_step(Row& r, float hi, float lo, double goal, bool part_of_total, u64 n0, u64 w0) {
    const int tid = threadIdx.x;
    const Steps steps((double)lo, (double)hi);
    for (int b = tid; b < (kWeigh ? 4 : 1) * kBuckets; b += kThreads) sts32(r.mem + kCounts + 4 * b, 0u);   // (the weights lie behind the counts)
    const unsigned hit = r.mem + kHit + 32 * r.hits;
    if (tid == 0) {
        sts32(r.mem + kListed, 0u);
        sts32(hit + 24, 0u);
    }
    __syncthreads();
    // (four at a time: a weight is a chain of twenty dependent operations)
    for (int base = tid; base < r.n; base += 4 * kThreads) {
        float v[4];
        bool in[4];
        u64 w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = base + e * kThreads;
            v[e] = r.x(min(i, r.n - 1));
            in[e] = i < r.n && r.kept(v[e], i) && v[e] <= hi && v[e] >= lo;
        }
        if (kWeigh) {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = r.weight(in[e] ? v[e] : r.low);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!in[e]) continue;
            const unsigned at = r.mem + kCounts + 4 * steps.of(v[e]);
            add_shared(at, 1u);
            if (kWeigh) {
                add_shared(at + 4 * kBuckets, (unsigned)w[e] & 0x7FFFu);
                add_shared(at + 8 * kBuckets, (unsigned)(w[e] >> 15) & 0x3FFFu);
                add_shared(at + 12 * kBuckets, (unsigned)(w[e] >> 29));
            }
        }
    }
    row_sync<kBlocks>();
    // each block takes its share of the steps, a thread `per` of them in a row
    const int share = kBuckets / (int)r.blocks, per = (share + kThreads - 1) / kThreads, from = (int)r.mine * share + tid * per;
    const bool busy = tid * per < share;
    constexpr int kPer = (kBuckets + kThreads - 1) / kThreads;
    unsigned n[kPer];
    u64 w[kPer], n_sum = 0, w_sum = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        n[e] = 0;
        w[e] = 0;
        if (busy && e < per) {
            constexpr int kMost = kBlocks ? kMostBlocks : 1;
            const unsigned at = r.mem + kCounts + 4 * (from + e);
            unsigned v[4][kMost];   // (all on the way at once; the repeated ones do not count)
#pragma unroll
            for (int k = 0; k < kMost; ++k)
#pragma unroll
                for (int x = 0; x < (kWeigh ? 4 : 1); ++x) v[x][k] = load32<kBlocks>(at + 4 * x * kBuckets, min((unsigned)k, r.blocks - 1));
#pragma unroll
            for (int k = 0; k < kMost; ++k)
                if ((unsigned)k < r.blocks) {
                    n[e] += v[0][k];
                    if (kWeigh) w[e] += v[1][k] + ((u64)v[2][k] << 15) + ((u64)v[3][k] << 29);
                }
        }
        n_sum += n[e];
        w_sum += w[e];
    }
    const u64 n_to = warp_scan(n_sum), w_to = kWeigh ? warp_scan(w_sum) : 0ull;
    if (lane_id() == 31) {
        sts64(r.mem + kWarpA + 8 * warp_id(), n_to);
        sts64(r.mem + kWarpB + 8 * warp_id(), w_to);
    }
    __syncthreads();
    u64 n_at = n_to - n_sum, w_at = w_to - w_sum, n_block = 0, w_block = 0;
    for (int k = 0; k < kWarps; ++k) {
        const u64 vn = lds64(r.mem + kWarpA + 8 * k), vw = kWeigh ? lds64(r.mem + kWarpB + 8 * k) : 0ull;
        if (k < warp_id()) n_at += vn, w_at += vw;
        n_block += vn;
        w_block += vw;
    }
    const unsigned slot = r.mem + kSlots + 16 * r.turn;
    if (tid == 0) {
        sts64(slot, n_block);
        sts64(slot + 8, w_block);
    }
    row_sync<kBlocks>();
    u64 n_below, w_below = 0, unused, total = 0;
    over_blocks<kBlocks>(r, slot, n_below, unused);
    if (kWeigh) over_blocks<kBlocks>(r, slot + 8, w_below, total);
    total += w0;
    n_at += n0 + n_below;
    w_at += w0 + w_below;
    r.turn ^= 1;
    if (part_of_total) goal *= (double)total;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        if (busy && e < per && n[e]) {
            const double before = kWeigh ? (double)w_at : (double)n_at, after = kWeigh ? (double)(w_at + w[e]) : (double)(n_at + n[e]);
            if (before < goal && after >= goal) {   // (one step of all)
                sts64(hit, n_at);
                sts64(hit + 8, w_at);
                sts32(hit + 16, n[e]);
                sts32(hit + 20, (unsigned)(from + e));
                sts32(hit + 24, 1u);
            }
        }
        n_at += n[e];
        w_at += w[e];
    }
    row_sync<kBlocks>();
    Hit h = {false, 0, 0, total, 0u, 0};
    const unsigned who = __ballot_sync(0xffffffffu, (unsigned)lane_id() < r.blocks && load32<kBlocks>(hit + 24, min((unsigned)lane_id(), r.blocks - 1)) != 0u);
    if (who) {
        const unsigned k = __ffs(who) - 1;
        h.found = true;
        h.n_before = load64<kBlocks>(hit, k);
        h.w_before = load64<kBlocks>(hit + 8, k);
        h.n = load32<kBlocks>(hit + 16, k);
        h.bucket = (int)load32<kBlocks>(hit + 20, k);
    }
    r.hits ^= 1;   // (a block resets this place again when everyone is past the other one)
    return h;
}

// Kept values of steps [from, to] of [lo, hi] (kCap at most over the row) to the first block's list, in any order.
template <bool kBlocks>
__device__ static __forceinline__ void gather(Row& r, float hi, float lo, int from, int to) {
    const Steps steps((double)lo, (double)hi);
    for (int base = threadIdx.x; base < r.n; base += 4 * kThreads) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = r.x(min(base + e * kThreads, r.n - 1));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = base + e * kThreads, b = steps.of(v[e]);
            if (i >= r.n || !r.kept(v[e], i) || v[e] < lo || v[e] > hi || b < from || b > to) continue;
            const unsigned at = take_shared(r.mem + kListed);
            if (at < kCap) sts64(r.mem + kList + 8 * at, (u64)~ordered(v[e]) << 32 | (unsigned)(r.first + i));
        }
    }
    row_sync<kBlocks>();
    if (!kBlocks || r.mine != 0) return;
    // a warp a block: its list goes behind those of the blocks before it
    const unsigned lane = lane_id();
    const int mine = (int)load32<kBlocks>(r.mem + kListed, min(lane, r.blocks - 1)), upto = (int)warp_scan(lane < r.blocks ? (u64)mine : 0ull);
    for (unsigned k = 1 + warp_id(); k < r.blocks; k += kWarps) {
        const int end = __shfl_sync(0xffffffffu, upto, k), base = end - __shfl_sync(0xffffffffu, mine, k);
        for (int i = lane; i < min(end, kCap) - base; i += 32) sts64(r.mem + kList + 8 * (base + i), load64<kBlocks>(r.mem + kList + 8 * i, k));
    }
    __syncthreads();
}

// n whole numbers at `list`, ascending; one block
__device__ static __forceinline__ void sort_list(unsigned list, int n) {
    int size = 2;
    while (size < n) size *= 2;
    for (int i = n + (int)threadIdx.x; i < size; i += kThreads) sts64(list + 8 * i, ~0ull);
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            for (int t = threadIdx.x; t < size / 2; t += kThreads) {
                const int a = 2 * t - (t & (j - 1)), b = a + j;
                const u64 va = lds64(list + 8 * a), vb = lds64(list + 8 * b);
                if ((va > vb) == ((a & k) == 0)) {
                    sts64(list + 8 * a, vb);
                    sts64(list + 8 * b, va);
                }
            }
            __syncthreads();
        }
}

// The sum of v of the threads before this one, and of all; one block.
__device__ static __forceinline__ u64 sum_before(const Row& r, u64 v, u64& all) {
    const u64 to = warp_scan(v);
    if (lane_id() == 31) sts64(r.mem + kWarpA + 8 * warp_id(), to);
    __syncthreads();
    u64 before = to - v;
    all = 0;
    for (int k = 0; k < kWarps; ++k) {
        const u64 w = lds64(r.mem + kWarpA + 8 * k);
        if (k < warp_id()) before += w;
        all += w;
    }
    __syncthreads();
    return before;
}
// the largest double below a positive one
__device__ static __forceinline__ double just_below(double v) { return __longlong_as_double(__double_as_longlong(v) - 1); }
// the logit of a list's entry
__device__ static __forceinline__ float logit_of(u64 key) { return unordered(~(unsigned)(key >> 32)); }

// The first block finishes a row whose candidates are all in its list (n of them): k or 0, p of `total` (of the first k where
// that is 0), min_p.  A short list is not sorted: every thread counts what stands before its candidate, and adds it up.
__device__ static __forceinline__ void finish_list(const Row& r, int n, int k, bool use_p, double p, u64 total, double u, int* out) {
    if (n <= kRanked) {
        constexpr int kOwn = kRanked / kThreads;
        u64 key[kOwn], w[kOwn], before[kOwn], run[kOwn], all = 0;
        int rank[kOwn];
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
            const int i = threadIdx.x + j * kThreads;
            key[j] = i < n ? lds64(r.mem + kList + 8 * i) : ~0ull;
            w[j] = i < n ? r.weight(logit_of(key[j])) : 0ull;
            if (i < n) sts64(r.mem + kHeld + 8 * i, w[j]);
            rank[j] = 0;
            before[j] = run[j] = 0;
        }
        __syncthreads();
        if (((int)threadIdx.x & ~31) < n)
            for (int i = 0; i < n; ++i) {
                const u64 other = lds64(r.mem + kList + 8 * i), weight = lds64(r.mem + kHeld + 8 * i);
#pragma unroll
                for (int j = 0; j < kOwn; ++j)
                    if (other < key[j]) {
                        ++rank[j];
                        before[j] += weight;
                    }
            }
        const int staying = k > 0 && k < n ? k : n;
#pragma unroll
        for (int j = 0; j < kOwn; ++j)   // (one thread has the last candidate that k leaves)
            if ((int)threadIdx.x + j * kThreads < n && rank[j] == staying - 1) sts64(r.mem + kTotal, before[j] + w[j]);
        __syncthreads();
        const double goal = p * (double)(total ? total : lds64(r.mem + kTotal));
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
            const int i = threadIdx.x + j * kThreads;
            const bool in = i < n && (rank[j] == 0 || (rank[j] < staying && (!use_p || (double)before[j] < goal) && (double)w[j] >= r.least));
            if (!in) w[j] = 0;
            if (i < n) sts64(r.mem + kHeld + 8 * i, w[j]);
        }
        __syncthreads();
        if (((int)threadIdx.x & ~31) < n)
            for (int i = 0; i < n; ++i) {   // in the order of the indices now
                const unsigned other = (unsigned)lds64(r.mem + kList + 8 * i);
                const u64 weight = lds64(r.mem + kHeld + 8 * i);
                all += weight;
#pragma unroll
                for (int j = 0; j < kOwn; ++j)
                    if (other < (unsigned)key[j]) run[j] += weight;
            }
        const double want = u * (double)all, reach = want < (double)all ? want : just_below((double)all);
#pragma unroll
        for (int j = 0; j < kOwn; ++j)
            if (w[j] && !((double)run[j] > reach) && (double)(run[j] + w[j]) > reach) *out = (int)(unsigned)key[j];
        return;
    }
    sort_list(r.mem + kList, n);
    const int i0 = kEach * threadIdx.x;
    u64 key[kEach], w[kEach], sum = 0, all;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        key[j] = i0 + j < n ? lds64(r.mem + kList + 8 * (i0 + j)) : 0ull;
        w[j] = i0 + j < n && (k <= 0 || i0 + j < k) ? r.weight(logit_of(key[j])) : 0ull;
        sum += w[j];
    }
    u64 before = sum_before(r, sum, all);
    const double goal = p * (double)(total ? total : all);
    int kept = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const bool in = i0 + j < n && (i0 + j == 0 || (w[j] > 0 && (!use_p || (double)before < goal) && (double)w[j] >= r.least));
        kept += __syncthreads_count(in);
        before += w[j];
        if (in) sts64(r.mem + kHeld + 8 * (i0 + j), (key[j] & 0xFFFFFFFFull) << 43 | w[j]);   // (kept are the first ones)
    }
    __syncthreads();
    sort_list(r.mem + kHeld, kept);   // by index now
    sum = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        key[j] = i0 + j < kept ? lds64(r.mem + kHeld + 8 * (i0 + j)) : 0ull;
        w[j] = key[j] & ((1ull << 43) - 1);
        sum += w[j];
    }
    before = sum_before(r, sum, all);
    const double want = u * (double)all, reach = want < (double)all ? want : just_below((double)all);
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        if (w[j] && !((double)before > reach) && (double)(before + w[j]) > reach) *out = (int)(key[j] >> 43);
        before += w[j];
    }
}

// Each warp of a block has its range of the block's logits, so that sums can be taken in the order of the indices.
__device__ static __forceinline__ void warp_range(const Row& r, int& lo, int& hi) {
    const int per = ((r.n + kWarps - 1) / kWarps + 31) & ~31;
    lo = min(r.n, warp_id() * per);
    hi = min(r.n, lo + per);
}

// The first index at which the running sum of f over the row exceeds share * total + offset (of the last value's, where the
// sum does not get there).  The thread that finds it calls `found`.
template <bool kBlocks, class F, class G>
__device__ static __forceinline__ void select(Row& r, double share, double offset, F f, G found) {
    int lo, hi;
    warp_range(r, lo, hi);
    u64 sum = 0;
    for (int base = lo + lane_id(); base < hi; base += 128) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = r.x(min(base + 32 * e, hi - 1));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const u64 w = f(v[e], min(base + 32 * e, hi - 1));
            sum += base + 32 * e < hi ? w : 0ull;
        }
    }
    sum = warp_reduce(sum, Add());
    __syncthreads();
    if (lane_id() == 0) sts64(r.mem + kWarpB + 8 * warp_id(), sum);
    __syncthreads();
    u64 block = 0, before = 0;
    for (int k = 0; k < kWarps; ++k) {
        const u64 w = lds64(r.mem + kWarpB + 8 * k);
        if (k < warp_id()) before += w;
        block += w;
    }
    const unsigned slot = r.mem + kSlots + 16 * r.turn;
    if (threadIdx.x == 0) sts64(slot, block);
    row_sync<kBlocks>();
    u64 below, total;
    over_blocks<kBlocks>(r, slot, below, total);
    before += below;
    r.turn ^= 1;
    const double want = share * (double)total + offset, reach = want < (double)total ? want : just_below((double)total);
    if (total && !((double)before > reach) && (double)(before + sum) > reach) {   // (one warp of all)
        for (int base = lo; base < hi; base += 32) {
            const int i = base + lane_id();
            const u64 v = i < hi ? f(r.x(i), i) : 0ull, to = before + warp_scan(v);
            const unsigned m = __ballot_sync(0xffffffffu, (double)to > reach);
            if (m) {
                if (lane_id() == __ffs(m) - 1) found(r.first + i);
                break;
            }
            before = __shfl_sync(0xffffffffu, to, 31);
        }
    }
    __syncwarp();
}

// The last kept value for a goal (a number of values, or p of the weight): sets r.last and r.last_index, or finishes the row
// where its candidates fit the list.  True: finished.
template <bool kBlocks, bool kWeigh>
__device__ static __forceinline__ bool cut(Row& r, float hi, float lo, double goal, int k, bool use_p, double p, double u, int* out) {
    Hit h = find_step<kBlocks, kWeigh>(r, hi, lo, goal, kWeigh, 0ull, 0ull);
    if (!h.found) return false;   // (fewer values than k: all are kept)
    if (kWeigh) goal *= (double)h.total;
    if (h.n_before + h.n <= kCap) {
        gather<kBlocks>(r, hi, lo, 0, h.bucket);
        if (r.mine == 0) finish_list(r, (int)(h.n_before + h.n), k, use_p, p, kWeigh ? h.total : 0ull, u, out);
        return true;
    }
    while (h.n > kCap) {   // a smaller step
        const Steps steps((double)lo, (double)hi);
        u64 most = 0, least = 0;   // (as ordered values, the smaller one inverted)
        for (int i = threadIdx.x; i < r.n; i += kThreads) {
            const float v = r.x(i);
            if (!r.kept(v, i) || v > hi || v < lo || steps.of(v) != h.bucket) continue;
            most = Max()(most, ordered(v));
            least = Max()(least, ~ordered(v));
        }
        largest<kBlocks>(r, most, least);
        hi = unordered((unsigned)most);
        lo = unordered(~(unsigned)least);
        if (!(lo < hi)) {   // equal values: so many of them, by index
            const float v = hi;
            u64 many;
            if (kWeigh) {
                const u64 w = r.weight(v);
                const double rest = ceil((goal - (double)h.w_before) / (double)w);
                many = rest < 1.0 ? 1ull : rest > (double)h.n ? h.n : (u64)rest;
                while (many > 1 && (double)(h.w_before + (many - 1) * w) >= goal) --many;
                while (many < h.n && (double)(h.w_before + many * w) < goal) ++many;
            } else {
                many = (u64)goal - h.n_before;
            }
            if (threadIdx.x == 0) sts32(r.mem + kLastIndex, 0u);
            select<kBlocks>(r, 0.0, (double)(many - 1), [&](float x, int i) -> u64 { return x == v && r.kept(x, i); },
                            [&](int index) { sts32(r.mem + kLastIndex, (unsigned)index + 1u); });
            row_sync<kBlocks>();
            const unsigned found = __reduce_max_sync(0xffffffffu, load32<kBlocks>(r.mem + kLastIndex, min((unsigned)lane_id(), r.blocks - 1)));
            r.last = v;
            r.last_index = (int)found - 1;
            return false;
        }
        h = find_step<kBlocks, kWeigh>(r, hi, lo, goal, false, h.n_before, h.w_before);
        if (!h.found) return false;
    }
    gather<kBlocks>(r, hi, lo, h.bucket, h.bucket);
    if (r.mine == 0) {   // the last one of the step's that is kept
        sort_list(r.mem + kList, (int)h.n);
        const int i0 = kEach * threadIdx.x;
        u64 key[kEach], w[kEach], sum = 0, all;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const bool there = i0 + j < (int)h.n;
            key[j] = there ? lds64(r.mem + kList + 8 * (i0 + j)) : 0ull;
            w[j] = !there ? 0ull : kWeigh ? r.weight(logit_of(key[j])) : 1ull;
            sum += w[j];
        }
        u64 before = (kWeigh ? h.w_before : h.n_before) + sum_before(r, sum, all);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (w[j] && (double)before < goal && (double)(before + w[j]) >= goal) {
                sts32(r.mem + kLast, ~(unsigned)(key[j] >> 32));
                sts32(r.mem + kLastIndex, (unsigned)key[j]);
            }
            before += w[j];
        }
    }
    row_sync<kBlocks>();
    r.last = unordered(load32<kBlocks>(r.mem + kLast, 0));
    r.last_index = (int)load32<kBlocks>(r.mem + kLastIndex, 0);
    return false;
}

};

template <class T, int kThreads, bool kBlocks>
__global__ void __launch_bounds__(kThreads, 512 / kThreads) sample_kernel(const T* __restrict__ logits, long long ld, int V, int part, unsigned blocks,
                                                             const float* __restrict__ us, const float* __restrict__ temperatures,
                                                             const int* __restrict__ top_ks, const float* __restrict__ top_ps,
                                                             const float* __restrict__ min_ps, int* __restrict__ out) {
    extern __shared__ __align__(16) unsigned char memory[];
    wait_for_earlier_kernels();
    const unsigned mem = (unsigned)__cvta_generic_to_shared(memory), mine = kBlocks ? blockIdx.x % blocks : 0u;
    const int b = blockIdx.x / blocks, first = min(V, (int)mine * part), n = min(V, first + part) - first;
    const double t = __ldg(temperatures + b), p = top_ps ? (double)__ldg(top_ps + b) : 1.0, least = min_ps ? (double)__ldg(min_ps + b) : 0.0;
    const int k = top_ks ? __ldg(top_ks + b) : 0;
    float u = __ldg(us + b);
    u = u >= 0.f ? fminf(u, 1.f) : 0.f;

    // this block's logits: 16 bytes at a time where they are aligned
    const T* src = logits + (size_t)b * ld + first;
    constexpr int kPer = 16 / (int)sizeof(T);
    const int head = min(n, (int)(((16 - (reinterpret_cast<uintptr_t>(src) & 15)) & 15) / sizeof(T))), body = (n - head) / kPer;
    float best = -INFINITY, least_v = INFINITY;   // (a thread's indices ascend: the first of equal ones stays)
    int best_at = 0;
    auto take = [&](float v, int i) {
        v = fmaxf(v, -INFINITY) + 0.f;   // (a NaN is -inf; one zero)
        sts32(mem + kLogits + 4 * i, __float_as_uint(v));
        if (v > best) {
            best = v;
            best_at = i;
        }
        least_v = fminf(least_v, v > -INFINITY ? v : INFINITY);
    };
    for (int i = threadIdx.x; i < head; i += kThreads) take(widen(src[i]), i);
#pragma unroll 4
    for (int j = threadIdx.x; j < body; j += kThreads) {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(src + head) + j);
        const T* f = reinterpret_cast<const T*>(&v);
#pragma unroll
        for (int e = 0; e < kPer; ++e) take(widen(f[e]), head + j * kPer + e);
    }
    for (int i = head + body * kPer + (int)threadIdx.x; i < n; i += kThreads) take(widen(src[i]), i);
    // largest value with the lowest index; smallest above -inf (inverted); zero: none
    u64 most = best > -INFINITY ? (u64)ordered(best) << 32 | ~(unsigned)(first + best_at) : 0ull, low = best > -INFINITY ? ~ordered(least_v) : 0ull;
    using S = Sampler<kThreads>;
    typename S::Row r{mem, n, first, blocks, mine, 0, 0, 0.0, 1.4426950408889634 / t, -INFINITY, -INFINITY, -1, least * kOne};
    S::template largest<kBlocks>(r, most, low);
    const float top = most ? unordered((unsigned)(most >> 32)) : -INFINITY;
    const int arg = most ? (int)~(unsigned)most : -1;
    // nothing to choose from, or the largest alone is kept
    const bool alone = arg < 0 || !(t > 0.0) || k == 1 || p <= 0.0 || !(least <= 1.0);
    if (alone) {
        if (mine == 0 && threadIdx.x == 0) out[b] = arg;
    } else {
        float lo = unordered(~(unsigned)low), hi = top;
        if (top == INFINITY) {   // infinite ones share the weight, the others have none
            for (int i = threadIdx.x; i < n; i += kThreads) sts32(mem + kLogits + 4 * i, __float_as_uint(r.x(i) == INFINITY ? 0.f : -INFINITY));
            __syncthreads();
            hi = lo = 0.f;
        }
        r.top = hi;
        r.low = lo = fmaxf(lo, __double2float_ru(r.top - kDeepest * t));
        if (!(lo < hi)) lo = hi - fmaxf(1.f, fabsf(hi) * 0.5f);   // (all the same)
        bool done = false;
        if (k > 0 && k < V) done = S::template cut<kBlocks, false>(r, hi, lo, (double)k, k, p < 1.0, p, u, out + b);
        if (!done && p < 1.0) done = S::template cut<kBlocks, true>(r, hi, lo, p, 0, true, p, u, out + b);
        if (!done)
            S::template select<kBlocks>(r, (double)u, 0.0,
                            [&](float v, int i) -> u64 {
                                const u64 w = r.weight(fmaxf(v, r.low));
                                return r.kept(v, i) && (double)w >= r.least ? w : 0ull;
                            },
                            [&](int index) { out[b] = index; });
    }
    row_sync<kBlocks>();   // (nobody leaves while another block may use its shared memory)
}

}  // namespace

qil_status launch_sample(const void* logits, qil_dtype type, long long ld, const float* u, const float* temperature, const int* top_k,
                         const float* top_p, const float* min_p, int* out, int B, int V, cudaStream_t st) {
    // Blocks of a row: of 4096 logits or more, eight at most (one row of 32 000, top-k and top-p: 12.3 us with eight, 14.7 with four,
    // 20.0 with two, 25.2 with one, of 512 threads each); fewer where the rows alone fill the GPU twice over, as long as two
    // blocks fit an SM's shared memory (64 rows of 32 000: 30.6 us with eight, 21.2 with four, of 256 threads each).
    unsigned blocks = 1;
    while (blocks < (unsigned)kMostBlocks && V > 4096 * (int)blocks) blocks *= 2;
    const auto part_of = [&](unsigned n) { return ((V + (int)n - 1) / (int)n + 7) & ~7; };
    while (blocks > 1 && (long long)B * blocks > 2 * num_sms() && (int)kLogits + 4 * part_of(blocks / 2) <= 112 * 1024) blocks /= 2;
    const int part = part_of(blocks);
    const size_t smem = kLogits + (size_t)part * 4;
    const dim3 grid((unsigned)B * blocks);
    auto go = [&](auto kernel, int threads, auto* x, std::atomic<unsigned long long>& allowed) {
        if (!allow_smem(kernel, (int)kLogits + QIL_SAMPLE_MAX_VOCAB / kMostBlocks * 4, allowed)) return QIL_ERR_CUDA;
        return launch_early_clusters(kernel, blocks, grid, threads, smem, st, x, ld, V, part, blocks, u, temperature, top_k, top_p, min_p, out);
    };
    auto of = [&](auto* x) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(x)>>;
        // 512 threads where every block has an SM (one row of 32 000: 12.3 us, with 256 13.0), else 256, two blocks an SM (64 rows of
        // 32 000, four blocks each: 29.5 us with 512, 21.2 with 256; 64 of 128 003, eight each, settings of every kind: 105 and 94)
        static std::atomic<unsigned long long> a{0}, b{0}, c{0}, d{0};
        if ((long long)B * blocks <= num_sms())
            return blocks == 1 ? go(sample_kernel<T, 512, false>, 512, x, a) : go(sample_kernel<T, 512, true>, 512, x, b);
        return blocks == 1 ? go(sample_kernel<T, 256, false>, 256, x, c) : go(sample_kernel<T, 256, true>, 256, x, d);
    };
    if (type == QIL_F32) return of(static_cast<const float*>(logits));
    if (type == QIL_BF16) return of(static_cast<const __nv_bfloat16*>(logits));
    return of(static_cast<const __half*>(logits));
}

}  // namespace qil
