// The quantised paged cache: rotary embedding with an append that quantises as it writes, and the read-back.
//   One scale per token and key head (bf16), with 4 bits also a zero point (bf16, a whole number), of the head's D values v:
//   8 bits   a = max |v|;  s = bf16(a / 127);  q = clamp(rint(v / s), -128, 127);  the code stands for q s
//   4 bits   lo = min(0, min v), hi = max(0, max v);  s = bf16((hi - lo) / 15);  z = clamp(rint(-lo / s), 0, 15);
//            q = clamp(rint(v / s) + z, 0, 15);  the code stands for (q - z) s
//   s < 2^-126: the head counts as zeros (s = 1); a value or a scale that is not finite: s = NaN, all codes zero.
// Every operation is an fp32 operation rounded on its own (a key is turned by two products and a sum, without a fused
// multiply-add), so that the codes are defined to the bit.  The scale is held in 16 bits because a code is rounded against the
// rounded scale: half a step more range at the most, and the products with it are exact in the kernels that read it.
//
// Both kernels are one pass.  Append: a thread turns 8 pairs or takes 16 values, the D / 16 threads of a head find its range by
// shuffles.  5466 tokens of 32 + 32 + 32 heads of 128: 57.1 us with 8 bits, 64.5 with 4, where the copy rate would allow 35 and 31:
// it waits for instructions, about 400 a warp, and for their latency (73 us with a division per code; with 62 registers a thread
// instead of 40, which six blocks an SM allow, 69; with the page by a division and a choice for every value of a head without
// codes, 61.7).  They are the definition's separate roundings, and what every thread does for its one head: the request and the
// page, 64 bytes of cosines and sines for 32 bytes of a turned head, and the 52 (4 bits: 76) bytes that 40 registers do not hold.
// Read-back: a warp takes up to 512 values of a token's keys and the same of its values; the same tokens 26.0 and
// 23.1 us, 79 and 75 % of the copy rate.
#include "kv_quant.cuh"

namespace qil {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ int page_shift(int page_size) { return 31 - __clz(page_size); }   // (a power of two)

// rint(v / s) + 1.5 2^23 by the reciprocal of s, where that decides: v times it is off by 2^-24 of 128 (8e-6) at most, so that the
// division itself has to be taken only within 2e-5 of a half (`far` collects the distances from whole numbers).
constexpr float kMagic = 12582912.f;
__device__ __forceinline__ float rounded(float v, float inv, float& far) {
    const float t = fmaf(v, inv, kMagic);
    far = fmaxf(far, fabsf(fmaf(v, inv, kMagic - t)));
    return t;
}
__device__ __forceinline__ uint2 bytes8(const float (&t)[8]) {
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lo = __byte_perm(__float_as_uint(t[4 * h]), __float_as_uint(t[4 * h + 1]), 0x0040);
        const uint32_t hi = __byte_perm(__float_as_uint(t[4 * h + 2]), __float_as_uint(t[4 * h + 3]), 0x0040);
        w[h] = __byte_perm(lo, hi, 0x5410);
    }
    return make_uint2(w[0], w[1]);
}
// (t - kMagic + z, at most 15, for each of eight: whole numbers below 2^16 are exact on the way)
__device__ __forceinline__ uint32_t nibbles8(const float (&t)[8], float z) {
    float q[8], w[2];
    const float less = z - kMagic;
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = fminf(t[e] + less, 15.f);
#pragma unroll
    for (int h = 0; h < 2; ++h) w[h] = fmaf(fmaf(fmaf(q[4 * h + 3], 16.f, q[4 * h + 2]), 16.f, q[4 * h + 1]), 16.f, q[4 * h]) + kMagic;
    return __byte_perm(__float_as_uint(w[0]), __float_as_uint(w[1]), 0x5410);
}

template <int kDim, int kBits>
__global__ void __launch_bounds__(kThreads, 6) rope_append_q_kernel(const __nv_bfloat16* __restrict__ qkv, const float* __restrict__ cos_sin,
                                                                 __nv_bfloat16* __restrict__ q_out, QuantCache kvq, PagedCache c, int max_pos,
                                                                 int pieces) {
    constexpr int kHalf = kDim / 2, kPer = kHalf / 8;   // threads of a head: 8 pairs or 16 values each
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
    size_t row = 0;   // of the cache: (page, head, slot)
    bool there = head < H;
    if (!there && known) {
        const int page_at = pos >> page_shift(c.page_size), slot = pos & (c.page_size - 1);
        const int page = page_at < c.max_pages ? __ldg(c.block_table + (size_t)seq * c.max_pages + page_at) : -1;
        there = page >= 0 && page < c.num_pages;
        row = ((size_t)(there ? page : 0) * Hk + (head - H - (turn ? 0 : Hk))) * c.page_size + slot;
    }
    if (!there) return;   // (the threads of a head agree on all of this)
    float a[8], b[8], u[8], v[8];
    unpack8(first, a);
    unpack8(second, b);
    if (turn) {
        const float4* cs = reinterpret_cast<const float4*>(cos_sin + (size_t)(known ? pos : 0) * kDim + o);
        const float4 co[2] = {__ldg(cs), __ldg(cs + 1)}, si[2] = {__ldg(cs + kHalf / 4), __ldg(cs + kHalf / 4 + 1)};
        const float cv[8] = {co[0].x, co[0].y, co[0].z, co[0].w, co[1].x, co[1].y, co[1].z, co[1].w};
        const float sv[8] = {si[0].x, si[0].y, si[0].z, si[0].w, si[1].x, si[1].y, si[1].z, si[1].w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            u[e] = __fsub_rn(__fmul_rn(a[e], cv[e]), __fmul_rn(b[e], sv[e]));
            v[e] = __fadd_rn(__fmul_rn(b[e], cv[e]), __fmul_rn(a[e], sv[e]));
        }
        if (head < H) {
            __nv_bfloat16* dst = q_out + ((size_t)t * H + head) * kDim + o;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                u[e] = known ? u[e] : 0.f;
                v[e] = known ? v[e] : 0.f;
            }
            *reinterpret_cast<uint4*>(dst) = pack8(u);
            *reinterpret_cast<uint4*>(dst + kHalf) = pack8(v);
            return;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            u[e] = a[e];
            v[e] = b[e];
        }
    }
    // the head's range over its threads
    float low = 0.f, high = 0.f, nan = 0.f;   // (8 bits: high alone, of |v|; nan: zero, or a NaN where a value is not finite)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        nan = fmaf(u[e], 0.f, fmaf(v[e], 0.f, nan));
        if (kBits == 8) {
            high = fmaxf(high, fmaxf(fabsf(u[e]), fabsf(v[e])));
        } else {
            low = fminf(low, fminf(u[e], v[e]));
            high = fmaxf(high, fmaxf(u[e], v[e]));
        }
    }
    high += nan;   // (stays a NaN in the maxima below by its bits: above infinity's)
    uint32_t most = __float_as_uint(fabsf(high));
    const unsigned mine = ((1u << kPer) - 1u) << (threadIdx.x & 31 & ~(kPer - 1));
#pragma unroll
    for (int x = 1; x < kPer; x <<= 1) {
        most = max(most, __shfl_xor_sync(mine, most, x));
        if (kBits == 4) low = fminf(low, __shfl_xor_sync(mine, low, x));
    }
    high = __uint_as_float(most);
    const float exact = kBits == 8 ? __fdiv_rn(high, 127.f) : __fdiv_rn(__fsub_rn(high, low), 15.f);
    float s = __bfloat162float(__float2bfloat16_rn(exact));
    const bool strange = !(high < INFINITY) || !(s < INFINITY), none = s < 1.17549435e-38f;
    if (strange || none) s = 1.f;
    const bool codes = !strange && !none;
    // (v / s is below 127.5, or 15.1: the scale is rounded by 2^-8 of it at most; only rint(v / s) + z can be one too large)
    const float inv = codes ? __frcp_rn(s) : 0.f;
    float z = 0.f;
    if (kBits == 4 && codes) z = rintf(__fdiv_rn(-low, s));
    float qu[8], qv[8], far = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {   // (0 times an infinity: NaN, which `far` passes over; the words are cleared below)
        qu[e] = rounded(u[e], inv, far);
        qv[e] = rounded(v[e], inv, far);
    }
    if (far > 0.49998f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            qu[e] = rintf(__fdiv_rn(u[e], s)) + kMagic;
            qv[e] = rintf(__fdiv_rn(v[e], s)) + kMagic;
        }
    }
    if (kBits == 8) {
        unsigned char* dst = static_cast<unsigned char*>(turn ? kvq.k : kvq.v) + row * kDim;
        uint2 x = bytes8(qu), y = bytes8(qv);
        if (!codes) x = y = make_uint2(0u, 0u);
        if (turn) {
            *reinterpret_cast<uint2*>(dst + o) = x;
            *reinterpret_cast<uint2*>(dst + o + kHalf) = y;
        } else {
            *reinterpret_cast<uint4*>(dst + 2 * o) = make_uint4(x.x, x.y, y.x, y.y);
        }
    } else {
        uint32_t* dst = static_cast<uint32_t*>(turn ? kvq.k : kvq.v) + row * (kDim / 8);
        uint2 x = make_uint2(nibbles8(qu, z), nibbles8(qv, z));
        if (!codes) x = make_uint2(0u, 0u);
        if (turn) {
            dst[o / 8] = x.x;
            dst[(o + kHalf) / 8] = x.y;
        } else {
            *reinterpret_cast<uint2*>(dst + 2 * o / 8) = x;
        }
    }
    if (o == 0) {
        const uint32_t held_scale = strange ? 0x7FC0u : __float_as_uint(s) >> 16;   // (s is a bf16 value)
        __nv_bfloat16* to = turn ? kvq.ks : kvq.vs;
        if (kBits == 8) reinterpret_cast<uint16_t*>(to)[row] = (uint16_t)held_scale;
        else reinterpret_cast<uint32_t*>(to)[row] = held_scale | (__float_as_uint(z) & 0xFFFF0000u);
    }
}

// 16 values of one head of one cached token
template <int kDim, int kBits>
__device__ __forceinline__ void read16(const void* codes, const __nv_bfloat16* scales, size_t row, int o, uint4 (&w)[2], uint32_t& par) {
    if (kBits == 8) {
        w[0] = __ldg(reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(codes) + row * kDim + o));
        par = __ldg(reinterpret_cast<const unsigned short*>(scales) + row);
    } else {
        const uint2 x = __ldg(reinterpret_cast<const uint2*>(static_cast<const uint32_t*>(codes) + row * (kDim / 8) + o / 8));
        w[0] = make_uint4(x.x, x.y, 0u, 0u);
        par = __ldg(reinterpret_cast<const uint32_t*>(scales) + row);
    }
}
template <int kBits>
__device__ __forceinline__ void write16(__nv_bfloat16* dst, const uint4 w, uint32_t par) {
    const float s = __uint_as_float(par << 16), z = __uint_as_float(par & 0xFFFF0000u);
    float f[2][8];
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const float q = kBits == 8 ? (float)(signed char)(x[e >> 2] >> (8 * (e & 3))) : (float)((x[e >> 3] >> (4 * (e & 7))) & 15u) - z;
        f[e >> 3][e & 7] = q * s;
    }
    *reinterpret_cast<uint4*>(dst) = pack8(f[0]);
    *reinterpret_cast<uint4*>(dst + 8) = pack8(f[1]);
}

template <int kDim, int kBits>
__global__ void __launch_bounds__(kThreads) kv_read_q_kernel(QuantCache kvq, PagedCache c, __nv_bfloat16* __restrict__ k_out,
                                                             __nv_bfloat16* __restrict__ v_out, int chunks) {
    constexpr int kPer = kDim / 16;
    wait_for_earlier_kernels();
    // (rows times heads are below 2^31, and so are the warps)
    const unsigned at = blockIdx.x * (kThreads / 32u) + (threadIdx.x >> 5), row_at = at / (unsigned)chunks;
    const int Hk = c.num_kv_heads, piece = (int)(at - row_at * chunks) * 32 + (threadIdx.x & 31);
    if (row_at >= (unsigned)c.total_q) return;   // (whole warps)
    const int t = (int)row_at;
    int seq = 0, lo = 0, hi = 0, kv = 0;
    const bool held = request_at_row(c.cu_q, c.kv_len, c.num_seqs, c.total_q, t, seq, lo, hi, kv);
    if (!held || t < lo || piece >= Hk * kPer) return;   // (a row of no request stays as it is)
    const int pos = kv - (hi - lo) + (t - lo), head = piece / kPer, o = (piece % kPer) * 16;
    const int page_at = pos >> page_shift(c.page_size), slot = pos & (c.page_size - 1);
    const int page = pos >= 0 && page_at < c.max_pages ? __ldg(c.block_table + (size_t)seq * c.max_pages + page_at) : -1;
    const size_t to = ((size_t)t * Hk + head) * kDim + o;
    uint4 kw[2] = {}, vw[2] = {};
    uint32_t kp = 0u, vp = 0u;   // (a scale of zero: zeros)
    if (page >= 0 && page < c.num_pages) {
        const size_t row = ((size_t)page * Hk + head) * c.page_size + slot;
        read16<kDim, kBits>(kvq.k, kvq.ks, row, o, kw, kp);
        read16<kDim, kBits>(kvq.v, kvq.vs, row, o, vw, vp);
    }
    write16<kBits>(k_out + to, kw[0], kp);
    write16<kBits>(v_out + to, vw[0], vp);
}

}  // namespace

qil_status launch_rope_append_q(const void* qkv, const float* cos_sin, void* q_out, const QuantCache& kvq, const PagedCache& c, int max_pos,
                                cudaStream_t st) {
    const int pieces = (c.num_heads + 2 * c.num_kv_heads) * (c.head_dim / 16);
    const dim3 grid((unsigned)c.total_q, (unsigned)((pieces + kThreads - 1) / kThreads));
    auto go = [&](auto kernel) {
        return launch_early(kernel, grid, kThreads, 0, st, reinterpret_cast<const __nv_bfloat16*>(qkv), cos_sin,
                            reinterpret_cast<__nv_bfloat16*>(q_out), kvq, c, max_pos, pieces);
    };
    if (c.head_dim == 128) return kvq.bits == 8 ? go(rope_append_q_kernel<128, 8>) : go(rope_append_q_kernel<128, 4>);
    return kvq.bits == 8 ? go(rope_append_q_kernel<64, 8>) : go(rope_append_q_kernel<64, 4>);
}

qil_status launch_kv_read_q(const QuantCache& kvq, const PagedCache& c, void* k_out, void* v_out, cudaStream_t st) {
    const int chunks = (c.num_kv_heads * (c.head_dim / 16) + 31) / 32;
    const long long warps = (long long)c.total_q * chunks;
    const dim3 grid((unsigned)((warps + kThreads / 32 - 1) / (kThreads / 32)));
    auto go = [&](auto kernel) {
        return launch_early(kernel, grid, kThreads, 0, st, kvq, c, reinterpret_cast<__nv_bfloat16*>(k_out),
                            reinterpret_cast<__nv_bfloat16*>(v_out), chunks);
    };
    if (c.head_dim == 128) return kvq.bits == 8 ? go(kv_read_q_kernel<128, 8>) : go(kv_read_q_kernel<128, 4>);
    return kvq.bits == 8 ? go(kv_read_q_kernel<64, 8>) : go(kv_read_q_kernel<64, 4>);
}

}  // namespace qil
