// What the attention kernels over the quantised cache share.  Rows, visibility and workspace are those of attn_paged.cuh.
#pragma once

#include "attn_paged.cuh"
#include "kv_quant.cuh"

namespace qil {

struct AttnQuantParams {
    AttnParams a;     // (a.k and a.v are unused)
    QuantCache kv;
};

// Pairs of codes as bf16 pairs, exact.  128 + n is 0x4300 | n for n < 128.
__device__ __forceinline__ uint32_t bf2_sub(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// (x & mask) | 0x43004300
template <uint32_t mask>
__device__ __forceinline__ uint32_t plus128(uint32_t x) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(x), "n"(mask), "n"(0x43004300u));
    return d;
}
// the signed bytes 0 and 2 of x: (128 + low 7 bits) - (128, or 256 where the sign bit is set)
__device__ __forceinline__ uint32_t bytes02(uint32_t x) { return bf2_sub(plus128<0x007F007Fu>(x), plus128<0x00800080u>(x)); }

qil_status launch_attn_few_q(const AttnQuantParams& p, cudaStream_t st);
qil_status launch_attn_many_q(const AttnQuantParams& p, cudaStream_t st);

}  // namespace qil
