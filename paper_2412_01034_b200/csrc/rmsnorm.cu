// Residual addition and root-mean-square norm of the decoder layer (the Llama-2 backbone of the OpenVLA deployment,
// App. A.4.2), with the output the next linear reads: bf16 (weight-only linears), or int8 codes and a scale per token
// (the W8A8 linear), or both.
//   h = x + residual (fp32)        residual_out = bf16(h)
//   y = h * rstd * w               rstd = 1 / sqrt(sum h^2 / K + eps)
//   s = max |y| / 127 (0 -> 1)     q = clamp(rint(y / s), -128, 127)
// The norm is taken of the unrounded sum.  Memory bound: x and the residual are read once, the row stays in registers
// between the statistics and the output.  max |y| = rstd * max |h w|, so that the sum of squares and the maximum need one
// reduction over the block, not two.  A block works on one row; a thread owns kVec vectors of 8 elements.
#include "layer_common.cuh"

namespace qil {

namespace {

template <int kVec>
__global__ void __launch_bounds__(1024) rmsnorm_kernel(const __nv_bfloat16* __restrict__ x, const __nv_bfloat16* __restrict__ residual,
                                                       const __nv_bfloat16* __restrict__ weight, __nv_bfloat16* __restrict__ residual_out,
                                                       __nv_bfloat16* __restrict__ y, int8_t* __restrict__ qy,
                                                       float* __restrict__ scales, int K, float eps) {
    __shared__ float s_sum[32], s_max[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    const size_t row = (size_t)blockIdx.x * K;
    const int nvec = K >> 3;
    float h[kVec][8], hw[kVec][8];
    float sum = 0.f, top = 0.f;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const int v = tid + i * blockDim.x;
        if (v < nvec) {
            unpack8(*reinterpret_cast<const uint4*>(x + row + 8 * (size_t)v), h[i]);
            float w[8];
            unpack8(__ldg(reinterpret_cast<const uint4*>(weight) + v), w);
            if (residual) {
                float r[8];
                unpack8(*reinterpret_cast<const uint4*>(residual + row + 8 * (size_t)v), r);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] += r[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sum = fmaf(h[i][j], h[i][j], sum);
                hw[i][j] = h[i][j] * w[j];
                top = fmaxf(top, fabsf(hw[i][j]));
            }
            if (residual_out) *reinterpret_cast<uint4*>(residual_out + row + 8 * (size_t)v) = pack8(h[i]);
        }
    }
    sum = warp_sum(sum);
    top = warp_max(top);
    if (lane == 0) {
        s_sum[warp] = sum;
        s_max[warp] = top;
    }
    __syncthreads();
    sum = warp_sum(lane < warps ? s_sum[lane] : 0.f);
    top = warp_max(lane < warps ? s_max[lane] : 0.f);
    const float rstd = 1.f / sqrtf(sum / (float)K + eps);
    const float most = top * rstd;                          // max |y|
    const float step = most == 0.f ? 1.f : most / 127.f;
    const float code = rstd / step;                         // y / step = (h w) * code
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const int v = tid + i * blockDim.x;
        if (v < nvec) {
            if (y) {
                float o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = hw[i][j] * rstd;
                *reinterpret_cast<uint4*>(y + row + 8 * (size_t)v) = pack8(o);
            }
            if (qy) {
                uint32_t q[2] = {0u, 0u};
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int c = max(-128, min(127, __float2int_rn(hw[i][j] * code)));
                    q[j >> 2] |= (uint32_t)(c & 0xFF) << (8 * (j & 3));
                }
                *reinterpret_cast<uint2*>(qy + row + 8 * (size_t)v) = make_uint2(q[0], q[1]);
            }
        }
    }
    if (qy && tid == 0) scales[blockIdx.x] = step;
}

}  // namespace

bool rmsnorm_supported(int K) { return K % 8 == 0 && K <= 32768; }

qil_status launch_rmsnorm(const void* x, const void* residual, const void* weight, void* residual_out, void* y, int8_t* qy,
                          float* scales, int M, int K, float eps, cudaStream_t st) {
    const int nvec = K / 8;
    const int vec = nvec <= 1024 ? 1 : nvec <= 2048 ? 2 : 4;
    const int threads = ((nvec + vec - 1) / vec + 31) / 32 * 32;
    auto go = [&](auto kernel) {
        kernel<<<(unsigned)M, threads, 0, st>>>(
            reinterpret_cast<const __nv_bfloat16*>(x), reinterpret_cast<const __nv_bfloat16*>(residual),
            reinterpret_cast<const __nv_bfloat16*>(weight), reinterpret_cast<__nv_bfloat16*>(residual_out),
            reinterpret_cast<__nv_bfloat16*>(y), qy, scales, K, eps);
    };
    if (vec == 1) go(rmsnorm_kernel<1>);
    else if (vec == 2) go(rmsnorm_kernel<2>);
    else go(rmsnorm_kernel<4>);
    return launch_status();
}

}  // namespace qil
