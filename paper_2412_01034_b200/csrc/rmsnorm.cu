// Residual addition and root-mean-square norm of the decoder layer (the Llama-2 backbone of the OpenVLA deployment,
// App. A.4.2), with the output the next linear reads: bf16 (weight-only linears), or int8 codes and a scale per token
// (the W8A8 linear), or both.
//   h = x + residual (fp32)        residual_out = bf16(h)
//   y = h * rstd * w               rstd = 1 / sqrt(sum h^2 / K + eps)
//   s = max |y| / 127 (0 -> 1)     q = clamp(rint(y / s), -128, 127)
// The norm is taken of the unrounded sum.  Memory bound: x and the residual are read once, the row stays in registers
// between the statistics and the output.  max |y| = rstd * max |h w|, so that the sum of squares and the maximum need one
// reduction over the block, not two.  A block works on one row at a time, a thread on kVec vectors of 8 elements; the
// next row's vectors are on their way while this one is reduced and written, and the weights are read once per block.
#include "layer_common.cuh"

namespace qil {

namespace {

// Where max |h w| is less, the factor of the codes (127 / max |h w|) would come near the end of fp32's range: such a row has
// the codes and the scale of zeros.  (Products lifted by a power of two instead cost up to 15 % of every row's time.)
constexpr float kLeast = 0x1p-119f;

template <int kVec, bool kResidual>
__global__ void __launch_bounds__(kVec == 1 ? 256 : 1024) rmsnorm_kernel(const __nv_bfloat16* x, const __nv_bfloat16* residual,
                                                       const __nv_bfloat16* __restrict__ weight, __nv_bfloat16* residual_out,
                                                       __nv_bfloat16* __restrict__ y, int8_t* __restrict__ qy,
                                                       float* __restrict__ scales, int M, int K, float eps) {
    __shared__ float s_sum[2][32], s_max[2][32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    const int nvec = K >> 3;
    wait_for_earlier_kernels();
    uint4 xv[kVec], rv[kVec], wv[kVec];
    // (threads past the row's end repeat its last vector and count for nothing: no condition around a load)
    auto load = [&](int row) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const size_t at = (size_t)row * K + 8 * (size_t)min(tid + i * (int)blockDim.x, nvec - 1);
            xv[i] = *reinterpret_cast<const uint4*>(x + at);
            if (kResidual) rv[i] = *reinterpret_cast<const uint4*>(residual + at);
        }
    };
    constexpr bool kAhead = kVec < 4;   // (four vectors of two rows would not fit the registers of 1024 threads)
    if (kAhead) load(blockIdx.x);
#pragma unroll
    for (int i = 0; i < kVec; ++i) wv[i] = __ldg(reinterpret_cast<const uint4*>(weight) + min(tid + i * (int)blockDim.x, nvec - 1));
    int half = 0;
#pragma unroll 1
    for (int row = blockIdx.x; row < M; row += gridDim.x, half ^= 1) {
        float h[kVec][8], sum = 0.f, top = kLeast;
        if (!kAhead) load(row);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            unpack8(xv[i], h[i]);
            if (kResidual) {
                float r[8];
                unpack8(rv[i], r);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] += r[j];
            }
        }
        if (kAhead && row + (int)gridDim.x < M) load(row + gridDim.x);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int v = tid + i * blockDim.x;
            float w[8];
            unpack8(wv[i], w);
            if (kResidual && residual_out && v < nvec) *reinterpret_cast<uint4*>(residual_out + (size_t)row * K + 8 * (size_t)v) = pack8(h[i]);
            float part = 0.f, most = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                part = fmaf(h[i][j], h[i][j], part);
                h[i][j] *= w[j];
                most = fmaxf(most, fabsf(h[i][j]));
            }
            sum += v < nvec ? part : 0.f;
            top = fmaxf(top, v < nvec ? most : 0.f);   // (a repeated vector may already hold the row's results, in place)
        }
        sum = warp_sum(sum);
        top = warp_max(top);
        if (lane == 0) {
            s_sum[half][warp] = sum;
            s_max[half][warp] = top;
        }
        __syncthreads();   // (the halves take turns: the next row's values cannot meet this row's readers)
        sum = warp_sum(lane < warps ? s_sum[half][lane] : 0.f);
        top = warp_max(lane < warps ? s_max[half][lane] : 0.f);
        const float rstd = 1.f / sqrtf(sum / (float)K + eps);
        const float most = top * rstd;                          // max |y|
        const float step = most == kLeast * rstd ? 1.f : most / 127.f;   // (a row with a NaN has a step of NaN, also one of NaN alone)
        const float code = rstd / step;                         // y / step = (h w) * code
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int v = tid + i * blockDim.x;
            if (v >= nvec) continue;
            const size_t at = (size_t)row * K + 8 * (size_t)v;
            if (qy) {
                // 1.5 * 2^23 + v: the nearest integer in the low bits (the conversion instructions run at a quarter of the
                // rate and set the pace).  |v| <= 127 up to rounding, so that no code needs the clamp.
                uint32_t q[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) q[j] = __float_as_uint(fmaf(h[i][j], code, 12582912.f));
#pragma unroll
                for (int j = 0; j < 8; j += 4)
                    q[j] = __byte_perm(__byte_perm(q[j], q[j + 1], 0x0040), __byte_perm(q[j + 2], q[j + 3], 0x0040), 0x5410);
                *reinterpret_cast<uint2*>(qy + at) = make_uint2(q[0], q[4]);
            }
            if (y) {
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] *= rstd;
                *reinterpret_cast<uint4*>(y + at) = pack8(h[i]);
            }
        }
        if (qy && tid == 0) scales[row] = step;
    }
}

}  // namespace

bool rmsnorm_supported(int K) { return K % 8 == 0 && K <= 32768; }

qil_status launch_rmsnorm(const void* x, const void* residual, const void* weight, void* residual_out, void* y, int8_t* qy,
                          float* scales, int M, int K, float eps, cudaStream_t st) {
    const int nvec = K / 8;
    const int vec = nvec <= 256 ? 1 : nvec <= 2048 ? 2 : 4;
    const int threads = ((nvec + vec - 1) / vec + 31) / 32 * 32;
    // One round of blocks, which take the rows in turn (64 registers a thread: 1024 threads per SM).  8192 rows of 4096 with
    // residual and int8 output: 41.3 us = 5.7 TB/s, 87 % of the copy rate (one vector a thread took 2 us more, one block per
    // row 12 us more); a single row 2.9 us.  Rows of more than 16384 take four vectors a thread, whose registers spill (72 to 76
    // bytes a thread, and no next row on the way): 1024 rows of 32768 49 us = 4.8 TB/s.
    const long long room = (long long)num_sms() * (threads < 1024 ? 1024 / threads : 1);
    const unsigned grid = (unsigned)(M < room ? M : room);
    auto go = [&](auto kernel) {
        return launch_early(kernel, dim3(grid), threads, 0, st, reinterpret_cast<const __nv_bfloat16*>(x),
                            reinterpret_cast<const __nv_bfloat16*>(residual), reinterpret_cast<const __nv_bfloat16*>(weight),
                            reinterpret_cast<__nv_bfloat16*>(residual_out), reinterpret_cast<__nv_bfloat16*>(y), qy, scales, M, K, eps);
    };
    if (vec == 1) return residual ? go(rmsnorm_kernel<1, true>) : go(rmsnorm_kernel<1, false>);
    if (vec == 2) return residual ? go(rmsnorm_kernel<2, true>) : go(rmsnorm_kernel<2, false>);
    return residual ? go(rmsnorm_kernel<4, true>) : go(rmsnorm_kernel<4, false>);
}

}  // namespace qil
