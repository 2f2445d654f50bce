// Product of e4m3 matrices with a scale for each block of 128 along the inner axis (and 128 rows of the weights).
//
//     out[m][n] = sum_b a_scale[m][b] w_scale[n / 128][b] sum_{k in block b} a[m][k] w[n][k]
#include "layer.cuh"

#include <cuda_fp8.h>

namespace sketchssm {

namespace {

constexpr int kTile = 32;

__device__ __forceinline__ float e4m3(unsigned char x) {
    const __half_raw h = __nv_cvt_fp8_to_halfraw(x, __NV_E4M3);
    return __half2float(__half(h));
}

__global__ void __launch_bounds__(256) scaled_matmul_kernel(const MatmulParams p) {
    __shared__ float sa[kTile][kTile + 1], sw[kTile][kTile + 1];
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int tid = (int)threadIdx.x, tn = tid & 31, tm = tid >> 5;
    const int m0 = (int)blockIdx.y * kTile, n0 = (int)blockIdx.x * kTile;
    float acc[4] = {};
    for (int b = 0; b < p.KB; ++b) {
        float part[4] = {};
        for (int k0 = b * 128; k0 < min(p.K, b * 128 + 128); k0 += kTile) {
            __syncthreads();
            for (int i = tid; i < kTile * kTile; i += 256) {
                const int r = i / kTile, k = k0 + i % kTile;
                sa[r][i % kTile] = m0 + r < p.M && k < p.K ? e4m3(p.a[(size_t)(m0 + r) * p.K + k]) : 0.f;
                sw[r][i % kTile] = n0 + r < p.N && k < p.K ? e4m3(p.w[(size_t)(n0 + r) * p.K + k]) : 0.f;
            }
            __syncthreads();
            for (int k = 0; k < kTile; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) part[i] = fmaf(sa[tm * 4 + i][k], sw[tn][k], part[i]);
        }
        const int n = n0 + tn;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int m = m0 + tm * 4 + i;
            if (m < p.M && n < p.N) acc[i] = fmaf(p.a_scale[(size_t)m * p.KB + b] * p.w_scale[(size_t)(n / 128) * p.KB + b], part[i], acc[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = m0 + tm * 4 + i, n = n0 + tn;
        if (m < p.M && n < p.N) {
            if (p.out_bf16) static_cast<__nv_bfloat16*>(p.out)[m * p.out_stride + n] = __float2bfloat16_rn(acc[i]);
            else static_cast<float*>(p.out)[m * p.out_stride + n] = acc[i];
        }
    }
}

}  // namespace

int launch_scaled_matmul(Ctx* ctx, const MatmulParams& p, cudaStream_t stream) {
    if ((p.M + kTile - 1) / kTile > 65535) return SKETCHSSM_UNSUPPORTED_SHAPE;
    return launch_layer(ctx, scaled_matmul_kernel, dim3((unsigned)((p.N + kTile - 1) / kTile), (unsigned)((p.M + kTile - 1) / kTile)), dim3(256), 0, stream, p);
}

}  // namespace sketchssm
