// Root-mean-square norm of rows (or of groups of a row) with what stands around it in a layer: the residual's addition before
// it, or the skip and the gate of the recurrence's output, and behind it the 8-bit rows with a scale for each block of 128
// that the next projection takes.
//
//     h = x + residual   or   h = (x + skip skip_weight) silu(gate);   y = h / sqrt(mean(h^2) + eps) weight
//     scale = max|y| / 448 over 128 elements,  out8 = e4m3(y 448 / max|y|)
//
// Every input is read once and every output written once, so HBM bounds it: a row (group) stays in the registers of the threads
// that share it, NV vectors of eight elements each, between the sum of squares and the result.  A block of 128 is sixteen
// neighbouring lanes' vectors, so its largest value takes four shuffles.  16384 rows of 2048 with the residual, bf16: 46 us, 5.1 TB/s.
#include "layer.cuh"

#include <cuda_fp8.h>

namespace sketchssm {

namespace {

// Eight consecutive elements as floats.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&f)[8]) {
    if constexpr (sizeof(T) == 2) {
        Vec16<T>::unpack(*reinterpret_cast<const uint4*>(p), f);
    } else {
        float a[4], b[4];
        Vec16<T>::unpack(reinterpret_cast<const uint4*>(p)[0], a);
        Vec16<T>::unpack(reinterpret_cast<const uint4*>(p)[1], b);
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[i] = a[i]; f[4 + i] = b[i]; }
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&f)[8]) {
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4*>(p) = Vec16<T>::pack(f);
    } else {
        reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
}

// blockDim.x threads (a multiple of 32) share a row; blockDim.y rows per CTA.  MODE 0: plain, 1: residual, 2: gate.
template <typename T, typename X, int NV, int MODE>
__global__ void __launch_bounds__(512) rms_norm_kernel(const NormParams p) {
    __shared__ float sums[32];
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int tx = (int)threadIdx.x, nt = (int)blockDim.x;
    const long long unit = (long long)blockIdx.x * blockDim.y + threadIdx.y;     // (row, group)
    const bool live = unit < (long long)p.rows * p.groups;
    const long long row = live ? unit / p.groups : 0;
    const int g0 = live ? (int)(unit - row * p.groups) * p.group : 0;
    float h[NV][8];
    float sq = 0.f;
    // Short rows: the weights are asked for with the row, not a round trip behind it.
    constexpr bool kAhead = NV == 1;
    float4 ahead[kAhead ? NV : 1][2];
    if constexpr (kAhead) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int i = (v * nt + tx) * 8;
            if (live && i < p.group) {
                ahead[v][0] = *reinterpret_cast<const float4*>(p.weight + g0 + i);
                ahead[v][1] = *reinterpret_cast<const float4*>(p.weight + g0 + i + 4);
            }
        }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int i = (v * nt + tx) * 8;                // inside the group
        const bool in = live && i < p.group;
        const int e = g0 + i;
#pragma unroll
        for (int j = 0; j < 8; ++j) h[v][j] = 0.f;
        if (in) {
            load8(static_cast<const X*>(p.x) + row * p.x_stride + e, h[v]);
            float f[8];
            if constexpr (MODE == 1) {
                load8(static_cast<const T*>(p.residual) + row * p.width + e, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[v][j] += f[j];
                store8(static_cast<T*>(p.residual_out) + row * p.width + e, h[v]);
            }
            if constexpr (MODE == 2) {
                if (p.skip != nullptr) {
                    load8(static_cast<const T*>(p.skip) + row * p.skip_stride + e, f);
                    const int per = p.width / p.skip_heads;
                    if ((per & 7) == 0) {
                        const float s = p.skip_weight[e / per];
#pragma unroll
                        for (int j = 0; j < 8; ++j) h[v][j] = fmaf(s, f[j], h[v][j]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) h[v][j] = fmaf(p.skip_weight[(e + j) / per], f[j], h[v][j]);
                    }
                }
                load8(static_cast<const T*>(p.gate) + row * p.gate_stride + e, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[v][j] *= silu<T>(f[j]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sq = fmaf(h[v][j], h[v][j], sq);
        }
    }
    sq = warp_sum(sq);
    if (nt > 32) {                                      // one row per CTA then
        if ((tx & 31) == 0) sums[tx >> 5] = sq;
        __syncthreads();
        sq = 0.f;
        for (int i = 0; i < nt / 32; ++i) sq += sums[i];
    }
    const float r = rsqrtf(sq / (float)p.group + p.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int i = (v * nt + tx) * 8;
        const bool in = live && i < p.group;
        const int e = g0 + i;
        float top = 0.f;
        if (in) {
            float4 w0, w1;
            if constexpr (kAhead) {
                w0 = ahead[v][0];
                w1 = ahead[v][1];
            } else {
                w0 = *reinterpret_cast<const float4*>(p.weight + e);
                w1 = *reinterpret_cast<const float4*>(p.weight + e + 4);
            }
            const float w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[v][j] = h[v][j] * r * w[j];
                top = fmaxf(top, fabsf(h[v][j]));
            }
            if (p.out != nullptr) store8(static_cast<T*>(p.out) + row * p.width + e, h[v]);
        }
        if (p.out8 != nullptr) {
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            if (in) {
                const float inv = top > 1e-30f ? 448.f / top : 0.f;
                uint32_t w[2];
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const __nv_fp8x2_storage_t lo = __nv_cvt_float2_to_fp8x2(make_float2(h[v][4 * q] * inv, h[v][4 * q + 1] * inv), __NV_SATFINITE, __NV_E4M3);
                    const __nv_fp8x2_storage_t hi = __nv_cvt_float2_to_fp8x2(make_float2(h[v][4 * q + 2] * inv, h[v][4 * q + 3] * inv), __NV_SATFINITE, __NV_E4M3);
                    w[q] = (uint32_t)lo | ((uint32_t)hi << 16);
                }
                *reinterpret_cast<uint2*>(static_cast<unsigned char*>(p.out8) + row * p.width + e) = make_uint2(w[0], w[1]);
                if ((e & 127) == 0) p.scale[row * ((p.width + 127) / 128) + e / 128] = top * (1.f / 448.f);
            }
        }
    }
}

template <typename T, typename X, int NV>
int norm_mode(Ctx* ctx, const NormParams& p, dim3 grid, dim3 block, cudaStream_t stream) {
    if (p.gate != nullptr) return launch_layer(ctx, rms_norm_kernel<T, X, NV, 2>, grid, block, 0, stream, p);
    if (p.residual != nullptr) return launch_layer(ctx, rms_norm_kernel<T, X, NV, 1>, grid, block, 0, stream, p);
    return launch_layer(ctx, rms_norm_kernel<T, X, NV, 0>, grid, block, 0, stream, p);
}

template <typename T, typename X>
int norm_types(Ctx* ctx, const NormParams& p, cudaStream_t stream) {
    const int vecs = (p.group + 7) / 8;                 // of the longest part that threads share
    const long long units = (long long)p.rows * p.groups;
    // Two vectors a thread (16384 rows of 2048: 46 us; four 50, eight in a warp without a barrier 74), with few rows one, for a short
    // chain; long rows as many as 512 threads leave.
    int nv = units * vecs >= (long long)sm_count(ctx) * 1024 ? 2 : 1;
    while (nv < 4 && (vecs + nv - 1) / nv > 512) nv *= 2;
    const int tx = ((vecs + nv - 1) / nv + 31) / 32 * 32;
    const int rows_per_cta = tx == 32 ? 4 : 1;
    const dim3 block((unsigned)tx, (unsigned)rows_per_cta), grid((unsigned)((units + rows_per_cta - 1) / rows_per_cta));
    if (nv == 4) return norm_mode<T, X, 4>(ctx, p, grid, block, stream);
    if (nv == 2) return norm_mode<T, X, 2>(ctx, p, grid, block, stream);
    return norm_mode<T, X, 1>(ctx, p, grid, block, stream);
}

}  // namespace

int launch_rms_norm(Ctx* ctx, const NormParams& p, bool bf16, cudaStream_t stream) {
    if (bf16) return p.x_bf16 ? norm_types<__nv_bfloat16, __nv_bfloat16>(ctx, p, stream) : norm_types<__nv_bfloat16, float>(ctx, p, stream);
    return p.x_bf16 ? norm_types<float, __nv_bfloat16>(ctx, p, stream) : norm_types<float, float>(ctx, p, stream);
}

}  // namespace sketchssm
