// Root-mean-square norm with the residual's addition before it, or of every head's output with the gate behind it, and the rows in 8-bit
// integers with a scale for each of them that the next projection takes.
//
//     h = x  or  x + residual;   y = h / sqrt(mean(h^2) + eps) weight   in groups of `group` elements;   with gate: y act(gate)
//     scale = max|y| / 127 over the row,  out8 = round(y 127 / max|y|)
//
// Every input is read once and every output written once, so HBM bounds it.  A row belongs to one CTA (four short rows to four warps of one)
// and stays in its threads' registers, NV vectors of eight elements each: a group's sum of squares and the row's largest value are both
// needed before an element of it can be written.  A group is whole vectors of neighbouring threads, any number of them: where it is
// not the row, every vector's own sum goes through shared memory and each thread adds up those of its group.
#include "layer.cuh"

namespace sketchssm {

namespace {

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

// To the nearest integer, ties to even, as a byte (what is not a number: 0).
__device__ __forceinline__ uint32_t byte_of(float x) {
    int i;
    asm("cvt.rni.sat.s8.f32 %0, %1;" : "=r"(i) : "f"(x));
    return (uint32_t)i & 0xffu;
}

// blockDim.x threads (a multiple of 32) share a row; blockDim.y rows per CTA, more than one only with 32 threads each.
// MODE 0: plain, 1: residual, 2: gate.  GROUPS: the row is more than one group.
template <typename T, typename X, int NV, int MODE, bool GROUPS>
__global__ void __launch_bounds__(512) integer_norm_kernel(const Norm8Params p) {
    extern __shared__ float part[];                     // GROUPS: [rows][width / 8] sums of squares
    __shared__ float sums[32], tops[32];
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int tx = (int)threadIdx.x, nt = (int)blockDim.x;
    const long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const bool live = row < p.rows;
    float h[NV][8];
    float sq = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int e = (v * nt + tx) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) h[v][j] = 0.f;
        if (live && e < p.width) {
            load8(static_cast<const X*>(p.x) + row * p.x_stride + e, h[v]);
            if constexpr (MODE == 1) {
                float f[8];
                load8(static_cast<const T*>(p.residual) + row * p.width + e, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[v][j] += f[j];
                store8(static_cast<T*>(p.residual_out) + row * p.width + e, h[v]);
            }
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s = fmaf(h[v][j], h[v][j], s);
            if constexpr (GROUPS) part[threadIdx.y * (p.width / 8) + e / 8] = s;
            sq += s;
        }
    }
    float r = 0.f;
    if constexpr (GROUPS) {
        if (nt > 32) __syncthreads();
        else __syncwarp();
    } else {
        sq = warp_sum(sq);
        if (nt > 32) {                                  // one row per CTA then
            if ((tx & 31) == 0) sums[tx >> 5] = sq;
            __syncthreads();
            sq = 0.f;
            for (int i = 0; i < nt / 32; ++i) sq += sums[i];
        }
        r = rsqrtf(sq / (float)p.width + p.eps);
    }
    float top = 0.f, odd = 0.f;                         // odd: not a number if a value is not finite
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int e = (v * nt + tx) * 8;
        if (live && e < p.width) {
            int w0 = e;
            if constexpr (GROUPS) {
                const int per = p.group / 8, g = e / p.group;
                const float* s = part + threadIdx.y * (p.width / 8) + g * per;
                float t = 0.f;
                for (int i = 0; i < per; ++i) t += s[i];
                r = rsqrtf(t / (float)p.group + p.eps);
                w0 = e - g * p.group;
            }
            const float4 wa = *reinterpret_cast<const float4*>(p.weight + w0), wb = *reinterpret_cast<const float4*>(p.weight + w0 + 4);
            const float w[8] = {wa.x, wa.y, wa.z, wa.w, wb.x, wb.y, wb.z, wb.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) h[v][j] = h[v][j] * r * w[j];
            if constexpr (MODE == 2) {
                float f[8];
                load8(static_cast<const T*>(p.gate) + row * p.gate_stride + e, f);
                if (p.sigmoid) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) h[v][j] *= 1.f / (1.f + expf(-f[j]));
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) h[v][j] *= f[j] / (1.f + expf(-f[j]));
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                top = fmaxf(top, fabsf(h[v][j]));
                odd = fmaf(h[v][j], 0.f, odd);
            }
            if (p.out != nullptr) store8(static_cast<T*>(p.out) + row * p.width + e, h[v]);
        }
    }
    // (a value that is not finite leaves a largest value that is not a number, which outlives the maxima below)
    top = odd == 0.f ? top : __int_as_float(0x7fffffff);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(__shfl_xor_sync(0xffffffffu, top, o)));
    if (nt > 32) {
        if ((tx & 31) == 0) tops[tx >> 5] = top;
        __syncthreads();
        for (int i = 0; i < nt / 32; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(tops[i]));
    }
    const float inv = top > 1e-30f ? 127.f / top : 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int e = (v * nt + tx) * 8;
        if (live && e < p.width) {
            uint32_t w[2];
#pragma unroll
            for (int q = 0; q < 2; ++q)
                w[q] = byte_of(h[v][4 * q] * inv) | byte_of(h[v][4 * q + 1] * inv) << 8 | byte_of(h[v][4 * q + 2] * inv) << 16 | byte_of(h[v][4 * q + 3] * inv) << 24;
            *reinterpret_cast<uint2*>(p.out8 + row * p.width + e) = make_uint2(w[0], w[1]);
        }
    }
    if (live && tx == 0) p.scale[row] = top * (1.f / 127.f);
}

template <typename T, typename X, int NV, int MODE>
int norm_groups(Ctx* ctx, const Norm8Params& p, dim3 grid, dim3 block, cudaStream_t stream) {
    if (p.group == p.width) return launch_layer(ctx, integer_norm_kernel<T, X, NV, MODE, false>, grid, block, 0, stream, p);
    return launch_layer(ctx, integer_norm_kernel<T, X, NV, MODE, true>, grid, block, (size_t)block.y * (p.width / 8) * 4, stream, p);
}
template <typename T, typename X, int NV>
int norm_mode(Ctx* ctx, const Norm8Params& p, dim3 grid, dim3 block, cudaStream_t stream) {
    if (p.gate != nullptr) return norm_groups<T, X, NV, 2>(ctx, p, grid, block, stream);
    if (p.residual != nullptr) return norm_groups<T, X, NV, 1>(ctx, p, grid, block, stream);
    return norm_groups<T, X, NV, 0>(ctx, p, grid, block, stream);
}
template <typename T, typename X>
int norm_types(Ctx* ctx, const Norm8Params& p, cudaStream_t stream) {
    const int vecs = p.width / 8;
    int nv = (long long)p.rows * vecs >= (long long)sm_count(ctx) * 1024 ? 2 : 1;
    while (nv < 4 && (vecs + nv - 1) / nv > 512) nv *= 2;
    const int tx = ((vecs + nv - 1) / nv + 31) / 32 * 32;
    const int rows_per_cta = tx == 32 ? 4 : 1;
    const dim3 block((unsigned)tx, (unsigned)rows_per_cta), grid((unsigned)((p.rows + rows_per_cta - 1) / rows_per_cta));
    if (nv == 4) return norm_mode<T, X, 4>(ctx, p, grid, block, stream);
    if (nv == 2) return norm_mode<T, X, 2>(ctx, p, grid, block, stream);
    return norm_mode<T, X, 1>(ctx, p, grid, block, stream);
}

}  // namespace

int launch_integer_norm(Ctx* ctx, const Norm8Params& p, bool bf16, bool x_bf16, cudaStream_t stream) {
    if (bf16) return x_bf16 ? norm_types<__nv_bfloat16, __nv_bfloat16>(ctx, p, stream) : norm_types<__nv_bfloat16, float>(ctx, p, stream);
    return x_bf16 ? norm_types<float, __nv_bfloat16>(ctx, p, stream) : norm_types<float, float>(ctx, p, stream);
}

}  // namespace sketchssm
