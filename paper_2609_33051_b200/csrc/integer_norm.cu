// Root-mean-square norm with the residual's addition before it, or of every head's output with the gate behind it, and the rows in 8-bit
// integers with a scale for each of them that the next projection takes.
//
//     h = x  or  x + residual;   y = h / sqrt(mean(h^2) + eps) weight   in groups of `group` elements;   with gate: y act(gate)
//     scale = max|y| / 127 over the row,  out8 = round(y 127 / max|y|)
//
// Every input is read once and every output written once, so HBM bounds it where instructions do not: 16384 rows of 2048 with the residual take 43 us,
// of which the bytes are 36 at 6.46 TB/s; 16384 rows of 4096 in groups of 128 with the gate 96 us (bytes: 52), with 33 instructions an
// element.  512 such rows take 5.3 us, 64 rows of 2048 with the residual 1.8 (from a graph, data larger than L2).  A row belongs to one CTA (four short rows to four warps of one)
// and stays in its threads' registers, NV vectors of eight elements each: a group's sum of squares and the row's largest value are both
// needed before an element of it can be written.  A group is whole vectors of neighbouring threads, any number of them: where it is
// not the row, and neighbouring lanes of a warp do not hold it, every vector's own sum goes through shared memory and each thread adds up those
// of its group.
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

// Eight elements as they were read.
template <typename T>
struct Row8 {
    uint4 a[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) a[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ void unpack(float (&f)[8]) const {
        constexpr int N = Vec16<T>::N;
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            float g[N];
            Vec16<T>::unpack(a[i], g);
#pragma unroll
            for (int j = 0; j < N; ++j) f[i * N + j] = g[j];
        }
    }
};

// The larger one; not a number if either is.
__device__ __forceinline__ float max_nan(float a, float b) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(b));
    return a;
}
// The largest of a warp's values, none of them negative: their bits are in the values' order, with what is not a number above all.
__device__ __forceinline__ float warp_top(float a) { return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(a))); }
// 1 / (1 + e^-x) by the quick instructions.
__device__ __forceinline__ float quick_sigmoid(float x) {
    float e, y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * -1.44269504f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(1.f + e));
    return y;
}
// Four values of at most 127 times 1 / inv to the nearest integers, ties to even, as bytes: the low ones of numbers that start at 1.5 * 2^23, where a
// step is one (the conversion instruction, a sixteenth as fast as this sum, bounded rows with a gate).
__device__ __forceinline__ uint32_t bytes_of(const float* h, float inv) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(fmaf(h[i], inv, 12582912.f));
    return __byte_perm(__byte_perm(u[0], u[1], 0x0040), __byte_perm(u[2], u[3], 0x0040), 0x5410);
}

// blockDim.x threads (a multiple of 32) share a row; blockDim.y rows per CTA, more than one only with 32 threads each.
// MODE 0: plain, 1: residual, 2: gate.  GROUPS: the row is more than one group.
template <typename T, typename X, int NV, int MODE, bool GROUPS>
__global__ void __launch_bounds__(512) integer_norm_kernel(const Norm8Params p) {
    extern __shared__ float part[];                     // GROUPS, not within warps: [rows][width / 8] sums of squares
    __shared__ float sums[32], tops[32];
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int tx = (int)threadIdx.x, nt = (int)blockDim.x;
    const long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const bool live = row < p.rows;
    // A group of up to 256 elements that is a power of two lies with neighbouring lanes of one warp.
    const int per = p.group / 8;
    const bool lanes = GROUPS && 32 % per == 0;
    // One vector a thread (few rows): all that it reads is under way before the first sum is waited for.  Two or more: the weights, which are in
    // the cache by then, are left for later, as their registers would cost resident rows.
    constexpr bool kAhead = NV == 1;
    float h[NV][8];
    Row8<T> side[NV];                                   // the residual's or the gate's elements
    float4 w[2];
    auto load_weight = [&](int e) {
        const float4* weight = reinterpret_cast<const float4*>(p.weight + (!GROUPS ? e : lanes ? e & (p.group - 1) : e % p.group));
        w[0] = weight[0];
        w[1] = weight[1];
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int e = (v * nt + tx) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) h[v][j] = 0.f;
        if (live && e < p.width) {
            load8(static_cast<const X*>(p.x) + row * p.x_stride + e, h[v]);
            if constexpr (MODE == 1) side[v].load(static_cast<const T*>(p.residual) + row * p.width + e);
            if constexpr (MODE == 2) side[v].load(static_cast<const T*>(p.gate) + row * p.gate_stride + e);
            if (kAhead) load_weight(e);
        }
    }
    float r[NV], sq = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int e = (v * nt + tx) * 8;
        r[v] = 0.f;
        if (live && e < p.width) {
            if constexpr (MODE == 1) {
                float f[8];
                side[v].unpack(f);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[v][j] += f[j];
                store8(static_cast<T*>(p.residual_out) + row * p.width + e, h[v]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) r[v] = fmaf(h[v][j], h[v][j], r[v]);
            if (GROUPS && !lanes) part[threadIdx.y * (p.width / 8) + e / 8] = r[v];
            sq += r[v];
        }
        if (GROUPS && lanes)
            for (int o = per / 2; o > 0; o >>= 1) r[v] += __shfl_xor_sync(0xffffffffu, r[v], o);
    }
    if constexpr (GROUPS) {
        if (!lanes) {
            if (nt > 32) __syncthreads();
            else __syncwarp();
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int e = (v * nt + tx) * 8;
                if (live && e < p.width) {
                    const float* s = part + threadIdx.y * (p.width / 8) + e / p.group * per;
                    r[v] = 0.f;
                    for (int i = 0; i < per; ++i) r[v] += s[i];
                }
            }
        }
    } else {
        sq = warp_sum(sq);
        if (nt > 32) {                                  // one row per CTA then
            if ((tx & 31) == 0) sums[tx >> 5] = sq;
            __syncthreads();
            sq = (tx & 31) < nt / 32 ? sums[tx & 31] : 0.f;
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);       // (of at most 16 warps)
            sq = __shfl_sync(0xffffffffu, sq, 0);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) r[v] = sq;
    }
    float top = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int e = (v * nt + tx) * 8;
        if (live && e < p.width) {
            const float s = rsqrtf(r[v] / (float)p.group + p.eps);
            if (!kAhead) load_weight(e);
            const float f8[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
#pragma unroll
            for (int j = 0; j < 8; ++j) h[v][j] = h[v][j] * s * f8[j];
            if constexpr (MODE == 2) {
                float f[8];
                side[v].unpack(f);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    // (Gates in bf16 are 2^-9 off themselves.  The quick instructions are 2^-22 off each and the rounding of the exponent is 2^-24 of
                    // it: less than 2^-18 for gates down to -32, and 2^-16 beyond, where next to nothing passes.)
                    if constexpr (sizeof(T) == 2) h[v][j] *= (p.sigmoid ? 1.f : f[j]) * quick_sigmoid(f[j]);
                    else h[v][j] *= (p.sigmoid ? 1.f : f[j]) / (1.f + expf(-f[j]));
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) top = max_nan(top, fabsf(h[v][j]));
            if (p.out != nullptr) store8(static_cast<T*>(p.out) + row * p.width + e, h[v]);
        }
    }
    top = warp_top(top);
    if (nt > 32) {
        if ((tx & 31) == 0) tops[tx >> 5] = top;
        __syncthreads();
        top = warp_top((tx & 31) < nt / 32 ? tops[tx & 31] : 0.f);
    }
    if (!(top < __int_as_float(0x7f800000))) top = __int_as_float(0x7fffffff);      // a row with an infinity, too, has no scale
    const float inv = top > 1e-30f ? 127.f / top : 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int e = (v * nt + tx) * 8;
        if (live && e < p.width) {
            const uint2 u = inv > 0.f ? make_uint2(bytes_of(h[v], inv), bytes_of(h[v] + 4, inv)) : make_uint2(0u, 0u);
            *reinterpret_cast<uint2*>(p.out8 + row * p.width + e) = u;
        }
    }
    if (live && tx == 0) p.scale[row] = top * (1.f / 127.f);
}

template <typename T, typename X, int NV, int MODE>
int norm_groups(Ctx* ctx, const Norm8Params& p, dim3 grid, dim3 block, cudaStream_t stream) {
    if (p.group == p.width) return launch_layer(ctx, integer_norm_kernel<T, X, NV, MODE, false>, grid, block, 0, stream, p);
    return launch_layer(ctx, integer_norm_kernel<T, X, NV, MODE, true>, grid, block, 32 % (p.group / 8) == 0 ? 0 : (size_t)block.y * (p.width / 8) * 4, stream, p);
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
    // Two vectors a thread where there are rows enough for all SMs: 16384 rows of 4096 with the gate in 96 us (119 with one, 116 with four), of 2048
    // with the residual in 43 (47, 48).
    int nv = (long long)p.rows * vecs >= (long long)sm_count(ctx) * 1024 ? 2 : 1;
    while (nv < 4 && (vecs + nv - 1) / nv > 512) nv *= 2;
    const int tx = ((vecs + nv - 1) / nv + 31) / 32 * 32;
    const int rows_per_cta = tx == 32 ? 4 : 1;
    const dim3 block((unsigned)tx, (unsigned)rows_per_cta), grid((unsigned)(((long long)p.rows + rows_per_cta - 1) / rows_per_cta));
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
