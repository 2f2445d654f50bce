// The operators around the recurrence (convolution, prompt scan, norm, 8-bit product): parameters and shared helpers.
#pragma once

#include "internal.cuh"

namespace sketchssm {

constexpr int kFaultScanWait = 5;      // prompt scan, tensor cores
constexpr int kFaultMatmulWait = 6;    // 8-bit product

// A batch of packed prompts as the kernels see it.
struct PromptsDev {
    const int* starts;
    const int* slots;
    const int* resume;
    int N, T, B;
};

struct ConvParams {
    PromptsDev pr;
    const float* weight;
    const float* bias;
    void* state;
    const void* x;
    void* out;
    long long x_stride, out_stride;
    int C, W, silu;
};

struct ConvStepParams {
    const float* weight;
    const float* bias;
    void* state;
    const void* x;
    const void* dt;
    const float* a;
    const float* dt_bias;
    void *q, *k, *v;
    float *beta, *decay;
    long long x_stride, dt_stride;
    int B, H, G, K, V, W;
};

struct ScanParams {
    PromptsDev pr;
    const void *q, *k, *v, *dt;
    const float *a, *dt_bias, *skip;
    void* out;
    float* state;
    float* work;
    int* status;
    long long q_stride, k_stride, v_stride, dt_stride, out_stride;
    int H, G, K, V, out_bf16;
    int cols;              // CUDA cores: value columns per CTA
    int segments;          // tensor cores: parts that a sequence's tokens are split into
};

struct NormParams {
    const void* x;
    const float* weight;
    const void* residual;
    void* residual_out;
    const void* gate;
    const void* skip;
    const float* skip_weight;
    void* out;
    void* out8;
    float* scale;
    long long x_stride, gate_stride, skip_stride;
    int rows, width, group, groups, skip_heads, x_bf16;
    float eps;
};

struct MatmulParams {
    const unsigned char *a, *w;
    const float *a_scale, *w_scale;
    void* out;
    int* status;
    long long out_stride;
    int M, N, K, KB, out_bf16;
};

int launch_causal_conv(Ctx* ctx, const ConvParams& p, bool bf16, cudaStream_t stream);
int launch_conv_step(Ctx* ctx, const ConvStepParams& p, bool bf16, cudaStream_t stream);
int launch_prompt_scan(Ctx* ctx, const ScanParams& p, bool bf16, cudaStream_t stream);       // CUDA cores, every configuration
int launch_prompt_scan_tc(Ctx* ctx, const ScanParams& p, bool bf16, cudaStream_t stream);    // tcgen05; UNSUPPORTED_SHAPE outside its domain
int prompt_scan_tc_segments(Ctx* ctx, int groups, int sequences, int tokens);     // parts that a sequence is split into
int launch_rms_norm(Ctx* ctx, const NormParams& p, bool bf16, cudaStream_t stream);
int launch_scaled_matmul(Ctx* ctx, const MatmulParams& p, cudaStream_t stream);
int launch_scaled_matmul_pair(Ctx* ctx, const MatmulParams& p, cudaStream_t stream);         // many rows; UNSUPPORTED_SHAPE where a 128 x 128 tile an SM is enough

// Prompt scan on tensor cores: at most this many segments (of all sequences of a batch together) keep a state in the scratch.  A unit
// of work is a segment for two blocks of 64 value columns; segments are made until 148 SMs have one, of at least four chunks of
// 128 tokens on the average.  (One prompt, 8 heads of 64 columns: 2048 tokens in segments of at least four chunks 59 us, of two 52, of
// eight 88; 512 tokens whole 31, in segments of two 39; 4096 tokens 68, 71 and 92.)
inline long long scan_segment_states(const sketchssm_config& c, long long tokens) {
    if (c.kind != SKETCHSSM_MAMBA2 || c.io_dtype != SKETCHSSM_BF16 || c.dk != 128 || c.dv % 64 != 0) return 0;
    const long long slabs = ((long long)c.heads * (c.dv / 64) + 1) / 2, n = 148 / slabs, most = tokens / 512;
    return (n < most ? n : most) < 2 ? 0 : n < most ? n : most;
}

inline int sm_count(Ctx* ctx) {
    if (ctx->sm_count == 0 && cudaDeviceGetAttribute(&ctx->sm_count, cudaDevAttrMultiProcessorCount, ctx->cfg.device) != cudaSuccess)
        ctx->sm_count = 148;
    return ctx->sm_count;
}

#ifdef __CUDACC__

// Launch with the programmatic-stream-serialization attribute.  The kernels wait for their predecessor before anything else and
// only then let their successor start: a successor that reads ahead of its own wait never overtakes what came before them.
template <typename P>
inline int launch_layer(Ctx* ctx, void (*kern)(const P), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, const P& p,
                        int cluster = 1) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = static_cast<sketchssm_ctx*>(ctx)->tune_pdl ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, p);
    if (e != cudaSuccess) {
        ctx->last_cuda_error = e;
        (void)cudaGetLastError();
        return SKETCHSSM_CUDA_ERROR;
    }
    ctx->last_launches += 1;
    return SKETCHSSM_OK;
}

// First row of sequence i, and the end of its rows; always inside [0, T] and begin <= end, whatever the array holds.
__device__ __forceinline__ int seq_start(const PromptsDev& pr, int i) {
    return min(max(pr.starts[i], 0), pr.T);
}
__device__ __forceinline__ int2 seq_rows(const PromptsDev& pr, int i) {
    const int b = seq_start(pr, i);
    return make_int2(b, max(b, seq_start(pr, i + 1)));
}
// The batch entry that a sequence's state goes to / comes from; -1: none.
__device__ __forceinline__ int seq_slot(const PromptsDev& pr, int i) {
    const int s = pr.slots != nullptr ? pr.slots[i] : i;
    return s >= 0 && s < pr.B ? s : -1;
}
__device__ __forceinline__ int seq_resume(const PromptsDev& pr, int i) {
    const int s = pr.resume != nullptr ? pr.resume[i] : -1;
    return s >= 0 && s < pr.B ? s : -1;
}

// Number of the N sequences that start before row t (starts ascend).  A whole warp calls it.
__device__ __forceinline__ int starts_before(const PromptsDev& pr, int t) {
    int n = 0;
    for (int j = threadIdx.x & 31; j - (int)(threadIdx.x & 31) < pr.N; j += 32)
        n += __popc(__ballot_sync(0xffffffffu, j < pr.N && pr.starts[j] < t));
    return n;
}

__device__ __forceinline__ float softplus(float x) { return fmaxf(x, 0.f) + log1pf(expf(-fabsf(x))); }

// 16 bytes of io elements as floats and back.
template <typename T>
struct Vec16;
template <>
struct Vec16<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void unpack(const uint4& u, float (&f)[4]) {
        f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};
template <>
struct Vec16<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void unpack(const uint4& u, float (&f)[8]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// y / (1 + exp(-y)); where the result is rounded to bfloat16 the exponential and the reciprocal are the fast ones (a few parts
// in 10^7, the rounding is 2^-9; with denormals flushed, which costs nothing here and saves half of their instructions).
template <typename T>
__device__ __forceinline__ float silu(float y) {
    if constexpr (sizeof(T) == 2) {
        float r;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + ex2(-1.4426950408889634f * y)));
        return y * r;
    } else {
        return y / (1.f + expf(-y));
    }
}

#endif  // __CUDACC__

}  // namespace sketchssm
