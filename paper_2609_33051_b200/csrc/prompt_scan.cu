// Selective scan of packed prompts on CUDA cores: every type, shape and precision that the library has.
//
//     S <- exp(a beta) S + beta k v^T,   out = S^T q + skip v,   token by token, S in fp32 registers.
//
// A CTA takes `cols` value columns of one head of one sequence; four neighbouring lanes share a column, a quarter of its K rows
// each, so the output of a token takes two shuffles.  Tokens come in blocks of 32 through shared memory as fp32.
// Bound by fp32 issue: K V multiply-adds for the state, as many for the output and K V multiplications for the decay, a token.
#include "layer.cuh"

namespace sketchssm {

namespace {

constexpr int kTok = 32;

template <typename T, int K>
__global__ void __launch_bounds__(256) prompt_scan_kernel(const ScanParams p) {
    constexpr int KQ = K / 4, KP = KQ + 4;             // rows per lane; quarters 4 floats apart from bank to bank
    extern __shared__ __align__(16) float sm[];
    const int cols = p.cols, nt = cols * 4, tid = (int)threadIdx.x;
    float* sk = sm;                                     // [kTok][4][KP]
    float* sq = sk + kTok * 4 * KP;
    float* sv = sq + kTok * 4 * KP;                     // [kTok][cols]
    float* sy = sv + kTok * cols;                       // [kTok][cols]
    float* sb = sy + kTok * cols;                       // beta, decay [kTok]
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int blocks = p.V / cols;
    const int unit = (int)blockIdx.x;
    const int seq = unit / (p.H * blocks), h = unit / blocks % p.H, c0 = unit % blocks * cols;
    const int g = h / (p.H / p.G);
    const int2 rows = seq_rows(p.pr, seq);
    const int src = seq_resume(p.pr, seq), dst = seq_slot(p.pr, seq);
    const int kq = tid & 3, col = tid >> 2;
    const size_t at = (size_t)h * K * p.V + (size_t)(kq * KQ) * p.V + c0 + col;
    const size_t entry = (size_t)p.H * K * p.V;
    float S[KQ];
#pragma unroll
    for (int i = 0; i < KQ; ++i) S[i] = src >= 0 ? p.state[src * entry + at + (size_t)i * p.V] : 0.f;
    const float a = p.a[h], bias = p.dt_bias != nullptr ? p.dt_bias[h] : 0.f, skip = p.skip != nullptr ? p.skip[h] : 0.f;
    for (int t0 = rows.x; t0 < rows.y; t0 += kTok) {
        const int n = min(kTok, rows.y - t0);
        __syncthreads();
        for (int i = tid; i < n * (K / 4); i += nt) {
            const int t = i / (K / 4), e = i % (K / 4) * 4;
            float f[4];
            load_io<4>(static_cast<const T*>(p.k) + (long long)(t0 + t) * p.k_stride + (size_t)g * K, e, f);
            *reinterpret_cast<float4*>(sk + (t * 4 + e / KQ) * KP + e % KQ) = make_float4(f[0], f[1], f[2], f[3]);
            load_io<4>(static_cast<const T*>(p.q) + (long long)(t0 + t) * p.q_stride + (size_t)g * K, e, f);
            *reinterpret_cast<float4*>(sq + (t * 4 + e / KQ) * KP + e % KQ) = make_float4(f[0], f[1], f[2], f[3]);
        }
        for (int i = tid; i < n * cols; i += nt) {
            const int t = i / cols, e = i % cols;
            sv[i] = (float)static_cast<const T*>(p.v)[(long long)(t0 + t) * p.v_stride + (size_t)h * p.V + c0 + e];
        }
        for (int t = tid; t < n; t += nt) {
            const float beta = softplus((float)static_cast<const T*>(p.dt)[(long long)(t0 + t) * p.dt_stride + h] + bias);
            sb[t] = beta;
            sb[kTok + t] = expf(a * beta);
        }
        __syncthreads();
        for (int t = 0; t < n; ++t) {
            const float v = sv[t * cols + col], bv = sb[t] * v, d = sb[kTok + t];
            const float4* k4 = reinterpret_cast<const float4*>(sk + (t * 4 + kq) * KP);
            const float4* q4 = reinterpret_cast<const float4*>(sq + (t * 4 + kq) * KP);
            float y0 = 0.f, y1 = 0.f;
#pragma unroll
            for (int i = 0; i < KQ / 4; ++i) {
                const float4 k = k4[i], q = q4[i];
                S[4 * i] = fmaf(d, S[4 * i], k.x * bv);
                S[4 * i + 1] = fmaf(d, S[4 * i + 1], k.y * bv);
                S[4 * i + 2] = fmaf(d, S[4 * i + 2], k.z * bv);
                S[4 * i + 3] = fmaf(d, S[4 * i + 3], k.w * bv);
                y0 = fmaf(S[4 * i], q.x, y0);
                y1 = fmaf(S[4 * i + 1], q.y, y1);
                y0 = fmaf(S[4 * i + 2], q.z, y0);
                y1 = fmaf(S[4 * i + 3], q.w, y1);
            }
            float y = y0 + y1;
            y += __shfl_xor_sync(0xffffffffu, y, 1);
            y += __shfl_xor_sync(0xffffffffu, y, 2);
            if (kq == 0) sy[t * cols + col] = fmaf(skip, v, y);
        }
        __syncthreads();
        for (int i = tid; i < n * cols; i += nt) {
            const int t = i / cols, e = i % cols;
            const long long o = (long long)(t0 + t) * p.out_stride + (long long)h * p.V + c0 + e;
            if (p.out_bf16) static_cast<__nv_bfloat16*>(p.out)[o] = __float2bfloat16_rn(sy[i]);
            else static_cast<float*>(p.out)[o] = sy[i];
        }
    }
    if (dst >= 0) {
#pragma unroll
        for (int i = 0; i < KQ; ++i) p.state[dst * entry + at + (size_t)i * p.V] = S[i];
    }
}

}  // namespace

int launch_prompt_scan(Ctx* ctx, const ScanParams& p0, bool bf16, cudaStream_t stream) {
    const int rc = launch_prompt_scan_tc(ctx, p0, bf16, stream);
    if (rc != SKETCHSSM_UNSUPPORTED_SHAPE) return rc;
    ScanParams p = p0;
    // 16 columns a CTA where 32 would leave SMs with less than two CTAs (V = 80 is five times 16)
    p.cols = p.V % 32 == 0 && (long long)p.pr.N * p.H * (p.V / 32) >= 2ll * sm_count(ctx) ? 32 : 16;
    const long long units = (long long)p.pr.N * p.H * (p.V / p.cols);
    if (units > 0x7fffffffll) return SKETCHSSM_UNSUPPORTED_SHAPE;
    const int kp = p.K / 4 + 4;
    const size_t smem = (size_t)(2 * kTok * 4 * kp + 2 * kTok * p.cols + 2 * kTok) * 4;
    auto kern = p.K == 128 ? (bf16 ? prompt_scan_kernel<__nv_bfloat16, 128> : prompt_scan_kernel<float, 128>)
                           : (bf16 ? prompt_scan_kernel<__nv_bfloat16, 64> : prompt_scan_kernel<float, 64>);
    const cudaError_t e = unlock_smem(ctx, kern);
    if (e != cudaSuccess) { ctx->last_cuda_error = e; return SKETCHSSM_CUDA_ERROR; }
    return launch_layer(ctx, kern, dim3((unsigned)units), dim3((unsigned)(p.cols * 4)), smem, stream, p);
}

}  // namespace sketchssm
