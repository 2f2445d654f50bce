// Selective scan of packed prompts on CUDA cores: every type, shape and precision that the library has.
//
//     S <- exp(a beta) S + beta k v^T,   out = S^T q + skip v,   token by token, S in fp32 registers.
//
// A CTA takes `cols` value columns of one head of one sequence.  A thread holds eight rows (two runs of four) of four columns, K / 8
// neighbouring lanes share the columns: a token is 48 two-element operations a thread, five loads of 16 bytes from shared memory
// and a sum over the lanes in which every step halves what a lane still has to add.  Tokens come in blocks of 32 through shared memory
// as fp32.  Bound by fp32 issue (three multiply-adds for an element of the state and a token), and with few heads by the chain of
// a token, about 250 cycles.
#include "pairs.cuh"

namespace sketchssm {

namespace {

constexpr int kTok = 32;

template <typename T, int K>
__global__ void __launch_bounds__(512) prompt_scan_kernel(const ScanParams p) {
    constexpr int LK = K / 8;                          // lanes that share four columns
    extern __shared__ __align__(16) float sm[];
    const int cols = p.cols, nt = (int)blockDim.x, tid = (int)threadIdx.x;
    float* sk = sm;                                     // [kTok][K]
    float* sq = sk + kTok * K;
    float* sv = sq + kTok * K;                          // [kTok][cols]
    float* sy = sv + kTok * cols;                       // [kTok][cols]
    float2* sb = reinterpret_cast<float2*>(sy + kTok * cols);      // beta, decay [kTok]
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int blocks = p.V / cols;
    const int unit = (int)blockIdx.x;
    const int seq = unit / (p.H * blocks), h = unit / blocks % p.H, c0 = unit % blocks * cols;
    const int g = h / (p.H / p.G);
    const int2 rows = seq_rows(p.pr, seq);
    const int src = seq_resume(p.pr, seq), dst = seq_slot(p.pr, seq);
    const int r = tid % LK, cg = tid / LK * 4;          // this thread's rows 4 r .. and K / 2 + 4 r .., columns cg ..
    const size_t entry = (size_t)p.H * K * p.V, at = (size_t)h * K * p.V + (size_t)(4 * r) * p.V + c0 + cg;
    uint64_t S[4][4];                                   // [pair of rows][column]
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const size_t o = src * entry + at + (size_t)(i / 2 * (K / 2) + i % 2 * 2) * p.V;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
        if (src >= 0) {
            a = *reinterpret_cast<const float4*>(p.state + o);
            b = *reinterpret_cast<const float4*>(p.state + o + p.V);
        }
        S[i][0] = pack2(a.x, b.x); S[i][1] = pack2(a.y, b.y); S[i][2] = pack2(a.z, b.z); S[i][3] = pack2(a.w, b.w);
    }
    const float a = p.a[h], bias = p.dt_bias != nullptr ? p.dt_bias[h] : 0.f, skip = p.skip != nullptr ? p.skip[h] : 0.f;
    const bool upper = (r & (LK / 2)) != 0, odd = (r & (LK / 4)) != 0;
    const int mine = (upper ? 2 : 0) + (odd ? 1 : 0);   // the column whose sum ends in this lane
    for (int t0 = rows.x; t0 < rows.y; t0 += kTok) {
        const int n = min(kTok, rows.y - t0);
        __syncthreads();
        for (int i = tid; i < n * (K / 4); i += nt) {
            const int t = i / (K / 4), e = i % (K / 4) * 4;
            float f[4], u[4];
            load_io<4>(static_cast<const T*>(p.k) + (long long)(t0 + t) * p.k_stride + (size_t)g * K, e, f);
            load_io<4>(static_cast<const T*>(p.q) + (long long)(t0 + t) * p.q_stride + (size_t)g * K, e, u);
            *reinterpret_cast<float4*>(sk + t * K + e) = make_float4(f[0], f[1], f[2], f[3]);
            *reinterpret_cast<float4*>(sq + t * K + e) = make_float4(u[0], u[1], u[2], u[3]);
        }
        for (int i = tid; i < n * (cols / 4); i += nt) {
            const int t = i / (cols / 4), e = i % (cols / 4) * 4;
            float f[4];
            load_io<4>(static_cast<const T*>(p.v) + (long long)(t0 + t) * p.v_stride + (size_t)h * p.V + c0, e, f);
            *reinterpret_cast<float4*>(sv + t * cols + e) = make_float4(f[0], f[1], f[2], f[3]);
        }
        for (int t = tid; t < n; t += nt) {
            const float beta = softplus((float)static_cast<const T*>(p.dt)[(long long)(t0 + t) * p.dt_stride + h] + bias);
            sb[t] = make_float2(beta, expf(a * beta));
        }
        __syncthreads();
#pragma unroll 2
        for (int t = 0; t < n; ++t) {
            const float2 bd = sb[t];
            const float4 v = *reinterpret_cast<const float4*>(sv + t * cols + cg);
            const ulonglong2 k0 = *reinterpret_cast<const ulonglong2*>(sk + t * K + 4 * r), k1 = *reinterpret_cast<const ulonglong2*>(sk + t * K + K / 2 + 4 * r);
            const ulonglong2 q0 = *reinterpret_cast<const ulonglong2*>(sq + t * K + 4 * r), q1 = *reinterpret_cast<const ulonglong2*>(sq + t * K + K / 2 + 4 * r);
            const uint64_t k[4] = {k0.x, k0.y, k1.x, k1.y}, q[4] = {q0.x, q0.y, q1.x, q1.y}, d = pack2(bd.y, bd.y);
            const float bv[4] = {bd.x * v.x, bd.x * v.y, bd.x * v.z, bd.x * v.w};
            float y[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint64_t b2 = pack2(bv[c], bv[c]);
                uint64_t y2 = 0ull;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    S[i][c] = fma2(d, S[i][c], mul2(k[i], b2));
                    y2 = fma2(S[i][c], q[i], y2);
                }
                float lo, hi;
                unpack2(y2, lo, hi);
                y[c] = lo + hi;
            }
            // the halves of the lanes add two columns each, their halves one, the rest of the way as usual
            const float s0 = upper ? y[0] : y[2], s1 = upper ? y[1] : y[3];
            float z0 = (upper ? y[2] : y[0]) + __shfl_xor_sync(0xffffffffu, s0, LK / 2);
            float z1 = (upper ? y[3] : y[1]) + __shfl_xor_sync(0xffffffffu, s1, LK / 2);
            float z = (odd ? z1 : z0) + __shfl_xor_sync(0xffffffffu, odd ? z0 : z1, LK / 4);
#pragma unroll
            for (int o = LK / 8; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
            if ((r & (LK / 4 - 1)) == 0) sy[t * cols + cg + mine] = z;
        }
        __syncthreads();
        for (int i = tid; i < n * (cols / 4); i += nt) {
            const int t = i / (cols / 4), e = i % (cols / 4) * 4;
            const float4 y = *reinterpret_cast<const float4*>(sy + t * cols + e), v = *reinterpret_cast<const float4*>(sv + t * cols + e);
            const float f[4] = {fmaf(skip, v.x, y.x), fmaf(skip, v.y, y.y), fmaf(skip, v.z, y.z), fmaf(skip, v.w, y.w)};
            const long long o = (long long)(t0 + t) * p.out_stride + (long long)h * p.V + c0;
            if (p.out_bf16) store_io<4>(static_cast<__nv_bfloat16*>(p.out) + o, e, f);
            else store_io<4>(static_cast<float*>(p.out) + o, e, f);
        }
    }
    if (dst >= 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const size_t o = dst * entry + at + (size_t)(i / 2 * (K / 2) + i % 2 * 2) * p.V;
            float4 a4, b4;
            unpack2(S[i][0], a4.x, b4.x); unpack2(S[i][1], a4.y, b4.y); unpack2(S[i][2], a4.z, b4.z); unpack2(S[i][3], a4.w, b4.w);
            *reinterpret_cast<float4*>(p.state + o) = a4;
            *reinterpret_cast<float4*>(p.state + o + p.V) = b4;
        }
    }
}

}  // namespace

int launch_prompt_scan(Ctx* ctx, const ScanParams& p0, bool bf16, cudaStream_t stream) {
    const int rc = launch_prompt_scan_tc(ctx, p0, bf16, stream);
    if (rc != SKETCHSSM_UNSUPPORTED_SHAPE) return rc;
    ScanParams p = p0;
    // All columns of a head in a CTA (keys and queries are then fetched once) where that gives the SMs four of them, else 16 or 32.
    const long long heads = (long long)p.pr.N * p.H;
    p.cols = heads >= 4ll * sm_count(ctx) ? p.V : p.V % 32 == 0 && heads * (p.V / 32) >= 4ll * sm_count(ctx) ? 32 : 16;
    const long long units = heads * (p.V / p.cols);
    if (units > 0x7fffffffll) return SKETCHSSM_UNSUPPORTED_SHAPE;
    const size_t smem = (size_t)(2 * kTok * p.K + 2 * kTok * p.cols + 2 * kTok) * 4;
    auto kern = p.K == 128 ? (bf16 ? prompt_scan_kernel<__nv_bfloat16, 128> : prompt_scan_kernel<float, 128>)
                           : (bf16 ? prompt_scan_kernel<__nv_bfloat16, 64> : prompt_scan_kernel<float, 64>);
    const cudaError_t e = unlock_smem(ctx, kern);
    if (e != cudaSuccess) { ctx->last_cuda_error = e; return SKETCHSSM_CUDA_ERROR; }
    return launch_layer(ctx, kern, dim3((unsigned)units), dim3((unsigned)(p.cols / 4 * (p.K / 8))), smem, stream, p);
}

}  // namespace sketchssm
