// Gated delta rule over packed prompts on CUDA cores: every type, shape and both kinds of decay that the library has.
//
//     S <- D S,   S <- S + beta k (v - S^T k)^T,   out = S^T q,   token by token, S in fp32 registers,
//
// k and q unit vectors (q times q_scale), beta = 1 / (1 + exp(-b)), D = exp(a softplus(dt + dt_bias)): a number a head (GDN) or a
// diagonal (KDA).  Keys and queries stay as they are: their norms are numbers of the token, which multiply S^T k, the new
// values and S^T q.
//
// A CTA takes `cols` value columns of one head of one sequence.  Eight neighbouring lanes share four columns, a thread holds sixteen
// rows (K = 128: four runs of four; eight with K = 64) of them: a token is four two-element operations for a pair of elements of
// the state.  S^T k is needed by all lanes before the state goes on (three shuffles a column); the sums for out are
// made for four tokens together, every step halving what a lane still has to add.  Tokens come through shared memory, 32 of them while the
// 32 before are worked on.  Bound by fp32 issue where there are many heads, and by the chain of a token, some 300 cycles, where there are few.
#include "pairs.cuh"

namespace sketchssm {

namespace {

constexpr int kTok = 32;

// 16 bytes from global to shared memory, not waited for.
__device__ __forceinline__ void copy16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Four consecutive elements as two pairs of floats.
__device__ __forceinline__ void four(const float* p, uint64_t& a, uint64_t& b) {
    const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(p);
    a = v.x;
    b = v.y;
}
__device__ __forceinline__ void four(const __nv_bfloat16* p, uint64_t& a, uint64_t& b) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    a = pack2(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u));
    b = pack2(__uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
}

// Elements of a stage of kTok tokens: keys, queries, values, and KDA's arguments of the decays.
template <bool KDA>
__host__ __device__ constexpr int stage_elements(int K, int cols) { return kTok * ((KDA ? 3 : 2) * K + cols); }

template <typename T, int K, bool KDA>
__global__ void __launch_bounds__(256) delta_scan_kernel(const DeltaParams p) {
    constexpr int LK = 8, RUNS = K / 32, RP = 2 * RUNS;        // lanes that share four columns; runs of four rows, pairs of rows of a thread
    extern __shared__ __align__(16) unsigned char sm[];
    const int cols = p.cols, nt = (int)blockDim.x, tid = (int)threadIdx.x, lane = tid & 31;
    const int stage = stage_elements<KDA>(K, cols);
    T* const raw = reinterpret_cast<T*>(sm);
    float* sy = reinterpret_cast<float*>(raw + 2 * stage);         // [kTok][cols]
    float4* sg = reinterpret_cast<float4*>(sy + kTok * cols);      // decay (GDN), 1 / |k|, beta, q_scale / |q|  [kTok]
    float* sd = reinterpret_cast<float*>(sg + kTok);               // KDA: decays [kTok][K]
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int blocks = p.V / cols;
    const int unit = (int)blockIdx.x;
    const int seq = unit / (p.H * blocks), h = unit / blocks % p.H, c0 = unit % blocks * cols;
    const int g = h / (p.H / p.G);
    const int2 rows = seq_rows(p.pr, seq);
    const int src = seq_resume(p.pr, seq), dst = seq_slot(p.pr, seq);
    const int r = tid % LK, cg = tid / LK * 4;          // this thread's rows 4 r + 32 j .., columns cg ..
    const size_t entry = (size_t)p.H * K * p.V, at = (size_t)h * K * p.V + (size_t)(4 * r) * p.V + c0 + cg;
    uint64_t S[RP][4];                                  // [pair of rows][column]
#pragma unroll
    for (int i = 0; i < RP; ++i) {
        const size_t o = src * entry + at + (size_t)(i / 2 * 32 + i % 2 * 2) * p.V;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
        if (src >= 0) {
            a = *reinterpret_cast<const float4*>(p.state + o);
            b = *reinterpret_cast<const float4*>(p.state + o + p.V);
        }
        S[i][0] = pack2(a.x, b.x); S[i][1] = pack2(a.y, b.y); S[i][2] = pack2(a.z, b.z); S[i][3] = pack2(a.w, b.w);
    }
    const float a = p.a[h];
    constexpr int E = 16 / (int)sizeof(T);
    float dt = 0.f, bl = 0.f;
    auto fetch = [&](int t0, T* to) {
        const int n = min(kTok, rows.y - t0);
        for (int i = tid; i < n * (K / E); i += nt) {
            const int t = i / (K / E), e = i % (K / E) * E;
            copy16(to + t * K + e, static_cast<const T*>(p.k) + (long long)(t0 + t) * p.k_stride + (size_t)g * K + e);
            copy16(to + kTok * K + t * K + e, static_cast<const T*>(p.q) + (long long)(t0 + t) * p.q_stride + (size_t)g * K + e);
            if constexpr (KDA)
                copy16(to + kTok * (2 * K + cols) + t * K + e, static_cast<const T*>(p.dt) + (long long)(t0 + t) * p.dt_stride + (size_t)h * K + e);
        }
        const int per = cols / E;
        for (int i = tid; i < n * per; i += nt) {
            const int t = i / per, e = i % per * E;
            copy16(to + 2 * kTok * K + t * cols + e, static_cast<const T*>(p.v) + (long long)(t0 + t) * p.v_stride + (size_t)h * p.V + c0 + e);
        }
        if (tid < n) {
            bl = (float)static_cast<const T*>(p.b)[(long long)(t0 + tid) * p.b_stride + h];
            if constexpr (!KDA) dt = (float)static_cast<const T*>(p.dt)[(long long)(t0 + tid) * p.dt_stride + h];
        }
    };
    if (rows.x < rows.y) fetch(rows.x, raw);
    int b = 0;
    for (int t0 = rows.x; t0 < rows.y; t0 += kTok, b ^= 1) {
        const int n = min(kTok, rows.y - t0);
        const T *sk = raw + b * stage, *sq = sk + kTok * K, *sv = sq + kTok * K;
        copies_done();
        const int n4 = (n + 3) & ~3;                    // tokens are worked on by four: those behind the last one change nothing
        if (n4 > n) {
            T* to = raw + b * stage;
            const T zero = (T)0.f;
            for (int i = n * K + tid; i < n4 * K; i += nt) {
                to[i] = zero;
                to[kTok * K + i] = zero;
                if constexpr (KDA) sd[i] = 1.f;
            }
            for (int i = n * cols + tid; i < n4 * cols; i += nt) to[2 * kTok * K + i] = zero;
        }
        float4 gate = make_float4(1.f, 0.f, 0.f, 0.f);
        if (tid < n) {
            gate.z = 1.f / (1.f + expf(-bl));
            if constexpr (!KDA) gate.x = expf(a * softplus(dt + (p.dt_bias != nullptr ? p.dt_bias[h] : 0.f)));
        }
        if (tid < kTok) sg[tid] = gate;
        __syncthreads();                                // this stage is there, and nobody reads the other one any more
        if (t0 + kTok < rows.y) fetch(t0 + kTok, raw + (b ^ 1) * stage);
        for (int t = tid >> 5; t < n; t += nt >> 5) {    // norms: a warp a token
            float k2 = 0.f, q2 = 0.f;
#pragma unroll
            for (int i = 0; i < K / 32; ++i) {
                const float kv = (float)sk[t * K + i * 32 + lane], qv = (float)sq[t * K + i * 32 + lane];
                k2 = fmaf(kv, kv, k2);
                q2 = fmaf(qv, qv, q2);
            }
            k2 = warp_sum(k2);
            q2 = warp_sum(q2);
            if (lane == 0) {
                sg[t].y = inv_length(k2, p.eps);
                sg[t].w = p.q_scale * inv_length(q2, p.eps);
            }
        }
        if constexpr (KDA) {
            const T* sx = sv + kTok * cols;
            const float* bias = p.dt_bias != nullptr ? p.dt_bias + (size_t)h * K : nullptr;
            for (int i = tid; i < n * K; i += nt) sd[i] = expf(a * softplus((float)sx[i] + (bias != nullptr ? bias[i % K] : 0.f)));
        }
        __syncthreads();
#pragma unroll 1
        for (int t4 = 0; t4 < n4; t4 += 4) {
            float y[16];                                // of four tokens and four columns
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int t = t4 + u;
                const float4 w = sg[t];
                uint64_t k[RP], q[RP], v01, v23;
                four(sv + t * cols + cg, v01, v23);
#pragma unroll
                for (int j = 0; j < RUNS; ++j) four(sk + t * K + j * 32 + 4 * r, k[2 * j], k[2 * j + 1]);
                if constexpr (KDA) {
#pragma unroll
                    for (int j = 0; j < RUNS; ++j) {
                        uint64_t d0, d1;
                        four(sd + t * K + j * 32 + 4 * r, d0, d1);
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            S[2 * j][c] = mul2(d0, S[2 * j][c]);
                            S[2 * j + 1][c] = mul2(d1, S[2 * j + 1][c]);
                        }
                    }
                }
                float x[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint64_t s = mul2(S[0][c], k[0]);
#pragma unroll
                    for (int i = 1; i < RP; ++i) s = fma2(S[i][c], k[i], s);
                    float lo, hi;
                    unpack2(s, lo, hi);
                    x[c] = lo + hi;
                }
#pragma unroll
                for (int o = LK / 2; o > 0; o >>= 1) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) x[c] += __shfl_xor_sync(0xffffffffu, x[c], o);
                }
#pragma unroll
                for (int j = 0; j < RUNS; ++j) four(sq + t * K + j * 32 + 4 * r, q[2 * j], q[2 * j + 1]);
                float v[4];
                unpack2(v01, v[0], v[1]);
                unpack2(v23, v[2], v[3]);
                const float read = w.x * w.y, put = w.z * w.y;
                const uint64_t d = pack2(w.x, w.x);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float nv = put * (v[c] - read * x[c]);
                    const uint64_t n2 = pack2(nv, nv);
                    uint64_t y2 = 0ull;
#pragma unroll
                    for (int i = 0; i < RP; ++i) {
                        if constexpr (KDA) S[i][c] = fma2(k[i], n2, S[i][c]);
                        else S[i][c] = fma2(d, S[i][c], mul2(k[i], n2));
                        y2 = fma2(S[i][c], q[i], y2);
                    }
                    float lo, hi;
                    unpack2(y2, lo, hi);
                    y[u * 4 + c] = (lo + hi) * w.w;
                }
            }
            // Sixteen sums over the lanes: in every step the halves of the lanes keep a half of the sums each.
#pragma unroll
            for (int s = 0; s < 3; ++s) {
                const int keep = 8 >> s, o = LK >> (s + 1);
                const bool up = (r & o) != 0;
#pragma unroll
                for (int i = 0; i < keep; ++i) {
                    const float give = up ? y[i] : y[keep + i];
                    y[i] = (up ? y[keep + i] : y[i]) + __shfl_xor_sync(0xffffffffu, give, o);
                }
            }
            *reinterpret_cast<float2*>(sy + (t4 + r / 2) * cols + cg + r % 2 * 2) = make_float2(y[0], y[1]);     // the two sums that ended in this lane
        }
        __syncthreads();
        for (int i = tid; i < n * (cols / 4); i += nt) {
            const int t = i / (cols / 4), e = i % (cols / 4) * 4;
            const float4 y = *reinterpret_cast<const float4*>(sy + t * cols + e);
            const float f[4] = {y.x, y.y, y.z, y.w};
            const long long o = (long long)(t0 + t) * p.out_stride + (long long)h * p.V + c0;
            if (p.out_bf16) store_io<4>(static_cast<__nv_bfloat16*>(p.out) + o, e, f);
            else store_io<4>(static_cast<float*>(p.out) + o, e, f);
        }
    }
    if (dst >= 0) {
#pragma unroll
        for (int i = 0; i < RP; ++i) {
            const size_t o = dst * entry + at + (size_t)(i / 2 * 32 + i % 2 * 2) * p.V;
            float4 a4, b4;
            unpack2(S[i][0], a4.x, b4.x); unpack2(S[i][1], a4.y, b4.y); unpack2(S[i][2], a4.z, b4.z); unpack2(S[i][3], a4.w, b4.w);
            *reinterpret_cast<float4*>(p.state + o) = a4;
            *reinterpret_cast<float4*>(p.state + o + p.V) = b4;
        }
    }
}

template <typename T, int K, bool KDA>
int launch_cores(Ctx* ctx, const DeltaParams& p, long long units, cudaStream_t stream) {
    const size_t smem = (size_t)2 * stage_elements<KDA>(K, p.cols) * sizeof(T) + (size_t)kTok * (p.cols * 4 + 16 + (KDA ? K * 4 : 0));
    const auto kern = delta_scan_kernel<T, K, KDA>;
    const cudaError_t e = unlock_smem(ctx, kern);
    if (e != cudaSuccess) { ctx->last_cuda_error = e; return SKETCHSSM_CUDA_ERROR; }
    return launch_layer(ctx, kern, dim3((unsigned)units), dim3((unsigned)(p.cols * 2)), smem, stream, p);      // eight lanes for four columns
}

}  // namespace

int launch_delta_scan(Ctx* ctx, const DeltaParams& p0, bool bf16, cudaStream_t stream) {
    const int rc = launch_delta_scan_tc(ctx, p0, bf16, stream);
    if (rc != SKETCHSSM_UNSUPPORTED_SHAPE) return rc;
    DeltaParams p = p0;
    // As many columns of a head in a CTA (keys, queries and decays are then fetched once for them) as leave every SM four CTAs.
    const long long heads = (long long)p.pr.N * p.H;
    p.cols = 16;
    for (int c : {p.V, p.V / 2, 32})
        if (p.V % c == 0 && c % 16 == 0 && c > p.cols && heads * (p.V / c) >= 4ll * sm_count(ctx)) p.cols = c;
    const long long units = heads * (p.V / p.cols);
    if (units > 0x7fffffffll) return SKETCHSSM_UNSUPPORTED_SHAPE;
    const bool kda = ctx->cfg.kind == SKETCHSSM_KDA;
    if (p.K == 64) {
        if (bf16) return kda ? launch_cores<__nv_bfloat16, 64, true>(ctx, p, units, stream) : launch_cores<__nv_bfloat16, 64, false>(ctx, p, units, stream);
        return kda ? launch_cores<float, 64, true>(ctx, p, units, stream) : launch_cores<float, 64, false>(ctx, p, units, stream);
    }
    if (bf16) return kda ? launch_cores<__nv_bfloat16, 128, true>(ctx, p, units, stream) : launch_cores<__nv_bfloat16, 128, false>(ctx, p, units, stream);
    return kda ? launch_cores<float, 128, true>(ctx, p, units, stream) : launch_cores<float, 128, false>(ctx, p, units, stream);
}

}  // namespace sketchssm
