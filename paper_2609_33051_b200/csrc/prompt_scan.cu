// Selective scan of packed prompts on CUDA cores: every type, shape and precision that the library has.
//
//     S <- exp(a beta) S + beta k v^T,   out = S^T q + skip v,   token by token, S in fp32 registers.
//
// A CTA takes `cols` value columns of one head of one sequence.  A thread holds eight rows (K = 128: two runs of four; four with
// K = 64) of four columns, sixteen neighbouring lanes share the columns: a token is 48 two-element operations a thread and five loads
// of 16 bytes from shared memory.  The sums over the lanes are made for four tokens and columns together: every step halves what a
// lane still has to add, and nothing waits for a token's own chain of shuffles (which took 400 cycles a token).  Tokens come through
// shared memory, 32 of them while the 32 before are worked on.  Bound by fp32 issue (three multiply-adds for an element of the state and a
// token), and with few heads by the chain of a token, about 300 cycles.  2000 fp32 tokens of 24 heads of 80 columns, seven ragged
// sequences: 150 to 220 us, what the longest of them takes (lengths that took 152 us took 208 split in time for more CTAs: the states and a
// second reading cost more than the longest sequence's tail).
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

template <typename T, int K>
__global__ void __launch_bounds__(512) prompt_scan_kernel(const ScanParams p) {
    constexpr int LK = 16, RUNS = K / 64, RP = 2 * RUNS;       // lanes that share four columns; runs and pairs of rows of a thread
    extern __shared__ __align__(16) unsigned char sm[];
    const int cols = p.cols, nt = (int)blockDim.x, tid = (int)threadIdx.x;
    const int stage = kTok * (2 * K + cols);            // elements: keys, queries [kTok][K], values [kTok][cols]; two stages
    T* const raw = reinterpret_cast<T*>(sm);
    float* sy = reinterpret_cast<float*>(raw + 2 * stage);         // [kTok][cols]
    float2* sb = reinterpret_cast<float2*>(sy + kTok * cols);      // beta, decay [kTok]
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int blocks = p.V / cols;
    const int unit = (int)blockIdx.x;
    const int seq = unit / (p.H * blocks), h = unit / blocks % p.H, c0 = unit % blocks * cols;
    const int g = h / (p.H / p.G);
    const int2 rows = seq_rows(p.pr, seq);
    const int src = seq_resume(p.pr, seq), dst = seq_slot(p.pr, seq);
    const int r = tid % LK, cg = tid / LK * 4;          // this thread's rows 4 r .. (and K / 2 + 4 r ..), columns cg ..
    const size_t entry = (size_t)p.H * K * p.V, at = (size_t)h * K * p.V + (size_t)(4 * r) * p.V + c0 + cg;
    uint64_t S[RP][4];                                  // [pair of rows][column]
#pragma unroll
    for (int i = 0; i < RP; ++i) {
        const size_t o = src * entry + at + (size_t)(i / 2 * (K / 2) + i % 2 * 2) * p.V;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
        if (src >= 0) {
            a = *reinterpret_cast<const float4*>(p.state + o);
            b = *reinterpret_cast<const float4*>(p.state + o + p.V);
        }
        S[i][0] = pack2(a.x, b.x); S[i][1] = pack2(a.y, b.y); S[i][2] = pack2(a.z, b.z); S[i][3] = pack2(a.w, b.w);
    }
    const float a = p.a[h], bias = p.dt_bias != nullptr ? p.dt_bias[h] : 0.f, skip = p.skip != nullptr ? p.skip[h] : 0.f;
    constexpr int E = 16 / (int)sizeof(T);
    float dt = 0.f;
    auto fetch = [&](int t0, T* to) {
        const int n = min(kTok, rows.y - t0);
        for (int i = tid; i < n * (K / E); i += nt) {
            const int t = i / (K / E), e = i % (K / E) * E;
            copy16(to + t * K + e, static_cast<const T*>(p.k) + (long long)(t0 + t) * p.k_stride + (size_t)g * K + e);
            copy16(to + kTok * K + t * K + e, static_cast<const T*>(p.q) + (long long)(t0 + t) * p.q_stride + (size_t)g * K + e);
        }
        const int per = cols / E;
        for (int i = tid; i < n * per; i += nt) {
            const int t = i / per, e = i % per * E;
            copy16(to + 2 * kTok * K + t * cols + e, static_cast<const T*>(p.v) + (long long)(t0 + t) * p.v_stride + (size_t)h * p.V + c0 + e);
        }
        if (tid < n) dt = (float)static_cast<const T*>(p.dt)[(long long)(t0 + tid) * p.dt_stride + h];
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
            for (int i = n * K + tid; i < n4 * K; i += nt) { to[i] = zero; to[kTok * K + i] = zero; }
            for (int i = n * cols + tid; i < n4 * cols; i += nt) to[2 * kTok * K + i] = zero;
            if (tid >= n && tid < n4) sb[tid] = make_float2(0.f, 1.f);
        }
        if (tid < n) {
            const float beta = softplus(dt + bias);
            sb[tid] = make_float2(beta, expf(a * beta));
        }
        __syncthreads();                                // this stage is there, and nobody reads the other one any more
        if (t0 + kTok < rows.y) fetch(t0 + kTok, raw + (b ^ 1) * stage);
#pragma unroll 1
        for (int t4 = 0; t4 < n4; t4 += 4) {
            float y[16];                                // of four tokens and four columns
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int t = t4 + u;
                const float2 bd = sb[t];
                uint64_t k[RP], q[RP], v01, v23;
                four(sv + t * cols + cg, v01, v23);
                four(sk + t * K + 4 * r, k[0], k[1]);
                four(sq + t * K + 4 * r, q[0], q[1]);
                if constexpr (RUNS == 2) {
                    four(sk + t * K + K / 2 + 4 * r, k[2], k[3]);
                    four(sq + t * K + K / 2 + 4 * r, q[2], q[3]);
                }
                const uint64_t d = pack2(bd.y, bd.y), beta2 = pack2(bd.x, bd.x);
                float bv[4];
                unpack2(mul2(beta2, v01), bv[0], bv[1]);
                unpack2(mul2(beta2, v23), bv[2], bv[3]);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint64_t b2 = pack2(bv[c], bv[c]);
                    uint64_t y2 = 0ull;
#pragma unroll
                    for (int i = 0; i < RP; ++i) {
                        S[i][c] = fma2(d, S[i][c], mul2(k[i], b2));
                        y2 = fma2(S[i][c], q[i], y2);
                    }
                    float lo, hi;
                    unpack2(y2, lo, hi);
                    y[u * 4 + c] = lo + hi;
                }
            }
            // Sixteen sums over the lanes: in every step the halves of the lanes keep a half of the sums each.
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int keep = 8 >> s, o = LK >> (s + 1);
                const bool up = (r & o) != 0;
#pragma unroll
                for (int i = 0; i < keep; ++i) {
                    const float give = up ? y[i] : y[keep + i];
                    y[i] = (up ? y[keep + i] : y[i]) + __shfl_xor_sync(0xffffffffu, give, o);
                }
            }
            sy[(t4 + r / 4) * cols + cg + r % 4] = y[0];             // the sum that ended in this lane
        }
        __syncthreads();
        for (int i = tid; i < n * (cols / 4); i += nt) {
            const int t = i / (cols / 4), e = i % (cols / 4) * 4;
            uint64_t y01, y23, v01, v23;
            four(sy + t * cols + e, y01, y23);
            four(sv + t * cols + e, v01, v23);
            float f[4];
            unpack2(fma2(pack2(skip, skip), v01, y01), f[0], f[1]);
            unpack2(fma2(pack2(skip, skip), v23, y23), f[2], f[3]);
            const long long o = (long long)(t0 + t) * p.out_stride + (long long)h * p.V + c0;
            if (p.out_bf16) store_io<4>(static_cast<__nv_bfloat16*>(p.out) + o, e, f);
            else store_io<4>(static_cast<float*>(p.out) + o, e, f);
        }
    }
    if (dst >= 0) {
#pragma unroll
        for (int i = 0; i < RP; ++i) {
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
    // As many columns of a head in a CTA (keys and queries are then fetched once for them) as leave every SM four CTAs.  (16 fp32 heads of 64
    // columns, sequences of 50 tokens: 24 of them 45 us in blocks of 32, 53 in 16, 50 in 64; 74 of them 106 in 64, 135 in 16; 10 of them 30 in
    // 16, 27 in 32.)
    const long long heads = (long long)p.pr.N * p.H;
    p.cols = 16;
    for (int c : {p.V, p.V / 2, 32})
        if (p.V % c == 0 && c % 8 == 0 && c > p.cols && heads * (p.V / c) >= 4ll * sm_count(ctx)) p.cols = c;
    const long long units = heads * (p.V / p.cols);
    if (units > 0x7fffffffll) return SKETCHSSM_UNSUPPORTED_SHAPE;
    const size_t smem = (size_t)2 * kTok * (2 * p.K + p.cols) * (bf16 ? 2 : 4) + (size_t)(kTok * p.cols + 2 * kTok) * 4;
    void (*kern)(const ScanParams);
    if (p.K == 64) kern = bf16 ? prompt_scan_kernel<__nv_bfloat16, 64> : prompt_scan_kernel<float, 64>;
    else kern = bf16 ? prompt_scan_kernel<__nv_bfloat16, 128> : prompt_scan_kernel<float, 128>;
    const int threads = p.cols * 4;                     // sixteen lanes for four columns
    const cudaError_t e = unlock_smem(ctx, kern);
    if (e != cudaSuccess) { ctx->last_cuda_error = e; return SKETCHSSM_CUDA_ERROR; }
    return launch_layer(ctx, kern, dim3((unsigned)units), dim3((unsigned)threads), smem, stream, p);
}

}  // namespace sketchssm
