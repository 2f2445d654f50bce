// Short causal convolution of every channel, for packed prompts and for one token of every sequence.
//
//     y[t][c] = bias[c] + sum_{j < W} weight[c][j] x[t - (W - 1) + j][c],   W = 2..4, optionally SiLU behind it.
//
// Prompts: every element is read and written once, so HBM bounds it.  A thread owns 16 bytes of channels and walks down a run
// of R rows with the last W - 1 of them in registers; only those rows are read twice, by the runs on both sides of a border.
// Ragged sequences: a run takes the rows of its R whose window lies inside their sequence, and of every sequence that starts
// in it at least the first W - 1 rows, over its own end if need be.  So one run alone reads a sequence's stored rows, and it
// writes the new ones afterwards: the slot may be the resume entry, without a second launch.
//
// 16384 tokens of 4352 bf16 channels: 57 us, 5.0 TB/s (a copy of the same bytes: 44 us); the exponentials and reciprocals of SiLU keep
// their pipe busy for 61 % of it.
#include "pairs.cuh"

namespace sketchssm {

namespace {

// What a thread of the prompt kernel reads of a row: four channels.  (Sixteen bytes of bf16, eight channels, took 153 registers: 12 warps
// an SM and 66 us for 16384 x 4352.)
template <typename T>
struct Four;
template <>
struct Four<float> {
    using Raw = uint4;
    static __device__ __forceinline__ void open(const uint4& u, uint64_t (&f)[2]) {
        f[0] = (uint64_t)u.y << 32 | u.x;
        f[1] = (uint64_t)u.w << 32 | u.z;
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4]) { return Vec16<float>::pack(f); }
};
template <>
struct Four<__nv_bfloat16> {
    using Raw = uint2;
    static __device__ __forceinline__ void open(const uint2& u, uint64_t (&f)[2]) {
        f[0] = pack2(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u));
        f[1] = pack2(__uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
    }
    static __device__ __forceinline__ uint2 pack(const float (&f)[4]) {
        __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
        return make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
    }
};

// The taps and the bias of N channels.
template <int W, int N>
__device__ __forceinline__ void load_taps(const float* weight, const float* bias, int c, float (&w)[W][N], float (&b)[N]) {
    float flat[N * W];
#pragma unroll
    for (int i = 0; i < N * W / 4; ++i) {
        const float4 f = reinterpret_cast<const float4*>(weight + (size_t)c * W)[i];
        flat[4 * i] = f.x; flat[4 * i + 1] = f.y; flat[4 * i + 2] = f.z; flat[4 * i + 3] = f.w;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
        b[e] = 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j) w[j][e] = flat[e * W + j];
    }
    if (bias != nullptr) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const float4 f = reinterpret_cast<const float4*>(bias + c)[i];
            b[4 * i] = f.x; b[4 * i + 1] = f.y; b[4 * i + 2] = f.z; b[4 * i + 3] = f.w;
        }
    }
}

template <typename T, int W, int R>
__global__ void __launch_bounds__(128) causal_conv_kernel(const ConvParams p) {
    using V = Four<T>;
    using Raw = typename V::Raw;
    constexpr int N = 4, U = 4, kBlock = 128;
    grid_dep_wait();
    grid_dep_launch_dependents();
    const PromptsDev& pr = p.pr;
    const int t0 = (int)blockIdx.x * R;
    const bool last = blockIdx.x == gridDim.x - 1;
    // The whole run is on its way to L2 while the sequences are looked up and the taps fetched.
    const int c0 = (int)blockIdx.y * kBlock * N;
    for (int r = (int)threadIdx.x; r < R && t0 + r < pr.T; r += kBlock)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(static_cast<const T*>(p.x) + (long long)(t0 + r) * p.x_stride + c0),
                     "r"((uint32_t)(min(kBlock * N, p.C - c0) * (int)sizeof(T)))
                     : "memory");
    const int i0 = starts_before(pr, t0);              // by whole warps, before any thread leaves
    const int c = ((int)blockIdx.y * kBlock + (int)threadIdx.x) * N;
    if (c >= p.C) return;
    const T* x = static_cast<const T*>(p.x) + c;
    T* out = static_cast<T*>(p.out) + c;
    T* state = static_cast<T*>(p.state) + c;
    uint64_t w[W][N / 2], b[N / 2];                    // pairs of channels
    {
        float wf[W][N], bf[N];
        load_taps<W, N>(p.weight, p.bias, c, wf, bf);
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
            b[e] = pack2(bf[2 * e], bf[2 * e + 1]);
#pragma unroll
            for (int j = 0; j < W; ++j) w[j][e] = pack2(wf[j][2 * e], wf[j][2 * e + 1]);
        }
    }
    uint64_t win[W - 1][N / 2];                        // the rows before the next one, oldest first
    auto row = [&](const Raw& u, T* to) {
        uint64_t f[N / 2];
        V::open(u, f);
        float y[N];
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
            uint64_t s = b[e];
#pragma unroll
            for (int j = 0; j < W - 1; ++j) s = fma2(w[j][e], win[j][e], s);
            unpack2(fma2(w[W - 1][e], f[e], s), y[2 * e], y[2 * e + 1]);
        }
        if (p.silu) {
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = silu<T>(y[e]);
        }
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
#pragma unroll
            for (int j = 0; j + 1 < W - 1; ++j) win[j][e] = win[j + 1][e];
            win[W - 2][e] = f[e];
        }
        *reinterpret_cast<Raw*>(to) = V::pack(y);
    };
    // Rows t .. end - 1, U at a time; the next U are under way while these are worked on.
    auto walk = [&](int t, int end) {
        const T* from = x + (long long)t * p.x_stride;
        T* to = out + (long long)t * p.out_stride;
        Raw in[U], next[U];
        if (t + U <= end) {
#pragma unroll
            for (int u = 0; u < U; ++u) next[u] = *reinterpret_cast<const Raw*>(from + u * p.x_stride);
#pragma unroll 1
            while (t + U <= end) {
                from += U * p.x_stride;
                t += U;
#pragma unroll
                for (int u = 0; u < U; ++u) in[u] = next[u];
                if (t + U <= end) {
#pragma unroll
                    for (int u = 0; u < U; ++u) next[u] = *reinterpret_cast<const Raw*>(from + u * p.x_stride);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    row(in[u], to);
                    to += p.out_stride;
                }
            }
        }
#pragma unroll 1
        for (; t < end; ++t) {
            row(*reinterpret_cast<const Raw*>(from), to);
            from += p.x_stride;
            to += p.out_stride;
        }
    };
    if (i0 > 0) {                                      // the sequence that began before this run
        const int2 r = seq_rows(pr, i0 - 1);
        const int t = max(t0, r.x + W - 1), end = min(r.y, t0 + R);
        if (t < end) {
#pragma unroll
            for (int j = 0; j < W - 1; ++j) V::open(*reinterpret_cast<const Raw*>(x + (long long)(t - (W - 1) + j) * p.x_stride), win[j]);
            walk(t, end);
        }
    }
    for (int i = i0; i < pr.N; ++i) {                  // those that begin in it
        const int2 r = seq_rows(pr, i);
        if (r.x >= t0 + R && !last) break;
        const int src = seq_resume(pr, i), dst = seq_slot(pr, i);
        Raw old[W - 1];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            old[j] = Raw{};
            if (src >= 0) old[j] = *reinterpret_cast<const Raw*>(state + ((size_t)src * (W - 1) + j) * p.C);
            V::open(old[j], win[j]);
        }
        walk(r.x, min(r.y, max(t0 + R, r.x + W - 1)));
        if (dst >= 0) {
            const int len = r.y - r.x;
            Raw nw[W - 1];
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {          // row len + j of (stored rows, prompt)
                nw[j] = Raw{};
                if (len + j >= W - 1) {
                    nw[j] = *reinterpret_cast<const Raw*>(x + (long long)(r.y - (W - 1) + j) * p.x_stride);
                } else {
#pragma unroll
                    for (int m = 0; m < W - 1; ++m)
                        if (m == len + j) nw[j] = old[m];
                }
            }
#pragma unroll
            for (int j = 0; j < W - 1; ++j) *reinterpret_cast<Raw*>(state + ((size_t)dst * (W - 1) + j) * p.C) = nw[j];
        }
    }
}

// One token.  Values: a thread convolves 16 bytes of channels for four batch entries with the taps in registers (read for
// every entry they are as many bytes as everything else), moves the stored rows on and writes.  Keys and queries go to every head of
// their group, which is most of what the call writes: a block convolves 32 pieces of 16 bytes into shared memory and all its threads
// copy them to the heads.  The last block of a batch entry makes the gates.
constexpr int kEntries = 4, kPieces = 32;

template <typename T, int W>
__device__ __forceinline__ void token_rows(const ConvStepParams& p, int b, int c, int C, uint4 (&in)[W]) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) in[j] = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.state) + ((size_t)b * (W - 1) + j) * C + c);
    in[W - 1] = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.x) + (long long)b * p.x_stride + c);
}
template <typename T, int W>
__device__ __forceinline__ void conv_values(const ConvStepParams& p, int b, int c, int C, const uint4 (&in)[W], const float (&w)[W][Vec16<T>::N],
                                            const float (&bias)[Vec16<T>::N], float (&y)[Vec16<T>::N]) {
    using V = Vec16<T>;
    constexpr int N = V::N;
    float f[N];
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = bias[e];
#pragma unroll
    for (int j = 0; j < W; ++j) {
        V::unpack(in[j], f);
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = fmaf(w[j][e], f[e], y[e]);
        if (j > 0) *reinterpret_cast<uint4*>(static_cast<T*>(p.state) + ((size_t)b * (W - 1) + j - 1) * C + c) = in[j];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = silu<T>(y[e]);
}
template <typename T, int W>
__device__ __forceinline__ uint4 conv_token(const ConvStepParams& p, int b, int c, int C, const uint4 (&in)[W], const float (&w)[W][Vec16<T>::N],
                                            const float (&bias)[Vec16<T>::N]) {
    float y[Vec16<T>::N];
    conv_values<T, W>(p, b, c, C, in, w, bias, y);
    return Vec16<T>::pack(y);
}

template <typename T, int W>
__global__ void __launch_bounds__(128) conv_step_kernel(const ConvStepParams p) {
    constexpr int N = Vec16<T>::N;
    __shared__ uint4 piece[kPieces];
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int tid = (int)threadIdx.x, hv = p.H * p.V, gk = p.G * p.K, C = hv + 2 * gk;
    const int v_blocks = (hv / N + 127) / 128 * ((p.B + kEntries - 1) / kEntries), k_blocks = (2 * gk / N + kPieces - 1) / kPieces * p.B;
    int i = (int)blockIdx.x;
    if (i < k_blocks) {
        const int b = i % p.B, first = hv + i / p.B * kPieces * N, n = min(kPieces, (C - first) / N), per = p.H / p.G;
        if (tid < n) {
            float w[W][N], bias[N];
            uint4 in[W];
            token_rows<T, W>(p, b, first + tid * N, C, in);
            load_taps<W, N>(p.weight, p.bias, first + tid * N, w, bias);
            piece[tid] = conv_token<T, W>(p, b, first + tid * N, C, in, w, bias);
        }
        __syncthreads();
        const int at = tid % kPieces, c = first - hv + at * N;
        if (at >= n) return;
        const bool key = c < gk;
        const int e = key ? c : c - gk;
        const uint4 r = piece[at];
        T* dst = static_cast<T*>(key ? p.k : p.q) + ((size_t)b * p.H + (size_t)(e / p.K) * per) * p.K + e % p.K;
        for (int h = tid / kPieces; h < per; h += 128 / kPieces) *reinterpret_cast<uint4*>(dst + (size_t)h * p.K) = r;
        return;
    }
    i -= k_blocks;
    if (i < v_blocks) {
        const int groups = (p.B + kEntries - 1) / kEntries, b0 = i % groups * kEntries, c = (i / groups * 128 + tid) * N;
        if (c >= hv) return;
        float w[W][N], bias[N];
        uint4 in[kEntries][W];
#pragma unroll
        for (int k = 0; k < kEntries; ++k)
            if (b0 + k < p.B) token_rows<T, W>(p, b0 + k, c, C, in[k]);
        load_taps<W, N>(p.weight, p.bias, c, w, bias);
#pragma unroll
        for (int k = 0; k < kEntries; ++k)
            if (b0 + k < p.B) *reinterpret_cast<uint4*>(static_cast<T*>(p.v) + (size_t)(b0 + k) * hv + c) = conv_token<T, W>(p, b0 + k, c, C, in[k], w, bias);
        return;
    }
    i = (i - v_blocks) * 128 + tid;
    if (i < p.B * p.H) {
        const int b = i / p.H, h = i % p.H;
        const T* dt = static_cast<const T*>(p.dt) + (long long)b * p.dt_stride;
        const float beta = softplus((float)dt[h] + (p.dt_bias != nullptr ? p.dt_bias[h] : 0.f));
        p.beta[i] = beta;
        p.decay[i] = expf(p.a[h] * beta);
    }
}

// One token of a delta-rule layer.  A warp takes 32 pieces of 16 bytes of channels for four batch entries, with the taps in registers: of values,
// or of keys and queries, which are whole rows of K there (8, 16 or 32 neighbouring lanes): their norm is a sum over those, of what the
// activation leaves in fp32, and the result, rounded once, goes to every head of the group.  The last blocks make the gates: beta, and the
// decay of a head or (KDA, 16 bytes a thread) of its channels.
// What bounds it: memory, behind two rounds of latency.  512 KDA entries of 32 heads take 22 to 26 us for 109 MB (17 at 6.46 TB/s); with eight bytes of
// channels a thread and an entry at a time it took 60.
template <typename T, int W, bool KDA>
__global__ void __launch_bounds__(128) delta_step_kernel(const DeltaStepParams d) {
    constexpr int N = Vec16<T>::N;
    const ConvStepParams& p = d.c;
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int tid = (int)threadIdx.x, hv = p.H * p.V, gk = p.G * p.K, C = hv + 2 * gk;
    const int sets = (p.B + kEntries - 1) / kEntries, v_warps = (hv / N + 31) / 32, warps = (v_warps + (2 * gk / N + 31) / 32) * sets;
    const int blocks = (warps + 3) / 4;
    if ((int)blockIdx.x < blocks) {
        const int w0 = (int)blockIdx.x * 4 + (tid >> 5);
        if (w0 >= warps) return;
        const int b0 = w0 % sets * kEntries, unit = w0 / sets;
        const bool value = unit < v_warps;
        const int c = (value ? unit * 32 : hv / N + (unit - v_warps) * 32) * N + (tid & 31) * N;
        const bool in = c < (value ? hv : C);
        float w[W][N], bias[N];
        uint4 rows[kEntries][W];
        if (in) {
#pragma unroll
            for (int k = 0; k < kEntries; ++k)
                if (b0 + k < p.B) token_rows<T, W>(p, b0 + k, c, C, rows[k]);
            load_taps<W, N>(p.weight, p.bias, c, w, bias);
        }
        if (value) {
            if (!in) return;
#pragma unroll
            for (int k = 0; k < kEntries; ++k)
                if (b0 + k < p.B) *reinterpret_cast<uint4*>(static_cast<T*>(p.v) + (size_t)(b0 + k) * hv + c) = conv_token<T, W>(p, b0 + k, c, C, rows[k], w, bias);
            return;
        }
        const bool key = c < hv + gk;
        const int e = key ? c - hv : c - hv - gk, per = p.H / p.G;
        const float scale = key ? 1.f : d.q_scale;
#pragma unroll
        for (int k = 0; k < kEntries; ++k) {
            if (b0 + k >= p.B) break;
            float y[N], sq = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) y[i] = 0.f;
            if (in) conv_values<T, W>(p, b0 + k, c, C, rows[k], w, bias, y);
#pragma unroll
            for (int i = 0; i < N; ++i) sq = fmaf(y[i], y[i], sq);
            for (int o = p.K / N / 2; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
            const float r = inv_length(sq, d.eps) * scale;
#pragma unroll
            for (int i = 0; i < N; ++i) y[i] *= r;
            if (in) {
                T* dst = static_cast<T*>(key ? p.k : p.q) + ((size_t)(b0 + k) * p.H + (size_t)(e / p.K) * per) * p.K + e % p.K;
                const uint4 u = Vec16<T>::pack(y);
                for (int h = 0; h < per; ++h) *reinterpret_cast<uint4*>(dst + (size_t)h * p.K) = u;
            }
        }
        return;
    }
    const long long j = ((long long)blockIdx.x - blocks) * 128 + tid;
    if constexpr (KDA) {
        const int per = p.K / N;                         // threads of a head
        if (j >= (long long)p.B * p.H * per) return;
        const int b = (int)(j / (p.H * per)), hk = (int)(j % (p.H * per)) * N, h = hk / p.K;
        float f[N], add[N];
        Vec16<T>::unpack(*reinterpret_cast<const uint4*>(static_cast<const T*>(p.dt) + (long long)b * p.dt_stride + hk), f);
#pragma unroll
        for (int e = 0; e < N; ++e) add[e] = p.dt_bias != nullptr ? p.dt_bias[hk + e] : 0.f;
        const float a = p.a[h];
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = expf(a * softplus(f[e] + add[e]));
        *reinterpret_cast<uint4*>(static_cast<T*>(d.decay) + (size_t)b * p.H * p.K + hk) = Vec16<T>::pack(f);
        if (hk % p.K == 0) p.beta[(size_t)b * p.H + h] = 1.f / (1.f + expf(-(float)static_cast<const T*>(d.b)[(long long)b * d.b_stride + h]));
    } else if (j < (long long)p.B * p.H) {
        const int b = (int)(j / p.H), h = (int)(j % p.H);
        const float x = (float)static_cast<const T*>(p.dt)[(long long)b * p.dt_stride + h] + (p.dt_bias != nullptr ? p.dt_bias[h] : 0.f);
        p.beta[j] = 1.f / (1.f + expf(-(float)static_cast<const T*>(d.b)[(long long)b * d.b_stride + h]));
        static_cast<float*>(d.decay)[j] = expf(p.a[h] * softplus(x));
    }
}

template <typename T, int W>
int conv_width(Ctx* ctx, const ConvParams& p, cudaStream_t stream) {
    const int bx = (p.C / 4 + 127) / 128;
    // Runs of 32 rows where they give every SM work, of 8 below that (short calls are latency: fewer rows in a row).
    const long long blocks32 = (long long)bx * ((p.pr.T + 31) / 32);
    const int r = blocks32 >= 4ll * sm_count(ctx) ? 32 : 8;
    const dim3 grid((unsigned)max(1, (p.pr.T + r - 1) / r), (unsigned)bx);
    return r == 32 ? launch_layer(ctx, causal_conv_kernel<T, W, 32>, grid, dim3(128), 0, stream, p)
                   : launch_layer(ctx, causal_conv_kernel<T, W, 8>, grid, dim3(128), 0, stream, p);
}

template <typename T, int W>
int step_width(Ctx* ctx, const ConvStepParams& p, cudaStream_t stream) {
    constexpr int N = Vec16<T>::N;
    const long long values = (long long)((p.H * p.V / N + 127) / 128) * ((p.B + kEntries - 1) / kEntries);
    const long long others = (long long)((2 * p.G * p.K / N + kPieces - 1) / kPieces) * p.B, gates = ((long long)p.B * p.H + 127) / 128;
    if (values + others + gates > 0x7fffffff) return SKETCHSSM_UNSUPPORTED_SHAPE;
    return launch_layer(ctx, conv_step_kernel<T, W>, dim3((unsigned)(values + others + gates)), dim3(128), 0, stream, p);
}

template <typename T, int W, bool KDA>
int delta_width(Ctx* ctx, const DeltaStepParams& d, cudaStream_t stream) {
    constexpr int N = Vec16<T>::N;
    const ConvStepParams& p = d.c;
    const long long warps = (long long)((p.H * p.V / N + 31) / 32 + (2 * p.G * p.K / N + 31) / 32) * ((p.B + kEntries - 1) / kEntries);
    const long long blocks = (warps + 3) / 4 + ((long long)p.B * p.H * (KDA ? p.K / N : 1) + 127) / 128;
    if (warps > 0x7fffffff || blocks > 0x7fffffff) return SKETCHSSM_UNSUPPORTED_SHAPE;
    return launch_layer(ctx, delta_step_kernel<T, W, KDA>, dim3((unsigned)blocks), dim3(128), 0, stream, d);
}
template <typename T>
int delta_step_types(Ctx* ctx, const DeltaStepParams& p, cudaStream_t stream) {
    const bool kda = ctx->cfg.kind == SKETCHSSM_KDA;
    switch (p.c.W) {
        case 2: return kda ? delta_width<T, 2, true>(ctx, p, stream) : delta_width<T, 2, false>(ctx, p, stream);
        case 3: return kda ? delta_width<T, 3, true>(ctx, p, stream) : delta_width<T, 3, false>(ctx, p, stream);
        default: return kda ? delta_width<T, 4, true>(ctx, p, stream) : delta_width<T, 4, false>(ctx, p, stream);
    }
}

}  // namespace

int launch_delta_step(Ctx* ctx, const DeltaStepParams& p, bool bf16, cudaStream_t stream) {
    return bf16 ? delta_step_types<__nv_bfloat16>(ctx, p, stream) : delta_step_types<float>(ctx, p, stream);
}

int launch_causal_conv(Ctx* ctx, const ConvParams& p, bool bf16, cudaStream_t stream) {
    switch (p.W) {
        case 2: return bf16 ? conv_width<__nv_bfloat16, 2>(ctx, p, stream) : conv_width<float, 2>(ctx, p, stream);
        case 3: return bf16 ? conv_width<__nv_bfloat16, 3>(ctx, p, stream) : conv_width<float, 3>(ctx, p, stream);
        default: return bf16 ? conv_width<__nv_bfloat16, 4>(ctx, p, stream) : conv_width<float, 4>(ctx, p, stream);
    }
}

int launch_conv_step(Ctx* ctx, const ConvStepParams& p, bool bf16, cudaStream_t stream) {
    switch (p.W) {
        case 2: return bf16 ? step_width<__nv_bfloat16, 2>(ctx, p, stream) : step_width<float, 2>(ctx, p, stream);
        case 3: return bf16 ? step_width<__nv_bfloat16, 3>(ctx, p, stream) : step_width<float, 3>(ctx, p, stream);
        default: return bf16 ? step_width<__nv_bfloat16, 4>(ctx, p, stream) : step_width<float, 4>(ctx, p, stream);
    }
}

}  // namespace sketchssm
