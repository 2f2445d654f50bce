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
__device__ __forceinline__ uint4 conv_token(const ConvStepParams& p, int b, int c, int C, const uint4 (&in)[W], const float (&w)[W][Vec16<T>::N],
                                            const float (&bias)[Vec16<T>::N]) {
    using V = Vec16<T>;
    constexpr int N = V::N;
    float y[N], f[N];
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
    return V::pack(y);
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

}  // namespace

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
