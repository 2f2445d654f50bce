// Short causal convolution of every channel, for packed prompts and for one token of every sequence.
//
//     y[t][c] = bias[c] + sum_{j < W} weight[c][j] x[t - (W - 1) + j][c],   W = 2..4, optionally SiLU behind it.
//
// Prompts: every element is read and written once, so HBM bounds it.  A thread owns 16 bytes of channels and walks down a run
// of R rows with the last W - 1 of them in registers; only those rows are read twice, by the runs on both sides of a border.
// Ragged sequences: a run takes the rows of its R whose window lies inside their sequence, and of every sequence that starts
// in it at least the first W - 1 rows, over its own end if need be.  So one run alone reads a sequence's stored rows, and it
// writes the new ones afterwards: the slot may be the resume entry, without a second launch.
#include "layer.cuh"

namespace sketchssm {

namespace {

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
__global__ void __launch_bounds__(64) causal_conv_kernel(const ConvParams p) {
    using V = Vec16<T>;
    constexpr int N = V::N, U = 8;                     // rows requested together
    grid_dep_wait();
    grid_dep_launch_dependents();
    const PromptsDev& pr = p.pr;
    const int t0 = (int)blockIdx.x * R;
    const bool last = blockIdx.x == gridDim.x - 1;
    const int i0 = starts_before(pr, t0);              // by whole warps, before any thread leaves
    const int c = ((int)blockIdx.y * 64 + (int)threadIdx.x) * N;
    if (c >= p.C) return;
    const T* x = static_cast<const T*>(p.x) + c;
    T* out = static_cast<T*>(p.out) + c;
    T* state = static_cast<T*>(p.state) + c;
    float w[W][N], b[N];
    load_taps<W, N>(p.weight, p.bias, c, w, b);
    uint4 win[W - 1];                                  // the rows before the next one, oldest first
    auto walk = [&](int t, int end) {
        while (t < end) {
            const int n = min(U, end - t);
            uint4 in[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (u < n) in[u] = *reinterpret_cast<const uint4*>(x + (long long)(t + u) * p.x_stride);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u < n) {
                    float y[N], f[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) y[e] = b[e];
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) {
                        V::unpack(win[j], f);
#pragma unroll
                        for (int e = 0; e < N; ++e) y[e] = fmaf(w[j][e], f[e], y[e]);
                    }
                    V::unpack(in[u], f);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        y[e] = fmaf(w[W - 1][e], f[e], y[e]);
                        if (p.silu) y[e] = silu<T>(y[e]);
                    }
#pragma unroll
                    for (int j = 0; j + 1 < W - 1; ++j) win[j] = win[j + 1];
                    win[W - 2] = in[u];
                    *reinterpret_cast<uint4*>(out + (long long)(t + u) * p.out_stride) = V::pack(y);
                }
            }
            t += n;
        }
    };
    if (i0 > 0) {                                      // the sequence that began before this run
        const int2 r = seq_rows(pr, i0 - 1);
        const int t = max(t0, r.x + W - 1), end = min(r.y, t0 + R);
        if (t < end) {
#pragma unroll
            for (int j = 0; j < W - 1; ++j) win[j] = *reinterpret_cast<const uint4*>(x + (long long)(t - (W - 1) + j) * p.x_stride);
            walk(t, end);
        }
    }
    for (int i = i0; i < pr.N; ++i) {                  // those that begin in it
        const int2 r = seq_rows(pr, i);
        if (r.x >= t0 + R && !last) break;
        const int src = seq_resume(pr, i), dst = seq_slot(pr, i);
        uint4 old[W - 1];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            old[j] = make_uint4(0u, 0u, 0u, 0u);
            if (src >= 0) old[j] = *reinterpret_cast<const uint4*>(state + ((size_t)src * (W - 1) + j) * p.C);
            win[j] = old[j];
        }
        walk(r.x, min(r.y, max(t0 + R, r.x + W - 1)));
        if (dst >= 0) {
            const int len = r.y - r.x;
            uint4 nw[W - 1];
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {          // row len + j of (stored rows, prompt)
                nw[j] = make_uint4(0u, 0u, 0u, 0u);
                if (len + j >= W - 1) {
                    nw[j] = *reinterpret_cast<const uint4*>(x + (long long)(r.y - (W - 1) + j) * p.x_stride);
                } else {
#pragma unroll
                    for (int m = 0; m < W - 1; ++m)
                        if (m == len + j) nw[j] = old[m];
                }
            }
#pragma unroll
            for (int j = 0; j < W - 1; ++j) *reinterpret_cast<uint4*>(state + ((size_t)dst * (W - 1) + j) * p.C) = nw[j];
        }
    }
}

// One token: a thread per 16 bytes of channels convolves, moves the stored rows on and writes the value, or the key or query to
// every head of its group; the last block of a batch entry makes the gates.
template <typename T, int W>
__global__ void __launch_bounds__(128) conv_step_kernel(const ConvStepParams p) {
    using V = Vec16<T>;
    constexpr int N = V::N;
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int b = (int)blockIdx.x, hv = p.H * p.V, gk = p.G * p.K, C = hv + 2 * gk;
    if (blockIdx.y == gridDim.y - 1) {
        const T* dt = static_cast<const T*>(p.dt) + (long long)b * p.dt_stride;
        for (int h = (int)threadIdx.x; h < p.H; h += 128) {
            const float beta = softplus((float)dt[h] + (p.dt_bias != nullptr ? p.dt_bias[h] : 0.f));
            p.beta[(size_t)b * p.H + h] = beta;
            p.decay[(size_t)b * p.H + h] = expf(p.a[h] * beta);
        }
        return;
    }
    const int c = ((int)blockIdx.y * 128 + (int)threadIdx.x) * N;
    if (c >= C) return;
    const T* x = static_cast<const T*>(p.x) + (long long)b * p.x_stride + c;
    T* state = static_cast<T*>(p.state) + (size_t)b * (W - 1) * C + c;
    uint4 in[W];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) in[j] = *reinterpret_cast<const uint4*>(state + (size_t)j * C);
    in[W - 1] = *reinterpret_cast<const uint4*>(x);
    float y[N], f[N], w[W][N];
    load_taps<W, N>(p.weight, p.bias, c, w, y);
#pragma unroll
    for (int j = 0; j < W; ++j) {
        V::unpack(in[j], f);
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = fmaf(w[j][e], f[e], y[e]);
        if (j > 0) *reinterpret_cast<uint4*>(state + (size_t)(j - 1) * C) = in[j];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = silu<T>(y[e]);
    const uint4 r = V::pack(y);
    if (c < hv) {
        *reinterpret_cast<uint4*>(static_cast<T*>(p.v) + (size_t)b * hv + c) = r;
        return;
    }
    const bool key = c < hv + gk;
    const int e = c - hv - (key ? 0 : gk), per = p.H / p.G;
    T* dst = static_cast<T*>(key ? p.k : p.q) + ((size_t)b * p.H + (size_t)(e / p.K) * per) * p.K + e % p.K;
    for (int h = 0; h < per; ++h) *reinterpret_cast<uint4*>(dst + (size_t)h * p.K) = r;
}

template <typename T, int W>
int conv_width(Ctx* ctx, const ConvParams& p, cudaStream_t stream) {
    const int vecs = p.C / Vec16<T>::N, bx = (vecs + 63) / 64;
    // Runs of 32 rows where they give every SM work, of 8 below that (short calls are latency: fewer rows in a row).
    const long long blocks32 = (long long)bx * ((p.pr.T + 31) / 32);
    const int r = blocks32 >= 4ll * sm_count(ctx) ? 32 : 8;
    const dim3 grid((unsigned)max(1, (p.pr.T + r - 1) / r), (unsigned)bx);
    return r == 32 ? launch_layer(ctx, causal_conv_kernel<T, W, 32>, grid, dim3(64), 0, stream, p)
                   : launch_layer(ctx, causal_conv_kernel<T, W, 8>, grid, dim3(64), 0, stream, p);
}

template <typename T, int W>
int step_width(Ctx* ctx, const ConvStepParams& p, cudaStream_t stream) {
    const int vecs = (p.H * p.V + 2 * p.G * p.K) / Vec16<T>::N;
    return launch_layer(ctx, conv_step_kernel<T, W>, dim3((unsigned)p.B, (unsigned)((vecs + 127) / 128 + 1)), dim3(128), 0, stream, p);
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
