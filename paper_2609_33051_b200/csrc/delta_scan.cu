// Gated delta rule over packed prompts on CUDA cores: every type, shape and both kinds of decay that the library has.
//
//     S <- D S,   S <- S + beta k (v - S^T k)^T,   out = S^T q,   token by token, S in fp32 registers,
//
// k and q unit vectors (q times q_scale), beta = 1 / (1 + exp(-b)), D = exp(a softplus(dt + dt_bias)): a number a head (GDN) or a
// diagonal (KDA).
//
// Four tokens are worked on together.  With E_a the decays of the first a + 1 of them, D_sa those between s and a, all at most one,
//     u_a = beta_a (v_a - S^T E_a k_a - sum_{s < a} <k_a, D_sa k_s> u_s),   out_a = S^T E_a q_a + sum_{s <= a} <q_a, D_sa k_s> u_s,
//     S <- E_3 S + sum_s D_s3 k_s u_s^T,
// so that S is read with four keys and four queries at once and moved on once, and the sums over the lanes, which everything waits for, are
// made once in four tokens.
//
// A CTA takes `cols` value columns of one head of one sequence, the longest sequences first.  LK neighbouring lanes share four columns: eight, so
// that a thread holds sixteen rows (K = 128: four runs of four) of them, or sixteen where there are few heads.  Tokens come through shared memory,
// a stage of them while the one before is worked on; what four tokens have to do with one another is worked out by a warp, its lanes over the
// channels.
//
// What bounds it: multiplications.  4096 KDA tokens in 8 prompts of 512, 32 heads, 64 columns a CTA, take 566 us (in ragged ones 574 to 970: 0.55 us for
// each token of the longest; token by token 1400); three products with
// 16384 elements of a state a token are 6.4 G, 180 us at the card's rate.  Per four tokens a thread has 416 instructions for two such
// products each, two cycles long, and 175 others in the same pipe; the longest prompt's CTAs end last.  1500 fp32 tokens in 7
// prompts of 24 heads of 80 columns, 16 columns a CTA: 181 to 222 us by their lengths (token by token 306), bound by the longest prompt's chain of
// sums over lanes.
#include "pairs.cuh"

namespace sketchssm {

namespace {

template <bool KDA>
constexpr int kTok = KDA ? 16 : 32;                    // tokens of a stage
constexpr int kNear = 36;                              // floats of four tokens: see group_sums

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

// Elements of a stage: keys, queries, values.
template <bool KDA>
__host__ __device__ constexpr int stage_elements(int K, int cols) { return kTok<KDA> * (2 * K + cols); }

// log(1 + exp(x)): the logarithm of 1 + y as 2 artanh(y / (2 + y)), by its series (the argument is at most a third; what is left out is below
// 2^-26 of the sum).
__device__ __forceinline__ float softplus_series(float x) {
    const float y = expf(-fabsf(x)), z = __fdividef(y, 2.f + y), z2 = z * z;
    float s = 1.f / 15.f;
    s = fmaf(s, z2, 1.f / 13.f);
    s = fmaf(s, z2, 1.f / 11.f);
    s = fmaf(s, z2, 1.f / 9.f);
    s = fmaf(s, z2, 1.f / 7.f);
    s = fmaf(s, z2, 1.f / 5.f);
    s = fmaf(s, z2, 1.f / 3.f);
    s = fmaf(s, z2, 1.f);
    return fmaxf(x, 0.f) + 2.f * z * s;
}

// KDA's decays of every token and channel, once for all value columns: [T][H][K] floats in the scratch.
template <typename T>
__global__ void __launch_bounds__(256) delta_decay_kernel(const DeltaParams p) {
    constexpr int N = Vec16<T>::N;
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int per = p.H * p.K / N;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= (long long)p.pr.T * per) return;
    const int t = (int)(i / per), e = (int)(i % per) * N;
    float f[N], bias[N];
    Vec16<T>::unpack(*reinterpret_cast<const uint4*>(static_cast<const T*>(p.dt) + (long long)t * p.dt_stride + e), f);
#pragma unroll
    for (int j = 0; j < N; ++j) bias[j] = p.dt_bias != nullptr ? p.dt_bias[e + j] : 0.f;
    const float a = p.a[e / p.K];
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = expf(a * softplus_series(f[j] + bias[j]));
    float* to = reinterpret_cast<float*>(p.work) + (long long)t * p.H * p.K + e;
#pragma unroll
    for (int j = 0; j < N / 4; ++j) *reinterpret_cast<float4*>(to + 4 * j) = make_float4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]);
}

// Thirty-two sums over the lanes of a warp: sum i ends in lane i.
__device__ __forceinline__ float sum_of_lane(float (&v)[32], int lane) {
#pragma unroll
    for (int s = 0; s < 5; ++s) {
        const int keep = 16 >> s;
        const bool up = (lane & keep) != 0;
#pragma unroll
        for (int i = 0; i < keep; ++i) {
            const float give = up ? v[i] : v[keep + i];
            v[i] = (up ? v[keep + i] : v[i]) + __shfl_xor_sync(0xffffffffu, give, keep);
        }
    }
    return v[0];
}
__host__ __device__ constexpr int below(int a, int s) { return a * (a - 1) / 2 + s; }          // (a, s < a) of four
__host__ __device__ constexpr int upto(int a, int s) { return a * (a + 1) / 2 + s; }           // (a, s <= a)

// What four tokens have to do with one another, by a warp.  k, q: their rows (T) in shared memory; gate: decays (GDN) and betas, [2][4].
// near: [0..3] what S^T k is taken times, [4..9] L, [10..13] beta, [14..23] P, [24..27] what S^T q is taken times, [28..31] what u is put with,
// [32] the decay of all four.  KDA: d holds the decays [4][K]; the keys and queries with their norms and decays go to kp, qp, km [4][K],
// the decay of all four tokens to d4 [K].
template <typename T, int K, bool KDA>
__device__ __forceinline__ void group_sums(const T* k, const T* q, const float* gate, float* near, float* sums, float* kp, float* qp, float* km, float* d4,
                                           const float* d, float eps, float q_scale, int lane) {
    constexpr int C = K / 32;                           // channels of a lane
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = 0.f;
    float kr[4][C], qr[4][C], dr[4][C];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        load_io<C>(k, a * K + lane * C, kr[a]);
        load_io<C>(q, a * K + lane * C, qr[a]);
        if constexpr (KDA) load_io<C>(d, a * K + lane * C, dr[a]);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            v[a] = fmaf(kr[a][c], kr[a][c], v[a]);
            v[4 + a] = fmaf(qr[a][c], qr[a][c], v[4 + a]);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            float x = kr[s][c];
            v[14 + upto(s, s)] = fmaf(qr[s][c], x, v[14 + upto(s, s)]);
#pragma unroll
            for (int a = s + 1; a < 4; ++a) {
                if constexpr (KDA) x *= dr[a][c];
                v[8 + below(a, s)] = fmaf(kr[a][c], x, v[8 + below(a, s)]);
                v[14 + upto(a, s)] = fmaf(qr[a][c], x, v[14 + upto(a, s)]);
            }
        }
    }
    const float mine = sum_of_lane(v, lane);
    __syncwarp();
    sums[lane] = lane < 4 ? inv_length(mine, eps) : lane < 8 ? q_scale * inv_length(mine, eps) : mine;
    __syncwarp();
    float n[4], m[4], g[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) { n[a] = sums[a]; m[a] = sums[4 + a]; g[a] = KDA ? 1.f : gate[a]; }
    if constexpr (KDA) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float e = 1.f;
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                e *= dr[a][c];
                float x = kr[a][c] * n[a];
                kr[a][c] = x * e;
                qr[a][c] *= m[a] * e;
#pragma unroll
                for (int s = a + 1; s < 4; ++s) x *= dr[s][c];
                v[a * C + c] = x;
            }
            dr[0][c] = e;
        }
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            float x[C];
#pragma unroll
            for (int c = 0; c < C; ++c) x[c] = v[a * C + c];
            store_io<C>(kp, a * K + lane * C, kr[a]);
            store_io<C>(qp, a * K + lane * C, qr[a]);
            store_io<C>(km, a * K + lane * C, x);
        }
        store_io<C>(d4, lane * C, dr[0]);
    }
    // (a lane a number)
    float e[4];
    e[0] = g[0];
#pragma unroll
    for (int a = 1; a < 4; ++a) e[a] = e[a - 1] * g[a];
    float out = 0.f;
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        float between = 1.f;                            // the decays of the tokens behind s up to a
#pragma unroll
        for (int s = 3; s >= 0; --s) {
            if (s <= a && lane == 14 + upto(a, s)) out = m[a] * n[s] * between * sums[14 + upto(a, s)];
            if (s < a && lane == 4 + below(a, s)) out = n[a] * n[s] * between * sums[8 + below(a, s)];
            if (s <= a) between *= g[s];
        }
        float behind = 1.f;
#pragma unroll
        for (int s = a + 1; s < 4; ++s) behind *= g[s];
        if (lane == a) out = e[a] * n[a];
        if (lane == 24 + a) out = e[a] * m[a];
        if (lane == 28 + a) out = behind * n[a];
        if (lane == 10 + a) out = gate[4 + a];
    }
    near[lane] = out;
    if (lane == 0) near[32] = e[3];
}

// The sequence in place `place` when they stand by their lengths, the longest first.  (Every CTA finds its own by comparing all with all: beyond 64
// sequences they are left as they are.  48 KDA sequences of 60 tokens on the average, 8 heads: 104 us, in their own order 118; 100 of 30: 127
// and 129; 200 of 16: 224 and 143.)
__device__ __forceinline__ int by_length(const PromptsDev& pr, int place) {
    __shared__ int found;
    if (pr.N < 2 || pr.N > 64) return place;
    for (int i = (int)threadIdx.x; i < pr.N; i += (int)blockDim.x) {
        const int2 mine = seq_rows(pr, i);
        int before = 0;
        for (int j = 0; j < pr.N; ++j) {
            const int2 other = seq_rows(pr, j);
            before += other.y - other.x > mine.y - mine.x || (other.y - other.x == mine.y - mine.x && j < i);
        }
        if (before == place) found = i;
    }
    __syncthreads();
    return found;
}

template <typename T, int K, bool KDA, int LK>
// (All the registers that it asks for, 170 to 190: with 168, three CTAs an SM, KDA's 566 us become 718.)
__global__ void __maxnreg__(255) delta_scan_kernel(const DeltaParams p) {
    constexpr int RUNS = K / (4 * LK), RP = 2 * RUNS, STEPS = LK == 8 ? 3 : 4;     // runs of four rows and pairs of rows of a thread; halvings of its lanes
    constexpr int TOK = kTok<KDA>, GR = TOK / 4;
    extern __shared__ __align__(16) unsigned char sm[];
    const int cols = p.cols, nt = (int)blockDim.x, tid = (int)threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int stage = stage_elements<KDA>(K, cols);
    T* const raw = reinterpret_cast<T*>(sm);
    float* sy = reinterpret_cast<float*>(raw + 2 * stage);         // [TOK][cols]
    float* near = sy + TOK * cols;                                 // [GR][kNear]
    float* gates = near + GR * kNear;                              // [GR][2][4]
    float* sums = gates + GR * 8;                                  // [16 warps][32]
    float* kp = sums + 16 * 32;                                     // KDA: [TOK][K] three times, [GR][K], and the decays [2][TOK][K]
    float *qp = kp + TOK * K, *km = qp + TOK * K, *d4 = km + TOK * K, *sd = d4 + GR * K;
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int blocks = p.V / cols;
    const int unit = (int)blockIdx.x;
    const int seq = by_length(p.pr, unit / (p.H * blocks)), h = unit / blocks % p.H, c0 = unit % blocks * cols;
    const int g = h / (p.H / p.G);
    const int2 rows = seq_rows(p.pr, seq);
    const int src = seq_resume(p.pr, seq), dst = seq_slot(p.pr, seq);
    const int r = tid % LK, cg = tid / LK * 4;          // this thread's rows 4 r + 4 LK j .., columns cg ..
    const size_t entry = (size_t)p.H * K * p.V, at = (size_t)h * K * p.V + (size_t)(4 * r) * p.V + c0 + cg;
    uint64_t S[RP][4];                                  // [pair of rows][column]
#pragma unroll
    for (int i = 0; i < RP; ++i) {
        const size_t o = src * entry + at + (size_t)(i / 2 * 4 * LK + i % 2 * 2) * p.V;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
        if (src >= 0) {
            a = *reinterpret_cast<const float4*>(p.state + o);
            b = *reinterpret_cast<const float4*>(p.state + o + p.V);
        }
        S[i][0] = pack2(a.x, b.x); S[i][1] = pack2(a.y, b.y); S[i][2] = pack2(a.z, b.z); S[i][3] = pack2(a.w, b.w);
    }
    const float a = p.a[h];
    constexpr int E = 16 / (int)sizeof(T);
    const int v_row = tid / (cols / E), v_piece = tid % (cols / E);      // (cols LK / 4 threads: LK E / 4 rows of values at a time)
    const int y_row = tid / (cols / 4), y_piece = tid % (cols / 4) * 4;  // (LK rows of outputs)
    float dt = 0.f, bl = 0.f;
    auto fetch = [&](int t0, T* to) {
        const int n = min(TOK, rows.y - t0);
        for (int i = tid; i < n * (K / E); i += nt) {
            const int t = i / (K / E), e = i % (K / E) * E;
            copy16(to + t * K + e, static_cast<const T*>(p.k) + (long long)(t0 + t) * p.k_stride + (size_t)g * K + e);
            copy16(to + TOK * K + t * K + e, static_cast<const T*>(p.q) + (long long)(t0 + t) * p.q_stride + (size_t)g * K + e);
        }
        if constexpr (KDA) {
            float* d = sd + (to == raw ? 0 : TOK * K);
            for (int i = tid; i < n * (K / 4); i += nt)
                copy16(d + i * 4, reinterpret_cast<const float*>(p.work) + ((long long)(t0 + i / (K / 4)) * p.H + h) * K + i % (K / 4) * 4);
        }
        for (int t = v_row, e = v_piece * E; t < n; t += LK * E / 4) {
            copy16(to + 2 * TOK * K + t * cols + e, static_cast<const T*>(p.v) + (long long)(t0 + t) * p.v_stride + (size_t)h * p.V + c0 + e);
        }
        if (tid < n) {
            bl = (float)static_cast<const T*>(p.b)[(long long)(t0 + tid) * p.b_stride + h];
            if constexpr (!KDA) dt = (float)static_cast<const T*>(p.dt)[(long long)(t0 + tid) * p.dt_stride + h];
        }
    };
    if (rows.x < rows.y) fetch(rows.x, raw);
    int b = 0;
    for (int t0 = rows.x; t0 < rows.y; t0 += TOK, b ^= 1) {
        const int n = min(TOK, rows.y - t0);
        const T *sk = raw + b * stage, *sq = sk + TOK * K, *sv = sq + TOK * K;
        copies_done();
        const int n4 = (n + 3) & ~3;                    // tokens behind the last one change nothing
        if (n4 > n) {
            T* to = raw + b * stage;
            const T zero = (T)0.f;
            for (int i = n * K + tid; i < n4 * K; i += nt) {
                to[i] = zero;
                to[TOK * K + i] = zero;
            }
            for (int i = n * cols + tid; i < n4 * cols; i += nt) to[2 * TOK * K + i] = zero;
            if constexpr (KDA)
                for (int i = n * K + tid; i < n4 * K; i += nt) sd[b * TOK * K + i] = 1.f;
        }
        if (tid < TOK) {
            float decay = 1.f, beta = 0.f;
            if (tid < n) {
                beta = 1.f / (1.f + expf(-bl));
                if constexpr (!KDA) decay = expf(a * softplus(dt + (p.dt_bias != nullptr ? p.dt_bias[h] : 0.f)));
            }
            gates[tid / 4 * 8 + tid % 4] = decay;
            gates[tid / 4 * 8 + 4 + tid % 4] = beta;
        }
        __syncthreads();                                // this stage is there, and nobody reads the other one any more
        if (t0 + TOK < rows.y) fetch(t0 + TOK, raw + (b ^ 1) * stage);
        for (int i = warp; i < n4 / 4; i += nt >> 5)
            group_sums<T, K, KDA>(sk + i * 4 * K, sq + i * 4 * K, gates + i * 8, near + i * kNear, sums + warp * 32, kp + i * 4 * K, qp + i * 4 * K, km + i * 4 * K, d4 + i * K,
                                  sd + (b * TOK + i * 4) * K, p.eps, p.q_scale, lane);
        __syncthreads();
#pragma unroll 1
        for (int i4 = 0; i4 < n4 / 4; ++i4) {
            const int t4 = i4 * 4;
            const float* w = near + i4 * kNear;
            // four rows 4 r + 4 LK j .. of a token's key, of its query, and of what its u is put with
            auto key = [&](int u, int j, uint64_t& x, uint64_t& y) {
                if constexpr (KDA) four(kp + (t4 + u) * K + j * 4 * LK + 4 * r, x, y);
                else four(sk + (t4 + u) * K + j * 4 * LK + 4 * r, x, y);
            };
            auto query = [&](int u, int j, uint64_t& x, uint64_t& y) {
                if constexpr (KDA) four(qp + (t4 + u) * K + j * 4 * LK + 4 * r, x, y);
                else four(sq + (t4 + u) * K + j * 4 * LK + 4 * r, x, y);
            };
            float x[16];                                // S^T k of four tokens and four columns
            {
                uint64_t s[4][4];
#pragma unroll
                for (int j = 0; j < RUNS; ++j) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        uint64_t k0, k1;
                        key(u, j, k0, k1);
#pragma unroll
                        for (int c = 0; c < 4; ++c) s[u][c] = fma2(S[2 * j + 1][c], k1, j > 0 ? fma2(S[2 * j][c], k0, s[u][c]) : mul2(S[2 * j][c], k0));
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float lo, hi;
                    unpack2(s[i / 4][i % 4], lo, hi);
                    x[i] = lo + hi;
                }
            }
            // Sixteen sums over LK lanes: in every step the halves of the lanes keep a half of the sums each, then they hand them back.
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const int keep = 8 >> s, o = LK >> (s + 1);
                const bool up = (r & o) != 0;
#pragma unroll
                for (int i = 0; i < keep; ++i) {
                    const float give = up ? x[i] : x[keep + i];
                    x[i] = (up ? x[keep + i] : x[i]) + __shfl_xor_sync(0xffffffffu, give, o);
                }
            }
            float y[16];                                // the same of S^T q, meanwhile
            {
                uint64_t s[4][4];
#pragma unroll
                for (int j = 0; j < RUNS; ++j) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        uint64_t q0, q1;
                        query(u, j, q0, q1);
#pragma unroll
                        for (int c = 0; c < 4; ++c) s[u][c] = fma2(S[2 * j + 1][c], q1, j > 0 ? fma2(S[2 * j][c], q0, s[u][c]) : mul2(S[2 * j][c], q0));
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float lo, hi;
                    unpack2(s[i / 4][i % 4], lo, hi);
                    y[i] = lo + hi;
                }
            }
#pragma unroll
            for (int s = STEPS - 1; s >= 0; --s) {
                const int have = 8 >> s, o = LK >> (s + 1);
                const bool up = (r & o) != 0;
#pragma unroll
                for (int i = 0; i < have; ++i) {
                    const float other = __shfl_xor_sync(0xffffffffu, x[i], o), own = x[i];
                    x[i] = up ? other : own;
                    x[have + i] = up ? own : other;
                }
            }
            float f[kNear];
#pragma unroll
            for (int i = 0; i < kNear / 4; ++i) {
                const float4 v = *reinterpret_cast<const float4*>(w + 4 * i);
                f[4 * i] = v.x; f[4 * i + 1] = v.y; f[4 * i + 2] = v.z; f[4 * i + 3] = v.w;
            }
            float u[4][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                uint64_t v01, v23;
                four(sv + (t4 + t) * cols + cg, v01, v23);
                float v[4];
                unpack2(v01, v[0], v[1]);
                unpack2(v23, v[2], v[3]);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float z = KDA ? v[c] - x[t * 4 + c] : fmaf(-f[t], x[t * 4 + c], v[c]);
#pragma unroll
                    for (int s = 0; s < t; ++s) z = fmaf(-f[4 + below(t, s)], u[s][c], z);
                    u[t][c] = f[10 + t] * z;
                }
            }
            // S moves on
            if constexpr (!KDA) {
                const uint64_t keep = pack2(f[32], f[32]);
#pragma unroll
                for (int i = 0; i < RP; ++i) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) S[i][c] = mul2(keep, S[i][c]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < RUNS; ++j) {
                    uint64_t d0, d1;
                    four(d4 + i4 * K + j * 4 * LK + 4 * r, d0, d1);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        S[2 * j][c] = mul2(d0, S[2 * j][c]);
                        S[2 * j + 1][c] = mul2(d1, S[2 * j + 1][c]);
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                uint64_t put[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float z = KDA ? u[t][c] : f[28 + t] * u[t][c];
                    put[c] = pack2(z, z);
                }
#pragma unroll
                for (int j = 0; j < RUNS; ++j) {
                    uint64_t k0, k1;
                    if constexpr (KDA) four(km + (t4 + t) * K + j * 4 * LK + 4 * r, k0, k1);
                    else key(t, j, k0, k1);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        S[2 * j][c] = fma2(k0, put[c], S[2 * j][c]);
                        S[2 * j + 1][c] = fma2(k1, put[c], S[2 * j + 1][c]);
                    }
                }
            }
            // out: every lane keeps one or two of its sixteen sums
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float z = 0.f;
#pragma unroll
                    for (int s = 0; s <= t; ++s) z = fmaf(f[14 + upto(t, s)], u[s][c], z);
                    // (the lanes' sum takes it once)
                    y[t * 4 + c] = (KDA ? y[t * 4 + c] : f[24 + t] * y[t * 4 + c]) + (r == 0 ? z : 0.f);
                }
            }
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const int keep = 8 >> s, o = LK >> (s + 1);
                const bool up = (r & o) != 0;
#pragma unroll
                for (int i = 0; i < keep; ++i) {
                    const float give = up ? y[i] : y[keep + i];
                    y[i] = (up ? y[keep + i] : y[i]) + __shfl_xor_sync(0xffffffffu, give, o);
                }
            }
            // the sums that ended in this lane
            if constexpr (LK == 8) *reinterpret_cast<float2*>(sy + (t4 + r / 2) * cols + cg + r % 2 * 2) = make_float2(y[0], y[1]);
            else sy[(t4 + r / 4) * cols + cg + r % 4] = y[0];
        }
        __syncthreads();
        for (int t = y_row, e = y_piece; t < n; t += LK) {
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
            const size_t o = dst * entry + at + (size_t)(i / 2 * 4 * LK + i % 2 * 2) * p.V;
            float4 a4, b4;
            unpack2(S[i][0], a4.x, b4.x); unpack2(S[i][1], a4.y, b4.y); unpack2(S[i][2], a4.z, b4.z); unpack2(S[i][3], a4.w, b4.w);
            *reinterpret_cast<float4*>(p.state + o) = a4;
            *reinterpret_cast<float4*>(p.state + o + p.V) = b4;
        }
    }
}

template <typename T, int K, bool KDA, int LK>
int launch_lanes(Ctx* ctx, const DeltaParams& p, long long units, cudaStream_t stream) {
    constexpr int TOK = kTok<KDA>;
    const size_t smem = (size_t)2 * stage_elements<KDA>(K, p.cols) * sizeof(T) + (size_t)(TOK * p.cols + TOK / 4 * (kNear + 8) + 512) * 4 +
                        (KDA ? (size_t)(5 * TOK + TOK / 4) * K * 4 : 0);
    const auto kern = delta_scan_kernel<T, K, KDA, LK>;
    const cudaError_t e = unlock_smem(ctx, kern);
    if (e != cudaSuccess) { ctx->last_cuda_error = e; return SKETCHSSM_CUDA_ERROR; }
    return launch_layer(ctx, kern, dim3((unsigned)units), dim3((unsigned)(p.cols * LK / 4)), smem, stream, p);
}

template <typename T, int K, bool KDA>
int launch_cores(Ctx* ctx, const DeltaParams& p0, cudaStream_t stream) {
    DeltaParams p = p0;
    // Many heads: 64 or 80 columns of one in a CTA (what four tokens have to do with one another is then worked out once for them), eight lanes for
    // four of them.  Where that leaves SMs with a CTA alone or none, the chain of a token counts: 32 columns, or 16 of 80, and sixteen lanes.
    // Measured, with 64 or 80 columns and with 32 or 16: KDA, 1136 tokens, one prompt of 32 heads 589 us and 433, two 608 and 453, four 622 and
    // 896 (16 columns: 1249); 8 prompts of 512 558 and 741.  fp32 GDN, 500 tokens, one prompt of 32 heads 152 and 121, four 262 and 350; 8
    // prompts of 300, 16 heads of V = 64 95 and 110; V = 80, 24 heads, 3 prompts of 500 238 and 201, 7 of 300 289 and 231, 16 of 200 both 297.
    const long long heads = (long long)p.pr.N * p.H;
    const bool many = p.V == 80 ? heads >= 2ll * sm_count(ctx) : heads * (p.V / 32) > (KDA ? 2ll : 1ll) * sm_count(ctx);
    p.cols = p.V == 80 ? (many ? 80 : 16) : many ? 64 : 32;
    const long long units = heads * (p.V / p.cols);
    if (units > 0x7fffffffll) return SKETCHSSM_UNSUPPORTED_SHAPE;
    if constexpr (KDA) {
        const long long vecs = (long long)p.pr.T * (p.H * K / Vec16<T>::N);
        if (vecs / 256 >= 0x7fffffffll) return SKETCHSSM_UNSUPPORTED_SHAPE;
        if (vecs > 0) {
            const int rc = launch_layer(ctx, delta_decay_kernel<T>, dim3((unsigned)((vecs + 255) / 256)), dim3(256), 0, stream, p);
            if (rc != SKETCHSSM_OK) return rc;
        }
    }
    return many ? launch_lanes<T, K, KDA, 8>(ctx, p, units, stream) : launch_lanes<T, K, KDA, 16>(ctx, p, units, stream);
}

}  // namespace

int launch_delta_scan(Ctx* ctx, const DeltaParams& p, bool bf16, cudaStream_t stream) {
    const int rc = launch_delta_scan_tc(ctx, p, bf16, stream);
    if (rc != SKETCHSSM_UNSUPPORTED_SHAPE) return rc;
    const bool kda = ctx->cfg.kind == SKETCHSSM_KDA;
    if (p.K == 64) {
        if (bf16) return kda ? launch_cores<__nv_bfloat16, 64, true>(ctx, p, stream) : launch_cores<__nv_bfloat16, 64, false>(ctx, p, stream);
        return kda ? launch_cores<float, 64, true>(ctx, p, stream) : launch_cores<float, 64, false>(ctx, p, stream);
    }
    if (bf16) return kda ? launch_cores<__nv_bfloat16, 128, true>(ctx, p, stream) : launch_cores<__nv_bfloat16, 128, false>(ctx, p, stream);
    return kda ? launch_cores<float, 128, true>(ctx, p, stream) : launch_cores<float, 128, false>(ctx, p, stream);
}

}  // namespace sketchssm
