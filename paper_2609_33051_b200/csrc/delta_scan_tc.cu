// Gated delta rule over packed prompts on tcgen05 + TMEM: GDN, bf16 tensors, K = V = 128.
//
// A sequence goes through in chunks of 64 tokens.  With c_t the sum of the chunk's log2 decays up to token t, unit keys k (a key as it is times
// r_t) and S the state before the chunk, what the tokens add is U, the solution of a unit lower triangular system:
//     (I + L) U = X,   L[t][s] = beta_t 2^(c_t - c_s) <k_t, k_s> for s < t,   X[t] = beta_t (v_t - 2^c_t S^T k_t)
//     Y[t] = 2^c_t S^T q_t + sum_{s <= t} P[t][s] U[s],   P[t][s] = 2^(c_t - c_s) <q_t, k_s>
//     S <- 2^c_end S + sum_s 2^(c_end - c_s) k_s U[s]^T
// T = (I + L)^-1 and P do not depend on the state: a first kernel makes them, all chunks at once, and leaves them in the scratch as
// matrix operands; a second one takes a sequence and head at a time through its chunks.
//
// There the state is kept transposed: 128 value columns are the lanes of tensor memory, so that everything a chunk reads of it is one
// operand in tensor memory times a tile of shared memory (keys, queries, T, P), and a lane's thread scales, adds and splits without
// another thread's help.  Per chunk: K S^T and, later, Q S^T;  X;  (T - I) X;  U and W = 2^(c_end - c) r U;  W K and U P;  S.
//
// Precision.  States are fp32, outputs sums of fp32 accuracy rounded once.  Keys and queries are exact bf16 operands.  S, X, T - I and W
// go to the tensor cores in three parts of bf16 (24 bits; products of parts below 2^-24 are left out), so that the state's error stays that of
// fp32 sums: with two parts of S, X and T it was 10 to 30 times larger.  What is for the outputs alone, S with the queries, P and
// U, goes in two parts (2^-16 of a term), where an output's own rounding is 2^-8 of their sum.  Sums of log decays are made in 64 bits and
// kept as a whole number and a rest of at most a half.
#include "tma.cuh"

#include <utility>

namespace sketchssm {

namespace {

using namespace tc;

constexpr int kQ = 64;                                 // tokens of a chunk
constexpr uint32_t kPart = 8192u;                      // 64 rows of 128 bytes
constexpr uint32_t kTOff = 0, kPOff = 3 * kPart, kGOff = 5 * kPart;
// gates of a chunk and head, 64 floats each: beta, beta 2^c r, 2^(c_end - c) r, q_scale 2^c / |q|, and 2^c_end
constexpr int kBeta = 0, kRead = 64, kPut = 128, kAsk = 192, kKeep = 256, kGates = 320;
constexpr uint32_t kBlock = kGOff + kGates * 4u;       // bytes of the scratch for a chunk of a head

struct DeltaArgs {
    CUtensorMap tq, tk, tv;
    DeltaParams p;
    int units;
};

// The first chunk of sequence i in the scratch: chunks of sequences that follow one another never meet, whatever their lengths are.
__device__ __forceinline__ int chunk_base(int row0, int i) { return row0 / kQ + i; }

__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool acc) { tc_mma_bf16(d, a, b, idesc, acc ? 1u : 0u); }
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc ? 1u : 0u)
        : "memory");
}
__device__ __forceinline__ void tmem_st8u(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void bulk_s2g(void* dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_u32(src)), "r"(bytes) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}

__device__ __forceinline__ uint32_t bf16x2(float a, float b) {
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
}
// Two floats as two parts of bfloat16 each: what the first leaves, rounded, is the second.
__device__ __forceinline__ void two_parts(uint64_t x, uint32_t& hi, uint32_t& lo) {
    float a, b;
    unpack2(x, a, b);
    hi = bf16x2(a, b);
    unpack2(fma2(pack2(__uint_as_float(hi << 16), __uint_as_float(hi & 0xffff0000u)), pack2(-1.f, -1.f), x), a, b);
    lo = bf16x2(a, b);
}
// Two floats as three parts each: the upper 16 bits of what is left, twice, and the rest rounded: 8 + 8 + 8 bits.
__device__ __forceinline__ void three_parts(uint64_t x, uint32_t& p0, uint32_t& p1, uint32_t& p2) {
    const uint64_t minus = pack2(-1.f, -1.f);
    uint32_t lo = (uint32_t)x & 0xffff0000u, hi = (uint32_t)(x >> 32) & 0xffff0000u;
    p0 = __byte_perm(lo, hi, 0x7632);
    x = fma2(pack2(__uint_as_float(lo), __uint_as_float(hi)), minus, x);
    lo = (uint32_t)x & 0xffff0000u;
    hi = (uint32_t)(x >> 32) & 0xffff0000u;
    p1 = __byte_perm(lo, hi, 0x7632);
    x = fma2(pack2(__uint_as_float(lo), __uint_as_float(hi)), minus, x);
    float a, b;
    unpack2(x, a, b);
    p2 = bf16x2(a, b);
}

constexpr uint32_t kTypes = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);      // bf16 x bf16 -> fp32, 128 rows

// ---- what does not depend on the state: T and P of every chunk ------------------------------------------------------------
//
// A CTA takes a chunk, a group and two of its heads.  One product gives the rows <k_t, k_s> (lanes 0..63) and <q_t, k_s> (64..127);
// threads 0..63 make -L of both heads from them, the others P.  T is found column by column: a thread holds a whole column in registers and
// takes from the rows below what each of its elements puts there, so that nothing is waited for; two warps a head.
// The columns from 32 on start at row 32: the heavy half changes schedulers with the CTA's number.

constexpr int kPrepThreads = 128;
constexpr uint32_t kPrepL = 4 * kPart;                 // behind the tile of K and Q rows (whose place P takes): -L of two heads, [s][t] floats
constexpr uint32_t kPrepNorm = kPrepL + 2u * kQ * kQ * 4u;        // 1 / |k|, 1 / |q|: [2][64]
constexpr uint32_t kPrepSum = kPrepNorm + 2u * kQ * 4u;           // of each head: whole, rest, beta: [2][3][64]
constexpr uint32_t kPrepBar = kPrepSum + 6u * kQ * 4u;
constexpr uint32_t kPrepSmem = kPrepBar + 32u + 1024u;

// What element S of a column puts into the rows below: l holds -L, [s][t].
template <int S>
__device__ __forceinline__ void take(uint64_t (&T)[32], const float* l) {
    float a, b;
    unpack2(T[S / 2], a, b);
    const float ts = S % 2 ? b : a;
    const uint64_t ts2 = pack2(ts, ts);
    if constexpr (S % 2 == 0) T[S / 2] = pack2(a, fmaf(l[S * kQ + S + 1], ts, b));
    constexpr int first = S / 2 + 1;                    // the first pair behind S
    if constexpr (first % 2 == 1 && first < 32) T[first] = fma2(*reinterpret_cast<const uint64_t*>(l + S * kQ + 2 * first), ts2, T[first]);
#pragma unroll
    for (int i = (first + 1) / 2; i < 16; ++i) {
        const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(l + S * kQ + 4 * i);
        T[2 * i] = fma2(v.x, ts2, T[2 * i]);
        T[2 * i + 1] = fma2(v.y, ts2, T[2 * i + 1]);
    }
}
template <int FIRST, int... I>
__device__ __forceinline__ void take_rows(uint64_t (&T)[32], const float* l, std::integer_sequence<int, I...>) { (take<FIRST + I>(T, l), ...); }

__global__ void __launch_bounds__(kPrepThreads, 3) delta_prep_kernel(const __grid_constant__ DeltaArgs g) {
    extern __shared__ unsigned char raw[];
    unsigned char* smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    float* minus_l = reinterpret_cast<float*>(smem + kPrepL);
    float* norms = reinterpret_cast<float*>(smem + kPrepNorm);
    float* sums = reinterpret_cast<float*>(smem + kPrepSum);
    uint64_t* bar = reinterpret_cast<uint64_t*>(smem + kPrepBar);
    uint32_t* slot = reinterpret_cast<uint32_t*>(bar + 2);
    const DeltaParams& p = g.p;
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int per = p.H / p.G, batches = (per + 1) / 2;
    int u = (int)blockIdx.x;
    const int batch = u % batches;
    u /= batches;
    const int group = u % p.G, chunk = u / p.G;
    if (tid == 0) {
        mbar_init(bar, 1);
        mbar_init(bar + 1, 1);
        mbar_fence_init();
    }
    if (warp == 1) tmem_alloc<64>(slot);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    grid_dep_wait();
    grid_dep_launch_dependents();
    const uint32_t tmem = *slot;
    // the sequence of this chunk: the last one whose first chunk is not behind it
    int n = 0;
    for (int j = lane; j - lane < p.pr.N; j += 32)
        n += __popc(__ballot_sync(0xffffffffu, j < p.pr.N && chunk_base(seq_start(p.pr, min(j, p.pr.N - 1)), j) <= chunk));
    bool ok = n > 0;
    int t0 = 0, valid = 0;
    if (ok) {
        const int2 rows = seq_rows(p.pr, n - 1);
        t0 = rows.x + (chunk - chunk_base(rows.x, n - 1)) * kQ;
        valid = min(kQ, rows.y - t0);
        ok = t0 >= rows.x && valid > 0;
    }
    if (ok) {
        if (tid == 0) {
            mbar_expect_tx(bar, 4 * kPart);
            for (int h = 0; h < 2; ++h) {
                tma_load(smem + h * 2 * kPart, &g.tk, group * 128 + h * 64, t0, bar);
                tma_load(smem + h * 2 * kPart + kPart, &g.tq, group * 128 + h * 64, t0, bar);
            }
        }
        const int h0 = group * per + batch * 2, heads = min(2, per - batch * 2);
        // gates, while the rows are under way: a warp a head, two neighbouring tokens a lane
        if (warp < heads) {
            const int h = h0 + warp;
            float* s = sums + warp * 3 * kQ;
            const float a2 = p.a[h] * 1.4426950408889634f, bias = p.dt_bias != nullptr ? p.dt_bias[h] : 0.f;
            double c[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int t = lane * 2 + i;
                float l = 0.f, beta = 0.f;
                if (t < valid) {
                    const long long r = t0 + t;
                    beta = 1.f / (1.f + expf(-__bfloat162float(static_cast<const __nv_bfloat16*>(p.b)[r * p.b_stride + h])));
                    l = a2 * softplus(__bfloat162float(static_cast<const __nv_bfloat16*>(p.dt)[r * p.dt_stride + h]) + bias);
                    if (l < -160.f) l = -160.f;         // (2^-160 is zero in fp32; the bound keeps the sums finite; NaN passes it)
                }
                s[2 * kQ + t] = beta;
                c[i] = i > 0 ? c[0] + (double)l : (double)l;
            }
            double before = c[1];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double up = __shfl_up_sync(0xffffffffu, before, o);
                if (lane >= o) before += up;
            }
            before = __shfl_up_sync(0xffffffffu, before, 1);
            if (lane == 0) before = 0.0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const double x = c[i] + before, w = rint(x);
                s[lane * 2 + i] = (float)w;
                s[kQ + lane * 2 + i] = (float)(x - w);
            }
        }
        ok = mbar_wait_bounded(bar, 0);
        // norms: a row of K or Q a thread
        {
            float sq = 0.f;
            const unsigned char* row = smem + (tid & 64) * 128 + (tid & 63) * 128;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float f[8];
                    Vec16<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4*>(row + h * 2 * kPart + ((i ^ (tid & 7)) * 16)), f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sq = fmaf(f[e], f[e], sq);
                }
            }
            norms[tid] = inv_length(sq, p.eps) * (tid < 64 ? 1.f : p.q_scale);
        }
        ok = __syncthreads_and(ok) != 0;
        if (warp == 0 && ok) {
            const uint64_t da = swizzled_desc(smem_u32(smem), 16u, 1024u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint64_t at = da + (uint32_t)(i / 4) * (2 * kPart >> 4) + (uint32_t)(i % 4) * 2u;
                if (elect()) mma_ss(tmem, at, at, kTypes | ((64u >> 3) << 17), i > 0);
            }
            if (elect()) tc_commit(bar + 1);
            __syncwarp();
        }
        // what the second kernel reads of the gates
        if (ok && tid < 64) {
            for (int j = 0; j < heads; ++j) {
                const float *s = sums + j * 3 * kQ, w = s[tid], r = s[kQ + tid];
                float* to = reinterpret_cast<float*>(p.work + ((size_t)chunk * p.H + h0 + j) * kBlock + kGOff);
                const bool in = tid < valid;
                const float e = exp2f(w) * exp2f(r), rest = exp2f(s[kQ - 1] - w) * exp2f(s[2 * kQ - 1] - r);
                to[kBeta + tid] = s[2 * kQ + tid];
                to[kRead + tid] = in ? s[2 * kQ + tid] * e * norms[tid] : 0.f;
                to[kPut + tid] = in ? rest * norms[tid] : 0.f;
                to[kAsk + tid] = in ? e * norms[64 + tid] : 0.f;
                if (tid == 63) to[kKeep] = e;
            }
        }
        ok = ok && mbar_wait_bounded(bar + 1, 0);
        ok = __syncthreads_and(ok) != 0;                // (from here on the tile's place is P's)
        if (ok) {
            tc_fence_after();
            const int t = tid & 63;
            const uint32_t lanes = (uint32_t)(warp * 32) << 16;
#pragma unroll 1
            for (int j = 0; j < heads; ++j) {
                const float *s = sums + j * 3 * kQ, w = s[t], r = s[kQ + t];
                const bool in = t < valid;
                if (tid < 64) {
                    const float mine = -s[2 * kQ + t] * norms[t];
                    float* to = minus_l + j * kQ * kQ + t;
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {
                        uint32_t d[16];
                        tmem_ld16_async(tmem + lanes + c * 16, d);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int e = c * 16 + i;
                            const float x = mine * norms[e] * __uint_as_float(d[i]) * ex2((w - s[e]) + (r - s[kQ + e]));
                            to[e * kQ] = in && e < t ? x : 0.f;
                        }
                    }
                } else {
                    const float mine = norms[64 + t];
                    unsigned char* to = smem + j * 2 * kPart + t * 128;
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {
                        uint32_t d[16], hi[8], lo[8];
                        tmem_ld16_async(tmem + lanes + c * 16, d);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            float x[2];
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                const int e = c * 16 + i + q;
                                const float y = mine * norms[e] * __uint_as_float(d[i + q]) * ex2((w - s[e]) + (r - s[kQ + e]));
                                x[q] = in && e <= t ? y : 0.f;
                            }
                            two_parts(pack2(x[0], x[1]), hi[i / 2], lo[i / 2]);
                        }
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            unsigned char* at = to + (((c * 2 + q) ^ (t & 7)) * 16);
                            *reinterpret_cast<uint4*>(at) = make_uint4(hi[4 * q], hi[4 * q + 1], hi[4 * q + 2], hi[4 * q + 3]);
                            *reinterpret_cast<uint4*>(at + kPart) = make_uint4(lo[4 * q], lo[4 * q + 1], lo[4 * q + 2], lo[4 * q + 3]);
                        }
                    }
                    proxy_fence();
                }
            }
            __syncthreads();
            if (tid == 64)
                for (int j = 0; j < heads; ++j) bulk_s2g(p.work + ((size_t)chunk * p.H + h0 + j) * kBlock + kPOff, smem + j * 2 * kPart, 2 * kPart);
            // column `col` of T: element t takes -L[t][s] T[s] from every s before it
            const int head = warp >> 1, col = (tid & 63) ^ ((blockIdx.x & 1) * 32);
            if (head < heads) {
                uint64_t T[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) T[i] = pack2(2 * i == col ? 1.f : 0.f, 2 * i + 1 == col ? 1.f : 0.f);
                const float* l = minus_l + head * kQ * kQ;
                if (col < 32) take_rows<0>(T, l, std::make_integer_sequence<int, 32>{});
                take_rows<32>(T, l, std::make_integer_sequence<int, 31>{});
                // T - I in three parts: rows t of 128 bytes, this thread's two of each
                unsigned char* to = p.work + ((size_t)chunk * p.H + h0 + head) * kBlock + kTOff + (col % 8) * 2;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    float x[2];
                    unpack2(T[i], x[0], x[1]);
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const int t = 2 * i + q;
                        float y = t > col ? x[q] : 0.f;
                        unsigned short* at = reinterpret_cast<unsigned short*>(to + t * 128 + (((col / 8) ^ (t & 7)) * 16));
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t top = __float_as_uint(y) & 0xffff0000u;
                            at[e * (kPart / 2)] = (unsigned short)(top >> 16);
                            y -= __uint_as_float(top);
                        }
                        at[2 * (kPart / 2)] = __bfloat16_as_ushort(__float2bfloat16_rn(y));
                    }
                }
            }
            if (tid == 64) tma_store_done();
        }
        if (!ok && tid == 0) record_fault(p.status, kFaultScanWait, 11);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_free<64>(tmem);
}

// ---- the chunks of a sequence, one after another ------------------------------------------------------------------------------
//
// Roles: warp 0 issues the copies, warp 1 the products; warps 4..11 hold the state, a lane of tensor memory and half of what is there to
// split a thread (64 keys' channels of S, 32 tokens of X, U, W and Y).  They meet through mbarriers alone; every wait is bounded.
// Operands go over in quarters (16 tokens, 32 channels), products follow them as they come; T and P are lower triangular, a quarter of
// them meets the tokens from itself on only.
// Tensor memory: three parts of S, whose place W K takes once Q S^T is there; three parts of X, then of W, and two of U; K S^T, then
// (T - I) X; Y.

constexpr int kThreads = 384;
constexpr uint32_t kKOff = 0, kQOff = 2 * kPart, kVOff = 4 * kPart, kWOff = 6 * kPart;
constexpr uint32_t kStage = (kWOff + kBlock + 1023u) & ~1023u;
constexpr uint32_t kBarOff = 2 * kStage;
enum { bFull = 0, bEmpty = 2, bS = 4, bX = 8, bRead = 9, bXP = 10, bU = 14, bWP = 15, bProd = 19, bAsk = 20, bScaled = 21, bY = 22, bYFree = 23, kBars = 24 };
constexpr uint32_t kMarkOff = kBarOff + kBars * 8u + 16u;        // [128]: see mark_of
constexpr uint32_t kSmemTc = kMarkOff + 128u * 4u + 1024u;

// columns of tensor memory: parts of S (half h, part i: 96 h + 32 i), W K; parts of X and W, of U (part i, tokens s: 32 i + s / 2); K S^T and (T - I) X; Y
constexpr uint32_t cS = 0, cW = 192, cU = 288, cX = 352, cY = 416;

// The products take every token's values into every token, and a zero weight times NaN or infinity is NaN: from a lane's first value
// that is not finite on, zeros go to the products, and the lane's outputs and state become NaN afterwards.  A mark of chunk n holds that
// token; the largest of several is the first token of the latest chunk, so that marks need no clearing.
__device__ __forceinline__ uint32_t mark_of(int n, int token) { return ((uint32_t)n << 7) + (uint32_t)(kQ - token); }

__global__ void __launch_bounds__(kThreads, 1) delta_scan_tc_kernel(const __grid_constant__ DeltaArgs g) {
    extern __shared__ unsigned char raw[];
    unsigned char* smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    uint64_t* bar = reinterpret_cast<uint64_t*>(smem + kBarOff);
    uint32_t* slot = reinterpret_cast<uint32_t*>(bar + kBars);
    uint32_t* marks = reinterpret_cast<uint32_t*>(smem + kMarkOff);
    const DeltaParams& p = g.p;
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 32) { prefetch_map(&g.tq); prefetch_map(&g.tk); prefetch_map(&g.tv); }
    if (tid == 0) {
        for (int i = 0; i < kBars; ++i) {
            int n = 1;                                  // copies and commits of products arrive once
            if (i == bEmpty || i == bEmpty + 1) n = 9;  // the products' commit and the eight warps
            if ((i >= bS && i < bX) || (i >= bXP && i < bU) || (i >= bWP && i < bProd)) n = 4;      // the four warps of a quarter
            if (i == bRead || i == bScaled || i == bYFree) n = 8;
            mbar_init(bar + i, n);
        }
        mbar_fence_init();
    }
    if (tid < 128) marks[tid] = 0u;
    if (warp == 1) tmem_alloc<512>(slot);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    grid_dep_wait();
    grid_dep_launch_dependents();
    const uint32_t tmem = *slot;
    const uint32_t sbase = smem_u32(smem);
    bool ok = true;
    int n = 0, m = 0;                                   // chunks so far, over all units of the CTA; those with a state before them

    if (warp == 0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (lane == 0) {
            for (int u = (int)blockIdx.x; u < g.units && ok; u += (int)gridDim.x) {
                const int head = u % p.H, seq = u / p.H, group = head / (p.H / p.G);
                const int2 rows = seq_rows(p.pr, seq);
                int chunk = chunk_base(rows.x, seq);
                for (int t = rows.x; t < rows.y; t += kQ, ++chunk, ++n) {
                    const int b = n & 1;
                    ok = n < 2 || mbar_wait_bounded(bar + bEmpty + b, (n / 2 - 1) & 1);
                    if (!ok) break;
                    unsigned char* to = smem + b * kStage;
                    mbar_expect_tx(bar + bFull + b, 6 * kPart + kBlock);
                    tma_load(to + kKOff, &g.tk, group * 128, t, bar + bFull + b);
                    tma_load(to + kKOff + kPart, &g.tk, group * 128 + 64, t, bar + bFull + b);
                    bulk_g2s(to + kWOff, p.work + ((size_t)chunk * p.H + head) * kBlock, kBlock, bar + bFull + b);
                    tma_load(to + kVOff, &g.tv, head * 128, t, bar + bFull + b);
                    tma_load(to + kVOff + kPart, &g.tv, head * 128 + 64, t, bar + bFull + b);
                    tma_load(to + kQOff, &g.tq, group * 128, t, bar + bFull + b);
                    tma_load(to + kQOff + kPart, &g.tq, group * 128 + 64, t, bar + bFull + b);
                }
            }
            if (!ok) record_fault(p.status, kFaultScanWait, 12);
            // Before the CTA ends the copies under way have ended (after a fault; otherwise they have been waited for), and the last arrivals
            // at the buffers' barriers are in.
            for (int i = n < 2 ? 0 : n - 2; i < n; ++i) mbar_wait_bounded(bar + (ok ? bEmpty : bFull) + (i & 1), (i / 2) & 1, ok ? 1u << 22 : 1u << 16);
        }
        __syncwarp();
    } else if (warp == 1) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        constexpr uint32_t kN64 = kTypes | ((64u >> 3) << 17), kProdDesc = kTypes | (1u << 16) | ((128u >> 3) << 17);
        for (int u = (int)blockIdx.x; u < g.units && ok; u += (int)gridDim.x) {
            const int seq = u / p.H;
            const int2 rows = seq_rows(p.pr, seq);
            const bool fresh0 = seq_resume(p.pr, seq) < 0;
            for (int t = rows.x; t < rows.y && ok; t += kQ, ++n) {
                const int b = n & 1, valid = min(kQ, rows.y - t);
                const bool live = !(fresh0 && t == rows.x);                      // S is not zero
                const uint32_t base = sbase + b * kStage;
                const uint64_t dk = swizzled_desc(base + kKOff, 16u, 1024u), dq = swizzled_desc(base + kQOff, 16u, 1024u);
                const uint64_t dt = swizzled_desc(base + kWOff + kTOff, 16u, 1024u), dp = swizzled_desc(base + kWOff + kPOff, 16u, 1024u);
                const uint64_t dkt = swizzled_desc(base + kKOff, kPart, 1024u);
                ok = warp_wait(bar + bFull + b, (n / 2) & 1);
                if (!ok) break;
                if (valid < kQ) {                        // rows of the next sequence are no part of this one
                    for (int r = valid + lane / 8; r < kQ; r += 4) {
                        unsigned char* k = smem + b * kStage + kKOff + r * 128 + lane % 8 * 16;
                        *reinterpret_cast<uint4*>(k) = *reinterpret_cast<uint4*>(k + kPart) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    proxy_fence();
                    __syncwarp();
                }
                if (live) {                              // K S^T: 32 channels at a time, three parts
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int q = i / 2 + i % 2 * 2;                         // quarters 0, 2, 1, 3
                        ok = ok && warp_wait(bar + bS + q, m & 1);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll
                        for (int e = 0; e < 6; ++e) {                            // (two steps of 16 channels, three parts)
                            const int step = e & 1, part = e >> 1;
                            if (elect())
                                mma_ts(tmem + cX, tmem + cS + (q / 2) * 96 + part * 32 + (q & 1) * 16 + step * 8,
                                       dk + (uint32_t)(q / 2) * (kPart >> 4) + (uint32_t)((q & 1) * 2 + step) * 2u, kN64, i > 0 || e > 0);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (elect()) tc_commit(bar + bX);
                    __syncwarp();
                }
                // (T - I) X, 16 tokens at a time
                ok = warp_wait(bar + bRead, n & 1);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int q = i / 2 + i % 2 * 2;
                    ok = ok && warp_wait(bar + bXP + q, n & 1);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t desc = kTypes | ((uint32_t)((64 - 16 * q) >> 3) << 17);
                    const uint64_t rows_q = dt + (uint32_t)q * (2048u >> 4) + (uint32_t)q * 2u;
#pragma unroll
                    for (int e = 0; e < 6; ++e) {                                // parts (T, X): 00 01 10 11 02 20
                        const int tp = e == 2 || e == 3 ? 1 : e == 5 ? 2 : 0, xp = e == 1 || e == 3 ? 1 : e == 4 ? 2 : 0;
                        if (elect()) mma_ts(tmem + cX + 16 * q, tmem + cW + xp * 32 + q * 8, rows_q + (uint32_t)tp * (kPart >> 4), desc, i > 0 || e > 0);
                    }
                    __syncwarp();
                }
                if (!ok) break;
                if (elect()) tc_commit(bar + bU);
                __syncwarp();
                ok = n < 1 || warp_wait(bar + bYFree, (n - 1) & 1);
                if (!ok) break;
                tc_fence_after();
                if (live) {                              // Q S^T in two parts
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int part = i >> 3, k = i & 7;
                        if (elect())
                            mma_ts(tmem + cY, tmem + cS + (k / 4) * 96 + part * 32 + (k & 3) * 8, dq + (uint32_t)(k / 4) * (kPart >> 4) + (uint32_t)(k & 3) * 2u,
                                   kN64, i > 0);
                    }
                    if (elect()) tc_commit(bar + bAsk);
                    __syncwarp();
                    ok = warp_wait(bar + bAsk, m & 1);   // (W K takes the place of S)
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {            // W K, 16 tokens at a time
                    const int q = i / 2 + i % 2 * 2;
                    ok = ok && warp_wait(bar + bWP + q, n & 1);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int e = 0; e < 3; ++e)
                        if (elect()) mma_ts(tmem + cS, tmem + cW + e * 32 + q * 8, dkt + (uint32_t)q * 128u, kProdDesc, i > 0 || e > 0);
                    __syncwarp();
                }
                if (!ok) break;
                if (elect()) tc_commit(bar + bProd);
                __syncwarp();
                if (live) {
                    ok = warp_wait(bar + bScaled, m & 1);
                    ++m;
                    if (!ok) break;
                    tc_fence_after();
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {            // U P
                    const uint32_t desc = kTypes | ((uint32_t)((64 - 16 * q) >> 3) << 17);
                    const uint64_t rows_q = dp + (uint32_t)q * (2048u >> 4) + (uint32_t)q * 2u;
#pragma unroll
                    for (int e = 0; e < 3; ++e)                                  // parts (P, U): 00 01 10
                        if (elect())
                            mma_ts(tmem + cY + 16 * q, tmem + cU + (e == 1) * 32 + q * 8, rows_q + (uint32_t)(e == 2) * (kPart >> 4), desc, live || q > 0 || e > 0);
                }
                if (elect()) {
                    tc_commit(bar + bY);
                    tc_commit(bar + bEmpty + b);
                }
                __syncwarp();
            }
        }
        if (!ok && lane == 0) record_fault(p.status, kFaultScanWait, 13);
        __syncwarp();
    } else if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    } else {
        // (384 threads start with 168 registers: 128 x 56 + 256 x 224 of 64512)
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const int quad = warp & 3, half = (warp - 4) >> 2, col = quad * 32 + lane;       // value column; half of the channels and tokens
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
        uint64_t S[32];                                 // channels 64 half ..
        auto arrive = [&](int i) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_one(bar + i);
        };
        // S as an operand: 16 columns of a part for 32 channels
        auto give_state = [&]() {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t a[3][8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) three_parts(S[q * 16 + c * 8 + i], a[0][i], a[1][i], a[2][i]);
#pragma unroll
                    for (int e = 0; e < 3; ++e) tmem_st8u(lanes + cS + half * 96 + e * 32 + q * 16 + c * 8, a[e]);
                }
                tmem_st_wait();
                arrive(bS + half * 2 + q);
            }
        };
        // Y of a chunk, behind the next one's X: where it goes, how many of this half's tokens there are, and from which on they are not finite
        __nv_bfloat16* y_to = nullptr;
        int y_tokens = 0, y_bad = 0, y_n = 0;
        auto write_y = [&]() {
            ok = warp_wait(bar + bY, y_n & 1);
            if (!ok) return;
            tc_fence_after();
            uint32_t d[32];
            tmem_ld32_async(lanes + cY + half * 32, d);
            tmem_ld_wait();
            arrive(bYFree);
            __nv_bfloat16* to = y_to;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                if (i < y_tokens) *to = __float2bfloat16_rn(i >= y_bad ? __int_as_float(0x7fffffff) : __uint_as_float(d[i]));
                to += p.out_stride;
            }
        };
        for (int u = (int)blockIdx.x; u < g.units && ok; u += (int)gridDim.x) {
            const int head = u % p.H, seq = u / p.H;
            const int2 rows = seq_rows(p.pr, seq);
            const int src = seq_resume(p.pr, seq), dst = seq_slot(p.pr, seq);
            const size_t at = (size_t)head * 128 * 128 + (size_t)half * 64 * 128 + col;
            if (src >= 0) {
                const float* from = p.state + (size_t)src * p.H * 128 * 128 + at;
#pragma unroll
                for (int i = 0; i < 32; ++i) S[i] = pack2(from[2 * i * 128], from[(2 * i + 1) * 128]);
                if (rows.x < rows.y) give_state();
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) S[i] = 0ull;
            }
            for (int t = rows.x; t < rows.y; t += kQ, ++n) {
                const int b = n & 1, valid = min(kQ, rows.y - t);
                const bool live = src >= 0 || t > rows.x;
                const float* gate = reinterpret_cast<const float*>(smem + b * kStage + kWOff + kGOff);
                ok = warp_wait(bar + bFull + b, (n / 2) & 1);
                if (!ok) break;
                // X of this half's tokens
                uint64_t X[16];
                {
                    const unsigned char* v = smem + b * kStage + kVOff + (col >> 6) * kPart + half * 32 * 128 + (col & 7) * 2;
                    const int cv = (col & 63) >> 3;
                    const ulonglong2* be = reinterpret_cast<const ulonglong2*>(gate + kBeta + half * 32);
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        float f[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int s = 2 * i + e;
                            const uint32_t w = *reinterpret_cast<const unsigned short*>(v + s * 128 + ((cv ^ (s & 7)) * 16));
                            f[e] = half * 32 + s < valid ? __uint_as_float(w << 16) : 0.f;
                        }
                        const ulonglong2 bb = be[i / 2];
                        X[i] = mul2(bb.x, pack2(f[0], f[1]));
                        X[i + 1] = mul2(bb.y, pack2(f[2], f[3]));
                    }
                }
                if (live) {
                    ok = warp_wait(bar + bX, m & 1);
                    if (!ok) break;
                    tc_fence_after();
                }
                uint32_t d[32];
                if (live) {
                    tmem_ld32_async(lanes + cX + half * 32, d);
                    tmem_ld_wait();
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) d[i] = 0u;
                }
                arrive(bRead);
                uint64_t odd = 0ull;
                {
                    const ulonglong2* rd = reinterpret_cast<const ulonglong2*>(gate + kRead + half * 32);
                    const uint64_t minus = pack2(-1.f, -1.f);
                    const int left = valid - half * 32;
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const ulonglong2 r = rd[i / 2];
                        // (rows behind the sequence: their scales are zeros, but what the products left of them may be anything)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (2 * i + e >= left) d[2 * i + e] = 0u;
                        X[i] = fma2(mul2(r.x, minus), pack2(__uint_as_float(d[2 * i]), __uint_as_float(d[2 * i + 1])), X[i]);
                        X[i + 1] = fma2(mul2(r.y, minus), pack2(__uint_as_float(d[2 * i + 2]), __uint_as_float(d[2 * i + 3])), X[i + 1]);
                        odd = fma2(X[i], 0ull, odd);
                        odd = fma2(X[i + 1], 0ull, odd);
                    }
                }
                {
                    float o0, o1;
                    unpack2(odd, o0, o1);
                    if (!(o0 + o1 == 0.f)) {
                        int first = kQ;
#pragma unroll
                        for (int i = 15; i >= 0; --i) {
                            float a, c;
                            unpack2(X[i], a, c);
                            if (!(fabsf(c) <= 3.4028235e38f)) first = half * 32 + 2 * i + 1;
                            if (!(fabsf(a) <= 3.4028235e38f)) first = half * 32 + 2 * i;
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float a, c;
                            unpack2(X[i], a, c);
                            X[i] = pack2(half * 32 + 2 * i >= first ? 0.f : a, half * 32 + 2 * i + 1 >= first ? 0.f : c);
                        }
                        atomicMax(marks + col, mark_of(n + 1, first));
                    }
                }
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    uint32_t a[3][8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) three_parts(X[q * 8 + i], a[0][i], a[1][i], a[2][i]);
#pragma unroll
                    for (int e = 0; e < 3; ++e) tmem_st8u(lanes + cW + e * 32 + half * 16 + q * 8, a[e]);
                    tmem_st_wait();
                    arrive(bXP + half * 2 + q);
                }
                if (y_to != nullptr) {
                    write_y();
                    if (!ok) break;
                }
                // U and W
                ok = warp_wait(bar + bU, n & 1);
                if (!ok) break;
                tc_fence_after();
                tmem_ld32_async(lanes + cX + half * 32, d);
                tmem_ld_wait();
                const uint32_t mark = reinterpret_cast<const volatile uint32_t*>(marks)[col];
                const bool bad = (mark >> 7) == (uint32_t)n + 1u;
                const int first = bad ? kQ - (int)(mark & 127u) - half * 32 : kQ;
                if (bad) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float a, c;
                        unpack2(X[i], a, c);
                        if (2 * i >= first) { a = 0.f; d[2 * i] = 0u; }
                        if (2 * i + 1 >= first) { c = 0.f; d[2 * i + 1] = 0u; }
                        X[i] = pack2(a, c);
                    }
                }
                {
                    const ulonglong2* put = reinterpret_cast<const ulonglong2*>(gate + kPut + half * 32);
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        uint32_t a[3][8], w[2][8];
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            const int j = q * 8 + i;
                            const ulonglong2 f = put[j / 2];
                            const uint64_t u0 = add2(X[j], pack2(__uint_as_float(d[2 * j]), __uint_as_float(d[2 * j + 1])));
                            const uint64_t u1 = add2(X[j + 1], pack2(__uint_as_float(d[2 * j + 2]), __uint_as_float(d[2 * j + 3])));
                            three_parts(mul2(f.x, u0), a[0][i], a[1][i], a[2][i]);
                            three_parts(mul2(f.y, u1), a[0][i + 1], a[1][i + 1], a[2][i + 1]);
                            two_parts(u0, w[0][i], w[1][i]);
                            two_parts(u1, w[0][i + 1], w[1][i + 1]);
                        }
#pragma unroll
                        for (int e = 0; e < 3; ++e) tmem_st8u(lanes + cW + e * 32 + half * 16 + q * 8, a[e]);
#pragma unroll
                        for (int e = 0; e < 2; ++e) tmem_st8u(lanes + cU + e * 32 + half * 16 + q * 8, w[e]);
                        tmem_st_wait();
                        arrive(bWP + half * 2 + q);
                    }
                }
                const float keep = gate[kKeep];
                if (live) {                              // Q S^T is there: its tokens' factors
                    ok = warp_wait(bar + bAsk, m & 1);
                    ++m;
                    if (!ok) break;
                    tc_fence_after();
                    tmem_ld32_async(lanes + cY + half * 32, d);
                    tmem_ld_wait();
                    const float4* ask = reinterpret_cast<const float4*>(gate + kAsk + half * 32);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float4 f = ask[2 * i], h = ask[2 * i + 1];
                        const float w[8] = {f.x, f.y, f.z, f.w, h.x, h.y, h.z, h.w};
                        uint32_t r[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) r[e] = __float_as_uint(w[e] * __uint_as_float(d[8 * i + e]));
                        tmem_st8u(lanes + cY + half * 32 + 8 * i, r);
                    }
                    tmem_st_wait();
                    arrive(bScaled);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive_one(bar + bEmpty + b);
                y_to = static_cast<__nv_bfloat16*>(p.out) + (long long)(t + half * 32) * p.out_stride + (long long)head * 128 + col;
                y_tokens = valid - half * 32;
                y_bad = first;
                y_n = n;
                // S
                ok = warp_wait(bar + bProd, n & 1);
                if (!ok) break;
                tc_fence_after();
                const uint64_t keep2 = pack2(keep, keep);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    tmem_ld32_async(lanes + cS + half * 64 + c * 32, d);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        S[c * 16 + i] = fma2(keep2, S[c * 16 + i], pack2(__uint_as_float(d[2 * i]), __uint_as_float(d[2 * i + 1])));
                }
                if (bad) {
                    const float nan = __int_as_float(0x7fffffff);
#pragma unroll
                    for (int i = 0; i < 32; ++i) S[i] = pack2(nan, nan);
                }
                // (both halves of W K have been read: the parts take their place)
                tc_fence_before();
                asm volatile("bar.sync %0, 64;" ::"r"(quad + 1) : "memory");
                tc_fence_after();
                if (t + kQ < rows.y) give_state();
            }
            if (!ok) break;
            if (dst >= 0) {
                float* to = p.state + (size_t)dst * p.H * 128 * 128 + at;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    float a, c;
                    unpack2(S[i], a, c);
                    to[2 * i * 128] = a;
                    to[(2 * i + 1) * 128] = c;
                }
            }
        }
        if (ok && y_to != nullptr) write_y();
        if (!ok && lane == 0) record_fault(p.status, kFaultScanWait, 14);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_free<512>(tmem);
}

}  // namespace

size_t delta_tc_work_bytes(const sketchssm_config& c, long long sequences, long long tokens) {
    if (c.kind != SKETCHSSM_GDN || c.io_dtype != SKETCHSSM_BF16 || c.dk != 128 || c.dv != 128 || sequences == 0 || tokens == 0) return 0;
    return (size_t)(tokens / kQ + sequences) * c.heads * kBlock;
}

int launch_delta_scan_tc(Ctx* ctx, const DeltaParams& p, bool bf16, cudaStream_t stream) {
    if (!bf16 || !p.out_bf16 || p.K != 128 || p.V != 128 || p.pr.T == 0 || ctx->cfg.kind != SKETCHSSM_GDN) return SKETCHSSM_UNSUPPORTED_SHAPE;
    DeltaArgs g;
    g.p = p;
    const long long units = (long long)p.pr.N * p.H, chunks = (long long)p.pr.T / kQ + p.pr.N;
    const long long preps = chunks * p.G * ((p.H / p.G + 1) / 2);
    if (units > (1 << 30) || preps > 0x7fffffffll) return SKETCHSSM_UNSUPPORTED_SHAPE;
    g.units = (int)units;
    if (!make_map(&g.tq, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.q, (uint64_t)p.G * 128, (uint64_t)p.pr.T, (uint64_t)p.q_stride * 2, kQ) ||
        !make_map(&g.tk, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.k, (uint64_t)p.G * 128, (uint64_t)p.pr.T, (uint64_t)p.k_stride * 2, kQ) ||
        !make_map(&g.tv, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.v, (uint64_t)p.H * 128, (uint64_t)p.pr.T, (uint64_t)p.v_stride * 2, kQ)) {
        ctx->last_cuda_error = cudaErrorInvalidValue;
        return SKETCHSSM_CUDA_ERROR;
    }
    cudaError_t e = unlock_smem(ctx, delta_prep_kernel);
    if (e == cudaSuccess) e = unlock_smem(ctx, delta_scan_tc_kernel);
    if (e != cudaSuccess) { ctx->last_cuda_error = e; return SKETCHSSM_CUDA_ERROR; }
    const int rc = launch_layer<DeltaArgs>(ctx, delta_prep_kernel, dim3((unsigned)preps), dim3(kPrepThreads), kPrepSmem, stream, g);
    if (rc != SKETCHSSM_OK) return rc;
    const unsigned grid = (unsigned)(units < sm_count(ctx) ? units : sm_count(ctx));
    return launch_layer<DeltaArgs>(ctx, delta_scan_tc_kernel, dim3(grid), dim3(kThreads), kSmemTc, stream, g);
}

}  // namespace sketchssm
