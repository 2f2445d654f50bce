// Selective scan of packed prompts on tcgen05 + TMEM: bf16 tensors, K = 128, value columns in blocks of 64.
//
// A sequence goes through in chunks of 128 tokens.  With c_t the sum of the chunk's log2 decays up to token t, per head:
//     Y   = diag(2^c_t) Q S + P V,      P[t][s] = <q_t, k_s> beta_s 2^(c_t - c_s)  for s <= t, else 0        (outputs, + skip V)
//     S  <- 2^c_end S + K^T W,          W[t] = beta_t 2^(c_end - c_t) v_t                                   (state)
// A CTA (one per SM, persistent) takes two column blocks of one group at a time ("sets": two heads of 64 columns, or both halves of
// one of 128), which share K, Q and the products Q K^T.
//
// Precision.  Outputs are sums of fp32 accuracy, rounded once to bf16, and states are fp32.  Q K^T is exact up to the fp32 sums.  The
// state is held in fp32 registers; W goes to the tensor cores in three bf16 parts, so that a term of S is off by less than 2^-22.  P below
// its diagonal, and S as an operand of Y, go there in two parts, off by 2^-16 of a term at most, where an output's own rounding is 2^-8 of
// their sum (in one part: outputs 1.3e-3 in the square mean from those of fp32 sums, now 5e-5; one prompt of 16384 tokens of 64 heads
// 268 us then, 327 now).  The diagonal, a token's own weight beta, is no part of P: it goes with the skip, in fp32.
// Sums of log2 decays run backward for c_end - c_t, so that what is small is exact; forward sums are kept as whole numbers, which are
// exact, and a rest of up to 64 in size, so that c_t - c_s is off by less than 2^-14.7 whatever was decayed before s.
//
// What bounds it: a chunk of a pair of heads takes about 10,500 cycles, and no unit is busy throughout: the tensor cores work a quarter of
// them, HBM would need 2800, the schedulers issue in half (the one with the longest rows of P in two thirds).  Two chains of about that
// length go round: Q K^T, P, P V, Y (the next Q K^T waits for P V, as P's second parts lie in its columns), and S as an operand, Q S, W in four
// quarters, their products, S.  16384 tokens of 64 heads in one prompt: 327 us (0.86 TB/s), in 48 ragged ones: 400 to 430 us by their
// lengths (1.1 TB/s); 100 tokens 13 us.
//
// Roles: warp 3 issues the copies (TMA, 128-byte swizzle), warp 1 the products of Y (Q K^T, Q S, P V), warp 2 those of the state,
// warp 0 makes the gates of a chunk; per set four warps ("A") turn Q K^T into P in tensor memory, add the skip and store Y, and eight
// ("B") make W, hold S, hand it on as an operand and scale Q S.  They meet through mbarriers alone; every wait is bounded.
// Tensor memory: Q K^T and then P's second parts 128 columns, Y 2 x 64, state products 2 x 64, P's first parts 2 x 64.
//
// Few sequences and heads: a sequence is split into segments.  A first launch (OUTPUTS = false) leaves every segment's own state and
// decay in the scratch, a second one starts each segment from the sum of those before it.
#include "tma.cuh"

namespace sketchssm {

namespace {

using namespace tc;

constexpr int kQ = 128;                                // tokens of a chunk
constexpr uint32_t kTile = 16384u;                     // 128 rows of 128 bytes
constexpr uint32_t kKOff = 0, kQOff = 3 * kTile, kVOff = 5 * kTile, kWOff = 9 * kTile;       // K of 64 tokens in three buffers, Q in one, V in two
constexpr uint32_t kKHalf = kTile / 2;                 // 64 of the 128 columns of such a K
constexpr uint32_t kWBuf = 32768u;                     // of a set: S in two parts, or W of 32 tokens in three, twice
constexpr uint32_t kGateOff = kWOff + 2 * kWBuf;       // [2 buffers][2 sets][6][128] floats and one more: see gates
constexpr uint32_t kGateSet = 6 * kQ + 4, kGateBuf = 2 * kGateSet;
constexpr uint32_t kBarOff = kGateOff + 2 * kGateBuf * 4;
constexpr int kThreads = 896;

enum { bFullK = 0, bEmptyK = 3, bFullQ = 6, bEmptyQ = 7, bFullV = 8, bEmptyV = 10, bGate = 12, bGateFree = 14, bDot = 16, bState = 17,
       bInter = 18, bP = 19, bY = 23, bYFree = 25, bW = 26, bProd = 28, bVRead = 30, bScaled = 34, kBars = 36 };
constexpr uint32_t kMarkOff = kBarOff + kBars * 8u + 16u;       // [2 buffers][2 sets][65]: see mark_of
constexpr uint32_t kMarks = 65;
constexpr uint32_t kOwnOff = kMarkOff + 4u * kMarks * 4u;       // [2 buffers][128]: <q_t, k_t>
constexpr uint32_t kSmemTc = kOwnOff + 2u * kQ * 4u + 1024u;

// columns of tensor memory
constexpr uint32_t kDot = 0, kY = 128, kProd = 256, kP = 384;

struct ScanArgs {
    CUtensorMap tq, tk, tv;
    ScanParams p;
    int slabs, slabs_per_group, blocks_per_group;      // pairs of column blocks: all, per group; column blocks per group
    int units;
};

// One unit: a segment of a sequence for one pair of column blocks.
struct Unit {
    int t0, t1;            // rows of the segment
    int seq, seg, group;
    int block0, live1;     // first column block; whether the second set has one of its own
    int last;              // this segment ends the sequence
};

__device__ __forceinline__ Unit decode_unit(const ScanArgs& g, int u) {
    Unit x;
    const int slab = u % g.slabs, r = u / g.slabs;
    x.seg = r % g.p.segments;
    x.seq = r / g.p.segments;
    x.group = slab / g.slabs_per_group;
    const int i = slab % g.slabs_per_group * 2;
    x.block0 = x.group * g.blocks_per_group + i;
    x.live1 = i + 1 < g.blocks_per_group;
    const int2 rows = seq_rows(g.p.pr, x.seq);
    const int chunks = (rows.y - rows.x + kQ - 1) / kQ;
    const int per = max(1, (chunks + g.p.segments - 1) / g.p.segments);
    x.t0 = min(rows.y, rows.x + x.seg * per * kQ);
    x.t1 = min(rows.y, x.t0 + per * kQ);
    x.last = x.seg == (chunks > 0 ? (chunks - 1) / per : 0);
    return x;
}
// The segment has work: tokens, or (a sequence without tokens) a state to hand on.
__device__ __forceinline__ bool unit_runs(const Unit& x, bool outputs) { return outputs ? x.t1 > x.t0 || x.last : !x.last && x.t1 > x.t0; }

__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool acc) { tc_mma_bf16(d, a, b, idesc, acc ? 1u : 0u); }
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc ? 1u : 0u)
        : "memory");
}
__device__ __forceinline__ void tmem_st16u(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
        "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

__device__ __forceinline__ void tmem_st8u(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}

// The products take every value of a chunk into every row, and a zero weight times NaN or infinity is NaN: values that are not finite go
// to the products as zeros, and a column's rows from the first of them on become NaN afterwards.  A mark of chunk n holds that row; the
// largest of several is the first row of the latest chunk, so that marks need no clearing.  (The 65th: of any column.)
// Looking for them cost one long prompt 2 % (269 us, 263, with P in one part), many short ones 0.6 %.
__device__ __forceinline__ uint32_t mark_of(int n, int row) { return ((uint32_t)n << 8) + (uint32_t)(kQ - row); }

// Adds products of the eight values, two by two, to two sums: not finite if one of the values is not (or if a product overflows: then
// for nothing).  Half as many instructions as a sum for each value.
__device__ __forceinline__ void odd_values(const uint4& v, uint32_t& a, uint32_t& b) {
    asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(a) : "r"(v.x), "r"(v.y));
    asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(b) : "r"(v.z), "r"(v.w));
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
// Buffer of K's half `half` (64 tokens) of chunk n, and its barriers' parity.
__device__ __forceinline__ uint32_t k_slot(int n, int half) { return (uint32_t)(2 * n + half) % 3u; }
__device__ __forceinline__ uint32_t k_phase(int n, int half) { return ((uint32_t)(2 * n + half) / 3u) & 1u; }

template <bool OUTPUTS>
__global__ void __launch_bounds__(kThreads, 1) prompt_scan_tc_kernel(const __grid_constant__ ScanArgs g) {
    extern __shared__ unsigned char raw[];
    unsigned char* smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    float* gates = reinterpret_cast<float*>(smem + kGateOff);
    uint64_t* bar = reinterpret_cast<uint64_t*>(smem + kBarOff);
    uint32_t* slot = reinterpret_cast<uint32_t*>(bar + kBars);
    const ScanParams& p = g.p;
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int per_head = p.V / 64;                     // column blocks of a head
    if (tid == 32) { prefetch_map(&g.tq); prefetch_map(&g.tk); prefetch_map(&g.tv); }
    if (tid == 0) {
        for (int i = 0; i < kBars; ++i) {
            int n = 1;                                  // copies and commits of products arrive once
            if (i >= bEmptyK && i < bFullQ) n = OUTPUTS ? 2 : 1;                // both product warps read K
            if (i >= bEmptyV && i < bGate) n = OUTPUTS ? 8 : 16;                               // A (without outputs: B) of both sets
            if (i >= bGateFree && i < bDot) n = OUTPUTS ? 24 : 16;
            if (i == bYFree) n = 8;                                             // the warps of both sets
            if (i == bState || i == bW || i == bW + 1) n = 16;
            if (i >= bP && i < bY) n = 8;                                       // (A)
            if (i >= bVRead) n = 8;                                              // (B) of one set
            mbar_init(bar + i, n);
        }
        mbar_fence_init();
    }
    if (OUTPUTS && tid < 4 * (int)kMarks) reinterpret_cast<uint32_t*>(smem + kMarkOff)[tid] = 0u;
    if (warp == 1) tmem_alloc<512>(slot);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    grid_dep_wait();
    grid_dep_launch_dependents();
    const uint32_t tmem = *slot;
    const uint32_t sbase = smem_u32(smem);
    bool ok = true;
    int n = 0;                                          // chunks so far, over all units of the CTA

    if (warp == 3) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        if (lane == 0) {
            int nk = 0, nv = 0, nq = 0;                 // copies issued: halves of K, V, Q
            auto load_k = [&](const Unit& x, int t) {
                const uint32_t slot = (uint32_t)nk % 3u;
                ok = ok && (nk < 3 || mbar_wait_bounded(bar + bEmptyK + slot, ((uint32_t)nk / 3u - 1u) & 1u));
                if (ok) {
                    mbar_expect_tx(bar + bFullK + slot, kTile);
                    tma_load(smem + kKOff + slot * kTile, &g.tk, x.group * 128, t, bar + bFullK + slot);
                    tma_load(smem + kKOff + slot * kTile + kKHalf, &g.tk, x.group * 128 + 64, t, bar + bFullK + slot);
                    ++nk;
                }
            };
            for (int u = (int)blockIdx.x; u < g.units && ok; u += (int)gridDim.x) {
                const Unit x = decode_unit(g, u);
                if (!unit_runs(x, OUTPUTS)) continue;
                for (int t = x.t0; t < x.t1 && ok; t += kQ) {
                    load_k(x, t);
                    const int b = nv & 1;
                    ok = ok && (nv < 2 || mbar_wait_bounded(bar + bEmptyV + b, (nv / 2 - 1) & 1));
                    if (ok) {
                        mbar_expect_tx(bar + bFullV + b, 2 * kTile);
                        tma_load(smem + kVOff + b * 2 * kTile, &g.tv, x.block0 * 64, t, bar + bFullV + b);
                        tma_load(smem + kVOff + (b * 2 + 1) * kTile, &g.tv, (x.block0 + x.live1) * 64, t, bar + bFullV + b);
                        ++nv;
                    }
                    if constexpr (OUTPUTS) {
                        ok = ok && (nq < 1 || mbar_wait_bounded(bar + bEmptyQ, (nq - 1) & 1));
                        if (ok) {
                            mbar_expect_tx(bar + bFullQ, 2 * kTile);
                            tma_load(smem + kQOff, &g.tq, x.group * 128, t, bar + bFullQ);
                            tma_load(smem + kQOff + kTile, &g.tq, x.group * 128 + 64, t, bar + bFullQ);
                            ++nq;
                        }
                    }
                    load_k(x, t + 64);                  // (last: its buffer is free when half of the chunk before has gone to the state)
                }
            }
            if (!ok) record_fault(p.status, kFaultScanWait, 1);
            // Before the CTA ends the copies under way have ended (after a fault; otherwise they have been waited for), and the products'
            // last arrivals at the buffers' barriers are in.
            for (int i = max(0, nk - 3); i < nk; ++i)
                mbar_wait_bounded(bar + (ok ? bEmptyK : bFullK) + i % 3, (i / 3) & 1, ok ? 1u << 22 : 1u << 16);
            for (int i = max(0, nv - 2); i < nv && !ok; ++i) mbar_wait_bounded(bar + bFullV + (i & 1), (i / 2) & 1, 1u << 16);
            if (nq > 0) mbar_wait_bounded(bar + (ok ? bEmptyQ : bFullQ), (nq - 1) & 1, 1u << 16);
        }
        __syncwarp();
    } else if (warp == 1) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        if constexpr (OUTPUTS) {
            constexpr uint32_t kTypes = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);      // bf16 x bf16 -> fp32, 128 rows
            constexpr uint32_t kDotDesc = kTypes | ((64u >> 3) << 17), kInterDesc = kTypes | (1u << 16) | ((128u >> 3) << 17);
            constexpr uint32_t kPDesc = kTypes | (1u << 16) | ((64u >> 3) << 17);
            const uint64_t dq = swizzled_desc(sbase + kQOff, 16u, 1024u), ds = swizzled_desc(sbase + kWOff, kWBuf, 1024u);
            int m = 0;                                  // chunks with a state before them
            for (int u = (int)blockIdx.x; u < g.units && ok; u += (int)gridDim.x) {
                const Unit x = decode_unit(g, u);
                if (!unit_runs(x, true)) continue;
                const bool fresh0 = x.seg == 0 && seq_resume(p.pr, x.seq) < 0;
                for (int t = x.t0; t < x.t1; t += kQ, ++n) {
                    const int b = n & 1;
                    const bool fresh = fresh0 && t == x.t0;                     // S is zero
                    // (P of the chunk before is made and used: its Q K^T, and the second parts of P in that one's place, are needed no more)
                    ok = (n < 1 || (warp_wait(bar + bY, (n - 1) & 1) && warp_wait(bar + bY + 1, (n - 1) & 1))) && warp_wait(bar + bFullQ, n & 1);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {                      // 64 tokens of K, 64 columns
                        const uint32_t slot = k_slot(n, half);
                        ok = ok && warp_wait(bar + bFullK + slot, k_phase(n, half));
                        if (!ok) break;
                        tc_fence_after();
                        const uint64_t dk = swizzled_desc(sbase + kKOff + slot * kTile, 16u, 1024u);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const uint32_t in = (uint32_t)(i % 4) * 2u;
                            if (elect())
                                mma_ss(tmem + kDot + half * 64, dq + (uint32_t)(i / 4) * (kTile >> 4) + in, dk + (uint32_t)(i / 4) * (kKHalf >> 4) + in, kDotDesc, i > 0);
                        }
                        if (elect()) tc_commit(bar + bEmptyK + slot);
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (elect()) tc_commit(bar + bDot);
                    __syncwarp();
                    ok = n < 1 || warp_wait(bar + bYFree, (n - 1) & 1);
                    if (!fresh) {
                        ok = ok && warp_wait(bar + bState, m & 1);
                        if (!ok) break;
                        ++m;
                        tc_fence_after();
#pragma unroll
                        for (int i = 0; i < 16; ++i)                             // S in two parts
                            if (elect())
                                mma_ss(tmem + kY, dq + (uint32_t)(i % 8 / 4) * (kTile >> 4) + (uint32_t)(i % 4) * 2u,
                                       ds + (uint32_t)(i / 8) * (kTile >> 4) + (uint32_t)(i % 8) * 128u, kInterDesc, i > 0);
                        if (elect()) tc_commit(bar + bInter);
                    }
                    if (elect()) tc_commit(bar + bEmptyQ);
                    __syncwarp();
                    ok = ok && warp_wait(bar + bFullV + b, (n / 2) & 1);
                    const uint64_t dv = swizzled_desc(sbase + kVOff + b * 2 * kTile, 16u, 1024u);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {                               // 32 columns of P at a time, as they are made
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            ok = ok && (j > 0 || warp_wait(bar + bP + c, n & 1)) && (fresh || c > 0 || warp_wait(bar + bScaled + j, (m - 1) & 1));
                            if (!ok) break;
                            tc_fence_after();
                            const uint64_t v = dv + (uint32_t)j * (kTile >> 4) + (uint32_t)c * 256u;
                            if (elect()) mma_ts(tmem + kY + j * 64, tmem + kP + j * 64 + c * 16, v, kPDesc, c > 0 || !fresh);
                            if (elect()) mma_ts(tmem + kY + j * 64, tmem + kP + j * 64 + c * 16 + 8, v + 128u, kPDesc, true);
                            if (elect()) mma_ts(tmem + kY + j * 64, tmem + kDot + c * 32 + j * 16, v, kPDesc, true);
                            if (elect()) mma_ts(tmem + kY + j * 64, tmem + kDot + c * 32 + j * 16 + 8, v + 128u, kPDesc, true);
                            if (c == 3 && elect()) tc_commit(bar + bY + j);
                            __syncwarp();
                        }
                    }
                    if (!ok) break;
                }
            }
            if (!ok && lane == 0) record_fault(p.status, kFaultScanWait, 2);
        }
        __syncwarp();
    } else if (warp == 2) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        constexpr uint32_t kDesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
        const uint64_t dw = swizzled_desc(sbase + kWOff, kWBuf, 1024u);
        for (int u = (int)blockIdx.x; u < g.units && ok; u += (int)gridDim.x) {
            const Unit x = decode_unit(g, u);
            if (!unit_runs(x, OUTPUTS)) continue;
            for (int t = x.t0; t < x.t1 && ok; t += kQ, ++n) {
#pragma unroll
                for (int h = 0; h < 4; ++h) {                                   // 32 tokens at a time, both sets' columns
                    const uint32_t slot = k_slot(n, h >> 1);
                    if ((h & 1) == 0) {
                        ok = ok && warp_wait(bar + bFullK + slot, k_phase(n, h >> 1));
                        const int valid = max(0, x.t1 - t - h * 32);
                        if (ok && valid < 64) {          // rows of the next sequence are no part of this one
                            for (int r = valid + lane / 8; r < 64; r += 4) {
                                unsigned char* k = smem + kKOff + slot * kTile + r * 128 + lane % 8 * 16;
                                *reinterpret_cast<uint4*>(k) = *reinterpret_cast<uint4*>(k + kKHalf) = make_uint4(0u, 0u, 0u, 0u);
                            }
                            proxy_fence();
                            __syncwarp();
                        }
                    }
                    ok = ok && warp_wait(bar + bW + (h & 1), h >> 1);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t dk = swizzled_desc(sbase + kKOff + slot * kTile, kKHalf, 1024u);
#pragma unroll
                    for (int i = 0; i < 6; ++i)
                        if (elect())
                            mma_ss(tmem + kProd, dk + (uint32_t)((h & 1) * 2 + i % 2) * 128u, dw + (uint32_t)(h & 1) * 768u + (uint32_t)(i / 2) * 256u + (uint32_t)(i % 2) * 128u,
                                   kDesc, i > 0 || h > 0);
                    if (elect()) {
                        tc_commit(bar + bProd + (h & 1));
                        if (h & 1) tc_commit(bar + bEmptyK + slot);
                    }
                    __syncwarp();
                }
            }
        }
        if (!ok && lane == 0) record_fault(p.status, kFaultScanWait, 3);
        __syncwarp();
    } else if (warp == 0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        // gates: four neighbouring tokens a lane
        for (int u = (int)blockIdx.x; u < g.units && ok; u += (int)gridDim.x) {
            const Unit x = decode_unit(g, u);
            if (!unit_runs(x, OUTPUTS)) continue;
            const int h0 = x.block0 / per_head, h1 = (x.block0 + x.live1) / per_head;
            float a2[2], bias[2], next[2][4];
            a2[0] = p.a[h0] * 1.4426950408889634f; a2[1] = p.a[h1] * 1.4426950408889634f;
            bias[0] = p.dt_bias != nullptr ? p.dt_bias[h0] : 0.f; bias[1] = p.dt_bias != nullptr ? p.dt_bias[h1] : 0.f;
            auto fetch = [&](int t) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = t + lane * 4 + i;
                    const __nv_bfloat16* dt = static_cast<const __nv_bfloat16*>(p.dt) + (long long)r * p.dt_stride;
                    next[0][i] = r < x.t1 ? __bfloat162float(dt[h0]) : 0.f;
                    next[1][i] = r < x.t1 ? __bfloat162float(dt[h1]) : 0.f;
                }
            };
            fetch(x.t0);
            for (int t = x.t0; t < x.t1; t += kQ, ++n) {
                const int b = n & 1;
                float beta[2][4];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) beta[j][i] = t + lane * 4 + i < x.t1 ? softplus(next[j][i] + bias[j]) : 0.f;
                if (t + kQ < x.t1) fetch(t + kQ);
                ok = n < 2 || warp_wait(bar + bGateFree + b, (n / 2 - 1) & 1);
                if (!ok) break;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    // (2^-160 is zero in fp32; the bound keeps the sums finite; NaN passes it)
                    float l[4], suf[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x2 = a2[j] * beta[j][i];
                        l[i] = t + lane * 4 + i < x.t1 ? (x2 < -160.f ? -160.f : x2) : 0.f;
                    }
                    suf[3] = 0.f;
#pragma unroll
                    for (int i = 2; i >= 0; --i) suf[i] = suf[i + 1] + l[i + 1];
                    float after = suf[0] + l[0];
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const float down = __shfl_down_sync(0xffffffffu, after, o);
                        if (lane + o < 32) after += down;
                    }
                    const float all = after;             // (in lane 0: of the chunk)
                    after = __shfl_down_sync(0xffffffffu, after, 1);
                    if (lane == 31) after = 0.f;
                    float w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = beta[j][i] * exp2f(after + suf[i]);
                    float* set = gates + b * kGateBuf + j * kGateSet;
                    float4* to = reinterpret_cast<float4*>(set) + lane;
                    to[0] = make_float4(w[0], w[1], w[2], w[3]);                  // beta 2^(c at the chunk's end - c)
                    if (lane == 0) set[6 * kQ] = exp2f(all);                     // 2^(c at the chunk's end)
                    if constexpr (OUTPUTS) {
                        // Forward sums of whole numbers and of what is left, at most a half each: the first are exact, the second at most 64
                        // in size, so that a difference of two sums is that of the tokens between them, whatever stands before them.
                        float whole[4], part[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float r = rintf(l[i]);
                            whole[i] = i > 0 ? whole[i - 1] + r : r;
                            part[i] = i > 0 ? part[i - 1] + (l[i] - r) : l[i] - r;
                        }
                        float whole0 = whole[3], part0 = part[3];
#pragma unroll
                        for (int o = 1; o < 32; o <<= 1) {
                            const float up = __shfl_up_sync(0xffffffffu, whole0, o), up2 = __shfl_up_sync(0xffffffffu, part0, o);
                            if (lane >= o) { whole0 += up; part0 += up2; }
                        }
                        whole0 = __shfl_up_sync(0xffffffffu, whole0, 1);
                        part0 = __shfl_up_sync(0xffffffffu, part0, 1);
                        if (lane == 0) whole0 = part0 = 0.f;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            whole[i] += whole0;
                            part[i] += part0;
                        }
                        const float end = __shfl_sync(0xffffffffu, whole[3], lane | 7), end2 = __shfl_sync(0xffffffffu, part[3], lane | 7);
                        float e[4], f[4], own[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            e[i] = exp2f(whole[i] + part[i]);
                            f[i] = beta[j][i] * ex2((end - whole[i]) + (end2 - part[i]));
                            own[i] = beta[j][i] + (l[i] - l[i]);                 // (NaN where the decay is: it would reach a state of zeros too)
                        }
                        to[32] = make_float4(e[0], e[1], e[2], e[3]);             // 2^c
                        to[64] = make_float4(whole[0], whole[1], whole[2], whole[3]);     // c, whole numbers
                        to[96] = make_float4(part[0], part[1], part[2], part[3]);         // c, the rest
                        to[128] = make_float4(f[0], f[1], f[2], f[3]);            // beta 2^(c at the end of the 32 tokens - c)
                        to[160] = make_float4(own[0], own[1], own[2], own[3]);    // beta
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive_one(bar + bGate + b);
            }
        }
        if (!ok && lane == 0) record_fault(p.status, kFaultScanWait, 4);
    } else if (warp < 12) {
        if constexpr (OUTPUTS) {
            // A: token row `row` of set j
            asm volatile("setmaxnreg.inc.sync.aligned.u32 96;");
            const int j = (warp - 4) >> 2, quad = warp & 3, row = quad * 32 + lane;
            const uint32_t lanes = (uint32_t)(quad * 32) << 16;
            const uint32_t tp = tmem + lanes + kP, td = tmem + lanes + kDot, ty = tmem + lanes + kY + j * 64;
            {
                uint32_t z[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) z[i] = 0u;
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_st16u(tp + j * 64 + c * 16, z);  // above the diagonal P stays zero
                tmem_st_wait();
            }
            for (int u = (int)blockIdx.x; u < g.units && ok; u += (int)gridDim.x) {
                const Unit x = decode_unit(g, u);
                if (!unit_runs(x, true)) continue;
                const int block = x.block0 + (j ? x.live1 : 0), head = block / per_head;
                const bool live = j == 0 || x.live1;
                const float skip = p.skip != nullptr ? p.skip[head] : 0.f;
                for (int t = x.t0; t < x.t1; t += kQ, ++n) {
                    const int b = n & 1, valid = min(kQ, x.t1 - t);
                    const float* gt = gates + b * kGateBuf + j * kGateSet;
                    unsigned char* v = smem + kVOff + (b * 2 + j) * kTile;
                    unsigned char* mine = v + row * 128;
                    ok = warp_wait(bar + bFullV + b, (n / 2) & 1);
                    if (ok && row >= valid) {                                    // rows of the next sequence are no part of this one
#pragma unroll
                        for (int i = 0; i < 8; ++i) reinterpret_cast<uint4*>(mine)[i] = make_uint4(0u, 0u, 0u, 0u);
                    }
                    if (valid < kQ) proxy_fence();
                    if (!ok) break;
                    uint32_t odd = 0u;
                    {
                        uint32_t a = 0u;
#pragma unroll
                        for (int i = 0; i < 8; ++i) odd_values(*reinterpret_cast<const uint4*>(mine + ((i ^ (row & 7)) * 16)), odd, a);
                        asm("{ .reg .b32 z; mov.b32 z, 0; fma.rn.bf16x2 %0, %0, z, z; fma.rn.bf16x2 %0, %1, z, %0; }" : "+r"(odd) : "r"(a));
                    }
                    const bool odd_row = (odd & 0x7fff7fffu) != 0u;
                    ok = warp_wait(bar + bGate + b, (n / 2) & 1) && warp_wait(bar + bDot, n & 1);
                    if (!ok) break;
                    tc_fence_after();
                    uint32_t* marks = reinterpret_cast<uint32_t*>(smem + kMarkOff) + (b * 2 + j) * kMarks;
                    if (__any_sync(0xffffffffu, odd_row)) {
                        ok = warp_wait(bar + bVRead + j * 2 + b, (n / 2) & 1);       // (the state takes the values as they are)
                        if (!ok) break;
                        if (odd_row) {
                            atomicMax(marks + 64, mark_of(n, row));
#pragma unroll 1
                            for (int e = 0; e < 64; ++e) {
                                unsigned short* at = reinterpret_cast<unsigned short*>(mine + (((e >> 3) ^ (row & 7)) * 16)) + (e & 7);
                                if ((*at & 0x7f80u) == 0x7f80u) {
                                    *at = 0;
                                    atomicMax(marks + e, mark_of(n, row));
                                }
                            }
                        }
                        proxy_fence();
                    }
                    // P: below the diagonal's 32 x 32 blocks its weight is 2^(c_t - c at the end of the columns' 32) times a factor of
                    // the column, both at most 1 (but for beta); in them it is one exponential an element.  A block is one warp's, for both
                    // sets (set 0's warps take those below the diagonal, set 1's those on it), so that the second parts can take the place of
                    // the Q K^T that they are made of, 16 columns a set.
                    auto made = [&](int c0, int c1) {    // this warp's part in blocks c0 .. c1 - 1, and its row of V, are there
                        tmem_st_wait();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0)
                            for (int c = c0; c < c1; ++c) mbar_arrive_one(bar + bP + c);
                    };
                    const float beta = gt[5 * kQ + row];
                    const float* g2 = gates + b * kGateBuf;
                    uint32_t d[32], f[8], f2[8];
                    if (j == 0) {
#pragma unroll 1
                        for (int c = quad + 1; c < 4; ++c) {
                            uint32_t z[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) z[i] = 0u;
                            tmem_st16u(td + c * 32, z);          // (the second parts above the diagonal)
                            tmem_st16u(td + c * 32 + 16, z);
                        }
                        made(quad, 4);
                        if (quad > 0) tmem_ld32_async(td, d);
#pragma unroll 1
                        for (int c = 0; c < quad; ++c) {
                            tmem_ld_wait();
#pragma unroll
                            for (int q = 0; q < 2; ++q) {                        // sets
                                const float* g1 = g2 + q * kGateSet;
                                const float r = ex2((g1[2 * kQ + row] - g1[2 * kQ + c * 32 + 31]) + (g1[3 * kQ + row] - g1[3 * kQ + c * 32 + 31]));
                                const uint64_t r2 = pack2(r, r);
                                const ulonglong2* f4 = reinterpret_cast<const ulonglong2*>(g1 + 4 * kQ + c * 32);
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
#pragma unroll
                                    for (int i = 0; i < 4; ++i) {
                                        const ulonglong2 w = f4[4 * h + i];
                                        const uint32_t* u = d + 16 * h + 4 * i;
                                        two_parts(mul2(pack2(__uint_as_float(u[0]), __uint_as_float(u[1])), mul2(r2, w.x)), f[2 * i], f2[2 * i]);
                                        two_parts(mul2(pack2(__uint_as_float(u[2]), __uint_as_float(u[3])), mul2(r2, w.y)), f[2 * i + 1], f2[2 * i + 1]);
                                    }
                                    tmem_st8u(tp + q * 64 + c * 16 + h * 8, f);
                                    tmem_st8u(td + c * 32 + q * 16 + h * 8, f2);
                                }
                            }
                            if (c + 1 < quad) tmem_ld32_async(td + (c + 1) * 32, d);
                            made(c, c + 1);
                        }
                    } else {
                        tmem_ld32_async(td + quad * 32, d);
                        made(0, quad);
                        made(quad + 1, 4);
                        tmem_ld_wait();
                        {
                            uint32_t o[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = (lane & 16) ? d[i + 16] : d[i];
#pragma unroll
                            for (int s = 8; s > 0; s >>= 1) {
#pragma unroll
                                for (int i = 0; i < s; ++i) o[i] = (lane & s) ? o[i + s] : o[i];
                            }
                            reinterpret_cast<uint32_t*>(smem + kOwnOff)[b * kQ + row] = o[0];
                        }
                        const uint64_t minus = pack2(-1.f, -1.f);
#pragma unroll
                        for (int q = 0; q < 2; ++q) {                            // sets
                            const float* g1 = g2 + q * kGateSet + 2 * kQ;
                            const uint64_t ct = pack2(g1[row], g1[row]), part = pack2(g1[kQ + row], g1[kQ + row]);
                            const ulonglong2* c4 = reinterpret_cast<const ulonglong2*>(g1 + quad * 32);
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const ulonglong2 a = c4[4 * h + i], a2 = c4[32 + 4 * h + i], bt = c4[96 + 4 * h + i];
                                    const uint32_t* u = d + 16 * h + 4 * i;
                                    float x0, x1, x2, x3;
                                    unpack2(add2(fma2(a.x, minus, ct), fma2(a2.x, minus, part)), x0, x1);
                                    unpack2(add2(fma2(a.y, minus, ct), fma2(a2.y, minus, part)), x2, x3);
                                    unpack2(mul2(mul2(pack2(__uint_as_float(u[0]), __uint_as_float(u[1])), bt.x), pack2(ex2(x0), ex2(x1))), x0, x1);
                                    unpack2(mul2(mul2(pack2(__uint_as_float(u[2]), __uint_as_float(u[3])), bt.y), pack2(ex2(x2), ex2(x3))), x2, x3);
                                    const int e = 16 * h + 4 * i;        // column e of the 32 is there up to the row before `lane`
                                    two_parts(pack2(lane > e ? x0 : 0.f, lane > e + 1 ? x1 : 0.f), f[2 * i], f2[2 * i]);
                                    two_parts(pack2(lane > e + 2 ? x2 : 0.f, lane > e + 3 ? x3 : 0.f), f[2 * i + 1], f2[2 * i + 1]);
                                }
                                tmem_st8u(tp + q * 64 + quad * 16 + h * 8, f);
                                tmem_st8u(td + quad * 32 + q * 16 + h * 8, f2);
                            }
                        }
                        made(quad, quad + 1);
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive_one(bar + bGateFree + b);
                    // Y: what the products left, and the skip; v's row becomes y's, then the warp stores its rows
                    ok = ok && warp_wait(bar + bY + j, n & 1) && warp_wait(bar + bVRead + j * 2 + b, (n / 2) & 1);
                    if (!ok) break;
                    tc_fence_after();
                    uint32_t o[2][32];
                    tmem_ld32_async(ty, o[0]);
                    tmem_ld32_async(ty + 32, o[1]);
                    tmem_ld_wait();
                    tc_fence_before();
                    __syncwarp();
                    const float own = reinterpret_cast<const volatile float*>(smem + kOwnOff)[b * kQ + row] * beta;
                    __syncwarp();
                    if (lane == 0) mbar_arrive_one(bar + bYFree);
                    const bool nan_here = reinterpret_cast<const volatile uint32_t*>(marks)[64] >= mark_of(n, row);
                    const uint64_t skip2 = pack2(skip + own, skip + own);
#pragma unroll
                    for (int c0 = 0; c0 < 8; c0 += 4) {
                        uint4 u[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) u[c] = *reinterpret_cast<const uint4*>(mine + (((c0 + c) ^ (row & 7)) * 16));
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t w[4] = {u[c].x, u[c].y, u[c].z, u[c].w};
                            uint32_t z[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int e = (c0 + c) % 4 * 8 + 2 * i;
                                float lo, hi;
                                unpack2(fma2(skip2, pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)),
                                             pack2(__uint_as_float(o[(c0 + c) / 4][e]), __uint_as_float(o[(c0 + c) / 4][e + 1]))), lo, hi);
                                z[i] = bf16x2(lo, hi);
                            }
                            *reinterpret_cast<uint4*>(mine + (((c0 + c) ^ (row & 7)) * 16)) = make_uint4(z[0], z[1], z[2], z[3]);
                        }
                    }
                    if (nan_here) {
#pragma unroll 1
                        for (int e = 0; e < 64; ++e)
                            if (reinterpret_cast<const volatile uint32_t*>(marks)[e] >= mark_of(n, row))
                                reinterpret_cast<unsigned short*>(mine + (((e >> 3) ^ (row & 7)) * 16))[e & 7] = 0x7fff;
                    }
                    __syncwarp();
                    // a warp's 32 rows of 128 bytes, eight lanes a row; the buffer is free before the stores are made
                    uint4 y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int r = i * 4 + lane / 8;
                        y[i] = *reinterpret_cast<const uint4*>(v + quad * 4096 + r * 128 + (((lane % 8) ^ (r & 7)) * 16));
                    }
                    proxy_fence();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_one(bar + bEmptyV + b);
                    if (live) {
                        unsigned char* out = static_cast<unsigned char*>(p.out) +
                                             ((long long)(t + quad * 32 + lane / 8) * p.out_stride + block * 64 + lane % 8 * 8) * 2;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            if (i * 4 + lane / 8 < valid - quad * 32) *reinterpret_cast<uint4*>(out) = y[i];
                            out += p.out_stride * 8;
                        }
                    }
                }
            }
            if (!ok && lane == 0) record_fault(p.status, kFaultScanWait, 5);
        }
    } else {
        // B: state row `row` of set j (896 threads start with 72 registers: 128 x 48 + 256 x 96 + 512 x 64 of 64512)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        const int j = (warp - 12) >> 3, quad = warp & 3, row = quad * 32 + lane, bt = (tid - 384) & 255, half = bt >> 7;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        unsigned char* buf = smem + kWOff + j * kWBuf;
        uint64_t S[16];                                 // pairs of columns: half `half` of the 64
        int m = 0;                                      // chunks with a state before them
        for (int u = (int)blockIdx.x; u < g.units && ok; u += (int)gridDim.x) {
            const Unit x = decode_unit(g, u);
            if (!unit_runs(x, OUTPUTS)) continue;
            const int block = x.block0 + (j ? x.live1 : 0);
            const bool live = j == 0 || x.live1;
            const int src = seq_resume(p.pr, x.seq);
            // The block's row of this thread in a state; and in the scratch: per sequence `segments` states (that before segment 0,
            // those left by segments 0, 1, ..) and behind them as many decays a head.  (Worked out where they are used, from a
            // number that the compiler cannot see through: kept over the chunks they cost the registers of the state.)
            auto at = [&](int row0) {
                int k = block;
                asm volatile("" : "+r"(k));
                return ((size_t)row0 * p.H + k / per_head) * 128 * p.V + (size_t)row * p.V + (k % per_head) * 64 + half * 32;
            };
            auto decay = [&](int i) {
                int k = block;
                asm volatile("" : "+r"(k));
                return p.work + (size_t)p.pr.N * p.segments * p.H * 128 * p.V + ((size_t)x.seq * p.segments + i) * p.H + k / per_head;
            };
            // A row is 256 bytes of a state, all of it asked for before the first use: a round trip a state.
            auto load = [&](const float* from) {
                const ulonglong2* f = reinterpret_cast<const ulonglong2*>(from);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const ulonglong2 v = f[i];
                    S[2 * i] = v.x;
                    S[2 * i + 1] = v.y;
                }
            };
            auto add = [&](const float* from, float keep) {                      // S <- keep S + a state
                const ulonglong2* f = reinterpret_cast<const ulonglong2*>(from);
                const uint64_t keep2 = pack2(keep, keep);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const ulonglong2 v = f[i];
                    S[2 * i] = fma2(keep2, S[2 * i], v.x);
                    S[2 * i + 1] = fma2(keep2, S[2 * i + 1], v.y);
                }
            };
            auto store = [&](float* to) {
#pragma unroll
                for (int i = 0; i < 8; ++i) reinterpret_cast<ulonglong2*>(to)[i] = make_ulonglong2(S[2 * i], S[2 * i + 1]);
            };
#pragma unroll
            for (int i = 0; i < 16; ++i) S[i] = 0ull;
            if (x.seg == 0) {
                // (a later segment's CTA may have written the entry already: the first launch kept a copy)
                if (src >= 0) load(OUTPUTS && !x.last ? p.work + at(x.seq * p.segments) : p.state + at(src));
                if (!OUTPUTS && live) store(p.work + at(x.seq * p.segments));
            } else if (OUTPUTS) {
                load(p.work + at(x.seq * p.segments + 1));
                for (int i = 2; i <= x.seg; ++i) add(p.work + at(x.seq * p.segments + i), *decay(i));
            }
            const bool fresh0 = x.seg == 0 && src < 0;
            float total = 1.f;
            for (int t = x.t0; t < x.t1; t += kQ, ++n) {
                const int b = n & 1, valid = min(kQ, x.t1 - t);
                const bool fresh = fresh0 && t == x.t0;
                if (OUTPUTS && !fresh) {                 // S as an operand: row n of 64 columns
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t hi[4], lo[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) two_parts(S[c * 4 + i], hi[i], lo[i]);
                        unsigned char* to = buf + row * 128 + (((half * 4 + c) ^ (row & 7)) * 16);
                        *reinterpret_cast<uint4*>(to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                        *reinterpret_cast<uint4*>(to + kTile) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                    }
                    proxy_fence();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_one(bar + bState);
                }
                ok = warp_wait(bar + bGate + b, (n / 2) & 1) && warp_wait(bar + bFullV + b, (n / 2) & 1);
                if (!ok) break;
                if (OUTPUTS && !fresh) {                 // Q S is there (and the buffer's S has been read): its rows times 2^c
                    ok = warp_wait(bar + bInter, m & 1);
                    ++m;
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t ty = tmem + lanes + kY + j * 64 + half * 32;
                    const float ec = gates[b * kGateBuf + j * kGateSet + kQ + row];
                    const uint64_t ec2 = pack2(ec, ec);
                    uint32_t d[16];
#pragma unroll 1
                    for (int c = 0; c < 2; ++c) {
                        tmem_ld16_async(ty + c * 16, d);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const uint64_t y = mul2(ec2, pack2(__uint_as_float(d[2 * i]), __uint_as_float(d[2 * i + 1])));
                            d[2 * i] = (uint32_t)y;
                            d[2 * i + 1] = (uint32_t)(y >> 32);
                        }
                        tmem_st16u(ty + c * 16, d);
                    }
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_one(bar + bScaled + j);
                }
                const float* w = gates + b * kGateBuf + j * kGateSet;
                const uint64_t minus = pack2(-1.f, -1.f);
#pragma unroll 1
                for (int h = 0; h < 4; ++h) {
                    if (h >= 2) {
                        ok = warp_wait(bar + bProd + (h & 1), 0);
                        if (!ok) break;
                    }
                    const int tt = bt >> 3, t32 = h * 32 + tt;                   // eight threads a token, 8 columns each
                    const uint64_t wt = pack2(w[t32], w[t32]);
                    const uint32_t inside = t32 < valid ? 0xffffffffu : 0u;
                    const unsigned char* v = smem + kVOff + (b * 2 + j) * kTile + t32 * 128;
                    unsigned char* to = buf + (h & 1) * 12288 + tt * 128;
                    {
                        const uint32_t off = (uint32_t)(((bt & 7) ^ (tt & 7)) * 16);
                        const uint4 vv = *reinterpret_cast<const uint4*>(v + off);
                        const uint32_t v4[4] = {vv.x & inside, vv.y & inside, vv.z & inside, vv.w & inside};
                        uint32_t q[3][4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            // the upper 16 bits of what is left, twice, and the rest rounded: 8 + 8 + 8 bits
                            uint64_t r = mul2(pack2(__uint_as_float(v4[i] << 16), __uint_as_float(v4[i] & 0xffff0000u)), wt);
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const uint32_t lo = (uint32_t)r & 0xffff0000u, hi = (uint32_t)(r >> 32) & 0xffff0000u;
                                q[e][i] = __byte_perm(lo, hi, 0x7632);
                                r = fma2(pack2(__uint_as_float(lo), __uint_as_float(hi)), minus, r);
                            }
                            float r0, r1;
                            unpack2(r, r0, r1);
                            q[2][i] = bf16x2(r0, r1);
                        }
#pragma unroll
                        for (int e = 0; e < 3; ++e)
                            *reinterpret_cast<uint4*>(to + e * 4096 + off) = make_uint4(q[e][0], q[e][1], q[e][2], q[e][3]);
                    }
                    proxy_fence();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive_one(bar + bW + (h & 1));
                        if (h == 3) mbar_arrive_one(OUTPUTS ? bar + bVRead + j * 2 + b : bar + bEmptyV + b);
                    }
                }
                if (!ok) break;
                const float keep = w[6 * kQ];
                total *= keep;
                ok = warp_wait(bar + bProd + 1, 1);
                if (!ok) break;
                tc_fence_after();
                const uint64_t keep2 = pack2(keep, keep);
                {
                    uint32_t d[2][16];
                    tmem_ld16_async(tmem + lanes + kProd + j * 64 + half * 32, d[0]);
                    tmem_ld16_async(tmem + lanes + kProd + j * 64 + half * 32 + 16, d[1]);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        S[i] = fma2(keep2, S[i], pack2(__uint_as_float(d[i / 8][2 * i % 16]), __uint_as_float(d[i / 8][2 * i % 16 + 1])));
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_one(bar + bGateFree + b);
            }
            if (!ok) break;
            if (live) {
                if constexpr (!OUTPUTS) {
                    store(p.work + at(x.seq * p.segments + x.seg + 1));
                    if (row == 0 && half == 0 && block % per_head == 0) *decay(x.seg + 1) = total;
                } else if (x.last) {
                    const int dst = seq_slot(p.pr, x.seq);
                    if (dst >= 0) store(p.state + at(dst));
                }
            }
        }
        if (!ok && lane == 0) record_fault(p.status, kFaultScanWait, 6);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_free<512>(tmem);
}

}  // namespace

// Segments of a sequence, from what the host knows of the lengths.
int prompt_scan_tc_segments(Ctx* ctx, int groups, int sequences, int tokens) {
    const sketchssm_config& c = ctx->cfg;
    const long long slabs = (long long)groups * ((c.heads / groups * (c.dv / 64) + 1) / 2);
    const long long all = scan_segment_states(c, tokens), n = (all < 148 / slabs ? all : 148 / slabs) / sequences;
    return n < 2 ? 1 : n > 16 ? 16 : (int)n;
}

int launch_prompt_scan_tc(Ctx* ctx, const ScanParams& p0, bool bf16, cudaStream_t stream) {
    ScanParams p = p0;
    if (!bf16 || !p.out_bf16 || p.K != 128 || p.V % 64 != 0 || p.pr.T == 0) return SKETCHSSM_UNSUPPORTED_SHAPE;
    p.segments = prompt_scan_tc_segments(ctx, p.G, p.pr.N, p.pr.T);
    ScanArgs g;
    g.p = p;
    g.blocks_per_group = p.H / p.G * (p.V / 64);
    g.slabs_per_group = (g.blocks_per_group + 1) / 2;
    g.slabs = g.slabs_per_group * p.G;
    const long long units = (long long)p.pr.N * p.segments * g.slabs;
    if (units > (1 << 30)) return SKETCHSSM_UNSUPPORTED_SHAPE;
    g.units = (int)units;
    if (!make_map(&g.tq, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.q, (uint64_t)p.G * 128, (uint64_t)p.pr.T, (uint64_t)p.q_stride * 2, kQ) ||
        !make_map(&g.tk, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.k, (uint64_t)p.G * 128, (uint64_t)p.pr.T, (uint64_t)p.k_stride * 2, kQ / 2) ||
        !make_map(&g.tv, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.v, (uint64_t)p.H * p.V, (uint64_t)p.pr.T, (uint64_t)p.v_stride * 2, kQ)) {
        ctx->last_cuda_error = cudaErrorInvalidValue;
        return SKETCHSSM_CUDA_ERROR;
    }
    cudaError_t e = unlock_smem(ctx, prompt_scan_tc_kernel<true>);
    if (e == cudaSuccess && p.segments > 1) e = unlock_smem(ctx, prompt_scan_tc_kernel<false>);
    if (e != cudaSuccess) { ctx->last_cuda_error = e; return SKETCHSSM_CUDA_ERROR; }
    const unsigned grid = (unsigned)(units < sm_count(ctx) ? units : sm_count(ctx));
    if (p.segments > 1) {
        const int rc = launch_layer<ScanArgs>(ctx, prompt_scan_tc_kernel<false>, dim3(grid), dim3(kThreads), kSmemTc, stream, g);
        if (rc != SKETCHSSM_OK) return rc;
    }
    return launch_layer<ScanArgs>(ctx, prompt_scan_tc_kernel<true>, dim3(grid), dim3(kThreads), kSmemTc, stream, g);
}

}  // namespace sketchssm
