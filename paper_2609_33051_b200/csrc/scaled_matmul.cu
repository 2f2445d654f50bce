// Product of e4m3 matrices with a scale for each block of 128 along the inner axis (and 128 rows of the weights), on tcgen05.
//
//     out[m][n] = sum_b a_scale[m][b] w_scale[n / 128][b] sum_{k in block b} a[m][k] w[n][k]
//
// The weights are the 128-row operand and the tokens the BN-column one: an accumulator lane is a weight row, a column a token.
// So a few tokens cost a narrow accumulator instead of a mostly empty 128-row one, the weights' scale is one number per tile and
// block, and a warp's stores of a token are 32 neighbouring elements of its row, whatever the row stride and the edges are.
// Each block of 128 goes through the tensor cores into an accumulator of its own (fp32, in tensor memory); the epilogue warps
// add it, times its scales, to sums in registers, two elements an instruction, while the next block is multiplied.
//
// Roles: one thread issues the copies (TMA, 128-byte swizzle: a row of a tile is exactly one block), one warp the products (an elected
// lane of the converged warp); two warps fetch the token scales, four blocks at a time and one such group ahead, and leave them, times
// the weights' scale, in shared memory; the other warps add.
// With few tiles (a decode step) the blocks are split over a cluster of up to eight CTAs; each of them adds up a share of the
// columns, from the sums in every rank's shared memory in the order of the ranks.
//
// What bounds it: 64 x 8512 x 2048 takes 7.6 us (8.3 replayed from a graph, as the times below are), of which the weights' bytes are 2.7 at
// the rate of HBM; the first tile arrives 3400 cycles after the start, the eight blocks of a CTA take another 2500, the sums' way to the
// other CTA and out 4000.
#include "tma.cuh"

namespace sketchssm {

namespace {

using namespace tc;

struct MatmulArgs {
    CUtensorMap tw, ta;
    MatmulParams p;
    int ks, n_tiles, tiles;
};

__device__ __forceinline__ void put(float* o, float y) { *o = y; }
__device__ __forceinline__ void put(__nv_bfloat16* o, float y) { *o = __float2bfloat16_rn(y); }

// AS accumulators of BN columns, NS stages of operand tiles, EW epilogue warps.
template <int BN, int EW, int NS, int AS>
struct MatmulSmem {
    static constexpr uint32_t kW = 128u * 128u, kA = (uint32_t)BN * 128u, kStage = kW + kA;
    static constexpr uint32_t kScales = NS * kStage;                       // [AS][BN] floats
    static constexpr uint32_t kBars = kScales + AS * BN * 4u;
    static constexpr uint32_t kTotal = kBars + (2 * NS + 3 * AS) * 8u + 16u;
    static constexpr uint32_t kBytes = kTotal + 1024u;                     // (the tiles start on 1024 bytes)
    static_assert(BN * 128u * 4u <= NS * kStage, "the sums of a split tile take the stages' place");
};

// The sums of a tile's BN columns that the KS CTAs of a cluster hold, a share of the columns by each: four rows of a column at a
// time, all loads of a thread under way together (a round trip to another SM's shared memory is about a thousand cycles).
template <int BN, int THREADS, int KS>
__device__ __forceinline__ void add_ranks(const MatmulArgs& g, unsigned char* smem, int tile, int rank) {
    constexpr int kPer = BN / KS, kItems = kPer * 32, kRounds = (kItems + THREADS - 1) / THREADS;
    const MatmulParams& p = g.p;
    const int m0 = tile / g.n_tiles * BN + rank * kPer, n0 = tile % g.n_tiles * 128;
    cluster_sync();
    float4 f[kRounds][KS];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        const int item = i * THREADS + (int)threadIdx.x;
        if (kItems % THREADS == 0 || item < kItems) {
#pragma unroll
            for (int q = 0; q < KS; ++q)
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f[i][q].x), "=f"(f[i][q].y), "=f"(f[i][q].z), "=f"(f[i][q].w)
                             : "r"(cluster_addr(smem + (uint32_t)(rank * kItems + item) * 16u, (uint32_t)q)) : "memory");
        }
    }
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
#pragma unroll
        for (int q = 1; q < KS; ++q) {
            f[i][0].x += f[i][q].x; f[i][0].y += f[i][q].y; f[i][0].z += f[i][q].z; f[i][0].w += f[i][q].w;
        }
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // this CTA needs the others' sums no more
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        const int item = i * THREADS + (int)threadIdx.x, m = m0 + item / 32, n = n0 + item % 32 * 4;
        if ((kItems % THREADS == 0 || item < kItems) && m < p.M) {
            const float y[4] = {f[i][0].x, f[i][0].y, f[i][0].z, f[i][0].w};
            const size_t o = (size_t)m * p.out_stride + n;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (n + j < p.N) {
                    if (p.out_bf16) put(static_cast<__nv_bfloat16*>(p.out) + o + j, y[j]);
                    else put(static_cast<float*>(p.out) + o + j, y[j]);
                }
            }
        }
    }
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");        // nobody reaches into a CTA that has ended
}

template <int BN, int EW, int NS, int AS, int MINB>
__global__ void __launch_bounds__(32 * (EW + 4), MINB) scaled_matmul_kernel(const __grid_constant__ MatmulArgs g) {
    using L = MatmulSmem<BN, EW, NS, AS>;
    constexpr int CW = BN / (EW / 4);                  // accumulator columns of an epilogue warp
    constexpr int CH = 16;                             // of one load
    constexpr int TM = AS * BN < 32 ? 32 : AS * BN;
    extern __shared__ unsigned char raw[];
    unsigned char* smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    float* scales = reinterpret_cast<float*>(smem + L::kScales);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBars);
    uint64_t *empty = full + NS, *acc_full = empty + NS, *acc_empty = acc_full + AS, *sc_full = acc_empty + AS;
    uint32_t* slot = reinterpret_cast<uint32_t*>(sc_full + AS);
    const MatmulParams& p = g.p;
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 32) { prefetch_map(&g.tw); prefetch_map(&g.ta); }
    if (tid == 0) {
        for (int i = 0; i < NS; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
        for (int i = 0; i < AS; ++i) { mbar_init(acc_full + i, 1); mbar_init(acc_empty + i, EW); mbar_init(sc_full + i, 2); }
        mbar_fence_init();
    }
    if (warp == 1) tmem_alloc<TM>(slot);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    int rank = (int)blockIdx.x % g.ks, first = (int)blockIdx.x / g.ks, step = (int)gridDim.x / g.ks;
    int kb0 = p.KB * rank / g.ks, kb1 = p.KB * (rank + 1) / g.ks;
    asm volatile("" : "+r"(rank), "+r"(first), "+r"(step), "+r"(kb0), "+r"(kb1));      // (worked out while the predecessor still runs)
    grid_dep_wait();
    grid_dep_launch_dependents();
    const uint32_t tmem = *slot;

    if (warp == 0) {
        if (lane == 0) {
            int it = 0;
            bool ok = true;
            for (int tile = first; tile < g.tiles && ok; tile += step) {
                const int n0 = tile % g.n_tiles * 128, m0 = tile / g.n_tiles * BN;
                for (int kb = kb0; kb < kb1; ++kb, ++it) {
                    const int s = it % NS;
                    if (it >= NS && !mbar_wait_bounded(empty + s, (it / NS - 1) & 1)) {
                        record_fault(p.status, kFaultMatmulWait, 1);
                        ok = false;
                        break;
                    }
                    mbar_expect_tx(full + s, L::kStage);
                    tma_load(smem + s * L::kStage, &g.tw, kb * 128, n0, full + s);
                    tma_load(smem + s * L::kStage + L::kW, &g.ta, kb * 128, m0, full + s);
                }
            }
            // before the CTA ends: no copy is under way (after a fault; otherwise all of them have been waited for), and the products'
            // last arrivals at the stages' barriers are in
            for (int i = it < NS ? 0 : it - NS; i < it; ++i) mbar_wait_bounded((ok ? empty : full) + i % NS, (i / NS) & 1);
        }
        __syncwarp();
    } else if (warp == 1) {
        constexpr uint32_t idesc = (1u << 4) | ((uint32_t)(BN >> 3) << 17) | ((128u >> 4) << 24);      // e4m3 x e4m3 -> fp32
        int it = 0;
        bool ok = true;
        for (int tile = first; tile < g.tiles && ok; tile += step) {
            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                const int s = it % NS, as = it % AS;
                ok = it < AS || warp_wait(acc_empty + as, (it / AS - 1) & 1);
                ok = ok && warp_wait(full + s, (it / NS) & 1);
                if (!ok) {
                    if (lane == 0) record_fault(p.status, kFaultMatmulWait, 2);
                    break;
                }
                tc_fence_after();
                const uint32_t base = smem_u32(smem) + (uint32_t)s * L::kStage;
                const uint64_t dw = swizzled_desc(base, 16u, 1024u), da = swizzled_desc(base + L::kW, 16u, 1024u);
#pragma unroll
                for (int j = 0; j < 4; ++j)            // 32 bytes of every row at a time
                    if (elect())
                        asm volatile(
                            "{\n\t.reg .pred p;\n\t"
                            "setp.ne.b32 p, %4, 0;\n\t"
                            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem + (uint32_t)(as * BN)),
                            "l"(dw + 2u * j), "l"(da + 2u * j), "r"(idesc), "r"((uint32_t)j)
                            : "memory");
                if (elect()) {
                    tc_commit(empty + s);
                    tc_commit(acc_full + as);
                }
                __syncwarp();
            }
        }
    } else if (warp < 4) {
        constexpr int PT = (BN + 63) / 64;             // tokens of a thread
        const int t = tid - 64;
        int it = 0;
        bool ok = true;
        for (int tile = first; tile < g.tiles && ok; tile += step) {
            const float* sw = p.w_scale + (size_t)(tile % g.n_tiles) * p.KB;
            const int m0 = tile / g.n_tiles * BN;
            // four blocks' scales at a time, one such group ahead of the one in use (nothing may be computed from them before
            // that: the first use waits for the load)
            auto fetch = [&](int kb, float (&f)[4][PT], float (&fw)[4]) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    fw[j] = kb + j < kb1 ? sw[kb + j] : 0.f;
#pragma unroll
                    for (int i = 0; i < PT; ++i) {
                        const int m = m0 + t + 64 * i;
                        f[j][i] = t + 64 * i < BN && m < p.M && kb + j < kb1 ? p.a_scale[(size_t)m * p.KB + kb + j] : 0.f;
                    }
                }
            };
            float now[4][PT], next[4][PT], now_w[4], next_w[4];
            fetch(kb0, next, next_w);
            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                if (((kb - kb0) & 3) == 0) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        now_w[j] = next_w[j];
#pragma unroll
                        for (int i = 0; i < PT; ++i) now[j][i] = next[j][i];
                    }
                    fetch(kb + 4, next, next_w);
                }
                const int as = it % AS;
                ok = it < AS || mbar_wait_bounded(acc_empty + as, (it / AS - 1) & 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) {
                    if (lane == 0) record_fault(p.status, kFaultMatmulWait, 3);
                    break;
                }
#pragma unroll
                for (int i = 0; i < PT; ++i) {
                    if (t + 64 * i < BN) scales[as * BN + t + 64 * i] = now[0][i] * now_w[0];
                    now[0][i] = now[1][i];
                    now[1][i] = now[2][i];
                    now[2][i] = now[3][i];
                }
                now_w[0] = now_w[1];
                now_w[1] = now_w[2];
                now_w[2] = now_w[3];
                __syncwarp();
                if (lane == 0) mbar_arrive_one(sc_full + as);
            }
        }
    } else {
        const int quad = warp & 3, half = (warp - 4) >> 2;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        int it = 0;
        bool ok = true;
        uint64_t acc[CW / 2];
        for (int tile = first; tile < g.tiles && ok; tile += step) {
#pragma unroll
            for (int c = 0; c < CW / 2; ++c) acc[c] = 0ull;
            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                const int as = it % AS;
                ok = mbar_wait_bounded(sc_full + as, (it / AS) & 1) && mbar_wait_bounded(acc_full + as, (it / AS) & 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) {
                    if (lane == 0) record_fault(p.status, kFaultMatmulWait, 4);
                    break;
                }
                tc_fence_after();
                const ulonglong2* sc = reinterpret_cast<const ulonglong2*>(scales + as * BN + half * CW);
#pragma unroll
                for (int c = 0; c < CW / CH; ++c) {
                    float d[CH];
                    tmem_ld16(tmem + (uint32_t)(as * BN + half * CW + c * CH) + lanes, d);
#pragma unroll
                    for (int j = 0; j < CH / 4; ++j) {
                        const ulonglong2 s4 = sc[c * (CH / 4) + j];
                        uint64_t* a = acc + c * (CH / 2) + 2 * j;
                        a[0] = fma2(pack2(d[4 * j], d[4 * j + 1]), s4.x, a[0]);
                        a[1] = fma2(pack2(d[4 * j + 2], d[4 * j + 3]), s4.y, a[1]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_one(acc_empty + as);
            }
            const int n = tile % g.n_tiles * 128 + quad * 32 + lane, m0 = tile / g.n_tiles * BN + half * CW;
            if (g.ks == 1) {
                if (n < p.N) {
                    const int cols = min(CW, p.M - m0);
                    auto store = [&](auto* out) {
                        out += (size_t)m0 * p.out_stride + n;
#pragma unroll
                        for (int c = 0; c < CW; ++c) {
                            float lo, hi;
                            unpack2(acc[c / 2], lo, hi);
                            if (c < cols) put(out, (c & 1) ? hi : lo);
                            out += p.out_stride;
                        }
                    };
                    if (p.out_bf16) store(static_cast<__nv_bfloat16*>(p.out));
                    else store(static_cast<float*>(p.out));
                }
            } else {
                // every product of this CTA has been waited for, so nothing reads or fills the stages any more
                float* sums = reinterpret_cast<float*>(smem) + (size_t)(half * CW) * 128 + quad * 32 + lane;
#pragma unroll
                for (int c = 0; c < CW; ++c) {
                    float lo, hi;
                    unpack2(acc[c / 2], lo, hi);
                    sums[c * 128] = (c & 1) ? hi : lo;
                }
            }
        }
    }
    if (g.ks == 2) add_ranks<BN, 32 * (EW + 4), 2>(g, smem, first, rank);      // a CTA of a cluster has one tile
    if (g.ks == 4) add_ranks<BN, 32 * (EW + 4), 4>(g, smem, first, rank);
    if (g.ks == 8) add_ranks<BN, 32 * (EW + 4), 8>(g, smem, first, rank);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_free<TM>(tmem);
}

template <int BN, int EW, int NS, int AS, int MINB>
int launch_tiles(Ctx* ctx, const MatmulParams& p, int ks, cudaStream_t stream) {
    MatmulArgs g;
    g.p = p;
    g.ks = ks;
    g.n_tiles = (p.N + 127) / 128;
    const long long tiles = (long long)g.n_tiles * ((p.M + BN - 1) / BN);
    if (tiles > (1 << 27)) return SKETCHSSM_UNSUPPORTED_SHAPE;
    g.tiles = (int)tiles;
    if (!make_map(&g.tw, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.w, (uint64_t)p.K, (uint64_t)p.N, (uint64_t)p.K, 128) ||
        !make_map(&g.ta, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.a, (uint64_t)p.K, (uint64_t)p.M, (uint64_t)p.K, BN)) {
        ctx->last_cuda_error = cudaErrorInvalidValue;
        return SKETCHSSM_CUDA_ERROR;
    }
    auto kern = scaled_matmul_kernel<BN, EW, NS, AS, MINB>;
    const cudaError_t e = unlock_smem(ctx, kern);
    if (e != cudaSuccess) { ctx->last_cuda_error = e; return SKETCHSSM_CUDA_ERROR; }
    const int grid = ks > 1 ? (int)tiles * ks : (int)(tiles < (long long)sm_count(ctx) * MINB ? tiles : sm_count(ctx) * MINB);
    return launch_layer<MatmulArgs>(ctx, kern, dim3((unsigned)grid), dim3(32 * (EW + 4)), MatmulSmem<BN, EW, NS, AS>::kBytes, stream, g, ks);
}

}  // namespace

int launch_scaled_matmul(Ctx* ctx, const MatmulParams& p, cudaStream_t stream) {
    const int sms = sm_count(ctx);
    const long long nt = (p.N + 127) / 128;
    if (p.M > 128) {
        const int rc = launch_scaled_matmul_pair(ctx, p, stream);
        if (rc != SKETCHSSM_UNSUPPORTED_SHAPE) return rc;
    }
    // The narrowest tile that holds the tokens.
    const int bn = p.M <= 16 ? 16 : p.M <= 32 ? 32 : p.M <= 64 ? 64 : 128;
    const long long tiles = nt * ((p.M + bn - 1) / bn);
    // Few tiles: the blocks split over a cluster, while that leaves a CTA two blocks and every SM one CTA.  (Two CTAs an SM: 9.3 us for
    // 64 x 8512 x 2048 against 8.3; the sums' way through distributed shared memory, some 10 bytes a cycle and SM, is what grows.)
    int ks = 1;
    while (ks < 8 && tiles * ks * 2 <= (long long)sms && p.KB >= ks * 4) ks *= 2;
    if (bn == 16) return launch_tiles<16, 4, 6, 4, 2>(ctx, p, ks, stream);
    if (bn == 32) return launch_tiles<32, 4, 5, 4, 2>(ctx, p, ks, stream);
    // (Eight stages where a CTA has an SM to itself: 64 x 8512 x 2048 in 8.3 us, 8.7 with four.  With four stages two CTAs fit on an SM, and
    // clusters of four and eight find their place more easily: 64 x 2048 x 4096 in 8.5 us, 11.4 with eight.)
    if (bn == 64) return ks <= 2 ? launch_tiles<64, 4, 8, 4, 1>(ctx, p, ks, stream) : launch_tiles<64, 4, 4, 4, 2>(ctx, p, ks, stream);
    return launch_tiles<128, 8, 6, 4, 1>(ctx, p, ks, stream);
}

}  // namespace sketchssm
