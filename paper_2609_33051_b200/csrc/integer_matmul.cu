// Product of 8-bit integer matrices with a scale for each row of either, on tcgen05: few rows.
//
//     out[m][n] = a_scale[m] w_scale[n] sum_k a[m][k] w[n][k],   the sum exact in 32-bit integers
//
// The weights are the 128-row operand and the tokens the BN-column one, so that a few tokens cost a narrow accumulator, the weights' scale
// is one number a thread, and a warp's stores of a token are 32 neighbouring elements of its row, whatever the row stride and the edges are.
// A tile's whole inner axis runs into one accumulator (tensor memory); there are two, so that one is scaled and stored while the next tile
// is multiplied.  With few tiles (a decode step) the inner axis is split over a cluster of up to eight CTAs; each of them adds up a share
// of the columns from every rank's shared memory: whole numbers, so that no order of theirs shows.
//
// Roles: one thread issues the copies (TMA, 128-byte swizzle), one warp the products (an elected lane of the converged warp), the
// others take the sums out.
//
// What bounds it (weights from memory, replayed from a graph): 64 x 12352 x 2048 takes 9.8 us, of which the weights' 25 MB are 3.9 at 6.46 TB/s;
// the rest is the start, the first copies' way and the end of 97 CTAs with one tile each, the fullest use of 148 SMs that tiles of 128 weights
// allow.  777 x 2049 x 4096, 119 tiles, 13.8 us: 125 MB of operands from L2 at 9 TB/s, near what it gives.
#include "tma.cuh"

namespace sketchssm {

namespace {

using namespace tc;

struct Int8Args {
    CUtensorMap tw, ta;
    MatmulParams p;
    int ks, n_tiles, tiles;
};

__device__ __forceinline__ void put(float* o, float y) { *o = y; }
__device__ __forceinline__ void put(__nv_bfloat16* o, float y) { *o = __float2bfloat16_rn(y); }

// NS stages of operand tiles.
template <int BN, int NS>
struct Int8Smem {
    static constexpr uint32_t kW = 128u * 128u, kA = (uint32_t)BN * 128u, kStage = kW + kA;
    static constexpr uint32_t kBars = NS * kStage;
    static constexpr uint32_t kBytes = kBars + (2 * NS + 4) * 8u + 16u + 1024u;      // (the tiles start on 1024 bytes)
    static_assert(BN * 128u * 4u <= NS * kStage, "the sums of a split tile take the stages' place");
};

// The sums of a tile's BN columns that the KS CTAs of a cluster hold, a share of the columns by each: four rows of a column at a
// time, all loads of a thread under way together.
template <int BN, int THREADS, int KS>
__device__ __forceinline__ void add_ranks(const Int8Args& g, unsigned char* smem, int tile, int rank) {
    constexpr int kPer = BN / KS, kItems = kPer * 32, kRounds = (kItems + THREADS - 1) / THREADS;
    const MatmulParams& p = g.p;
    const int m0 = tile / g.n_tiles * BN + rank * kPer, n0 = tile % g.n_tiles * 128;
    float as[kRounds], ws[kRounds][4];                  // (asked for before the wait)
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        const int item = i * THREADS + (int)threadIdx.x, m = m0 + item / 32, n = n0 + item % 32 * 4;
        const bool in = (kItems % THREADS == 0 || item < kItems) && m < p.M;
        as[i] = in ? p.a_scale[m] : 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) ws[i][j] = in && n + j < p.N ? p.w_scale[n + j] : 0.f;
    }
    cluster_sync();
    int4 f[kRounds][KS];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        const int item = i * THREADS + (int)threadIdx.x;
        if (kItems % THREADS == 0 || item < kItems) {
#pragma unroll
            for (int q = 0; q < KS; ++q)
                asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(f[i][q].x), "=r"(f[i][q].y), "=r"(f[i][q].z), "=r"(f[i][q].w)
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
            const int y[4] = {f[i][0].x, f[i][0].y, f[i][0].z, f[i][0].w};
            const size_t o = (size_t)m * p.out_stride + n;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (n + j < p.N) {
                    const float s = (float)y[j] * as[i] * ws[i][j];
                    if (p.out_bf16) put(static_cast<__nv_bfloat16*>(p.out) + o + j, s);
                    else put(static_cast<float*>(p.out) + o + j, s);
                }
            }
        }
    }
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");        // nobody reaches into a CTA that has ended
}

template <int BN, int EW, int NS, int MINB>
__global__ void __launch_bounds__(32 * (EW + 4), MINB) integer_matmul_kernel(const __grid_constant__ Int8Args g) {
    using L = Int8Smem<BN, NS>;
    constexpr int CW = BN / (EW / 4);                  // accumulator columns of an epilogue warp
    constexpr int CH = 16;                             // of one load
    constexpr int TM = 2 * BN < 32 ? 32 : 2 * BN;
    extern __shared__ unsigned char raw[];
    unsigned char* smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBars);
    uint64_t *empty = full + NS, *acc_full = empty + NS, *acc_empty = acc_full + 2;
    uint32_t* slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
    const MatmulParams& p = g.p;
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 32) { prefetch_map(&g.tw); prefetch_map(&g.ta); }
    if (tid == 0) {
        for (int i = 0; i < NS; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(acc_full + i, 1); mbar_init(acc_empty + i, EW); }
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
                        record_fault(p.status, kFaultMatmulWait, 21);
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
        constexpr uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | ((128u >> 4) << 24);      // s8 x s8 -> s32
        int it = 0, n = 0;
        bool ok = true;
        for (int tile = first; tile < g.tiles && ok; tile += step, ++n) {
            const int as = n & 1;
            ok = n < 2 || warp_wait(acc_empty + as, (n / 2 - 1) & 1);
            for (int kb = kb0; kb < kb1 && ok; ++kb, ++it) {
                const int s = it % NS;
                ok = warp_wait(full + s, (it / NS) & 1);
                if (!ok) break;
                tc_fence_after();
                const uint32_t base = smem_u32(smem) + (uint32_t)s * L::kStage;
                const uint64_t dw = swizzled_desc(base, 16u, 1024u), da = swizzled_desc(base + L::kW, 16u, 1024u);
#pragma unroll
                for (int j = 0; j < 4; ++j)            // 32 bytes of every row at a time
                    if (elect())
                        asm volatile(
                            "{\n\t.reg .pred p;\n\t"
                            "setp.ne.b32 p, %4, 0;\n\t"
                            "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem + (uint32_t)(as * BN)),
                            "l"(dw + 2u * j), "l"(da + 2u * j), "r"(idesc), "r"((uint32_t)(j | (kb - kb0)))
                            : "memory");
                if (elect()) {
                    tc_commit(empty + s);
                    if (kb == kb1 - 1) tc_commit(acc_full + as);
                }
                __syncwarp();
            }
            if (!ok && lane == 0) record_fault(p.status, kFaultMatmulWait, 22);
        }
    } else if (warp >= 4) {
        const int quad = warp & 3, half = (warp - 4) >> 2;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        int it = 0;
        for (int tile = first; tile < g.tiles; tile += step, ++it) {
            const int as = it & 1;
            const int n = tile % g.n_tiles * 128 + quad * 32 + lane, m0 = tile / g.n_tiles * BN + half * CW;
            const float ws = n < p.N ? p.w_scale[n] : 0.f;
            bool ok = mbar_wait_bounded(acc_full + as, (it / 2) & 1);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) {
                if (lane == 0) record_fault(p.status, kFaultMatmulWait, 23);
                break;
            }
            tc_fence_after();
            // (a split tile's products have all been waited for, so nothing reads or fills the stages any more)
            int* sums = reinterpret_cast<int*>(smem) + (size_t)(half * CW) * 128 + quad * 32 + lane;
#pragma unroll
            for (int c = 0; c < CW / CH; ++c) {
                uint32_t d[CH];
                tmem_ld16_async(tmem + (uint32_t)(as * BN + half * CW + c * CH) + lanes, d);
                tmem_ld_wait();
                if (g.ks > 1) {
#pragma unroll
                    for (int j = 0; j < CH; ++j) sums[(c * CH + j) * 128] = (int)d[j];
                } else {
                    const int cols = min(CH, p.M - m0 - c * CH);
                    float sc[CH];
#pragma unroll
                    for (int j = 0; j < CH; ++j) sc[j] = j < cols ? p.a_scale[m0 + c * CH + j] : 0.f;
                    auto store = [&](auto* out) {
                        out += (size_t)(m0 + c * CH) * p.out_stride + n;
#pragma unroll
                        for (int j = 0; j < CH; ++j) {
                            if (j < cols && n < p.N) put(out, (float)(int)d[j] * sc[j] * ws);
                            out += p.out_stride;
                        }
                    };
                    if (p.out_bf16) store(static_cast<__nv_bfloat16*>(p.out));
                    else store(static_cast<float*>(p.out));
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_one(acc_empty + as);
        }
    }
    __syncwarp();
    if (g.ks == 2) add_ranks<BN, 32 * (EW + 4), 2>(g, smem, first, rank);      // a CTA of a cluster has one tile
    if (g.ks == 4) add_ranks<BN, 32 * (EW + 4), 4>(g, smem, first, rank);
    if (g.ks == 8) add_ranks<BN, 32 * (EW + 4), 8>(g, smem, first, rank);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_free<TM>(tmem);
}

template <int BN, int EW, int NS, int MINB>
int launch_tiles(Ctx* ctx, const MatmulParams& p, int ks, cudaStream_t stream) {
    Int8Args g;
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
    auto kern = integer_matmul_kernel<BN, EW, NS, MINB>;
    const cudaError_t e = unlock_smem(ctx, kern);
    if (e != cudaSuccess) { ctx->last_cuda_error = e; return SKETCHSSM_CUDA_ERROR; }
    const int grid = ks > 1 ? (int)tiles * ks : (int)(tiles < (long long)sm_count(ctx) * MINB ? tiles : sm_count(ctx) * MINB);
    return launch_layer<Int8Args>(ctx, kern, dim3((unsigned)grid), dim3(32 * (EW + 4)), Int8Smem<BN, NS>::kBytes, stream, g, ks);
}

}  // namespace

int launch_integer_matmul(Ctx* ctx, const MatmulParams& p, cudaStream_t stream) {
    const int sms = sm_count(ctx);
    const long long nt = (p.N + 127) / 128;
    if (p.M > 128) {
        const int rc = launch_integer_matmul_pair(ctx, p, stream);
        if (rc != SKETCHSSM_UNSUPPORTED_SHAPE) return rc;
    }
    // The narrowest tile that holds the tokens (1 x 12352 x 2048: 8.1 us; 64: 9.8; 128: 10.8).
    const int bn = p.M <= 16 ? 16 : p.M <= 32 ? 32 : p.M <= 64 ? 64 : 128;
    const long long tiles = nt * ((p.M + bn - 1) / bn);
    // Few tiles: the inner axis split over a cluster, while that leaves a CTA two blocks and every SM one CTA.  (Clusters of eight CTAs that have an SM
    // to themselves find no place for more than about half of the SMs at a time: 128 x 2048 x 4096 in 8.9 us with clusters of four, 15.0 with
    // eight; but 100 x 1024 x 8192, 8 tiles, 10.7 and 9.0.  Not split: 13.5 us for the first; 64 x 2048 x 4096 12.3, split 7.9.)
    int ks = 1;
    while (ks < 8 && tiles * ks * 2 <= (long long)(bn == 128 && ks == 4 ? sms / 2 : sms) && p.KB >= ks * 4) ks *= 2;
    if (bn == 16) return launch_tiles<16, 4, 6, 2>(ctx, p, ks, stream);
    if (bn == 32) return launch_tiles<32, 4, 5, 2>(ctx, p, ks, stream);
    // (64 x 12352 x 2048, not split: 9.8 us with eight stages, 10.6 with four and two CTAs an SM; 64 x 2048 x 4096, by eight: 11.6 and 7.9.)
    if (bn == 64) return ks <= 2 ? launch_tiles<64, 4, 8, 1>(ctx, p, ks, stream) : launch_tiles<64, 4, 4, 2>(ctx, p, ks, stream);
    return launch_tiles<128, 8, 6, 1>(ctx, p, ks, stream);
}

}  // namespace sketchssm
