// The product of integer_matmul.cu for many rows: tiles of 256 tokens x BN weights, 256 or 128, on pairs of SMs (tcgen05, cta_group::2).
//
// A pair shares both operands, half of each in either SM: a block of 128 of the inner axis is 32 KB of copies for an SM.  The tokens are the
// accumulator's lanes, the weights its columns.  The inner axis runs into one accumulator of BN columns; there are two, so that a tile is
// scaled and stored while the next one is multiplied.
//
// Roles per CTA: one thread issues the copies of its half (they report to the leader's barrier), one warp of the leader the products;
// BN / 16 warps take a tile's sums out (32 lanes, 64 columns each), times both scales, and store them through shared memory (TMA), or
// directly where a row or the row stride is no multiple of 16 bytes.
//
// What bounds it: the operands' way from L2, and the power cap.  16384 x 12352 x 2048 to bf16 takes 331 us by itself (L2 flushed, the card idle before it) and
// 350 one after another for a second, at 1430 to 1520 MHz of 1965: 2.50 and 2.37 Pop/s; 3136 tiles of 1 MB of operands are 9.0 to 9.5 TB/s.  (293 were
// seen on a cooler card.)  The output's 405 MB are 63 us of memory.  With four stages 330 and 362; five are what 227 KB hold beside the stores'
// staging.  Bands of 8 or 16 tiles of tokens, walked down a band first so that fewer operand tiles are in use at a time, gain nothing.
#include "tma.cuh"

namespace sketchssm {

namespace {

using namespace tc;

constexpr uint32_t kHalf = 128u * 128u;                // of the tokens
template <int BN, int NS>
struct PairShape {
    static constexpr int kEpiWarps = BN / 16, kThreads = 32 * (4 + kEpiWarps);
    static constexpr uint32_t kStageBytes = kHalf + (uint32_t)BN / 2u * 128u;
    static constexpr uint32_t kOut = NS * kStageBytes, kBars = kOut + kEpiWarps * 4096u, kSmem = kBars + (2 * NS + 4) * 8u + 16u + 1024u;
};

struct PairArgs {
    CUtensorMap ta, tw, to;
    MatmulParams p;
    int n_tiles, tiles, tma_out;
};

// A copy whose bytes are counted by a barrier of the leader of the pair.
__device__ __forceinline__ void tma_load_pair(void* dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
            smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
// Arrives at a barrier of both CTAs once the products issued so far are done.
__device__ __forceinline__ void commit_pair(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
                 "h"((uint16_t)3)
                 : "memory");
}

template <int BN, int kStages>
__global__ void __launch_bounds__(PairShape<BN, kStages>::kThreads, 1) integer_matmul_pair_kernel(const __grid_constant__ PairArgs g) {
    using L = PairShape<BN, kStages>;
    constexpr int kEpiWarps = L::kEpiWarps, kColumns = 2 * BN;         // two accumulators
    constexpr uint32_t kStageBytes = L::kStageBytes, kOut = L::kOut, kBars = L::kBars;
    extern __shared__ unsigned char raw[];
    unsigned char* smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + kBars);        // the leader's: both halves are there
    uint64_t *empty = full + kStages, *acc_full = empty + kStages, *acc_empty = acc_full + 2;     // acc_empty: the leader's
    uint32_t* slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
    const MatmulParams& p = g.p;
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = (int)blockIdx.x & 1, first = (int)blockIdx.x >> 1, step = (int)gridDim.x >> 1;
    if (tid == 64) { prefetch_map(&g.ta); prefetch_map(&g.tw); }
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(acc_full + i, 1); mbar_init(acc_empty + i, 2 * kEpiWarps); }
        mbar_fence_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "n"(kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    grid_dep_wait();
    grid_dep_launch_dependents();
    const uint32_t tmem = *slot;

    if (warp == 0) {
        if (lane == 0) {
            int it = 0;
            bool ok = true;
            for (int tile = first; tile < g.tiles && ok; tile += step) {
                const int m = tile / g.n_tiles * 256 + rank * 128, n = tile % g.n_tiles * BN + rank * (BN / 2);
                for (int kb = 0; kb < p.KB; ++kb, ++it) {
                    const int s = it % kStages;
                    if (it >= kStages && !mbar_wait_bounded(empty + s, (it / kStages - 1) & 1)) {
                        record_fault(p.status, kFaultMatmulWait, 31);
                        ok = false;
                        break;
                    }
                    if (rank == 0) mbar_expect_tx(full + s, 2u * kStageBytes);
                    const uint32_t bar = cluster_addr(full + s, 0);
                    unsigned char* dst = smem + (uint32_t)s * kStageBytes;
                    tma_load_pair(dst, &g.ta, kb * 128, m, bar);
                    tma_load_pair(dst + kHalf, &g.tw, kb * 128, n, bar);
                }
            }
            // before the CTAs end: no copy is under way (after a fault; otherwise all of them have been waited for), and the products'
            // last arrivals at the stages' barriers are in
            for (int i = it < kStages ? 0 : it - kStages; i < it; ++i) {
                if (ok) mbar_wait_bounded(empty + i % kStages, (i / kStages) & 1);
                else if (rank == 0) mbar_wait_bounded(full + i % kStages, (i / kStages) & 1);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            constexpr uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | ((256u >> 4) << 24);      // s8 x s8 -> s32
            int it = 0, n = 0;
            bool ok = true;
            for (int tile = first; tile < g.tiles && ok; tile += step, ++n) {
                const int as = n & 1;
                ok = n < 2 || warp_wait(acc_empty + as, (n / 2 - 1) & 1);
                for (int kb = 0; kb < p.KB && ok; ++kb, ++it) {
                    const int s = it % kStages;
                    ok = warp_wait(full + s, (it / kStages) & 1);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t base = smem_u32(smem) + (uint32_t)s * kStageBytes;
                    const uint64_t da = swizzled_desc(base, 16u, 1024u), dw = swizzled_desc(base + kHalf, 16u, 1024u);
#pragma unroll
                    for (int j = 0; j < 4; ++j)        // 32 bytes of every row at a time
                        if (elect())
                            asm volatile(
                                "{\n\t.reg .pred p;\n\t"
                                "setp.ne.b32 p, %4, 0;\n\t"
                                "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem + (uint32_t)(as * BN)),
                                "l"(da + 2u * j), "l"(dw + 2u * j), "r"(idesc), "r"((uint32_t)(j | kb))
                                : "memory");
                    if (elect()) {
                        commit_pair(empty + s);
                        if (kb == p.KB - 1) commit_pair(acc_full + as);
                    }
                    __syncwarp();
                }
                if (!ok && lane == 0) record_fault(p.status, kFaultMatmulWait, 32);
            }
        }
        __syncwarp();
    } else if (warp >= 4) {
        const int quad = warp & 3, part = (warp - 4) >> 2;             // 32 lanes, 64 columns
        const uint32_t at0 = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(part * 64);
        unsigned char* stage = smem + kOut + (uint32_t)(warp - 4) * 4096u;
        const uint32_t release = cluster_addr(acc_empty, 0);
        int it = 0;
        for (int tile = first; tile < g.tiles; tile += step, ++it) {
            const int as = it & 1;
            const int m0 = tile / g.n_tiles * 256 + rank * 128 + quad * 32, n0 = tile % g.n_tiles * BN + part * 64;
            const float s = m0 + lane < p.M ? p.a_scale[m0 + lane] : 0.f;
            const float w0 = n0 + lane < p.N ? p.w_scale[n0 + lane] : 0.f, w1 = n0 + 32 + lane < p.N ? p.w_scale[n0 + 32 + lane] : 0.f;
            bool ok = mbar_wait_bounded(acc_full + as, (it / 2) & 1);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) {
                if (lane == 0) record_fault(p.status, kFaultMatmulWait, 33);
                break;
            }
            tc_fence_after();
            uint32_t d[2][32];
            tmem_ld32_async(at0 + (uint32_t)(as * BN), d[0]);
            tmem_ld32_async(at0 + (uint32_t)(as * BN + 32), d[1]);
            tmem_ld_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(release + 8u * (uint32_t)as) : "memory");
#pragma unroll
            for (int c = 0; c < 32; ++c) {
                d[0][c] = __float_as_uint((float)(int)d[0][c] * s * __shfl_sync(0xffffffffu, w0, c));
                d[1][c] = __float_as_uint((float)(int)d[1][c] * s * __shfl_sync(0xffffffffu, w1, c));
            }
            // through shared memory, 128 bytes of a row at a time: 64 elements, or 32
            const int per = p.out_bf16 ? 64 : 32;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                if (p.out_bf16 && r >= 1) break;
                if (lane == 0) tma_store_read();
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint4 u;
                    if (p.out_bf16) {
                        float f[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(d[c / 4][c % 4 * 8 + j]);
                        u = Vec16<__nv_bfloat16>::pack(f);
                    } else {
                        u = make_uint4(d[r][c * 4], d[r][c * 4 + 1], d[r][c * 4 + 2], d[r][c * 4 + 3]);
                    }
                    *reinterpret_cast<uint4*>(stage + lane * 128 + ((c ^ (lane & 7)) * 16)) = u;
                }
                const int n = n0 + r * per;
                if (g.tma_out) {
                    proxy_fence();
                    __syncwarp();
                    if (lane == 0 && m0 < p.M && n < p.N) tma_store(&g.to, n, m0, stage);
                } else {
                    __syncwarp();
                    const int rows = min(32, p.M - m0);
                    for (int i = 0; i < rows; ++i) {
                        const unsigned char* row = stage + i * 128;
                        const size_t o = (size_t)(m0 + i) * p.out_stride + n;
                        if (p.out_bf16) {
#pragma unroll
                            for (int c = lane; c < 64; c += 32)
                                if (n + c < p.N)
                                    static_cast<__nv_bfloat16*>(p.out)[o + c] = reinterpret_cast<const __nv_bfloat16*>(row + ((c >> 3) ^ (i & 7)) * 16)[c & 7];
                        } else if (n + lane < p.N) {
                            static_cast<float*>(p.out)[o + lane] = reinterpret_cast<const float*>(row + ((lane >> 2) ^ (i & 7)) * 16)[lane & 3];
                        }
                    }
                    __syncwarp();
                }
            }
        }
        if (lane == 0) tma_store_done();
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();                                    // nobody reaches into a CTA that has ended
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kColumns));
}

template <int BN, int NS>
int launch_pairs(Ctx* ctx, const MatmulParams& p, cudaStream_t stream) {
    using L = PairShape<BN, NS>;
    const long long nt = (p.N + BN - 1) / BN, tiles = nt * ((p.M + 255) / 256);
    const int pairs = sm_count(ctx) / 2;
    if (tiles > (1 << 27)) return SKETCHSSM_UNSUPPORTED_SHAPE;
    PairArgs g;
    g.p = p;
    g.n_tiles = (int)nt;
    g.tiles = (int)tiles;
    const int size = p.out_bf16 ? 2 : 4;
    g.tma_out = (p.out_stride * size) % 16 == 0 && (p.N * (long long)size) % 16 == 0;     // (a store ends on 16 bytes of a row)
    if (!make_map(&g.ta, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.a, (uint64_t)p.K, (uint64_t)p.M, (uint64_t)p.K, 128) ||
        !make_map(&g.tw, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.w, (uint64_t)p.K, (uint64_t)p.N, (uint64_t)p.K, BN / 2) ||
        (g.tma_out && !make_map(&g.to, p.out_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, size, p.out, (uint64_t)p.N,
                                (uint64_t)p.M, (uint64_t)p.out_stride * size, 32))) {
        ctx->last_cuda_error = cudaErrorInvalidValue;
        return SKETCHSSM_CUDA_ERROR;
    }
    const auto kern = integer_matmul_pair_kernel<BN, NS>;
    const cudaError_t e = unlock_smem(ctx, kern);
    if (e != cudaSuccess) { ctx->last_cuda_error = e; return SKETCHSSM_CUDA_ERROR; }
    const int grid = 2 * (int)(tiles < pairs ? tiles : pairs);
    return launch_layer<PairArgs>(ctx, kern, dim3((unsigned)grid), dim3(L::kThreads), L::kSmem, stream, g, 2);
}

}  // namespace

int launch_integer_matmul_pair(Ctx* ctx, const MatmulParams& p, cudaStream_t stream) {
    // From where the other kernel's 128 x 128 tiles are more than the SMs, so that some of them would take two.  (256 x 9472 x 2048, 148 such tiles:
    // 11.0 us there, 11.9 here; 256 x 9600, 150 of them, 15.3 and 11.8; 777 x 2049 x 4096, 119, 14.7 and 19.6; 4096 x 2048 x 4096, 512, 45.4
    // and 28.2.)
    const long long small = (long long)((p.N + 127) / 128) * ((p.M + 127) / 128);
    if (small > sm_count(ctx)) return launch_pairs<256, 5>(ctx, p, stream);
    // Down to half as many, pairs with tiles of 256 x 128, one each, bring a quarter fewer operands than two tiles there, but their stores are slower
    // where rows are no whole 16 bytes.  (300 x 4096 x 2048: 10.1 us there, 9.3 here; 640 x 2048 x 4096 14.6 and 13.7; 256 x 9472 x 2048 11.6
    // and 11.0; 777 x 2049 x 4096 14.9 and 16.7.  Fewer tiles are split there.)
    const int size = p.out_bf16 ? 2 : 4;
    const long long wide = (long long)((p.N + 127) / 128) * ((p.M + 255) / 256);
    if (2 * small > sm_count(ctx) && 2 * wide <= sm_count(ctx) && (p.out_stride * size) % 16 == 0 && (p.N * (long long)size) % 16 == 0)
        return launch_pairs<128, 7>(ctx, p, stream);
    return SKETCHSSM_UNSUPPORTED_SHAPE;
}

}  // namespace sketchssm
