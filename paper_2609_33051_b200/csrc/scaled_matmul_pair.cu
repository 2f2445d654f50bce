// The 8-bit product of scaled_matmul.cu for many rows: tiles of 256 tokens x 256 weights on pairs of SMs (tcgen05, cta_group::2).
//
// What bounds it: an SM's tensor cores take a block of 128 x 256 x 128 in about 500 cycles, in which a single CTA would have to
// bring 48 KB of operands from L2; 148 SMs doing that ask for more than L2 gives (about 10 TB/s: 321 us of copies alone for
// 16384 x 8512 x 2048).  A pair shares the weights, half of them in either SM: 32 KB a block.  And here the tokens are the
// accumulator's lanes, the weights its columns (the other way round than for few tokens): a thread's scale is one number a block,
// where scales read per column from shared memory, which the operands keep busy, made the sums 1700 cycles a block.
//
// Roles per CTA: one thread issues the copies of its half (they report to the leader's barrier), one warp of the leader the products
// (an elected lane of the converged warp: from a branch that one lane takes, an issue takes 95 cycles and a block 600); two warps
// fetch scales, eight blocks at a time; sixteen warps add a block's accumulator (32 lanes, 64 columns each), times its scale, to
// sums in registers and at the end store them through shared memory (TMA), or directly where a row or the row stride is no
// multiple of 16 bytes.  They release an accumulator with an arrival at the leader's barrier of the default (CTA) scope: reads of
// tensor memory are ordered by the tcgen05 fences, and a release of cluster scope waited 900 cycles for the stores before it.
#include "tma.cuh"

namespace sketchssm {

namespace {

using namespace tc;

constexpr int kStages = 4, kEpiWarps = 16, kThreads = 32 * (4 + kEpiWarps);
constexpr int kScaleBlocks = 8;                        // blocks whose scales are fetched together, in two buffers
constexpr uint32_t kHalf = 128u * 128u, kStageBytes = 2u * kHalf;
constexpr uint32_t kOut = kStages * kStageBytes, kScales = kOut + kEpiWarps * 4096u;
constexpr uint32_t kScaleBuf = kScaleBlocks * 130u;    // floats: 128 tokens and two column blocks of each
constexpr uint32_t kBars = kScales + 2u * kScaleBuf * 4u;
constexpr uint32_t kSmem = kBars + (2 * kStages + 8) * 8u + 16u + 1024u;

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
__global__ void __launch_bounds__(kThreads, 1) scaled_matmul_pair_kernel(const __grid_constant__ PairArgs g) {
    extern __shared__ unsigned char raw[];
    unsigned char* smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + kBars);        // the leader's: both halves are there
    uint64_t *empty = full + kStages, *acc_full = empty + kStages, *acc_empty = acc_full + 2;     // acc_empty: the leader's
    uint64_t *sc_full = acc_empty + 2, *sc_empty = sc_full + 2;
    uint32_t* slot = reinterpret_cast<uint32_t*>(sc_empty + 2);
    float* scales = reinterpret_cast<float*>(smem + kScales);
    const MatmulParams& p = g.p;
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = (int)blockIdx.x & 1, first = (int)blockIdx.x >> 1, step = (int)gridDim.x >> 1;
    if (tid == 64) { prefetch_map(&g.ta); prefetch_map(&g.tw); }
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(acc_full + i, 1); mbar_init(acc_empty + i, 2 * kEpiWarps); mbar_init(sc_full + i, 2); mbar_init(sc_empty + i, kEpiWarps); }
        mbar_fence_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(slot)) : "memory");
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
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (lane == 0) {
            int it = 0;
            bool ok = true;
            for (int tile = first; tile < g.tiles && ok; tile += step) {
                const int m = tile / g.n_tiles * 256 + rank * 128, n = tile % g.n_tiles * 256 + rank * 128;
                for (int kb = 0; kb < p.KB; ++kb, ++it) {
                    const int s = it % kStages;
                    if (it >= kStages && !mbar_wait_bounded(empty + s, (it / kStages - 1) & 1)) {
                        record_fault(p.status, kFaultMatmulWait, 11);
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
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (rank == 0) {
            constexpr uint32_t idesc = (1u << 4) | ((256u >> 3) << 17) | ((256u >> 4) << 24);      // e4m3 x e4m3 -> fp32
            int it = 0;
            bool ok = true;
            for (int tile = first; tile < g.tiles && ok; tile += step) {
                for (int kb = 0; kb < p.KB; ++kb, ++it) {
                    const int s = it % kStages, as = it & 1;
                    ok = it < 2 || warp_wait(acc_empty + as, (it / 2 - 1) & 1);
                    ok = ok && warp_wait(full + s, (it / kStages) & 1);
                    if (!ok) {
                        if (lane == 0) record_fault(p.status, kFaultMatmulWait, 12);
                        break;
                    }
                    tc_fence_after();
                    const uint32_t base = smem_u32(smem) + (uint32_t)s * kStageBytes;
                    const uint64_t da = swizzled_desc(base, 16u, 1024u), dw = swizzled_desc(base + kHalf, 16u, 1024u);
#pragma unroll
                    for (int j = 0; j < 4; ++j)        // 32 bytes of every row at a time
                        if (elect())
                            asm volatile(
                                "{\n\t.reg .pred p;\n\t"
                                "setp.ne.b32 p, %4, 0;\n\t"
                                "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem + (uint32_t)(as * 256)),
                                "l"(da + 2u * j), "l"(dw + 2u * j), "r"(idesc), "r"((uint32_t)j)
                                : "memory");
                    if (elect()) {
                        commit_pair(empty + s);
                        commit_pair(acc_full + as);
                    }
                    __syncwarp();
                }
            }
        }
        __syncwarp();
    } else if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        // Scales: eight blocks of 128 tokens and two column blocks, all loads of a group under way together.
        constexpr int kEach = kScaleBlocks * 128 / 64;
        const int t = tid - 64;
        int group = 0;
        bool ok = true;
        for (int tile = first; tile < g.tiles && ok; tile += step) {
            const int m0 = tile / g.n_tiles * 256 + rank * 128, nb0 = tile % g.n_tiles * 2;
            for (int kb0 = 0; kb0 < p.KB; kb0 += kScaleBlocks, ++group) {
                float v[kEach], w = 0.f;
                const int kb = kb0 + t % kScaleBlocks;
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    const int m = m0 + i * (64 / kScaleBlocks) + t / kScaleBlocks;
                    v[i] = m < p.M && kb < p.KB ? p.a_scale[(size_t)m * p.KB + kb] : 0.f;
                }
                if (t < 2 * kScaleBlocks && kb < p.KB && (nb0 + t / kScaleBlocks) * 128 < p.N)
                    w = p.w_scale[(size_t)(nb0 + t / kScaleBlocks) * p.KB + kb];
                ok = group < 2 || mbar_wait_bounded(sc_empty + (group & 1), (group / 2 - 1) & 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) {
                    if (lane == 0) record_fault(p.status, kFaultMatmulWait, 14);
                    break;
                }
                float* sc = scales + (group & 1) * kScaleBuf + t % kScaleBlocks * 130;
#pragma unroll
                for (int i = 0; i < kEach; ++i) sc[i * (64 / kScaleBlocks) + t / kScaleBlocks] = v[i];
                if (t < 2 * kScaleBlocks) sc[128 + t / kScaleBlocks] = w;
                __syncwarp();
                if (lane == 0) mbar_arrive_one(sc_full + (group & 1));
            }
        }
    } else {
        // (640 threads start with 96 registers: 128 x 56 + 512 x 104 of 61440)
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        const int quad = warp & 3, part = (warp - 4) >> 2;             // 32 lanes, 64 columns
        const uint32_t at0 = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(part * 64);
        unsigned char* stage = smem + kOut + (uint32_t)(warp - 4) * 4096u;
        const uint32_t release = cluster_addr(acc_empty, 0);
        int it = 0, group = 0;
        bool ok = true;
        uint64_t acc[32];
        for (int tile = first; tile < g.tiles && ok; tile += step) {
#pragma unroll
            for (int c = 0; c < 32; ++c) acc[c] = 0ull;
            for (int kb = 0; kb < p.KB; ++kb, ++it) {
                if (kb % kScaleBlocks == 0) {
                    ok = mbar_wait_bounded(sc_full + (group & 1), (group >> 1) & 1);
                    ++group;
                }
                const float* sc = scales + ((group - 1) & 1) * kScaleBuf + kb % kScaleBlocks * 130;
                const int as = it & 1;
                ok = ok && mbar_wait_bounded(acc_full + as, (it / 2) & 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) {
                    if (lane == 0) record_fault(p.status, kFaultMatmulWait, 13);
                    break;
                }
                tc_fence_after();
                const float s = sc[quad * 32 + lane] * sc[128 + (part >> 1)];
                const uint64_t s2 = pack2(s, s);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t d[32];
                    tmem_ld32_async(at0 + (uint32_t)(as * 256 + c * 32), d);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        acc[c * 16 + j] = fma2(pack2(__uint_as_float(d[2 * j]), __uint_as_float(d[2 * j + 1])), s2, acc[c * 16 + j]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(release + 8u * (uint32_t)as) : "memory");
                    if (kb % kScaleBlocks == kScaleBlocks - 1 || kb == p.KB - 1) mbar_arrive_one(sc_empty + ((group - 1) & 1));
                }
            }
            const int m0 = tile / g.n_tiles * 256 + rank * 128 + quad * 32, n0 = tile % g.n_tiles * 256 + part * 64;
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
                        for (int j = 0; j < 4; ++j) unpack2(acc[c * 4 + j], f[2 * j], f[2 * j + 1]);
                        u = Vec16<__nv_bfloat16>::pack(f);
                    } else {
                        const uint64_t lo = acc[r * 16 + c * 2], hi = acc[r * 16 + c * 2 + 1];
                        u = make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
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
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

}  // namespace

int launch_scaled_matmul_pair(Ctx* ctx, const MatmulParams& p, cudaStream_t stream) {
    const long long nt = (p.N + 255) / 256, tiles = nt * ((p.M + 255) / 256);
    const int pairs = sm_count(ctx) / 2;
    // From where the other kernel's 128 x 128 tiles are more than the SMs, so that some of them would take two.  (Inner axis 2048: 256 x 9472,
    // 148 such tiles, 11.5 us there and 12.8 here; 256 x 11264, 176 of them, 18.6 and 13.2; 1024 x 2304, 144, 11.3 and 12.9; 1024 x 3328,
    // 208, 19.0 and 13.4.)
    const long long small = (long long)((p.N + 127) / 128) * ((p.M + 127) / 128);
    if (small <= sm_count(ctx) || tiles > (1 << 27)) return SKETCHSSM_UNSUPPORTED_SHAPE;
    PairArgs g;
    g.p = p;
    g.n_tiles = (int)nt;
    g.tiles = (int)tiles;
    const int size = p.out_bf16 ? 2 : 4;
    g.tma_out = (p.out_stride * size) % 16 == 0 && (p.N * (long long)size) % 16 == 0;     // (a store ends on 16 bytes of a row)
    if (!make_map(&g.ta, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.a, (uint64_t)p.K, (uint64_t)p.M, (uint64_t)p.K, 128) ||
        !make_map(&g.tw, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.w, (uint64_t)p.K, (uint64_t)p.N, (uint64_t)p.K, 128) ||
        (g.tma_out && !make_map(&g.to, p.out_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, size, p.out, (uint64_t)p.N,
                                (uint64_t)p.M, (uint64_t)p.out_stride * size, 32))) {
        ctx->last_cuda_error = cudaErrorInvalidValue;
        return SKETCHSSM_CUDA_ERROR;
    }
    const cudaError_t e = unlock_smem(ctx, scaled_matmul_pair_kernel);
    if (e != cudaSuccess) { ctx->last_cuda_error = e; return SKETCHSSM_CUDA_ERROR; }
    const int grid = 2 * (int)(tiles < pairs ? tiles : pairs);
    return launch_layer<PairArgs>(ctx, scaled_matmul_pair_kernel, dim3((unsigned)grid), dim3(kThreads), kSmem, stream, g, 2);
}

}  // namespace sketchssm
