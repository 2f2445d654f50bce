// Gated delta rule over packed prompts on tcgen05 + TMEM: GDN, bf16 tensors, K = V = 128.
//
// A sequence goes through in chunks of 64 tokens.  With c_t the sum of the chunk's log2 decays up to token t, unit keys k (a key as it is times
// r_t) and S the state before the chunk, what the tokens add is U, the solution of a unit lower triangular system:
//     U = diag(beta) T X,   T = (I + L)^-1,   L[t][s] = 2^(c_t - c_s) <k_t, k_s> beta_s for s < t,   X[t] = v_t - 2^c_t S^T k_t
//     Y[t] = 2^c_t S^T q_t + sum_{s <= t} P[t][s] U[s],   P[t][s] = 2^(c_t - c_s) <q_t, k_s>
//     S <- 2^c_end S + sum_s 2^(c_end - c_s) k_s U[s]^T
// T and P do not depend on the state: a first kernel makes them, all chunks at once, and leaves them in the scratch as
// matrix operands; a second one takes a sequence and head at a time through its chunks.
//
// There the state is kept transposed: 128 value columns are the lanes of tensor memory, so that everything a chunk reads of it is one
// operand in tensor memory times a tile of shared memory (keys, queries, T, P), and a lane's thread scales, adds and splits without
// another thread's help.  Per chunk: K S^T and, later, Q S^T;  X;  (T - I) X;  U and W = 2^(c_end - c) r U;  W K and U P;  S.
//
// Precision.  States are fp32, outputs sums of fp32 accuracy rounded once.  What the tensor cores multiply are fp16 operands in two parts of 11
// bits each (the product of the second parts is left out), summed in fp32.  fp16 has the bits but not the range, so everything is scaled by
// powers of two, which round nothing: keys and queries by one each, to lengths between a half and one (then one part holds all of their bits
// but those below 2^-24 of the length), and a lane's state, X, U and W by one for the lane and chunk, from the largest value v in it and the length
// of the state before it.  A token leaves the state's squared length at most at d^2 |S|^2 + v^2 (a convex mean along its key), a chunk at 2^(2 c_end) |S|^2
// + 64 v^2, which bounds it from where it was measured on; so |U| is at most 9 v + |S|, |W| twice that, and is brought below 2^15.  T and P are at most
// one as they are, T because the rows' step sizes are left to U (a part ends at 2^-24, and rows of small ones would lose their bits: with
// b = -7 everywhere states were 4e-5 off), and are made kTile times as large, so that what has decayed to 2^-25 of a large value ends there, and not
// that of one.  In bf16 the same accuracy took three parts, half as many products again and more than twice the time to split.
// Sums of log decays are made in 64 bits and kept as a whole number and a rest of at most a half.
//
// What bounds it.  The second kernel: a chunk's chain of products and of the warps' work between them, 3.0 to 3.3 us of which the products are less
// than a third; a sequence's chunks follow one another.  16384 tokens of 32 heads (SM clock 1965 MHz): one prompt 604 us (126 the first kernel; 291, 22
// and 160 the passes over five segments, see decode_unit; 881 whole), 48 ragged prompts 450 to 464 by their lengths.  The warp that lays out V needs
// nearly as long for a chunk as the chain: without its look at the sizes the passes take 274 and 152.  The first kernel: waiting, for loads
// and for its own warps, and memory, of which it reads and writes 0.45 GB (3.6 TB/s).  100 tokens: 24 us, half of it the first kernel.
#include "tma.cuh"

#include <cuda_fp16.h>

#include <utility>

namespace sketchssm {

namespace {

using namespace tc;

constexpr int kQ = 64;                                 // tokens of a chunk
constexpr uint32_t kPart = 8192u;                      // 64 rows of 128 bytes
constexpr float kTile = 16384.f;                       // factor of T and P
// The scratch: for a chunk of a head two parts of T - I, two of P and the gates; for one of a group the rows of K and Q, half of the channels at a time
constexpr uint32_t kTOff = 0, kPOff = 2 * kPart, kGOff = 4 * kPart, kRows = 4 * kPart;
// gates, 64 floats each: beta, -2^c r, 2^(c_end - c) r, 2^c kTile / |q| (r and 1 / |q| of the scaled rows), and 2^c_end and whether no beta is below kLeastBeta
constexpr int kBeta = 0, kRead = 64, kPut = 128, kAsk = 192, kKeep = 256, kPlain = 257, kGates = 320;
// behind them, and not copied with them: a token's decay, r and 1 / |q|, for chunks taken token by token
constexpr int kDecay = kGates, kKey = kGates + 64, kQuery = kGates + 128, kFloats = kGates + 192;
constexpr uint32_t kCopied = kGOff + kGates * 4u, kBlock = kGOff + kFloats * 4u;

// Numbers of very different size.  A column's scale is its chunk's largest; an operand is 2^-25 off at that scale where it is small, so a token keeps the
// accuracy of its own column's numbers only while those, scaled, stay above some floor: the larger one of its value and the one before it (whose
// weight the state has), or what earlier ones and the state were, less what has decayed since; and no value counts that beta keeps out.  Where they
// do not (a value or a state 2^16 times as large as the others that a chunk meets, beta below 2^-12 throughout) the columns of a pair of warps go through
// the chunk token by token, in fp32, and the products meet zeros: 50 to 100 us instead of 3.  It is looked at where two neighbouring tokens are
// below the floor (of normal numbers one in ten million columns and chunks), or the state that a unit begins with, or a beta below kLeastBeta; a look
// takes 2 us, and 12 where nobody has run its instructions lately.
// (The floor: 2^-25 is 2^-18 of it, and what shows of it in outputs and states, measured where there was no floor, a twentieth of that: the tests' bound
// is 2^-18.7.  With a floor of 1 / 32 there were looks in one of four calls of 16384 tokens.)
constexpr float kFloor = 1.f / 128.f, kLeastBeta = 1.f / 4096.f;

struct DeltaArgs {
    CUtensorMap tq, tk, tv;
    DeltaParams p;
    // of the scratch, behind the heads' blocks: rows of K and Q; sequences by their lengths; states between segments
    unsigned char* rows;
    int* order;
    float* states;
    int units, preps;
    int segments, turns, pass; // parts that a sequence is split into; units of the first pass a CTA; 0: whole ones, 1, 2: see decode_unit
};

// What a CTA of the second kernel takes at a time: a sequence and head, or a segment of one.
struct Unit {
    int t0, t1;                // rows
    int seq, head, chunk;      // chunk: of the first row, in the scratch
    int seg, kind;             // kWhole and kFirst begin with the stored state, kLater with the segment's, kAlone with zeros, kMap with the unit matrix
    bool outputs;
};
enum { kWhole, kFirst, kLater, kAlone, kMap };

// The first chunk of sequence i in the scratch: chunks of sequences that follow one another never meet, whatever their lengths are.
__device__ __forceinline__ int chunk_base(int row0, int i) { return row0 / kQ + i; }

// Unit number `it` of this CTA.  Whole sequences go out in the order of their lengths, the longest first, to and fro over the CTAs.
// Few sequences and heads leave most of the card idle for as long as the longest takes.  Then a sequence is split into n segments.  What
// a segment makes of a state is linear: S <- M S + N.  The first pass takes the first segment with its outputs, and of each that others follow N
// (from a state of zeros) and M (from the unit matrix, without values); a small kernel goes through them, and the second pass takes
// all others from the states that they begin with.  In the first pass a CTA takes a first segment, or `turns` of the other units, and the first
// segment is that many times as long.
__device__ __forceinline__ bool decode_unit(const DeltaArgs& g, int it, Unit& x) {
    const DeltaParams& p = g.p;
    const int G = (int)gridDim.x, i = (int)blockIdx.x;
    int u;
    x.kind = kWhole;
    x.seg = 0;
    if (g.pass == 1) {
        const int pairs = p.pr.N * p.H;
        if (i < pairs) {
            if (it > 0) return false;
            x.kind = kFirst;
            u = i;
        } else {
            const int k = (i - pairs) * g.turns + it;
            if (it >= g.turns || k >= g.units) return false;
            x.kind = (k & 1) ? kMap : kAlone;
            x.seg = k / 2 / pairs + 1;
            u = k / 2 % pairs;
        }
    } else {
        const int k = it * G + ((it & 1) ? G - 1 - i : i);
        if (k >= g.units) return false;
        u = k;
        if (g.pass == 2) {
            x.kind = kLater;
            x.seg = k % (g.segments - 1) + 1;
            u = k / (g.segments - 1);
        }
    }
    x.head = u % p.H;
    x.seq = u / p.H;
    if (g.order != nullptr) x.seq = min(max(g.order[x.seq], 0), p.pr.N - 1);
    x.outputs = x.kind <= kLater;
    const int2 rows = seq_rows(p.pr, x.seq);
    const int chunks = (rows.y - rows.x + kQ - 1) / kQ;
    if (g.pass == 0) {
        x.t0 = rows.x;
        x.t1 = rows.y;
        x.chunk = chunk_base(rows.x, x.seq);
    } else {
        const int all = g.turns + g.segments - 1, per = (chunks + all - 1) / all, first = x.seg == 0 ? 0 : (g.turns + x.seg - 1) * per;
        x.t0 = (int)min((long long)rows.y, rows.x + (long long)first * kQ);
        x.t1 = (int)min((long long)rows.y, x.t0 + (long long)(x.seg == 0 ? g.turns * per : per) * kQ);
        x.chunk = chunk_base(rows.x, x.seq) + first;
    }
    return true;
}
// The stored state before the unit, and whether it is one (not zeros).
__device__ __forceinline__ bool has_state(const DeltaArgs& g, const Unit& x) {
    return x.kind >= kLater ? x.kind != kAlone : seq_resume(g.p.pr, x.seq) >= 0;
}
// State i of a sequence and head in the scratch: before segments 1 .. n - 1; then N and M of segments 1 .. n - 2.
__device__ __forceinline__ float* scratch_state(const DeltaArgs& g, int seq, int head, int i) {
    return g.states + (((size_t)seq * g.p.H + head) * (3 * g.segments - 5) + i) * 128 * 128;
}

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
__device__ __forceinline__ uint32_t half_pair(float a, float b) {
    __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
}
// Two floats as two parts of fp16 each: what the first leaves, rounded, is the second.  (The mixed multiply-add takes the halves as they are;
// brought back to fp32 first, two conversions on the same pipe, they cost three times as much.)
__device__ __forceinline__ void two_parts(uint64_t x, uint32_t& hi, uint32_t& lo) {
    float a, b, c, d;
    unpack2(x, a, b);
    hi = half_pair(a, b);
    asm("{\n\t.reg .b16 h, l, m;\n\tmov.b32 {l, h}, %2;\n\tmov.b16 m, 0xBC00;\n\t"
        "fma.rn.f32.f16 %0, l, m, %3;\n\tfma.rn.f32.f16 %1, h, m, %4;\n\t}"
        : "=f"(c), "=f"(d)
        : "r"(hi), "f"(a), "f"(b));
    lo = half_pair(c, d);
}
__device__ __forceinline__ void bulk_s2g(void* dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_u32(src)), "r"(bytes) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}

constexpr uint32_t kTypes = (1u << 4) | ((128u >> 4) << 24);      // fp16 x fp16 -> fp32, 128 rows

// ---- what does not depend on the state: T and P of every chunk ------------------------------------------------------------
//
// A CTA takes a chunk, a group and two of its heads.  The gates' arguments, 64 rows far apart, are what it waits for longest: they are used behind the
// norms only.  The rows of K and Q are scaled to fp16 in place (and kept for the second kernel).  One product
// gives <k_t, k_s> (lanes 0..63) and <q_t, k_s> (64..127).  Of four warps a head, two make P from the latter and store it, two make -L and from
// it T, in blocks of sixteen by sixteen: D_b, the inverses of the diagonal ones, column by column, a column a thread, all four at once; then
//     T[b][c] = D_b sum_{c <= e < b} -L[b][e] T[e][c],   T[b][b] = D_b,
// transposed, so that what one product leaves in registers is the next one's first operand (mma.sync, in two parts as above: operands of this
// size are in registers before a tcgen05 product could be set up).  (All of it column by column is as many multiply-adds on CUDA
// cores, but their second operands, broadcast from shared memory at 128 bytes a cycle, were most of 160 us for 16384 tokens of 32 heads.)

constexpr int kPrepThreads = 256;
// behind the tile of K and Q rows, whose place -L of both heads takes (two parts, rows t), then T: the diagonal blocks of -L, [4][s][t] floats
// a head; their inverses, [4][2 parts][t][s]; 1 / |k|, 1 / |q|, and 1 / |k| or zero: [3][64]; halves of their squares; whole, rest, beta: [2][3][64]; beta / |k|: [2][64]
constexpr uint32_t kPrepDiag = 4 * kPart, kPrepInv = kPrepDiag + 2u * 4096u;
constexpr uint32_t kPrepNorm = kPrepInv + 2u * 4096u, kPrepHalf = kPrepNorm + 3u * kQ * 4u, kPrepSum = kPrepHalf + 4u * kQ * 4u;
constexpr uint32_t kPrepPut = kPrepSum + 6u * kQ * 4u, kPrepBar = kPrepPut + 2u * kQ * 4u;
constexpr uint32_t kPrepSmem = kPrepBar + 32u + 1024u;

// Element S of sixteen neighbouring ones of a column puts -L[t][s] of itself into those behind it: l holds their block of -L, [s][t].
template <int S>
__device__ __forceinline__ void take_near(uint64_t (&T)[8], const float* l) {
    float a, b;
    unpack2(T[S / 2], a, b);
    const float ts = S % 2 ? b : a;
    const uint64_t ts2 = pack2(ts, ts);
    if constexpr (S % 2 == 0) T[S / 2] = pack2(a, fmaf(l[S * 16 + S + 1], ts, b));
    constexpr int first = S / 2 + 1;                    // the first pair behind S
    if constexpr (first % 2 == 1) T[first] = fma2(*reinterpret_cast<const uint64_t*>(l + S * 16 + 2 * first), ts2, T[first]);
#pragma unroll
    for (int i = (first + 1) / 2; i < 4; ++i) {
        const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(l + S * 16 + 4 * i);
        T[2 * i] = fma2(v.x, ts2, T[2 * i]);
        T[2 * i + 1] = fma2(v.y, ts2, T[2 * i + 1]);
    }
}
template <int... I>
__device__ __forceinline__ void take_fifteen(uint64_t (&T)[8], const float* l, std::integer_sequence<int, I...>) { (take_near<I>(T, l), ...); }

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void stmatrix4_trans(uint32_t at, const uint32_t (&r)[4]) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void mma_block(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// c (16 x 16, two tiles of 8 columns) += a b^T: a in two parts, of b two parts of sixteen rows of sixteen.
__device__ __forceinline__ void mma_sixteen(float (&c)[2][4], const uint32_t (&hi)[4], const uint32_t (&lo)[4], uint32_t b_hi, uint32_t b_lo) {
    uint32_t bh[4], bl[4];                              // (first eight rows: both halves of their columns; the other eight)
    ldmatrix4(bh, b_hi);
    ldmatrix4(bl, b_lo);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        mma_block(c[i], hi, bh[2 * i], bh[2 * i + 1]);
        mma_block(c[i], hi, bl[2 * i], bl[2 * i + 1]);
        mma_block(c[i], lo, bh[2 * i], bh[2 * i + 1]);
    }
}
// What a product leaves as the first operand of the next: both of its operands are kTile times what they stand for, and so is this one.  (It is at most
// one: what a key reads of the state that a value of one has left.)
__device__ __forceinline__ void as_operand(const float (&c)[2][4], uint32_t (&hi)[4], uint32_t (&lo)[4]) {
    const uint64_t back = pack2(1.f / kTile, 1.f / kTile);
#pragma unroll
    for (int i = 0; i < 4; ++i) two_parts(mul2(pack2(c[i >> 1][(i & 1) * 2], c[i >> 1][(i & 1) * 2 + 1]), back), hi[i], lo[i]);
}
// Byte of element (row, column) of a part: rows of 128 bytes in the 128-byte swizzle.
__device__ __forceinline__ uint32_t at_swizzled(int row, int col) { return (uint32_t)(row * 128 + (((col >> 3) ^ (row & 7)) * 16) + (col & 7) * 2); }

__global__ void __launch_bounds__(kPrepThreads, 3) delta_prep_kernel(const __grid_constant__ DeltaArgs g) {
    extern __shared__ unsigned char raw[];
    unsigned char* smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    float* norms = reinterpret_cast<float*>(smem + kPrepNorm);
    float *sums = reinterpret_cast<float*>(smem + kPrepSum), *puts = reinterpret_cast<float*>(smem + kPrepPut);
    uint64_t* bar = reinterpret_cast<uint64_t*>(smem + kPrepBar);
    uint32_t* slot = reinterpret_cast<uint32_t*>(bar + 2);
    const DeltaParams& p = g.p;
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int per = p.H / p.G, batches = (per + 1) / 2;
    int u = (int)blockIdx.x;
    if (u == g.preps) {                                  // (one CTA more: every sequence's place by its number of chunks)
        grid_dep_wait();
        grid_dep_launch_dependents();
        // (sorted by counting: a length's exponent and first three bits are its class; which of a class comes first is left open, and changes nothing
        // but the time)
        int* count = reinterpret_cast<int*>(smem);
        auto place = [&](int i) {
            const int2 rows = seq_rows(p.pr, i);
            const int chunks = (rows.y - rows.x + kQ - 1) / kQ;
            return kPrepThreads - 1 - (chunks > 0 ? min((int)(__float_as_uint((float)chunks) >> 20) - (127 << 3) + 1, kPrepThreads - 1) : 0);
        };
        count[tid] = 0;
        __syncthreads();
        for (int i = tid; i < p.pr.N; i += kPrepThreads) atomicAdd(count + place(i), 1);
        __syncthreads();
        const int mine = count[tid];
        int before = mine;                               // of the classes up to this one
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, before, o);
            if (lane >= o) before += up;
        }
        int* totals = count + kPrepThreads;
        if (lane == 31) totals[warp] = before;
        __syncthreads();
        for (int w = 0; w < warp; ++w) before += totals[w];
        count[tid] = before - mine;
        __syncthreads();
        for (int i = tid; i < p.pr.N; i += kPrepThreads) g.order[min(atomicAdd(count + place(i), 1), p.pr.N - 1)] = i;
        return;
    }
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
    auto not_behind = [&](int j, int end) { return __popc(__ballot_sync(0xffffffffu, j < end && chunk_base(seq_start(p.pr, min(j, p.pr.N - 1)), j) <= chunk)); };
    int n = 0, end = p.pr.N;                             // (n of them are not behind it, those from `end` on are)
    while (end - n > 32) {
        const int step = (end - n + 31) / 32, m = not_behind(n + (lane + 1) * step - 1, end);
        n += m * step;
        end = min(end, n + step);
    }
    n += not_behind(n + lane, end);
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
        const int mine = warp >> 2, role = warp & 3;     // this warp's head of the two; what it does for it
        // the gates' arguments: a warp a head, two neighbouring tokens a lane (asked for here, and used behind the norms)
        float x[2] = {0.f, 0.f}, y[2] = {0.f, 0.f}, a2 = 0.f, bias = 0.f;
        if (role == 0 && mine < heads) {
            const int h = h0 + mine;
            a2 = p.a[h] * 1.4426950408889634f;
            bias = p.dt_bias != nullptr ? p.dt_bias[h] : 0.f;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (lane * 2 + i < valid) {
                    const long long r = t0 + lane * 2 + i;
                    x[i] = __bfloat162float(static_cast<const __nv_bfloat16*>(p.b)[r * p.b_stride + h]);
                    y[i] = __bfloat162float(static_cast<const __nv_bfloat16*>(p.dt)[r * p.dt_stride + h]);
                }
        }
        ok = mbar_wait_bounded(bar, 0);
        ok = __syncthreads_and(ok) != 0;
        // norms: half a row of K or Q a thread, which it then scales; rows behind the sequence are zeros
        if (ok) {
            const int r = tid & 127;
            unsigned char* row = smem + (tid >> 7) * 2 * kPart + r * 128;
            float* halves = reinterpret_cast<float*>(smem + kPrepHalf);
            uint64_t sq[4] = {0ull, 0ull, 0ull, 0ull};
            uint4 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = *reinterpret_cast<const uint4*>(row + ((i ^ (r & 7)) * 16));
                float f[8];
                Vec16<__nv_bfloat16>::unpack(v[i], f);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint64_t x = pack2(f[2 * e], f[2 * e + 1]);
                    sq[e] = fma2(x, x, sq[e]);
                }
            }
            float even, odd;
            unpack2(add2(add2(sq[0], sq[1]), add2(sq[2], sq[3])), even, odd);
            halves[tid] = even + odd;
            __syncthreads();
            const float inv = inv_length(halves[r] + halves[r + 128], p.eps), scale = __uint_as_float(__float_as_uint(inv) & 0x7f800000u);
            const bool fine = inv == inv;                // (a row that is not finite: zeros, and a factor that is not a number)
            if (tid < 128) norms[r] = fine ? inv / scale : inv;
            if (tid < 64) norms[128 + r] = fine ? inv / scale : 0.f;
            const bool in = (r & 63) < valid && fine;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float f[8];
                Vec16<__nv_bfloat16>::unpack(v[i], f);
                uint32_t h[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) h[e] = in ? half_pair(f[2 * e] * scale, f[2 * e + 1] * scale) : 0u;
                *reinterpret_cast<uint4*>(row + ((i ^ (r & 7)) * 16)) = make_uint4(h[0], h[1], h[2], h[3]);
            }
            proxy_fence();
        }
        ok = __syncthreads_and(ok) != 0;
        if (tid == 64 && ok && batch == 0) bulk_s2g(g.rows + ((size_t)chunk * p.G + group) * kRows, smem, kRows);
        if (warp == 1 && ok) {
            const uint64_t da = swizzled_desc(smem_u32(smem), 16u, 1024u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint64_t at = da + (uint32_t)(i / 4) * (2 * kPart >> 4) + (uint32_t)(i % 4) * 2u;
                if (elect()) mma_ss(tmem, at, at, kTypes | ((64u >> 3) << 17), i > 0);
            }
            if (elect()) tc_commit(bar + 1);
            __syncwarp();
        }
        // gates, while the product is made
        if (ok && role == 0 && mine < heads) {
            float *s = sums + mine * 3 * kQ, *put = puts + mine * kQ;
            bool plain = true;
            double c[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bool in = lane * 2 + i < valid;
                float l = a2 * softplus(y[i] + bias);
                if (l < -160.f) l = -160.f;             // (2^-160 is zero in fp32; the bound keeps the sums finite)
                // What is not finite counts in beta, by which its token is known: sums, L and T stay finite, as products of sixteen rows
                // would carry it to the tokens before.
                float beta = 1.f / (1.f + expf(-x[i]));
                if (!(l <= 3.4028235e38f)) {
                    l = 0.f;
                    beta = __int_as_float(0x7fffffff);
                }
                s[2 * kQ + lane * 2 + i] = in ? beta : 0.f;
                put[lane * 2 + i] = in && beta == beta ? beta * norms[128 + lane * 2 + i] : 0.f;
                plain = plain && (!in || beta >= kLeastBeta);
                c[i] = (i > 0 ? c[0] : 0.0) + (double)(in ? l : 0.f);
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
            plain = __all_sync(0xffffffffu, plain);
            if (lane == 0) reinterpret_cast<float*>(p.work + ((size_t)chunk * p.H + h0 + mine) * kBlock + kGOff)[kPlain] = plain ? 1.f : 0.f;
        }
        ok = ok && mbar_wait_bounded(bar + 1, 0);
        if (tid == 64) tma_store_read();
        ok = __syncthreads_and(ok) != 0;                // (from here on the tile's place is -L's)
        // what the second kernel reads of the gates
        if (ok && role >= 2 && mine < heads) {
            const int t = tid & 63;
            const float *s = sums + mine * 3 * kQ, w = s[t], r = s[kQ + t];
            float* to = reinterpret_cast<float*>(p.work + ((size_t)chunk * p.H + h0 + mine) * kBlock + kGOff);
            const bool in = t < valid;
            const float e = exp2f(w) * exp2f(r), rest = exp2f(s[kQ - 1] - w) * exp2f(s[2 * kQ - 1] - r);
            to[kBeta + t] = s[2 * kQ + t];
            to[kRead + t] = in ? fmaf(s[2 * kQ + t], 0.f, -e * norms[t]) : 0.f;      // (not a number where beta is none: see the marks)
            to[kPut + t] = in ? rest * norms[t] : 0.f;
            to[kAsk + t] = in ? e * kTile * norms[64 + t] : 0.f;
            if (t == 63) to[kKeep] = e;
            to[kDecay + t] = exp2f((t > 0 ? w - s[t - 1] : w) + (t > 0 ? r - s[kQ + t - 1] : r));
            to[kKey + t] = in ? norms[t] : 0.f;
            to[kQuery + t] = in ? norms[64 + t] : 0.f;
        }
        if (ok && mine < heads) {
            tc_fence_after();
            const int t = tid & 63;
            const uint32_t lanes = (uint32_t)(role * 32) << 16;
            const uint64_t minus = pack2(-1.f, -1.f);
            const float* s = sums + mine * 3 * kQ;
            const uint64_t w = pack2(s[t], s[t]), r = pack2(s[kQ + t], s[kQ + t]);
            // tokens e0 .. e0 + 15 of the row: the product times the row's factor, the columns' and the decay between.  (Rows behind the sequence
            // are zeros as K's and Q's are.)
            auto tokens = [&](int e0, uint64_t factor, const float* columns, uint64_t (&x)[8]) {
                uint32_t d[16];
                tmem_ld16_async(tmem + lanes + e0, d);
                tmem_ld_wait();
                const ulonglong2 *w4 = reinterpret_cast<const ulonglong2*>(s + e0), *r4 = reinterpret_cast<const ulonglong2*>(s + kQ + e0),
                                 *n4 = reinterpret_cast<const ulonglong2*>(columns + e0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const ulonglong2 we = w4[i], re = r4[i], ne = n4[i];
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        float a, b;
                        unpack2(add2(fma2(q ? we.y : we.x, minus, w), fma2(q ? re.y : re.x, minus, r)), a, b);
                        const uint64_t f = mul2(mul2(factor, q ? ne.y : ne.x), pack2(__uint_as_float(d[4 * i + 2 * q]), __uint_as_float(d[4 * i + 2 * q + 1])));
                        x[2 * i + q] = mul2(f, pack2(ex2(a), ex2(b)));
                    }
                }
            };
            // sixteen tokens of row t, times kTile, in two parts
            auto put = [&](unsigned char* to, int e0, const uint64_t (&x)[8]) {
                uint32_t hi[8], lo[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) two_parts(mul2(x[i], pack2(kTile, kTile)), hi[i], lo[i]);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    unsigned char* at = to + t * 128 + (((e0 / 8 + q) ^ (t & 7)) * 16);
                    *reinterpret_cast<uint4*>(at) = make_uint4(hi[4 * q], hi[4 * q + 1], hi[4 * q + 2], hi[4 * q + 3]);
                    *reinterpret_cast<uint4*>(at + kPart) = make_uint4(lo[4 * q], lo[4 * q + 1], lo[4 * q + 2], lo[4 * q + 3]);
                }
            };
            // the same to memory, where a sector is written at once: two pieces of sixteen bytes, in the order that the swizzle gives them
            auto put_out = [&](unsigned char* to, int e0, const uint64_t (&x)[8]) {
                uint32_t h[2][8];
#pragma unroll
                for (int i = 0; i < 8; ++i) two_parts(x[i], h[0][i], h[1][i]);
                unsigned char* at = to + t * 128 + (((e0 / 8) ^ (t & 6)) * 16);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    uint32_t a[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) a[i] = (t & 1) ? h[e][i ^ 4] : h[e][i];
                    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at + e * kPart), "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]),
                                 "r"(a[4]), "r"(a[5]), "r"(a[6]), "r"(a[7])
                                 : "memory");
                }
            };
            unsigned char* block = p.work + ((size_t)chunk * p.H + h0 + mine) * kBlock;
            if (role >= 2) {
                const uint64_t factor = pack2(kTile * norms[64 + t], kTile * norms[64 + t]);
                const int last = 32 * (role & 1) + 32;   // (a warp's rows end there)
#pragma unroll 1
                for (int e0 = 0; e0 < last; e0 += 16) {  // (blocks above the diagonal are not read)
                    uint64_t x[8];
                    tokens(e0, factor, norms + 128, x);
                    if (e0 + 16 > last - 32) {           // (the diagonal is in these rows)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            float a, b;
                            unpack2(x[i], a, b);
                            x[i] = pack2(e0 + 2 * i <= t ? a : 0.f, e0 + 2 * i + 1 <= t ? b : 0.f);
                        }
                    }
                    if (e0 <= t) put_out(block + kPOff, e0, x);
                }
            } else {
                unsigned char* L = smem + mine * 2 * kPart;
                float* diag = reinterpret_cast<float*>(smem + kPrepDiag + mine * 4096);
                {
                    const float f = -norms[128 + t];
#pragma unroll 1
                    for (int e0 = 0; e0 < 32 * role + 32; e0 += 16) {
                        uint64_t x[8];
                        tokens(e0, pack2(f, f), puts + mine * kQ, x);      // (what it leaves on and above the diagonal nobody reads)
                        put(L, e0, x);
                        if (e0 == (t & 48)) {
                            float* to = diag + e0 * 16 + (t & 15);
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                float a, b;
                                unpack2(x[i], a, b);
                                to[2 * i * 16] = a;
                                to[(2 * i + 1) * 16] = b;
                            }
                        }
                    }
                }
                __syncwarp();
                // the inverses: this warp's two blocks, a column a lane
                {
                    const int blk = t >> 4, c = t & 15;
                    uint64_t x[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = pack2(2 * i == c ? 1.f : 0.f, 2 * i + 1 == c ? 1.f : 0.f);
                    take_fifteen(x, diag + blk * 256, std::make_integer_sequence<int, 15>{});
                    unsigned short* to = reinterpret_cast<unsigned short*>(smem + kPrepInv + mine * 4096 + blk * 1024) + c;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        uint32_t hi, lo;
                        two_parts(mul2(x[i], pack2(kTile, kTile)), hi, lo);
                        to[2 * i * 16] = (unsigned short)hi;
                        to[(2 * i + 1) * 16] = (unsigned short)(hi >> 16);
                        to[2 * i * 16 + 256] = (unsigned short)lo;
                        to[(2 * i + 1) * 16 + 256] = (unsigned short)(lo >> 16);
                    }
                }
                asm volatile("bar.sync %0, 64;" ::"r"(mine + 1) : "memory");    // L and the inverses are there
                // T: block columns 0 and 3 by one warp, 1 and 2 by the other.  Of block column c the blocks c .. 3.
                const uint32_t l_at = smem_u32(L), inv_at = smem_u32(smem + kPrepInv + mine * 4096) + (uint32_t)((lane & 7) + (lane >> 4) * 8) * 32u + (uint32_t)((lane >> 3) & 1) * 16u;
                uint32_t th[5][4], tl[5][4];             // blocks: of the first block column, up to four; of the second one or two
                auto column = [&](auto first, auto at0) {
                    constexpr int C = decltype(first)::value, A = decltype(at0)::value;
#pragma unroll
                    for (int b = C; b < 4; ++b) {
                        float c[2][4], d[2][4];
#pragma unroll
                        for (int i = 0; i < 8; ++i) c[i >> 2][i & 3] = d[i >> 2][i & 3] = 0.f;
                        if (b == C) {
                            // (a product's lane has row lane / 4, and eight more, and columns 2 (lane % 4) and one more of either tile)
                            const int m = lane >> 2, k = (lane & 3) * 2;
                            c[0][0] = c[1][2] = m == k ? kTile * kTile : 0.f;
                            c[0][1] = c[1][3] = m == k + 1 ? kTile * kTile : 0.f;
                        } else {
#pragma unroll
                            for (int e = C; e < b; ++e) {
                                const uint32_t at = l_at + at_swizzled(b * 16 + (lane & 7) + (lane >> 4) * 8, e * 16 + ((lane >> 3) & 1) * 8);
                                mma_sixteen(c, th[A + e - C], tl[A + e - C], at, at + kPart);
                            }
                        }
                        uint32_t ch[4], cl[4];
                        as_operand(c, ch, cl);
                        mma_sixteen(d, ch, cl, inv_at + b * 1024, inv_at + b * 1024 + 512);
                        as_operand(d, th[A + b - C], tl[A + b - C]);
                    }
                };
                auto store = [&](auto first, auto at0) {
                    constexpr int C = decltype(first)::value, A = decltype(at0)::value;
#pragma unroll
                    for (int b = C; b < 4; ++b) {        // (blocks above the diagonal are not read)
                        // (tiles of the operand: rows 0..7 and 8..15 of columns 0..7, then of 8..15; stored transposed: T's rows are its columns)
                        const uint32_t at = l_at + at_swizzled(b * 16 + (lane & 7) + (lane >> 4) * 8, C * 16 + ((lane >> 3) & 1) * 8);
                        stmatrix4_trans(at, th[A + b - C]);
                        stmatrix4_trans(at + kPart, tl[A + b - C]);
                    }
                };
                using I0 = std::integral_constant<int, 0>;
                using I1 = std::integral_constant<int, 1>;
                using I2 = std::integral_constant<int, 2>;
                using I3 = std::integral_constant<int, 3>;
                using I4 = std::integral_constant<int, 4>;
                if (role == 0) {
                    column(I0{}, I0{});
                    column(I3{}, I4{});
                } else {
                    column(I1{}, I0{});
                    column(I2{}, I3{});
                }
                asm volatile("bar.sync %0, 64;" ::"r"(mine + 1) : "memory");    // (nobody reads L any more)
                if (role == 0) {
                    store(I0{}, I0{});
                    store(I3{}, I4{});
                } else {
                    store(I1{}, I0{});
                    store(I2{}, I3{});
                }
                asm volatile("bar.sync %0, 64;" ::"r"(mine + 1) : "memory");
                {                                        // the diagonal's part of T X is added in fp32
                    unsigned short* to = reinterpret_cast<unsigned short*>(L + at_swizzled(t, t));
                    to[0] = to[kPart / 2] = 0;
                }
                proxy_fence();
                asm volatile("bar.sync %0, 64;" ::"r"(mine + 1) : "memory");
                if (t == 0) {
                    bulk_s2g(block + kTOff, L, 2 * kPart);
                    tma_store_done();
                }
            }
        }
        if (tid == 64) tma_store_done();
        if (!ok && tid == 0) record_fault(p.status, kFaultScanWait, 11);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_free<64>(tmem);
}

// ---- the chunks of a sequence, one after another ------------------------------------------------------------------------------
//
// Roles: warp 0 issues the copies, warp 1 the products; warp 2 brings two tokens of every value column together and finds the columns' largest
// values, warp 3 takes Y apart again and stores it; warps 4..11 hold the state, a lane of tensor memory and half of what is there to split
// a thread (64 keys' channels of S, 32 tokens of X, U and W); warps 12..15 scale Y, a lane a thread.  They meet through mbarriers alone; every wait is bounded.
// A chunk is a chain of four products and what stands between them: K S^T, X, (T - I) X, W, W K, S.  Everything else is done while a product
// of the chain runs or by other warps: the next chunk's V behind K S^T, U behind W K.
// T and P are lower triangular, 16 tokens of them meet the tokens from themselves on only.
// Tensor memory: two parts of S, of X, then of W, and of U; K S^T, then (T - I) X; Y; W K.
//
// What bounds it: the splitting.  Conversions, comparisons and two-element multiply-adds all issue every other cycle of a scheduler, and an
// arrival at a barrier costs a warp 26 of its scheduler's cycles, a poll 16: few warps, and few barriers between them (sixteen warps with
// a barrier for every quarter took half as long again).

constexpr int kWarps = 8, kThreads = 32 * (8 + kWarps);
constexpr uint32_t kWOff = kRows, kStage = (kWOff + kCopied + 1023u) & ~1023u;
constexpr uint32_t kVOff = 2 * kStage;                 // two buffers: rows of 256 bytes, then pairs of rows, [32][128] pairs of bf16
constexpr uint32_t kYOff = kVOff + 4 * kPart;          // the same
constexpr uint32_t kBarOff = kYOff + 2 * kPart;
// (bUP has two that take turns: nothing but its arrivals holds the state's warps back until the Y warps have seen them, and those could be a
// chunk ahead of a late one, which then would not see that phase end.  Two chunks ahead they are never: U of the next chunk but one waits for Y.
// bOutFree has two as well: the state's warps, which ask for it now and then, may come when it is two phases back.)
enum { bFull = 0, bEmpty = 2, bRaw = 4, bFullV = 6, bEmptyV = 8, bS = 10, bXP = 12, bWP = 13, bUP = 14, bX = 16, bU = 17, bProd = 18, bAsk = 19, bY = 20, bOut = 21,
       bOutFree = 22, bJoin = 24, bScaled = 25, bPair = 26, kBars = 30 };
constexpr uint32_t kMarkOff = (kBarOff + kBars * 8u + 4u + 15u) & ~15u;  // [128]: see mark_of
constexpr uint32_t kLargeOff = kMarkOff + 128u * 4u;             // [4][128][2]: the largest values of chunk n at n & 3, and the least of its pairs' larger ones
constexpr uint32_t kMostOff = kLargeOff + 1024u * 4u;             // [2][2][128]: the largest elements of the state, by halves
constexpr uint32_t kAsideOff = kMostOff + 512u * 4u;              // [2][2][128]: for Y of chunk n at n & 1, its factor and the first token that is not finite
constexpr uint32_t kPairOff = kAsideOff + 512u * 4u;              // [2][2][2][128]: what the halves of a column read by a key and a query
constexpr uint32_t kRowsOff = kPairOff + 1024u * 4u;              // [4][2][256]: for every pair of warps a token's key and query, of two tokens in turn
constexpr uint32_t kSmemTc = kRowsOff + 2048u * 4u + 1024u;

// columns of tensor memory: parts of S (part i, channel k: 64 i + k / 2); of X and W, of U (part i, token s: 32 i + s / 2); K S^T and (T - I) X; Y; W K
constexpr uint32_t cS = 0, cW = 128, cU = 192, cX = 256, cY = 320, cP = 384;

// The products take every token's values into every token, and a zero weight times NaN or infinity is NaN: from a lane's first value
// that is not finite on, zeros go to the products, and the lane's outputs and state become NaN afterwards.  A mark of chunk n holds that
// token; the largest of several is the first token of the latest chunk, so that marks need no clearing.
__device__ __forceinline__ uint32_t mark_of(int n, int token) { return ((uint32_t)n << 7) + (uint32_t)(kQ - token); }

// To the outputs' warps in the place of a column's first token that is not finite (kQ: none): its outputs are there already.
constexpr int kOutputsThere = -1;

// The scale for what is bounded by `all`: where that, times the scale, would be beyond 2^14 or below 2^11 (the second parts would lose bits), a new one.
// Returns the new scale over the old one.
__device__ __forceinline__ float new_scale(float all, float& up, float& down) {
    const float now = all * up;
    if (now <= 16384.f && (now >= 2048.f || all == 0.f)) return 1.f;
    const int e = max(-100, (int)((__float_as_uint(all) & 0x7f800000u) >> 23) - 127);     // (below 2^(e + 1); below 2^13 then)
    const float old = down;
    up = __uint_as_float((uint32_t)(127 + 12 - e) << 23);
    down = __uint_as_float((uint32_t)(127 - 12 + e) << 23);
    return up * old;
}
__device__ __forceinline__ void arrive_warp(uint64_t* bar, int lane) {
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive_one(bar);
}
// Channels 32 i .. of a half of S as an operand, in the lanes at `lanes`.
__device__ __forceinline__ void give_state(const uint64_t (&S)[32], int i, uint32_t lanes, uint64_t* bar, int lane) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        uint32_t a[2][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) two_parts(S[i * 16 + c * 8 + j], a[0][j], a[1][j]);
#pragma unroll
        for (int e = 0; e < 2; ++e) tmem_st8u(lanes + cS + e * 64 + i * 16 + c * 8, a[e]);
    }
    tmem_st_wait();
    arrive_warp(bar, lane);
}
// Bounds sqrt(a^2 + b^2), a and b not negative.
__device__ __forceinline__ float longer(float a, float b) {
    const float m = fmaxf(a, b), n = fminf(a, b);
    return fmaf(0.5f * n, __fdividef(n, fmaxf(m, 1e-30f)), m);
}
constexpr float kLength = 11.4f;                        // bounds the length of 128 elements of at most one

// A chunk for the 32 columns of two warps, half of the channels each: whether its numbers are too far apart for one scale, and then the chunk, token by
// token.  The values are where the outputs will stand.
struct Alone {
    uint64_t S[32];            // times 1 / down
    unsigned char *smem, *stage;
    uint64_t *bar, *pair;      // pair: where the two meet
    const float* rest;         // the chunk's gates in the scratch
    const volatile float *most, *next;         // the largest elements of the state's halves, 128 apart; the next chunk's largest value
    float up, down, length, q_scale;
    uint32_t lanes;            // of tensor memory, and this half's columns there
    int n, m, o, col, half, valid, met;
    bool zero, outputs, live, more, ok;
};
__device__ __noinline__ bool token_by_token(Alone& g) {
    const int lane = (int)threadIdx.x & 31, half = g.half, valid = g.valid;
    const bool outputs = g.outputs;
    const float up = g.up, q_scale = g.q_scale;
    unsigned char* const stage = g.stage;
    uint64_t* const pair = g.pair;
    int met = g.met;
    auto meet = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive_one(pair);
        const bool ok = warp_wait(pair, met & 1);
        ++met;
        if (!ok) g.ok = false;
        return ok;
    };
    const float* beta = reinterpret_cast<const float*>(stage + kWOff + kGOff) + kBeta;
    volatile unsigned short* value = reinterpret_cast<volatile unsigned short*>(g.smem + kYOff + g.col * 4);     // of token t: at(t)
    auto at = [](int t) { return (t >> 1) * 256 + (t & 1); };
    // (a lane has two tokens' decays, keys' and queries' factors)
    const float d0 = __ldcg(g.rest + kDecay + lane), d1 = __ldcg(g.rest + kDecay + 32 + lane), k0 = __ldcg(g.rest + kKey + lane),
                k1 = __ldcg(g.rest + kKey + 32 + lane), q0 = __ldcg(g.rest + kQuery + lane), q1 = __ldcg(g.rest + kQuery + 32 + lane);
    auto of = [](float low, float high, int i) { return __shfl_sync(0xffffffffu, i < 32 ? low : high, i & 31); };
    if (!meet()) return false;
    {
        float a = 0.f, last = fmaxf(g.most[0], g.most[128]);
        g.met = met;
        g.length = fminf(g.length, kLength * last);
        if (__all_sync(0xffffffffu, last * beta[kKeep - kBeta] * up >= kFloor)) return false;      // (the state alone is large enough, up to the last token)
        bool nothing = g.zero, over = false, alone = false;      // neither a state nor a value so far; nothing behind it is finite
#pragma unroll 1
        for (int i = 0; i < valid; ++i) {
            const float size = __uint_as_float((uint32_t)(value[at(i)] & 0x7fff) << 16), counts = beta[i] >= kLeastBeta ? size : 0.f;
            a = fmaxf(fmaxf(counts, last), of(d0, d1, i) * a);
            last = counts;
            over = over || !(size <= 3.4028235e38f);
            if (over || (nothing && size == 0.f)) continue;
            if (!(a * up >= kFloor)) alone = true;
            nothing = false;
        }
        if (!__any_sync(0xffffffffu, alone)) return false;
    }
    uint64_t S[32];                                     // channels 64 half ..
    const uint64_t down2 = pack2(g.down, g.down);
#pragma unroll
    for (int i = 0; i < 32; ++i) S[i] = mul2(down2, g.S[i]);
    // Keys and queries as floats, a token's at a time, by its half of the channels: two a lane.  [key, query][64]
    float* const row = reinterpret_cast<float*>(g.smem + kRowsOff) + (g.col >> 5) * 512 + half * 128;
    auto spread = [&](int t) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const __half2 w = *reinterpret_cast<const __half2*>(stage + half * (2 * kPart) + i * kPart + t * 128 + (((lane >> 2) ^ (t & 7)) * 16) + (lane & 3) * 4);
            *reinterpret_cast<float2*>(row + (t & 1) * 256 + i * 64 + lane * 2) = __half22float2(w);
        }
        __syncwarp();
    };
    // the state times one of them
    auto read_by = [&](const float* x) {
        uint64_t sum[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(x + 4 * i);
            sum[i % 2 * 2] = fma2(S[2 * i], w.x, sum[i % 2 * 2]);
            sum[i % 2 * 2 + 1] = fma2(S[2 * i + 1], w.y, sum[i % 2 * 2 + 1]);
        }
        float lo, hi;
        unpack2(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), lo, hi);
        return lo + hi;
    };
    volatile float* both = reinterpret_cast<volatile float*>(g.smem + kPairOff) + g.col;
    float asked = 0.f;                                  // by the query of the token before
#pragma unroll 1
    for (int i = 0; i <= valid; ++i) {
        volatile float* to = both + (i & 1) * 512;
        const float* x = row + (i & 1) * 256;
        if (i < valid) spread(i);
        to[half * 256] = i < valid ? read_by(x) : 0.f;
        to[half * 256 + 128] = asked;
        if (!meet()) return false;
        const float query = of(q0, q1, i > 0 ? i - 1 : 0);
        if (half == 0 && i > 0 && outputs) value[at(i - 1)] = __bfloat16_as_ushort(__float2bfloat16_rn(q_scale * query * (to[128] + to[256 + 128])));
        if (i == valid) break;
        const float d = of(d0, d1, i), r = of(k0, k1, i);
        const float u = beta[i] * fmaf(-(d * r), to[0] + to[256], __uint_as_float((uint32_t)value[at(i)] << 16));
        const uint64_t d2 = pack2(d, d), u2 = pack2(u * r, u * r);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(x + 4 * j);
            S[2 * j] = fma2(u2, w.x, mul2(d2, S[2 * j]));
            S[2 * j + 1] = fma2(u2, w.y, mul2(d2, S[2 * j + 1]));
        }
        asked = outputs ? read_by(x + 64) : 0.f;
    }
    // The state is the one behind the chunk; zeros go to the products, for the other columns' sake.
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        float a, b;
        unpack2(S[i], a, b);
        most = fmaxf(most, fmaxf(fabsf(a), fabsf(b)));
    }
    both[half * 256 + (valid & 1 ? 0 : 512)] = most;    // (the other one than the last token's)
    if (!meet()) return false;
    most = fmaxf(both[valid & 1 ? 0 : 512], both[256 + (valid & 1 ? 0 : 512)]);
    g.met = met;
    auto wait = [&](int i, int k) { return g.ok = warp_wait(g.bar + i, k & 1); };
    if (g.live && !wait(bX, g.m)) return false;
    tc_fence_after();
    const uint32_t none[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < 4; ++e) tmem_st8u(g.lanes + cW + (e >> 1) * 32 + half * 16 + (e & 1) * 8, none);
    tmem_st_wait();
    arrive_warp(g.bar + bXP, lane);
    if (!wait(bU, g.n)) return false;
    tc_fence_after();
    arrive_warp(g.bar + bWP, lane);
    if (outputs) {
#pragma unroll
        for (int e = 0; e < 4; ++e) tmem_st8u(g.lanes + cU + (e >> 1) * 32 + half * 16 + (e & 1) * 8, none);
        if (half == 0) {
            volatile float* aside = reinterpret_cast<volatile float*>(g.smem + kAsideOff) + (g.o & 1) * 256 + g.col;
            aside[0] = 0.f;
            aside[128] = __int_as_float(kOutputsThere);
        }
        tmem_st_wait();
        arrive_warp(g.bar + bUP + (g.o & 1), lane);
    }
    g.up = g.down = 1.f;
    if (g.more) {
        if (!wait(bFullV + ((g.n + 1) & 1), (g.n + 1) >> 1)) return false;
        g.length = kLength * most;
        const float r = new_scale(9.f * *g.next + g.length, g.up, g.down);
        const uint64_t r2 = pack2(r, r);
#pragma unroll
        for (int i = 0; i < 32; ++i) S[i] = mul2(r2, S[i]);
    }
    if (!wait(bProd, g.n)) return false;
    tc_fence_after();
    if (g.more) {
        give_state(S, 0, g.lanes + half * 32, g.bar + bS, lane);
        give_state(S, 1, g.lanes + half * 32, g.bar + bS + 1, lane);
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) g.S[i] = S[i];
    return true;
}

__device__ __forceinline__ bool finite16(uint32_t bf) { return (bf & 0x7f80u) != 0x7f80u; }

__global__ void __launch_bounds__(kThreads, 1) delta_scan_tc_kernel(const __grid_constant__ DeltaArgs g) {
    extern __shared__ unsigned char raw[];
    unsigned char* smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    uint64_t* bar = reinterpret_cast<uint64_t*>(smem + kBarOff);
    uint32_t* slot = reinterpret_cast<uint32_t*>(bar + kBars);
    uint32_t* marks = reinterpret_cast<uint32_t*>(smem + kMarkOff);
    const DeltaParams& p = g.p;
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 32) prefetch_map(&g.tv);
    if (tid == 0) {
        for (int i = 0; i < kBars; ++i) {
            int n = 1;                                  // copies, commits of products and single warps arrive once
            if (i == bEmptyV || i == bEmptyV + 1 || (i >= bS && i < bX) || i == bJoin) n = kWarps;
            if (i == bOut || i == bScaled) n = 4;
            if (i >= bPair) n = 2;
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
            Unit x;
            for (int it = 0; ok && decode_unit(g, it, x); ++it) {
                const int head = x.head, group = head / (p.H / p.G);
                int chunk = x.chunk;
                if (has_state(g, x) && x.kind != kMap) {         // (two chunks ahead of the warps that read it)
                    const float* from = x.kind == kLater ? scratch_state(g, x.seq, x.head, x.seg - 1)
                                                         : p.state + ((size_t)seq_resume(p.pr, x.seq) * p.H + x.head) * 128 * 128;
                    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from), "r"(128 * 128 * 4) : "memory");
                }
                for (int t = x.t0; t < x.t1; t += kQ, ++chunk, ++n) {
                    const int b = n & 1;
                    ok = n < 2 || mbar_wait_bounded(bar + bEmpty + b, (n / 2 - 1) & 1);
                    if (!ok) break;
                    unsigned char* to = smem + b * kStage;
                    mbar_expect_tx(bar + bFull + b, kRows + kCopied);
                    bulk_g2s(to, g.rows + ((size_t)chunk * p.G + group) * kRows, kRows, bar + bFull + b);
                    bulk_g2s(to + kWOff, p.work + ((size_t)chunk * p.H + head) * kBlock, kCopied, bar + bFull + b);
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
        Unit x;
        int o = 0, om = 0;                              // chunks with outputs; those of them with a state before them
        for (int it = 0; ok && decode_unit(g, it, x); ++it) {
            const bool stored = has_state(g, x);
            for (int t = x.t0; t < x.t1 && ok; t += kQ, ++n) {
                const int b = n & 1;
                const bool live = stored || t > x.t0;                            // S is not zero
                const uint32_t base = sbase + b * kStage;
                const uint64_t dk = swizzled_desc(base, 16u, 1024u), dq = swizzled_desc(base + kPart, 16u, 1024u);
                const uint64_t dt = swizzled_desc(base + kWOff + kTOff, 16u, 1024u), dp = swizzled_desc(base + kWOff + kPOff, 16u, 1024u);
                const uint64_t dkt = swizzled_desc(base, 2 * kPart, 1024u);
                ok = warp_wait(bar + bFull + b, (n / 2) & 1);
                if (!ok) break;
                if (live) {                              // K S^T: first the first 32 channels of both halves
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        ok = ok && warp_wait(bar + bS + i, m & 1);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll
                        for (int e = 0; e < 8; ++e) {                            // (two halves, two steps of 16 channels, two parts)
                            const int half = e >> 2, step = (e >> 1) & 1, part = e & 1;
                            if (elect())
                                mma_ts(tmem + cX, tmem + cS + part * 64 + half * 32 + i * 16 + step * 8,
                                       dk + (uint32_t)half * (2 * kPart >> 4) + (uint32_t)(i * 2 + step) * 2u, kN64, i > 0 || e > 0);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (elect()) tc_commit(bar + bX);
                    __syncwarp();
                    ++m;
                }
                ok = warp_wait(bar + bXP, n & 1);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int q = 0; q < 4; ++q) {            // (T - I) X, 16 tokens at a time
                    const uint32_t desc = kTypes | ((uint32_t)((64 - 16 * q) >> 3) << 17);
                    const uint64_t rows_q = dt + (uint32_t)q * (2048u >> 4) + (uint32_t)q * 2u;
#pragma unroll
                    for (int e = 0; e < 3; ++e)                                  // parts (T, X): 00 01 10
                        if (elect())
                            mma_ts(tmem + cX + 16 * q, tmem + cW + (e == 1) * 32 + q * 8, rows_q + (uint32_t)(e == 2) * (kPart >> 4), desc, q > 0 || e > 0);
                }
                if (elect()) tc_commit(bar + bU);
                __syncwarp();
                if (x.outputs) {
                    ok = o < 1 || warp_wait(bar + bOut, (o - 1) & 1);
                    if (!ok) break;
                    tc_fence_after();
                }
                if (live && x.outputs) {                 // Q S^T
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int part = i >> 3, k = i & 7;
                        if (elect())
                            mma_ts(tmem + cY, tmem + cS + part * 64 + k * 8, dq + (uint32_t)(k / 4) * (2 * kPart >> 4) + (uint32_t)(k & 3) * 2u, kN64, i > 0);
                    }
                    if (elect()) tc_commit(bar + bAsk);
                    __syncwarp();
                }
                ok = warp_wait(bar + bWP, n & 1);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int e = 0; e < 8; ++e)              // W K
                    if (elect()) mma_ts(tmem + cP, tmem + cW + (e & 1) * 32 + (e >> 1) * 8, dkt + (uint32_t)(e >> 1) * 128u, kProdDesc, e > 0);
                if (elect()) tc_commit(bar + bProd);
                __syncwarp();
                if (!x.outputs) {                        // (what the other warps read of the stage they have read: W is made of it)
                    if (elect()) tc_commit(bar + bEmpty + b);
                    __syncwarp();
                    continue;
                }
                ok = warp_wait(bar + bUP + (o & 1), (o >> 1) & 1) && (!live || warp_wait(bar + bScaled, om & 1));
                if (!ok) break;
                ++o;
                if (live) ++om;
                tc_fence_after();
#pragma unroll
                for (int q = 0; q < 4; ++q) {            // U P
                    const uint32_t desc = kTypes | ((uint32_t)((64 - 16 * q) >> 3) << 17);
                    const uint64_t rows_q = dp + (uint32_t)q * (2048u >> 4) + (uint32_t)q * 2u;
#pragma unroll
                    for (int e = 0; e < 3; ++e)                                  // parts (P, U): 00 01 10
                        if (elect())
                            mma_ts(tmem + cY + 16 * q, tmem + cU + (e == 1) * 32 + q * 8, rows_q + (uint32_t)(e == 2) * (kPart >> 4), desc, live || q > 0 || e > 0);
                }
                if (elect()) {                           // (what the other warps read of the stage they have read: U and Y's factors)
                    tc_commit(bar + bY);
                    tc_commit(bar + bEmpty + b);
                }
                __syncwarp();
            }
        }
        if (!ok && lane == 0) record_fault(p.status, kFaultScanWait, 13);
        __syncwarp();
    } else if (warp == 2) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        // V, copied a chunk ahead: four columns a lane; two rows at a time become one of pairs, in their place
        Unit next, x;
        uint32_t last[2] = {0u, 0u};                    // the sizes of the token before
        int next_it = 0, next_n = 0, next_t = 0;
        bool there = decode_unit(g, 0, next);
        if (there) next_t = next.t0;
        auto copy = [&]() {                              // the next copy, if there is one
            while (there && next_t >= next.t1) {
                there = decode_unit(g, ++next_it, next);
                if (there) next_t = next.t0;
            }
            if (!there) return;
            const int b = next_n & 1;
            ok = ok && (next_n < 2 || warp_wait(bar + bEmptyV + b, (next_n / 2 - 1) & 1));
            if (!ok) return;
            if (lane == 0) {
                mbar_expect_tx(bar + bRaw + b, 2 * kPart);
                tma_load(smem + kVOff + b * 2 * kPart, &g.tv, next.head * 128, next_t, bar + bRaw + b);
            }
            __syncwarp();
            ++next_n;
            next_t += kQ;
        };
        copy();
        for (int it = 0; ok && decode_unit(g, it, x); ++it) {
            for (int t = x.t0; t < x.t1; t += kQ, ++n) {
                const int b = n & 1, valid = x.kind == kMap ? 0 : min(kQ, x.t1 - t);     // (M is made without values)
                copy();
                ok = ok && warp_wait(bar + bRaw + b, (n / 2) & 1);
                if (!ok) break;
                unsigned char* v = smem + kVOff + b * 2 * kPart;
                // The largest size, and the least of all tokens' larger one of their size and that of the token before, two columns at a time.  (As whole
                // numbers: sizes in bf16 are in their order, with what is not finite above all.  max(y, min(x, z)) is the lesser one of y's two pairs.)
                uint32_t top[2] = {0u, 0u}, least[2] = {0x7f7f7f7fu, 0x7f7f7f7fu};
                if (t == x.t0) last[0] = last[1] = 0x7f7f7f7fu;          // (a unit's first token: see where it begins)
                auto load = [&](uint2 (&a)[2], uint2 (&c)[2], int r) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        a[i] = *reinterpret_cast<const uint2*>(v + (r + i) * 512 + lane * 8);
                        c[i] = *reinterpret_cast<const uint2*>(v + (r + i) * 512 + 256 + lane * 8);
                    }
                };
                auto store = [&](const uint2& a, const uint2& c, int r) {
                    *reinterpret_cast<uint4*>(v + r * 512 + lane * 16) =
                        make_uint4(__byte_perm(a.x, c.x, 0x5410), __byte_perm(a.x, c.x, 0x7632), __byte_perm(a.y, c.y, 0x5410), __byte_perm(a.y, c.y, 0x7632));
                };
                auto take = [&](const uint2 (&a)[2], const uint2 (&c)[2], int r) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t y0 = (j ? a[0].y : a[0].x) & 0x7fff7fffu, z0 = (j ? c[0].y : c[0].x) & 0x7fff7fffu;
                        const uint32_t y1 = (j ? a[1].y : a[1].x) & 0x7fff7fffu, z1 = (j ? c[1].y : c[1].x) & 0x7fff7fffu;
                        top[j] = __vimax3_u16x2(__vimax3_u16x2(top[j], y0, z0), y1, z1);
                        least[j] = __vimin3_u16x2(least[j], __vmaxu2(y0, __vminu2(last[j], z0)), __vmaxu2(y1, __vminu2(z0, z1)));
                        last[j] = z1;
                    }
                    __syncwarp();                        // (rows are read by other lanes than write them)
                    store(a[0], c[0], r);
                    store(a[1], c[1], r + 1);
                };
                const int whole = valid / 8 * 4;         // pairs of rows that are all there, four at a time: two are loaded while two are worked on
                {
                    uint2 a[2], c[2], d[2], e[2];
                    if (whole > 0) load(a, c, 0);
#pragma unroll 1
                    for (int r = 0; r < whole; r += 4) {
                        load(d, e, r + 2);
                        take(a, c, r);
                        if (r + 4 < whole) load(a, c, r + 4);
                        take(d, e, r + 2);
                    }
                }
#pragma unroll 1
                for (int r = whole; r < 32; ++r) {       // rows of the next sequence are no part of this one
                    uint2 a = make_uint2(0u, 0u), c = a;
                    if (2 * r < valid) {
                        a = *reinterpret_cast<const uint2*>(v + r * 512 + lane * 8);
                        if (2 * r + 1 < valid) c = *reinterpret_cast<const uint2*>(v + r * 512 + 256 + lane * 8);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const uint32_t y = (j ? a.y : a.x) & 0x7fff7fffu, z = 2 * r + 1 < valid ? (j ? c.y : c.x) & 0x7fff7fffu : 0x7f7f7f7fu;
                            top[j] = __vmaxu2(top[j], y);
                            if (2 * r + 1 < valid) top[j] = __vmaxu2(top[j], z);
                            least[j] = __vminu2(least[j], __vmaxu2(y, __vminu2(last[j], z)));
                            last[j] = z;
                        }
                        __syncwarp();
                    }
                    store(a, c, r);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (!finite16(top[i / 2] >> (i % 2 * 16))) {                 // (tokens before it keep their accuracy: of those that are finite)
                        uint32_t most = 0u;
                        __threadfence_block();
#pragma unroll 1
                        for (int r = 0; r < 32; ++r) {
                            const uint32_t w = *reinterpret_cast<const volatile uint32_t*>(v + r * 512 + lane * 16 + i * 4) & 0x7fff7fffu;
                            most = __vmaxu2(most, (finite16(w) ? w & 0xffffu : 0u) | (finite16(w >> 16) ? w & 0xffff0000u : 0u));
                        }
                        most = max(most & 0xffffu, most >> 16);
                        top[i / 2] = i % 2 ? __byte_perm(top[i / 2], most, 0x5410) : __byte_perm(most, top[i / 2], 0x7610);
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    *reinterpret_cast<float4*>(smem + kLargeOff + (n & 3) * 1024 + lane * 32 + i * 16) =
                        make_float4(__uint_as_float(top[i] << 16), __uint_as_float(least[i] << 16), __uint_as_float(top[i] & 0xffff0000u), __uint_as_float(least[i] & 0xffff0000u));
                proxy_fence();                           // (the next copy writes where this warp has)
                __syncwarp();
                if (lane == 0) mbar_arrive_one(bar + bFullV + b);
            }
        }
        if (!ok && lane == 0) record_fault(p.status, kFaultScanWait, 16);
        // (as above)
        for (int i = next_n < 2 ? 0 : next_n - 2; i < next_n; ++i) mbar_wait_bounded(bar + (ok ? bEmptyV : bRaw) + (i & 1), (i / 2) & 1, ok ? 1u << 22 : 1u << 16);
        __syncwarp();
    } else if (warp == 3) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        // Y: four columns a lane, two rows at a time
        Unit x;
        for (int it = 0; ok && decode_unit(g, it, x); ++it) {
            if (!x.outputs) continue;
            const int head = x.head;
            for (int t = x.t0; t < x.t1; t += kQ, ++n) {
                const int valid = min(kQ, x.t1 - t);
                ok = warp_wait(bar + bOut, n & 1);
                if (!ok) break;
                unsigned char* to = static_cast<unsigned char*>(p.out) + ((long long)t * p.out_stride + (long long)head * 128 + lane * 4) * 2;
                const long long step = p.out_stride * 2;
#pragma unroll 4
                for (int r = 0; r < 32; ++r) {
                    const uint4 w = *reinterpret_cast<const uint4*>(smem + kYOff + r * 512 + lane * 16);
                    if (2 * r < valid) *reinterpret_cast<uint2*>(to) = make_uint2(__byte_perm(w.x, w.y, 0x5410), __byte_perm(w.z, w.w, 0x5410));
                    to += step;
                    if (2 * r + 1 < valid) *reinterpret_cast<uint2*>(to) = make_uint2(__byte_perm(w.x, w.y, 0x7632), __byte_perm(w.z, w.w, 0x7632));
                    to += step;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive_one(bar + bOutFree + (n & 1));
            }
        }
        if (!ok && lane == 0) record_fault(p.status, kFaultScanWait, 15);
        __syncwarp();
    } else if (warp >= 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        // Y of a value column: Q S^T times its tokens' factors, and what U P has added to it
        const int col = (warp & 3) * 32 + lane;
        const uint32_t at = tmem + ((uint32_t)((warp & 3) * 32) << 16) + cY;
        const float* aside = reinterpret_cast<const float*>(smem + kAsideOff) + col;
        Unit x;
        int o = 0;                                      // chunks with outputs
        for (int it = 0; ok && decode_unit(g, it, x); ++it) {
            if (!x.outputs) {
                n += (x.t1 - x.t0 + kQ - 1) / kQ;
                continue;
            }
            const bool stored = has_state(g, x);
            for (int t = x.t0; t < x.t1; t += kQ, ++n, ++o) {
                if (stored || t > x.t0) {
                    const float* gate = reinterpret_cast<const float*>(smem + (n & 1) * kStage + kWOff + kGOff) + kAsk;
                    ok = warp_wait(bar + bFull + (n & 1), (n / 2) & 1) && warp_wait(bar + bAsk, m & 1);
                    if (!ok) break;
                    ++m;
                    tc_fence_after();
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t d[32];
                        tmem_ld32_async(at + h * 32, d);
                        tmem_ld_wait();
                        const ulonglong2* ask = reinterpret_cast<const ulonglong2*>(gate + h * 32);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t r[8];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const ulonglong2 w = ask[2 * i + e];
                                const uint64_t y0 = mul2(w.x, pack2(__uint_as_float(d[8 * i + 4 * e]), __uint_as_float(d[8 * i + 4 * e + 1])));
                                const uint64_t y1 = mul2(w.y, pack2(__uint_as_float(d[8 * i + 4 * e + 2]), __uint_as_float(d[8 * i + 4 * e + 3])));
                                r[4 * e] = (uint32_t)y0;
                                r[4 * e + 1] = (uint32_t)(y0 >> 32);
                                r[4 * e + 2] = (uint32_t)y1;
                                r[4 * e + 3] = (uint32_t)(y1 >> 32);
                            }
                            tmem_st8u(at + h * 32 + 8 * i, r);
                        }
                    }
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_one(bar + bScaled);
                }
                ok = warp_wait(bar + bUP + (o & 1), (o >> 1) & 1);
                if (!ok) break;
                const float scale = reinterpret_cast<const volatile float*>(aside)[(o & 1) * 256];
                const int first = __float_as_int(reinterpret_cast<const volatile float*>(aside)[(o & 1) * 256 + 128]);
                ok = warp_wait(bar + bY, o & 1) && (o < 1 || warp_wait(bar + bOutFree + ((o - 1) & 1), ((o - 1) >> 1) & 1));
                if (!ok) break;
                tc_fence_after();
                const uint64_t scale2 = pack2(scale, scale);
                uint32_t* to = reinterpret_cast<uint32_t*>(smem + kYOff) + col;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t d[32];
                    tmem_ld32_async(at + h * 32, d);
                    tmem_ld_wait();
                    if (first < kQ) {
                        if (first == kOutputsThere) continue;                    // (the same for the whole warp)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (h * 32 + i >= first) d[i] = 0x7fffffffu;
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float a, c;
                        unpack2(mul2(scale2, pack2(__uint_as_float(d[2 * i]), __uint_as_float(d[2 * i + 1]))), a, c);
                        const __nv_bfloat162 y = __floats2bfloat162_rn(a, c);
                        to[(h * 16 + i) * 128] = *reinterpret_cast<const uint32_t*>(&y);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_one(bar + bOut);
            }
        }
        if (!ok && lane == 0) record_fault(p.status, kFaultScanWait, 17);
    } else {
        // (512 threads start with 128 registers: 128 x 56 + 256 x 192 + 128 x 72 are all 65536)
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        const int quad = warp & 3, half = (warp - 4) >> 2, col = quad * 32 + lane;       // value column; half of the channels and tokens
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
        const float2* large = reinterpret_cast<const float2*>(smem + kLargeOff) + col;
        float* most = reinterpret_cast<float*>(smem + kMostOff) + col;
        uint64_t S[32];                                 // channels 64 half .., times `up`
        uint32_t f[16];                                 // the next chunk's values of this half, two tokens each
        float up = 1.f, down = 1.f;                     // the lane's scale and its inverse
        float length = 0.f;                             // bounds the length of the lane's state before the chunk
        bool zero = false;                              // a lane without a state before the unit
        bool doubt = false;                             // the least of the chunk's numbers may be too small for its scale
        int met = 0;                                    // meetings of a column's halves
        int units = 0;                                  // with tokens, so far
        auto arrive = [&](int i) { arrive_warp(bar + i, lane); };
        auto fetch = [&](int c, uint32_t* begin = nullptr) {     // begin: for the chunk's first two values
            const int b = c & 1;
            ok = warp_wait(bar + bFullV + b, (c / 2) & 1);
            if (!ok) return;
            const uint32_t* v = reinterpret_cast<const uint32_t*>(smem + kVOff + b * 2 * kPart) + half * 16 * 128 + col;
#pragma unroll
            for (int i = 0; i < 16; ++i) f[i] = v[i * 128];
            if (begin != nullptr) *begin = v[half * -16 * 128];
            __syncwarp();
            if (lane == 0) mbar_arrive_one(bar + bEmptyV + b);
        };
        // The largest element of this half of the state, for the other half too.
        auto state_most = [&](int c) {
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                float a, d;
                unpack2(S[i], a, d);
                top = fmaxf(top, fmaxf(fabsf(a), fabsf(d)));
            }
            most[((c & 1) * 2 + half) * 128] = top * down;
        };
        auto most_of = [&](int c) {
            const volatile float* from = most + (c & 1) * 256;
            return fmaxf(from[0], from[128]);
        };
        auto rescale = [&](int c) {
            const float2 sizes = large[(c & 3) * 128];
            const float all = 9.f * sizes.x + length;
            const float r = new_scale(all, up, down);
            doubt = !(sizes.y * up >= kFloor) && all != 0.f;
            return r;
        };
        auto give = [&](int i) { give_state(S, i, lanes + half * 32, bar + bS + i, lane); };
        Unit x;
        int o = 0;                                      // chunks with outputs
        for (int it = 0; ok && decode_unit(g, it, x); ++it) {
            const int2 rows = make_int2(x.t0, x.t1);
            const bool stored = has_state(g, x);
            const size_t at = (size_t)half * 64 * 128 + col;
            if (stored && x.kind != kMap) {
                const float* from = (x.kind == kLater ? scratch_state(g, x.seq, x.head, x.seg - 1)
                                                      : p.state + ((size_t)seq_resume(p.pr, x.seq) * p.H + x.head) * 128 * 128) + at;
#pragma unroll
                for (int i = 0; i < 32; ++i) S[i] = pack2(from[2 * i * 128], from[(2 * i + 1) * 128]);
            } else {
                const int one = x.kind == kMap ? col - half * 64 : -1;
#pragma unroll
                for (int i = 0; i < 32; ++i) S[i] = pack2(2 * i == one ? 1.f : 0.f, 2 * i + 1 == one ? 1.f : 0.f);
            }
            up = down = 1.f;
            if (rows.x < rows.y) {
                uint32_t begin = 0u;
                fetch(n, &begin);
                if (!ok) break;
                state_most(n);
                arrive(bJoin);
                ok = warp_wait(bar + bJoin, units & 1);
                ++units;
                if (!ok) break;
                length = kLength * most_of(n);
                zero = length == 0.f;
                const float r = rescale(n), first = __uint_as_float(begin << 16 & 0x7fff0000u);
                // (Without a state the first token, if it is small by itself, keeps some bits less than the others.)
                doubt = doubt || (zero ? first > 0.f && !(first * up >= kFloor / 128.f) : !(most_of(n) * up >= kFloor));
                const uint64_t r2 = pack2(r, r);
                if (stored) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) S[i] = mul2(r2, S[i]);
                    give(0);
                    give(1);
                }
            }
            int t = rows.x;
            bool checked = x.kind == kMap;               // (a map has no values, and what it is off by decays as it does)
            while (ok && t < rows.y) {
                for (; t < rows.y; t += kQ, ++n) {
                    const int b = n & 1, left = rows.y - t - half * 32;              // tokens of the sequence from this half on
                    const bool live = stored || t > rows.x, more = t + kQ < rows.y;
                    const float* gate = reinterpret_cast<const float*>(smem + b * kStage + kWOff + kGOff) + half * 32;
                    ok = warp_wait(bar + bFull + b, (n / 2) & 1);
                    if (!ok) break;
                    const bool plain = gate[kPlain - half * 32] != 0.f;
                    if (__any_sync(0xffffffffu, doubt || !plain) && !checked) break;
                    checked = x.kind == kMap;
                    // X of this half's tokens: the values, scaled (times powers of two in bf16), less what the state has for their keys
                    uint64_t X[16];
                    {
                        const uint32_t up16 = __float_as_uint(up) >> 16;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float a, c;
                            asm("{\n\t.reg .b16 l, h, s, x;\n\tmov.b32 {l, h}, %2;\n\tmov.b32 {s, x}, %3;\n\t"
                                "fma.rn.f32.bf16 %0, l, s, 0f00000000;\n\tfma.rn.f32.bf16 %1, h, s, 0f00000000;\n\t}"
                                : "=f"(a), "=f"(c)
                                : "r"(f[i]), "r"(up16));
                            X[i] = pack2(a, c);
                        }
                    }
                    if (more) {
                        fetch(n + 1);
                        if (!ok) break;
                    }
                    uint32_t d[32];
                    const ulonglong2* rd = reinterpret_cast<const ulonglong2*>(gate + kRead);
                    if (live) {
                        ok = warp_wait(bar + bX, m & 1);
                        if (!ok) break;
                        ++m;
                        tc_fence_after();
                        tmem_ld32_async(lanes + cX + half * 32, d);
                        tmem_ld_wait();
                    } else {                                 // (a key that is not finite counts, whatever it is taken of)
#pragma unroll
                        for (int i = 0; i < 32; ++i) d[i] = 0u;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const ulonglong2 r = rd[i];
                        X[2 * i] = fma2(r.x, pack2(__uint_as_float(d[4 * i]), __uint_as_float(d[4 * i + 1])), X[2 * i]);
                        X[2 * i + 1] = fma2(r.y, pack2(__uint_as_float(d[4 * i + 2]), __uint_as_float(d[4 * i + 3])), X[2 * i + 1]);
                    }
                    {
                        uint32_t a[4][8], odd = 0u;          // first parts of 16 tokens, of 16 more; second parts
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            two_parts(X[i], a[i / 8][i % 8], a[2 + i / 8][i % 8]);
                            asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(odd) : "r"(a[i / 8][i % 8] & 0x7fff7fffu));
                        }
                        auto store = [&]() {
#pragma unroll
                            for (int e = 0; e < 4; ++e) tmem_st8u(lanes + cW + (e >> 1) * 32 + half * 16 + (e & 1) * 8, a[e]);
                        };
                        const bool wild = (odd & 0x7c00u) == 0x7c00u || (odd & 0x7c000000u) == 0x7c000000u;
                        if (!__any_sync(0xffffffffu, wild)) {
                            store();
                        } else {
                            int first = 32;
#pragma unroll
                            for (int i = 15; i >= 0; --i) {
                                if ((a[i / 8][i % 8] & 0x7c000000u) == 0x7c000000u) first = 2 * i + 1;
                                if ((a[i / 8][i % 8] & 0x7c00u) == 0x7c00u) first = 2 * i;
                            }
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const uint32_t keep = (2 * i < first ? 0xffffu : 0u) | (2 * i + 1 < first ? 0xffff0000u : 0u);
                                a[i / 8][i % 8] &= keep;
                                a[2 + i / 8][i % 8] &= keep;
                            }
                            if (first < 32 && first < left) atomicMax(marks + col, mark_of(n + 1, half * 32 + first));
                            store();
                        }
                        tmem_st_wait();
                        arrive(bXP);
                    }
                    // U and W
                    ok = warp_wait(bar + bU, n & 1);
                    if (!ok) break;
                    tc_fence_after();
                    tmem_ld32_async(lanes + cX + half * 32, d);
                    const uint32_t mark = reinterpret_cast<const volatile uint32_t*>(marks)[col];
                    const bool bad = (mark >> 7) == (uint32_t)n + 1u;
                    const int first = bad ? kQ - (int)(mark & 127u) - half * 32 : 32;
                    const float end = gate[kKeep - half * 32], keep = bad ? __int_as_float(0x7fffffff) : end;       // (NaN: all of the lane's state)
                    tmem_ld_wait();
                    {
                        const ulonglong2 *put = reinterpret_cast<const ulonglong2*>(gate + kPut), *beta = reinterpret_cast<const ulonglong2*>(gate + kBeta);
                        const uint64_t back = pack2(1.f / kTile, 1.f / kTile);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const ulonglong2 be = beta[i];
                            X[2 * i] = mul2(be.x, fma2(back, pack2(__uint_as_float(d[4 * i]), __uint_as_float(d[4 * i + 1])), X[2 * i]));
                            X[2 * i + 1] = mul2(be.y, fma2(back, pack2(__uint_as_float(d[4 * i + 2]), __uint_as_float(d[4 * i + 3])), X[2 * i + 1]));
                        }
                        auto store = [&]() {
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                uint32_t a[2][8];
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const ulonglong2 w = put[q * 4 + i];
                                    two_parts(mul2(w.x, X[q * 8 + 2 * i]), a[0][2 * i], a[1][2 * i]);
                                    two_parts(mul2(w.y, X[q * 8 + 2 * i + 1]), a[0][2 * i + 1], a[1][2 * i + 1]);
                                }
#pragma unroll
                                for (int e = 0; e < 2; ++e) tmem_st8u(lanes + cW + e * 32 + half * 16 + q * 8, a[e]);
                            }
                            tmem_st_wait();
                            arrive(bWP);
                            if (!x.outputs) return;
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                uint32_t a[2][8];
#pragma unroll
                                for (int i = 0; i < 8; ++i) two_parts(X[q * 8 + i], a[0][i], a[1][i]);
#pragma unroll
                                for (int e = 0; e < 2; ++e) tmem_st8u(lanes + cU + e * 32 + half * 16 + q * 8, a[e]);
                            }
                        };
                        if (!__any_sync(0xffffffffu, first < 32)) {
                            store();
                        } else {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                float b0, b1;
                                unpack2(X[i], b0, b1);
                                X[i] = pack2(2 * i >= first ? 0.f : b0, 2 * i + 1 >= first ? 0.f : b1);
                            }
                            store();
                        }
                    }
                    if (x.outputs) {
                        if (half == 0) {
                            float* aside = reinterpret_cast<float*>(smem + kAsideOff) + (o & 1) * 256 + col;
                            aside[0] = p.q_scale * down * (1.f / kTile);
                            aside[128] = __int_as_float(bad ? kQ - (int)(mark & 127u) : kQ);
                        }
                        tmem_st_wait();
                        arrive(bUP + (o & 1));
                        ++o;
                    }
                    float r = down;
                    if (more) {
                        const float big = large[(n & 3) * 128].x;
                        length = longer(end * length, 8.f * big);
                        r = rescale(n + 1);
                    }
                    const uint64_t r2 = pack2(r, r), keep2 = pack2(keep * r, keep * r);
                    const bool same = __all_sync(0xffffffffu, r == 1.f);
                    // S, times the next chunk's scale (behind the last chunk as it is)
                    ok = warp_wait(bar + bProd, n & 1);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        tmem_ld32_async(lanes + cP + half * 64 + i * 32, d);
                        tmem_ld_wait();
                        if (same) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) S[i * 16 + j] = fma2(keep2, S[i * 16 + j], pack2(__uint_as_float(d[2 * j]), __uint_as_float(d[2 * j + 1])));
                        } else {
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                S[i * 16 + j] = fma2(r2, pack2(__uint_as_float(d[2 * j]), __uint_as_float(d[2 * j + 1])), mul2(keep2, S[i * 16 + j]));
                        }
                        if (more) give(i);
                    }
                }
                if (!ok || t >= rows.y) break;
                // A chunk whose numbers may be too far apart.
                if (o > 0) ok = warp_wait(bar + bOutFree + ((o - 1) & 1), ((o - 1) >> 1) & 1);
                if (!ok) break;
                Alone c;
                uint32_t* v = reinterpret_cast<uint32_t*>(smem + kYOff) + half * 16 * 128 + col;
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i * 128] = f[i];
#pragma unroll
                for (int i = 0; i < 32; ++i) c.S[i] = S[i];
                state_most(n);
                c.smem = smem;
                c.stage = smem + (n & 1) * kStage;
                c.bar = bar;
                c.pair = bar + bPair + quad;
                c.rest = reinterpret_cast<const float*>(p.work + ((size_t)(x.chunk + (t - rows.x) / kQ) * p.H + x.head) * kBlock + kGOff);
                c.most = most + (n & 1) * 256;
                c.next = &large[((n + 1) & 3) * 128].x;
                c.up = up;
                c.down = down;
                c.length = length;
                c.q_scale = p.q_scale;
                c.lanes = lanes;
                c.n = n;
                c.m = m;
                c.o = o;
                c.col = col;
                c.half = half;
                c.valid = min(kQ, rows.y - t);
                c.met = met;
                c.zero = t == rows.x && zero;
                c.outputs = x.outputs;
                c.live = stored || t > rows.x;
                c.more = t + kQ < rows.y;
                c.ok = true;
                const bool alone = token_by_token(c);
                met = c.met;
                ok = c.ok;
                if (!ok) break;
#pragma unroll
                for (int i = 0; i < 32; ++i) S[i] = c.S[i];
                length = c.length;                       // (measured now)
                if (alone) {
                    up = c.up;
                    down = c.down;
                    if (c.live) ++m;
                    if (x.outputs) ++o;
                    t += kQ;
                    ++n;
                    if (t >= rows.y) break;
                    fetch(n);
                    const float2 sizes = large[(n & 3) * 128];
                    doubt = !(sizes.y * up >= kFloor) && (sizes.x > 0.f || length > 0.f);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) f[i] = v[i * 128];
                    checked = true;
                }
            }
            if (!ok) break;
            const int dst = x.kind == kWhole || (x.kind == kLater && x.seg == g.segments - 1) ? seq_slot(p.pr, x.seq) : -1;
            float* to = dst >= 0 ? p.state + ((size_t)dst * p.H + x.head) * 128 * 128
                        : x.kind == kFirst ? scratch_state(g, x.seq, x.head, 0)
                        : x.kind >= kAlone ? scratch_state(g, x.seq, x.head, g.segments - 1 + 2 * (x.seg - 1) + (x.kind == kMap)) : nullptr;
            if (to != nullptr) {
                to += at;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    float a, c;
                    unpack2(S[i], a, c);
                    to[2 * i * 128] = a;
                    to[(2 * i + 1) * 128] = c;
                }
            }
        }
        if (!ok && lane == 0) record_fault(p.status, kFaultScanWait, 14);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_free<512>(tmem);
}

// The states that segments 2 .. n - 1 begin with: one after the other M S + N.  A CTA takes 32 value columns of a sequence and head; a thread
// four rows of four columns.  The next M comes while one is multiplied.
constexpr int kJoinThreads = 256;
constexpr uint32_t kJoinMat = 128u * 132u;
constexpr uint32_t kJoinSmem = (2u * kJoinMat + 128u * 32u) * 4u;
__global__ void __launch_bounds__(kJoinThreads) delta_join_kernel(const DeltaArgs g) {
    extern __shared__ __align__(16) float mat[];         // two times M [128][132], S [128][32]
    float* sx = mat + 2 * kJoinMat;
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int tid = (int)threadIdx.x, n = g.segments, c0 = (int)blockIdx.x % 4 * 32, head = (int)blockIdx.x / 4 % g.p.H, seq = (int)blockIdx.x / 4 / g.p.H;
    auto copy = [&](int s) {
        const float* M = scratch_state(g, seq, head, n - 1 + 2 * (s - 1) + 1);
        float* to = mat + (s & 1) * kJoinMat;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int e = i * kJoinThreads + tid;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to + e / 32 * 132 + e % 32 * 4)), "l"(M + e * 4) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    copy(1);
    for (int i = tid; i < 1024; i += kJoinThreads)
        *reinterpret_cast<float4*>(sx + i * 4) = *reinterpret_cast<const float4*>(scratch_state(g, seq, head, 0) + i / 8 * 128 + c0 + i % 8 * 4);
    const int k = tid / 8, c = tid % 8 * 4;              // rows k, k + 32, ..
    for (int s = 1; s < n - 1; ++s) {
        const float* N = scratch_state(g, seq, head, n - 1 + 2 * (s - 1)) + k * 128 + c0 + c;
        float4 y[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] = *reinterpret_cast<const float4*>(N + q * 32 * 128);
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();                                 // M and S are there, and nobody reads the other M any more
        if (s + 1 < n - 1) copy(s + 1);
        const float* M = mat + (s & 1) * kJoinMat + k * 132;
#pragma unroll 2
        for (int j = 0; j < 128; j += 4) {
            float m[4][4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 v = *reinterpret_cast<const float4*>(M + q * 32 * 132 + j);
                m[q][0] = v.x; m[q][1] = v.y; m[q][2] = v.z; m[q][3] = v.w;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float4 x = *reinterpret_cast<const float4*>(sx + (j + e) * 32 + c);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    y[q].x = fmaf(m[q][e], x.x, y[q].x); y[q].y = fmaf(m[q][e], x.y, y[q].y);
                    y[q].z = fmaf(m[q][e], x.z, y[q].z); y[q].w = fmaf(m[q][e], x.w, y[q].w);
                }
            }
        }
        __syncthreads();                                 // nobody reads S any more
        float* to = scratch_state(g, seq, head, s) + k * 128 + c0 + c;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            *reinterpret_cast<float4*>(sx + (k + q * 32) * 32 + c) = y[q];
            *reinterpret_cast<float4*>(to + q * 32 * 128) = y[q];
        }
    }
}

}  // namespace

// bf16 rows in tiles of 64 x 128 elements, as they are.
static bool make_rows_map(CUtensorMap* map, const void* base, uint64_t cols, uint64_t rows, uint64_t stride) {
    const auto encode = tensor_map_encoder();
    if (encode == nullptr) return false;
    const cuuint64_t dims[2] = {cols, rows}, strides[1] = {stride};
    const cuuint32_t box[2] = {128, kQ}, steps[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Segments of a sequence (1: none) and units of the first pass a CTA, for the least time, estimated for sequences of the average length: turns + 1
// times a segment's chunks at 3 us each, and what the small kernel and the units' starts take, some 30 us and 8 a segment.  Each pass has an
// SM for each of its CTAs: in the first one of every first segment and one for `turns` of the 2 (n - 2) others, in the second n - 1.
// One prompt, a key head for each head, whole and split: 16384 tokens of 4 heads 773 and 237 us, of 32 948 and 673, of 64 1169 and 1085; 2048 of 16
// heads 120 and 102.  16384 of 32 heads, a key head for two: 881 and 606 (five segments, two turns; three and one took a sixth longer).
struct Split {
    int segments, turns;
};
static Split delta_split(long long sequences, long long heads, long long tokens, int sms) {
    const long long pairs = sequences * heads, chunks = (tokens / sequences + kQ - 1) / kQ;
    Split best = {1, 1};
    long long least = 3 * chunks;
    for (int turns = 1; turns <= 4; ++turns)
        for (int n = 3; n <= 16; ++n) {
            if ((n - 1) * pairs > sms || pairs + (2 * (n - 2) * pairs + turns - 1) / turns > sms) break;
            const long long per = (chunks + turns + n - 2) / (turns + n - 1), time = 3 * (turns + 1) * per + 30 + 8 * (n - 2);
            if (time < least) {
                least = time;
                best = {n, turns};
            }
        }
    return best;
}

// Tokens of a batch up to which the CUDA cores are faster whatever the sequences are: 1 token of 4 heads in 5.6 us, 19.5 here; 16 sequences of 2
// tokens, 32 heads, 28.1 and 51.2; one of 32 tokens, 32 heads, 11.8 and 20.1; one of 64 19.9 and 20.1.  (More sequences of a few tokens would be faster
// there too, 256 of 4, 4 heads, 45 and 86, but one long one among them would not, and the lengths are not known here.)
constexpr long long kFewTokens = 32;

// (The scratch's size is asked for without a device: it holds for so many SMs, and no more of them are counted on.)
constexpr int kMostSms = 148;

size_t delta_tc_work_bytes(const sketchssm_config& c, long long sequences, long long tokens) {
    if (c.kind != SKETCHSSM_GDN || c.io_dtype != SKETCHSSM_BF16 || c.dk != 128 || c.dv != 128 || sequences == 0 || tokens <= kFewTokens) return 0;
    // (The groups are not known here: every head may be one.  Fewer sequences than asked for may be split into more segments: of all of them
    // together 3 n - 5 states, less than three times the SMs.  Sequences below 15 chunks are not split.)
    const size_t states = c.heads <= kMostSms / 2 && 3 * tokens > 64 * 38 ? 3 * kMostSms : 0;
    return (size_t)(tokens / kQ + sequences) * c.heads * (kBlock + kRows) + ((size_t)sequences * 4 + 15) / 16 * 16 + states * 128 * 128 * 4 + 16;
}

int launch_delta_scan_tc(Ctx* ctx, const DeltaParams& p, bool bf16, cudaStream_t stream) {
    if (!bf16 || !p.out_bf16 || p.K != 128 || p.V != 128 || p.pr.T <= kFewTokens || ctx->cfg.kind != SKETCHSSM_GDN) return SKETCHSSM_UNSUPPORTED_SHAPE;
    DeltaArgs g;
    g.p = p;
    g.p.work += -reinterpret_cast<uintptr_t>(p.work) & 31u;     // (whole sectors are written there; the scratch begins on 16 bytes)
    const long long units = (long long)p.pr.N * p.H, chunks = (long long)p.pr.T / kQ + p.pr.N;
    const long long preps = chunks * p.G * ((p.H / p.G + 1) / 2);
    if (units > (1 << 30) || preps >= 0x7fffffffll) return SKETCHSSM_UNSUPPORTED_SHAPE;
    const Split split = delta_split(p.pr.N, p.H, p.pr.T, sm_count(ctx) < kMostSms ? sm_count(ctx) : kMostSms);
    g.segments = split.segments;
    g.turns = split.turns;
    g.preps = (int)preps;
    g.rows = g.p.work + (size_t)chunks * p.H * kBlock;
    unsigned char* behind = g.rows + (size_t)chunks * p.H * kRows;
    const bool sort = g.segments == 1 && p.pr.N > 1;
    g.order = sort ? reinterpret_cast<int*>(behind) : nullptr;
    g.states = reinterpret_cast<float*>(behind + ((size_t)p.pr.N * 4 + 15) / 16 * 16);
    if (!make_map(&g.tq, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.q, (uint64_t)p.G * 128, (uint64_t)p.pr.T, (uint64_t)p.q_stride * 2, kQ) ||
        !make_map(&g.tk, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.k, (uint64_t)p.G * 128, (uint64_t)p.pr.T, (uint64_t)p.k_stride * 2, kQ) ||
        !make_rows_map(&g.tv, p.v, (uint64_t)p.H * 128, (uint64_t)p.pr.T, (uint64_t)p.v_stride * 2)) {
        ctx->last_cuda_error = cudaErrorInvalidValue;
        return SKETCHSSM_CUDA_ERROR;
    }
    cudaError_t e = unlock_smem(ctx, delta_prep_kernel);
    if (e == cudaSuccess) e = unlock_smem(ctx, delta_scan_tc_kernel);
    if (e == cudaSuccess && g.segments > 1) e = unlock_smem(ctx, delta_join_kernel);
    if (e != cudaSuccess) { ctx->last_cuda_error = e; return SKETCHSSM_CUDA_ERROR; }
    int rc = launch_layer<DeltaArgs>(ctx, delta_prep_kernel, dim3((unsigned)(preps + sort)), dim3(kPrepThreads), kPrepSmem, stream, g);
    auto scan = [&](int pass, long long parts) {
        g.pass = pass;
        g.units = (int)(units * parts);
        const long long ctas = pass == 1 ? units + (g.units + g.turns - 1) / g.turns : g.units;
        const unsigned grid = (unsigned)(pass == 1 || ctas < sm_count(ctx) ? ctas : sm_count(ctx));
        return launch_layer<DeltaArgs>(ctx, delta_scan_tc_kernel, dim3(grid), dim3(kThreads), kSmemTc, stream, g);
    };
    if (rc == SKETCHSSM_OK && g.segments == 1) return scan(0, 1);
    if (rc == SKETCHSSM_OK) rc = scan(1, 2 * (g.segments - 2));
    if (rc == SKETCHSSM_OK) rc = launch_layer<DeltaArgs>(ctx, delta_join_kernel, dim3((unsigned)(units * 4)), dim3(kJoinThreads), kJoinSmem, stream, g);
    return rc == SKETCHSSM_OK ? scan(2, g.segments - 1) : rc;
}

}  // namespace sketchssm
