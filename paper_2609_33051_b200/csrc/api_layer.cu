// C ABI of the operators around the recurrence: argument checking and kernel dispatch.
#include "layer.cuh"

using namespace sketchssm;

namespace {

// What every call asks first.
int begin_call(sketchssm_ctx* ctx) {
    if (ctx == nullptr) return SKETCHSSM_INVALID_ARG;
    ctx->last_launches = 0;
    return ctx->bound ? SKETCHSSM_OK : SKETCHSSM_NOT_BOUND;
}

inline bool good(const void* p) { return p != nullptr && aligned16(p); }
inline bool good_or_null(const void* p) { return aligned16(p); }
inline bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool dtype_ok(int d) { return d == SKETCHSSM_F32 || d == SKETCHSSM_BF16; }
// Row stride of rows of `width` elements of `size` bytes: at least a row, and rows 16-byte aligned.
inline bool stride_ok(int64_t stride, int64_t width, int size) {
    return stride >= width && stride <= ((int64_t)1 << 31) && (stride * size) % 16 == 0;
}

int check_prompts(const sketchssm_ctx* ctx, const sketchssm_prompts* pr, PromptsDev* out) {
    if (pr == nullptr || pr->sequences < 0 || pr->tokens < 0) return SKETCHSSM_INVALID_ARG;
    if (pr->sequences > 0 && pr->starts == nullptr) return SKETCHSSM_INVALID_ARG;
    if (!aligned_to(pr->starts, 4) || !aligned_to(pr->slots, 4) || !aligned_to(pr->resume, 4)) return SKETCHSSM_INVALID_ARG;
    if (pr->slots == nullptr && pr->sequences > ctx->cfg.batch) return SKETCHSSM_INVALID_ARG;
    // rows are numbered in 32 bits, with room for a tile behind the last one
    if (pr->tokens > (1 << 30) || pr->sequences > (1 << 24)) return SKETCHSSM_UNSUPPORTED_SHAPE;
    *out = PromptsDev{pr->starts, pr->slots, pr->resume, pr->sequences, pr->tokens, ctx->cfg.batch};
    return SKETCHSSM_OK;
}

// The arguments of the delta rule's decays: a number a head (GDN), or K of them (KDA), whose rows are read 16 bytes at a time.
bool decay_ok(const sketchssm_ctx* ctx, const void* dt, int64_t stride) {
    const sketchssm_config& c = ctx->cfg;
    return c.kind == SKETCHSSM_KDA ? aligned16(dt) && stride_ok(stride, (int64_t)c.heads * c.dk, ctx->io_size) : stride >= c.heads;
}

}  // namespace

extern "C" {

int sketchssm_causal_conv(sketchssm_ctx* ctx, const sketchssm_prompts* prompts, int channels, int width, const void* weight,
                          const void* bias, void* state, const void* x, int64_t x_stride, void* out, int64_t out_stride,
                          uint32_t flags, void* stream) {
    int rc = begin_call(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    ConvParams p{};
    rc = check_prompts(ctx, prompts, &p.pr);
    if (rc != SKETCHSSM_OK) return rc;
    if (flags & ~SKETCHSSM_SILU) return SKETCHSSM_INVALID_ARG;
    if (channels < 1) return SKETCHSSM_INVALID_ARG;
    if (width < 2 || width > 4 || channels > (1 << 20) || (channels * ctx->io_size) % 16 != 0) return SKETCHSSM_UNSUPPORTED_SHAPE;
    if (!good(weight) || !good_or_null(bias) || !good(state)) return SKETCHSSM_INVALID_ARG;
    if (p.pr.T > 0 && (!good(x) || !good(out))) return SKETCHSSM_INVALID_ARG;
    if (!stride_ok(x_stride, channels, ctx->io_size) || !stride_ok(out_stride, channels, ctx->io_size)) return SKETCHSSM_INVALID_ARG;
    if (p.pr.N == 0) return SKETCHSSM_OK;
    rc = set_device(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    p.weight = static_cast<const float*>(weight); p.bias = static_cast<const float*>(bias); p.state = state;
    p.x = x; p.out = out; p.x_stride = x_stride; p.out_stride = out_stride;
    p.C = channels; p.W = width; p.silu = (flags & SKETCHSSM_SILU) ? 1 : 0;
    return launch_causal_conv(ctx, p, ctx->cfg.io_dtype == SKETCHSSM_BF16, static_cast<cudaStream_t>(stream));
}

int sketchssm_conv_step(sketchssm_ctx* ctx, int groups, int width, const void* weight, const void* bias, void* state,
                        const void* x, int64_t x_stride, const void* dt, int64_t dt_stride, const void* a,
                        const void* dt_bias, void* q, void* k, void* v, void* beta, void* decay, void* stream) {
    int rc = begin_call(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    const sketchssm_config& c = ctx->cfg;
    if (c.kind != SKETCHSSM_MAMBA2) return SKETCHSSM_UNSUPPORTED_SHAPE;
    if (groups < 1 || c.heads % groups != 0) return SKETCHSSM_INVALID_ARG;
    if (width < 2 || width > 4) return SKETCHSSM_UNSUPPORTED_SHAPE;
    const void* ps[10] = {weight, state, x, a, q, k, v, beta, decay, dt};
    for (const void* p : ps)
        if (p == nullptr || (p != dt && p != a && !aligned16(p))) return SKETCHSSM_INVALID_ARG;
    if (!good_or_null(bias) || !aligned_to(dt_bias, 4) || !aligned_to(a, 4) || !aligned_to(dt, ctx->io_size)) return SKETCHSSM_INVALID_ARG;
    const int64_t channels = (int64_t)c.heads * c.dv + 2ll * groups * c.dk;
    if (channels > (1 << 20)) return SKETCHSSM_UNSUPPORTED_SHAPE;
    if (!stride_ok(x_stride, channels, ctx->io_size) || dt_stride < c.heads) return SKETCHSSM_INVALID_ARG;
    rc = set_device(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    ConvStepParams p{};
    p.weight = static_cast<const float*>(weight); p.bias = static_cast<const float*>(bias); p.state = state;
    p.x = x; p.dt = dt; p.a = static_cast<const float*>(a); p.dt_bias = static_cast<const float*>(dt_bias);
    p.q = q; p.k = k; p.v = v; p.beta = static_cast<float*>(beta); p.decay = static_cast<float*>(decay);
    p.x_stride = x_stride; p.dt_stride = dt_stride;
    p.B = c.batch; p.H = c.heads; p.G = groups; p.K = c.dk; p.V = c.dv; p.W = width;
    return launch_conv_step(ctx, p, c.io_dtype == SKETCHSSM_BF16, static_cast<cudaStream_t>(stream));
}

int sketchssm_prompt_work_bytes(const sketchssm_ctx* ctx, int sequences, int tokens, size_t* bytes) {
    if (ctx == nullptr || bytes == nullptr || sequences < 0 || tokens < 0) return SKETCHSSM_INVALID_ARG;
    const sketchssm_config& c = ctx->cfg;
    const size_t states = sequences > 0 ? (size_t)scan_segment_states(c, tokens) : 0;
    *bytes = (states * c.heads * ((size_t)c.dk * c.dv + 1) * 4 + 15) & ~(size_t)15;
    return SKETCHSSM_OK;
}

int sketchssm_prompt_scan(sketchssm_ctx* ctx, const sketchssm_prompts* prompts, int groups, const void* q, int64_t q_stride,
                          const void* k, int64_t k_stride, const void* v, int64_t v_stride, const void* dt, int64_t dt_stride,
                          const void* a, const void* dt_bias, const void* skip, void* out, int64_t out_stride, int out_dtype,
                          void* work, size_t work_bytes, void* stream) {
    int rc = begin_call(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    const sketchssm_config& c = ctx->cfg;
    ScanParams p{};
    rc = check_prompts(ctx, prompts, &p.pr);
    if (rc != SKETCHSSM_OK) return rc;
    if (c.kind != SKETCHSSM_MAMBA2) return SKETCHSSM_UNSUPPORTED_SHAPE;
    if (groups < 1 || c.heads % groups != 0 || !dtype_ok(out_dtype)) return SKETCHSSM_INVALID_ARG;
    if (p.pr.T > 0) {
        const void* ps[4] = {q, k, v, out};
        for (const void* x : ps)
            if (!good(x)) return SKETCHSSM_INVALID_ARG;
        if (dt == nullptr) return SKETCHSSM_INVALID_ARG;
    }
    if (a == nullptr || !aligned_to(a, 4) || !aligned_to(dt_bias, 4) || !aligned_to(skip, 4) || !aligned_to(dt, ctx->io_size))
        return SKETCHSSM_INVALID_ARG;
    const int64_t gk = (int64_t)groups * c.dk, hv = (int64_t)c.heads * c.dv;
    if (!stride_ok(q_stride, gk, ctx->io_size) || !stride_ok(k_stride, gk, ctx->io_size) || !stride_ok(v_stride, hv, ctx->io_size) ||
        !stride_ok(out_stride, hv, out_dtype == SKETCHSSM_BF16 ? 2 : 4) || dt_stride < c.heads)
        return SKETCHSSM_INVALID_ARG;
    size_t need = 0;
    rc = sketchssm_prompt_work_bytes(ctx, p.pr.N, p.pr.T, &need);
    if (rc != SKETCHSSM_OK) return rc;
    if (work_bytes < need || (need > 0 && !good(work))) return SKETCHSSM_INVALID_ARG;
    if (p.pr.N == 0) return SKETCHSSM_OK;
    rc = set_device(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    p.q = q; p.k = k; p.v = v; p.dt = dt;
    p.a = static_cast<const float*>(a); p.dt_bias = static_cast<const float*>(dt_bias); p.skip = static_cast<const float*>(skip);
    p.out = out; p.state = static_cast<float*>(ctx->bufs.state); p.work = static_cast<float*>(work);
    p.status = static_cast<int*>(ctx->bufs.status);
    p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride; p.dt_stride = dt_stride; p.out_stride = out_stride;
    p.H = c.heads; p.G = groups; p.K = c.dk; p.V = c.dv; p.out_bf16 = out_dtype == SKETCHSSM_BF16;
    return launch_prompt_scan(ctx, p, c.io_dtype == SKETCHSSM_BF16, static_cast<cudaStream_t>(stream));
}

int sketchssm_rms_norm(sketchssm_ctx* ctx, int rows, int width, int group, float eps, const void* x, int64_t x_stride,
                       int x_dtype, const void* weight, const void* residual, void* residual_out, const void* gate,
                       int64_t gate_stride, const void* skip, int64_t skip_stride, const void* skip_weight, int skip_heads,
                       void* out, void* out8, void* scale, void* stream) {
    int rc = begin_call(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    if (rows < 0 || width < 1 || group < 0 || !(eps >= 0.f) || !dtype_ok(x_dtype)) return SKETCHSSM_INVALID_ARG;
    if ((width & 7) || width > 16384) return SKETCHSSM_UNSUPPORTED_SHAPE;
    if (group == 0 || group == width) {
        group = width;
    } else {
        if (group > width || width % group != 0) return SKETCHSSM_INVALID_ARG;
        if (group % 128 != 0) return SKETCHSSM_UNSUPPORTED_SHAPE;
    }
    if ((residual == nullptr) != (residual_out == nullptr) || (out8 == nullptr) != (scale == nullptr)) return SKETCHSSM_INVALID_ARG;
    if (out == nullptr && out8 == nullptr) return SKETCHSSM_INVALID_ARG;
    if (residual != nullptr && gate != nullptr) return SKETCHSSM_INVALID_ARG;
    if ((skip == nullptr) != (skip_weight == nullptr) || (skip != nullptr && gate == nullptr)) return SKETCHSSM_INVALID_ARG;
    if (skip != nullptr && (skip_heads < 1 || width % skip_heads != 0)) return SKETCHSSM_INVALID_ARG;
    if (!good(weight) || !aligned_to(skip_weight, 4) || !aligned_to(scale, 4)) return SKETCHSSM_INVALID_ARG;
    if (rows > 0 && x == nullptr) return SKETCHSSM_INVALID_ARG;
    const void* ps[7] = {x, residual, residual_out, gate, skip, out, out8};
    for (const void* p : ps)
        if (!aligned16(p)) return SKETCHSSM_INVALID_ARG;
    const int xs = x_dtype == SKETCHSSM_BF16 ? 2 : 4;
    if (!stride_ok(x_stride, width, xs) || (gate != nullptr && !stride_ok(gate_stride, width, ctx->io_size)) ||
        (skip != nullptr && !stride_ok(skip_stride, width, ctx->io_size)))
        return SKETCHSSM_INVALID_ARG;
    if (rows == 0) return SKETCHSSM_OK;
    if ((int64_t)rows * (width / group) > 0x7fffffff) return SKETCHSSM_UNSUPPORTED_SHAPE;
    rc = set_device(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    NormParams p{};
    p.x = x; p.weight = static_cast<const float*>(weight); p.residual = residual; p.residual_out = residual_out;
    p.gate = gate; p.skip = skip; p.skip_weight = static_cast<const float*>(skip_weight);
    p.out = out; p.out8 = out8; p.scale = static_cast<float*>(scale);
    p.x_stride = x_stride; p.gate_stride = gate_stride; p.skip_stride = skip_stride;
    p.rows = rows; p.width = width; p.group = group; p.groups = width / group; p.skip_heads = skip_heads;
    p.x_bf16 = x_dtype == SKETCHSSM_BF16; p.eps = eps;
    return launch_rms_norm(ctx, p, ctx->cfg.io_dtype == SKETCHSSM_BF16, static_cast<cudaStream_t>(stream));
}

int sketchssm_scaled_matmul(sketchssm_ctx* ctx, int rows, int cols, int inner, const void* a, const void* a_scale,
                            const void* w, const void* w_scale, void* out, int64_t out_stride, int out_dtype, void* stream) {
    int rc = begin_call(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    if (rows < 0 || cols < 1 || inner < 1 || !dtype_ok(out_dtype)) return SKETCHSSM_INVALID_ARG;
    // rows and columns are numbered in 32 bits, with room for a tile behind the last one
    if (inner % 16 != 0 || rows > (1 << 30) || cols > (1 << 30) || inner > (1 << 30)) return SKETCHSSM_UNSUPPORTED_SHAPE;
    if (out_stride < cols) return SKETCHSSM_INVALID_ARG;
    if (!good(w) || w_scale == nullptr || !aligned_to(w_scale, 4)) return SKETCHSSM_INVALID_ARG;
    if (rows == 0) return SKETCHSSM_OK;
    if (!good(a) || a_scale == nullptr || !aligned_to(a_scale, 4) || !good(out)) return SKETCHSSM_INVALID_ARG;
    rc = set_device(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    MatmulParams p{};
    p.a = static_cast<const unsigned char*>(a); p.w = static_cast<const unsigned char*>(w);
    p.a_scale = static_cast<const float*>(a_scale); p.w_scale = static_cast<const float*>(w_scale);
    p.out = out; p.status = static_cast<int*>(ctx->bufs.status); p.out_stride = out_stride;
    p.M = rows; p.N = cols; p.K = inner; p.KB = (inner + 127) / 128; p.out_bf16 = out_dtype == SKETCHSSM_BF16;
    return launch_scaled_matmul(ctx, p, static_cast<cudaStream_t>(stream));
}

int sketchssm_delta_step(sketchssm_ctx* ctx, int groups, int width, float eps, float q_scale, const void* weight, const void* bias, void* state,
                         const void* x, int64_t x_stride, const void* b, int64_t b_stride, const void* dt, int64_t dt_stride, const void* a,
                         const void* dt_bias, void* q, void* k, void* v, void* beta, void* decay, void* stream) {
    int rc = begin_call(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    const sketchssm_config& c = ctx->cfg;
    if (c.kind == SKETCHSSM_MAMBA2) return SKETCHSSM_UNSUPPORTED_SHAPE;
    if (groups < 1 || c.heads % groups != 0 || !(eps > 0.f) || !(q_scale == q_scale)) return SKETCHSSM_INVALID_ARG;
    if (width < 2 || width > 4) return SKETCHSSM_UNSUPPORTED_SHAPE;
    const void* ps[8] = {weight, state, x, q, k, v, beta, decay};
    for (const void* p : ps)
        if (!good(p)) return SKETCHSSM_INVALID_ARG;
    if (b == nullptr || dt == nullptr || a == nullptr || !good_or_null(bias) || !aligned_to(dt_bias, 4) || !aligned_to(a, 4) || !aligned_to(b, ctx->io_size) ||
        !aligned_to(dt, ctx->io_size))
        return SKETCHSSM_INVALID_ARG;
    const int64_t channels = (int64_t)c.heads * c.dv + 2ll * groups * c.dk;
    if (channels > (1 << 20) || (int64_t)c.heads * c.dk > (1 << 20)) return SKETCHSSM_UNSUPPORTED_SHAPE;
    if (!stride_ok(x_stride, channels, ctx->io_size) || b_stride < c.heads || !decay_ok(ctx, dt, dt_stride)) return SKETCHSSM_INVALID_ARG;
    rc = set_device(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    DeltaStepParams p{};
    p.c.weight = static_cast<const float*>(weight); p.c.bias = static_cast<const float*>(bias); p.c.state = state;
    p.c.x = x; p.c.dt = dt; p.c.a = static_cast<const float*>(a); p.c.dt_bias = static_cast<const float*>(dt_bias);
    p.c.q = q; p.c.k = k; p.c.v = v; p.c.beta = static_cast<float*>(beta);
    p.c.x_stride = x_stride; p.c.dt_stride = dt_stride;
    p.c.B = c.batch; p.c.H = c.heads; p.c.G = groups; p.c.K = c.dk; p.c.V = c.dv; p.c.W = width;
    p.b = b; p.b_stride = b_stride; p.decay = decay; p.eps = eps; p.q_scale = q_scale;
    return launch_delta_step(ctx, p, c.io_dtype == SKETCHSSM_BF16, static_cast<cudaStream_t>(stream));
}

int sketchssm_delta_work_bytes(const sketchssm_ctx* ctx, int sequences, int tokens, size_t* bytes) {
    if (ctx == nullptr || bytes == nullptr || sequences < 0 || tokens < 0) return SKETCHSSM_INVALID_ARG;
    const sketchssm_config& c = ctx->cfg;
    *bytes = c.kind == SKETCHSSM_KDA ? (sequences > 0 ? (size_t)tokens * c.heads * c.dk * 4 : 0) : delta_tc_work_bytes(c, sequences, tokens);
    return SKETCHSSM_OK;
}

int sketchssm_delta_scan(sketchssm_ctx* ctx, const sketchssm_prompts* prompts, int groups, float eps, float q_scale, const void* q, int64_t q_stride,
                         const void* k, int64_t k_stride, const void* v, int64_t v_stride, const void* b, int64_t b_stride, const void* dt,
                         int64_t dt_stride, const void* a, const void* dt_bias, void* out, int64_t out_stride, int out_dtype, void* work,
                         size_t work_bytes, void* stream) {
    int rc = begin_call(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    const sketchssm_config& c = ctx->cfg;
    DeltaParams p{};
    rc = check_prompts(ctx, prompts, &p.pr);
    if (rc != SKETCHSSM_OK) return rc;
    if (c.kind == SKETCHSSM_MAMBA2) return SKETCHSSM_UNSUPPORTED_SHAPE;
    if (groups < 1 || c.heads % groups != 0 || !dtype_ok(out_dtype) || !(eps > 0.f) || !(q_scale == q_scale)) return SKETCHSSM_INVALID_ARG;
    if (p.pr.T > 0) {
        const void* ps[4] = {q, k, v, out};
        for (const void* x : ps)
            if (!good(x)) return SKETCHSSM_INVALID_ARG;
        if (b == nullptr || dt == nullptr) return SKETCHSSM_INVALID_ARG;
    }
    if (a == nullptr || !aligned_to(a, 4) || !aligned_to(dt_bias, 4) || !aligned_to(b, ctx->io_size) || !aligned_to(dt, ctx->io_size)) return SKETCHSSM_INVALID_ARG;
    const int64_t gk = (int64_t)groups * c.dk, hv = (int64_t)c.heads * c.dv;
    if (!stride_ok(q_stride, gk, ctx->io_size) || !stride_ok(k_stride, gk, ctx->io_size) || !stride_ok(v_stride, hv, ctx->io_size) ||
        !stride_ok(out_stride, hv, out_dtype == SKETCHSSM_BF16 ? 2 : 4) || b_stride < c.heads || !decay_ok(ctx, dt, dt_stride))
        return SKETCHSSM_INVALID_ARG;
    size_t need = 0;
    // (GDN into fp32 goes over CUDA cores, which need none)
    if (c.kind == SKETCHSSM_KDA || out_dtype == SKETCHSSM_BF16) rc = sketchssm_delta_work_bytes(ctx, p.pr.N, p.pr.T, &need);
    if (rc != SKETCHSSM_OK) return rc;
    if (work_bytes < need || (need > 0 && !good(work))) return SKETCHSSM_INVALID_ARG;
    if (p.pr.N == 0) return SKETCHSSM_OK;
    rc = set_device(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    p.q = q; p.k = k; p.v = v; p.b = b; p.dt = dt;
    p.a = static_cast<const float*>(a); p.dt_bias = static_cast<const float*>(dt_bias);
    p.out = out; p.state = static_cast<float*>(ctx->bufs.state); p.work = static_cast<unsigned char*>(work);
    p.status = static_cast<int*>(ctx->bufs.status);
    p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride; p.b_stride = b_stride; p.dt_stride = dt_stride; p.out_stride = out_stride;
    p.eps = eps; p.q_scale = q_scale;
    p.H = c.heads; p.G = groups; p.K = c.dk; p.V = c.dv; p.out_bf16 = out_dtype == SKETCHSSM_BF16;
    return launch_delta_scan(ctx, p, c.io_dtype == SKETCHSSM_BF16, static_cast<cudaStream_t>(stream));
}

int sketchssm_integer_norm(sketchssm_ctx* ctx, int rows, int width, int group, float eps, const void* x, int64_t x_stride, int x_dtype,
                        const void* weight, const void* residual, void* residual_out, const void* gate, int64_t gate_stride, uint32_t flags,
                        void* out, void* out8, void* scale, void* stream) {
    int rc = begin_call(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    if (rows < 0 || width < 1 || group < 1 || !(eps >= 0.f) || !dtype_ok(x_dtype) || (flags & ~SKETCHSSM_SIGMOID)) return SKETCHSSM_INVALID_ARG;
    if (group > width || width % group != 0) return SKETCHSSM_INVALID_ARG;
    if ((group & 7) || width > 16384) return SKETCHSSM_UNSUPPORTED_SHAPE;
    if ((residual == nullptr) != (residual_out == nullptr) || (residual != nullptr && gate != nullptr)) return SKETCHSSM_INVALID_ARG;
    if (!good(weight) || !aligned_to(scale, 4)) return SKETCHSSM_INVALID_ARG;
    if (rows > 0 && (x == nullptr || out8 == nullptr || scale == nullptr)) return SKETCHSSM_INVALID_ARG;
    const void* ps[6] = {x, residual, residual_out, gate, out, out8};
    for (const void* p : ps)
        if (!aligned16(p)) return SKETCHSSM_INVALID_ARG;
    if (!stride_ok(x_stride, width, x_dtype == SKETCHSSM_BF16 ? 2 : 4) || (gate != nullptr && !stride_ok(gate_stride, width, ctx->io_size)))
        return SKETCHSSM_INVALID_ARG;
    if (rows == 0) return SKETCHSSM_OK;
    rc = set_device(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    Norm8Params p{};
    p.x = x; p.weight = static_cast<const float*>(weight); p.residual = residual; p.residual_out = residual_out; p.gate = gate;
    p.out = out; p.out8 = static_cast<signed char*>(out8); p.scale = static_cast<float*>(scale);
    p.x_stride = x_stride; p.gate_stride = gate_stride;
    p.rows = rows; p.width = width; p.group = group; p.sigmoid = (flags & SKETCHSSM_SIGMOID) ? 1 : 0; p.eps = eps;
    return launch_integer_norm(ctx, p, ctx->cfg.io_dtype == SKETCHSSM_BF16, x_dtype == SKETCHSSM_BF16, static_cast<cudaStream_t>(stream));
}

int sketchssm_integer_matmul(sketchssm_ctx* ctx, int rows, int cols, int inner, const void* a, const void* a_scale, const void* w,
                          const void* w_scale, void* out, int64_t out_stride, int out_dtype, void* stream) {
    int rc = begin_call(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    if (rows < 0 || cols < 1 || inner < 1 || !dtype_ok(out_dtype)) return SKETCHSSM_INVALID_ARG;
    // rows and columns are numbered in 32 bits, with room for a tile behind the last one; 2^14 x inner has to stay below 2^31
    if (inner % 16 != 0 || rows > (1 << 30) || cols > (1 << 30) || inner >= (1 << 17)) return SKETCHSSM_UNSUPPORTED_SHAPE;
    if (out_stride < cols) return SKETCHSSM_INVALID_ARG;
    if (!good(w) || w_scale == nullptr || !aligned_to(w_scale, 4)) return SKETCHSSM_INVALID_ARG;
    if (rows == 0) return SKETCHSSM_OK;
    if (!good(a) || a_scale == nullptr || !aligned_to(a_scale, 4) || !good(out)) return SKETCHSSM_INVALID_ARG;
    rc = set_device(ctx);
    if (rc != SKETCHSSM_OK) return rc;
    MatmulParams p{};
    p.a = static_cast<const unsigned char*>(a); p.w = static_cast<const unsigned char*>(w);
    p.a_scale = static_cast<const float*>(a_scale); p.w_scale = static_cast<const float*>(w_scale);
    p.out = out; p.status = static_cast<int*>(ctx->bufs.status); p.out_stride = out_stride;
    p.M = rows; p.N = cols; p.K = inner; p.KB = (inner + 127) / 128; p.out_bf16 = out_dtype == SKETCHSSM_BF16;
    return launch_integer_matmul(ctx, p, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
