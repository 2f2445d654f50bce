"""Refusals and host-side sizes of the operators around the recurrence, without a GPU: every one of these calls ends before any
CUDA call is made (the addresses are only checked, never dereferenced)."""
import ctypes

import pytest
import torch

from paper_2609_33051_b200 import binding, build

OK, INVALID, SHAPE, UNBOUND = 0, -1, -2, -3
P, Q = 1 << 20, (1 << 20) + 2          # an aligned address and one that is not


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def context(lib, bind=True, **kw):
    cfg = dict(kind=0, batch=4, heads=8, dk=128, dv=64, rank=8, buf_len=4, io_dtype=1, out_dtype=0, device=0)
    cfg.update(kw)
    ctx = ctypes.c_void_p()
    assert lib.sketchssm_create(ctypes.byref(binding.Config(**cfg)), ctypes.byref(ctx)) == OK
    if bind:
        assert lib.sketchssm_bind(ctx, ctypes.byref(binding.Buffers(*([P] * 7), None, None))) == OK
    return ctx


def prompts(sequences=0, tokens=16, starts=P, slots=P, resume=P):
    return binding.PromptBatch(sequences, tokens, starts, slots, resume)


def conv(lib, ctx, pr=None, C=64, W=4, weight=P, bias=P, state=P, x=P, xs=64, out=P, os=64, flags=1):
    return lib.sketchssm_causal_conv(ctx, ctypes.byref(pr or prompts()), C, W, weight, bias, state, x, xs, out, os, flags, None)


def test_conv_refusals(lib):
    ctx = context(lib)
    assert conv(lib, ctx) == OK                                        # no sequences: nothing to do
    assert conv(lib, ctx, bias=None) == OK
    assert lib.sketchssm_causal_conv(ctx, None, 64, 4, P, P, P, P, 64, P, 64, 0, None) == INVALID
    assert conv(lib, None) == INVALID
    assert conv(lib, context(lib, bind=False)) == UNBOUND
    for bad in (dict(W=1), dict(W=5), dict(C=60, xs=64, os=64)):
        assert conv(lib, ctx, **bad) == SHAPE, bad
    for bad in (dict(C=0), dict(weight=None), dict(weight=Q), dict(bias=Q), dict(state=None), dict(state=Q), dict(x=None), dict(x=Q),
                dict(out=None), dict(out=Q), dict(xs=56), dict(xs=68), dict(os=63), dict(flags=2),
                dict(pr=prompts(sequences=-1)), dict(pr=prompts(tokens=-1)), dict(pr=prompts(sequences=1, starts=None)),
                dict(pr=prompts(starts=Q)), dict(pr=prompts(slots=Q)), dict(pr=prompts(resume=Q)),
                dict(pr=prompts(sequences=5, slots=None))):
        assert conv(lib, ctx, **bad) == INVALID, bad
    assert conv(lib, ctx, pr=prompts(tokens=(1 << 30) + 1)) == SHAPE
    f32 = context(lib, io_dtype=0)
    assert conv(lib, f32, C=60, xs=60, os=60) == OK and conv(lib, f32, C=62, xs=64, os=64) == SHAPE


def step(lib, ctx, G=2, W=4, weight=P, bias=P, state=P, x=P, xs=1024, dt=P, ds=8, a=P, dt_bias=P, q=P, k=P, v=P, beta=P, decay=P):
    return lib.sketchssm_conv_step(ctx, G, W, weight, bias, state, x, xs, dt, ds, a, dt_bias, q, k, v, beta, decay, None)


def test_conv_step_refusals(lib):
    ctx = context(lib)
    assert step(lib, None) == INVALID
    assert step(lib, context(lib, bind=False)) == UNBOUND
    assert step(lib, context(lib, kind=1, dv=128)) == SHAPE
    assert step(lib, ctx, W=1) == SHAPE and step(lib, ctx, W=5) == SHAPE
    for bad in (dict(G=0), dict(G=3), dict(weight=None), dict(bias=Q), dict(state=None), dict(x=Q), dict(xs=1016), dict(xs=1028),
                dict(dt=None), dict(dt=P + 1), dict(ds=7), dict(a=None), dict(a=Q), dict(dt_bias=Q), dict(q=None), dict(k=Q), dict(v=None), dict(beta=Q),
                dict(decay=None)):
        assert step(lib, ctx, **bad) == INVALID, bad


def scan(lib, ctx, pr=None, G=2, q=P, qs=256, k=P, ks=256, v=P, vs=512, dt=P, ds=8, a=P, dt_bias=P, skip=P, out=P, os=512, od=1,
         work=P, wb=1 << 40):
    return lib.sketchssm_prompt_scan(ctx, ctypes.byref(pr or prompts()), G, q, qs, k, ks, v, vs, dt, ds, a, dt_bias, skip, out, os, od,
                                     work, wb, None)


def test_scan_refusals(lib):
    ctx = context(lib)
    assert scan(lib, ctx) == OK and scan(lib, ctx, dt_bias=None, skip=None) == OK
    assert scan(lib, ctx, pr=prompts(tokens=0), q=None, k=None, v=None, dt=None, out=None) == OK
    assert scan(lib, None) == INVALID
    assert scan(lib, context(lib, bind=False)) == UNBOUND
    assert scan(lib, context(lib, kind=2, dv=128)) == SHAPE              # the delta rules have no prompt scan here
    for bad in (dict(G=0), dict(G=3), dict(q=None), dict(k=Q), dict(v=None), dict(dt=None), dict(dt=P + 1), dict(out=Q), dict(a=None),
                dict(a=Q), dict(dt_bias=Q), dict(skip=Q), dict(qs=248), dict(ks=260), dict(vs=504), dict(os=500), dict(ds=7), dict(od=2),
                dict(pr=prompts(sequences=-1)), dict(pr=prompts(sequences=2, starts=None)), dict(pr=prompts(sequences=9, slots=None))):
        assert scan(lib, ctx, **bad) == INVALID, bad


def test_scan_scratch(lib):
    ctx, n = context(lib), ctypes.c_size_t(7)
    assert lib.sketchssm_prompt_work_bytes(None, 1, 1, ctypes.byref(n)) == INVALID
    assert lib.sketchssm_prompt_work_bytes(ctx, 1, 1, None) == INVALID
    assert lib.sketchssm_prompt_work_bytes(ctx, -1, 1, ctypes.byref(n)) == INVALID
    assert lib.sketchssm_prompt_work_bytes(ctx, 0, 0, ctypes.byref(n)) == OK and n.value == 0
    assert lib.sketchssm_prompt_work_bytes(ctx, 1, 1000, ctypes.byref(n)) == OK and n.value == 0          # too short to split
    # 8 heads of 64 columns: four pairs, so up to 37 segments fill 148 SMs; 4096 tokens make 8 of 512
    assert lib.sketchssm_prompt_work_bytes(ctx, 3, 4096, ctypes.byref(n)) == OK and n.value == 8 * 8 * (128 * 64 + 1) * 4
    assert lib.sketchssm_prompt_work_bytes(ctx, 1, 1 << 20, ctypes.byref(n)) == OK and n.value == 37 * 8 * (128 * 64 + 1) * 4
    for other in (context(lib, io_dtype=0), context(lib, heads=200), context(lib, dv=80), context(lib, dk=64)):
        assert lib.sketchssm_prompt_work_bytes(other, 1, 1 << 20, ctypes.byref(n)) == OK and n.value == 0
    assert scan(lib, ctx, pr=prompts(tokens=4096), wb=0, work=None) == OK                                # no sequences: no scratch
    assert scan(lib, ctx, pr=prompts(sequences=1, tokens=4096), wb=8 * 8 * (128 * 64 + 1) * 4 - 1) == INVALID
    assert scan(lib, ctx, pr=prompts(sequences=1, tokens=4096), work=Q) == INVALID
    assert scan(lib, ctx, pr=prompts(sequences=1, tokens=4096), work=None) == INVALID


def norm(lib, ctx, rows=0, width=256, group=0, eps=1e-5, x=P, xs=256, xd=1, weight=P, res=None, res_out=None, gate=None, gs=256,
         skip=None, ss=256, sw=None, heads=0, out=P, out8=P, scale=P):
    return lib.sketchssm_rms_norm(ctx, rows, width, group, eps, x, xs, xd, weight, res, res_out, gate, gs, skip, ss, sw, heads, out,
                                  out8, scale, None)


def test_norm_refusals(lib):
    ctx = context(lib)
    assert norm(lib, ctx) == OK and norm(lib, ctx, out=None) == OK and norm(lib, ctx, out8=None, scale=None) == OK
    assert norm(lib, ctx, group=128) == OK and norm(lib, ctx, group=256) == OK
    assert norm(lib, ctx, gate=P, skip=P, sw=P, heads=4) == OK and norm(lib, ctx, res=P, res_out=P) == OK
    assert norm(lib, None) == INVALID
    assert norm(lib, context(lib, bind=False)) == UNBOUND
    for bad in (dict(width=252), dict(width=16392, xs=16392), dict(group=64)):
        assert norm(lib, ctx, **bad) == SHAPE, bad
    for bad in (dict(rows=-1), dict(width=0), dict(group=-1), dict(group=512), dict(group=192), dict(eps=-1.0), dict(eps=float("nan")),
                dict(xd=2), dict(x=Q), dict(xs=248), dict(xs=260), dict(weight=None), dict(weight=Q), dict(res=P), dict(res_out=P),
                dict(res=Q, res_out=P), dict(out=None, out8=None, scale=None), dict(scale=None), dict(out8=None), dict(out=Q),
                dict(out8=Q), dict(gate=P, res=P, res_out=P), dict(skip=P, sw=P, heads=4), dict(gate=P, skip=P), dict(gate=P, sw=P),
                dict(gate=P, skip=P, sw=P, heads=0), dict(gate=P, skip=P, sw=P, heads=3), dict(gate=P, gs=8), dict(gate=Q),
                dict(gate=P, skip=P, sw=P, heads=4, ss=12), dict(rows=1, x=None)):
        assert norm(lib, ctx, **bad) == INVALID, bad


def matmul(lib, ctx, M=0, N=256, K=128, a=P, sa=P, w=P, sw=P, out=P, os=256, od=1):
    return lib.sketchssm_scaled_matmul(ctx, M, N, K, a, sa, w, sw, out, os, od, None)


def test_matmul_refusals(lib):
    ctx = context(lib)
    assert matmul(lib, ctx) == OK and matmul(lib, ctx, N=255) == OK
    assert matmul(lib, None) == INVALID
    assert matmul(lib, context(lib, bind=False)) == UNBOUND
    assert matmul(lib, ctx, K=120) == SHAPE
    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(w=None), dict(w=Q), dict(sw=None), dict(sw=Q), dict(os=255), dict(od=2)):
        assert matmul(lib, ctx, **bad) == INVALID, bad
    for bad in (dict(a=None), dict(a=Q), dict(sa=None), dict(sa=Q), dict(out=None), dict(out=Q)):
        assert matmul(lib, ctx, M=1, **bad) == INVALID, bad


def test_matmul_refuses_rows_that_a_tile_could_number_past_32_bits(lib):
    ctx = context(lib)
    for bad in (dict(M=2 ** 30 + 1), dict(M=2 ** 31 - 1), dict(N=2 ** 30 + 1, os=2 ** 30 + 1), dict(K=2 ** 30 + 16)):
        assert matmul(lib, ctx, **bad) == SHAPE, bad
    assert matmul(lib, ctx, N=2 ** 30, os=2 ** 30) == OK and matmul(lib, ctx, K=2 ** 30) == OK


def test_prompts_of_the_binding():
    i = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    p = binding.Prompts(i(0, 3, 3, 9), 9, slots=i(2, 0, 1), resume=i(-1, 5, -1))
    assert p.sequences == 3 and p.tokens == 9 and p.c.starts == p.starts.data_ptr() and p.on(torch.device("cpu"))
    assert binding.Prompts(i(0), 0).sequences == 0
    for args, kw in (((i(), 9), {}), ((i(0, 3), -1), {}), ((torch.tensor([0, 3]), 3), {}), ((i(0, 3), 3), dict(slots=i(0, 1))),
                     ((i(0, 3), 3), dict(resume=i())), ((i(0, 1, 2, 3)[::3], 3), {})):
        with pytest.raises(ValueError):
            binding.Prompts(*args, **kw)


def test_the_binding_refuses_tensors_that_do_not_fit():
    """The extension module's checks come before the library's, and before any CUDA call: a CPU tensor is refused by name."""
    build.build()
    m = binding.SketchSSM("mamba2", 2, 4, 128, 64, 8, 4, device=0, allocate=False)

    class Stream:
        cuda_stream = 0

    x = torch.zeros(3, 256, dtype=torch.bfloat16)
    w = torch.ones(256)
    pr = binding.Prompts(torch.tensor([0, 3], dtype=torch.int32), 3)
    with pytest.raises(ValueError, match=r"x is a BFloat16 tensor \(3, 256, \) on cuda:0"):
        m.rms_norm(x, w, out=x, stream=Stream)
    with pytest.raises(ValueError, match="x is f32 or bf16"):
        m.rms_norm(x.half(), w, out=x, stream=Stream)
    with pytest.raises(ValueError, match="x has 2 axes"):
        m.rms_norm(x[0], w, out=x, stream=Stream)
    with pytest.raises(ValueError, match="x is a tensor"):
        m.rms_norm(None, w, out=x, stream=Stream)
    with pytest.raises(ValueError, match="prompts lie on the layer's device"):
        m.causal_conv(pr, x, torch.ones(256, 4), None, x, x, stream=Stream)
    with pytest.raises(ValueError, match="prompts lie on the layer's device"):
        m.prompt_scan(pr, x, x, x, x, w, x, stream=Stream)
    with pytest.raises(ValueError, match="weight has 2 axes"):
        m.conv_step(x, x, w, None, x, w, None, {n: x for n in ("q", "k", "v", "beta", "decay")}, stream=Stream)
    a = torch.zeros(3, 256, dtype=torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="out is a Float tensor"):
        m.scaled_matmul(a, w, a, w, torch.zeros(3, 3), stream=Stream)
    with pytest.raises(ValueError, match="out is f32 or bf16"):
        m.scaled_matmul(a, w, a, w, a, stream=Stream)
    m.close()
    assert m._norm[1] == 0                     # a closed layer's context is not handed on


def test_the_binding_refuses_sizes_beyond_the_librarys_numbers():
    """The library takes sizes as ints: longer axes are refused before they are cut (views of one element: nothing is allocated)."""
    build.build()
    m = binding.SketchSSM("mamba2", 2, 4, 128, 64, 8, 4, device=0, allocate=False)

    class Stream:
        cuda_stream = 0

    long = 2 ** 32 + 4
    w = torch.ones(16)
    for t in (torch.bfloat16, torch.float32):
        x = torch.zeros(1, dtype=t)
        for size in ((long, 16), (3, long)):
            with pytest.raises(ValueError, match="longer than"):
                m.rms_norm(x.expand(*size), w, out=x, stream=Stream)
    a = torch.zeros(1, dtype=torch.uint8).view(torch.float8_e4m3fn)
    for a_size, w_size in (((long, 16), (8, 16)), ((3, long), (8, long)), ((3, 16), (long, 16))):
        with pytest.raises(ValueError, match="longer than"):
            m.scaled_matmul(a.expand(*a_size), w, a.expand(*w_size), w, torch.zeros(3, 8), stream=Stream)
    x = torch.zeros(3, 16, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="groups is out of range"):
        m.conv_step(x, x, torch.ones(16, 4), None, x, w, None, {n: x for n in ("q", "k", "v", "beta", "decay")}, groups=2 ** 32 + 1, stream=Stream)
    m.close()
    with pytest.raises(ValueError, match="tokens"):
        binding.Prompts(torch.tensor([0, 3], dtype=torch.int32), long)
