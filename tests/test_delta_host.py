"""Refusals of the delta-rule layer's operators and of the 8-bit integer ones, without a GPU: every one of these calls ends before any CUDA call
is made (the addresses are only checked, never dereferenced)."""
import ctypes

import pytest
import torch

from paper_2609_33051_b200 import binding, build
from tests.test_layer_host import INVALID, OK, SHAPE, UNBOUND, P, Q, context, prompts

GDN, KDA, NAN = 1, 2, float("nan")


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def scan(lib, ctx, pr=None, G=2, eps=1e-6, qs_=0.1, q=P, qs=256, k=P, ks=256, v=P, vs=1024, b=P, bs=8, dt=P, ds=1024, a=P, dt_bias=P, out=P, os=1024, od=1,
         work=P, wb=1 << 40):
    return lib.sketchssm_delta_scan(ctx, ctypes.byref(pr or prompts()), G, eps, qs_, q, qs, k, ks, v, vs, b, bs, dt, ds, a, dt_bias, out, os, od, work, wb, None)


@pytest.mark.parametrize("kind", [GDN, KDA])
def test_scan_refusals(lib, kind):
    ctx = context(lib, kind=kind, dv=128)
    assert scan(lib, ctx) == OK and scan(lib, ctx, dt_bias=None) == OK and scan(lib, ctx, b=P + 2, bs=9) == OK
    assert scan(lib, ctx, pr=prompts(tokens=0), q=None, k=None, v=None, b=None, dt=None, out=None) == OK
    assert scan(lib, None) == INVALID
    assert scan(lib, context(lib, kind=kind, dv=128, bind=False)) == UNBOUND
    assert scan(lib, context(lib, kind=0, dv=128)) == SHAPE               # Mamba-2 has a scan of its own
    for bad in (dict(G=0), dict(G=3), dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN), dict(qs_=NAN), dict(q=None), dict(k=Q), dict(v=None), dict(b=None),
                dict(b=P + 1), dict(bs=7), dict(dt=None), dict(dt=P + 1), dict(ds=7), dict(out=Q), dict(a=None), dict(a=Q), dict(dt_bias=Q), dict(qs=248), dict(ks=260),
                dict(vs=1016), dict(os=1028), dict(od=2), dict(pr=prompts(sequences=-1)), dict(pr=prompts(sequences=2, starts=None)),
                dict(pr=prompts(sequences=9, slots=None))):
        assert scan(lib, ctx, **bad) == INVALID, bad
    assert scan(lib, ctx, pr=prompts(tokens=(1 << 30) + 1)) == SHAPE
    # the decays' arguments: a number a head at any stride, or rows of K for every head that are read 16 bytes at a time
    assert scan(lib, ctx, ds=8) == (OK if kind == GDN else INVALID)
    assert scan(lib, ctx, dt=P + 2) == (OK if kind == GDN else INVALID)
    assert scan(lib, ctx, ds=1028) == (OK if kind == GDN else INVALID)


def test_scan_scratch_refusals(lib):
    ctx, n = context(lib, kind=GDN, dv=128), ctypes.c_size_t(7)
    assert lib.sketchssm_delta_work_bytes(None, 1, 1, ctypes.byref(n)) == INVALID
    assert lib.sketchssm_delta_work_bytes(ctx, 1, 1, None) == INVALID
    assert lib.sketchssm_delta_work_bytes(ctx, -1, 1, ctypes.byref(n)) == INVALID
    assert lib.sketchssm_delta_work_bytes(ctx, 1, -1, ctypes.byref(n)) == INVALID
    assert lib.sketchssm_delta_work_bytes(ctx, 0, 0, ctypes.byref(n)) == OK and n.value == 0
    for tokens in (1, 64, 1000):
        assert lib.sketchssm_delta_work_bytes(ctx, 3, tokens, ctypes.byref(n)) == OK and n.value % 16 == 0
        if n.value:
            for bad in (dict(wb=n.value - 1), dict(work=None), dict(work=Q)):
                assert scan(lib, ctx, pr=prompts(sequences=3, tokens=tokens), **bad) == INVALID


@pytest.mark.parametrize("kind", [GDN, KDA])
def test_scan_into_fp32_needs_scratch_for_kda_alone(lib, kind):
    """GDN goes over CUDA cores then, whatever the number of tokens, and the tensor cores' scratch is not asked for: such a call gets as far as its device
    (one that no machine has)."""
    ctx, n = context(lib, kind=kind, dv=128, device=1000), ctypes.c_size_t(0)
    assert lib.sketchssm_delta_work_bytes(ctx, 3, 1000, ctypes.byref(n)) == OK and n.value > 0
    for none in (dict(work=None, wb=0), dict(work=Q), dict(wb=n.value - 1)):
        got = scan(lib, ctx, pr=prompts(sequences=3, tokens=1000), od=0, **none)
        assert (got == INVALID) == (kind == KDA), none
    assert scan(lib, ctx, pr=prompts(sequences=0, tokens=1000), od=0, work=None, wb=0) == OK


@pytest.mark.parametrize("kind", [GDN, KDA])
def test_no_sequences_need_no_scratch(lib, kind):
    ctx, n = context(lib, kind=kind, dv=128), ctypes.c_size_t(7)
    assert lib.sketchssm_delta_work_bytes(ctx, 0, 100, ctypes.byref(n)) == OK and n.value == 0
    assert scan(lib, ctx, pr=prompts(sequences=0, tokens=100), work=None, wb=0) == OK


def step(lib, ctx, G=2, W=4, eps=1e-6, qs=0.1, weight=P, bias=P, state=P, x=P, xs=1536, b=P, bs=8, dt=P, ds=1024, a=P, dt_bias=P, q=P, k=P, v=P, beta=P,
         decay=P):
    return lib.sketchssm_delta_step(ctx, G, W, eps, qs, weight, bias, state, x, xs, b, bs, dt, ds, a, dt_bias, q, k, v, beta, decay, None)


@pytest.mark.parametrize("kind", [GDN, KDA])
def test_step_refusals(lib, kind):
    ctx = context(lib, kind=kind, dv=128)
    assert step(lib, None) == INVALID
    assert step(lib, context(lib, kind=kind, dv=128, bind=False)) == UNBOUND
    assert step(lib, context(lib, kind=0, dv=128)) == SHAPE
    assert step(lib, ctx, W=1) == SHAPE and step(lib, ctx, W=5) == SHAPE
    for bad in (dict(G=0), dict(G=3), dict(eps=0.0), dict(eps=NAN), dict(qs=NAN), dict(weight=None), dict(bias=Q), dict(state=None), dict(x=Q), dict(xs=1528),
                dict(xs=1540), dict(b=None), dict(b=P + 1), dict(bs=7), dict(dt=None), dict(dt=P + 1), dict(ds=7), dict(a=None), dict(a=Q), dict(dt_bias=Q), dict(q=None),
                dict(k=Q), dict(v=None), dict(beta=Q), dict(decay=None)):
        assert step(lib, ctx, **bad) == INVALID, bad
    if kind == KDA:
        for bad in (dict(dt=P + 2), dict(ds=1016), dict(ds=1028)):
            assert step(lib, ctx, **bad) == INVALID, bad


def norm(lib, ctx, rows=0, width=256, group=256, eps=1e-5, x=P, xs=256, xd=1, weight=P, res=None, res_out=None, gate=None, gs=256, flags=0, out=P, out8=P, scale=P):
    return lib.sketchssm_integer_norm(ctx, rows, width, group, eps, x, xs, xd, weight, res, res_out, gate, gs, flags, out, out8, scale, None)


def test_norm_refusals(lib):
    ctx = context(lib)
    assert norm(lib, ctx) == OK and norm(lib, ctx, out=None) == OK and norm(lib, ctx, group=64) == OK and norm(lib, ctx, flags=1, gate=P) == OK
    assert norm(lib, ctx, res=P, res_out=P) == OK and norm(lib, ctx, width=240, group=80) == OK
    assert norm(lib, None) == INVALID
    assert norm(lib, context(lib, bind=False)) == UNBOUND
    for bad in (dict(width=252, group=252), dict(width=16392, xs=16392, group=16392), dict(group=4)):
        assert norm(lib, ctx, **bad) == SHAPE, bad
    for bad in (dict(rows=-1), dict(width=0), dict(group=0), dict(group=512), dict(group=96), dict(eps=-1.0), dict(eps=NAN), dict(xd=2), dict(x=Q), dict(xs=248),
                dict(xs=260), dict(weight=None), dict(weight=Q), dict(res=P), dict(res_out=P), dict(res=Q, res_out=P), dict(out=Q), dict(out8=Q), dict(scale=Q),
                dict(gate=P, res=P, res_out=P), dict(gate=P, gs=8), dict(gate=Q), dict(flags=2), dict(rows=1, x=None), dict(rows=1, out8=None), dict(rows=1, scale=None)):
        assert norm(lib, ctx, **bad) == INVALID, bad


def matmul(lib, ctx, M=0, N=256, K=128, a=P, sa=P, w=P, sw=P, out=P, os=256, od=1):
    return lib.sketchssm_integer_matmul(ctx, M, N, K, a, sa, w, sw, out, os, od, None)


def test_matmul_refusals(lib):
    ctx = context(lib)
    assert matmul(lib, ctx) == OK and matmul(lib, ctx, N=255) == OK and matmul(lib, ctx, K=2 ** 17 - 16) == OK
    assert matmul(lib, None) == INVALID
    assert matmul(lib, context(lib, bind=False)) == UNBOUND
    for bad in (dict(K=120), dict(K=2 ** 17), dict(M=2 ** 30 + 1), dict(N=2 ** 30 + 1, os=2 ** 30 + 1)):
        assert matmul(lib, ctx, **bad) == SHAPE, bad
    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(w=None), dict(w=Q), dict(sw=None), dict(sw=Q), dict(os=255), dict(od=2)):
        assert matmul(lib, ctx, **bad) == INVALID, bad
    for bad in (dict(a=None), dict(a=Q), dict(sa=None), dict(sa=Q), dict(out=None), dict(out=Q)):
        assert matmul(lib, ctx, M=1, **bad) == INVALID, bad


def test_the_binding_refuses_tensors_that_do_not_fit():
    """The extension module's checks come before the library's, and before any CUDA call: a CPU tensor is refused by name."""
    build.build()
    m = binding.SketchSSM("kda", 2, 4, 128, 128, 8, 4, device=0, allocate=False)

    class Stream:
        cuda_stream = 0

    bf, f = torch.bfloat16, torch.float32
    x, w, c = torch.zeros(3, 256, dtype=bf), torch.ones(256), torch.zeros(3, 256, dtype=torch.int8)
    pr = binding.Prompts(torch.tensor([0, 3], dtype=torch.int32), 3)
    with pytest.raises(ValueError, match="prompts lie on the layer's device"):
        m.delta_scan(pr, x, x, x, x, x, w, x, stream=Stream)
    with pytest.raises(ValueError, match="weight has 2 axes"):
        m.delta_step(x, x, x, w, None, x, w, None, {n: x for n in ("q", "k", "v", "beta", "decay")}, stream=Stream)
    with pytest.raises(ValueError, match="groups is out of range"):
        m.delta_step(x, x, x, x, None, x, w, None, {n: x for n in ("q", "k", "v", "beta", "decay")}, groups=2 ** 32 + 1, stream=Stream)
    with pytest.raises(ValueError, match=r"x is a BFloat16 tensor \(3, 256, \) on cuda:0"):
        m.integer_norm(x, w, c, w, stream=Stream)
    with pytest.raises(ValueError, match="act is silu or sigmoid"):
        m.integer_norm(x, w, c, w, act="relu", stream=Stream)
    with pytest.raises(ValueError, match="weight has 1 axes"):
        m.integer_norm(x, x, c, w, stream=Stream)
    with pytest.raises(ValueError, match="out is a Float tensor"):
        m.integer_matmul(c, w, c, w, torch.zeros(3, 3, dtype=f), stream=Stream)
    with pytest.raises(ValueError, match="out is f32 or bf16"):
        m.integer_matmul(c, w, c, w, c, stream=Stream)
    long = 2 ** 32 + 4
    with pytest.raises(ValueError, match="longer than"):
        m.integer_matmul(c[:1, :1].expand(long, 16), w, c[:1, :1].expand(8, 16), w, x, stream=Stream)
    m.close()
    assert m._delta_scan[1] == 0 and m._norm8[1] == 0          # a closed layer's context is not handed on
