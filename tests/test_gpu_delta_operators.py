"""The operators of a delta-rule layer (GDN, KDA) and of 8-bit integer projections against their plain 64-bit forms, at the sizes and layouts
where they can go wrong.

Tolerances.  u = 2^-24 is half a step of fp32.
- scan: delta_ref.scan derives the bound of fp32 arithmetic; then one rounding to the type.
- token: convolution and SiLU as in the Mamba-2 layer's test (1e-5 of the absolute sum A); a key is that over its length, which is off by no
  more than its largest element's share; gates a few ulp; one rounding.
- norm: fp32 sums of at most 64 terms a thread, exponentials and divisions of a few ulp: 1e-5 of the result; one rounding, or half a scale.
- product: the sums are exact; one conversion and two products: 3 u, and one rounding."""
import pytest
import torch

from paper_2609_33051_b200 import binding
from tests import delta_ref as dref
from tests import layer_ref as ref
from tests.test_gpu_layer_operators import batch_of, rand, strided

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DEV = "cuda:0"
TYPE = binding.TORCH_DTYPE


def layer(B=4, H=8, K=128, V=128, io="bf16", kind="gdn"):
    return binding.SketchSSM(kind, B, H, K, V, 8, 4, io=io, device=0)


# ---- scan ------------------------------------------------------------------------------------------------------------

SCAN = [
    # kind, lengths, heads, groups, K, V, io, out, slots, resume, rows before and behind
    ("gdn", [1], 1, 1, 128, 128, "bf16", "bf16", None, None, 0, 0),
    ("kda", [1], 2, 1, 128, 128, "bf16", "f32", [1], [1], 0, 0),
    ("gdn", [0], 2, 1, 128, 128, "bf16", "bf16", [1], [0], 0, 0),
    ("kda", [0, 3, 0], 3, 3, 64, 64, "f32", "f32", [2, 1, 0], [2, -1, -1], 1, 2),
    ("gdn", [63], 4, 2, 128, 128, "bf16", "bf16", None, None, 0, 0),
    ("gdn", [64], 4, 2, 128, 128, "bf16", "bf16", None, [3], 0, 0),
    ("gdn", [65], 4, 4, 128, 128, "bf16", "bf16", [3], [3], 0, 0),
    ("kda", [65], 4, 2, 128, 128, "bf16", "bf16", None, [3], 0, 0),
    ("gdn", [129], 3, 1, 128, 80, "bf16", "f32", None, None, 0, 0),
    ("kda", [33], 3, 1, 128, 80, "f32", "bf16", None, None, 0, 0),
    ("gdn", [257, 1, 0, 64], 5, 1, 128, 128, "bf16", "bf16", [3, 0, 2, -1], [7, -1, 6, 5], 3, 5),
    ("kda", [130, 126, 2], 6, 2, 64, 64, "bf16", "f32", [99, 1, 2], None, 0, 130),
    ("gdn", [33, 70], 2, 1, 128, 80, "f32", "f32", [0, 1], [0, 1], 0, 0),
    ("gdn", [700], 2, 1, 128, 128, "bf16", "f32", None, None, 0, 0),
    ("gdn", [515, 389], 6, 3, 128, 128, "bf16", "bf16", None, [0, -1], 0, 0),
    ("kda", [300, 5], 2, 2, 128, 128, "bf16", "bf16", None, [6, 7], 0, 7),
    ("gdn", [1100], 1, 1, 64, 64, "bf16", "bf16", None, None, 0, 0),
    ("gdn", [300], 3, 3, 128, 64, "bf16", "bf16", None, [6], 0, 7),
    ("kda", [200], 2, 1, 128, 64, "f32", "f32", None, None, 0, 0),
    ("gdn", [40] * 60, 16, 4, 128, 128, "f32", "f32", [-1] * 55 + [0, 1, 2, 3, 4], [i % 3 + 5 if i % 4 else -1 for i in range(60)], 0, 0),
    ("kda", [20, 41] * 40, 8, 8, 64, 64, "f32", "f32", [-1] * 75 + [0, 1, 2, 3, 4], None, 0, 0),
    # sequences split into segments: one from a stored state into the same entry, ragged ones with an empty and a short one, many segments
    ("gdn", [3300], 2, 1, 128, 128, "bf16", "bf16", [4], [4], 0, 3),
    ("gdn", [5000, 0, 90, 7500], 3, 3, 128, 128, "bf16", "bf16", [0, 1, 2, 3], [-1, 6, 2, 3], 2, 0),
    ("gdn", [9100], 1, 1, 128, 128, "bf16", "bf16", None, None, 0, 0),
    ("gdn", [70, 128, 63] * 20, 8, 4, 128, 128, "bf16", "bf16", [-1] * 55 + [0, 1, 2, 3, 4], [i % 3 + 5 if i % 4 else -1 for i in range(60)], 0, 0),
]


def scan_inputs(kind, lengths, H, G, K, V, io, B, first=0, tail=0, seed=0):
    gen, dt = torch.Generator().manual_seed(seed + sum(lengths) + H), TYPE[io]
    T, ch = first + sum(lengths) + tail, ((H, K) if kind == "kda" else (H,))
    # decays of a token from nearly one to nearly nothing
    return dict(q=rand(gen, T, G, K, dtype=dt), k=rand(gen, T, G, K, dtype=dt), v=rand(gen, T, H, V, dtype=dt), b=rand(gen, T, H, dtype=dt),
                dt=rand(gen, T, *ch, dtype=dt), a=-torch.exp(2.7 * torch.rand(H, generator=gen)) * torch.linspace(0.01, 1, H),
                bias=rand(gen, *ch) - 3, state=rand(gen, B, H, K, V))


NAMES = ("q", "k", "v", "b", "dt", "a")


def run_scan(m, pr, x, out, bias=True, **kw):
    d = {n: x[n].to(DEV) for n in x}
    m.delta_scan(pr, d["q"], d["k"], d["v"], d["b"], d["dt"], d["a"], out, dt_bias=d["bias"] if bias else None, **kw)
    m.check_status()


def check_scan(m, x, starts, pr, slots, resume, out_dtype, bias=True, **kw):
    st = x["state"]
    m.state.copy_(st)
    dt_bias = x["bias"] if bias else None
    want, tol, new, new_tol = dref.scan(starts, slots, resume, *(x[n] for n in NAMES), dt_bias, st, m.B, **kw)
    T, H, V = x["v"].shape
    out = strided(torch.full((T, H, V), float("nan"), dtype=TYPE[out_dtype]), 8)
    dt = strided(x["dt"], 8, 16) if m.kind == "kda" else strided(x["dt"], 1, 2)
    m.delta_scan(pr, strided(x["q"], 8), strided(x["k"], 16, 8), strided(x["v"], 24), strided(x["b"], 3, 1), dt, x["a"].to(DEV), out,
                 dt_bias=None if dt_bias is None else dt_bias.to(DEV), **{n: kw[n] for n in ("eps", "q_scale") if n in kw})
    m.check_status()
    ref.close(out, want, ref.half_step(TYPE[out_dtype]) * want.abs() + tol, "out")
    ref.close(m.state, new, new_tol, "state")
    kept = [s for s in (slots if slots is not None else range(len(starts) - 1)) if 0 <= s < m.B]
    rest = [s for s in range(m.B) if s not in kept]
    assert torch.equal(m.state[rest].cpu(), st[rest])
    return out


@pytest.mark.parametrize("kind,lengths,H,G,K,V,io,od,slots,resume,first,tail", SCAN)
def test_scan(kind, lengths, H, G, K, V, io, od, slots, resume, first, tail):
    starts, pr = batch_of(lengths, slots, resume, first, tail)
    check_scan(layer(8, H, K, V, io, kind), scan_inputs(kind, lengths, H, G, K, V, io, 8, first, tail), starts, pr, slots, resume, od)


@pytest.mark.parametrize("kind,od", [("gdn", "bf16"), ("gdn", "f32"), ("kda", "bf16"), ("kda", "f32")])
def test_scan_without_bias_and_with_other_scales(kind, od):
    starts, pr = batch_of([140, 9])
    x = scan_inputs(kind, [140, 9], 4, 2, 128, 128, "bf16", 8)
    x["k"] = x["k"] * 64
    check_scan(layer(8, 4, kind=kind), x, starts, pr, None, None, od, bias=False, eps=0.5, q_scale=-3.0)


@pytest.mark.parametrize("kind", ["gdn", "kda"])
@pytest.mark.parametrize("dt,a,b", [(-200.0, -1.0, 0.0), (60.0, -16.0, 0.0), (0.0, 0.0, 30.0), (8.0, -1e-4, -100.0), (30.0, -1e30, 100.0)])
def test_scan_with_extreme_gates(kind, dt, a, b):
    """Decays of zero and of one, step sizes of zero and of one, and sums of log decays far beyond fp32's range of exponentials."""
    x = scan_inputs(kind, [300], 2, 1, 128, 128, "bf16", 8)
    x["dt"], x["b"] = (x["dt"].float() + dt).to(torch.bfloat16), (x["b"].float() + b).to(torch.bfloat16)
    x["a"] = torch.full((2,), a)
    starts, pr = batch_of([300], None, [1])
    for od in ("bf16", "f32"):
        check_scan(layer(8, 2, kind=kind), x, starts, pr, None, [1], od)


@pytest.mark.parametrize("kind,lengths", [("gdn", [300]), ("gdn", [64, 1, 130]), ("kda", [150])])
def test_scan_of_keys_that_repeat(kind, lengths):
    """The same key again and again, with step sizes near one and no decay: what the chunks' triangular systems are worst at."""
    x = scan_inputs(kind, lengths, 2, 1, 128, 128, "bf16", 8, seed=3)
    x["k"] = x["k"][:1].expand_as(x["k"]).contiguous()
    x["k"][::3] *= -2
    x["b"] = torch.full_like(x["b"], 6.0)
    x["a"] = torch.full((2,), -1e-3)
    starts, pr = batch_of(lengths, None, [i + 3 for i in range(len(lengths))])
    for od in ("bf16", "f32"):
        check_scan(layer(8, 2, kind=kind), x, starts, pr, None, [i + 3 for i in range(len(lengths))], od)


@pytest.mark.parametrize("kind", ["gdn", "kda"])
def test_scan_keeps_fp32s_accuracy(kind):
    """Over many chunks the state's error, as a length, stays a few times that of fp32 sums in chunks (1.3e-7 here): products in parts of bf16
    that lost a part of a term would show as 4e-6."""
    lengths = [1500, 900]
    x = scan_inputs(kind, lengths, 4, 2, 128, 128, "bf16", 4, seed=1)
    x["a"] = torch.linspace(-4, -0.5, 4)
    x["bias"] = x["bias"] - 1
    starts, pr = batch_of(lengths, None, [2, 3])
    for od, most in (("bf16", 2.0e-3), ("f32", 1e-6)):
        m = layer(4, 4, kind=kind)
        m.state.copy_(x["state"])
        want, _, new, _ = dref.scan(starts, None, [2, 3], *(x[n] for n in NAMES), x["bias"], x["state"], 4)
        out = torch.empty(2400, 4, 128, dtype=TYPE[od], device=DEV)
        run_scan(m, pr, x, out)
        assert (m.state[:2].cpu().double() - new[:2]).norm() <= 1e-6 * new[:2].norm()
        assert (out.cpu().double() - want).norm() <= most * want.norm()


@pytest.mark.parametrize("kind,od", [("gdn", "bf16"), ("gdn", "f32"), ("kda", "bf16")])
@pytest.mark.parametrize("lengths", [[140, 150, 40], [1, 5, 1]])
def test_scan_hands_on_a_nan_of_the_gates(kind, od, lengths):
    """Rates, step sizes and decays that are NaN: the head is NaN from that token on, in outputs and state, and nothing else is."""
    x = scan_inputs(kind, lengths, 4, 2, 128, 128, "bf16", 4, seed=5)
    starts, pr = batch_of(lengths)
    T, at = sum(lengths), lengths[0] + lengths[1] // 2
    x["a"][2] = float("nan")
    x["dt"][at, 0] = float("nan")                 # sequence 1, head 0
    x["b"][at, 1] = float("nan")                  # sequence 1, head 1
    m = layer(4, 4, kind=kind)
    out = torch.zeros(T, 4, 128, dtype=TYPE[od], device=DEV)
    run_scan(m, pr, x, out)
    bad = torch.zeros(T, 4, dtype=torch.bool)
    bad[:, 2] = bad[at:lengths[0] + lengths[1], :2] = True
    assert torch.equal(torch.isnan(out).all(2).cpu(), bad) and torch.equal(torch.isnan(out).any(2).cpu(), bad)
    state = torch.zeros(4, 4, dtype=torch.bool)
    state[:len(lengths), 2] = state[1, :2] = True
    assert torch.equal(torch.isnan(m.state).all(3).all(2).cpu(), state) and torch.equal(torch.isnan(m.state).any(3).any(2).cpu(), state)


@pytest.mark.parametrize("kind,lengths,H,G", [("gdn", [300, 7, 0, 141, 1], 3, 1), ("gdn", [140, 2, 128], 4, 2), ("kda", [140, 2], 2, 1)])
def test_scan_does_not_look_ahead(kind, lengths, H, G):
    """What is not finite changes no output of a token before it, of another column (values), head (keys, queries) or sequence; a column of the
    state that a value was not finite in, and all of a head's from such a key on, is not finite, and so are its outputs."""
    x = scan_inputs(kind, lengths, H, G, 128, 128, "bf16", 8, seed=9)
    T, nan, inf = sum(lengths), float("nan"), float("inf")
    for t, h, c, value in ((0, H - 1, 3, nan), (1, 0, 0, nan), (70, 0, 63, inf), (70, 0, 10, -inf), (127, 1, 5, inf), (100, 1, 5, nan), (131, 1, 127, nan),
                           (T - 1, 0, 7, nan)):
        x["v"][t, h, c] = value
    x["k"][135, 0, 3], x["q"][20, 0, 0] = nan, nan
    x["state"][6, 0, 5, 9] = inf
    resume = [6] + [-1] * (len(lengths) - 1)
    starts, pr = batch_of(lengths, None, resume)
    want, tol, new, new_tol = dref.scan(starts, None, resume, *(x[n] for n in NAMES), x["bias"], x["state"], 8)
    for od in ("bf16", "f32"):
        m = layer(8, H, kind=kind)
        m.state.copy_(x["state"])
        out = torch.zeros(T, H, 128, dtype=TYPE[od], device=DEV)
        run_scan(m, pr, x, out)
        for got, exp, bound in ((out, want, ref.half_step(TYPE[od]) * want.abs() + tol), (m.state[:len(lengths)], new[:len(lengths)], new_tol[:len(lengths)])):
            there = torch.isfinite(exp)
            assert torch.equal(torch.isfinite(got.cpu()), there)
            ref.close(ref.f64(got)[there], exp[there], bound[there], "finite ones")


@pytest.mark.parametrize("kind,od", [("gdn", "bf16"), ("gdn", "f32"), ("kda", "bf16")])
def test_what_rows_outside_the_sequences_hold_changes_nothing(kind, od):
    """NaN before, behind and in the rows of a batch that belong to no sequence; none of them is written."""
    lens, first, tail = [130, 0, 60], 5, 40
    x = scan_inputs(kind, lens, 4, 1, 128, 128, "bf16", 8, first, tail)
    starts, pr = batch_of(lens, None, [3, 4, 5], first, tail)
    clean = check_scan(layer(8, 4, kind=kind), x, starts, pr, None, [3, 4, 5], od)
    for n in ("q", "k", "v", "b", "dt"):
        x[n][:first] = x[n][starts[-1]:] = float("nan")
    got = check_scan(layer(8, 4, kind=kind), x, starts, pr, None, [3, 4, 5], od)
    assert torch.equal(got[first:-tail], clean[first:-tail])


@pytest.mark.parametrize("kind,od", [("gdn", "bf16"), ("kda", "f32")])
def test_scan_in_pieces_is_the_whole(kind, od):
    """A prompt in three calls that go on from the stored state, on another stream, equals the prompt in one."""
    x = scan_inputs(kind, [450], 4, 1, 128, 128, "bf16", 8, seed=9)
    m, s = layer(8, 4, kind=kind), torch.cuda.Stream()
    want, tol, new, new_tol = dref.scan([0, 450], None, None, *(x[n] for n in NAMES), x["bias"], x["state"], 8)
    d = {n: x[n].to(DEV) for n in x}
    out = torch.zeros(450, 4, 128, dtype=TYPE[od], device=DEV)
    s.wait_stream(torch.cuda.current_stream())
    for i, (lo, hi) in enumerate(((0, 130), (130, 131), (131, 450))):
        _, pr = batch_of([hi - lo], [0], [0 if i else -1])
        torch.cuda.synchronize()
        m.delta_scan(pr, *(d[n][lo:hi] for n in ("q", "k", "v", "b", "dt")), d["a"], out[lo:hi], dt_bias=d["bias"], stream=s)
    s.synchronize()
    ref.close(out, want, ref.half_step(TYPE[od]) * want.abs() + tol, "out")
    ref.close(m.state[:1], new[:1], new_tol[:1], "state")


@pytest.mark.parametrize("kind,od", [("gdn", "bf16"), ("kda", "f32")])
def test_scan_replayed_from_a_graph_with_other_lengths(kind, od):
    """The lengths and entries are read when the kernels run: a replay takes the ones that the arrays hold then."""
    x = scan_inputs(kind, [200, 100], 4, 2, 128, 128, "bf16", 8, seed=4)
    m = layer(8, 4, kind=kind)
    starts, pr = batch_of([200, 100], [0, 1], [-1, -1])
    d = {n: x[n].to(DEV) for n in x}
    out = torch.zeros(300, 4, 128, dtype=TYPE[od], device=DEV)
    work = m.new_delta_work(2, 300)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.delta_scan(pr, *(d[n] for n in NAMES), out, dt_bias=d["bias"], work=work)
    for lens, slots, resume in (([200, 100], [0, 1], [-1, -1]), ([3, 297], [5, 2], [7, -1]), ([0, 10], [3, 3 + 1], [6, 6])):
        starts = ref.starts_of(lens)
        for t, v in ((pr.starts, starts), (pr.slots, slots), (pr.resume, resume)):
            t.copy_(torch.tensor(v, dtype=torch.int32))
        m.state.copy_(x["state"])
        out.fill_(float("nan"))
        want, tol, new, new_tol = dref.scan(starts, slots, resume, *(x[n] for n in NAMES), x["bias"], x["state"], 8)
        g.replay()
        torch.cuda.synchronize()
        ref.close(out, want, ref.half_step(TYPE[od]) * want.abs() + tol, "out")
        ref.close(m.state, new, new_tol, "state")
    m.check_status()


@pytest.mark.parametrize("kind,od", [("gdn", "bf16"), ("gdn", "f32"), ("kda", "bf16")])
def test_scan_stays_inside_its_arrays_whatever_starts_holds(kind, od):
    """Row numbers that do not ascend or leave the batch are cut to it: some outputs are senseless, none is outside."""
    m = layer(4, 2, kind=kind)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    d = {n: t.to(DEV) for n, t in scan_inputs(kind, [64], 2, 1, 128, 128, "bf16", 4).items()}
    wide = torch.full((96, 2, 128), 7.0, dtype=TYPE[od], device=DEV)
    work = torch.zeros(m.new_delta_work(2, 64).numel() + 4096 if m.new_delta_work(2, 64) is not None else 4096, dtype=torch.uint8, device=DEV)
    used = work.numel() - 4096
    work[used:] = 77
    for starts in (i32(40, 10, 64), i32(-5, 1000, 20), i32(64, 64, 64), i32(-9, -9, -3), i32(0, 64, 3)):
        pr = binding.Prompts(starts, 64, i32(-7, 1 << 30), i32(1 << 30, -1))
        m.delta_scan(pr, *(d[n] for n in NAMES), wide[16:80], work=work)
    m.check_status()
    assert (wide[:16] == 7).all() and (wide[80:] == 7).all() and (work[used:] == 77).all()


def test_scan_twice_is_the_same_to_the_bit():
    x = scan_inputs("gdn", [700, 30, 333], 8, 4, 128, 128, "bf16", 4, seed=2)
    starts, pr = batch_of([700, 30, 333])
    m, outs = layer(4, 8), []
    for _ in range(2):
        m.state.copy_(x["state"])
        out = torch.empty(1063, 8, 128, dtype=torch.bfloat16, device=DEV)
        run_scan(m, pr, x, out)
        outs.append((out.view(torch.int16), m.state.clone().view(torch.int32)))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


# ---- a token ---------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("kind,B,H,G,K,V,W,io", [("gdn", 1, 32, 16, 128, 128, 4, "bf16"), ("kda", 3, 8, 8, 64, 64, 3, "f32"), ("gdn", 5, 24, 2, 128, 80, 2, "bf16"),
                                                 ("kda", 37, 6, 3, 128, 128, 4, "f32"), ("kda", 130, 32, 32, 128, 128, 4, "bf16"), ("gdn", 9, 3, 1, 64, 128, 4, "f32"),
                                                 ("kda", 2, 5, 1, 64, 64, 4, "bf16")])
def test_step(kind, B, H, G, K, V, W, io):
    gen, dt_ = torch.Generator().manual_seed(B + H), TYPE[io]
    C, ch = H * V + 2 * G * K, ((H, K) if kind == "kda" else (H,))
    x, b, dt = rand(gen, B, C, dtype=dt_), rand(gen, B, H, dtype=dt_, scale=3), rand(gen, B, *ch, dtype=dt_, scale=3)
    w, cb, a, bias = rand(gen, C, W, scale=0.5), rand(gen, C), -torch.exp(rand(gen, H)), rand(gen, *ch)
    st = rand(gen, B, W - 1, C, dtype=dt_)
    x[0, H * V:H * V + K] = 0                                          # (one key of the bias alone)
    m, state = layer(B, H, K, V, io, kind), st.to(DEV)
    t = m.new_token_buffers()
    dtd = strided(dt.flatten(1), 8, 16) if kind == "kda" else strided(dt, 3, 5)
    m.delta_step(strided(x, 16, 8), strided(b, 3, 2), dtd, w.to(DEV), cb.to(DEV), state, a.to(DEV), bias.to(DEV), t, groups=G, eps=1e-3, q_scale=0.7)
    full = torch.cat([st, x[:, None]], 1).double()
    terms = full * w.double().T
    y, mag = terms.sum(1) + cb.double(), terms.abs().sum(1) + cb.double().abs()
    y = ref.silu(y)
    spread = lambda z: z.repeat_interleave(H // G, 1)  # noqa: E731
    ref.close(t["v"], y[:, :H * V].unflatten(1, (H, V)), (ref.half_step(dt_) * y.abs() + 1e-5 * mag)[:, :H * V].unflatten(1, (H, V)), "v")
    for name, cut, scale in (("k", slice(H * V, H * V + G * K), 1.0), ("q", slice(H * V + G * K, C), 0.7)):
        z, e = y[:, cut].unflatten(1, (G, K)), 1e-5 * mag[:, cut].unflatten(1, (G, K))
        length = torch.sqrt((z * z).sum(-1, keepdim=True) + 1e-3)
        want = scale * z / length
        # off by its own error, and by that of the length (at most the length of the errors), and a few roundings of sums of 128
        tol = scale * e / length + want.abs() * (e.norm(dim=-1, keepdim=True) / length + 20 * U) + ref.half_step(dt_) * want.abs()
        ref.close(t[name], spread(want), spread(tol), name)
    ref.close(t["beta"], 1 / (1 + torch.exp(-b.double())), 8 * U, "beta")
    D = dref.decays(dt, a, bias)
    arg = ref.softplus(dt.double().reshape(B, H, -1) + bias.double().reshape(H, -1))
    # the argument of the exponential is off by 10 u of itself, the result by that and 2 ulp; then (KDA) one rounding
    tol = (16 * U * (arg + 1) * a.double().abs()[:, None] + 4 * U) * D + 1e-38
    if kind == "kda":
        ref.close(t["decay"], D, tol + ref.half_step(dt_) * D, "decay")
    else:
        ref.close(t["decay"], D[..., 0], tol[..., 0], "decay")
    assert torch.equal(state.cpu().double(), full[:, 1:])


def test_step_replayed_moves_the_rows_on():
    gen, bf = torch.Generator().manual_seed(8), torch.bfloat16
    C = 4 * 128 + 2 * 2 * 128
    x, b, dt = rand(gen, 3, C, dtype=bf).to(DEV), rand(gen, 3, 4, dtype=bf).to(DEV), rand(gen, 3, 4, dtype=bf).to(DEV)
    w, a, st = rand(gen, C, 4).to(DEV), -torch.ones(4, device=DEV), rand(gen, 3, 3, C, dtype=bf).to(DEV)
    m = layer(3, 4)
    t, g, s = m.new_token_buffers(), torch.cuda.CUDAGraph(), torch.cuda.Stream()
    old = st.clone()
    with torch.cuda.graph(g, stream=s):
        m.delta_step(x, b, dt, w, None, st, a, None, t, groups=2)
    for i in range(2):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(st, torch.cat([old[:, 2:], x[:, None], x[:, None]], 1))


# ---- norm ------------------------------------------------------------------------------------------------------------

NORM = [
    # rows, width, group, io, x, mode, act
    (1, 8, 8, "bf16", "bf16", "plain", "silu"),
    (3, 136, 136, "f32", "f32", "residual", "silu"),
    (5, 256, 128, "bf16", "f32", "gated", "silu"),
    (6, 240, 80, "bf16", "f32", "gated", "sigmoid"),
    (1, 2048, 2048, "bf16", "bf16", "residual", "silu"),
    (7, 4096, 128, "bf16", "f32", "gated", "sigmoid"),
    (2, 4104, 4104, "f32", "bf16", "gated", "silu"),
    (4, 16384, 16384, "f32", "f32", "plain", "silu"),
    (257, 5128, 5128, "bf16", "bf16", "residual", "silu"),
    (1300, 1920, 80, "bf16", "bf16", "gated", "silu"),
    (1025, 248, 8, "bf16", "f32", "gated", "silu"),
    (130, 512, 256, "f32", "f32", "plain", "silu"),
    (700, 16384, 64, "bf16", "bf16", "gated", "silu"),
    (3000, 1024, 512, "bf16", "bf16", "residual", "silu"),
]


@pytest.mark.parametrize("rows,D,group,io,xt,mode,act", NORM)
def test_norm(rows, D, group, io, xt, mode, act):
    gen, dt = torch.Generator().manual_seed(rows + D), TYPE[io]
    x, w = rand(gen, rows, D, dtype=TYPE[xt], scale=3), 1 + 0.3 * rand(gen, group)
    if rows > 2:
        x[1] = 0                                             # a row of zeros
        x[2, :group] *= 1e-3
    kw = {}
    if mode == "residual":
        kw = dict(residual=rand(gen, rows, D, dtype=dt))
        if rows > 2:
            kw["residual"][1] = 0
    if mode == "gated":
        kw = dict(gate=rand(gen, rows, D, dtype=dt, scale=2))
    m = layer(1, io=io)
    h, want = dref.norm8(x, w, 1e-5, act=act, **kw)
    dev = {n: t.to(DEV) if n == "residual" else strided(t, 8, 16) for n, t in kw.items()}
    out, out8, scale = torch.empty(rows, D, dtype=dt, device=DEV), torch.empty(rows, D, dtype=torch.int8, device=DEV), torch.empty(rows, device=DEV)
    if mode == "residual":
        dev["residual_out"] = dev["residual"]                # in place
    xd = strided(x, 8)
    m.integer_norm(xd, w.to(DEV), out8, scale, out=out, act=act, **dev)
    assert m.last_launch_count() == 1
    # a cancellation in h = x + residual leaves an absolute error of its terms' size
    slack = 1e-5 * want.abs()
    if mode == "residual":
        ref.close(dev["residual_out"], h, (ref.half_step(dt) + U) * h.abs(), "residual")
        slack = slack + 4 * U * (x.double().abs() + kw["residual"].double().abs()) * (want / h).abs().nan_to_num(0.0)
    ref.close(out, want, ref.half_step(dt) * want.abs() + slack + 1e-37, "out")
    top = want.abs().amax(1)
    ref.close(scale, top / 127, (4 * U * top + slack.amax(1)) / 127, "scale")
    s = scale.cpu().double()[:, None]
    ref.close(out8.cpu().double() * s, want, 0.5 * s + 1.1 * slack + 200 * U * want.abs(), "out8")
    assert rows < 3 or (out8[1] == 0).all()
    if mode != "residual":
        alone = torch.empty_like(out8)
        m.integer_norm(xd, w.to(DEV), alone, scale, act=act, **dev)
        assert torch.equal(alone, out8)


@pytest.mark.parametrize("group", [64, 512])
def test_norm_keeps_what_is_not_finite_to_its_row(group):
    gen = torch.Generator().manual_seed(3)
    x, w = rand(gen, 600, 512), torch.ones(group)
    m, outs = layer(1, io="f32"), []
    for bad in (False, True):
        if bad:
            x[5, 7], x[100, 500], x[7, 300] = float("nan"), float("inf"), -float("inf")
        out8, scale = torch.empty(600, 512, dtype=torch.int8, device=DEV), torch.empty(600, device=DEV)
        m.integer_norm(x.to(DEV), w.to(DEV), out8, scale)
        outs.append((out8, scale))
    rest = [i for i in range(600) if i not in (5, 7, 100)]
    for a, b in zip(*outs):
        assert torch.equal(a[rest], b[rest])
    assert torch.isnan(outs[1][1][[5, 7, 100]]).all() and torch.isfinite(outs[1][1][rest]).all()


# ---- product ---------------------------------------------------------------------------------------------------------


def integers(gen, n, k):
    return torch.randint(-128, 128, (n, k), generator=gen, dtype=torch.int32).to(torch.int8), torch.rand(n, generator=gen) + 0.01


@pytest.mark.parametrize("M,N,K,od,pad", [(1, 1, 16, "f32", 0), (1, 128, 128, "bf16", 0), (3, 127, 144, "f32", 5), (17, 129, 256, "bf16", 7),
                                          (64, 513, 2048, "bf16", 8), (65, 200, 112, "bf16", 0), (129, 257, 400, "f32", 3),
                                          (128, 256, 384, "bf16", 0), (300, 520, 1040, "f32", 0), (1000, 1000, 512, "bf16", 24),
                                          (513, 2056, 272, "bf16", 0), (2049, 384, 640, "bf16", 0), (700, 4160, 1152, "f32", 0),
                                          (16, 12352, 2048, "bf16", 0), (130, 12352, 528, "bf16", 0), (2100, 2200, 272, "f32", 0),
                                          (2100, 2201, 144, "bf16", 2), (1801, 2500, 912, "bf16", 4), (5000, 1030, 128, "f32", 1),
                                          (4099, 4100, 16, "bf16", 4), (5, 300, 65536, "f32", 0), (33, 40000, 64, "bf16", 0), (2300, 5000, 2064, "f32", 0)])
def test_matmul(M, N, K, od, pad):
    gen = torch.Generator().manual_seed(M + N + K)
    (a, sa), (w, sw) = integers(gen, M, K), integers(gen, N, K)
    m = layer(1)
    wide = torch.full((M, N + pad), 7.0, dtype=TYPE[od], device=DEV)
    out = wide[:, :N]
    m.integer_matmul(a.to(DEV), sa.to(DEV), w.to(DEV), sw.to(DEV), out)
    m.check_status()
    want = (a.double() @ w.double().T) * sa.double()[:, None] * sw.double()
    ref.close(out, want, (ref.half_step(TYPE[od]) + 3 * U) * want.abs(), "out")
    assert (wide[:, N:] == 7).all()


@pytest.mark.parametrize("value", [-128, 127])
def test_matmul_of_the_largest_sums(value):
    """2^14 x 131056, just below what 32 bits hold."""
    K = 2 ** 17 - 16
    a, w, one = torch.full((3, K), -128, dtype=torch.int8, device=DEV), torch.full((130, K), value, dtype=torch.int8, device=DEV), torch.ones(130, device=DEV)
    m, out = layer(1), torch.empty(3, 130, device=DEV)
    m.integer_matmul(a, one[:3], w, one, out)
    m.check_status()
    assert (out == torch.tensor(-128.0 * value * K)).all()                # (a multiple of 2^11 or 2^18, below 2^31 in size)


def test_matmul_keeps_a_scale_that_is_not_finite_to_its_row_and_column():
    gen = torch.Generator().manual_seed(1)
    for M, N in ((200, 300), (20, 300), (2100, 2200)):
        (a, sa), (w, sw) = integers(gen, M, 256), integers(gen, N, 256)
        sa[7], sw[150] = float("nan"), float("nan")
        m, out = layer(1), torch.empty(M, N, device=DEV)
        m.integer_matmul(a.to(DEV), sa.to(DEV), w.to(DEV), sw.to(DEV), out)
        want = (a.double() @ w.double().T) * sa.double()[:, None] * sw.double()
        ref.close(out, want, 3 * U * want.abs())


def test_matmul_replayed_and_without_rows():
    gen = torch.Generator().manual_seed(2)
    (a, sa), (w, sw) = integers(gen, 40, 512), integers(gen, 640, 512)
    m, out = layer(1), torch.empty(40, 640, device=DEV)
    ad, sad, wd, swd = a.to(DEV), sa.to(DEV), w.to(DEV), sw.to(DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.integer_matmul(ad, sad, wd, swd, out)
    b, sb = integers(gen, 40, 512)
    ad.copy_(b), sad.copy_(sb)
    g.replay()
    torch.cuda.synchronize()
    want = (b.double() @ w.double().T) * sb.double()[:, None] * sw.double()
    ref.close(out, want, 3 * U * want.abs())
    first = out.clone()
    m.integer_matmul(ad[:0], sad[:0], wd, swd, out[:0])
    assert torch.equal(out, first) and m.last_launch_count() == 0
    m.integer_norm(torch.empty(0, 64, device=DEV), torch.ones(64, device=DEV), torch.empty(0, 64, dtype=torch.int8, device=DEV), torch.empty(0, device=DEV))
    assert m.last_launch_count() == 0
