"""The operators around the recurrence against their plain 64-bit forms, at the sizes and layouts where they can go wrong.

Tolerances.  u = 2^-24 is half a step of fp32.  A result is a sum of terms; A is the sum of their absolute values.
- convolution: at most 5 fused multiply-adds (5 u A), SiLU by the fast exponential and division (arguments below 32: 32 x 2^-22 in
  the exponential, 2^-22 in the division, |silu'| <= 1.1): 1e-5 A covers both; then one rounding to the type.
- scan: a term goes through as many decays as tokens follow it (expf 2 ulp, a multiplication, an addition: 6 u each), and through
  sums over K: (6 n + K + 16) u A, n the sequence's length; then one rounding.  Where the products go through bfloat16 parts the
  kernel's own comment says how many: TERMS below.
- norm: fp32 sums of at most 64 terms a thread, exponentials and divisions of a few ulp: 1e-5 of the result; one rounding.
  8 bits: half a step 2^-4 of the value, or 2^-10 scales among the subnormals.
- product: the values are exact in fp32, K additions of 2 u each: K 2^-23 A; one rounding."""
import pytest
import torch

from paper_2609_33051_b200 import binding
from tests import layer_ref as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DEV = "cuda:0"
TYPE = binding.TORCH_DTYPE


def layer(B=4, H=8, K=128, V=64, io="bf16", kind="mamba2"):
    return binding.SketchSSM(kind, B, H, K, V, 8, 4, io=io, device=0)


def rand(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(dtype)


def strided(t, pad, front=0):
    """The same rows on the device, as a column range of a wider matrix."""
    flat = t.flatten(1)
    wide = torch.full((t.shape[0], front + flat.shape[1] + pad), float("nan"), dtype=t.dtype, device=DEV)
    view = wide[:, front:front + flat.shape[1]]
    view.copy_(flat)
    return view.unflatten(1, t.shape[1:]) if t.dim() > 2 else view


def batch_of(lengths, slots=None, resume=None, first=0, tail=0):
    starts = ref.starts_of(lengths, first)
    i32 = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    return starts, binding.Prompts(i32(starts), starts[-1] + tail, i32(slots), i32(resume))


# ---- convolution -----------------------------------------------------------------------------------------------------

CONV = [
    # lengths, channels, width, io, silu, slots, resume, rows before and behind
    ([1], 8, 4, "bf16", True, None, None, 0, 0),
    ([2], 16, 3, "bf16", False, [3], [3], 0, 0),
    ([3], 8, 4, "f32", True, [1], [0], 0, 0),
    ([0], 8, 2, "f32", False, [1], [1], 0, 0),
    ([0, 0, 5, 0], 24, 4, "bf16", True, [3, 2, 1, 0], [3, -1, 5, 0], 3, 4),
    ([7, 1, 1, 1, 2, 30, 3, 9], 520, 4, "bf16", True, [0, 1, 2, 3, 4, -1, 6, 99], [0, -1, 7, 8, 9, 9, 6, 99], 2, 5),
    ([31, 2, 31, 33, 1], 136, 3, "f32", True, None, [5, 5, 5, 5, 5], 0, 1),
    ([300, 0, 1, 211], 1032, 4, "bf16", True, [1, 0, 2, 5], [1, 9, -1, 8], 0, 0),
    ([29, 6], 64, 2, "bf16", False, None, None, 0, 0),
    ([4100], 4352, 4, "bf16", True, [2], [2], 0, 0),             # runs of 32 rows
    ([33, 31, 30, 1, 2, 3, 2900, 1100], 4352, 4, "bf16", True, None, [0, 1, 2, 3, 4, 5, 6, 7], 1, 2),
]


@pytest.mark.parametrize("lengths,C,W,io,act,slots,resume,first,tail", CONV)
def test_conv(lengths, C, W, io, act, slots, resume, first, tail):
    gen, B = torch.Generator().manual_seed(C + W), 10
    starts, pr = batch_of(lengths, slots, resume, first, tail)
    T, dt = pr.tokens, TYPE[io]
    x, w, b = rand(gen, T, C, dtype=dt), rand(gen, C, W, scale=0.5), rand(gen, C, scale=0.2)
    st = rand(gen, B, W - 1, C, dtype=dt)
    m = layer(B=B, io=io)
    want, mag, new = ref.conv(starts, slots, resume, x, w, b, st, act, B)
    out = strided(torch.full((T, C), float("nan"), dtype=dt), 8, 8)
    state = st.to(DEV)
    m.causal_conv(pr, strided(x, 16), w.to(DEV), b.to(DEV), state, out, silu=act)
    assert m.last_launch_count() == 1
    ref.close(out, want, ref.half_step(dt) * want.abs() + 1e-5 * mag, "out")
    assert torch.equal(state.cpu().double(), new)


def test_conv_without_bias_on_another_stream_and_replayed():
    gen = torch.Generator().manual_seed(5)
    starts, pr = batch_of([70, 5, 60], None, [0, 1, -1])
    x, w, st = rand(gen, 135, 64, dtype=torch.bfloat16), rand(gen, 64, 4), rand(gen, 4, 3, 64, dtype=torch.bfloat16)
    m, xd, wd, state = layer(), x.to(DEV), w.to(DEV), st.to(DEV)
    out = torch.empty_like(xd)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        m.causal_conv(pr, xd, wd, None, state, out)
    for _ in range(2):                                       # the state goes on from replay to replay
        want, mag, new = ref.conv(starts, None, [0, 1, -1], x, w, None, state.cpu(), True, 4)
        g.replay()
        torch.cuda.synchronize()
        ref.close(out, want, 2.0 ** -8 * want.abs() + 1e-5 * mag)
        assert torch.equal(state.cpu().double(), new)


@pytest.mark.parametrize("B,H,G,K,V,W,io", [(1, 64, 1, 128, 64, 4, "bf16"), (3, 8, 8, 64, 64, 3, "f32"), (5, 24, 2, 128, 80, 2, "bf16"),
                                            (37, 6, 3, 128, 128, 4, "f32"), (256, 64, 1, 128, 64, 4, "bf16")])
def test_conv_step(B, H, G, K, V, W, io):
    gen, dt_ = torch.Generator().manual_seed(B + H), TYPE[io]
    C = H * V + 2 * G * K
    x, dt = rand(gen, B, C, dtype=dt_), rand(gen, B, H, dtype=dt_, scale=3)
    w, b, a, bias = rand(gen, C, W, scale=0.5), rand(gen, C), -torch.exp(rand(gen, H)), rand(gen, H)
    st = rand(gen, B, W - 1, C, dtype=dt_)
    m, state = layer(B, H, K, V, io), st.to(DEV)
    t = m.new_token_buffers()
    m.conv_step(strided(x, 16, 8), strided(dt, 3, 5), w.to(DEV), b.to(DEV), state, a.to(DEV), bias.to(DEV), t, groups=G)
    full = torch.cat([st, x[:, None]], 1).double()
    terms = full * w.double().T
    y, mag = terms.sum(1) + b.double(), terms.abs().sum(1) + b.double().abs()
    y = ref.silu(y)
    spread = lambda z: z.unflatten(1, (G, K)).repeat_interleave(H // G, 1)  # noqa: E731
    for name, cut, shape in (("v", slice(0, H * V), None), ("k", slice(H * V, H * V + G * K), G), ("q", slice(H * V + G * K, C), G)):
        want, tol = y[:, cut], ref.half_step(dt_) * y[:, cut].abs() + 1e-5 * mag[:, cut]
        want, tol = (spread(want), spread(tol)) if shape else (want.unflatten(1, (H, V)), tol.unflatten(1, (H, V)))
        ref.close(t[name], want, tol, name)
    beta = ref.softplus(dt.double() + bias.double())
    ref.close(t["beta"], beta, 8 * U * (beta + 1), "beta")
    # the argument of the exponential is off by 10 u of itself, the result by that and 2 ulp
    ref.close(t["decay"], torch.exp(beta * a.double()), (16 * U * (beta + 1) * a.double().abs() + 4 * U) * torch.exp(beta * a.double()) + 1e-38, "decay")
    assert torch.equal(state.cpu().double(), full[:, 1:])


# ---- scan ------------------------------------------------------------------------------------------------------------

SCAN = [
    # lengths, heads, groups, K, V, io, out, slots, resume, rows before and behind
    ([1], 1, 1, 128, 64, "bf16", "bf16", None, None, 0, 0),
    ([1], 2, 1, 128, 64, "bf16", "f32", [1], [1], 0, 0),
    ([0], 2, 1, 128, 64, "bf16", "bf16", [1], [0], 0, 0),
    ([0, 3, 0], 3, 3, 64, 64, "f32", "f32", [2, 1, 0], [2, -1, -1], 1, 2),
    ([127], 4, 2, 128, 64, "bf16", "bf16", None, None, 0, 0),
    ([128], 4, 2, 128, 128, "bf16", "bf16", None, [3], 0, 0),
    ([129], 3, 1, 128, 80, "bf16", "f32", None, None, 0, 0),
    ([257, 1, 0, 64], 5, 1, 128, 64, "bf16", "bf16", [3, 0, 2, -1], [7, -1, 6, 5], 3, 5),
    ([130, 126, 2], 6, 2, 64, 64, "bf16", "f32", [99, 1, 2], None, 0, 130),
    ([33, 70], 2, 1, 128, 80, "f32", "f32", [0, 1], [0, 1], 0, 0),
    ([700], 2, 1, 128, 64, "bf16", "f32", None, None, 0, 0),
    ([515, 389], 7, 7, 128, 64, "bf16", "bf16", None, [0, -1], 0, 0),
    ([300, 5], 2, 2, 128, 128, "bf16", "f32", None, [6, 7], 0, 7),
    ([300], 3, 3, 128, 80, "bf16", "bf16", None, [6], 0, 7),
    ([1100], 1, 1, 64, 64, "bf16", "bf16", None, None, 0, 0),
    # sequences split into segments: one from a stored state into the same entry, ragged ones with an empty one among them, two groups
    # of three heads, halves of 128 columns
    ([2100], 2, 1, 128, 64, "bf16", "bf16", [4], [4], 0, 3),
    ([1500, 0, 90, 1025], 3, 1, 128, 64, "bf16", "bf16", [0, 1, 2, 3], [-1, 6, 2, 3], 2, 0),
    ([1111, 1000], 6, 2, 128, 64, "bf16", "bf16", [3, 2], [2, -1], 0, 0),
    ([1200], 2, 2, 128, 128, "bf16", "bf16", None, [0], 0, 0),
    ([200] * 40, 8, 1, 128, 64, "bf16", "bf16", [-1] * 35 + [0, 1, 2, 3, 4], [i % 3 + 5 if i % 4 else -1 for i in range(40)], 0, 0),
]
# How many half steps 2^-8 of bfloat16 the products may be off by, measured by A, for the type of the output.  With bf16 outputs a term
# goes into its product either by way of the scores or by way of the state, and either is rounded once: one half step; the log2 of a
# score's weight is off by 2^-10 at most where sums of decays are long, its exponential by ln 2 of that: 0.18 half steps, and 0.02
# for the fast logarithm and exponential.  With fp32 outputs nothing is rounded below fp32.
TERMS = {"bf16": 1.2, "f32": 0.0}


def scan_inputs(lengths, H, G, K, V, io, B, first=0, tail=0, seed=0):
    gen, dt = torch.Generator().manual_seed(seed + sum(lengths) + H), TYPE[io]
    T = first + sum(lengths) + tail
    return dict(q=rand(gen, T, G, K, dtype=dt), k=rand(gen, T, G, K, dtype=dt), v=rand(gen, T, H, V, dtype=dt),
                dt=rand(gen, T, H, dtype=dt), a=-torch.exp(2.7 * torch.rand(H, generator=gen)) * torch.linspace(0.01, 1, H),
                bias=rand(gen, H) - 1, skip=rand(gen, H), state=rand(gen, B, H, K, V))


def check_scan(m, x, starts, pr, slots, resume, out_dtype, bias=True, skip=True, state=None):
    st = x["state"] if state is None else state
    m.state.copy_(st)
    dt_bias, sk = x["bias"] if bias else None, x["skip"] if skip else None
    want, mag, new, new_mag = ref.scan(starts, slots, resume, x["q"], x["k"], x["v"], x["dt"], x["a"], dt_bias, sk, st, m.B)
    T, H, V = x["v"].shape
    out = strided(torch.full((T, H, V), float("nan"), dtype=TYPE[out_dtype]), 8)
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    m.prompt_scan(pr, strided(x["q"], 8), strided(x["k"], 16, 8), strided(x["v"], 24), strided(x["dt"], 1, 2), dev(x["a"]), out,
                  dt_bias=dev(dt_bias), skip=dev(sk))
    m.check_status()
    n = max([b - a for a, b in zip(starts, starts[1:])] + [0])
    rel = (6 * n + m.K + 16) * U
    ref.close(out, want, ref.half_step(TYPE[out_dtype]) * want.abs() + (rel + TERMS[out_dtype] * 2.0 ** -8) * mag, "out")
    ref.close(m.state, new, rel * new_mag, "state")
    kept = [s for s in (slots if slots is not None else range(len(starts) - 1)) if 0 <= s < m.B]
    rest = [s for s in range(m.B) if s not in kept]
    assert torch.equal(m.state[rest].cpu(), st[rest])
    return out


@pytest.mark.parametrize("lengths,H,G,K,V,io,od,slots,resume,first,tail", SCAN)
def test_scan(lengths, H, G, K, V, io, od, slots, resume, first, tail):
    starts, pr = batch_of(lengths, slots, resume, first, tail)
    m = layer(8, H, K, V, io)
    check_scan(m, scan_inputs(lengths, H, G, K, V, io, 8, first, tail), starts, pr, slots, resume, od)


@pytest.mark.parametrize("bias,skip", [(False, True), (True, False), (False, False)])
def test_scan_without_bias_and_skip(bias, skip):
    starts, pr = batch_of([140, 9])
    m = layer(8, 4, 128, 64)
    check_scan(m, scan_inputs([140, 9], 4, 1, 128, 64, "bf16", 8), starts, pr, None, None, "bf16", bias, skip)


@pytest.mark.parametrize("dt,a", [(-200.0, -1.0), (60.0, -16.0), (0.0, 0.0), (8.0, -1e-4), (30.0, -1e30)])
def test_scan_with_extreme_gates(dt, a):
    """Step sizes of zero, decays of zero and of one, and sums of their logarithms far beyond fp32's range of exponentials."""
    x = scan_inputs([300], 2, 1, 128, 64, "bf16", 8)
    x["dt"] = (x["dt"].float() + dt).to(torch.bfloat16)
    x["a"] = torch.full((2,), a)
    starts, pr = batch_of([300], None, [1])
    check_scan(layer(8, 2, 128, 64), x, starts, pr, None, [1], "f32")


@pytest.mark.parametrize("lengths", [[140, 150, 40], [1, 5, 1], [60, 2300]])
def test_scan_hands_on_a_nan_of_the_gates(lengths):
    """Rates and step sizes that are NaN: the head is NaN from that token on, in outputs and state, and nothing else is."""
    x = scan_inputs(lengths, 4, 2, 128, 64, "bf16", 4, seed=5)
    starts, pr = batch_of(lengths)
    T, at = sum(lengths), lengths[0] + lengths[1] // 2
    x["a"][2] = float("nan")
    x["dt"][at, 0] = float("nan")                 # sequence 1, head 0
    m = layer(4, 4, 128, 64)
    out = torch.zeros(T, 4, 64, dtype=torch.bfloat16, device=DEV)
    m.prompt_scan(pr, *(x[n].to(DEV) for n in ("q", "k", "v", "dt", "a")), out, dt_bias=x["bias"].to(DEV), skip=x["skip"].to(DEV))
    m.check_status()
    bad = torch.zeros(T, 4, dtype=torch.bool)
    bad[:, 2] = bad[at:lengths[0] + lengths[1], 0] = True
    assert torch.equal(torch.isnan(out).all(2).cpu(), bad) and torch.equal(torch.isnan(out).any(2).cpu(), bad)
    state = torch.zeros(4, 4, dtype=torch.bool)
    state[:len(lengths), 2] = state[1, 0] = True
    assert torch.equal(torch.isnan(m.state).all(3).all(2).cpu(), state) and torch.equal(torch.isnan(m.state).any(3).any(2).cpu(), state)


@pytest.mark.parametrize("lengths,H,G,V", [([300, 7, 0, 141, 1], 3, 1, 64), ([140, 2, 128], 4, 2, 128), ([1400], 2, 1, 64)])
def test_scan_in_chunks_does_not_look_ahead(lengths, H, G, V):
    """bf16 outputs, which are made 128 tokens at a time: what is not finite changes no output of a token before it, of another
    column (values) or head (keys, queries); everything else is as in the test of the same sizes."""
    x = scan_inputs(lengths, H, G, 128, V, "bf16", 8, seed=9)
    T, nan, inf = sum(lengths), float("nan"), float("inf")
    for t, h, c, value in ((0, H - 1, 3, nan), (1, 0, 0, nan), (70, 0, 63, inf), (70, 0, 10, -inf), (127, 1, 5, inf), (100, 1, 5, nan), (131, 1, V - 1, nan),
                           (T - 1, 0, 7, nan), (T - 2, 1, 31, -inf)):
        x["v"][t, h, c] = value
    x["k"][135, 0, 3], x["q"][20, 0, 0] = nan, inf
    starts, pr = batch_of(lengths)
    m = layer(8, H, 128, V)
    m.state.copy_(x["state"])
    want, mag, new, new_mag = ref.scan(starts, None, None, *(x[n] for n in ("q", "k", "v", "dt", "a", "bias", "skip", "state")), m.B)
    out = torch.zeros(T, H, V, dtype=torch.bfloat16, device=DEV)
    m.prompt_scan(pr, *(x[n].to(DEV) for n in ("q", "k", "v", "dt", "a")), out, dt_bias=x["bias"].to(DEV), skip=x["skip"].to(DEV))
    m.check_status()
    rel = (6 * max(lengths) + 144) * U
    for got, exp, tol in ((out, want, ref.half_step(torch.bfloat16) * want.abs() + (rel + TERMS["bf16"] * 2.0 ** -8) * mag), (m.state, new, rel * new_mag)):
        there = torch.isfinite(exp)
        assert torch.equal(torch.isfinite(got.cpu()), there)
        ref.close(ref.f64(got)[there], exp[there], tol[there], "finite ones")


def test_scan_keeps_what_is_not_finite_to_its_own_sequence_and_head():
    x = scan_inputs([140, 150, 40], 4, 2, 128, 64, "bf16", 8, seed=3)
    starts, pr = batch_of([140, 150, 40], None, [3, 4, 5])
    m = layer(8, 4, 128, 64)
    clean, bad = [], torch.zeros(330, 4, dtype=torch.bool)
    x["v"][145, 1, 5] = float("nan")              # sequence 1, head 1
    x["k"][300, 0, 7] = float("inf")              # sequence 2, heads 0 and 1
    x["state"][4, 3, 2, 2] = float("nan")         # sequence 1, head 3
    x["q"][10, 1, 0] = float("nan")               # one token of sequence 0, heads 2 and 3
    m.state.copy_(x["state"])
    want, mag, new, new_mag = ref.scan(starts, None, [3, 4, 5], *(x[n] for n in ("q", "k", "v", "dt", "a", "bias", "skip", "state")), m.B)
    out = torch.zeros(330, 4, 64, dtype=torch.float32, device=DEV)
    m.prompt_scan(pr, *(x[n].to(DEV) for n in ("q", "k", "v", "dt", "a")), out, dt_bias=x["bias"].to(DEV), skip=x["skip"].to(DEV))
    m.check_status()
    bad[145:290, 1] = bad[300:330, 0] = bad[300:330, 1] = bad[140:290, 3] = bad[10, 2:] = True
    good = ~bad[:, :, None].expand_as(want)
    tol = ((6 * 150 + 144) * U + TERMS["f32"] * 2.0 ** -8) * mag + U * want.abs()
    got = out.cpu().double()
    assert ((got - want).abs() - tol)[good].max() <= 0
    # what the plain form leaves finite or not is the same per token and head where no chunk is shared
    assert torch.isnan(got[145, 1, 5]) and torch.isnan(got[10, 2:]).all()
    st, keep = m.state.cpu().double(), torch.ones(8, 4, dtype=torch.bool)
    keep[1, 1] = keep[1, 3] = keep[2, :2] = keep[4, 3] = False
    assert ((st - new).abs() - (6 * 150 + 144) * U * new_mag)[keep].max() <= 0


@pytest.mark.parametrize("od", ["bf16", "f32"])
def test_what_rows_outside_the_sequences_hold_changes_nothing(od):
    """NaN before, behind and in the rows of a batch that belong to no sequence; none of them is written."""
    lens, first, tail = [130, 0, 60], 5, 40
    x = scan_inputs(lens, 4, 1, 128, 64, "bf16", 8, first, tail)
    starts, pr = batch_of(lens, None, [3, 4, 5], first, tail)
    clean = check_scan(layer(8, 4, 128, 64), x, starts, pr, None, [3, 4, 5], od)
    for n in ("q", "k", "v", "dt"):
        x[n][:first] = x[n][starts[-1]:] = float("nan")
    assert torch.equal(check_scan(layer(8, 4, 128, 64), x, starts, pr, None, [3, 4, 5], od)[first:-tail], clean[first:-tail])
    m, st = layer(8), torch.zeros(8, 3, 256, dtype=torch.bfloat16, device=DEV)
    w, out = rand(torch.Generator().manual_seed(1), 256, 4).to(DEV), torch.full((pr.tokens, 256), 7.0, dtype=torch.bfloat16, device=DEV)
    m.causal_conv(pr, x["v"].flatten(1).to(DEV), w, None, st, out)
    assert torch.isfinite(out).all() and (out[:first] == 7).all() and (out[starts[-1]:] == 7).all() and torch.isfinite(st).all()


def test_norm_keeps_what_is_not_finite_to_its_row():
    gen = torch.Generator().manual_seed(3)
    x, w = rand(gen, 600, 512), torch.ones(512)
    m = layer(1, io="f32")
    outs = []
    for bad in (False, True):
        if bad:
            x[5, 7], x[100, 0] = float("nan"), float("inf")
        out8, scale, out = torch.empty(600, 512, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(600, 4, device=DEV), torch.empty(600, 512, device=DEV)
        m.rms_norm(x.to(DEV), w.to(DEV), out=out, out8=out8, scale=scale)
        outs.append((out8.view(torch.uint8), scale, out))
    rest = [i for i in range(600) if i not in (5, 100)]
    for a, b in zip(*outs):
        assert torch.equal(a[rest], b[rest])
    assert torch.isnan(outs[1][2][5]).all()


def test_scan_in_pieces_is_the_whole():
    """A prompt in three calls that go on from the stored state, on another stream, equals the prompt in one."""
    x = scan_inputs([450], 4, 1, 128, 64, "bf16", 8, seed=9)
    m, s = layer(8, 4, 128, 64), torch.cuda.Stream()
    want, mag, new, new_mag = ref.scan([0, 450], None, None, *(x[n] for n in ("q", "k", "v", "dt", "a", "bias", "skip", "state")), 8)
    d = {n: x[n].to(DEV) for n in x}
    out = torch.zeros(450, 4, 64, dtype=torch.float32, device=DEV)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for i, (lo, hi) in enumerate(((0, 130), (130, 131), (131, 450))):
            _, pr = batch_of([hi - lo], [0], [0 if i else -1])
            m.prompt_scan(pr, *(d[n][lo:hi] for n in ("q", "k", "v", "dt")), d["a"], out[lo:hi], dt_bias=d["bias"], skip=d["skip"])
    s.synchronize()
    rel = (6 * 450 + 144) * U
    ref.close(out, want, (rel + TERMS["f32"] * 2.0 ** -8) * mag, "out")
    ref.close(m.state[:1], new[:1], rel * new_mag[:1], "state")


def test_scan_replayed_from_a_graph_with_other_lengths():
    """The lengths and entries are read when the kernels run: a replay takes the ones that the arrays hold then."""
    x = scan_inputs([200, 100], 4, 1, 128, 64, "bf16", 8, seed=4)
    m = layer(8, 4, 128, 64)
    starts, pr = batch_of([200, 100], [0, 1], [-1, -1])
    d = {n: x[n].to(DEV) for n in x}
    out = torch.zeros(300, 4, 64, dtype=torch.float32, device=DEV)
    work = m.new_prompt_work(2, 300)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.prompt_scan(pr, *(d[n] for n in ("q", "k", "v", "dt", "a")), out, dt_bias=d["bias"], skip=d["skip"], work=work)
    for lens, slots, resume in (([200, 100], [0, 1], [-1, -1]), ([3, 297], [5, 2], [7, -1]), ([0, 10], [3, 3 + 1], [6, 6])):
        starts = ref.starts_of(lens)
        for t, v in ((pr.starts, starts), (pr.slots, slots), (pr.resume, resume)):
            t.copy_(torch.tensor(v, dtype=torch.int32))
        m.state.copy_(x["state"])
        out.fill_(float("nan"))
        want, mag, new, new_mag = ref.scan(starts, slots, resume, *(x[n] for n in ("q", "k", "v", "dt", "a", "bias", "skip", "state")), 8)
        g.replay()
        torch.cuda.synchronize()
        rel = (6 * 300 + 144) * U
        ref.close(out, want, (rel + TERMS["f32"] * 2.0 ** -8) * mag, "out")
        ref.close(m.state, new, rel * new_mag, "state")
    m.check_status()


def test_scan_and_conv_stay_inside_their_arrays_whatever_starts_holds():
    """Row numbers that do not ascend or leave the batch are cut to it: some outputs are senseless, none is outside."""
    m = layer(4, 2, 128, 64)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    x = scan_inputs([64], 2, 1, 128, 64, "bf16", 4)
    d = {n: x[n].to(DEV) for n in x}
    wide = torch.full((96, 2, 64), 7.0, device=DEV)
    cw = torch.full((96, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    st = torch.zeros(4, 3, 128, dtype=torch.bfloat16, device=DEV)
    for starts in (i32(40, 10, 64), i32(-5, 1000, 20), i32(64, 64, 64), i32(-9, -9, -3)):
        pr = binding.Prompts(starts, 64, i32(-7, 1 << 30), i32(1 << 30, -1))
        m.prompt_scan(pr, *(d[n] for n in ("q", "k", "v", "dt", "a")), wide[16:80])
        m.causal_conv(pr, d["v"].flatten(1), torch.ones(128, 4, device=DEV), None, st, cw[16:80])
    m.check_status()
    assert (wide[:16] == 7).all() and (wide[80:] == 7).all() and (cw[:16] == 7).all() and (cw[80:] == 7).all()


# ---- norm ------------------------------------------------------------------------------------------------------------

NORM = [
    # rows, width, group, io, x, mode, skip heads
    (1, 8, 0, "bf16", "bf16", "plain", 0),
    (3, 136, 0, "f32", "f32", "residual", 0),
    (5, 256, 128, "bf16", "f32", "gated", 4),
    (1, 2048, 0, "bf16", "bf16", "residual", 0),
    (7, 4096, 2048, "bf16", "f32", "gated", 64),
    (2, 4104, 0, "f32", "bf16", "gated", 3),
    (4, 16384, 0, "f32", "f32", "plain", 0),
    (257, 5128, 0, "bf16", "bf16", "residual", 0),
    (1300, 1928, 0, "bf16", "bf16", "gated", 0),
    (1025, 248, 0, "bf16", "f32", "gated", 31),
    (130, 512, 128, "f32", "f32", "gated", 8),
    (700, 16384, 8192, "bf16", "bf16", "gated", 128),
]


@pytest.mark.parametrize("rows,D,group,io,xt,mode,heads", NORM)
def test_norm(rows, D, group, io, xt, mode, heads):
    gen, dt = torch.Generator().manual_seed(rows + D), TYPE[io]
    x, w = rand(gen, rows, D, dtype=TYPE[xt], scale=3), 1 + 0.3 * rand(gen, D)
    if rows > 2:
        x[1] = 0                                             # a row of zeros
        x[2, :128] *= 1e-3
    kw = {}
    if mode == "residual":
        kw = dict(residual=rand(gen, rows, D, dtype=dt))
        if rows > 2:
            kw["residual"][1] = 0
    if mode == "gated":
        kw = dict(gate=rand(gen, rows, D, dtype=dt, scale=2))
        if heads:
            kw.update(skip=rand(gen, rows, D, dtype=dt), skip_weight=rand(gen, heads))
    m = layer(1, io=io)
    h, want = ref.norm(x, w, 1e-5, group, **kw)
    dev = {n: t.to(DEV) if n in ("residual", "skip_weight") else strided(t, 8, 16) for n, t in kw.items()}
    out, out8 = torch.empty(rows, D, dtype=dt, device=DEV), torch.empty(rows, D, dtype=torch.float8_e4m3fn, device=DEV)
    scale = torch.empty(rows, -(-D // 128), device=DEV)
    xd = strided(x, 8)
    if mode == "residual":
        dev["residual_out"] = dev["residual"]                # in place
    m.rms_norm(xd, w.to(DEV), out=out, out8=out8, scale=scale, group=group, **dev)
    # a cancellation in h = x + ... leaves an absolute error of its terms' size
    terms = (x.double().abs() + (kw["skip"].double() * kw["skip_weight"].double().repeat_interleave(D // heads)).abs()) if heads else x.double().abs()
    if mode == "gated":
        terms = terms * ref.silu(kw["gate"].double()).abs()
    ratio = (want / h).abs().nan_to_num(0.0)
    slack = 1e-5 * want.abs() + 4 * U * terms * ratio
    if mode == "residual":
        ref.close(dev["residual_out"], h, (ref.half_step(dt) + U) * h.abs() + U * x.double().abs(), "residual")
        slack = slack + 4 * U * kw["residual"].double().abs() * ratio
    ref.close(out, want, ref.half_step(dt) * want.abs() + slack + 1e-37, "out")
    blocks = torch.nn.functional.pad(want, (0, scale.shape[1] * 128 - D)).unflatten(1, (-1, 128))
    top = blocks.abs().amax(-1)
    loose = torch.nn.functional.pad(slack, (0, scale.shape[1] * 128 - D)).unflatten(1, (-1, 128)).amax(-1)
    ref.close(scale, top / 448, (4 * U * top + loose) / 448, "scale")
    spread = scale.cpu().double().repeat_interleave(128, 1)[:, :D]
    ref.close(out8.float().cpu().double() * spread, want, 2.0 ** -4 * want.abs() + 2.0 ** -10 * spread + 1.1 * slack, "out8")
    # either output alone is the same
    alone8, alone = torch.empty_like(out8), torch.empty_like(out)
    if mode != "residual":
        m.rms_norm(xd, w.to(DEV), out8=alone8, scale=scale, group=group, **dev)
        m.rms_norm(xd, w.to(DEV), out=alone, group=group, **dev)
        assert torch.equal(alone8.view(torch.uint8), out8.view(torch.uint8)) and torch.equal(alone, out)


# ---- product ---------------------------------------------------------------------------------------------------------


def quantised(gen, n, k, rows):
    x = torch.randn(n, k, generator=gen)
    q = (x * 100).to(torch.float8_e4m3fn)
    return q, torch.rand(-(-n // rows), -(-k // 128), generator=gen) + 0.01


@pytest.mark.parametrize("M,N,K,od,pad", [(1, 1, 16, "f32", 0), (1, 128, 128, "bf16", 0), (3, 127, 144, "f32", 5), (17, 129, 256, "bf16", 7),
                                          (64, 513, 2048, "bf16", 8), (65, 200, 112, "bf16", 0), (129, 257, 400, "f32", 3),
                                          (128, 256, 384, "bf16", 0), (300, 520, 1040, "f32", 0), (1000, 1000, 512, "bf16", 24),
                                          (513, 2056, 272, "bf16", 0), (2049, 384, 640, "bf16", 0), (700, 4160, 1152, "f32", 0),
                                          (16, 8512, 2048, "bf16", 0), (130, 8512, 528, "bf16", 0), (2100, 2200, 272, "f32", 0),
                                          (2100, 2201, 144, "bf16", 2), (1801, 2500, 912, "bf16", 4), (5000, 1030, 128, "f32", 1),
                                          (4099, 4100, 16, "bf16", 4)])
def test_matmul(M, N, K, od, pad):
    gen = torch.Generator().manual_seed(M + N + K)
    a, sa = quantised(gen, M, K, 1)
    w, sw = quantised(gen, N, K, 128)
    m = layer(1)
    wide = torch.full((M, N + pad), 7.0, dtype=TYPE[od], device=DEV)
    out = wide[:, :N]
    m.scaled_matmul(a.to(DEV), sa.to(DEV), w.to(DEV), sw.to(DEV), out)
    m.check_status()
    want, mag = ref.matmul(a, sa, w, sw)
    ref.close(out, want, ref.half_step(TYPE[od]) * want.abs() + K * 2.0 ** -23 * mag, "out")
    assert (wide[:, N:] == 7).all()


def test_matmul_keeps_what_is_not_finite_to_its_row_and_column():
    gen = torch.Generator().manual_seed(1)
    a, sa = quantised(gen, 200, 256, 1)
    w, sw = quantised(gen, 300, 256, 128)
    a[7, 3] = w[150, 200] = float("nan")
    sa[9, 0] = float("inf")
    m, out = layer(1), torch.empty(200, 300, device=DEV)
    m.scaled_matmul(a.to(DEV), sa.to(DEV), w.to(DEV), sw.to(DEV), out)
    want, mag = ref.matmul(a, sa, w, sw)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(out.cpu()), fine) and not fine[7].any() and not fine[:, 150].any() and not fine[9].any()
    assert ((out.cpu().double() - want).abs() - 256 * 2.0 ** -23 * mag)[fine].max() <= 0


def test_matmul_rows_do_not_depend_on_the_batch_and_replay():
    """Captured and replayed with other inputs; no rows at all; twice the same answer to the bit."""
    gen = torch.Generator().manual_seed(2)
    (a, sa), (w, sw) = quantised(gen, 40, 512, 1), quantised(gen, 640, 512, 128)
    m, out = layer(1), torch.empty(40, 640, device=DEV)
    ad, sad, wd, swd = a.to(DEV), sa.to(DEV), w.to(DEV), sw.to(DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.scaled_matmul(ad, sad, wd, swd, out)
    b, sb = quantised(gen, 40, 512, 1)
    ad.copy_(b), sad.copy_(sb)
    g.replay()
    torch.cuda.synchronize()
    want, mag = ref.matmul(b, sb, w, sw)
    ref.close(out, want, 512 * 2.0 ** -23 * mag)
    first = out.clone()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int32), first.view(torch.int32))
    m.scaled_matmul(ad[:0], sad[:0], wd, swd, out[:0])
    assert torch.equal(out.view(torch.int32), first.view(torch.int32)) and m.last_launch_count() == 0
