"""The operators of a delta-rule layer in a row, as a layer runs them: a prompt, the sketch, decode steps, a flush.

The recurrence alone: a prompt in one scan against the same tokens given one by one to the token's operator and the library's exact decode.
The whole layer passes two roundings to 8-bit integers on the way, where values that differ by a bf16 rounding can fall on either side; its
bound is derived at the test."""
import pytest
import torch

from paper_2609_33051_b200 import binding, layer
from tests import delta_ref as dref
from tests import layer_ref as ref
from tests.test_gpu_layer_together import prompts, rand

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("kind,H,G,K,V,W", [("gdn", 4, 2, 128, 128, 4), ("kda", 4, 4, 128, 128, 4), ("gdn", 3, 1, 128, 80, 3), ("kda", 2, 1, 64, 64, 2)])
def test_a_prompt_and_its_tokens_one_by_one(kind, H, G, K, V, W):
    """Keys, queries and (KDA) decays of a token are stored in bf16, 2^-9 off: a token adds at most six such errors to a column of the state (two
    readings by the key, its outer product, the value, the decay, and a rounding of the value), and one to an output."""
    B, L, T, bf = 3, 4, 11, torch.bfloat16
    gen = torch.Generator().manual_seed(H + V)
    C, D = H * V + 2 * G * K, (H * K if kind == "kda" else H)
    x, b, dt = rand(gen, B, T, C, dtype=bf).to(DEV), rand(gen, B, T, H, dtype=bf).to(DEV), rand(gen, B, T, D, dtype=bf).to(DEV)
    w, cb, a = rand(gen, C, W, scale=0.5).to(DEV), rand(gen, C).to(DEV), -torch.exp(rand(gen, H)).to(DEV)
    bias = (rand(gen, *((H, K) if kind == "kda" else (H,))) - 2).to(DEV)
    m, s = (binding.SketchSSM(kind, B, H, K, V, 8, L, io="bf16", device=0) for _ in range(2))
    start, rows = rand(gen, B, H, K, V).to(DEV), rand(gen, B, W - 1, C, dtype=bf).to(DEV)
    own = torch.arange(B, dtype=torch.int32, device=DEV)
    pr = binding.Prompts(T * torch.arange(B + 1, dtype=torch.int32, device=DEV), B * T, slots=own, resume=own)
    m.state.copy_(start)
    conv_a, conv_b = rows.clone(), rows.clone()
    c = torch.empty(B * T, C, dtype=bf, device=DEV)
    m.causal_conv(pr, x.view(B * T, C), w, cb, conv_a, c)
    v, k, q = c[:, :H * V].unflatten(1, (H, V)), c[:, H * V:H * V + G * K].unflatten(1, (G, K)), c[:, H * V + G * K:].unflatten(1, (G, K))
    y = torch.empty(B * T, H, V, device=DEV)
    m.delta_scan(pr, q, k, v, b.view(B * T, H), dt.view(B * T, D), a, y, dt_bias=bias)
    s.state.copy_(start)
    t, n = s.new_token_buffers(), 0
    outs = torch.empty(B, T, H, V, device=DEV)
    for i in range(T):
        s.delta_step(x[:, i], b[:, i], dt[:, i], w, cb, conv_b, a, bias, t, groups=G)
        assert torch.equal(t["v"], v.view(B, T, H, V)[:, i])
        args = [t[z] for z in ("q", "k", "v", "beta", "decay")]
        if n == L - 1:
            s.state_update(n, *args, t["out"])
        else:
            s.full_read_decode(n, *args, t["out"])
        n = (n + 1) % L
        outs[:, i] = t["out"]
    s.state_update(n, flags=binding.NO_SKETCH)          # what is left in the ring
    m.check_status(), s.check_status()
    assert torch.equal(conv_a, conv_b)
    args = ([T * i for i in range(B + 1)], None, list(range(B)), q, k, v, b.view(B * T, H), dt.view(B * T, D) if kind == "gdn" else dt.view(B * T, H, K), a, bias, start, B)
    want, tol, new, new_tol = dref.scan(*args)
    ref.close(y, want, tol + 2.0 ** -24 * want.abs(), "scan")
    ref.close(m.state, new, new_tol, "state")
    want, tol, new, new_tol = dref.scan(*args, rel=6 * 2.0 ** -9)
    ref.close(outs.view(B * T, H, V), want, tol, "steps")
    ref.close(s.state, new, new_tol, "state by steps")


def weights(gen, kind, width, H, G, K, V, W):
    C, inner, D = H * V + 2 * G * K, H * V, (H * K if kind == "kda" else H)
    return dict(norm=1 + 0.1 * rand(gen, width), w_in=rand(gen, inner + C + H + D, width, scale=width ** -0.5), conv_weight=rand(gen, C, W, scale=0.5),
                conv_bias=0.1 * rand(gen, C), a=-torch.exp(rand(gen, H)), dt_bias=rand(gen, *((H, K) if kind == "kda" else (H,))) - 2,
                head_norm=1 + 0.1 * rand(gen, V), w_out=rand(gen, width, inner, scale=inner ** -0.5))


def plain_layer(kind, act, w, x, residual, H, G, K, V, starts):
    """The layer in 64 bits, with the roundings of what is stored: 8-bit integer activations and weights, bf16 between the calls."""
    def quant(z):
        scale = z.abs().amax(1, keepdim=True) / 127
        return torch.round(z / scale) * scale

    def weight(z):
        q8, scale = layer.quantise_integer(z)
        return q8.double() * scale.double()[:, None]

    bf = lambda z: z.to(torch.bfloat16).double()  # noqa: E731
    inner, C = H * V, H * V + 2 * G * K
    h = x.double() + residual.double()
    p = bf(quant(dref.norm8(h, w["norm"], 1e-5)[1]) @ weight(w["w_in"]).T)
    gate, xbc, b, dt = p[:, :inner], p[:, inner:inner + C], p[:, inner + C:inner + C + H], p[:, inner + C + H:]
    c = bf(ref.conv(starts, None, None, xbc, w["conv_weight"], w["conv_bias"], torch.zeros(8, w["conv_weight"].shape[1] - 1, C), True, 8)[0])
    v, k, q = c[:, :inner].unflatten(1, (H, V)), c[:, inner:inner + G * K].unflatten(1, (G, K)), c[:, inner + G * K:].unflatten(1, (G, K))
    y = bf(dref.scan(starts, None, None, q, k, v, b, dt.unflatten(1, (H, K)) if kind == "kda" else dt, w["a"], w["dt_bias"], torch.zeros(8, H, K, V), 8)[0].flatten(1))
    return bf(quant(dref.norm8(y, w["head_norm"], 1e-5, gate=gate, act=act)[1]) @ weight(w["w_out"]).T), bf(h)


@pytest.mark.parametrize("kind,act,G,V", [("gdn", "silu", 2, 128), ("kda", "sigmoid", 4, 128), ("gdn", "silu", 4, 80)])
def test_a_layer_over_prompts_and_then_token_by_token(kind, act, G, V):
    """Prompts of 70 and 25 tokens, then 6 tokens each (a window of 4: decode steps and a flush), against the layer over the whole
    sequences in 64 bits.

    Bound: stored values of either side differ by a bf16 rounding (up to 2^-8 of them) here and there.  A step of the integers is about a
    thirtieth of a row's mean value, so such a difference crosses a border in one of eight values and is a step there: sqrt(1 / 8) / 30 of
    the row in the square mean, 2^-6.4, twice in a row, and the roundings of a token's unit keys add 2^-9 a token: below 2^-5."""
    H, K, W, width = 4, 128, 4, 256
    gen = torch.Generator().manual_seed(21)
    w, lens, more = weights(gen, kind, width, H, G, K, V, W), (70, 25), 6
    x = [rand(gen, n + more, width, dtype=torch.bfloat16) for n in lens]
    r = [rand(gen, n + more, width, dtype=torch.bfloat16) for n in lens]
    want, res = zip(*(plain_layer(kind, act, w, a, b, H, G, K, V, [0, a.shape[0]]) for a, b in zip(x, r)))
    lay = layer.DeltaLayer(kind, 2, H, K, V, G, 8, 4, act=act, **w)
    first, residual = torch.cat([a[:n] for a, n in zip(x, lens)]).to(DEV), torch.cat([a[:n] for a, n in zip(r, lens)]).to(DEV)
    out = lay.prompt(prompts([0, 70, 95]), first, residual)
    off = lambda got, exp: float((ref.f64(got) - exp).norm() / exp.norm())  # noqa: E731
    full = torch.cat([a[:n] for a, n in zip(want, lens)])
    assert off(out, full) <= 2.0 ** -5
    assert torch.equal(ref.f64(residual), torch.cat([a[:n] for a, n in zip(res, lens)]))
    lay.begin_window()
    for i in range(more):
        tok, rr = (torch.stack([a[n + i] for a, n in zip(z, lens)]).to(DEV) for z in (x, r))
        got = lay.step(i % 4, tok, rr, exact=True)
        assert off(got, torch.stack([a[n + i] for a, n in zip(want, lens)])) <= 2.0 ** -5, i
        assert torch.equal(ref.f64(rr), torch.stack([a[n + i] for a, n in zip(res, lens)]))
    lay.m.check_status()
    # between windows: the ring's tokens go into the states, another prompt goes on from them, the sketch is built again
    lay.end_window(2)
    pr = binding.Prompts(torch.tensor([0, 3], dtype=torch.int32, device=DEV), 3, *(torch.tensor([1], dtype=torch.int32, device=DEV) for _ in range(2)))
    lay.prompt(pr, first[:3])
    lay.begin_window()
    assert torch.isfinite(lay.step(0, first[:2])).all()
    lay.m.check_status()


@pytest.mark.parametrize("kind", ["gdn", "kda"])
def test_a_layers_token_in_a_graph_and_calls_on_another_stream(kind):
    """A decode step of the layer, captured once and replayed for other tokens, gives what the calls give; so do calls on a stream that is
    not the current one."""
    H, G, K, V, W, width, B = 2, 1, 128, 128, 4, 128, 5
    gen = torch.Generator().manual_seed(4)
    w = weights(gen, kind, width, H, G, K, V, W)
    a, b = (layer.DeltaLayer(kind, B, H, K, V, G, 8, 4, **w) for _ in range(2))
    x0, side = rand(gen, 121, width, dtype=torch.bfloat16).to(DEV), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    first = a.prompt(prompts([0, 3, 9, 9, 120, 121]), x0)
    a.begin_window()
    other = b.prompt(prompts([0, 3, 9, 9, 120, 121]), x0, stream=side)
    b.begin_window(stream=side)
    x = rand(gen, B, width, dtype=torch.bfloat16).to(DEV)
    torch.cuda.synchronize()
    assert torch.equal(first, other) and torch.equal(a.m.state, b.m.state)
    keep = [t.clone() for t in (a.conv_state, a.m.ring)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = a.step(0, x)
    for t, old in zip((a.conv_state, a.m.ring), keep):
        t.copy_(old)
    x.copy_(rand(gen, B, width, dtype=torch.bfloat16))
    g.replay()
    want = b.step(0, x)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(a.conv_state, b.conv_state)


@pytest.mark.parametrize("kind", ["gdn", "kda"])
def test_a_layer_over_prompts_without_tokens(kind):
    """Sequences of no tokens, and no sequences: states and stored rows of the sequences' slots start from zeros, others stay."""
    H, G, K, V, width = 4, 1, 128, 128, 256
    lay = layer.DeltaLayer(kind, 3, H, K, V, G, 8, 4, **weights(torch.Generator().manual_seed(1), kind, width, H, G, K, V, 4))
    lay.m.state.fill_(3.0), lay.conv_state.fill_(2.0)
    empty = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    pr = binding.Prompts(torch.zeros(3, dtype=torch.int32, device=DEV), 0, slots=torch.tensor([2, 0], dtype=torch.int32, device=DEV))
    assert lay.prompt(pr, empty(0, width), empty(0, width)).shape == (0, width)
    for t, old in ((lay.m.state, 3.0), (lay.conv_state, 2.0)):
        assert (t[0] == 0).all() and (t[1] == old).all() and (t[2] == 0).all()
    none = binding.Prompts(torch.zeros(1, dtype=torch.int32, device=DEV), 0)
    assert lay.prompt(none, empty(0, width)).shape == (0, width)
    assert (lay.m.state[1] == 3).all()
    lay.m.check_status()


def test_a_layer_refuses_what_does_not_fit():
    w = weights(torch.Generator().manual_seed(1), "gdn", 128, 2, 1, 128, 128, 4)
    with pytest.raises(ValueError, match="kind is gdn or kda"):
        layer.DeltaLayer("mamba2", 1, 2, 128, 128, 1, 8, 4, **w)
    with pytest.raises(ValueError, match="act is silu or sigmoid"):
        layer.DeltaLayer("gdn", 1, 2, 128, 128, 1, 8, 4, act="relu", **w)
    with pytest.raises(ValueError, match="w_in has"):
        layer.DeltaLayer("kda", 1, 2, 128, 128, 1, 8, 4, **w)
