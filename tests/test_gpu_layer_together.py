"""The operators around the recurrence in a row, as a layer runs them: a prompt, the sketch, decode steps, a flush.

The recurrence alone is compared to the rounding of its outputs: a prompt in one scan against the same tokens given one by one to the
convolution's token form and the library's exact decode.  The whole layer passes two roundings to e4m3 on the way, where values that
differ by a bf16 rounding can fall on either side; its bound is derived at the test."""
import pytest
import torch

from paper_2609_33051_b200 import binding, layer
from tests import layer_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(dtype)


def prompts(starts):
    return binding.Prompts(torch.tensor(starts, dtype=torch.int32, device=DEV), starts[-1])


@pytest.mark.parametrize("H,G,K,V,W", [(4, 2, 128, 64, 4), (3, 1, 128, 80, 3), (8, 8, 64, 64, 2), (2, 1, 128, 128, 4)])
def test_a_prompt_and_its_tokens_one_by_one(H, G, K, V, W):
    """conv -> scan over a prompt, and conv_step -> full read / state update for its tokens: equal values, keys and queries, states within
    fp32 sums of the window, outputs within their roundings."""
    B, L, T, bf = 3, 4, 11, torch.bfloat16
    gen = torch.Generator().manual_seed(H + V)
    C = H * V + 2 * G * K
    x, dt = rand(gen, B, T, C, dtype=bf).to(DEV), rand(gen, B, T, H, dtype=bf).to(DEV)
    w, b, a = rand(gen, C, W, scale=0.5).to(DEV), rand(gen, C).to(DEV), -torch.exp(rand(gen, H)).to(DEV)
    bias, skip = rand(gen, H).to(DEV), rand(gen, H).to(DEV)
    m, s = (binding.SketchSSM("mamba2", B, H, K, V, 8, L, io="bf16", device=0) for _ in range(2))
    start, rows = rand(gen, B, H, K, V).to(DEV), rand(gen, B, W - 1, C, dtype=bf).to(DEV)
    own = torch.arange(B, dtype=torch.int32, device=DEV)
    pr = binding.Prompts(T * torch.arange(B + 1, dtype=torch.int32, device=DEV), B * T, slots=own, resume=own)
    m.state.copy_(start)
    conv_a, conv_b = rows.clone(), rows.clone()
    c = torch.empty(B * T, C, dtype=bf, device=DEV)
    m.causal_conv(pr, x.view(B * T, C), w, b, conv_a, c)
    v, k, q = c[:, :H * V].unflatten(1, (H, V)), c[:, H * V:H * V + G * K].unflatten(1, (G, K)), c[:, H * V + G * K:].unflatten(1, (G, K))
    y = torch.empty(B * T, H, V, device=DEV)
    m.prompt_scan(pr, q, k, v, dt.view(B * T, H), a, y, dt_bias=bias, skip=skip)
    s.state.copy_(start)
    t, n = s.new_token_buffers(), 0
    outs = torch.empty(B, T, H, V, device=DEV)
    spread = lambda z: z.view(B, T, G, K).repeat_interleave(H // G, 2)  # noqa: E731
    for i in range(T):
        s.conv_step(x[:, i], dt[:, i], w, b, conv_b, a, bias, t, groups=G)
        assert torch.equal(t["v"], v.view(B, T, H, V)[:, i]) and torch.equal(t["k"], spread(k)[:, i]) and torch.equal(t["q"], spread(q)[:, i])
        args = [t[z] for z in ("q", "k", "v", "beta", "decay")]
        if n == L - 1:
            s.state_update(n, *args, t["out"])
        else:
            s.full_read_decode(n, *args, t["out"])
        n = (n + 1) % L
        outs[:, i] = t["out"] + skip[:, None] * t["v"].float()
    s.state_update(n, flags=binding.NO_SKETCH)          # what is left in the ring
    m.check_status(), s.check_status()
    assert torch.equal(conv_a, conv_b)
    want, mag, new, new_mag = ref.scan([T * i for i in range(B + 1)], None, list(range(B)), q, k, v, dt.view(B * T, H), a, bias, skip, start, B)
    # the scan as its own test has it; the flushes split their operands in two parts of bf16 (2^-16 of a term each)
    rel = (6 * T + K + 16) * 2.0 ** -24
    ref.close(y, want, rel * mag, "scan")
    ref.close(outs.view(B * T, H, V), want, (rel + 3 * 2.0 ** -16) * mag, "steps")
    ref.close(m.state, new, rel * new_mag, "state")
    ref.close(s.state, new, (rel + 3 * 2.0 ** -16) * new_mag, "state by steps")


def weights(gen, width, H, G, K, V, W):
    C, inner = H * V + 2 * G * K, H * V
    return dict(norm=1 + 0.1 * rand(gen, width), w_in=rand(gen, 2 * inner + 2 * G * K + H, width, scale=width ** -0.5), conv_weight=rand(gen, C, W, scale=0.5),
                conv_bias=0.1 * rand(gen, C), a=-torch.exp(rand(gen, H)), dt_bias=rand(gen, H) - 1, skip=rand(gen, H),
                gate_norm=1 + 0.1 * rand(gen, inner), w_out=rand(gen, width, inner, scale=inner ** -0.5))


def plain_layer(w, x, residual, H, G, K, V, starts):
    """The layer in 64 bits, with the roundings of what is stored: e4m3 activations and weights, bf16 between the calls."""
    def quant(z):
        top = torch.nn.functional.pad(z, (0, -z.shape[1] % 128)).unflatten(1, (-1, 128)).abs().amax(-1).repeat_interleave(128, 1)[:, :z.shape[1]]
        return ((z * 448 / top).float().to(torch.float8_e4m3fn).double() * top / 448)

    def weight(z):
        q8, scale = layer.quantise_weight(z)
        return q8.double() * scale.double().repeat_interleave(128, 0)[:z.shape[0]].repeat_interleave(128, 1)[:, :z.shape[1]]

    bf = lambda z: z.to(torch.bfloat16).double()  # noqa: E731
    inner, C = H * V, H * V + 2 * G * K
    h = x.double() + residual.double()
    p = bf(quant(ref.norm(h, w["norm"], 1e-5, 0)[1]) @ weight(w["w_in"]).T)
    gate, xbc, dt = p[:, :inner], p[:, inner:inner + C], p[:, inner + C:]
    c = bf(ref.conv(starts, None, None, xbc, w["conv_weight"], w["conv_bias"], torch.zeros(8, w["conv_weight"].shape[1] - 1, C), True, 8)[0])
    v, k, q = c[:, :inner].unflatten(1, (H, V)), c[:, inner:inner + G * K].unflatten(1, (G, K)), c[:, inner + G * K:].unflatten(1, (G, K))
    y = bf(ref.scan(starts, None, None, q, k, v, dt, w["a"], w["dt_bias"], w["skip"], torch.zeros(8, H, K, V), 8)[0].flatten(1))
    return bf(quant(ref.norm(y, w["gate_norm"], 1e-5, 0, gate=gate)[1]) @ weight(w["w_out"]).T), bf(h)


def test_a_layer_over_prompts_and_then_token_by_token():
    """Prompts of 40 and 25 tokens, then 6 tokens each (a window of 4: decode steps and a flush), against the layer over the whole
    sequences in 64 bits.

    Bound: stored values of either side differ by a bf16 rounding (up to 2^-8 of them) here and there, and where such a value lies next to a
    border of e4m3 the two roundings differ by a step, 2^-3 of it.  A difference of up to 2^-8 reaches a border in one of 2^4 values,
    so an activation is off by sqrt(2^-4) 2^-3 = 2^-5 of itself in the square mean, twice in a row: 2^-4 of the result."""
    H, G, K, V, W, width = 4, 2, 128, 64, 4, 256
    gen = torch.Generator().manual_seed(21)
    w, lens, more = weights(gen, width, H, G, K, V, W), (40, 25), 6
    x = [rand(gen, n + more, width, dtype=torch.bfloat16) for n in lens]
    r = [rand(gen, n + more, width, dtype=torch.bfloat16) for n in lens]
    want, res = zip(*(plain_layer(w, a, b, H, G, K, V, [0, a.shape[0]]) for a, b in zip(x, r)))
    lay = layer.Mamba2Layer(2, H, K, V, G, 8, 4, **{n: t for n, t in w.items()})
    first, residual = torch.cat([a[:n] for a, n in zip(x, lens)]).to(DEV), torch.cat([a[:n] for a, n in zip(r, lens)]).to(DEV)
    out = lay.prompt(prompts([0, 40, 65]), first, residual)
    off = lambda got, exp: float((ref.f64(got) - exp).norm() / exp.norm())  # noqa: E731
    full = torch.cat([a[:n] for a, n in zip(want, lens)])
    assert off(out, full) <= 2.0 ** -4
    assert torch.equal(ref.f64(residual), torch.cat([a[:n] for a, n in zip(res, lens)]))
    lay.begin_window()
    for i in range(more):
        tok, rr = (torch.stack([a[n + i] for a, n in zip(z, lens)]).to(DEV) for z in (x, r))
        got = lay.step(i % 4, tok, rr, exact=True)
        assert off(got, torch.stack([a[n + i] for a, n in zip(want, lens)])) <= 2.0 ** -4, i
        assert torch.equal(ref.f64(rr), torch.stack([a[n + i] for a, n in zip(res, lens)]))
    lay.m.check_status()


def test_a_layers_token_in_a_graph():
    """A decode step of the layer, captured once and replayed for other tokens, gives what the calls give."""
    H, G, K, V, W, width, B = 2, 1, 128, 64, 4, 128, 5
    gen = torch.Generator().manual_seed(4)
    w = weights(gen, width, H, G, K, V, W)
    a, b = (layer.Mamba2Layer(B, H, K, V, G, 8, 4, **w) for _ in range(2))
    for lay in (a, b):
        lay.prompt(prompts([0, 3, 9, 9, 20, 21]), rand(torch.Generator().manual_seed(1), 21, width, dtype=torch.bfloat16).to(DEV))
        lay.begin_window()
    x = rand(gen, B, width, dtype=torch.bfloat16).to(DEV)
    torch.cuda.synchronize()
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


def test_what_a_call_allocates_belongs_to_its_stream(monkeypatch):
    """Tensors that a call makes and drops are made on the stream that the caller named: their memory would otherwise go to the current
    stream's next tensors while the kernels still use it."""
    H, G, K, V, W, width, B = 4, 1, 128, 64, 4, 256, 3
    gen = torch.Generator().manual_seed(6)
    w = weights(gen, width, H, G, K, V, W)
    a, b = (layer.Mamba2Layer(B, H, K, V, G, 8, 4, **w) for _ in range(2))
    lens = [0, 1100, 1103, 1110]
    x, tok = rand(gen, lens[-1], width, dtype=torch.bfloat16).to(DEV), rand(gen, B, width, dtype=torch.bfloat16).to(DEV)
    pr = prompts(lens)
    want = a.prompt(pr, x)
    a.begin_window()
    want_tok = a.step(0, tok)
    args = [torch.zeros(lens[-1], *d, dtype=torch.bfloat16, device=DEV) for d in ((G, K), (G, K), (H, V), (H,))]
    y = torch.zeros(lens[-1], H, V, device=DEV)
    torch.cuda.synchronize()
    side, seen, empty = torch.cuda.Stream(), [], torch.empty

    def watched(*args, **kw):
        seen.append(torch.cuda.current_stream())
        return empty(*args, **kw)

    monkeypatch.setattr(torch, "empty", watched)
    out = b.prompt(pr, x, stream=side)
    b.begin_window(stream=side)
    out_tok = b.step(0, tok, stream=side)
    assert len(seen) > 9 and all(s == side for s in seen)
    assert torch.cuda.current_stream() != side
    del seen[:]
    b.m.prompt_scan(pr, *args, a.a, y, stream=side)
    assert seen == [side]                      # the scan's scratch
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(out_tok, want_tok)
