"""A layer's prompts between decode steps, and its gated norm in groups."""
import pytest
import torch

from paper_2609_33051_b200 import binding, layer
from tests.test_gpu_layer_together import rand, weights

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
H, G, K, V, W, WIDTH, L = 4, 2, 128, 64, 4, 256, 4


def make(seed=3, B=2, **kw):
    return layer.Mamba2Layer(B, H, K, V, G, 8, L, **weights(torch.Generator().manual_seed(seed), WIDTH, H, G, K, V, W), **kw)


def one_prompt(n, slot):
    return binding.Prompts(torch.tensor([0, n], dtype=torch.int32, device=DEV), n, slots=torch.tensor([slot], dtype=torch.int32, device=DEV))


@pytest.mark.parametrize("before", [1, 2, 3])
def test_a_prompt_between_decode_steps(before):
    """A sequence decodes `before` tokens of a window; another one's prompt is taken in; both decode on.  The first has the states of a layer
    that never stopped, the second those of a layer that held it alone: sums of the same terms in another order, the flushes' in two parts of
    bf16 (2^-16 of a term; far below 2^-12 of the state's norm)."""
    gen, after = torch.Generator().manual_seed(before), 3
    first, second = (rand(gen, n, WIDTH, dtype=torch.bfloat16).to(DEV) for n in (30, 20))
    tokens = [rand(gen, 2, WIDTH, dtype=torch.bfloat16).to(DEV) for _ in range(before + after)]
    lay, alone, other = make(), make(), make()
    for a in (lay, alone):
        a.prompt(one_prompt(30, 0), first)
        a.begin_window()
    for i in range(before):
        lay.step(i, tokens[i], exact=True)
    lay.end_window(before)
    lay.prompt(one_prompt(20, 1), second)
    lay.begin_window()
    other.prompt(one_prompt(20, 1), second)
    other.begin_window()
    for i in range(after):
        lay.step(i, tokens[before + i], exact=True)
        other.step(i, tokens[before + i], exact=True)
    for i in range(before + after):
        alone.step(i % L, tokens[i], exact=True)
    lay.end_window(after), other.end_window(after), alone.end_window((before + after) % L)
    off = lambda a, b: float((a - b).norm() / b.norm())  # noqa: E731
    assert off(lay.m.state[0], alone.m.state[0]) <= 2.0 ** -12 and off(lay.m.state[1], other.m.state[1]) <= 2.0 ** -12
    assert torch.equal(lay.conv_state[0], alone.conv_state[0]) and torch.equal(lay.conv_state[1], other.conv_state[1])
    assert off(lay.m.state[0], make().m.state[0] + 1) > 0.1                   # (there is a state)
    lay.m.check_status()


def test_the_ring_of_an_ended_window_is_empty():
    """What the steps left in the ring is in the states: a window that ends early and one that goes on have the same."""
    a, b = make(), make()
    x = [rand(torch.Generator().manual_seed(i), 2, WIDTH, dtype=torch.bfloat16).to(DEV) for i in range(L)]
    for i in range(L):
        a.step(i, x[i])
        b.step(i, x[i]) if i < 2 else b.step(i - 2, x[i])
        if i == 1:
            b.end_window(2)
            b.begin_window()
    b.end_window(2)
    assert float((a.m.state - b.m.state).norm() / a.m.state.norm()) <= 2.0 ** -12


@pytest.mark.parametrize("group", [0, 128])
def test_the_gated_norm_in_groups(group):
    """The layer's prompt and step are the library's calls in a row, the norm in the groups that were asked for."""
    lay, m, inner = make(norm_group=group), None, H * V
    m, t = lay.m, 50
    x = rand(torch.Generator().manual_seed(9), t, WIDTH, dtype=torch.bfloat16).to(DEV)
    out = lay.prompt(one_prompt(t, 0), x)
    e4m3, bf = torch.float8_e4m3fn, torch.bfloat16
    new = lambda r, c, dtype=bf: torch.empty(r, c, dtype=dtype, device=DEV)  # noqa: E731

    def project(z, kw, w, scale):
        z8, s = new(z.shape[0], z.shape[1], e4m3), new(z.shape[0], -(-z.shape[1] // 128), torch.float32)
        m.rms_norm(z, out8=z8, scale=s, **kw)
        return m.scaled_matmul(z8, s, w, scale, new(z.shape[0], w.shape[0]))

    p = project(x, dict(weight=lay.norm), lay.w_in, lay.w_in_scale)
    c = m.causal_conv(one_prompt(t, 0), p[:, inner:inner + lay.channels], lay.conv_weight, lay.conv_bias, m.new_conv_state(lay.channels, W), new(t, lay.channels))
    v, k, q = c[:, :inner].unflatten(1, (H, V)), c[:, inner:inner + G * K].unflatten(1, (G, K)), c[:, inner + G * K:].unflatten(1, (G, K))
    y = new(t, inner)
    m.prompt_scan(one_prompt(t, 0), q, k, v, p[:, inner + lay.channels:inner + lay.channels + H], lay.a, y.unflatten(1, (H, V)), dt_bias=lay.dt_bias, skip=lay.skip)
    want = project(y, dict(weight=lay.gate_norm, gate=p[:, :inner], group=group), lay.w_out, lay.w_out_scale)
    assert torch.equal(out, want)
    whole = project(y, dict(weight=lay.gate_norm, gate=p[:, :inner]), lay.w_out, lay.w_out_scale)
    assert torch.equal(out, whole) == (group == 0)
    lay.begin_window()
    a, b = make(norm_group=group), make()
    for z in (a, b):
        z.m.state.copy_(m.state), z.conv_state.copy_(lay.conv_state), z.begin_window()
    assert torch.equal(a.step(0, x[:2]), b.step(0, x[:2])) == (group == 0)
