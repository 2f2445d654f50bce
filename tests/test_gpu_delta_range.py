"""The delta rule's scan over numbers of very different size: step sizes, values and states that a chunk's common scale has to hold.  Tolerances are
delta_ref's bound of fp32 arithmetic, and, where the error as a whole is looked at, what the other tests of the operator allow it."""
import pytest
import torch

from tests import delta_ref as dref
from tests import layer_ref as ref
from tests.test_gpu_delta_operators import DEV, NAMES, batch_of, check_scan, layer, run_scan, scan_inputs

pytestmark = pytest.mark.gpu


def inputs(lengths, H=2, **kw):
    return scan_inputs("gdn", lengths, H, 1, 128, 128, "bf16", 8, **kw)


@pytest.mark.parametrize("size", [1e6, 1e8])
@pytest.mark.parametrize("od", ["bf16", "f32"])
def test_a_large_state_that_decays_over_chunks(size, od):
    """A stored state far above the values, of which a chunk leaves a five-hundredth or so: the tokens hundreds of places behind it have their own size's
    accuracy."""
    x = inputs([1000], seed=12)
    x["state"] = x["state"] * size
    x["a"], x["bias"] = torch.full((2,), -1.0), torch.full((2,), -2.3)
    x["dt"] = x["dt"] * 0.1
    starts, pr = batch_of([1000], None, [1])
    check_scan(layer(8, 2), x, starts, pr, None, [1], od)


@pytest.mark.parametrize("b", [-5.0, -7.0])
def test_small_step_sizes_keep_their_bits(b):
    """Outputs and states are as small as the step sizes, and still right to the accuracy of their own size: the bounds of
    test_scan_keeps_fp32s_accuracy, for decays of a length that does not grow with the prompt."""
    x = inputs([300], seed=11)
    x["b"] = (x["b"].float() * 0.25 + b).to(torch.bfloat16)
    x["a"] = torch.tensor([-4.0, -0.5])
    starts, pr = batch_of([300])
    m = layer(8, 2)
    want, _, new, _ = dref.scan(starts, None, None, *(x[n] for n in NAMES), x["bias"], x["state"], 8)
    out = torch.empty(300, 2, 128, dtype=torch.bfloat16, device=DEV)
    run_scan(m, pr, x, out)
    assert (m.state[:1].cpu().double() - new[:1]).norm() <= 1e-6 * new[:1].norm()
    assert (out.cpu().double() - want).norm() <= 2.0e-3 * want.norm()


@pytest.mark.parametrize("od", ["bf16", "f32"])
def test_what_has_decayed_of_larger_values_leaves_no_trace(od):
    """Values some hundred times as large at a chunk's start, of which a token leaves two thirds: the tokens that meet nothing of them are right to their
    own size."""
    x = inputs([300], seed=20)
    x["v"][64:67] *= 256
    x["v"][130, :, ::3] *= 512
    x["a"], x["bias"], x["dt"] = torch.full((2,), -1.0), torch.full((2,), -0.7), x["dt"] * 0.1
    starts, pr = batch_of([300], None, [1])
    check_scan(layer(8, 2), x, starts, pr, None, [1], od)


@pytest.mark.parametrize("od", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", [[300], [70, 1, 100], [129]])
@pytest.mark.parametrize("size", [2.0 ** 12, 2.0 ** 18, 2.0 ** 24, 2.0 ** 32, 1e30, -1e38])
def test_a_large_value_changes_no_token_before_it(size, lengths, od):
    """Values of any finite size at places of a chunk, in some columns: earlier tokens, other columns, and what comes when it has decayed, to the same
    bound."""
    x = inputs(lengths, seed=13)
    x["a"] = torch.tensor([-16.0, -0.5])                     # one head forgets it, the other one does not
    x["bias"] = x["bias"] + 2
    T = sum(lengths)
    for t, h, c in ((0, 0, 3), (40, 0, 5), (40, 1, 5), (63, 1, 64), (64, 0, 127), (100, 1, 31), (101, 1, 31), (T - 1, 0, 40)):
        x["v"][t, h, c] = size
    starts, pr = batch_of(lengths, None, None)
    check_scan(layer(8, 2), x, starts, pr, None, None, od)


@pytest.mark.parametrize("od", ["bf16", "f32"])
@pytest.mark.parametrize("a", [-16.0, -4.0, -0.05])
@pytest.mark.parametrize("size", [1e-30, 1e3, 1e6, 1e12, 1e30])
def test_a_stored_state_of_any_size(size, a, od):
    """A stored state far from the values' size, with decays that take it below them within a token, within a chunk, and not at all."""
    x = inputs([200, 140], seed=14)
    x["state"] = x["state"] * size
    x["a"], x["bias"] = torch.full((2,), a), x["bias"] + 3
    starts, pr = batch_of([200, 140], None, [1, 5])
    check_scan(layer(8, 2), x, starts, pr, None, [1, 5], od)


@pytest.mark.parametrize("a", [-16.0, -0.5])
@pytest.mark.parametrize("size", [2.0 ** -8, 2.0 ** -20, 2.0 ** -60, 0.0])
def test_tokens_of_small_values_between_others(size, a):
    """Runs of small values, or of none, before, between and behind others, from zeros and from a stored state of zeros."""
    x = inputs([260, 90], seed=15)
    x["v"][:30] *= size
    x["v"][70:200] *= size
    x["v"][250:270] *= size
    x["v"][300:, :, ::2] *= size
    x["a"], x["bias"] = torch.full((2,), a), x["bias"] + 2
    x["state"][3] = 0
    starts, pr = batch_of([260, 90], None, [-1, 3])
    want, tol, new, new_tol = dref.scan(starts, None, [-1, 3], *(x[n] for n in NAMES), x["bias"], x["state"], 8)
    m = layer(8, 2)
    m.state.copy_(x["state"])
    out = torch.empty(350, 2, 128, dtype=torch.bfloat16, device=DEV)
    run_scan(m, pr, x, out)
    # Below 2^-126 numbers are multiples of 2^-133 in bf16, and of 2^-149 in fp32: what decays to that is off by half of the former, and each of its
    # forty roundings by half of the latter.
    ref.close(out, want, ref.half_step(torch.bfloat16) * want.abs() + tol + 2.0 ** -134 + 40 * 2.0 ** -150, "out")
    ref.close(m.state[:2], new[:2], new_tol[:2] + 40 * 2.0 ** -150, "state")


@pytest.mark.parametrize("b", [-9.0, -12.0, -16.0, -24.0])
def test_tiny_step_sizes_keep_their_bits(b):
    """As above, where the state is so small beside the values that a common scale would leave it no bits."""
    x = inputs([200], seed=16)
    x["b"] = (x["b"].float() * 0.25 + b).to(torch.bfloat16)
    x["a"] = torch.tensor([-4.0, -0.5])
    starts, pr = batch_of([200])
    m = layer(8, 2)
    want, _, new, _ = dref.scan(starts, None, None, *(x[n] for n in NAMES), x["bias"], x["state"], 8)
    out = torch.empty(200, 2, 128, dtype=torch.bfloat16, device=DEV)
    run_scan(m, pr, x, out)
    assert (m.state[:1].cpu().double() - new[:1]).norm() <= 1e-6 * new[:1].norm()
    assert (out.cpu().double() - want).norm() <= 2.0e-3 * want.norm()


@pytest.mark.parametrize("H", [2, 3])
def test_large_values_in_a_prompt_of_segments(H):
    """A prompt that is split into segments: large values in the first one, in a middle one and in the last one."""
    x = inputs([3300], H, seed=17)
    x["a"] = torch.linspace(-8, -0.5, H)
    for t, h, c in ((50, 0, 3), (1500, 1, 7), (1501, 0, 9), (2000, 1, 70), (3290, 0, 100)):
        x["v"][t, h, c] = 2.0 ** 26
    starts, pr = batch_of([3300], [4], [4])
    check_scan(layer(8, H), x, starts, pr, [4], [4], "bf16")


def test_large_values_beside_ones_that_are_not_finite():
    """NaN and infinity reach what they reach, and nothing before them, in chunks that are taken token by token too."""
    x = inputs([200, 60], seed=18)
    inf, nan = float("inf"), float("nan")
    for t, h, c, value in ((10, 0, 5, 1e30), (20, 0, 5, inf), (30, 1, 6, 1e25), (31, 1, 8, nan), (75, 0, 9, -1e20), (220, 0, 4, 1e30), (230, 1, 4, nan)):
        x["v"][t, h, c] = value
    x["k"][130, 0, 7] = nan
    x["v"][129, 0, 11] = 1e28
    x["q"][225, 0, 0] = nan
    x["a"][:] = -8.0
    starts, pr = batch_of([200, 60], None, [6, -1])
    want, tol, new, new_tol = dref.scan(starts, None, [6, -1], *(x[n] for n in NAMES), x["bias"], x["state"], 8)
    m = layer(8, 2)
    m.state.copy_(x["state"])
    out = torch.zeros(260, 2, 128, dtype=torch.bfloat16, device=DEV)
    run_scan(m, pr, x, out)
    for got, exp, bound in ((out, want, ref.half_step(torch.bfloat16) * want.abs() + tol), (m.state[:2], new[:2], new_tol[:2])):
        there = torch.isfinite(exp)
        assert torch.equal(torch.isfinite(got.cpu()), there)
        ref.close(ref.f64(got)[there], exp[there], bound[there], "finite ones")


def test_large_values_twice_are_the_same_to_the_bit():
    x = inputs([700, 30], 4, seed=19)
    x["v"][::37, 1, 5] = 1e12
    x["a"][:] = -6.0
    starts, pr = batch_of([700, 30])
    m, outs = layer(8, 4), []
    for _ in range(2):
        m.state.copy_(x["state"])
        out = torch.empty(730, 4, 128, dtype=torch.bfloat16, device=DEV)
        run_scan(m, pr, x, out)
        outs.append((out.view(torch.int16), m.state.clone().view(torch.int32)))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.parametrize("kind,od", [("gdn", "bf16"), ("gdn", "f32"), ("kda", "bf16")])
def test_infinite_gates_are_what_the_formulas_give(kind, od):
    """Step sizes of nothing and of one, decays of nothing and of one, from arguments that are infinite: nothing that is not finite comes of them."""
    x = scan_inputs(kind, [200, 20], 2, 1, 128, 128, "bf16", 8, seed=21)
    inf = float("inf")
    for t, h, value in ((3, 0, inf), (70, 1, -inf), (71, 1, inf), (130, 0, -inf), (210, 1, -inf)):
        x["b"][t, h] = value
    for t, h, value in ((5, 0, -inf), (66, 1, inf), (100, 0, inf), (140, 1, -inf), (205, 0, inf)):
        x["dt"][t, h] = value
    starts, pr = batch_of([200, 20], None, [1, 5])
    check_scan(layer(8, 2, kind=kind), x, starts, pr, None, [1, 5], od)


def test_a_long_sequence_without_decays():
    """Nothing decays, and the bound behind a column's scale grows with every chunk while the state does not: 94 chunks of one sequence (among others, so
    that it is not split) keep the accuracy of test_scan_keeps_fp32s_accuracy."""
    lengths = [6000] + [10] * 18
    x = scan_inputs("gdn", lengths, 4, 2, 128, 128, "bf16", 19, seed=22)
    x["a"] = torch.tensor([0.0, -1e-5, -1e-3, 0.0])
    x["k"][:, 1, 64:] = 0                                # half of the rows of the states of two heads stay zeros
    starts, pr = batch_of(lengths)
    m = layer(19, 4)
    want, _, new, _ = dref.scan(starts, None, None, *(x[n] for n in NAMES), x["bias"], x["state"], 19)
    out = torch.empty(sum(lengths), 4, 128, dtype=torch.bfloat16, device=DEV)
    run_scan(m, pr, x, out)
    assert (m.state.cpu().double() - new).norm() <= 1e-6 * new.norm()
    assert (out.cpu().double() - want).norm() <= 2.0e-3 * want.norm()


@pytest.mark.parametrize("a", [-16.0, -2.0])
@pytest.mark.parametrize("phase", [0, 1, 2, 3])
def test_small_neighbours_between_large_ones(phase, a):
    """Two small values between two large ones, again and again, wherever the pairs begin."""
    x = inputs([200, 67], seed=23)
    t = (torch.arange(267) + phase) % 4
    x["v"][t < 2] *= 2.0 ** -30
    x["a"], x["bias"] = torch.full((2,), a), x["bias"] + 3
    starts, pr = batch_of([200, 67], None, [1, -1])
    check_scan(layer(8, 2), x, starts, pr, None, [1, -1], "bf16")


@pytest.mark.parametrize("seed", range(6))
def test_sizes_drawn_at_random(seed):
    """Values, keys, states and gates over dozens of powers of two, drawn for every token and column, every token, every column."""
    gen, lengths = torch.Generator().manual_seed(seed), [[200], [65, 130], [64, 1, 33]][seed % 3]
    x, T = inputs(lengths, seed=30 + seed), sum(lengths)
    powers = lambda spread, *shape: 2.0 ** (spread * torch.randn(*shape, generator=gen))  # noqa: E731
    x["v"] = (x["v"].float() * powers(8, *((T, 2, 128), (T, 1, 1), (1, 1, 128))[seed // 2])).to(torch.bfloat16)
    if seed % 2:
        x["k"] = (x["k"].float() * powers(4, T, 1, 128)).to(torch.bfloat16)
        x["state"] = x["state"] * powers(12, 8, 2, 128, 128)
        x["b"], x["dt"] = x["b"] * 4, x["dt"] * 4
    x["a"] = -torch.exp(3 * torch.rand(2, generator=gen) - 1)
    resume = [1] + [-1] * (len(lengths) - 1)
    starts, pr = batch_of(lengths, None, resume)
    check_scan(layer(8, 2), x, starts, pr, None, resume, "bf16")
