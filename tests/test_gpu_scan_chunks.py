"""The prompt scan with bfloat16 tensors and outputs, K = 128, which goes through in chunks of 128 tokens: its outputs are sums of fp32
accuracy, rounded once.

Tolerance.  u = 2^-24; A is the sum of the absolute terms, n the sequence's length.  As for the token-by-token scan a term is off by
(6 n + K + 16) u.  A weight of another token and the state go to their products in two parts of bfloat16, off by 2^-8 of 2^-8: 2^-16 of
a term, which takes one of the two ways.  A weight's log2 is a difference of two sums of fractions of up to 64 in size, each of at most ten
roundings of 2^-19: 2^-14.7, ln 2 of that in the weight.  Together less than 2^-14 of A, and one rounding of the result."""
import pytest
import torch

from paper_2609_33051_b200 import binding
from tests import layer_ref as ref
from tests.test_gpu_layer_operators import DEV, SCAN, U, batch_of, layer, scan_inputs, strided

pytestmark = pytest.mark.gpu
PARTS = 2.0 ** -14
BF16 = torch.bfloat16
INPUTS = ("q", "k", "v", "dt", "a", "bias", "skip", "state")


def on_device(x):
    return {n: t.to(DEV) for n, t in x.items()}


def held(m, x, out, starts, slots, resume, parts=PARTS, state=None):
    """Outputs and states against the plain 64-bit scan, with the tolerance above."""
    want, mag, new, new_mag = ref.scan(starts, slots, resume, *(x[n] for n in INPUTS[:-1]), x["state"] if state is None else state, m.B)
    n = max([b - a for a, b in zip(starts, starts[1:])] + [0])
    rel = (6 * n + m.K + 16) * U
    ref.close(out, want, ref.half_step(BF16) * want.abs() + (rel + parts) * mag, "out")
    ref.close(m.state, new, rel * new_mag, "state")


def run(m, pr, x, **kw):
    T, H, V = x["v"].shape
    out = strided(torch.full((T, H, V), float("nan"), dtype=BF16), 8)
    m.state.copy_(x["state"])
    m.prompt_scan(pr, strided(x["q"], 8), strided(x["k"], 16, 8), strided(x["v"], 24), strided(x["dt"], 1, 2), x["a"].to(DEV), out,
                  dt_bias=x["bias"].to(DEV), skip=x["skip"].to(DEV), **kw)
    m.check_status()
    return out


SIZES = [c[:5] + c[7:] for c in SCAN if c[5] == c[6] == "bf16"]


@pytest.mark.parametrize("lengths,H,G,K,V,slots,resume,first,tail", SIZES)
def test_outputs_are_rounded_once(lengths, H, G, K, V, slots, resume, first, tail):
    """(K = 64 and V = 80 are summed token by token: no parts there.)"""
    starts, pr = batch_of(lengths, slots, resume, first, tail)
    m, x = layer(8, H, K, V), scan_inputs(lengths, H, G, K, V, "bf16", 8, first, tail, seed=1)
    held(m, x, run(m, pr, x), starts, slots, resume, PARTS if K == 128 and V % 64 == 0 else 0.0)


@pytest.mark.parametrize("lengths,H,G,V", [([300], 3, 1, 64), ([128, 250, 60], 2, 2, 128), ([1300], 2, 1, 64)])
@pytest.mark.parametrize("behind", [20, 61, 96, 125])
def test_tokens_behind_a_strong_reset(lengths, H, G, V, behind):
    """Tokens that all but clear the state (log2 decays near -140 each), then small steps: their weights are near one, while the sums of
    the chunk's log2 decays are in the thousands."""
    x = scan_inputs(lengths, H, G, 128, V, "bf16", 4, seed=behind)
    gen = torch.Generator().manual_seed(behind)
    place = torch.cat([torch.arange(n) % 128 for n in lengths])[:, None]
    strong, weak = 6 + 2 * torch.rand(x["dt"].shape, generator=gen), -6 + torch.rand(x["dt"].shape, generator=gen)
    x["dt"], x["bias"] = torch.where(place < behind, strong, weak).to(BF16), torch.zeros(H)
    x["a"] = -12 - 4 * torch.rand(H, generator=gen)
    starts, pr = batch_of(lengths)
    m = layer(4, H, 128, V)
    held(m, x, run(m, pr, x), starts, None, None)


@pytest.mark.parametrize("dt,a", [(-200.0, -1.0), (60.0, -16.0), (0.0, 0.0), (8.0, -1e-4), (30.0, -1e30), (3.0, -3.0), (-5.0, -16.0)])
@pytest.mark.parametrize("lengths", [[300], [1100]])
def test_extreme_gates(dt, a, lengths):
    """Step sizes of zero, decays of zero and of one, and sums of their logarithms far beyond fp32's range of exponentials."""
    x = scan_inputs(lengths, 2, 1, 128, 64, "bf16", 8)
    x["dt"] = (x["dt"].float() + dt).to(BF16)
    x["a"] = torch.full((2,), a)
    starts, pr = batch_of(lengths, None, [1])
    m = layer(8, 2, 128, 64)
    held(m, x, run(m, pr, x), starts, None, [1])


def test_a_prompt_in_pieces_on_another_stream():
    """A prompt in four calls that go on from the stored state, one of them split into segments, is the prompt in one."""
    x = scan_inputs([1500], 4, 1, 128, 64, "bf16", 8, seed=9)
    m, s, d = layer(8, 4, 128, 64), torch.cuda.Stream(), on_device(x)
    out = torch.zeros(1500, 4, 64, dtype=BF16, device=DEV)
    m.state.copy_(d["state"])
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for i, (lo, hi) in enumerate(((0, 130), (130, 131), (131, 1400), (1400, 1500))):
            _, pr = batch_of([hi - lo], [0], [0 if i else -1])
            m.prompt_scan(pr, *(d[n][lo:hi] for n in ("q", "k", "v", "dt")), d["a"], out[lo:hi], dt_bias=d["bias"], skip=d["skip"])
    s.synchronize()
    m.check_status()
    held(m, x, out, [0, 1500], None, None)


@pytest.mark.parametrize("H,T,batches", [
    (4, 300, (([200, 100], [0, 1], [-1, -1]), ([3, 297], [5, 2], [7, -1]), ([0, 10], [3, 4], [6, 6]))),
    # in segments: the longest sequence is another one in every replay, and ends in another segment
    (2, 2300, (([1200, 1100], [0, 1], [-1, -1]), ([100, 2200], [5, 2], [7, -1]), ([2300, 0], [3, 4], [3, 6]), ([0, 700], [2, 6], [-1, 2]))),
])
def test_replays_with_other_lengths(H, T, batches):
    x = scan_inputs([T], H, 1, 128, 64, "bf16", 8, seed=4)
    m, d = layer(8, H, 128, 64), on_device(x)
    _, pr = batch_of(*batches[0])
    out, work = torch.empty(T, H, 64, dtype=BF16, device=DEV), m.new_prompt_work(2, T)
    assert (work is not None) == (T > 1000)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.prompt_scan(pr, *(d[n] for n in ("q", "k", "v", "dt", "a")), out, dt_bias=d["bias"], skip=d["skip"], work=work)
    for lens, slots, resume in batches:
        starts = ref.starts_of(lens)
        for t, v in ((pr.starts, starts), (pr.slots, slots), (pr.resume, resume)):
            t.copy_(torch.tensor(v, dtype=torch.int32))
        m.state.copy_(d["state"])
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        m.check_status()
        held(m, x, out, starts, slots, resume)


@pytest.mark.parametrize("T", [64, 1100])
def test_it_stays_inside_its_arrays_whatever_starts_holds(T):
    """Row numbers that do not ascend or leave the batch are cut to it: some outputs are senseless, none is outside."""
    m, x = layer(4, 2, 128, 64), scan_inputs([T], 2, 1, 128, 64, "bf16", 4)
    d = on_device(x)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    wide = torch.full((T + 32, 2, 64), 7.0, dtype=BF16, device=DEV)
    m.state.copy_(d["state"])
    for starts in (i32(40, 10, T), i32(-5, 1000000, 20), i32(T, T, T), i32(-9, -9, -3)):
        pr = binding.Prompts(starts, T, i32(-7, 1 << 30), i32(1 << 30, -1))
        m.prompt_scan(pr, *(d[n] for n in ("q", "k", "v", "dt", "a")), wide[16:T + 16])
    m.check_status()
    assert (wide[:16] == 7).all() and (wide[T + 16:] == 7).all() and torch.equal(m.state, d["state"])


def test_what_is_not_finite_stays_in_its_sequence_and_head():
    x = scan_inputs([140, 150, 40], 4, 2, 128, 64, "bf16", 8, seed=3)
    x["v"][145, 1, 5] = float("nan")              # sequence 1, head 1
    x["k"][300, 0, 7] = float("inf")              # sequence 2, heads 0 and 1
    x["state"][4, 3, 2, 2] = float("nan")         # sequence 1, head 3
    x["q"][10, 1, 0] = float("nan")               # one token of sequence 0, heads 2 and 3
    starts, pr = batch_of([140, 150, 40], None, [3, 4, 5])
    m = layer(8, 4, 128, 64)
    got = ref.f64(run(m, pr, x))
    want, mag, new, new_mag = ref.scan(starts, None, [3, 4, 5], *(x[n] for n in INPUTS), m.B)
    bad = torch.zeros(330, 4, dtype=torch.bool)
    bad[145:290, 1] = bad[300:330, :2] = bad[140:290, 3] = bad[10, 2:] = True
    good = ~bad[:, :, None].expand_as(want)
    rel = (6 * 150 + 144) * U
    assert ((got - want).abs() - (2.0 ** -8 * want.abs() + (rel + PARTS) * mag))[good].max() <= 0
    assert torch.isnan(got[145:290, 1, 5]).all() and torch.isnan(got[10, 2:]).all() and torch.isnan(got[140:290, 3, 2]).all()
    st, keep = ref.f64(m.state), torch.ones(8, 4, dtype=torch.bool)
    keep[1, 1] = keep[1, 3] = keep[2, :2] = keep[4, 3] = False
    assert ((st - new).abs() - rel * new_mag)[keep].max() <= 0
