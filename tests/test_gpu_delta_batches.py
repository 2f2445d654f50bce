"""Delta scans of batches with many sequences (found by halving, sorted by counting, or left in their order), of the numbers of tokens at which the
path changes, and of two batches at once.  Bounds as for the scan's other tests."""
import random

import pytest
import torch

from tests.test_gpu_delta_operators import DEV, check_scan, layer, run_scan, scan_inputs
from tests.test_gpu_layer_operators import batch_of

pytestmark = pytest.mark.gpu


def lengths_of(n, longest, seed):
    r = random.Random(seed)
    return [r.choice((0, 1, 2, 3, r.randint(0, 7), r.randint(0, longest) if i % 41 == 5 else 1)) for i in range(n)]


@pytest.mark.parametrize("kind,n,longest,H,G,io,od", [("gdn", 33, 200, 3, 1, "bf16", "bf16"), ("gdn", 257, 300, 2, 2, "bf16", "bf16"), ("gdn", 1100, 150, 1, 1, "bf16", "bf16"),
                                                     ("gdn", 65, 90, 2, 1, "bf16", "f32"), ("kda", 64, 80, 2, 2, "bf16", "bf16"), ("kda", 150, 50, 1, 1, "f32", "f32")])
def test_many_sequences(kind, n, longest, H, G, io, od):
    lengths = lengths_of(n, longest, n)
    slots, resume = [-1] * n, [-1 if i % 3 else 5 + i % 3 for i in range(n)]
    for s, i in enumerate((0, n // 2, n - 1, n - 2, 5)):
        slots[i] = s
    starts, pr = batch_of(lengths, slots, resume)
    check_scan(layer(8, H, 128, 128, io, kind), scan_inputs(kind, lengths, H, G, 128, 128, io, 8), starts, pr, slots, resume, od)


@pytest.mark.parametrize("lengths", [[32], [33], [1] * 32, [1] * 33, [0, 31, 0], [30, 0, 3], [2, 2, 2]])
def test_few_tokens_on_either_path(lengths):
    starts, pr = batch_of(lengths, None, [(i + 3) % 40 for i in range(len(lengths))])
    check_scan(layer(40, 4), scan_inputs("gdn", lengths, 4, 2, 128, 128, "bf16", 40), starts, pr, None, [(i + 3) % 40 for i in range(len(lengths))], "bf16")


@pytest.mark.parametrize("kind", ["gdn", "kda"])
def test_two_batches_at_once(kind):
    """Two contexts on two streams, each with its own scratch, one batch in whole sequences and one (GDN) in segments: as one after the other."""
    todo = []
    for lengths, B in (([100, 0, 700] + [9] * 30, 40), ([3200], 3)):
        x = {n: t.to(DEV) for n, t in scan_inputs(kind, lengths, 2, 1, 128, 128, "bf16", B).items()}
        starts, pr = batch_of(lengths, None, None)
        m = layer(B, 2, kind=kind)
        out = torch.empty_like(x["v"])
        m.state.copy_(x["state"])
        run_scan(m, pr, x, out)
        todo.append((m, pr, x, out, m.state.clone(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    again = [torch.full_like(t[3], float("nan")) for t in todo]
    for m, _, x, *_ in todo:
        m.state.copy_(x["state"])
    torch.cuda.synchronize()
    for _ in range(3):
        for (m, pr, x, _, _, stream), out in zip(todo, again):
            m.delta_scan(pr, x["q"], x["k"], x["v"], x["b"], x["dt"], x["a"], out, dt_bias=x["bias"], stream=stream)
    torch.cuda.synchronize()
    for (m, _, _, out, state, _), o in zip(todo, again):
        m.check_status()
        assert torch.equal(o, out) and torch.equal(m.state, state)


def test_a_graph_that_brings_its_own_scratch():
    """Captured without a scratch given, between other captured calls whose scratch the graph's memory may hand out again: replayed twice, as the
    calls one by one."""
    lengths = [[200, 64, 90], [500]]
    m = layer(8, 4)
    xs = [{n: t.to(DEV) for n, t in scan_inputs("gdn", ls, 4, 2, 128, 128, "bf16", 8).items()} for ls in lengths]
    prs = [batch_of(ls, [i + 4 * j for i in range(len(ls))], None)[1] for j, ls in enumerate(lengths)]
    want = [torch.empty_like(x["v"]) for x in xs]
    for pr, x, out in zip(prs, xs, want):
        run_scan(m, pr, x, out)
    state = m.state.clone()
    outs = [torch.empty_like(x["v"]) for x in xs]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for pr, x, out in zip(prs, xs, outs):
            m.delta_scan(pr, x["q"], x["k"], x["v"], x["b"], x["dt"], x["a"], out, dt_bias=x["bias"])
    for _ in range(2):
        m.state.zero_()
        for o in outs:
            o.fill_(float("nan"))
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        assert torch.equal(m.state[[0, 1, 2, 4]], state[[0, 1, 2, 4]])
    m.check_status()


@pytest.mark.parametrize("kind,lengths", [("gdn", [100, 0, 321]), ("gdn", [3500]), ("kda", [70, 33])])
def test_what_the_scratch_holds_before_changes_nothing(kind, lengths):
    """Scratch of zeros, of bytes that are no numbers in any type, and at an address of the smallest alignment: the same to the bit."""
    x = {n: t.to(DEV) for n, t in scan_inputs(kind, lengths, 4, 2, 128, 128, "bf16", 4).items()}
    pr, m = batch_of(lengths, None, None)[1], layer(4, 4, kind=kind)
    need = m.new_delta_work(len(lengths), sum(lengths)).numel()
    got = []
    for fill, at in ((0, 0), (255, 0), (255, 16)):
        work = torch.full((need + 64,), fill, dtype=torch.uint8, device=DEV)
        out = torch.empty_like(x["v"])
        run_scan(m, pr, x, out, work=work[at:at + need])
        got.append((out, m.state.clone()))
        assert (work[:at] == fill).all() and (work[at + need:] == fill).all()
    for out, state in got[1:]:
        assert torch.equal(out, got[0][0]) and torch.equal(state, got[0][1])
