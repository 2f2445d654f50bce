"""The delta rule's scan over numbers of very different size: step sizes, values and states that a chunk's common scale has to hold.  Tolerances are
delta_ref's bound of fp32 arithmetic, and, where the error as a whole is looked at, what the other tests of the operator allow it."""
import pytest
import torch

from tests import delta_ref as dref
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
