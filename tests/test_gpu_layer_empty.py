"""The operators around the recurrence without rows, tokens or sequences: nothing to do, and no refusal."""
import pytest
import torch

from paper_2609_33051_b200 import binding, layer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def empty(*size, dtype=torch.bfloat16):
    return torch.empty(*size, dtype=dtype, device=DEV)


@pytest.mark.parametrize("mode", ["plain", "residual", "gate", "skip"])
@pytest.mark.parametrize("outputs", ["both", "io", "8 bits"])
def test_norm_of_no_rows(mode, outputs):
    m = binding.SketchSSM("mamba2", 2, 4, 128, 64, 8, 4, io="bf16", device=0)
    kw = {}
    if mode == "residual":
        kw = dict(residual=empty(0, 256), residual_out=empty(0, 256))
    if mode in ("gate", "skip"):
        kw = dict(gate=empty(0, 256))
    if mode == "skip":
        kw.update(skip=empty(0, 512)[:, 256:], skip_weight=torch.ones(4, device=DEV))
    if outputs != "8 bits":
        kw["out"] = empty(0, 256)
    if outputs != "io":
        kw.update(out8=empty(0, 256, dtype=torch.float8_e4m3fn), scale=empty(0, 2, dtype=torch.float32))
    m.rms_norm(empty(0, 256), torch.ones(256, device=DEV), **kw)
    assert m.last_launch_count() == 0
    m.check_status()


def test_norm_of_no_rows_still_wants_an_output():
    m = binding.SketchSSM("mamba2", 2, 4, 128, 64, 8, 4, io="bf16", device=0)
    x, w = empty(0, 256), torch.ones(256, device=DEV)
    for kw in ({}, dict(out=x, residual=x), dict(out8=empty(0, 256, dtype=torch.float8_e4m3fn)), dict(out=x, skip=x, gate=x)):
        with pytest.raises(binding.SketchSSMError):
            m.rms_norm(x, w, **kw)


def test_a_layer_over_prompts_without_tokens():
    """Sequences of no tokens, and no sequences: states and stored rows of the sequences' slots start from zeros, others stay."""
    gen = torch.Generator().manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    H, G, K, V, width = 4, 1, 128, 64, 256
    C = H * V + 2 * G * K
    lay = layer.Mamba2Layer(3, H, K, V, G, 8, 4, norm=torch.ones(width), w_in=rand(2 * H * V + 2 * G * K + H, width), conv_weight=rand(C, 4),
                            conv_bias=rand(C), a=-torch.exp(rand(H)), dt_bias=rand(H), skip=rand(H), gate_norm=torch.ones(H * V), w_out=rand(width, H * V))
    lay.m.state.fill_(3.0), lay.conv_state.fill_(2.0)
    pr = binding.Prompts(torch.zeros(3, dtype=torch.int32, device=DEV), 0, slots=torch.tensor([2, 0], dtype=torch.int32, device=DEV))
    assert lay.prompt(pr, empty(0, width), empty(0, width)).shape == (0, width)
    for t, old in ((lay.m.state, 3.0), (lay.conv_state, 2.0)):
        assert (t[0] == 0).all() and (t[1] == old).all() and (t[2] == 0).all()
    none = binding.Prompts(torch.zeros(1, dtype=torch.int32, device=DEV), 0)
    assert lay.prompt(none, empty(0, width)).shape == (0, width)
    assert (lay.m.state[1] == 3).all()
    lay.m.check_status()
