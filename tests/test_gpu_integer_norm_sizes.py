"""The norm with rows of 8-bit integers at the ends of what it takes."""
import pytest
import torch

from paper_2609_33051_b200 import binding
from tests import delta_ref as dref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_as_many_rows_as_an_int_holds():
    """2^31 - 1 rows, four of which a CTA takes: the number of CTAs is not to be had in 32 bits with a sign."""
    rows = 2 ** 31 - 1
    if torch.cuda.mem_get_info(0)[0] < 70 << 30:
        pytest.skip("64 GB of device memory are not free")
    m = binding.SketchSSM("gdn", 1, 1, 64, 64, 8, 4, io="bf16", device=0)
    gen = torch.Generator().manual_seed(1)
    some, w = torch.randn(5, 8, generator=gen).to(torch.bfloat16), torch.rand(8, generator=gen) + 0.5
    x = torch.zeros(rows, 8, dtype=torch.bfloat16, device=DEV)
    x[-5:] = some.to(DEV)
    out8, scale = torch.empty(rows, 8, dtype=torch.int8, device=DEV), torch.empty(rows, device=DEV)
    m.integer_norm(x, w.to(DEV), out8, scale)
    m.check_status()
    _, want = dref.norm8(some, w, 1e-5)
    top = want.abs().amax(1)
    assert ((scale[-5:].cpu().double() - top / 127).abs() <= 1e-5 * top / 127).all()
    s = scale[-5:].cpu().double()[:, None]
    assert ((out8[-5:].cpu().double() * s - want).abs() <= 0.5 * s + 1.2e-5 * want.abs()).all()
    assert int(out8[:1000].abs().amax()) == 0 and float(scale[:1000].amax()) == 0.0
    del x, out8, scale
    torch.cuda.empty_cache()
