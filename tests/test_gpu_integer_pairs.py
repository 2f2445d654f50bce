"""Products of 8-bit integers at the sizes where pairs of SMs take tiles of 256 x 128, and at those just beside.  Bound as for the product's other
tests: exact sums, one conversion and two products, 3 u, and one rounding."""
import pytest
import torch

from tests import layer_ref as ref
from tests.test_gpu_delta_operators import DEV, TYPE, U, integers, layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K,od,pad", [(129, 9472, 208, "bf16", 8), (129, 4737, 208, "bf16", 7), (300, 4096, 2048, "f32", 0), (300, 6144, 272, "bf16", 0),
                                          (640, 2048, 400, "bf16", 16), (256, 9408, 1040, "f32", 4), (256, 9412, 1040, "f32", 1), (777, 1984, 80, "bf16", 0),
                                          (257, 3968, 16, "f32", 0), (1280, 1792, 1168, "bf16", 0), (2304, 1024, 128, "f32", 0), (384, 3136, 8192, "bf16", 0)])
def test_middling_products(M, N, K, od, pad):
    gen = torch.Generator().manual_seed(M + N + K)
    (a, sa), (w, sw) = integers(gen, M, K), integers(gen, N, K)
    m = layer(1)
    wide = torch.full((M, N + pad), 7.0, dtype=TYPE[od], device=DEV)
    m.integer_matmul(a.to(DEV), sa.to(DEV), w.to(DEV), sw.to(DEV), wide[:, :N])
    m.check_status()
    want = (a.double() @ w.double().T) * sa.double()[:, None] * sw.double()
    ref.close(wide[:, :N], want, (ref.half_step(TYPE[od]) + 3 * U) * want.abs(), "out")
    assert (wide[:, N:] == 7).all()
