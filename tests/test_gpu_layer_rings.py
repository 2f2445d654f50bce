"""Sizes that bring the kernels' buffers round and give a CTA more than one tile, for every width of tile: the tolerances are those of the
tests of the same operators."""
import pytest
import torch

from tests import layer_ref as ref
from tests.test_gpu_layer_operators import DEV, TYPE, U, batch_of, layer, quantised, scan_inputs

pytestmark = pytest.mark.gpu

# rows, columns, inner.  A CTA has its share of the inner axis' blocks of 128 for each of its tiles; the buffers hold 4 to 8 blocks.
MATMUL = [
    (7, 9600, 2048), (20, 9600, 2048), (64, 9600, 2048), (100, 9600, 2048),          # 16 blocks a CTA
    (3, 38016, 272), (20, 38016, 272), (64, 19100, 656), (100, 19100, 1152),         # a second tile
    (16, 2048, 8192), (30, 2048, 8192), (50, 2048, 8192),                            # clusters of eight with 8 blocks each
    (256, 2048, 4096), (200, 1000, 7000),                                            # clusters of four and more, 128 columns
    (64, 4096, 2304), (64, 8512, 4096),                                              # clusters of two
    (4099, 2500, 2320),                                                              # pairs of SMs: three tiles, 19 blocks
]


@pytest.mark.parametrize("M,N,K", MATMUL)
@pytest.mark.parametrize("od", ["bf16", "f32"])
def test_matmul(M, N, K, od):
    K = K // 16 * 16
    gen = torch.Generator().manual_seed(M + N + K)
    (a, sa), (w, sw) = quantised(gen, M, K, 1), quantised(gen, N, K, 128)
    m, out = layer(1), torch.empty(M, N, dtype=TYPE[od], device=DEV)
    m.scaled_matmul(a.to(DEV), sa.to(DEV), w.to(DEV), sw.to(DEV), out)
    m.check_status()
    want, mag = ref.matmul(a, sa, w, sw)
    ref.close(out, want, ref.half_step(TYPE[od]) * want.abs() + K * 2.0 ** -23 * mag, "out")


# sequences, heads, K, V, io, out: heads times sequences decide how many value columns a CTA takes
@pytest.mark.parametrize("N,H,K,V,io,od", [
    (40, 16, 64, 64, "bf16", "bf16"), (40, 16, 128, 64, "f32", "f32"), (20, 16, 64, 64, "f32", "f32"), (20, 16, 128, 64, "bf16", "f32"),
    (25, 24, 128, 80, "bf16", "bf16"), (25, 24, 128, 80, "f32", "f32"), (13, 24, 128, 80, "bf16", "f32"),
    (40, 16, 128, 128, "bf16", "f32"), (20, 16, 128, 128, "f32", "f32"), (10, 16, 128, 128, "bf16", "f32"), (60, 10, 128, 128, "f32", "bf16"),
])
def test_scan_on_cuda_cores(N, H, K, V, io, od):
    lengths = [(7 * i) % 41 for i in range(N)]
    starts, pr = batch_of(lengths, list(range(N)), [i if i % 3 else -1 for i in range(N)])
    resume = [i if i % 3 else -1 for i in range(N)]
    x = scan_inputs(lengths, H, 2, K, V, io, N, seed=2)
    m, d = layer(N, H, K, V, io), {n: t.to(DEV) for n, t in x.items()}
    m.state.copy_(d["state"])
    out = torch.empty(starts[-1], H, V, dtype=TYPE[od], device=DEV)
    m.prompt_scan(pr, *(d[n] for n in ("q", "k", "v", "dt", "a")), out, dt_bias=d["bias"], skip=d["skip"])
    want, mag, new, new_mag = ref.scan(starts, list(range(N)), resume, *(x[n] for n in ("q", "k", "v", "dt", "a", "bias", "skip", "state")), N)
    rel = (6 * 40 + K + 16) * U
    ref.close(out, want, ref.half_step(TYPE[od]) * want.abs() + rel * mag, "out")
    ref.close(m.state, new, rel * new_mag, "state")


@pytest.mark.parametrize("M,N,K", [(256, 9472, 272), (256, 9473, 272), (257, 9472, 144), (1153, 2176, 272), (1100, 2100, 1040), (300, 11264, 400)])
def test_matmul_around_a_tile_for_every_sm(M, N, K):
    """As many tiles of 128 x 128 as the card has SMs, a few more and half as many again: where one kernel hands over to the other."""
    gen = torch.Generator().manual_seed(M + N)
    (a, sa), (w, sw) = quantised(gen, M, K, 1), quantised(gen, N, K, 128)
    m, out = layer(1), torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    m.scaled_matmul(a.to(DEV), sa.to(DEV), w.to(DEV), sw.to(DEV), out)
    m.check_status()
    want, mag = ref.matmul(a, sa, w, sw)
    ref.close(out, want, 2.0 ** -8 * want.abs() + K * 2.0 ** -23 * mag, "out")
