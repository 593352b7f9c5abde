"""Every way in which products in MXFP4 are computed (tests/test_mxfp4_choice.py sees to it that none is left out), with results of every
type, stored and added."""
import pytest
import torch

from paper_2106_10796_amd import binding as B
from test_gpu_mxfp4 import TYPES, check_product, on_gpu, random_mx

pytestmark = pytest.mark.gpu

RINGS = [(1, 130, 300), (16, 8191, 513), (5, 8210, 700), (16, 8193, 2049), (2, 25090, 129),       # one fragment of rows: 8 waves, 4
         (17, 4090, 300), (200, 500, 2050), (17, 4100, 300), (31, 6000, 1153), (32, 8200, 513),   # two: 8 waves, 4
         (33, 4090, 385), (100, 2040, 1025)]                                                      # four
TILES = [(64, 8200, 300), (1030, 700, 513), (65, 4090, 8200), (500, 1020, 16400), (1000, 1030, 16400), (1000, 2050, 16390),
         (513, 8200, 300), (2050, 4100, 300), (4400, 4099, 300), (4400, 4099, 1025), (4352, 4099, 1800), (2100, 9000, 1800),
         (5100, 4130, 1800), (4130, 5100, 1800), (66000, 100, 1801), (75800, 250, 1800)]
WAYS = RINGS + TILES


@pytest.mark.parametrize("M,N,K", WAYS)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_product(M, N, K, dtype, accumulate):
    check_product(M, N, K, dtype, seed=M + K, accumulate=accumulate, ld=N + 7)


@pytest.mark.parametrize("M,N,K", RINGS)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_a_ring_stores_into_any_address(M, N, K, dtype, accumulate):
    (ac, as_), (bc, bs) = random_mx(M, K, 1), random_mx(N, K, 2)
    a, b, ws = on_gpu(ac, as_, M, K), on_gpu(bc, bs, N, K), B.new_mxfp4_workspace([(M, N, K)])
    want = torch.ones(M, N, dtype=TYPES[dtype], device="cuda")
    B.cdsgd_mxfp4_matmul(a, b, want, ws, accumulate=accumulate)
    for offset in range(1, 16 // want.element_size()):
        flat = torch.ones(M * N + 32, dtype=want.dtype, device="cuda")
        out = flat[offset:offset + M * N].view(M, N)
        B.cdsgd_mxfp4_matmul(a, b, out, ws, accumulate=accumulate)
        assert torch.equal(out, want)
        assert bool((flat[:offset] == 1).all()) and bool((flat[offset + M * N:] == 1).all())
