"""Microscaled 4-bit products of scales at both ends of their range."""
import numpy as np
import pytest
import torch

from oracle import mx4
from test_gpu_mx4 import dev, gemm, random_container

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exponent", [0, -134, 60, 100])
@pytest.mark.parametrize("M", [4, 30, 70, 300, 1030])
def test_every_pair_of_scales_whose_product_is_the_same(M, exponent):
    """All blocks' products in units of 2^exponent, from scales as far apart as the format goes: sums of 1024 multiples of a quarter below 36 units have
    18 bits and are exact, those of 2^-134 in fp32's subnormal range (the smallest is 2^-149, a quarter of a unit 2^-136)."""
    N, K, total = 72, 1024, exponent + 254
    rng = np.random.default_rng(M)
    lo, hi = max(0, total - 254), min(254, total)
    blocks = rng.integers(lo, hi + 1, (4, 8))
    blocks[0, :2], blocks[3, 6:] = (lo, hi), (hi, lo)
    A, B = (([t[0] for t in random_container(rng, r, K)][0], np.ascontiguousarray(np.broadcast_to(s[:, None], (4, r, 8)).astype(np.uint8)))
            for r, s in ((M, blocks), (N, total - blocks)))
    want, _ = mx4.product(A, B)
    got = gemm(M, N, K, torch.float32, dev(A), dev(B)).double().cpu().numpy()
    assert np.array_equal(got, want)
