"""Microscaled 4-bit operators whose workgroups take more than one launch (tests/test_mx4_launches.py holds these sizes to that), against calls that
take one: a batch of matrices of one row is a matrix of as many rows, its containers the same bytes.  Everything is equal bit for bit."""
import numpy as np
import pytest
import torch

import paper_2105_04246_amd as hq
from test_mx4_launches import DEQUANTIZE, N

pytestmark = pytest.mark.gpu


def needs(gb):
    if torch.cuda.mem_get_info()[0] < gb << 30:
        pytest.skip("needs %d GB of free memory" % gb)


def containers(rows, n, batch=1):
    q, s = hq.new_mx4(rows, n, batch=batch)
    return q.fill_(0xA5), s.fill_(0xA5)


def values(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").mul_(torch.exp2(torch.randint(-9, 9, (shape[0], 1), generator=g, device="cuda").float())).to(dtype)


def same(got, want):
    for g, w in zip(got, want):
        assert torch.equal(g.view(-1), w.view(-1))


def one_matrix(x, seed=None):
    """Along the rows of x, few workgroups."""
    q = containers(*x.shape)
    args = (hq.mx4_type(x.dtype), x, x.shape[0], x.shape[1], 1, None)
    if seed is None:
        hq.hq_mx4_quantize(*args, *q, None, None)
    else:
        hq.hq_mx4_quantize_sr(*args, seed, *q, None, None)
    return q


def test_quantize_along_the_rows():
    needs(8)
    x, q = values((N, 32), torch.bfloat16, 1), containers(1, 32, N)
    hq.hq_mx4_quantize(hq.HQ_BF16, x, 1, 32, N, None, *q, None, None)
    same(q, one_matrix(x))


def test_quantize_along_the_columns():
    needs(8)
    x, q = values((N, 32), torch.bfloat16, 2), containers(1, 32, N)
    hq.hq_mx4_quantize(hq.HQ_BF16, x, 32, 1, N, None, None, None, *q)
    same(q, one_matrix(x))


@pytest.mark.parametrize("seed", [None, 0x123456789ABCDEF])
def test_quantize_both_ways(seed):
    needs(8)
    x, q, qt = values((N, 1), torch.float32, 3), containers(1, 1, N), containers(1, 1, N)
    args = (hq.HQ_FP32, x, 1, 1, N, None)
    if seed is None:
        hq.hq_mx4_quantize(*args, *q, *qt)
    else:
        hq.hq_mx4_quantize_sr(*args, seed, *q, *qt)
    want = one_matrix(x, seed)
    same(q, want)
    same(qt, want)


def test_dequantize():
    needs(8)
    g = torch.Generator(device="cuda").manual_seed(4)
    q = torch.randint(0, 256, (DEQUANTIZE, 1, 128), dtype=torch.uint8, generator=g, device="cuda")
    s = torch.randint(100, 150, (DEQUANTIZE, 1, 8), dtype=torch.uint8, generator=g, device="cuda")
    got, want = (torch.full((DEQUANTIZE, 8), float("nan"), device="cuda") for _ in range(2))
    hq.hq_mx4_dequantize(q, s, 1, 8, DEQUANTIZE, None, hq.HQ_FP32, got)
    hq.hq_mx4_dequantize(q, s, DEQUANTIZE, 8, 1, None, hq.HQ_FP32, want)
    assert torch.equal(got, want) and bool(want.any())


def test_products_by_expert_over_nothing():
    """The row belongs to the last expert, whose last columns lie in the second launch."""
    E, cols = 4096, 1 << 18
    offs = torch.tensor([0] * E + [1], dtype=torch.int32, device="cuda")
    out = torch.full((1, cols), float("nan"), device="cuda")
    hq.hq_mx4_gemm_grouped(hq.mx4_problem(1, cols, 0, E), None, None, None, None, offs, out)
    assert bool((out == 0).all())


def test_weight_gradients_by_expert():
    """Three rows, for the first expert, one in the middle and the last: products of grid values, exact."""
    needs(16)
    E, cols, owners = 4096, (1 << 19) + 64, (0, 2000, 4095)
    rng = np.random.default_rng(5)
    g, x = (torch.from_numpy(rng.choice((1, 2, 3, 4, 6), s) * rng.choice((-1, 1), s)).to("cuda", torch.bfloat16) for s in ((3, 1), (3, cols)))
    o = np.zeros(E + 1, np.int32)
    for e in owners:
        o[e + 1:] += 1
    offs = torch.from_numpy(o).cuda()
    gt, xt = hq.new_mx4(1, 3, E), hq.new_mx4(cols, 3, E)
    hq.hq_mx4_quantize(hq.HQ_BF16, g, 3, 1, E, offs, None, None, *gt)
    hq.hq_mx4_quantize(hq.HQ_BF16, x, 3, cols, E, offs, None, None, *xt)
    p = hq.mx4_problem(1, cols, 3, E, hq.HQ_BF16)
    need = hq.hq_mx4_workspace_bytes(hq.HQ_ENTRY_MX4_WGRAD_GROUPED, p)
    out = torch.full((E, 1, cols), float("nan"), dtype=torch.bfloat16, device="cuda")
    hq.hq_mx4_wgrad_grouped(p, *gt, *xt, offs, out, torch.empty(max(16, need), dtype=torch.uint8, device="cuda"), need)
    for k, e in enumerate(owners):
        assert torch.equal(out[e, 0], g[k] * x[k])
        out[e] = 0
    for part in out.split(256):
        assert bool((part == 0).all())
