"""Microscaled 4-bit products whose operands lie beyond 4 GB, in the tiles (tests/test_mx4_launches.py holds these sizes to them).  Random codes under scales
of 1: their sums (multiples of a quarter below 2^24 quarters) are exact in fp32 in any order."""
import pytest
import torch

import paper_2105_04246_amd as hq

pytestmark = pytest.mark.gpu


def plain(codes, rows):
    return codes, torch.full((codes.shape[0], rows, 8), 127, dtype=torch.uint8, device="cuda")


def random_codes(seed, *shape):
    return torch.randint(0, 256, shape, dtype=torch.uint8, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def gemm(A, B, M, N, K):
    p = hq.mx4_problem(M, N, K)
    need = hq.hq_mx4_workspace_bytes(hq.HQ_ENTRY_MX4_GEMM, p)
    out = torch.full((M, N), float("nan"), device="cuda")
    hq.hq_mx4_gemm(p, *A, *B, out, torch.empty(max(16, need), dtype=torch.uint8, device="cuda"), need)
    return out


def part(c, start, stop):
    """Chunks start .. stop of a container, copied to where their offsets are small."""
    return tuple(t[start:stop].clone() for t in c)


def needs(gb):
    if torch.cuda.mem_get_info()[0] < gb << 30:
        pytest.skip("needs %d GB of free memory" % gb)


FAR_EXPERTS = [(72, 131072, 8192, 9), (2000, 131072, 8192, 9)]                       # rows, N, K, experts
FAR_WEIGHTS = [(40, 1 << 22, 9 * 256), (300, 1 << 22, 9 * 256)]                      # M, N, K
FAR_GRADIENTS = [(1 << 22, 40, 2560, 2), (1 << 22, 300, 2560, 2)]                    # M, N, rows, experts


@pytest.mark.parametrize("rows,N,K,E", FAR_EXPERTS)
def test_weights_of_the_last_expert_beyond_4_gb(rows, N, K, E):
    needs(16)
    chunks = hq.hq_mx4_chunks(K)
    A, B = plain(random_codes(1, chunks, rows, 128), rows), plain(random_codes(2, E * chunks, N, 128), N)
    assert (E - 1) * chunks * N * 128 >= 1 << 32
    offs = torch.tensor([0] * E + [rows], dtype=torch.int32, device="cuda")
    got = torch.full((rows, N), float("nan"), device="cuda")
    hq.hq_mx4_gemm_grouped(hq.mx4_problem(rows, N, K, E), *A, *B, offs, got)
    want = gemm(A, part(B, (E - 1) * chunks, E * chunks), rows, N, K)
    assert torch.equal(got, want) and bool(want.any())


@pytest.mark.parametrize("M,N,K", FAR_WEIGHTS)
def test_last_chunk_of_a_product_beyond_4_gb(M, N, K):
    """The product is the one over the first eight chunks and the one over the ninth, added."""
    needs(32)
    A, B = plain(random_codes(3, 9, M, 128), M), plain(random_codes(4, 9, N, 128), N)
    assert 8 * N * 128 >= 1 << 32
    got = gemm(A, B, M, N, K)
    want = gemm(part(A, 0, 8), part(B, 0, 8), M, N, 8 * 256) + gemm(part(A, 8, 9), part(B, 8, 9), M, N, 256)
    assert torch.equal(got, want) and bool(want.any())


@pytest.mark.parametrize("M,N,T,E", FAR_GRADIENTS)
def test_rows_of_the_last_expert_beyond_4_gb(M, N, T, E):
    needs(48)
    A, B = plain(random_codes(5, 10, M, 128), M), plain(random_codes(6, 10, N, 128), N)
    offs = torch.tensor([0, 2048, T], dtype=torch.int32, device="cuda")
    p = hq.mx4_problem(M, N, T, E)
    cap = hq.hq_mx4_chunks(T, E)
    A, B = (tuple(torch.cat([t, torch.full_like(t[:cap - 10], 255)]) for t in c) for c in (A, B))
    out = torch.full((E, M, N), float("nan"), device="cuda")
    need = hq.hq_mx4_workspace_bytes(hq.HQ_ENTRY_MX4_WGRAD_GROUPED, p)
    hq.hq_mx4_wgrad_grouped(p, *A, *B, offs, out, torch.empty(max(16, need), dtype=torch.uint8, device="cuda"), need)
    for e, (start, stop) in enumerate(((0, 8), (8, 10))):
        want = gemm(part(A, start, stop), part(B, start, stop), M, N, 256 * (stop - start))
        assert torch.equal(out[e], want) and bool(want.any())
