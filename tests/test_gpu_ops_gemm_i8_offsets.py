"""Grouped int8 product with offsets that no dispatch writes: experts that claim the same rows many times over."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_11562_b200 import build as B
    B.build()
    from paper_2609_11562_b200 import entwine as E


def _claims(G, M):
    """Every other expert claims all rows, those between none."""
    return torch.tensor([0, M] * (G // 2) + [0], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("M,N,G", [(5000, 600, 64), (300, 40000, 8), (130, 20, 1024), (40, 300, 16)])
def test_rows_claimed_many_times(M, N, G):
    """All experts are alike, so that whichever computes a row gives the same; what lies behind the rows stays."""
    K = 64
    g = torch.Generator(device="cuda").manual_seed(M)
    a = torch.randint(-128, 128, (M, K), generator=g, device="cuda", dtype=torch.int8)
    b = torch.randint(-128, 128, (1, N, K), generator=g, device="cuda", dtype=torch.int8).repeat(G, 1, 1)
    out = torch.full((M + 70, N), -9.0, device="cuda")
    E.gemm_i8_grouped(a, torch.ones(M, device="cuda"), b, torch.ones(G, N, device="cuda"), _claims(G, M), out[:M])
    E.ops_status()
    assert torch.equal(out[:M].double(), a.double() @ b[0].double().T)
    assert bool((out[M:] == -9).all())


def test_claims_whose_tiles_pass_32_bits():
    """512 claims of 2^30 rows are 2^31 tiles of 256 rows.  Only one channel, so that the result is the first column."""
    M, G, K = 1 << 30, 1024, 16
    a = torch.zeros(M, K, dtype=torch.int8, device="cuda")
    a[:, 0].random_(-128, 128)
    b = torch.zeros(G, 1, K, dtype=torch.int8, device="cuda")
    b[:, 0, 0] = 1
    out = torch.full((M, 1), -999.0, dtype=torch.bfloat16, device="cuda")
    E.gemm_i8_grouped(a, torch.ones(M, device="cuda"), b, torch.ones(G, 1, device="cuda"), _claims(G, M), out)
    E.ops_status()
    for r in range(0, M, 1 << 28):
        assert torch.equal(out[r:r + (1 << 28), 0], a[r:r + (1 << 28), 0].to(torch.bfloat16))
    del a, out
    torch.cuda.empty_cache()
