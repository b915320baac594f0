"""Bounded device-side waits of the 4-bit products: a block of codes that never comes makes them give up, say so and leave the
GPU usable.  The block is withheld by the host (it is not loaded), under a short budget."""
import pytest
import torch

import mxf4_reference as R

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_11562_b200 import build as B
    B.build()
    from paper_2609_11562_b200 import entwine as E

BUDGET_NS = 20_000_000


@pytest.fixture
def withheld():
    def withhold(block):
        E.ops_set_option(E.OPS_OPT_WAIT_BUDGET_NS, BUDGET_NS)
        E.ops_set_option(E.OPS_OPT_WITHHOLD_BLOCK, block)

    def restore():
        E.ops_set_option(E.OPS_OPT_WAIT_BUDGET_NS, 2_000_000_000)
        E.ops_set_option(E.OPS_OPT_WITHHOLD_BLOCK, -1)
    E.ops_status()
    withhold.off = restore
    yield withhold
    restore()
    torch.cuda.synchronize()


def _operand(rows, K, seed):
    """Scales 1: sums of multiples of 1/4 below 36 K, exact in fp32."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randint(0, 256, (rows, -(-K // 32) * 16), generator=g, device="cuda", dtype=torch.uint8)[:, :K // 2]
    return q, torch.full((rows, -(-K // 128) * 4), 127, device="cuda", dtype=torch.uint8)[:, :-(-K // 32)]


def _wide(q, s, K):
    return torch.from_numpy(R.decode(q.cpu().numpy(), s.cpu().numpy(), K)).cuda()


# M, N, K, withheld block of 256, channels of the first tile.  Narrow tiles, K split over a cluster and not, more blocks than the
# ring has stages and fewer; pairs, a tile for each, the same.
CASES = [(16, 8192, 3584, 0, 128), (16, 8192, 3584, 2, 128), (8, 128, 2048, 0, 128), (64, 1000, 6000, 2, 128), (60, 2560, 200, 0, 128),
         (128, 300, 4200, 1, 128), (30, 4000, 16000, 6, 128),
         (600, 2560, 2816, 0, 256), (600, 2560, 2816, 10, 256), (600, 2560, 2816, 5, 256), (400, 3000, 200, 0, 256), (400, 3000, 400, 1, 256),
         (192, 16384, 4000, 15, 256)]


@pytest.mark.parametrize("M,N,K,block,first", CASES)
def test_a_wait_that_runs_out_is_reported(withheld, M, N, K, block, first):
    a, sa = _operand(M, K, 1)
    b, sb = _operand(N, K, 2)
    want = _wide(a, sa, K) @ _wide(b, sb, K).T
    out = torch.empty(M, N, device="cuda")
    withheld(block)
    E.gemm_mxf4(a, sa, b, sb, out)
    with pytest.raises(E.EntwineError) as e:
        E.ops_status()
    assert e.value.code == E.ERR_TIMEOUT
    assert torch.equal(out[:, first:].double(), want[:, first:])    # the tiles that lacked nothing
    withheld.off()
    E.ops_status()
    out.fill_(float("nan"))
    E.gemm_mxf4(a, sa, b, sb, out)
    E.ops_status()
    assert torch.equal(out.double(), want)


@pytest.mark.parametrize("counts,N,K,block", [([3, 0, 5, 1], 512, 1024, 1), ([64] * 16, 640, 1024, 1), ([300, 0, 700], 1000, 2000, 0)])
def test_a_wait_that_runs_out_with_experts(withheld, counts, N, K, block):
    G, M = len(counts), sum(counts)
    a, sa = _operand(M, K, 3)
    b, sb = _operand(G * N, K, 4)
    b, sb = b.unflatten(0, (G, N)), sb.unflatten(0, (G, N))
    off = torch.tensor([0] + counts, device="cuda").cumsum(0).int()
    expert = torch.repeat_interleave(torch.arange(G, device="cuda"), torch.tensor(counts, device="cuda"))
    want = torch.cat([_wide(a[expert == g], sa[expert == g], K) @ _wide(b[g], sb[g], K).T for g in range(G)])
    out = torch.empty(M, N, device="cuda")
    withheld(block)
    E.gemm_mxf4_grouped(a, sa, b, sb, off, out)
    with pytest.raises(E.EntwineError) as e:
        E.ops_status()
    assert e.value.code == E.ERR_TIMEOUT
    withheld.off()
    E.gemm_mxf4_grouped(a, sa, b, sb, off, out)
    E.ops_status()
    assert torch.equal(out.double(), want)


def test_both_products_failures_are_counted_together(withheld):
    K = 512
    a, sa = _operand(16, K, 5)
    out = torch.empty(16, 16, device="cuda")
    i, one = torch.ones(16, 64, dtype=torch.int8, device="cuda"), torch.ones(16, device="cuda")
    before = E.ops_failed_waits()
    withheld(0)
    E.gemm_mxf4(a, sa, a, sa, out)
    after_one = E.ops_failed_waits()
    E.gemm_i8(i, one, i, one, out)
    withheld.off()
    assert before < after_one < E.ops_failed_waits()
    with pytest.raises(E.EntwineError):  # (this thread is told once, so that later queries start anew)
        E.ops_status()
    E.ops_status()
