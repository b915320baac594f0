"""Bounded device-side waits of the int8 products: a block of operands that never comes makes them give up, say so and
leave the GPU usable.  The block is withheld by the host (it is not loaded), under a short budget."""
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_11562_b200 import build as B
    B.build()
    from paper_2609_11562_b200 import entwine as E

BUDGET_NS = 20_000_000


@pytest.fixture
def withheld():
    """Sets the withheld block under a short budget; both are put back afterwards."""
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


def _operands(M, N, K, experts=0):
    """Small values: every sum is exact in fp32 (K * 64 < 2^24)."""
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    pitch = -(-K // 16) * 16
    shape = (experts, N, pitch) if experts else (N, pitch)
    a = torch.randint(-8, 9, (M, pitch), generator=g, device="cuda", dtype=torch.int8)[:, :K]
    b = torch.randint(-8, 9, shape, generator=g, device="cuda", dtype=torch.int8)[..., :K]
    return a, torch.ones(M, device="cuda"), b, torch.ones(shape[:-1], device="cuda")


# M, N, K, withheld block, channels of the first tile.  Narrow tiles: K split over a cluster and not, more blocks than
# the ring has stages and fewer, the first block, a middle one and the last.  Pairs: the same.
NARROW = [(16, 8192, 3584, 0, 128), (16, 8192, 3584, 6, 128), (8, 128, 1024, 0, 128), (64, 1000, 4000, 3, 128), (100, 6000, 200, 1, 128),
          (128, 300, 2100, 3, 128), (30, 19200, 4096, 20, 128)]
PAIRS = [(600, 2560, 1408, 0, 256), (600, 2560, 1408, 10, 256), (600, 2560, 1408, 5, 256), (700, 3000, 200, 0, 256), (700, 3000, 200, 1, 256),
         (500, 4096, 2000, 13, 256)]


@pytest.mark.parametrize("M,N,K,block,first", NARROW + PAIRS)
def test_a_wait_that_runs_out_is_reported(withheld, M, N, K, block, first):
    a, sa, b, sb = _operands(M, N, K)
    want = a.double() @ b.double().T
    out = torch.empty(M, N, device="cuda")
    withheld(block)
    E.gemm_i8(a, sa, b, sb, out)
    with pytest.raises(E.EntwineError) as e:
        E.ops_status()
    assert e.value.code == E.ERR_TIMEOUT
    assert torch.equal(out[:, first:].double(), want[:, first:])    # the tiles that lacked nothing
    withheld.off()
    E.ops_status()
    out.fill_(float("nan"))
    E.gemm_i8(a, sa, b, sb, out)
    E.ops_status()
    assert torch.equal(out.double(), want)


@pytest.mark.parametrize("counts,N,K,block", [([3, 0, 5, 1], 512, 1024, 1), ([64] * 64, 640, 512, 1), ([300, 0, 700], 3000, 1000, 0)])
def test_a_wait_that_runs_out_with_experts(withheld, counts, N, K, block):
    G, M = len(counts), sum(counts)
    a, sa, b, sb = _operands(M, N, K, G)
    off = torch.tensor([0] + counts, device="cuda").cumsum(0).int()
    expert = torch.repeat_interleave(torch.arange(G, device="cuda"), torch.tensor(counts, device="cuda"))
    want = torch.cat([a[expert == g].double() @ b[g].double().T for g in range(G)])
    out = torch.empty(M, N, device="cuda")
    withheld(block)
    E.gemm_i8_grouped(a, sa, b, sb, off, out)
    with pytest.raises(E.EntwineError) as e:
        E.ops_status()
    assert e.value.code == E.ERR_TIMEOUT
    withheld.off()
    E.gemm_i8_grouped(a, sa, b, sb, off, out)
    E.ops_status()
    assert torch.equal(out.double(), want)


def test_a_captured_call_keeps_its_settings(withheld):
    a, sa, b, sb = _operands(40, 500, 700)
    out, side = torch.empty(40, 500, device="cuda"), torch.cuda.Stream()
    withheld(2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        E.gemm_i8(a, sa, b, sb, out)
    withheld.off()
    with torch.cuda.stream(side):
        graph.replay()
    with pytest.raises(E.EntwineError) as e:
        E.ops_status(side)
    assert e.value.code == E.ERR_TIMEOUT
    E.gemm_i8(a, sa, b, sb, out)
    E.ops_status()
    assert torch.equal(out.double(), a.double() @ b.double().T)


def _timed_out(stream=None):
    try:
        E.ops_status(stream)
    except E.EntwineError as e:
        assert e.code == E.ERR_TIMEOUT
        return True
    return False


def test_a_query_takes_no_failure_from_another_thread(withheld):
    """Whoever asks first, on whatever stream, the thread whose product it was is told too."""
    a, sa, b, sb = _operands(16, 1000, 600)
    out, side = torch.empty(16, 1000, device="cuda"), torch.cuda.Stream()
    with ThreadPoolExecutor(1) as other:
        other.submit(_timed_out).result()             # (that thread's first query: what failed before it)
        before, others = E.ops_failed_waits(), other.submit(E.ops_failed_waits).result()
        assert before == others
        withheld(0)
        E.gemm_i8(a, sa, b, sb, out)
        withheld.off()
        torch.cuda.synchronize()
        assert other.submit(_timed_out, side).result()
        assert not other.submit(_timed_out, side).result()
        assert _timed_out()
        assert not _timed_out() and not other.submit(_timed_out).result()
        assert E.ops_failed_waits(side) > before      # and whoever kept the number sees it, whatever was asked between
        now = E.ops_failed_waits()
        E.gemm_i8(a, sa, b, sb, out)
        assert E.ops_failed_waits() == now and torch.equal(out.double(), a.double() @ b.double().T)


def test_status_on_a_capturing_stream_is_refused():
    side, x = torch.cuda.Stream(), torch.zeros(8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        x.add_(1)
        for ask in (E.ops_status, E.ops_failed_waits):
            with pytest.raises(E.EntwineError) as e:
                ask(side)
            assert e.value.code == E.ERR_INVALID
    graph.replay()
    torch.cuda.synchronize()
    assert x[0].item() == 1
