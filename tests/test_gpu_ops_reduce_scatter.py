"""The int8 product as the first half of the ReduceScatter: quantise, multiply, and let the library's consumer reduce and
scatter the partial output, as entwine_gemm_rs does with its own bf16 product."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_11562_b200 import build as B
    B.build()
    from paper_2609_11562_b200 import entwine as E


@pytest.mark.parametrize("M,N,K,W,rank", [(1024, 512, 384, 4, 1), (2048, 768, 1000, 8, 7)])
def test_int8_partial_output_reduced_and_scattered(M, N, K, W, rank):
    g, R = torch.Generator(device="cuda").manual_seed(M), M // W
    x = torch.randn(M, K, generator=g, device="cuda").to(torch.bfloat16)
    weight = torch.randn(N, K, generator=g, device="cuda") / K ** 0.5
    peers = torch.randn(W - 1, M, N, generator=g, device="cuda").to(torch.bfloat16)
    pitch = -(-K // 16) * 16
    xq, wq = (torch.zeros(n, pitch, dtype=torch.int8, device="cuda")[:, :K] for n in (M, N))
    xs, ws = torch.empty(M, device="cuda"), torch.empty(N, device="cuda")
    partial = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    out, send = torch.empty(R, N, dtype=torch.bfloat16, device="cuda"), torch.empty(W - 1, R, N, dtype=torch.bfloat16, device="cuda")
    plan = E.Plan(M, N, pitch // 64 * 64 + 64, W, E.ORDER_INTERLEAVED, 4, rank=rank)   # (the consumer reads no operand)
    E.quant_i8(weight, wq, ws)
    E.quant_i8(x, xq, xs)
    E.gemm_i8(xq, xs, wq, ws, partial)
    plan.comm_only(partial, peers, out, send)
    assert plan.last_status()["code"] == E.OK
    E.ops_status()
    ref = (xq.double() @ wq.double().T) * xs.double()[:, None] * ws.double()
    assert bool(((partial.double() - ref).abs() <= 3 * 2.0 ** -24 * ref.abs() * 1.01 + 2.0 ** -8 * ref.abs()).all())
    others = [d for d in range(W) if d != rank]
    for q, d in enumerate(others):
        assert torch.equal(send[q], partial[d * R:(d + 1) * R])
    mine = slice(rank * R, (rank + 1) * R)
    terms = torch.cat([peers[:, mine].double(), partial[None, mine].double()])
    # W - 1 additions in fp32 and one rounding to bf16
    tol = (W - 1) * 2.0 ** -24 * terms.abs().sum(0) * 1.01 + 2.0 ** -8 * terms.sum(0).abs()
    assert bool(((out.double() - terms.sum(0)).abs() <= tol).all())
    plan.destroy()
