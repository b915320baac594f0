"""The operators around the ReduceScatter together, as a block uses them: the reduced shard through dropout, residual and
layer norm (one call), to 4 bits, through the product and the next ReduceScatter; and the gradients of the training part."""
import numpy as np
import pytest
import torch

import mxf4_reference as R4
import philox_reference as RP

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_11562_b200 import build as B
    B.build()
    from paper_2609_11562_b200 import entwine as E


def test_shard_to_norm_to_four_bits_to_the_next_reduce_scatter():
    W, R, H, N = 4, 512, 1024, 512  # ranks, rows of a shard, hidden size, output size of the next product
    M = W * R
    g = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    partial, peers = rand(M, H).bfloat16(), rand(W - 1, M, H).bfloat16()
    plan = E.Plan(M, H, 256, W, E.ORDER_INTERLEAVED, 0, rank=1)
    shard, send = torch.empty(R, H, dtype=torch.bfloat16, device="cuda"), torch.empty(W - 1, R, H, dtype=torch.bfloat16, device="cuda")
    plan.comm_only(partial, peers, shard, send)
    # dropout + residual + norm of rank 1's rows
    residual, weight, bias, rng = rand(R, H).bfloat16(), 1 + 0.1 * rand(H), rand(H), torch.tensor([5, 6], device="cuda")
    hidden, normed = torch.empty_like(shard), torch.empty_like(shard)
    E.layer_norm(shard, weight, bias, normed, residual=residual, hidden=hidden, p=0.1, rng=rng, row0=R)
    # four bits, the product with a weight of N channels, its ReduceScatter
    x, sx = (torch.empty(R, n, dtype=torch.uint8, device="cuda") for n in (H // 2, H // 32))
    w, sw = (torch.empty(N, n, dtype=torch.uint8, device="cuda") for n in (H // 2, H // 32))
    E.quant_mxf4(normed, x, sx)
    E.quant_mxf4(rand(N, H) / 32, w, sw)
    out = torch.empty(R, N, dtype=torch.bfloat16, device="cuda")
    E.gemm_mxf4(x, sx, w, sw, out)
    peers2 = rand(W - 1, R, N).bfloat16()
    plan2 = E.Plan(R, N, 256, W, E.ORDER_INTERLEAVED, 0, rank=1)
    shard2, send2 = torch.empty(R // W, N, dtype=torch.bfloat16, device="cuda"), torch.empty(W - 1, R // W, N, dtype=torch.bfloat16, device="cuda")
    plan2.comm_only(out, peers2, shard2, send2)
    plan.last_status()
    plan2.last_status()
    E.ops_status()
    # each step from the step before, in 64 bits
    reduced = partial.double()[R:2 * R] + peers.double()[:, R:2 * R].sum(0)
    assert float((shard.double() - reduced).abs().max()) <= 2.0 ** -8 * float(reduced.abs().max())
    h = residual.double() + shard.double() * torch.from_numpy(RP.factors(0.1, 5, 6, R, R, H)).cuda()
    assert bool(((hidden.double() - h).abs() <= 2.0 ** -8 * h.abs() + 1e-5).all())
    h = hidden.double()
    y = (h - h.mean(1, keepdim=True)) / torch.sqrt(h.var(1, correction=0, keepdim=True) + 1e-5) * weight.double() + bias.double()
    assert bool(((normed.double() - y).abs() <= 2.0 ** -8 * y.abs() + 1e-4).all())
    q, s = R4.encode(normed.double().cpu().numpy())
    assert np.array_equal(x.cpu().numpy(), q) and np.array_equal(sx.cpu().numpy(), s)
    u, v = (torch.from_numpy(R4.decode(a.cpu().numpy(), b.cpu().numpy(), H)).cuda() for a, b in ((x, sx), (w, sw)))
    ref = u @ v.T
    size = (H + 1) * 2.0 ** -23 * (u.abs() @ v.abs().T)
    assert bool(((out.double() - ref).abs() <= size + 2.0 ** -8 * (ref.abs() + size)).all())
    r2 = R // W
    reduced = out.double()[r2:2 * r2] + peers2.double()[:, r2:2 * r2].sum(0)
    assert float((shard2.double() - reduced).abs().max()) <= 2.0 ** -8 * float(reduced.abs().max())


def test_training_step_of_two_shards_is_that_of_the_whole():
    """Two ranks' halves of the rows, each with its row0, against one call on all of them; the weight's gradients add up."""
    M, H, p = 512, 2048, 0.15
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    x, residual, dout, down = (rand(M, H) for _ in range(4))
    weight, bias, rng = 1 + 0.1 * rand(H), rand(H), torch.tensor([7, 8], device="cuda")

    def step(rows, row0):
        n = rows.stop - rows.start
        hidden, y, dx, dres = (torch.empty(n, H, dtype=torch.bfloat16, device="cuda") for _ in range(4))
        mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        dw, db = torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
        E.layer_norm(x[rows], weight, bias, y, mean=mean, rstd=rstd, residual=residual[rows], hidden=hidden, p=p, rng=rng, row0=row0)
        E.layer_norm_bwd(dout[rows], hidden, weight, mean, rstd, dx, dw, db, torch.empty(E.layer_norm_bwd_work(n, H), device="cuda"),
                         dhidden=down[rows], dresidual=dres, p=p, rng=rng, row0=row0)
        return (y, hidden, dx, dres), (dw, db)

    whole, sums = step(slice(0, M), 100)
    halves = [step(slice(a, a + M // 2), 100 + a) for a in (0, M // 2)]
    half = 2.0 ** -7  # two roundings to bf16 of values that are 2^-20 apart
    for i, t in enumerate(whole):
        parts = torch.cat([halves[0][0][i], halves[1][0][i]])
        assert bool(((t.double() - parts.double()).abs() <= half * t.double().abs() + 1e-4).all())
    for i, t in enumerate(sums):
        n = (halves[0][1][i] + halves[1][1][i]).double()
        assert bool(((t.double() - n).abs() <= M * 2.0 ** -22 * (8 * dout.double().abs().sum(0))).all())


def test_expert_layer_in_four_bits():
    """Tokens quantised, sorted by expert with their scales, multiplied with their experts' matrices, returned with weights."""
    T, k, G, H, N = 200, 3, 12, 512, 384
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(T, H, generator=g, device="cuda").bfloat16()
    ids = torch.rand(T, G, generator=g, device="cuda").topk(k, dim=1).indices.int()
    ids[3, 1] = -1
    weights = torch.rand(T, k, generator=g, device="cuda")
    q, s = (torch.empty(T, n, dtype=torch.uint8, device="cuda") for n in (H // 2, H // 32))
    E.quant_mxf4(x, q, s)
    b, sb = (torch.empty(G * N, n, dtype=torch.uint8, device="cuda") for n in (H // 2, H // 32))
    E.quant_mxf4(torch.randn(G * N, H, generator=g, device="cuda") / 22, b, sb)
    rows, row_scale = (torch.zeros(T * k, n, dtype=torch.uint8, device="cuda") for n in (H // 2, H // 32))
    offsets, row_of = torch.empty(G + 1, dtype=torch.int32, device="cuda"), torch.empty(T, k, dtype=torch.int32, device="cuda")
    i8 = torch.int8  # the dispatch moves bytes
    E.moe_dispatch(q.view(i8), ids, G, rows.view(i8), offsets, row_of)
    E.moe_dispatch(s.view(i8), ids, G, row_scale.view(i8), offsets, row_of)
    y = torch.zeros(T * k, N, dtype=torch.bfloat16, device="cuda")
    E.gemm_mxf4_grouped(rows, row_scale, b.unflatten(0, (G, N)), sb.unflatten(0, (G, N)), offsets, y)
    out = torch.empty(T, N, dtype=torch.bfloat16, device="cuda")
    E.moe_combine(y, weights, row_of, out)
    E.ops_status()
    u = torch.from_numpy(R4.decode(q.cpu().numpy(), s.cpu().numpy(), H)).cuda()
    v = torch.from_numpy(R4.decode(b.cpu().numpy(), sb.cpu().numpy(), H)).cuda().unflatten(0, (G, N))
    ref, size = torch.zeros(T, N, dtype=torch.float64, device="cuda"), torch.zeros(T, N, dtype=torch.float64, device="cuda")
    for e in range(G):
        for j in range(k):
            t = (ids[:, j] == e).nonzero()[:, 0]
            one = weights[t, j, None].double() * (u[t] @ v[e].T)
            ref[t] += one
            size[t] += one.abs() + 0.01
    # y rounded to bf16, the weighted sum rounded to bf16
    assert bool(((out.double() - ref).abs() <= 2.0 ** -7 * size).all())
