"""The operators where their loops turn more than once and where their launch shapes change: many assignments a token, long
rows, many tokens, few tokens of long rows, a vocabulary's channels, far more experts than rows."""
import numpy as np
import pytest
import torch

from test_gpu_ops_gemm_i8 import _check, _grouped, _levels, _scales
from test_gpu_ops_rows import FLOATING, TINY, _check_dispatch, _dispatch, _half_step, _ids, _laid_out, _name, _rand, _sort_ref

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_11562_b200 import entwine as E


# more assignments than are placed together (eight), in the single launch and behind the sort
@pytest.mark.parametrize("T,k,n_experts,H", [(20, 17, 33, 520), (100, 9, 16, 40), (1, 2048, 1024, 24), (300, 9, 64, 264), (600, 17, 20, 136)])
def test_dispatch_of_many_assignments(T, k, n_experts, H):
    for i, dtype in enumerate((torch.bfloat16, torch.float32, torch.int8)):
        ids = _ids(T, k, n_experts, T + i).to((torch.int64, torch.int32)[i % 2])
        x = _rand((T, H), dtype, i)
        scale = torch.rand(T).cuda() if dtype == torch.int8 else None
        for pitch, shift in ((H, 0), (H + 3, 1)):
            _check_dispatch(x, ids, n_experts, _dispatch(_laid_out(x, pitch, shift), ids.cuda(), n_experts, scale), scale)


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.int8), ids=_name)
@pytest.mark.parametrize("T,H", [(40, 8195), (1100, 5120), (700, 20000)])
def test_dispatch_of_long_rows(T, H, dtype):
    ids, x = _ids(T, 3, 12, T), _rand((T, H), dtype, 5)
    scale = torch.rand(T).cuda()
    for pitch, shift in ((-(-H // 16) * 16, 0), (H, 3)):
        _check_dispatch(x, ids, 12, _dispatch(_laid_out(x, pitch, shift), ids.cuda(), 12, scale), scale)


# a CTA a token (1024 tokens and more) and a row over several CTAs; one turn over a row and several; one, two, four and
# nine assignments
@pytest.mark.parametrize("dtype", FLOATING, ids=_name)
@pytest.mark.parametrize("k", [1, 2, 4, 9])
@pytest.mark.parametrize("T,H", [(1100, 4096), (1100, 5123), (16, 8195), (1030, 1000), (3, 40000)])
def test_return_and_gradients_of_long_rows(T, H, k, dtype):
    n_experts, u, tiny = 20, 2.0 ** -24, TINY[dtype]
    ids = _ids(T, k, n_experts, T + k)
    _, rr = _sort_ref(ids, n_experts)
    row_of = torch.from_numpy(rr).cuda()
    there, at = row_of >= 0, row_of.clamp(min=0).long()
    y, g = _rand((T * k, H), dtype, 1).cuda(), _rand((T, H), dtype, 2).cuda()
    y[int(there.sum()):] = float("nan")                    # rows that nobody owns
    w = torch.rand(T, k, generator=torch.Generator().manual_seed(3)).cuda() - 0.2
    w[~there] = float("nan")
    w64, g64 = torch.where(there, w, 0).double(), g.double()
    y64 = [torch.where(there[:, j, None], y[at[:, j]], 0).double() for j in range(k)]

    def close(got, ref, mag):
        """k fused multiply-adds in fp32, each off by at most u times a partial sum of magnitudes, and one rounding."""
        assert bool(torch.isfinite(got).all())
        assert bool(((got.double() - ref).abs() <= (k + 1) * u * mag * (1 + 2.0 ** -7) + _half_step(dtype) * ref.abs() + tiny).all())

    for pitch, shift in ((-(-H // 8) * 8, 0), (H + 3, 1)):
        yd, gd = _laid_out(y, pitch, shift, fill=float("nan")), _laid_out(g, pitch, shift, fill=float("nan"))
        new = lambda n: _laid_out(torch.full((n, H), 9.0, dtype=dtype), pitch, shift)  # noqa: E731
        out, dx, dy, dw = new(T), new(T), new(T * k), torch.full((T, k), 9.0, device="cuda")
        E.moe_combine(yd, w, row_of, out)
        close(out, sum(y64[j] * w64[:, j, None] for j in range(k)), sum(y64[j].abs() * w64[:, j, None].abs() for j in range(k)))
        E.moe_dispatch_bwd(yd, row_of, dx)
        close(dx, sum(y64), sum(v.abs() for v in y64))
        E.moe_combine_bwd(gd, yd, w, row_of, dy, dw)
        want = torch.full((T * k, H), 9.0, dtype=torch.float64, device="cuda")
        for j in range(k):
            t = there[:, j].nonzero()[:, 0]
            want[at[t, j]] = w64[t, j, None] * g64[t]
            # H additions in any order
            assert bool(((dw[:, j].double() - (g64 * y64[j]).sum(1)).abs() <= H * u * (g64 * y64[j]).abs().sum(1) * (1 + 2.0 ** -7)).all())
        # the fp32 product, then the rounding of the type
        assert bool(((dy.double() - want).abs() <= (u + _half_step(dtype)) * (1 + 2.0 ** -7) * want.abs() + tiny).all())
        assert not bool(dw[~there].any())


# few tokens through a vocabulary: one matrix whose channels alone fill every pair twice
@pytest.mark.parametrize("dtype", FLOATING, ids=_name)
@pytest.mark.parametrize("M,N,K", [(1, 37900, 48), (16, 37889, 520), (33, 40000, 264), (97, 38000, 136), (128, 37900, 1000)])
def test_gemm_i8_few_tokens_many_channels(M, N, K, dtype):
    a, b, sa, sb = _levels(M, K, 1), _levels(N, K, 2), _scales(M, 3), _scales(N, 4)
    for bias, extra in ((None, 0), (torch.randn(N, device="cuda"), 5)):
        store = torch.full((M + 1, N + extra), -9.0, dtype=dtype, device="cuda")
        out = store[:M, :N]
        E.gemm_i8(a, sa, b, sb, out, bias=bias)
        _check(out, a, sa, b, sb, bias)
        assert bool((store[:, N:] == -9).all()) and bool((store[M:] == -9).all())
    E.ops_status()


# far more experts than rows, and few rows at a length that is split
@pytest.mark.parametrize("counts,N,K", [([1] * 8 + [0] * 120, 1024, 4096), ([0] * 127 + [3], 256, 2048), ([0, 2] * 30 + [0] * 900, 128, 700),
                                        ([1, 0, 0, 1], 130, 8192)])
def test_grouped_far_more_experts_than_rows(counts, N, K):
    for dtype in (torch.bfloat16, torch.float32):
        _grouped(counts, N, K, dtype, False, 0)
        _grouped(counts, N, K, dtype, True, 5, seed=3, first=2)


def test_gradient_of_a_short_row_agrees_with_differences():
    """Rows of 3 and 20 elements: <c, combine(y, w)> is linear in y and in w, so differences are exact but for rounding."""
    for H in (3, 20):
        T, k, n_experts = 5, 2, 3
        ids = _ids(T, k, n_experts, H)
        _, rr = _sort_ref(ids, n_experts)
        there, row_of = rr >= 0, torch.from_numpy(rr).cuda()
        y, c = _rand((T * k, H), torch.float32, 1), _rand((T, H), torch.float32, 2)
        w = torch.rand(T, k, generator=torch.Generator().manual_seed(3))
        dy, dw = torch.zeros(T * k, H, device="cuda"), torch.empty(T, k, device="cuda")
        E.moe_combine_bwd(c.cuda(), y.cuda(), w.cuda(), row_of, dy, dw)
        y64, c64, w64 = y.double().numpy(), c.double().numpy(), w.double().numpy()

        def loss(y, w):
            return (c64[:, None] * w[..., None] * np.where(there[..., None], y[np.maximum(rr, 0)], 0)).sum()

        for at in np.ndindex(*y64.shape):
            d = np.zeros_like(y64)
            d[at] = 1.0
            assert abs((loss(y64 + d, w64) - loss(y64 - d, w64)) / 2 - float(dy[at])) <= 1e-6
        for at in np.ndindex(*w64.shape):
            d = np.zeros_like(w64)
            d[at] = 1.0
            # H products of a few units, each sum off by at most H * 2^-24 of their magnitudes
            assert abs((loss(y64, w64 + d) - loss(y64, w64 - d)) / 2 - float(dw[at])) <= 1e-4
