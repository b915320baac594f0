"""Layer norm and its gradients for rows of millions of columns: what a thread adds up of a row may not lose bits with the
row's length."""
import math

import pytest
import torch

import test_gpu_ops_norm as N

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_11562_b200 import build as B
    B.build()
    from paper_2609_11562_b200 import entwine as E

U = N.U


@pytest.fixture(autouse=True)
def depth_that_does_not_grow(monkeypatch):
    """Eight values are added in fp32, their sums in more bits, the result rounded once: at most eight roundings, whatever the
    row's length, and one that turns the sum into fp32."""
    monkeypatch.setattr(N, "_depth", lambda cols: 10)


def _rows(cols, dtype):
    """Rows whose fp32 sums are rounded to the same side again and again: equal values, two values in turn (their distances from
    the mean are equal), a large mean under small differences; and one of random numbers."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(4, cols, dtype=dtype, device="cuda")
    x[0] = 0.1
    x[0, ::1000] = 0.2
    x[1, 0::2], x[1, 1::2] = 0.7, 0.1
    x[2] = torch.randn(cols, generator=g, device="cuda") + 8
    x[3] = torch.randn(cols, generator=g, device="cuda")
    return x


@pytest.mark.parametrize("keep", [True, False])
@pytest.mark.parametrize("dtype", N.FLOATING, ids=N._id)
@pytest.mark.parametrize("cols", [(1 << 20) + 8, (1 << 24) + 5])
def test_layer_norm(cols, dtype, keep):
    x = _rows(cols, dtype)
    w, b = 1 + 0.2 * torch.randn(cols, device="cuda"), torch.randn(cols, device="cuda")
    out, hidden = torch.empty_like(x), torch.empty_like(x) if keep else None
    mean, rstd = torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    E.layer_norm(x, w, b, out, eps=1e-3, mean=mean, rstd=rstd, hidden=hidden)
    assert not keep or torch.equal(hidden, x)
    N._check_norm(x, w, b, 1e-3, out, mean, rstd)


@pytest.mark.parametrize("dtype", N.FLOATING, ids=N._id)
@pytest.mark.parametrize("cols", [(1 << 20) + 8, (1 << 24) + 5])
def test_gradients(cols, dtype):
    h, dout = _rows(cols, dtype), _rows(cols, dtype).flip(0).contiguous()
    w = torch.ones(cols, device="cuda")
    mean, rstd = N._stats(h)
    dx, dw, db = torch.empty_like(h), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    E.layer_norm_bwd(dout, h, w, mean, rstd, dx, dw, db, torch.empty(E.layer_norm_bwd_work(4, cols), device="cuda"))
    N._check_grad(dout, h, w, mean, rstd, None, None, dx, None, dw, db)


def test_a_row_that_is_not_finite_stays_so():
    """(a sum that carries its rounding error along would make a NaN of an infinite mean)"""
    cols = 40000
    x = torch.randn(3, cols, device="cuda")
    x[0, 777], x[1, 39999] = math.inf, math.nan
    out, mean, rstd = torch.empty_like(x), torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    w = torch.ones(cols, device="cuda")
    E.layer_norm(x, w, None, out, mean=mean, rstd=rstd)
    assert bool(torch.isinf(mean[0])) and bool(torch.isnan(mean[1])) and bool(torch.isnan(out[:2]).all()) and bool(torch.isfinite(out[2]).all())
