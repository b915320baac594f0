"""The forms that large calls take, against the definitions in 64 bits: rows with four groups a thread, rings that turn more
than once, CTA pairs with several tiles of several blocks each.  The bounds are those of the smaller calls' tests."""
import functools
import math

import numpy as np
import pytest
import torch

import mxf4_reference
import philox_on_device
import philox_reference
import test_gpu_ops_mxf4 as Q
import test_gpu_ops_norm as N

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_11562_b200 import build as B
    B.build()
    from paper_2609_11562_b200 import entwine as E

FLOATING, U = N.FLOATING, N.U
_id = N._id


def _factors(p, row0, rows, cols):
    return philox_on_device.factors(p, N.SEED, N.OFFSET, row0, rows, cols)


@pytest.mark.parametrize("p,row0,rows,cols", [(0.1, 0, 5, 64), (0.3, (1 << 32) - 9, 9, 1021), (0.999, 77, 40, 7)])
def test_the_mask_on_the_device_is_that_of_the_host(p, row0, rows, cols):
    assert torch.equal(_factors(p, row0, rows, cols).cpu(), torch.from_numpy(philox_reference.factors(p, N.SEED, N.OFFSET, row0, rows, cols)))


# ------------------------------------------------------------------------------------------
# dropout: from 2^20 elements on, four groups a thread; rows longer than a CTA's threads go in several chunks
# ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", FLOATING, ids=_id)
@pytest.mark.parametrize("rows,cols,shift,pad", [(1100, 1024, 0, 0), (1100, 1021, 0, 3), (1100, 1021, 0, 0), (1100, 1024, 1, 6), (70, 20000, 0, 0),
                                                 (60, 20003, 0, 0), (9000, 130, 0, 6)])
def test_dropout(rows, cols, shift, pad, dtype):
    m = N._Rows(rows, cols, dtype, shift, pad)
    for p, with_residual in ((0.1, True), (0.5, False)):
        x, r, out = m.random(), m.random() if with_residual else None, m.out()
        E.dropout(x, out, p, N._rng(), row0=77, residual=r)
        f = _factors(p, 77, rows, cols)
        y = x.double() * f
        ref = y + r.double() if with_residual else y
        N._near(out, ref, 2 * U * y.abs() + U * ref.abs())
        if not with_residual:
            assert bool((out[f == 0] == 0).all())
    m.untouched_around()


# ------------------------------------------------------------------------------------------
# layer norm: from 2048 rows on, four groups a thread where they divide a row evenly or nearly
# ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", FLOATING, ids=_id)
@pytest.mark.parametrize("rows,cols,shift,pad", [(2100, 1024, 0, 0), (2100, 5128, 0, 0), (2051, 5131, 0, 5), (2100, 2040, 0, 0), (2100, 1021, 0, 0),
                                                 (2049, 16384, 0, 0), (700, 1536, 0, 0), (700, 1021, 0, 3)])
def test_layer_norm(rows, cols, shift, pad, dtype):
    m = N._Rows(rows, cols, dtype, shift, pad, seed=rows)
    for p, res, hid, wtype in ((0.0, False, True, torch.float32), (0.1, True, True, dtype), (0.3, False, True, torch.float32), (0.0, True, True, dtype)):
        x, out = m.random(1.0, 0.5), m.out()
        r, hidden = m.random(2.0) if res else None, m.out()
        w, b = (1 + 0.2 * torch.randn(cols, device="cuda")).to(wtype), torch.randn(cols, device="cuda").to(wtype)
        mean, rstd = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
        E.layer_norm(x, w, b, out, eps=1e-3, mean=mean, rstd=rstd, residual=r, hidden=hidden, p=p, rng=N._rng(), row0=11)
        y = x.double() * (_factors(p, 11, rows, cols) if p else 1.0)
        ref = y + r.double() if res else y
        N._near(hidden, ref, 2 * U * y.abs() + U * ref.abs())
        N._check_norm(hidden, w, b, 1e-3, out, mean, rstd)
        alone = m.out()  # without what else it writes it writes the same
        E.layer_norm(x, w, b, alone, eps=1e-3, residual=r, p=p, rng=N._rng(), row0=11)
        assert torch.equal(alone, out)
        m.untouched_around()
        m.written.clear()


# ------------------------------------------------------------------------------------------
# gradients: a CTA's rows pass through two or three places of shared memory, each of them used several times
# ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", FLOATING, ids=_id)
@pytest.mark.parametrize("rows,cols,shift,pad", [(4000, 1024, 0, 0), (2000, 2560, 0, 0), (1500, 5120, 0, 0), (1501, 1027, 0, 5), (1400, 4613, 0, 3),
                                                 (1300, 5632, 0, 0), (1000, 8192, 0, 0), (900, 12288, 0, 0), (1500, 1021, 0, 0), (1200, 5121, 0, 0),
                                                 (900, 12291, 1, 0)])
def test_layer_norm_gradients(rows, cols, shift, pad, dtype):
    m = N._Rows(rows, cols, dtype, shift, pad, seed=cols)
    for p, down, both, wtype in ((0.0, False, False, dtype), (0.1, True, True, torch.float32)):
        dout, h = m.random(), m.random(2.0, 0.3)
        dhidden = m.random() if down else None
        w = (1 + 0.2 * torch.randn(cols, device="cuda")).to(wtype)
        mean, rstd = N._stats(h)
        dx, dres = m.out(), m.out() if both else None
        dw, db = torch.full((cols,), math.nan, device="cuda"), torch.full((cols,), math.nan, device="cuda")
        need = E.layer_norm_bwd_work(rows, cols)
        work = torch.full((need + 1,), 5.0, device="cuda")
        E.layer_norm_bwd(dout, h, w, mean, rstd, dx, dw, db, work[:need], dhidden=dhidden, dresidual=dres, p=p, rng=N._rng(), row0=5)
        N._check_grad(dout, h, w, mean, rstd, dhidden, _factors(p, 5, rows, cols) if p else None, dx, dres, dw, db)
        assert float(work[need]) == 5.0
        m.untouched_around()
        m.written.clear()


# ------------------------------------------------------------------------------------------
# quantiser and way back: from 2^20 elements on, two pieces or four groups a thread
# ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", FLOATING, ids=_id)
@pytest.mark.parametrize("rows,cols,pad", [(1100, 1024, 0), (1100, 1021, 3), (1100, 1021, 0), (8300, 130, 0), (30, 40000, 0), (27, 40003, 2)])
def test_quantiser_and_way_back(rows, cols, pad, dtype):
    x = Q._hard_rows(rows, cols + pad, dtype, rows + cols)[:, :cols]
    q, s, qw, sw = Q._places(rows, cols)
    E.quant_mxf4(x, q, s)
    rq, rs = mxf4_reference.encode(x.double().cpu().numpy())
    assert np.array_equal(s.cpu().numpy(), rs)
    assert np.array_equal(q.cpu().numpy(), rq)
    assert bool((qw[:, q.shape[1]:] == 255).all()) and bool((sw[:, s.shape[1]:] == 255).all())
    wide = torch.full((rows, cols + pad), 7.0, dtype=dtype, device="cuda")
    E.dequant_mxf4(q, s, wide[:, :cols])
    assert torch.equal(wide[:, :cols], torch.from_numpy(mxf4_reference.decode(rq, rs, cols)).cuda().to(dtype))
    assert bool((wide[:, cols:] == 7.0).all())


# ------------------------------------------------------------------------------------------
# product on pairs: several tiles a pair, whose blocks of 256 elements end inside a group of four scales' stages, at its end,
# or one behind it
# ------------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=1)
def _product(M, N_, K):
    a, sa = Q._operand(M, K, 1, 1)
    b, sb = Q._operand(N_, K, 2, 1)
    return a, sa, b, sb, Q._wide(a, sa, K) @ Q._wide(b, sb, K).T


@pytest.mark.parametrize("M,N_,K", [(4500, 2048, 2816), (4500, 2048, 2304), (4500, 2048, 1024), (4500, 2048, 1280), (4500, 2048, 640),
                                    (4500, 2048, 500), (8000, 4096, 1600), (130, 40000, 3500)])
@pytest.mark.parametrize("dtype", FLOATING, ids=_id)
def test_product_of_exact_sums(M, N_, K, dtype):
    """Terms are multiples of 1/4 up to 36 * 4: exact in fp32 for 576 K < 2^24."""
    assert 144 * 4 * K < 2 ** 24
    a, sa, b, sb, ref = _product(M, N_, K)
    whole = torch.full((M + 2, N_ + 8), 9.0, dtype=dtype, device="cuda")
    out = whole[1:M + 1, :N_]
    for _ in range(3):
        out.fill_(8.0)
        E.gemm_mxf4(a, sa, b, sb, out)
        Q._check_sums(out, ref, torch.zeros_like(ref), K)
    out.fill_(9.0)
    assert bool((whole == 9.0).all())
    E.ops_status()


@pytest.mark.parametrize("dtype", FLOATING, ids=_id)
@pytest.mark.parametrize("counts,N_,K", [((700, 0, 350, 1200, 65, 900, 300, 513), 2048, 1280), ((700, 0, 350, 1200, 65, 900, 300, 513), 2048, 2336),
                                         ((30, 1, 0, 90, 17, 64, 5, 33) * 4, 2304, 1536), ((16,) * 64, 1536, 1100),
                                         # few rows and tiles: narrow tiles, K shared by the CTAs of a cluster
                                         ((16, 0, 9, 40, 3, 16, 20, 1), 512, 4096), ((64, 30, 70, 64), 1000, 3000)])
def test_grouped_product_of_exact_sums(counts, N_, K, dtype):
    Q._grouped(counts, N_, K, dtype, bias=True, spare=5, first=3)
