"""CPU tests of the 4-bit operators, dropout and layer norm: what is refused before any CUDA call, by the C entry points and
by the binding, what the binding hands over, and the references that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

import mxf4_reference
import philox_reference
from paper_2609_11562_b200 import build as B

B.build()
from paper_2609_11562_b200 import entwine as E  # noqa: E402

L = E._lib
P = 1 << 20  # an aligned address that is never followed: every call below is refused first
NAN = float("nan")


def _all_refused(fn, good, bad):
    for i, v in bad:
        args = list(good)
        args[i] = v
        assert fn(*args) == E.ERR_INVALID, (i, v)


def test_quantiser_refusals():
    #       x, dtype, rows, cols, ldx, q, ldq, scale, lds, stream
    good = [P, E.DTYPE_BF16, 4, 65, 65, P, 33, P, 3, None]
    _all_refused(L.entwine_quant_mxf4, good, [
        (0, None), (0, P + 1), (1, E.DTYPE_I8), (1, 9), (1, -1), (2, -1), (2, 1 << 31), (3, 0), (3, -1), (3, 1 << 31), (4, 64), (5, None),
        (6, 32), (7, None), (8, 2)])
    #       q, ldq, scale, lds, rows, cols, x, dtype, ldx, stream
    good = [P, 33, P, 3, 4, 65, P, E.DTYPE_FP32, 65, None]
    _all_refused(L.entwine_dequant_mxf4, good, [
        (0, None), (1, 32), (2, None), (3, 2), (4, -1), (5, 0), (6, None), (6, P + 2), (7, E.DTYPE_I8), (8, 64)])
    assert L.entwine_quant_mxf4(None, E.DTYPE_BF16, 0, 64, 64, None, 32, None, 2, None) == E.OK
    assert L.entwine_dequant_mxf4(None, 32, None, 2, 0, 64, None, E.DTYPE_BF16, 64, None) == E.OK


def test_product_refusals():
    #       A, lda, scale_a, ldsa, B, ldb, scale_b, ldsb, bias, C, c_dtype, ldc, M, N, K, stream
    good = [P, 32, P, 4, P, 32, P, 4, P, P, E.DTYPE_BF16, 32, 4, 32, 64, None]
    _all_refused(L.entwine_gemm_mxf4, good, [
        (0, None), (0, P + 8), (1, 31), (1, 40), (2, None), (2, P + 2), (3, 1), (3, 6), (4, None), (4, P + 4), (5, 16), (5, 36), (6, None), (6, P + 1),
        (7, 0), (7, 5), (8, P + 2), (9, None), (9, P + 1), (10, E.DTYPE_I8), (10, 5), (11, 31), (12, -1), (12, 2147418112), (13, 0),
        (13, 2147483393), (14, 0), (14, 65), (14, (1 << 24) + 1)])
    assert L.entwine_gemm_mxf4(None, 32, None, 4, None, 32, None, 4, None, None, 0, 32, 0, 32, 64, None) == E.OK
    #       A, lda, scale_a, ldsa, B, ldb, expert_stride, scale_b, ldsb, scale_stride, bias, offsets, C, c_dtype, ldc, M, N, K, G, stream
    good = [P, 32, P, 4, P, 32, 1024, P, 4, 128, P, P, P, E.DTYPE_FP32, 32, 4, 32, 64, 4, None]
    _all_refused(L.entwine_gemm_mxf4_grouped, good, [
        (0, None), (1, 24), (2, P + 1), (3, 2), (4, P + 8), (5, 33), (6, 1016), (6, 1000), (6, 1008), (7, None), (7, P + 2), (8, 6), (9, 126), (9, 120),
        (10, P + 1), (11, None), (11, P + 2), (12, P + 2), (13, 3), (14, 16), (15, -4), (16, 0), (16, 1 << 30), (17, 80), (18, 0), (18, 1025)])


def test_dropout_refusals():
    #       x, dtype, rows, cols, ldx, residual, ldr, p, rng, row0, out, ldo, stream
    good = [P, E.DTYPE_BF16, 4, 64, 64, P, 64, 0.5, P, 0, P, 64, None]
    bad_drop = [(7, -0.1), (7, 1.0), (7, NAN), (7, 1 - 2.0 ** -18), (8, None), (8, P + 4), (9, -1), (9, (1 << 32) - 3)]
    _all_refused(L.entwine_dropout, good, bad_drop + [
        (0, None), (0, P + 1), (1, E.DTYPE_I8), (1, 4), (2, -1), (2, 1 << 31), (3, 0), (3, 1 << 31), (4, 63), (5, P + 1), (6, 63), (10, None),
        (10, P + 1), (11, 63)])
    assert L.entwine_dropout(None, E.DTYPE_BF16, 0, 64, 64, None, 0, 0.0, None, 0, None, 64, None) == E.OK
    #       x, dtype, rows, cols, ldx, residual, ldr, p, rng, row0, weight, bias, w_dtype, eps, hidden, ldh, out, ldo, mean, rstd, stream
    good = [P, E.DTYPE_FP16, 4, 64, 64, P, 64, 0.5, P, 0, P, P, E.DTYPE_FP32, 1e-5, P, 64, P, 64, P, P, None]
    _all_refused(L.entwine_layer_norm, good, bad_drop + [
        (0, None), (0, P + 1), (1, E.DTYPE_I8), (2, -1), (2, 1 << 31), (3, 0), (3, 1 << 31), (4, 63), (5, P + 1), (6, 63), (10, None), (10, P + 2),
        (11, P + 2), (12, E.DTYPE_BF16), (12, E.DTYPE_I8), (13, -1.0), (13, NAN), (14, P + 1), (15, 63), (16, None), (16, P + 1), (17, 63),
        (18, P + 2), (19, P + 1)])
    assert L.entwine_layer_norm(None, E.DTYPE_FP16, 0, 64, 64, None, 0, 0.0, None, 0, None, None, E.DTYPE_FP16, 0.0, None, 0, None, 64, None, None,
                                None) == E.OK


def test_gradient_refusals():
    n = E.layer_norm_bwd_work(4, 64)
    assert n > 0
    #       dout, dtype, rows, cols, ldo, hidden, ldh, weight, w_dtype, mean, rstd, dhidden, lddh, p, rng, row0, dx, lddx, dresidual, lddr,
    #       dweight, dbias, work, work_floats, stream
    good = [P, E.DTYPE_BF16, 4, 64, 64, P, 64, P, E.DTYPE_BF16, P, P, P, 64, 0.5, P, 0, P, 64, P, 64, P, P, P, n, None]
    _all_refused(L.entwine_layer_norm_bwd, good, [
        (0, None), (0, P + 1), (1, E.DTYPE_I8), (2, -1), (2, 1 << 31), (3, 0), (3, 1 << 31), (4, 63), (5, None), (5, P + 1), (6, 63), (7, None),
        (7, P + 1), (8, E.DTYPE_FP16), (9, None), (9, P + 2), (10, None), (10, P + 1), (11, P + 1), (12, 63), (13, 1.0), (13, NAN), (14, None),
        (14, P + 4), (15, -1), (15, 1 << 32), (16, None), (16, P + 1), (17, 63), (18, P + 1), (19, 63), (20, None), (20, P + 2), (21, P + 2),
        (22, None), (22, P + 1), (23, n - 1), (23, 0), (23, -1)])
    floats = ctypes.c_int64(0)
    for args in ((-1, 64), (1 << 31, 64), (4, 0), (4, 1 << 31)):
        assert L.entwine_layer_norm_bwd_work(*args, ctypes.byref(floats)) == E.ERR_INVALID
    assert L.entwine_layer_norm_bwd_work(4, 64, None) == E.ERR_INVALID
    with pytest.raises(E.EntwineError):
        E.layer_norm_bwd_work(-1, 64)


@pytest.mark.parametrize("rows", [0, 1, 7, 1000, 10 ** 6, (1 << 31) - 1])
@pytest.mark.parametrize("cols", [1, 64, 4096, 8192, 8200, 16384, 100000, 2147418111])
def test_workspace_holds_a_sum_of_both_gradients_and_stays_small(rows, cols):
    n = E.layer_norm_bwd_work(rows, cols)
    assert n % (2 * cols) == 0 and 1 <= n // (2 * cols) <= 8192


def test_binding_refuses_host_tensors():
    x, b, n = torch.zeros(4, 64), torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(64)
    for call in (lambda: E.quant_mxf4(x, b, b), lambda: E.dequant_mxf4(b, b, x), lambda: E.gemm_mxf4(b, b, b, b, x),
                 lambda: E.gemm_mxf4_grouped(b, b, b, b, b, x), lambda: E.dropout(x, x, 0.1, n), lambda: E.dropout_bwd(x, x, 0.1, n),
                 lambda: E.layer_norm(x, n, n, x), lambda: E.layer_norm_bwd(x, x, n, n, n, x, n, n, n), lambda: E.quant_mxf4([[1.0]], b, b)):
        with pytest.raises(E.EntwineError) as e:
            call()
        assert e.value.code == E.ERR_INVALID


class _Tensor(torch.Tensor):
    """A host tensor that says it lies on a device."""

    place = 0

    @staticmethod
    def on(t, device=0):
        t = t.as_subclass(_Tensor)
        t.place = device
        return t

    def get_device(self):
        return self.place


def f(*s, dtype=torch.float32):
    return _Tensor.on(torch.zeros(*s, dtype=dtype))


def u8(*s):
    return f(*s, dtype=torch.uint8)


def i64(*s):
    return f(*s, dtype=torch.int64)


@pytest.fixture
def recorded():
    """The binding with the library replaced by functions that note what they are given, and device 0 as the current one."""
    calls, keep, addresses = [], [], {}
    for name in E.OP_SYMBOLS:
        fn = ctypes.CFUNCTYPE(ctypes.c_int, *E._OP_ARGS[name])(lambda *a, name=name: calls.append((name, a)) or E.OK)
        keep.append(fn)
        addresses[name] = ctypes.cast(fn, ctypes.c_void_p).value
    dtypes = (torch.bfloat16, torch.float16, torch.float32, torch.int8, torch.int32, torch.int64, torch.uint8)
    E._opcalls.bind(addresses, dtypes, E.EntwineError, lambda: 0, lambda dev: 0)
    yield calls
    E._bind_ops()


def test_binding_refuses_what_does_not_fit(recorded):
    x, q, s, n, r = f(4, 65), u8(4, 33), u8(4, 3), f(65), i64(2)
    o = i64(5).int().as_subclass(_Tensor)
    o.place = 0
    norm = lambda **k: E.layer_norm(*[k.pop(a, d) for a, d in (("x", x), ("weight", n), ("bias", n), ("out", x))], stream=0, **k)  # noqa: E731

    def grad(**k):
        k = {**dict(dout=x, hidden=x, weight=n, mean=f(4), rstd=f(4), dx=x, dweight=n, dbias=n, work=f(9000), stream=0), **k}
        E.layer_norm_bwd(**k)

    bad = [
        lambda: E.quant_mxf4(x, u8(4, 32), s, stream=0), lambda: E.quant_mxf4(x, q, u8(4, 2), stream=0), lambda: E.quant_mxf4(x, q, u8(3, 3), stream=0),
        lambda: E.quant_mxf4(x, f(4, 33), s, stream=0), lambda: E.quant_mxf4(x, f(4, 33, dtype=torch.int8), s, stream=0),
        lambda: E.quant_mxf4(i64(4, 65), q, s, stream=0), lambda: E.quant_mxf4(f(65), q, s, stream=0),
        lambda: E.quant_mxf4(_Tensor.on(torch.zeros(65, 4).t()), q, s, stream=0), lambda: E.quant_mxf4(x, q, _Tensor.on(u8(4, 3), 1), stream=0),
        lambda: E.dequant_mxf4(u8(4, 34), s, x, stream=0), lambda: E.dequant_mxf4(q, s, u8(4, 65), stream=0),
        lambda: E.gemm_mxf4(q, s, u8(7, 32), u8(7, 3), f(4, 7), stream=0), lambda: E.gemm_mxf4(q, s, u8(7, 33), u8(7, 3), f(4, 8), stream=0),
        lambda: E.gemm_mxf4(q, u8(4, 2), u8(7, 33), u8(7, 3), f(4, 7), stream=0), lambda: E.gemm_mxf4(q, s, u8(7, 33), u8(7, 4), f(4, 7), stream=0),
        lambda: E.gemm_mxf4(q, s, u8(7, 33), u8(7, 3), f(4, 7), bias=f(8), stream=0), lambda: E.gemm_mxf4(q, s, u8(7, 33), u8(7, 3), i64(4, 7), stream=0),
        lambda: E.gemm_mxf4_grouped(q, s, u8(7, 33), u8(7, 3), o, f(4, 7), stream=0),
        lambda: E.gemm_mxf4_grouped(q, s, u8(4, 7, 33), u8(4, 7, 2), o, f(4, 7), stream=0),
        lambda: E.gemm_mxf4_grouped(q, s, u8(4, 7, 33), u8(3, 7, 3), o, f(4, 7), stream=0),
        lambda: E.gemm_mxf4_grouped(q, s, u8(3, 7, 33), u8(3, 7, 3), o, f(4, 7), stream=0),
        lambda: E.gemm_mxf4_grouped(q, s, u8(4, 7, 33), u8(4, 7, 3), o, f(4, 6), stream=0),
        lambda: E.dropout(x, f(4, 64), 0.1, r, stream=0), lambda: E.dropout(x, f(4, 65, dtype=torch.float16), 0.1, r, stream=0),
        lambda: E.dropout(x, x, 0.1, None, stream=0), lambda: E.dropout(x, x, 0.1, i64(3), stream=0), lambda: E.dropout(x, x, 0.1, f(2), stream=0),
        lambda: E.dropout(x, x, 1.0, r, stream=0), lambda: E.dropout(x, x, NAN, r, stream=0), lambda: E.dropout(x, x, -0.5, r, stream=0),
        lambda: E.dropout(x, x, 0.1, r, row0=1 << 70, stream=0), lambda: E.dropout(x, x, 0.1, r, residual=f(3, 65), stream=0),
        lambda: norm(weight=f(64)), lambda: norm(weight=f(65, dtype=torch.float16)), lambda: norm(bias=f(65, dtype=torch.float16)),
        lambda: norm(out=f(4, 66)), lambda: norm(mean=f(5)), lambda: norm(rstd=f(4, dtype=torch.float16)), lambda: norm(residual=f(4, 64)),
        lambda: norm(hidden=f(5, 65)), lambda: norm(p=0.1), lambda: norm(p=2.0, rng=r), lambda: norm(x=f(4, 65, 1)),
        lambda: grad(hidden=f(4, 64)), lambda: grad(mean=f(3)), lambda: grad(rstd=None), lambda: grad(dx=f(4, 65, dtype=torch.bfloat16)),
        lambda: grad(dweight=f(65, dtype=torch.float16)), lambda: grad(dbias=f(64)), lambda: grad(work=f(3, 3)), lambda: grad(work=i64(9000)),
        lambda: grad(dhidden=f(3, 65)), lambda: grad(dresidual=f(4, 66)), lambda: grad(p=0.5), lambda: grad(work=_Tensor.on(f(9000), 1)),
    ]
    for call in bad:
        with pytest.raises(E.EntwineError) as e:
            call()
        assert e.value.code == E.ERR_INVALID
    assert not recorded
    with pytest.raises(TypeError):
        E.dropout(x, x, "much", r, stream=0)


def test_binding_hands_sizes_and_distances_over(recorded):
    x, h = f(6, 72)[:, :65], f(6, 80)[:, :65]
    q, s, w, ws = u8(6, 48)[:, :33], u8(6, 8)[:, :3], u8(7, 64)[:, :33], u8(7, 4)[:, :3]
    at = lambda t: t.data_ptr()  # noqa: E731
    E.quant_mxf4(x, q, s, stream=3)
    assert recorded.pop() == ("entwine_quant_mxf4", (at(x), E.DTYPE_FP32, 6, 65, 72, at(q), 48, at(s), 8, 3))
    E.dequant_mxf4(q, s, x, stream=3)
    assert recorded.pop() == ("entwine_dequant_mxf4", (at(q), 48, at(s), 8, 6, 65, at(x), E.DTYPE_FP32, 72, 3))
    out, bias = f(6, 9, dtype=torch.float16)[:, :7], f(7)
    E.gemm_mxf4(q, s, w, ws, out, bias=bias, stream=3)
    assert recorded.pop() == ("entwine_gemm_mxf4", (at(q), 48, at(s), 8, at(w), 64, at(ws), 4, at(bias), at(out), E.DTYPE_FP16, 9, 6, 7, 66, 3))
    g, gs, off = u8(2, 9, 64)[:, :7, :33], u8(2, 8, 4)[:, :7, :3], f(3, dtype=torch.int32)
    E.gemm_mxf4_grouped(q, s, g, gs, off, out, stream=3)
    assert recorded.pop() == ("entwine_gemm_mxf4_grouped", (at(q), 48, at(s), 8, at(g), 64, 576, at(gs), 4, 32, None, at(off), at(out), E.DTYPE_FP16, 9,
                                                           6, 7, 66, 2, 3))
    r = i64(2)
    E.dropout(x, h, 0.25, r, row0=9, residual=x, stream=3)
    assert recorded.pop() == ("entwine_dropout", (at(x), E.DTYPE_FP32, 6, 65, 72, at(x), 72, 0.25, at(r), 9, at(h), 80, 3))
    E.dropout_bwd(x, h, 0.25, r, row0=9, stream=3)
    assert recorded.pop() == ("entwine_dropout", (at(x), E.DTYPE_FP32, 6, 65, 72, None, 0, 0.25, at(r), 9, at(h), 80, 3))
    n, m = f(65), f(6)
    E.layer_norm(x, n, None, h, eps=0.5, mean=m, residual=x, hidden=h, p=0.25, rng=r, row0=9, stream=3)
    assert recorded.pop() == ("entwine_layer_norm", (at(x), E.DTYPE_FP32, 6, 65, 72, at(x), 72, 0.25, at(r), 9, at(n), None, E.DTYPE_FP32, 0.5, at(h), 80,
                                                    at(h), 80, at(m), None, 3))
    work = f(5000)
    E.layer_norm_bwd(x, h, n, m, m, x, n, None, work, dhidden=h, dresidual=h, p=0.25, rng=r, row0=9, stream=3)
    assert recorded.pop() == ("entwine_layer_norm_bwd", (at(x), E.DTYPE_FP32, 6, 65, 72, at(h), 80, at(n), E.DTYPE_FP32, at(m), at(m), at(h), 80, 0.25, at(r),
                                                        9, at(x), 72, at(h), 80, at(n), None, at(work), 5000, 3))
    assert not recorded


def test_the_generator_gives_the_published_numbers():
    """The known answers that its authors publish for all-zero and all-one counters and keys."""
    one = 0xFFFFFFFF
    for fill, want in ((0, (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)), (one, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD))):
        got = philox_reference.philox([np.full(1, fill)] * 4, (fill, fill))
        assert tuple(int(w[0]) for w in got) == want


def test_reference_codes():
    x = np.array([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -0.75, 6.0, 0.26]])
    q, s = mxf4_reference.encode(x)
    assert s.tolist() == [[127]]
    assert mxf4_reference.decode(q, s, 12).tolist() == [[0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, -0.0, -1.0, 6.0, 0.5]]
