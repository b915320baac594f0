"""CPU tests of the operators beside the fused call: every symbol of include/entwine_ops.h is exported and bound, and
calls that cannot be right are refused before any CUDA call, by the C entry points and by the binding."""
import ctypes
import os
import re

import pytest
import torch

from paper_2609_11562_b200 import build as B

B.build()
from paper_2609_11562_b200 import entwine as E  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
L = E._lib
P = 1 << 20  # an aligned address that is never followed: every call below is refused first


def test_every_declared_operator_is_exported_and_bound():
    header = open(os.path.join(ROOT, "include", "entwine_ops.h")).read()
    declared = set(re.findall(r"^int (entwine_[a-z0-9_]+)\(", header, flags=re.M))
    assert declared == set(E.OP_SYMBOLS) and declared
    lib = ctypes.CDLL(E.LIB_PATH)
    for name in declared:
        assert hasattr(lib, name), name
    for name, value in re.findall(r"(ENTWINE_(?:BF16|FP16|FP32|I8)) = (\d)", header):
        assert getattr(E, name.replace("ENTWINE_", "DTYPE_")) == int(value)


def _vary(good, bad):
    """The good argument list with one argument replaced, for each (index, value) of bad."""
    for i, v in bad:
        args = list(good)
        args[i] = v
        yield i, v, args


def _all_refused(fn, good, bad):
    for i, v, args in _vary(good, bad):
        assert fn(*args) == E.ERR_INVALID, (i, v)


def test_quant_i8_refusals():
    good = [P, E.DTYPE_BF16, 4, 64, 64, P, 64, P, None]
    _all_refused(L.entwine_quant_i8, good, [
        (0, None), (0, P + 1), (1, E.DTYPE_I8), (1, 9), (1, -1), (2, -1), (2, 1 << 31), (3, 0), (3, -4), (4, 63), (5, None),
        (6, 63), (7, None), (7, P + 2)])
    assert L.entwine_quant_i8(None, E.DTYPE_BF16, 0, 64, 64, None, 64, None, None) == E.OK  # nothing to do


def test_gemm_i8_refusals():
    #       A, lda, scale_a, B, ldb, scale_b, bias, C, c_dtype, ldc, M, N, K, stream
    good = [P, 64, P, P, 64, P, P, P, E.DTYPE_BF16, 32, 4, 32, 64, None]
    _all_refused(L.entwine_gemm_i8, good, [
        (0, None), (0, P + 8), (1, 63), (1, 72), (1, 48), (2, None), (2, P + 1), (3, None), (3, P + 4), (4, 72), (5, None),
        (6, P + 2), (7, None), (7, P + 1), (8, E.DTYPE_I8), (8, 5), (9, 31), (10, -1), (10, 1 << 31), (11, 0), (11, 1 << 31),
        (12, 0), (12, 65), (12, 131072)])
    assert L.entwine_gemm_i8(None, 64, None, None, 64, None, None, None, 0, 32, 0, 32, 64, None) == E.OK
    #       A, lda, scale_a, B, ldb, expert_stride, scale_b, bias, offsets, C, c_dtype, ldc, M, N, K, G, stream
    good = [P, 64, P, P, 64, 2048, P, P, P, P, E.DTYPE_FP32, 32, 4, 32, 64, 4, None]
    _all_refused(L.entwine_gemm_i8_grouped, good, [
        (0, None), (1, 56), (3, P + 8), (4, 65), (5, 2040), (5, 1024), (6, None), (7, P + 1), (8, None), (8, P + 2), (9, P + 2), (10, 3),
        (11, 16), (12, -4), (13, 0), (14, 80), (15, 0), (15, 1025), (13, 1 << 30)])


def test_moe_dispatch_refusals():
    #       x, dtype, T, H, ldx, x_scale, ids, ids64, k, E, rows, ldr, row_scale, offsets, row_of, stream
    good = [P, E.DTYPE_BF16, 4, 64, 64, P, P, 1, 2, 8, P, 64, P, P, P, None]
    _all_refused(L.entwine_moe_dispatch, good, [
        (0, None), (0, P + 1), (1, 7), (2, -1), (2, 1 << 31), (3, 0), (4, 63), (5, None), (5, P + 2), (6, None), (6, P + 4), (8, 0),
        (8, -1), (8, 1 << 30), (9, 0), (9, 1025), (10, None), (11, 63), (12, None), (12, P + 1), (13, None), (13, P + 2),
        (14, None), (14, P + 1)])


def test_moe_return_refusals():
    #       y, dtype, n_rows, H, ldy, row_of, T, k, dx, ldx, stream
    good = [P, E.DTYPE_FP32, 8, 64, 64, P, 4, 2, P, 64, None]
    _all_refused(L.entwine_moe_dispatch_bwd, good, [
        (0, None), (0, P + 2), (1, E.DTYPE_I8), (2, -1), (3, 0), (4, 63), (5, None), (6, -1), (7, 0), (7, 1 << 30), (8, None), (9, 63)])
    good = [P, E.DTYPE_FP32, 8, 64, 64, P, P, 4, 2, P, 64, None]
    _all_refused(L.entwine_moe_combine, good, [
        (0, None), (1, E.DTYPE_I8), (2, -1), (3, 0), (4, 63), (5, None), (5, P + 2), (6, None), (7, -1), (8, 0), (9, None), (10, 63)])
    assert L.entwine_moe_combine(None, E.DTYPE_FP32, 0, 64, 64, None, None, 0, 2, None, 64, None) == E.OK
    #       dout, dtype, T, H, ldo, y, n_rows, ldy, w, row_of, k, dy, lddy, dw, stream
    good = [P, E.DTYPE_FP16, 4, 64, 64, P, 8, 64, P, P, 2, P, 64, P, None]
    _all_refused(L.entwine_moe_combine_bwd, good, [
        (0, None), (0, P + 1), (1, E.DTYPE_I8), (2, -1), (3, 0), (4, 63), (5, None), (6, -1), (7, 63), (8, None), (9, None),
        (10, 0), (11, None), (12, 63), (13, None), (13, P + 2)])


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 8)
    for call in (lambda: E.quant_i8(x, x, x), lambda: E.moe_dispatch(x, x, 4, x, x, x), lambda: E.moe_dispatch_bwd(x, x, x),
                 lambda: E.moe_combine(x, x, x, x), lambda: E.moe_combine_bwd(x, x, x, x, x, x),
                 lambda: E.quant_i8([[1.0]], x, x)):
        with pytest.raises(E.EntwineError) as e:
            call()
        assert e.value.code == E.ERR_INVALID


class _Tensor(torch.Tensor):
    """A host tensor that says it lies on a device."""

    @staticmethod
    def on(t, device):
        t = t.as_subclass(_Tensor)
        t.place = device
        return t

    def get_device(self):
        return self.place


_I, _V = ctypes.c_int64, ctypes.c_void_p


@pytest.fixture
def recorded():
    """The binding with the library replaced by functions that note their names, and device 0 as the current one."""
    calls, keep, addresses = [], [], {}
    for name in E.OP_SYMBOLS:
        fn = ctypes.CFUNCTYPE(ctypes.c_int, *E._OP_ARGS[name])(lambda *a, name=name: calls.append((name, a)) or E.OK)
        keep.append(fn)
        addresses[name] = ctypes.cast(fn, _V).value
    dtypes = (torch.bfloat16, torch.float16, torch.float32, torch.int8, torch.int32, torch.int64)
    E._opcalls.bind(addresses, dtypes, E.EntwineError, lambda: 0, lambda dev: 0)
    yield calls
    E._bind_ops()


def test_binding_refuses_tensors_of_another_device(recorded):
    x, q, s = torch.zeros(4, 8), torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4)
    for devices in ((1, 0, 0), (0, 1, 0), (0, 0, 1)):
        args = [_Tensor.on(t, d) for t, d in zip((x, q, s), devices)]
        with pytest.raises(E.EntwineError, match="current CUDA device"):
            E.quant_i8(*args, stream=0)
    assert not recorded


def test_binding_refuses_what_does_not_fit(recorded):
    on = lambda t: _Tensor.on(t, 0)  # noqa: E731
    f = lambda *s: on(torch.zeros(*s))  # noqa: E731
    i8, i32 = lambda *s: on(torch.zeros(*s, dtype=torch.int8)), lambda *s: on(torch.zeros(*s, dtype=torch.int32))  # noqa: E731
    bad = [
        lambda: E.quant_i8(f(4, 8), i8(4, 7), f(4), stream=0),
        lambda: E.quant_i8(f(4, 8), f(4, 8), f(4), stream=0),
        lambda: E.quant_i8(f(4, 8), i8(4, 8), f(5), stream=0),
        lambda: E.quant_i8(f(4, 8, 2), i8(4, 8), f(4), stream=0),
        lambda: E.quant_i8(on(torch.zeros(8, 4).t()), i8(4, 8), f(4), stream=0),
        lambda: E.quant_i8(on(torch.zeros(1, 8).expand(4, 8)), i8(4, 8), f(4), stream=0),
        lambda: E.quant_i8(on(torch.zeros(4, 8, dtype=torch.float64)), i8(4, 8), f(4), stream=0),
        lambda: E.moe_dispatch(f(4, 8), i32(5, 2), 3, f(8, 8), i32(4), i32(4, 2), stream=0),
        lambda: E.moe_dispatch(f(4, 8), f(4, 2), 3, f(8, 8), i32(4), i32(4, 2), stream=0),
        lambda: E.moe_dispatch(f(4, 8), i32(4, 2), 3, f(7, 8), i32(4), i32(4, 2), stream=0),
        lambda: E.moe_dispatch(f(4, 8), i32(4, 2), 3, i8(8, 8), i32(4), i32(4, 2), stream=0),
        lambda: E.moe_dispatch(f(4, 8), i32(4, 2), 3, f(8, 8), i32(3), i32(4, 2), stream=0),
        lambda: E.moe_dispatch(f(4, 8), i32(4, 2), 3, f(8, 8), i32(4), i32(2, 4), stream=0),
        lambda: E.moe_dispatch(f(4, 8), i32(4, 2), 3, f(8, 8), i32(4), i32(4, 2), x_scale=f(4), stream=0),
        lambda: E.moe_dispatch(f(4, 8), i32(4, 2), 3, f(8, 8), i32(4), i32(4, 2), x_scale=f(4), row_scale=f(4), stream=0),
        lambda: E.moe_dispatch_bwd(f(8, 8), i32(4, 2), f(4, 9), stream=0),
        lambda: E.moe_dispatch_bwd(i8(8, 8), i32(4, 2), i8(4, 8), stream=0),
        lambda: E.moe_dispatch_bwd(f(8, 8), i32(8), f(4, 8), stream=0),
        lambda: E.moe_combine(f(8, 8), f(4, 3), i32(4, 2), f(4, 8), stream=0),
        lambda: E.moe_combine(f(8, 8), i32(4, 2), i32(4, 2), f(4, 8), stream=0),
        lambda: E.moe_combine(f(8, 8), f(4, 2), i32(4, 2), f(5, 8), stream=0),
        lambda: E.moe_combine_bwd(f(4, 8), f(8, 9), f(4, 2), i32(4, 2), f(8, 9), f(4, 2), stream=0),
        lambda: E.moe_combine_bwd(f(4, 8), f(8, 8), f(4, 2), i32(5, 2), f(8, 8), f(4, 2), stream=0),
        lambda: E.moe_combine_bwd(f(4, 8), f(8, 8), f(4, 2), i32(4, 2), f(7, 8), f(4, 2), stream=0),
        lambda: E.moe_combine_bwd(f(4, 8), f(8, 8), f(4, 2), i32(4, 2), f(8, 8), f(2, 4), stream=0),
        lambda: E.gemm_i8(i8(4, 16), f(4), i8(6, 32), f(6), f(4, 6), stream=0),
        lambda: E.gemm_i8(i8(4, 16), f(4), i8(6, 16), f(6), f(4, 5), stream=0),
        lambda: E.gemm_i8(i8(4, 16), f(4), i8(6, 16), f(6), i8(4, 6), stream=0),
        lambda: E.gemm_i8(i8(4, 16), f(3), i8(6, 16), f(6), f(4, 6), stream=0),
        lambda: E.gemm_i8(i8(4, 16), f(4), i8(6, 16), f(4), f(4, 6), stream=0),
        lambda: E.gemm_i8(i8(4, 16), f(4), i8(6, 16), f(6), f(4, 6), bias=f(4), stream=0),
        lambda: E.gemm_i8(f(4, 16), f(4), i8(6, 16), f(6), f(4, 6), stream=0),
        lambda: E.gemm_i8(on(i8(16, 4).t()), f(4), i8(6, 16), f(6), f(4, 6), stream=0),
        lambda: E.gemm_i8_grouped(i8(4, 16), f(4), i8(6, 16), f(6), i32(3), f(4, 6), stream=0),
        lambda: E.gemm_i8_grouped(i8(4, 16), f(4), i8(2, 6, 16), f(2, 6), i32(2), f(4, 6), stream=0),
        lambda: E.gemm_i8_grouped(i8(4, 16), f(4), i8(2, 6, 16), f(6, 2), i32(3), f(4, 6), stream=0),
        lambda: E.gemm_i8_grouped(i8(4, 16), f(4), i8(2, 6, 32), f(2, 6), i32(3), f(4, 6), stream=0),
        lambda: E.gemm_i8_grouped(i8(4, 16), f(4), on(torch.zeros(1, 6, 16, dtype=torch.int8).expand(2, 6, 16)), f(2, 6), i32(3), f(4, 6), stream=0),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(E.EntwineError) as e:
            call()
        assert e.value.code == E.ERR_INVALID, i
    assert not recorded  # nothing reached the library


def test_binding_passes_what_fits(recorded):
    on = lambda t: _Tensor.on(t, 0)  # noqa: E731
    f = lambda *s: on(torch.zeros(*s))  # noqa: E731
    i8, i32 = lambda *s: on(torch.zeros(*s, dtype=torch.int8)), lambda *s: on(torch.zeros(*s, dtype=torch.int32))  # noqa: E731
    x, q, scale = on(torch.zeros(4, 16)[:, :8]), i8(4, 8), f(4)
    E.quant_i8(x, q, scale, stream=7)
    assert recorded.pop() == ("entwine_quant_i8", (x.data_ptr(), E.DTYPE_FP32, 4, 8, 16, q.data_ptr(), 8, scale.data_ptr(), 7))
    E.quant_i8(x, q, scale)                             # the current stream, here the default one (a null handle)
    assert recorded.pop()[1][-1] is None
    a, b, sb, out, bias = i8(4, 16), on(torch.zeros(6, 48, dtype=torch.int8)[:, :16]), f(6), f(4, 6), f(6)
    E.gemm_i8(a, scale, b, sb, out, bias=bias, stream=0)
    assert recorded.pop() == ("entwine_gemm_i8", (a.data_ptr(), 16, scale.data_ptr(), b.data_ptr(), 48, sb.data_ptr(), bias.data_ptr(),
                                                  out.data_ptr(), E.DTYPE_FP32, 6, 4, 6, 16, None))
    e, se, off = on(torch.zeros(3, 6, 32, dtype=torch.int8)[:, :, :16]), f(3, 6), i32(4)
    E.gemm_i8_grouped(a, scale, e, se, off, out, stream=0)
    assert recorded.pop() == ("entwine_gemm_i8_grouped", (a.data_ptr(), 16, scale.data_ptr(), e.data_ptr(), 32, 192, se.data_ptr(), None,
                                                          off.data_ptr(), out.data_ptr(), E.DTYPE_FP32, 6, 4, 6, 16, 3, None))
    t, ids, rows, row_of = f(4, 8), on(torch.zeros(4, 2, dtype=torch.int64)), f(8, 8), i32(4, 2)
    E.moe_dispatch(t, ids, 3, rows, off, row_of, stream=0)
    assert recorded.pop() == ("entwine_moe_dispatch", (t.data_ptr(), E.DTYPE_FP32, 4, 8, 8, None, ids.data_ptr(), 1, 2, 3, rows.data_ptr(),
                                                       8, None, off.data_ptr(), row_of.data_ptr(), None))
    rs = f(8)
    E.moe_dispatch(t, i32(4, 2), 3, rows, off, row_of, x_scale=scale, row_scale=rs, stream=0)
    got = recorded.pop()[1]
    assert (got[5], got[7], got[12]) == (scale.data_ptr(), 0, rs.data_ptr())
    E.moe_dispatch_bwd(rows, row_of, t, stream=0)
    assert recorded.pop() == ("entwine_moe_dispatch_bwd", (rows.data_ptr(), E.DTYPE_FP32, 8, 8, 8, row_of.data_ptr(), 4, 2, t.data_ptr(), 8, None))
    w, dw = f(4, 2), f(4, 2)
    E.moe_combine(rows, w, row_of, t, stream=0)
    assert recorded.pop() == ("entwine_moe_combine", (rows.data_ptr(), E.DTYPE_FP32, 8, 8, 8, w.data_ptr(), row_of.data_ptr(), 4, 2, t.data_ptr(),
                                                      8, None))
    dy = f(8, 8)
    E.moe_combine_bwd(t, rows, w, row_of, dy, dw, stream=0)
    assert recorded.pop() == ("entwine_moe_combine_bwd", (t.data_ptr(), E.DTYPE_FP32, 4, 8, 8, rows.data_ptr(), 8, 8, w.data_ptr(), row_of.data_ptr(),
                                                          2, dy.data_ptr(), 8, dw.data_ptr(), None))
    assert not recorded


def test_an_error_of_the_library_is_raised(recorded):
    E._opcalls.bind({n: ctypes.cast(keep, _V).value for n, keep in _failing().items()},
                    (torch.bfloat16, torch.float16, torch.float32, torch.int8, torch.int32, torch.int64), E.EntwineError, lambda: 0, lambda dev: 0)
    on = lambda t: _Tensor.on(t, 0)  # noqa: E731
    with pytest.raises(E.EntwineError, match="entwine_quant_i8") as e:
        E.quant_i8(on(torch.zeros(4, 8)), on(torch.zeros(4, 8, dtype=torch.int8)), on(torch.zeros(4)))
    assert e.value.code == E.ERR_CUDA


_kept = {}


def _failing():
    for name in E.OP_SYMBOLS:
        _kept[name] = ctypes.CFUNCTYPE(ctypes.c_int, *E._OP_ARGS[name])(lambda *a: E.ERR_CUDA)
    return _kept
