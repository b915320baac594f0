"""ctypes binding over the C-ABI library (include/entwine.h, include/entwine_ops.h).

Argument marshalling only: every step of the path runs in the CUDA library.  Importing this
module fails loudly if libentwine.so has not been built, an operator if its marshalling module has not (there is
no fallback).
Device-buffer arguments are torch CUDA tensors (bf16, contiguous) or raw integer addresses;
`stream` is a torch.cuda.Stream, a raw handle or None (the current torch stream).

The operators beside the fused call (quant_i8, moe_dispatch and the others at the end of this file) take
torch CUDA tensors only: sizes, row distances and element types are read from them, and what does not fit
together is refused with EntwineError(ERR_INVALID) before anything is launched.  Their arguments are marshalled by an
extension module (csrc/opcalls.c), because their smallest calls are as short as a ctypes call.  A call works on its
tensors after it has returned: one that is freed before that, on another stream than its allocation's, needs
Tensor.record_stream as with any kernel.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libentwine.so")
if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2609_11562_b200.build` "
        "(or __graft_entry__.build()); this package has no CPU fallback")
_lib = ctypes.CDLL(LIB_PATH)


class _NoOpcalls:
    """Stands where the operators' marshalling module could not be loaded: everything else works without it."""

    def __init__(self, why: ImportError):
        self._why = why

    def on_first_call(self, f):
        pass

    def __getattr__(self, name):
        raise ImportError(f"the operators need the extension module _opcalls, which could not be loaded ({self._why}): "
                          "build it with `python -m paper_2609_11562_b200.build`") from self._why


try:
    from . import _opcalls
except ImportError as e:
    _opcalls = _NoOpcalls(e)

ORDER_ROW_MAJOR, ORDER_INTERLEAVED, ORDER_M_MAJOR = 0, 1, 2
OK, ERR_INVALID, ERR_RESOURCES, ERR_CUDA, ERR_TIMEOUT, ERR_INTERNAL = 0, -1, -2, -3, -4, -5
ERR_TOO_LARGE = -6
OPT_RANK, OPT_BLOCK_N, OPT_WAIT_BUDGET_NS, OPT_TAIL_HELP = 1, 2, 3, 4
OPT_WITHHOLD_PEER, OPT_NUM_SMS, OPT_POISON_PARTIAL, OPT_PAIR_CTAS, OPT_COLOCATE = 5, 6, 7, 8, 9
OPT_PREFETCH, OPT_STAGES, OPT_L2_HINTS, OPT_LISTS, OPT_RELEASE_GROUP = 10, 11, 12, 13, 14
OPT_KBLOCKS_PER_STAGE, OPT_LDA, OPT_LDB, OPT_REG_CONSUMER, OPT_SPLIT_LAST_WAVE, OPT_B_LAYOUT = 15, 16, 17, 18, 19, 20
OPT_CONSUMER_TMA = 21
B_LAYOUT_NK, B_LAYOUT_KN = 0, 1
RELEASE_PARTITION, RELEASE_WHOLE = -1, -2
(EXPORT_COUNTS, EXPORT_ORDER, EXPORT_TILES, EXPORT_FLAG_SEQ, EXPORT_LIST_OFFS, EXPORT_TASKS,
 EXPORT_PEER_OFFS) = range(7)

# every symbol include/entwine.h declares
SYMBOLS = ("entwine_plan", "entwine_set_option", "entwine_gemm_rs", "entwine_gemm_rs_host",
           "entwine_gemm_only", "entwine_comm_only", "entwine_read_partial", "entwine_plan_export",
           "entwine_last_status", "entwine_destroy", "entwine_strerror", "entwine_gemm_rs_static",
           "entwine_gemm_rs_norm", "entwine_heap_bytes", "entwine_gemm_rs_pull",
           "entwine_gemm_rs_host_begin", "entwine_gemm_rs_host_wait", "entwine_last_sm_clock",
           "entwine_plan_workspace_bytes", "entwine_plan_set_workspace")

_vp, _i64, _int, _f64 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_double
_lib.entwine_plan.argtypes = [ctypes.POINTER(_vp), _i64, _i64, _i64, _int, _int, _int]
_lib.entwine_set_option.argtypes = [_vp, _int, _i64]
_lib.entwine_gemm_rs_norm.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_float, _vp, _vp, _vp, _vp]
_lib.entwine_gemm_rs.argtypes = [_vp] * 7
_lib.entwine_heap_bytes.argtypes = [_vp, ctypes.POINTER(_i64), ctypes.POINTER(_i64)]
_lib.entwine_gemm_rs_pull.argtypes = [_vp, _vp, _vp, _vp, _i64, ctypes.c_uint32, _int, _vp, _vp]
_lib.entwine_gemm_rs_host.argtypes = [_vp] * 6
_lib.entwine_gemm_rs_host_begin.argtypes = [_vp] * 6
_lib.entwine_gemm_rs_host_wait.argtypes = [_vp]
_lib.entwine_gemm_only.argtypes = [_vp] * 4
_lib.entwine_comm_only.argtypes = [_vp, _vp, _vp, _vp, _vp, _int, _vp]
_lib.entwine_read_partial.argtypes = [_vp, _vp, _vp]
_lib.entwine_plan_export.argtypes = [_vp, _int, _vp, ctypes.POINTER(ctypes.c_size_t)]
_lib.entwine_last_status.argtypes = [_vp, ctypes.POINTER(_i64)]
_lib.entwine_last_sm_clock.argtypes = [_vp, ctypes.POINTER(_i64)]
_lib.entwine_plan_workspace_bytes.argtypes = [_vp, ctypes.POINTER(ctypes.c_size_t)]
_lib.entwine_plan_set_workspace.argtypes = [_vp, _vp, ctypes.c_size_t]
_lib.entwine_destroy.argtypes = [_vp]
_lib.entwine_gemm_rs_static.argtypes = [_vp] * 7 + [ctypes.POINTER(_i64)]
_lib.entwine_strerror.argtypes = [_int]
_lib.entwine_strerror.restype = ctypes.c_char_p
# every symbol include/entwine_ops.h declares, with its argument types
_OP_ARGS = {
    "entwine_quant_i8": [_vp, _int, _i64, _i64, _i64, _vp, _i64, _vp, _vp],
    "entwine_gemm_i8": [_vp, _i64, _vp, _vp, _i64, _vp, _vp, _vp, _int, _i64, _i64, _i64, _i64, _vp],
    "entwine_gemm_i8_grouped": [_vp, _i64, _vp, _vp, _i64, _i64, _vp, _vp, _vp, _vp, _int, _i64, _i64, _i64, _i64, _i64, _vp],
    "entwine_ops_status": [_vp],
    "entwine_ops_failed_waits": [_vp, ctypes.POINTER(ctypes.c_uint64)],
    "entwine_ops_set_option": [_int, _i64],
    "entwine_moe_dispatch": [_vp, _int, _i64, _i64, _i64, _vp, _vp, _int, _i64, _i64, _vp, _i64, _vp, _vp, _vp, _vp],
    "entwine_moe_dispatch_bwd": [_vp, _int, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _vp],
    "entwine_moe_combine": [_vp, _int, _i64, _i64, _i64, _vp, _vp, _i64, _i64, _vp, _i64, _vp],
    "entwine_moe_combine_bwd": [_vp, _int, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _i64, _vp, _i64, _vp, _vp],
    "entwine_quant_mxf4": [_vp, _int, _i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp],
    "entwine_dequant_mxf4": [_vp, _i64, _vp, _i64, _i64, _i64, _vp, _int, _i64, _vp],
    "entwine_gemm_mxf4": [_vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _int, _i64, _i64, _i64, _i64, _vp],
    "entwine_gemm_mxf4_grouped": [_vp, _i64, _vp, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _vp, _int, _i64, _i64, _i64,
                                  _i64, _i64, _vp],
    "entwine_dropout": [_vp, _int, _i64, _i64, _i64, _vp, _i64, _f64, _vp, _i64, _vp, _i64, _vp],
    "entwine_layer_norm": [_vp, _int, _i64, _i64, _i64, _vp, _i64, _f64, _vp, _i64, _vp, _vp, _int, ctypes.c_float, _vp, _i64,
                           _vp, _i64, _vp, _vp, _vp],
    "entwine_layer_norm_bwd_work": [_i64, _i64, ctypes.POINTER(_i64)],
    "entwine_layer_norm_bwd": [_vp, _int, _i64, _i64, _i64, _vp, _i64, _vp, _int, _vp, _vp, _vp, _i64, _f64, _vp, _i64, _vp, _i64,
                               _vp, _i64, _vp, _vp, _vp, _i64, _vp],
}
OP_SYMBOLS = tuple(_OP_ARGS)
for _name, _args in _OP_ARGS.items():
    getattr(_lib, _name).argtypes = _args
    getattr(_lib, _name).restype = _int
for _name in SYMBOLS:
    if _name != "entwine_strerror":
        getattr(_lib, _name).restype = _int


class EntwineError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {strerror(code)} ({code})")


def strerror(code: int) -> str:
    return _lib.entwine_strerror(code).decode()


def _check(code: int, what: str):
    if code != OK:
        raise EntwineError(code, what)


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(s):
    if s is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(s, int):
        return s
    return s.cuda_stream


_EXPORT_DTYPE = {EXPORT_COUNTS: np.int64, EXPORT_ORDER: np.int32, EXPORT_TILES: np.int32,
                 EXPORT_FLAG_SEQ: np.int32, EXPORT_LIST_OFFS: np.int32, EXPORT_TASKS: np.int64,
                 EXPORT_PEER_OFFS: np.int64}


class Plan:
    """entwine_plan / entwine_destroy as a Python object; methods mirror the C entry points."""

    def __init__(self, M, N, K_local, W, tile_order=ORDER_INTERLEAVED, n_comm_sms=0, **options):
        self._h = _vp()
        _check(_lib.entwine_plan(ctypes.byref(self._h), M, N, K_local, W, tile_order, n_comm_sms),
               "entwine_plan")
        self.M, self.N, self.K, self.W = M, N, K_local, W
        self.tile_order, self.n_comm_sms = tile_order, n_comm_sms
        self.rank = 0
        keys = {"rank": OPT_RANK, "block_n": OPT_BLOCK_N, "wait_budget_ns": OPT_WAIT_BUDGET_NS,
                "tail_help": OPT_TAIL_HELP, "num_sms": OPT_NUM_SMS, "poison_partial": OPT_POISON_PARTIAL,
                "pair_ctas": OPT_PAIR_CTAS, "colocate": OPT_COLOCATE, "prefetch": OPT_PREFETCH, "stages": OPT_STAGES, "l2_hints": OPT_L2_HINTS, "lists": OPT_LISTS, "release_group": OPT_RELEASE_GROUP,
                "kblocks_per_stage": OPT_KBLOCKS_PER_STAGE, "reg_consumer": OPT_REG_CONSUMER, "split_last_wave": OPT_SPLIT_LAST_WAVE, "b_layout": OPT_B_LAYOUT, "consumer_tma": OPT_CONSUMER_TMA, "lda": OPT_LDA, "ldb": OPT_LDB}
        # num_sms first: it bounds the others
        for name in sorted(options, key=lambda n: {"num_sms": 0, "b_layout": 1}.get(n, 2)):
            self.set_option(keys[name], options[name])

    def set_option(self, key, value):
        _check(_lib.entwine_set_option(self._h, key, int(value)), f"entwine_set_option({key})")
        if key == OPT_RANK:
            self.rank = int(value)

    def gemm_rs(self, A, B, peer_partials, out_shard, send_bufs, stream=None):
        _check(_lib.entwine_gemm_rs(self._h, _ptr(A), _ptr(B), _ptr(peer_partials), _ptr(out_shard),
                                    _ptr(send_bufs), _stream(stream)), "entwine_gemm_rs")

    def gemm_rs_norm(self, A, B, peer_partials, residual, weight, eps, hidden_out, norm_out, send_bufs,
                     stream=None):
        _check(_lib.entwine_gemm_rs_norm(self._h, _ptr(A), _ptr(B), _ptr(peer_partials), _ptr(residual),
                                         _ptr(weight), float(eps), _ptr(hidden_out), _ptr(norm_out),
                                         _ptr(send_bufs), _stream(stream)), "entwine_gemm_rs_norm")

    def heap_bytes(self):
        """(least bytes of one rank's heap segment, offset of its flag array)."""
        seg, off = _i64(0), _i64(0)
        _check(_lib.entwine_heap_bytes(self._h, ctypes.byref(seg), ctypes.byref(off)), "entwine_heap_bytes")
        return seg.value, off.value

    def gemm_rs_pull(self, A, B, heap, heap_stride, epoch, out_shard, produce_only=False, stream=None):
        _check(_lib.entwine_gemm_rs_pull(self._h, _ptr(A), _ptr(B), _ptr(heap), int(heap_stride), int(epoch),
                                         1 if produce_only else 0, _ptr(out_shard), _stream(stream)),
               "entwine_gemm_rs_pull")

    def gemm_rs_host(self, A, B, peer_partials, out_shard, send_bufs):
        """Host tensors (CPU, bf16, contiguous; pinned for speed)."""
        _check(_lib.entwine_gemm_rs_host(self._h, _ptr(A), _ptr(B), _ptr(peer_partials),
                                         _ptr(out_shard), _ptr(send_bufs)), "entwine_gemm_rs_host")

    def gemm_rs_host_begin(self, A, B, peer_partials, out_shard, send_bufs):
        """Enqueue one host-buffer call (at most two outstanding); pair with gemm_rs_host_wait."""
        _check(_lib.entwine_gemm_rs_host_begin(self._h, _ptr(A), _ptr(B), _ptr(peer_partials),
                                               _ptr(out_shard), _ptr(send_bufs)), "entwine_gemm_rs_host_begin")

    def gemm_rs_host_wait(self):
        _check(_lib.entwine_gemm_rs_host_wait(self._h), "entwine_gemm_rs_host_wait")

    def gemm_rs_static(self, A, B, peer_partials, out_shard, send_bufs, stream=None, want_status=True):
        """The fused call on the library's fixed scratch array: for callers that must not
        allocate device memory (see include/entwine.h).  Problems above the array's limits raise
        EntwineError(ERR_TOO_LARGE).  With want_status the call synchronises the stream and
        returns the status dict; overlapping calls on one device race."""
        out = (_i64 * 8)() if want_status else None
        code = _lib.entwine_gemm_rs_static(self._h, _ptr(A), _ptr(B), _ptr(peer_partials), _ptr(out_shard),
                                           _ptr(send_bufs), _stream(stream), out)
        _check(code, "entwine_gemm_rs_static")
        if not want_status:
            return None
        names = ("code", "cta", "where", "flags_published", "tiles_reduced", "tiles_pushed",
                 "t_gemm_ns", "t_end_ns")
        return {k: int(v) for k, v in zip(names, out)}

    def gemm_only(self, A, B, stream=None):
        _check(_lib.entwine_gemm_only(self._h, _ptr(A), _ptr(B), _stream(stream)), "entwine_gemm_only")

    def comm_only(self, partial, peer_partials, out_shard, send_bufs, n_ctas=0, stream=None):
        _check(_lib.entwine_comm_only(self._h, _ptr(partial), _ptr(peer_partials), _ptr(out_shard),
                                      _ptr(send_bufs), n_ctas, _stream(stream)), "entwine_comm_only")

    def read_partial(self, dst, stream=None):
        _check(_lib.entwine_read_partial(self._h, _ptr(dst), _stream(stream)), "entwine_read_partial")

    def export(self, what) -> np.ndarray:
        n = ctypes.c_size_t(0)
        _check(_lib.entwine_plan_export(self._h, what, None, ctypes.byref(n)), "entwine_plan_export")
        buf = np.zeros(n.value // np.dtype(_EXPORT_DTYPE[what]).itemsize, _EXPORT_DTYPE[what])
        cap = ctypes.c_size_t(buf.nbytes)
        _check(_lib.entwine_plan_export(self._h, what, buf.ctypes.data_as(_vp), ctypes.byref(cap)),
               "entwine_plan_export")
        return buf

    def counts(self) -> dict:
        c = self.export(EXPORT_COUNTS)
        names = ("P_blk", "Q", "cpb", "x", "n_tasks", "n_reduce", "n_push", "flags_published",
                 "peer_flags_prepublished", "min_flag_reads", "bytes_peer_read", "bytes_own_read",
                 "bytes_push_write", "bytes_out_write", "n_gemm_ctas", "n_comm_ctas")
        return {k: int(v) for k, v in zip(names, c)}

    def last_status(self, check=True) -> dict:
        out = (_i64 * 8)()
        code = _lib.entwine_last_status(self._h, out)
        names = ("code", "cta", "where", "flags_published", "tiles_reduced", "tiles_pushed",
                 "t_gemm_ns", "t_end_ns")
        st = {k: int(v) for k, v in zip(names, out)}
        if check and code != OK:
            raise EntwineError(code, f"device status {st}")
        return st

    def workspace_bytes(self) -> int:
        n = ctypes.c_size_t(0)
        _check(_lib.entwine_plan_workspace_bytes(self._h, ctypes.byref(n)), "entwine_plan_workspace_bytes")
        return int(n.value)

    def set_workspace(self, buf, nbytes=None):
        """buf: a CUDA tensor (kept alive by this object) or a raw device address with nbytes."""
        if buf is None:
            _check(_lib.entwine_plan_set_workspace(self._h, None, 0), "entwine_plan_set_workspace")
            self._ws = None
            return
        n = nbytes if nbytes is not None else buf.numel() * buf.element_size()
        _check(_lib.entwine_plan_set_workspace(self._h, _ptr(buf), n), "entwine_plan_set_workspace")
        self._ws = buf

    def last_sm_clock_mhz(self) -> float:
        """SM clock of the launch that the last last_status() call reported (0.0 if unknown)."""
        out = (_i64 * 2)()
        _check(_lib.entwine_last_sm_clock(self._h, out), "entwine_last_sm_clock")
        return out[0] / out[1] * 1e3 if out[1] > 0 else 0.0

    def destroy(self):
        if self._h:
            _lib.entwine_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


# ------------------------------------------------------------------------------------------
# operators beside the fused call (include/entwine_ops.h)
# ------------------------------------------------------------------------------------------
DTYPE_BF16, DTYPE_FP16, DTYPE_FP32, DTYPE_I8 = 0, 1, 2, 3
OPS_OPT_WAIT_BUDGET_NS, OPS_OPT_WITHHOLD_BLOCK = 1, 2


def _bind_ops():
    """Hands the marshalling module the library's entry points and what it asks torch for, before the operators' first
    call: with raw addresses and stream handles the rest of the module needs no torch."""
    import torch
    addresses = {name: ctypes.cast(getattr(_lib, name), _vp).value for name in OP_SYMBOLS}
    dtypes = (torch.bfloat16, torch.float16, torch.float32, torch.int8, torch.int32, torch.int64, torch.uint8)
    # the current stream's handle where torch gives it alone: building a Stream object takes 3 us, as long as a short kernel
    stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
    _opcalls.bind(addresses, dtypes, EntwineError, torch.cuda.current_device, stream)


_opcalls.on_first_call(_bind_ops)


def quant_i8(x, q, scale, stream=None):
    """Rows to int8 with a scale each: scale = amax / 127, q = rint(127 x / amax), ties to even.
    x [M, K] bf16, fp16 or fp32; q [M, K] int8; scale [M] fp32."""
    _opcalls.quant_i8(x, q, scale, stream)


def gemm_i8(a, scale_a, b, scale_b, out, bias=None, stream=None):
    """out[m, n] = scale_a[m] scale_b[n] sum_k a[m, k] b[n, k] (+ bias[n]).  a [M, K], b [N, K] int8 with rows on 16-byte
    boundaries; scale_a [M], scale_b [N], bias [N] fp32; out [M, N] bf16, fp16 or fp32."""
    _opcalls.gemm_i8(a, scale_a, b, scale_b, out, bias, stream)


def gemm_i8_grouped(a, scale_a, b, scale_b, offsets, out, bias=None, stream=None):
    """Rows [offsets[g], offsets[g+1]) of a times expert g's matrix: b [G, N, K] int8, scale_b and bias [G, N] fp32,
    offsets [G+1] int32 on the device; the rest as gemm_i8.  Rows of no expert are left as they were."""
    _opcalls.gemm_i8_grouped(a, scale_a, b, scale_b, offsets, out, bias, stream)


def ops_status(stream=None):
    """Synchronises the stream; raises EntwineError(ERR_TIMEOUT) if bounded device-side waits of products on the current
    device have run out since this thread's last query: whosever product it was, all of this thread's since then may be
    incomplete.  Other threads are told by their own queries."""
    _check(_lib.entwine_ops_status(_stream(stream)), "entwine_ops_status")


def ops_failed_waits(stream=None) -> int:
    """Synchronises the stream; the number of products' waits that have run out on the current device since the library
    was loaded.  Unchanged from before some calls to after them: these are complete."""
    n = ctypes.c_uint64(0)
    _check(_lib.entwine_ops_failed_waits(_stream(stream), ctypes.byref(n)), "entwine_ops_failed_waits")
    return n.value


def ops_set_option(key, value):
    """A setting of the process for its later products: the budget of their device-side waits, or fault injection
    (include/entwine_ops.h)."""
    _check(_lib.entwine_ops_set_option(key, int(value)), f"entwine_ops_set_option({key})")


def moe_dispatch(x, ids, n_experts, rows, offsets, row_of, x_scale=None, row_scale=None, stream=None):
    """Tokens sorted by expert.  x [T, H] bf16, fp16, fp32 or int8; ids [T, k] int32 or int64, an id outside
    [0, n_experts) drops the assignment; rows [T*k, H]; offsets [n_experts+1] int32; row_of [T, k] int32 (-1:
    dropped); x_scale [T] -> row_scale [T*k] fp32, both or neither.  Rows behind offsets[-1] are left as they were."""
    _opcalls.moe_dispatch(x, ids, n_experts, rows, offsets, row_of, x_scale, row_scale, stream)


def moe_dispatch_bwd(d_rows, row_of, dx, stream=None):
    """Gradient of moe_dispatch: dx[t] = sum_j d_rows[row_of[t, j]] in fp32, j ascending.  d_rows [n, H], dx [T, H]."""
    _opcalls.moe_dispatch_bwd(d_rows, row_of, dx, stream)


def moe_combine(y, weights, row_of, out, stream=None):
    """out[t] = sum_j weights[t, j] y[row_of[t, j]] in fp32, j ascending.  y [n, H], out [T, H] of one type, weights
    [T, k] fp32."""
    _opcalls.moe_combine(y, weights, row_of, out, stream)


def moe_combine_bwd(dout, y, weights, row_of, dy, dw, stream=None):
    """Gradients of moe_combine: dy[row_of[t, j]] = weights[t, j] dout[t], dw[t, j] = <dout[t], y[row_of[t, j]]>
    (fp32; 0 where dropped).  Rows of dy that no assignment names are left as they were."""
    _opcalls.moe_combine_bwd(dout, y, weights, row_of, dy, dw, stream)


def quant_mxf4(x, q, scale, stream=None):
    """Rows to 4-bit floats (e2m1) with a power-of-two scale per 32 elements (e8m0), the OCP MXFP4 format.  x [M, K] bf16,
    fp16 or fp32; q [M, ceil(K/2)] uint8, element 2i in the lower half of byte i; scale [M, ceil(K/32)] uint8."""
    _opcalls.quant_mxf4(x, q, scale, stream)


def dequant_mxf4(q, scale, x, stream=None):
    """Back to values, rounded once to x's type: x = code 2^(scale - 127), NaN where scale is 255."""
    _opcalls.dequant_mxf4(q, scale, x, stream)


def gemm_mxf4(a, scale_a, b, scale_b, out, bias=None, stream=None):
    """out[m, n] = sum_k a[m, k] b[n, k] (+ bias[n]) of the values that codes and scales stand for.  a [M, ceil(K/2)],
    b [N, ceil(K/2)] uint8 with rows on 16-byte boundaries; scale_a [M, ceil(K/32)], scale_b [N, ceil(K/32)] uint8 with rows on
    4-byte boundaries (a contiguous [N, 90] needs a copy with rows of 92); of an odd K the last upper half is zero, as quant_mxf4
    writes it; bias [N] fp32; out [M, N] bf16, fp16 or fp32."""
    _opcalls.gemm_mxf4(a, scale_a, b, scale_b, out, bias, stream)


def gemm_mxf4_grouped(a, scale_a, b, scale_b, offsets, out, bias=None, stream=None):
    """Rows [offsets[g], offsets[g+1]) of a times expert g's matrix: b [G, N, ceil(K/2)], scale_b [G, N, ceil(K/32)] uint8, bias
    [G, N] fp32, offsets [G+1] int32 on the device; the rest as gemm_mxf4.  Rows of no expert are left as they were."""
    _opcalls.gemm_mxf4_grouped(a, scale_a, b, scale_b, offsets, out, bias, stream)


def dropout(x, out, p, rng, row0=0, residual=None, stream=None):
    """out = residual + dropout(x): kept with probability 1 - p (to the nearest 2^-16) by a number computed from rng, the
    row's number row0 + r and the column; the mask is not stored.  rng: int64 [2] on the device, seed and offset (None is
    allowed with p = 0); x, out, residual [M, K] of one type, bf16, fp16 or fp32."""
    _opcalls.dropout(x, out, p, rng, row0, residual, stream)


def dropout_bwd(dout, dx, p, rng, row0=0, stream=None):
    """Gradient of dropout: the same mask and factor on dout."""
    _opcalls.dropout(dout, dx, p, rng, row0, None, stream)


def layer_norm(x, weight, bias, out, eps=1e-5, mean=None, rstd=None, residual=None, hidden=None, p=0.0, rng=None, row0=0,
               stream=None):
    """hidden = residual + dropout(x) (rounded to x's type), out = (hidden - mean) rstd weight + bias.  x, out, residual, hidden
    [M, K] of one type; weight and bias (or None) [K] of that type or fp32; mean, rstd [M] fp32 for the gradients; p, rng, row0
    as in dropout.  Outputs that are None are not written."""
    _opcalls.layer_norm(x, weight, bias, out, eps, mean, rstd, residual, hidden, p, rng, row0, stream)


def layer_norm_bwd_work(rows, cols) -> int:
    """fp32 elements of layer_norm_bwd's workspace."""
    n = _i64(0)
    _check(_lib.entwine_layer_norm_bwd_work(int(rows), int(cols), ctypes.byref(n)), "entwine_layer_norm_bwd_work")
    return n.value


def layer_norm_bwd(dout, hidden, weight, mean, rstd, dx, dweight, dbias, work, dhidden=None, dresidual=None, p=0.0, rng=None,
                   row0=0, stream=None):
    """Gradients of layer_norm: dx [M, K] (of x, through the dropout), dresidual [M, K] (of the residual and of hidden; None: not
    written), dweight and dbias (or None) [K] fp32.  dhidden: the gradient that reaches hidden itself.  work: contiguous fp32,
    layer_norm_bwd_work(M, K) elements or more, one for each call that may overlap."""
    _opcalls.layer_norm_bwd(dout, hidden, weight, mean, rstd, dx, dweight, dbias, work, dhidden, dresidual, p, rng, row0, stream)
