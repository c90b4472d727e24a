"""Python binding of the MI355X quantized DiT linear layer (DiffPro, arXiv 2511.11446).

Argument marshalling only: every step (DAQ, INT8 GEMM, dequantization, plan walk)
runs inside ``libdiffpro_qlinear.so`` (hand-written HIP for gfx950) through the C
ABI of ``include/diffpro_qlinear.h``.  PyTorch supplies device memory and the
current stream, nothing else.  There is no CPU or PyTorch fallback: if the
library is missing or a call fails, an exception is raised.

A call that is given `stream` (a torch stream or a handle) runs there: its inputs have to be ready
on that stream and to live until it is done with them, and what it returns is ready on that stream.
"""
import ctypes
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdiffpro_qlinear.so")

QL_OK = 0
STATUS_NAMES = {0: "QL_OK", 1: "QL_ERR_NULL", 2: "QL_ERR_SHAPE", 3: "QL_ERR_ALIGN", 4: "QL_ERR_UNSUPPORTED",
                5: "QL_ERR_WORKSPACE", 6: "QL_ERR_DEVICE"}

# every symbol include/diffpro_qlinear.h declares
EXPORTS = ("ql_status_string", "ql_last_device_error", "ql_version", "daq_workspace_bytes", "daq_quantize",
           "qlinear_workspace_bytes", "qlinear_w8a8", "qlinear_w4a8", "qgemm_w8a8", "qgemm_w4a8",
           "ql_pack_w4_host", "ql_plan_create", "ql_plan_destroy", "ql_plan_num_layers",
           "ql_plan_workspace_bytes", "qlinear_plan_run", "ql_set_gemm_variant", "ql_num_gemm_variants",
           "ql_gemm_variant_name", "daq_quantize_robust", "qlinear_plan_run_robust", "ql_time_bin",
           "qlinear_w4a8_g", "qgemm_w4a8_g", "qlinear_w8a8_fused", "qlinear_w4a8_fused", "qlinear_f16", "ql_repack_w4_pairs_host", "ql_prepack_w4", "daq_quantize_rowmax", "qlinear_plan_run_ex", "qlinear_w8a8_noalloc", "qlinear_noalloc_max_bytes",
           "ql_schedule_topk", "ql_plan_greedy", "ql_gptq_quantize_host", "daq_quantize_ln",
           "daq_cg_workspace_bytes", "daq_quantize_cg", "qlinear_grouped_workspace_bytes", "qlinear_grouped", "ql_pack_bits_host",
           "ql_unpack_bits_host", "ql_zero_point_fold_host",
           "attention_f16_workspace_bytes", "attention_f16", "daq_kv_append", "attention_kv8_workspace_bytes", "attention_kv8")


class QlError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        extra = ""
        if status == 6:
            extra = " (hipError %d)" % lib().ql_last_device_error()
        super().__init__("%s failed: %s%s" % (where, STATUS_NAMES.get(status, status), extra))


class ql_debug(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("a_scales", ctypes.c_void_p), ("acc", ctypes.c_void_p)]


class ql_layer_desc(ctypes.Structure):
    _fields_ = [("K", ctypes.c_int64), ("N", ctypes.c_int64), ("w_bits", ctypes.c_int32), ("group", ctypes.c_int32),
                ("w", ctypes.c_void_p), ("w_scale", ctypes.c_void_p), ("bias", ctypes.c_void_p)]


_lib = None
_i64, _vp, _sz, _int = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int


def ensure_built():
    """For the entry scripts (tests, smoke check, benchmark): compile the library if no built one is there.
    The binding itself never builds and never falls back: lib() raises when the library is missing."""
    if not os.path.exists(LIB_PATH):
        from . import build as _build
        _build.build()
    return LIB_PATH


def lib():
    """Load the HIP library (built in-tree by ``python -m paper_2511_11446_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("%s is missing: build it with `python -m paper_2511_11446_amd.build` "
                          "(there is no fallback path)" % LIB_PATH)
    # PyTorch-ROCm ships its own HIP runtime (soname libamdhip64.so.7).  Loading torch first makes the
    # dynamic loader resolve this library's libamdhip64.so.7 dependency to that same copy, so torch's
    # device pointers and streams and this library's kernels live in ONE runtime.  The other order
    # would put two HIP runtimes in the process, and the second one finds no device.
    import torch  # noqa: F401
    L = ctypes.CDLL(LIB_PATH)
    L.ql_status_string.restype = ctypes.c_char_p
    L.ql_status_string.argtypes = [_int]
    L.ql_gemm_variant_name.restype = ctypes.c_char_p
    L.ql_gemm_variant_name.argtypes = [_int]
    L.daq_workspace_bytes.restype = _sz
    L.daq_workspace_bytes.argtypes = [_i64, _i64, _i64]
    L.qlinear_workspace_bytes.restype = _sz
    L.qlinear_workspace_bytes.argtypes = [_i64, _i64, _i64]
    L.daq_quantize.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _sz, _vp]
    lin = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _i64, _vp, ctypes.POINTER(ql_debug), _vp, _sz, _vp]
    L.qlinear_w8a8.argtypes = lin
    L.qlinear_w4a8.argtypes = lin
    gem = [_vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _i64, _vp, _vp, _vp]
    L.qgemm_w8a8.argtypes = gem
    L.qgemm_w4a8.argtypes = gem
    L.ql_pack_w4_host.argtypes = [_vp, _i64, _i64, _vp]
    L.ql_plan_create.argtypes = [ctypes.POINTER(ql_layer_desc), ctypes.c_int32, _i64, ctypes.POINTER(_vp)]
    L.ql_plan_destroy.argtypes = [_vp]
    L.ql_plan_destroy.restype = None
    L.ql_plan_num_layers.argtypes = [_vp]
    L.ql_plan_num_layers.restype = ctypes.c_int32
    L.ql_plan_workspace_bytes.argtypes = [_vp, _i64, _i64]
    L.ql_plan_workspace_bytes.restype = _sz
    L.qlinear_plan_run.argtypes = [_vp, ctypes.POINTER(_vp), ctypes.POINTER(_vp), _i64, _i64, _vp, _sz, _vp]
    L.qlinear_w4a8_g.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _i64, _vp, ctypes.POINTER(ql_debug), _vp, _sz, _vp]
    L.qlinear_w4a8_g.restype = _int
    L.qgemm_w4a8_g.argtypes = [_vp, _vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _i64, _vp, _vp, _vp]
    L.qgemm_w4a8_g.restype = _int
    L.qlinear_w8a8_fused.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _i64, ctypes.POINTER(ql_fusion), _vp, _vp, _sz, _vp]
    L.qlinear_w8a8_fused.restype = _int
    L.qlinear_w4a8_fused.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _i64, ctypes.POINTER(ql_fusion), _vp, _vp, _sz, _vp]
    L.qlinear_w4a8_fused.restype = _int
    L.ql_repack_w4_pairs_host.argtypes = [_vp, _i64, _i64, _vp]
    L.ql_repack_w4_pairs_host.restype = _int
    L.ql_prepack_w4.argtypes = [_vp, _i64, _i64, _vp, _vp]
    L.ql_prepack_w4.restype = _int
    L.daq_quantize_rowmax.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _sz, _vp]
    L.daq_quantize_rowmax.restype = _int
    L.qlinear_plan_run_ex.argtypes = [_vp, ctypes.POINTER(_vp), ctypes.POINTER(_vp), _i64, _i64, _vp, ctypes.POINTER(ctypes.POINTER(ql_fusion)), _vp, _sz, _vp]
    L.qlinear_plan_run_ex.restype = _int
    L.qlinear_f16.argtypes = [_vp, _i64, _i64, _vp, _vp, _i64, ctypes.POINTER(ql_fusion), _vp, _vp]
    L.qlinear_f16.restype = _int
    L.qlinear_plan_run_robust.argtypes = [_vp, ctypes.POINTER(_vp), ctypes.POINTER(_vp), _i64, _i64, _vp, _vp, _sz, _vp]
    L.qlinear_plan_run_robust.restype = _int
    L.daq_quantize_robust.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _sz, _vp]
    L.daq_quantize_robust.restype = _int
    L.ql_time_bin.argtypes = [_i64, _i64]
    L.ql_time_bin.restype = _int
    L.ql_set_gemm_variant.argtypes = [_int]
    L.qlinear_noalloc_max_bytes.restype = _sz
    L.qlinear_noalloc_max_bytes.argtypes = []
    L.qlinear_w8a8_noalloc.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _i64, _vp, _vp]
    L.qlinear_w8a8_noalloc.restype = _int
    i32 = ctypes.c_int32
    L.attention_f16_workspace_bytes.restype = _sz
    L.attention_f16_workspace_bytes.argtypes = [_i64, _i64, i32, i32, i32, i32]
    L.attention_f16.argtypes = [_vp, _vp, _i64, _i64, _vp, _i64, _i64, _i64, _vp, _vp, _sz, _vp]
    L.attention_f16.restype = _int
    L.daq_kv_append.argtypes = [_vp, _vp, _vp]
    L.daq_kv_append.restype = _int
    L.attention_kv8_workspace_bytes.restype = _sz
    L.attention_kv8_workspace_bytes.argtypes = [_i64, i32, i32, i32, i32]
    L.attention_kv8.argtypes = [_vp, _vp, _vp, _sz, _vp]
    L.attention_kv8.restype = _int
    _lib = L
    return L


def _check(status, where):
    if status != QL_OK:
        raise QlError(status, where)


# The binding's own cost is what a loop of small calls sees (a launch costs the host 3.6 us): addresses go through as plain
# integers and the current stream's handle is fetched without building a Stream object (0.1 instead of 2.8 us).

def _ptr(t):
    return None if t is None else t.data_ptr()


_raw_stream = None


def _stream(stream):
    if stream is None:
        global _raw_stream
        if _raw_stream is None:
            import torch
            get, dev = getattr(torch._C, "_cuda_getCurrentRawStream", None), torch.cuda.current_device
            _raw_stream = (lambda: get(dev())) if get is not None else (lambda: torch.cuda.current_stream().cuda_stream)
        return _raw_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


_torch = None


def _load_torch():
    global _torch
    import torch
    _torch = torch
    return torch


def _need(t, dtype, shape=None, name="tensor"):
    torch = _torch or _load_torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda or not t.is_contiguous() or t.dtype != dtype:
        raise TypeError("%s must be a contiguous CUDA tensor of %s" % (name, dtype))
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    return t


def workspace(nbytes, device="cuda", stream=None):
    """A 256-byte aligned scratch tensor of at least nbytes, for use on `stream` (default: the current one)."""
    torch = _torch or _load_torch()
    return _empty((max(int(nbytes), 256),), torch.uint8, device, stream)


def _empty(shape, dtype, device, stream, returned=False):
    """A tensor that a call makes for itself and uses on `stream`: from that stream's memory, as memory that was freed on the current stream may
    still be written by what waits there.  One that is returned is the current stream's too: freed, it waits for what that one does with it."""
    torch = _torch or _load_torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    cuda = torch.cuda
    if not isinstance(stream, cuda.Stream):
        handle = _stream(stream)
        stream = cuda.ExternalStream(handle) if handle else cuda.default_stream()
    with cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    if returned:
        t.record_stream(cuda.current_stream(t.device))
    return t


def daq_workspace_bytes(M, K, R):
    return int(lib().daq_workspace_bytes(M, K, R))


def qlinear_workspace_bytes(M, K, R):
    return int(lib().qlinear_workspace_bytes(M, K, R))


def daq_quantize(x, R, q=None, scales=None, ws=None, stream=None):
    """x fp16 [M,K] -> (q int8 [M,K], scales fp32 [M/R])."""
    import torch
    _need(x, torch.float16, name="x")
    M, K = x.shape
    if q is None:
        q = _empty((M, K), torch.int8, x.device, stream, True)
    if scales is None:
        scales = _empty((max(M // max(R, 1), 1),), torch.float32, x.device, stream, True)
    if ws is None and R > 1:
        ws = workspace(daq_workspace_bytes(M, K, R), x.device, stream)
    rc = lib().daq_quantize(_ptr(x), M, K, R, _ptr(q), _ptr(scales), _ptr(ws), 0 if ws is None else ws.numel(),
                            _stream(stream))
    _check(rc, "daq_quantize")
    return q, scales


def daq_quantize_rowmax(x, R, row_absmax, q=None, scales=None, ws=None, stream=None):
    """DAQ with the row maxima given (int32 [M], binary16 bit patterns, as a fused layer's row_absmax output leaves them)."""
    import torch
    _need(x, torch.float16, name="x")
    M, K = x.shape
    _need(row_absmax, torch.int32, (M,), "row_absmax")
    if q is None:
        q = _empty((M, K), torch.int8, x.device, stream, True)
    if scales is None:
        scales = _empty((max(M // max(R, 1), 1),), torch.float32, x.device, stream, True)
    if ws is None and R > 1:
        ws = workspace(daq_workspace_bytes(M, K, R), x.device, stream)
    rc = lib().daq_quantize_rowmax(_ptr(x), M, K, R, _ptr(row_absmax), _ptr(q), _ptr(scales), _ptr(ws),
                                   0 if ws is None else ws.numel(), _stream(stream))
    _check(rc, "daq_quantize_rowmax")
    return q, scales


def daq_quantize_ln(x, R=1, shift=None, scale=None, rows_per_mod=1, eps=1e-6, want_h=False, want_q=True, ws=None, stream=None):
    """LayerNorm + modulation + DAQ: x fp16 [M,K] -> dict(q int8, scales fp32 [M/R], h fp16 (if want_h or R > 1))."""
    import torch
    _need(x, torch.float16, name="x")
    M, K = x.shape
    out = {}
    if want_h or R > 1:
        out["h"] = _empty((M, K), torch.float16, x.device, stream, True)
    if want_q:
        out["q"] = _empty((M, K), torch.int8, x.device, stream, True)
        out["scales"] = _empty((max(M // max(R, 1), 1),), torch.float32, x.device, stream, True)
    if ws is None and R > 1 and want_q:
        ws = workspace(daq_workspace_bytes(M, K, R), x.device, stream)
    fn = lib().daq_quantize_ln
    fn.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _i64, ctypes.c_float, _vp, _vp, _vp, _vp, _sz, _vp]
    rc = fn(_ptr(x), M, K, R, _ptr(shift), _ptr(scale), rows_per_mod, eps, _ptr(out.get("h")), _ptr(out.get("q")),
            _ptr(out.get("scales")), _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream))
    _check(rc, "daq_quantize_ln")
    return out


def daq_quantize_cg(x, R, act_group, stream=None):
    """Eq. (4) with channel groups: x fp16 [M,K] -> (q int8 [M,K], alpha fp32 [M/R, K/act_group])."""
    import torch
    _need(x, torch.float16, name="x")
    M, K = x.shape
    q = _empty((M, K), torch.int8, x.device, stream, True)
    sc = _empty((M // R, K // act_group), torch.float32, x.device, stream, True)
    L = lib()
    L.daq_cg_workspace_bytes.restype = _sz
    L.daq_cg_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64]
    ws = workspace(L.daq_cg_workspace_bytes(M, K, R, act_group), x.device, stream)
    L.daq_quantize_cg.argtypes = [_vp, _i64, _i64, _i64, _i64, _vp, _vp, _vp, _sz, _vp]
    _check(L.daq_quantize_cg(_ptr(x), M, K, R, act_group, _ptr(q), _ptr(sc), _ptr(ws), ws.numel(), _stream(stream)), "daq_quantize_cg")
    return q, sc


def qlinear_grouped(x, R, w, w_scale, group, bias=None, act_group=0, storage=8, debug=False, y=None, stream=None):
    """Group-scaled layer for any weight width: storage 8 = int8 codes [N,K], 4 = packed nibbles [N,K/2];
    act_group = 0 (row scales) or group (one activation scale per scale block and channel group)."""
    import torch
    _need(x, torch.float16, name="x")
    M, K = x.shape
    N = w.shape[0]
    G = K // group
    if y is None:
        y = _empty((M, N), torch.float16, x.device, stream, True)
    L = lib()
    L.qlinear_grouped_workspace_bytes.restype = _sz
    L.qlinear_grouped_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64]
    ws = workspace(L.qlinear_grouped_workspace_bytes(M, K, R, act_group), x.device, stream)
    out, dbg = {"y": y}, None
    if debug:
        out["q"] = _empty((M, K), torch.int8, x.device, stream, True)
        out["s_a"] = _empty((M // R,) if act_group == 0 else (M // R, G), torch.float32, x.device, stream, True)
        out["P"] = _empty((M, G, N), torch.int32, x.device, stream, True)
        dbg = ctypes.pointer(ql_debug(out["q"].data_ptr(), out["s_a"].data_ptr(), out["P"].data_ptr()))
    L.qlinear_grouped.argtypes = [_vp, _i64, _i64, _i64, _i64, _vp, ctypes.c_int32, _vp, _i64, _vp, _i64, _vp, ctypes.POINTER(ql_debug),
                                  _vp, _sz, _vp]
    rc = L.qlinear_grouped(_ptr(x), M, K, R, act_group, _ptr(w), storage, _ptr(w_scale), group, _ptr(bias), N, _ptr(y), dbg, _ptr(ws),
                           ws.numel(), _stream(stream))
    _check(rc, "qlinear_grouped")
    return out if debug else y


def pack_bits_host(codes, bits):
    import numpy as np
    codes = np.ascontiguousarray(codes, dtype=np.int8)
    N, K = codes.shape
    out = np.empty((N, K * bits // 8), np.uint8)
    _check(lib().ql_pack_bits_host(codes.ctypes.data_as(_vp), _i64(N), _i64(K), ctypes.c_int32(bits), out.ctypes.data_as(_vp)), "ql_pack_bits_host")
    return out


def unpack_bits_host(packed, bits, K):
    import numpy as np
    packed = np.ascontiguousarray(packed, dtype=np.uint8)
    N = packed.shape[0]
    out = np.empty((N, K), np.int8)
    _check(lib().ql_unpack_bits_host(packed.ctypes.data_as(_vp), _i64(N), _i64(K), ctypes.c_int32(bits), out.ctypes.data_as(_vp)), "ql_unpack_bits_host")
    return out


def zero_point_fold_host(codes, zeros, group):
    import numpy as np
    codes = np.ascontiguousarray(codes, dtype=np.int8)
    zeros = np.ascontiguousarray(zeros, dtype=np.int32)
    N, K = codes.shape
    out = np.empty((N, K), np.int8)
    _check(lib().ql_zero_point_fold_host(codes.ctypes.data_as(_vp), zeros.ctypes.data_as(_vp), _i64(N), _i64(K), _i64(group),
                                         out.ctypes.data_as(_vp)), "ql_zero_point_fold_host")
    return out


class ql_fusion(ctypes.Structure):
    _fields_ = [("act", ctypes.c_int32), ("reserved", ctypes.c_int32), ("residual", ctypes.c_void_p),
                ("gate", ctypes.c_void_p), ("gate_rows", ctypes.c_int64), ("row_absmax", ctypes.c_void_p)]


ACT_NONE, ACT_GELU_TANH = 0, 1


def qlinear_fused(x, R, w, w_scale, bias=None, bits=8, group=128, act=ACT_NONE, residual=None, gate=None, gate_rows=1,
                  y=None, ws=None, stream=None, row_absmax=None):
    """The layer with activation, gate and residual folded into its epilogue:
    h = fp16(act(u)); y = fp16(fma(gate, h, residual)).  bits = 8 (w int8 [N,K]) or 4 (w packed [N,K/2], group).
    row_absmax: int32 [M] device tensor that receives every row's largest |y| as a binary16 bit pattern, or None."""
    import torch
    _need(x, torch.float16, name="x")
    M, K = x.shape
    N = w.shape[0]
    if residual is not None:
        _need(residual, torch.float16, (M, N), "residual")
    if gate is not None:
        _need(gate, torch.float16, (M // gate_rows, N), "gate")
    if y is None:
        y = _empty((M, N), torch.float16, x.device, stream, True)
    if ws is None:
        ws = workspace(qlinear_workspace_bytes(M, K, R), x.device, stream)
    if row_absmax is not None:
        _need(row_absmax, torch.int32, (M,), "row_absmax")
    fu = ql_fusion(act, 0, None if residual is None else residual.data_ptr(), None if gate is None else gate.data_ptr(), gate_rows,
                   None if row_absmax is None else row_absmax.data_ptr())
    if bits == 8:
        rc = lib().qlinear_w8a8_fused(_ptr(x), M, K, R, _ptr(w), _ptr(w_scale), _ptr(bias), N, ctypes.byref(fu), _ptr(y),
                                      _ptr(ws), ws.numel(), _stream(stream))
    else:
        rc = lib().qlinear_w4a8_fused(_ptr(x), M, K, R, _ptr(w), _ptr(w_scale), group, _ptr(bias), N, ctypes.byref(fu),
                                      _ptr(y), _ptr(ws), ws.numel(), _stream(stream))
    _check(rc, "qlinear_w%da8_fused" % bits)
    return y


def qlinear_f16(x, w, bias=None, act=ACT_NONE, residual=None, gate=None, gate_rows=1, y=None, stream=None, row_absmax=None):
    """A layer left in FP16: x fp16 [M,K], w fp16 [N,K] -> y fp16 [M,N] (fp32 accumulation)."""
    import torch
    _need(x, torch.float16, name="x")
    _need(w, torch.float16, name="w")
    M, K = x.shape
    N = w.shape[0]
    if y is None:
        y = _empty((M, N), torch.float16, x.device, stream, True)
    fu = ql_fusion(act, 0, None if residual is None else residual.data_ptr(), None if gate is None else gate.data_ptr(), gate_rows,
                   None if row_absmax is None else row_absmax.data_ptr())
    _check(lib().qlinear_f16(_ptr(x), M, K, _ptr(w), _ptr(bias), N, ctypes.byref(fu), _ptr(y), _stream(stream)), "qlinear_f16")
    return y


class _DaqParams(ctypes.Structure):
    _fields_ = [("p_ppm", ctypes.c_int32), ("a_bits", ctypes.c_int32)]


def daq_quantize_robust(x, R, p_ppm=999000, a_bits=8, q=None, scales=None, ws=None, stream=None):
    """Percentile-clipped DAQ: x fp16 [M,K] -> (q int8 [M,K] with |q| <= 2^(a_bits-1)-1, scales fp32 [M/R])."""
    import torch
    _need(x, torch.float16, name="x")
    M, K = x.shape
    if q is None:
        q = _empty((M, K), torch.int8, x.device, stream, True)
    if scales is None:
        scales = _empty((max(M // max(R, 1), 1),), torch.float32, x.device, stream, True)
    if ws is None and R > 1:
        ws = workspace(daq_workspace_bytes(M, K, R), x.device, stream)
    prm = _DaqParams(p_ppm, a_bits)
    rc = lib().daq_quantize_robust(_ptr(x), M, K, R, ctypes.byref(prm), _ptr(q), _ptr(scales), _ptr(ws),
                                   0 if ws is None else ws.numel(), _stream(stream))
    _check(rc, "daq_quantize_robust")
    return q, scales


def time_bin(step, num_steps):
    return int(lib().ql_time_bin(step, num_steps))


def _qlinear(fn_name, x, R, w, w_scale, bias, N, y, debug, ws, stream, group=128):
    import torch
    _need(x, torch.float16, name="x")
    M, K = x.shape
    if y is None:
        y = _empty((M, N), torch.float16, x.device, stream, True)
    if ws is None:
        ws = workspace(qlinear_workspace_bytes(M, K, R), x.device, stream)
    dbg = None
    out = {"y": y}
    if debug:
        G = K // group
        out["q"] = _empty((M, K), torch.int8, x.device, stream, True)
        out["s_a"] = _empty((M // R,), torch.float32, x.device, stream, True)
        shape = (M, N) if fn_name == "qlinear_w8a8" else (M, G, N)
        out["acc" if fn_name == "qlinear_w8a8" else "P"] = acc = _empty(shape, torch.int32, x.device, stream, True)
        dbg = ctypes.pointer(ql_debug(out["q"].data_ptr(), out["s_a"].data_ptr(), acc.data_ptr()))
    if fn_name == "qlinear_w4a8" and group != 128:
        fn_name = "qlinear_w4a8_g"
        rc = lib().qlinear_w4a8_g(_ptr(x), M, K, R, _ptr(w), _ptr(w_scale), group, _ptr(bias), N, _ptr(y), dbg, _ptr(ws),
                                  ws.numel(), _stream(stream))
    else:
        rc = getattr(lib(), fn_name)(_ptr(x), M, K, R, _ptr(w), _ptr(w_scale), _ptr(bias), N, _ptr(y), dbg, _ptr(ws),
                                     ws.numel(), _stream(stream))
    _check(rc, fn_name)
    return out if debug else y


def qlinear_w8a8(x, R, w, w_scale, bias=None, y=None, debug=False, ws=None, stream=None):
    """DAQ + INT8 GEMM + dequantization.  w int8 [N,K], w_scale fp32 [N], bias fp16 [N] or None."""
    import torch
    _need(w, torch.int8, name="w")
    _need(w_scale, torch.float32, (w.shape[0],), "w_scale")
    if bias is not None:
        _need(bias, torch.float16, (w.shape[0],), "bias")
    if w.shape[1] != x.shape[1]:
        raise ValueError("w must be [N,K]")
    return _qlinear("qlinear_w8a8", x, R, w, w_scale, bias, w.shape[0], y, debug, ws, stream)


def qlinear_w8a8_noalloc(x, R, w, w_scale, bias, y, stream=None):
    """qlinear_w8a8 on the library's own fixed scratch: the call allocates nothing; y is the caller's."""
    M, K = x.shape
    _check(lib().qlinear_w8a8_noalloc(_ptr(x), M, K, R, _ptr(w), _ptr(w_scale), _ptr(bias), w.shape[0], _ptr(y), _stream(stream)),
           "qlinear_w8a8_noalloc")
    return y


def qlinear_w4a8(x, R, w4, w_scale, bias=None, y=None, debug=False, ws=None, stream=None, group=128):
    """Same with packed 4-bit weights: w4 uint8 [N,K/2], w_scale fp16 [N,K/group]."""
    import torch
    _need(w4, torch.uint8, name="w4")
    K = x.shape[1]
    if w4.shape[1] * 2 != K:
        raise ValueError("w4 must be [N,K/2]")
    _need(w_scale, torch.float16, (w4.shape[0], K // group), "w_scale")
    if bias is not None:
        _need(bias, torch.float16, (w4.shape[0],), "bias")
    return _qlinear("qlinear_w4a8", x, R, w4, w_scale, bias, w4.shape[0], y, debug, ws, stream, group)


def _qgemm(fn_name, q, a_scales, R, w, w_scale, bias, N, y, acc, stream):
    import torch
    _need(q, torch.int8, name="q")
    _need(a_scales, torch.float32, name="a_scales")
    M, K = q.shape
    if y is None:
        y = _empty((M, N), torch.float16, q.device, stream, True)
    rc = getattr(lib(), fn_name)(_ptr(q), _ptr(a_scales), M, K, R, _ptr(w), _ptr(w_scale), _ptr(bias), N, _ptr(y),
                                 _ptr(acc), _stream(stream))
    _check(rc, fn_name)
    return y


def qgemm_w8a8(q, a_scales, R, w, w_scale, bias=None, y=None, acc=None, stream=None):
    return _qgemm("qgemm_w8a8", q, a_scales, R, w, w_scale, bias, w.shape[0], y, acc, stream)


def qgemm_w4a8(q, a_scales, R, w4, w_scale, bias=None, y=None, acc=None, stream=None, group=128):
    if group == 128:
        return _qgemm("qgemm_w4a8", q, a_scales, R, w4, w_scale, bias, w4.shape[0], y, acc, stream)
    import torch
    M, K = q.shape
    N = w4.shape[0]
    if y is None:
        y = _empty((M, N), torch.float16, q.device, stream, True)
    rc = lib().qgemm_w4a8_g(_ptr(q), _ptr(a_scales), M, K, R, _ptr(w4), _ptr(w_scale), group, _ptr(bias), N, _ptr(y),
                            _ptr(acc), _stream(stream))
    _check(rc, "qgemm_w4a8_g")
    return y


def ql_pack_w4_host(codes):
    """numpy int8 [N,K] in [-8,7] -> numpy uint8 [N,K/2] in the library's 4-bit storage order."""
    import numpy as np
    codes = np.ascontiguousarray(codes, dtype=np.int8)
    N, K = codes.shape
    out = np.empty((N, K // 2), np.uint8)
    rc = lib().ql_pack_w4_host(codes.ctypes.data_as(_vp), N, K, out.ctypes.data_as(_vp))
    _check(rc, "ql_pack_w4_host")
    return out


MASK_NONE, MASK_CAUSAL, MASK_PREFIX = 0, 1, 2


class ql_attention(ctypes.Structure):
    _fields_ = [("T_q", _i64), ("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
                ("mask", ctypes.c_int32), ("scale", ctypes.c_float), ("cap", ctypes.c_float), ("reserved", ctypes.c_int32),
                ("prefix", _vp), ("slopes", _vp), ("cu_q", _vp), ("q", _vp), ("q_row", _i64), ("q_head", _i64),
                ("o", _vp), ("o_row", _i64), ("o_head", _i64), ("row_absmax", _vp)]


class ql_kv_cache(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("num_pages", _i64), ("page", ctypes.c_int32),
                ("scale_tokens", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32), ("page_table", _vp), ("len_k", _vp),
                ("B", ctypes.c_int32), ("max_pages", ctypes.c_int32)]


class ql_kv_new(ctypes.Structure):
    _fields_ = [("T", _i64), ("Hq", ctypes.c_int32), ("rot_pairs", ctypes.c_int32), ("cu", _vp), ("q", _vp), ("k", _vp), ("v", _vp),
                ("q_row", _i64), ("q_head", _i64), ("k_row", _i64), ("k_head", _i64), ("v_row", _i64), ("v_head", _i64),
                ("rot", _vp), ("rot_rows", _i64), ("rot_dim", ctypes.c_int32), ("reserved", ctypes.c_int32), ("pos", _vp),
                ("q_out", _vp), ("k_out", _vp), ("v_out", _vp)]


# The structures above as packed bytes: what a call needs of them costs a tenth of filling a ctypes object field by field (3 us)
_ATTENTION = struct.Struct("=q5iffi3QQqqQqqQ")
_KV_CACHE = struct.Struct("=4Qq4i2Q2i")
_KV_NEW = struct.Struct("=q2iQ3Q6qQq2iQ3Q")


def _heads(t, name, dev, H=None, D=None):
    """A [T, H, D] binary16 view whose rows and heads may be strided: (pointer, row stride, head stride)."""
    torch = _torch or _load_torch()
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.float16 or t.dim() != 3 or not t.is_cuda:
        raise TypeError("%s must be a [T, heads, D] CUDA tensor of torch.float16" % name)
    if t.get_device() != dev:
        _elsewhere(t, name)
    n, heads, d = t.shape
    row, head, one = t.stride()
    if one != 1:
        raise TypeError("%s must have its channels next to each other" % name)
    if (H is not None and heads != H) or (D is not None and d != D):
        raise ValueError("%s has shape %s, expected [T, %s, %s]" % (name, tuple(t.shape), H, D))
    # the stride of a single row or head means nothing
    return t.data_ptr(), row if n > 1 else 0, head if heads > 1 else 0


def _elsewhere(t, name):
    """The calls run on the current device's stream: what they are given has to be there."""
    raise ValueError("%s is on %s, the current device is cuda:%d" % (name, t.device, _torch._C._cuda_getDevice()))


def _here(stream, dev):
    if getattr(stream, "device_index", dev) != dev:
        raise ValueError("stream is on cuda:%d, the current device is cuda:%d" % (stream.device_index, dev))


def _at(t, dtype, shape, name, dev):
    """The address of a small argument (0: none)."""
    if t is None:
        return 0
    if _need(t, dtype, shape, name).get_device() != dev:
        _elsewhere(t, name)
    return t.data_ptr()


def _current():
    try:
        return (_torch or _load_torch())._C._cuda_getDevice()
    except RuntimeError:   # no device: no tensor can be on it
        return -1


def _attention_form(dev, q, B, Hkv, cu_q, mask, prefix, scale, cap, slopes, o, row_absmax, stream):
    torch = _torch or _load_torch()
    qp, q_row, q_head = _heads(q, "q", dev)
    T, Hq, D = q.shape
    if o is None:
        o = _empty((T, Hq, D), torch.float16, q.device, stream, True)
    op, o_row, o_head = _heads(o, "o", dev, Hq, D)
    if o.shape[0] != T:
        raise ValueError("o has %d rows, expected %d" % (o.shape[0], T))
    cu, pre = _at(cu_q, torch.int32, (B + 1,), "cu_q", dev), _at(prefix, torch.int32, (B,), "prefix", dev)
    sl, am = _at(slopes, torch.float32, (Hq,), "slopes", dev), _at(row_absmax, torch.int32, (T,), "row_absmax", dev)
    return _ATTENTION.pack(T, B, Hq, Hkv, D, mask, D ** -0.5 if scale is None else scale, cap, 0, pre, sl, cu, qp, q_row, q_head, op, o_row, o_head, am), o


def attention_f16_workspace_bytes(T_q, T_k, B, Hq, Hkv, D):
    return int(lib().attention_f16_workspace_bytes(T_q, T_k, B, Hq, Hkv, D))


def attention_f16(q, k, v, batch=None, cu_q=None, cu_k=None, mask=MASK_NONE, prefix=None, scale=None, cap=0.0, slopes=None, o=None,
                  row_absmax=None, ws=None, stream=None):
    """Softmax attention: q fp16 [T_q, Hq, D], k, v fp16 [T_k, Hkv, D] (views with strided rows and heads, such as the columns of a fused qkv
    layer's output) -> o fp16 [T_q, Hq, D].  Sequences one behind the other: `batch` of equal length, or int32 [B+1] first rows in cu_q / cu_k.
    scale: default D ** -0.5; cap: tanh cap of the scores (0: none; 2^-10 to 2^10); slopes fp32 [Hq]: bias by distance; mask MASK_NONE / _CAUSAL / _PREFIX
    (prefix int32 [B]); row_absmax: int32 [T_q] that receives every row's largest |o| as a binary16 bit pattern, for daq_quantize_rowmax."""
    dev = _current()
    _here(stream, dev)
    kp, k_row, k_head = _heads(k, "k", dev)
    T_k, Hkv, D = k.shape
    vp, v_row, v_head = _heads(v, "v", dev, Hkv, D)
    if v.shape[0] != T_k or q.shape[-1] != D:
        raise ValueError("k has shape %s, v %s and q %s" % (tuple(k.shape), tuple(v.shape), tuple(q.shape)))
    B = batch if batch is not None else cu_q.shape[0] - 1 if cu_q is not None else cu_k.shape[0] - 1 if cu_k is not None else 1
    cu = _at(cu_k, _torch.int32, (B + 1,), "cu_k", dev)
    a, o = _attention_form(dev, q, B, Hkv, cu_q, mask, prefix, scale, cap, slopes, o, row_absmax, stream)
    if ws is None:
        ws = workspace(attention_f16_workspace_bytes(q.shape[0], T_k, B, q.shape[1], Hkv, D), q.device, stream)
    elif ws.get_device() != dev:
        _elsewhere(ws, "ws")
    _check(lib().attention_f16(a, kp, k_row, k_head, vp, v_row, v_head, T_k, cu, _ptr(ws), ws.numel(), _stream(stream)),
           "attention_f16")
    return o


class KvCache8:
    """A paged cache of keys and values in 8 bits: k int8 [pages, Hkv, page, D], v int8 [pages, Hkv, page/64, D, 64],
    k_scale, v_scale fp32 [pages, Hkv, page/scale_tokens] (CUDA tensors, kept here; the layout is the header's ql_kv_cache)."""

    def __init__(self, k, v, k_scale, v_scale):
        import torch
        _need(k, torch.int8, name="k")
        P, H, page, D = k.shape
        _need(v, torch.int8, (P, H, page // 64, D, 64), "v")
        _need(k_scale, torch.float32, name="k_scale")
        _need(v_scale, torch.float32, tuple(k_scale.shape), "v_scale")
        if k_scale.dim() != 3 or tuple(k_scale.shape[:2]) != (P, H) or k_scale.shape[2] < 1 or page % k_scale.shape[2]:
            raise ValueError("k_scale has shape %s, expected [%d, %d, page / scale_tokens]" % (tuple(k_scale.shape), P, H))
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.num_pages, self.heads, self.page, self.D, self.scale_tokens = P, H, page, D, page // k_scale.shape[2]
        self._devices = tuple(t.get_device() for t in (k, v, k_scale, v_scale))
        self._fields = (k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), P, page, self.scale_tokens, H, D)

    @classmethod
    def empty(cls, num_pages, heads, D, page=64, scale_tokens=64, device="cuda"):
        import torch
        if page < 64 or page % 64 or scale_tokens not in (1, 16, 32, 64):
            raise ValueError("page has to be a multiple of 64 and scale_tokens 1, 16, 32 or 64, not %s and %s" % (page, scale_tokens))
        z = dict(device=device)
        scales = (num_pages, heads, page // scale_tokens)
        return cls(torch.zeros((num_pages, heads, page, D), dtype=torch.int8, **z),
                   torch.zeros((num_pages, heads, page // 64, D, 64), dtype=torch.int8, **z),
                   torch.zeros(scales, dtype=torch.float32, **z), torch.zeros(scales, dtype=torch.float32, **z))

    def desc(self, page_table, len_k):
        """The header's ql_kv_cache for these pages and lengths, as bytes, and the number of sequences."""
        torch = _torch or _load_torch()
        B, max_pages = _need(page_table, torch.int32, name="page_table").shape
        dev = _current()
        if page_table.get_device() != dev:
            _elsewhere(page_table, "page_table")
        if self._devices != (dev, dev, dev, dev):
            name = ("k", "v", "k_scale", "v_scale")[[d == dev for d in self._devices].index(False)]
            _elsewhere(getattr(self, name), "the cache's " + name)
        return _KV_CACHE.pack(*self._fields, page_table.data_ptr(), _at(len_k, torch.int32, (B,), "len_k", dev), B, max_pages), B


def daq_kv_append(cache, k, v, page_table, len_k, cu=None, q=None, rot=None, rot_pairs=False, pos=None, q_out=None, k_out=None, v_out=None,
                  stream=None):
    """New keys and values fp16 [T, Hkv, D] (strided views) into the cache, k and q rotated by rot fp32 [rows, rot_dim/2, 2] (cos, sin) at row pos
    (int32 [T]; default: the token's place in its sequence).  len_k int32 [B] counts the new tokens; cu int32 [B+1]: first new row of each sequence
    (default: T / B each).  q_out fp16 [T, Hq, D]: the rotated q (made where q is given); k_out, v_out fp16 [T, Hkv, D]: what the cache now holds.
    Returns q_out."""
    torch = _torch or _load_torch()
    c, B = cache.desc(page_table, len_k)
    dev = _current()
    _here(stream, dev)
    kp, k_row, k_head = _heads(k, "k", dev, cache.heads, cache.D)
    vp, v_row, v_head = _heads(v, "v", dev, cache.heads, cache.D)
    T = k.shape[0]
    if v.shape[0] != T:
        raise ValueError("k has %d rows and v %d" % (T, v.shape[0]))
    Hq = qp = q_row = q_head = qo = 0
    if q is not None:
        qp, q_row, q_head = _heads(q, "q", dev, None, cache.D)
        Hq = q.shape[1]
        if q.shape[0] != T:
            raise ValueError("q has %d rows and k %d" % (q.shape[0], T))
        if q_out is None:
            q_out = _empty((T, Hq, cache.D), torch.float16, q.device, stream, True)
        qo = _at(q_out, torch.float16, (T, Hq, cache.D), "q_out", dev)
    ko, vo = _at(k_out, torch.float16, (T, cache.heads, cache.D), "k_out", dev), _at(v_out, torch.float16, (T, cache.heads, cache.D), "v_out", dev)
    cup, pp, rp = _at(cu, torch.int32, (B + 1,), "cu", dev), _at(pos, torch.int32, (T,), "pos", dev), _at(rot, torch.float32, None, "rot", dev)
    rows = half = 0
    if rot is not None:
        rows, half, two = rot.shape
        if two != 2 or not rows or not half:     # (the address of an empty table is none: no rotation)
            raise ValueError("rot must be [rows, rot_dim / 2, 2]")
    n = _KV_NEW.pack(T, Hq, 1 if rot_pairs else 0, cup, qp, kp, vp, q_row, q_head, k_row, k_head, v_row, v_head, rp, rows, 2 * half, 0, pp, qo, ko, vo)
    _check(lib().daq_kv_append(c, n, _stream(stream)), "daq_kv_append")
    return q_out


def attention_kv8_workspace_bytes(T_q, B, Hq, Hkv, D):
    return int(lib().attention_kv8_workspace_bytes(T_q, B, Hq, Hkv, D))


def attention_kv8(q, cache, page_table, len_k, cu_q=None, mask=MASK_CAUSAL, prefix=None, scale=None, cap=0.0, slopes=None, o=None,
                  row_absmax=None, ws=None, stream=None):
    """attention_f16 over the 8-bit cache: q fp16 [T_q, Hq, D], page_table int32 [B, max_pages], len_k int32 [B] -> o fp16 [T_q, Hq, D]."""
    c, B = cache.desc(page_table, len_k)
    dev = _current()
    _here(stream, dev)
    a, o = _attention_form(dev, q, B, cache.heads, cu_q, mask, prefix, scale, cap, slopes, o, row_absmax, stream)
    if q.shape[2] != cache.D:
        raise ValueError("q has heads of %d, the cache of %d" % (q.shape[2], cache.D))
    if ws is None:
        ws = workspace(attention_kv8_workspace_bytes(q.shape[0], B, q.shape[1], cache.heads, cache.D), q.device, stream)
    elif ws.get_device() != dev:
        _elsewhere(ws, "ws")
    _check(lib().attention_kv8(a, c, _ptr(ws), ws.numel(), _stream(stream)), "attention_kv8")
    return o


class Plan:
    """A per-layer weight-bit plan (Algorithm 2, Phase B): list of dicts(K, N, bits, w, w_scale, bias[, group]) of CUDA
    tensors; group = k per weight scale of a 4-bit layer (default 128)."""

    def __init__(self, layers, M_max):
        self._keep = layers  # the plan stores raw pointers: keep the tensors alive
        arr = (ql_layer_desc * len(layers))()
        for i, l in enumerate(layers):
            arr[i] = ql_layer_desc(l["K"], l["N"], l["bits"], l.get("group", 128) if l["bits"] == 4 else 0, l["w"].data_ptr(),
                                   0 if l.get("w_scale") is None else l["w_scale"].data_ptr(),
                                   0 if l.get("bias") is None else l["bias"].data_ptr())
        h = _vp()
        _check(lib().ql_plan_create(arr, len(layers), M_max, ctypes.byref(h)), "ql_plan_create")
        self.handle = h
        self.L = len(layers)
        self.M_max = M_max

    def workspace_bytes(self, M, R):
        return int(lib().ql_plan_workspace_bytes(self.handle, M, R))

    def run(self, x_in, y_out, M, R, ws, stream=None):
        """x_in / y_out: lists of L CUDA tensors ([M,K_l] fp16 / [M,N_l] fp16)."""
        xs = (_vp * self.L)(*[t.data_ptr() for t in x_in])
        ys = (_vp * self.L)(*[t.data_ptr() for t in y_out])
        _check(lib().qlinear_plan_run(self.handle, xs, ys, M, R, _ptr(ws), ws.numel(), _stream(stream)),
               "qlinear_plan_run")

    def run_ptrs(self, xs, ys, M, R, ws, stream_ptr):
        """Same with pre-marshalled pointer arrays (keeps Python out of a timed loop)."""
        _check(lib().qlinear_plan_run(self.handle, xs, ys, M, R, _ptr(ws), ws.numel(), stream_ptr), "qlinear_plan_run")

    def run_ptrs_robust(self, xs, ys, M, R, p_ppm, a_bits, ws, stream_ptr):
        prm = _DaqParams(p_ppm, a_bits)
        _check(lib().qlinear_plan_run_robust(self.handle, xs, ys, M, R, ctypes.byref(prm), _ptr(ws), ws.numel(), stream_ptr),
               "qlinear_plan_run_robust")

    def run_ex(self, x_in, y_out, M, R, ws, fusions=None, p_ppm=None, a_bits=8, stream=None):
        """The plan walk with optional percentile DAQ (p_ppm) and per-layer glue: fusions = list of None or
        dict(act, residual, gate, gate_rows) per layer."""
        xs = (_vp * self.L)(*[t.data_ptr() for t in x_in])
        ys = (_vp * self.L)(*[t.data_ptr() for t in y_out])
        prm = None if p_ppm is None else ctypes.byref(_DaqParams(p_ppm, a_bits))
        fus = None
        keep = []
        if fusions is not None:
            arr = (ctypes.POINTER(ql_fusion) * self.L)()
            for i, f in enumerate(fusions):
                if f is None:
                    continue
                fu = ql_fusion(f.get("act", 0), 0, None if f.get("residual") is None else f["residual"].data_ptr(),
                               None if f.get("gate") is None else f["gate"].data_ptr(), f.get("gate_rows", 1),
                               None if f.get("row_absmax") is None else f["row_absmax"].data_ptr())
                keep.append(fu)
                arr[i] = ctypes.pointer(fu)
            fus = arr
        _check(lib().qlinear_plan_run_ex(self.handle, xs, ys, M, R, prm, fus, _ptr(ws), ws.numel(), _stream(stream)),
               "qlinear_plan_run_ex")

    def close(self):
        if self.handle:
            lib().ql_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class ql_planner_layer(ctypes.Structure):
    _fields_ = [("n_options", ctypes.c_int32), ("reserved", ctypes.c_int32), ("bits", ctypes.POINTER(ctypes.c_int32)),
                ("c_lat", ctypes.POINTER(ctypes.c_double)), ("c_mem", ctypes.POINTER(ctypes.c_double)),
                ("sensitivity", ctypes.c_double)]


def schedule_topk(delta, candidates, T, rho_ppm, k):
    """Step 4, eq. (6): the k kept timesteps (ascending) = protected tail + the largest-delta steps of the rest."""
    import numpy as np
    d = np.ascontiguousarray(delta, dtype=np.float64)
    c = np.ascontiguousarray(candidates, dtype=np.int32)
    out = np.empty((max(k, 0),), np.int32)
    rc = lib().ql_schedule_topk(d.ctypes.data_as(_vp), c.ctypes.data_as(_vp), ctypes.c_int32(len(c)), ctypes.c_int32(T),
                                ctypes.c_int32(rho_ppm), ctypes.c_int32(k), out.ctypes.data_as(_vp))
    _check(rc, "ql_schedule_topk")
    return out


def plan_greedy(drift, c_step, layers, B_lat, B_mem, rho_ppm, eps=1e-12):
    """Algorithm 2, Phase A.  layers: list of dict(bits=[...], c_lat=[...], c_mem=[...], sensitivity=s).
    Returns dict(bits=[L], kept=[T] bool, C_lat, C_mem, feasible)."""
    import numpy as np
    dr = np.ascontiguousarray(drift, dtype=np.float64)
    cs = np.ascontiguousarray(c_step, dtype=np.float64)
    T, L = len(dr), len(layers)
    arr = (ql_planner_layer * L)()
    keep = []
    for i, l in enumerate(layers):
        b = np.ascontiguousarray(l["bits"], dtype=np.int32)
        cl = np.ascontiguousarray(l["c_lat"], dtype=np.float64)
        cm = np.ascontiguousarray(l["c_mem"], dtype=np.float64)
        keep += [b, cl, cm]
        arr[i] = ql_planner_layer(len(b), 0, b.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                                  cl.ctypes.data_as(ctypes.POINTER(ctypes.c_double)),
                                  cm.ctypes.data_as(ctypes.POINTER(ctypes.c_double)), float(l["sensitivity"]))
    bits = np.empty((L,), np.int32)
    kept = np.empty((T,), np.uint8)
    cl_out, cm_out, feas = ctypes.c_double(), ctypes.c_double(), ctypes.c_int32()
    fn = lib().ql_plan_greedy
    fn.argtypes = [_vp, _vp, ctypes.c_int32, ctypes.POINTER(ql_planner_layer), ctypes.c_int32, ctypes.c_double, ctypes.c_double,
                   ctypes.c_int32, ctypes.c_double, _vp, _vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double),
                   ctypes.POINTER(ctypes.c_int32)]
    rc = fn(dr.ctypes.data_as(_vp), cs.ctypes.data_as(_vp), T, arr, L, B_lat, B_mem, rho_ppm, eps, bits.ctypes.data_as(_vp),
            kept.ctypes.data_as(_vp), ctypes.byref(cl_out), ctypes.byref(cm_out), ctypes.byref(feas))
    _check(rc, "ql_plan_greedy")
    return dict(bits=bits, kept=kept.astype(bool), C_lat=cl_out.value, C_mem=cm_out.value, feasible=bool(feas.value))


def gptq_quantize_host(W, H, bits, group, symmetric=True, damp=0.01, scale_fp16=False):
    """Step 2, GPTQ: W fp32 [N,K], H float64 [K,K] -> (codes int8 [N,K], scales fp32 [N,K/group], zeros int32 [N,K/group])."""
    import numpy as np
    W = np.ascontiguousarray(W, dtype=np.float32)
    H = np.ascontiguousarray(H, dtype=np.float64)
    N, K = W.shape
    codes = np.empty((N, K), np.int8)
    scales = np.empty((N, K // group), np.float32)
    zeros = np.zeros((N, K // group), np.int32)
    fn = lib().ql_gptq_quantize_host
    fn.argtypes = [_vp, _i64, _i64, _vp, ctypes.c_int32, _i64, ctypes.c_int32, ctypes.c_double, ctypes.c_int32, _vp, _vp, _vp]
    rc = fn(W.ctypes.data_as(_vp), N, K, H.ctypes.data_as(_vp), bits, group, 1 if symmetric else 0, damp, 1 if scale_fp16 else 0,
            codes.ctypes.data_as(_vp), scales.ctypes.data_as(_vp), zeros.ctypes.data_as(_vp))
    _check(rc, "ql_gptq_quantize_host")
    return codes, scales, zeros


def set_gemm_variant(v):
    _check(lib().ql_set_gemm_variant(v), "ql_set_gemm_variant")


def gemm_variants():
    L = lib()
    return [L.ql_gemm_variant_name(i).decode() for i in range(L.ql_num_gemm_variants())]


def prepack_w4(pairs, stream=None):
    """Device uint8 [N,K/2] in pair order (low nibble = even k, high nibble = odd k) -> a new device tensor in the
    library's 4-bit storage order."""
    N, K2 = pairs.shape
    out = _empty(pairs.shape, pairs.dtype, pairs.device, stream, True)
    _check(lib().ql_prepack_w4(_ptr(pairs), N, K2 * 2, _ptr(out), _stream(stream)), "ql_prepack_w4")
    return out


def ql_repack_w4_pairs_host(pairs):
    """uint8 [N,K/2] in pair order (low nibble = even k, high nibble = odd k) -> the library's 4-bit storage order."""
    import numpy as np
    pairs = np.ascontiguousarray(pairs, dtype=np.uint8)
    N, K2 = pairs.shape
    out = np.empty_like(pairs)
    _check(lib().ql_repack_w4_pairs_host(pairs.ctypes.data_as(_vp), N, K2 * 2, out.ctypes.data_as(_vp)), "ql_repack_w4_pairs_host")
    return out
