"""Thin binding of libqmm.so (include/qmm.h).  Argument marshalling only: every step of the path runs in the HIP kernels.
torch is used for device memory and the current stream.  All calls go through ctypes; quantized_operand, scale_quantize, gemm,
metric and the operators around a feed-forward block first try the native short path for plain tensors (csrc/qmm_host.cpp), which does
the same with a fifth of the host time.  There is no CPU fallback: a missing or unloadable library raises."""
import collections
import ctypes
import importlib.util
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqmm.so")
HOST_PATH = os.path.join(_HERE, "_qmm_host.so")

INT8, E4M3, E5M2, BF16 = 0, 1, 2, 3
DT_BF16, DT_F32 = 0, 1
RTNE, STOCHASTIC = 0, 1
SILU, GELU = 0, 1
FORMATS = {"int8": INT8, "e4m3": E4M3, "e5m2": E5M2, "bf16": BF16}
EXPORTS = ["qmm_num_scales", "qmm_scale_workspace_size", "qmm_scale", "qmm_scale_static", "qmm_quantize", "qmm_scale_quantize_workspace_size", "qmm_scale_quantize", "qmm_scale_multi_workspace_size", "qmm_scale_multi", "qmm_quantize_multi",
           "qmm_gemm_workspace_size",
           "qmm_gemm", "qmm_gemm_nsr_workspace_size", "qmm_gemm_nsr", "qmm_metric_workspace_size", "qmm_metric", "qmm_dequantize", "qmm_rmsnorm_quantize", "qmm_rmsnorm_backward_workspace_size", "qmm_rmsnorm_backward", "qmm_gemm_gated_workspace_size", "qmm_gemm_gated", "qmm_gated_backward",
           "qmm_num_block_scales", "qmm_quantize_blocks", "qmm_gemm_blocks_workspace_size", "qmm_gemm_blocks", "qmm_dropout", "qmm_layernorm_quantize",
           "qmm_layernorm_backward_workspace_size", "qmm_layernorm_backward",
           "qmm_moments_workspace_size", "qmm_moments", "qmm_mfma_rate", "qmm_hbm_rate", "qmm_status_string", "qmm_version"]


class QmmError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: status {status} ({status_string(status)})")


class Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("contract_axis", ctypes.c_int32),
                ("batch", ctypes.c_int64), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("batch_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


class Granularity(ctypes.Structure):
    _fields_ = [("per_channel", ctypes.c_int32), ("batch_inner", ctypes.c_int32), ("batch_groups", ctypes.c_int64)]


class Operand(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("format", ctypes.c_int32), ("is_codes", ctypes.c_int32),
                ("delta", ctypes.c_void_p), ("gran", Granularity)]


class BlockOperand(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("format", ctypes.c_int32), ("block_rows", ctypes.c_int32), ("delta", ctypes.c_void_p)]


_lib = None
_short = None


class _NoShortPath:
    """Stands for a native short path that was not built: every call goes through ctypes."""
    @staticmethod
    def _decline(*_):
        return None
    scale_quantize = quantized_operand = gemm = metric = rmsnorm_quantize = rmsnorm_backward = gemm_gated = gated_backward = _decline
    quantize_blocks = gemm_blocks = dropout = layernorm_quantize = layernorm_backward = _decline


def _host():
    """Load the native short path (_qmm_host.so, built with libqmm.so).  It saves host time only: where it has not been built the
    calls go through ctypes, to the same kernels; one that is there and cannot be loaded raises."""
    global _short
    if _short is None:
        lib()
        if not os.path.exists(HOST_PATH):
            _short = _NoShortPath
            return _short
        spec = importlib.util.spec_from_file_location("_qmm_host", HOST_PATH)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.setup(Operand)
        module.setup_blocks(BlockOperand)
        _short = module
    return _short


def lib():
    """Load libqmm.so (built in-tree by paper_2408_02897_amd.build).  Raises if it is absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2408_02897_amd.build` first "
                               "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, u64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_uint64, ctypes.c_int, ctypes.c_size_t
        TP, GP, OP = ctypes.POINTER(Tensor), ctypes.POINTER(Granularity), ctypes.POINTER(Operand)
        L.qmm_num_scales.restype = i64; L.qmm_num_scales.argtypes = [TP, GP]
        L.qmm_scale_workspace_size.restype = sz; L.qmm_scale_workspace_size.argtypes = [TP, GP]
        L.qmm_scale.restype = i32; L.qmm_scale.argtypes = [TP, i32, GP, vp, vp, sz, vp]
        L.qmm_scale_static.restype = i32; L.qmm_scale_static.argtypes = [TP, i32, GP, vp, vp]
        L.qmm_quantize.restype = i32; L.qmm_quantize.argtypes = [TP, i32, GP, vp, i32, u64, u64, vp, vp]
        L.qmm_scale_quantize_workspace_size.restype = sz; L.qmm_scale_quantize_workspace_size.argtypes = [TP, GP]
        L.qmm_scale_quantize.restype = i32; L.qmm_scale_quantize.argtypes = [TP, i32, GP, i32, u64, u64, vp, vp, vp, sz, vp]
        L.qmm_scale_multi_workspace_size.restype = sz; L.qmm_scale_multi_workspace_size.argtypes = [i32, vp, vp]
        L.qmm_scale_multi.restype = i32; L.qmm_scale_multi.argtypes = [i32, vp, i32, vp, vp, vp, sz, vp]
        L.qmm_quantize_multi.restype = i32; L.qmm_quantize_multi.argtypes = [i32, vp, i32, vp, vp, i32, u64, vp, vp, vp]
        L.qmm_gemm_workspace_size.restype = sz; L.qmm_gemm_workspace_size.argtypes = [OP, OP, i64, i64, i64, i64]
        L.qmm_gemm.restype = i32; L.qmm_gemm.argtypes = [OP, OP, i64, i64, i64, i64, vp, i32, vp, vp, sz, vp]
        L.qmm_gemm_nsr_workspace_size.restype = sz; L.qmm_gemm_nsr_workspace_size.argtypes = [i64, i64, i64]
        L.qmm_gemm_nsr.restype = i32; L.qmm_gemm_nsr.argtypes = [OP, OP, i64, i64, i64, i64, vp, i32, vp, vp, vp, sz, vp]
        L.qmm_metric_workspace_size.restype = sz; L.qmm_metric_workspace_size.argtypes = [i64]
        L.qmm_metric.restype = i32; L.qmm_metric.argtypes = [vp, i32, vp, vp, i64, vp, vp, sz, vp]
        L.qmm_dequantize.restype = i32; L.qmm_dequantize.argtypes = [vp, i64, i64, i64, i32, GP, vp, vp, i32, vp]
        L.qmm_rmsnorm_quantize.restype = i32; L.qmm_rmsnorm_quantize.argtypes = [TP, TP, vp, i32, ctypes.c_float, i32, i32, u64, u64, vp, vp, vp, vp, vp, vp]
        L.qmm_rmsnorm_backward_workspace_size.restype = sz; L.qmm_rmsnorm_backward_workspace_size.argtypes = [TP]
        L.qmm_rmsnorm_backward.restype = i32; L.qmm_rmsnorm_backward.argtypes = [TP, TP, vp, vp, i32, TP, vp, vp, vp, sz, vp]
        L.qmm_gemm_gated_workspace_size.restype = sz; L.qmm_gemm_gated_workspace_size.argtypes = [OP, OP, i64, i64, i64, i64]
        L.qmm_gemm_gated.restype = i32; L.qmm_gemm_gated.argtypes = [OP, OP, i64, i64, i64, i64, i32, vp, vp, i32, vp, sz, vp]
        L.qmm_gated_backward.restype = i32; L.qmm_gated_backward.argtypes = [TP, TP, i32, i32, i32, u64, u64, vp, vp, vp, vp]
        BP, f32 = ctypes.POINTER(BlockOperand), ctypes.c_float
        L.qmm_num_block_scales.restype = i64; L.qmm_num_block_scales.argtypes = [i64, i64, i64, i32]
        L.qmm_quantize_blocks.restype = i32; L.qmm_quantize_blocks.argtypes = [TP, i32, i32, i32, u64, u64, vp, vp, vp, vp, vp]
        L.qmm_gemm_blocks_workspace_size.restype = sz; L.qmm_gemm_blocks_workspace_size.argtypes = [i64, i64, i64, i64]
        L.qmm_gemm_blocks.restype = i32; L.qmm_gemm_blocks.argtypes = [BP, BP, i64, i64, i64, i64, vp, i32, vp, sz, vp]
        L.qmm_dropout.restype = i32; L.qmm_dropout.argtypes = [TP, f32, u64, u64, vp, vp]
        L.qmm_layernorm_quantize.restype = i32
        L.qmm_layernorm_quantize.argtypes = [TP, TP, vp, vp, i32, f32, f32, u64, u64, i32, i32, i32, u64, u64, vp, vp, vp, vp, vp, vp, vp]
        L.qmm_layernorm_backward_workspace_size.restype = sz; L.qmm_layernorm_backward_workspace_size.argtypes = [TP]
        L.qmm_layernorm_backward.restype = i32; L.qmm_layernorm_backward.argtypes = [TP, TP, vp, vp, vp, i32, TP, f32, u64, u64, vp, vp, vp, vp, vp, sz, vp]
        L.qmm_moments_workspace_size.restype = sz; L.qmm_moments_workspace_size.argtypes = [i64]
        L.qmm_moments.restype = i32; L.qmm_moments.argtypes = [vp, i32, i64, ctypes.c_double, vp, vp, sz, vp]
        L.qmm_mfma_rate.restype = i32
        L.qmm_mfma_rate.argtypes = [i32, i32, vp, i64, i64, i32, vp, ctypes.POINTER(ctypes.c_double), vp]
        L.qmm_hbm_rate.restype = i32; L.qmm_hbm_rate.argtypes = [vp, vp, i64, i32, vp, vp]
        L.qmm_status_string.restype = ctypes.c_char_p; L.qmm_status_string.argtypes = [i32]
        L.qmm_version.restype = i32; L.qmm_version.argtypes = []
        _lib = L
    return _lib


def status_string(status):
    return lib().qmm_status_string(int(status)).decode()


def _check(status, where):
    if status != 0:
        raise QmmError(status, where)


def _stream():
    """The current stream's handle as a number (what torch.cuda.current_stream().cuda_stream is, without the Stream object
    made for it: 0.2 instead of 3.1 us, on every call)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return DT_BF16
    if t.dtype == torch.float32:
        return DT_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def tensor_desc(x, contract_axis):
    """Descriptor of a 2-D [rows, cols] or 3-D [batch, rows, cols] device tensor with contiguous columns."""
    shape, stride = x.shape, x.stride()
    assert len(shape) in (2, 3) and x.is_cuda
    if len(shape) == 2:
        (r, c), b, batch_stride = shape, 1, shape[0] * stride[0]
    else:
        (b, r, c), batch_stride = shape, stride[0]
    assert stride[-1] == 1 or c <= 1, "columns must be contiguous"
    return Tensor(x.data_ptr(), _dtype_code(x), contract_axis, b, r, c, batch_stride, stride[-2])


def granularity(per_channel=False, batch_groups=1, batch_inner=1):
    """Scale group of matrix b: (b // batch_inner) % batch_groups."""
    return Granularity(int(per_channel), int(batch_inner), int(batch_groups))


def _workspace(nbytes, device):
    return torch.empty(max(int(nbytes), 16), dtype=torch.uint8, device=device)


def _scratch(nbytes, device):
    """(tensor to keep until the call is enqueued, pointer, size) of a workspace; nothing is allocated for none."""
    if nbytes == 0:
        return None, None, 0
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return ws, ws.data_ptr(), nbytes


def scale(x, contract_axis, fmt, per_channel=False, batch_groups=1, out=None, workspace=None, batch_inner=1):
    """qmm_scale: step sizes (float32 device tensor of qmm_num_scales elements)."""
    L = lib()
    t, g = tensor_desc(x, contract_axis), granularity(per_channel, batch_groups, batch_inner)
    n = L.qmm_num_scales(ctypes.byref(t), ctypes.byref(g))
    if out is None:
        out = torch.empty(n, dtype=torch.float32, device=x.device)
    need = L.qmm_scale_workspace_size(ctypes.byref(t), ctypes.byref(g))
    if workspace is None:
        workspace = _workspace(need, x.device)
    _check(L.qmm_scale(ctypes.byref(t), fmt, ctypes.byref(g), out.data_ptr(), workspace.data_ptr(),
                       workspace.numel(), _stream()), "qmm_scale")
    return out


def scale_static(x, contract_axis, fmt, per_channel=False, batch_groups=1, out=None, batch_inner=1):
    """qmm_scale_static: qmm_scale with the library's own scratch array (no workspace, nothing allocated by the call
    itself when `out` is given)."""
    L = lib()
    t, g = tensor_desc(x, contract_axis), granularity(per_channel, batch_groups, batch_inner)
    if out is None:
        out = torch.empty(L.qmm_num_scales(ctypes.byref(t), ctypes.byref(g)), dtype=torch.float32, device=x.device)
    _check(L.qmm_scale_static(ctypes.byref(t), fmt, ctypes.byref(g), out.data_ptr(), _stream()), "qmm_scale_static")
    return out


def quantize(x, contract_axis, fmt, delta, per_channel=False, batch_groups=1, mode=RTNE, seed=0, offset=0, out=None,
             batch_inner=1):
    """qmm_quantize: uint8 codes [batch, non-contracting, contracting]."""
    L = lib()
    t, g = tensor_desc(x, contract_axis), granularity(per_channel, batch_groups, batch_inner)
    nc, kc = (t.rows, t.cols) if contract_axis == 1 else (t.cols, t.rows)
    if out is None:
        out = torch.empty((t.batch, nc, kc), dtype=torch.uint8, device=x.device)
    assert delta.dtype == torch.float32 and delta.numel() == L.qmm_num_scales(ctypes.byref(t), ctypes.byref(g))
    _check(L.qmm_quantize(ctypes.byref(t), fmt, ctypes.byref(g), delta.data_ptr(), mode, seed, offset,
                          out.data_ptr(), _stream()), "qmm_quantize")
    return out


class MultiDesc:
    """Host-side argument arrays of qmm_scale_multi / qmm_quantize_multi for a fixed list of tensors (built once,
    reused: the arrays hold raw pointers, the object keeps their owners alive)."""
    def __init__(self, xs, contract_axis=1, per_channel=False, batch_groups=1):
        n = len(xs)
        self.count = n
        self.t = (Tensor * n)(*[tensor_desc(x, contract_axis) for x in xs])
        self.g = (Granularity * n)(*[granularity(per_channel, batch_groups) for _ in xs])
        self._keep = list(xs)
        self.device = xs[0].device
        self.shapes = [(d.batch, d.rows, d.cols) if contract_axis == 1 else (d.batch, d.cols, d.rows) for d in self.t]
        self.num_scales = [lib().qmm_num_scales(ctypes.byref(self.t[i]), ctypes.byref(self.g[i])) for i in range(n)]

    @staticmethod
    def pointers(tensors):
        arr = (ctypes.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])
        arr._keep = list(tensors)
        return arr


def scale_multi(desc, fmt, outs=None, workspace=None, out_ptrs=None):
    """qmm_scale_multi on a MultiDesc: list of step-size tensors."""
    L = lib()
    if outs is None:
        outs = [torch.empty(n, dtype=torch.float32, device=desc.device) for n in desc.num_scales]
    if out_ptrs is None:
        out_ptrs = MultiDesc.pointers(outs)
    if workspace is None:
        workspace = _workspace(L.qmm_scale_multi_workspace_size(desc.count, desc.t, desc.g), desc.device)
    _check(L.qmm_scale_multi(desc.count, desc.t, fmt, desc.g, out_ptrs, workspace.data_ptr(), workspace.numel(), _stream()),
           "qmm_scale_multi")
    return outs


def quantize_multi(desc, fmt, deltas, mode=RTNE, seed=0, offsets=None, outs=None, delta_ptrs=None, out_ptrs=None):
    """qmm_quantize_multi on a MultiDesc: list of uint8 code tensors."""
    L = lib()
    if outs is None:
        outs = [torch.empty(s, dtype=torch.uint8, device=desc.device) for s in desc.shapes]
    if delta_ptrs is None:
        delta_ptrs = MultiDesc.pointers(deltas)
    if out_ptrs is None:
        out_ptrs = MultiDesc.pointers(outs)
    offs = (ctypes.c_uint64 * desc.count)(*offsets) if offsets is not None else None
    _check(L.qmm_quantize_multi(desc.count, desc.t, fmt, desc.g, delta_ptrs, mode, seed, offs, out_ptrs, _stream()),
           "qmm_quantize_multi")
    return outs


def operand(data, fmt, delta=None, per_channel=False, batch_groups=1, is_codes=True, batch_inner=1):
    assert data.is_contiguous()
    op = Operand(data.data_ptr(), fmt, int(is_codes), delta.data_ptr() if delta is not None else None,
                 granularity(per_channel, batch_groups, batch_inner))
    op._keep = (data, delta)   # the struct holds raw device pointers: keep their owners alive with it
    return op


def gemm(a, b, out_dtype=torch.float32, want_acc=False, out=None, acc_out=None, want_y=True):
    """qmm_gemm on two (data, Operand) pairs built by `operand`: a = (tensor [batch,M,K], Operand) etc.
    Returns y (and the raw accumulators when want_acc)."""
    if want_y and not want_acc and acc_out is None:
        r = (_short or _host()).gemm(a, b, out_dtype, out)
        if type(r) is int:
            _check(r, "qmm_gemm")
        if r is not None:
            return r
    L = lib()
    (ta, oa), (tb, ob) = a, b
    sa, sb = ta.shape, tb.shape
    if len(sa) == 2:
        sa, sb = (1, *sa), (1, *sb)
    bt, m, k = sa
    n = sb[1]
    assert sb[0] == bt and sb[2] == k
    dev = ta.device
    y = out
    if y is None and want_y:
        y = torch.empty((bt, m, n), dtype=out_dtype, device=dev)
    acc = acc_out
    if acc is None and want_acc:
        acc = torch.empty((bt, m, n), dtype=torch.int32 if oa.format == INT8 else torch.float32, device=dev)
    pa, pb = ctypes.byref(oa), ctypes.byref(ob)
    ws, ws_ptr, ws_bytes = _scratch(L.qmm_gemm_workspace_size(pa, pb, bt, m, n, k), dev)
    ydt = DT_BF16 if (y is not None and y.dtype == torch.bfloat16) else DT_F32
    _check(L.qmm_gemm(pa, pb, bt, m, n, k, y.data_ptr() if y is not None else None, ydt,
                      acc.data_ptr() if acc is not None else None, ws_ptr, ws_bytes, _stream()), "qmm_gemm")
    return (y, acc) if want_acc else y


def gemm_nsr(a, b, y_ref, out_dtype=torch.bfloat16, out=None, out2=None, workspace=None):
    """qmm_gemm_nsr: y as `gemm` gives it, and a device tensor of 2 float64: sum (y - y_ref)^2, sum y_ref^2."""
    L = lib()
    (ta, oa), (tb, ob) = a, b
    if ta.dim() == 2:
        ta = ta.unsqueeze(0); tb = tb.unsqueeze(0)
    bt, m, k = ta.shape
    n = tb.shape[1]
    assert tb.shape[0] == bt and tb.shape[2] == k
    assert y_ref.dtype == torch.float32 and y_ref.is_contiguous() and y_ref.numel() == bt * m * n
    dev = ta.device
    y = out if out is not None else torch.empty((bt, m, n), dtype=out_dtype, device=dev)
    if out2 is None:
        out2 = torch.empty(2, dtype=torch.float64, device=dev)
    ws = workspace if workspace is not None else _workspace(L.qmm_gemm_nsr_workspace_size(bt, m, n), dev)
    ydt = DT_BF16 if y.dtype == torch.bfloat16 else DT_F32
    _check(L.qmm_gemm_nsr(ctypes.byref(oa), ctypes.byref(ob), bt, m, n, k, y.data_ptr(), ydt, y_ref.data_ptr(),
                          out2.data_ptr(), ws.data_ptr(), ws.numel(), _stream()), "qmm_gemm_nsr")
    return y, out2


def scale_quantize(x, contract_axis, fmt, per_channel=False, batch_groups=1, mode=RTNE, seed=0, offset=0, batch_inner=1):
    """qmm_scale_quantize: (uint8 codes [batch, non-contracting, contracting], step sizes) as scale and quantize give them."""
    r = (_short or _host()).scale_quantize(x, contract_axis, fmt, per_channel, batch_groups, mode, seed, offset, batch_inner)
    if type(r) is int:
        _check(r, "qmm_scale_quantize")
    if r is not None:
        return r
    L = lib()
    t, g = tensor_desc(x, contract_axis), granularity(per_channel, batch_groups, batch_inner)
    nc, kc = (t.rows, t.cols) if contract_axis == 1 else (t.cols, t.rows)
    dev = x.device
    delta = torch.empty(batch_groups * (nc if per_channel else 1), dtype=torch.float32, device=dev)     # qmm_num_scales
    codes = torch.empty((t.batch, nc, kc), dtype=torch.uint8, device=dev)
    tp, gp = ctypes.byref(t), ctypes.byref(g)
    ws, ws_ptr, ws_bytes = _scratch(L.qmm_scale_quantize_workspace_size(tp, gp), dev)
    _check(L.qmm_scale_quantize(tp, fmt, gp, mode, seed, offset, delta.data_ptr(), codes.data_ptr(), ws_ptr, ws_bytes, _stream()),
           "qmm_scale_quantize")
    return codes, delta


def quantized_operand(x, contract_axis, fmt, per_channel=False, batch_groups=1, mode=RTNE, seed=0, batch_inner=1):
    """scale + quantize; returns ((codes, Operand), delta)."""
    r = (_short or _host()).quantized_operand(x, contract_axis, fmt, per_channel, batch_groups, mode, seed, 0, batch_inner)
    if type(r) is int:
        _check(r, "qmm_scale_quantize")
    if r is not None:
        return r
    c, d = scale_quantize(x, contract_axis, fmt, per_channel, batch_groups, mode, seed, batch_inner=batch_inner)
    return (c, operand(c, fmt, d, per_channel, batch_groups, batch_inner=batch_inner)), d


def reference_gemm(x, w, out=None):
    """High-precision product of bfloat16 operands x [batch,M,K], w [batch,N,K] -> float32."""
    assert x.dtype == torch.bfloat16 and w.dtype == torch.bfloat16
    x = x.contiguous(); w = w.contiguous()
    return gemm((x, operand(x, BF16, is_codes=False)), (w, operand(w, BF16, is_codes=False)), torch.float32, out=out)


def metric(y, y_ref, denom=None, out=None, workspace=None):
    """qmm_metric: 16 float64 on the device (layout in include/qmm.h)."""
    r = (_short or _host()).metric(y, y_ref, denom, out, workspace)
    if type(r) is int:
        _check(r, "qmm_metric")
    if r is not None:
        return r
    L = lib()
    assert y.is_contiguous() and y_ref.is_contiguous() and y_ref.dtype == torch.float32
    n = y.numel()
    assert y_ref.numel() == n and (denom is None or (denom.numel() == n and denom.dtype == torch.float32))
    if out is None:
        out = torch.empty(16, dtype=torch.float64, device=y.device)
    if workspace is None:
        workspace = _workspace(L.qmm_metric_workspace_size(n), y.device)
    _check(L.qmm_metric(y.data_ptr(), _dtype_code(y), y_ref.data_ptr(), denom.data_ptr() if denom is not None else None,
                        n, out.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream()), "qmm_metric")
    return out


def dequantize(codes, fmt, delta, per_channel=False, batch_groups=1, out_dtype=torch.float32, out=None, batch_inner=1):
    """qmm_dequantize: values of the uint8 device tensor codes [batch, rows, K] (or [rows, K])."""
    L = lib()
    assert codes.dtype == torch.uint8 and codes.is_contiguous() and codes.is_cuda
    c3 = codes if codes.dim() == 3 else codes.unsqueeze(0)
    b, r, k = c3.shape
    g = granularity(per_channel, batch_groups, batch_inner)
    assert delta.dtype == torch.float32 and delta.numel() == batch_groups * (r if per_channel else 1)
    if out is None:
        out = torch.empty(codes.shape, dtype=out_dtype, device=codes.device)
    _check(L.qmm_dequantize(codes.data_ptr(), b, r, k, fmt, ctypes.byref(g), delta.data_ptr(), out.data_ptr(),
                            _dtype_code(out), _stream()), "qmm_dequantize")
    return out


# ---- around a feed-forward block: what stands in front of and between its products

Normed = collections.namedtuple("Normed", "codes delta h y rstd")
GatedGradient = collections.namedtuple("GatedGradient", "codes delta dgu")


def _row_desc(x, shape=None, dtype=None):
    """tensor_desc of a tensor of rows, after the checks that the library cannot make: extents and type of another tensor."""
    assert shape is None or tuple(x.shape) == tuple(shape), f"shape {tuple(x.shape)}, not {tuple(shape)}"
    assert dtype is None or x.dtype == dtype, f"{x.dtype}, not {dtype}"
    return tensor_desc(x, 1)


def _on(device, *tensors):
    """Kernels run on the current device's stream: all tensors of a call are there."""
    for t in tensors:
        if t is not None and (not t.is_cuda or t.device.index != torch._C._cuda_getDevice()):
            raise ValueError(f"a tensor on {t.device}, which is not the current GPU")
    return device


def _dense_out(t, shape, dtype):
    assert t.is_contiguous() and tuple(t.shape) == tuple(shape) and t.dtype == dtype, "an output is contiguous, of its shape and type"
    return t


def _weight_args(weight, cols):
    if weight is None:
        return None, DT_F32
    assert weight.shape == (cols,) and weight.is_contiguous(), "one weight per column"
    return weight.data_ptr(), _dtype_code(weight)


def rmsnorm_quantize(x, weight, fmt, residual=None, eps=1e-6, mode=RTNE, seed=0, offset=0, want_y=False, want_rstd=False, h_out=None):
    """qmm_rmsnorm_quantize on [rows, cols] or [batch, rows, cols]: Normed(codes [batch, rows, cols], delta, h, y, rstd).  codes and delta are an
    operand with per_channel=True and batch_groups=batch; h is x + residual (x without one), y and rstd are None unless wanted.
    `h_out`: where h goes, e.g. the residual itself."""
    r = (_short or _host()).rmsnorm_quantize(x, weight, fmt, residual, eps, mode, seed, offset, want_y, want_rstd, h_out)
    if type(r) is int:
        _check(r, "qmm_rmsnorm_quantize")
    if r is not None:
        return Normed._make(r)
    L = lib()
    dev = _on(x.device, x, weight, residual, h_out)
    t = _row_desc(x)
    r = None if residual is None else _row_desc(residual, x.shape, x.dtype)
    w_ptr, w_type = _weight_args(weight, t.cols)
    h = x
    if residual is not None:
        h = torch.empty(x.shape, dtype=x.dtype, device=dev) if h_out is None else _dense_out(h_out, x.shape, x.dtype)
    else:
        assert h_out is None, "without a residual h is x"
    codes = torch.empty((t.batch, t.rows, t.cols), dtype=torch.uint8, device=dev)
    delta = torch.empty(t.batch * t.rows, dtype=torch.float32, device=dev)
    y = torch.empty(x.shape, dtype=x.dtype, device=dev) if want_y else None
    rstd = torch.empty(t.batch * t.rows, dtype=torch.float32, device=dev) if want_rstd else None
    _check(L.qmm_rmsnorm_quantize(ctypes.byref(t), None if r is None else ctypes.byref(r), w_ptr, w_type, eps, fmt, mode, seed, offset,
                                  None if r is None else h.data_ptr(), None if y is None else y.data_ptr(), None if rstd is None else rstd.data_ptr(),
                                  delta.data_ptr(), codes.data_ptr(), _stream()), "qmm_rmsnorm_quantize")
    return Normed(codes, delta, h, y, rstd)


def rmsnorm_backward(dy, h, rstd, weight, dresidual=None, want_dw=True, dx_out=None):
    """qmm_rmsnorm_backward: (dx, dw); dw is float32, or None unless wanted.  `dx_out`: where dx goes, e.g. dy itself."""
    r = (_short or _host()).rmsnorm_backward(dy, h, rstd, weight, dresidual, want_dw, dx_out)
    if type(r) is int:
        _check(r, "qmm_rmsnorm_backward")
    if r is not None:
        return r
    L = lib()
    dev = _on(dy.device, dy, h, rstd, weight, dresidual, dx_out)
    t, th = _row_desc(dy), _row_desc(h, dy.shape, dy.dtype)
    r = None if dresidual is None else _row_desc(dresidual, dy.shape, dy.dtype)
    w_ptr, w_type = _weight_args(weight, t.cols)
    assert rstd.dtype == torch.float32 and rstd.is_contiguous() and rstd.numel() == t.batch * t.rows, "one rstd per row"
    dx = torch.empty(dy.shape, dtype=dy.dtype, device=dev) if dx_out is None else _dense_out(dx_out, dy.shape, dy.dtype)
    dw = torch.empty(t.cols, dtype=torch.float32, device=dev) if want_dw else None
    ws, ws_ptr, ws_bytes = _scratch(L.qmm_rmsnorm_backward_workspace_size(ctypes.byref(t)) if want_dw else 0, dev)
    _check(L.qmm_rmsnorm_backward(ctypes.byref(t), ctypes.byref(th), rstd.data_ptr(), w_ptr, w_type, None if r is None else ctypes.byref(r),
                                  dx.data_ptr(), None if dw is None else dw.data_ptr(), ws_ptr, ws_bytes, _stream()), "qmm_rmsnorm_backward")
    return dx, dw


def _check_operand(t, op, batch, rows):
    """An operand reads what its tensor holds: the same memory, elements of its format, a step size for every row of every group (of an operand made by
    `operand` or quantized_operand, which know their tensors).  What the library refuses itself is left to it."""
    if (op.data or 0) != t.data_ptr() or not t.is_contiguous():
        raise ValueError("an operand of another tensor")
    if (op.format == BF16 or op.is_codes) and t.element_size() != (2 if op.format == BF16 else 1):
        raise ValueError(f"{t.dtype} in an operand of format {op.format}")
    delta = getattr(op, "_keep", (None, None))[1]
    if delta is None:
        return
    groups = min(op.gran.batch_groups, (batch - 1) // max(op.gran.batch_inner, 1) + 1)
    need = max(groups, 0) * (rows if op.gran.per_channel else 1)
    if delta.dtype != torch.float32 or not delta.is_contiguous() or delta.numel() < need or (op.delta or 0) != delta.data_ptr():
        raise ValueError(f"{delta.numel()} step sizes of {delta.dtype}, not {need} of float32 side by side")
    _on(t.device, delta)


def gemm_gated(a, b, activation=SILU, out_dtype=torch.bfloat16, want_gu=False):
    """qmm_gemm_gated on two (data, Operand) pairs as `gemm` takes them, b = ([batch, 2 F, K], Operand) with the gate's rows first:
    h [batch, M, F], or (h, gu [batch, M, 2 F]) when want_gu.  An operand that describes more than its tensors hold: ValueError."""
    r = (_short or _host()).gemm_gated(a, b, activation, out_dtype, want_gu)
    if type(r) is int:
        _check(r, "qmm_gemm_gated")
    if r is not None:
        return r if want_gu else r[0]
    L = lib()
    (ta, oa), (tb, ob) = a, b
    dev = _on(ta.device, ta, tb)
    sa, sb = ta.shape, tb.shape
    if len(sa) == 2:
        sa, sb = (1, *sa), (1, *sb)
    bt, m, k = sa
    assert len(sb) == 3 and sb[0] == bt and sb[2] == k and sb[1] % 2 == 0, "b is [batch, 2 F, K]"
    f = sb[1] // 2
    _check_operand(ta, oa, bt, m)
    _check_operand(tb, ob, bt, 2 * f)
    h = torch.empty((bt, m, f), dtype=out_dtype, device=dev)
    gu = torch.empty((bt, m, 2 * f), dtype=out_dtype, device=dev) if want_gu else None
    pa, pb = ctypes.byref(oa), ctypes.byref(ob)
    ws, ws_ptr, ws_bytes = _scratch(L.qmm_gemm_gated_workspace_size(pa, pb, bt, m, f, k), dev)
    _check(L.qmm_gemm_gated(pa, pb, bt, m, f, k, activation, h.data_ptr(), None if gu is None else gu.data_ptr(), _dtype_code(h),
                            ws_ptr, ws_bytes, _stream()), "qmm_gemm_gated")
    return (h, gu) if want_gu else h


def gated_backward(dh, gu, activation=SILU, fmt=E5M2, mode=RTNE, seed=0, offset=0, want_codes=True, want_dgu=False, dgu_out=None):
    """qmm_gated_backward on dh [.., F] and gu [.., 2 F]: GatedGradient(codes [batch, rows, 2 F], delta, dgu), None for what is not wanted.
    codes and delta are an operand with per_channel=True and batch_groups=batch.  `dgu_out`: where dgu goes, e.g. gu itself."""
    r = (_short or _host()).gated_backward(dh, gu, activation, fmt, mode, seed, offset, want_codes, want_dgu, dgu_out)
    if type(r) is int:
        _check(r, "qmm_gated_backward")
    if r is not None:
        return GatedGradient._make(r)
    L = lib()
    dev = _on(dh.device, dh, gu, dgu_out)
    t, tg = _row_desc(dh), _row_desc(gu, (*dh.shape[:-1], 2 * dh.shape[-1]), dh.dtype)
    codes = torch.empty((t.batch, t.rows, 2 * t.cols), dtype=torch.uint8, device=dev) if want_codes else None
    delta = torch.empty(t.batch * t.rows, dtype=torch.float32, device=dev) if want_codes else None
    dgu = None
    if dgu_out is not None:
        dgu = _dense_out(dgu_out, gu.shape, gu.dtype)
    elif want_dgu:
        dgu = torch.empty(gu.shape, dtype=gu.dtype, device=dev)
    assert codes is not None or dgu is not None, "nothing is wanted"
    _check(L.qmm_gated_backward(ctypes.byref(t), ctypes.byref(tg), activation, fmt, mode, seed, offset, None if dgu is None else dgu.data_ptr(),
                                None if delta is None else delta.data_ptr(), None if codes is None else codes.data_ptr(), _stream()), "qmm_gated_backward")
    return GatedGradient(codes, delta, dgu)


# ---- layers whose products have a step size for every block of 128

BLOCK = 128
LayerNormed = collections.namedtuple("LayerNormed", "codes delta h y mean rstd")
LayerNormGradient = collections.namedtuple("LayerNormGradient", "dh dx dw db")


def _block_scales(batch, rows, k, block_rows):
    return (batch, -(-k // BLOCK), -(-rows // max(int(block_rows), 1)))


def quantize_blocks(x, contract_axis, fmt, block_rows=1, mode=RTNE, seed=0, offset=0, both=False):
    """qmm_quantize_blocks on [rows, cols] or [batch, rows, cols]: (codes [batch, non-contracting, contracting], delta [batch, blocks of 128 along the
    contracting axis, rows of blocks]).  `both`: a pair of such pairs, the second one contracted over the other axis."""
    r = (_short or _host()).quantize_blocks(x, contract_axis, fmt, block_rows, mode, seed, offset, both)
    if type(r) is int:
        _check(r, "qmm_quantize_blocks")
    if r is not None:
        return (r[:2], r[2:]) if both else r
    L = lib()
    dev = _on(x.device, x)
    t = tensor_desc(x, contract_axis)
    if block_rows not in (1, BLOCK):
        raise ValueError("block_rows is 1 or 128")

    def outputs(axis):
        nc, kc = (t.rows, t.cols) if axis == 1 else (t.cols, t.rows)
        return (torch.empty((t.batch, nc, kc), dtype=torch.uint8, device=dev),
                torch.empty(_block_scales(t.batch, nc, kc, block_rows), dtype=torch.float32, device=dev))
    codes, delta = outputs(contract_axis)
    other = outputs(1 - contract_axis) if both else (None, None)
    _check(L.qmm_quantize_blocks(ctypes.byref(t), fmt, block_rows, mode, seed, offset, delta.data_ptr(), codes.data_ptr(),
                                 other[1].data_ptr() if both else None, other[0].data_ptr() if both else None, _stream()), "qmm_quantize_blocks")
    return ((codes, delta), other) if both else (codes, delta)


def block_operand(codes, fmt, delta, block_rows=1):
    """One side of gemm_blocks: uint8 codes [rows, K] or [batch, rows, K] and their step sizes as quantize_blocks gives them: [batch, blocks of 128 along K, rows of
    blocks], without its first axis for one matrix, or those values in a row.  (In another order, such as [rows, blocks], as many values are another matrix's.)"""
    if codes.dtype != torch.uint8 or codes.dim() not in (2, 3) or not codes.is_contiguous():
        raise ValueError("codes are a contiguous uint8 tensor [rows, K] or [batch, rows, K]")
    if block_rows not in (1, BLOCK):
        raise ValueError("block_rows is 1 or 128")
    batch, rows, k = codes.shape if codes.dim() == 3 else (1, *codes.shape)
    need = _block_scales(batch, rows, k, block_rows)
    shapes = (need, (need[0] * need[1] * need[2],), *([need[1:]] if batch == 1 else []))
    if delta.dtype != torch.float32 or not delta.is_contiguous() or tuple(delta.shape) not in shapes or delta.device != codes.device:
        raise ValueError(f"step sizes {tuple(delta.shape)} of {delta.dtype}, not {need} of float32 side by side on the codes' device")
    op = BlockOperand(codes.data_ptr(), fmt, block_rows, delta.data_ptr())
    op._keep = (codes, delta)
    return op


def _check_block_operand(t, op):
    """An operand reads what its tensors hold: the codes it was made for, and a step size for every block (block_rows may have been set since)."""
    codes, delta = getattr(op, "_keep", (None, None))
    if codes is None:
        raise ValueError("not an operand that block_operand made")
    need = _block_scales(*(codes.shape if codes.dim() == 3 else (1, *codes.shape)), op.block_rows)
    if op.block_rows in (1, BLOCK) and delta.numel() != need[0] * need[1] * need[2]:
        raise ValueError(f"{delta.numel()} step sizes, not {need}")
    if codes.data_ptr() != t.data_ptr() or codes.shape != t.shape or op.data != codes.data_ptr() or op.delta != delta.data_ptr():
        if t.numel():
            raise ValueError("an operand of another tensor")


def gemm_blocks(a, b, out_dtype=torch.float32, out=None):
    """qmm_gemm_blocks on two (codes, BlockOperand) pairs: y [batch, M, N]."""
    r = (_short or _host()).gemm_blocks(a, b, out_dtype, out)
    if type(r) is int:
        _check(r, "qmm_gemm_blocks")
    if r is not None:
        return r
    L = lib()
    (ta, oa), (tb, ob) = a, b
    dev = _on(ta.device, ta, tb, out)
    _check_block_operand(ta, oa)
    _check_block_operand(tb, ob)
    sa, sb = ta.shape, tb.shape
    if len(sa) == 2:
        sa, sb = (1, *sa), (1, *sb)
    bt, m, k = sa
    if len(sb) != 3 or sb[0] != bt or sb[2] != k:
        raise ValueError(f"operands {tuple(ta.shape)} and {tuple(tb.shape)}")
    n = sb[1]
    y = torch.empty((bt, m, n), dtype=out_dtype, device=dev) if out is None else _dense_out(out, (bt, m, n), out.dtype)
    ws, ws_ptr, ws_bytes = _scratch(L.qmm_gemm_blocks_workspace_size(bt, m, n, k), dev)
    _check(L.qmm_gemm_blocks(ctypes.byref(oa), ctypes.byref(ob), bt, m, n, k, y.data_ptr(), _dtype_code(y), ws_ptr, ws_bytes, _stream()), "qmm_gemm_blocks")
    return y


def dropout(x, p, seed, offset=0, out=None):
    """qmm_dropout of [rows, cols] or [batch, rows, cols]; the gradient is the same call on the upstream gradient.  `out`: where it goes, e.g. x itself."""
    r = (_short or _host()).dropout(x, p, seed, offset, out)
    if type(r) is int:
        _check(r, "qmm_dropout")
    if r is not None:
        return r
    L = lib()
    dev = _on(x.device, x, out)
    t = _row_desc(x)
    y = torch.empty(x.shape, dtype=x.dtype, device=dev) if out is None else _dense_out(out, x.shape, x.dtype)
    _check(L.qmm_dropout(ctypes.byref(t), p, seed, offset, y.data_ptr(), _stream()), "qmm_dropout")
    return y


def layernorm_quantize(x, weight, bias, fmt=None, block=False, residual=None, eps=1e-5, dropout=0.0, dropout_seed=0, dropout_offset=0, mode=RTNE, seed=0,
                       offset=0, want_y=False, want_stats=False, h_out=None):
    """qmm_layernorm_quantize on [rows, cols] or [batch, rows, cols]: LayerNormed(codes [batch, rows, cols], delta, h, y, mean, rstd).  fmt None: no codes.  With
    `block` delta is [batch, blocks of 128 columns, rows], an operand of gemm_blocks, else [batch * rows], an operand of gemm with per_channel=True and
    batch_groups=batch.  h is dropout(x) + residual (x without either); y (without codes: always there), mean and rstd are None unless wanted.
    `h_out`: where h goes, e.g. the residual itself."""
    r = (_short or _host()).layernorm_quantize(x, weight, bias, fmt, block, residual, eps, dropout, dropout_seed, dropout_offset, mode, seed, offset, want_y, want_stats, h_out)
    if type(r) is int:
        _check(r, "qmm_layernorm_quantize")
    if r is not None:
        return LayerNormed._make(r)
    L = lib()
    dev = _on(x.device, x, weight, bias, residual, h_out)
    t = _row_desc(x)
    r = None if residual is None else _row_desc(residual, x.shape, x.dtype)
    w_ptr, w_type = _weight_args(weight, t.cols)
    b_ptr, b_type = _weight_args(bias, t.cols)
    assert weight is None or bias is None or w_type == b_type, "weight and bias of one type"
    dropout = ctypes.c_float(dropout).value                    # as the library gets it: what is 0 there makes no h
    new_h = residual is not None or dropout > 0
    h = x
    if new_h:
        h = torch.empty(x.shape, dtype=x.dtype, device=dev) if h_out is None else _dense_out(h_out, x.shape, x.dtype)
    else:
        assert h_out is None, "without a residual and dropout h is x"
    codes = delta = None
    if fmt is not None:
        codes = torch.empty((t.batch, t.rows, t.cols), dtype=torch.uint8, device=dev)
        delta = torch.empty(_block_scales(t.batch, t.rows, t.cols, 1) if block else (t.batch * t.rows,), dtype=torch.float32, device=dev)
    y = torch.empty(x.shape, dtype=x.dtype, device=dev) if want_y or fmt is None else None
    mean, rstd = (torch.empty(t.batch * t.rows, dtype=torch.float32, device=dev) for _ in range(2)) if want_stats else (None, None)
    ptr = lambda o: None if o is None else o.data_ptr()
    _check(L.qmm_layernorm_quantize(ctypes.byref(t), None if r is None else ctypes.byref(r), w_ptr, b_ptr, b_type if weight is None else w_type, eps, dropout,
                                    dropout_seed, dropout_offset, 0 if fmt is None else fmt, BLOCK if block else 0, mode, seed, offset, ptr(h) if new_h else None,
                                    ptr(y), ptr(mean), ptr(rstd), ptr(delta), ptr(codes), _stream()), "qmm_layernorm_quantize")
    return LayerNormed(codes, delta, h, y, mean, rstd)


def layernorm_backward(dy, h, mean, rstd, weight, dresidual=None, dropout=0.0, dropout_seed=0, dropout_offset=0, want_dw=True, dh_out=None, dx_out=None):
    """qmm_layernorm_backward: LayerNormGradient(dh, dx, dw, db): of the residual, of x (dh itself without dropout), of weight and bias (float32, None unless
    wanted).  `dh_out`, `dx_out`: where they go, e.g. dy itself."""
    r = (_short or _host()).layernorm_backward(dy, h, mean, rstd, weight, dresidual, dropout, dropout_seed, dropout_offset, want_dw, dh_out, dx_out)
    if type(r) is int:
        _check(r, "qmm_layernorm_backward")
    if r is not None:
        return LayerNormGradient._make(r)
    L = lib()
    dev = _on(dy.device, dy, h, mean, rstd, weight, dresidual, dh_out, dx_out)
    t, th = _row_desc(dy), _row_desc(h, dy.shape, dy.dtype)
    r = None if dresidual is None else _row_desc(dresidual, dy.shape, dy.dtype)
    w_ptr, w_type = _weight_args(weight, t.cols)
    for s in (mean, rstd):
        assert s.dtype == torch.float32 and s.is_contiguous() and s.numel() == t.batch * t.rows, "one mean and rstd per row"
    dh = torch.empty(dy.shape, dtype=dy.dtype, device=dev) if dh_out is None else _dense_out(dh_out, dy.shape, dy.dtype)
    dropout = ctypes.c_float(dropout).value                    # as the library gets it: with 0 there is no dx
    if dropout > 0:
        dx = torch.empty(dy.shape, dtype=dy.dtype, device=dev) if dx_out is None else _dense_out(dx_out, dy.shape, dy.dtype)
    else:
        assert dx_out is None, "without dropout dx is dh"
        dx = dh
    dw, db = (torch.empty(t.cols, dtype=torch.float32, device=dev) for _ in range(2)) if want_dw else (None, None)
    ws, ws_ptr, ws_bytes = _scratch(L.qmm_layernorm_backward_workspace_size(ctypes.byref(t)) if want_dw else 0, dev)
    _check(L.qmm_layernorm_backward(ctypes.byref(t), ctypes.byref(th), mean.data_ptr(), rstd.data_ptr(), w_ptr, w_type, None if r is None else ctypes.byref(r), dropout,
                                    dropout_seed, dropout_offset, dh.data_ptr(), dx.data_ptr() if dropout > 0 else None, None if dw is None else dw.data_ptr(),
                                    None if db is None else db.data_ptr(), ws_ptr, ws_bytes, _stream()), "qmm_layernorm_backward")
    return LayerNormGradient(dh, dx, dw, db)


MOMENT_FIELDS = ("n", "mean", "m2", "m3", "m4", "absmax", "nan_cnt", "rsv")


def moments(x, center=0.0, out=None, workspace=None):
    """qmm_moments over all elements of the contiguous device tensor x: 8 float64 on the device (MOMENT_FIELDS)."""
    L = lib()
    assert x.is_contiguous() and x.is_cuda
    n = x.numel()
    if out is None:
        out = torch.empty(8, dtype=torch.float64, device=x.device)
    if workspace is None:
        workspace = _workspace(L.qmm_moments_workspace_size(n), x.device)
    _check(L.qmm_moments(x.data_ptr(), _dtype_code(x), n, float(center), out.data_ptr(), workspace.data_ptr(),
                         workspace.numel(), _stream()), "qmm_moments")
    return out


def mfma_rate(codes, fmt_a, fmt_b, rounds=2000, workgroups=None, sink=None):
    """qmm_mfma_rate on the bytes of the uint8 device tensor `codes`; returns (sink tensor, operations launched)."""
    L = lib()
    assert codes.dtype == torch.uint8 and codes.is_contiguous() and codes.is_cuda
    if workgroups is None:
        workgroups = torch.cuda.get_device_properties(codes.device).multi_processor_count
    if sink is None:
        sink = torch.empty(workgroups * 256, dtype=torch.float32, device=codes.device)
    assert sink.numel() >= workgroups * 256 and sink.dtype == torch.float32
    flops = ctypes.c_double(0.0)
    _check(L.qmm_mfma_rate(fmt_a, fmt_b, codes.data_ptr(), codes.numel(), int(rounds), int(workgroups), sink.data_ptr(),
                           ctypes.byref(flops), _stream()), "qmm_mfma_rate")
    return sink, flops.value


def hbm_rate(src, dst=None, workgroups=1024, sink=None):
    """qmm_hbm_rate over the bytes of the contiguous device tensor src (copied to dst when given); returns the sink."""
    L = lib()
    assert src.is_contiguous() and src.is_cuda and (dst is None or (dst.is_contiguous() and dst.numel() * dst.element_size() == src.numel() * src.element_size()))
    if sink is None:
        sink = torch.empty(workgroups * 256, dtype=torch.int32, device=src.device)
    _check(L.qmm_hbm_rate(src.data_ptr(), dst.data_ptr() if dst is not None else None, src.numel() * src.element_size(),
                          int(workgroups), sink.data_ptr(), _stream()), "qmm_hbm_rate")
    return sink


METRIC_FIELDS = ("S_ee", "S_rr", "S_ae", "S_ar", "M_e", "M_r", "RE_sum", "RE_max", "RE_cnt",
                 "BE_sum", "BE_max", "BE_cnt", "n", "nan_cnt", "rsv0", "rsv1")
