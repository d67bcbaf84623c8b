"""Python binding of libqconv.so (the C ABI in include/qconv.h).

Argument marshalling only: every step of the quantized path runs in the HIP
kernels of the shared library.  PyTorch supplies device memory and the
current stream.  If the library is not built, every call raises -- there is
no fallback implementation.
"""
from __future__ import annotations

import ctypes
import operator
import os
import struct
from array import array

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libqconv.so")

QCONV_OK, QCONV_EINVAL, QCONV_EUNSUPPORTED, QCONV_EWORKSPACE, QCONV_EOVERFLOW, QCONV_EHIP = 0, -1, -2, -3, -4, -5
QCONV_ESCRATCH = -6
ALGO_AUTO, ALGO_BITPLANE, ALGO_MFMA_I8, ALGO_MFMA_FP4, ALGO_MFMA_F16 = 0, 1, 2, 3, 4
EPI_INT32, EPI_SCALE_F32, EPI_BN_F32, EPI_BN_PACK = 0, 1, 2, 3
EPI_POOL2, EPI_RESIDUAL = 1, 2
F32_FMAF_CHAIN, F32_MFMA, F32_BF16X6 = 0, 1, 2
DT_F32, DT_F16, DT_BF16 = 0, 1, 2
ACT_SILU, ACT_GELU, ACT_RELU = 0, 1, 2
OP_NAMES = {1: "XNOR", 2: "SHIFT", 3: "XNOR-ADDER", 4: "SHIFT-ADDER", 5: "MAC"}

EXPORTED = (
    "qconv_error_string", "qconv_version", "qconv_inference_op", "qconv_packed_act_bytes",
    "qconv_pack_act", "qconv_packed_weight_bytes", "qconv_pack_weight", "qconv_fold_bn",
    "qconv_out_size", "qconv_forward", "qnet_create", "qnet_destroy", "qnet_add_conv_f32",
    "qnet_add_maxpool_f32", "qnet_add_quantize", "qnet_add_qconv", "qnet_add_avgpool",
    "qnet_add_fc_f32", "qnet_workspace_bytes", "qnet_forward", "qnet_forward_range", "qnet_num_layers",
    "qnet_forward_noalloc", "qnet_noalloc_bytes", "qnet_noalloc_limit", "qnet_set_f32_algo", "qnet_layer_fused_into",
    "qnet_layer_kernel",
    "qnet_tensor_info", "qconv_resolve_algo",
    "qconv_kernel_name", "aqe_forward", "aqe_backward", "aqe_sgd_clip",
    "qconv_ffn_pre_floats", "qconv_ffn_forward_bytes", "qconv_ffn_forward", "qconv_ffn_backward_bytes", "qconv_ffn_backward",
    "qconv_q4_code_bytes", "qconv_q4_scale_bytes", "qconv_q4_pack", "qconv_q4_workspace_bytes", "qconv_q4_linear",
    "qconv_q4_gated", "aqe_grad_norm_bytes", "aqe_grad_norm", "aqe_clip_grads",
    "qconv_moe_sort_bytes", "qconv_moe_sort", "qconv_moe_gather", "qconv_moe_combine", "qconv_moe_combine_backward",
    "qconv_moe_forward_bytes", "qconv_moe_gated_forward", "qconv_moe_linear_forward", "qconv_moe_backward_bytes",
    "qconv_moe_gated_backward", "qconv_moe_linear_backward",
    "qconv_lora_mid_floats", "qconv_lora_forward_bytes", "qconv_lora_forward", "qconv_lora_backward_bytes",
    "qconv_lora_backward",
)


class QconvError(RuntimeError):
    def __init__(self, status: int, what: str = ""):
        self.status = status
        msg = _lib_or_none().qconv_error_string(status).decode() if _lib_or_none() else str(status)
        super().__init__(f"{what}: {msg} ({status})" if what else f"{msg} ({status})")


class qconv_desc(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int) for name in
                ("n", "cin", "h", "w", "cout", "kh", "kw", "stride", "pad", "a_bits", "w_bits", "algo")]


class qconv_epilogue(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int), ("flags", ctypes.c_int), ("scale", ctypes.c_void_p),
                ("bn_k", ctypes.c_void_p), ("bn_b", ctypes.c_void_p), ("residual", ctypes.c_void_p),
                ("out_bits", ctypes.c_int), ("out_thresholds", ctypes.c_void_p)]


class qconv_ffn_desc(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int) for name in ("m", "k", "f", "dtype", "act")] + \
               [(name, ctypes.c_int64) for name in ("ld_x", "ld_w", "ld_h")]


class qconv_q4_desc(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int) for name in ("m", "n", "k", "group", "dtype")] + \
               [(name, ctypes.c_int64) for name in ("ld_x", "ld_y")]


class qconv_moe_rows_desc(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int) for name in ("tokens", "slots", "width", "dtype")] + \
               [(name, ctypes.c_int64) for name in ("ld_tokens", "ld_rows")]


class qconv_moe_desc(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int) for name in ("rows", "groups", "k", "f", "dtype", "act")] + \
               [(name, ctypes.c_int64) for name in ("ld_x", "ld_w", "ld_h")]


class qconv_lora_desc(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int) for name in ("m", "groups", "rank", "k", "n", "dtype")] + \
               [(name, ctypes.c_int64) for name in ("ld_x", "ld_y", "ld_out")]


_lib = None


def _lib_or_none():
    return _lib


def lib() -> ctypes.CDLL:
    """Load the HIP library; raise loudly if it was not built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`"
                           " (the quantized path has no CPU fallback)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    L.qconv_error_string.restype = ctypes.c_char_p
    L.qconv_error_string.argtypes = [i32]
    L.qconv_version.restype = i32
    L.qconv_inference_op.argtypes = [i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    L.qconv_packed_act_bytes.restype = sz
    L.qconv_packed_act_bytes.argtypes = [i32] * 5
    L.qconv_pack_act.argtypes = [vp, i32, i32, i32, i32, i32, vp, vp, vp]
    L.qconv_packed_weight_bytes.restype = sz
    L.qconv_packed_weight_bytes.argtypes = [i32] * 5
    L.qconv_pack_weight.argtypes = [vp, i32, i32, i32, i32, i32, vp, vp, vp, vp]
    L.qconv_fold_bn.argtypes = [vp, vp, vp, vp, ctypes.c_double, i32, vp, vp]
    L.qconv_out_size.argtypes = [i32] * 4
    L.qconv_forward.argtypes = [ctypes.POINTER(qconv_desc), vp, vp, ctypes.POINTER(qconv_epilogue), vp, vp, vp]
    L.qconv_resolve_algo.argtypes = [ctypes.POINTER(qconv_desc), ctypes.POINTER(qconv_epilogue)]
    L.qconv_kernel_name.argtypes = [ctypes.POINTER(qconv_desc), ctypes.POINTER(qconv_epilogue), i32,
                                    ctypes.c_char_p, i32]
    i64 = ctypes.c_int64
    f32 = ctypes.c_float
    L.aqe_forward.argtypes = [vp, i64, i32, f32, vp, vp, i64, vp, vp]
    L.aqe_backward.argtypes = [vp, vp, i64, f32, vp, vp]
    L.aqe_sgd_clip.argtypes = [vp, vp, i64, f32, vp]
    ffn = q4 = vp  # a descriptor by reference, or its bytes
    L.qconv_ffn_pre_floats.restype = sz
    L.qconv_ffn_pre_floats.argtypes = [i32, i32]
    L.qconv_ffn_forward_bytes.restype = sz
    L.qconv_ffn_forward_bytes.argtypes = [ffn]
    L.qconv_ffn_forward.argtypes = [ffn] + [vp] * 6 + [sz, vp]
    L.qconv_ffn_backward_bytes.restype = sz
    L.qconv_ffn_backward_bytes.argtypes = [ffn]
    L.qconv_ffn_backward.argtypes = [ffn] + [vp] * 9 + [sz, vp]
    L.qconv_q4_code_bytes.restype = sz
    L.qconv_q4_code_bytes.argtypes = [i32] * 3
    L.qconv_q4_scale_bytes.restype = sz
    L.qconv_q4_scale_bytes.argtypes = [i32] * 3
    L.qconv_q4_pack.argtypes = [vp, i32, i32, i32, i64, i32, i32, vp, vp, vp]
    L.qconv_q4_workspace_bytes.restype = sz
    L.qconv_q4_workspace_bytes.argtypes = [q4, i32]
    L.qconv_q4_linear.argtypes = [q4] + [vp] * 6 + [sz, vp]
    L.qconv_q4_gated.argtypes = [q4] + [vp] * 5 + [i32] + [vp] * 2 + [sz, vp]
    L.qconv_moe_sort_bytes.restype = sz
    L.qconv_moe_sort_bytes.argtypes = [i32] * 3
    L.qconv_moe_sort.argtypes = [vp] + [i32] * 3 + [i64, i32] + [vp] * 4 + [sz, vp]
    rows = moe = vp
    L.qconv_moe_gather.argtypes = [rows] + [vp] * 4
    L.qconv_moe_combine.argtypes = [rows] + [vp] * 5
    L.qconv_moe_combine_backward.argtypes = [rows] + [vp] * 5 + [i64, vp, vp]
    for gated in (L.qconv_moe_forward_bytes, L.qconv_moe_backward_bytes):
        gated.restype = sz
        gated.argtypes = [moe, i32]
    L.qconv_moe_gated_forward.argtypes = [moe] + [vp] * 7 + [sz, vp]
    L.qconv_moe_linear_forward.argtypes = [moe] + [vp] * 5 + [sz, vp]
    L.qconv_moe_gated_backward.argtypes = [moe] + [vp] * 10 + [sz, vp]
    L.qconv_moe_linear_backward.argtypes = [moe] + [vp] * 7 + [sz, vp]
    lora = vp
    L.qconv_lora_mid_floats.restype = sz
    L.qconv_lora_mid_floats.argtypes = [i32] * 2
    L.qconv_lora_forward_bytes.restype = sz
    L.qconv_lora_forward_bytes.argtypes = [lora, i32]
    L.qconv_lora_forward.argtypes = [lora] + [vp] * 10 + [sz, vp]
    L.qconv_lora_backward_bytes.restype = sz
    L.qconv_lora_backward_bytes.argtypes = [lora]
    L.qconv_lora_backward.argtypes = [lora] + [vp] * 12 + [sz, vp]
    L.aqe_grad_norm_bytes.restype = sz
    L.aqe_grad_norm_bytes.argtypes = [i32, vp]
    L.aqe_grad_norm.argtypes = [i32] + [vp] * 5 + [sz, vp]
    L.aqe_clip_grads.argtypes = [i32] + [vp] * 4 + [f32, vp, vp, sz, vp]
    L.qnet_create.restype = vp
    L.qnet_create.argtypes = [i32, i32, i32]
    L.qnet_destroy.argtypes = [vp]
    L.qnet_add_conv_f32.argtypes = [vp, i32, vp, i32, i32, i32, i32, vp, vp, i32, i32]
    L.qnet_add_maxpool_f32.argtypes = [vp, i32, i32, i32, i32]
    L.qnet_add_quantize.argtypes = [vp, i32, i32]
    L.qnet_add_qconv.argtypes = [vp, i32, vp, i32, i32, i32, i32, i32, i32, vp, vp, i32, i32]
    L.qnet_add_avgpool.argtypes = [vp, i32]
    L.qnet_add_fc_f32.argtypes = [vp, i32, vp, vp, i32]
    L.qnet_workspace_bytes.restype = sz
    L.qnet_workspace_bytes.argtypes = [vp, i32]
    L.qnet_forward.argtypes = [vp, vp, i32, vp, vp, sz, vp]
    L.qnet_forward_range.argtypes = [vp, vp, i32, vp, vp, sz, i32, i32, vp]
    L.qnet_num_layers.argtypes = [vp]
    L.qnet_forward_noalloc.argtypes = [vp, vp, i32, vp, vp]
    L.qnet_noalloc_bytes.restype = sz
    L.qnet_noalloc_bytes.argtypes = [vp, i32]
    L.qnet_noalloc_limit.restype = sz
    L.qnet_noalloc_limit.argtypes = []
    L.qnet_set_f32_algo.argtypes = [vp, i32]
    L.qnet_layer_fused_into.argtypes = [vp, i32]
    L.qnet_layer_kernel.argtypes = [vp, i32, i32, ctypes.c_char_p, i32]
    L.qnet_tensor_info.argtypes = [vp, i32, i32] + [ctypes.POINTER(i32)] * 4 + [ctypes.POINTER(sz)]
    _lib = L
    return L


def _check(rc: int, what: str) -> int:
    if rc < 0:
        raise QconvError(rc, what)
    return rc


def _ptr(t):
    return None if t is None else t.data_ptr()


# The two lookups behind torch.cuda.current_stream().cuda_stream, without the
# Stream object (3 us a call, as much as a launch); None where torch lacks them.
_raw_stream = None


def _stream(stream):
    global _raw_stream
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        import torch

        get, dev = (getattr(torch._C, f, None) for f in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
        cur = torch.cuda.current_stream
        cur()  # initialises the device, and raises where there is none
        _raw_stream = (lambda: get(dev())) if get and dev else (lambda: cur().cuda_stream)
    return _raw_stream()


# threshold values a quantizer of `bits` reads (Eq. 21: one delta; Eq. 22: three)
_THR_COUNT = {1: 0, 2: 1, 3: 3}


def _host_thr(vals, bits: int, what: str):
    """Host float array of the thresholds for `bits` (None = the defaults).
    The C side reads exactly 1 value for 2 bits and 3 for 3 bits, so the
    length is checked here; 1-bit and 16-bit quantizers take none."""
    if vals is None:
        return None
    vals = [float(v) for v in (vals.tolist() if hasattr(vals, "tolist") else vals)]
    need = _THR_COUNT.get(bits, 0)
    if need == 0:
        return None
    if len(vals) != need:
        raise ValueError(f"{what}: {bits}-bit thresholds take {need} value(s), got {len(vals)}")
    return (ctypes.c_float * need)(*vals)


def planes(bits: int) -> int:
    return {1: 1, 2: 2, 3: 4}[bits]


def out_size(n: int, k: int, stride: int, pad: int) -> int:
    return _check(lib().qconv_out_size(n, k, stride, pad), "qconv_out_size")


def inference_op(m_bits: int, n_bits: int):
    op, prec = ctypes.c_int(), ctypes.c_int()
    _check(lib().qconv_inference_op(m_bits, n_bits, ctypes.byref(op), ctypes.byref(prec)), "qconv_inference_op")
    return OP_NAMES[op.value], prec.value


def packed_act_words(n, c, h, w, bits) -> int:
    return lib().qconv_packed_act_bytes(n, c, h, w, bits) // 4


def packed_weight_words(cout, cin, kh, kw, bits) -> int:
    return lib().qconv_packed_weight_bytes(cout, cin, kh, kw, bits) // 4


def pack_act(x, bits: int, thresholds=None, out=None, stream=None):
    """fp32 NCHW device tensor -> packed bitplanes [n][h][w][cw][P] (int32 view);
    bits = 16: the fp16 channel-last tensor [n][h][w][cw * 32] (int32 view)."""
    n, c, h, w = x.shape
    if out is None:
        import torch

        out = torch.empty(packed_act_words(n, c, h, w, bits), dtype=torch.int32, device=x.device)
    t = _host_thr(thresholds, bits, "pack_act")
    _check(lib().qconv_pack_act(_ptr(x), n, c, h, w, bits, t, _ptr(out), _stream(stream)), "qconv_pack_act")
    return out


def pack_weight(w, bits: int, base_thresholds=None, stream=None, out=None):
    """fp32 OIHW device tensor -> (packed weights, s_c); out = (words, scale)
    reuses existing buffers."""
    cout, cin, kh, kw = w.shape
    if out is None:
        import torch

        out = torch.empty(packed_weight_words(cout, cin, kh, kw, bits), dtype=torch.int32, device=w.device)
        scale = torch.empty(cout, dtype=torch.float32, device=w.device)
    else:
        out, scale = out
    t = _host_thr(base_thresholds, bits, "pack_weight")
    _check(lib().qconv_pack_weight(_ptr(w), cout, cin, kh, kw, bits, t, _ptr(out), _ptr(scale), _stream(stream)),
           "qconv_pack_weight")
    return out, scale


def _empty_like(x):
    import torch

    return torch.empty_like(x)


def aqe_forward(x, bits: int, alpha: float, thresholds=None, scale=None, group_size: int = 0, out=None, stream=None):
    """AQE forward y = alpha h(x) + (1 - alpha) x (device fp32 tensors);
    weights: pass scale (s_c per group) and group_size (values per group)."""
    y = _empty_like(x) if out is None else out
    t = _host_thr(thresholds, bits, "aqe_forward")
    _check(lib().aqe_forward(_ptr(x), x.numel(), bits, float(alpha), t, _ptr(scale), int(group_size), _ptr(y),
                             _stream(stream)), "aqe_forward")
    return y


def aqe_backward(x, gy, alpha: float, out=None, stream=None):
    """AQE backward gx = 2 alpha gy 1{|x| <= 1}."""
    gx = _empty_like(gy) if out is None else out
    _check(lib().aqe_backward(_ptr(x), _ptr(gy), x.numel(), float(alpha), _ptr(gx), _stream(stream)), "aqe_backward")
    return gx


def aqe_sgd_clip(w, g, lr: float, stream=None):
    """In place: w = clip(w - lr g, -1, 1)."""
    _check(lib().aqe_sgd_clip(_ptr(w), _ptr(g), w.numel(), float(lr), _stream(stream)), "aqe_sgd_clip")
    return w


# ---------------------------------------------------------------------------
# Fully connected operators and the gradient norm.  They work on the tensors'
# memory: autograd records nothing (ffn_backward is the gradient), and what is
# written in place does not change a tensor's version.
# ---------------------------------------------------------------------------

class _Dtypes(dict):
    """torch type -> DT_*, -1 for the types the operators do not take."""

    def __missing__(self, key):
        import torch

        self.update({torch.float32: DT_F32, torch.float16: DT_F16, torch.bfloat16: DT_BF16})
        return self.setdefault(key, -1)


_dtypes = _Dtypes()


def _dtype_code(t) -> int:
    return _dtypes[t.dtype]


def _new(shape, dtype, like, stream):
    """A new tensor that belongs to the stream the kernels run on (freed memory
    is handed out again in that stream's order)."""
    if stream is None:
        return like.new_empty(shape) if dtype is like.dtype else like.new_empty(shape, dtype=dtype)
    import torch

    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


_current_device = None  # torch's lookup, once it has a device


def _on_gpu(t, what: str, stream):
    """Kernels go to a stream of the current device: it has to be the tensors'."""
    global _current_device
    if not t.is_cuda:
        raise ValueError(f"{what}: tensors are on the GPU, got one on {t.device}")
    if _current_device is None:
        import torch

        _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    d = t.get_device()
    if d != _current_device() or (stream is not None and stream.device_index != d):
        raise ValueError(f"{what}: tensors are on cuda:{d}, the current device is cuda:{_current_device()}"
                         + (f", the stream is of cuda:{stream.device_index}" if stream is not None else ""))


# A call for one token takes 3 us on the GPU, so the checks below ask each
# property of a tensor once and by its cheapest name.

def _ld(t, s, what: str) -> int:
    """Row stride of a matrix of shape s with unit column stride."""
    rows, cols = s
    ld, unit = t.stride()
    if unit != 1 and cols > 1:
        raise ValueError(f"{what}: columns must be contiguous (strides {t.stride()})")
    if rows <= 1:
        return cols  # no second row
    if ld < cols:
        raise ValueError(f"{what}: row stride {ld} is below the {cols} columns")
    return ld


def _rows(t, rows, cols, like, what: str) -> int:
    """Row stride of a matrix [rows][cols] of the type and on the device of `like`."""
    s = t.shape
    if len(s) != 2 or s[0] != rows or s[1] != cols:
        raise ValueError(f"{what}: shape {tuple(s)}, expected ({rows}, {cols})")
    if t.dtype is not like.dtype or t.get_device() != like.get_device():
        raise ValueError(f"{what}: {t.dtype} on {t.device}, expected {like.dtype} on {like.device}")
    return _ld(t, s, what)


def _workspace(ws, nbytes: int, like, what: str, stream):
    """The caller's workspace (checked on the C side for its size) or a new one."""
    if ws is None:
        if not nbytes:
            return None, 0
        import torch

        return _new((nbytes,), torch.uint8, like, stream), nbytes
    if ws.device != like.device or not ws.is_contiguous():
        raise ValueError(f"{what}: the workspace is a contiguous tensor on {like.device}")
    return ws, ws.numel() * ws.element_size()


# Descriptors as bytes: filling a ctypes structure takes 1 us.
_FFN_DESC = struct.Struct("5i4x3q")
_Q4_DESC = struct.Struct("5i4x2q")


def _ffn_sizes(x, w_gate, what, stream):
    """(m, k, f) of a feed-forward call."""
    s, w = x.shape, w_gate.shape
    if len(s) != 2 or len(w) != 2:
        raise ValueError(f"{what}: x and the weights are matrices")
    _on_gpu(x, what, stream)
    return s[0], s[1], w[0]


def _ffn_desc(x, w_gate, w_up, act, ld_h, m, k, f, what):
    ld_w = _rows(w_gate, f, k, x, what)
    if _rows(w_up, f, k, x, what) != ld_w:
        raise ValueError(f"{what}: w_gate and w_up have different row strides")
    return _FFN_DESC.pack(_int(m), _int(k), _int(f), _dtypes[x.dtype], act, _ld(x, (m, k), what), ld_w, ld_h)


def _int(v: int) -> int:
    if v > 0x7fffffff:
        raise QconvError(QCONV_EUNSUPPORTED, "a size past 2^31")
    return v


def ffn_forward(x, w_gate, w_up, act: int = ACT_SILU, keep_pre: bool = False, pre=None, out=None,
                workspace=None, stream=None):
    """h = act(x w_gate^T) * (x w_up^T) for 16-bit x [m][k] and weights [f][k]
    -> (h [m][f], pre).  keep_pre (or a buffer `pre` of a former call) keeps
    what ffn_backward needs, else pre is None.  h has no autograd graph."""
    m, k, f = _ffn_sizes(x, w_gate, "ffn_forward", stream)
    d = _ffn_desc(x, w_gate, w_up, act, f if out is None else _rows(out, m, f, x, "ffn_forward out"), m, k, f,
                  "ffn_forward")
    L = lib()
    h = _new((m, f), x.dtype, x, stream) if out is None else out
    if pre is not None:
        _check_pre(pre, m, f, x, "ffn_forward")
    elif keep_pre:
        import torch

        pre = _new((L.qconv_ffn_pre_floats(m, f),), torch.float32, x, stream)
    ws, nbytes = _workspace(workspace, L.qconv_ffn_forward_bytes(d), x, "ffn_forward", stream)
    _check(L.qconv_ffn_forward(d, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), h.data_ptr(), _ptr(pre), _ptr(ws),
                               nbytes, _stream(stream)), "qconv_ffn_forward")
    return h, pre


def _check_pre(pre, m, f, like, what):
    import torch

    if pre.dtype != torch.float32 or pre.device != like.device or not pre.is_contiguous() or \
            pre.numel() < lib().qconv_ffn_pre_floats(m, f):
        raise ValueError(f"{what}: pre holds at least {lib().qconv_ffn_pre_floats(m, f)} contiguous fp32 values")


def ffn_backward(x, w_gate, w_up, pre, gh, act: int = ACT_SILU, need_x: bool = True, need_w: bool = True, out=None,
                 workspace=None, stream=None):
    """From gh [m][f] and the forward's pre -> (gx [m][k], gw_gate [f][k],
    gw_up [f][k]) in x's type; None for what need_x / need_w leave out.  out:
    contiguous tensors to write instead of new ones."""
    m, k, f = _ffn_sizes(x, w_gate, "ffn_backward", stream)
    d = _ffn_desc(x, w_gate, w_up, act, _rows(gh, m, f, x, "ffn_backward gh"), m, k, f, "ffn_backward")
    _check_pre(pre, m, f, x, "ffn_backward")
    gx, gg, gu = out if out is not None else (None, None, None)
    shapes = [(m, k), (f, k), (f, k)]
    for i, (t, need) in enumerate(zip((gx, gg, gu), (need_x, need_w, need_w))):
        if t is not None and (not t.is_contiguous() or _rows(t, *shapes[i], x, "ffn_backward out") != k):
            raise ValueError("ffn_backward: out tensors are contiguous")
    new = lambda t, need, s: (_new(s, x.dtype, x, stream) if t is None else t) if need else None
    gx, gg, gu = new(gx, need_x, shapes[0]), new(gg, need_w, shapes[1]), new(gu, need_w, shapes[2])
    ws, nbytes = _workspace(workspace, lib().qconv_ffn_backward_bytes(d), x, "ffn_backward", stream)
    _check(lib().qconv_ffn_backward(d, _ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(pre), _ptr(gh), _ptr(gx),
                                    _ptr(gg), _ptr(gu), _ptr(ws), nbytes, _stream(stream)), "qconv_ffn_backward")
    return gx, gg, gu


def q4_pack(w, group: int = 64, top: int = 6, out=None, stream=None):
    """A matrix [n][k] (fp32 or 16-bit) -> (codes uint8 [n][kp / 2], scales
    bf16 [n][kp / group]): 4-bit E2M1 codes with a scale per `group` values of
    a row; top: the magnitude a group's largest value maps to (6, or 4 for
    weights that sit on the levels of 1..3 bits).  The products take any bf16
    scales, those made here fastest."""
    import torch

    if w.dim() != 2:
        raise ValueError("q4_pack: w is a matrix")
    _on_gpu(w, "q4_pack", stream)
    n, k = w.shape
    ld = _rows(w, n, k, w, "q4_pack")
    if out is None:
        cb, sb = lib().qconv_q4_code_bytes(n, k, group), lib().qconv_q4_scale_bytes(n, k, group)
        out = (_new((n, cb // n if n else 0), torch.uint8, w, stream),
               _new((n, sb // (2 * n) if n else 0), torch.bfloat16, w, stream))
    else:
        _q4_group(*out, n, k, w, "q4_pack", group)
    codes, scales = out
    _check(lib().qconv_q4_pack(_ptr(w), _dtype_code(w), n, k, ld, group, top, _ptr(codes), _ptr(scales),
                               _stream(stream)), "qconv_q4_pack")
    return codes, scales


def _q4_group(codes, scales, n, k, like, what, group=None) -> int:
    """The group size of packed weights [n][k], their buffers checked against it."""
    import torch

    dev = like.get_device()
    if codes.dtype is not torch.uint8 or scales.dtype is not torch.bfloat16 or codes.get_device() != dev or \
            scales.get_device() != dev or not codes.is_contiguous() or not scales.is_contiguous():
        raise ValueError(f"{what}: codes are uint8 and scales bf16, contiguous, on {like.device}")
    cs, ss = codes.shape, scales.shape
    if group is None:
        group = 2 * cs[1] // ss[1] if len(cs) == 2 and len(ss) == 2 and ss[1] else 0
    if group not in (32, 64, 128):
        raise ValueError(f"{what}: groups of {group} values (32, 64 and 128 are supported)")
    groups = (k + group - 1) // group
    if cs != (n, groups * group // 2) or ss != (n, groups):
        raise ValueError(f"{what}: codes {tuple(cs)} and scales {tuple(ss)} are not those of a ({n}, {k}) weight")
    return group


def _q4_sizes(x, codes, scales, what, stream):
    """(m, n, k, group) of a product with packed weights."""
    s, c = x.shape, codes.shape
    if len(s) != 2 or len(c) != 2:
        raise ValueError(f"{what}: x and codes are matrices")
    _on_gpu(x, what, stream)
    m, k = s
    n = c[0]
    return m, n, k, _q4_group(codes, scales, n, k, x, what)


def _q4_desc(x, m, n, k, group, out, what):
    return _Q4_DESC.pack(_int(m), _int(n), _int(k), group, _dtypes[x.dtype], _ld(x, (m, k), what),
                         n if out is None else _rows(out, m, n, x, what))


def q4_linear(x, codes, scales, bias=None, out=None, workspace=None, stream=None):
    """y [m][n] = x [m][k] w^T + bias with 4-bit weights (q4_pack); x and y
    fp16 or bf16, bias fp32 [n]."""
    m, n, k, group = _q4_sizes(x, codes, scales, "q4_linear", stream)
    d = _q4_desc(x, m, n, k, group, out, "q4_linear")
    if bias is not None:
        import torch

        if bias.dtype is not torch.float32 or bias.get_device() != x.get_device() or bias.shape != (n,) or \
                not bias.is_contiguous():
            raise ValueError(f"q4_linear: bias is a contiguous fp32 vector of {n} on {x.device}")
        bias = bias.data_ptr()
    L = lib()
    y = _new((m, n), x.dtype, x, stream) if out is None else out
    ws, nbytes = _workspace(workspace, L.qconv_q4_workspace_bytes(d, 0), x, "q4_linear", stream)
    _check(L.qconv_q4_linear(d, x.data_ptr(), codes.data_ptr(), scales.data_ptr(), bias, y.data_ptr(), _ptr(ws), nbytes,
                             _stream(stream)), "qconv_q4_linear")
    return y


def q4_gated(x, gate_codes, gate_scales, up_codes, up_scales, act: int = ACT_SILU, out=None, workspace=None,
             stream=None):
    """h [m][n] = act(x w_gate^T) * (x w_up^T) with 4-bit weights."""
    m, n, k, group = _q4_sizes(x, gate_codes, gate_scales, "q4_gated", stream)
    if _q4_group(up_codes, up_scales, n, k, x, "q4_gated up") != group:
        raise ValueError("q4_gated: gate and up weights have different groups")
    d = _q4_desc(x, m, n, k, group, out, "q4_gated")
    L = lib()
    y = _new((m, n), x.dtype, x, stream) if out is None else out
    ws, nbytes = _workspace(workspace, L.qconv_q4_workspace_bytes(d, 1), x, "q4_gated", stream)
    _check(L.qconv_q4_gated(d, x.data_ptr(), gate_codes.data_ptr(), gate_scales.data_ptr(), up_codes.data_ptr(),
                            up_scales.data_ptr(), act, y.data_ptr(), _ptr(ws), nbytes, _stream(stream)),
           "qconv_q4_gated")
    return y


# ---------------------------------------------------------------------------
# Rows that go to different weights: tokens sorted by expert and back, the
# experts' products, adapters of many requests.  Which rows belong to which
# weight stays on the device (offsets); no call waits for it.  A result over
# what the call still reads is refused.
# ---------------------------------------------------------------------------

_ROWS_DESC = struct.Struct("4i2q")
_MOE_DESC = struct.Struct("6i3q")
_LORA_DESC = struct.Struct("6i3q")


def _indices(t, like, what: str, numel=None):
    """An index tensor: contiguous int32 on the device of `like`."""
    import torch

    if t.dtype is not torch.int32 or t.get_device() != like.get_device() or not t.is_contiguous() or \
            (numel is not None and t.numel() != numel):
        raise ValueError(f"{what}: contiguous int32{'' if numel is None else f' of {numel} values'} on {like.device}")
    return t


def moe_sort(ids, groups: int, out=None, workspace=None, stream=None):
    """The order that brings the rows of each group together.  ids [tokens] or
    [tokens][slots], int32 or int64: an assignment's group (expert, adapter), or
    a value outside [0, groups) for none -> int32 (offsets [groups + 1]: where
    each group's rows start; order [tokens * slots]: the assignments by group,
    stably, those of none last; place, of ids' shape: an assignment's row, -1 for
    none).  groups is at most 4096."""
    import torch

    _on_gpu(ids, "moe_sort", stream)
    if ids.dim() not in (1, 2) or ids.dtype not in (torch.int32, torch.int64):
        raise ValueError("moe_sort: ids are int32 or int64, [tokens] or [tokens][slots]")
    tokens, slots = ids.shape if ids.dim() == 2 else (ids.shape[0], 1)
    if slots < 1:
        raise ValueError("moe_sort: ids have at least one slot")
    if ids.dim() == 2:
        ld = _ld(ids, (tokens, slots), "moe_sort")
    else:
        ld = ids.stride(0) if tokens > 1 else 1
        if ld < 1:
            raise ValueError("moe_sort: ids share memory")
    n = _int(tokens * slots)
    shapes = (groups + 1,), (n,), tuple(ids.shape)
    if out is None:
        if groups < 1:
            raise QconvError(QCONV_EINVAL, "moe_sort")
        out = tuple(_new(s, torch.int32, ids, stream) for s in shapes)
    elif any(tuple(_indices(t, ids, "moe_sort out").shape) != s for t, s in zip(out, shapes, strict=True)):
        raise ValueError(f"moe_sort: out has the shapes {shapes}")
    offsets, order, place = out
    L = lib()
    ws, nbytes = _workspace(workspace, L.qconv_moe_sort_bytes(tokens, slots, groups), ids, "moe_sort", stream)
    _check(L.qconv_moe_sort(ids.data_ptr(), ids.dtype is torch.int64, tokens, slots, ld, groups, offsets.data_ptr(),
                            order.data_ptr(), place.data_ptr(), _ptr(ws), nbytes, _stream(stream)), "qconv_moe_sort")
    return offsets, order, place


def _place(place, tokens, like, what):
    """(slots, place's address)."""
    if place.dim() not in (1, 2) or place.shape[0] != tokens:
        raise ValueError(f"{what}: place is [{tokens}] or [{tokens}][slots], got {tuple(place.shape)}")
    _indices(place, like, what + " place")
    return place.shape[1] if place.dim() == 2 else 1


def _weights(weights, place, like, what):
    import torch

    if weights is not None and (weights.dtype is not torch.float32 or weights.shape != place.shape or
                                weights.get_device() != like.get_device() or not weights.is_contiguous()):
        raise ValueError(f"{what}: weights are contiguous fp32 of place's shape on {like.device}")
    return _ptr(weights)


def _matrix(t, what, stream):
    if t.dim() != 2:
        raise ValueError(f"{what}: a matrix, got {tuple(t.shape)}")
    _on_gpu(t, what, stream)
    return t.shape


def moe_gather(x, place, out=None, stream=None):
    """rows [tokens * slots][width] of x [tokens][width] by place (moe_sort):
    rows[place[t][s]] = x[t].  fp32 or 16-bit; rows that no place names are left
    as they are.  out shares no value with x."""
    tokens, width = _matrix(x, "moe_gather", stream)
    slots = _place(place, tokens, x, "moe_gather")
    n = tokens * slots
    ld = width if out is None else _rows(out, n, width, x, "moe_gather out")
    d = _ROWS_DESC.pack(_int(tokens), _int(slots), _int(width), _dtypes[x.dtype], _ld(x, (tokens, width), "moe_gather"), ld)
    rows = _new((n, width), x.dtype, x, stream) if out is None else out
    _check(lib().qconv_moe_gather(d, x.data_ptr(), place.data_ptr(), rows.data_ptr(), _stream(stream)),
           "qconv_moe_gather")
    return rows


def moe_combine(rows, place, weights=None, out=None, stream=None):
    """y [tokens][width] = the rows of each token's slots times weights (fp32 of
    place's shape; None: ones), summed in fp32 and rounded once.  out shares no
    value with rows."""
    n, width = _matrix(rows, "moe_combine", stream)
    tokens = place.shape[0] if place.dim() else 0
    slots = _place(place, tokens, rows, "moe_combine")
    if n != tokens * slots:
        raise ValueError(f"moe_combine: {n} rows for {tokens} x {slots} places")
    w = _weights(weights, place, rows, "moe_combine")
    ld = width if out is None else _rows(out, tokens, width, rows, "moe_combine out")
    d = _ROWS_DESC.pack(_int(tokens), _int(slots), _int(width), _dtypes[rows.dtype], ld, _ld(rows, (n, width), "moe_combine"))
    y = _new((tokens, width), rows.dtype, rows, stream) if out is None else out
    _check(lib().qconv_moe_combine(d, rows.data_ptr(), place.data_ptr(), w, y.data_ptr(), _stream(stream)),
           "qconv_moe_combine")
    return y


def moe_gather_backward(grows, place, out=None, stream=None):
    """The gradient of moe_gather's x: each token's rows of grows, summed."""
    return moe_combine(grows, place, None, out, stream)


def moe_combine_backward(gy, rows, place, weights=None, need_rows: bool = True, need_w: bool = True, out=None,
                         stream=None):
    """From gy [tokens][width] -> (the gradient of moe_combine's rows, of its
    weights: fp32 of place's shape); None for what need_rows / need_w leave out.
    Gradients of rows that no place names are left as they are.  out: tensors (or
    None) to write instead of new ones; they may be rows and weights themselves,
    but share no value with gy."""
    import torch

    tokens, width = _matrix(gy, "moe_combine_backward", stream)
    slots = _place(place, tokens, gy, "moe_combine_backward")
    n = tokens * slots
    ld_rows = _rows(rows, n, width, gy, "moe_combine_backward rows")
    w = _weights(weights, place, gy, "moe_combine_backward")
    grows, gw = out if out is not None else (None, None)
    ld = width if grows is None else _rows(grows, n, width, gy, "moe_combine_backward out")
    if gw is not None:
        _weights(gw, place, gy, "moe_combine_backward out")
    d = _ROWS_DESC.pack(_int(tokens), _int(slots), _int(width), _dtypes[gy.dtype],
                        _ld(gy, (tokens, width), "moe_combine_backward"), ld_rows)
    grows = (_new((n, width), gy.dtype, gy, stream) if grows is None else grows) if need_rows else None
    gw = (_new(place.shape, torch.float32, gy, stream) if gw is None else gw) if need_w else None
    _check(lib().qconv_moe_combine_backward(d, gy.data_ptr(), rows.data_ptr(), place.data_ptr(), w, _ptr(grows), ld,
                                            _ptr(gw), _stream(stream)), "qconv_moe_combine_backward")
    return grows, gw


def _expert_weights(w, k, like, what):
    """(groups, f, row stride) of weights [groups][f][k], one group's rows right after the other's."""
    s = w.shape
    if len(s) != 3 or s[2] != k or w.dtype is not like.dtype or w.get_device() != like.get_device():
        raise ValueError(f"{what}: weights are [groups][f][{k}] {like.dtype} on {like.device}, got {tuple(s)} {w.dtype}")
    step, ld, unit = w.stride()
    groups, f = s[0], s[1]
    if f == 1 and groups > 1:
        ld = step  # one row a group
    elif f <= 1:
        ld = k
    if (unit != 1 and k > 1) or ld < k or (groups > 1 and step != f * ld):
        raise ValueError(f"{what}: columns are contiguous and one group's rows follow the other's (strides {w.stride()})")
    return groups, f, ld


def _moe_args(x, ws, offsets, act, what, stream, out):
    """(rows, k, groups, f, descriptor) of an experts' product; out: [rows][f] or None."""
    rows, k = _matrix(x, what, stream)
    groups, f, ld_w = _expert_weights(ws[0], k, x, what)
    if len(ws) == 2 and (_expert_weights(ws[1], k, x, what) != (groups, f, ld_w)):
        raise ValueError(f"{what}: w_gate and w_up have different shapes or strides")
    _indices(offsets, x, what + " offsets", groups + 1)
    ld_h = f if out is None else _rows(out, rows, f, x, what)
    return rows, k, groups, f, _MOE_DESC.pack(_int(rows), groups, _int(k), _int(f), _dtypes[x.dtype], act,
                                              _ld(x, (rows, k), what), ld_w, ld_h)


def moe_gated_forward(x, w_gate, w_up, offsets, act: int = ACT_SILU, keep_pre: bool = False, pre=None, out=None,
                      workspace=None, stream=None):
    """ffn_forward with the weights [groups][f][k] of each row's group: rows
    offsets[g] .. offsets[g + 1] of x [rows][k] are group g's -> (h [rows][f],
    pre).  Rows of no group are left as they are.  out shares no value with x or
    the weights."""
    rows, k, groups, f, d = _moe_args(x, (w_gate, w_up), offsets, act, "moe_gated_forward", stream, out)
    L = lib()
    h = _new((rows, f), x.dtype, x, stream) if out is None else out
    if pre is not None:
        _check_pre(pre, rows, f, x, "moe_gated_forward")
    elif keep_pre:
        import torch

        pre = _new((L.qconv_ffn_pre_floats(rows, f),), torch.float32, x, stream)
    ws, nbytes = _workspace(workspace, L.qconv_moe_forward_bytes(d, 1), x, "moe_gated_forward", stream)
    _check(L.qconv_moe_gated_forward(d, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), offsets.data_ptr(),
                                     h.data_ptr(), _ptr(pre), _ptr(ws), nbytes, _stream(stream)),
           "qconv_moe_gated_forward")
    return h, pre


def moe_linear_forward(x, w, offsets, out=None, workspace=None, stream=None):
    """y [rows][f] = x w_g^T with the weights [groups][f][k] of each row's group.
    out shares no value with x or w."""
    rows, k, groups, f, d = _moe_args(x, (w,), offsets, 0, "moe_linear_forward", stream, out)
    L = lib()
    y = _new((rows, f), x.dtype, x, stream) if out is None else out
    ws, nbytes = _workspace(workspace, L.qconv_moe_forward_bytes(d, 0), x, "moe_linear_forward", stream)
    _check(L.qconv_moe_linear_forward(d, x.data_ptr(), w.data_ptr(), offsets.data_ptr(), y.data_ptr(), _ptr(ws), nbytes,
                                      _stream(stream)), "qconv_moe_linear_forward")
    return y


def _grad_outs(out, shapes, needs, like, what, stream):
    """The gradients to write: those of `out` (contiguous) or new ones, None where not needed."""
    out = (None,) * len(shapes) if out is None else out
    for t, s in zip(out, shapes, strict=True):
        if t is not None and (tuple(t.shape) != s or t.dtype is not like.dtype or not t.is_contiguous() or
                              t.get_device() != like.get_device()):
            raise ValueError(f"{what}: out tensors are contiguous {like.dtype} on {like.device}, of the shapes {shapes}")
    return [(_new(s, like.dtype, like, stream) if t is None else t) if need else None
            for t, s, need in zip(out, shapes, needs)]


def moe_gated_backward(x, w_gate, w_up, offsets, pre, gh, act: int = ACT_SILU, need_x: bool = True, need_w: bool = True,
                       out=None, workspace=None, stream=None):
    """From gh [rows][f] and the forward's pre -> (gx [rows][k], gw_gate and
    gw_up [groups][f][k]) in x's type; None for what need_x / need_w leave out.
    The gradients of both products are rounded to x's type on the way (with fp16
    infinite past 65504: the loss is scaled as for any gradient).
    out: contiguous tensors (or None) to write instead of new ones, which share no
    value with what is still read: the gradient of x is written first.  Rows of no
    group are left as they are, weights of no row get zeros."""
    rows, k, groups, f, d = _moe_args(x, (w_gate, w_up), offsets, act, "moe_gated_backward", stream, gh)
    _check_pre(pre, rows, f, x, "moe_gated_backward")
    gx, gg, gu = _grad_outs(out, ((rows, k), (groups, f, k), (groups, f, k)), (need_x, need_w, need_w), x,
                            "moe_gated_backward", stream)
    L = lib()
    ws, nbytes = _workspace(workspace, L.qconv_moe_backward_bytes(d, 1), x, "moe_gated_backward", stream)
    _check(L.qconv_moe_gated_backward(d, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), offsets.data_ptr(),
                                      pre.data_ptr(), gh.data_ptr(), _ptr(gx), _ptr(gg), _ptr(gu), _ptr(ws), nbytes,
                                      _stream(stream)), "qconv_moe_gated_backward")
    return gx, gg, gu


def moe_linear_backward(x, w, offsets, gy, need_x: bool = True, need_w: bool = True, out=None, workspace=None,
                        stream=None):
    """From gy [rows][f] -> (gx [rows][k], gw [groups][f][k]), as moe_gated_backward."""
    rows, k, groups, f, d = _moe_args(x, (w,), offsets, 0, "moe_linear_backward", stream, gy)
    gx, gw = _grad_outs(out, ((rows, k), (groups, f, k)), (need_x, need_w), x, "moe_linear_backward", stream)
    L = lib()
    ws, nbytes = _workspace(workspace, L.qconv_moe_backward_bytes(d, 0), x, "moe_linear_backward", stream)
    _check(L.qconv_moe_linear_backward(d, x.data_ptr(), w.data_ptr(), offsets.data_ptr(), gy.data_ptr(), _ptr(gx),
                                       _ptr(gw), _ptr(ws), nbytes, _stream(stream)), "qconv_moe_linear_backward")
    return gx, gw


def _lora_args(x, a, b, offsets, order, scale, y, out, what, stream):
    """(m, groups, rank, k, n, descriptor) of an adapters' call."""
    import torch

    m, k = _matrix(x, what, stream)
    dev = x.get_device()
    sa, sb = a.shape, b.shape
    if len(sa) != 3 or len(sb) != 3 or sa[2] != k or sb[0] != sa[0] or sb[2] != sa[1] or a.dtype is not x.dtype or \
            b.dtype is not x.dtype or a.get_device() != dev or b.get_device() != dev or not a.is_contiguous() or \
            not b.is_contiguous():
        raise ValueError(f"{what}: a is [adapters][rank][{k}] and b [adapters][n][rank], contiguous {x.dtype} on {x.device}")
    groups, rank, n = sa[0], sa[1], sb[1]
    _indices(offsets, x, what + " offsets", groups + 1)
    _indices(order, x, what + " order", m)
    if scale is not None and (scale.dtype is not torch.float32 or scale.shape != (groups,) or scale.get_device() != dev or
                              not scale.is_contiguous()):
        raise ValueError(f"{what}: scale is a contiguous fp32 vector of {groups} on {x.device}")
    ld_y = _rows(y, m, n, x, what)
    return m, groups, rank, k, n, _LORA_DESC.pack(_int(m), groups, rank, _int(k), _int(n), _dtypes[x.dtype],
                                                  _ld(x, (m, k), what), ld_y,
                                                  ld_y if out is None else _rows(out, m, n, x, what + " out"))


def _check_mid(mid, m, rank, like, what):
    import torch

    if mid.dtype is not torch.float32 or mid.get_device() != like.get_device() or not mid.is_contiguous() or \
            mid.numel() < lib().qconv_lora_mid_floats(m, rank):
        raise ValueError(f"{what}: mid holds at least {lib().qconv_lora_mid_floats(m, rank)} contiguous fp32 values")


def lora_forward(y, x, a, b, offsets, order, scale=None, keep_mid: bool = False, mid=None, out=None, workspace=None,
                 stream=None):
    """Adds to y [m][n], a shared projection's result for x [m][k], each token's
    low-rank adapter: y[t] + scale[g] (x[t] a_g^T) b_g^T with a [adapters][rank][k],
    b [adapters][n][rank], scale fp32 [adapters] (None: ones) -> (out, mid).  In
    place, or into `out`; neither may share a value with x, a, b or mid.  offsets and
    order are moe_sort's of the tokens' adapters (ids [m]); a token of none keeps its y.
    An infinity among the operands may give a NaN in its place: the second product
    takes x a_g^T in two parts.  keep_mid (or a buffer `mid` of a former
    call) keeps what lora_backward needs, else mid is None.  rank is at most 256."""
    m, groups, rank, k, n, d = _lora_args(x, a, b, offsets, order, scale, y, out, "lora_forward", stream)
    L = lib()
    if mid is not None:
        _check_mid(mid, m, rank, x, "lora_forward")
    elif keep_mid:
        import torch

        mid = _new((L.qconv_lora_mid_floats(m, rank),), torch.float32, x, stream)
    to = y if out is None else out
    ws, nbytes = _workspace(workspace, L.qconv_lora_forward_bytes(d, mid is not None), x, "lora_forward", stream)
    _check(L.qconv_lora_forward(d, x.data_ptr(), a.data_ptr(), b.data_ptr(), offsets.data_ptr(), order.data_ptr(),
                                _ptr(scale), y.data_ptr(), to.data_ptr(), _ptr(mid), _ptr(ws), nbytes, _stream(stream)),
           "qconv_lora_forward")
    return to, mid


def lora_backward(x, a, b, offsets, order, mid, gy, scale=None, need_x: bool = True, need_w: bool = True, out=None,
                  workspace=None, stream=None):
    """From gy [m][n] and the forward's mid -> (gx [m][k]: the adapters' part of
    x's gradient, ga, gb) in x's type; None for what need_x / need_w leave out.
    out: contiguous tensors (or None) to write instead of new ones, which share no
    value with x or gy where ga and gb are wanted."""
    m, groups, rank, k, n, d = _lora_args(x, a, b, offsets, order, scale, gy, None, "lora_backward", stream)
    _check_mid(mid, m, rank, x, "lora_backward")
    gx, ga, gb = _grad_outs(out, ((m, k), (groups, rank, k), (groups, n, rank)), (need_x, need_w, need_w), x,
                            "lora_backward", stream)
    L = lib()
    ws, nbytes = _workspace(workspace, L.qconv_lora_backward_bytes(d), x, "lora_backward", stream)
    _check(L.qconv_lora_backward(d, x.data_ptr(), a.data_ptr(), b.data_ptr(), offsets.data_ptr(), order.data_ptr(),
                                 _ptr(scale), mid.data_ptr(), gy.data_ptr(), _ptr(gx), _ptr(ga), _ptr(gb), _ptr(ws),
                                 nbytes, _stream(stream)), "qconv_lora_backward")
    return gx, ga, gb


def _dense(t) -> bool:
    """Whether a tensor's values fill one range of memory, in any order of its dimensions."""
    if t.is_contiguous():
        return True
    want = 1
    for size, stride in sorted(((s, st) for s, st in zip(t.shape, t.stride()) if s != 1), key=lambda v: v[1]):
        if stride != want:
            return False
        want *= size
    return True


def _same_layout(a, b) -> bool:
    """Whether two dense tensors of as many values hold them in the same order."""
    return (a.is_contiguous() and b.is_contiguous()) or \
        (a.shape == b.shape and all(n == 1 or i == j for n, i, j in zip(a.shape, a.stride(), b.stride())))


def _grad_arrays(grads, what, stream):
    """(count, pointers, sizes, types, dense order) of a list of gradients as C
    arrays.  One pass per property with the tensors' own methods: a model has
    hundreds of gradients, and a Python loop body costs more than the kernels."""
    import torch

    T = torch.Tensor
    n = len(grads)
    types = list(map(operator.attrgetter("dtype"), grads))
    codes = array("i", [_dtypes[types[0]]]) * n if n and types.count(types[0]) == n else \
        array("i", map(_dtypes.__getitem__, types))
    if n:
        _on_gpu(grads[0], what, stream)
    plain = all(map(T.is_contiguous, grads))
    if len(set(map(T.get_device, grads))) > 1 or -1 in codes or not (plain or all(map(_dense, grads))):
        raise ValueError(f"{what}: gradients are dense fp32, fp16 or bf16 tensors on one device")
    return n, array("Q", map(T.data_ptr, grads)), array("q", map(T.numel, grads)), codes, plain


def _addr(a):
    """Address of an array.array's values, which its owner keeps alive."""
    return a.buffer_info()[0]


def _norm_out(grads, norm, what, stream):
    import torch

    if norm is None:
        return _new((), torch.float32, grads[0] if len(grads) else torch.empty(0, device="cuda"), stream)
    if norm.dtype != torch.float32 or norm.numel() != 1 or (len(grads) and norm.device != grads[0].device):
        raise ValueError(f"{what}: norm is one fp32 value on the gradients' device")
    _on_gpu(norm, what, stream)  # there may be no gradient to compare it with
    return norm


def aqe_grad_norm(grads, norm=None, workspace=None, stream=None):
    """The 2-norm over all values of a list of gradients, as a device scalar."""
    n, ptrs, sizes, types, _ = _grad_arrays(grads, "aqe_grad_norm", stream)
    norm = _norm_out(grads, norm, "aqe_grad_norm", stream)
    ws, nbytes = _workspace(workspace, lib().aqe_grad_norm_bytes(n, _addr(sizes)), norm, "aqe_grad_norm", stream)
    _check(lib().aqe_grad_norm(n, _addr(ptrs), _addr(sizes), _addr(types), _ptr(norm), _ptr(ws), nbytes,
                               _stream(stream)), "aqe_grad_norm")
    return norm


def aqe_clip_grads(grads, max_norm: float, out=None, norm=None, workspace=None, stream=None):
    """Scale a list of gradients so that their joint norm is at most max_norm,
    in place or into the tensors of `out` (same sizes, types and layouts); returns
    the norm before, as a device scalar.  A tensor is listed once."""
    n, ptrs, sizes, types, plain = _grad_arrays(grads, "aqe_clip_grads", stream)
    outs = ptrs
    if out is not None:
        m, outs, out_sizes, out_types, out_plain = _grad_arrays(out, "aqe_clip_grads", stream)
        if m != n or out_sizes != sizes or out_types != types or (n and out[0].device != grads[0].device) or \
                not (plain and out_plain or all(map(_same_layout, out, grads))):
            raise ValueError("aqe_clip_grads: out holds one tensor per gradient, of its size, layout, type and device")
    norm = _norm_out(grads, norm, "aqe_clip_grads", stream)
    ws, nbytes = _workspace(workspace, lib().aqe_grad_norm_bytes(n, _addr(sizes)), norm, "aqe_clip_grads", stream)
    _check(lib().aqe_clip_grads(n, _addr(ptrs), _addr(outs), _addr(sizes), _addr(types), float(max_norm), _ptr(norm),
                                _ptr(ws), nbytes, _stream(stream)), "aqe_clip_grads")
    return norm


def fold_bn(gamma, beta, mean, var, eps):
    """Host fold of BN parameters (numpy/CPU arrays) -> (k, b) float32 numpy."""
    import numpy as np

    g, b, m, v = (np.ascontiguousarray(np.asarray(a, dtype=np.float32)) for a in (gamma, beta, mean, var))
    c = g.size
    k = np.empty(c, np.float32)
    bb = np.empty(c, np.float32)
    P = lambda a: a.ctypes.data_as(ctypes.c_void_p)
    _check(lib().qconv_fold_bn(P(g), P(b), P(m), P(v), ctypes.c_double(float(eps)), c, P(k), P(bb)), "qconv_fold_bn")
    return k, bb


def conv(act_packed, w_packed, n, cin, h, w, cout, k, stride, pad, a_bits, w_bits, mode=EPI_INT32,
         flags=0, scale=None, bn_k=None, bn_b=None, residual=None, out_bits=0, out=None, out_packed=None,
         algo=ALGO_AUTO, stream=None, out_thresholds=None):
    """qconv_forward; allocates the outputs the epilogue needs when not given."""
    if (out is None and mode != EPI_BN_PACK) or (out_packed is None and mode == EPI_BN_PACK):
        import torch

        ho, wo = out_size(h, k, stride, pad), out_size(w, k, stride, pad)
        if flags & EPI_POOL2:
            ho, wo = ho // 2, wo // 2
        dev = act_packed.device
        if mode == EPI_BN_PACK:
            out_packed = torch.empty(packed_act_words(n, cout, ho, wo, out_bits), dtype=torch.int32, device=dev)
        else:
            dt = torch.int32 if mode == EPI_INT32 else torch.float32
            out = torch.empty((n, cout, ho, wo), dtype=dt, device=dev)
    d = qconv_desc(n, cin, h, w, cout, k, k, stride, pad, a_bits, w_bits, algo)
    thr = _host_thr(out_thresholds, out_bits, "conv") if out_thresholds is not None else None  # alive across the call
    e = qconv_epilogue(mode, flags, _ptr(scale), _ptr(bn_k), _ptr(bn_b), _ptr(residual), out_bits,
                       ctypes.cast(thr, ctypes.c_void_p) if thr is not None else None)
    rc = lib().qconv_forward(ctypes.byref(d), _ptr(act_packed), _ptr(w_packed), ctypes.byref(e), _ptr(out),
                             _ptr(out_packed), _stream(stream))
    if rc < 0:
        out_size(h, k, stride, pad), out_size(w, k, stride, pad)  # an impossible geometry is reported as that
        raise QconvError(rc, "qconv_forward")
    return out, out_packed


ALGO_NAMES = {ALGO_BITPLANE: "bitplane", ALGO_MFMA_I8: "mfma_i8", ALGO_MFMA_FP4: "mfma_fp4", ALGO_MFMA_F16: "mfma_f16"}


def resolve_algo(n, cin, h, w, cout, k, stride, pad, a_bits, w_bits, mode=EPI_INT32, flags=0, out_bits=0,
                 algo=ALGO_AUTO) -> int:
    """The concrete algorithm qconv_forward would run (launches nothing)."""
    d = qconv_desc(n, cin, h, w, cout, k, k, stride, pad, a_bits, w_bits, algo)
    e = qconv_epilogue(mode, flags, None, None, None, None, out_bits, None)
    return _check(lib().qconv_resolve_algo(ctypes.byref(d), ctypes.byref(e)), "qconv_resolve_algo")


def kernel_name(n, cin, h, w, cout, k, stride, pad, a_bits, w_bits, mode=EPI_INT32, flags=0, out_bits=0,
                algo=ALGO_AUTO, packed_out=False) -> str:
    """The GPU kernel instantiation qconv_forward would launch on the current
    device, as a profiler names it (launches nothing)."""
    d = qconv_desc(n, cin, h, w, cout, k, k, stride, pad, a_bits, w_bits, algo)
    e = qconv_epilogue(mode, flags, None, None, None, None, out_bits, None)
    buf = ctypes.create_string_buffer(128)
    _check(lib().qconv_kernel_name(ctypes.byref(d), ctypes.byref(e), int(bool(packed_out)), buf, 128),
           "qconv_kernel_name")
    return buf.value.decode()


class Net:
    """A qnet layer list (tensor ids as in include/qconv.h)."""

    def __init__(self, in_c: int, in_h: int, in_w: int, f32_algo: int = F32_MFMA):
        self._h = lib().qnet_create(in_c, in_h, in_w)
        if not self._h:
            raise QconvError(QCONV_EINVAL, "qnet_create")
        _check(lib().qnet_set_f32_algo(self._h, int(f32_algo)), "qnet_set_f32_algo")
        self.f32_algo = f32_algo
        self._keep = []  # device tensors the layers point at
        self.layers = []  # per layer: what was added (kind, source, parameters), for reports

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.qnet_destroy(self._h)
            self._h = None

    def _add(self, rc, what, *keep, **info):
        self._keep.extend(k for k in keep if k is not None)
        tid = _check(rc, what)
        self.layers.append(dict(kind=what.replace("qnet_add_", ""), dst=tid, **info))
        return tid

    def fused_into(self, layer):
        """The earlier layer whose epilogue writes layer `layer`'s tensor, or None."""
        if layer < 0:
            return None
        r = _check(lib().qnet_layer_fused_into(self._h, layer), "qnet_layer_fused_into")
        return None if r == layer else r

    def layer_kernel(self, layer, batch):
        """The GPU kernel layer `layer` launches ("" when an earlier layer writes its tensor)."""
        buf = ctypes.create_string_buffer(128)
        _check(lib().qnet_layer_kernel(self._h, layer, batch, buf, 128), "qnet_layer_kernel")
        return buf.value.decode()

    def _mark_fused(self, tid):
        """Record (for reports) which layer writes the tensor a layer just added."""
        li = tid - 1
        prod = self.fused_into(li)
        self.layers[li]["fused_into"] = prod
        if prod is not None:
            key = "pool_dst" if self.layers[li]["kind"] == "maxpool_f32" else "pack_dst"
            self.layers[prod][key] = tid
        return tid

    def conv_f32(self, src, w, bn_k, bn_b, stride=1, pad=0, relu=False, out_bits=0):
        cout, _, k, _ = w.shape
        return self._add(lib().qnet_add_conv_f32(self._h, src, _ptr(w), cout, k, stride, pad, _ptr(bn_k), _ptr(bn_b),
                                                 int(relu), out_bits), "qnet_add_conv_f32", w, bn_k, bn_b,
                         src=src, cout=cout, k=k, stride=stride, pad=pad, out_bits=out_bits)

    def maxpool_f32(self, src, k, stride, pad):
        return self._mark_fused(self._add(lib().qnet_add_maxpool_f32(self._h, src, k, stride, pad),
                                          "qnet_add_maxpool_f32", src=src, k=k, stride=stride, pad=pad))

    def quantize(self, src, bits):
        return self._mark_fused(self._add(lib().qnet_add_quantize(self._h, src, bits), "qnet_add_quantize", src=src,
                                          out_bits=bits))

    def qconv(self, src, w_packed, cout, k, stride, pad, w_bits, bn_k, bn_b, pool2=False, residual_src=-1,
              out_bits=0):
        return self._add(lib().qnet_add_qconv(self._h, src, _ptr(w_packed), cout, k, stride, pad, w_bits, int(pool2),
                                              _ptr(bn_k), _ptr(bn_b), residual_src, out_bits),
                         "qnet_add_qconv", w_packed, bn_k, bn_b, src=src, cout=cout, k=k, stride=stride, pad=pad,
                         w_bits=w_bits, pool2=bool(pool2), residual_src=residual_src, out_bits=out_bits)

    def avgpool(self, src):
        return self._add(lib().qnet_add_avgpool(self._h, src), "qnet_add_avgpool", src=src)

    def fc_f32(self, src, w, bias=None):
        return self._add(lib().qnet_add_fc_f32(self._h, src, _ptr(w), _ptr(bias), w.shape[0]), "qnet_add_fc_f32",
                         w, bias, src=src, cout=w.shape[0])

    def workspace_bytes(self, batch):
        return lib().qnet_workspace_bytes(self._h, batch)

    def tensor_info(self, tid, batch):
        c, h, w, b = (ctypes.c_int() for _ in range(4))
        off = ctypes.c_size_t()
        _check(lib().qnet_tensor_info(self._h, tid, batch, ctypes.byref(c), ctypes.byref(h), ctypes.byref(w),
                                      ctypes.byref(b), ctypes.byref(off)), "qnet_tensor_info")
        return c.value, h.value, w.value, b.value, off.value

    def forward(self, x, logits, workspace, stream=None):
        nbytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
        _check(lib().qnet_forward(self._h, _ptr(x), x.shape[0], _ptr(logits), _ptr(workspace), nbytes,
                                  _stream(stream)), "qnet_forward")
        return logits

    def forward_range(self, x, logits, workspace, first, count, stream=None):
        """Layers [first, first + count) of forward() on the same workspace."""
        nbytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
        _check(lib().qnet_forward_range(self._h, _ptr(x), x.shape[0], _ptr(logits), _ptr(workspace), nbytes,
                                        int(first), int(count), _stream(stream)), "qnet_forward_range")
        return logits

    def forward_noalloc(self, x, logits, stream=None):
        """forward() on the library's fixed scratch array instead of a workspace."""
        _check(lib().qnet_forward_noalloc(self._h, _ptr(x), x.shape[0], _ptr(logits), _stream(stream)),
               "qnet_forward_noalloc")
        return logits

    def noalloc_bytes(self, batch):
        return lib().qnet_noalloc_bytes(self._h, batch)

    def num_layers(self):
        return _check(lib().qnet_num_layers(self._h), "qnet_num_layers")
