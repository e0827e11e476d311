"""ctypes binding of libdsqconv: the same names as ``include/dsqconv.h``.

Argument marshalling only; calls whose arguments all have their plain form go through
the native ``_marshal`` module instead of ctypes (csrc/marshal.cpp) where it loads: it is
built against one PyTorch, and without it, with a warning, every call takes the ctypes path.
PyTorch supplies device memory (``data_ptr()``)
and the HIP stream handle (``torch.cuda.current_stream().cuda_stream`` is
PyTorch-ROCm's name for the hipStream_t); every step of the path runs in the
library's HIP kernels.  There is no CPU fallback: if the shared library has
not been built, the first call raises.
"""
import ctypes as C
import os
import warnings
from dataclasses import dataclass

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdsqconv.so")

DSQ_NHWC, DSQ_NCHW = 0, 1
DSQ_OK = 0
DSQ_CONV_MANY_IN_FLIGHT = 0x10
DSQ_CONV_ACT_DENSE3 = 0x20
DSQ_CONV_NEXT_DENSE3 = 0x40
DSQ_CONV_NEXT_SUMS_ZERO = 0x80
DSQ_PACK_CONTAINER, DSQ_PACK_DENSE3 = 0, 1
DSQ_F32, DSQ_F16, DSQ_BF16 = 0, 1, 2


def DSQ_CONV_KERNEL(k):
    return k & 15

EXPORTS = [
    "dsq_act_packed_bytes", "dsq_act_packed_bytes_ex", "dsq_wgt_packed_bytes", "dsq_wgt_aux_bytes",
    "dsq_quantize_act", "dsq_quantize_act_ex", "dsq_pack_weights", "dsq_pack_weights_for", "dsq_conv2d", "dsq_conv2d_requant", "dsq_conv2d_wq",
    "dsq_soft_quantize_fwd", "dsq_soft_quantize_bwd",
    "dsq_conv2d_plan", "dsq_status_string",
    "dsq_code_row_bytes", "dsq_rms_norm_bwd_bytes", "dsq_w4_packed_bytes", "dsq_w4_scale_bytes",
    "dsq_rms_norm", "dsq_rms_norm_bwd", "dsq_pack_weights_w4", "dsq_linear_w4", "dsq_linear_w4a8",
    "dsq_qk_norm_rope_bwd_bytes", "dsq_attention_bwd_bytes", "dsq_attention_cache_bytes",
    "dsq_qk_norm_rope", "dsq_qk_norm_rope_bwd", "dsq_attention", "dsq_attention_bwd", "dsq_attention_cache",
]


class DsqError(RuntimeError):
    def __init__(self, status, message):
        super().__init__("libdsqconv: %s (status %d)" % (message, status))
        self.status = status


class dsq_conv_desc(C.Structure):
    _fields_ = [(n, C.c_int) for n in
                ("N", "C_in", "H", "W", "C_out", "R", "S", "stride", "pad", "bits", "flags")]


_lib = None


def load_library():
    """Load libdsqconv.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            "libdsqconv.so is missing at %s: build it first "
            "(python -c 'import __graft_entry__ as g; g.build()'). "
            "There is no fallback path." % LIB_PATH)
    lib = C.CDLL(LIB_PATH)
    vp, sz, i, f = C.c_void_p, C.c_size_t, C.c_int, C.c_float
    lib.dsq_act_packed_bytes.restype = sz
    lib.dsq_act_packed_bytes.argtypes = [i] * 5
    lib.dsq_act_packed_bytes_ex.restype = sz
    lib.dsq_act_packed_bytes_ex.argtypes = [i] * 6
    lib.dsq_quantize_act_ex.restype = i
    lib.dsq_quantize_act_ex.argtypes = [vp, i, i, i, i, i, f, f, i, i, vp, sz, vp, vp]
    lib.dsq_wgt_packed_bytes.restype = sz
    lib.dsq_wgt_packed_bytes.argtypes = [i] * 5
    lib.dsq_wgt_aux_bytes.restype = sz
    lib.dsq_wgt_aux_bytes.argtypes = [i] * 3
    lib.dsq_quantize_act.restype = i
    lib.dsq_quantize_act.argtypes = [vp, i, i, i, i, i, f, f, i, vp, sz, vp, vp]
    lib.dsq_pack_weights.restype = i
    lib.dsq_pack_weights.argtypes = [vp, vp, vp, vp, i, i, i, i, i, vp, sz, vp, sz, vp]
    lib.dsq_pack_weights_for.restype = i
    lib.dsq_pack_weights_for.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, vp, sz, vp, sz, vp]
    lib.dsq_conv2d.restype = i
    lib.dsq_conv2d.argtypes = [C.POINTER(dsq_conv_desc), vp, vp, f, f, vp, vp, vp, i, vp, vp]
    lib.dsq_conv2d_requant.restype = i
    lib.dsq_conv2d_requant.argtypes = [C.POINTER(dsq_conv_desc), vp, vp, f, f, vp, vp, vp, vp, i, f, f, i,
                                       vp, sz, vp, vp]
    lib.dsq_conv2d_wq.restype = i
    lib.dsq_conv2d_wq.argtypes = [C.POINTER(dsq_conv_desc), vp, i, vp, vp, vp, i, vp]
    lib.dsq_soft_quantize_fwd.restype = i
    lib.dsq_soft_quantize_fwd.argtypes = [vp, sz, f, f, f, i, vp, vp]
    lib.dsq_soft_quantize_bwd.restype = i
    lib.dsq_soft_quantize_bwd.argtypes = [vp, vp, sz, f, f, f, i, vp, vp, vp]
    lib.dsq_conv2d_plan.restype = i
    lib.dsq_conv2d_plan.argtypes = [C.POINTER(dsq_conv_desc), i, f, C.c_char_p, sz]
    i64 = C.c_int64
    for name, args in (("dsq_code_row_bytes", [i]), ("dsq_rms_norm_bwd_bytes", [i, i]), ("dsq_w4_packed_bytes", [i, i]),
                       ("dsq_w4_scale_bytes", [i, i, i])):
        getattr(lib, name).restype = sz
        getattr(lib, name).argtypes = args
    lib.dsq_rms_norm.restype = i
    lib.dsq_rms_norm.argtypes = [vp, i64, vp, i64, vp, i, i, i, f, vp, vp, vp, sz, vp, vp, vp]
    lib.dsq_rms_norm_bwd.restype = i
    lib.dsq_rms_norm_bwd.argtypes = [vp, i64, vp, vp, vp, i64, vp, i64, i, i, i, vp, vp, vp, sz, vp]
    heads = [vp, i64, i64]
    for name, args in (("dsq_qk_norm_rope_bwd_bytes", [i] * 4), ("dsq_attention_bwd_bytes", [i] * 2), ("dsq_attention_cache_bytes", [i] * 5)):
        getattr(lib, name).restype = sz
        getattr(lib, name).argtypes = args
    rotation = [vp, vp, f, vp, i, vp, vp, i, i]
    for name, args in (
            ("dsq_qk_norm_rope", heads * 3 + [i] * 5 + rotation + heads * 2 + [vp, vp, i64, i, vp, vp]),
            ("dsq_qk_norm_rope_bwd", heads * 2 + [i] * 5 + rotation + heads * 4 + [vp, vp, vp, sz, vp]),
            ("dsq_attention", heads * 3 + [i] * 6 + [vp, vp, i, i, f] + heads + [vp, vp]),
            ("dsq_attention_bwd", heads * 4 + [vp] + heads + [i] * 6 + [vp, vp, i, i, f] + heads * 3 + [vp, sz, vp]),
            ("dsq_attention_cache", heads + [i] * 5 + [vp, i, i, vp, vp, i64, i, vp, i64, i, vp, vp, i, f] + heads + [vp, sz, vp])):
        getattr(lib, name).restype = i
        getattr(lib, name).argtypes = args
    lib.dsq_pack_weights_w4.restype = i
    lib.dsq_pack_weights_w4.argtypes = [vp, vp, vp, vp, i, i, i, vp, sz, vp, sz, vp]
    lib.dsq_linear_w4.restype = i
    lib.dsq_linear_w4.argtypes = [vp, i64, i, i, i, i, i, vp, vp, vp, vp, i64, vp]
    lib.dsq_linear_w4a8.restype = i
    lib.dsq_linear_w4a8.argtypes = [vp, sz, vp, i, i, i, i, vp, vp, vp, i, vp, i64, vp]
    lib.dsq_status_string.restype = C.c_char_p
    lib.dsq_status_string.argtypes = [i]
    _lib = lib
    return lib


_marshal = None


class _NoMarshal:
    """In the module's place where it does not load: leaves every call to the ctypes path."""

    @staticmethod
    def quantize_act(*args):
        return None

    conv2d = conv2d_requant = conv2d_wq = soft_quantize_fwd = soft_quantize_bwd = quantize_act
    rms_norm = rms_norm_bwd = linear_w4 = linear_w4a8 = quantize_act
    qk_norm_rope = qk_norm_rope_bwd = attention = attention_bwd = attention_cache = quantize_act


def load_marshal():
    """The native marshalling module, bound to the library's entry points; where it is missing or does not load
    (built for another PyTorch), a warning and a stand-in that leaves the calls to ctypes: 5 us a call, same results."""
    global _marshal
    if _marshal is None:
        lib = load_library()
        try:
            from . import _marshal as module
        except ImportError as e:
            warnings.warn("the _marshal module of paper_1908_05033_amd is missing or does not load (%s): calls are marshalled "
                          "by ctypes, some 5 us slower each (python -c 'import __graft_entry__ as g; g.build()' builds it)" % e,
                          RuntimeWarning, stacklevel=3)
            _marshal = _NoMarshal
            return _marshal
        module.init(dsq_conv_desc, *(C.cast(getattr(lib, name), C.c_void_p).value for name in
                                     ("dsq_quantize_act", "dsq_conv2d", "dsq_conv2d_requant", "dsq_conv2d_wq",
                                      "dsq_soft_quantize_fwd", "dsq_soft_quantize_bwd")))
        module.init_lm(*(C.cast(getattr(lib, name), C.c_void_p).value for name in
                         ("dsq_rms_norm", "dsq_rms_norm_bwd", "dsq_linear_w4", "dsq_linear_w4a8", "dsq_code_row_bytes",
                          "dsq_w4_packed_bytes", "dsq_w4_scale_bytes")))
        module.init_heads(*(C.cast(getattr(lib, name), C.c_void_p).value for name in
                            ("dsq_qk_norm_rope", "dsq_qk_norm_rope_bwd", "dsq_attention", "dsq_attention_bwd", "dsq_attention_cache")))
        _marshal = module
    return _marshal


def _check(status):
    if status != DSQ_OK:
        raise DsqError(status, load_library().dsq_status_string(status).decode())


def _dev_ptr(t, dtype=None, allow_none=False):
    if t is None:
        if allow_none:
            return None
        raise DsqError(1, "a required tensor is None")
    if isinstance(t, int):          # raw device address
        return t
    if not t.is_cuda:
        raise TypeError("libdsqconv takes device tensors")
    if dtype is not None and t.dtype != dtype:
        raise TypeError("expected %s, got %s" % (dtype, t.dtype))
    if not t.is_contiguous():
        raise TypeError("tensor must be contiguous")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def dsq_act_packed_bytes(N, H, W, C, bits):
    return int(load_library().dsq_act_packed_bytes(N, H, W, C, bits))


def dsq_act_packed_bytes_ex(N, H, W, C, bits, packing):
    return int(load_library().dsq_act_packed_bytes_ex(N, H, W, C, bits, packing))


def dsq_wgt_packed_bytes(C_out, C_in, R, S, bits):
    return int(load_library().dsq_wgt_packed_bytes(C_out, C_in, R, S, bits))


def dsq_wgt_aux_bytes(C_out, R, S):
    return int(load_library().dsq_wgt_aux_bytes(C_out, R, S))


def dsq_quantize_act(x, layout, N, C, H, W, l, u, bits, codes_packed, pix_code_sum, stream=None):
    status = (_marshal or load_marshal()).quantize_act(x, layout, N, C, H, W, l, u, bits, codes_packed, pix_code_sum, stream)
    if status is None:
        _check(load_library().dsq_quantize_act(
            _dev_ptr(x, torch.float32), layout, N, C, H, W, l, u, bits,
            _dev_ptr(codes_packed, torch.uint8), codes_packed.numel() if codes_packed is not None else 0,
            _dev_ptr(pix_code_sum, torch.int32), _stream(stream)))
    elif status != DSQ_OK:
        _check(status)


def dsq_quantize_act_ex(x, layout, N, C, H, W, l, u, bits, packing, codes_packed, pix_code_sum, stream=None):
    _check(load_library().dsq_quantize_act_ex(
        _dev_ptr(x, torch.float32), layout, N, C, H, W, l, u, bits, packing,
        _dev_ptr(codes_packed, torch.uint8), codes_packed.numel() if codes_packed is not None else 0,
        _dev_ptr(pix_code_sum, torch.int32), _stream(stream)))


def dsq_pack_weights(w_oihw, l_w, u_w, codes_oihw, C_out, C_in, R, S, bits, w_packed, w_aux,
                     stream=None):
    _check(load_library().dsq_pack_weights(
        _dev_ptr(w_oihw, torch.float32, True), _dev_ptr(l_w, torch.float32),
        _dev_ptr(u_w, torch.float32), _dev_ptr(codes_oihw, torch.uint8, True),
        C_out, C_in, R, S, bits,
        _dev_ptr(w_packed, torch.uint8), w_packed.numel() if w_packed is not None else 0,
        _dev_ptr(w_aux, torch.uint8), w_aux.numel() if w_aux is not None else 0,
        _stream(stream)))


def dsq_pack_weights_for(w_oihw, l_w, u_w, codes_oihw, C_out, C_in, R, S, bits_w, bits_act, w_packed, w_aux,
                         stream=None):
    _check(load_library().dsq_pack_weights_for(
        _dev_ptr(w_oihw, torch.float32, True), _dev_ptr(l_w, torch.float32),
        _dev_ptr(u_w, torch.float32), _dev_ptr(codes_oihw, torch.uint8, True),
        C_out, C_in, R, S, bits_w, bits_act,
        _dev_ptr(w_packed, torch.uint8), w_packed.numel() if w_packed is not None else 0,
        _dev_ptr(w_aux, torch.uint8), w_aux.numel() if w_aux is not None else 0,
        _stream(stream)))


def dsq_conv2d(desc, act_packed, pix_code_sum, l_a, u_a, w_packed, w_aux, out, out_layout,
               acc_or_none=None, stream=None):
    status = (_marshal or load_marshal()).conv2d(desc, act_packed, pix_code_sum, l_a, u_a, w_packed, w_aux, out, out_layout, acc_or_none, stream)
    if status is None:
        _check(load_library().dsq_conv2d(
            C.byref(desc) if desc is not None else None,
            _dev_ptr(act_packed, torch.uint8), _dev_ptr(pix_code_sum, torch.int32), l_a, u_a,
            _dev_ptr(w_packed, torch.uint8), _dev_ptr(w_aux, torch.uint8),
            _dev_ptr(out, torch.float32), out_layout,
            _dev_ptr(acc_or_none, torch.int32, True), _stream(stream)))
    elif status != DSQ_OK:
        _check(status)


def dsq_conv2d_requant(desc, act_packed, pix_code_sum, l_a, u_a, w_packed, w_aux, scale, shift, relu,
                       l_next, u_next, bits_next, codes_next, pix_code_sum_next, stream=None):
    status = (_marshal or load_marshal()).conv2d_requant(desc, act_packed, pix_code_sum, l_a, u_a, w_packed, w_aux, scale, shift,
                                                        relu, l_next, u_next, bits_next, codes_next, pix_code_sum_next, stream)
    if status is None:
        _check(load_library().dsq_conv2d_requant(
            C.byref(desc) if desc is not None else None,
            _dev_ptr(act_packed, torch.uint8), _dev_ptr(pix_code_sum, torch.int32), l_a, u_a,
            _dev_ptr(w_packed, torch.uint8), _dev_ptr(w_aux, torch.uint8),
            _dev_ptr(scale, torch.float32, True), _dev_ptr(shift, torch.float32, True), int(bool(relu)),
            l_next, u_next, bits_next,
            _dev_ptr(codes_next, torch.uint8), codes_next.numel() if codes_next is not None else 0,
            _dev_ptr(pix_code_sum_next, torch.int32), _stream(stream)))
    elif status != DSQ_OK:
        _check(status)


def dsq_conv2d_wq(desc, x, x_layout, w_packed, w_aux, out, out_layout, stream=None):
    status = (_marshal or load_marshal()).conv2d_wq(desc, x, x_layout, w_packed, w_aux, out, out_layout, stream)
    if status is None:
        _check(load_library().dsq_conv2d_wq(
            C.byref(desc) if desc is not None else None, _dev_ptr(x, torch.float32), x_layout,
            _dev_ptr(w_packed, torch.uint8), _dev_ptr(w_aux, torch.uint8), _dev_ptr(out, torch.float32), out_layout,
            _stream(stream)))
    elif status != DSQ_OK:
        _check(status)


def dsq_soft_quantize_fwd(x, l, u, alpha, bits, y, stream=None):
    status = (_marshal or load_marshal()).soft_quantize_fwd(x, l, u, alpha, bits, y, stream)
    if status is None:
        _check(load_library().dsq_soft_quantize_fwd(_dev_ptr(x, torch.float32), x.numel(), l, u, alpha, bits,
                                                    _dev_ptr(y, torch.float32), _stream(stream)))
    elif status != DSQ_OK:
        _check(status)


def dsq_soft_quantize_bwd(x, grad_y, l, u, alpha, bits, grad_x, grad_alpha_l_u, stream=None):
    status = (_marshal or load_marshal()).soft_quantize_bwd(x, grad_y, l, u, alpha, bits, grad_x, grad_alpha_l_u, stream)
    if status is None:
        _check(load_library().dsq_soft_quantize_bwd(
            _dev_ptr(x, torch.float32), _dev_ptr(grad_y, torch.float32), x.numel(), l, u, alpha, bits,
            _dev_ptr(grad_x, torch.float32), _dev_ptr(grad_alpha_l_u, torch.float64), _stream(stream)))
    elif status != DSQ_OK:
        _check(status)


def dsq_conv2d_plan(desc, chained=False, l_a=0.0):
    buf = C.create_string_buffer(512)
    _check(load_library().dsq_conv2d_plan(C.byref(desc), int(bool(chained)), l_a, buf, len(buf)))
    return buf.value.decode()


# ---------------------------------------------------------------------------
# Layers of language models.  Rows of floats are tensors of two dimensions whose rows may lie
# apart (stride(1) is 1); their shapes and type are taken from them.
# ---------------------------------------------------------------------------

_DTYPES = {torch.float32: DSQ_F32, torch.float16: DSQ_F16, torch.bfloat16: DSQ_BF16}


def dsq_code_row_bytes(dim):
    return int(load_library().dsq_code_row_bytes(dim))


def dsq_rms_norm_bwd_bytes(rows, dim):
    return int(load_library().dsq_rms_norm_bwd_bytes(rows, dim))


def dsq_w4_packed_bytes(N, K):
    return int(load_library().dsq_w4_packed_bytes(N, K))


def dsq_w4_scale_bytes(N, K, group):
    return int(load_library().dsq_w4_scale_bytes(N, K, group))


def _here(t, name):
    """A device tensor of the current device: the stream and the kernel are that device's."""
    if not isinstance(t, torch.Tensor):
        raise DsqError(1, "%s is a required tensor" % name) if t is None else TypeError("%s: expected a tensor" % name)
    if not t.is_cuda:
        raise TypeError("libdsqconv takes device tensors")
    if t.get_device() != torch.cuda.current_device():
        raise TypeError("%s is on another device than the current one" % name)
    return t


def _rows(t, name, shape=None, dtype=None, strided=True, allow_none=False):
    """(address, distance of rows) of a tensor [rows, elements], (None, 0) where it may be None."""
    if t is None and allow_none:
        return None, 0
    _here(t, name)
    if t.dim() != 2 or (shape is not None and tuple(t.shape) != tuple(shape)):
        raise DsqError(4, "%s has the shape %s%s" % (name, list(t.shape), "" if shape is None else ", expected %s" % list(shape)))
    if dtype is None:
        if t.dtype not in _DTYPES:
            raise TypeError("%s: expected float32, float16 or bfloat16, got %s" % (name, t.dtype))
    elif t.dtype != dtype:
        raise TypeError("%s: expected %s, got %s" % (name, dtype, t.dtype))
    if t.numel() and t.shape[1] > 1 and t.stride(1) != 1:
        raise TypeError("%s: the elements of a row must lie side by side" % name)
    stride = t.stride(0) if t.shape[0] > 1 else t.shape[1]
    if not strided and stride != t.shape[1]:
        raise TypeError("%s must be contiguous" % name)
    return t.data_ptr(), stride


def _vector(t, name, n, dtype, allow_none=False):
    """Address of a contiguous tensor of n elements."""
    if t is None and allow_none:
        return None
    if _here(t, name).dtype != dtype:
        raise TypeError("%s: expected %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous():
        raise TypeError("%s must be contiguous" % name)
    if t.numel() != n:
        raise DsqError(4, "%s has %d elements, expected %d" % (name, t.numel(), n))
    return t.data_ptr()


def _bytes(t, name, allow_none=False):
    """(address, size) of a uint8 buffer."""
    if t is None and allow_none:
        return None, 0
    if _here(t, name).dtype != torch.uint8:
        raise TypeError("%s: expected %s, got %s" % (name, torch.uint8, t.dtype))
    if not t.is_contiguous():
        raise TypeError("%s must be contiguous" % name)
    return t.data_ptr(), t.numel()


def _code_rows(t, name, rows, dim):
    """Address of int8 rows with their pitch."""
    return _rows(t, name, (rows, dsq_code_row_bytes(dim)), torch.int8, strided=False)[0]


def dsq_rms_norm(x, residual, weight, eps, sum_out, y, codes, scales, rstd, stream=None):
    """x, residual [rows, dim]; sum_out, y [rows, dim]; codes int8 [rows, dsq_code_row_bytes(dim)]; all but x may be None."""
    status = (_marshal or load_marshal()).rms_norm(x, residual, weight, eps, sum_out, y, codes, scales, rstd, stream)
    if status is not None:
        if status != DSQ_OK:
            _check(status)
        return
    xp, xs = _rows(x, "x")
    (rows, dim), dt = x.shape, x.dtype
    rp, rs = _rows(residual, "residual", x.shape, dt, allow_none=True)
    _check(load_library().dsq_rms_norm(
        xp, xs, rp, rs, _vector(weight, "weight", dim, dt, True), _DTYPES[dt], rows, dim, eps,
        _rows(sum_out, "sum_out", x.shape, dt, False, True)[0], _rows(y, "y", x.shape, dt, False, True)[0],
        None if codes is None else _code_rows(codes, "codes", rows, dim), 0 if codes is None else codes.numel(),
        _vector(scales, "scales", rows, torch.float32, True), _vector(rstd, "rstd", rows, torch.float32, True), _stream(stream)))


def dsq_rms_norm_bwd(h, weight, rstd, grad_y, grad_sum, grad_x, grad_weight, workspace, stream=None):
    """h, grad_y, grad_sum, grad_x [rows, dim]; grad_weight float32 [dim]; workspace uint8 of dsq_rms_norm_bwd_bytes(rows, dim)."""
    status = (_marshal or load_marshal()).rms_norm_bwd(h, weight, rstd, grad_y, grad_sum, grad_x, grad_weight, workspace, stream)
    if status is not None:
        if status != DSQ_OK:
            _check(status)
        return
    hp, hs = _rows(h, "h")
    (rows, dim), dt = h.shape, h.dtype
    gp, gs = _rows(grad_y, "grad_y", h.shape, dt)
    sp, ss = _rows(grad_sum, "grad_sum", h.shape, dt, allow_none=True)
    ws, nbytes = _bytes(workspace, "workspace", True)
    _check(load_library().dsq_rms_norm_bwd(
        hp, hs, _vector(weight, "weight", dim, dt, True), _vector(rstd, "rstd", rows, torch.float32), gp, gs, sp, ss,
        _DTYPES[dt], rows, dim, _rows(grad_x, "grad_x", h.shape, dt, False)[0],
        _vector(grad_weight, "grad_weight", dim, torch.float32, True), ws, nbytes, _stream(stream)))


def dsq_pack_weights_w4(w, codes, scale, zero, N, K, group, w_packed, w_scales, stream=None):
    """w float32 or codes uint8 [N, K]; scale float32 and zero uint8 [N, ceil(K / group)] or None."""
    groups = N * -(-K // group) if group > 0 else 0
    wp, wn = _bytes(w_packed, "w_packed")
    sp, sn = _bytes(w_scales, "w_scales")
    _check(load_library().dsq_pack_weights_w4(
        _vector(w, "w", N * K, torch.float32, True), _vector(codes, "codes", N * K, torch.uint8, True),
        _vector(scale, "scale", groups, torch.float32, True), _vector(zero, "zero", groups, torch.uint8, True),
        N, K, group, wp, wn, sp, sn, _stream(stream)))


def _packed(w_packed, w_scales, N, K, group):
    wp, wn = _bytes(w_packed, "w_packed")
    sp, sn = _bytes(w_scales, "w_scales")
    if wn < dsq_w4_packed_bytes(N, K) or sn < dsq_w4_scale_bytes(N, K, group):
        raise DsqError(7, "w_packed or w_scales is smaller than a layer of %d x %d in groups of %d" % (N, K, group))
    return wp, sp


def dsq_linear_w4(x, w_packed, w_scales, N, K, group, bias, out, stream=None):
    """x [M, K], out [M, N], bias [N] or None, of one type."""
    status = (_marshal or load_marshal()).linear_w4(x, w_packed, w_scales, N, K, group, bias, out, stream)
    if status is not None:
        if status != DSQ_OK:
            _check(status)
        return
    xp, xs = _rows(x, "x", (x.shape[0], K) if isinstance(x, torch.Tensor) and x.dim() == 2 else None)
    op, os_ = _rows(out, "out", (x.shape[0], N), x.dtype)
    wp, sp = _packed(w_packed, w_scales, N, K, group)
    _check(load_library().dsq_linear_w4(xp, xs, _DTYPES[x.dtype], x.shape[0], N, K, group, wp, sp,
                                        _vector(bias, "bias", N, x.dtype, True), op, os_, _stream(stream)))


def dsq_linear_w4a8(codes, scales, w_packed, w_scales, N, K, group, bias, out, stream=None):
    """codes int8 [M, dsq_code_row_bytes(K)], scales float32 [M]; out [M, N] and bias [N] or None, of one type."""
    status = (_marshal or load_marshal()).linear_w4a8(codes, scales, w_packed, w_scales, N, K, group, bias, out, stream)
    if status is not None:
        if status != DSQ_OK:
            _check(status)
        return
    op, os_ = _rows(out, "out", (out.shape[0], N) if isinstance(out, torch.Tensor) and out.dim() == 2 else None)
    M = out.shape[0]
    cp = _code_rows(codes, "codes", M, K)
    wp, sp = _packed(w_packed, w_scales, N, K, group)
    _check(load_library().dsq_linear_w4a8(cp, codes.numel(), _vector(scales, "scales", M, torch.float32), M, N, K, group, wp, sp,
                                          _vector(bias, "bias", N, out.dtype, True), _DTYPES[out.dtype], op, os_, _stream(stream)))


# ---------------------------------------------------------------------------
# Heads of a block: tensors [rows, heads, dim] whose rows and heads may lie apart (stride(2) is 1).
# ---------------------------------------------------------------------------

def dsq_qk_norm_rope_bwd_bytes(rows, q_heads, kv_heads, dim):
    return int(load_library().dsq_qk_norm_rope_bwd_bytes(rows, q_heads, kv_heads, dim))


def dsq_attention_bwd_bytes(q_rows, q_heads):
    return int(load_library().dsq_attention_bwd_bytes(q_rows, q_heads))


def dsq_attention_cache_bytes(sequences, max_rows, q_heads, kv_heads, dim):
    return int(load_library().dsq_attention_cache_bytes(sequences, max_rows, q_heads, kv_heads, dim))


def _heads(t, name, shape=None, dtype=None, allow_none=False):
    """(address, distance of rows, distance of heads) of a tensor [rows, heads, dim]; zeros where it may be None.
    Entries of the shape that are None are not compared."""
    if t is None and allow_none:
        return None, 0, 0
    _here(t, name)
    if t.dim() != 3 or (shape is not None and any(n is not None and n != m for n, m in zip(shape, t.shape))):
        raise DsqError(4, "%s has the shape %s%s" % (name, list(t.shape), "" if shape is None else ", expected %s" % list(shape)))
    if t.dtype not in _DTYPES if dtype is None else t.dtype != dtype:
        raise TypeError("%s: expected %s, got %s" % (name, "float32, float16 or bfloat16" if dtype is None else dtype, t.dtype))
    rows, heads, dim = t.shape
    if t.numel() and dim > 1 and t.stride(2) != 1:
        raise TypeError("%s: the elements of a head must lie side by side" % name)
    return t.data_ptr(), t.stride(0) if rows > 1 else heads * dim, t.stride(1) if heads > 1 else dim


def _rotation(positions, rows, pair_axis, frequencies):
    """positions, axes, pair_axis, frequencies, rope_dim as the library takes them."""
    pairs = frequencies.numel() if isinstance(frequencies, torch.Tensor) else 0
    axes = positions.shape[0] if isinstance(positions, torch.Tensor) and positions.dim() == 2 else 1
    return (_vector(positions, "positions", axes * rows, torch.int32, True), axes, _vector(pair_axis, "pair_axis", pairs, torch.uint8, True),
            _vector(frequencies, "frequencies", pairs, torch.float32, True), 2 * pairs)


def _both(q, k):
    """rows, query heads, key heads, dim and type of q and k, one of which may be None."""
    one = q if q is not None else k
    _heads(one, "q")
    rows, heads, dim = one.shape
    if q is not None and k is not None:
        _heads(k, "k", (rows, None, dim), q.dtype)
    return rows, 0 if q is None else heads, 0 if k is None else k.shape[1], dim, one.dtype


def dsq_qk_norm_rope(q, k, v, q_weight, k_weight, eps, positions, pair_axis, frequencies, interleaved, q_out, k_out, k_cache, v_cache,
                     slots, stream=None):
    """q [rows, q_heads, dim], k and v [rows, kv_heads, dim]; weights [dim]; positions int32 [rows] or [axes, rows]; frequencies
    float32 and pair_axis uint8 [rope_dim / 2]; caches [pages, kv_heads, page, dim]; slots int64 [rows].  What is not wanted is None."""
    status = (_marshal or load_marshal()).qk_norm_rope(q, k, v, q_weight, k_weight, eps, positions, pair_axis, frequencies, interleaved, q_out,
                                                       k_out, k_cache, v_cache, slots, stream)
    if status is not None:
        if status != DSQ_OK:
            _check(status)
        return
    rows, hq, hk, dim, dt = _both(q, k)
    pages, page = 0, 0
    if k_cache is not None:
        pages, page = _cache(k_cache, "k_cache", hk, dim, dt)
        if v_cache is not None and _cache(v_cache, "v_cache", hk, dim, dt) != (pages, page):
            raise DsqError(4, "k_cache and v_cache have different shapes")
    elif v_cache is not None or slots is not None:
        raise DsqError(1, "k_cache is a required tensor where v_cache or slots is given")
    _check(load_library().dsq_qk_norm_rope(
        *_heads(q, "q", allow_none=True), *_heads(k, "k", allow_none=True), *_heads(v, "v", (rows, hk, dim), dt, True), _DTYPES[dt], rows, hq, hk, dim,
        _vector(q_weight, "q_weight", dim, dt, True), _vector(k_weight, "k_weight", dim, dt, True), eps,
        *_rotation(positions, rows, pair_axis, frequencies), int(bool(interleaved)), *_heads(q_out, "q_out", (rows, hq, dim), dt, True),
        *_heads(k_out, "k_out", (rows, hk, dim), dt, True), None if k_cache is None else k_cache.data_ptr(),
        None if v_cache is None else v_cache.data_ptr(), pages, page, _vector(slots, "slots", rows, torch.int64, True), _stream(stream)))


def dsq_qk_norm_rope_bwd(q, k, q_weight, k_weight, eps, positions, pair_axis, frequencies, interleaved, grad_q_out, grad_k_out, grad_q, grad_k,
                         grad_q_weight, grad_k_weight, workspace, stream=None):
    """As dsq_qk_norm_rope; gradients in the shapes of q and k; of the weights float32 [dim] or None; workspace uint8 of
    dsq_qk_norm_rope_bwd_bytes(..)."""
    status = (_marshal or load_marshal()).qk_norm_rope_bwd(q, k, q_weight, k_weight, eps, positions, pair_axis, frequencies, interleaved, grad_q_out, grad_k_out,
                                                           grad_q, grad_k, grad_q_weight, grad_k_weight, workspace, stream)
    if status is not None:
        if status != DSQ_OK:
            _check(status)
        return
    rows, hq, hk, dim, dt = _both(q, k)
    like = lambda t, name, heads: _heads(t, name, (rows, heads, dim), dt, heads == 0)
    ws, nbytes = _bytes(workspace, "workspace", True)
    _check(load_library().dsq_qk_norm_rope_bwd(
        *_heads(q, "q", allow_none=True), *_heads(k, "k", allow_none=True), _DTYPES[dt], rows, hq, hk, dim,
        _vector(q_weight, "q_weight", dim, dt, True), _vector(k_weight, "k_weight", dim, dt, True), eps,
        *_rotation(positions, rows, pair_axis, frequencies), int(bool(interleaved)), *like(grad_q_out, "grad_q_out", hq),
        *like(grad_k_out, "grad_k_out", hk), *like(grad_q, "grad_q", hq), *like(grad_k, "grad_k", hk),
        _vector(grad_q_weight, "grad_q_weight", dim, torch.float32, True), _vector(grad_k_weight, "grad_k_weight", dim, torch.float32, True),
        ws, nbytes, _stream(stream)))


def _prompts(q, k, v, q_starts, k_starts):
    """Rows, keys, heads, dim, type, addresses of the starts and the number of sequences."""
    _heads(q, "q")
    (rows, hq, dim), dt = q.shape, q.dtype
    _heads(k, "k", (None, None, dim), dt)
    _heads(v, "v", k.shape, dt)
    sequences = 1
    if q_starts is not None:
        sequences = max(0, _here(q_starts, "q_starts").numel() - 1)
    starts = [_vector(t, name, sequences + 1, torch.int32, True) for t, name in ((q_starts, "q_starts"), (k_starts, "k_starts"))]
    return rows, k.shape[0], hq, k.shape[1], dim, dt, starts, sequences


def dsq_attention(q, k, v, q_starts, k_starts, causal, scale, out, lse, stream=None):
    """q, out [rows, q_heads, dim]; k, v [keys, kv_heads, dim]; starts int32 [sequences + 1] or None; lse float32 [q_heads, rows] or None."""
    status = (_marshal or load_marshal()).attention(q, k, v, q_starts, k_starts, causal, scale, out, lse, stream)
    if status is not None:
        if status != DSQ_OK:
            _check(status)
        return
    rows, keys, hq, hk, dim, dt, starts, sequences = _prompts(q, k, v, q_starts, k_starts)
    _check(load_library().dsq_attention(
        *_heads(q, "q"), *_heads(k, "k"), *_heads(v, "v"), _DTYPES[dt], rows, keys, hq, hk, dim, *starts, sequences, int(bool(causal)), scale,
        *_heads(out, "out", q.shape, dt), _vector(lse, "lse", hq * rows, torch.float32, True), _stream(stream)))


def dsq_attention_bwd(q, k, v, out, lse, grad_out, q_starts, k_starts, causal, scale, grad_q, grad_k, grad_v, workspace, stream=None):
    """As dsq_attention, with its out and lse; gradients in the shapes of what they belong to; workspace uint8 of
    dsq_attention_bwd_bytes(rows, q_heads)."""
    status = (_marshal or load_marshal()).attention_bwd(q, k, v, out, lse, grad_out, q_starts, k_starts, causal, scale, grad_q, grad_k,
                                                        grad_v, workspace, stream)
    if status is not None:
        if status != DSQ_OK:
            _check(status)
        return
    rows, keys, hq, hk, dim, dt, starts, sequences = _prompts(q, k, v, q_starts, k_starts)
    ws, nbytes = _bytes(workspace, "workspace", True)
    _check(load_library().dsq_attention_bwd(
        *_heads(q, "q"), *_heads(k, "k"), *_heads(v, "v"), *_heads(out, "out", q.shape, dt), _vector(lse, "lse", hq * rows, torch.float32),
        *_heads(grad_out, "grad_out", q.shape, dt), _DTYPES[dt], rows, keys, hq, hk, dim, *starts, sequences, int(bool(causal)), scale,
        *_heads(grad_q, "grad_q", q.shape, dt), *_heads(grad_k, "grad_k", k.shape, dt), *_heads(grad_v, "grad_v", k.shape, dt),
        ws, nbytes, _stream(stream)))


def _cache(t, name, heads, dim, dtype):
    """Pages and page size of a cache [pages, heads, page, dim]."""
    if _here(t, name).dtype != dtype:
        raise TypeError("%s: expected %s, got %s" % (name, dtype, t.dtype))
    if t.dim() != 4 or t.shape[1] != heads or t.shape[3] != dim:
        raise DsqError(4, "%s has the shape %s, expected [pages, %d, page, %d]" % (name, list(t.shape), heads, dim))
    if not t.is_contiguous():
        raise TypeError("%s must be contiguous" % name)
    return t.shape[0], t.shape[2]


def dsq_attention_cache(q, q_starts, max_rows, k_cache, v_cache, page_table, lengths, tree, scale, out, workspace, stream=None):
    """q, out [rows, q_heads, dim]; q_starts int32 [sequences + 1] or None; caches [pages, kv_heads, page, dim]; page_table int32
    [sequences, pages of each] whose rows may lie apart; lengths int32 [sequences]; tree int64 [rows, words] or None; workspace uint8 of
    dsq_attention_cache_bytes(sequences, max_rows, q_heads, kv_heads, dim)."""
    status = (_marshal or load_marshal()).attention_cache(q, q_starts, max_rows, k_cache, v_cache, page_table, lengths, tree, scale, out, workspace, stream)
    if status is not None:
        if status != DSQ_OK:
            _check(status)
        return
    qp = _heads(q, "q")
    (rows, hq, dim), dt = q.shape, q.dtype
    if _here(k_cache, "k_cache").dim() != 4:
        raise DsqError(4, "k_cache has the shape %s, expected [pages, kv_heads, page, dim]" % list(k_cache.shape))
    hk = k_cache.shape[1]
    pages, page = _cache(k_cache, "k_cache", hk, dim, dt)
    if _cache(v_cache, "v_cache", hk, dim, dt) != (pages, page):
        raise DsqError(4, "k_cache and v_cache have different shapes")
    sequences = _here(lengths, "lengths").numel()
    tp, tr = _rows(page_table, "page_table", (sequences, page_table.shape[-1]) if isinstance(page_table, torch.Tensor) and page_table.dim() else None,
                   torch.int32)
    words = 0
    if tree is not None:
        if _here(tree, "tree").dim() != 2 or not tree.shape[1]:
            raise DsqError(4, "tree has the shape %s, expected [%d, words]" % (list(tree.shape), rows))
        words = tree.shape[1]
    ws, nbytes = _bytes(workspace, "workspace")
    _check(load_library().dsq_attention_cache(
        *qp, _DTYPES[dt], rows, hq, hk, dim, _vector(q_starts, "q_starts", sequences + 1, torch.int32, True), sequences, max_rows,
        k_cache.data_ptr(), v_cache.data_ptr(), pages, page, tp, tr, page_table.shape[1], _vector(lengths, "lengths", sequences, torch.int32),
        _vector(tree, "tree", rows * words, torch.int64, True), words, scale, *_heads(out, "out", q.shape, dt), ws, nbytes, _stream(stream)))


# ---------------------------------------------------------------------------
# Small conveniences: buffer allocation for one layer (still no arithmetic).
# ---------------------------------------------------------------------------

@dataclass
class LayerBuffers:
    desc: dsq_conv_desc
    act_packed: torch.Tensor
    pix_code_sum: torch.Tensor
    w_packed: torch.Tensor
    w_aux: torch.Tensor
    out: torch.Tensor          # NHWC float32 [N, Ho, Wo, C_out]
    acc: torch.Tensor = None   # NHWC int32, optional


def make_desc(N, C_in, H, W, C_out, R, S, stride, pad, bits, flags=0):
    return dsq_conv_desc(N, C_in, H, W, C_out, R, S, stride, pad, bits, flags)


def alloc_layer(N, C_in, H, W, C_out, R, S, stride, pad, bits, device="cuda", with_acc=False, flags=0):
    """Device buffers for one layer, sized by the library's own size queries."""
    Ho = (H + 2 * pad - R) // stride + 1
    Wo = (W + 2 * pad - S) // stride + 1
    u8 = dict(dtype=torch.uint8, device=device)
    return LayerBuffers(
        desc=make_desc(N, C_in, H, W, C_out, R, S, stride, pad, bits, flags),
        act_packed=torch.empty(dsq_act_packed_bytes(N, H, W, C_in, bits), **u8),
        pix_code_sum=torch.empty(N * H * W, dtype=torch.int32, device=device),
        w_packed=torch.empty(dsq_wgt_packed_bytes(C_out, C_in, R, S, bits), **u8),
        w_aux=torch.empty(dsq_wgt_aux_bytes(C_out, R, S), **u8),
        out=torch.empty((N, Ho, Wo, C_out), dtype=torch.float32, device=device),
        acc=torch.empty((N, Ho, Wo, C_out), dtype=torch.int32, device=device) if with_acc else None,
    )
