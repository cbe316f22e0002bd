"""ctypes binding of include/dcnv4.h: same names, argument marshalling only.

The tensor arguments are torch tensors on the GPU (torch is used for device memory and
streams, nothing else); every step of the operator runs inside libdcnv4.so.  If the
library has not been built the import of it fails loudly -- there is no fallback path.

With `stream`, results and workspaces that the caller does not bring are memory of that stream, as torch's are of the current one:
memory of the current one may still be read there by what was queued before, and would go back to it while the call writes.  Who
uses such results on another stream waits for the call first and, where they are given back before that use has ended, marks them
(torch.Tensor.record_stream).
"""
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdcnv4.so")

DCNV4_F32, DCNV4_F16 = 0, 1
DCNV4_OK = 0

# every symbol include/dcnv4.h declares
EXPORTS = (
    "dcnv4_output_hw", "dcnv4_forward", "dcnv4_backward", "dcnv4_forward_merged", "dcnv4_backward_merged",
    "dcnv4_forward_softmax", "dcnv4_backward_softmax",
    "dcnv4_linear", "dcnv4_depthwise3x3", "dcnv4_module_forward", "dcnv4_module_workspace_bytes",
    "dcnv4_module_forward_static", "dcnv4_module_static_workspace_limit",
    "dcnv4_layer_norm", "dcnv4_layer_norm_backward", "dcnv4_layer_norm_workspace_bytes",
    "dcnv4_dropout", "dcnv4_dropout_backward",
    "dcnv4_dropout_add_layer_norm", "dcnv4_dropout_add_layer_norm_backward",
    "dcnv4_linear_cross_entropy", "dcnv4_linear_cross_entropy_backward", "dcnv4_linear_cross_entropy_workspace_bytes",
    "dcnv4_linear_backward", "dcnv4_linear_backward_workspace_bytes",
    "dcnv4_gated_linear", "dcnv4_gated_linear_backward", "dcnv4_gated_linear_workspace_bytes",
    "dcnv4_norm_scale_add_norm", "dcnv4_norm_scale_add_norm_backward", "dcnv4_norm_scale_add_norm_workspace_bytes",
    "dcnv4_adamw",
    "dcnv4_forward_algorithmic_bytes", "dcnv4_backward_algorithmic_bytes",
    "dcnv4_forward_merged_algorithmic_bytes", "dcnv4_backward_merged_algorithmic_bytes",
    "dcnv4_set_option", "dcnv4_last_kernel_name", "dcnv4_status_string",
)

_lib = None


class AdamwTensor(ctypes.Structure):
    """dcnv4_adamw_tensor."""
    _fields_ = [("n", ctypes.c_longlong), ("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("scales", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("lr", ctypes.c_double), ("weight_decay", ctypes.c_double)]


class Dcnv4Error(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        super().__init__(f"{where}: status {status} ({dcnv4_status_string(status)})")


def load_library():
    """Load libdcnv4.so (built in-tree by paper_2401_06197_amd.build); raise if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2401_06197_amd.build` "
            "(the DCNv4 operator has no fallback implementation)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, ci, cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    ip = ctypes.POINTER(ctypes.c_int)
    lib.dcnv4_output_hw.argtypes = [ci] * 10 + [ip, ip]
    lib.dcnv4_output_hw.restype = ci
    geo = [ci] * 13 + [cf, ci, vp]
    lib.dcnv4_forward.argtypes = [vp] * 4 + geo
    lib.dcnv4_forward.restype = ci
    lib.dcnv4_backward.argtypes = [vp] * 7 + geo
    lib.dcnv4_backward.restype = ci
    lib.dcnv4_forward_softmax.argtypes = [vp] * 4 + geo
    lib.dcnv4_forward_softmax.restype = ci
    lib.dcnv4_backward_softmax.argtypes = [vp] * 7 + geo
    lib.dcnv4_backward_softmax.restype = ci
    lib.dcnv4_forward_merged.argtypes = [vp] * 3 + geo
    lib.dcnv4_forward_merged.restype = ci
    lib.dcnv4_backward_merged.argtypes = [vp] * 5 + geo
    lib.dcnv4_backward_merged.restype = ci
    for f in (lib.dcnv4_forward_algorithmic_bytes, lib.dcnv4_backward_algorithmic_bytes,
              lib.dcnv4_forward_merged_algorithmic_bytes, lib.dcnv4_backward_merged_algorithmic_bytes):
        f.argtypes = [ci] * 8
        f.restype = ctypes.c_longlong
    lib.dcnv4_linear.argtypes = [vp] * 4 + [ctypes.c_longlong, ci, ci, ci, vp]
    lib.dcnv4_linear.restype = ci
    lib.dcnv4_depthwise3x3.argtypes = [vp] * 4 + [ci] * 5 + [vp]
    lib.dcnv4_depthwise3x3.restype = ci
    lib.dcnv4_module_forward.argtypes = [vp] * 10 + [ctypes.c_longlong, vp] + geo
    lib.dcnv4_module_forward.restype = ci
    lib.dcnv4_module_forward_static.argtypes = [vp] * 10 + geo
    lib.dcnv4_module_forward_static.restype = ci
    lib.dcnv4_module_static_workspace_limit.argtypes = []
    lib.dcnv4_module_static_workspace_limit.restype = ctypes.c_longlong
    lib.dcnv4_module_workspace_bytes.argtypes = [ci] * 8
    lib.dcnv4_module_workspace_bytes.restype = ctypes.c_longlong
    ll, ull = ctypes.c_longlong, ctypes.c_ulonglong
    drop = [cf, ull, ull, vp]
    lib.dcnv4_layer_norm.argtypes = [vp] * 6 + [ll, ci, cf, ci, vp]
    lib.dcnv4_layer_norm_backward.argtypes = [vp] * 9 + [ll, ll, ci, ci, vp]
    lib.dcnv4_layer_norm_workspace_bytes.argtypes = [ll, ci]
    lib.dcnv4_layer_norm_workspace_bytes.restype = ll
    lib.dcnv4_dropout.argtypes = [vp] * 3 + [ll] + drop + [ci, vp]
    lib.dcnv4_dropout_backward.argtypes = [vp] * 2 + [ll] + drop + [ci, vp]
    lib.dcnv4_dropout_add_layer_norm.argtypes = [vp] * 8 + [ll, ci] + drop + [cf, ci, vp]
    lib.dcnv4_dropout_add_layer_norm_backward.argtypes = [vp] * 11 + [ll, ll, ci] + drop + [ci, vp]
    lib.dcnv4_linear_cross_entropy.argtypes = [vp] * 7 + [ll, ll, ci, ci, ll, ci, vp]
    lib.dcnv4_linear_cross_entropy_backward.argtypes = [vp] * 10 + [ll, ll, ci, ci, ll, ci, vp]
    lib.dcnv4_linear_cross_entropy_workspace_bytes.argtypes = [ll, ci, ci, ci, ci]
    lib.dcnv4_linear_cross_entropy_workspace_bytes.restype = ll
    lib.dcnv4_linear_cross_entropy.restype = lib.dcnv4_linear_cross_entropy_backward.restype = ci
    for f in (lib.dcnv4_layer_norm, lib.dcnv4_layer_norm_backward, lib.dcnv4_dropout, lib.dcnv4_dropout_backward,
              lib.dcnv4_dropout_add_layer_norm, lib.dcnv4_dropout_add_layer_norm_backward):
        f.restype = ci
    lib.dcnv4_linear_backward.argtypes = [vp] * 7 + [ll, ll, ci, ci, ci, vp]
    lib.dcnv4_gated_linear.argtypes = [vp] * 5 + [ll, ll, ci, ci, ci, ci, vp]
    lib.dcnv4_gated_linear_backward.argtypes = [vp] * 8 + [ll, ll, ci, ci, ci, ci, vp]
    lib.dcnv4_linear_backward.restype = lib.dcnv4_gated_linear.restype = lib.dcnv4_gated_linear_backward.restype = ci
    lib.dcnv4_linear_backward_workspace_bytes.argtypes = [ll, ci, ci, ci]
    lib.dcnv4_gated_linear_workspace_bytes.argtypes = [ll, ci, ci, ci, ci]
    lib.dcnv4_linear_backward_workspace_bytes.restype = lib.dcnv4_gated_linear_workspace_bytes.restype = ll
    lib.dcnv4_norm_scale_add_norm.argtypes = [vp] * 14 + [ll, ci, ci, ci, cf, ci, vp]
    lib.dcnv4_norm_scale_add_norm_backward.argtypes = [vp] * 22 + [ll, ll, ci, ci, ci, ci, vp]
    lib.dcnv4_norm_scale_add_norm.restype = lib.dcnv4_norm_scale_add_norm_backward.restype = ci
    lib.dcnv4_norm_scale_add_norm_workspace_bytes.argtypes = [ll, ci, ci]
    lib.dcnv4_norm_scale_add_norm_workspace_bytes.restype = ll
    cd = ctypes.c_double
    lib.dcnv4_adamw.argtypes = [ctypes.POINTER(AdamwTensor), ci, cd, cd, cd, ll, vp, vp, ull, ci, ci, vp]
    lib.dcnv4_adamw.restype = ci
    lib.dcnv4_set_option.argtypes = [ctypes.c_char_p, ci]
    lib.dcnv4_set_option.restype = ci
    lib.dcnv4_last_kernel_name.argtypes = [ci]
    lib.dcnv4_last_kernel_name.restype = ctypes.c_char_p
    lib.dcnv4_status_string.argtypes = [ci]
    lib.dcnv4_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _pair(v):
    if type(v) is int:
        return v, v
    return (int(v), int(v)) if isinstance(v, int) else (int(v[0]), int(v[1]))


def dcnv4_status_string(status):
    return load_library().dcnv4_status_string(int(status)).decode()


def dcnv4_output_hw(H, W, kernel=3, stride=1, pad=1, dilation=1):
    (kh, kw), (sh, sw), (ph, pw), (dh, dw) = map(_pair, (kernel, stride, pad, dilation))
    ho, wo = ctypes.c_int(0), ctypes.c_int(0)
    rc = load_library().dcnv4_output_hw(H, W, kh, kw, sh, sw, ph, pw, dh, dw, ctypes.byref(ho), ctypes.byref(wo))
    if rc:
        raise Dcnv4Error(rc, "dcnv4_output_hw")
    return ho.value, wo.value


def dcnv4_set_option(key, value):
    rc = load_library().dcnv4_set_option(key.encode(), int(value))
    if rc:
        raise Dcnv4Error(rc, f"dcnv4_set_option({key!r}, {value})")


def dcnv4_last_kernel_name(backward):
    s = load_library().dcnv4_last_kernel_name(int(backward))
    return s.decode() if s else None


def dcnv4_forward_algorithmic_bytes(N, H, W, G, Cg, Ho, Wo, dtype):
    return int(load_library().dcnv4_forward_algorithmic_bytes(N, H, W, G, Cg, Ho, Wo, dtype))


def dcnv4_backward_algorithmic_bytes(N, H, W, G, Cg, Ho, Wo, dtype):
    return int(load_library().dcnv4_backward_algorithmic_bytes(N, H, W, G, Cg, Ho, Wo, dtype))


def dcnv4_forward_merged_algorithmic_bytes(N, H, W, G, Cg, Ho, Wo, dtype):
    return int(load_library().dcnv4_forward_merged_algorithmic_bytes(N, H, W, G, Cg, Ho, Wo, dtype))


def dcnv4_backward_merged_algorithmic_bytes(N, H, W, G, Cg, Ho, Wo, dtype):
    return int(load_library().dcnv4_backward_merged_algorithmic_bytes(N, H, W, G, Cg, Ho, Wo, dtype))


def _dtype_code(t):
    import torch
    dt = t.dtype
    if dt is torch.float32:
        return DCNV4_F32
    if dt is torch.float16:
        return DCNV4_F16
    raise TypeError(f"dcnv4: unsupported tensor dtype {dt}")


def _check(name, t, ref):
    if not t.is_cuda:
        raise ValueError(f"dcnv4: {name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"dcnv4: {name} must be contiguous")
    if t.dtype != ref.dtype or t.device != ref.device:
        raise ValueError(f"dcnv4: {name} must share dtype and device with x")


def _check_all(x, named):
    """_check of x and of each (name, tensor), whose messages are only made where one does not pass.  (A small call is bound by
    this module: forward and backward of 1x14x14x64 took 36 us, 21 of them here.)"""
    at, dt = x.get_device(), x.dtype
    if at < 0 or not x.is_cuda or not x.is_contiguous():
        _check("x", x, x)
    for name, t in named:
        if t.get_device() != at or t.dtype is not dt or not t.is_contiguous():
            _check(name, t, x)


def _uninitialised(x, shape, stream=None):
    """A plain tensor of x's type on its device, whatever subclass x is of, and of the stream that the call runs on.  (new_empty keeps the
    subclass; it takes 1.2 us where torch.empty takes 1.6.)"""
    import torch
    if stream is not None:
        with torch.cuda.stream(stream):
            return _uninitialised(x, shape)
    return x.new_empty(shape) if type(x) is torch.Tensor else torch.empty(shape, dtype=x.dtype, device=x.device)


def _empty_like(stream, *tensors):
    """torch.empty_like of each, of the stream that the call runs on."""
    import torch
    if stream is not None:
        with torch.cuda.stream(stream):
            return _empty_like(None, *tensors)
    return tuple(map(torch.empty_like, tensors))


def _stream_ptr(stream, device):
    import torch
    if stream is not None:
        return stream.cuda_stream
    # (the handle itself, where torch gives it: the function is not part of its interface.  A Stream object around it takes 1.9 us)
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return torch.cuda.current_stream(device).cuda_stream
    return raw(torch.cuda.current_device() if device.index is None else device.index)


def _call(device, entry, args):
    """The library's entry point on `device`; the switch of devices is left out where it would change nothing.  (Small
    calls are bound by this module: forward of 64x7x7x1024 fp16 15.6 -> 13.6 us a call without the switch and with the
    output size worked out in _conv_hw.)"""
    import torch
    f = getattr(load_library(), entry)
    if torch.cuda.current_device() == device.index:
        rc = f(*args)
    else:
        with torch.cuda.device(device):
            rc = f(*args)
    if rc:
        raise Dcnv4Error(rc, entry)


_INT_MAX = 2 ** 31 - 1


def _conv_hw(H, W, kh, kw, sh, sw, ph, pw, dh, dw):
    """dcnv4_output_hw, worked out here (a call into the library costs more than the arithmetic)."""
    eh, ew = H + 2 * ph - dh * (kh - 1) - 1, W + 2 * pw - dw * (kw - 1) - 1
    if (0 < H and 0 < W and 0 < kh < _INT_MAX and 0 < kw < _INT_MAX and 0 < sh < _INT_MAX and 0 < sw < _INT_MAX
            and 0 <= ph < _INT_MAX and 0 <= pw < _INT_MAX and 0 < dh < _INT_MAX and 0 < dw < _INT_MAX
            and 0 <= eh < _INT_MAX and 0 <= ew < _INT_MAX):
        return eh // sh + 1, ew // sw + 1
    return dcnv4_output_hw(H, W, (kh, kw), (sh, sw), (ph, pw), (dh, dw))          # (refuses, or settles what is left)


def _shape_args(x, offset, mask, kernel, stride, pad, dilation):
    (kh, kw), (sh, sw), (ph, pw), (dh, dw) = _pair(kernel), _pair(stride), _pair(pad), _pair(dilation)
    xshape, oshape, mshape = x.shape, offset.shape, mask.shape
    if len(xshape) != 4 or len(oshape) != 6 or len(mshape) != 5:
        raise ValueError("dcnv4: expected x [N,H,W,C], offset [N,Ho,Wo,G,K,2], mask [N,Ho,Wo,G,K]")
    N, H, W, C = xshape
    G = mshape[3]
    if G < 1 or C % G:
        raise ValueError("dcnv4: C must be a multiple of G")
    Ho, Wo = _conv_hw(H, W, kh, kw, sh, sw, ph, pw, dh, dw)
    K = kh * kw
    if mshape != (N, Ho, Wo, G, K) or oshape != (N, Ho, Wo, G, K, 2):
        raise ValueError(f"dcnv4: offset/mask shapes {tuple(oshape)}/{tuple(mshape)} do not match "
                         f"N={N} Ho={Ho} Wo={Wo} G={G} K={K}")
    return (N, H, W, G, C // G, kh, kw, sh, sw, ph, pw, dh, dw), (N, Ho, Wo, C)


def dcnv4_forward(x, offset, mask, kernel=3, stride=1, pad=1, dilation=1, offset_scale=1.0, out=None, stream=None,
                  prepare_only=False, _entry="dcnv4_forward"):
    """y [N,Ho,Wo,C] = DCNv4 aggregation of x [N,H,W,C] (Eq. 1-2 of the paper, no softmax).

    With prepare_only the checked argument tuple for load_library().dcnv4_forward is returned
    instead of launching (for launch loops that must not pay the checks every time)."""
    geo, yshape = _shape_args(x, offset, mask, kernel, stride, pad, dilation)
    _check_all(x, (("offset", offset), ("mask", mask)))
    if out is None:
        out = _uninitialised(x, yshape, stream)
    else:
        _check("out", out, x)
        if tuple(out.shape) != yshape:
            raise ValueError("dcnv4: out has the wrong shape")
    args = (x.data_ptr(), offset.data_ptr(), mask.data_ptr(), out.data_ptr(), *geo,
            float(offset_scale), _dtype_code(x), _stream_ptr(stream, x.device))
    if prepare_only:
        return args
    _call(x.device, _entry, args)
    return out


def dcnv4_forward_softmax(x, offset, mask_logits, **kw):
    """dcnv4_forward with m = softmax of mask_logits over the 9 taps (the DCNv3 form)."""
    return dcnv4_forward(x, offset, mask_logits, _entry="dcnv4_forward_softmax", **kw)


def dcnv4_backward_softmax(x, offset, mask_logits, grad_y, **kw):
    """(grad_x, grad_offset, grad_mask_logits) of dcnv4_forward_softmax."""
    return dcnv4_backward(x, offset, mask_logits, grad_y, _entry="dcnv4_backward_softmax", **kw)


def dcnv4_backward(x, offset, mask, grad_y, kernel=3, stride=1, pad=1, dilation=1, offset_scale=1.0,
                   out=None, stream=None, prepare_only=False, _entry="dcnv4_backward"):
    """(grad_x, grad_offset, grad_mask) of dcnv4_forward for upstream gradient grad_y."""
    geo, yshape = _shape_args(x, offset, mask, kernel, stride, pad, dilation)
    _check_all(x, (("offset", offset), ("mask", mask), ("grad_y", grad_y)))
    if grad_y.shape != yshape:
        raise ValueError("dcnv4: grad_y has the wrong shape")
    if out is None:
        gx, go, gm = _empty_like(stream, x, offset, mask)
    else:
        gx, go, gm = out
        for name, t, ref in (("grad_x", gx, x), ("grad_offset", go, offset), ("grad_mask", gm, mask)):
            _check(name, t, x)
            if t.shape != ref.shape:
                raise ValueError(f"dcnv4: {name} has the wrong shape")
    args = (x.data_ptr(), offset.data_ptr(), mask.data_ptr(), grad_y.data_ptr(),
            gx.data_ptr(), go.data_ptr(), gm.data_ptr(), *geo,
            float(offset_scale), _dtype_code(x), _stream_ptr(stream, x.device))
    if prepare_only:
        return args
    _call(x.device, _entry, args)
    return gx, go, gm


def _merged_shape_args(x, om, kernel, stride, pad, dilation):
    (kh, kw), (sh, sw), (ph, pw), (dh, dw) = _pair(kernel), _pair(stride), _pair(pad), _pair(dilation)
    xshape, oshape = x.shape, om.shape
    if len(xshape) != 4 or len(oshape) != 5 or oshape[4] != 32:
        raise ValueError("dcnv4: expected x [N,H,W,C] and offset_mask [N,Ho,Wo,G,32]")
    N, H, W, C = xshape
    G = oshape[3]
    if G < 1 or C % G:
        raise ValueError("dcnv4: C must be a multiple of G")
    Ho, Wo = _conv_hw(H, W, kh, kw, sh, sw, ph, pw, dh, dw)
    if oshape != (N, Ho, Wo, G, 32):
        raise ValueError(f"dcnv4: offset_mask shape {tuple(oshape)} does not match N={N} Ho={Ho} Wo={Wo} G={G}")
    return (N, H, W, G, C // G, kh, kw, sh, sw, ph, pw, dh, dw), (N, Ho, Wo, C)


def dcnv4_forward_merged(x, offset_mask, kernel=3, stride=1, pad=1, dilation=1, offset_scale=1.0, out=None, stream=None,
                         prepare_only=False):
    """dcnv4_forward with the offsets and mask values in one tensor [N,Ho,Wo,G,32]: 18 offsets, 9 mask
    values, 5 unused entries per (pixel, group)."""
    geo, yshape = _merged_shape_args(x, offset_mask, kernel, stride, pad, dilation)
    _check_all(x, (("offset_mask", offset_mask),))
    if out is None:
        out = _uninitialised(x, yshape, stream)
    else:
        _check("out", out, x)
        if tuple(out.shape) != yshape:
            raise ValueError("dcnv4: out has the wrong shape")
    args = (x.data_ptr(), offset_mask.data_ptr(), out.data_ptr(), *geo,
            float(offset_scale), _dtype_code(x), _stream_ptr(stream, x.device))
    if prepare_only:
        return args
    _call(x.device, "dcnv4_forward_merged", args)
    return out


def dcnv4_backward_merged(x, offset_mask, grad_y, kernel=3, stride=1, pad=1, dilation=1, offset_scale=1.0,
                          out=None, stream=None, prepare_only=False):
    """(grad_x, grad_offset_mask) of dcnv4_forward_merged; grad_offset_mask is laid out like offset_mask."""
    geo, yshape = _merged_shape_args(x, offset_mask, kernel, stride, pad, dilation)
    _check_all(x, (("offset_mask", offset_mask), ("grad_y", grad_y)))
    if grad_y.shape != yshape:
        raise ValueError("dcnv4: grad_y has the wrong shape")
    if out is None:
        gx, gom = _empty_like(stream, x, offset_mask)
    else:
        gx, gom = out
        for name, t, ref in (("grad_x", gx, x), ("grad_offset_mask", gom, offset_mask)):
            _check(name, t, x)
            if t.shape != ref.shape:
                raise ValueError(f"dcnv4: {name} has the wrong shape")
    args = (x.data_ptr(), offset_mask.data_ptr(), grad_y.data_ptr(), gx.data_ptr(), gom.data_ptr(), *geo,
            float(offset_scale), _dtype_code(x), _stream_ptr(stream, x.device))
    if prepare_only:
        return args
    _call(x.device, "dcnv4_backward_merged", args)
    return gx, gom


def dcnv4_linear(x, w, b=None, out=None, stream=None, prepare_only=False):
    """y[..., o] = sum_k x[..., k] * w[o, k] + b[o]: a linear layer over the last axis of x (a 1x1
    point-wise convolution of an NHWC map), on the matrix cores."""
    if x.dim() < 2 or w.dim() != 2 or w.shape[1] != x.shape[-1] or (b is not None and tuple(b.shape) != (w.shape[0],)):
        raise ValueError("dcnv4: expected x [..., K], w [Nout, K], b [Nout]")
    for name, t in (("x", x), ("w", w)) + ((("b", b),) if b is not None else ()):
        _check(name, t, x)
    yshape = tuple(x.shape[:-1]) + (w.shape[0],)
    if out is None:
        out = _uninitialised(x, yshape, stream)
    else:
        _check("out", out, x)
        if tuple(out.shape) != yshape:
            raise ValueError("dcnv4: out has the wrong shape")
    P = x.numel() // x.shape[-1]
    args = (x.data_ptr(), w.data_ptr(), b.data_ptr() if b is not None else None, out.data_ptr(), P, x.shape[-1],
            w.shape[0], _dtype_code(x), _stream_ptr(stream, x.device))
    if prepare_only:
        return args
    _call(x.device, "dcnv4_linear", args)
    return out


def dcnv4_depthwise3x3(x, w, b=None, out=None, stream=None):
    """y[n,h,w,c] = b[c] + sum_ij w[i,j,c] * x[n,h+i-1,w+j-1,c] (zero padding): x [N,H,W,C], w [3,3,C]."""
    import torch
    if x.dim() != 4 or tuple(w.shape) != (3, 3, x.shape[3]) or (b is not None and tuple(b.shape) != (x.shape[3],)):
        raise ValueError("dcnv4: expected x [N,H,W,C], w [3,3,C], b [C]")
    for name, t in (("x", x), ("w", w)) + ((("b", b),) if b is not None else ()):
        _check(name, t, x)
    if out is None:
        out = _empty_like(stream, x)[0]
    else:
        _check("out", out, x)
        if out.shape != x.shape:
            raise ValueError("dcnv4: out has the wrong shape")
    N, H, W, C = x.shape
    with torch.cuda.device(x.device):
        rc = load_library().dcnv4_depthwise3x3(x.data_ptr(), w.data_ptr(), b.data_ptr() if b is not None else None,
                                               out.data_ptr(), N, H, W, C, _dtype_code(x), _stream_ptr(stream, x.device))
    if rc:
        raise Dcnv4Error(rc, "dcnv4_depthwise3x3")
    return out


def dcnv4_module_workspace_bytes(N, H, W, G, Cg, dtype, lightweight, depthwise=False):
    return int(load_library().dcnv4_module_workspace_bytes(N, H, W, G, Cg, dtype, int(bool(lightweight)), int(bool(depthwise))))


def dcnv4_module_forward(x, w_om, b_om, G, w_in=None, b_in=None, w_out=None, b_out=None, w_dw=None, b_dw=None, kernel=3,
                         stride=1, pad=1, dilation=1, offset_scale=1.0, workspace=None, out=None, stream=None,
                         prepare_only=False):
    """Forward of the DCNv4 module: (value projection,) ONE linear layer for offsets and modulation
    scalars, the operator, (output projection).  w_om [G*32, C] / b_om [G*32] in the merged layout
    (row g*32 + e: entry e of group g; 0..17 offsets, 18..26 scalars, 27..31 ignored); w_in, w_out
    [C, C] or both None (the lightweight variant); w_dw [3, 3, C] / b_dw [C]: the optional depthwise
    convolution in front of the offset/scalar layer."""
    if x.dim() != 4 or x.shape[3] % G:
        raise ValueError("dcnv4: expected x [N,H,W,C] with C a multiple of G")
    N, H, W, C = x.shape
    (kh, kw), (sh, sw), (ph, pw), (dh, dw) = map(_pair, (kernel, stride, pad, dilation))
    if (w_in is None) != (w_out is None):
        raise ValueError("dcnv4: the input and output projections come together")
    shapes = [("w_om", w_om, (G * 32, C)), ("b_om", b_om, (G * 32,)), ("w_in", w_in, (C, C)), ("b_in", b_in, (C,)),
              ("w_out", w_out, (C, C)), ("b_out", b_out, (C,)), ("w_dw", w_dw, (3, 3, C)), ("b_dw", b_dw, (C,))]
    for name, t, shape in shapes:
        if t is not None:
            _check(name, t, x)
            if tuple(t.shape) != shape:
                raise ValueError(f"dcnv4: {name} must have shape {shape}")
    _check("x", x, x)
    light = w_in is None
    need = dcnv4_module_workspace_bytes(N, H, W, G, C // G, _dtype_code(x), light, w_dw is not None)
    if workspace is None:
        workspace = _workspace(x, None, need, stream)[0]
    elif not workspace.is_cuda or workspace.device != x.device or not workspace.is_contiguous():
        raise ValueError("dcnv4: workspace must be a contiguous tensor on x's device")
    if out is None:
        out = _empty_like(stream, x)[0]
    else:
        _check("out", out, x)
        if out.shape != x.shape:
            raise ValueError("dcnv4: out has the wrong shape")
    ptr = lambda t: t.data_ptr() if t is not None else None
    args = (x.data_ptr(), ptr(w_in), ptr(b_in), ptr(w_dw), ptr(b_dw), w_om.data_ptr(), ptr(b_om), ptr(w_out), ptr(b_out), workspace.data_ptr(),
            workspace.numel() * workspace.element_size(), out.data_ptr(), N, H, W, G, C // G, kh, kw, sh, sw, ph, pw,
            dh, dw, float(offset_scale), _dtype_code(x), _stream_ptr(stream, x.device))
    if prepare_only:
        return args
    _call(x.device, "dcnv4_module_forward", args)
    return out


def dcnv4_module_static_workspace_limit():
    return int(load_library().dcnv4_module_static_workspace_limit())


def dcnv4_module_forward_static(x, w_om, b_om, G, out, w_in=None, b_in=None, w_out=None, b_out=None, w_dw=None, b_dw=None,
                                kernel=3, stride=1, pad=1, dilation=1, offset_scale=1.0, stream=None):
    """dcnv4_module_forward with the workspace in the library's built-in buffer: nothing is allocated, here
    or in the library (the caller passes `out`).  Raises Dcnv4Error (status 6) if the call needs more than
    dcnv4_module_static_workspace_limit() bytes."""
    args = dcnv4_module_forward(x, w_om, b_om, G, w_in=w_in, b_in=b_in, w_out=w_out, b_out=b_out, w_dw=w_dw, b_dw=b_dw,
                                kernel=kernel, stride=stride, pad=pad, dilation=dilation, offset_scale=offset_scale,
                                workspace=x, out=out, stream=stream, prepare_only=True)
    args = args[:9] + args[11:]                      # the same arguments without (workspace, workspace_bytes)
    import torch
    with torch.cuda.device(x.device):
        rc = load_library().dcnv4_module_forward_static(*args)
    if rc:
        raise Dcnv4Error(rc, "dcnv4_module_forward_static")
    return out


# Operators on rows [..., C].  Optional tensors may be None; statistics and losses are float32.  (Small calls are bound by this module:
# a layer norm of 49 x 1024 takes the GPU 3 us.  So checks make nothing that a call without fault does not need.)

def _rows(x):
    shape = x.shape
    if len(shape) < 1 or shape[-1] < 1:
        raise ValueError("dcnv4: expected x [..., C]")
    C = shape[-1]
    return x.numel() // C, C


def _check_like(x, named):
    """_check_all, and the shape of each (name, tensor, shape); tensors that are None are left out."""
    at, dt = x.get_device(), x.dtype
    if at < 0 or not x.is_cuda or not x.is_contiguous():
        _check("x", x, x)
    for name, t, shape in named:
        if t is None:
            continue
        if t.get_device() != at or t.dtype is not dt or not t.is_contiguous():
            _check(name, t, x)
        if t.shape != shape:
            raise ValueError(f"dcnv4: {name} must have shape {tuple(shape)}")


def _check_plain(name, t, at, shape, dtype):
    if t is None or t.get_device() != at or t.dtype is not dtype or not t.is_contiguous() or t.shape != shape:
        raise ValueError(f"dcnv4: {name} must be a contiguous tensor of {dtype} and shape {tuple(shape)} on x's device")


def _new_like(x, stream):
    """_uninitialised(x, x.shape), faster (1.2 us, 1.8 with the shape); of the stream that the call runs on."""
    import torch
    if stream is not None:
        with torch.cuda.stream(stream):
            return _new_like(x, None)
    return torch.empty_like(x) if type(x) is torch.Tensor else _uninitialised(x, x.shape)


def _new(x, shape, dtype):
    import torch
    if type(x) is not torch.Tensor:
        return torch.empty(shape, dtype=dtype, device=x.device)
    if dtype is not x.dtype:
        return x.new_empty(shape, dtype=dtype)
    return torch.empty_like(x) if shape == x.shape else x.new_empty(shape)


def _outputs(x, out, specs, stream):
    """The output tensors: those of `out`, checked, or new ones of the stream that the call runs on.  specs: (name, shape, dtype), None for one that
    is not wanted."""
    if out is None:
        import torch
        if stream is not None:
            with torch.cuda.stream(stream):
                return _outputs(x, None, specs, None)
        made, shape, dtype, last = [], None, None, None
        for s in specs:
            if s is None:
                made.append(None)
                continue
            # (the same shape again is made faster: 0.9 us for 1.5)
            if s[2] is dtype and s[1] == shape:
                last = torch.empty_like(last)
            else:
                last = _new(x, s[1], s[2])
            _, shape, dtype = s
            made.append(last)
        return made
    out = list(out) if isinstance(out, (tuple, list)) else [out]
    if len(out) != len(specs):
        raise ValueError(f"dcnv4: out must hold {len(specs)} tensors")
    for t, s in zip(out, specs):
        if (t is None) != (s is None):
            raise ValueError("dcnv4: out must hold a tensor for every result, and None where there is none")
        if t is not None:
            _check_plain(s[0], t, x.get_device(), s[1], s[2])
    return out


def _workspace(x, workspace, need, stream):
    """(workspace, bytes): the caller's, or a new one.  A new one is of the stream that the call runs on: it is given back when the call
    returns, and only what comes later on that stream may have it."""
    import torch
    if workspace is None:
        need = max(need, 16)
        if stream is None:
            return torch.empty(need, dtype=torch.uint8, device=x.device), need
        with torch.cuda.stream(stream):
            return torch.empty(need, dtype=torch.uint8, device=x.device), need
    if workspace.get_device() != x.get_device() or not workspace.is_contiguous():
        raise ValueError("dcnv4: workspace must be a contiguous tensor on x's device")
    return workspace, workspace.nbytes


def _prepared(args, *held):
    """The arguments alone (prepare_only), whose tensors the caller has to hold."""
    if any(t is None for t in held):
        raise ValueError("dcnv4: prepare_only needs out, and a workspace where there is one")
    return args


_MASK64 = 2 ** 64 - 1


def _offset_ptr(x, offset_on_device):
    import torch
    if offset_on_device is None:
        return None
    if offset_on_device.get_device() != x.get_device() or offset_on_device.dtype is not torch.int64 or offset_on_device.numel() != 1:
        raise ValueError("dcnv4: offset_on_device must be one int64 on x's device")
    return offset_on_device.data_ptr()


def dcnv4_layer_norm_workspace_bytes(P, C):
    return int(load_library().dcnv4_layer_norm_workspace_bytes(P, C))


def dcnv4_layer_norm(x, gamma=None, beta=None, eps=1e-6, stats=False, out=None, stream=None, prepare_only=False):
    """y = (x - mean) * rstd * gamma + beta over the last axis of x [..., C].  With `stats` (y, mean, rstd), mean and
    rstd float32 [...], which dcnv4_layer_norm_backward takes.  `out`: y, or the three."""
    import torch
    P, C = _rows(x)
    _check_like(x, (("gamma", gamma, (C,)), ("beta", beta, (C,))))
    mean = rstd = None
    if stats:
        stat, f32 = x.shape[:-1], torch.float32
        y, mean, rstd = _outputs(x, out, (("y", x.shape, x.dtype), ("mean", stat, f32), ("rstd", stat, f32)), stream)
    else:
        y = _new_like(x, stream) if out is None else _outputs(x, out, (("y", x.shape, x.dtype),), stream)[0]
    args = (x.data_ptr(), None if gamma is None else gamma.data_ptr(), None if beta is None else beta.data_ptr(), y.data_ptr(),
            None if mean is None else mean.data_ptr(), None if rstd is None else rstd.data_ptr(), P, C, float(eps), _dtype_code(x),
            _stream_ptr(stream, x.device))
    if prepare_only:
        return _prepared(args, out)
    _call(x.device, "dcnv4_layer_norm", args)
    return (y, mean, rstd) if stats else y


def dcnv4_layer_norm_backward(x, gamma, mean, rstd, grad_y, workspace=None, out=None, stream=None, prepare_only=False, beta=None):
    """(grad_x, grad_gamma, grad_beta) of dcnv4_layer_norm.  grad_gamma is None where gamma is; grad_beta too, unless beta is given (a norm
    with beta alone)."""
    import torch
    P, C = _rows(x)
    shape, dt, at = x.shape, x.dtype, x.get_device()
    _check_like(x, (("gamma", gamma, (C,)), ("beta", beta, (C,)), ("grad_y", grad_y, shape)))
    _check_plain("mean", mean, at, shape[:-1], torch.float32)
    _check_plain("rstd", rstd, at, shape[:-1], torch.float32)
    if gamma is None and beta is None:
        (gx, gg, gb), size = _outputs(x, out, (("grad_x", shape, dt), None, None), stream), 0
        space = None
    else:
        gx, gg, gb = _outputs(x, out, (("grad_x", shape, dt), None if gamma is None else ("grad_gamma", (C,), dt), ("grad_beta", (C,), dt)), stream)
        space, size = _workspace(x, workspace, dcnv4_layer_norm_workspace_bytes(P, C) if workspace is None else 0, stream)
    ptr = torch.Tensor.data_ptr
    args = (ptr(x), None if gamma is None else ptr(gamma), ptr(mean), ptr(rstd), ptr(grad_y), ptr(gx), None if gg is None else ptr(gg),
            None if gb is None else ptr(gb), None if space is None else ptr(space), size, P, C, _dtype_code(x),
            _stream_ptr(stream, x.device))
    if prepare_only:
        return _prepared(args, out, *(() if space is None else (workspace,)))
    _call(x.device, "dcnv4_layer_norm_backward", args)
    return gx, gg, gb


def dcnv4_dropout(x, p, seed, offset=0, offset_on_device=None, residual=None, out=None, stream=None, prepare_only=False):
    """[residual +] dropout of x: element i is dropped where its bits of the generator (include/dcnv4.h) at (seed, offset) say so,
    else scaled by 1 / (1 - p).  seed and offset: 64 bits, of either sign.  offset_on_device: one int64 on the GPU, added to
    offset as the kernel runs (captured graphs)."""
    shape = x.shape
    _check_like(x, (("residual", residual, shape),))
    y = _new_like(x, stream) if out is None else _outputs(x, out, (("out", shape, x.dtype),), stream)[0]
    args = (x.data_ptr(), None if residual is None else residual.data_ptr(), y.data_ptr(), x.numel(), float(p), int(seed) & _MASK64, int(offset) & _MASK64,
            _offset_ptr(x, offset_on_device), _dtype_code(x), _stream_ptr(stream, x.device))
    if prepare_only:
        return _prepared(args, out)
    _call(x.device, "dcnv4_dropout", args)
    return y


def dcnv4_dropout_backward(grad_y, p, seed, offset=0, offset_on_device=None, out=None, stream=None, prepare_only=False):
    """grad_x of dcnv4_dropout with the same p, seed and offset (that of the residual is grad_y itself)."""
    shape = grad_y.shape
    _check_all(grad_y, ())
    gx = _new_like(grad_y, stream) if out is None else _outputs(grad_y, out, (("out", shape, grad_y.dtype),), stream)[0]
    args = (grad_y.data_ptr(), gx.data_ptr(), grad_y.numel(), float(p), int(seed) & _MASK64, int(offset) & _MASK64, _offset_ptr(grad_y, offset_on_device),
            _dtype_code(grad_y), _stream_ptr(stream, grad_y.device))
    if prepare_only:
        return _prepared(args, out)
    _call(grad_y.device, "dcnv4_dropout_backward", args)
    return gx


def dcnv4_dropout_add_layer_norm(x, residual, gamma, beta, p, seed, offset=0, offset_on_device=None, eps=1e-6, out=None, stream=None,
                                 prepare_only=False):
    """(z, y, mean, rstd): z = residual + dropout(x), y = layer norm of z over the last axis."""
    import torch
    P, C = _rows(x)
    shape, dt, f32 = x.shape, x.dtype, torch.float32
    _check_like(x, (("residual", residual, shape), ("gamma", gamma, (C,)), ("beta", beta, (C,))))
    stat = shape[:-1]
    z, y, mean, rstd = _outputs(x, out, (("z", shape, dt), ("y", shape, dt), ("mean", stat, f32), ("rstd", stat, f32)), stream)
    ptr = torch.Tensor.data_ptr
    args = (ptr(x), ptr(residual), None if gamma is None else ptr(gamma), None if beta is None else ptr(beta), ptr(z), ptr(y), ptr(mean),
            ptr(rstd), P, C, float(p), int(seed) & _MASK64, int(offset) & _MASK64, _offset_ptr(x, offset_on_device), float(eps), _dtype_code(x),
            _stream_ptr(stream, x.device))
    if prepare_only:
        return _prepared(args, out)
    _call(x.device, "dcnv4_dropout_add_layer_norm", args)
    return z, y, mean, rstd


def dcnv4_dropout_add_layer_norm_backward(z, gamma, mean, rstd, grad_y, p, seed, offset=0, offset_on_device=None, grad_z=None,
                                          workspace=None, out=None, stream=None, prepare_only=False, beta=None):
    """(grad_x, grad_residual, grad_gamma, grad_beta) of dcnv4_dropout_add_layer_norm; grad_z: the gradient of z from what else
    reads it.  The last two are None as in dcnv4_layer_norm_backward."""
    import torch
    P, C = _rows(z)
    shape, dt, at = z.shape, z.dtype, z.get_device()
    _check_like(z, (("gamma", gamma, (C,)), ("beta", beta, (C,)), ("grad_y", grad_y, shape), ("grad_z", grad_z, shape)))
    _check_plain("mean", mean, at, shape[:-1], torch.float32)
    _check_plain("rstd", rstd, at, shape[:-1], torch.float32)
    specs = (("grad_x", shape, dt), ("grad_residual", shape, dt))
    if gamma is None and beta is None:
        (gx, gr, gg, gb), size = _outputs(z, out, specs + (None, None), stream), 0
        space = None
    else:
        gx, gr, gg, gb = _outputs(z, out, specs + (None if gamma is None else ("grad_gamma", (C,), dt), ("grad_beta", (C,), dt)), stream)
        space, size = _workspace(z, workspace, dcnv4_layer_norm_workspace_bytes(P, C) if workspace is None else 0, stream)
    ptr = torch.Tensor.data_ptr
    args = (ptr(z), None if gamma is None else ptr(gamma), ptr(mean), ptr(rstd), ptr(grad_y), None if grad_z is None else ptr(grad_z), ptr(gx),
            ptr(gr), None if gg is None else ptr(gg), None if gb is None else ptr(gb), None if space is None else ptr(space), size,
            P, C, float(p), int(seed) & _MASK64, int(offset) & _MASK64, _offset_ptr(z, offset_on_device), _dtype_code(z), _stream_ptr(stream, z.device))
    if prepare_only:
        return _prepared(args, out, *(() if space is None else (workspace,)))
    _call(z.device, "dcnv4_dropout_add_layer_norm_backward", args)
    return gx, gr, gg, gb


def dcnv4_linear_cross_entropy_workspace_bytes(P, K, V, dtype, backward):
    return int(load_library().dcnv4_linear_cross_entropy_workspace_bytes(P, K, V, dtype, int(bool(backward))))


def _loss_args(x, w, target, b, workspace, backward, stream):
    import torch
    P, K = _rows(x)
    if w.dim() != 2 or w.shape[1] != K:
        raise ValueError("dcnv4: expected x [..., K], w [V, K]")
    V = w.shape[0]
    _check_like(x, (("w", w, w.shape), ("b", b, (V,))))
    _check_plain("target", target, x.get_device(), x.shape[:-1], torch.int64)
    need = dcnv4_linear_cross_entropy_workspace_bytes(P, K, V, _dtype_code(x), backward) if workspace is None else 0
    return P, K, V, *_workspace(x, workspace, need, stream)


def dcnv4_linear_cross_entropy(x, w, target, b=None, ignore_index=-100, workspace=None, out=None, stream=None, prepare_only=False):
    """(loss, lse), float32 [...]: loss = lse - logit[target] with logits x w^T + b that are never stored.  x [..., K], w [V, K],
    target [...] int64; rows whose target is ignore_index have loss 0."""
    import torch
    P, K, V, space, size = _loss_args(x, w, target, b, workspace, False, stream)
    stat, f32 = x.shape[:-1], torch.float32
    loss, lse = _outputs(x, out, (("loss", stat, f32), ("lse", stat, f32)), stream)
    ptr = torch.Tensor.data_ptr
    args = (ptr(x), ptr(w), None if b is None else ptr(b), ptr(target), ptr(loss), ptr(lse), ptr(space), size, P, K, V, int(ignore_index),
            _dtype_code(x), _stream_ptr(stream, x.device))
    if prepare_only:
        return _prepared(args, out, workspace)
    _call(x.device, "dcnv4_linear_cross_entropy", args)
    return loss, lse


def dcnv4_linear_cross_entropy_backward(x, w, target, lse, grad_loss, b=None, ignore_index=-100, workspace=None, out=None, stream=None,
                                        prepare_only=False):
    """(grad_x, grad_w, grad_b) of dcnv4_linear_cross_entropy for grad_loss [...] float32, from its lse; grad_b is None where b is."""
    import torch
    P, K, V, space, size = _loss_args(x, w, target, b, workspace, True, stream)
    shape, dt, at = x.shape, x.dtype, x.get_device()
    _check_plain("lse", lse, at, shape[:-1], torch.float32)
    _check_plain("grad_loss", grad_loss, at, shape[:-1], torch.float32)
    gx, gw, gb = _outputs(x, out, (("grad_x", shape, dt), ("grad_w", w.shape, dt), None if b is None else ("grad_b", (V,), dt)), stream)
    ptr = torch.Tensor.data_ptr
    args = (ptr(x), ptr(w), None if b is None else ptr(b), ptr(target), ptr(lse), ptr(grad_loss), ptr(gx), ptr(gw), None if gb is None else ptr(gb),
            ptr(space), size, P, K, V, int(ignore_index), _dtype_code(x), _stream_ptr(stream, x.device))
    if prepare_only:
        return _prepared(args, out, workspace)
    _call(x.device, "dcnv4_linear_cross_entropy_backward", args)
    return gx, gw, gb


FIRST_NORM, SECOND_NORM = 1, 2


def dcnv4_norm_scale_add_norm_workspace_bytes(P, C, gates):
    return int(load_library().dcnv4_norm_scale_add_norm_workspace_bytes(P, C, gates))


def _end_args(x, scale, gate, first, second, rows):
    """(P, C, gates, norms, gamma1, beta1, gamma2, beta2) of a block's end, checked; rows: (name, tensor of x's shape or None)."""
    shape = x.shape
    P, C = _rows(x)
    norms, gamma1, beta1, gamma2, beta2, gates = 0, None, None, None, None, 0
    if first is not None:
        norms, (gamma1, beta1) = FIRST_NORM, first
    if second is not None:
        norms, (gamma2, beta2) = norms | SECOND_NORM, second
    vector = (C,)
    _check_like(x, (("scale", scale, vector), ("gamma1", gamma1, vector), ("beta1", beta1, vector), ("gamma2", gamma2, vector), ("beta2", beta2, vector),
                    *[(name, t, shape) for name, t in rows]))
    if gate is not None:
        import torch
        if len(shape) < 2:
            raise ValueError("dcnv4: expected x [N, ..., C] with gate [N]")
        gates = shape[0]
        _check_plain("gate", gate, x.get_device(), (gates,), torch.float32)
    return P, C, gates, norms, gamma1, beta1, gamma2, beta2


def _ptr(t):
    return None if t is None else t.data_ptr()


def dcnv4_norm_scale_add_norm(x, residual, scale=None, gate=None, first=None, second=None, eps=1e-6, stats=True, out=None, stream=None,
                              prepare_only=False):
    """(z, y, mean1, rstd1, mean2, rstd2): z = residual + gate * scale * first(x), y = second(z), x [N, ..., C].  first, second: None (no such norm) or a
    layer norm's (gamma, beta), each of which may be None.  scale [C]; gate [N] float32, one for each image.  y and the statistics of
    norms that there are not are None; without `stats` all of these (and not in `out` either)."""
    import torch
    P, C, gates, norms, gamma1, beta1, gamma2, beta2 = _end_args(x, scale, gate, first, second, (("residual", residual),))
    shape, dt, f32 = x.shape, x.dtype, torch.float32
    stat = shape[:-1] if stats else None
    one, two = stats and first is not None, stats and second is not None
    z, y, mean1, rstd1, mean2, rstd2 = results = _outputs(x, out, (
        ("z", shape, dt), None if second is None else ("y", shape, dt), ("mean1", stat, f32) if one else None, ("rstd1", stat, f32) if one else None,
        ("mean2", stat, f32) if two else None, ("rstd2", stat, f32) if two else None), stream)
    args = (*[None if t is None else t.data_ptr() for t in (x, residual, gamma1, beta1, scale, gate, gamma2, beta2, z, y, mean1, rstd1, mean2, rstd2)],
            P, C, gates, norms, float(eps), _dtype_code(x), _stream_ptr(stream, x.device))
    if prepare_only:
        return _prepared(args, out)
    _call(x.device, "dcnv4_norm_scale_add_norm", args)
    return tuple(results)


def dcnv4_norm_scale_add_norm_backward(x, z, scale, gate, first, second, stats, grad_y, grad_z=None, grad_gate=True, workspace=None, out=None,
                                       stream=None, prepare_only=False):
    """(grad_x, grad_residual, grad_scale, grad_gate, grad_gamma1, grad_beta1, grad_gamma2, grad_beta2) of dcnv4_norm_scale_add_norm, from its z and
    stats = (mean1, rstd1, mean2, rstd2), None where there is no such norm.  grad_y is None without a second norm, where grad_residual is grad_z itself (in `out`: None).
    Gradients of what is None are None; so is the gates' with grad_gate=False."""
    import torch
    if second is None:
        if grad_y is not None or grad_z is None:
            raise ValueError("dcnv4: without a second norm there is grad_z, and no grad_y")
        z = None
    elif grad_y is None or z is None:
        raise ValueError("dcnv4: a second norm's backward pass takes z and grad_y")
    P, C, gates, norms, gamma1, beta1, gamma2, beta2 = _end_args(x, scale, gate, first, second, (("z", z), ("grad_y", grad_y), ("grad_z", grad_z)))
    shape, dt, at, f32, vector = x.shape, x.dtype, x.get_device(), torch.float32, (C,)
    if stats is None or len(stats) != 4:
        raise ValueError("dcnv4: stats must be (mean1, rstd1, mean2, rstd2)")
    mean1, rstd1, mean2, rstd2 = stats
    if second is not None:
        _check_plain("mean2", mean2, at, shape[:-1], f32)
        _check_plain("rstd2", rstd2, at, shape[:-1], f32)
    if first is not None:
        _check_plain("mean1", mean1, at, shape[:-1], f32)
        _check_plain("rstd1", rstd1, at, shape[:-1], f32)
    of = lambda name, t: None if t is None else (name, vector, dt)
    specs = (("grad_x", shape, dt), None if second is None else ("grad_residual", shape, dt), of("grad_scale", scale),
             ("grad_gate", (gates,), f32) if gate is not None and grad_gate else None, of("grad_gamma1", gamma1), of("grad_beta1", beta1),
             of("grad_gamma2", gamma2), of("grad_beta2", beta2))
    results = _outputs(x, out, specs, stream)
    space, size = None, 0
    if any(s is not None for s in specs[2:]):
        space, size = _workspace(x, workspace, dcnv4_norm_scale_add_norm_workspace_bytes(P, C, gates) if workspace is None else 0, stream)
    args = (*[None if t is None else t.data_ptr() for t in (x, z, gamma1, beta1, scale, gate, gamma2, mean1, rstd1, mean2, rstd2, grad_y, grad_z,
                                                            *results, space)], size, P, C, gates, norms, _dtype_code(x), _stream_ptr(stream, x.device))
    if prepare_only:
        return _prepared(args, out, *(() if space is None else (workspace,)))
    _call(x.device, "dcnv4_norm_scale_add_norm_backward", args)
    return (results[0], grad_z if second is None else results[1], *results[2:])


def dcnv4_linear_backward_workspace_bytes(P, K, Nout, dtype):
    return int(load_library().dcnv4_linear_backward_workspace_bytes(P, K, Nout, dtype))


def dcnv4_linear_backward(x, w, grad_y, b=None, need_x=True, workspace=None, out=None, stream=None, prepare_only=False, need_w=True):
    """(grad_x, grad_w, grad_b) of dcnv4_linear for grad_y [..., Nout]; grad_b is None where b is, grad_x with need_x=False (a first layer), grad_w with
    need_w=False (a layer that is not trained).  Sizes as in include/dcnv4.h, which are more than dcnv4_linear takes."""
    P, K = _rows(x)
    if w.dim() != 2 or w.shape[1] != K:
        raise ValueError("dcnv4: expected x [..., K], w [Nout, K]")
    N, shape, dt = w.shape[0], x.shape, x.dtype
    _check_like(x, (("w", w, w.shape), ("b", b, (N,)), ("grad_y", grad_y, (*shape[:-1], N))))
    gx, gw, gb = _outputs(x, out, (("grad_x", shape, dt) if need_x else None, ("grad_w", w.shape, dt) if need_w else None,
                                   None if b is None else ("grad_b", (N,), dt)), stream)
    space, size = _workspace(x, workspace, dcnv4_linear_backward_workspace_bytes(P, K, N, _dtype_code(x)) if workspace is None else 0, stream)
    args = (x.data_ptr(), w.data_ptr(), grad_y.data_ptr(), _ptr(gx), _ptr(gw), _ptr(gb), space.data_ptr(), size, P, K, N, _dtype_code(x),
            _stream_ptr(stream, x.device))
    if prepare_only:
        return _prepared(args, out, workspace)
    _call(x.device, "dcnv4_linear_backward", args)
    return gx, gw, gb


ACTIVATIONS = {"silu": 0, "gelu": 1}


def dcnv4_gated_linear_workspace_bytes(P, K, F, dtype, backward):
    return int(load_library().dcnv4_gated_linear_workspace_bytes(P, K, F, dtype, int(bool(backward))))


def _gated_args(x, w, b, activation):
    P, K = _rows(x)
    if w.dim() != 3 or w.shape[0] != 2 or w.shape[2] != K:
        raise ValueError("dcnv4: expected x [..., K], w [2, F, K]")
    if activation not in ACTIVATIONS:
        raise ValueError(f"dcnv4: activation must be one of {', '.join(ACTIVATIONS)}")
    F = w.shape[1]
    _check_like(x, (("w", w, w.shape), ("b", b, (2, F))))
    return P, K, F, ACTIVATIONS[activation]


def dcnv4_gated_linear(x, w, b=None, activation="silu", workspace=None, out=None, stream=None, prepare_only=False):
    """h = act(x w[0]^T + b[0]) * (x w[1]^T + b[1]): x [..., K], w [2, F, K], b [2, F], h [..., F]; activation "silu" or "gelu" (with erf)."""
    P, K, F, act = _gated_args(x, w, b, activation)
    h, = _outputs(x, out, (("h", (*x.shape[:-1], F), x.dtype),), stream)
    code = _dtype_code(x)
    space, size = None, 0
    if code == DCNV4_F32 or workspace is not None:
        space, size = _workspace(x, workspace, dcnv4_gated_linear_workspace_bytes(P, K, F, code, False) if workspace is None else 0, stream)
    args = (x.data_ptr(), w.data_ptr(), _ptr(b), h.data_ptr(), _ptr(space), size, P, K, F, act, code, _stream_ptr(stream, x.device))
    if prepare_only:
        return _prepared(args, out, *(() if code == DCNV4_F16 else (workspace,)))
    _call(x.device, "dcnv4_gated_linear", args)
    return h


def dcnv4_gated_linear_backward(x, w, grad_h, b=None, activation="silu", need_x=True, workspace=None, out=None, stream=None, prepare_only=False, need_w=True,
                                need_b=True):
    """(grad_x, grad_w, grad_b) of dcnv4_gated_linear for grad_h [..., F]; grad_b is None where b is, grad_x with need_x=False (a first layer), grad_w and
    grad_b with need_w=False and need_b=False (a layer that is not trained)."""
    P, K, F, act = _gated_args(x, w, b, activation)
    shape, dt = x.shape, x.dtype
    _check_like(x, (("grad_h", grad_h, (*shape[:-1], F)),))
    gx, gw, gb = _outputs(x, out, (("grad_x", shape, dt) if need_x else None, ("grad_w", w.shape, dt) if need_w else None,
                                   ("grad_b", (2, F), dt) if need_b and b is not None else None), stream)
    code = _dtype_code(x)
    space, size = _workspace(x, workspace, dcnv4_gated_linear_workspace_bytes(P, K, F, code, True) if workspace is None else 0, stream)
    args = (x.data_ptr(), w.data_ptr(), _ptr(b), grad_h.data_ptr(), _ptr(gx), _ptr(gw), _ptr(gb), space.data_ptr(), size, P, K, F, act, code,
            _stream_ptr(stream, x.device))
    if prepare_only:
        return _prepared(args, out, workspace)
    _call(x.device, "dcnv4_gated_linear_backward", args)
    return gx, gw, gb


class AdamwPlan:
    """The tensors of a dcnv4_adamw_step, checked and listed once (dcnv4_adamw_plan makes it).  It holds their memory and works there at each
    step: a tensor that is given other memory needs a new plan.  Gradients among them: where autograd makes them anew (torch's zero_grad() drops them unless
    it is called with set_to_none=False), an old plan's step reads the old ones."""

    def __init__(self, records, held, device, state_bits, dtype):
        self.records, self.held, self.device, self.state_bits, self.dtype = records, held, device, state_bits, dtype

    def __len__(self):
        return len(self.records)

    def set(self, lr=None, weight_decay=None):
        """Other learning rates or weight decays from the next step on: a number, or one for each tensor."""
        # (both are looked at before the first is set)
        new = [(name, _each(values, len(self), name)) for name, values in (("lr", lr), ("weight_decay", weight_decay)) if values is not None]
        for name, values in new:
            for record, value in zip(self.records, values):
                setattr(record, name, value)


def _each(values, count, name):
    values = [float(v) for v in values] if isinstance(values, (list, tuple)) else [float(values)] * count
    if len(values) != count:
        raise ValueError(f"dcnv4: {name} must be a number, or one for each of {count} tensors")
    return values


def dcnv4_adamw_plan(params, grads, exp_avgs, exp_avg_sqs, lr, weight_decay=0.0, scales=None, copies=None):
    """What dcnv4_adamw_step takes: lists of as many tensors each, of any shapes.  params float32; grads all float32 or all float16; exp_avgs and
    exp_avg_sqs all float32, or, for states of 8 bits, all torch.float8_e4m3fn (m, and the root of v), with `scales`: float32 [(n + 255) // 256, 2]
    for a tensor of n elements (m is exp_avg * scales[:, 0], the root of v exp_avg_sq * scales[:, 1], a scale for each 256 elements; zeros to
    start with).  copies (with float16 gradients): float16 tensors, or None in the place of one, that get the parameters after each step.  lr,
    weight_decay: a number, or one for each tensor."""
    import torch
    params, grads, ms, vs = list(params), list(grads), list(exp_avgs), list(exp_avg_sqs)
    count = len(params)
    lists = [("grads", grads), ("exp_avgs", ms), ("exp_avg_sqs", vs)]
    scales = [None] * count if scales is None else list(scales)
    copies = [None] * count if copies is None else list(copies)
    lists += [("scales", scales), ("copies", copies)]
    if count < 1 or any(len(l) != count for _, l in lists):
        raise ValueError("dcnv4: expected lists of as many tensors each, one at least")
    if not params[0].is_cuda:
        raise ValueError("dcnv4: params must be GPU tensors")
    at, device, state = params[0].get_device(), params[0].device, ms[0].dtype
    if state is not torch.float32 and state is not torch.float8_e4m3fn:
        raise TypeError(f"dcnv4: unsupported state dtype {state}")
    eight, dtype = state is torch.float8_e4m3fn, _dtype_code(grads[0])
    written, read = [], []
    for i, (p, g, m, v, s, c) in enumerate(zip(params, grads, ms, vs, scales, copies)):
        n, shape = p.numel(), p.shape
        _check_plain(f"params[{i}]", p, at, shape, torch.float32)
        _check_plain(f"grads[{i}]", g, at, shape, grads[0].dtype)
        _check_plain(f"exp_avgs[{i}]", m, at, shape, state)
        _check_plain(f"exp_avg_sqs[{i}]", v, at, shape, state)
        if eight != (s is not None):
            raise ValueError("dcnv4: states of 8 bits come with scales, and no others")
        if eight:
            _check_plain(f"scales[{i}]", s, at, ((n + 255) // 256, 2), torch.float32)
        if c is not None:
            if dtype != DCNV4_F16:
                raise ValueError("dcnv4: copies come with float16 gradients")
            _check_plain(f"copies[{i}]", c, at, shape, torch.float16)
        written += [(t.data_ptr(), t.data_ptr() + t.nbytes, True) for t in (p, m, v, s, c) if t is not None]
        read.append((g.data_ptr(), g.data_ptr() + g.nbytes, False))
    # what is written overlaps nothing else (gradients may)
    end, last = 0, False
    for first, after, out in sorted(written + read):
        if first < end and (out or last):
            raise ValueError("dcnv4: parameters, states and copies must not share memory")
        if after > end:
            end, last = after, out
    records = (AdamwTensor * count)()
    ptr = lambda t: None if t is None else t.data_ptr()
    for r, p, g, m, v, s, c in zip(records, params, grads, ms, vs, scales, copies):
        r.n, r.param, r.grad, r.m, r.v, r.scales, r.copy = p.numel(), ptr(p), ptr(g), ptr(m), ptr(v), ptr(s), ptr(c)
    # (the memory that is listed, whatever the caller's tensors are made to hold later)
    held = tuple([None if t is None else t.detach() for t in l] for l in (params, grads, ms, vs, scales, copies))
    plan = AdamwPlan(records, held, device, 8 if eight else 32, dtype)
    plan.set(lr=lr, weight_decay=weight_decay)
    return plan


def dcnv4_adamw_step(plan, step, betas=(0.9, 0.999), eps=1e-8, seed=0, step_on_device=None, factors_on_device=None, stream=None):
    """A step of AdamW (include/dcnv4.h) over the plan's tensors, in place.  step: the number of this step, from 1 on; step_on_device: one int64 on
    the GPU that is added to it (captured graphs).  factors_on_device: two float32 on the GPU, which gradients and learning rates are multiplied
    with; a first one that is not finite leaves everything as it is.  seed: of the rounding of states of 8 bits."""
    import torch
    factors = None
    if factors_on_device is not None:
        _check_plain("factors_on_device", factors_on_device, plan.device.index, (2,), torch.float32)
        factors = factors_on_device.data_ptr()
    args = (plan.records, len(plan), float(betas[0]), float(betas[1]), float(eps), int(step), _offset_ptr(plan.held[0][0], step_on_device), factors,
            int(seed) & _MASK64, plan.state_bits, plan.dtype, _stream_ptr(stream, plan.device))
    _call(plan.device, "dcnv4_adamw", args)
