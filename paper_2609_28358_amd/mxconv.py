"""ctypes binding of libmxconv.so (include/mxconv.h).

Argument marshalling only: output tensors are allocated with torch on the
caller's device, pointers and the current HIP stream are passed through, and
every step runs in the library's HIP kernels.  A missing library raises; there
is no fallback path.
"""
import ctypes
import functools
import os
from array import array
from operator import attrgetter, itemgetter

import torch

E4M3, E2M1, E2M3, E3M2 = 0, 1, 2, 3
F32, BF16 = 0, 1
NCHW, NHWC, CBF, CBF_BF16 = 0, 1, 2, 3
ACT, WEIGHT = 0, 1
FN_NONE, FN_RELU, FN_SILU = 0, 1, 2
FN_PRE_OUT = 0x100      # or-ed into fwd_quant's fn: act_out receives the pre-activation
FN_BF16 = 0x200         # or-ed into fwd_quant / dgrad_quant / quantize_sum's fn: bf16 full-precision tensors
KEEP_PAD = 0x100        # or-ed into quantize's layout: padding channels' codes already +0, not written

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmxconv.so")
_lib = None


class MxconvError(RuntimeError):
    pass


QMULTI_MAX = 24
FP6_SLACK = 16          # bytes of read slack at the end of an FP6 code buffer


class MxcConv(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in
                ("n", "cin", "cout", "h", "w", "kh", "kw", "sh", "sw", "ph", "pw")]


class MxcWJob(ctypes.Structure):
    _fields_ = [("conv", ctypes.POINTER(MxcConv)), ("fmt", ctypes.c_int32), ("workspace", ctypes.c_void_p),
                ("ws_bytes", ctypes.c_size_t), ("gw", ctypes.c_void_p)]


WREDUCE_MAX = 32
CONCAT_MAX = 4
TERMS_MAX = 4


class MxcLinear(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("rows", "outs", "ins")]


class MxcNorm(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("gates", ctypes.c_int64), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("scale", ctypes.c_float), ("eps", ctypes.c_float), ("w_post", ctypes.c_void_p),
                ("gate", ctypes.c_void_p), ("w_pre", ctypes.c_void_p)]


class MxcPart(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("ncb", ctypes.c_int32),
                ("up", ctypes.c_int32)]


class MxcTerm(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("c_src", ctypes.c_int32), ("c_off", ctypes.c_int32),
                ("down", ctypes.c_int32)]


class MxcQJob(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p)] + [(k, ctypes.c_int32) for k in
                                           ("dtype", "layout", "role", "fmt", "n", "c", "h", "w")] + \
               [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("conv", ctypes.POINTER(MxcConv)), ("col_codes", ctypes.c_void_p), ("col_scales", ctypes.c_void_p)]


def lib():
    """Load the in-tree library (built by paper_2609_28358_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise MxconvError(f"{LIB_PATH} is missing: build it with "
                          "`python -m paper_2609_28358_amd.build` (no CPU fallback exists)")
    L = ctypes.CDLL(LIB_PATH)
    P, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    CP, LP, NP = (ctypes.POINTER(t) for t in (MxcConv, MxcLinear, MxcNorm))
    sigs = {
        "mxconv_codes_bytes": (sz, [i32] * 6),
        "mxconv_scales_bytes": (sz, [i32] * 6),
        "mxconv_out_size": (i32, [CP, ctypes.POINTER(i32), ctypes.POINTER(i32)]),
        "mxconv_im2col_codes_bytes": (sz, [CP, i32]),
        "mxconv_im2col_scales_bytes": (sz, [CP, i32]),
        "mxconv_wgrad_workspace_bytes": (sz, [CP, i32]),
        "mxconv_quantize": (i32, [P, i32, i32, i32, i32, i32, i32, i32, i32, P, P, P]),
        "mxconv_quantize_multi": (i32, [i32, ctypes.POINTER(MxcQJob), P]),
        "mxconv_quantize_sr": (i32, [P, i32, i32, i32, i32, i32, i32, i32, i32, ctypes.c_uint64, P, P, P]),
        "mxconv_nvfp_scales_bytes": (sz, [i32] * 6),
        "mxconv_nvfp_workspace_bytes": (sz, []),
        "mxconv_nvfp_quantize": (i32, [P, i32, i32, i32, i32, i32, i32, i32, i32, P, P, P, P, sz, P]),
        "mxconv_nvfp_fwd": (i32, [CP, i32, P, P, P, P, P, P, P, i32, P]),
        "mxconv_nvfp_dgrad": (i32, [CP, i32, P, P, P, P, P, P, P, i32, P]),
        "mxconv_nvfp_wgrad_workspace_bytes": (sz, [CP, i32]),
        "mxconv_nvfp_wgrad": (i32, [CP, i32, P, P, P, P, P, P, P, P, sz, P]),
        "mxconv_im2col_cbf": (i32, [CP, i32, P, P, P, P, P]),
        "mxconv_fwd": (i32, [CP, i32, P, P, P, P, P, i32, P]),
        "mxconv_dgrad": (i32, [CP, i32, P, P, P, P, P, i32, P]),
        "mxconv_wgrad": (i32, [CP, i32, P, P, P, P, P, P, sz, P]),
        "mxconv_wgrad_deferred": (i32, [CP, i32, P, P, P, P, P, P, sz, P]),
        "mxconv_backward": (i32, [CP, i32, P, P, P, P, P, P, P, i32, P, P, sz, i32, P]),
        "mxconv_wgrad_reduce_multi": (i32, [i32, ctypes.POINTER(MxcWJob), P]),
        "mxconv_fwd_quant": (i32, [CP, i32, P, P, P, P, i32, i32, P, P, P, P]),
        "mxconv_dgrad_quant": (i32, [CP, i32, P, P, P, P, i32, P, i32, P, P, P, P]),
        "mxconv_dgrad_quant_sr": (i32, [CP, i32, P, P, P, P, i32, P, i32, P, P, P, ctypes.c_uint64, P]),
        "mxconv_naive_codes_bytes": (sz, [i64, i64, i32]),
        "mxconv_naive_scales_bytes": (sz, [i64, i64]),
        "mxconv_naive_im2col_f32": (i32, [CP, P, P, P]),
        "mxconv_naive_quantize_1d": (i32, [P, i64, i64, i32, i32, P, P, P]),
        "mxconv_naive_fwd": (i32, [CP, i32, P, P, P, P, P, P]),
        "mxconv_naive_dgrad": (i32, [CP, i32, P, P, P, P, P, P, P]),
        "mxconv_naive_wgrad": (i32, [CP, i32, P, P, P, P, P, P]),
        "mxconv_wgrad_noalloc": (i32, [CP, i32, P, P, P, P, P, P]),
        "mxconv_concat_cbf": (i32, [i32, i32, i32, i32, i32, ctypes.POINTER(MxcPart), P, P, P]),
        "mxconv_quantize_sum": (i32, [i32, i32, i32, i32, i32, i32, ctypes.POINTER(MxcTerm), i32, P, P, P, P, P]),
        "mxconv_quantize_sum_sr": (i32, [i32, i32, i32, i32, i32, i32, ctypes.POINTER(MxcTerm), i32, P, P, P, P,
                                         ctypes.c_uint64, P]),
        "mxconv_linear_workspace_bytes": (sz, [i32, LP]),
        "mxconv_linear_fwd": (i32, [LP, i32, P, P, P, P, P, i32, P, i64, P, i64, P, i64, i32, P, sz, P]),
        "mxconv_linear_dgrad": (i32, [LP, i32, P, P, P, P, i32, P, i64, P, i64, P, i64, i32, P, sz, P]),
        "mxconv_linear_wgrad": (i32, [LP, i32, P, P, P, P, P, P, P, sz, P]),
        "mxconv_norm_fwd": (i32, [NP, P, i64, P, i64, P, i64, P, i64, P]),
        "mxconv_norm_workspace_bytes": (sz, [NP]),
        "mxconv_norm_bwd": (i32, [NP, P, i64, P, i64, P, i64, P, i64, P, i64, P, i64, P, P, P, P, sz, P]),
        "mxconv_grad_clip_workspace_bytes": (sz, []),
        "mxconv_grad_clip": (i32, [i32, P, ctypes.c_double, P, P, sz, P]),
        "mxconv_strerror": (ctypes.c_char_p, [i32]),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def pair(first, second):
    """The `fmt` argument of a GEMM entry point whose two MX operands have
    these formats (first, second in the call's argument order)."""
    return first if first == second else 0x10 | (first << 2) | second


def strerror(rc):
    return lib().mxconv_strerror(rc).decode()


def _check(rc, what):
    if rc != 0:
        raise MxconvError(f"{what}: {strerror(rc)} (code {rc})")


# Host cost of a call.  Most calls on small layers take less time on the GPU
# than on the host, so what a call needs from a layer or a shape alone (its
# struct, sizes) is computed once per distinct description, in bounded caches,
# and pointers and the stream are passed as plain integers.  Measured per call
# (32 -> 32 channels at 8x8, batch 32): quantize into a given output 8.1 -> 5.0
# us, fwd 12.0 -> 8.0, backward 14.1 -> 10.4, fwd_quant 14.2 -> 9.2.
_CACHED = 4096
_conv_fields = itemgetter("n", "cin", "cout", "h", "w", "kh", "kw", "sh", "sw", "ph", "pw")


def _conv_key(cv):
    return tuple(map(int, _conv_fields(cv)))


def _ptr(t):
    return t.data_ptr() if t is not None else None


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _raw_device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


def conv_struct(cv):
    return MxcConv(*_conv_key(cv))


@functools.lru_cache(maxsize=_CACHED, typed=True)
def _conv_of(key):
    """The layer's struct, shared by its calls (the library only reads it)."""
    return MxcConv(*key)


def _conv(cv):
    return ctypes.byref(_conv_of(_conv_key(cv)))


@functools.lru_cache(maxsize=_CACHED, typed=True)
def codes_bytes(role, fmt, n, c, h, w):
    return lib().mxconv_codes_bytes(role, fmt, n, c, h, w)


@functools.lru_cache(maxsize=_CACHED, typed=True)
def scales_bytes(role, fmt, n, c, h, w):
    return lib().mxconv_scales_bytes(role, fmt, n, c, h, w)


@functools.lru_cache(maxsize=_CACHED, typed=True)
def _out_size(key):
    ho, wo = ctypes.c_int(), ctypes.c_int()
    _check(lib().mxconv_out_size(ctypes.byref(_conv_of(key)), ctypes.byref(ho), ctypes.byref(wo)), "out_size")
    return ho.value, wo.value


def out_size(cv):
    return _out_size(_conv_key(cv))


@functools.lru_cache(maxsize=_CACHED, typed=True)
def _wgrad_workspace_bytes(key, fmt):
    return lib().mxconv_wgrad_workspace_bytes(ctypes.byref(_conv_of(key)), fmt)


def wgrad_workspace_bytes(cv, fmt):
    return _wgrad_workspace_bytes(_conv_key(cv), fmt)


@functools.lru_cache(maxsize=_CACHED, typed=True)
def _nvfp_wgrad_workspace_bytes(key, fmt):
    return lib().mxconv_nvfp_wgrad_workspace_bytes(ctypes.byref(_conv_of(key)), fmt)


def nvfp_wgrad_workspace_bytes(cv, fmt):
    return _nvfp_wgrad_workspace_bytes(_conv_key(cv), fmt)


class MxTensor:
    """Codes and E8M0 scales of one quantized tensor (device uint8 tensors)."""

    def __init__(self, codes, scales, role, fmt, shape):
        self.codes, self.scales, self.role, self.fmt, self.shape = codes, scales, role, fmt, tuple(shape)

    @staticmethod
    def empty(role, fmt, shape, device):
        n, c, h, w = shape
        nb = codes_bytes(role, fmt, n, c, h, w)
        ns = scales_bytes(role, fmt, n, c, h, w)
        if nb == 0:
            raise MxconvError(f"invalid MX tensor geometry {shape} role {role} fmt {fmt}")
        codes = torch.empty(nb, dtype=torch.uint8, device=device)
        if fmt in (E2M3, E3M2):
            codes[-FP6_SLACK:].zero_()     # read slack, never written by the library: keep it defined
        return MxTensor(codes, torch.empty(ns, dtype=torch.uint8, device=device), role, fmt, shape)


_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


def _quant_args(src, layout, shape):
    if shape is None:
        if layout == NHWC:
            n, h, w, c = src.shape
            shape = (n, c, h, w)
        elif layout == NCHW:
            shape = tuple(src.shape)
        else:
            raise ValueError("shape is required for the CBF layout")
    dtype = _DTYPES.get(src.dtype)
    if dtype is None:
        raise MxconvError(f"unsupported dtype {src.dtype}")
    if not src.is_contiguous():
        raise MxconvError("src must be contiguous")
    return dtype, tuple(map(int, shape))


def quantize(src, role, fmt, layout=NCHW, shape=None, out=None, stream=None, keep_pad=False):
    """Quantize `src` (fp32 or bf16 device tensor) once.  `shape` is the
    logical (n, c, h, w); it defaults to src.shape for NCHW.  keep_pad: the
    codes of `out`'s padding channels already hold +0 codes (MXC_KEEP_PAD)."""
    dtype, shape = _quant_args(src, layout, shape)
    if out is None:
        if keep_pad:
            raise MxconvError("keep_pad needs an output whose padding codes are +0")
        out = MxTensor.empty(role, fmt, shape, src.device)
    _check(lib().mxconv_quantize(_ptr(src), dtype, layout | (KEEP_PAD if keep_pad else 0), role, fmt, *shape,
                                 _ptr(out.codes), _ptr(out.scales), _stream(stream)), "mxconv_quantize")
    return out


def quantize_multi(items, stream=None):
    """Several quantize() calls in one library call (one launch for the CBF
    batch-block-32 activations and OIHW weights among them).  items: tuples
    (src, role, fmt, layout, shape, out[, col]); col = (cv, col_codes,
    col_scales) also writes the activation's CBF im2col for layer cv into the
    two uint8 device tensors (sizes: mxconv_im2col_{codes,scales}_bytes).
    Returns the MX tensors."""
    if len(items) > QMULTI_MAX:
        raise MxconvError(f"at most {QMULTI_MAX} tensors per call")
    jobs = (MxcQJob * max(1, len(items)))()
    outs = []
    for k, item in enumerate(items):
        src, role, fmt, layout, shape, out = item[:6]
        col = item[6] if len(item) > 6 else None
        dtype, shape = _quant_args(src, layout, shape)
        if out is None:
            out = MxTensor.empty(role, fmt, shape, src.device)
        jobs[k] = MxcQJob(src.data_ptr(), dtype, layout, role, fmt, *shape, out.codes.data_ptr(),
                          out.scales.data_ptr())
        if col is not None:
            cv, cc, cs = col
            jobs[k].conv = ctypes.pointer(_conv_of(_conv_key(cv)))
            jobs[k].col_codes = cc.data_ptr()
            jobs[k].col_scales = cs.data_ptr()
        outs.append(out)
    _check(lib().mxconv_quantize_multi(len(items), jobs, _stream(stream)), "mxconv_quantize_multi")
    return outs


def quantize_sr(src, role, fmt, seed, layout=NCHW, shape=None, out=None, stream=None):
    """quantize() with stochastic rounding of the elements under `seed`."""
    dtype, shape = _quant_args(src, layout, shape)
    if out is None:
        out = MxTensor.empty(role, fmt, shape, src.device)
    _check(lib().mxconv_quantize_sr(_ptr(src), dtype, layout, role, fmt, *shape, int(seed) & (2 ** 64 - 1),
                                    _ptr(out.codes), _ptr(out.scales), _stream(stream)), "mxconv_quantize_sr")
    return out


class NvfpTensor:
    """A tensor in the two-level NVFP format: codes (MX-CBF layout), E4M3
    block scales, and the per-tensor scale (a one-element float tensor)."""

    def __init__(self, codes, scales, tscale, role, fmt, shape):
        self.codes, self.scales, self.tscale = codes, scales, tscale
        self.role, self.fmt, self.shape = role, fmt, tuple(shape)


def nvfp_quantize(src, role, fmt, layout=NCHW, shape=None, workspace=None, stream=None):
    """Eqs. (4)-(6) on the GPU: CBF activations (batch block 32) or OIHW weights."""
    dtype, shape = _quant_args(src, layout, shape)
    L = lib()
    nb = L.mxconv_codes_bytes(role, fmt, *shape)
    ns = L.mxconv_nvfp_scales_bytes(role, fmt, *shape)
    if nb == 0 or ns == 0:
        raise MxconvError(f"invalid NVFP tensor geometry {shape} role {role} fmt {fmt}")
    out = NvfpTensor(torch.empty(nb, dtype=torch.uint8, device=src.device),
                     torch.empty(ns, dtype=torch.uint8, device=src.device),
                     torch.empty(4, dtype=torch.float32, device=src.device), role, fmt, shape)
    wsb = L.mxconv_nvfp_workspace_bytes()
    if workspace is None:
        workspace = torch.empty(wsb, dtype=torch.uint8, device=src.device)
    _check(L.mxconv_nvfp_quantize(_ptr(src), dtype, layout, role, fmt, *shape, _ptr(out.codes), _ptr(out.scales),
                                  _ptr(out.tscale), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                  _stream(stream)), "mxconv_nvfp_quantize")
    return out


def nvfp_fwd(cv, w, x, layout=NCHW, out=None, stream=None):
    """Y = W * X on NVFP operands (NvfpTensor): NVFP4, NVFP6 E2M3, NVFP8, or
    NVFP4 weights with NVFP6 E3M2 activations."""
    y = _out((cv["n"], cv["cout"], *out_size(cv)), layout, batch_block(cv["n"]), x.codes.device, out)
    _check(lib().mxconv_nvfp_fwd(_conv(cv), pair(w.fmt, x.fmt), _ptr(w.codes), _ptr(w.scales), _ptr(w.tscale),
                                 _ptr(x.codes), _ptr(x.scales), _ptr(x.tscale), _ptr(y), layout, _stream(stream)),
           "mxconv_nvfp_fwd")
    return y


def nvfp_dgrad(cv, w, gy, layout=NCHW, out=None, stream=None):
    gx = _out((cv["n"], cv["cin"], cv["h"], cv["w"]), layout, batch_block(cv["n"]), gy.codes.device, out)
    _check(lib().mxconv_nvfp_dgrad(_conv(cv), pair(w.fmt, gy.fmt), _ptr(w.codes), _ptr(w.scales),
                                   _ptr(w.tscale), _ptr(gy.codes), _ptr(gy.scales), _ptr(gy.tscale), _ptr(gx), layout,
                                   _stream(stream)), "mxconv_nvfp_dgrad")
    return gx


def nvfp_wgrad(cv, gy, x, out=None, workspace=None, stream=None):
    gw = out if out is not None else torch.empty((cv["cout"], cv["cin"], cv["kh"], cv["kw"]),
                                                 dtype=torch.float32, device=x.codes.device)
    fmt = pair(gy.fmt, x.fmt)
    need = nvfp_wgrad_workspace_bytes(cv, fmt)
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.codes.device)
    wsz = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().mxconv_nvfp_wgrad(_conv(cv), fmt, _ptr(gy.codes), _ptr(gy.scales),
                                   _ptr(gy.tscale), _ptr(x.codes), _ptr(x.scales), _ptr(x.tscale), _ptr(gw),
                                   _ptr(workspace), wsz, _stream(stream)), "mxconv_nvfp_wgrad")
    return gw


def im2col_cbf(cv, x, stream=None):
    c = _conv(cv)
    nb = lib().mxconv_im2col_codes_bytes(c, x.fmt)
    ns = lib().mxconv_im2col_scales_bytes(c, x.fmt)
    codes = torch.empty(nb, dtype=torch.uint8, device=x.codes.device)
    scales = torch.empty(ns, dtype=torch.uint8, device=x.codes.device)
    _check(lib().mxconv_im2col_cbf(c, x.fmt, _ptr(x.codes), _ptr(x.scales), _ptr(codes),
                                   _ptr(scales), _stream(stream)), "mxconv_im2col_cbf")
    return codes, scales


def _want(t, dtype, what):
    """A device tensor argument must have the element type the call reads or
    writes through its pointer."""
    if t is not None and t.dtype != dtype:
        raise MxconvError(f"{what} must be {dtype}, got {t.dtype}")


def _out(shape, layout, bn, device, out):
    n, c, h, w = shape
    dtype = torch.bfloat16 if layout == CBF_BF16 else torch.float32
    if out is not None:
        _want(out, dtype, "the output")
        return out
    if layout in (CBF, CBF_BF16):
        return torch.empty((n // bn, h, w, c, bn), dtype=dtype, device=device)
    return torch.empty((n, c, h, w), dtype=dtype, device=device)


def batch_block(n):
    return 32 if n >= 32 else n


def fwd(cv, w, x, layout=NCHW, out=None, stream=None):
    ho, wo = out_size(cv)
    y = _out((cv["n"], cv["cout"], ho, wo), layout, batch_block(cv["n"]), x.codes.device, out)
    _check(lib().mxconv_fwd(_conv(cv), pair(w.fmt, x.fmt), _ptr(w.codes), _ptr(w.scales),
                            _ptr(x.codes), _ptr(x.scales), _ptr(y), layout, _stream(stream)), "mxconv_fwd")
    return y


def dgrad(cv, w, gy, layout=NCHW, out=None, stream=None):
    gx = _out((cv["n"], cv["cin"], cv["h"], cv["w"]), layout, batch_block(cv["n"]), gy.codes.device, out)
    _check(lib().mxconv_dgrad(_conv(cv), pair(w.fmt, gy.fmt), _ptr(w.codes), _ptr(w.scales),
                              _ptr(gy.codes), _ptr(gy.scales), _ptr(gx), layout, _stream(stream)),
           "mxconv_dgrad")
    return gx


def wgrad(cv, gy, x, out=None, workspace=None, stream=None, deferred=False):
    """G_W = G_Y * X^T.  deferred: leave the split-K partial sums in the
    workspace for wgrad_reduce_multi (the workspace must then be passed)."""
    gw = out if out is not None else torch.empty((cv["cout"], cv["cin"], cv["kh"], cv["kw"]),
                                                 dtype=torch.float32, device=x.codes.device)
    need = wgrad_workspace_bytes(cv, pair(gy.fmt, x.fmt))
    if workspace is None and need:
        if deferred:
            raise MxconvError("a deferred weight gradient needs the caller's workspace")
        workspace = torch.empty(need, dtype=torch.uint8, device=x.codes.device)
    wsz = workspace.numel() * workspace.element_size() if workspace is not None else 0
    fn, name = (lib().mxconv_wgrad_deferred, "mxconv_wgrad_deferred") if deferred else (lib().mxconv_wgrad,
                                                                                          "mxconv_wgrad")
    _check(fn(_conv(cv), pair(gy.fmt, x.fmt), _ptr(gy.codes), _ptr(gy.scales),
              _ptr(x.codes), _ptr(x.scales), _ptr(gw), _ptr(workspace), wsz, _stream(stream)), name)
    return gw


def backward(cv, w, gy, x, layout=NCHW, gx_out=None, gw_out=None, workspace=None, stream=None, deferred=False):
    """Input and weight gradients of one layer from one call: (G_X, G_W), bit
    for bit what dgrad() and wgrad() give (one launch where the layer allows)."""
    f = pair(w.fmt, gy.fmt)
    if pair(gy.fmt, x.fmt) != f:
        raise MxconvError("backward needs the same format pair for (W, G_Y) and (G_Y, X)")
    dev = gy.codes.device
    gx = _out((cv["n"], cv["cin"], cv["h"], cv["w"]), layout, batch_block(cv["n"]), dev, gx_out)
    gw = gw_out if gw_out is not None else torch.empty((cv["cout"], cv["cin"], cv["kh"], cv["kw"]),
                                                       dtype=torch.float32, device=dev)
    need = wgrad_workspace_bytes(cv, f)
    if workspace is None and need:
        if deferred:
            raise MxconvError("a deferred weight gradient needs the caller's workspace")
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    wsz = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().mxconv_backward(_conv(cv), f, _ptr(w.codes), _ptr(w.scales), _ptr(gy.codes),
                                 _ptr(gy.scales), _ptr(x.codes), _ptr(x.scales), _ptr(gx), layout, _ptr(gw),
                                 _ptr(workspace), wsz, 1 if deferred else 0, _stream(stream)), "mxconv_backward")
    return gx, gw


def wgrad_reduce_multi(items, stream=None):
    """Finish deferred weight gradients in one launch.  items: tuples
    (cv, fmt, workspace, gw) of the deferred calls (fmt as passed to them:
    pair(gy.fmt, x.fmt))."""
    if len(items) > WREDUCE_MAX:
        raise MxconvError(f"at most {WREDUCE_MAX} layers per call")
    jobs = (MxcWJob * max(1, len(items)))()
    for k, (cv, fmt, ws, gw) in enumerate(items):
        jobs[k] = MxcWJob(ctypes.pointer(_conv_of(_conv_key(cv))), fmt, ws.data_ptr() if ws is not None else None,
                          ws.numel() * ws.element_size() if ws is not None else 0, gw.data_ptr())
    _check(lib().mxconv_wgrad_reduce_multi(len(items), jobs, _stream(stream)), "mxconv_wgrad_reduce_multi")


def fwd_quant(cv, w, x, fn=FN_NONE, out_fmt=None, out=None, act_out=None, stream=None):
    """Forward with the quantizing epilogue: MX codes of fn(W * X) for
    (n, cout, Ho, Wo); `act_out` (CBF fp32, optional) receives the values
    that were quantized (with FN_PRE_OUT: W * X; with FN_BF16 | FN_PRE_OUT
    it is bf16 and receives W * X rounded to bf16).  Returns the MxTensor."""
    _want(act_out, torch.bfloat16 if (fn & FN_BF16) and (fn & FN_PRE_OUT) else torch.float32, "act_out")
    ho, wo = out_size(cv)
    out_fmt = x.fmt if out_fmt is None else out_fmt
    shape = (cv["n"], cv["cout"], ho, wo)
    y = out if out is not None else MxTensor.empty(ACT, out_fmt, shape, x.codes.device)
    _check(lib().mxconv_fwd_quant(_conv(cv), pair(w.fmt, x.fmt), _ptr(w.codes), _ptr(w.scales),
                                  _ptr(x.codes), _ptr(x.scales), fn, out_fmt, _ptr(y.codes), _ptr(y.scales),
                                  _ptr(act_out), _stream(stream)), "mxconv_fwd_quant")
    return y


def dgrad_quant(cv, w, gy, fn=FN_NONE, z=None, out_fmt=None, out=None, act_out=None, stream=None, sr_seed=None):
    """Input gradient with the quantizing epilogue: MX codes of
    (W^T * G_Y) . fn'(z) for (n, cin, h, w); z is the CBF pre-activation of
    this layer's input (not needed for FN_NONE), fp32, or bf16 with FN_BF16.
    act_out (optional) is fp32.  sr_seed: round the codes stochastically
    (mxconv_dgrad_quant_sr) with this 64-bit seed."""
    _want(z, torch.bfloat16 if fn & FN_BF16 else torch.float32, "z")
    _want(act_out, torch.float32, "act_out")
    out_fmt = gy.fmt if out_fmt is None else out_fmt
    shape = (cv["n"], cv["cin"], cv["h"], cv["w"])
    g = out if out is not None else MxTensor.empty(ACT, out_fmt, shape, gy.codes.device)
    args = (_conv(cv), pair(w.fmt, gy.fmt), _ptr(w.codes), _ptr(w.scales), _ptr(gy.codes),
            _ptr(gy.scales), fn, _ptr(z), out_fmt, _ptr(g.codes), _ptr(g.scales), _ptr(act_out))
    if sr_seed is None:
        _check(lib().mxconv_dgrad_quant(*args, _stream(stream)), "mxconv_dgrad_quant")
    else:
        _check(lib().mxconv_dgrad_quant_sr(*args, sr_seed, _stream(stream)), "mxconv_dgrad_quant_sr")
    return g


# ---------------------------------------------------------------- network steps
def concat_cbf(parts, out=None, stream=None):
    """Concatenate MX-CBF activations along channels, whole blocks, in order.
    parts: MxTensors, or (MxTensor, up) with up = 1 for a 2x nearest-neighbour
    upsampling of that part.  Returns the MxTensor of (n, 32 * sum ncb, h, w)."""
    if not 1 <= len(parts) <= CONCAT_MAX:
        raise MxconvError(f"1 to {CONCAT_MAX} parts")
    arr = (MxcPart * len(parts))()
    nb, hw, fmt = 0, None, None
    for k, p in enumerate(parts):
        t, up = (p, 0) if isinstance(p, MxTensor) else p
        n, c, h, w = t.shape
        ncb = (c + 31) // 32
        arr[k] = MxcPart(t.codes.data_ptr(), t.scales.data_ptr(), ncb, up)
        nb += ncb
        hw = (h * 2, w * 2) if up else (h, w)
        fmt, dev = t.fmt, t.codes.device
    shape = (n, 32 * nb, hw[0], hw[1])
    y = out if out is not None else MxTensor.empty(ACT, fmt, shape, dev)
    _check(lib().mxconv_concat_cbf(fmt, shape[0], shape[2], shape[3], len(parts), arr, _ptr(y.codes), _ptr(y.scales),
                                   _stream(stream)), "mxconv_concat_cbf")
    return y


def quantize_sum(terms, shape, fmt, fn=FN_NONE, z=None, out=None, vals=None, stream=None, sr_seed=None):
    """MX codes of fn'(z) . (sum of terms) for the (n, c, h, w) tensor `shape`.
    terms: tuples (src, c_src, c_off, down) with src a CBF device tensor
    [n/32][hs][ws][c_src][32]; terms and z are fp32, or bf16 with FN_BF16;
    vals (optional) is fp32.  sr_seed: round the codes stochastically
    (mxconv_quantize_sum_sr) with this 64-bit seed."""
    if not 1 <= len(terms) <= TERMS_MAX:
        raise MxconvError(f"1 to {TERMS_MAX} terms")
    dt = torch.bfloat16 if fn & FN_BF16 else torch.float32
    _want(z, dt, "z")
    _want(vals, torch.float32, "vals")
    arr = (MxcTerm * len(terms))()
    for k, (src, c_src, c_off, down) in enumerate(terms):
        _want(src, dt, f"term {k}")
        arr[k] = MxcTerm(src.data_ptr(), c_src, c_off, down)
    n, c, h, w = shape
    g = out if out is not None else MxTensor.empty(ACT, fmt, shape, terms[0][0].device)
    args = (fmt, n, c, h, w, len(terms), arr, fn, _ptr(z), _ptr(g.codes), _ptr(g.scales), _ptr(vals))
    if sr_seed is None:
        _check(lib().mxconv_quantize_sum(*args, _stream(stream)), "mxconv_quantize_sum")
    else:
        _check(lib().mxconv_quantize_sum_sr(*args, sr_seed, _stream(stream)), "mxconv_quantize_sum_sr")
    return g


# ---------------------------------------------------------------- linear layers, residual norms, clipping
# These calls check what a pointer cannot say (device, type, strides, sizes),
# run with the tensors' device current, and allocate on the stream they launch
# on: a workspace freed at return is reused only by later work of that stream.
LINEAR_FWD, LINEAR_DGRAD, LINEAR_WGRAD = 0, 1, 2


def _place(device, stream):
    """The context of a call -- the stream where one is given, else the tensors'
    device where it is not the current one -- or None."""
    if device.type != "cuda":
        raise MxconvError(f"tensors must be on a GPU, got {device}")
    if stream is not None:
        if stream.device != device:
            raise MxconvError(f"the stream is on {stream.device}, the tensors on {device}")
        return torch.cuda.stream(stream)
    here = _raw_device() if _raw_device is not None else torch.cuda.current_device()
    return None if device.index == here else torch.cuda.device(device)


def _launch(fn, device, stream, *args):
    """fn(raw stream, *args), a call's launching part, in its context."""
    place = _place(device, stream)
    if place is None:
        return fn(_raw_stream(device.index) if _raw_stream is not None else _stream(None), *args)
    with place:
        return fn(_stream(stream), *args)


def _rows_cols(t, what, shape, dtype, device):
    """The row stride of a row-major full-precision matrix argument."""
    if t.dtype != dtype:
        raise MxconvError(f"{what} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise MxconvError(f"{what} must be {shape[0]} x {shape[1]}, got {tuple(t.shape)}")
    if t.device != device:
        raise MxconvError(f"{what} must be on {device}, got {t.device}")
    ld, step = t.stride()
    if step != 1 and shape[1] > 1:
        raise MxconvError(f"{what} must have unit column stride")
    return ld if shape[0] > 1 else shape[1]


def _vector(t, what, shape, device):
    """An fp32 parameter argument."""
    if t.dtype != torch.float32 or t.shape != shape or t.device != device or not t.is_contiguous():
        raise MxconvError(f"{what} must be a contiguous fp32 tensor of shape {tuple(shape)} on {device}")


@functools.lru_cache(maxsize=_CACHED)
def _mx_geometry(role, fmt, shape):
    """(rows, columns, code bytes, scale bytes) of an MX matrix, or None."""
    r, c, h, w = shape
    if h != 1 or w != 1 or (role == ACT and r % 32) or not codes_bytes(WEIGHT, fmt, r, c, 1, 1):
        return None
    return r, c, codes_bytes(WEIGHT, fmt, r, c, 1, 1), scales_bytes(WEIGHT, fmt, r, c, 1, 1)


def _mx_matrix(q, what):
    """(rows, columns, device) of an MX matrix argument: shape (R, C, 1, 1) with
    32-row blocks."""
    g = _mx_geometry(q.role, q.fmt, q.shape)
    if g is None:
        raise MxconvError(f"{what} must be an MX matrix: shape (R, C, 1, 1), role WEIGHT (or ACT with R a multiple of 32)")
    c, s = q.codes, q.scales
    dev = c.device
    if (c.dtype != torch.uint8 or s.dtype != torch.uint8 or c.numel() < g[2] or s.numel() < g[3] or
            not (c.is_contiguous() and s.is_contiguous()) or s.get_device() != c.get_device()):
        raise MxconvError(f"{what}: codes and scales must be contiguous uint8 tensors of the matrix's size on one device")
    return g[0], g[1], dev


@functools.lru_cache(maxsize=_CACHED)
def _linear_of(rows, outs, ins):
    """The layer's struct (only read by the library) and its workspace sizes."""
    s = MxcLinear(rows, outs, ins)
    return ctypes.byref(s), tuple(lib().mxconv_linear_workspace_bytes(op, ctypes.byref(s)) for op in range(3))


def _dtype_code(dtype):
    code = _DTYPES.get(dtype)
    if code is None:
        raise MxconvError(f"unsupported dtype {dtype}")
    return code


def linear_workspace_bytes(op, rows, outs, ins):
    return _linear_of(rows, outs, ins)[1][op]


def _workspace(ws, need, device):
    """(tensor to keep, pointer, bytes) of a call's workspace."""
    if ws is None:
        if not need:
            return None, None, 0
        ws = torch.empty(need, dtype=torch.uint8, device=device)
        return ws, ws.data_ptr(), need
    if ws.device != device or not ws.is_contiguous():
        raise MxconvError(f"the workspace must be a contiguous tensor on {device}")
    return ws, ws.data_ptr(), ws.numel() * ws.element_size()


def quantize_matrix(m, fmt, out=None, stream=None):
    """The MX matrix of a contiguous fp32 or bf16 matrix [R][C], an operand of
    the linear products in any of its roles: quantize() with role WEIGHT and
    shape (R, C, 1, 1)."""
    if m.dim() != 2:
        raise MxconvError("quantize_matrix needs a matrix")
    return quantize(m, WEIGHT, fmt, shape=(m.shape[0], m.shape[1], 1, 1), out=out, stream=stream)


def linear(w, x, bias=None, fn=FN_NONE, residual=None, dtype=torch.bfloat16, out=None, pre_out=None, workspace=None,
           stream=None):
    """Y = fn(X W^T + bias) + residual, [rows][outs] of `dtype`, from the MX
    matrices W [outs][ins] and X [rows][ins] (mxconv_linear_fwd).  pre_out
    receives X W^T + bias."""
    (outs, ins, wdev), (rows, k, dev) = _mx_matrix(w, "w"), _mx_matrix(x, "x")
    if k != ins or wdev != dev:
        raise MxconvError(f"w is {outs} x {ins} on {wdev}, x {rows} x {k} on {dev}")
    if bias is not None:
        _vector(bias, "bias", (outs,), dev)
    return _launch(_linear, dev, stream, (rows, outs), ins, w, x, bias, fn, residual, dtype, out, pre_out, workspace, dev)


def _linear(raw, shape, ins, w, x, bias, fn, residual, dtype, out, pre_out, workspace, dev):
    code = _dtype_code(dtype)
    y = out if out is not None else x.codes.new_empty(shape, dtype=dtype)
    ldr = _rows_cols(residual, "residual", shape, dtype, dev) if residual is not None else 0
    ldz = _rows_cols(pre_out, "pre_out", shape, dtype, dev) if pre_out is not None else 0
    ldy = _rows_cols(y, "the output", shape, dtype, dev) if out is not None else shape[1]
    s, need = _linear_of(shape[0], shape[1], ins)
    ws, wp, wb = _workspace(workspace, need[0], dev)
    _check(lib().mxconv_linear_fwd(s, pair(w.fmt, x.fmt), w.codes.data_ptr(), w.scales.data_ptr(), x.codes.data_ptr(),
                                   x.scales.data_ptr(), _ptr(bias), fn, _ptr(residual), ldr, y.data_ptr(), ldy,
                                   _ptr(pre_out), ldz, code, wp, wb, raw), "mxconv_linear_fwd")
    return y


def linear_dgrad(w, dz, fn=FN_NONE, z=None, add=None, dtype=torch.bfloat16, out=None, workspace=None, stream=None):
    """dX = fn'(z) . (dZ W) + add, [rows][ins] of `dtype`, from the MX matrices
    W [outs][ins] and dZ [rows][outs] (mxconv_linear_dgrad)."""
    (outs, ins, wdev), (rows, n, dev) = _mx_matrix(w, "w"), _mx_matrix(dz, "dz")
    if n != outs or wdev != dev:
        raise MxconvError(f"w is {outs} x {ins} on {wdev}, dz {rows} x {n} on {dev}")
    return _launch(_linear_dgrad, dev, stream, (rows, ins), outs, w, dz, fn, z, add, dtype, out, workspace, dev)


def _linear_dgrad(raw, shape, outs, w, dz, fn, z, add, dtype, out, workspace, dev):
    code = _dtype_code(dtype)
    dx = out if out is not None else dz.codes.new_empty(shape, dtype=dtype)
    ldz = _rows_cols(z, "z", shape, dtype, dev) if z is not None else 0
    lda = _rows_cols(add, "add", shape, dtype, dev) if add is not None else 0
    ldx = _rows_cols(dx, "the output", shape, dtype, dev) if out is not None else shape[1]
    s, need = _linear_of(shape[0], outs, shape[1])
    ws, wp, wb = _workspace(workspace, need[1], dev)
    _check(lib().mxconv_linear_dgrad(s, pair(w.fmt, dz.fmt), w.codes.data_ptr(), w.scales.data_ptr(), dz.codes.data_ptr(),
                                     dz.scales.data_ptr(), fn, _ptr(z), ldz, _ptr(add), lda, dx.data_ptr(), ldx, code, wp, wb,
                                     raw), "mxconv_linear_dgrad")
    return dx


def linear_wgrad(dz, x, bias=True, out=None, bias_out=None, workspace=None, stream=None):
    """(dW, db): dZ^T X, fp32 [outs][ins], and the column sums of dZ, fp32
    [outs] (None with bias=False), from the MX matrices dZ [rows][outs] and
    X [rows][ins] (mxconv_linear_wgrad)."""
    (rows, outs, gdev), (r2, ins, dev) = _mx_matrix(dz, "dz"), _mx_matrix(x, "x")
    if r2 != rows or gdev != dev:
        raise MxconvError(f"dz is {rows} x {outs} on {gdev}, x {r2} x {ins} on {dev}")
    return _launch(_linear_wgrad, dev, stream, rows, outs, ins, dz, x, bias, out, bias_out, workspace, dev)


def _linear_wgrad(raw, rows, outs, ins, dz, x, bias, dw, db, workspace, dev):
    if dw is None:
        dw = x.codes.new_empty((outs, ins), dtype=torch.float32)
    else:
        _vector(dw, "the output", (outs, ins), dev)
    if db is not None:
        _vector(db, "bias_out", (outs,), dev)
    elif bias:
        db = x.codes.new_empty((outs,), dtype=torch.float32)
    s, need = _linear_of(rows, outs, ins)
    ws, wp, wb = _workspace(workspace, need[2], dev)
    _check(lib().mxconv_linear_wgrad(s, pair(dz.fmt, x.fmt), dz.codes.data_ptr(), dz.scales.data_ptr(), x.codes.data_ptr(),
                                     x.scales.data_ptr(), dw.data_ptr(), _ptr(db), wp, wb, raw), "mxconv_linear_wgrad")
    return dw, db


def _norm_struct(y, w_post, gate, scale, w_pre, eps):
    if y.dim() != 2 or y.dtype not in _DTYPES:
        raise MxconvError("the residual norms need fp32 or bf16 matrices")
    rows, d = y.shape
    if gate is not None and gate.dim() == 1:
        gate = gate[None]
    if gate is not None and (gate.dim() != 2 or gate.shape[0] == 0 or rows % gate.shape[0]):
        raise MxconvError(f"gate must be [d] or [gates][d] with gates dividing the {rows} rows, got {tuple(gate.shape)}")
    gates = gate.shape[0] if gate is not None else 1
    dev = y.device
    if w_post is not None:
        _vector(w_post, "w_post", (d,), dev)
    if w_pre is not None:
        _vector(w_pre, "w_pre", (d,), dev)
    if gate is not None:
        _vector(gate, "gate", (gates, d), dev)
    return MxcNorm(rows, gates, d, _DTYPES[y.dtype], scale, eps, _ptr(w_post), _ptr(gate), _ptr(w_pre)), gates


def norm_workspace_bytes(rows, d, gates=1, gate=True, post=True, pre=True):
    """Workspace of norm_residual_backward for `rows` rows of length d with
    these parameters (with fewer parameters it is no larger)."""
    return _norm_workspace_bytes(rows, gates, d, gate, post, pre)


@functools.lru_cache(maxsize=_CACHED)
def _norm_workspace_bytes(rows, gates, d, gate, post, pre):
    some = 16                                         # only whether a pointer is NULL is looked at
    s = MxcNorm(rows, gates, d, F32, 1.0, 0.0, some if post else None, some if gate else None, some if pre else None)
    return lib().mxconv_norm_workspace_bytes(ctypes.byref(s))


def norm_residual(x, y, w_post=None, gate=None, scale=1.0, w_pre=None, eps=1e-6, h_out=None, u_out=None, stream=None):
    """(H, U): H = x + scale * gate . N(y; w_post) and U = N(H; w_pre), N(v; w)
    = w . v / sqrt(mean(v^2) + eps) by rows (mxconv_norm_fwd).  x, y: [rows][d],
    fp32 or bf16; w_post, w_pre: fp32 [d] or None (N(y) is y; no U); gate: fp32
    [d], [gates][d] (each for rows / gates consecutive rows) or None."""
    s, gates = _norm_struct(y, w_post, gate, scale, w_pre, eps)
    return _launch(_norm_residual, y.device, stream, s, x, y, w_pre is not None, h_out, u_out, y.device)


def _norm_residual(raw, s, x, y, pre, h, u, dev):
    shape, dt = y.shape, y.dtype
    # a row-major y (checked here): empty_like() is contiguous
    ldx, ldy = _rows_cols(x, "x", shape, dt, dev), _rows_cols(y, "y", shape, dt, dev)
    ldh = ldu = shape[1]
    if h is None:
        h = torch.empty_like(y)
    else:
        ldh = _rows_cols(h, "h_out", shape, dt, dev)
    if not pre:
        u = None
    elif u is None:
        u = torch.empty_like(y)
    else:
        ldu = _rows_cols(u, "u_out", shape, dt, dev)
    _check(lib().mxconv_norm_fwd(ctypes.byref(s), x.data_ptr(), ldx, y.data_ptr(), ldy, h.data_ptr(), ldh, _ptr(u), ldu,
                                 raw), "mxconv_norm_fwd")
    return h, u


def norm_residual_backward(dh, du, h, y, w_post=None, gate=None, scale=1.0, w_pre=None, eps=1e-6, dx_out=None, dy_out=None,
                           dw_pre_out=None, dw_post_out=None, dgate_out=None, workspace=None, stream=None):
    """(dX, dY, dw_pre, dw_post, dgate) of norm_residual from the gradients dh
    of H and du of U, with H and y of the forward pass (mxconv_norm_bwd).  du
    and h may be None without w_pre; the gradients of absent parameters are
    None; dgate is [gates][d]."""
    s, gates = _norm_struct(y, w_post, gate, scale, w_pre, eps)
    if w_pre is None:
        du = h = None
    elif du is None or h is None:
        raise MxconvError("the backward pass of w_pre needs du and h")
    return _launch(_norm_backward, y.device, stream, s, gates, dh, du, h, y, w_post is not None, gate is not None, dx_out,
                   dy_out, dw_pre_out, dw_post_out, dgate_out, workspace, y.device)


def _result(t, what, shape, dev, like):
    """An fp32 output: the caller's, or a new one (like another tensor)."""
    if t is None:
        return like.new_empty(shape, dtype=torch.float32)
    _vector(t, what, shape, dev)
    return t


def _norm_backward(raw, s, gates, dh, du, h, y, post, gate, dx, dy, dw_pre, dw_post, dgate, workspace, dev):
    shape, dt = y.shape, y.dtype
    rows, d = shape
    lddh, ldy = _rows_cols(dh, "dh", shape, dt, dev), _rows_cols(y, "y", shape, dt, dev)
    lddu = ldh = lddx = lddy = d
    if h is not None:
        lddu, ldh = _rows_cols(du, "du", shape, dt, dev), _rows_cols(h, "h", shape, dt, dev)
    dw_pre = _result(dw_pre, "dw_pre_out", (d,), dev, y) if h is not None else None
    dw_post = _result(dw_post, "dw_post_out", (d,), dev, y) if post else None
    dgate = _result(dgate, "dgate_out", (gates, d), dev, y) if gate else None
    if dx is None:
        dx = torch.empty_like(y)
    else:
        lddx = _rows_cols(dx, "dx_out", shape, dt, dev)
    if dy is None:
        dy = torch.empty_like(y)
    else:
        lddy = _rows_cols(dy, "dy_out", shape, dt, dev)
    ws, wp, wb = _workspace(workspace, _norm_workspace_bytes(rows, gates, d, gate, post, h is not None), dev)
    _check(lib().mxconv_norm_bwd(ctypes.byref(s), dh.data_ptr(), lddh, _ptr(du), lddu, _ptr(h), ldh, y.data_ptr(), ldy,
                                 dx.data_ptr(), lddx, dy.data_ptr(), lddy, _ptr(dw_pre), _ptr(dw_post), _ptr(dgate), wp, wb,
                                 raw), "mxconv_norm_bwd")
    return dx, dy, dw_pre, dw_post, dgate


def _descriptors(tensors, dev):
    """Pointers, sizes and types of contiguous fp32 / bf16 tensors on device
    `dev`, a list each (by map(): a step has hundreds of tensors)."""
    types = list(map(_dtype_of, tensors))
    if not set(types) <= _DTYPES.keys() or set(map(torch.Tensor.get_device, tensors)) != {dev.index} or \
            not all(map(torch.Tensor.is_contiguous, tensors)):
        raise MxconvError(f"gradients and their outputs must be contiguous fp32 or bf16 tensors on {dev}")
    return list(map(torch.Tensor.data_ptr, tensors)), list(map(torch.Tensor.numel, tensors)), types


_dtype_of = attrgetter("dtype")


def _clip(tensors, outs, max_norm, norm_out, workspace, stream):
    if not tensors:
        raise MxconvError("no tensors")
    dev = tensors[0].device
    if dev.type != "cuda":
        raise MxconvError(f"tensors must be on a GPU, got {dev}")
    ptrs, sizes, types = _descriptors(tensors, dev)
    desc = array("q", bytes(32 * len(ptrs)))          # mxc_gtensor: src, dst, n, dtype
    desc[0::4] = array("q", ptrs)
    desc[2::4] = array("q", sizes)
    desc[3::4] = array("q", map(_DTYPES.get, types))
    if outs is not None:
        dst = ptrs
        if outs is not tensors:
            outs = list(outs)
            if len(outs) != len(tensors):
                raise MxconvError(f"{len(outs)} outputs for {len(tensors)} tensors")
            dst, osizes, otypes = _descriptors(outs, dev)
            if osizes != sizes or otypes != types:
                raise MxconvError("an output must have its gradient's size and type")
        desc[1::4] = array("q", dst)
    return _launch(_clip_launch, dev, stream, len(ptrs), desc, max_norm, norm_out, workspace, dev)


def _clip_launch(raw, count, desc, max_norm, norm, workspace, dev):
    if norm is None:
        norm = torch.empty((), dtype=torch.float32, device=dev)
    elif norm.dtype != torch.float32 or norm.numel() != 1 or norm.device != dev:
        raise MxconvError(f"norm_out must be one fp32 element on {dev}")
    ws, wp, wb = _workspace(workspace, _clip_workspace_bytes(), dev)
    _check(lib().mxconv_grad_clip(count, desc.buffer_info()[0], max_norm, norm.data_ptr(), wp, wb, raw), "mxconv_grad_clip")
    return norm


@functools.lru_cache(maxsize=None)
def _clip_workspace_bytes():
    return lib().mxconv_grad_clip_workspace_bytes()


def grad_norm(tensors, norm_out=None, workspace=None, stream=None):
    """The Euclidean norm of all elements of the tensors, an fp32 device scalar."""
    return _clip(list(tensors), None, float("inf"), norm_out, workspace, stream)


def grad_clip(tensors, max_norm, out=None, norm_out=None, workspace=None, stream=None):
    """Scale the tensors (contiguous fp32 or bf16) by min(1, max_norm / (norm +
    1e-6)), norm = their Euclidean norm together, into `out` (tensors of the
    same sizes and types, sharing no memory with each other or with a gradient
    other than their own; None: in place).  Returns the norm before scaling, an
    fp32 device scalar; nothing is synchronized (mxconv_grad_clip)."""
    tensors = list(tensors)
    return _clip(tensors, tensors if out is None else out, max_norm, norm_out, workspace, stream)


# ---------------------------------------------------------------- naive comparator
# Channels-last GEMM form: P = n*Ho*Wo positions (n, ho, wo), K = kh*kw*cin
# (kh, kw, ci); X, G_Y, G_X NHWC fp32; W, G_W OHWI fp32 ([cout][K]).
class LineMatrix:
    """A 1-D-blocked matrix: codes [lines][Lp] and scales [lines][Lp/32]."""

    def __init__(self, codes, scales, fmt, lines, length):
        self.codes, self.scales, self.fmt, self.lines, self.length = codes, scales, fmt, lines, length


def naive_im2col_f32(cv, x, out=None, stream=None):
    ho, wo = out_size(cv)
    col = out if out is not None else torch.empty((cv["n"] * ho * wo, cv["kh"] * cv["kw"] * cv["cin"]),
                                                  dtype=torch.float32, device=x.device)
    _check(lib().mxconv_naive_im2col_f32(_conv(cv), _ptr(x), _ptr(col), _stream(stream)),
           "mxconv_naive_im2col_f32")
    return col


def naive_quantize_1d(m, direction, fmt, out=None, stream=None):
    """Quantize a contiguous fp32 [rows][cols] device matrix with 1-D blocks
    of 32 along its rows (direction 0) or columns (direction 1)."""
    rows, cols = m.shape
    lines, length = (rows, cols) if direction == 0 else (cols, rows)
    if out is None:
        nb = lib().mxconv_naive_codes_bytes(lines, length, fmt)
        ns = lib().mxconv_naive_scales_bytes(lines, length)
        if nb == 0:
            raise MxconvError(f"invalid line matrix {lines} x {length}")
        out = LineMatrix(torch.empty(nb, dtype=torch.uint8, device=m.device),
                         torch.empty(ns, dtype=torch.uint8, device=m.device), fmt, lines, length)
    if m.dtype != torch.float32 or not m.is_contiguous():
        raise MxconvError("naive_quantize_1d needs a contiguous fp32 matrix")
    _check(lib().mxconv_naive_quantize_1d(_ptr(m), rows, cols, direction, fmt, _ptr(out.codes),
                                          _ptr(out.scales), _stream(stream)), "mxconv_naive_quantize_1d")
    return out


def naive_fwd(cv, col_q, w_q, out=None, stream=None):
    ho, wo = out_size(cv)
    y = out if out is not None else torch.empty((cv["n"] * ho * wo, cv["cout"]), dtype=torch.float32,
                                                device=col_q.codes.device)
    _check(lib().mxconv_naive_fwd(_conv(cv), col_q.fmt, _ptr(col_q.codes),
                                  _ptr(col_q.scales), _ptr(w_q.codes), _ptr(w_q.scales), _ptr(y),
                                  _stream(stream)), "mxconv_naive_fwd")
    return y


def naive_dgrad(cv, gy_q, wt_q, gcol=None, out=None, stream=None):
    ho, wo = out_size(cv)
    dev = gy_q.codes.device
    if gcol is None:
        gcol = torch.empty((cv["n"] * ho * wo, cv["kh"] * cv["kw"] * cv["cin"]), dtype=torch.float32,
                           device=dev)
    gx = out if out is not None else torch.empty((cv["n"], cv["h"], cv["w"], cv["cin"]),
                                                 dtype=torch.float32, device=dev)
    _check(lib().mxconv_naive_dgrad(_conv(cv), gy_q.fmt, _ptr(gy_q.codes),
                                    _ptr(gy_q.scales), _ptr(wt_q.codes), _ptr(wt_q.scales), _ptr(gcol),
                                    _ptr(gx), _stream(stream)), "mxconv_naive_dgrad")
    return gx


def naive_wgrad(cv, gyt_q, xt_q, out=None, stream=None):
    gw = out if out is not None else torch.empty((cv["cout"], cv["kh"] * cv["kw"] * cv["cin"]),
                                                 dtype=torch.float32, device=gyt_q.codes.device)
    _check(lib().mxconv_naive_wgrad(_conv(cv), gyt_q.fmt, _ptr(gyt_q.codes),
                                    _ptr(gyt_q.scales), _ptr(xt_q.codes), _ptr(xt_q.scales), _ptr(gw),
                                    _stream(stream)), "mxconv_naive_wgrad")
    return gw
