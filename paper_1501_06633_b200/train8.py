"""ctypes binding of the 8-bit training operators of ``libmaxdnn.so``: same names as
``include/maxdnn.h``, argument marshalling only.  Tensors are torch CUDA tensors; matrices may be
views with a row pitch (``stride(0)``) that matches the descriptor.  8-bit values are
``torch.float8_e4m3fn`` / ``torch.float8_e5m2``, scales ``torch.float8_e8m0fnu`` (or ``uint8`` bytes)."""
from __future__ import annotations

import ctypes
import warnings

from .binding import OK, MaxdnnError, load_library

__all__ = [
    "DTYPE_F32", "DTYPE_BF16", "DTYPE_F16", "DTYPE_E4M3", "DTYPE_E5M2", "DTYPE_E8M0",
    "BLOCK_ROW", "BLOCK_COL", "BLOCK_TILE", "MAJOR_K", "MAJOR_MN",
    "ACT_SILU", "ACT_GELU", "ACT_GELU_TANH",
    "Quant8Desc", "Gemm8Desc", "LayerNormDesc", "Act8Desc",
    "quant8", "dequant8", "gemm8", "layer_norm_fprop", "layer_norm_bprop_workspace",
    "layer_norm_bprop", "act8_fprop", "act8_bprop", "empty_packed", "empty_scales",
]

DTYPE_F32, DTYPE_BF16, DTYPE_F16, DTYPE_E4M3, DTYPE_E5M2, DTYPE_E8M0 = range(6)
BLOCK_ROW, BLOCK_COL, BLOCK_TILE = range(3)
MAJOR_K, MAJOR_MN = range(2)
ACT_SILU, ACT_GELU, ACT_GELU_TANH = range(3)

_vp = ctypes.c_void_p
torch = None      # imported with the library, at the first call
_current_device = _current_raw_stream = None
_TYPES = ()       # the tensor types of each DTYPE_* code


def _round16(n):
    return -(-int(n) // 16) * 16


def _or(value, default):
    return int(default if value is None else value)


class Quant8Desc(ctypes.Structure):
    """maxdnn_quant8_desc."""

    _fields_ = [("rows", ctypes.c_int32), ("cols", ctypes.c_int32), ("ldx", ctypes.c_int64),
                ("ldq", ctypes.c_int64), ("x_type", ctypes.c_int32), ("q_type", ctypes.c_int32)]

    @classmethod
    def make(cls, rows, cols, x_type=DTYPE_BF16, q_type=DTYPE_E4M3, ldx=None, ldq=None) -> "Quant8Desc":
        return cls(int(rows), int(cols), _or(ldx, cols), _or(ldq, _round16(cols)), int(x_type), int(q_type))


class Gemm8Desc(ctypes.Structure):
    """maxdnn_gemm8_desc."""

    _fields_ = [(n, ctypes.c_int32) for n in ("M", "N", "K")] + \
               [(n, ctypes.c_int64) for n in ("lda", "ldb", "ldc")] + \
               [(n, ctypes.c_int32) for n in ("a_type", "b_type", "c_type", "a_major", "b_major", "a_block",
                                              "b_block", "a_scale_type", "b_scale_type")]

    @classmethod
    def make(cls, M, N, K, a_type=DTYPE_E4M3, b_type=DTYPE_E4M3, c_type=DTYPE_BF16, a_major=MAJOR_K,
             b_major=MAJOR_K, a_block=None, b_block=BLOCK_TILE, a_scale_type=DTYPE_E8M0,
             b_scale_type=DTYPE_E8M0, lda=None, ldb=None, ldc=None) -> "Gemm8Desc":
        if a_block is None:
            a_block = BLOCK_ROW if a_major == MAJOR_K else BLOCK_COL
        return cls(int(M), int(N), int(K), _or(lda, _round16(K if a_major == MAJOR_K else M)),
                   _or(ldb, _round16(K if b_major == MAJOR_K else N)), _or(ldc, N), int(a_type), int(b_type),
                   int(c_type), int(a_major), int(b_major), int(a_block), int(b_block), int(a_scale_type),
                   int(b_scale_type))


class LayerNormDesc(ctypes.Structure):
    """maxdnn_layer_norm_desc."""

    _fields_ = [("rows", ctypes.c_int32), ("cols", ctypes.c_int32), ("ldx", ctypes.c_int64),
                ("ldy", ctypes.c_int64), ("ldq", ctypes.c_int64), ("x_type", ctypes.c_int32),
                ("y_type", ctypes.c_int32), ("w_type", ctypes.c_int32), ("q_type", ctypes.c_int32),
                ("eps", ctypes.c_float)]

    @classmethod
    def make(cls, rows, cols, eps=1e-5, x_type=DTYPE_BF16, y_type=None, w_type=DTYPE_F32, q_type=DTYPE_E4M3,
             ldx=None, ldy=None, ldq=None) -> "LayerNormDesc":
        return cls(int(rows), int(cols), _or(ldx, cols), _or(ldy, cols), _or(ldq, _round16(cols)), int(x_type),
                   _or(y_type, x_type), int(w_type), int(q_type), float(eps))


class Act8Desc(ctypes.Structure):
    """maxdnn_act8_desc."""

    _fields_ = [("rows", ctypes.c_int32), ("cols", ctypes.c_int32)] + \
               [(n, ctypes.c_int64) for n in ("ldh", "lda", "ldq", "ldc")] + \
               [(n, ctypes.c_int32) for n in ("x_type", "h_type", "q_type", "act", "gated")]

    @classmethod
    def make(cls, rows, cols, act=ACT_SILU, gated=True, x_type=DTYPE_BF16, h_type=None, q_type=DTYPE_E4M3,
             ldh=None, lda=None, ldq=None, ldc=None) -> "Act8Desc":
        wide = int(cols) * (2 if gated else 1)
        return cls(int(rows), int(cols), _or(ldh, wide), _or(lda, cols), _or(ldq, _round16(cols)),
                   _or(ldc, _round16(wide)), int(x_type), _or(h_type, x_type), int(q_type), int(act),
                   1 if gated else 0)


_lib = None


class _NoPlain:
    """Stands in where the marshalling module is not built: every call goes through the checks below."""

    quant8 = dequant8 = gemm8 = layer_norm_fprop = layer_norm_bprop = act8_fprop = act8_bprop = staticmethod(lambda *a: -1)


_plain = _NoPlain


def _usable(module):
    """Whether the module was built for this torch, whose tensors it reads by the layout of its headers."""
    built = getattr(module, "torch_version", "(unknown)")
    if built != torch.__version__:
        warnings.warn("_train8 was built for torch %s, this is %s: its calls are marshalled in Python; "
                      "python -m paper_1501_06633_b200.build renews it" % (built, torch.__version__))
    return built == torch.__version__


def _load_plain(lib):
    """The module that checks and passes on the arguments of plain calls (csrc/train8_binding.cpp)."""
    if not torch.cuda.is_available():
        return _NoPlain
    try:
        from . import _train8
    except ImportError:
        return _NoPlain
    if not _usable(_train8):
        return _NoPlain
    _train8.bind(*(ctypes.cast(getattr(lib, "maxdnn_" + n), ctypes.c_void_p).value for n in (
        "quant8", "dequant8", "gemm8", "layer_norm_fprop", "layer_norm_bprop", "act8_fprop", "act8_bprop")))
    return _train8


def _raw_stream(device):
    return torch.cuda.current_stream(device).cuda_stream


def _library():
    global _lib, torch, _TYPES, _current_device, _current_raw_stream, _plain
    if _lib is None:
        lib = load_library()
        import torch
        # what torch.cuda.current_device() and current_stream().cuda_stream return, without the
        # objects around them: a small layer's call is bound by the host
        _current_device, _current_raw_stream = torch.cuda.current_device, _raw_stream
        if (torch.cuda.is_available() and hasattr(torch._C, "_cuda_getDevice")
                and hasattr(torch._C, "_cuda_getCurrentRawStream")):
            torch.cuda.init()
            _current_device, _current_raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
        _TYPES = ((torch.float32,), (torch.bfloat16,), (torch.float16,),
                  (torch.float8_e4m3fn, torch.uint8), (torch.float8_e5m2, torch.uint8),
                  (torch.float8_e8m0fnu, torch.uint8))
        P, sz = ctypes.POINTER, ctypes.c_size_t
        for name, args in (
                ("maxdnn_quant8", [P(Quant8Desc)] + [_vp] * 9),
                ("maxdnn_dequant8", [P(Quant8Desc), ctypes.c_int] + [_vp] * 4),
                ("maxdnn_gemm8", [P(Gemm8Desc)] + [_vp] * 6),
                ("maxdnn_layer_norm_fprop", [P(LayerNormDesc)] + [_vp] * 11),
                ("maxdnn_layer_norm_bprop_workspace", [P(LayerNormDesc), P(sz)]),
                ("maxdnn_layer_norm_bprop", [P(LayerNormDesc)] + [_vp] * 10 + [sz, _vp]),
                ("maxdnn_act8_fprop", [P(Act8Desc)] + [_vp] * 7),
                ("maxdnn_act8_bprop", [P(Act8Desc)] + [_vp] * 5)):
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = ctypes.c_int, args
        _plain = _load_plain(lib)
        _lib = lib
    return _lib


def _raise(status, where):
    if status != OK:
        raise MaxdnnError(status, where)


def _mat(t, dtype, rows, cols, ld, what):
    """Address of a [rows][cols] matrix with row pitch ld: a 2-d view with these strides, or any
    contiguous tensor of rows x cols elements where ld = cols."""
    try:
        if (t.is_cuda and t.shape == (rows, cols) and t.stride() == (ld, 1) and t.dtype in _TYPES[dtype]
                and t.get_device() == _current_device()):
            return t.data_ptr()
    except (AttributeError, IndexError):
        pass
    _on_device(t, what)
    if not 0 <= dtype < len(_TYPES) or t.dtype not in _TYPES[dtype]:
        raise TypeError("%s has dtype %s, which is not what the descriptor says" % (what, t.dtype))
    if t.dim() == 2 and t.shape[0] == rows and t.shape[1] == cols:
        if rows and ((cols > 1 and t.stride(1) != 1) or (rows > 1 and cols and t.stride(0) != ld)):
            raise ValueError("%s has strides %s, expected (%d, 1)" % (what, tuple(t.stride()), ld))
    elif t.numel() != rows * cols or not t.is_contiguous() or (ld != cols and rows > 1):
        raise ValueError("%s has shape %s, expected (%d, %d) with row pitch %d" % (what, tuple(t.shape), rows, cols, ld))
    return t.data_ptr()


def _on_device(t, what):
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise TypeError("%s must be a CUDA tensor" % what)
    if t.get_device() != _current_device():
        raise ValueError("%s is not on the current device" % what)


def _vec(t, dtype, n, what):
    """Address of a contiguous tensor of n elements."""
    _on_device(t, what)
    if not 0 <= dtype < len(_TYPES) or t.dtype not in _TYPES[dtype]:
        raise TypeError("%s has dtype %s, which is not what the descriptor says" % (what, t.dtype))
    if t.numel() != n or not t.is_contiguous():
        raise ValueError("%s has shape %s, expected %d contiguous elements" % (what, tuple(t.shape), n))
    return t.data_ptr()


def _blocks(n):
    return -(-n // 128)


def _n_scales(block, rows, cols):
    return (_blocks(cols) * rows, _blocks(rows) * cols, _blocks(rows) * _blocks(cols))[block]


def _scales(t, n, what):
    return _vec(t, DTYPE_E8M0, n, what)


def _stream(stream):
    return _current_raw_stream(_current_device()) if stream is None else stream.cuda_stream


def _pair(pair, dtype, rows, cols, ld, n_scales, what):
    """(values, scales) of a packed result that may not be wanted."""
    if pair is None:
        return None, None
    q, s = pair
    return _mat(q, dtype, rows, cols, ld, what), _scales(s, n_scales, "scales of " + what)


def empty_packed(rows, cols, dtype=DTYPE_E4M3, device="cuda"):
    """An 8-bit matrix whose rows start at multiples of 16 bytes, as a [rows][cols] view."""
    _library()
    wide = torch.empty(rows, _round16(cols), dtype=torch.uint8, device=device)
    return wide.view(_TYPES[dtype][0])[:, :cols]


def empty_scales(block, rows, cols, device="cuda"):
    """Scales of a packed [rows][cols] matrix in their layout for `block`."""
    _library()
    shape = ((_blocks(cols), rows), (_blocks(rows), cols), (_blocks(rows), _blocks(cols)))[block]
    return torch.empty(shape, dtype=torch.uint8, device=device).view(torch.float8_e8m0fnu)


def quant8(desc: Quant8Desc, x, row=None, col=None, tile=None, x_scale=None, stream=None) -> None:
    """maxdnn_quant8: packs x into the forms asked for; row, col, tile: (values, scales)."""
    lib = _library()
    none = (None, None)
    status = _plain.quant8(desc, x, x_scale, *(row or none), *(col or none), *(tile or none),
                           None if stream is None else stream.cuda_stream)
    if status >= 0:
        return _raise(status, "maxdnn_quant8")
    r, c = desc.rows, desc.cols
    px = _mat(x, desc.x_type, r, c, desc.ldx, "x")
    ps = None if desc.x_type < DTYPE_E4M3 else _scales(x_scale, _n_scales(BLOCK_ROW, r, c), "x_scale")
    out = []
    for block, pair, what in ((BLOCK_ROW, row, "row"), (BLOCK_COL, col, "col"), (BLOCK_TILE, tile, "tile")):
        out += _pair(pair, desc.q_type, r, c, desc.ldq, _n_scales(block, r, c), what)
    _raise(lib.maxdnn_quant8(ctypes.byref(desc), px, ps, *out, _stream(stream)), "maxdnn_quant8")


def dequant8(desc: Quant8Desc, q, s, x, block=BLOCK_ROW, stream=None) -> None:
    """maxdnn_dequant8: the values that a packed matrix stands for."""
    lib = _library()
    status = _plain.dequant8(desc, block, q, s, x,
                           None if stream is None else stream.cuda_stream)
    if status >= 0:
        return _raise(status, "maxdnn_dequant8")
    r, c = desc.rows, desc.cols
    _raise(lib.maxdnn_dequant8(
        ctypes.byref(desc), block, _mat(q, desc.q_type, r, c, desc.ldq, "q"),
        _scales(s, _n_scales(block, r, c) if 0 <= block <= 2 else -1, "s"),
        _mat(x, desc.x_type, r, c, desc.ldx, "x"), _stream(stream)), "maxdnn_dequant8")


def _operand(t, s, dtype, major, block, scale_type, mn, k, ld, what):
    rows, cols = (mn, k) if major == MAJOR_K else (k, mn)
    p = _mat(t, dtype, rows, cols, ld, what)
    n = _n_scales(block, rows, cols) if 0 <= block <= 2 else -1
    return p, _vec(s, scale_type, n, "scales of " + what)


def gemm8(desc: Gemm8Desc, a, a_scale, b, b_scale, c, stream=None) -> None:
    """maxdnn_gemm8: C[m, n] = sum_k a[m, k] b[n, k] of packed matrices."""
    lib = _library()
    status = _plain.gemm8(desc, a, a_scale, b, b_scale, c,
                           None if stream is None else stream.cuda_stream)
    if status >= 0:
        return _raise(status, "maxdnn_gemm8")
    M, N, K = desc.M, desc.N, desc.K
    pa, psa = _operand(a, a_scale, desc.a_type, desc.a_major, desc.a_block, desc.a_scale_type, M, K, desc.lda, "a")
    pb, psb = _operand(b, b_scale, desc.b_type, desc.b_major, desc.b_block, desc.b_scale_type, N, K, desc.ldb, "b")
    pc = _mat(c, desc.c_type, M, N, desc.ldc, "c")
    _raise(lib.maxdnn_gemm8(ctypes.byref(desc), pa, psa, pb, psb, pc, _stream(stream)), "maxdnn_gemm8")


def layer_norm_fprop(desc: LayerNormDesc, x, gamma=None, beta=None, y=None, mean=None, rstd=None, packed=None,
                     checkpoint=None, stream=None) -> None:
    """maxdnn_layer_norm_fprop; packed: (q, s) of y, checkpoint: (c, sc) of x."""
    lib = _library()
    none = (None, None)
    status = _plain.layer_norm_fprop(desc, x, gamma, beta, y, mean, rstd, *(packed or none), *(checkpoint or none),
                           None if stream is None else stream.cuda_stream)
    if status >= 0:
        return _raise(status, "maxdnn_layer_norm_fprop")
    r, c = desc.rows, desc.cols
    f32, w, n = DTYPE_F32, desc.w_type, _n_scales(BLOCK_ROW, r, c)
    q, s = _pair(packed, desc.q_type, r, c, desc.ldq, n, "packed")
    k, sk = _pair(checkpoint, desc.q_type, r, c, desc.ldq, n, "checkpoint")
    _raise(lib.maxdnn_layer_norm_fprop(
        ctypes.byref(desc), _mat(x, desc.x_type, r, c, desc.ldx, "x"), None if gamma is None else _vec(gamma, w, c, "gamma"),
        None if beta is None else _vec(beta, w, c, "beta"), None if y is None else _mat(y, desc.y_type, r, c, desc.ldy, "y"),
        None if mean is None else _vec(mean, f32, r, "mean"), None if rstd is None else _vec(rstd, f32, r, "rstd"), q, s, k, sk, _stream(stream)),
        "maxdnn_layer_norm_fprop")


def layer_norm_bprop_workspace(desc: LayerNormDesc) -> int:
    """Bytes of device scratch maxdnn_layer_norm_bprop needs for dgamma and dbeta."""
    n = ctypes.c_size_t()
    _raise(_library().maxdnn_layer_norm_bprop_workspace(ctypes.byref(desc), ctypes.byref(n)),
           "maxdnn_layer_norm_bprop_workspace")
    return int(n.value)


def layer_norm_bprop(desc: LayerNormDesc, dy, x, gamma, mean, rstd, dx, dgamma=None, dbeta=None, workspace=None,
                     x_scale=None, stream=None) -> None:
    """maxdnn_layer_norm_bprop; x: wide, or the checkpoint with its x_scale."""
    lib = _library()
    status = _plain.layer_norm_bprop(desc, dy, x, x_scale, gamma, mean, rstd, dx, dgamma, dbeta, workspace,
                           None if stream is None else stream.cuda_stream)
    if status >= 0:
        return _raise(status, "maxdnn_layer_norm_bprop")
    r, c, f32 = desc.rows, desc.cols, DTYPE_F32
    if workspace is not None:
        _on_device(workspace, "workspace")
        if not workspace.is_contiguous():
            raise TypeError("workspace must be a contiguous CUDA tensor")
    _raise(lib.maxdnn_layer_norm_bprop(
        ctypes.byref(desc), _mat(dy, desc.y_type, r, c, desc.ldy, "dy"), _mat(x, desc.x_type, r, c, desc.ldx, "x"),
        None if desc.x_type < DTYPE_E4M3 else _scales(x_scale, _n_scales(BLOCK_ROW, r, c), "x_scale"),
        None if gamma is None else _vec(gamma, desc.w_type, c, "gamma"), _vec(mean, f32, r, "mean"), _vec(rstd, f32, r, "rstd"),
        _mat(dx, desc.y_type, r, c, desc.ldy, "dx"), None if dgamma is None else _vec(dgamma, f32, c, "dgamma"),
        None if dbeta is None else _vec(dbeta, f32, c, "dbeta"), None if workspace is None else workspace.data_ptr(),
        0 if workspace is None else workspace.numel() * workspace.element_size(), _stream(stream)),
        "maxdnn_layer_norm_bprop")


def act8_fprop(desc: Act8Desc, h, a=None, packed=None, checkpoint=None, stream=None) -> None:
    """maxdnn_act8_fprop; packed: (q, s) of the result, checkpoint: (c, sc) of h."""
    lib = _library()
    none = (None, None)
    status = _plain.act8_fprop(desc, h, a, *(packed or none), *(checkpoint or none),
                           None if stream is None else stream.cuda_stream)
    if status >= 0:
        return _raise(status, "maxdnn_act8_fprop")
    r, c, many = desc.rows, desc.cols, 1 + desc.gated
    n = _n_scales(BLOCK_ROW, r, c)
    q, s = _pair(packed, desc.q_type, r, c, desc.ldq, n, "packed")
    k, sk = _pair(checkpoint, desc.q_type, r, many * c, desc.ldc, many * n, "checkpoint")
    _raise(lib.maxdnn_act8_fprop(
        ctypes.byref(desc), _mat(h, desc.x_type, r, many * c, desc.ldh, "h"),
        None if a is None else _mat(a, desc.x_type, r, c, desc.lda, "a"), q, s, k, sk, _stream(stream)), "maxdnn_act8_fprop")


def act8_bprop(desc: Act8Desc, da, h, dh, h_scale=None, stream=None) -> None:
    """maxdnn_act8_bprop; h: wide, or the checkpoint with its h_scale."""
    lib = _library()
    status = _plain.act8_bprop(desc, da, h, h_scale, dh,
                           None if stream is None else stream.cuda_stream)
    if status >= 0:
        return _raise(status, "maxdnn_act8_bprop")
    r, c, many = desc.rows, desc.cols, 1 + desc.gated
    packed = desc.h_type >= DTYPE_E4M3
    _raise(lib.maxdnn_act8_bprop(
        ctypes.byref(desc), _mat(da, desc.x_type, r, c, desc.lda, "da"),
        _mat(h, desc.h_type, r, many * c, desc.ldc if packed else desc.ldh, "h"),
        _scales(h_scale, many * _n_scales(BLOCK_ROW, r, c), "h_scale") if packed else None,
        _mat(dh, desc.x_type, r, many * c, desc.ldh, "dh"), _stream(stream)), "maxdnn_act8_bprop")
