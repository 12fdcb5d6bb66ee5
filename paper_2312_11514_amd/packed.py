"""Norms with the residual's addition, and projections with weights in 4 bits: ctypes binding of lif_add_norm and the lif_packed calls of
include/lif.h, argument marshalling only.

    qkv = PackedLinear(n_out=6144, n_in=4096, group=128)
    qkv.quantize(weight)                                  # once; or qkv.pack(codes, scales), from a checkpoint in 4 bits
    add_norm(y, normed, residual=x, total=x, weight=w)    # x += y, normed = norm(x)
    qkv.multiply(normed, out)

    codes, scales = torch.empty(rows, 4096, dtype=torch.int8, device="cuda"), torch.empty(rows, 1, device="cuda")
    add_norm(y, codes, residual=x, total=x, weight=w, scales=scales)          # the same in 8 bits
    qkv.multiply(codes, out, scales=scales)
"""
from __future__ import annotations

import ctypes as C
import struct

from . import binding as _b
from .binding import LIF_INVALID_ARG, LifError

# lif_norm_rows and lif_packed_rows, filled in one go; the bytes themselves are the argument, so that threads share none
_NORM, _PRODUCT, _CONFIG = struct.Struct("@7P4q5if"), struct.Struct("@4P2q2i"), struct.Struct("@5i")
assert _NORM.size == C.sizeof(_b.LifNormRows) and _PRODUCT.size == C.sizeof(_b.LifPackedRows) and _CONFIG.size == C.sizeof(_b.LifPackedConfig)


def _refuse(message):
    raise LifError(LIF_INVALID_ARG, message)


class _Torch:
    """What the calls need of torch again and again (imported with the first of them)."""
    ready = False

    @classmethod
    def bind(cls):
        import torch
        lib = _b.load_library()
        cls.int8, cls.float32, cls.uint8 = torch.int8, torch.float32, torch.uint8
        cls.codes = {torch.float32: _b.LIF_F32, torch.float16: _b.LIF_F16, torch.bfloat16: _b.LIF_BF16}
        cls.types = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
        cls.device = staticmethod(getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device)
        cls.add_norm, cls.multiply = lib.lif_add_norm, lib.lif_packed_multiply
        cls.ready = True


def _stride(t, what):
    """Elements between the rows of [..., width]."""
    if t.is_contiguous():
        return t.shape[-1]
    shape, strides = t.shape, t.stride()
    if strides[-1] == 1:
        stride = None
        for n, s in zip(reversed(shape[:-1]), reversed(strides[:-1])):
            if n == 1:
                continue
            if stride is None:
                stride, below = s, n * s
            elif s != below:
                break
            else:
                below = n * s
        else:
            return shape[-1] if stride is None else stride
    _refuse(f"{what} must have its elements one after the other and its rows at one stride")


def _like(t, shape, dtype, device, what):
    """The stride of rows that have to be as others are."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device:
        _refuse(f"{what} must be {list(shape)} of {dtype} beside the rows")
    return shape[-1] if t.is_contiguous() else _stride(t, what)


def _floats(t, n, device, what):
    if t.dtype is not _Torch.float32 or t.numel() != n or t.get_device() != device or not t.is_contiguous():
        _refuse(f"{what} must be a contiguous float32 tensor of {n} elements beside the rows")
    return t.data_ptr()


def add_norm(x, out, *, norm=_b.NORM_RMS, eps=1e-5, weight=None, bias=None, residual=None, total=None, scales=None, group=0):
    """lif_add_norm: h = residual + x, total = h, out = norm(h).

    x, residual, total, out [..., width] of one type (float32, float16 or bfloat16), rows at one stride; total and out may be x or the residual.
    With scales (float32, [rows] or, with a group of 32, 64 or 128, [rows, ceil(width / group)]) out is int8.  weight, bias: float32 [width] or None."""
    if not _Torch.ready:
        _Torch.bind()
    dtype, shape, device = x.dtype, x.shape, x.get_device()
    code = _Torch.codes.get(dtype)
    if code is None or not shape:
        _refuse("x must be float32, float16 or bfloat16 rows")
    if device < 0 or device != _Torch.device():
        _refuse("x must be on the current GPU")
    width = shape[-1]
    rows = x.numel() // width if width else 0
    r_ptr = r_stride = t_ptr = t_stride = s_ptr = 0
    if scales is None:
        out_stride = _like(out, shape, dtype, device, "out")
    else:
        if group not in (0, 32, 64, 128):
            _refuse("group must be 0, 32, 64 or 128")
        out_stride = _like(out, shape, _Torch.int8, device, "out")
        s_ptr = _floats(scales, rows * (-(-width // group) if group else 1), device, "scales")
    if residual is not None:
        r_ptr, r_stride = residual.data_ptr(), _like(residual, shape, dtype, device, "residual")
    if total is not None:
        t_ptr, t_stride = total.data_ptr(), _like(total, shape, dtype, device, "total")
    w_ptr, b_ptr = _floats(weight, width, device, "weight") if weight is not None else 0, _floats(bias, width, device, "bias") if bias is not None else 0
    try:
        args = _NORM.pack(x.data_ptr(), r_ptr, t_ptr, out.data_ptr(), s_ptr, w_ptr, b_ptr, _stride(x, "x"), r_stride, t_stride, out_stride, rows, width, code,
                          norm, group, eps)
    except (struct.error, OverflowError) as e:
        _refuse(f"the number of rows, norm, group or eps: {e}")
    rc = _Torch.add_norm(args, _b._stream())
    if rc:
        _b._check(rc)


class PackedLinear:
    """A matrix [n_out, n_in] in 4 bits behind the C ABI, a scale (and with zeros=True a zero point) for every `group` inputs.  Owns (through torch)
    the codes and the words of the groups.  All calls enqueue on torch's current stream and return immediately; multiply() and dequantize() may run on
    several streams at once."""

    def __init__(self, n_out, n_in, *, group=128, zeros=False, dtype="f16", device="cuda"):
        import torch
        self.lib = _b.load_library()
        if not _Torch.ready:
            _Torch.bind()
        if dtype not in _Torch.types:
            _refuse("dtype must be f32, f16 or bf16")
        self.tdtype = _Torch.types[dtype]
        try:                                               # (ctypes takes numbers of more bits for others)
            self.cfg = _b.LifPackedConfig.from_buffer_copy(_CONFIG.pack(n_out, n_in, group, int(bool(zeros)), _Torch.codes[self.tdtype]))
        except struct.error as e:
            _refuse(f"configuration: {e}")
        code_bytes, group_bytes = self.lib.lif_packed_code_bytes(C.byref(self.cfg)), self.lib.lif_packed_group_bytes(C.byref(self.cfg))
        if code_bytes == 0:
            _refuse("configuration rejected by lif_packed_code_bytes")
        self.n_out, self.n_in, self.group, self.row_groups = n_out, n_in, group, -(-n_in // group)
        self.codes = torch.empty(code_bytes, dtype=torch.uint8, device=device)
        self.groups = torch.empty(group_bytes // 4, dtype=torch.int32, device=device)
        self.buf = _b.LifPackedBuffers(self.codes.data_ptr(), self.groups.data_ptr(), code_bytes, group_bytes)
        h = C.c_void_p()
        _b._check(self.lib.lif_packed_create(C.byref(self.cfg), C.byref(self.buf), C.byref(h)))
        self.handle = h
        self._gpu = self.codes.get_device()

    def close(self):
        if getattr(self, "handle", None):
            self.lib.lif_packed_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _here(self):
        if self._gpu < 0 or self._gpu != _Torch.device():
            _refuse("the weights must be on the current GPU")

    def _full(self, weight):
        self._here()
        if weight.dtype is not self.tdtype or weight.shape != (self.n_out, self.n_in) or weight.get_device() != self._gpu:
            _refuse(f"weight must be [{self.n_out}, {self.n_in}] of the matrix's type beside it")
        return weight.data_ptr(), _stride(weight, "weight")

    def quantize(self, weight):
        """lif_packed_quantize: from full weights [n_out, n_in]."""
        ptr, stride = self._full(weight)
        _b._check(self.lib.lif_packed_quantize(self.handle, ptr, stride, _b._stream()))

    def pack(self, codes, scales, zeros=None):
        """lif_packed_pack: from uint8 [n_out, n_in / 2], two codes in a byte, the lower input in the lower half; float32 [n_out, groups of a row]; uint8
        [n_out, groups of a row] if the matrix has zero points."""
        self._here()
        for t, dtype, columns, what in ((codes, _Torch.uint8, self.n_in // 2, "codes"), (scales, _Torch.float32, self.row_groups, "scales"),
                                        (zeros, _Torch.uint8, self.row_groups, "zeros")):
            if t is None and what != "zeros":
                _refuse(f"{what} must be given")
            if t is not None and (t.dtype is not dtype or t.shape != (self.n_out, columns) or t.get_device() != self._gpu or not t.is_contiguous()):
                _refuse(f"{what} must be a contiguous {dtype} tensor [{self.n_out}, {columns}] beside the matrix")
        _b._check(self.lib.lif_packed_pack(self.handle, codes.data_ptr(), scales.data_ptr(), _b._ptr(zeros), _b._stream()))

    def dequantize(self, out):
        """lif_packed_dequantize: what the weights stand for, into out [n_out, n_in]."""
        ptr, stride = self._full(out)
        _b._check(self.lib.lif_packed_dequantize(self.handle, ptr, stride, _b._stream()))

    def multiply(self, x, out, bias=None, scales=None):
        """lif_packed_multiply: out [..., n_out] = x [..., n_in] times the matrix (+ bias, float32 [n_out]).  x is of the matrix's type, or int8 with scales,
        float32, [rows] or [rows, groups of a row]."""
        shape, device, dtype, n_in = x.shape, self._gpu, self.tdtype, self.n_in
        if device < 0 or device != _Torch.device():
            _refuse("the weights must be on the current GPU")
        if not shape or shape[-1] != n_in or x.dtype is not (dtype if scales is None else _Torch.int8) or x.get_device() != device:
            _refuse(f"x must be [..., {n_in}] of the matrix's type (int8 if there are scales) beside it")
        rows = x.numel() // n_in
        s_ptr = x_group = 0
        if scales is not None:
            groups = self.row_groups
            if groups > 1 and scales.numel() != rows:
                x_group, s_ptr = self.group, _floats(scales, rows * groups, device, "scales")
            else:
                s_ptr = _floats(scales, rows, device, "scales")
        b_ptr, out_stride = _floats(bias, self.n_out, device, "bias") if bias is not None else 0, _like(out, (*shape[:-1], self.n_out), dtype, device, "out")
        try:
            args = _PRODUCT.pack(x.data_ptr(), s_ptr, b_ptr, out.data_ptr(), _stride(x, "x"), out_stride, rows, x_group)
        except struct.error as e:
            _refuse(f"the number of rows: {e}")
        rc = _Torch.multiply(self.handle, args, _b._stream())
        if rc:
            _b._check(rc)
