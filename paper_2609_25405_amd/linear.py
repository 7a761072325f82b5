"""A layer's norms and products as operators on torch tensors: RMS norm with the residual's addition,
products with bias, activation and residual, the same for ragged groups of rows, and the 8-bit blocks
that they read and write.

Marshalling around include/orthrus/linear.h; the arithmetic runs in liborthrus.so, on torch's current stream
unless ``stream`` names another.  Tensors live on the current device.
"""
from __future__ import annotations

import struct
from ctypes import byref
from typing import Optional, Union

import torch

from . import _abi as A
from . import _abi_linear as L
from .ops import _check, _need, _room, _stream

BLOCK = L.ORTHRUS_MX8_BLOCK
_pack = struct.Struct("=QQqqi4x").pack          # an orthrus_matrix (a ctypes struct takes three times as long to make)
_DTYPES = {torch.float32: A.ORTHRUS_F32, torch.bfloat16: A.ORTHRUS_BF16}
_ACTS = {None: L.ORTHRUS_ACT_NONE, "relu": L.ORTHRUS_ACT_RELU, "silu": L.ORTHRUS_ACT_SILU, "gelu": L.ORTHRUS_ACT_GELU,
         "gelu_tanh": L.ORTHRUS_ACT_GELU_TANH}


def _up(n: int, to: int) -> int:
    return -(-n // to) * to


class Mx8:
    """Rows in 8-bit blocks: e4m3 ``codes`` [rows][width] and one e8m0 scale for each 32 consecutive
    elements of a row, ``scales`` [rows][ceil(width / 32)].  Elements of a row lie side by side; rows may be apart."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor):
        _need(codes.dtype == torch.float8_e4m3fn and codes.dim() == 2, "codes")
        rows, width = codes.shape
        _need(scales.dtype == torch.float8_e8m0fnu and scales.shape == (rows, -(-width // BLOCK)), "scales")
        self._tensors, self._shape = (codes, scales), codes.shape
        self._device = codes.get_device()
        _need(scales.get_device() == self._device, "codes and scales on one device")
        at, scales_at, stride, scale_stride = codes.data_ptr(), scales.data_ptr(), _row_stride(codes, "codes"), _row_stride(scales, "scales")
        self._ref = _pack(at, scales_at, stride, scale_stride, L.ORTHRUS_MX8)
        self._aligned = (at | stride) % 16 == 0 and (scales_at | scale_stride) % 4 == 0

    @classmethod
    def empty(cls, rows: int, width: int, device="cuda") -> "Mx8":
        """Room for rows that the products can read: codes 16 and scales 4 bytes aligned."""
        codes = torch.empty((rows, _up(width, 16)), dtype=torch.float8_e4m3fn, device=device)
        scales = torch.empty((rows, _up(-(-width // BLOCK), 4)), dtype=torch.float8_e8m0fnu, device=device)
        return cls(codes[:, :width], scales[:, :-(-width // BLOCK)])

    @classmethod
    def of(cls, codes: torch.Tensor, scales: torch.Tensor) -> "Mx8":
        """A copy of codes and scale bytes (uint8 or e8m0) that the products can read."""
        m = cls.empty(*codes.shape, device=codes.device)
        m.codes.view(torch.uint8).copy_(codes.view(torch.uint8))
        m.scales.view(torch.uint8).copy_(scales.view(torch.uint8))
        return m

    # the tensors stay the ones the rows were made of
    codes = property(lambda self: self._tensors[0])
    scales = property(lambda self: self._tensors[1])
    shape = property(lambda self: self._shape)

    def get_device(self) -> int:
        return self._device


Rows = Union[torch.Tensor, Mx8]


def _aligned(t: torch.Tensor, to: int) -> torch.Tensor:
    es = t.element_size()
    if t.stride(1) == 1 and t.data_ptr() % to == 0 and (t.shape[0] < 2 or t.stride(0) * es % to == 0):
        return t
    room = torch.empty((t.shape[0], _up(t.shape[1] * es, to) // es), dtype=t.dtype, device=t.device)[:, :t.shape[1]]
    if es == 1:
        room.view(torch.uint8).copy_(t.view(torch.uint8))
    else:
        room.copy_(t)
    return room


def aligned(t: Rows) -> Rows:
    """``t`` [rows][k] if its rows begin where the products read them, at multiples of 16 bytes (scales of 8-bit blocks: of 4), else
    with a copy, on the current stream, of what does not."""
    if t.__class__ is not Mx8:
        return _aligned(t, 16)
    return t if t._aligned else Mx8(_aligned(t.codes, 16), _aligned(t.scales, 4))


def _row_stride(t: torch.Tensor, what: str) -> int:
    rows, width = t.shape
    stride, inner = t.stride()
    if (inner != 1 and width > 1) or (rows > 1 and stride < width):
        raise A.OrthrusError(A.ORTHRUS_EINVAL, what + " strides")
    return stride if rows > 1 else _up(width, 16)          # (one row's stride is nobody's)


# A call costs the host about as much as a small launch costs the device: few and cheap checks, and no more calls than they need.
_OTHER_DEVICE = "tensor on another device than the current one"
_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
_BF16, _F32 = torch.bfloat16, torch.float32
_lib = None


def _load():
    global _lib
    _lib = L.load()
    return _lib


def _here(dev: int, *others) -> None:
    """The tensors of a call belong to the current device, whose stream is the default one."""
    if dev < 0 or dev != _device():
        raise A.OrthrusError(A.ORTHRUS_EINVAL, _OTHER_DEVICE)
    for t in others:
        if t is not None and t.get_device() != dev:
            raise A.OrthrusError(A.ORTHRUS_EINVAL, _OTHER_DEVICE)


def _ref(t: Optional[Rows], shape, dev: int, what: str):
    """t [rows][width] on device `dev` as the argument of a call."""
    if t is None:
        return None
    if t.shape != shape:
        raise A.OrthrusError(A.ORTHRUS_EINVAL, what + " shape")
    if t.__class__ is Mx8:
        if t._device != dev:
            raise A.OrthrusError(A.ORTHRUS_EINVAL, _OTHER_DEVICE)
        return t._ref
    if t.get_device() != dev:
        raise A.OrthrusError(A.ORTHRUS_EINVAL, _OTHER_DEVICE)
    stride, inner = t.stride()
    if inner != 1 or shape[0] < 2 or stride < shape[1]:
        stride = _row_stride(t, what)
    dtype = t.dtype
    if dtype is _BF16:
        return _pack(t.data_ptr(), 0, stride, 0, 1)
    if dtype is _F32:
        return _pack(t.data_ptr(), 0, stride, 0, 0)
    raise A.OrthrusError(A.ORTHRUS_EUNSUPPORTED, what + " dtype")


def _shape2(t: Rows, what: str):
    shape = t.shape
    if len(shape) != 2:
        raise A.OrthrusError(A.ORTHRUS_EINVAL, what + " shape")
    return shape


def convert(x: Rows, y: Rows, stream: Optional[int] = None) -> None:
    """y = x in y's type: fp32 or bf16 rows to 8-bit blocks, or back (rounded; what fp32 or bf16
    rows became is exact in either)."""
    shape = _shape2(x, "x")
    dev = x.get_device()
    _here(dev)
    rc = (_lib or _load()).orthrus_convert(_ref(x, shape, dev, "x"), _ref(y, shape, dev, "y"), *shape,
                                           _raw_stream(dev) if stream is None else stream)
    if rc:
        raise A.OrthrusError(rc, "orthrus_convert")


def norm(x: torch.Tensor, y: Rows, gain: Optional[torch.Tensor] = None, eps: float = 1e-5, add: Optional[torch.Tensor] = None,
         total: Optional[torch.Tensor] = None, stream: Optional[int] = None) -> None:
    """RMS norm of the rows of s = x + add: y = s * gain / sqrt(mean(s^2) + eps), and total = s if given.  total or y
    may be x or add; nothing else that is written may share memory with another argument."""
    shape = _shape2(x, "x")
    dev = x.get_device()
    _here(dev, gain)
    at = None
    if gain is not None:
        if gain.dtype is not _F32 or gain.numel() != shape[1] or not gain.is_contiguous():
            raise A.OrthrusError(A.ORTHRUS_EINVAL, "gain")
        at = gain.data_ptr()
    rc = (_lib or _load()).orthrus_norm(_ref(x, shape, dev, "x"), _ref(add, shape, dev, "add"), _ref(total, shape, dev, "total"), at, eps,
                                        _ref(y, shape, dev, "y"), *shape, _raw_stream(dev) if stream is None else stream)
    if rc:
        raise A.OrthrusError(rc, "orthrus_norm")


def _lend(t: torch.Tensor, stream: Optional[int], dev: int) -> None:
    """Makes memory just taken on the current stream safe to write on another: what used it before may still be queued, and it is
    not given to others before the other stream is done with it."""
    if stream is None or stream == _raw_stream(dev):
        return
    other = torch.cuda.ExternalStream(stream, device=dev) if stream else torch.cuda.default_stream(dev)
    other.wait_stream(torch.cuda.current_stream(dev))
    t.record_stream(other)


class LinearWeights:
    """Weights in the layout that the products read, packed once from ``matrix`` [groups n][k] (bf16 tensor
    or Mx8), or, with ``up`` of the same shape and type, from a pair: y = act(x matrix^T) * (x up^T)."""

    def __init__(self, matrix: Rows, up: Optional[Rows] = None, groups: int = 1, stream: Optional[int] = None):
        all_rows, k = shape = _shape2(matrix, "matrix")
        _need(groups > 0 and all_rows % groups == 0, "groups")
        dev = matrix.get_device()
        _here(dev)
        m, second = _ref(matrix, shape, dev, "matrix"), _ref(up, shape, dev, "up")
        dtype = L.ORTHRUS_MX8 if isinstance(matrix, Mx8) else _DTYPES[matrix.dtype]
        self._struct = L.orthrus_linear_weights(None, dtype, all_rows // groups, k, int(up is not None), groups)
        nbytes = int(L.load().orthrus_linear_packed_bytes(byref(self._struct)))
        if nbytes == 0:
            raise A.OrthrusError(A.ORTHRUS_EUNSUPPORTED if dtype == A.ORTHRUS_F32 else A.ORTHRUS_EINVAL, "orthrus_linear_packed_bytes")
        self._packed = torch.empty(nbytes, dtype=torch.uint8, device=f"cuda:{dev}")
        self._struct.packed = self._packed.data_ptr()
        self._ref = byref(self._struct)
        self._sizes = (all_rows // groups, k, groups, up is not None)
        self._device = dev
        _lend(self._packed, stream, dev)
        _check(L.load().orthrus_linear_pack(self._ref, m, second, _stream(stream, dev)), "orthrus_linear_pack")

    # bytes and sizes stay the ones that were packed
    packed = property(lambda self: self._packed)
    n = property(lambda self: self._sizes[0])
    k = property(lambda self: self._sizes[1])
    groups = property(lambda self: self._sizes[2])
    gated = property(lambda self: self._sizes[3])

    def get_device(self) -> int:
        return self._device


def linear_workspace(w: LinearWeights, rows: int, device="cuda") -> Optional[torch.Tensor]:
    """The workspace of products of up to ``rows`` rows (None where they need none)."""
    n = int(L.load().orthrus_linear_bytes(w._ref, rows))
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _product(w, x, offsets, y, bias, act, residual, workspace, stream):
    shape = _shape2(x, "x")
    rows = shape[0]
    n, k, groups, gated = w._sizes
    if shape[1] != k:
        raise A.OrthrusError(A.ORTHRUS_EINVAL, "x width")
    ws, ws_bytes = _room(workspace)
    dev = x.get_device()
    _here(dev, w, offsets, bias, workspace)
    out = (rows, n)
    e = None
    if bias is not None or act is not None or residual is not None:
        e = L.orthrus_epilogue()
        if act not in _ACTS:
            raise A.OrthrusError(A.ORTHRUS_EINVAL, "act")
        e.act = _ACTS[act]
        if bias is not None:
            _need(bias.dtype == torch.float32 and bias.numel() == groups * (2 if gated else 1) * n and bias.shape[-1] == n and
                  bias.is_contiguous(), "bias")
            e.bias = bias.data_ptr()
        if residual is not None:
            e.residual = L.orthrus_matrix.from_buffer_copy(_ref(residual, out, dev, "residual"))
        e = byref(e)
    lib, stream = _lib or _load(), _raw_stream(dev) if stream is None else stream
    at, to = _ref(x, shape, dev, "x"), _ref(y, out, dev, "y")
    if offsets is None:
        rc = lib.orthrus_linear(w._ref, at, rows, e, to, ws, ws_bytes, stream)
    else:
        rc = lib.orthrus_linear_grouped(w._ref, at, offsets.data_ptr(), rows, e, to, ws, ws_bytes, stream)
    if rc:
        raise A.OrthrusError(rc, "orthrus_linear" if offsets is None else "orthrus_linear_grouped")


def linear(w: LinearWeights, x: Rows, y: Rows, bias: Optional[torch.Tensor] = None, act: Optional[str] = None,
           residual: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream: Optional[int] = None) -> None:
    """y = act(x W^T + bias) + residual, or for pairs of weights act(x W^T + bias) * (x U^T + bias_u) + residual.  x [rows][k] of
    the weights' type, rows 16 bytes aligned (`aligned`, `Mx8.empty`); y [rows][n] fp32, bf16 or Mx8; bias fp32 [n], pairs [2][n];
    act None, relu, silu, gelu or gelu_tanh; residual fp32 or bf16 [rows][n], which may be y; workspace: linear_workspace."""
    _product(w, x, None, y, bias, act, residual, workspace, stream)


def linear_grouped(w: LinearWeights, x: Rows, offsets: torch.Tensor, y: Rows, bias: Optional[torch.Tensor] = None, act: Optional[str] = None,
                   residual: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream: Optional[int] = None) -> None:
    """`linear` of groups of rows: row r of [offsets[g], offsets[g + 1]) through the weights and bias ([groups][n], pairs
    [groups][2][n]) of group g.  offsets: int32 [groups + 1] on the device, ascending.  Rows of y outside all groups are left as they
    were."""
    _need(offsets.dtype == torch.int32 and offsets.shape == (w._sizes[2] + 1,) and offsets.is_contiguous(), "offsets")
    _product(w, x, offsets, y, bias, act, residual, workspace, stream)
