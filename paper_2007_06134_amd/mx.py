"""Microscaled messages on torch tensors: the ``adpsgd_mx_*`` calls of ``include/adpsgd.h``.

What a worker sends at a synchronization is its difference from the model that
all workers share, in 4 (E2M1) or 8 bits (E4M3) an element, blocks of 32
elements sharing a power of two.  Every function runs on the current stream of
its tensors' device, waits for nothing and can be captured into a graph;
outputs and workspaces that the caller does not pass come from torch's
allocator.

No gradient flows through a call: tensors that require one are refused unless
gradients are switched off (``torch.no_grad()``).  What a call writes then counts
for autograd as torch's own writes do; writes to tensors that require no
gradient are not counted, as those of the engine are not.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from ._native import MX_E2M1, MX_E4M3, _check, adpsgd_mx_rows, lib

BLOCK = 32                                # elements that share a scale
_ROW_BYTES = {MX_E2M1: 16, MX_E4M3: 32}   # of codes, a block

# The smallest calls take a few microseconds on the GPU, so the checks below are
# made of the cheapest queries of a tensor (a device is its index, -1 off the GPU).
_U8, _F32, _F64, _I64 = torch.uint8, torch.float32, torch.float64, torch.int64
_gradients = torch.is_grad_enabled
_current_device = torch._C._cuda_getDevice
_current_stream = torch._C._cuda_getCurrentRawStream


def _run(fn, dev: int, *args) -> None:
    """fn(*args, current stream) of device dev, made the current device for it."""
    if _current_device() == dev:
        rc = fn(*args, _current_stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _current_stream(dev))
    if rc:
        _check(rc)


class MxRows:
    """K rows of P elements: codes [K, >= ceil(P / 32) * 16 (E2M1) or * 32 (E4M3)] and scales
    [K, >= ceil(P / 32)], uint8, rows at strides that are multiples of 16 bytes.  The tensors keep their
    memory for as long as the rows are used: what they hold may be written, they are not resized."""

    __slots__ = ("_codes", "_scales", "_P", "_format", "_K", "_dev", "_c", "_ref")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, P: int, format: int = MX_E2M1):
        per = _ROW_BYTES.get(format)
        if per is None:
            raise ValueError("format must be MX_E2M1 or MX_E4M3")
        if P < 0:
            raise ValueError("P must be >= 0")
        n = -(-P // BLOCK)
        K, code_ld = _bytes(codes, n * per, "codes")
        K2, scale_ld = _bytes(scales, n, "scales")
        dev = codes.get_device()
        if K != K2 or scales.get_device() != dev:
            raise ValueError("codes and scales must have one row a worker on one device")
        if not 1 <= K <= 65536:
            raise ValueError("there must be 1 to 65536 rows")
        _check_size(K, P)
        self._codes, self._scales, self._P, self._format, self._K, self._dev = codes, scales, P, format, K, dev
        self._c = adpsgd_mx_rows(codes.data_ptr(), scales.data_ptr(), code_ld, scale_ld, P, K, format)
        self._ref = C.byref(self._c)

    @classmethod
    def empty(cls, K: int, P: int, format: int = MX_E2M1, device="cuda") -> "MxRows":
        """Rows to be written, at adpsgd_mx_code_stride and adpsgd_mx_scale_stride."""
        if format not in _ROW_BYTES:
            raise ValueError("format must be MX_E2M1 or MX_E4M3")
        if not 1 <= K <= 65536 or P < 0:
            raise ValueError("K must be in [1, 65536] and P >= 0")
        _check_size(K, P)
        return cls(torch.empty((K, lib.adpsgd_mx_code_stride(format, P)), dtype=_U8, device=device),
                   torch.empty((K, lib.adpsgd_mx_scale_stride(P)), dtype=_U8, device=device), P, format)

    codes = property(lambda self: self._codes)
    scales = property(lambda self: self._scales)
    K = property(lambda self: self._K)
    P = property(lambda self: self._P)
    format = property(lambda self: self._format)
    device = property(lambda self: self._codes.device)


def _check_size(K: int, P: int) -> None:
    """The library's limits, before memory of that size is asked for."""
    if P > 1 << 34 or (P + 255 >> 8) * K >= 1 << 31:
        raise ValueError("P must be at most 2^34 and K * P below 2^39")


def _bytes(t: torch.Tensor, need: int, name: str) -> Tuple[int, int]:
    """Rows of a byte matrix and their distance; of a single row or empty ones, whose stride means
    nothing, their length in whole units of 16."""
    if t.dtype is not _U8 or t.dim() != 2 or t.get_device() < 0:
        raise ValueError(f"{name} must be a uint8 matrix on a GPU")
    K, w = t.shape
    if w < need or (w > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must have rows of at least {need} contiguous bytes")
    return K, t.stride(0) if K > 1 and w > 0 else -(-w // 16) * 16


def _no_grad(name: str) -> None:
    if _gradients():
        raise ValueError(f"{name} requires a gradient, and none flows through this call: use torch.no_grad() or detach()")


def _matrix(t: torch.Tensor, K: int, P: int, dev: int, name: str) -> int:
    """Row stride of a float32 [K, P] tensor."""
    if t.dtype is not _F32 or t.shape != (K, P) or t.get_device() != dev:
        raise ValueError(f"{name} must be float32 [{K}, {P}] on device {dev}")
    if t.requires_grad:
        _no_grad(name)
    return _row_stride(t, K, P, name)


def _row_stride(t: torch.Tensor, K: int, P: int, name: str) -> int:
    ld, one = t.stride()
    if one != 1 and P > 1:
        raise ValueError(f"{name} must have contiguous rows")
    if K == 1:
        return P
    if ld < P:
        raise ValueError(f"{name} must have rows that do not overlap")
    return ld


def _vector(t: Optional[torch.Tensor], P: int, dev: int, name: str) -> Optional[int]:
    if t is None:
        return None
    if t.dtype is not _F32 or t.dim() != 1 or t.numel() != P or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous float32 [{P}] on device {dev}")
    if t.requires_grad:
        _no_grad(name)
    return t.data_ptr()


def _written(*tensors: Optional[torch.Tensor]) -> None:
    """Of a call without gradients (with them it takes no tensor that this is for)."""
    for t in tensors:
        if t is not None and t.requires_grad:
            torch.autograd.graph.increment_version(t)


def _offsets(t: torch.Tensor, dev: int) -> int:
    if t.dtype is not _I64 or t.dim() != 1 or t.shape[0] < 2 or t.get_device() != dev or t.stride(0) != 1:
        raise ValueError(f"offsets must be contiguous int64 [T + 1] on device {dev}")
    return t.shape[0] - 1


def mx_quantize(x: torch.Tensor, base: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, *,
                format: Optional[int] = None, residual_out: Optional[torch.Tensor] = None,
                out: Optional[MxRows] = None) -> MxRows:
    """The messages of the K workers whose parameters are x [K, P]: (x - base) + residual in `format`.

    base [P] and residual [K, P] count as zero where they are None.  What the message leaves out is
    written to residual_out, by default to residual itself, and not kept where both are None.
    out: rows to write (their format is the one used)."""
    dev = x.get_device()
    if x.dtype is not _F32 or x.dim() != 2 or dev < 0:
        raise ValueError("x must be a float32 matrix on a GPU")
    if x.requires_grad:
        _no_grad("x")
    K, P = x.shape
    x_ld = _row_stride(x, K, P, "x")
    base_ptr = _vector(base, P, dev, "base")
    r_in = r_out = None
    r_ld = 0
    if residual is not None:
        r_ld, r_in = _matrix(residual, K, P, dev, "residual"), residual.data_ptr()
        if residual_out is None:
            r_out = r_in
    if residual_out is not None:
        ld, r_out = _matrix(residual_out, K, P, dev, "residual_out"), residual_out.data_ptr()
        if residual is not None and ld != r_ld:
            raise ValueError("residual and residual_out must have the same row stride")
        r_ld = ld
    if out is None:
        out = MxRows.empty(K, P, MX_E2M1 if format is None else format, x.device)
    elif out._K != K or out._P != P or out._dev != dev or (format is not None and format != out._format):
        raise ValueError(f"out must be rows of the format for [{K}, {P}] on device {dev}")
    _run(lib.adpsgd_mx_quantize, dev, out._ref, x.data_ptr(), x_ld, base_ptr, r_in, r_out, r_ld)
    if not _gradients():
        _written(residual if residual_out is None else residual_out)
    return out


def mx_dequantize(rows: MxRows, base: Optional[torch.Tensor] = None, *,
                  out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """What the rows say: base + their values, float32 [K, P]."""
    dev = rows._dev
    base_ptr = _vector(base, rows._P, dev, "base")
    if out is None:
        out = torch.empty((rows._K, rows._P), dtype=_F32, device=rows._codes.device)
    ld = _matrix(out, rows._K, rows._P, dev, "out")
    _run(lib.adpsgd_mx_dequantize, dev, rows._ref, base_ptr, out.data_ptr(), ld)
    if not _gradients():
        _written(out)
    return out


# A call's output of sums, its workspace and the workspace's bytes: for T tensors, where the offsets are.  The
# engine makes them before it sends anything and hands them to the call (_buffers).
def average_buffers(rows: MxRows, T: int, offsets: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor, int]:
    need = lib.adpsgd_mx_average_workspace(rows._K, rows._P, T)
    return offsets.new_empty(T, dtype=_F64), offsets.new_empty(need + 7 >> 3), need


def product_buffers(a: MxRows, T: int, offsets: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor, int]:
    need = lib.adpsgd_mx_product_workspace(a._K, a._P, T)
    return offsets.new_empty((T, a._K, a._K), dtype=_F32), offsets.new_empty(need + 7 >> 3), need


def mx_average(rows: MxRows, offsets: torch.Tensor, base: Optional[torch.Tensor] = None, *,
               x: Optional[torch.Tensor] = None, base_out: Optional[torch.Tensor] = None,
               _buffers: Optional[tuple] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The synchronization: (base + the rows' mean, float32 [P]; every tensor's variance, float64 [T]).

    offsets: int64 [T + 1] on the device, the tensors' boundaries as for ``Adpsgd`` (0 first, P last;
    the values are not checked).  The new model is also written to every row of x [K, P] where that is
    given, and to base_out (which may be base; a new tensor by default)."""
    dev, K, P = rows._dev, rows._K, rows._P
    T = _offsets(offsets, dev)
    base_ptr = _vector(base, P, dev, "base")
    x_ptr, x_ld = None, 0
    if x is not None:
        x_ld, x_ptr = _matrix(x, K, P, dev, "x"), x.data_ptr()
    if base_out is None:
        base_out = torch.empty((P,), dtype=_F32, device=rows._codes.device)
    out_ptr = _vector(base_out, P, dev, "base_out")
    var, work, need = _buffers or average_buffers(rows, T, offsets)
    _run(lib.adpsgd_mx_average, dev, rows._ref, T, offsets.data_ptr(), base_ptr, out_ptr, x_ptr, x_ld, var.data_ptr(),
         work.data_ptr(), need)
    if not _gradients():
        _written(x, base_out)
    return base_out, var


def mx_product(a: MxRows, offsets: torch.Tensor, b: Optional[MxRows] = None, *,
               _buffers: Optional[tuple] = None) -> torch.Tensor:
    """Inner products of the rows of a with those of b (of a, where b is None) for every tensor:
    float32 [T, K, K].  K is at most 256; a and b have the same format, K and P."""
    dev, K = a._dev, a._K
    T = _offsets(offsets, dev)
    if b is not None and b._dev != dev:
        raise ValueError("a and b must be on one device")
    if K > 256 or (b is not None and (b._format != a._format or b._K != K or b._P != a._P)):
        # (the library says why, before any memory is taken)
        _run(lib.adpsgd_mx_product, dev, a._ref, None if b is None else b._ref, T, offsets.data_ptr(), None, None, 0)
    out, work, need = _buffers or product_buffers(a, T, offsets)
    _run(lib.adpsgd_mx_product, dev, a._ref, None if b is None else b._ref, T, offsets.data_ptr(), out.data_ptr(),
         work.data_ptr(), need)
    return out
