"""8-bit rows and matrices on a GPU: e4m3 elements with a power-of-two scale for
each block of 128 (include/moeca.h states the stored form).

``QuantRows`` are rows that are quantised as they are written into slots and
read back by slot; ``QuantMatrix`` holds one weight matrix, or a stack of them,
with a scale per 128 x 128 block; ``linear`` multiplies rows with a matrix.
torch provides device memory and the stream; the arithmetic runs in the
library's kernels.  Calls run on their tensors' device, on its current stream
unless one is given, to which a tensor that such a call makes then belongs.
"""
from __future__ import annotations

import torch

from . import _lib

_BF16, _FP32 = torch.bfloat16, torch.float32
_CODE = {_BF16: _lib.MOECA_DTYPE_BF16, _FP32: _lib.MOECA_DTYPE_FP32}


def _dtype(t):
    code = _CODE.get(t.dtype)
    if code is None:
        raise TypeError(f"rows are bfloat16 or float32, not {t.dtype}")
    return code


def _launch(fn, device, stream, *args):
    """Call ``fn(*args, stream)`` of the library with the device current.  (A call of
    a few microseconds: the guard is entered only where another device is current,
    and the current stream's handle is asked for without making an object of it.)"""
    index = device.index
    if index is None or device.type != "cuda":
        raise ValueError(f"the tensors are on {device}, not on a GPU")
    if stream is not None and stream.device != device:
        raise ValueError(f"the stream is one of {stream.device}, the tensors are on {device}")
    raw = torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream
    if torch.cuda.current_device() == index:
        rc = fn(*args, raw)
    else:
        with torch.cuda.device(index):
            rc = fn(*args, raw)
    if rc != _lib.MOECA_OK:
        _lib._check(rc)


def _empty(shape, dtype, device, stream):
    """A new tensor that belongs to the call's stream: one of the current stream could
    still be in use there when a call on another writes it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _rows(t, width, device, what):
    """(pointer, rows, row stride) of a 2-d tensor of the activation type."""
    shape = t.shape
    if len(shape) != 2 or shape[1] != width:
        raise ValueError(f"{what}: expected rows of width {width}, got {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, expected {device}")
    rows = shape[0]
    ld, inner = t.stride()
    if rows > 0 and width > 1 and inner != 1:
        raise ValueError(f"{what}: the elements of a row must be contiguous")
    if rows <= 1:
        ld = width
    if ld < width:
        raise ValueError(f"{what}: rows overlap (stride {ld}, width {width})")
    return t.data_ptr() or None, rows, ld


def _indexes(slot, rows, device):
    if slot is None:
        return None
    if slot.dtype != torch.int32 or slot.dim() != 1 or not slot.is_contiguous():
        raise ValueError("slots are a contiguous int32 vector")
    if slot.device != device:
        raise ValueError(f"slots are on {slot.device}, expected {device}")
    if rows is not None and slot.shape[0] != rows:
        raise ValueError(f"{slot.shape[0]} slots for {rows} rows")
    return slot.data_ptr() or None


def _bytes(t, shape, what):
    """A dense 8-bit tensor of this shape, as uint8."""
    if t.element_size() != 1 or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{what}: expected contiguous bytes of shape {tuple(shape)}, "
                         f"got {t.dtype} {tuple(t.shape)}")
    return t.view(torch.uint8)


class QuantRows:
    """``slots`` rows of width K: ``q`` [slots][pitch], ``scale`` [slots][scale pitch]
    and, if wanted, ``norm`` [slots] (fp32, of the stored values).  New buffers
    start as zeros."""

    def __init__(self, slots, K, *, device="cuda:0", q=None, scale=None, norm=False):
        self.slots, self.K = int(slots), int(K)
        if self.slots < 0 or self.K < 1:
            raise ValueError("slots must be >= 0 and K >= 1")
        self._lib = _lib.load()
        self.pitch, self.scale_pitch = _lib.moeca_quant_pitch(K), _lib.moeca_quant_scale_pitch(K)
        if (q is None) != (scale is None):
            raise ValueError("q and scale come together")
        if q is None:
            q = torch.zeros(self.slots, self.pitch, dtype=torch.uint8, device=device)
            scale = torch.zeros(self.slots, self.scale_pitch, dtype=torch.uint8, device=device)
        self.q = _bytes(q, (self.slots, self.pitch), "q")
        self.device = self.q.device
        self.scale = _bytes(scale, (self.slots, self.scale_pitch), "scale")
        if norm is True:
            norm = torch.zeros(self.slots, device=self.q.device)
        self.norm = None if norm is None or norm is False else norm
        if self.norm is not None and (self.norm.dtype != torch.float32 or self.norm.ndim != 1 or
                                      self.norm.shape[0] != self.slots or
                                      not self.norm.is_contiguous()):
            raise ValueError("norm: expected a contiguous float32 vector, one per slot")
        for t in (self.scale, self.norm):
            if t is not None and t.device != self.q.device:
                raise ValueError("q, scale and norm must be on one device")

    def write(self, x, slot=None, stream=None):
        """Quantise the rows of ``x`` [rows][K] into ``slot`` (int32, default row r into
        slot r); a slot outside the range leaves its row out."""
        p, rows, ld = _rows(x, self.K, self.device, "x")
        at = _indexes(slot, rows, self.device)
        if rows == 0:
            return
        _launch(self._lib.moeca_quant_rows, self.device, stream, p, _dtype(x), rows, self.K, ld,
                at, self.slots, self.q.data_ptr(), self.scale.data_ptr(),
                None if self.norm is None else self.norm.data_ptr())

    def read(self, slot=None, dtype=None, out=None, stream=None):
        """The values of rows ``slot`` (default: all), in ``out`` or a new tensor of
        ``dtype`` (bfloat16); a slot outside the range gives zeros."""
        at = _indexes(slot, None, self.device)
        rows = self.slots if slot is None else slot.shape[0]
        if out is None:
            out = _empty((rows, self.K), dtype or _BF16, self.device, stream)
        elif dtype is not None and out.dtype != dtype:
            raise TypeError(f"out is {out.dtype}, not {dtype}")
        p, n, ld = _rows(out, self.K, self.device, "out")
        if n != rows:
            raise ValueError(f"out has {n} rows for {rows}")
        if rows == 0:
            return out
        _launch(self._lib.moeca_dequant_rows, self.device, stream, self.q.data_ptr(),
                self.scale.data_ptr(), self.slots, self.K, at, rows, p, _dtype(out), ld)
        return out


class QuantMatrix:
    """A weight matrix of N rows (out) and K inputs, or a stack of n of them: ``q``
    [n][N][pitch], ``scale`` [n][ceil(N / 128)][scale pitch] (one matrix: without n)."""

    def __init__(self, q, scale, N, K):
        self._lib = _lib.load()
        self.N, self.K = int(N), int(K)
        lead = tuple(q.shape[:-2])
        if len(lead) > 1:
            raise ValueError("q has two dimensions, or three for a stack")
        self.q = _bytes(q, lead + (self.N, _lib.moeca_quant_pitch(K)), "q")
        self.scale = _bytes(scale, lead + (-(-self.N // 128), _lib.moeca_quant_scale_pitch(K)),
                            "scale")
        self.device = self.q.device
        if self.scale.device != self.device:
            raise ValueError("q and scale must be on one device")


def quantize_matrix(W, stream=None) -> QuantMatrix:
    """Quantise W [N][K], or a stack [n][N][K], bfloat16 or float32."""
    if W.ndim not in (2, 3) or not W.is_contiguous():
        raise ValueError("W is a contiguous [N][K] or [n][N][K] tensor")
    N, K = W.shape[-2:]
    lead = tuple(W.shape[:-2])
    q = _empty(lead + (N, _lib.moeca_quant_pitch(K)), torch.uint8, W.device, stream)
    s = _empty(lead + (-(-N // 128), _lib.moeca_quant_scale_pitch(K)), torch.uint8, W.device,
               stream)
    _launch(_lib.load().moeca_quant_matrix, W.device, stream, W.data_ptr(), _dtype(W),
            lead[0] if lead else 1, N, K, q.data_ptr(), s.data_ptr())
    return QuantMatrix(q, s, N, K)


def linear_workspace(M, K, device="cuda:0"):
    """A workspace for ``linear`` calls of up to M rows of width K, one at a time."""
    return torch.empty(_lib.moeca_quant_linear_bytes(M, K), dtype=torch.uint8, device=device)


def linear(x, W: QuantMatrix, bias=None, out=None, workspace=None, stream=None):
    """x W^T (+ bias) for rows x [M][K] (bfloat16 or float32; quantised by the call)
    and one quantised matrix; ``out`` [M][N] is of x's type and overlaps no other
    operand.  Products are exact for float32 results and for up to 16 rows; others
    take the 8-bit matrix instructions (include/moeca.h states their precision).  Without a
    ``workspace`` one is allocated for the call, which then has to run on the
    current stream."""
    if W.q.ndim != 2:
        raise ValueError("linear takes one matrix, not a stack")
    device = W.device
    px, M, ldx = _rows(x, W.K, device, "x")
    dt = _dtype(x)
    if out is None:
        out = _empty((M, W.N), x.dtype, device, stream)
    elif out.dtype != x.dtype:
        raise TypeError(f"out is {out.dtype}, x {x.dtype}")
    po, n, ldo = _rows(out, W.N, device, "out")
    if n != M:
        raise ValueError(f"out has {n} rows, x {M}")
    if bias is not None and (bias.dtype != torch.float32 or tuple(bias.shape) != (W.N,) or
                             not bias.is_contiguous() or bias.device != device):
        raise ValueError(f"bias: expected a contiguous float32 vector of {W.N} on {device}")
    if M == 0:
        return out
    if px == po:
        raise ValueError("out is x: the product's blocks read x while others write out")
    if workspace is None:
        if stream is not None and stream != torch.cuda.current_stream(device):
            raise ValueError("a call on another stream needs a workspace of its own")
        workspace = linear_workspace(M, W.K, device)
    elif workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"workspace: expected contiguous bytes on {device}")
    _launch(W._lib.moeca_quant_linear, device, stream, px, dt, M, W.K, ldx, W.q.data_ptr(),
            W.scale.data_ptr(), W.N, None if bias is None else bias.data_ptr(), po, ldo,
            workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return out
