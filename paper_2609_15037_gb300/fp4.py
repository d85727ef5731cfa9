"""MXFP4 operands and their products: torch-allocated buffers around
moara_fp4_quantize, moara_fp4_dequantize, moara_fp4_product and
moara_fp4_linear.  Every computation happens in the library's kernels."""

from __future__ import annotations

import torch

from . import _host
from . import binding as B
from .adamw import _TYPES, allocating_on, entry_address, stream_handle

_QUANTIZE, _DEQUANTIZE, _PRODUCT, _LINEAR, _LINEAR_BYTES = (
    entry_address("moara_fp4_" + f) for f in ("quantize", "dequantize", "product", "linear", "linear_workspace_bytes"))


class Fp4Matrix:
    """A rows x cols matrix in MXFP4 (layouts of moara.h): codes `q`, scales `sf`."""

    __slots__ = "rows", "cols", "device", "_ptrs", "_both", "_q", "_sf"

    def __init__(self, rows, cols, q=None, sf=None, device=0):
        self.rows, self.cols, self.device = rows, cols, device
        sizes = B.moara_fp4_bytes(rows, cols)
        if q is None and sf is None:
            # one allocation: the codes, and the scales from the next 256 bytes on
            start = (sizes[0] + 255) // 256 * 256
            self._both, at = _host.bytes(start + sizes[1], device)
            self._ptrs = at, at + start
            return
        self._both = None
        for x, size in zip((q, sf), sizes):
            if (x is None or x.dtype != torch.uint8 or not x.is_contiguous() or x.numel() != size
                    or x.get_device() != device):
                raise ValueError(f"q and sf, contiguous uint8 tensors of {sizes} bytes on cuda:{device}, or neither are needed")
        # tensors of its own on the same memory: q and sf keep their identity where their storage is
        # replaced
        self._q, self._sf = q.detach(), sf.detach()
        self._ptrs = q.data_ptr(), sf.data_ptr()

    @property
    def q(self):
        return self._q if self._both is None else self._both[:B.moara_fp4_bytes(self.rows, self.cols)[0]]

    @property
    def sf(self):
        return self._sf if self._both is None else self._both[self._ptrs[1] - self._ptrs[0]:]

    def record_stream(self, stream):
        """As torch.Tensor.record_stream: once this operand is released, its memory is taken
        again only behind what `stream` (a torch.cuda.Stream or a cudaStream_t handle) has been
        given by then."""
        if not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(int(stream), device=self.device)
        for x in (self._q, self._sf) if self._both is None else (self._both,):
            x.record_stream(stream)


def _operand(buffer, rows, cols, device):
    """The operand in a buffer of the native module: (tensor, address of q, of sf)."""
    a = Fp4Matrix.__new__(Fp4Matrix)
    a.rows, a.cols, a.device, a._both, a._ptrs = rows, cols, device, buffer[0], buffer[1:]
    return a


class Fp4Group:
    """A context for MXFP4 operands and products on one device.

    The products of a weight W (n x k) with activations x and their gradient dy:

        x_r, x_c = fp4.quantize(x, rows=True, cols=True)
        w_r, w_c = fp4.quantize(W, rows=True, cols=True)    # after each step
        y = fp4.product(x_r, w_r)                           # x W^T
        dy_r, dy_c = fp4.quantize(dy, rows=True, cols=True)
        dx = fp4.product(dy_r, w_c)                         # dy W
        dW = fp4.product(dy_c, x_c)                         # dy^T x, G of MoaraGroup.step

    Streams are cudaStream_t handles; None is torch's current stream.  A call orders nothing
    between streams: an input that was made on another one has to be complete, and has to live
    until the call's work is done (record_stream of the tensor or operand)."""

    def __init__(self, device=0):
        self.device = device
        self.ctx = None
        self.ctx = B.moara_create(B.moara_default_hparams(), device)

    def _matrix(self, m, rows, cols, stream):
        if m is None:
            if stream is None:
                return Fp4Matrix(rows, cols, device=self.device)
            with allocating_on(stream, self.device):
                return Fp4Matrix(rows, cols, device=self.device)
        if (m.rows, m.cols) != (rows, cols):
            raise ValueError(f"out: an operand of {rows} x {cols} is needed")
        return self._here(m)

    def _here(self, m):
        """An operand, whose addresses are this group's device's."""
        if m.device != self.device:
            raise ValueError(f"an operand on cuda:{m.device}, expected cuda:{self.device}")
        return m

    def _bf16(self, out, dtype):
        """Whether a new output is bf16 (an output that is given has its own type)."""
        bf16 = _TYPES.get(dtype)
        if bf16 is None and out is None:
            raise ValueError("dtype must be float32 or bfloat16")
        return bf16

    def _done(self, got, name):
        """What a call of the native module gave: a tensor, or an error code to raise."""
        if got.__class__ is int:
            B._check(got, self.ctx, name)
        return got

    def quantize(self, x, rows=True, cols=False, out=None, out_cols=None, stream=None):
        """The operand of x (rows), of its transpose (cols), or both from one
        read of x; into out and out_cols where they are given."""
        if not rows and not cols:
            raise ValueError("rows, cols or both")
        if out is None and out_cols is None and stream is None:
            got = _host.fp4_quantize(_QUANTIZE, self.ctx, x, rows, cols, self.device, stream_handle(None, self.device))
            if got.__class__ is int:
                B._check(got, self.ctx, "moara_fp4_quantize")
            r, c, m, k = got
            if not cols:
                return _operand(r, m, k, self.device)
            b = _operand(c, k, m, self.device)
            return (_operand(r, m, k, self.device), b) if rows else b
        ptr, dtype, m, k, ld = _host.matrix(x, self.device)
        a = self._matrix(out, m, k, stream) if rows else None
        b = self._matrix(out_cols, k, m, stream) if cols else None
        q, sf = a._ptrs if rows else (0, 0)
        qt, sft = b._ptrs if cols else (0, 0)
        B.moara_fp4_quantize(self.ctx, ptr, dtype, m, k, ld, q, sf, qt, sft, stream_handle(stream, self.device))
        return (a, b) if rows and cols else a if rows else b

    def dequantize(self, a, dtype=torch.bfloat16, out=None, stream=None):
        """The values of an operand (bfloat16 holds them exactly)."""
        args = (_DEQUANTIZE, self.ctx, *self._here(a)._ptrs, a.rows, a.cols, out, self._bf16(out, dtype), self.device,
                stream_handle(stream, self.device))
        if stream is None:
            return self._done(_host.fp4_dequantize(*args), "moara_fp4_dequantize")
        with allocating_on(stream, self.device):
            return self._done(_host.fp4_dequantize(*args), "moara_fp4_dequantize")

    def product(self, a, b, dtype=torch.bfloat16, out=None, stream=None):
        """a b^T of two operands with the same number of columns."""
        if a.cols != b.cols:
            raise ValueError(f"{a.cols} and {b.cols} columns")
        args = (_PRODUCT, self.ctx, a.rows, b.rows, a.cols, *self._here(a)._ptrs, *self._here(b)._ptrs, out,
                self._bf16(out, dtype), self.device, stream_handle(stream, self.device))
        if stream is None:
            return self._done(_host.fp4_product(*args), "moara_fp4_product")
        with allocating_on(stream, self.device):
            return self._done(_host.fp4_product(*args), "moara_fp4_product")

    def linear(self, x, b, dtype=torch.bfloat16, out=None, stream=None):
        """x b^T with x (float32 or bfloat16) quantised by rows on the way."""
        args = (_LINEAR, self.ctx, x, b.rows, b.cols, *self._here(b)._ptrs, out, self._bf16(out, dtype), self.device,
                stream_handle(stream, self.device), _LINEAR_BYTES)
        if stream is None:
            return self._done(_host.fp4_linear(*args), "moara_fp4_linear")
        with allocating_on(stream, self.device):
            return self._done(_host.fp4_linear(*args), "moara_fp4_linear")

    def status(self, stream=None):
        """Reads and clears the device status word (0, or an error a kernel recorded)."""
        return B.moara_get_device_status(self.ctx, stream_handle(stream, self.device))

    def close(self):
        if self.ctx:
            B.moara_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
