"""MXFP4 operands and their products: torch-allocated buffers around
moara_fp4_quantize, moara_fp4_dequantize, moara_fp4_product and
moara_fp4_linear.  Every computation happens in the library's kernels."""

from __future__ import annotations

import functools

import torch

from . import binding as B
from .adamw import _TYPES, allocating_on, stream_handle


_linear_bytes = functools.lru_cache(maxsize=4096)(B.moara_fp4_linear_workspace_bytes)


class Fp4Matrix:
    """A rows x cols matrix in MXFP4 (layouts of moara.h): codes `q`, scales `sf`."""

    __slots__ = "rows", "cols", "_sizes", "_ptrs", "_both", "_start", "_q", "_sf"

    def __init__(self, rows, cols, q=None, sf=None, device=0):
        self.rows, self.cols = rows, cols
        if rows < 1 or cols < 1:
            B.moara_fp4_bytes(rows, cols)                   # raises
        # moara_fp4_bytes, without the call
        nq = rows * ((cols + 31) // 32) * 16
        sizes = self._sizes = nq, (rows + 127) // 128 * ((cols + 127) // 128) * 512
        if q is None and sf is None:
            # one allocation: the codes, and the scales from the next 256 bytes on
            start = self._start = (nq + 255) // 256 * 256
            both = self._both = torch.empty(start + sizes[1], dtype=torch.uint8,
                                            device=device if isinstance(device, torch.device) else torch.device("cuda", device))
            at = both.data_ptr()
            self._ptrs = at, at + start
            return
        self._both = None
        for x, size in zip((q, sf), sizes):
            if x is None or x.dtype != torch.uint8 or not x.is_contiguous() or x.numel() != size:
                raise ValueError(f"q and sf, contiguous uint8 tensors of {sizes} bytes, or neither are needed")
        self._q, self._sf = q, sf
        self._ptrs = q.data_ptr(), sf.data_ptr()

    @property
    def q(self):
        return self._q if self._both is None else self._both[:self._sizes[0]]

    @property
    def sf(self):
        return self._sf if self._both is None else self._both[self._start:]


class Fp4Group:
    """A context for MXFP4 operands and products on one device.

    The products of a weight W (n x k) with activations x and their gradient dy:

        x_r, x_c = fp4.quantize(x, rows=True, cols=True)
        w_r, w_c = fp4.quantize(W, rows=True, cols=True)    # after each step
        y = fp4.product(x_r, w_r)                           # x W^T
        dy_r, dy_c = fp4.quantize(dy, rows=True, cols=True)
        dx = fp4.product(dy_r, w_c)                         # dy W
        dW = fp4.product(dy_c, x_c)                         # dy^T x, G of MoaraGroup.step

    Streams are cudaStream_t handles; None is torch's current stream."""

    def __init__(self, device=0):
        self.device = device
        self.ctx = None
        self.ctx = B.moara_create(B.moara_default_hparams(), device)
        self._dev = torch.device("cuda", device)

    def _strided(self, x, what):
        """(address, type, row pitch) of a matrix whose rows are contiguous."""
        if x.dim() != 2 or x.dtype not in _TYPES or x.get_device() != self.device:
            raise ValueError(f"{what}: a float32 or bfloat16 matrix on cuda:{self.device} is needed")
        rows, cols = x.shape
        if cols > 1 and x.stride(1) != 1:
            raise ValueError(f"{what}: the entries of a row must be contiguous")
        return x.data_ptr(), _TYPES[x.dtype], x.stride(0) if rows > 1 else max(cols, 1)

    def _out(self, out, rows, cols, dtype, stream):
        if out is None:
            if dtype not in _TYPES:
                raise ValueError("dtype must be float32 or bfloat16")
            if stream is None:
                return torch.empty((rows, cols), dtype=dtype, device=self._dev)
            with allocating_on(stream, self.device):
                return torch.empty((rows, cols), dtype=dtype, device=self._dev)
        if tuple(out.shape) != (rows, cols):
            raise ValueError(f"out: shape {(rows, cols)} is needed")
        return out

    def _matrix(self, m, rows, cols, stream):
        if m is None:
            if stream is None:
                return Fp4Matrix(rows, cols, device=self._dev)
            with allocating_on(stream, self.device):
                return Fp4Matrix(rows, cols, device=self._dev)
        if (m.rows, m.cols) != (rows, cols):
            raise ValueError(f"out: an operand of {rows} x {cols} is needed")
        return m

    def quantize(self, x, rows=True, cols=False, out=None, out_cols=None, stream=None):
        """The operand of x (rows), of its transpose (cols), or both from one
        read of x; into out and out_cols where they are given."""
        if not rows and not cols:
            raise ValueError("rows, cols or both")
        ptr, dtype, ld = self._strided(x, "x")
        m, k = x.shape
        a = self._matrix(out, m, k, stream) if rows else None
        b = self._matrix(out_cols, k, m, stream) if cols else None
        q, sf = a._ptrs if rows else (0, 0)
        qt, sft = b._ptrs if cols else (0, 0)
        B.moara_fp4_quantize(self.ctx, ptr, dtype, m, k, ld, q, sf, qt, sft, stream_handle(stream, self.device))
        return (a, b) if rows and cols else a if rows else b

    def dequantize(self, a, dtype=torch.bfloat16, out=None, stream=None):
        """The values of an operand (bfloat16 holds them exactly)."""
        out = self._out(out, a.rows, a.cols, dtype, stream)
        ptr, dt, ld = self._strided(out, "out")
        B.moara_fp4_dequantize(self.ctx, *a._ptrs, a.rows, a.cols, ptr, dt, ld, stream_handle(stream, self.device))
        return out

    def product(self, a, b, dtype=torch.bfloat16, out=None, stream=None):
        """a b^T of two operands with the same number of columns."""
        if a.cols != b.cols:
            raise ValueError(f"{a.cols} and {b.cols} columns")
        m, n, k = a.rows, b.rows, a.cols
        out = self._out(out, m, n, dtype, stream)
        ptr, dt, ld = self._strided(out, "out")
        B.moara_fp4_product(self.ctx, m, n, k, *a._ptrs, *b._ptrs, ptr, dt, ld, stream_handle(stream, self.device))
        return out

    def linear(self, x, b, dtype=torch.bfloat16, out=None, stream=None):
        """x b^T with x (float32 or bfloat16) quantised by rows on the way."""
        xp, xd, ldx = self._strided(x, "x")
        m, k = x.shape
        if k != b.cols:
            raise ValueError(f"{k} and {b.cols} columns")
        n = b.rows
        out = self._out(out, m, n, dtype, stream)
        ptr, dt, ld = self._strided(out, "out")
        ws, size = self._workspace(_linear_bytes(m, n, k), stream)
        B.moara_fp4_linear(self.ctx, m, n, k, xp, xd, ldx, *b._ptrs, ptr, dt, ld, ws.data_ptr() if size else 0, size,
                           stream_handle(stream, self.device))
        return out

    def _workspace(self, size, stream):
        if size == 0:
            return None, 0
        if stream is None:
            return torch.empty(size, dtype=torch.uint8, device=self._dev), size
        with allocating_on(stream, self.device):
            return torch.empty(size, dtype=torch.uint8, device=self._dev), size

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
