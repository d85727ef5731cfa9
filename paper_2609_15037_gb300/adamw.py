"""AdamW over the parameters that have no projector, and the norm of their
gradients: host-side bookkeeping over moara_adamw_step, moara_adamw_moments and
moara_grad_norm.  Every computation happens in the library's kernels."""

from __future__ import annotations

import contextlib
import ctypes
import struct

import numpy as np
import torch

from . import _host
from . import binding as B

_TYPES = {torch.float32: B.MOARA_DTYPE_F32, torch.bfloat16: B.MOARA_DTYPE_BF16}
_STATES = {"f32": B.MOARA_DTYPE_F32, "block8": B.MOARA_DTYPE_BLOCK8}
_DESC = np.dtype(B.moara_adamw_tensor)
_PACK = struct.Struct("<q7Q3iI2f")          # the same as one record
_SIZE = _PACK.size


def entry_address(name):
    return ctypes.cast(getattr(B.lib, name), ctypes.c_void_p).value


_STEP, _MOMENTS, _NORM = (entry_address("moara_" + f) for f in ("adamw_step", "adamw_moments", "grad_norm"))


def _listed(xs):
    return xs if isinstance(xs, (list, tuple)) else list(xs)


def _current_stream(device):
    return torch.cuda.current_stream(device).cuda_stream


# the same without building a Stream object (1 us of a call's 5 to 10)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _current_stream)
_recording = torch.cuda.is_current_stream_capturing


def stream_handle(stream, device):
    """A cudaStream_t: `stream`, or torch's current stream on `device` for None."""
    return _current_stream(device) if stream is None else int(stream)


def allocating_on(stream, device):
    """Context in which torch allocates for work on `stream` (None: the current one)."""
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(torch.cuda.ExternalStream(int(stream), device=device))


class AdamWGroup:
    """Tensors that take AdamW steps together, with their moments.

    Streams are cudaStream_t handles; None is torch's current stream."""

    def __init__(self, beta1=0.9, beta2=0.999, eps=1e-8, seed=0, device=0):
        self.device = device
        self.hp = B.moara_adamw_hparams(beta1, beta2, eps, seed)
        self.ctx = None
        self.ctx = B.moara_create(B.moara_default_hparams(), device)
        self._dev = torch.device("cuda", device)
        self.params, self.copies, self.states = [], [], []
        self._table, self._room, self._all = np.zeros(0, _DESC), 0, None
        self._workspace = {}

    def _check(self, x, what, n=None, dtypes=tuple(_TYPES)):
        if x.dtype not in dtypes or x.get_device() != self.device or not x.is_contiguous():
            raise ValueError(f"{what}: a contiguous tensor of {dtypes} on cuda:{self.device} is needed")
        if n is not None and x.numel() != n:
            raise ValueError(f"{what}: {x.numel()} entries, expected {n}")
        return x

    def add(self, param, copy=None, state="f32", weight_decay=0.0, lr_scale=1.0, exp_avg=None, exp_avg_sq=None,
            exp_avg_scale=None, exp_avg_sq_scale=None, id=None):
        """Registers `param` (fp32 or bf16, updated in place) and returns its
        index.  copy: a bf16 tensor that receives the new values of an fp32
        param.  state: "f32" or "block8" moments, zero unless given (layouts of
        moara.h).  id: which random bits the 8-bit rounding takes (default: the
        index)."""
        if state not in _STATES:
            raise ValueError(f"state must be one of {tuple(_STATES)}")
        n = self._check(param, "param").numel()
        if copy is not None:
            self._check(copy, "copy", n, (torch.bfloat16,))
        code = torch.uint8 if state == "block8" else torch.float32
        blocks = -(-n // B.MOARA_ADAMW_BLOCK)

        def kept(x, what, size, dtype):
            return torch.zeros(size, dtype=dtype, device=self._dev) if x is None else self._check(x, what, size, (dtype,))
        s = {"exp_avg": kept(exp_avg, "exp_avg", n, code), "exp_avg_sq": kept(exp_avg_sq, "exp_avg_sq", n, code)}
        if state == "block8":
            s["exp_avg_scale"] = kept(exp_avg_scale, "exp_avg_scale", blocks, torch.float32)
            s["exp_avg_sq_scale"] = kept(exp_avg_sq_scale, "exp_avg_sq_scale", blocks, torch.float32)
        i = len(self.params)
        self._grow(i + 1)
        at = [x.data_ptr() for x in s.values()] + [0] * (4 - len(s))
        _PACK.pack_into(self._table, i * _SIZE, n, param.data_ptr(), 0, 0 if copy is None else copy.data_ptr(), *at,
                        _TYPES[param.dtype], 0, _STATES[state], i if id is None else id, weight_decay, lr_scale)
        self.params.append(param)
        self.copies.append(copy)
        self.states.append(s)
        return i

    def _grow(self, count):
        """Room for `count` descriptors."""
        if count > self._room:
            grown = np.zeros(max(16, 2 * count), _DESC)
            grown[:self._room] = self._table[:self._room]
            self._table, self._room = grown, len(grown)
        self._all = None

    def _chosen(self, ids):
        """The descriptors of a call, and their address."""
        if self._all is None:                       # they and their address are kept
            self._all = self._table[:len(self.params)], self._table.ctypes.data
        if ids is None:
            return self._all
        d = self._all[0][list(ids)]
        return d, d.ctypes.data

    def step(self, grads, t, lr, grad_scale=None, ids=None, stream=None):
        """One AdamW step at step t (1-based): grads[i] (fp32 or bf16) of every
        registered tensor, or of those in ids.  grad_scale: a one-element
        float32 device tensor that multiplies every gradient, or None."""
        d, at = self._chosen(ids)
        code = _host.adamw_step(_STEP, self.ctx, len(d), at, _listed(grads), ctypes.addressof(self.hp), t, lr, grad_scale,
                                self.device, stream_handle(stream, self.device))
        if code:
            B._check(code, self.ctx, "moara_adamw_step")

    def moments(self, exp_avg=None, exp_avg_sq=None, ids=None, stream=None):
        """The moments as fp32 tensors (lists, one per tensor); into the given
        ones, if any."""
        d, at = self._chosen(ids)
        n = len(d)
        if exp_avg is None or exp_avg_sq is None:
            sizes = d["n"].tolist()
            with allocating_on(stream, self.device):
                exp_avg, exp_avg_sq = ([torch.empty(k, device=self._dev) for k in sizes] if x is None else x
                                       for x in (exp_avg, exp_avg_sq))
        code = _host.adamw_moments(_MOMENTS, self.ctx, n, at, _listed(exp_avg), _listed(exp_avg_sq), self.device,
                                   stream_handle(stream, self.device))
        if code:
            B._check(code, self.ctx, "moara_adamw_moments")
        return exp_avg, exp_avg_sq

    def _norm_workspace(self, count, handle):
        """(tensor, address, bytes, gradients that it serves); zero before its first call."""
        # a recorded graph has its own, which no later call replaces or shares
        recorded = _recording()
        kept = None if recorded else self._workspace.get(handle)
        if kept is None or count > kept[3]:
            ws = torch.zeros(B.moara_grad_norm_workspace_bytes(count), dtype=torch.uint8, device=self._dev)
            kept = ws, ws.data_ptr(), ws.numel(), count
            if not recorded:
                self._workspace[handle] = kept
        return kept

    def grad_norm(self, grads, max_norm=0.0, extra_sq=None, out=None, stream=None):
        """{sum of squares, norm, clipping coefficient} of any gradients (fp32 or
        bf16), a float32 tensor of three.  extra_sq: a one-element float32 device
        tensor added to the sum under the root, or None.  The first element is
        what MoaraGroup.set_clip_extra takes, the last what step takes."""
        grads = _listed(grads)
        if stream is None:
            handle = _current_stream(self.device)
            ws = self._norm_workspace(len(grads), handle)
            got = _host.grad_norm(_NORM, self.ctx, grads, max_norm, extra_sq, out, ws[1], ws[2], self.device, handle)
        else:
            with allocating_on(stream, self.device):
                ws = self._norm_workspace(len(grads), int(stream))
                got = _host.grad_norm(_NORM, self.ctx, grads, max_norm, extra_sq, out, ws[1], ws[2], self.device, int(stream))
        if got.__class__ is int:
            B._check(got, self.ctx, "moara_grad_norm")
        return got

    def state_dict(self):
        return [{k: v.detach().clone() for k, v in s.items()} for s in self.states]

    def load_state_dict(self, sd):
        """Into the registered tensors' moments; nothing is taken of one that does not fit."""
        like = [{k: (v.dtype, v.shape) for k, v in s.items()} for s in sd]
        if like != [{k: (v.dtype, v.shape) for k, v in s.items()} for s in self.states]:
            raise ValueError("load_state_dict: the moments of other tensors")
        for s, new in zip(self.states, sd):
            for k, v in s.items():
                v.copy_(new[k])

    def close(self):
        if self.ctx:
            B.moara_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
