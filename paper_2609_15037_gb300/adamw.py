"""AdamW over the parameters that have no projector, and the norm of their
gradients: host-side bookkeeping over moara_adamw_step, moara_adamw_moments and
moara_grad_norm.  Every computation happens in the library's kernels."""

from __future__ import annotations

import bisect
import contextlib
import ctypes
import struct
import types

import numpy as np
import torch

from . import _host
from . import binding as B

_TYPES = {torch.float32: B.MOARA_DTYPE_F32, torch.bfloat16: B.MOARA_DTYPE_BF16}
_STATES = {"f32": B.MOARA_DTYPE_F32, "block8": B.MOARA_DTYPE_BLOCK8}
_DESC = np.dtype(B.moara_adamw_tensor)
_PACK = struct.Struct("<q7Q3iI2f")          # the same as one record
_SIZE = _PACK.size
_PLACES = np.dtype([("storage", np.uint64, 4), ("data", np.uint64, 4)])     # of a tensor's moments: host.cpp


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


class _Ranges:
    """Disjoint ranges of addresses."""

    def __init__(self):
        self._begin, self._end = [], []

    def add(self, at, sizes):
        """The memory at these addresses (0: none), all of it or nothing; ValueError where it
        overlaps a range or itself."""
        taken = []
        for begin, size in zip(at, sizes):
            if begin == 0:
                continue
            end = begin + size
            i = bisect.bisect_right(self._begin, begin)
            if (i and self._end[i - 1] > begin) or (i < len(self._begin) and self._begin[i] < end):
                for b in taken:
                    j = bisect.bisect_left(self._begin, b)
                    del self._begin[j], self._end[j]
                raise ValueError("the tensor, its copy or its moments overlap registered ones")
            self._begin.insert(i, begin)
            self._end.insert(i, end)
            taken.append(begin)


class AdamWGroup:
    """Tensors that take AdamW steps together, with their moments.

    A registered parameter or copy whose storage is replaced (an assignment to .data,
    module.to) is followed to its new place and type, and refused where it no longer fits; the
    memory of the moments is the group's from add on.  What a step
    writes (parameters, copies, moments) must not overlap: a tensor is registered once, and
    taken once per call.
    Streams are cudaStream_t handles; None is torch's current stream.  A call orders nothing
    between streams: a tensor that was made on another one has to be complete, and has to live
    until the call's work is done (torch.Tensor.record_stream)."""

    def __init__(self, beta1=0.9, beta2=0.999, eps=1e-8, seed=0, device=0):
        self.device = device
        self.hp = B.moara_adamw_hparams(beta1, beta2, eps, seed)
        self.ctx = None
        self.ctx = B.moara_create(B.moara_default_hparams(), device)
        self._dev = torch.device("cuda", device)
        self.params, self.copies, self.states = [], [], []
        self._own = []          # of each tensor: four tensors, or None, on its moments' memory
        self._ranges = _Ranges()
        self._table, self._places, self._places_at = np.zeros(0, _DESC), np.zeros(0, _PLACES), 0
        self._room, self._all = 0, None
        self._workspace = {}

    def _check(self, x, what, n=None, dtypes=tuple(_TYPES)):
        if x.dtype not in dtypes or x.get_device() != self.device or not x.is_contiguous():
            raise ValueError(f"{what}: a contiguous tensor of {dtypes} on cuda:{self.device} is needed")
        if n is not None and x.numel() != n:
            raise ValueError(f"{what}: {x.numel()} entries, expected {n}")
        return x

    def _check_kept(self, kept, n, state):
        """Checks a tensor's (param, copy, exp_avg, exp_avg_sq, exp_avg_scale, exp_avg_sq_scale), the
        last two None for f32 moments; their addresses."""
        param, copy, *moments = kept
        self._check(param, "param", n)
        if copy is not None:
            self._check(copy, "copy", n, (torch.bfloat16,))
        code = torch.uint8 if state == "block8" else torch.float32
        self._check(moments[0], "exp_avg", n, (code,))
        self._check(moments[1], "exp_avg_sq", n, (code,))
        if state == "block8":
            blocks = -(-n // B.MOARA_ADAMW_BLOCK)
            self._check(moments[2], "exp_avg_scale", blocks, (torch.float32,))
            self._check(moments[3], "exp_avg_sq_scale", blocks, (torch.float32,))
        return [0 if x is None else x.data_ptr() for x in kept]

    @staticmethod
    def _bytes(n, dtype, state):
        """Of what _check_kept takes."""
        code, blocks = 1 if state == "block8" else 4, 4 * -(-n // B.MOARA_ADAMW_BLOCK)
        return 4 * n if dtype is torch.float32 else 2 * n, 2 * n, code * n, code * n, blocks, blocks

    def add(self, param, copy=None, state="f32", weight_decay=0.0, lr_scale=1.0, exp_avg=None, exp_avg_sq=None,
            exp_avg_scale=None, exp_avg_sq_scale=None, id=None):
        """Registers `param` (fp32 or bf16, updated in place) and returns its
        index.  copy: a bf16 tensor that receives the new values of an fp32
        param.  state: "f32" or "block8" moments, zero unless given (layouts of
        moara.h).  id: which random bits the 8-bit rounding takes (default: the
        index)."""
        if state not in _STATES:
            raise ValueError(f"state must be one of {tuple(_STATES)}")
        n = param.numel()
        blocks = -(-n // B.MOARA_ADAMW_BLOCK)

        def kept(x, size, dtype):
            return torch.zeros(size, dtype=dtype, device=self._dev) if x is None else x
        code = torch.uint8 if state == "block8" else torch.float32
        s = {"exp_avg": kept(exp_avg, n, code), "exp_avg_sq": kept(exp_avg_sq, n, code)}
        if state == "block8":
            s["exp_avg_scale"] = kept(exp_avg_scale, blocks, torch.float32)
            s["exp_avg_sq_scale"] = kept(exp_avg_sq_scale, blocks, torch.float32)
        tensors = param, copy, *s.values(), *(None,) * (4 - len(s))
        at = self._check_kept(tensors, n, state)
        i = len(self.params)
        self._grow(i + 1)
        own = _host.own(tensors[2:], self._places_at + i * _PLACES.itemsize)
        _PACK.pack_into(self._table, i * _SIZE, n, at[0], 0, *at[1:],
                        _TYPES[param.dtype], 0, _STATES[state], i if id is None else id, weight_decay, lr_scale)
        sizes = self._bytes(n, param.dtype, state)
        try:
            self._ranges.add(at, sizes)
        except ValueError:      # or they lie where a replaced storage was
            self._follow()
            self._ranges.add(at, sizes)
        self.params.append(param)
        self.copies.append(copy)
        self.states.append(types.MappingProxyType(s))
        self._own.append(own)
        return i

    def _grow(self, count):
        """Room for `count` descriptors."""
        if count > self._room:
            grown = np.zeros(max(16, 2 * count), _DESC)
            grown[:self._room] = self._table[:self._room]
            places = np.zeros(len(grown), _PLACES)
            places[:self._room] = self._places[:self._room]
            self._table, self._places, self._room = grown, places, len(grown)
            self._places_at = places.ctypes.data
        self._all = None

    def _chosen(self, ids):
        """The descriptors of a call, their number and address, the address of the moments' places,
        and the parameters and copies."""
        if self._all is None:                       # they and their address are kept
            n = len(self.params)
            self._all = self._table[:n], n, self._table.ctypes.data, self._places_at, self.params, self.copies
        if ids is None:
            return self._all
        rows = np.arange(len(self.params))[ids]
        at = rows.tolist()
        if len(set(at)) != len(at):
            raise ValueError("ids: a tensor is listed twice")
        d, places = self._all[0][rows], self._places[rows]
        return (d, len(at), d.ctypes.data, places.ctypes.data, [self.params[i] for i in at], [self.copies[i] for i in at],
                places)

    def _follow(self):
        """The descriptors of tensors whose storage was replaced (an assignment to .data,
        module.to) or taken anew in place: their new places and types.  One that no longer fits is
        refused."""
        n = len(self.params)
        d, places, at, ranges = self._table[:n], self._places[:n], [], _Ranges()
        for p, c, own, size, state in zip(self.params, self.copies, self._own, d["n"].tolist(), d["state_dtype"].tolist()):
            x, state = (p, c, *own), "block8" if state == B.MOARA_DTYPE_BLOCK8 else "f32"
            at.append(self._check_kept(x, size, state))
            for y in x:
                if y is not None and y.untyped_storage().nbytes() < (y.storage_offset() + y.numel()) * y.element_size():
                    raise ValueError("the storage of a registered tensor was freed")
            ranges.add(at[-1], self._bytes(size, p.dtype, state))
        fields = "param", "param_bf16", "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale"
        for name, column in zip(fields, zip(*at)):
            d[name] = column
        d["param_dtype"] = [_TYPES[p.dtype] for p in self.params]
        for i, own in enumerate(self._own):
            places["data"][i] = [0 if x is None else x.untyped_storage().data_ptr() for x in own]
        self._ranges = ranges

    def _check_code(self, code, name):
        if code is None:
            raise RuntimeError("registered tensors change during the call")
        if code:
            B._check(code, self.ctx, name)

    def step(self, grads, t, lr, grad_scale=None, ids=None, stream=None):
        """One AdamW step at step t (1-based): grads[i] (fp32 or bf16) of every
        registered tensor, or of those in ids.  grad_scale: a one-element
        float32 device tensor that multiplies every gradient, or None."""
        grads, ids = _listed(grads), ids if ids is None else list(ids)
        stream = stream_handle(stream, self.device)
        for _ in range(2):                          # again where tensors were found in other places
            c = self._chosen(ids)
            code = _host.adamw_step(_STEP, self.ctx, c[1], c[2], grads, ctypes.addressof(self.hp), t, lr, grad_scale,
                                    self.device, stream, c[3], c[4], c[5])
            if code is not None:
                break
            self._follow()
        if code != 0:
            self._check_code(code, "moara_adamw_step")

    def moments(self, exp_avg=None, exp_avg_sq=None, ids=None, stream=None):
        """The moments as fp32 tensors (lists, one per tensor); into the given
        ones, if any."""
        ids = ids if ids is None else list(ids)
        if exp_avg is None or exp_avg_sq is None:
            sizes = self._chosen(ids)[0]["n"].tolist()
            with allocating_on(stream, self.device):
                exp_avg, exp_avg_sq = ([torch.empty(k, device=self._dev) for k in sizes] if x is None else x
                                       for x in (exp_avg, exp_avg_sq))
        m, v = _listed(exp_avg), _listed(exp_avg_sq)
        stream = stream_handle(stream, self.device)
        for _ in range(2):
            c = self._chosen(ids)
            code = _host.adamw_moments(_MOMENTS, self.ctx, c[1], c[2], m, v, self.device, stream, c[3])
            if code is not None:
                break
            self._follow()
        if code != 0:
            self._check_code(code, "moara_adamw_moments")
        return m, v

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
        return [{k: v.clone() for k, v in zip(s, own)} for s, own in zip(self.states, self._own)]

    def load_state_dict(self, sd):
        """Into the registered tensors' moments; nothing is taken of one that does not fit."""
        like = [{k: (v.dtype, v.shape) for k, v in s.items()} for s in sd]
        if like != [{k: (v.dtype, v.shape) for k, v in zip(s, own)} for s, own in zip(self.states, self._own)]:
            raise ValueError("load_state_dict: the moments of other tensors")
        for s, own, new in zip(self.states, self._own, sd):
            for k, v in zip(s, own):
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
