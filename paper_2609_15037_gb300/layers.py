"""Operators of a decoder's layers beside its products: root-mean-square norm, causal
attention over packed sequences, clipped policy loss; torch-allocated buffers around
moara_rms_norm, moara_rms_norm_quantize, moara_rms_norm_backward, moara_attention,
moara_attention_backward and moara_policy_loss.  Every computation happens in the
library's kernels."""

from __future__ import annotations

import ctypes

import torch

from . import _host
from . import binding as B
from .adamw import _TYPES, allocating_on, entry_address, record_on, stream_handle
from .fp4 import _operand

(_NORM, _NORM_QUANTIZE, _NORM_BACKWARD, _NORM_BYTES, _ATTENTION, _ATTENTION_BACKWARD, _LOSS, _LOSS_BYTES) = (
    entry_address("moara_" + f) for f in (
        "rms_norm", "rms_norm_quantize", "rms_norm_backward", "rms_norm_backward_workspace_bytes", "attention",
        "attention_backward", "policy_loss", "policy_loss_workspace_bytes"))


class Sequences:
    """Packed sequences of the given lengths (zero among them), one behind the other, as the
    attention takes them; made once and used by every layer, and by graphs recorded with it,
    which read its device memory."""

    def __init__(self, lengths, device=0, stream=None):
        self.lengths = [int(x) for x in lengths]
        self.device = device
        size = B.moara_sequences_bytes(self.lengths)
        host = torch.empty(max(1, size), dtype=torch.uint8)
        self._desc = B.moara_sequences_init(self.lengths, host.data_ptr(), size)
        self.tokens = self._desc.tokens
        with allocating_on(stream, device):
            # complete when this returns, for every stream
            self._tiles = host.to(torch.device("cuda", device))
        self._desc.tiles = self._tiles.data_ptr()
        self._at = ctypes.addressof(self._desc)

    def record_stream(self, stream):
        """As torch.Tensor.record_stream: once this list is released, its memory is taken
        again only behind what `stream` (a torch.cuda.Stream or a cudaStream_t handle) has been
        given by then."""
        record_on(stream, self.device, (self._tiles,))


class LayerGroup:
    """A context for the operators of a decoder's layers on one device.

    A layer's way, with the products of Fp4Group between:

        seqs = layer.sequences(lengths)                              # once a step
        h, (a, at), s = layer.norm_quantize(x, gain, residual=h, cols=True)
        qkv = fp4.product(a, w_qkv).view(tokens, heads + 2 * kv_heads, dim)
        out, lse, rest = layer.attention(q, k, v, seqs, train=True)
        ...
        dq, dk, dv = layer.attention_backward(dout, q, k, v, out, lse, seqs, rest=rest)
        dx, dgain = layer.norm_backward(dy, h, gain, s, dh=dh)       # of x and of the residual

    and behind the head's product

        sums, logp, dlogits = layer.policy_loss(logits, targets, old, adv, ref=ref, kl=0.05)

    Streams are cudaStream_t handles; None is torch's current stream.  A call orders nothing
    between streams: an input that was made on another one has to be complete, and has to live
    until the call's work is done (record_stream of the tensor, operand or list)."""

    def __init__(self, device=0):
        self.device = device
        self.ctx = None
        self.ctx = B.moara_create(B.moara_default_hparams(), device)

    def _call(self, name, fn, args, stream):
        if stream is None:
            got = fn(*args)
        else:
            with allocating_on(stream, self.device):
                got = fn(*args)
        if got.__class__ is int:
            B._check(got, self.ctx, name)
        return got

    def sequences(self, lengths, stream=None):
        return Sequences(lengths, self.device, stream)

    def _seqs(self, seqs):
        if seqs.device != self.device:
            raise ValueError(f"sequences on cuda:{seqs.device}, expected cuda:{self.device}")
        return seqs._at

    def norm(self, x, gain, residual=None, eps=1e-6, dtype=torch.bfloat16, h=None, out=None, stream=None):
        """(h, y, rstd) with h = x + residual in their type (x itself without one), y = h rstd gain
        in `dtype` and rstd = 1 / sqrt(mean h^2 + eps) of each row, which the gradients take.
        x, residual: float32 or bfloat16 matrices, gain: float32.  Into h and out where they are
        given; h may be x or the residual, out any of the three."""
        bf16 = _TYPES.get(dtype)
        if bf16 is None and out is None:
            raise ValueError("dtype must be float32 or bfloat16")
        return self._call("moara_rms_norm", _host.rms_norm, (
            _NORM, self.ctx, x, gain, residual, eps, bf16, h, out, self.device, stream_handle(stream, self.device)), stream)

    def norm_quantize(self, x, gain, residual=None, eps=1e-6, rows=True, cols=False, h=None, stream=None):
        """(h, operand, rstd) as norm with y as an Fp4Matrix, by rows (rows), by columns
        (cols), or a pair of both; y itself is not stored."""
        if not rows and not cols:
            raise ValueError("rows, cols or both")
        h, r, c, rstd, m, k = self._call("moara_rms_norm_quantize", _host.rms_norm_quantize, (
            _NORM_QUANTIZE, self.ctx, x, gain, residual, eps, rows, cols, h, self.device, stream_handle(stream, self.device)), stream)
        a = _operand(r, m, k, self.device) if rows else None
        b = _operand(c, k, m, self.device) if cols else None
        return h, (a, b) if rows and cols else a if rows else b, rstd

    def norm_backward(self, dy, h, gain, rstd, dh=None, out=None, stream=None):
        """(dx, dgain) from the gradient of y and, where it is given, that of h (dh, of h's
        type, what flows past the norm): dx, of h's type, is the gradient of x and of the residual.
        Into `out` where it is given, which may be dy, h or dh."""
        return self._call("moara_rms_norm_backward", _host.rms_norm_backward, (
            _NORM_BACKWARD, self.ctx, dy, h, gain, rstd, dh, out, self.device, stream_handle(stream, self.device), _NORM_BYTES), stream)

    def attention(self, q, k, v, seqs, scale=None, train=False, stream=None):
        """(out, lse) of causal attention inside the sequences; with train, (out, lse, rest),
        whose `rest` is what the rounding of out dropped.  q: tokens x heads x dim, k and v: tokens
        x kv_heads x dim, bfloat16, of any pitches that are multiples of 8 (slices of one
        projection), dim a multiple of 8 up to 128, kv_heads a divisor of heads.  scale: 1 / sqrt(dim) for None.
        Tokens behind the last sequence get zeros."""
        scale = q.shape[-1] ** -0.5 if scale is None else scale
        got = self._call("moara_attention", _host.attention, (
            _ATTENTION, self.ctx, self._seqs(seqs), q, k, v, scale, train, self.device, stream_handle(stream, self.device)), stream)
        return got if train else got[:2]

    def attention_backward(self, dout, q, k, v, out, lse, seqs, rest=None, scale=None, stream=None):
        """(dq, dk, dv) from the gradient of out and what attention(..., train=True) gave.
        Without `rest` the gradient of q is less exact where sequences are long."""
        scale = q.shape[-1] ** -0.5 if scale is None else scale
        return self._call("moara_attention_backward", _host.attention_backward, (
            _ATTENTION_BACKWARD, self.ctx, self._seqs(seqs), dout, q, k, v, out, lse, rest, scale, self.device,
            stream_handle(stream, self.device)), stream)

    def policy_loss(self, logits, targets, old, adv, weights=None, ref=None, clip=(0.2, 0.2), kl=0.0, grad=True, out=None,
                    stream=None):
        """(sums, logp, dlogits) of the clipped policy loss: sums = {loss, weighted KL term,
        weight of the clipped tokens}, logp the targets' log-probabilities, dlogits (None
        without `grad`) the loss's gradient, into `out` where it is given, which may be the logits.
        targets: int64; old, adv, weights (None: 1 / tokens), ref: float32 of one entry a token.
        The ratio is clipped to 1 - clip[0] .. 1 + clip[1].  kl: factor of the KL term to `ref`, which is
        not read where the factor is 0 (the second sum is 0 then)."""
        low, high = 1.0 - clip[0], 1.0 + clip[1]
        if kl and ref is None:
            raise ValueError("a KL term needs ref")
        return self._call("moara_policy_loss", _host.policy_loss, (
            _LOSS, self.ctx, logits, targets, old, adv, weights, ref if kl else None, low, high, kl, grad, out, self.device,
            stream_handle(stream, self.device), _LOSS_BYTES), stream)

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
