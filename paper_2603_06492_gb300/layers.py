"""The operators of ``libnoble.so`` in front of a projection, for torch tensors: layer norm with
the residual stream, and embedding.

    training     embed_forward, norm_forward  /  norm_backward, embed_backward
    generation   embed_forward, norm_forward, on buffers without gradients

As in ``attention``, buffer classes allocate the caller-owned memory of one shape with torch,
functions check and marshal arguments and return views of their buffers, which the next call
overwrites, and every step runs in the library's kernels.  ``include/noble.h`` defines each
operator.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding
from .attention import _TORCH, _code
from .binding import _check, _stream_handle


def _at(x, name, dtype, shape, device):
    """Address of a contiguous tensor of the given shape, type and device; None stays None."""
    if x is None:
        return None
    if x.dtype is not dtype or x.shape != shape or x.device != device or not x.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor {list(shape)} on {device}, got {x.dtype} "
                         f"{list(x.shape)} on {x.device}")
    return x.data_ptr()


def _place(x):
    """The device of a buffer's tensors, and its index; no tensor is on that of buffers without a GPU."""
    return (x.device, x.device.index) if x.is_cuda else ("a GPU, which these buffers are not on", -1)


def _stream(stream, buf):
    """Handle of the stream of a call, whose device has to be the current one."""
    handle = _stream_handle(stream)
    if buf._index != _current():
        raise ValueError(f"the buffers are on {buf.device}, the current device is {_current()}")
    return handle


_current = torch.cuda.current_device


# ---------------------------------------------------------------- layer norm
class NormBuffers:
    """Outputs and workspace of the norm of T rows of d elements: ``y``, with residual ``sum``, the
    stream behind the addition; with gradients ``dx``, ``dgain``, ``dbias``."""

    def __init__(self, T, d, dtype, eps=1e-5, residual=False, device="cuda", with_grads=True):
        self.T, self.d, self.residual = T, d, residual
        self.desc = binding.NormDesc(T, d, eps, _code(dtype), 0)
        self.dtype = _TORCH[self.desc.dtype]
        new = dict(dtype=self.dtype, device=device)
        self.y = torch.empty((T, d), **new)
        self.device, self._index = _place(self.y)
        self._lib = binding.load()
        self.sum = torch.empty((T, d), **new) if residual else None
        self._ref, self._rows, self._row = ctypes.byref(self.desc), (T, d), (d,)
        self._out = (self.sum.data_ptr() if residual else None, self.y.data_ptr())
        self.stats = None
        if with_grads:
            self.stats = torch.empty((T, 2), dtype=torch.float32, device=device)
            self.workspace_bytes = binding.load().noble_norm_bwd_workspace_bytes(self._ref)
            self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=device)
            self.dx = torch.empty((T, d), **new)
            self.dgain, self.dbias = (torch.empty(d, dtype=torch.float32, device=device) for _ in range(2))

    def _rows_of(self, x, name):
        return _at(x, name, self.dtype, self._rows, self.device)

    def _features(self, x, name):
        return _at(x, name, torch.float32, self._row, self.device)


def norm_forward(buf: NormBuffers, x, gain=None, bias=None, res=None, stream=None):
    """Layer norm of x [T, d] into ``buf.y``; with residual buffers of x + res, which goes to
    ``buf.sum``."""
    if (res is not None) != buf.residual:
        raise ValueError("buffers with residual take res, others do not")
    _check(buf._lib.noble_norm_fwd(buf._ref, buf._rows_of(x, "x"), buf._rows_of(res, "res"),
                                   buf._features(gain, "gain"), buf._features(bias, "bias"), *buf._out,
                                   None if buf.stats is None else buf.stats.data_ptr(), _stream(stream, buf)))
    return buf.y


def norm_backward(buf: NormBuffers, dy, s, gain=None, dstream=None, stream=None):
    """Gradients of norm_forward on the same buffers: ``buf.dx`` (of x, and of res), ``buf.dgain``,
    ``buf.dbias``.  ``s``: what was normed, ``buf.sum`` or x; ``dstream``: the gradient that reaches
    it by the residual stream."""
    if buf.stats is None:
        raise ValueError("buffers without gradients")
    _check(buf._lib.noble_norm_bwd(buf._ref, buf._rows_of(dy, "dy"), buf._rows_of(s, "s"), buf.stats.data_ptr(),
                                   buf._features(gain, "gain"), buf._rows_of(dstream, "dstream"),
                                   buf.dx.data_ptr(), buf.dgain.data_ptr(), buf.dbias.data_ptr(),
                                   buf.workspace.data_ptr(), buf.workspace_bytes, _stream(stream, buf)))
    return buf.dx


# ---------------------------------------------------------------- embedding
class EmbedBuffers:
    """Output ``y`` [T, d] of the embedding of T tokens by a table of ``vocab`` rows; with gradients
    ``dtable`` [vocab, d] (fp32) and its workspace."""

    def __init__(self, T, vocab, d, dtype, scale=1.0, device="cuda", with_grads=True):
        self.T, self.vocab, self.d = T, vocab, d
        self.desc = binding.EmbedDesc(T, vocab, d, scale, _code(dtype), 0)
        self.dtype = _TORCH[self.desc.dtype]
        self.y = torch.empty((T, d), dtype=self.dtype, device=device)
        self.device, self._index = _place(self.y)
        self._lib = binding.load()
        self._ref, self._tokens, self._rows, self._table = ctypes.byref(self.desc), (T,), (T, d), (vocab, d)
        self.dtable = None
        if with_grads:
            self.workspace_bytes = binding.load().noble_embed_bwd_workspace_bytes(self._ref)
            self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=device)
            self.dtable = torch.empty((vocab, d), dtype=torch.float32, device=device)


def embed_forward(buf: EmbedBuffers, ids, table, stream=None):
    """Scaled rows of table [vocab, d] by ids [T] (int32; negative: padding) into ``buf.y``."""
    _check(buf._lib.noble_embed_fwd(buf._ref, _at(ids, "ids", torch.int32, buf._tokens, buf.device),
                                    _at(table, "table", buf.dtype, buf._table, buf.device), buf.y.data_ptr(),
                                    _stream(stream, buf)))
    return buf.y


def embed_backward(buf: EmbedBuffers, ids, dy, stream=None):
    """The table's gradient into ``buf.dtable``, every row of it."""
    if buf.dtable is None:
        raise ValueError("buffers without gradients")
    _check(buf._lib.noble_embed_bwd(buf._ref, _at(ids, "ids", torch.int32, buf._tokens, buf.device),
                                    _at(dy, "dy", buf.dtype, buf._rows, buf.device), buf.dtable.data_ptr(),
                                    buf.workspace.data_ptr(), buf.workspace_bytes, _stream(stream, buf)))
    return buf.dtable
