"""The attention operators of ``libnoble.so`` for torch tensors: what stands between a
QKV and an output projection.

    training     rope_forward, attn_forward  /  attn_backward, rope_backward
    generation   kv_append, attn_paged, over a PagedCache

As in ``binding``, buffer classes allocate the caller-owned memory of one shape with
torch, functions check and marshal arguments, and every step runs in the library's
kernels.  Functions return views of their buffers, which the next call overwrites.
``include/noble.h`` defines each operator.

A QKV projection's output is packed by head: the n_q queries of a token, then its n_kv
keys, then its n_kv values, d features each.
"""
from __future__ import annotations

import ctypes
import math
import struct

import torch

from . import binding
from .binding import NOBLE_BF16, NOBLE_FP32, _check, _p, _stream_handle

NOBLE_ROPE_INTERLEAVED, NOBLE_ROPE_NORM = 1, 2
NOBLE_ATTN_CAUSAL, NOBLE_ATTN_SIMT_ONLY = 1, 2

_TORCH = {NOBLE_BF16: torch.bfloat16, NOBLE_FP32: torch.float32}
_PACK = struct.Struct("=Qqq").pack_into  # noble_heads
_HEADS = 24


def _code(dtype) -> int:
    return {"bf16": NOBLE_BF16, "fp32": NOBLE_FP32}[dtype] if isinstance(dtype, str) else dtype


class _Slots:
    """noble_heads arguments of a call, packed side by side."""

    def __init__(self, n):
        self.mem = (ctypes.c_char * (_HEADS * n))()
        base = ctypes.addressof(self.mem)
        self.at = [ctypes.c_void_p(base + _HEADS * i) for i in range(n)]

    def put(self, i, x, shape, dtype):
        """Tensor [T, n, d] as argument i; its features are next to each other."""
        if x.shape != shape or x.dtype is not dtype or not x.is_cuda:
            raise ValueError(f"expected a {dtype} CUDA tensor {list(shape)}, got {x.dtype} {list(x.shape)} on {x.device}")
        row, head, one = x.stride()
        if one != 1:
            raise ValueError("the features of a head have to be next to each other")
        _PACK(self.mem, _HEADS * i, x.data_ptr(), row, head)

    def raw(self, i, p, row, head):
        _PACK(self.mem, _HEADS * i, p, row, head)


def _flat(x, name, dtype, shape):
    """Address of a contiguous device tensor of the given shape; None stays None."""
    if x is None:
        return None
    if x.shape != shape or x.dtype is not dtype or not x.is_cuda or not x.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} CUDA tensor {list(shape)}, got {x.dtype} "
                         f"{list(x.shape)} on {x.device}")
    return x.data_ptr()


# ---------------------------------------------------------------- rotary positions
def rope_table(positions, rot, base=10000.0, factor=1.0, original=1.0, low_turns=0.0, high_turns=0.0, amplitude=1.0,
               device="cuda", stream=None):
    """cos and sin of every position and frequency, [positions, rot]; ``factor`` and what
    follows scale the frequencies by parts for longer contexts (noble_rope_table)."""
    table = torch.empty((positions, rot), dtype=torch.float32, device=device)
    s = binding.RopeScaling(base, factor, original, low_turns, high_turns, amplitude)
    _check(binding.load().noble_rope_table(positions, rot, ctypes.byref(s), _p(table), _stream_handle(stream)))
    return table


class RopeBuffers:
    """Outputs and workspace of the rotation (and norms) of T tokens' queries and keys.

    ``q`` [T, n_q, d] and ``k`` [T, n_kv, d]; with gradients ``dqkv``, laid out as the
    projection's output, of which ``dxq`` and ``dxk`` are the parts that rope_backward
    writes and ``dxv`` the place of the values' gradient, and ``dgain_q``, ``dgain_k``."""

    def __init__(self, T, n_q, n_kv, d, dtype, rot=None, positions=1, norm=True, eps=1e-6, interleaved=False,
                 device="cuda", with_grads=True):
        self.T, self.n_q, self.n_kv, self.d, self.rot = T, n_q, n_kv, d, d if rot is None else rot
        self.positions = positions
        flags = (NOBLE_ROPE_INTERLEAVED if interleaved else 0) | (NOBLE_ROPE_NORM if norm else 0)
        self.desc = binding.RopeDesc(T, n_q, n_kv, d, self.rot, positions, eps, _code(dtype), flags)
        self.dtype = _TORCH[self.desc.dtype]
        new = dict(dtype=self.dtype, device=device)
        self.q, self.k = torch.empty((T, n_q, d), **new), torch.empty((T, n_kv, d), **new)
        self._h = _Slots(7)
        self._ref = ctypes.byref(self.desc)
        self._q, self._k = (T, n_q, d), (T, n_kv, d)
        self._qkv, self._pos, self._table, self._gain = (T, (n_q + 2 * n_kv) * d), (T,), (positions, self.rot), (d,)
        step = d * (2 if self.desc.dtype == NOBLE_BF16 else 4)
        self._to_k, self._to_v = n_q * step, (n_q + n_kv) * step
        if with_grads:
            self.workspace_bytes = binding.load().noble_rope_bwd_workspace_bytes(self._ref)
            self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=device)
            self.dqkv = torch.empty((T, (n_q + 2 * n_kv) * d), **new)
            h = self.dqkv.view(T, n_q + 2 * n_kv, d)
            self.dxq, self.dxk, self.dxv = h[:, :n_q], h[:, n_q:n_q + n_kv], h[:, n_q + n_kv:]
            self.dgain_q, self.dgain_k = (torch.empty(d, dtype=torch.float32, device=device) for _ in range(2))

    def _put_qkv(self, qkv):
        """The queries, keys and values of a packed projection output as arguments 0 to 2."""
        if qkv.shape != self._qkv or qkv.dtype is not self.dtype or not qkv.is_cuda:
            raise ValueError(f"expected a {self.dtype} CUDA tensor {list(self._qkv)}, got {qkv.dtype} {list(qkv.shape)} on "
                             f"{qkv.device}")
        p, (row, one), d, mem = qkv.data_ptr(), qkv.stride(), self.d, self._h.mem
        if one != 1:
            raise ValueError("the rows of a projection's output have to be contiguous")
        _PACK(mem, 0, p, row, d)
        _PACK(mem, _HEADS, p + self._to_k, row, d)
        _PACK(mem, 2 * _HEADS, p + self._to_v, row, d)

    def _common(self, pos, table, gain_q, gain_k):
        return (_flat(pos, "pos", torch.int32, self._pos), _flat(table, "table", torch.float32, self._table),
                _flat(gain_q, "gain_q", torch.float32, self._gain), _flat(gain_k, "gain_k", torch.float32, self._gain))


def rope_forward(buf: RopeBuffers, qkv, pos, table, gain_q=None, gain_k=None, stream=None):
    """Normed and rotated queries and keys into ``buf.q`` and ``buf.k``."""
    buf._put_qkv(qkv)
    pos, table, gain_q, gain_k = buf._common(pos, table, gain_q, gain_k)
    h = buf._h
    h.put(3, buf.q, buf._q, buf.dtype)
    h.put(4, buf.k, buf._k, buf.dtype)
    _check(binding.load().noble_rope_fwd(buf._ref, h.at[0], h.at[1], pos, table, gain_q, gain_k, h.at[3], h.at[4],
                                         _stream_handle(stream)))
    return buf.q, buf.k


def rope_backward(buf: RopeBuffers, dq, dk, qkv, pos, table, gain_q=None, gain_k=None, stream=None):
    """Gradients of rope_forward: the parts ``buf.dxq``, ``buf.dxk`` of ``buf.dqkv``, and
    ``buf.dgain_q``, ``buf.dgain_k``."""
    buf._put_qkv(qkv)
    pos, table, gain_q, gain_k = buf._common(pos, table, gain_q, gain_k)
    h = buf._h
    h.put(3, dq, buf._q, buf.dtype)
    h.put(4, dk, buf._k, buf.dtype)
    h.put(5, buf.dxq, buf._q, buf.dtype)
    h.put(6, buf.dxk, buf._k, buf.dtype)
    _check(binding.load().noble_rope_bwd(buf._ref, h.at[3], h.at[4], h.at[0], h.at[1], pos, table, gain_q, gain_k,
                                         h.at[5], h.at[6], buf.dgain_q.data_ptr(), buf.dgain_k.data_ptr(),
                                         buf.workspace.data_ptr(), buf.workspace_bytes, _stream_handle(stream)))
    return buf.dxq, buf.dxk


# ---------------------------------------------------------------- the cache
class PagedCache:
    """Keys and values in pages, [pages, page_size, n_kv, d] each; ``k`` and ``v`` may be
    given, with any strides but a contiguous last dimension and the same for both."""

    def __init__(self, pages, page_size, n_kv, d, dtype, k=None, v=None, device="cuda"):
        self.pages, self.page_size, self.n_kv, self.d = pages, page_size, n_kv, d
        self.dtype = _TORCH[_code(dtype)]
        shape = (pages, page_size, n_kv, d)
        self.k = torch.empty(shape, dtype=self.dtype, device=device) if k is None else k
        self.v = torch.empty(shape, dtype=self.dtype, device=device) if v is None else v
        for x in (self.k, self.v):
            if x.shape != shape or x.dtype is not self.dtype or not x.is_cuda or x.stride(3) != 1:
                raise ValueError(f"expected a {self.dtype} CUDA tensor {list(shape)} of contiguous features")
        if self.k.stride() != self.v.stride():
            raise ValueError("the keys and the values of a cache need the same strides")
        self.c = binding.KvCache(self.k.data_ptr(), self.v.data_ptr(), pages, page_size, *self.k.stride()[:3])
        self._ref = ctypes.byref(self.c)


def kv_append(buf: RopeBuffers, cache: PagedCache, qkv, pos, slots, table, gain_q=None, gain_k=None, stream=None):
    """Normed and rotated queries into ``buf.q``; keys (normed and rotated) and values into
    the cache, token t at slots[t] = page * page_size + place (negative: not stored)."""
    if cache.n_kv != buf.n_kv or cache.d != buf.d or cache.dtype is not buf.dtype:
        raise ValueError("the cache has other heads or another type than the buffers")
    buf._put_qkv(qkv)
    pos, table, gain_q, gain_k = buf._common(pos, table, gain_q, gain_k)
    h = buf._h
    h.put(3, buf.q, buf._q, buf.dtype)
    _check(binding.load().noble_kv_append(buf._ref, h.at[0], h.at[1], h.at[2], pos,
                                          _flat(slots, "slots", torch.int64, buf._pos), table, gain_q, gain_k, h.at[3],
                                          cache._ref, _stream_handle(stream)))
    return buf.q


# ---------------------------------------------------------------- attention
class AttnBuffers:
    """Outputs and workspace of attention over T packed tokens of n_docs documents:
    ``o`` [T, n_q, d], ``lse`` [n_q, T]; with gradients ``dq``, ``dk``, ``dv`` and the
    backward's workspace.  ``dv`` may be given: the place of the values in a packed gradient."""

    def __init__(self, T, n_q, n_kv, d, dtype, n_docs=1, causal=True, window=0, scale=None, softcap=0.0, flags=0,
                 device="cuda", with_grads=True, dv=None):
        self.T, self.n_q, self.n_kv, self.d, self.n_docs = T, n_q, n_kv, d, n_docs
        flags |= NOBLE_ATTN_CAUSAL if causal else 0
        self.desc = binding.AttnDesc(T, n_docs, n_q, n_kv, d, window, 1.0 / math.sqrt(d) if scale is None else scale,
                                     softcap, _code(dtype), flags)
        self.dtype = _TORCH[self.desc.dtype]
        new = dict(dtype=self.dtype, device=device)
        self.o = torch.empty((T, n_q, d), **new)
        self.lse = torch.empty((n_q, T), dtype=torch.float32, device=device)
        self._h = _Slots(8)
        self._q, self._k, self._docs = (T, n_q, d), (T, n_kv, d), (n_docs + 1,)
        self._ref = ctypes.byref(self.desc)
        if with_grads:
            self.workspace_bytes = binding.load().noble_attn_bwd_workspace_bytes(self._ref)
            self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=device)
            self.dq, self.dk = torch.empty((T, n_q, d), **new), torch.empty((T, n_kv, d), **new)
            self.dv = torch.empty((T, n_kv, d), **new) if dv is None else dv

    def _inputs(self, q, k, v, doc_start, prefix, slope):
        h, t = self._h, self.dtype
        h.put(0, q, self._q, t)
        h.put(1, k, self._k, t)
        h.put(2, v, self._k, t)
        h.put(3, self.o, self._q, t)
        return (_flat(doc_start, "doc_start", torch.int32, self._docs), _flat(prefix, "prefix", torch.int32, (self.n_docs,)),
                _flat(slope, "slope", torch.float32, (self.n_q,)))


def attn_forward(buf: AttnBuffers, q, k, v, doc_start, prefix=None, slope=None, stream=None):
    """Attention of q [T, n_q, d] over k, v [T, n_kv, d] into ``buf.o``, and ``buf.lse``."""
    doc, pre, slo = buf._inputs(q, k, v, doc_start, prefix, slope)
    at = buf._h.at
    _check(binding.load().noble_attn_fwd(buf._ref, at[0], at[1], at[2], doc, pre, slo, at[3], buf.lse.data_ptr(),
                                         _stream_handle(stream)))
    return buf.o, buf.lse


def attn_backward(buf: AttnBuffers, d_o, q, k, v, doc_start, prefix=None, slope=None, stream=None):
    """Gradients of attn_forward, whose ``buf.o`` and ``buf.lse`` it reads, into ``buf.dq``,
    ``buf.dk`` and ``buf.dv``."""
    doc, pre, slo = buf._inputs(q, k, v, doc_start, prefix, slope)
    h, t = buf._h, buf.dtype
    h.put(4, d_o, buf._q, t)
    h.put(5, buf.dq, buf._q, t)
    h.put(6, buf.dk, buf._k, t)
    h.put(7, buf.dv, buf._k, t)
    at = h.at
    _check(binding.load().noble_attn_bwd(buf._ref, at[4], at[0], at[1], at[2], doc, pre, slo, at[3], buf.lse.data_ptr(),
                                         at[5], at[6], at[7], buf.workspace.data_ptr(), buf.workspace_bytes,
                                         _stream_handle(stream)))
    return buf.dq, buf.dk, buf.dv


class PagedBuffers:
    """Output and workspace of attention of n_seq sequences' newest q_len tokens over a
    cache: ``o`` [n_seq * q_len, n_q, d], and with_lse ``lse`` [n_seq * q_len, n_q].
    ``max_len``: no sequence is longer."""

    def __init__(self, n_seq, q_len, n_q, n_kv, d, dtype, max_len, window=0, scale=None, softcap=0.0, device="cuda",
                 with_lse=False):
        self.n_seq, self.rows, self.n_q, self.n_kv, self.d = n_seq, n_seq * q_len, n_q, n_kv, d
        self.desc = binding.PagedDesc(n_seq, q_len, n_q, n_kv, d, 0, max_len, window,
                                      1.0 / math.sqrt(d) if scale is None else scale, softcap, _code(dtype), 0)
        self.dtype = _TORCH[self.desc.dtype]
        self.o = torch.empty((self.rows, n_q, d), dtype=self.dtype, device=device)
        self.lse = torch.empty((self.rows, n_q), dtype=torch.float32, device=device) if with_lse else None
        self._h = _Slots(2)
        self._q, self._seqs = (self.rows, n_q, d), (n_seq,)
        self._ref = ctypes.byref(self.desc)
        self.workspace_bytes = binding.load().noble_attn_paged_workspace_bytes(self._ref)
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=device)


def attn_paged(buf: PagedBuffers, q, cache: PagedCache, page_table, kv_len, slope=None, stream=None):
    """Attention of q [n_seq * q_len, n_q, d] over the cache into ``buf.o``; row n of
    page_table [n_seq, pages of a sequence] lists the pages of sequence n, kv_len [n_seq]
    its tokens, the new ones included."""
    if cache.n_kv != buf.n_kv or cache.d != buf.d or cache.dtype is not buf.dtype:
        raise ValueError("the cache has other heads or another type than the buffers")
    h = buf._h
    h.put(0, q, buf._q, buf.dtype)
    h.put(1, buf.o, buf._q, buf.dtype)
    wide = page_table.shape[-1]
    buf.desc.max_pages = wide
    _check(binding.load().noble_attn_paged(
        buf._ref, h.at[0], cache._ref, _flat(page_table, "page_table", torch.int32, (buf.n_seq, wide)),
        _flat(kv_len, "kv_len", torch.int32, buf._seqs), _flat(slope, "slope", torch.float32, (buf.n_q,)), h.at[1],
        _p(buf.lse), buf.workspace.data_ptr(), buf.workspace_bytes, _stream_handle(stream)))
    return buf.o
