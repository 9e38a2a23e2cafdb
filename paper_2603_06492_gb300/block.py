"""The attention half of a transformer block: NOBLE QKV projection, head norms and rotation,
attention, NOBLE output projection -- forward and backward for training on packed
documents, and one step of generation over a paged cache.

Nothing is computed here: the block keeps buffers and calls the operators in order.
"""
from __future__ import annotations

import torch

from . import attention as A, binding as B


class AttentionBlock:
    """Sizes and options of a block.  ``params`` of its calls: ``{"qkv": ..., "out": ...}``, each
    a projection's parameters as for ``binding.forward``, and ``gain_q``, ``gain_k`` [d]."""

    def __init__(self, d_model, n_q, n_kv, d, r, dtype="bf16", rot=None, positions=4096, norm=True, causal=True, window=0,
                 softcap=0.0, table=None):
        self.d_model, self.n_q, self.n_kv, self.d, self.r, self.dtype = d_model, n_q, n_kv, d, r, dtype
        self.rope = dict(rot=d if rot is None else rot, positions=positions, norm=norm)
        self.scores = dict(window=window, softcap=softcap)
        self.causal = causal
        self.qkv_width = (n_q + 2 * n_kv) * d
        self.table = A.rope_table(positions, self.rope["rot"]) if table is None else table

    # ---------------------------------------------------------------- training
    def buffers(self, T, n_docs=1):
        """Buffers of a training step on T packed tokens."""
        heads = (self.n_q, self.n_kv, self.d, self.dtype)
        b = {"qkv": B.NobleLinearBuffers(T, self.d_model, self.qkv_width, self.r, self.dtype),
             "out": B.NobleLinearBuffers(T, self.n_q * self.d, self.d_model, self.r, self.dtype),
             "rope": A.RopeBuffers(T, *heads, **self.rope)}
        # the values' gradient goes to its place in the projection's
        b["attn"] = A.AttnBuffers(T, *heads, n_docs=n_docs, causal=self.causal, **self.scores, dv=b["rope"].dxv)
        return b

    def _values(self, qkv):
        return qkv.view(-1, self.n_q + 2 * self.n_kv, self.d)[:, self.n_q + self.n_kv:]

    def forward(self, b, x, params, pos, doc_start, prefix=None):
        qkv = B.forward(b["qkv"], x, params["qkv"])
        q, k = A.rope_forward(b["rope"], qkv, pos, self.table, params.get("gain_q"), params.get("gain_k"))
        o, _ = A.attn_forward(b["attn"], q, k, self._values(qkv), doc_start, prefix)
        return B.forward(b["out"], o.view(-1, self.n_q * self.d), params["out"])

    def backward(self, b, x, dy, params, pos, doc_start, prefix=None):
        """dx and the gradients of every parameter, after ``forward`` on the same buffers."""
        qkv, rope, attn = b["qkv"].y, b["rope"], b["attn"]
        d_o, out = B.backward(b["out"], attn.o.view(-1, self.n_q * self.d), dy, params["out"])
        dq, dk, _ = A.attn_backward(attn, d_o.view(-1, self.n_q, self.d), rope.q, rope.k, self._values(qkv), doc_start,
                                    prefix)
        A.rope_backward(rope, dq, dk, qkv, pos, self.table, params.get("gain_q"), params.get("gain_k"))
        dx, inner = B.backward(b["qkv"], x, rope.dqkv, params["qkv"])
        grads = {"qkv": inner, "out": out}
        if self.rope["norm"]:
            grads.update(gain_q=rope.dgain_q, gain_k=rope.dgain_k)
        return dx, grads

    # ---------------------------------------------------------------- generation
    def cache(self, pages, page_size):
        return A.PagedCache(pages, page_size, self.n_kv, self.d, self.dtype)

    def step_buffers(self, n_seq, max_len, q_len=1):
        """Buffers of a step of n_seq sequences by q_len tokens each."""
        T, heads, flag = n_seq * q_len, (self.n_q, self.n_kv, self.d, self.dtype), B.NOBLE_FLAG_INFERENCE
        return {"qkv": B.NobleLinearBuffers(T, self.d_model, self.qkv_width, self.r, self.dtype, with_grads=False, flags=flag),
                "out": B.NobleLinearBuffers(T, self.n_q * self.d, self.d_model, self.r, self.dtype, with_grads=False, flags=flag),
                "rope": A.RopeBuffers(T, *heads, **self.rope, with_grads=False),
                "paged": A.PagedBuffers(n_seq, q_len, *heads, max_len=max_len, **self.scores)}

    def step(self, b, cache, x, params, pos, slots, page_table, kv_len):
        """The newest tokens' outputs; their keys and values join the cache first."""
        qkv = B.forward(b["qkv"], x, params["qkv"])
        q = A.kv_append(b["rope"], cache, qkv, pos, slots, self.table, params.get("gain_q"), params.get("gain_k"))
        o = A.attn_paged(b["paged"], q, cache, page_table, kv_len)
        return B.forward(b["out"], o.view(-1, self.n_q * self.d), params["out"])

    def fill(self, b, cache, qkv, pos, slots, params):
        """Keys and values of prompts that ``forward`` has read into the cache; ``b``: RopeBuffers
        of as many tokens."""
        A.kv_append(b, cache, qkv, pos, slots, self.table, params.get("gain_q"), params.get("gain_k"))


def page_slots(page_table, seq, pos, page_size):
    """Slots of tokens at ``pos`` of sequences ``seq`` (int64 tensors)."""
    return page_table[seq, pos // page_size].to(torch.int64) * page_size + pos % page_size
