"""The attention half of a transformer block: NOBLE QKV projection, head norms and rotation,
attention, NOBLE output projection -- forward and backward for training on packed
documents, and one step of generation over a paged cache; a stack of them between its table of
tokens and its last norm; and the optimizer of its parameters.

Nothing is computed here: these keep buffers and call the operators in order.
"""
from __future__ import annotations

import torch

from . import attention as A, binding as B, layers as L


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


class Stack:
    """Attention halves one behind the other, from tokens to the last norm: the table's rows are the
    residual stream, each half reads a layer norm of it and adds its output.

    ``params`` of its calls: ``{"table": [vocab, d_model], "norms": [{"gain", "bias"}, ...], "blocks":
    [...]}``, with a norm more than blocks, and the blocks' as for ``AttentionBlock``.  Its options go to
    every half; all of them share one table of rotations, ``table`` if given."""

    def __init__(self, vocab, blocks, d_model, *heads, dtype="bf16", scale=1.0, eps=1e-5, **options):
        self.vocab, self.d_model, self.dtype, self.scale, self.eps = vocab, d_model, dtype, scale, eps
        if blocks < 0:
            raise ValueError(f"{blocks} blocks")
        self.blocks = []
        for _ in range(blocks):
            self.blocks.append(AttentionBlock(d_model, *heads, dtype=dtype, **options))
            options["table"] = self.blocks[0].table

    def _ends(self, T, with_grads):
        norm = dict(dtype=self.dtype, eps=self.eps, with_grads=with_grads)
        return {"embed": L.EmbedBuffers(T, self.vocab, self.d_model, self.dtype, scale=self.scale, with_grads=with_grads),
                "norms": [L.NormBuffers(T, self.d_model, residual=i > 0, **norm) for i in range(len(self.blocks) + 1)]}

    def _through(self, b, ids, params, half):
        """The last norm's output; half(i, x): block i's on x."""
        norms, stream = params["norms"], L.embed_forward(b["embed"], ids, params["table"])
        x = L.norm_forward(b["norms"][0], stream, norms[0]["gain"], norms[0]["bias"])
        for i in range(len(self.blocks)):
            n = b["norms"][i + 1]
            x = L.norm_forward(n, half(i, x), norms[i + 1]["gain"], norms[i + 1]["bias"], res=stream)
            stream = n.sum
        return x

    # ---------------------------------------------------------------- training
    def buffers(self, T, n_docs=1):
        """Buffers of a training step on T packed tokens."""
        return {**self._ends(T, True), "blocks": [blk.buffers(T, n_docs) for blk in self.blocks]}

    def forward(self, b, ids, params, pos, doc_start, prefix=None):
        return self._through(b, ids, params,
                             lambda i, x: self.blocks[i].forward(b["blocks"][i], x, params["blocks"][i], pos, doc_start, prefix))

    def backward(self, b, ids, dx, params, pos, doc_start, prefix=None):
        """Gradients of every parameter, in the layout of ``params``, after ``forward`` on the same buffers."""
        norms, blocks, dstream = [], [], None
        for i in range(len(self.blocks), -1, -1):
            n = b["norms"][i]
            dstream = L.norm_backward(n, dx, n.sum if i else b["embed"].y, params["norms"][i]["gain"], dstream)
            norms.insert(0, {"gain": n.dgain, "bias": n.dbias})
            if i:
                dx, g = self.blocks[i - 1].backward(b["blocks"][i - 1], b["norms"][i - 1].y, dstream, params["blocks"][i - 1], pos,
                                                    doc_start, prefix)
                blocks.insert(0, g)
        return {"table": L.embed_backward(b["embed"], ids, dstream), "norms": norms, "blocks": blocks}

    # ---------------------------------------------------------------- generation
    def caches(self, pages, page_size):
        return [blk.cache(pages, page_size) for blk in self.blocks]

    def step_buffers(self, n_seq, max_len, q_len=1):
        """Buffers of a step of n_seq sequences by q_len tokens each."""
        return {**self._ends(n_seq * q_len, False), "blocks": [blk.step_buffers(n_seq, max_len, q_len) for blk in self.blocks]}

    def step(self, b, caches, ids, params, pos, slots, page_table, kv_len):
        """The last norm's output for the newest tokens; their keys and values join the caches first."""
        return self._through(b, ids, params, lambda i, x: self.blocks[i].step(b["blocks"][i], caches[i], x, params["blocks"][i],
                                                                             pos, slots, page_table, kv_len))


class Update:
    """Optimizer of a Stack's parameters: orthogonalised momentum for the matrices of its
    projections, AdamW for everything else.  Keeps fp32 parameters and moments; the operands that
    the layers read (bf16, or the parameters themselves in fp32) are written in the same pass.

    ``multipliers``: arguments of ``binding.noble_linear_lr_multipliers``, whose rule then sets the
    learning rates of each projection's groups beside ``lr`` and ``lr_matrices``; ``{}`` are the paper's
    values (W_up, M, omega and phi train faster).  The paper has them for AdamW alone: ``gamma=0, gamma_M=0``
    leave W_up and M, whose steps are orthogonal here, at 1.  None: every multiplier is 1.

    ``precise``: 22 bits in the products of large matrices; without, their changes are about 1e-3 of
    their norm off, in fp32 parameters too (noble_muon_step)."""

    _MATRICES = {"W", "W_down", "W_up", "M"}
    _GRADS = {"W": "dW", "bias": "dbias", "W_down": "dW_down", "W_up": "dW_up", "M": "dM", "omega1": "domega1", "phi1": "dphi1",
              "omega2": "domega2", "phi2": "dphi2"}

    def __init__(self, params, grads, precise=False, multipliers=None):
        self.steps, self.precise, self.muon, self.adamw = 0, precise, [], []
        for matrix, p, g, mult in self._leaves(params, grads, multipliers):
            fp32 = p.dtype is torch.float32
            t = {"param": p if fp32 else p.float(), "param_bf16": None if fp32 else p, "grad": g, "decay": p.dim() == 2,
                 "lr_mult": mult}
            moments = ("momentum",) if matrix else ("exp_avg", "exp_avg_sq")
            t.update({k: torch.zeros_like(t["param"]) for k in moments})
            (self.muon if matrix else self.adamw).append(t)
        self.workspace = B.muon_workspace(self.muon, precise)

    @staticmethod
    def _rates(p, multipliers):
        """Learning-rate multipliers of a projection's parameters that are not 1."""
        if multipliers is None or p.get("W_down") is None:
            return {}
        (d_out, d_in), r = p["W"].shape, len(p["W_down"])
        dtype = "fp32" if p["W"].dtype is torch.float32 else "bf16"
        _, up, m, omega, phi = B.noble_linear_lr_multipliers(B.make_desc(1, d_in, d_out, r, dtype), **multipliers)
        return {"W_up": up, "M": m, "omega1": omega, "omega2": omega, "phi1": phi, "phi2": phi}

    def _leaves(self, params, grads, multipliers):
        yield False, params["table"], grads["table"], 1.0
        for p, g in zip(params["norms"], grads["norms"]):
            yield from ((False, p[k], g[k], 1.0) for k in ("gain", "bias"))
        for p, g in zip(params["blocks"], grads["blocks"]):
            yield from ((False, p[k], g[k], 1.0) for k in ("gain_q", "gain_k") if p.get(k) is not None and k in g)
            for name in ("qkv", "out"):
                rates = self._rates(p[name], multipliers)
                yield from ((k in self._MATRICES, p[name][k], g[name][d], rates.get(k, 1.0)) for k, d in self._GRADS.items()
                            if p[name].get(k) is not None)

    def step(self, lr, lr_matrices, weight_decay=0.01):
        """One step from the gradients that the Stack's buffers hold."""
        self.steps += 1
        B.noble_muon_step(self.muon, lr_matrices, weight_decay=weight_decay, precise=self.precise, workspace=self.workspace)
        B.noble_adamw_step(self.adamw, lr, weight_decay=weight_decay, step=self.steps)
