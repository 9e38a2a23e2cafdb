"""The measured cases of the attention operators, through their public entry points.

A case is one call, or one forward and backward, on buffers that a program keeps.  Kinds:

    "rope"    per-head RMS norm of the queries and keys and their rotation by position,
              read from the packed output of a QKV projection; with "step" also the
              gradients with respect to that output and to the norms' gains
    "append"  the same on new tokens of a serving batch, the keys and values written
              into the pages of a cache on the way
    "attn"    attention over packed documents (causal, windowed, with a prefix that all
              see, capped scores, a bias by distance); with "step" also dq, dk and dv
    "paged"   attention of the newest tokens of a serving batch over that cache

The plain forms below are elementary torch operations in 32 bits.  Sizes are those of the
package's configurations (1024- and 2048-wide decoders, a 768-wide ViT of 197 tokens per
image) or generic ones of the same ranges.  Lengths of documents and of cached sequences
come from the case ("layout"), so that the work does too; everything else from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

PAD = -1.0e30  # scores of places that nothing sees, before they are set to exactly zero


# ---------------------------------------------------------------- cases
def _rope(T, n_q, n_kv, d, rot, dtype="bf16", interleaved=False, norm=True, step=True, name=None):
    c = {"kind": "rope", "T": T, "n_q": n_q, "n_kv": n_kv, "d": d, "rot": rot, "dtype": dtype,
         "interleaved": interleaved, "norm": norm, "step": step}
    return {**c, "name": name} if name else c


def _append(T, n_q, n_kv, d, rot, page, dtype="bf16", interleaved=False, norm=True, name=None):
    c = {"kind": "append", "T": T, "n_q": n_q, "n_kv": n_kv, "d": d, "rot": rot, "page": page, "dtype": dtype,
         "interleaved": interleaved, "norm": norm}
    return {**c, "name": name} if name else c


def _attn(T, n_q, n_kv, d, docs, layout, dtype="bf16", causal=True, window=0, prefix=False, softcap=0.0, alibi=False,
          pad=0, step=True, name=None):
    c = {"kind": "attn", "T": T, "n_q": n_q, "n_kv": n_kv, "d": d, "docs": docs, "layout": layout, "dtype": dtype,
         "causal": causal, "window": window, "prefix": prefix, "softcap": softcap, "alibi": alibi, "pad": pad,
         "step": step}
    return {**c, "name": name} if name else c


def _paged(seqs, q_len, n_q, n_kv, d, page, longest, layout, dtype="bf16", window=0, softcap=0.0, alibi=False,
           name=None):
    c = {"kind": "paged", "seqs": seqs, "q_len": q_len, "n_q": n_q, "n_kv": n_kv, "d": d, "page": page,
         "longest": longest, "layout": layout, "dtype": dtype, "window": window, "softcap": softcap, "alibi": alibi}
    return {**c, "name": name} if name else c


def listed():
    return [
        # the fp32 mode of a small model, as a check of a training run: launches and gaps
        _rope(256, 2, 2, 64, 64, "fp32", name="rope-fp32-tiny-step"),
        # training the 2048-wide decoder: 16 sequences of 1024 tokens
        _rope(16384, 16, 16, 128, 128, name="rope-large-step"),
        # generating: one token of each of 24 sequences, grouped heads
        _append(24, 16, 4, 128, 128, 64, name="append-decode-24"),
        # reading prompts of no particular length, part of each head rotated in pairs
        _append(7001, 16, 16, 64, 32, 16, interleaved=True, norm=False, name="append-prompt-7001"),
        # the fp32 mode on one 1024-token sequence of the 1024-wide decoder
        _attn(1024, 16, 16, 64, 1, 0, "fp32", name="attn-fp32-sequence-step"),
        # training the 1024-wide decoder: 8 sequences of 1024 tokens
        _attn(8192, 16, 16, 64, 8, 0, name="attn-base-step"),
        # training a ViT: 64 images of 197 tokens, nothing masked within an image
        _attn(64 * 197, 12, 12, 64, 64, 0, causal=False, name="attn-vit-64-images-step"),
        # packed text of no particular length, each document with a prefix that all of it
        # sees, capped scores, grouped heads, and rows at the end that belong to nothing
        _attn(7001, 16, 4, 128, 11, 5, prefix=True, softcap=30.0, pad=37, name="attn-ragged-prefix-step"),
        # one long document of the 2048-wide decoder
        _attn(16384, 16, 16, 128, 1, 0, name="attn-long-step"),
        # generating with the 1024-wide decoder: 24 sequences up to its 1024 positions
        _paged(24, 1, 16, 16, 64, 16, 1024, 3, name="paged-decode-24"),
        # four proposed tokens checked at once on one long context, grouped heads
        _paged(1, 4, 16, 4, 128, 64, 131072, 0, name="paged-check-4-long"),
        # a full serving batch of long ragged contexts, grouped heads
        _paged(64, 1, 32, 4, 128, 64, 32768, 7, name="paged-decode-64-long"),
    ]


def _log_uniform(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))


def _heads(rng, most=32):
    n_kv = rng.choice((1, 2, 3, 4, 8, 12, 16))
    group = rng.choice((1, 1, 2, 4, 7, 8))
    return min(n_kv * group, most) // n_kv * n_kv or n_kv, n_kv


def draw(rng):
    kind = rng.choice(("rope", "append", "attn", "attn", "paged", "paged"))
    dtype = "fp32" if rng.random() < 0.2 else "bf16"
    d = rng.choice((32, 64, 64, 80, 96, 128, 128))
    n_q, n_kv = _heads(rng)
    if kind in ("rope", "append"):
        T = _log_uniform(rng, 1, 16384)
        rot = rng.choice((d, d, d // 2, d // 4))
        if kind == "rope":
            return _rope(T, n_q, n_kv, d, rot, dtype, rng.random() < 0.3, rng.random() < 0.7, rng.random() < 0.7)
        return _append(T, n_q, n_kv, d, rot, rng.choice((1, 16, 48, 64, 128)), dtype, rng.random() < 0.3,
                       rng.random() < 0.7)
    softcap = rng.choice((0.0, 0.0, 15.0, 50.0))
    if kind == "paged":
        while True:
            seqs = _log_uniform(rng, 1, 128)
            c = _paged(seqs, rng.choice((1, 1, 1, 2, 5, 8)), n_q, n_kv, d, rng.choice((16, 48, 64, 128)),
                       _log_uniform(rng, 1, 131072), rng.randrange(1000), dtype, rng.choice((0, 0, 128, 1000)),
                       softcap, rng.random() < 0.25)
            # the plain form's gathered copies, and no more work than the largest listed case
            if seqs * c["longest"] * n_kv * d <= 1e9 and seqs * c["q_len"] * n_q * c["longest"] <= 5e8:
                return c
    while True:
        T = _log_uniform(rng, 1, 16384 if dtype == "bf16" else 4096)
        docs = min(T, rng.choice((1, 1, 2, 5, 16, 64)))
        pad = rng.choice((0, 0, 1, 50)) if T > 100 else 0
        causal = rng.random() < 0.8
        c = _attn(T, n_q, n_kv, d, docs, rng.randrange(1000), dtype, causal, rng.choice((0, 0, 100, 1024)),
                  causal and rng.random() < 0.3, softcap, rng.random() < 0.25, pad, rng.random() < 0.75)
        longest = max(_doc_lengths(c))
        # no more work than the largest listed case, and the plain form's score matrices
        top = 5e10 if dtype == "fp32" else 3.8e12
        if len(_doc_lengths(c)) * n_q * longest ** 2 <= 4.3e9 and work(c)["flops"] <= top:
            return c


def _doc_lengths(c):
    """Lengths of the case's documents: even ones (layout 0) or ragged ones, some empty."""
    n, total = c["docs"], c["T"] - c["pad"]
    if c["layout"] == 0:
        assert total % n == 0
        return [total // n] * n
    rng = random.Random(c["layout"])
    cuts = sorted(rng.randint(0, total) for _ in range(n - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [total])]


def _prefixes(c):
    rng = random.Random(c["layout"] + 1)
    return [rng.randint(0, n) for n in _doc_lengths(c)]


def _kv_lengths(c):
    """Tokens in the cache of each sequence, the newest included; one of them the longest."""
    rng = random.Random(c["layout"])
    out = [rng.randint(min(c["q_len"], c["longest"]), c["longest"]) for _ in range(c["seqs"])]
    out[rng.randrange(c["seqs"])] = c["longest"]
    return out


# ---------------------------------------------------------------- inputs
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


class _Random:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, shape, dtype, std=1.0):
        return (torch.randn(shape, generator=self.g, device="cuda") * std).to(dtype)

    def around_one(self, shape):
        return 1.0 + 0.2 * torch.randn(shape, generator=self.g, device="cuda")

    def perm(self, n):
        return torch.randperm(n, generator=self.g, device="cuda")

    def ints(self, n, hi):
        return torch.randint(0, hi, (n,), generator=self.g, device="cuda")


POSITIONS = 32768  # of the rotation tables


def _table(rot):
    """cos and sin of each position and frequency, [positions][rot]: rot / 2 cosines, then as many sines."""
    freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(POSITIONS, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.cat([a.cos(), a.sin()], 1).float()


EPS = 1e-6


def _split(c, qkv):
    T, nq, nkv, d = c["T"], c["n_q"], c["n_kv"], c["d"]
    h = qkv.view(T, nq + 2 * nkv, d)
    return h[:, :nq], h[:, nq:nq + nkv], h[:, nq + nkv:]


def _tensors(c, seed):
    """The device tensors of a case."""
    r, dt, d, nq, nkv = _Random(seed), _dtype(c), c["d"], c["n_q"], c["n_kv"]
    s = {}
    if c["kind"] in ("rope", "append"):
        T = c["T"]
        s["qkv"] = r.normal((T, (nq + 2 * nkv) * d), dt)
        s["gain_q"] = r.around_one((d,)) if c["norm"] else None
        s["gain_k"] = r.around_one((d,)) if c["norm"] else None
        s["table"] = _table(c["rot"])
        if c["kind"] == "rope":
            # sequences of 1024 tokens, packed
            s["pos"] = (torch.arange(T, device="cuda") % 1024).int()
            if c["step"]:
                s["dq"] = r.normal((T, nq, d), dt)
                s["dk"] = r.normal((T, nkv, d), dt)
        else:
            # anywhere in their contexts, on pages of a pool that others use too
            s["pos"] = r.ints(T, POSITIONS).int()
            pages = -(-(T + 256) // c["page"])
            s["k_cache"] = r.normal((pages, c["page"], nkv, d), dt)
            s["v_cache"] = r.normal((pages, c["page"], nkv, d), dt)
            s["slots"] = r.perm(pages * c["page"])[:T].contiguous()
    elif c["kind"] == "attn":
        T = c["T"]
        # queries and keys out of their norms and rotation; values in place in the projection's output
        s["q"], s["k"] = r.normal((T, nq, d), dt, 1.2), r.normal((T, nkv, d), dt, 1.2)
        s["v"] = r.normal((T, (nq + 2 * nkv) * d), dt).view(T, nq + 2 * nkv, d)[:, nq + nkv:]
        if c["step"]:
            s["do"] = r.normal((T, nq, d), dt)
        lens = _doc_lengths(c)
        s["doc_start"] = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
        s["prefix"] = torch.tensor(_prefixes(c), dtype=torch.int32, device="cuda") if c["prefix"] else None
        s["slopes"] = _slopes(nq) if c["alibi"] else None
    else:
        lens, page = _kv_lengths(c), c["page"]
        most = -(-c["longest"] // page)
        need = [-(-n // page) for n in lens]
        pages = sum(need) + 3
        s["q"] = r.normal((c["seqs"] * c["q_len"], nq, d), dt, 1.2)
        s["k_cache"] = r.normal((pages, page, nkv, d), dt, 1.2)
        s["v_cache"] = r.normal((pages, page, nkv, d), dt)
        order = r.perm(pages).int()
        table = torch.zeros((c["seqs"], most), dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = order[at:at + n]
            at += n
        s["page_table"] = table
        s["kv_len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["slopes"] = _slopes(nq) if c["alibi"] else None
    return s


def _slopes(n):
    """Slopes of the distance bias: a geometric sequence over the heads."""
    return torch.tensor([2.0 ** (-8.0 * (i + 1) / n) for i in range(n)], dtype=torch.float32, device="cuda")


def prepare(case, seed):
    c = case
    s = _tensors(c, seed)
    s["case"] = c
    if c["kind"] == "attn":
        s["longest"] = max(_doc_lengths(c))
    if own:
        from paper_2603_06492_gb300 import attention as A
        dims = (c["n_q"], c["n_kv"], c["d"], c["dtype"])
        if c["kind"] in ("rope", "append"):
            s["buf"] = A.RopeBuffers(c["T"], *dims, rot=c["rot"], positions=POSITIONS, norm=c["norm"], eps=EPS,
                                     interleaved=c["interleaved"], with_grads=c.get("step", False))
            if c["kind"] == "append":
                s["cache"] = A.PagedCache(*s["k_cache"].shape, c["dtype"], k=s["k_cache"], v=s["v_cache"])
        elif c["kind"] == "attn":
            s["buf"] = A.AttnBuffers(c["T"], *dims, n_docs=c["docs"], causal=c["causal"], window=c["window"],
                                     softcap=c["softcap"], with_grads=c["step"])
        else:
            s["cache"] = A.PagedCache(*s["k_cache"].shape, c["dtype"], k=s["k_cache"], v=s["v_cache"])
            s["buf"] = A.PagedBuffers(c["seqs"], c["q_len"], *dims, max_len=c["longest"], window=c["window"],
                                      softcap=c["softcap"])
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(c, s)
    return {"rope": _plain_rope, "append": _plain_append, "attn": _plain_attn, "paged": _plain_paged}[c["kind"]](c, s)


def _run_own(c, s):
    from paper_2603_06492_gb300 import attention as A
    if c["kind"] == "rope":
        b, x = s["buf"], (s["qkv"], s["pos"], s["table"], s["gain_q"], s["gain_k"])
        out = {}
        out["q"], out["k"] = A.rope_forward(b, *x)
        if c["step"]:
            out["dxq"], out["dxk"] = A.rope_backward(b, s["dq"], s["dk"], *x)
            if c["norm"]:
                out["dgain_q"], out["dgain_k"] = b.dgain_q, b.dgain_k
        return out
    if c["kind"] == "append":
        yq = A.kv_append(s["buf"], s["cache"], s["qkv"], s["pos"], s["slots"], s["table"], s["gain_q"], s["gain_k"])
        return {"q": yq, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if c["kind"] == "attn":
        b = s["buf"]
        o, lse = A.attn_forward(b, s["q"], s["k"], s["v"], s["doc_start"], s["prefix"], s["slopes"])
        out = {"o": o, "lse": lse}
        if c["step"]:
            out["dq"], out["dk"], out["dv"] = A.attn_backward(b, s["do"], s["q"], s["k"], s["v"], s["doc_start"],
                                                              s["prefix"], s["slopes"])
        return out
    return {"o": A.attn_paged(s["buf"], s["q"], s["cache"], s["page_table"], s["kv_len"], s["slopes"])}


def _rotate(c, x, cs, sn):
    """The first `rot` features of each head, in pairs, by the angle of (cos, sin)."""
    rot = c["rot"]
    if c["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cs - b * sn, b * cs + a * sn], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cs - b * sn, b * cs + a * sn], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _angles(c, s):
    cs, sn = s["table"][s["pos"].long()].split(c["rot"] // 2, -1)
    return cs[:, None], sn[:, None]


def _norm_rotate(c, x, gain, cs, sn):
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain
    return _rotate(c, x, cs, sn)


def _norm_rotate_grad(c, x, gain, dy, cs, sn):
    x, dn = x.float(), _rotate(c, dy.float(), cs, -sn)
    if gain is None:
        return dn, None
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    xh = x * r
    g = dn * gain
    return r * (g - xh * (g * xh).mean(-1, keepdim=True)), (dn * xh).sum((0, 1))


def _plain_rope(c, s):
    dt = _dtype(c)
    q, k, _ = _split(c, s["qkv"])
    cs, sn = _angles(c, s)
    out = {"q": _norm_rotate(c, q, s["gain_q"], cs, sn).to(dt), "k": _norm_rotate(c, k, s["gain_k"], cs, sn).to(dt)}
    if c["step"]:
        dxq, dgq = _norm_rotate_grad(c, q, s["gain_q"], s["dq"], cs, sn)
        dxk, dgk = _norm_rotate_grad(c, k, s["gain_k"], s["dk"], cs, sn)
        out["dxq"], out["dxk"] = dxq.to(dt), dxk.to(dt)
        if c["norm"]:
            out["dgain_q"], out["dgain_k"] = dgq, dgk
    return out


def _plain_append(c, s):
    dt = _dtype(c)
    q, k, v = _split(c, s["qkv"])
    cs, sn = _angles(c, s)
    s["k_cache"].view(-1, c["n_kv"], c["d"])[s["slots"]] = _norm_rotate(c, k, s["gain_k"], cs, sn).to(dt)
    s["v_cache"].view(-1, c["n_kv"], c["d"])[s["slots"]] = v
    return {"q": _norm_rotate(c, q, s["gain_q"], cs, sn).to(dt), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _score(c, s, i, j):
    """The cap and the bias of scaled scores, as a function, for query and key positions i and j."""
    cap = c["softcap"]

    def f(x):
        if cap:
            x = cap * torch.tanh(x / cap)
        if s["slopes"] is not None:
            x = x - s["slopes"].view(1, -1, 1, 1) * (i - j).abs().float()
        return x
    return f


def _plain_attn(c, s):
    dt, T, nq, nkv, d = _dtype(c), c["T"], c["n_q"], c["n_kv"], c["d"]
    G, L, n = nq // nkv, s["longest"], c["docs"]
    start = s["doc_start"].long()
    lens = start[1:] - start[:-1]
    at = torch.arange(L, device="cuda")
    real = at < lens[:, None]                                   # [n][L]
    rows = torch.where(real, start[:-1, None] + at, 0)          # token of each padded place

    def padded(x, rep=1):                                       # [T][h][d] -> [n][h * rep][L][d]
        x = (x.float()[rows] * real[..., None, None]).transpose(1, 2)
        return x.repeat_interleave(rep, 1) if rep > 1 else x

    to = torch.where(real, rows, T)                             # one more row takes the padding

    def packed(x, empty=0.0):                                   # back to [T][h][d]
        out = torch.full((T + 1, x.shape[1], x.shape[3]), empty, device="cuda")
        out[to] = x.transpose(1, 2)
        return out[:T]

    q, k, v = padded(s["q"]), padded(s["k"], G), padded(s["v"], G)
    i, j = at[:, None], at[None, :]
    seen = real[:, None, :, None] & real[:, None, None, :]
    if c["causal"]:
        ok = (j <= i)[None, None]
        if s["prefix"] is not None:
            ok = ok | (j < s["prefix"].view(-1, 1, 1, 1))
        seen = seen & ok
    if c["window"]:
        seen = seen & (i - j < c["window"])
        if not c["causal"]:
            seen = seen & (j - i < c["window"])
    scale = 1.0 / math.sqrt(d)
    z = _score(c, s, i, j)((q @ k.transpose(-1, -2)) * scale)
    z = torch.where(seen, z, PAD)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - top) * seen
    total = p.sum(-1, keepdim=True)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    p = p / torch.where(total > 0, total, 1.0)
    o = p @ v
    out = {"o": packed(o).to(dt), "lse": packed(lse, -math.inf)[..., 0].t().contiguous()}
    if not c["step"]:
        return out
    do = padded(s["do"])
    dv = p.transpose(-1, -2) @ do
    dz = p * (do @ v.transpose(-1, -2) - (do * o).sum(-1, keepdim=True))
    if c["softcap"]:
        x = (q @ k.transpose(-1, -2)) * scale
        dz = dz * (1.0 - torch.tanh(x / c["softcap"]).square())
    dq, dk = dz @ k * scale, dz.transpose(-1, -2) @ q * scale
    shared = lambda x: x.view(n, nkv, G, L, d).sum(2)  # noqa: E731
    out["dq"], out["dk"], out["dv"] = packed(dq).to(dt), packed(shared(dk)).to(dt), packed(shared(dv)).to(dt)
    return out


def _plain_paged(c, s):
    dt, nq, nkv, d, n, m = _dtype(c), c["n_q"], c["n_kv"], c["d"], c["seqs"], c["q_len"]
    L = c["longest"]
    kv = [x[s["page_table"].long()].flatten(1, 2)[:, :L].float().transpose(1, 2) for x in (s["k_cache"], s["v_cache"])]
    j = torch.arange(L, device="cuda")
    i = (s["kv_len"].long()[:, None] - m + torch.arange(m, device="cuda"))[:, None, :, None]   # [n][1][m][1]
    seen = j <= i
    if c["window"]:
        seen = seen & (i - j < c["window"])
    q = s["q"].float().view(n, m, nkv, nq // nkv, d).permute(0, 2, 3, 1, 4)                     # [n][kv][g][m][d]
    z = (q.flatten(2, 3) @ kv[0].transpose(-1, -2) / math.sqrt(d)).view(n, nq, m, L)
    z = torch.where(seen, _score(c, s, i, j)(z), PAD)
    p = torch.exp(z - z.amax(-1, keepdim=True)) * seen
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    v = kv[1] * (j < s["kv_len"][:, None])[:, None, :, None]
    o = (p.view(n, nkv, nq // nkv * m, L) @ v).view(n, nq, m, d)
    return {"o": o.transpose(1, 2).reshape(n * m, nq, d).to(dt)}


# ---------------------------------------------------------------- what a pass cannot do without
def _pairs(c):
    """Visible (query, key) pairs of one head of an "attn" case."""
    total, w = 0, c["window"]
    pre = _prefixes(c) if c["prefix"] else [0] * c["docs"]
    for n, p in zip(_doc_lengths(c), pre):
        if not w and not p:
            total += n * (n + 1) // 2 if c["causal"] else n * n
        elif not w:
            total += p * p + (n * (n + 1) - p * (p + 1)) // 2
        else:
            for i in range(n):
                hi = max(i + 1, p) if c["causal"] else min(n, i + w)
                total += max(0, hi - max(0, i - w + 1))
    return total


def work(case):
    c = case
    es, nq, nkv, d = (2 if c["dtype"] == "bf16" else 4), c["n_q"], c["n_kv"], c["d"]
    if c["kind"] in ("rope", "append"):
        T = c["T"]
        b = 4.0 * T + 4.0 * min(T, 1024 if c["kind"] == "rope" else T) * c["rot"] + (8.0 * d if c["norm"] else 0.0)
        flops = T * (nq + nkv) * (3.0 * c["rot"] + (4.0 * d if c["norm"] else 0.0))
        if c["kind"] == "append":
            b += 8.0 * T + es * T * d * (2.0 * nq + 4.0 * nkv)
        else:
            b += 2.0 * es * T * d * (nq + nkv)
            if c["step"]:
                b += 2.0 * es * T * d * (nq + nkv) + (8.0 * d if c["norm"] else 0.0)
                flops *= 3.0
        return {"bytes": b, "flops": flops}
    if c["kind"] == "attn":
        T = c["T"]
        b = es * T * d * (2.0 * nq + 2.0 * nkv) + 4.0 * T * nq
        if c["step"]:
            b += es * T * d * (2.0 * nq + 2.0 * nkv)
        return {"bytes": b, "flops": (14.0 if c["step"] else 4.0) * d * nq * _pairs(c)}
    keys = seen = 0
    for n in _kv_lengths(c):
        rows = range(n - c["q_len"], n)
        lo = max(0, rows[0] - c["window"] + 1) if c["window"] else 0
        keys += n - lo
        seen += sum(max(0, i + 1 - (max(0, i - c["window"] + 1) if c["window"] else 0)) for i in rows)
    b = es * d * (2.0 * nkv * keys + 2.0 * nq * c["seqs"] * c["q_len"]) + 4.0 * keys / c["page"] + 4.0 * c["seqs"]
    return {"bytes": b, "flops": 4.0 * d * nq * seen}


# ---------------------------------------------------------------- 64-bit results
def exact(case, seed):
    c = case
    s = _tensors(c, seed)
    if c["kind"] in ("rope", "append"):
        return _exact_rope(c, s)
    if c["kind"] == "attn":
        # 64-bit products run at about a TFLOP/s
        if c["docs"] * c["n_q"] * max(_doc_lengths(c)) ** 2 * c["d"] > 3e11:
            return None
        return _exact_attn(c, s)
    return _exact_paged(c, s)


def _exact_rope(c, s):
    T, d, rot = c["T"], c["d"], c["rot"]
    half = rot // 2
    # the rotation as one matrix per token, [T][d][d]
    first = torch.arange(0, rot, 2, device="cuda") if c["interleaved"] else torch.arange(half, device="cuda")
    second = first + (1 if c["interleaved"] else half)
    t = s["table"].double()[s["pos"].long()]

    def turn(x, sign):
        y = x.clone()
        cs, sn = t[:, None, :half], sign * t[:, None, half:]
        y[..., first] = x[..., first] * cs - x[..., second] * sn
        y[..., second] = x[..., first] * sn + x[..., second] * cs
        return y

    x = s["qkv"].double().view(T, -1, d)
    nq, nkv = c["n_q"], c["n_kv"]
    out = {}
    for name, part, gain in (("q", x[:, :nq], s["gain_q"]), ("k", x[:, nq:nq + nkv], s["gain_k"])):
        if gain is not None:
            size = (part.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt()
            y = turn(part / size * gain.double(), 1.0)
        else:
            y = turn(part, 1.0)
        out[name] = y
        if c.get("step"):
            w = turn(s["d" + name].double(), -1.0)
            if gain is not None:
                out["dgain_" + name] = (w * part / size).sum((0, 1))
                gw = w * gain.double()
                w = gw / size - part * (gw * part).sum(-1, keepdim=True) / (d * size.pow(3))
            out["dx" + name] = w
    if c["kind"] == "append":
        cache = {n: s[n].double().view(-1, nkv, d) for n in ("k_cache", "v_cache")}
        cache["k_cache"].index_copy_(0, s["slots"], out.pop("k"))
        cache["v_cache"].index_copy_(0, s["slots"], x[:, nq + nkv:])
        out.update({n: t.view(s[n].shape) for n, t in cache.items()})
    return out


def _exact_attn(c, s):
    T, nq, nkv, d = c["T"], c["n_q"], c["n_kv"], c["d"]
    f64 = dict(dtype=torch.float64, device="cuda")
    o, dq = torch.zeros((T, nq, d), **f64), torch.zeros((T, nq, d), **f64)
    dk, dv = torch.zeros((T, nkv, d), **f64), torch.zeros((T, nkv, d), **f64)
    lse = torch.full((nq, T), -math.inf, **f64)
    start = s["doc_start"].tolist()
    pre = s["prefix"].tolist() if s["prefix"] is not None else None
    cap, w = c["softcap"], c["window"]
    for n, (a, b) in enumerate(zip(start, start[1:])):
        if a == b:
            continue
        far = torch.arange(b - a, device="cuda")[:, None] - torch.arange(b - a, device="cuda")  # query minus key
        hidden = torch.zeros_like(far, dtype=torch.bool)
        if c["causal"]:
            hidden |= far < 0
            if pre:
                hidden[:, :pre[n]] = False
        if w:
            hidden |= far >= w
            if not c["causal"]:
                hidden |= far <= -w
        for h in range(nq):
            g = h // (nq // nkv)
            q, k, v = s["q"][a:b, h].double(), s["k"][a:b, g].double(), s["v"][a:b, g].double()
            z = q @ k.T / math.sqrt(d)
            t = None
            if cap:
                t = torch.tanh(z / cap)
                z = cap * t
            if s["slopes"] is not None:
                z = z - float(s["slopes"][h]) * far.abs()
            z = z.masked_fill(hidden, -math.inf)
            lse[h, a:b] = torch.logsumexp(z, -1)
            p = torch.exp(z - lse[h, a:b, None])
            o[a:b, h] = p @ v
            if c["step"]:
                do = s["do"][a:b, h].double()
                dv[a:b, g] += p.T @ do
                dp = do @ v.T
                dz = p * (dp - (p * dp).sum(-1, keepdim=True))
                if cap:
                    dz = dz * (1.0 - t * t)
                dq[a:b, h] = dz @ k / math.sqrt(d)
                dk[a:b, g] += dz.T @ q / math.sqrt(d)
    out = {"o": o, "lse": lse}
    if c["step"]:
        out.update(dq=dq, dk=dk, dv=dv)
    return out


def _exact_paged(c, s):
    nq, nkv, d, m, page = c["n_q"], c["n_kv"], c["d"], c["q_len"], c["page"]
    o = torch.zeros((c["seqs"], m, nq, d), dtype=torch.float64, device="cuda")
    q = s["q"].double().view(c["seqs"], m, nq, d)
    for n, length in enumerate(_kv_lengths(c)):
        ids = s["page_table"][n, :-(-length // page)].long()
        k = s["k_cache"][ids].flatten(0, 1)[:length].double()
        v = s["v_cache"][ids].flatten(0, 1)[:length].double()
        for t in range(m):
            at = length - m + t
            if at < 0:
                continue
            lo = max(0, at - c["window"] + 1) if c["window"] else 0
            kk = k[lo:at + 1].repeat_interleave(nq // nkv, 1)
            vv = v[lo:at + 1].repeat_interleave(nq // nkv, 1)
            z = torch.einsum("hd,lhd->hl", q[n, t], kk) / math.sqrt(d)
            if c["softcap"]:
                z = c["softcap"] * torch.tanh(z / c["softcap"])
            if s["slopes"] is not None:
                z = z - s["slopes"].double()[:, None] * (at - torch.arange(lo, at + 1, device="cuda"))
            o[n, t] = torch.einsum("hl,lhd->hd", torch.softmax(z, -1), vv)
    return {"o": o.view(-1, nq, d)}
