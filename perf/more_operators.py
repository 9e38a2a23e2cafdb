"""The measured cases of the operators around the projections of a training step, through
their public entry points.

A case is one call, or one forward and backward, on buffers that a program keeps.  Kinds:

    "norm"   layer norm of T rows, with "res" of the sum of a layer's output and the
             residual stream (which is stored); with "step" also the gradients with respect
             to that sum, to the gain and to the bias
    "embed"  rows of a table by token, scaled; with "step" also the gradient of the table
    "muon"   one optimizer step of a group of matrices by orthogonalised momentum: the new
             momentum and, as a rank of a data-parallel job computes it for the others, the
             update in bf16; or with "precise" the new parameters and their bf16 copies

The plain forms below are elementary torch operations in 32 bits.  Sizes are those of the
package's configurations (1024- and 2048-wide decoders, a 768-wide ViT of 197 tokens per
image, ranks 64 and 128) or generic ones of the same ranges.
"""
from __future__ import annotations

import math
import random

import torch

own = False


# ---------------------------------------------------------------- cases
def _norm(T, d, dtype="bf16", res=False, step=True, name=None):
    c = {"kind": "norm", "T": T, "d": d, "dtype": dtype, "res": res, "step": step}
    return {**c, "name": name} if name else c


def _embed(T, vocab, d, tokens, dtype="bf16", pad=0, scale=1.0, step=True, name=None):
    c = {"kind": "embed", "T": T, "vocab": vocab, "d": d, "tokens": tokens, "dtype": dtype, "pad": pad, "scale": scale,
         "step": step}
    return {**c, "name": name} if name else c


def _muon(shapes, precise=False, nesterov=True, name=None):
    c = {"kind": "muon", "shapes": ",".join("%dx%d" % s for s in shapes), "precise": precise, "nesterov": nesterov}
    return {**c, "name": name} if name else c


def _layer(d_in, d_out, r):
    """The matrices of a NOBLE layer: W, W_down, W_up, M."""
    return [(d_out, d_in), (r, d_in), (d_out, r), (r, r)]


def listed():
    return [
        # generating: one token of each of 24 sequences, the residual stream of the 2048-wide decoder
        _norm(24, 2048, res=True, step=False, name="norm-decode-24"),
        # the fp32 mode on one 1024-token sequence of the 1024-wide decoder
        _norm(1024, 1024, "fp32", name="norm-fp32-sequence-step"),
        # training a ViT: 256 images of 197 tokens
        _norm(256 * 197, 768, name="norm-vit-256-images-step"),
        # training the 2048-wide decoder: 16 sequences of 1024 tokens, residual stream
        _norm(16384, 2048, res=True, name="norm-large-residual-step"),
        # generating: one token of each of 24 sequences, rows scaled by the square root of the width
        _embed(24, 50257, 2048, "words", scale=2048 ** 0.5, step=False, name="embed-decode-24"),
        # training the 1024-wide decoder: 8 sequences of 1024 tokens of text
        _embed(8192, 50257, 1024, "words", name="embed-base-step"),
        # the fp32 mode on prompts of no particular length, a small table, padding at the end of each
        _embed(7001, 1003, 264, "even", "fp32", pad=300, scale=0.5, name="embed-ragged-fp32-step"),
        # a long batch of the 2048-wide decoder and a table for many languages
        _embed(65536, 131072, 2048, "words", name="embed-long-step"),
        # the bottleneck of one layer of the 1024-wide decoder
        _muon([(64, 1024), (1024, 64), (64, 64)], name="muon-bottleneck-update"),
        # the FFN up projection of the 1024-wide decoder with its branch
        _muon(_layer(1024, 4096, 64), name="muon-base-ffn-up-update"),
        # odd sizes, parameters updated in place at 32-bit accuracy
        _muon([(1009, 2755), (333, 77), (1, 40)], precise=True, nesterov=False, name="muon-ragged-precise-step"),
        # the FFN up projection of the 2048-wide decoder with its branch
        _muon(_layer(2048, 8192, 128), name="muon-large-ffn-up-update"),
    ]


def _log_uniform(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))


def _width(rng, lo, hi):
    return 8 * _log_uniform(rng, lo // 8, hi // 8)


def draw(rng):
    kind = rng.choice(("norm", "norm", "embed", "embed", "muon", "muon"))
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    if kind == "norm":
        while True:
            c = _norm(_log_uniform(rng, 1, 65536), _width(rng, 64, 8192), dtype, rng.random() < 0.5, rng.random() < 0.7)
            if c["T"] * c["d"] <= 256 * 197 * 768:
                return c
    if kind == "embed":
        while True:
            c = _embed(_log_uniform(rng, 1, 65536), _log_uniform(rng, 2, 131072), _width(rng, 64, 4096),
                       rng.choice(("words", "words", "even", "one")), dtype, 0, rng.choice((1.0, 0.5, 32.0)),
                       rng.random() < 0.75)
            c["pad"] = rng.choice((0, 0, c["T"] // 7))
            if work(c)["bytes"] <= work(_embed(65536, 131072, 2048, "words"))["bytes"]:
                return c
    most = work(_muon(_layer(2048, 8192, 128)))["flops"]
    while True:
        shapes = [(_log_uniform(rng, 1, 8192), _log_uniform(rng, 1, 8192)) for _ in range(rng.choice((1, 1, 2, 5)))]
        precise = rng.random() < 0.4
        c = _muon(shapes, precise, rng.random() < 0.7)
        # 32-bit accuracy takes a multiple of the products
        if work(c)["flops"] * (4 if precise else 1) <= most:
            return c


def _shapes(c):
    return [tuple(int(n) for n in s.split("x")) for s in c["shapes"].split(",")]


# ---------------------------------------------------------------- inputs
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _tokens(c, g):
    """Token numbers as they come: by rank with frequency 1 / (rank + 2.7) ("words", the table's
    order shuffled), all alike likely ("even"), or one only ("one"); -1 where there is padding."""
    T, V = c["T"], c["vocab"]
    if c["tokens"] == "words":
        u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
        rank = (2.7 * ((V + 2.7) / 2.7) ** u - 2.7).long().clamp_(0, V - 1)
        ids = torch.randperm(V, generator=g, device="cuda")[rank]
    elif c["tokens"] == "even":
        ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    else:
        ids = torch.randint(0, V, (1,), generator=g, device="cuda").expand(T).clone()
    if c["pad"]:
        ids[torch.randperm(T, generator=g, device="cuda")[:c["pad"]]] = -1
    return ids.int()


def _tensors(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, dtype=torch.float32, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=g, device="cuda") * std + mean).to(dtype)

    s = {"case": c}
    if c["kind"] == "norm":
        shape, dt = (c["T"], c["d"]), _dtype(c)
        # rows of a residual stream: some features stand out
        s["x"] = (normal(shape) * (1.0 + 3.0 * torch.rand(c["d"], generator=g, device="cuda") ** 8)).to(dt)
        if c["res"]:
            s["res"] = normal(shape, dt, 0.5, 0.1)
        s["gain"], s["bias"] = normal((c["d"],), std=0.2, mean=1.0), normal((c["d"],), std=0.1)
        if c["step"]:
            s["dy"] = normal(shape, dt)
            if c["res"]:
                s["dstream"] = normal(shape, dt)
    elif c["kind"] == "embed":
        s["ids"] = _tokens(c, g)
        s["table"] = normal((c["vocab"], c["d"]), _dtype(c), 0.02)
        if c["step"]:
            s["dy"] = normal((c["T"], c["d"]), _dtype(c))
    else:
        # gradients: noise of a batch, and what the batch has in common in a few directions
        s["tensors"] = []
        for rows, cols in _shapes(c):
            k = min(rows, cols, 16)
            common = normal((rows, k)) @ normal((k, cols), std=(4.0 / k) ** 0.5)
            t = {"grad": (common + normal((rows, cols), std=2.0)) * 1e-3,
                 "momentum": (common + normal((rows, cols))) * 1e-2}
            if c["precise"]:
                t["param"] = normal((rows, cols), std=0.02)
                t["param_bf16"] = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
            else:
                t["update"] = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
            s["tensors"].append(t)
    return s


EPS = 1e-5
MUON = {"lr": 0.01, "momentum": 0.95, "weight_decay": 0.01, "steps": 5, "eps": 1e-7}
ABC = (3.4445, -4.7750, 2.0315)  # of a step of the iteration


def prepare(case, seed):
    s = _tensors(case, seed)
    if own:
        from paper_2603_06492_gb300 import binding as B, layers as L
        c = case
        if c["kind"] == "norm":
            s["buf"] = L.NormBuffers(c["T"], c["d"], c["dtype"], eps=EPS, residual=c["res"], with_grads=c["step"])
        elif c["kind"] == "embed":
            s["buf"] = L.EmbedBuffers(c["T"], c["vocab"], c["d"], c["dtype"], scale=c["scale"], with_grads=c["step"])
        else:
            s["workspace"] = B.muon_workspace(s["tensors"], precise=c["precise"])
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(c, s)
    return {"norm": _plain_norm, "embed": _plain_embed, "muon": _plain_muon}[c["kind"]](c, s)


def _run_own(c, s):
    from paper_2603_06492_gb300 import binding as B, layers as L
    if c["kind"] == "norm":
        b, out = s["buf"], {}
        out["y"] = L.norm_forward(b, s["x"], s["gain"], s["bias"], res=s.get("res"))
        if c["res"]:
            out["sum"] = b.sum
        if c["step"]:
            out["dx"] = L.norm_backward(b, s["dy"], b.sum if c["res"] else s["x"], s["gain"], dstream=s.get("dstream"))
            out["dgain"], out["dbias"] = b.dgain, b.dbias
        return out
    if c["kind"] == "embed":
        out = {"y": L.embed_forward(s["buf"], s["ids"], s["table"])}
        if c["step"]:
            out["dtable"] = L.embed_backward(s["buf"], s["ids"], s["dy"])
        return out
    B.noble_muon_step(s["tensors"], **MUON, nesterov=c["nesterov"], precise=c["precise"], workspace=s["workspace"])
    return _muon_outputs(s)


def _muon_outputs(s):
    return [{k: v for k, v in t.items() if k != "grad"} for t in s["tensors"]]


def _plain_norm(c, s):
    x = s["x"].float()
    out = {}
    if c["res"]:
        out["sum"] = (x + s["res"].float()).to(_dtype(c))
        x = out["sum"].float()  # what is normed is the stream as it is stored
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((x - mean) * (x - mean)).mean(1, keepdim=True) + EPS)
    xh = (x - mean) * rstd
    out["y"] = (xh * s["gain"] + s["bias"]).to(_dtype(c))
    if c["step"]:
        dy = s["dy"].float()
        w = dy * s["gain"]
        dx = rstd * (w - w.mean(1, keepdim=True) - xh * (w * xh).mean(1, keepdim=True))
        if c["res"]:
            dx = dx + s["dstream"].float()
        out["dx"] = dx.to(_dtype(c))
        out["dgain"], out["dbias"] = (dy * xh).sum(0), dy.sum(0)
    return out


def _plain_embed(c, s):
    ids = s["ids"].long()
    there = (ids >= 0)[:, None]
    rows = ids.clamp(min=0)
    out = {"y": (s["table"][rows].float() * c["scale"] * there).to(_dtype(c))}
    if c["step"]:
        total = torch.zeros((c["vocab"], c["d"]), dtype=torch.float32, device="cuda")
        out["dtable"] = total.index_add_(0, rows, s["dy"].float() * there).mul_(c["scale"])
    return out


def _plain_muon(c, s):
    for t in s["tensors"]:
        g, m = t["grad"], t["momentum"]
        m.mul_(MUON["momentum"]).add_(g)
        u = g + MUON["momentum"] * m if c["nesterov"] else m
        x = u / (torch.sqrt((u * u).sum()) + MUON["eps"])
        tall = x.shape[0] > x.shape[1]
        x = x.T if tall else x
        for _ in range(MUON["steps"]):
            a = x @ x.T
            x = ABC[0] * x + (ABC[1] * a + ABC[2] * (a @ a)) @ x
        o = x.T if tall else x
        if "update" in t:
            t["update"].copy_(o)
        if "param" in t:
            p, lr = t["param"], MUON["lr"]
            scale = math.sqrt(max(1.0, p.shape[0] / p.shape[1]))
            p.copy_(p - lr * MUON["weight_decay"] * p - lr * scale * o)
            t["param_bf16"].copy_(p)
    return _muon_outputs(s)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    if c["kind"] == "norm":
        n = c["T"] * c["d"]
        size = 4 if c["dtype"] == "fp32" else 2
        # forward: x (and the stream) in, y (and the stream) out; backward: dy (and the stream's
        # gradient) in, dx out -- with a step the normed rows are read once
        tensors = (4 if c["res"] else 2) + ((3 if c["res"] else 2) if c["step"] else 0)
        return {"bytes": tensors * n * size, "flops": n * (8 + (12 if c["step"] else 0))}
    if c["kind"] == "embed":
        size = 4 if c["dtype"] == "fp32" else 2
        T, V, d = c["T"], c["vocab"], c["d"]
        live = T - c["pad"]
        # distinct rows that so many tokens read
        distinct = {"one": min(live, 1), "even": V * -math.expm1(live * math.log1p(-1.0 / V)) if V > 1 else 1,
                    "words": 0}[c["tokens"]]
        if c["tokens"] == "words":
            top, whole = math.log((V + 2.7) / 2.7), min(V, 4096)
            ranks = [k + 0.5 for k in range(whole)]
            weights = [1.0] * whole
            while whole < V:  # wider and wider steps of rank
                step = min(V - whole, whole // 8)
                ranks.append(whole + step / 2)
                weights.append(float(step))
                whole += step
            distinct = sum(w * -math.expm1(-live / ((r + 2.7) * top)) for r, w in zip(ranks, weights))
        total = distinct * d * size + T * d * size + 4 * T
        if c["step"]:
            total += live * d * size + 4 * V * d
        return {"bytes": total, "flops": T * d * (2 if c["step"] else 1)}
    nbytes = flops = 0.0
    for rows, cols in _shapes(c):
        m, n = min(rows, cols), max(rows, cols)
        # gradient and momentum in, momentum out, and the update, or parameters in and out and their copy
        nbytes += rows * cols * (12 + (10 if c["precise"] else 2))
        # of the symmetric products half is enough
        flops += MUON["steps"] * (m * (m + 1.0) * n + m * m * (m + 1.0) + 2.0 * m * m * n)
    return {"bytes": nbytes, "flops": flops}


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    """What run returns, from the definitions in 64 bits."""
    c = case
    s = _tensors(c, seed)
    if c["kind"] == "norm":
        return _exact_norm(c, s)
    return _exact_embed(c, s) if c["kind"] == "embed" else _exact_muon(c, s)


def _exact_norm(c, s):
    z = s["x"].double()
    out = {}
    if c["res"]:
        out["sum"] = (z + s["res"].double()).to(_dtype(c)).double()
        z = out["sum"]
    n = c["d"]
    centred = z - torch.einsum("td->t", z)[:, None] / n
    spread = torch.sqrt(torch.einsum("td,td->t", centred, centred) / n + EPS)[:, None]
    unit = centred / spread
    out["y"] = torch.addcmul(s["bias"].double(), unit, s["gain"].double())
    if c["step"]:
        dy = s["dy"].double()
        out["dgain"], out["dbias"] = torch.einsum("td,td->d", dy, unit), torch.einsum("td->d", dy)
        w = dy * s["gain"].double()
        # the projection of w off the constant row and off unit, whose square is n (1 - EPS / spread^2)
        along = torch.einsum("td,td->t", w, unit)[:, None] / n
        dx = (w - torch.einsum("td->t", w)[:, None] / n - along * unit) / spread
        out["dx"] = dx + s["dstream"].double() if c["res"] else dx
    return out


def _exact_embed(c, s):
    live = torch.nonzero(s["ids"] >= 0).flatten()
    rows = s["ids"][live].long()
    y = torch.zeros((c["T"], c["d"]), dtype=torch.float64, device="cuda")
    y[live] = c["scale"] * s["table"].double()[rows]
    out = {"y": y}
    if c["step"]:
        # tokens in order of their numbers, each run of equal ones added up by itself
        order = torch.argsort(rows, stable=True)
        kept, counts = torch.unique_consecutive(rows[order], return_counts=True)
        total = torch.zeros((c["vocab"], c["d"]), dtype=torch.float64, device="cuda")
        if len(live):
            total[kept] = c["scale"] * torch.segment_reduce(s["dy"].double()[live][order], "sum", lengths=counts, axis=0)
        out["dtable"] = total
    return out


def _exact_muon(c, s):
    out = []
    for t in s["tensors"]:
        grad, momentum = t["grad"].double(), t["momentum"].double()
        momentum = MUON["momentum"] * momentum + grad
        u = grad + MUON["momentum"] * momentum if c["nesterov"] else momentum
        # the iteration on the smaller side's products alone: X_k = P_k X_0 with P_k from X_0's
        # singular vectors, which no step changes
        x = u / (torch.linalg.matrix_norm(u) + MUON["eps"])
        left, sigma, right = torch.linalg.svd(x, full_matrices=False) if x.numel() <= 1 << 16 else (None, None, None)
        if left is not None:
            for _ in range(MUON["steps"]):
                sigma = sigma * (ABC[0] + ABC[1] * sigma ** 2 + ABC[2] * sigma ** 4)
            o = left @ torch.diag(sigma) @ right
        else:
            wide = x if x.shape[0] <= x.shape[1] else x.mT
            eye = torch.eye(wide.shape[0], dtype=torch.float64, device="cuda")
            for _ in range(MUON["steps"]):
                gram = wide @ wide.mT
                wide = (ABC[0] * eye + gram @ (ABC[1] * eye + ABC[2] * gram)) @ wide
            o = wide if x.shape[0] <= x.shape[1] else wide.mT
        r = {"momentum": momentum}
        if c["precise"]:
            p = t["param"].double()
            scale = max(1.0, p.shape[0] / p.shape[1]) ** 0.5
            r["param"] = (1.0 - MUON["lr"] * MUON["weight_decay"]) * p - MUON["lr"] * scale * o
            r["param_bf16"] = r["param"]
        else:
            r["update"] = o
        out.append(r)
    return out


if __name__ == "__main__":
    for one in listed():
        print(one["name"], work(one))
    print(draw(random.Random(0)))
