"""The attention half of a block, its operators run together: a training step against the
64-bit definitions of all of them, and generation against the training forward.

Tolerances: four operators one behind the other, each within its own (1e-5 of fp32
operands, 1e-2 of bf16 ones), of which errors of the first meet the gains of the others:
4 of them each way is 8e-5 for fp32 gradients.  Generation in bf16 rounds q, k, v and o
as training does, and may differ by their roundings, 2^-8 of each.
"""
import math

import numpy as np
import pytest
import torch

import oracle
from tests import attention_ref as ref
from tests.gpu_helpers import rel_err

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import oracle as o
    from paper_2603_06492_gb300 import binding
    from paper_2603_06492_gb300.build import build
    build()
    o.build()
    binding.load()


def _layer(T, d_in, d_out, r, dtype, seed):
    from paper_2603_06492_gb300.inputs import Layer, make_layer_inputs
    return make_layer_inputs(Layer("block", T, d_in, d_out, r, dtype), seed, init="strong_branch")


def _oracle(inp, x, dy=None):
    from paper_2603_06492_gb300.inputs import to_paper_orientation
    p = to_paper_orientation(dict(inp, x=x, **({"dy": dy} if dy is not None else {})))
    args = [p[k] for k in ("W_down", "omega1", "phi1", "M", "omega2", "phi2", "W_up")]
    if dy is None:
        return oracle.fwd(p["x"], p["W"], p["bias"], *args)
    return oracle.bwd(p["x"], p["W"], *args, p["dy"])


def _setup(T, dtype, softcap=0.0):
    from paper_2603_06492_gb300 import binding as B
    from paper_2603_06492_gb300.block import AttentionBlock
    dm, nq, nkv, d, r = 128, 4, 2, 32, 16
    blk = AttentionBlock(dm, nq, nkv, d, r, dtype, positions=512, softcap=softcap)
    qkv, out = _layer(T, dm, blk.qkv_width, r, dtype, 1), _layer(T, nq * d, dm, r, dtype, 2)
    g = torch.Generator().manual_seed(3)
    gains = [1 + 0.2 * torch.randn(d, generator=g) for _ in range(2)]
    dev = {"qkv": B.params_to_device(qkv, dtype), "out": B.params_to_device(out, dtype), "gain_q": gains[0].cuda(),
           "gain_k": gains[1].cuda()}
    return blk, qkv, out, gains, dev


def test_training_step():
    T, docs, softcap = 150, [0, 60, 61, 150], 8.0
    blk, qkv, out, gains, dev = _setup(T, "fp32", softcap)
    nq, nkv, d = blk.n_q, blk.n_kv, blk.d
    pos = torch.tensor([i - a for a, b in zip(docs, docs[1:]) for i in range(a, b)]).int()
    b = blk.buffers(T, n_docs=3)
    args = (dev, pos.cuda(), torch.tensor(docs, dtype=torch.int32, device="cuda"))
    y = blk.forward(b, dev["qkv"]["x"], *args)
    dx, grads = blk.backward(b, dev["qkv"]["x"], dev["out"]["dy"], *args)
    torch.cuda.synchronize()
    # the same in 64 bits
    f64 = lambda a: torch.from_numpy(np.asarray(a, dtype=np.float64))  # noqa: E731
    table = blk.table.cpu()
    z = f64(_oracle(qkv, qkv["x"])).view(T, -1, d)
    xq, xk, v = z[:, :nq], z[:, nq:nq + nkv], z[:, nq + nkv:]
    q, k = (ref.rope(x, pos, table, d, False, g) for x, g in zip((xq, xk), gains))
    seen = ref.masks(T, docs)
    o, _ = ref.attention(q, k, v, seen, 1 / math.sqrt(d), softcap)
    want_y = _oracle(out, o.view(T, -1).numpy())
    go = _oracle(out, o.view(T, -1).numpy(), out["dy"])
    _, _, dq, dk, dv = ref.attention(q, k, v, seen, 1 / math.sqrt(d), softcap, None, f64(go["dx"]).view(T, nq, d))
    (_, dxq, dgq), (_, dxk, dgk) = (ref.rope(x, pos, table, d, False, g, dy=t) for x, g, t in
                                    ((xq, gains[0], dq), (xk, gains[1], dk)))
    gi = _oracle(qkv, qkv["x"], torch.cat([dxq, dxk, dv], 1).reshape(T, -1).numpy())
    pairs = {"y": (y, want_y), "dx": (dx, gi["dx"]), "gain_q": (grads["gain_q"], dgq), "gain_k": (grads["gain_k"], dgk)}
    for name, mine, theirs in (("qkv", grads["qkv"], gi), ("out", grads["out"], go)):
        for w in ("dW", "dW_down", "dW_up"):
            pairs[name + w] = (mine[w].T, theirs[w])
        for w in ("dM", "domega1", "dphi1", "domega2", "dphi2", "dbias"):
            pairs[name + w] = (mine[w], theirs[w])
    errs = {n: rel_err(a.detach().double().cpu().numpy(), np.asarray(w)) for n, (a, w) in pairs.items()}
    assert max(errs.values()) <= 8e-5, errs


@pytest.mark.parametrize("dtype,tol", [("fp32", 4e-5), ("bf16", 4e-2)])
def test_generation_is_the_training_forward(dtype, tol):
    from paper_2603_06492_gb300 import attention as A
    from paper_2603_06492_gb300.block import page_slots
    lens, page = [37, 64, 5], 16
    T, n = sum(lens), len(lens)
    docs = [0, 37, 101, 106]
    blk, _, _, _, dev = _setup(T, dtype)
    pos = torch.cat([torch.arange(m) for m in lens]).cuda()
    seq = torch.cat([torch.full((m,), i) for i, m in enumerate(lens)]).cuda()
    b = blk.buffers(T, n_docs=n)
    x = dev["qkv"]["x"]
    y = blk.forward(b, x, dev, pos.int(), torch.tensor(docs, dtype=torch.int32, device="cuda")).clone()
    # all but each sequence's last token as a prompt, the last one as a step
    cache = blk.cache(12, page)
    table = torch.randperm(12, generator=torch.Generator().manual_seed(1)).view(3, 4).int().cuda()
    last = torch.tensor([m - 1 for m in docs[1:]], device="cuda")
    slots = page_slots(table, seq, pos, page)
    slots[last] = -1
    blk.fill(A.RopeBuffers(T, blk.n_q, blk.n_kv, blk.d, dtype, **blk.rope, with_grads=False), cache, b["qkv"].y, pos.int(),
             slots, dev)
    step = blk.step_buffers(n, max_len=64)
    got = blk.step(step, cache, x[last].contiguous(), dev, pos[last].int(), page_slots(table, seq[last], pos[last], page), table,
                   torch.tensor(lens, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert rel_err(got.float().cpu(), y[last].float().cpu()) <= tol
