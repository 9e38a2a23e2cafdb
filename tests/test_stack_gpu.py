"""A stack of attention halves from tokens to the last norm, its operators run together: a training
step and its update against the 64-bit definitions of all of them, and generation against the
training forward.

Tolerances: a half is four operators each way, 8e-5 for its gradients in fp32 (test_block_gpu.py);
two halves, three norms and the table are twelve each way, each within 1e-5: 2.4e-4.  The update of
a matrix in pairs is within 3e-4 of itself (steps * products * growth, as in test_muon_gpu.py, of
what its gradient is off too), AdamW's change of a parameter is lr times a ratio of moments of the
first step, whose magnitude is 1 but where the gradient is near 0.  Generation in bf16 rounds as
training does, and may differ by its roundings through two halves, 2^-8 of each of eight.
"""
import numpy as np
import pytest
import torch

import oracle
from tests import attention_ref as ref
from tests.gpu_helpers import rel_err
from tests.test_block_gpu import _layer, _oracle

pytestmark = pytest.mark.gpu
VOCAB, DM, NQ, NKV, D, R = 97, 128, 4, 2, 32, 16


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2603_06492_gb300 import binding
    from paper_2603_06492_gb300.build import build
    build()
    oracle.build()
    binding.load()


def _setup(T, dtype, blocks=2):
    from paper_2603_06492_gb300 import binding as B
    from paper_2603_06492_gb300.block import Stack
    stack = Stack(VOCAB, blocks, DM, NQ, NKV, D, R, dtype=dtype, scale=3.0, positions=512)
    g = torch.Generator().manual_seed(7)
    rn = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    host = {"table": rn(VOCAB, DM).to(dt), "norms": [{"gain": 1 + 0.2 * rn(DM), "bias": 0.1 * rn(DM)} for _ in range(blocks + 1)],
            "blocks": [{"qkv": _layer(T, DM, stack.blocks[0].qkv_width, R, dtype, 20 + i), "out": _layer(T, NQ * D, DM, R, dtype, 30 + i),
                        "gain_q": 1 + 0.2 * rn(D), "gain_k": 1 + 0.2 * rn(D)} for i in range(blocks)]}
    dev = {"table": host["table"].cuda(), "norms": [{k: v.cuda() for k, v in n.items()} for n in host["norms"]], "blocks": []}
    for p in host["blocks"]:
        q = {n: {k: v for k, v in B.params_to_device(p[n], dtype).items() if k not in ("x", "dy")} for n in ("qkv", "out")}
        dev["blocks"].append({**q, "gain_q": p["gain_q"].cuda(), "gain_k": p["gain_k"].cuda()})
    ids = torch.randint(0, VOCAB, (T,), generator=g).int()
    ids[5] = -1  # padding
    return stack, host, dev, ids, g


def _f64(a):
    return torch.from_numpy(np.asarray(a, dtype=np.float64))


def _norm(z, p, dy=None, eps=1e-5):
    mean = z.mean(1, keepdim=True)
    r = 1 / torch.sqrt(((z - mean) ** 2).mean(1, keepdim=True) + eps)
    n = (z - mean) * r
    if dy is None:
        return n * p["gain"].double() + p["bias"].double()
    w = dy * p["gain"].double()
    return r * (w - w.mean(1, keepdim=True) - n * (w * n).mean(1, keepdim=True)), (dy * n).sum(0), dy.sum(0)


def _half(p, x, pos, table, seen, dy=None):
    """Output of an attention half on x, or its gradients."""
    z = _f64(_oracle(p["qkv"], x.numpy())).view(len(x), -1, D)
    xq, xk, v = z[:, :NQ], z[:, NQ:NQ + NKV], z[:, NQ + NKV:]
    q, k = (ref.rope(a, pos, table, D, False, g) for a, g in ((xq, p["gain_q"]), (xk, p["gain_k"])))
    o, _ = ref.attention(q, k, v, seen, D ** -0.5, 0.0)
    flat = o.reshape(len(x), -1).numpy()
    if dy is None:
        return _f64(_oracle(p["out"], flat))
    go = _oracle(p["out"], flat, dy.numpy())
    _, _, dq, dk, dv = ref.attention(q, k, v, seen, D ** -0.5, 0.0, None, _f64(go["dx"]).view(len(x), NQ, D))
    (_, dxq, dgq), (_, dxk, dgk) = (ref.rope(a, pos, table, D, False, g, dy=t)
                                    for a, g, t in ((xq, p["gain_q"], dq), (xk, p["gain_k"], dk)))
    gi = _oracle(p["qkv"], x.numpy(), torch.cat([dxq, dxk, dv], 1).reshape(len(x), -1).numpy())
    return _f64(gi["dx"]), {"qkv": gi, "out": go, "gain_q": dgq, "gain_k": dgk}


NAMES = ("W", "W_down", "W_up", "M", "omega1", "phi1", "omega2", "phi2", "bias")


def _reference(stack, host, ids, pos, docs, dy):
    T = len(ids)
    seen, table, live = ref.masks(T, docs), stack.blocks[0].table.cpu(), (ids >= 0)[:, None]
    streams = [host["table"].double()[ids.long().clamp(min=0)] * 3.0 * live]
    xs = [_norm(streams[0], host["norms"][0])]
    for i, p in enumerate(host["blocks"]):
        streams.append(streams[-1] + _half(p, xs[-1], pos, table, seen))
        xs.append(_norm(streams[-1], host["norms"][i + 1]))
    want, dstream, dx = {"y": xs[-1]}, 0.0, dy.double()
    for i in range(len(host["blocks"]), -1, -1):
        d, want[f"gain{i}"], want[f"bias{i}"] = _norm(streams[i], host["norms"][i], dx)
        dstream = d + dstream
        if i:
            dx, g = _half(host["blocks"][i - 1], xs[i - 1], pos, table, seen, dstream)
            for name in ("qkv", "out"):
                for n in NAMES:
                    w = _f64(g[name]["d" + n])
                    want[f"{i - 1}.{name}.{n}"] = w.T if n in ("W", "W_down", "W_up") else w
            want[f"{i - 1}.gain_q"], want[f"{i - 1}.gain_k"] = g["gain_q"], g["gain_k"]
    rows = ids.long()
    want["table"] = torch.zeros((VOCAB, DM), dtype=torch.float64).index_add_(0, rows[rows >= 0], 3.0 * dstream[rows >= 0])
    return want


def _flat(grads):
    out = {"table": grads["table"]}
    for i, n in enumerate(grads["norms"]):
        out[f"gain{i}"], out[f"bias{i}"] = n["gain"], n["bias"]
    for i, g in enumerate(grads["blocks"]):
        for name in ("qkv", "out"):
            out.update({f"{i}.{name}.{n}": g[name]["d" + n] for n in NAMES})
        out[f"{i}.gain_q"], out[f"{i}.gain_k"] = g["gain_q"], g["gain_k"]
    return out


def test_training_step_and_update():
    from paper_2603_06492_gb300.block import Update
    T, docs = 150, [0, 60, 61, 150]
    stack, host, dev, ids, g = _setup(T, "fp32")
    pos = torch.tensor([i - a for a, b in zip(docs, docs[1:]) for i in range(a, b)]).int()
    dy = torch.randn((T, DM), generator=g)
    args = (dev, pos.cuda(), torch.tensor(docs, dtype=torch.int32, device="cuda"))
    b = stack.buffers(T, n_docs=3)
    y = stack.forward(b, ids.cuda(), *args)
    grads = stack.backward(b, ids.cuda(), dy.cuda(), *args)
    torch.cuda.synchronize()
    want = _reference(stack, host, ids, pos, docs, dy)
    got = {"y": y, **_flat(grads)}
    errs = {n: rel_err(got[n].double().cpu().numpy(), want[n].numpy()) for n in want}
    assert max(errs.values()) <= 2.4e-4, sorted(errs.items(), key=lambda e: -e[1])[:5]

    # the update, from the gradients above
    u, old = Update(dev, grads, precise=True), y.clone()
    before = [t["param"].double().cpu() for t in u.muon + u.adamw]
    u.step(lr=1e-2, lr_matrices=0.1, weight_decay=0.0)
    torch.cuda.synchronize()
    for i, (t, p) in enumerate(zip(u.muon + u.adamw, before)):
        gr, change = t["grad"].double().cpu(), t["param"].double().cpu() - p
        if i < len(u.muon):
            x = gr / gr.norm()
            x = x.T if gr.shape[0] > gr.shape[1] else x
            for _ in range(5):
                a = x @ x.T
                x = 3.4445 * x + (-4.7750 * a + 2.0315 * a @ a) @ x
            x = x.T if gr.shape[0] > gr.shape[1] else x
            moved = -0.1 * max(1.0, gr.shape[0] / gr.shape[1]) ** 0.5 * x
            assert (change - moved).norm() <= 3e-4 * moved.norm() + 2.0 ** -22 * p.norm()
        else:
            moved = -1e-2 * gr / (gr.abs() + 1e-8)
            assert bool(((change - moved).abs() <= 1e-5 * moved.abs() + 2.0 ** -22 * p.abs() + 1e-7).all())
    # and the next forward reads the new parameters
    assert not torch.equal(stack.forward(b, ids.cuda(), *args), old)


def test_bf16_update_writes_the_operands():
    from paper_2603_06492_gb300.block import Update
    T = 64
    stack, _, dev, ids, g = _setup(T, "bf16", blocks=1)
    args = (dev, torch.arange(T).int().cuda(), torch.tensor([0, T], dtype=torch.int32, device="cuda"))
    b = stack.buffers(T)
    first = stack.forward(b, ids.cuda(), *args).clone()
    grads = stack.backward(b, ids.cuda(), torch.randn((T, DM), generator=g).bfloat16().cuda(), *args)
    u = Update(dev, grads)
    for _ in range(2):
        u.step(lr=1e-3, lr_matrices=0.02)
    torch.cuda.synchronize()
    for t in u.muon + u.adamw:
        assert t["param"].isfinite().all()
        if t["param_bf16"] is not None:
            assert torch.equal(t["param_bf16"], t["param"].bfloat16())
    assert {p.data_ptr() for p in (dev["table"], dev["blocks"][0]["qkv"]["W"])} <= {t["param_bf16"].data_ptr() for t in u.muon + u.adamw
                                                                                 if t["param_bf16"] is not None}
    assert not torch.equal(stack.forward(b, ids.cuda(), *args), first)


@pytest.mark.parametrize("dtype,tol", [("fp32", 1e-4), ("bf16", 8 * 2.0 ** -7)])
def test_generation_is_the_training_forward(dtype, tol):
    from paper_2603_06492_gb300 import attention as A
    from paper_2603_06492_gb300.block import page_slots
    lens, page = [37, 64, 5], 16
    T, n, docs = sum(lens), len(lens), [0, 37, 101, 106]
    stack, _, dev, ids, _ = _setup(T, dtype)
    ids = ids.clamp(min=0).cuda()
    pos = torch.cat([torch.arange(m) for m in lens]).cuda()
    seq = torch.cat([torch.full((m,), i) for i, m in enumerate(lens)]).cuda()
    b = stack.buffers(T, n_docs=n)
    y = stack.forward(b, ids, dev, pos.int(), torch.tensor(docs, dtype=torch.int32, device="cuda")).clone()
    caches = stack.caches(12, page)
    table = torch.randperm(12, generator=torch.Generator().manual_seed(1)).view(3, 4).int().cuda()
    last = torch.tensor([m - 1 for m in docs[1:]], device="cuda")
    slots = page_slots(table, seq, pos, page)
    slots[last] = -1
    for i, blk in enumerate(stack.blocks):
        blk.fill(A.RopeBuffers(T, NQ, NKV, D, dtype, **blk.rope, with_grads=False), caches[i], b["blocks"][i]["qkv"].y, pos.int(), slots,
                 dev["blocks"][i])
    step = stack.step_buffers(n, max_len=64)
    got = stack.step(step, caches, ids[last].contiguous(), dev, pos[last].int(), page_slots(table, seq[last], pos[last], page), table,
                     torch.tensor(lens, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert rel_err(got.float().cpu(), y[last].float().cpu()) <= tol
