"""The learning rates of a Stack's optimizer: the paper's multipliers by group, against the oracle's
formula on the host, and in the steps that the parameters take on a GPU."""
import pytest
import torch

import oracle.adamw
from paper_2603_06492_gb300 import binding as B
from paper_2603_06492_gb300.block import Update

DM, WIDTH, R, V, D = 64, 96, 16, 30, 16
NAMES = ("W", "bias", "W_down", "W_up", "M", "omega1", "phi1", "omega2", "phi2")
ONE = ("table", "gain", "bias", "gain_q", "gain_k")


def _model(device, dtype=torch.float32, blocks=2, branch=True):
    """Parameters and gradients of a stack, none of them zero."""
    g = torch.Generator().manual_seed(2)
    new = lambda *s, dt=torch.float32: (torch.randn(s, generator=g) + 3.0 * torch.randint(0, 2, s, generator=g) - 1.5).to(device, dt)  # noqa: E731

    def layer(d_in, d_out):
        shapes = {"W": (d_out, d_in), "bias": (d_out,), "W_down": (R, d_in), "W_up": (d_out, R), "M": (R, R), "omega1": (R,),
                  "phi1": (R,), "omega2": (R,), "phi2": (R,)}
        names = NAMES if branch else ("W", "bias")
        return ({n: new(*shapes[n], dt=dtype if n in ("W", "W_down", "W_up") else torch.float32) for n in names},
                {"d" + n: new(*shapes[n]) for n in names})

    norm = lambda: {"gain": new(DM), "bias": new(DM)}  # noqa: E731
    params = {"table": new(V, DM, dt=dtype), "norms": [norm() for _ in range(blocks + 1)], "blocks": []}
    grads = {"table": new(V, DM), "norms": [norm() for _ in range(blocks + 1)], "blocks": []}
    for _ in range(blocks):
        (pi, gi), (po, go) = layer(DM, WIDTH), layer(64, DM)
        params["blocks"].append({"qkv": pi, "out": po, "gain_q": new(D), "gain_k": new(D)})
        grads["blocks"].append({"qkv": gi, "out": go, "gain_q": new(D), "gain_k": new(D)})
    return params, grads


def _named(grads):
    """Address of each gradient -> its parameter's name and the projection's sizes."""
    out = {grads["table"].data_ptr(): ("table", None)}
    for n in grads["norms"]:
        out.update({n[k].data_ptr(): (k, None) for k in n})
    for b in grads["blocks"]:
        out.update({b[k].data_ptr(): (k, None) for k in ("gain_q", "gain_k")})
        for name, size in (("qkv", (DM, WIDTH)), ("out", (64, DM))):
            out.update({t.data_ptr(): (k[1:], size) for k, t in b[name].items()})
    return out


def _want(name, size, rule):
    if rule is None or size is None:
        return 1.0
    names = {"gamma_M": "gamma_m"}
    groups = oracle.adamw.lr_multipliers(*size, R, **{names.get(k, k): v for k, v in rule.items()})
    return groups[name.rstrip("12")]


@pytest.mark.parametrize("rule", [None, {}, dict(gamma=0.0, gamma_M=0.0), dict(gamma=0.2, gamma_M=0.1, omega_mult=2.0, phi_mult=0.0)])
def test_groups(monkeypatch, rule):
    monkeypatch.setattr(B, "muon_workspace", lambda tensors, precise: None)
    params, grads = _model("cpu")
    u, named = Update(params, grads, multipliers=rule), _named(grads)
    seen = [(named[t["grad"].data_ptr()], t["lr_mult"]) for t in u.muon + u.adamw]
    assert len(seen) == len(named) == 1 + 6 + 2 * (2 + 18)
    for (name, size), mult in seen:
        assert mult == pytest.approx(_want(name, size, rule), rel=1e-6), name


def test_without_a_branch(monkeypatch):
    monkeypatch.setattr(B, "muon_workspace", lambda tensors, precise: None)
    u = Update(*_model("cpu", branch=False), multipliers={})
    assert len(u.muon) == 4 and all(t["lr_mult"] == 1.0 for t in u.muon + u.adamw)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_steps(dtype):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    moved = []
    for rule in (None, {}):
        params, grads = _model("cuda", dtype)
        u, named = Update(params, grads, multipliers=rule), _named(grads)
        before = [t["param"].double() for t in u.muon + u.adamw]
        u.step(lr=1e-2, lr_matrices=0.05, weight_decay=0.0)
        torch.cuda.synchronize()
        moved.append([t["param"].double() - p for t, p in zip(u.muon + u.adamw, before)])
    # the changes themselves repeat to fp32's rounding, 2^-22 of them; p - change is off by a rounding of p, at most 8, twice
    for i, t in enumerate(u.muon + u.adamw):
        mult = _want(*named[t["grad"].data_ptr()], {})
        off = (moved[1][i] - mult * moved[0][i]).abs().max()
        assert moved[0][i].any() and off <= 2.0 ** -22 * moved[1][i].abs().max() + (1 + mult) * 8 * 2.0 ** -24, (mult, off)
