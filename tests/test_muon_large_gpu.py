"""The optimizer step on matrices whose products take several rounds of the pairs, tiles of 256 columns and
splits of them (test_muon_plan.py shows which), against its definition in 64 bits on the device.

Tolerances as in test_muon_gpu.py: twice the error of the same iteration in 64 bits with A, B and X rounded to 11 or 22 bits,
and the sums.  A product over K columns adds K / 16 times to its accumulator, and an add cuts up to 2^-23 of
the partial sum off, half that in the mean, and a partial sum of like terms is half of the whole in the mean:
K / 16 * 2^-25, or 2^-21 where that is more.  A step has one sum over the larger side and two over the smaller
one, and grows an error by 3.5 at most.
"""
import math

import pytest
import torch

from tests.test_muon_gpu import ABC, U, _near, lib  # noqa: F401

pytestmark = pytest.mark.gpu
PRECISE = 2  # NOBLE_MUON_PRECISE


def _layer(d_in, d_out, r):
    """The matrices of a NOBLE layer: W, W_down, W_up, M."""
    return [(d_out, d_in), (r, d_in), (d_out, r), (r, r)]


CALLS = [(shapes, precise) for shapes in (
    [(2900, 3100)], [(5000, 2300)], [(1500, 1600)], [(2048, 8192)], _layer(1024, 4096, 64), _layer(2048, 8192, 128),
    [(1100, 2300), (700, 900), (260, 3000), (1, 40), (300, 300), (90, 1000)]) for precise in (False, True)]


def _iterate(u, bits=None):
    def rnd(x):
        if bits is None:
            return x
        m, e = torch.frexp(x)
        return torch.ldexp(torch.round(m * 2.0 ** bits), e - bits)

    x = u / (torch.linalg.matrix_norm(u) + 1e-7)
    tall = x.shape[0] > x.shape[1]
    x = rnd(x.T if tall else x)
    eye = torch.eye(len(x), dtype=torch.float64, device="cuda")
    for _ in range(5):
        a = rnd(x @ x.T)
        x = rnd(rnd(ABC[0] * eye + ABC[1] * a + ABC[2] * a @ a) @ x)
    return x.T if tall else x


def _tensors(shapes, seed):
    # noise, and what a batch has in common in a few directions
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    out = []
    for rows, cols in shapes:
        k = min(rows, cols, 16)
        common = rn(rows, k) @ rn(k, cols) * (4.0 / k) ** 0.5
        out.append({"grad": (common + 2.0 * rn(rows, cols)) * 1e-3, "momentum": (common + rn(rows, cols)) * 1e-2,
                    "param": 0.02 * rn(rows, cols)})
    return out


def _tolerance(u, want, precise):
    rows, cols = u.shape
    rough = _iterate(u, 22 if precise or min(rows, cols) <= 256 else 11)
    sums = [max(2.0 ** -21, n / 16 * 2.0 ** -25) for n in (max(rows, cols), min(rows, cols), min(rows, cols))]
    return 2 * ((rough - want).norm() / want.norm()).item() + 5 * 4 * sum(sums) + 4 * U


@pytest.mark.parametrize("shapes,precise", CALLS)
def test_against_64_bits(shapes, precise):
    from paper_2603_06492_gb300 import binding as B
    hp = dict(lr=0.5, momentum=0.95, weight_decay=0.1, precise=precise)
    t, runs = _tensors(shapes, 1), []
    for fill in (255, 0):  # whatever the workspace holds
        dev = [{**{k: v.clone() for k, v in x.items()}, **{k: torch.full(x["grad"].shape, float("nan"), dtype=torch.bfloat16, device="cuda")
                                                           for k in ("param_bf16", "update")}} for x in t]
        B.noble_muon_step(dev, workspace=B.muon_workspace(dev, precise).fill_(fill), **hp)
        torch.cuda.synchronize()
        B.noble_get_device_status(None)
        runs.append(dev)
    assert all(torch.equal(a[k], b[k]) for a, b in zip(*runs) for k in a)
    for x, d in zip(t, runs[0]):
        rows, cols = x["grad"].shape
        g, m = x["grad"].double(), x["momentum"].double()
        m = 0.95 * m + g
        assert bool(((d["momentum"].double() - m).abs() <= 2 * U * (m.abs() + g.abs() + (m - g).abs())).all())
        u = g + 0.95 * m
        want = _iterate(u)
        rel = _tolerance(u, want, precise)
        _near(d["update"], want.cpu(), rel + 2.0 ** -8, (rows, cols))
        moved = -0.5 * math.sqrt(max(1.0, rows / cols)) * want
        p = x["param"].double() * (1 - 0.5 * 0.1)
        off = d["param"].double() - (p + moved)
        room = 4 * U * (p.norm() + moved.norm())
        assert off.norm() <= rel * moved.norm() + room, ((off.norm() / moved.norm()).item(), rel)
        # no tile of 32 x 32 is off by more than eight times its share of that, and no element by 16 times the largest one's
        edge = torch.nn.functional.pad(off, (0, -cols % 32, 0, -rows % 32)).view((rows + 31) // 32, 32, (cols + 31) // 32, 32)
        share = 32 / math.sqrt(max(rows, 32) * max(cols, 32))
        assert edge.square().sum((1, 3)).sqrt().max() <= 8 * share * (rel * moved.norm() + room)
        assert off.abs().max() <= 16 * (rel * moved.abs().max() + 4 * U * p.abs().max())
        assert torch.equal(d["param_bf16"], d["param"].bfloat16())


@pytest.mark.parametrize("tall", [False, True])
def test_elements_beyond_32_bits(tall):
    # 2^31 + 524288 elements: one in each row of the smaller side and a column of its own, so that X X^T is diagonal
    # and a step takes each element s to s (a + b s^2 + c s^4)
    from paper_2603_06492_gb300 import binding as B
    m, k = 32776, 65536
    shape = (k, m) if tall else (m, k)
    i = torch.arange(m, device="cuda")
    j = torch.where(i < 32768, 2 * i, k - 1 - 2 * (i - 32768))
    at = (j, i) if tall else (i, j)
    value = (1.0 + i % 7) * (1 - 2 * (i % 2))
    t = {"grad": torch.zeros(shape, device="cuda"), "momentum": torch.zeros(shape, device="cuda"),
         "param": torch.full(shape, 0.25, device="cuda"), "update": torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda")}
    t["grad"][at] = value
    B.noble_muon_step([t], lr=1.0, nesterov=False, steps=1, eps=0.0)
    torch.cuda.synchronize()
    B.noble_get_device_status(None)
    assert torch.equal(t["momentum"], t["grad"])
    s = value.double() / value.double().norm()
    want = s * (ABC[0] + ABC[1] * s ** 2 + ABC[2] * s ** 4)
    # X, A, B and the new X to 11 bits each, the update to 8
    rel = 4 * 2.0 ** -11
    assert bool(((t["update"][at].double() - want).abs() <= (rel + 2.0 ** -8) * want.abs()).all())
    moved = 0.25 - t["param"][at].double()
    scale = math.sqrt(max(1.0, shape[0] / shape[1]))
    assert bool(((moved - scale * want).abs() <= rel * scale * want.abs() + 2 * U).all())
    t["update"][at] = 0.0
    t["param"][at] = 0.25
    assert not t["update"].any() and bool((t["param"] == 0.25).all())


def test_update_of_a_stack():
    # what Update calls by default, two steps of it: parameters with copies in bf16, products in 11 bits
    from paper_2603_06492_gb300.block import Update
    g = torch.Generator(device="cuda").manual_seed(6)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    d, r = 1024, 64
    shapes = {"W": (3 * d, d), "W_down": (r, d), "W_up": (3 * d, r), "M": (r, r)}
    params = {"table": rn(50, d).bfloat16(), "norms": [], "blocks": [{n: {k: rn(*s).bfloat16() for k, s in shapes.items()} for n in ("qkv", "out")}]}
    grads = {"table": rn(50, d), "norms": [], "blocks": [{n: {"d" + k: rn(*s) for k, s in shapes.items()} for n in ("qkv", "out")}]}
    u = Update(params, grads)
    assert len(u.muon) == 8
    p = [t["param"].double() for t in u.muon]
    m, off = [torch.zeros_like(x) for x in p], [0.0] * len(p)
    for _ in range(2):
        u.step(lr=1e-3, lr_matrices=0.1, weight_decay=0.01)
        for i, t in enumerate(u.muon):
            rows, cols = t["grad"].shape
            m[i] = 0.95 * m[i] + t["grad"].double()
            blend = t["grad"].double() + 0.95 * m[i]
            want = _iterate(blend)
            moved = 0.1 * math.sqrt(max(1.0, rows / cols)) * want
            p[i] = p[i] * (1 - 0.1 * 0.01) - moved
            # of the first step's error the second one keeps nearly all
            off[i] += _tolerance(blend, want, False) * moved.norm() + 4 * U * (p[i].norm() + moved.norm())
    torch.cuda.synchronize()
    for t, want, room in zip(u.muon, p, off):
        assert (t["param"].double() - want).norm() <= room
        assert torch.equal(t["param_bf16"], t["param"].bfloat16())


@pytest.mark.parametrize("precise", [False, True])
@pytest.mark.parametrize("shape", [(1, 65536), (65536, 3), (200, 65536), (65536, 257)])
def test_longest_sums(shape, precise):
    from paper_2603_06492_gb300 import binding as B
    t = _tensors([shape], 8)[0]
    want = _iterate(t["grad"].double() + 0.95 * (0.95 * t["momentum"].double() + t["grad"].double()))
    rel = _tolerance(t["grad"].double() + 0.95 * (0.95 * t["momentum"].double() + t["grad"].double()), want, precise)
    t["param"].zero_()
    B.noble_muon_step([t], lr=1.0, precise=precise)
    torch.cuda.synchronize()
    B.noble_get_device_status(None)
    off = -t["param"].double() / math.sqrt(max(1.0, shape[0] / shape[1])) - want
    assert off.norm() <= rel * want.norm() and off.abs().max() <= 16 * rel * want.abs().max(), (off.norm() / want.norm(), rel)


def test_two_calls_at_once():
    # on streams and workspaces of their own: what one holds of the device, the other waits for
    from paper_2603_06492_gb300 import binding as B
    groups = [_tensors(s, 9) for s in ([(64, 1024), (100, 90)], [(1024, 2048), (64, 1024)], [(1500, 1600)])]
    copies = lambda: [[{k: v.clone() for k, v in t.items()} for t in g] for g in groups]  # noqa: E731
    want = copies()
    for g in want:
        B.noble_muon_step(g, 0.1)
    streams, work = [torch.cuda.Stream() for _ in groups], [B.muon_workspace(g) for g in groups]
    for _ in range(10):
        got = copies()
        torch.cuda.synchronize()
        for g, s, w in zip(got, streams, work):
            B.noble_muon_step(g, 0.1, workspace=w, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(a[k], b[k]) for x, y in zip(got, want) for a, b in zip(x, y) for k in a)
    B.noble_get_device_status(None)
