"""The optimizer step by orthogonalised momentum against its definition in 64 bits.

How far X may be off comes from the same iteration on the CPU in 64 bits with the
roundings that the formats have (A, B and X of each step to 11 or 22 bits): twice that,
as other roundings of the same size give other errors, and for sums in fp32
steps * 3 products * 2^-21 * 4 (a sum is off by 2^-21 of its terms, and one step grows an error by 3.5 at most).
An output in bf16 is rounded once more, 2^-8 of its values.  All of it relative to norms; no
element is off by more than 16 times that of the largest element, which a wrong tile would be.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ABC = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2603_06492_gb300 import binding
    from paper_2603_06492_gb300.build import build
    build()
    binding.load()


def _iterate(u, steps, eps, bits=None):
    def rnd(x):
        if bits is None:
            return x
        m, e = torch.frexp(x)
        return torch.ldexp(torch.round(m * 2.0 ** bits), e - bits)

    x = u / (torch.linalg.matrix_norm(u) + eps)
    tall = x.shape[0] > x.shape[1]
    x = rnd(x.T if tall else x)
    eye = torch.eye(len(x), dtype=torch.float64)
    for _ in range(steps):
        a = rnd(x @ x.T)
        x = rnd(rnd(ABC[0] * eye + ABC[1] * a + ABC[2] * a @ a) @ x)
    return x.T if tall else x


def _near(got, want, rel, what):
    got = got.double().cpu()
    off = got - want
    norm = want.norm()
    assert got.isfinite().all(), what
    assert off.norm() <= rel * norm, (what, (off.norm() / norm).item(), rel)
    assert off.abs().max() <= 16 * rel * want.abs().max(), (what, off.abs().max().item())


def _inputs(shapes, seed=0, spread=0.0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for rows, cols in shapes:
        scale = torch.exp(spread * torch.randn((rows, 1), generator=g))
        rn = lambda: torch.randn((rows, cols), generator=g)  # noqa: E731
        out.append({"grad": 1e-3 * scale * rn(), "momentum": 1e-2 * scale * rn(), "param": 0.02 * rn()})
    return out


def _run(tensors, out=("param", "param_bf16", "update"), **kw):
    from paper_2603_06492_gb300 import binding as B
    dev = []
    for t in tensors:
        d = {k: t[k].cuda() for k in ("grad", "momentum")}
        if "param" in out:
            d["param"] = t["param"].cuda()
        for k in ("param_bf16", "update"):
            if k in out:
                d[k] = torch.full(t["grad"].shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        d.update({k: t[k] for k in ("lr_mult", "decay") if k in t})
        dev.append(d)
    B.noble_muon_step(dev, **kw)
    torch.cuda.synchronize()
    B.noble_get_device_status(None)
    return dev


def _check(tensors, lr=0.5, momentum=0.95, weight_decay=0.1, nesterov=True, steps=5, eps=1e-7, precise=False,
           out=("param", "param_bf16", "update")):
    dev = _run(tensors, out, lr=lr, momentum=momentum, weight_decay=weight_decay, nesterov=nesterov, steps=steps, eps=eps,
               precise=precise)
    for t, d in zip(tensors, dev):
        rows, cols = t["grad"].shape
        what = (rows, cols, steps)
        g, m = t["grad"].double(), t["momentum"].double()
        m = momentum * m + g
        assert bool(((d["momentum"].double().cpu() - m).abs() <= 2 * U * (m.abs() + g.abs() + (m - g).abs())).all()), what
        u = g + momentum * m if nesterov else m
        want = _iterate(u, steps, eps)
        bits = 22 if precise or min(rows, cols) <= 256 else 11
        rough = _iterate(u, steps, eps, bits)
        rel = 2 * ((rough - want).norm() / want.norm()).item() + steps * 3 * 4 * 2.0 ** -21 + 4 * U
        if "update" in out:
            _near(d["update"], want, rel + 2.0 ** -8, what)
        if "param" in out:
            a = lr * t.get("lr_mult", 1.0)
            p = t["param"].double()
            # the parameters' own roundings, and the change's error
            moved = a * math.sqrt(max(1.0, rows / cols)) * want
            base = p * (1 - a * weight_decay) if t.get("decay", True) else p
            off = d["param"].double().cpu() - (base - moved)
            assert off.norm() <= rel * moved.norm() + 4 * U * (p.norm() + moved.norm()), (what, off.norm(), moved.norm(), rel)
            if "param_bf16" in out:
                assert torch.equal(d["param_bf16"], d["param"].bfloat16())
    return dev


SHAPES = [(1, 1), (1, 40), (40, 1), (2, 3), (7, 5), (8, 8), (64, 64), (65, 63), (128, 128), (130, 70), (16, 1000), (1024, 64),
          (255, 257), (256, 256), (257, 300), (300, 1100), (1030, 520), (512, 512), (513, 2000)]


@pytest.mark.parametrize("precise", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_sizes(shape, precise):
    _check(_inputs([shape]), precise=precise)


@pytest.mark.parametrize("steps", [0, 1, 2, 3, 4, 7])
@pytest.mark.parametrize("shape", [(300, 600), (90, 33), (700, 100)])
def test_steps(shape, steps):
    _check(_inputs([shape], 1), steps=steps)


@pytest.mark.parametrize("shapes", [
    [(128, 2048)], [(129, 2048)], [(128, 2049)], [(2041, 127)], [(1, 2048)], [(128, 129), (128, 127)],
    [(64, 1024), (1024, 64), (64, 64)], [(5, 1500), (1, 1), (100, 260), (77, 640)], [(128, 128)] * 16,
    [(33 + 5 * i, 2000 - 100 * i) for i in range(18)], [(100, 300), (140, 300)]])
def test_small_groups(shapes):
    # all iterate in one launch up to 128 rows and 2048 columns, on one to eight blocks each
    _check(_inputs(shapes, 11))


def test_small_alone_and_in_company():
    # blocks of another count add up in another order, and larger matrices take all along to their launches
    t = _inputs([(100, 260), (70, 2000), (300, 300)], 12)
    for n in (1, 2, 3):
        dev = _check(t[:n])
        again = _run(t[:n], lr=0.5, weight_decay=0.1, momentum=0.95, eps=1e-7)
        assert all(torch.equal(a[k], b[k]) for a, b in zip(dev, again) for k in ("param", "momentum", "update"))


@pytest.mark.parametrize("precise", [False, True])
def test_spectra(precise):
    # rows of very different sizes, and a matrix of few directions with little noise
    _check(_inputs([(320, 500)], 2, spread=1.5), precise=precise)
    _check(_inputs([(120, 500)], 2, spread=1.5), precise=precise)
    g = torch.Generator().manual_seed(4)
    t = _inputs([(400, 400)], 3)
    t[0]["momentum"] = torch.randn((400, 5), generator=g) @ torch.randn((5, 400), generator=g) + 0.05 * torch.randn((400, 400), generator=g)
    _check(t, precise=precise)


def test_many_tensors():
    shapes = [(1 + 37 * i % 300, 5 + 53 * i % 290) for i in range(37)]
    tensors = _inputs(shapes, 5)
    for i, t in enumerate(tensors):
        t["lr_mult"], t["decay"] = 0.25 * (i % 5), bool(i % 2)
    _check(tensors)
    _check(tensors, nesterov=False, precise=True)


@pytest.mark.parametrize("out", [("update",), ("param",), ("param", "param_bf16"), ("param", "update")])
def test_outputs(out):
    _check(_inputs([(300, 280), (64, 512)], 6), out=out)


@pytest.mark.parametrize("hp", [dict(momentum=0.0), dict(momentum=0.0, nesterov=False), dict(weight_decay=0.0), dict(lr=0.0),
                                dict(eps=0.0), dict(eps=10.0)])
def test_hyperparameters(hp):
    _check(_inputs([(270, 400), (20, 10)], 7), **hp)


@pytest.mark.parametrize("size", [1e-30, 1e-22, 1e-12, 1e10, 1e22, 1e35])
def test_sizes_of_gradients(size):
    t = _inputs([(290, 310), (3, 5)], 8)
    for x in t:
        x["grad"], x["momentum"] = x["grad"] * size, x["momentum"] * size
    _check(t, eps=0.0)


def test_zero_and_empty_and_non_finite():
    t = _inputs([(300, 300), (300, 300), (40, 70), (300, 300)], 9)
    good = _run([t[0]], lr=0.1)
    t[1]["grad"].zero_(), t[1]["momentum"].zero_()
    t[2]["grad"][3, 4] = float("nan")
    t[3]["grad"][0, 0] = float("inf")
    empty = {k: torch.empty((0, 5)) for k in ("grad", "momentum", "param")}
    dev = _run([t[0], t[1], empty, t[2], t[3]], lr=0.1, weight_decay=0.0, eps=0.0)
    assert not dev[1]["update"].any() and torch.equal(dev[1]["param"].cpu(), t[1]["param"])
    assert dev[3]["update"].isnan().all() and dev[4]["update"].isnan().all()
    u = (t[0]["grad"] + 0.95 * (0.95 * t[0]["momentum"] + t[0]["grad"])).double()
    _near(dev[0]["update"], _iterate(u, 5, 0.0), 0.02, "beside others")
    _near(good[0]["update"], _iterate(u, 5, 1e-7), 0.02, "alone")


def test_small_non_finite_stays_alone():
    t = _inputs([(100, 700), (64, 64), (90, 20)], 13)
    good = _run(t, lr=0.1)
    t[1]["grad"][3, 4] = float("nan")
    dev = _run(t, lr=0.1)
    assert all(torch.equal(dev[i][k], good[i][k]) for i in (0, 2) for k in ("param", "update"))
    assert not dev[1]["update"].isfinite().any()


def test_result_is_orthogonal():
    # a spectrum within a factor of 100: five steps bring every singular value into [0.3, 1.25]
    g = torch.Generator().manual_seed(10)
    q, _ = torch.linalg.qr(torch.randn((300, 300), generator=g, dtype=torch.float64))
    r, _ = torch.linalg.qr(torch.randn((700, 300), generator=g, dtype=torch.float64))
    u = ((q * torch.logspace(-2, 0, 300, dtype=torch.float64)) @ r.T).float()
    t = {"grad": u, "momentum": torch.zeros_like(u), "param": torch.zeros_like(u)}
    for precise in (False, True):
        x = _run([t], ("update",), lr=0.0, nesterov=False, precise=precise)[0]["update"].double().cpu()
        s = torch.linalg.svdvals(x)
        assert s.max() <= 1.25 and s.min() >= 0.3, (s.min(), s.max())


@pytest.mark.parametrize("precise", [False, True])
@pytest.mark.parametrize("shapes", [[(300, 900), (512, 64), (64, 64), (1100, 300)], [(100, 900), (513, 61), (64, 64)]])
def test_repeats_streams_and_graphs(precise, shapes):
    from paper_2603_06492_gb300 import binding as B
    t = _inputs(shapes, 11)
    want = _run(t, lr=0.1, precise=precise)
    again = _run(t, lr=0.1, precise=precise)
    keys = ("param", "param_bf16", "momentum", "update")
    assert all(torch.equal(a[k], b[k]) for a, b in zip(want, again) for k in keys)
    first = [{k: (t[i][k].cuda() if k in t[i] else torch.empty_like(want[i][k])) for k in (*keys, "grad")} for i in range(len(t))]
    dev = [{k: v.clone() for k, v in d.items()} for d in first]
    ws = B.muon_workspace(dev, precise)
    ws.fill_(255)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    B.noble_muon_step(dev, 0.1, precise=precise, workspace=ws, stream=side)
    side.synchronize()
    assert all(torch.equal(a[k], b[k]) for a, b in zip(dev, want) for k in keys)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.noble_muon_step(dev, 0.1, precise=precise, workspace=ws)
    for _ in range(2):
        for d, f in zip(dev, first):
            for k in d:
                d[k].copy_(f[k])
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a[k], b[k]) for a, b in zip(dev, want) for k in keys)


def test_neighbours_keep_their_values():
    # odd sizes: nothing behind a tensor or the workspace is touched
    from paper_2603_06492_gb300 import binding as B
    rows, cols = 131, 77
    n = rows * cols
    t = _inputs([(rows, cols)], 12)[0]
    room = {k: torch.full((n + 64,), 3.0, dtype=torch.bfloat16 if k in ("update", "param_bf16") else torch.float32, device="cuda")
            for k in ("param", "param_bf16", "grad", "momentum", "update")}
    dev = {k: v[:n].view(rows, cols) for k, v in room.items()}
    for k in ("param", "grad", "momentum"):
        dev[k].copy_(t[k])
    need = B.muon_workspace([dev]).numel()
    ws = torch.full((need + 4096,), 171, dtype=torch.uint8, device="cuda")
    B.noble_muon_step([dev], 0.1, workspace=ws[:need])
    torch.cuda.synchronize()
    assert bool((ws[need:] == 171).all()) and all(bool((v[n:] == 3.0).all()) for v in room.values())
    assert torch.equal(dev["grad"].cpu(), t["grad"])
