"""Layer norm, with and without the residual stream, and its gradients, against the
definition in 64 bits.

Tolerances, of u = 2^-24: a bf16 output is rounded once, 2^-8 of its value at most.  In
fp32, a mean of d elements is off by at most (d / 32 + 16) u of the largest element
(a lane's elements one by one, then a tree; d / 32 bounds the lane's), and every element
of y and dx by a few such errors: 4 (d / 32 + 16) u of the largest product that goes into
it.  dgain and dbias add up to 512 rows one by one, then parts: (rows of a part + parts / 32 + 64) u
of the sum of the terms' magnitudes, and the terms are off as y is.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp32": U}


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2603_06492_gb300 import binding
    from paper_2603_06492_gb300.build import build
    build()
    binding.load()


def _inputs(T, d, dtype, seed=0, offset=0.3):
    g = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    x, res, dy, dstream = ((rn(T, d) * s + o).to(DT[dtype]) for s, o in ((1.5, offset), (0.5, 0.0), (1.0, 0.1), (1.0, 0.0)))
    return x, res, dy, dstream, 1 + 0.2 * rn(d), 0.1 * rn(d)


def _reference(x, res, dy, dstream, gain, bias, eps, dtype):
    s = x if res is None else (x.double() + res.double()).to(DT[dtype])
    z = s.double()
    mean = z.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((z - mean) ** 2).mean(1, keepdim=True) + eps)
    n = (z - mean) * rstd
    ga = torch.ones(x.shape[1]) if gain is None else gain
    y = n * ga.double() + (0 if bias is None else bias.double())
    w = dy.double() * ga.double()
    dx = rstd * (w - w.mean(1, keepdim=True) - n * (w * n).mean(1, keepdim=True))
    if dstream is not None:
        dx = dx + dstream.double()
    big = {"y": (n * ga).abs().amax() + z.abs().amax() * rstd.amax() * ga.abs().amax() + 1,
           "dx": rstd.amax() * w.abs().amax() * (2 + n.abs().amax() ** 2) * (1 + z.abs().amax() * rstd.amax())
           + (0 if dstream is None else dstream.double().abs().amax())}
    return s, y, dx, (dy.double() * n).sum(0), dy.double().sum(0), n, big


def _close(got, want, tol, what):
    off = (got.double().cpu() - want).abs()
    assert bool((off <= tol).all()), (what, off.max().item(), (off / tol).max().item())


def _check(T, d, dtype, res=True, gain=True, bias=True, eps=1e-5, seed=0, offset=0.3):
    from paper_2603_06492_gb300 import layers as L
    x, r, dy, dstream, ga, bi = _inputs(T, d, dtype, seed, offset)
    r, dstream = (r, dstream) if res else (None, None)
    ga, bi = ga if gain else None, bi if bias else None
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    b = L.NormBuffers(T, d, dtype, eps=eps, residual=res)
    for out in (b.y, b.dx, b.dgain, b.dbias):
        out.fill_(float("nan"))
    y = L.norm_forward(b, cu(x), cu(ga), cu(bi), res=cu(r))
    s, wy, wdx, wdg, wdb, n, big = _reference(x, r, dy, dstream, ga, bi, eps, dtype)
    if res:
        assert torch.equal(b.sum.cpu(), s)
    dx = L.norm_backward(b, cu(dy), b.sum if res else cu(x), cu(ga), dstream=cu(dstream))
    each = 4 * (d / 32 + 16) * U
    _close(y, wy, HALF[dtype] * wy.abs() + each * big["y"], "y")
    _close(dx, wdx, HALF[dtype] * wdx.abs() + each * big["dx"], "dx")
    rows = min(512, max(1, -(-T // 152)))  # of a part
    adds = (rows + (T / rows) / 32 + 64) * U
    many = dy.double().abs().sum(0)
    _close(b.dgain, wdg, (adds + each) * (many * n.abs().amax() + many * big["y"]), "dgain")
    _close(b.dbias, wdb, adds * many, "dbias")
    return b


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,d", [(1, 8), (3, 16), (5, 64), (2, 136), (24, 256), (33, 264), (7, 512), (300, 768), (9, 1000), (64, 1024),
                                 (17, 1032), (11, 2048), (5, 2056), (3, 4096), (2, 5504), (4, 8192), (1, 8200), (2, 16384), (3, 16376),
                                 # rows through the ring
                                 (607, 8), (608, 8), (650, 136), (700, 768), (611, 776), (700, 1000), (640, 1032), (609, 2056),
                                 (608, 4104), (700, 5504), (613, 7680), (609, 7688), (610, 8200), (608, 16384)])
def test_sizes(T, d, dtype):
    _check(T, d, dtype)
    _check(T, d, dtype, res=False, seed=1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("res,gain,bias", [(True, False, True), (False, True, False), (True, False, False), (False, False, True)])
def test_parts_left_out(res, gain, bias, dtype):
    _check(50, 320, dtype, res, gain, bias)


@pytest.mark.parametrize("T", [151, 303, 304, 608, 609, 2432, 2433, 9000, 160000])
def test_rows(T):
    # parts of one row more or less, many parts, parts of 512 rows
    _check(T, 64, "bf16")


@pytest.mark.parametrize("T", [40, 640])
@pytest.mark.parametrize("d", [512, 2048])
def test_large_mean(T, d):
    # the variance is of what is left after the mean: 1000 +- 1.5 in fp32
    _check(T, d, "fp32", res=False, offset=1000.0)


@pytest.mark.parametrize("T", [20, 640])
def test_small_eps(T):
    _check(T, 256, "fp32", eps=1e-30)
    _check(T, 256, "fp32", eps=0.0)


def test_sums_of_like_rows():
    # 65536 equal rows: sums stay short of what running sums would lose
    from paper_2603_06492_gb300 import layers as L
    T, d = 65536, 64
    x, _, dy, _, ga, bi = _inputs(1, d, "fp32")
    b = L.NormBuffers(T, d, "fp32")
    X, DY = x.expand(T, d).contiguous().cuda(), dy.expand(T, d).contiguous().cuda()
    L.norm_forward(b, X, ga.cuda(), bi.cuda())
    L.norm_backward(b, DY, X, ga.cuda())
    want = T * dy[0].double()
    _close(b.dbias, want, 700 * U * want.abs(), "dbias")


@pytest.mark.parametrize("T", [20, 700])
def test_non_finite_rows_stay_apart(T):
    from paper_2603_06492_gb300 import layers as L
    d = 256
    x, r, dy, ds, ga, bi = (t.cuda() for t in _inputs(T, d, "bf16"))
    b = L.NormBuffers(T, d, "bf16", residual=True)
    y0 = L.norm_forward(b, x, ga, bi, res=r).clone()
    d0 = L.norm_backward(b, dy, b.sum, ga, dstream=ds).clone()
    x[3, 5], x[7, 0], dy[7] = float("nan"), float("inf"), float("nan")
    y1 = L.norm_forward(b, x, ga, bi, res=r)
    d1 = L.norm_backward(b, dy, b.sum, ga, dstream=ds)
    keep = [i for i in range(T) if i not in (3, 7)]
    assert torch.equal(y0[keep], y1[keep]) and torch.equal(d0[keep], d1[keep])
    assert y1[3].isnan().all() and y1[7].isnan().all()


@pytest.mark.parametrize("T", [37, 1000])
def test_in_place(T):
    # sum over x, y over res; dx over dy or over dstream
    from paper_2603_06492_gb300 import binding as B, layers as L
    d = 1024
    x, r, dy, ds, ga, bi = (t.cuda() for t in _inputs(T, d, "bf16"))
    b = L.NormBuffers(T, d, "bf16", residual=True)
    y0 = L.norm_forward(b, x, ga, bi, res=r).clone()
    s0, dx0 = b.sum.clone(), L.norm_backward(b, dy, b.sum, ga, dstream=ds).clone()
    x1, r1 = x.clone(), r.clone()
    lib, p, st = B.load(), lambda t: t.data_ptr(), B._stream_handle(None)
    B._check(lib.noble_norm_fwd(b._ref, p(x1), p(r1), p(ga), p(bi), p(x1), p(r1), p(b.stats), st))
    assert torch.equal(x1, s0) and torch.equal(r1, y0)
    for which in (0, 1):
        t = [dy.clone(), ds.clone()]
        B._check(lib.noble_norm_bwd(b._ref, p(t[0]), p(s0), p(b.stats), p(ga), p(t[1]), p(t[which]), p(b.dgain), p(b.dbias),
                                    p(b.workspace), b.workspace_bytes, st))
        assert torch.equal(t[which], dx0)


def test_gradients_are_optional_and_empty_batches():
    from paper_2603_06492_gb300 import binding as B, layers as L
    x, _, dy, _, ga, _ = (t.cuda() for t in _inputs(30, 128, "fp32"))
    b = L.NormBuffers(30, 128, "fp32")
    L.norm_forward(b, x, ga)
    dx = L.norm_backward(b, dy, x, ga).clone()
    dg, db = b.dgain.clone(), b.dbias.clone()
    lib, p, st = B.load(), lambda t: t.data_ptr(), B._stream_handle(None)
    for skip_g, skip_b in ((True, False), (False, True), (True, True)):
        for t in (b.dx, b.dgain, b.dbias):
            t.fill_(7.0)
        B._check(lib.noble_norm_bwd(b._ref, p(dy), p(x), p(b.stats), p(ga), None, p(b.dx), None if skip_g else p(b.dgain),
                                    None if skip_b else p(b.dbias), p(b.workspace), b.workspace_bytes, st))
        assert torch.equal(b.dx, dx)
        assert torch.equal(b.dgain, torch.full_like(dg, 7.0) if skip_g else dg)
        assert torch.equal(b.dbias, torch.full_like(db, 7.0) if skip_b else db)
    e = L.NormBuffers(0, 128, "fp32")
    e.dgain.fill_(3.0), e.dbias.fill_(3.0)
    L.norm_forward(e, x[:0], ga)
    L.norm_backward(e, dy[:0], x[:0], ga)
    assert not e.dgain.any() and not e.dbias.any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_inference_repeats_streams_and_graphs(dtype):
    from paper_2603_06492_gb300 import layers as L
    T, d = 1000, 768
    x, r, dy, ds, ga, bi = (t.cuda() for t in _inputs(T, d, dtype))
    b, light = L.NormBuffers(T, d, dtype, residual=True), L.NormBuffers(T, d, dtype, residual=True, with_grads=False)

    def step(stream=None):
        L.norm_forward(b, x, ga, bi, res=r, stream=stream)
        L.norm_backward(b, dy, b.sum, ga, dstream=ds, stream=stream)

    step()
    want = [t.clone() for t in (b.y, b.sum, b.dx, b.dgain, b.dbias)]
    assert torch.equal(L.norm_forward(light, x, ga, bi, res=r), want[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert all(torch.equal(t, w) for t, w in zip((b.y, b.sum, b.dx, b.dgain, b.dbias), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    dy.neg_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(b.y, want[0]) and torch.equal(b.dgain, -want[3]) and torch.equal(b.dbias, -want[4])


def test_gradients_against_differences():
    # L = sum(y t) along random directions, central differences of the definition in 64 bits
    from paper_2603_06492_gb300 import layers as L
    T, d, eps = 6, 64, 1e-5
    x, _, t, _, ga, bi = _inputs(T, d, "fp32", seed=5)
    b = L.NormBuffers(T, d, "fp32", eps=eps)
    L.norm_forward(b, x.cuda(), ga.cuda(), bi.cuda())
    dx = L.norm_backward(b, t.cuda(), x.cuda(), ga.cuda())
    g = torch.Generator().manual_seed(9)
    loss = lambda x, ga, bi: (torch.nn.functional.layer_norm(x, (d,), ga, bi, eps) * t.double()).sum()  # noqa: E731
    for _ in range(3):
        v = [torch.randn(s.shape, generator=g).double() for s in (x, ga, bi)]
        h = 1e-5
        at = lambda k: loss(*(p.double() + k * h * q for p, q in zip((x, ga, bi), v)))  # noqa: E731
        slope = (at(1) - at(-1)) / (2 * h)
        mine = sum((a.double().cpu() * q).sum() for a, q in zip((dx, b.dgain, b.dbias), v))
        # third derivatives of rows of O(1): h^2 of the sum of magnitudes; the gradients' own errors 1e-5 of it
        assert abs(mine - slope) <= 1e-5 * sum((a.double().cpu() * q).abs().sum() for a, q in zip((dx, b.dgain, b.dbias), v))


def test_offsets_beyond_32_bits():
    # 2.2e9 elements: the last rows come out as in a call of their own
    from paper_2603_06492_gb300 import layers as L
    T, d, n = 532000, 4096, 700
    g = torch.Generator(device="cuda").manual_seed(2)
    x, dy = (torch.empty((T, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x.fill_(1.0), dy.zero_()
    x[:, 0] = 3.0
    x[-n:], dy[-n:] = (torch.randn((n, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    ga, bi = torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    b, few = L.NormBuffers(T, d, "bf16"), L.NormBuffers(n, d, "bf16")
    assert torch.equal(L.norm_forward(b, x, ga, bi)[-n:], L.norm_forward(few, x[-n:], ga, bi))
    assert torch.equal(L.norm_backward(b, dy, x, ga)[-n:], L.norm_backward(few, dy[-n:], x[-n:], ga))
    assert torch.allclose(b.dgain, few.dgain, rtol=0, atol=1e-3) and torch.allclose(b.dbias, few.dbias, rtol=0, atol=1e-3)
