"""Norm and rotation of queries and keys, its gradients, and appending to a paged cache,
against their definitions in 64 bits.

Error: max |got - ref| / max |ref|.  Elementwise work: fp32 1e-5 (2^-24 a step, sums of up
to 256 squares), bf16 1e-2 (an output is rounded once, to 2^-9 of itself); gain gradients
are fp32 sums over tokens and heads and within 1e-5 for either type.
"""
import math

import pytest
import torch

from tests import attention_ref as ref
from tests.gpu_helpers import TOL, rel_err

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2603_06492_gb300 import binding
    from paper_2603_06492_gb300.build import build
    build()
    binding.load()


def _table(n, rot, seed=1):
    a = torch.rand((n, rot // 2), generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * 6.3
    return torch.cat([a.cos(), a.sin()], 1).float()


def _case(T, nq, nkv, d, rot, dtype, norm=True, positions=50, seed=0):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn((T, (nq + 2 * nkv) * d), generator=g).to(DT[dtype])
    pos = torch.randint(0, positions, (T,), generator=g).int()
    gains = [1 + 0.3 * torch.randn(d, generator=g) for _ in range(2)] if norm else [None, None]
    dq, dk = (torch.randn((T, n, d), generator=g).to(DT[dtype]) for n in (nq, nkv))
    return qkv, pos, _table(positions, rot), gains, dq, dk


def _cuda(*xs):
    return [None if x is None else x.cuda() for x in xs]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("T,nq,nkv,d,rot,interleaved", [
    (1, 1, 1, 8, 8, False), (1, 3, 1, 64, 64, True), (5, 16, 4, 128, 128, False), (37, 7, 2, 128, 64, False),
    (19, 2, 2, 64, 32, True), (33, 3, 3, 80, 20, False), (33, 3, 3, 80, 20, True), (9, 4, 2, 96, 96, False),
    (21, 5, 1, 40, 6, False), (21, 5, 1, 40, 6, True), (12, 2, 1, 256, 256, False), (12, 2, 1, 256, 130, True),
    (8, 33, 3, 64, 0, False), (600, 4, 4, 72, 48, False), (600, 9, 3, 16, 16, True), (3, 1, 1, 24, 2, True)])
def test_rope(T, nq, nkv, d, rot, interleaved, norm, dtype):
    from paper_2603_06492_gb300 import attention as A, binding
    qkv, pos, table, (gq, gk), dq, dk = _case(T, nq, nkv, d, rot, dtype, norm)
    buf = A.RopeBuffers(T, nq, nkv, d, dtype, rot=rot, positions=50, norm=norm, interleaved=interleaved)
    args = _cuda(qkv, pos, table, gq, gk)
    for x in (buf.q, buf.k, buf.dqkv, buf.dgain_q, buf.dgain_k):
        x.fill_(float("nan"))
    yq, yk = A.rope_forward(buf, *args)
    dxq, dxk = A.rope_backward(buf, *_cuda(dq, dk), *args)
    torch.cuda.synchronize()
    binding.noble_get_device_status(None)
    h = qkv.view(T, nq + 2 * nkv, d)
    for x, y, dx, dy, gain, dgain in ((h[:, :nq], yq, dxq, dq, gq, buf.dgain_q),
                                      (h[:, nq:nq + nkv], yk, dxk, dk, gk, buf.dgain_k)):
        wy, wdx, wdg = ref.rope(x, pos, table, rot, interleaved, gain, 1e-6, norm, dy)
        assert rel_err(y.float().cpu(), wy) <= TOL[dtype]
        # d = 8 and all alike: dx may cancel; it is held to dy's scale then
        assert float((dx.double().cpu() - wdx).abs().max()) <= TOL[dtype] * max(float(wdx.abs().max()), float(dy.abs().max()))
        if norm:
            assert rel_err(dgain.cpu(), wdg) <= 1e-5
    assert torch.isnan(buf.dxv).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_zero_heads_and_defaults(dtype):
    # a head of zeros: eps keeps its norm and gradients finite; gains default to ones
    from paper_2603_06492_gb300 import attention as A
    qkv, pos, table, _, dq, dk = _case(4, 2, 1, 64, 64, dtype)
    qkv[1] = 0
    buf = A.RopeBuffers(4, 2, 1, 64, dtype, positions=50)
    args = _cuda(qkv, pos, table)
    yq, _ = A.rope_forward(buf, *args)
    dxq, _ = A.rope_backward(buf, *_cuda(dq, dk), *args)
    wy, wdx, wdg = ref.rope(qkv.view(4, 4, 64)[:, :2], pos, table, 64, False, None, 1e-6, True, dq)
    assert rel_err(yq.float().cpu(), wy) <= TOL[dtype] and rel_err(dxq.float().cpu(), wdx) <= TOL[dtype]
    assert rel_err(buf.dgain_q.cpu(), wdg) <= 1e-5


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [64, 20])
def test_gradient_against_differences(interleaved, rot):
    # <dx, u> and <dgain, w> against the 64-bit definition's central differences
    from paper_2603_06492_gb300 import attention as A
    T, nq, nkv, d = 11, 3, 2, 64
    qkv, pos, table, (gq, gk), dq, dk = _case(T, nq, nkv, d, rot, "fp32")
    buf = A.RopeBuffers(T, nq, nkv, d, "fp32", rot=rot, positions=50, interleaved=interleaved)
    args = _cuda(qkv, pos, table, gq, gk)
    dxq, _ = A.rope_backward(buf, *_cuda(dq, dk), *args)
    x = qkv.view(T, -1, d)[:, :nq].double()
    g = torch.Generator().manual_seed(3)
    u, w = torch.randn(x.shape, generator=g, dtype=torch.float64), torch.randn(d, generator=g, dtype=torch.float64)
    value = lambda x, gain: float((ref.rope(x, pos, table, rot, interleaved, gain) * dq.double()).sum())  # noqa: E731
    h = 1e-5
    dx = (value(x + h * u, gq.double()) - value(x - h * u, gq.double())) / (2 * h)
    dg = (value(x, gq.double() + h * w) - value(x, gq.double() - h * w)) / (2 * h)
    assert abs(float((dxq.double().cpu() * u).sum()) - dx) <= 1e-5 * float(u.norm() * dxq.double().norm().cpu())
    assert abs(float((buf.dgain_q.double().cpu() * w).sum()) - dg) <= 1e-5 * float(w.norm() * buf.dgain_q.double().norm().cpu())


def test_in_place_and_strides():
    # the packed projection output as its own result, through the C entry point
    from paper_2603_06492_gb300 import attention as A, binding
    T, nq, nkv, d = 50, 4, 2, 64
    qkv, pos, table, (gq, gk), dq, dk = _case(T, nq, nkv, d, d, "bf16")
    buf = A.RopeBuffers(T, nq, nkv, d, "bf16", positions=50)
    args = _cuda(qkv, pos, table, gq, gk)
    yq, yk = (x.clone() for x in A.rope_forward(buf, *args))
    wide = torch.zeros((T, (nq + 2 * nkv) * d + 24), dtype=torch.bfloat16, device="cuda")
    x = wide[:, 8:8 + (nq + 2 * nkv) * d]
    x.copy_(args[0])
    A.rope_forward(buf, x, *args[1:])
    assert torch.equal(buf.q, yq) and torch.equal(buf.k, yk)
    import ctypes
    row = wide.stride(0)
    hq, hk = (binding.Heads(x.data_ptr() + 2 * o, row, d) for o in (0, nq * d))
    r = [ctypes.byref(hq), ctypes.byref(hk)]
    binding._check(binding.load().noble_rope_fwd(buf._ref, *r, *(t.data_ptr() for t in args[1:]), *r, None))
    torch.cuda.synchronize()
    h = x.view(T, -1, d) if x.is_contiguous() else x.reshape(T, -1, d)
    assert torch.equal(h[:, :nq], yq) and torch.equal(h[:, nq:nq + nkv], yk)
    assert torch.equal(h[:, nq + nkv:], args[0].view(T, -1, d)[:, nq + nkv:]) and not wide[:, :8].any() and not wide[:, -16:].any()


@pytest.mark.parametrize("bad", [-1, 50, 2 ** 31 - 1, -2 ** 31])
def test_position_beyond_the_table(bad):
    from paper_2603_06492_gb300 import attention as A, binding
    qkv, pos, table, (gq, gk), dq, dk = _case(6, 2, 1, 64, 64, "bf16")
    pos[3] = bad
    buf = A.RopeBuffers(6, 2, 1, 64, "bf16", positions=50)
    args = _cuda(qkv, pos, table, gq, gk)
    yq, _ = A.rope_forward(buf, *args)
    with pytest.raises(binding.NobleError):
        binding.noble_get_device_status(None)
    assert not yq[3].any() and yq[2].any()
    dxq, _ = A.rope_backward(buf, *_cuda(dq, dk), *args)
    with pytest.raises(binding.NobleError):
        binding.noble_get_device_status(None)
    assert not dxq[3].any() and torch.isfinite(buf.dgain_q).all()


@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0), dict(factor=4.0, low_turns=math.inf, high_turns=math.inf),
                                dict(factor=8.0, original=4096.0, low_turns=1.0, high_turns=32.0, amplitude=1.2)])
@pytest.mark.parametrize("rot", [2, 64, 128])
def test_table(rot, kw):
    from paper_2603_06492_gb300 import attention as A
    n = 5000
    got = A.rope_table(n, rot, **kw).cpu().double()
    p = dict(base=10000.0, factor=1.0, original=1.0, low_turns=0.0, high_turns=0.0, amplitude=1.0)
    p.update(kw)
    for i in range(rot // 2):
        f = p["base"] ** (-2.0 * i / rot)
        if p["factor"] != 1.0:
            t = p["original"] * f / (2 * math.pi)
            g = 1.0 if t >= p["high_turns"] else 0.0 if t <= p["low_turns"] else \
                (t - p["low_turns"]) / (p["high_turns"] - p["low_turns"])
            f = f * (g + (1 - g) / p["factor"])
        a = torch.arange(n, dtype=torch.float64) * f
        # fp32 results of fp64 angles: 2^-24 of values up to 1.2, and 2^-52 of an angle of 5000
        assert float((got[:, i] - p["amplitude"] * a.cos()).abs().max()) <= 1.2e-7
        assert float((got[:, rot // 2 + i] - p["amplitude"] * a.sin()).abs().max()) <= 1.2e-7


# ---------------------------------------------------------------- the cache
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("T,nq,nkv,d,rot,interleaved,page", [
    (1, 4, 1, 64, 64, False, 16), (24, 16, 4, 128, 128, False, 64), (77, 3, 3, 80, 20, True, 1), (130, 8, 2, 96, 48, False, 7),
    (9, 2, 1, 8, 8, True, 128)])
def test_append(T, nq, nkv, d, rot, interleaved, page, norm, dtype):
    from paper_2603_06492_gb300 import attention as A, binding
    qkv, pos, table, (gq, gk), _, _ = _case(T, nq, nkv, d, rot, dtype, norm)
    pages = -(-T // page) + 2
    g = torch.Generator().manual_seed(9)
    slots = torch.randperm(pages * page, generator=g)[:T].clone()
    if T > 5:
        slots[3] = -1
    cache = A.PagedCache(pages, page, nkv, d, dtype)
    cache.k.fill_(7.0), cache.v.fill_(-7.0)
    buf = A.RopeBuffers(T, nq, nkv, d, dtype, rot=rot, positions=50, norm=norm, interleaved=interleaved, with_grads=False)
    yq = A.kv_append(buf, cache, *_cuda(qkv, pos, slots, table, gq, gk))
    torch.cuda.synchronize()
    binding.noble_get_device_status(None)
    h = qkv.view(T, nq + 2 * nkv, d)
    assert rel_err(yq.float().cpu(), ref.rope(h[:, :nq], pos, table, rot, interleaved, gq, 1e-6, norm)) <= TOL[dtype]
    k = torch.full((pages * page, nkv, d), 7.0, dtype=torch.float64)
    v = torch.full((pages * page, nkv, d), -7.0).to(DT[dtype])
    real = slots >= 0
    k[slots[real]] = ref.rope(h[:, nq:nq + nkv], pos, table, rot, interleaved, gk, 1e-6, norm)[real]
    v[slots[real]] = h[:, nq + nkv:][real]
    assert rel_err(cache.k.float().cpu().view(-1, nkv, d), k) <= TOL[dtype]
    assert torch.equal(cache.v.cpu().view(-1, nkv, d), v)


def test_append_layout_and_bounds():
    """Keys and values interleaved in one allocation, heads outside of tokens; slots beyond
    the cache are left out and reported."""
    from paper_2603_06492_gb300 import attention as A, binding
    T, nq, nkv, d, page, pages = 10, 4, 2, 64, 8, 4
    qkv, pos, table, (gq, gk), _, _ = _case(T, nq, nkv, d, d, "bf16")
    both = torch.zeros((pages, 2, nkv, page, d), dtype=torch.bfloat16, device="cuda")
    k, v = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
    cache = A.PagedCache(pages, page, nkv, d, "bf16", k=k, v=v)
    plain = A.PagedCache(pages, page, nkv, d, "bf16")
    plain.k.zero_(), plain.v.zero_()
    buf = A.RopeBuffers(T, nq, nkv, d, "bf16", positions=50, with_grads=False)
    slots = torch.tensor([0, 9, 31, 17, -5, 3, 32, 2 ** 40, 12, 30])
    for c in (plain, cache):
        A.kv_append(buf, c, *_cuda(qkv, pos, slots, table, gq, gk))
        with pytest.raises(binding.NobleError):
            binding.noble_get_device_status(None)
    assert torch.equal(k, plain.k) and torch.equal(v, plain.v)
    touched = plain.v.view(-1, nkv * d).any(1).cpu()
    assert touched.nonzero()[:, 0].tolist() == [0, 3, 9, 12, 17, 30, 31]


def test_append_beyond_32_bits():
    # element offsets beyond 2^32 in a cache of 9 GB
    from paper_2603_06492_gb300 import attention as A
    nkv, d, page = 8, 128, 64
    pages = (2 ** 32 + 2 ** 22) // (nkv * d * page)
    qkv, pos, table, (gq, gk), _, _ = _case(3, 8, nkv, d, d, "bf16")
    cache = A.PagedCache(pages, page, nkv, d, "bf16")
    last = pages * page - 1
    cache.v[-1].zero_(), cache.v[0].zero_()
    buf = A.RopeBuffers(3, 8, nkv, d, "bf16", positions=50, with_grads=False)
    A.kv_append(buf, cache, *_cuda(qkv, pos, torch.tensor([last, 5, last - 70]), table, gq, gk))
    v = qkv.view(3, -1, d)[:, 16:]
    assert torch.equal(cache.v[-1, -1].cpu(), v[0]) and torch.equal(cache.v[0, 5].cpu(), v[1])
    assert torch.equal(cache.v.view(-1, nkv, d)[last - 70].cpu(), v[2]) and not cache.v[0, :5].any()
