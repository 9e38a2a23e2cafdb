"""Paths of the attention operators that small calls do not take: tokens beyond a batch per warp in the
rotation, tables of documents that do not fit shared memory, long documents, element offsets
beyond 2^32, and calls captured in a graph.  Errors and tolerances as in test_rope_gpu.py and
test_attention_gpu.py."""
import math

import pytest
import torch

from tests import attention_ref as ref
from tests.gpu_helpers import TOL, rel_err
from tests.test_attention_gpu import _check, _compare, _inputs
from tests.test_rope_gpu import _case, _cuda

pytestmark = pytest.mark.gpu
both = pytest.mark.parametrize("dtype", ["bf16", "fp32"])
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2603_06492_gb300 import binding
    from paper_2603_06492_gb300.build import build
    build()
    binding.load()


@pytest.fixture(autouse=True)
def no_device_error():
    from paper_2603_06492_gb300 import binding
    binding.noble_debug_rows_again()
    yield
    binding.noble_get_device_status(None)
    assert binding.noble_debug_rows_again() == 0


# ---------------------------------------------------------------- rotation
# more than 24 * 152 batches forward, 2 * 152 * 8 backward: all batches of a token by one warp, a ring
# that goes round, sums over several units of a warp
@both
@pytest.mark.parametrize("T,nq,nkv,d,rot,interleaved,norm", [
    (1300, 16, 4, 128, 128, False, True), (1300, 17, 4, 128, 64, True, True), (1900, 35, 3, 64, 64, False, True),
    (1300, 30, 9, 80, 20, False, True), (1300, 30, 9, 80, 20, True, False), (1237, 40, 1, 64, 32, True, False),
    (1300, 9, 8, 256, 256, False, True), (3700, 3, 2, 16, 6, False, True)])
def test_many_tokens_rotate(T, nq, nkv, d, rot, interleaved, norm, dtype):
    from paper_2603_06492_gb300 import attention as A
    qkv, pos, table, (gq, gk), dq, dk = _case(T, nq, nkv, d, rot, dtype, norm)
    buf = A.RopeBuffers(T, nq, nkv, d, dtype, rot=rot, positions=50, norm=norm, interleaved=interleaved)
    args = _cuda(qkv, pos, table, gq, gk)
    for x in (buf.q, buf.k, buf.dqkv, buf.dgain_q, buf.dgain_k):
        x.fill_(float("nan"))
    yq, yk = A.rope_forward(buf, *args)
    dxq, dxk = A.rope_backward(buf, *_cuda(dq, dk), *args)
    h = qkv.view(T, nq + 2 * nkv, d)
    for x, y, dx, dy, gain, dgain in ((h[:, :nq], yq, dxq, dq, gq, buf.dgain_q),
                                      (h[:, nq:nq + nkv], yk, dxk, dk, gk, buf.dgain_k)):
        wy, wdx, wdg = ref.rope(x, pos, table, rot, interleaved, gain, 1e-6, norm, dy)
        assert rel_err(y.float().cpu(), wy) <= TOL[dtype] and rel_err(dx.float().cpu(), wdx) <= TOL[dtype]
        if norm:
            assert rel_err(dgain.cpu(), wdg) <= 1e-5


@both
@pytest.mark.parametrize("T,nq,nkv,d,rot,interleaved", [(1300, 16, 4, 128, 128, False), (1300, 16, 16, 64, 32, True), (1300, 30, 9, 80, 20, False)])
def test_many_tokens_are_appended(T, nq, nkv, d, rot, interleaved, dtype):
    from paper_2603_06492_gb300 import attention as A
    qkv, pos, table, (gq, gk), _, _ = _case(T, nq, nkv, d, rot, dtype)
    page, pages = 16, T // 16 + 3
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(9))[:T]
    cache = A.PagedCache(pages, page, nkv, d, dtype)
    cache.k.zero_(), cache.v.zero_()
    buf = A.RopeBuffers(T, nq, nkv, d, dtype, rot=rot, positions=50, interleaved=interleaved, with_grads=False)
    yq = A.kv_append(buf, cache, *_cuda(qkv, pos, slots, table, gq, gk))
    h = qkv.view(T, nq + 2 * nkv, d)
    assert rel_err(yq.float().cpu(), ref.rope(h[:, :nq], pos, table, rot, interleaved, gq)) <= TOL[dtype]
    k = torch.zeros((pages * page, nkv, d), dtype=torch.float64)
    v = torch.zeros((pages * page, nkv, d), dtype=DT[dtype])
    k[slots], v[slots] = ref.rope(h[:, nq:nq + nkv], pos, table, rot, interleaved, gk), h[:, nq + nkv:]
    assert rel_err(cache.k.float().cpu().view(-1, nkv, d), k) <= TOL[dtype]
    assert torch.equal(cache.v.cpu().view(-1, nkv, d), v)


# ---------------------------------------------------------------- documents
@pytest.mark.parametrize("n", [127, 128, 1023, 1024, 1500])
@pytest.mark.parametrize("kw", [dict(), dict(causal=False, window=5), dict(prefix=True)])
def test_many_documents(n, kw):
    # starts in shared memory of all kernels, of some, of none; some documents empty
    T, g = 1800, torch.Generator().manual_seed(n)
    docs = sorted(torch.randint(3, T - 2, (n - 1,), generator=g).tolist())
    docs = [3, *docs, T - 2]
    kw = dict(kw)
    if kw.pop("prefix", False):
        kw["prefix"] = torch.randint(0, 9, (n,), generator=g).tolist()
    _check(T, 2, 1, 64, docs, "bf16", **kw)


@both
def test_long_document(dtype):
    _check(5000, 2, 1, 128, [0, 5000], dtype)


# ---------------------------------------------------------------- offsets
@both
def test_offsets_beyond_32_bits(dtype):
    """All tensors side by side in rows of 2^24 elements, of which 300 make 5e9."""
    from paper_2603_06492_gb300 import attention as A
    T, nq, nkv, d, docs = 300, 4, 2, 64, [0, 130, 300]
    mem = torch.empty((T, 2 ** 24), dtype=DT[dtype], device="cuda")
    used = 0

    def place(x):
        nonlocal used
        n = x.shape[1]
        out = mem[:, used:used + n * d].view(T, n, d)
        used += n * d
        return out.copy_(x)
    q, k, v, d_o = _inputs(T, nq, nkv, d, dtype)
    buf = A.AttnBuffers(T, nq, nkv, d, dtype, n_docs=2)
    qd, kd, vd, dod = (place(x) for x in (q, k, v, d_o))
    buf.o, buf.dq, buf.dk, buf.dv = (place(torch.full_like(x, float("nan"))) for x in (buf.o, buf.dq, buf.dk, buf.dv))
    dd = torch.tensor(docs, dtype=torch.int32, device="cuda")
    A.attn_forward(buf, qd, kd, vd, dd)
    A.attn_backward(buf, dod, qd, kd, vd, dd)
    got = [x.float().cpu() for x in (buf.o, buf.lse, buf.dq, buf.dk, buf.dv)]
    _compare(got, ref.attention(q, k, v, ref.masks(T, docs), 1 / math.sqrt(d), 0.0, None, d_o), dtype)
    # the rotation on the same rows
    qkv, pos, table, (gq, gk), dq, dk = _case(T, nq, nkv, d, d, dtype)
    r = A.RopeBuffers(T, nq, nkv, d, dtype, positions=50)
    wide = mem[:, used:used + qkv.shape[1]].copy_(qkv)
    used += qkv.shape[1]
    r.q, r.k = (place(torch.full_like(x, float("nan"))) for x in (r.q, r.k))
    r.dxq, r.dxk = (place(torch.full_like(x, float("nan"))) for x in (dq, dk))
    dqd, dkd = place(dq), place(dk)
    args = (wide, *_cuda(pos, table, gq, gk))
    A.rope_forward(r, *args)
    A.rope_backward(r, dqd, dkd, *args)
    x = qkv.view(T, -1, d)[:, :nq]
    wy, wdx, wdg = ref.rope(x, pos, table, d, False, gq, 1e-6, True, dq)
    assert rel_err(r.q.float().cpu(), wy) <= TOL[dtype] and rel_err(r.dxq.float().cpu(), wdx) <= TOL[dtype]
    assert rel_err(r.dgain_q.cpu(), wdg) <= 1e-5


# ---------------------------------------------------------------- graphs
@both
def test_captured_training_step(dtype):
    from paper_2603_06492_gb300 import attention as A
    T, nq, nkv, d = 700, 8, 2, 64
    qkv, pos, table, (gq, gk), _, _ = _case(T, nq, nkv, d, d, dtype)
    d_o = _inputs(T, nq, nkv, d, dtype)[3].cuda()
    args = _cuda(qkv, pos, table, gq, gk)
    docs = torch.tensor([0, 333, T], dtype=torch.int32, device="cuda")
    r = A.RopeBuffers(T, nq, nkv, d, dtype, positions=50)
    b = A.AttnBuffers(T, nq, nkv, d, dtype, n_docs=2, dv=r.dxv)

    def step():
        q, k = A.rope_forward(r, *args)
        v = args[0].view(T, -1, d)[:, nq + nkv:]
        A.attn_forward(b, q, k, v, docs)
        dq, dk, _ = A.attn_backward(b, d_o, q, k, v, docs)
        A.rope_backward(r, dq, dk, *args)
    outs = (b.o, b.lse, r.dqkv, r.dgain_q, r.dgain_k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        args[0].copy_(torch.randn(args[0].shape, generator=torch.Generator().manual_seed(7)).to(DT[dtype]))
        step()
        want = [x.clone() for x in outs]
        for x in outs:
            x.fill_(float("nan"))
        graph.replay()
        for x, w in zip(outs, want):
            assert torch.equal(x, w)


@both
def test_captured_generation_step(dtype):
    from paper_2603_06492_gb300 import attention as A
    n, nq, nkv, d, page, pages = 5, 8, 2, 64, 16, 64
    qkv, pos, table, (gq, gk), _, _ = _case(n, nq, nkv, d, d, dtype)
    args = _cuda(qkv, pos, table, gq, gk)
    cache = A.PagedCache(pages, page, nkv, d, dtype)
    cache.k.normal_(), cache.v.normal_()
    pages_of = torch.randperm(pages).int()[:60].view(n, 12).cuda()
    lens = torch.tensor([3, 100, 17, 192, 64], dtype=torch.int32, device="cuda")
    slots = torch.zeros(n, dtype=torch.int64, device="cuda")
    r = A.RopeBuffers(n, nq, nkv, d, dtype, positions=50, with_grads=False)
    p = A.PagedBuffers(n, 1, nq, nkv, d, dtype, max_len=1000)

    def step():
        q = A.kv_append(r, cache, args[0], args[1], slots, *args[2:])
        A.attn_paged(p, q, cache, pages_of, lens)
    graph = torch.cuda.CUDAGraph()
    at = lambda: pages_of[torch.arange(n, device="cuda"), ((lens - 1) // page).long()].long() * page + (lens - 1) % page  # noqa: E731
    slots.copy_(at())
    with torch.cuda.graph(graph):
        step()
    for grow in (0, -1):
        lens += grow
        slots.copy_(at())
        step()
        want = p.o.clone()
        p.o.fill_(float("nan"))
        graph.replay()
        assert torch.equal(p.o, want) and torch.isfinite(want).all()


# ---------------------------------------------------------------- a caller's error
@pytest.mark.parametrize("flags", [0, 2])
@pytest.mark.parametrize("docs", [[400, 0, 700], [0, 600, 100, 650], [690, 300, 200, 100, 0], [-50, 10 ** 9, 5, 300], [5, 5, 3, 3]])
@pytest.mark.parametrize("kw", [dict(), dict(causal=False), dict(window=40), dict(prefix=[200, -5, 10 ** 6, 7])])
def test_starts_that_do_not_ascend(docs, kw, flags):
    """Results are undefined, but calls end without an error of the device and leave the memory around
    their outputs as it is."""
    from paper_2603_06492_gb300 import attention as A, binding
    T, nq, nkv, d = 700, 4, 2, 64
    kw = dict(kw)
    prefix = kw.pop("prefix", None)
    x = [t.cuda() for t in _inputs(T, nq, nkv, d, "bf16")]
    buf = A.AttnBuffers(T, nq, nkv, d, "bf16", n_docs=len(docs) - 1, flags=flags, **kw)
    mem = torch.full((4, T + 256, nq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    buf.o, buf.dq, buf.dk, buf.dv = (mem[i, 128:-128, :n] for i, n in enumerate((nq, nq, nkv, nkv)))
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    rest = (ints(docs), None if prefix is None else ints((prefix * 2)[:len(docs) - 1]))
    A.attn_forward(buf, *x[:3], *rest)
    A.attn_backward(buf, x[3], *x[:3], *rest)
    binding.noble_get_device_status(None)
    binding.noble_debug_rows_again()
    assert (mem[:, :128] == 7).all() and (mem[:, -128:] == 7).all() and (mem[2:, :, nkv:] == 7).all()
