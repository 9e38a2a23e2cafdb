"""Attention over packed documents against its definition in 64 bits.

Error of an output: max |got - ref| / max |ref|.  Tolerances: fp32 operands 1e-5, sums of
a few hundred terms in fp32 (2^-24 each, and as much for the exponential of a score of
about 10); bf16 operands 1e-2: an output is rounded to 2^-9 of itself, after sums whose
probabilities (or score gradients) were each rounded to 2^-9, so that 2^-7 bounds it.
"""
import math

import pytest
import torch

from tests import attention_ref as ref
from tests.gpu_helpers import TOL, rel_err

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2603_06492_gb300 import binding
    from paper_2603_06492_gb300.build import build
    build()
    binding.load()


@pytest.fixture(autouse=True)
def no_device_error(request):
    """No error, and no row computed again but in the tests whose inputs are not finite."""
    from paper_2603_06492_gb300 import binding
    binding.noble_debug_rows_again()
    yield
    binding.noble_get_device_status(None)
    again = binding.noble_debug_rows_again()
    assert again == 0 or request.node.name.startswith("test_values"), again


DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _inputs(T, nq, nkv, d, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    rn = lambda n: torch.randn((T, n, d), generator=g).to(DT[dtype])  # noqa: E731
    return rn(nq), rn(nkv), rn(nkv), rn(nq)


def _layout(x, how):
    """The same values in device memory of another layout."""
    T, n, d = x.shape
    x = x.cuda()
    if how == "packed":  # part of wider rows
        out = torch.full((T, n + 3, d), float("nan"), dtype=x.dtype, device="cuda")[:, 1:n + 1]
    elif how == "heads":  # [heads][tokens][features]
        out = torch.empty((n, T, d), dtype=x.dtype, device="cuda").transpose(0, 1)
    elif how == "wide":  # features are part of a wider last dimension
        out = torch.full((T, n, d + 16), float("nan"), dtype=x.dtype, device="cuda")[:, :, 8:8 + d]
    else:
        return x.contiguous()
    return out.copy_(x)


def _run(q, k, v, d_o, docs, dtype, causal=True, prefix=None, window=0, softcap=0.0, slope=None, scale=None, flags=0,
         layout="", stream=None):
    from paper_2603_06492_gb300 import attention as A
    T, nq, d = q.shape
    buf = A.AttnBuffers(T, nq, k.shape[1], d, dtype, n_docs=len(docs) - 1, causal=causal, window=window, scale=scale,
                        softcap=softcap, flags=flags)
    if layout:
        buf.o, buf.dq = _layout(buf.o, layout), _layout(buf.dq, layout)
        buf.dk, buf.dv = _layout(buf.dk, layout), _layout(buf.dv, layout)
    for x in (buf.o, buf.lse, buf.dq, buf.dk, buf.dv):
        x.fill_(float("nan"))
    dev = [_layout(x, layout) for x in (q, k, v, d_o)]
    ints = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    rest = (ints(docs), ints(prefix), slope.cuda() if slope is not None else None)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    A.attn_forward(buf, *dev[:3], *rest, stream=stream)
    A.attn_backward(buf, dev[3], *dev[:3], *rest, stream=stream)
    torch.cuda.synchronize()
    return [x.float().cpu() for x in (buf.o, buf.lse, buf.dq, buf.dk, buf.dv)]


NAMES = ("o", "lse", "dq", "dk", "dv")


def _compare(got, want, dtype, names=NAMES):
    errs = {}
    for n, a, b in zip(names, got, want):
        if n == "lse":
            assert torch.equal(torch.isinf(a), torch.isinf(b)), "rows that see nothing"
            a, b = torch.where(torch.isinf(a), 0.0, a), torch.where(torch.isinf(b), 0.0, b)
        assert torch.isfinite(a).all(), n
        # gradients of rows that see one key only are zero, and compared as such
        scale = float(b.abs().max()) if b.numel() else 0.0
        errs[n] = rel_err(a, b) if scale > 1e-6 else float((a - b).abs().max())
    # lse of bf16 operands is a 32-bit result like the others' but for the scores' rounding of sums
    bad = {n: e for n, e in errs.items() if not e <= (1e-5 if n == "lse" else TOL[dtype])}
    assert not bad, (bad, errs)


def _check(T, nq, nkv, d, docs, dtype, causal=True, prefix=None, window=0, softcap=0.0, alibi=False, scale=None, flags=0,
           layout="", seed=0):
    q, k, v, d_o = _inputs(T, nq, nkv, d, dtype, seed)
    slope = torch.tensor([2.0 ** (-4.0 * (h + 1) / nq) for h in range(nq)]) if alibi else None
    got = _run(q, k, v, d_o, docs, dtype, causal, prefix, window, softcap, slope, scale, flags, layout)
    seen = ref.masks(T, docs, causal, prefix, window)
    want = ref.attention(q, k, v, seen, 1.0 / math.sqrt(d) if scale is None else scale, softcap, slope, d_o)
    _compare(got, want, dtype)


PATHS = [("bf16", 0), ("bf16", 2), ("fp32", 0)]  # tensor cores, bf16 and fp32 on the CUDA cores
path = pytest.mark.parametrize("dtype,flags", PATHS)


@path
@pytest.mark.parametrize("d", [8, 40, 64, 72, 96, 128])
@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 127, 128, 129, 200, 257, 300])
def test_sizes(T, d, dtype, flags):
    _check(T, 2, 1, d, [0, T], dtype, flags=flags)


@path
@pytest.mark.parametrize("docs", [
    [0, 300], [0, 1, 2, 3, 300], [0, 128, 256, 300], [0, 64, 64, 64, 193, 300], [0, 0, 300, 300],
    [5, 130, 260], [0, 299], [130, 200], [300, 300], [0, 0], [0, 100, 101, 102, 229, 290]])
@pytest.mark.parametrize("causal", [True, False])
def test_documents(docs, causal, dtype, flags):
    # tokens before the first and after the last document see nothing
    _check(300, 2, 2, 64, docs, dtype, causal=causal, flags=flags)


@path
@pytest.mark.parametrize("kw", [
    dict(window=1), dict(window=7), dict(window=128), dict(window=1000), dict(window=20, causal=False),
    dict(prefix=[0, 40, 1000]), dict(prefix=[37, 1, 64], window=30), dict(softcap=2.0), dict(softcap=30.0, alibi=True),
    dict(alibi=True), dict(alibi=True, causal=False), dict(scale=0.0), dict(scale=-0.3), dict(scale=2.0, softcap=5.0)])
def test_masks_and_scores(kw, dtype, flags):
    _check(333, 4, 2, 64, [0, 111, 190, 330], dtype, flags=flags, **kw)


@path
@pytest.mark.parametrize("nq,nkv", [(1, 1), (7, 1), (6, 3), (16, 2)])
def test_shared_heads(nq, nkv, dtype, flags):
    # the gradients of a key head add up over the query heads that share it
    _check(150, nq, nkv, 128, [0, 70, 150], dtype, flags=flags)


@path
@pytest.mark.parametrize("layout", ["packed", "heads", "wide"])
def test_layouts(layout, dtype, flags):
    _check(140, 4, 2, 72, [0, 90, 140], dtype, layout=layout, flags=flags)


@path
def test_more_blocks_than_sms(dtype, flags):
    # every block of a chip's worth takes several pieces of work
    _check(1030, 12, 4, 64, [0, 500, 510, 1029], dtype, flags=flags)


@path
@pytest.mark.parametrize("d", [64, 128])
def test_long_rows(d, dtype, flags):
    _check(900, 2, 1, d, [0, 900], dtype, causal=False, flags=flags)


@path
def test_scores_that_grow(dtype, flags):
    # maxima that rise from block to block: every earlier sum has to be scaled down
    T, d = 700, 64
    q, k, v, d_o = _inputs(T, 1, 1, d, dtype)
    ramp = (torch.arange(T) / 20.0)[:, None, None]
    q[..., 0], k[..., :1] = 8.0, ramp.to(k.dtype)
    seen = ref.masks(T, [0, T], False)
    got = _run(q, k, v, d_o, [0, T], dtype, causal=False, flags=flags)
    want = ref.attention(q, k, v, seen, 1 / math.sqrt(d), 0.0, None, d_o)
    _compare(got[:2] + got[3:], want[:2] + want[3:], dtype, NAMES[:2] + NAMES[3:])
    # dq = sum of ds k, whose sum of ds is 0: what the keys have in common, up to 35, cancels
    # exactly in it and not in its rounding, which is relative to the sum of |ds k|
    z = (q.double()[:, 0] @ k.double()[:, 0].T) / math.sqrt(d)
    p, dp = torch.softmax(z, 1), d_o.double()[:, 0] @ v.double()[:, 0].T
    ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(d)
    size = float((ds.abs() @ k.double()[:, 0].abs()).max())
    assert float((got[2].double() - want[2]).abs().max()) <= TOL[dtype] * size


@path
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_values_that_nothing_sees(bad, dtype, flags):
    """Tokens of no document, and other documents' tokens, may hold anything."""
    T, docs, d = 300, [7, 60, 140, 290], 64
    q, k, v, d_o = _inputs(T, 2, 1, d, dtype)
    clean = [x.clone() for x in (q, k, v, d_o)]
    out = torch.ones(T, dtype=torch.bool)
    out[docs[0]:docs[-1]] = False
    for x, c in zip((q, k, v, d_o), clean):
        x[out] = bad
        c[out] = 0.0
    want = ref.attention(*clean[:3], ref.masks(T, docs), 1 / math.sqrt(d), 0.0, None, clean[3])
    _compare(_run(q, k, v, d_o, docs, dtype, flags=flags), want, dtype)
    # a whole document of such values: the others' results stay
    for x in (q, k, v, d_o):
        x[60:140] = bad
    got = _run(q, k, v, d_o, docs, dtype, flags=flags)
    keep = torch.ones(T, dtype=torch.bool)
    keep[60:140] = False
    for n, a, b in zip(NAMES, got, want):
        a, b = (a[:, keep], b[:, keep]) if n == "lse" else (a[keep], b[keep])
        if n == "lse":
            a, b = a[:, 7:-10], b[:, 7:-10]
        assert torch.isfinite(a).all(), n
        assert rel_err(a, b) <= TOL[dtype], n


@path
def test_values_in_the_future(dtype, flags):
    """A key that a query does not see yet does not change its output."""
    T, d, at = 200, 64, 150
    q, k, v, d_o = _inputs(T, 2, 2, d, dtype)
    want = ref.attention(q, k, v, ref.masks(T, [0, T]), 1 / math.sqrt(d))
    k[at:], v[at:] = float("inf"), float("nan")
    got = _run(q, k, v, d_o, [0, T], dtype, flags=flags)
    assert rel_err(got[0][:at], want[0][:at]) <= TOL[dtype] and rel_err(got[1][:, :at], want[1][:, :at]) <= 1e-5
    assert torch.isnan(got[0][at:]).any()


@path
def test_repeated_calls_agree(dtype, flags):
    T = 1500
    q, k, v, d_o = _inputs(T, 8, 2, 128, dtype)
    docs = [0, 1000, 1500]
    first = _run(q, k, v, d_o, docs, dtype, flags=flags)
    for a, b in zip(first, _run(q, k, v, d_o, docs, dtype, flags=flags, stream=torch.cuda.Stream())):
        assert torch.equal(a, b)


def test_no_tokens():
    from paper_2603_06492_gb300 import attention as A
    buf = A.AttnBuffers(0, 2, 1, 64, "bf16", n_docs=0)
    e = lambda n: torch.empty((0, n, 64), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    docs = torch.zeros(1, dtype=torch.int32, device="cuda")
    A.attn_forward(buf, e(2), e(1), e(1), docs)
    A.attn_backward(buf, e(2), e(2), e(1), e(1), docs)


@pytest.mark.parametrize("dtype,flags,softcap", [("fp32", 0, 0.0), ("fp32", 0, 3.0), ("bf16", 0, 0.0), ("bf16", 0, 3.0)])
def test_gradients_against_differences(dtype, flags, softcap):
    """<gradient, u> against the central difference of sum(o * do) along u.

    The differences are those of the 64-bit definition on the same inputs: h = 1e-4 leaves
    h^2 = 1e-8 and 1e-16 / h; what remains is the gradients' own error, which adds up in
    quadrature over the outputs: the tolerance of one output is ample."""
    T, nq, nkv, d, docs = 70, 2, 1, 64, [0, 30, 70]
    q, k, v, d_o = _inputs(T, nq, nkv, d, dtype)
    got = _run(q, k, v, d_o, docs, dtype, softcap=softcap, flags=flags)
    seen = ref.masks(T, docs)
    g = torch.Generator().manual_seed(5)

    def value(*x):
        return float((ref.attention(*x, seen, 1 / math.sqrt(d), softcap)[0] * d_o.double()).sum())
    for n in range(3):
        x = [t.double() for t in (q, k, v)]
        u = torch.randn(x[n].shape, generator=g, dtype=torch.float64)
        h = 1e-4
        up, down = list(x), list(x)
        up[n], down[n] = x[n] + h * u, x[n] - h * u
        diff = (value(*up) - value(*down)) / (2 * h)
        grad = got[2 + n].double()
        assert abs(float((grad * u).sum()) - diff) <= TOL[dtype] * float(grad.norm() * u.norm()) / math.sqrt(u.numel()) * 10


@path
@pytest.mark.parametrize("d", [64, 128])
def test_several_pieces_per_block(d, dtype, flags):
    """More work than a chip takes at once, of row blocks that see different key tiles: the
    same documents side by side in many heads, each head as if it were alone."""
    T, docs, n = 2000, [0, 260, 300, 301, 930, 1500, 1995], 40
    q, k, v, d_o = _inputs(T, 2, 1, d, dtype)
    wide = lambda x, m: x.repeat(1, m // x.shape[1], 1)  # noqa: E731
    seen = ref.masks(T, docs, True, [100, 0, 0, 300, 7, 1], 150)
    want = ref.attention(q, k, v, seen, 1 / math.sqrt(d), 0.0, None, d_o)
    got = _run(wide(q, n), wide(k, n // 2), wide(v, n // 2), wide(d_o, n), docs, dtype,
               prefix=[100, 0, 0, 300, 7, 1], window=150, flags=flags)
    want = [wide(want[0], n), want[1].repeat(n // 2, 1), wide(want[2], n), wide(want[3], n // 2), wide(want[4], n // 2)]
    _compare(got, want, dtype)


@pytest.mark.parametrize("kw", [dict(), dict(softcap=5.0), dict(softcap=30.0), dict(softcap=5.0, alibi=True), dict(alibi=True),
                                dict(window=700), dict(causal=False)])
@pytest.mark.parametrize("nq,nkv,d", [(16, 4, 128), (8, 8, 64)])
def test_no_row_again_at_length(nq, nkv, d, kw):
    """Long sequences keep the warps of a block running ahead of each other for many steps;
    a step that is used before all of them are through shows as rows that are not finite
    (no_device_error counts them) or as results that differ from call to call."""
    from paper_2603_06492_gb300 import attention as A
    T = 4096
    g = torch.Generator(device="cuda").manual_seed(1)
    rn = lambda n: torch.randn((T, n, d), generator=g, device="cuda").bfloat16()  # noqa: E731
    q, k, v, d_o = rn(nq), rn(nkv), rn(nkv), rn(nq)
    docs = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    kw = dict(kw)
    slope = torch.tensor([2.0 ** (-8.0 * (h + 1) / nq) for h in range(nq)], device="cuda") if kw.pop("alibi", False) else None
    buf = A.AttnBuffers(T, nq, nkv, d, "bf16", **kw)
    first = None
    for _ in range(4):
        A.attn_forward(buf, q, k, v, docs, None, slope)
        A.attn_backward(buf, d_o, q, k, v, docs, None, slope)
        now = [x.clone() for x in (buf.o, buf.lse, buf.dq, buf.dk, buf.dv)]
        first = first or now
        for n, a, b in zip(NAMES, first, now):
            assert torch.equal(a, b), n


@path
@pytest.mark.parametrize("nq,nkv,d", [(12, 2, 128), (5, 1, 64), (16, 4, 40), (14, 2, 96)])
@pytest.mark.parametrize("kw", [dict(), dict(causal=False), dict(softcap=4.0, alibi=True), dict(window=70)])
def test_few_key_heads(nq, nkv, d, kw, dtype, flags):
    # query heads of a key head in several parts, whose gradients are added up
    _check(413, nq, nkv, d, [0, 90, 91, 380], dtype, flags=flags, seed=4, **kw)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_that_nothing_sees_of_few_key_heads(bad):
    q, k, v, d_o = _inputs(300, 8, 1, 64, "bf16", 5)
    docs = [0, 130, 280]
    clean = [x.clone() for x in (q, k, v, d_o)]
    for x, c in zip((q, k, v, d_o), clean):
        x[280:], c[280:] = bad, 0.0
    want = ref.attention(*clean[:3], ref.masks(300, docs), 1 / math.sqrt(64), 0.0, None, clean[3])
    _compare(_run(q, k, v, d_o, docs, "bf16"), want, "bf16")
