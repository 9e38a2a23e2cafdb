"""Infinities and NaN where a query does not see them, at lengths and in numbers at which rows that
are computed again take longer than a block's warps wait for each other, and where every
block has some.  Errors and tolerances as in test_attention_gpu.py; two results of the library are
held to twice that, since each may be off by it."""
import math

import pytest
import torch

from tests import attention_ref as ref
from tests.gpu_helpers import TOL, rel_err
from tests.test_attention_gpu import NAMES, _inputs, _run

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
def no_device_error():
    from paper_2603_06492_gb300 import binding
    yield
    binding.noble_get_device_status(None)


def _part(x, name, keep):
    return x[:, keep] if name == "lse" else x[keep]


def test_rows_again_of_a_long_document():
    """Keys 64 to 127 share their tile of queries with another document's, which hold NaN: 64 rows
    over 8 heads and 32700 queries each, about a second and a half, in a block that has further work."""
    T, d, docs = 32768, 128, [0, 64, 32768]
    q, k, v, d_o = _inputs(T, 16, 2, d, "bf16")
    q[:64], k[:64], v[:64], d_o[:64] = 0, 0, 0, 0
    want = _run(q, k, v, d_o, docs, "bf16")
    q[:64], k[:64], v[:64], d_o[:64] = (float("nan"),) * 4
    got = _run(q, k, v, d_o, docs, "bf16")
    keep = torch.arange(T) >= 64
    for n, a, b in zip(NAMES, got, want):
        a, b = _part(a, n, keep), _part(b, n, keep)
        assert torch.isfinite(a).all(), n
        assert rel_err(a, b) <= 2 * TOL["bf16"], n
        # all but the two blocks around it (256 queries, 128 keys) are the tiles' results as before
        assert torch.equal(a[..., 256:] if n == "lse" else a[256:], b[..., 256:] if n == "lse" else b[256:]), n


@pytest.mark.parametrize("nq,nkv,d,bad,kw", [
    (16, 16, 64, float("nan"), dict()), (16, 16, 128, float("inf"), dict()), (16, 16, 64, -float("inf"), dict(causal=False)),
    (16, 2, 128, float("nan"), dict(softcap=5.0)), (16, 16, 128, float("nan"), dict(softcap=5.0)), (16, 4, 40, float("inf"), dict(window=33))])
def test_rows_again_in_every_block(nq, nkv, d, bad, kw):
    """Every second document of 90 tokens holds such values, with more blocks than SMs."""
    from paper_2603_06492_gb300 import binding
    T, step = 2770, 90
    docs = list(range(0, T, step)) + [T]
    q, k, v, d_o = _inputs(T, nq, nkv, d, "bf16")
    spoilt = torch.arange(T) // step % 2 == 1
    want = ref.attention(q, k, v, ref.masks(T, docs, kw.get("causal", True), None, kw.get("window", 0)), 1 / math.sqrt(d),
                         kw.get("softcap", 0.0), None, d_o)
    for x in (q, k, v, d_o):
        x[spoilt] = bad
    binding.noble_debug_rows_again()
    got = _run(q, k, v, d_o, docs, "bf16", **kw)
    assert binding.noble_debug_rows_again() > 0
    for n, a, b in zip(NAMES, got, want):
        a, b = _part(a, n, ~spoilt), _part(b, n, ~spoilt)
        assert torch.isfinite(a).all(), n
        assert rel_err(a, b) <= (1e-5 if n == "lse" else TOL["bf16"]), n


def test_nothing_finite():
    # a training step that has diverged: NaN everywhere, and an end
    T, d = 16384, 128
    q, k, v, d_o = (x.fill_(float("nan")) for x in _inputs(T, 8, 8, d, "bf16"))
    for n, x in zip(NAMES, _run(q, k, v, d_o, [0, T], "bf16")):
        assert torch.isnan(x).all(), n


@pytest.mark.parametrize("docs,nq,nkv,d,kw", [
    ([0, 333, 1290], 4, 4, 64, dict()), ([0, 333, 1290], 16, 2, 128, dict(causal=False)), ([0, 333, 1290], 3, 1, 40, dict(softcap=5.0)),
    ([0, 333, 1290], 16, 2, 128, dict(softcap=5.0)), ([0, 333, 1290], 16, 2, 128, dict(window=150)),
    ([70, 129, 1281], 4, 4, 64, dict(causal=False)), ([70, 129, 1281], 16, 2, 128, dict()), ([70, 129, 1281], 3, 1, 40, dict(window=150)),
    ([70, 129, 1281], 4, 4, 128, dict(prefix=[30, 500])), ([70, 129, 1281], 16, 2, 64, dict(softcap=5.0, causal=False))])
def test_padding_counts_for_nothing(docs, nq, nkv, d, kw):
    """What is behind the last document leaves every bit as it is and no row to compute again."""
    from paper_2603_06492_gb300 import binding
    T = 1400
    q, k, v, d_o = _inputs(T, nq, nkv, d, "bf16")
    first = None
    for bad in (0.0, float("nan"), float("inf"), 3e38):
        for x in (q, k, v, d_o):
            x[docs[-1]:] = bad
        binding.noble_debug_rows_again()
        now = _run(q, k, v, d_o, docs, "bf16", **kw)
        assert binding.noble_debug_rows_again() == 0
        first = first or now
        for n, a, b in zip(NAMES, first, now):
            assert torch.equal(a, b), (n, bad)
    seen = ref.masks(T, docs, kw.get("causal", True), kw.get("prefix"), kw.get("window", 0))
    want = ref.attention(q, k, v, seen, 1 / math.sqrt(d), kw.get("softcap", 0.0), None, d_o)
    for n, a, b in zip(NAMES, first, want):
        assert torch.equal(torch.isinf(a), torch.isinf(b)), n
        assert rel_err(torch.where(torch.isinf(a), 0.0, a), torch.where(torch.isinf(b), 0.0, b)) <= (
            1e-5 if n == "lse" else TOL["bf16"]), n
