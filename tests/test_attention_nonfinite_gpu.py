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
