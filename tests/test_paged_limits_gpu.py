"""Attention over the cache at the ends of its ranges: lengths, bounds and windows near 2^31,
and windows behind a length that is cut.  Errors and tolerances as in test_paged_gpu.py."""
import math

import pytest
import torch

from tests import attention_ref as ref
from tests.gpu_helpers import TOL, rel_err
from tests.test_paged_gpu import DT, _case, _compare, _run, both

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2603_06492_gb300 import binding
    from paper_2603_06492_gb300.build import build
    build()
    binding.load()


@both
@pytest.mark.parametrize("max_len,d", [(64, 64), (1024, 64), (1024, 128)])
def test_window_behind_a_cut_length(max_len, d, dtype):
    # the length is cut to max_len, a multiple of a chunk, and the window lies behind that
    from paper_2603_06492_gb300 import binding
    case = _case([2000, 50], 1, 4, 2, d, 64, dtype)
    q, k, v, table, n = case
    got = _run(case, 1, dtype, max_len=max_len, window=128)
    with pytest.raises(binding.NobleError):
        binding.noble_get_device_status(None)
    assert not got[0][0].any() and torch.equal(got[1][0], torch.full_like(got[1][0], -math.inf))
    want = ref.paged(q, k, v, table, n, 1, 1 / math.sqrt(d), 128)
    _compare([x[1:] for x in got], [x[1:] for x in want], dtype)


@pytest.mark.parametrize("dtype,n_seq,d", [("bf16", 320, 128), ("bf16", 640, 64), ("fp32", 160, 128)])
def test_no_bound_on_the_length(dtype, n_seq, d):
    """max_len = 2^31 - 1 where the batch alone fills the chip, so that one chunk takes it all."""
    from paper_2603_06492_gb300 import binding
    case = _case([1 + i % 40 for i in range(n_seq)], 1, 8, 8, d, 16, dtype)
    q, k, v, table, n = case
    got = _run(case, 1, dtype, max_len=2 ** 31 - 1)
    binding.noble_get_device_status(None)
    _compare(got, ref.paged(q, k, v, table, n, 1, 1 / math.sqrt(d)), dtype)


def _one_page(n, dtype):
    """A sequence of n tokens whose first page, of 2^20, is the cache's first and whose others all
    are its second: 8 features of one head, keys and values 0."""
    page = 2 ** 20
    k, v = (torch.zeros((2, page, 1, 8), dtype=DT[dtype], device="cuda") for _ in range(2))
    table = torch.ones((1, -(-n // page)), dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    return k, v, table


def _run_long(n, dtype, k, v, table, max_len, window=0):
    from paper_2603_06492_gb300 import attention as A, binding
    cache = A.PagedCache(2, k.shape[1], 1, 8, dtype, k=k, v=v)
    buf = A.PagedBuffers(1, 1, 1, 1, 8, dtype, max_len, window=window, scale=1.0, with_lse=True)
    q = torch.zeros((1, 1, 8), dtype=DT[dtype], device="cuda")
    q[..., 0] = 1.0
    A.attn_paged(buf, q, cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    binding.noble_get_device_status(None)
    return buf.o.float().cpu().flatten(), float(buf.lse)


@pytest.mark.parametrize("dtype", ["bf16"])
def test_longest_sequence(dtype):
    """2^31 - 65536 tokens; the last of them outweighs the others by e^20 to 2^31."""
    n = 2 ** 31 - 65536
    k, v, table = _one_page(n, dtype)
    last = n - 1
    table[0, last // 2 ** 20] = 0
    k[0, last % 2 ** 20, 0, 0], v[0, last % 2 ** 20] = 40.0, 1.0
    table[0, 0] = 1
    o, lse = _run_long(n, dtype, k, v, table, 2 ** 31 - 1)
    assert float((o - 1).abs().max()) <= TOL[dtype] and abs(lse - 40.0) <= 1e-5 * 40


def test_lengths_beyond_the_longest_are_reported():
    from paper_2603_06492_gb300 import binding
    n = 2 ** 31 - 65536
    k, v, table = _one_page(2 ** 31 - 1, "bf16")
    with pytest.raises(binding.NobleError):
        _run_long(n + 1, "bf16", k, v, table, 2 ** 31 - 1)


def test_window_beyond_30_bits():
    """A window of 2^30 + 500 of 2^30 + 1000 tokens: 500 to 600 are seen and outweigh all others
    (100 e^30 to 2^30 e^0), those before 500 would outweigh them."""
    n, window = 2 ** 30 + 1000, 2 ** 30 + 500
    k, v, table = _one_page(n, "bf16")
    k[0, 500:600, 0, 0], v[0, 500:600] = 30.0, 1.0
    k[0, :500, 0, 0], v[0, :500] = 60.0, -1.0
    o, lse = _run_long(n, "bf16", k, v, table, n, window)
    assert float((o - 1).abs().max()) <= TOL["bf16"] and abs(lse - 30.0 - math.log(100)) <= 1e-5 * 35
