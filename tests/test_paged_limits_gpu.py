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
