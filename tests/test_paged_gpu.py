"""Attention of new tokens over a paged cache against its definition in 64 bits.  Errors and
tolerances as in test_attention_gpu.py."""
import math

import pytest
import torch

from tests import attention_ref as ref
from tests.gpu_helpers import TOL, rel_err

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
both = pytest.mark.parametrize("dtype", ["bf16", "fp32"])


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2603_06492_gb300 import binding
    from paper_2603_06492_gb300.build import build
    build()
    binding.load()


@pytest.fixture(autouse=True)
def no_row_again(request):
    """No row is computed again but in the test whose inputs are not finite."""
    from paper_2603_06492_gb300 import binding
    binding.noble_debug_rows_again()
    yield
    again = binding.noble_debug_rows_again()
    assert again == 0 or request.node.name.startswith(("test_values", "test_callers")), again


def _case(lens, q_len, nq, nkv, d, page, dtype, seed=0, spare=3, unwritten=float("nan")):
    """Sequences on shuffled pages; what no sequence has written holds NaN."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + spare
    k, v = (torch.randn((pages, page, nkv, d), generator=g).to(DT[dtype]) for _ in range(2))
    written = torch.zeros((pages, page), dtype=torch.bool)
    order = torch.randperm(pages, generator=g).int()
    table = torch.full((len(lens), max(need + [1])), 2 ** 30, dtype=torch.int32)  # entries past a sequence's end
    at = 0
    for i, n in enumerate(lens):
        table[i, :need[i]] = order[at:at + need[i]]
        for j in range(n):
            written[table[i, j // page], j % page] = True
        at += need[i]
    k[~written], v[~written] = unwritten, unwritten
    q = torch.randn((len(lens) * q_len, nq, d), generator=g).to(DT[dtype])
    return q, k, v, table, torch.tensor(lens, dtype=torch.int32)


def _run(case, q_len, dtype, max_len=None, window=0, softcap=0.0, slope=None, cache=None, stream=None):
    from paper_2603_06492_gb300 import attention as A
    q, k, v, table, lens = case
    pages, page, nkv, d = k.shape
    if cache is None:
        cache = A.PagedCache(pages, page, nkv, d, dtype, k=k.cuda(), v=v.cuda())
    buf = A.PagedBuffers(len(lens), q_len, q.shape[1], nkv, d, dtype, int(lens.max()) if max_len is None else max_len,
                         window=window, softcap=softcap, with_lse=True)
    buf.o.fill_(float("nan")), buf.lse.fill_(float("nan"))
    args = q.cuda(), cache, table.cuda(), lens.cuda(), slope.cuda() if slope is not None else None
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    A.attn_paged(buf, *args, stream=stream)
    torch.cuda.synchronize()
    return buf.o.float().cpu(), buf.lse.cpu()


def _compare(got, want, dtype):
    assert torch.equal(torch.isinf(got[1]), torch.isinf(want[1]))
    clean = [torch.where(torch.isinf(x), 0.0, x) for x in (got[1], want[1])]
    assert torch.isfinite(got[0]).all()
    for a, b, tol in ((got[0], want[0], TOL[dtype]), (*clean, 1e-5)):
        assert (rel_err(a, b) if float(b.abs().max()) > 0 else float(a.abs().max())) <= tol


def _check(lens, q_len, nq, nkv, d, page, dtype, window=0, softcap=0.0, alibi=False, **kw):
    from paper_2603_06492_gb300 import binding
    case = _case(lens, q_len, nq, nkv, d, page, dtype)
    slope = torch.tensor([2.0 ** (-4.0 * (h + 1) / nq) for h in range(nq)]) if alibi else None
    got = _run(case, q_len, dtype, window=window, softcap=softcap, slope=slope, **kw)
    binding.noble_get_device_status(None)
    q, k, v, table, n = case
    _compare(got, ref.paged(q, k, v, table, n, q_len, 1 / math.sqrt(d), window, softcap, slope), dtype)


@both
@pytest.mark.parametrize("d", [8, 40, 64, 72, 96, 128])
@pytest.mark.parametrize("page", [1, 16, 48, 64, 100])
def test_sizes(page, d, dtype):
    _check([1, 15, 16, 17, 63, 64, 65, 200, 0], 1, 4, 2, d, page, dtype)


@both
@pytest.mark.parametrize("q_len,nq,nkv", [(1, 1, 1), (1, 7, 1), (2, 16, 2), (5, 6, 3), (8, 8, 1), (64, 2, 1), (3, 32, 1)])
def test_rows(q_len, nq, nkv, dtype):
    # sequences shorter than their new tokens: the first of those see nothing
    _check([q_len, 300, max(q_len - 1, 0), 0, 1, 129], q_len, nq, nkv, 64, 16, dtype)


@both
@pytest.mark.parametrize("kw", [dict(window=1), dict(window=50), dict(window=5000), dict(softcap=3.0), dict(alibi=True),
                                dict(softcap=20.0, alibi=True, window=300)])
@pytest.mark.parametrize("q_len", [1, 4])
def test_masks_and_scores(q_len, kw, dtype):
    _check([5, 700, 333, 1500], q_len, 8, 2, 128, 64, dtype, **kw)


@both
@pytest.mark.parametrize("lens,max_len", [([3000], None), ([3000, 1, 2999], None), ([70, 700, 7], 100000), ([2500] * 3, 2500)])
def test_split_sequences(lens, max_len, dtype):
    # one sequence over many blocks, and long bounds for short sequences
    _check(lens, 2, 8, 2, 64, 32, dtype, max_len=max_len)


@both
def test_many_sequences(dtype):
    _check([(37 * i) % 250 for i in range(200)], 1, 2, 1, 64, 16, dtype)


@both
def test_values_that_a_row_does_not_see(dtype):
    """Of one sequence's new tokens, the later ones' values do not change the earlier ones'
    results, whatever they are."""
    case = _case([100, 64], 4, 4, 2, 64, 16, dtype)
    q, k, v, table, n = case
    want = ref.paged(q, k, v, table, n, 4, 1 / math.sqrt(64))
    for s, length in enumerate((100, 64)):
        j = length - 1
        k[table[s, j // 16], j % 16], v[table[s, j // 16], j % 16] = float("inf"), float("nan")
    got = _run(case, 4, dtype)
    keep = torch.tensor([r % 4 != 3 for r in range(8)])
    _compare([x[keep] for x in got], [x[keep] for x in want], dtype)
    assert torch.isnan(got[0][~keep]).any()


@both
def test_layouts_streams_and_repeats(dtype):
    from paper_2603_06492_gb300 import attention as A
    case = _case([900, 40], 2, 8, 2, 64, 16, dtype)
    q, k, v, table, n = case
    first = _run(case, 2, dtype)
    pages, page, nkv, d = k.shape
    mem = torch.zeros((pages, nkv, 2, page, d), dtype=DT[dtype], device="cuda")
    kk, vv = mem[:, :, 0].transpose(1, 2), mem[:, :, 1].transpose(1, 2)
    kk.copy_(k), vv.copy_(v)
    cache = A.PagedCache(pages, page, nkv, d, dtype, k=kk, v=vv)
    for a, b in zip(first, _run(case, 2, dtype, cache=cache, stream=torch.cuda.Stream())):
        assert torch.equal(a, b)


@both
def test_callers_errors_are_reported(dtype):
    from paper_2603_06492_gb300 import binding
    # a page number outside the cache: its keys are left out
    case = _case([100, 50], 1, 2, 1, 64, 16, dtype)
    q, k, v, table, n = case
    want = ref.paged(q, k, v, table, n, 1, 1 / 8)
    for bad in (-1, k.shape[0], 2 ** 31 - 1):
        t = table.clone()
        t[0, 2] = bad
        got = _run((q, k, v, t, n), 1, dtype)
        with pytest.raises(binding.NobleError):
            binding.noble_get_device_status(None)
        assert torch.isfinite(got[0]).all() and rel_err(got[0][1], want[0][1]) <= TOL[dtype]
    # lengths beyond the table or the stated bound
    for max_len in (None, 60):
        n2 = n.clone()
        n2[0] = 10 ** 6 if max_len is None else 100
        got = _run((q, k, v, table, n2), 1, dtype, max_len=10 ** 6 if max_len is None else 60)
        with pytest.raises(binding.NobleError):
            binding.noble_get_device_status(None)
        assert rel_err(got[0][1], want[0][1]) <= TOL[dtype]


def test_cache_beyond_32_bits():
    """Element offsets beyond 2^32: a sequence on the last pages of a 9 GB cache."""
    from paper_2603_06492_gb300 import attention as A
    nkv, d, page = 8, 128, 64
    pages = (2 ** 32 + 2 ** 22) // (nkv * d * page)
    small = _case([150, 90], 1, 16, nkv, d, page, "bf16")
    q, k, v, table, n = small
    want = ref.paged(q, k, v, table, n, 1, 1 / math.sqrt(d))
    cache = A.PagedCache(pages, page, nkv, d, "bf16")
    off = pages - k.shape[0]
    cache.k[off:].copy_(k), cache.v[off:].copy_(v)
    far = torch.where(table < k.shape[0], table + off, table)
    _compare(_run((q, k, v, far, n), 1, "bf16", cache=cache), want, "bf16")
