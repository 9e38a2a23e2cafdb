"""Norm and embedding at the largest numbers of rows, tokens and table rows that their descriptors allow, on
buffers of up to 34 GB.  Sums are of whole numbers, so that they are exact."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2603_06492_gb300 import binding
    from paper_2603_06492_gb300.build import build
    build()
    binding.load()
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T", [60, 3000])
def test_largest_table(T):
    from paper_2603_06492_gb300 import layers as L
    V, d = 2 ** 28, 8
    g = torch.Generator(device="cuda").manual_seed(T)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda").int()
    ids[:3] = torch.tensor([0, V - 1, 2 ** 27], dtype=torch.int32)
    ids[T // 2:T // 2 + 20] = V - 1  # a longer list
    table = torch.zeros((V, d), dtype=torch.bfloat16, device="cuda")
    rows, place = torch.unique(ids.long(), return_inverse=True)
    values = torch.randn((len(rows), d), generator=g, device="cuda").bfloat16()
    table[rows] = values
    dy = torch.randint(-8, 9, (T, d), generator=g, device="cuda").bfloat16()
    b = L.EmbedBuffers(T, V, d, "bf16")
    b.dtable.fill_(7.0)
    assert torch.equal(L.embed_forward(b, ids, table), values[place])
    got = L.embed_backward(b, ids, dy)
    assert torch.equal(got[rows], torch.zeros((len(rows), d), device="cuda").index_add_(0, place, dy.float()))
    got[rows] = 0.0
    assert not any(bool(part.any()) for part in got.split(2 ** 26))


@pytest.mark.parametrize("spread", [1, 1000])
def test_most_tokens(spread):
    # 64 windows of tokens, by one block each list
    from paper_2603_06492_gb300 import layers as L
    T, V, d = 2 ** 24, 1001, 8
    g = torch.Generator(device="cuda").manual_seed(spread)
    ids = torch.randint(V - spread, V, (T,), generator=g, device="cuda").int()
    dy = torch.randint(-4, 5, (T, d), generator=g, device="cuda").bfloat16()
    b = L.EmbedBuffers(T, V, d, "bf16")
    b.dtable.fill_(7.0)
    got = L.embed_backward(b, ids, dy).double()
    assert torch.equal(got, torch.zeros((V, d), dtype=torch.float64, device="cuda").index_add_(0, ids.long(), dy.double()))


def test_most_rows():
    from paper_2603_06492_gb300 import binding as B
    T, d = 2 ** 31 - 1, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    for part in x.split(2 ** 27):
        part.normal_(generator=g)
    gain, bias = torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    y, stats = torch.empty_like(x), torch.empty((T, 2), device="cuda")
    dgain, dbias = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    desc = ctypes.byref(B.NormDesc(T, d, 1e-5, 0, 0))
    need = B.load().noble_norm_bwd_workspace_bytes(desc)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    places = [slice(0, 1000), slice(2 ** 28 - 500, 2 ** 28 + 500), slice(2 ** 29 - 500, 2 ** 29 + 500), slice(T - 1000, T)]
    B._check(B.load().noble_norm_fwd(desc, x.data_ptr(), None, gain.data_ptr(), bias.data_ptr(), None, y.data_ptr(), stats.data_ptr(),
                                     B._stream_handle(None)))
    want = []
    for p in places:
        z = x[p].double()
        n = (z - z.mean(1, keepdim=True)) / torch.sqrt(z.var(1, unbiased=False, keepdim=True) + 1e-5)
        w = n * gain.double() + bias.double()
        # one rounding to bf16; in fp32 n is off by a few u of 1 / deviation times the largest element
        slack = 64 * U * (1 + z.abs().amax(1, keepdim=True) * stats[p, 1:].double()) * gain.abs().max().double()
        assert bool(((y[p].double() - w).abs() <= 2.0 ** -8 * w.abs() + slack).all())
        v = gain.double()  # of dy = 1
        want.append((v - v.mean() - n * (v * n).mean(1, keepdim=True)) * stats[p, 1:].double())
    dy = y.fill_(1.0)
    B._check(B.load().noble_norm_bwd(desc, dy.data_ptr(), x.data_ptr(), stats.data_ptr(), gain.data_ptr(), None, dy.data_ptr(),
                                     dgain.data_ptr(), dbias.data_ptr(), work.data_ptr(), need, B._stream_handle(None)))
    torch.cuda.synchronize()
    B.noble_get_device_status(None)
    for p, w in zip(places, want):
        z = x[p].double()
        slack = 64 * U * (1 + z.abs().amax(1, keepdim=True) * stats[p, 1:].double()) * gain.abs().max().double() * stats[p, 1:].double()
        assert bool(((dy[p].double() - w).abs() <= 2.0 ** -8 * w.abs() + slack).all())
    # a part of 512 ones is exact, and so are sums of parts up to 2^33 in steps of 512; the last part has 511
    assert bool(((dbias.double() - T).abs() <= 4 * U * T).all())
    # n has mean 0 and variance 1 over the rows: a sum of 2^31 of them is 5 times 2^15.5 off 0 at most, and its 2^22 parts
    # are added up with errors of 2^17 u of a running sum that stays below 2^18
    assert bool((dgain.abs() <= 5 * 2.0 ** 15.5 + 2.0 ** 11).all())
