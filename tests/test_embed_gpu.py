"""Embedding and its table's gradient against the definition in 64 bits.

Tolerances, of u = 2^-24: y is one product and one rounding, u and, in bf16, 2^-8 of its
value; a row of the gradient is a sum of c products' terms in fp32, (c + 2) u of the sum of
their magnitudes."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
FEW = 1024  # tokens of the path with one launch


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2603_06492_gb300 import binding
    from paper_2603_06492_gb300.build import build
    build()
    binding.load()


def _ids(T, V, how, seed=0):
    g = torch.Generator().manual_seed(seed)
    if how == "one":
        return torch.full((T,), V // 2, dtype=torch.int32)
    if how == "last":
        return torch.full((T,), V - 1, dtype=torch.int32)
    if how == "skewed":
        ids = ((V + 2.7) / 2.7) ** torch.rand(T, generator=g, dtype=torch.float64) * 2.7 - 2.7
        ids = torch.randperm(V, generator=g)[ids.long().clamp(0, V - 1)]
    else:
        ids = torch.randint(0, V, (T,), generator=g)
    if how == "padded":
        ids[torch.randperm(T, generator=g)[:T // 3 + 1]] = -1
        ids[:1] = -2 ** 31
    return ids.int()


def _check(T, V, d, dtype, how, scale=1.0, seed=0):
    from paper_2603_06492_gb300 import layers as L
    g = torch.Generator().manual_seed(seed + 1)
    ids = _ids(T, V, how, seed)
    table, dy = torch.randn((V, d), generator=g).to(DT[dtype]), torch.randn((T, d), generator=g).to(DT[dtype])
    b = L.EmbedBuffers(T, V, d, dtype, scale=scale)
    b.y.fill_(float("nan")), b.dtable.fill_(float("nan"))
    live = ids >= 0
    dy[~live] = float("nan")  # what padding holds does not matter
    y = L.embed_forward(b, ids.cuda(), table.cuda()).cpu().double()
    got = L.embed_backward(b, ids.cuda(), dy.cuda()).cpu().double()
    rows = ids.long()
    want = torch.zeros((T, d), dtype=torch.float64)
    want[live] = scale * table.double()[rows[live]]
    half = 2.0 ** -8 if dtype == "bf16" else U
    assert bool(((y - want).abs() <= (half + U) * want.abs()).all())
    grad, mag, count = (torch.zeros((V, w), dtype=torch.float64) for w in (d, d, 1))
    grad.index_add_(0, rows[live], dy.double()[live])
    mag.index_add_(0, rows[live], dy.double()[live].abs())
    count.index_add_(0, rows[live], torch.ones((int(live.sum()), 1), dtype=torch.float64))
    off = (got - scale * grad).abs()
    assert bool((off <= (count + 2) * U * abs(scale) * mag).all()), (off.max().item(), how)
    return b, ids.cuda(), dy.cuda()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,V,d", [(1, 1, 8), (1, 100, 64), (7, 3, 264), (24, 1000, 2048), (100, 63, 520), (257, 65, 1000),
                                   (FEW - 1, 500, 136), (FEW, 64, 256), (FEW + 1, 64, 256), (3000, 7, 40), (5000, 1001, 264),
                                   (4097, 20000, 128), (64, 2, 72), (65, 2, 72), (1000, 2100, 136), (FEW, 5000, 264), (6000, 16, 64),
                                   (16385, 70000, 16), (70000, 11, 8)])
@pytest.mark.parametrize("how", ["even", "skewed", "padded", "one"])
def test_sizes(T, V, d, dtype, how):
    _check(T, V, d, dtype, how, scale=0.5 if how == "even" else 1.0)


@pytest.mark.parametrize("T", [FEW, 2 * FEW])
@pytest.mark.parametrize("scale", [0.0, -3.0, 45.254833])
def test_scales(T, scale):
    _check(T, 300, 64, "bf16", "skewed", scale)


@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000])
@pytest.mark.parametrize("T", [1024, 3000])
def test_lengths_of_lists(T, n):
    # one row with exactly n tokens, spread among others
    from paper_2603_06492_gb300 import layers as L
    V, d = 5000, 72
    g = torch.Generator().manual_seed(n)
    ids = torch.randint(0, V - 1, (T,), generator=g)
    ids[torch.randperm(T, generator=g)[:n]] = V - 1
    dy = torch.randint(-8, 9, (T, d), generator=g).float()  # sums are exact
    b = L.EmbedBuffers(T, V, d, "fp32")
    got = L.embed_backward(b, ids.int().cuda(), dy.cuda()).cpu()
    assert torch.equal(got, torch.zeros(V, d).index_add_(0, ids, dy))


def test_wide_rows_and_many_tokens():
    _check(3, 5, 65536, "bf16", "even")
    _check(2500, 9, 16392, "bf16", "skewed")
    _check(300000, 3, 8, "fp32", "skewed")   # lists beyond one window of the bit map
    _check(600000, 100, 16, "bf16", "last")


def test_all_padding():
    for T in (5, 3000):
        from paper_2603_06492_gb300 import layers as L
        b = L.EmbedBuffers(T, 50, 64, "bf16")
        b.dtable.fill_(1.0)
        ids = torch.full((T,), -1, dtype=torch.int32, device="cuda")
        assert not L.embed_forward(b, ids, torch.ones((50, 64), dtype=torch.bfloat16, device="cuda")).any()
        assert not L.embed_backward(b, ids, torch.full((T, 64), float("nan"), dtype=torch.bfloat16, device="cuda")).any()


def test_no_tokens():
    from paper_2603_06492_gb300 import layers as L
    b = L.EmbedBuffers(0, 10, 16, "fp32")
    b.dtable.fill_(1.0)
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    L.embed_forward(b, ids, torch.ones((10, 16), device="cuda"))
    assert not L.embed_backward(b, ids, torch.empty((0, 16), device="cuda")).any()


@pytest.mark.parametrize("T", [10, 4000])
def test_tokens_beyond_the_table(T):
    # reported, and treated as padding
    from paper_2603_06492_gb300 import binding as B, layers as L
    V, d = 40, 32
    ids = torch.arange(T, dtype=torch.int32) % V
    bad = ids.clone()
    bad[3], bad[T - 1] = V, 2 ** 31 - 1
    padded = ids.clone()
    padded[3] = padded[T - 1] = -1
    dy, table = torch.randn(T, d).cuda(), torch.randn(V, d).cuda()
    b = L.EmbedBuffers(T, V, d, "fp32")
    y, g = (t.clone() for t in (L.embed_forward(b, padded.cuda(), table), L.embed_backward(b, padded.cuda(), dy)))
    B.noble_get_device_status(None)
    for call, want in ((lambda: L.embed_forward(b, bad.cuda(), table), y), (lambda: L.embed_backward(b, bad.cuda(), dy), g)):
        got = call()
        with pytest.raises(B.NobleError):
            B.noble_get_device_status(None)
        assert torch.equal(got, want)
    B.noble_get_device_status(None)


@pytest.mark.parametrize("T", [1500, 20000])
def test_repeats_streams_and_graphs(T):
    from paper_2603_06492_gb300 import layers as L
    b, ids, dy = _check(T, 3001, 256, "bf16", "skewed")
    dy = dy.nan_to_num()
    want = L.embed_backward(b, ids, dy).clone()
    b.workspace.fill_(255)  # whatever an earlier call left there
    for _ in range(5):
        assert torch.equal(L.embed_backward(b, ids, dy), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    L.embed_backward(b, ids, dy, stream=side)
    side.synchronize()
    assert torch.equal(b.dtable, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.embed_backward(b, ids, dy)
    for _ in range(2):
        b.dtable.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.dtable, want)
    dy.neg_()
    ids.copy_(ids.flip(0))
    dy.copy_(dy.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    # the same sums in the other order
    assert ((b.dtable + want).abs().max() <= 1e-3).item()


def test_workspace_stays_in_its_size():
    from paper_2603_06492_gb300 import binding as B, layers as L
    for T, V, how in ((5000, 40, "one"), (3333, 33, "even"), (9000, 100, "skewed"), (2049, 1, "one")):
        b = L.EmbedBuffers(T, V, 64, "bf16")
        room = torch.full((b.workspace_bytes + 4096,), 171, dtype=torch.uint8, device="cuda")
        ids, dy = _ids(T, V, how).cuda(), torch.randn(T, 64).bfloat16().cuda()
        B._check(B.load().noble_embed_bwd(b._ref, ids.data_ptr(), dy.data_ptr(), b.dtable.data_ptr(), room.data_ptr(),
                                          b.workspace_bytes, B._stream_handle(None)))
        torch.cuda.synchronize()
        assert bool((room[b.workspace_bytes:] == 171).all())


@pytest.mark.parametrize("T", [60, 5000])
def test_offsets_beyond_32_bits(T):
    # 2.2e9 elements of the table: rows at both ends, on the device
    from paper_2603_06492_gb300 import layers as L
    V, d = 540001, 4096
    g = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.randint(V - 50, V, (T,), generator=g, device="cuda").int()
    ids[::7] = torch.randint(0, 50, (len(ids[::7]),), generator=g, device="cuda").int()
    table = torch.empty((V, d), dtype=torch.bfloat16, device="cuda")
    for rows in (slice(0, 50), slice(V - 50, V)):
        table[rows] = torch.randn((50, d), generator=g, device="cuda").bfloat16()
    dy = torch.randint(-8, 9, (T, d), generator=g, device="cuda").bfloat16()  # sums are exact
    b = L.EmbedBuffers(T, V, d, "bf16")
    b.dtable.fill_(7.0)
    assert torch.equal(L.embed_forward(b, ids, table), table[ids.long()])
    got = L.embed_backward(b, ids, dy)
    for lo in (0, V - 50):
        inside = (ids >= lo) & (ids < lo + 50)
        want = torch.zeros((50, d), device="cuda").index_add_(0, ids[inside].long() - lo, dy[inside].float())
        assert torch.equal(got[lo:lo + 50], want)
    assert not any(bool(got[i:i + 50000].any()) for i in range(50, V - 50, 50000) if i + 50000 <= V - 50)
