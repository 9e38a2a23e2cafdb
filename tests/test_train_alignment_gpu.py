"""Buffers at 16 bytes past a multiple of 32, which is all that the interface asks for: the operators
around the projections give the bits that they give on buffers of torch's own, aligned to more."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2603_06492_gb300 import binding
    from paper_2603_06492_gb300.build import build
    build()
    binding.load()


def _placed(shape, dtype, off):
    """An uninitialised tensor whose address is ``off`` past a multiple of 256, and the bytes around it,
    all of them 171."""
    n = torch.Size(shape).numel() * dtype.itemsize
    room = torch.full((n + 1024,), 171, dtype=torch.uint8, device="cuda")
    start = -room.data_ptr() % 256 + off
    return room[start:start + n].view(dtype).view(shape), (room[:start], room[start + n:])


def _untouched(around):
    return all(bool((r == 171).all()) for r in around)


# the list path with one row of several pieces, whose sums go to the workspace; lists of one piece; few tokens
@pytest.mark.parametrize("T,V,many", [(3000, 500, 400), (1500, 40, 0), (20000, 70000, 9000), (512, 5000, 100)])
@pytest.mark.parametrize("d", [8, 264, 520])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_embedding_gradient(T, V, many, d, dtype):
    from paper_2603_06492_gb300 import binding as B
    g = torch.Generator(device="cuda").manual_seed(T)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda").int()
    ids[torch.randperm(T, generator=g, device="cuda")[:many]] = V // 3
    dy = torch.randn((T, d), generator=g, device="cuda").to(dtype)
    desc = ctypes.byref(B.EmbedDesc(T, V, d, 0.5, 0 if dtype is torch.bfloat16 else 1, 0))
    need, want = B.load().noble_embed_bwd_workspace_bytes(desc), None
    for out_off, work_off in ((0, 0), (0, 16), (16, 0), (16, 16)):
        out, out_around = _placed((V, d), torch.float32, out_off)
        work, work_around = _placed((need,), torch.uint8, work_off)
        B._check(B.load().noble_embed_bwd(desc, ids.data_ptr(), dy.data_ptr(), out.data_ptr(), work.data_ptr(), need,
                                          B._stream_handle(None)))
        torch.cuda.synchronize()
        B.noble_get_device_status(None)
        want = out.clone() if want is None else want
        assert torch.equal(out, want) and _untouched(out_around) and _untouched(work_around), (out_off, work_off)
    sums = torch.zeros((V, d), dtype=torch.float64, device="cuda").index_add_(0, ids.long(), dy.double())
    size = torch.zeros((V, d), dtype=torch.float64, device="cuda").index_add_(0, ids.long(), dy.double().abs())
    # a sum of n terms is off by n u of their magnitudes, its product by u
    count = torch.bincount(ids.long(), minlength=V)[:, None].double()
    assert bool(((want.double() - 0.5 * sums).abs() <= (count + 2) * 2.0 ** -24 * 0.5 * size).all())
