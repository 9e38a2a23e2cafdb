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


def _copies(tensors, off):
    """Copies of the tensors at ``off``, and what is around them."""
    out, around = {}, []
    for k, t in tensors.items():
        out[k], room = _placed(t.shape, t.dtype, off)
        out[k].copy_(t)
        around += room
    return out, around


@pytest.mark.parametrize("T,d", [(3, 8), (50, 264), (700, 2048), (200, 768), (9, 16384)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm(T, d, dtype):
    from paper_2603_06492_gb300 import binding as B
    g = torch.Generator(device="cuda").manual_seed(d)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    first = {**{k: rn(T, d).to(dtype) for k in ("x", "res", "dy", "dstream", "sum", "y", "dx")}, **{k: rn(d) for k in ("gain", "bias", "dgain", "dbias")},
             "stats": rn(T, 2)}
    desc = ctypes.byref(B.NormDesc(T, d, 1e-5, 0 if dtype is torch.bfloat16 else 1, 0))
    need = B.load().noble_norm_bwd_workspace_bytes(desc)
    first["workspace"] = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    got = []
    for off in (0, 16):
        t, around = _copies(first, off)
        p = {k: v.data_ptr() for k, v in t.items()}
        B._check(B.load().noble_norm_fwd(desc, p["x"], p["res"], p["gain"], p["bias"], p["sum"], p["y"], p["stats"], B._stream_handle(None)))
        B._check(B.load().noble_norm_bwd(desc, p["dy"], p["sum"], p["stats"], p["gain"], p["dstream"], p["dx"], p["dgain"], p["dbias"],
                                         p["workspace"], need, B._stream_handle(None)))
        torch.cuda.synchronize()
        B.noble_get_device_status(None)
        assert _untouched(around)
        got.append(t)
    assert all(torch.equal(got[0][k], got[1][k]) for k in first if k != "workspace")
    # one of the two against the definition: test_norm_gpu.py has the tolerances
    z = (first["x"].double() + first["res"].double()).to(dtype).double()
    want = torch.nn.functional.layer_norm(z, (d,), first["gain"].double(), first["bias"].double(), 1e-5)
    half = 2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -24
    assert bool(((got[0]["y"].double() - want).abs() <= half * want.abs() + 4 * (d / 32 + 16) * 2.0 ** -24 * 4 * want.abs().max()).all())


@pytest.mark.parametrize("shapes", [[(300, 310)], [(301, 77), (64, 100)], [(128, 2048), (9, 7)], [(1100, 2300), (300, 400)]])
@pytest.mark.parametrize("precise", [False, True])
def test_optimizer_step(shapes, precise):
    from paper_2603_06492_gb300 import binding as B
    g = torch.Generator(device="cuda").manual_seed(5)
    first = [{**{k: torch.randn(s, generator=g, device="cuda") for k in ("param", "grad", "momentum")},
              **{k: torch.empty(s, dtype=torch.bfloat16, device="cuda") for k in ("param_bf16", "update")}} for s in shapes]
    need, got = B.muon_workspace(first, precise).numel(), []
    for off in (0, 16):
        copies = [_copies(t, off) for t in first]
        work, around = _placed((need,), torch.uint8, off)
        B.noble_muon_step([t for t, _ in copies], 0.1, precise=precise, workspace=work)
        torch.cuda.synchronize()
        B.noble_get_device_status(None)
        assert _untouched(around) and all(_untouched(r) for _, r in copies)
        got.append([t for t, _ in copies])
    assert all(a[k].isfinite().all() and torch.equal(a[k], b[k]) for a, b in zip(*got) for k in a)
