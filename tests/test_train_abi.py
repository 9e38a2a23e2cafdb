"""Refusals of layer norm, embedding and the optimizer step by orthogonalised momentum, on the
host: a wrong argument gives its status before any device is touched; a right call reaches
the device check."""
import ctypes
import os
import re

import pytest
import torch

from paper_2603_06492_gb300 import binding as B
from paper_2603_06492_gb300.build import CSRC, build

FAKE = 0x100000  # aligned, never dereferenced
INVALID, MISALIGNED, UNSUPPORTED, SMALL, NO_DEVICE = 1, 2, 3, 4, 7
NAN, INF = float("nan"), float("inf")
ROOM = 1 << 40


@pytest.fixture(scope="module")
def lib():
    build()
    return B.load()


def _refused(fn, args, status):
    if status == NO_DEVICE and torch.cuda.is_available():
        pytest.skip("device present: an accepted call would read the fake pointers")
    with pytest.raises(B.NobleError) as e:
        B._check(fn(*args))
    assert e.value.status == status, str(e.value)


NORM = dict(T=10, d=64, eps=1e-5, dtype=0, flags=0)
EMBED = dict(T=10, vocab=100, d=64, scale=1.0, dtype=0, flags=0)


@pytest.mark.parametrize("over,status", [
    ({}, NO_DEVICE), (dict(d=16384), NO_DEVICE), (dict(eps=0.0), NO_DEVICE), (dict(T=-1), INVALID), (dict(eps=-1e-5), INVALID),
    (dict(eps=NAN), INVALID), (dict(eps=INF), INVALID), (dict(T=2 ** 31), UNSUPPORTED), (dict(d=0), UNSUPPORTED),
    (dict(d=12), UNSUPPORTED), (dict(d=16392), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(flags=1), UNSUPPORTED)])
def test_norm_descriptors(lib, over, status):
    d = ctypes.byref(B.NormDesc(**{**NORM, **over}))
    _refused(lib.noble_norm_fwd, (d, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE + 4096, FAKE, None), status)
    _refused(lib.noble_norm_bwd, (d, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE + 4096, FAKE, ROOM, None), status)
    assert (lib.noble_norm_bwd_workspace_bytes(d) == 0) == (status in (INVALID, UNSUPPORTED))


FWD, BWD = [FAKE] * 5 + [FAKE + 4096, FAKE], [FAKE] * 7 + [FAKE + 4096, FAKE]


@pytest.mark.parametrize("at,value,status", [
    (0, None, INVALID), (0, FAKE + 8, MISALIGNED), (1, None, NO_DEVICE), (1, FAKE + 2, MISALIGNED), (2, None, NO_DEVICE),
    (2, FAKE + 4, MISALIGNED), (3, None, NO_DEVICE), (4, None, INVALID), (4, FAKE + 4096, INVALID), (5, None, INVALID),
    (6, None, NO_DEVICE), (6, FAKE + 8, MISALIGNED)])
def test_norm_forward_pointers(lib, at, value, status):
    args = list(FWD)
    args[at] = value
    _refused(lib.noble_norm_fwd, (ctypes.byref(B.NormDesc(**NORM)), *args, None), status)


@pytest.mark.parametrize("at,value,status", [
    (0, None, INVALID), (1, None, INVALID), (2, None, INVALID), (3, None, NO_DEVICE), (4, None, NO_DEVICE), (4, FAKE + 2, MISALIGNED),
    (5, None, INVALID), (6, None, NO_DEVICE), (6, FAKE + 4096, INVALID), (7, None, NO_DEVICE), (8, None, INVALID),
    (8, FAKE + 128, NO_DEVICE), (8, FAKE + 4, MISALIGNED)])
def test_norm_backward_pointers(lib, at, value, status):
    args = list(BWD)
    args[at] = value
    _refused(lib.noble_norm_bwd, (ctypes.byref(B.NormDesc(**NORM)), *args, ROOM, None), status)


def test_norm_sizes(lib):
    d = B.NormDesc(**NORM)
    need = lib.noble_norm_bwd_workspace_bytes(ctypes.byref(d))
    _refused(lib.noble_norm_bwd, (ctypes.byref(d), *BWD, need - 1, None), SMALL)
    # nothing to do: no device is asked for
    d.T = 0
    assert lib.noble_norm_fwd(ctypes.byref(d), None, None, None, None, None, None, None, None) == 0


@pytest.mark.parametrize("over,status", [
    ({}, NO_DEVICE), (dict(vocab=2 ** 28), NO_DEVICE), (dict(scale=0.0), NO_DEVICE), (dict(T=-1), INVALID), (dict(vocab=0), INVALID),
    (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID), (dict(T=2 ** 24 + 1), UNSUPPORTED), (dict(vocab=2 ** 28 + 1), UNSUPPORTED),
    (dict(d=4), UNSUPPORTED), (dict(d=65544), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(flags=2), UNSUPPORTED)])
def test_embed_descriptors(lib, over, status):
    d = ctypes.byref(B.EmbedDesc(**{**EMBED, **over}))
    _refused(lib.noble_embed_fwd, (d, FAKE, FAKE, FAKE, None), status)
    _refused(lib.noble_embed_bwd, (d, FAKE, FAKE, FAKE, FAKE, ROOM, None), status)
    assert (lib.noble_embed_bwd_workspace_bytes(d) == 0) == (status in (INVALID, UNSUPPORTED))


@pytest.mark.parametrize("at", [0, 1, 2, 3])
@pytest.mark.parametrize("value,status", [(None, INVALID), (FAKE + 4, MISALIGNED)])
def test_embed_pointers(lib, at, value, status):
    d = ctypes.byref(B.EmbedDesc(**EMBED))
    args = [FAKE] * 4
    args[at] = value
    if at < 3:
        _refused(lib.noble_embed_fwd, (d, *args[:3], None), status)
    _refused(lib.noble_embed_bwd, (d, *args, ROOM, None), status)


@pytest.mark.parametrize("T", [1, 10, 5000, 2 ** 24])
def test_embed_workspace(lib, T):
    d = B.EmbedDesc(**{**EMBED, "T": T})
    need = lib.noble_embed_bwd_workspace_bytes(ctypes.byref(d))
    assert need % 256 == 0
    _refused(lib.noble_embed_bwd, (ctypes.byref(d), FAKE, FAKE, FAKE, FAKE, need - 1, None), SMALL)
    _refused(lib.noble_embed_bwd, (ctypes.byref(d), FAKE, FAKE, FAKE, FAKE, need, None), NO_DEVICE)


MUON = dict(param=FAKE, param_bf16=FAKE + 0x100000, grad=FAKE + 0x200000, momentum=FAKE + 0x300000, update=FAKE + 0x400000,
            rows=20, cols=30, lr_mult=1.0, decay=1)
HP = dict(lr=0.01, momentum=0.95, weight_decay=0.01, eps=1e-7, steps=5, flags=1)


def _muon(lib, tensors, status, hp=None, room=ROOM, ws=FAKE):
    arr = (B.MuonTensor * len(tensors))(*[B.MuonTensor(**t) for t in tensors])
    _refused(lib.noble_muon_step, (arr, len(tensors), ctypes.byref(B.MuonHparams(**{**HP, **(hp or {})})), ws, room, None), status)


@pytest.mark.parametrize("over,status", [
    ({}, NO_DEVICE), (dict(param=None, param_bf16=None), NO_DEVICE), (dict(update=None), NO_DEVICE), (dict(param_bf16=None), NO_DEVICE),
    (dict(param=None), INVALID), (dict(param=None, param_bf16=None, update=None), INVALID), (dict(grad=None), INVALID),
    (dict(momentum=None), INVALID), (dict(grad=FAKE + 8), MISALIGNED), (dict(update=FAKE + 0x400008), MISALIGNED),
    (dict(rows=-1), INVALID), (dict(cols=-3), INVALID), (dict(rows=65537), UNSUPPORTED), (dict(cols=65537), UNSUPPORTED),
    (dict(lr_mult=-1.0), INVALID), (dict(lr_mult=NAN), INVALID), (dict(lr_mult=INF), INVALID), (dict(grad=FAKE), INVALID),
    (dict(momentum=FAKE), INVALID), (dict(update=FAKE + 0x100000), INVALID), (dict(momentum=FAKE + 0x200000), INVALID)])
def test_muon_tensors(lib, over, status):
    _muon(lib, [{**MUON, **over}], status)


@pytest.mark.parametrize("hp,status", [
    (dict(lr=-1.0), INVALID), (dict(lr=NAN), INVALID), (dict(lr=INF), INVALID), (dict(momentum=1.0), INVALID),
    (dict(momentum=-0.1), INVALID), (dict(momentum=NAN), INVALID), (dict(weight_decay=-1.0), INVALID), (dict(weight_decay=INF), INVALID),
    (dict(eps=-1e-9), INVALID), (dict(eps=NAN), INVALID), (dict(steps=-1), INVALID), (dict(steps=17), INVALID),
    (dict(steps=0), NO_DEVICE), (dict(eps=0.0, momentum=0.0, lr=0.0), NO_DEVICE), (dict(flags=4), UNSUPPORTED), (dict(flags=3), NO_DEVICE)])
def test_muon_hparams(lib, hp, status):
    _muon(lib, [MUON], status, hp)


@pytest.mark.parametrize("mine", ["param", "param_bf16", "momentum", "update"])
@pytest.mark.parametrize("theirs", ["param", "param_bf16", "momentum", "update", "grad"])
def test_muon_memory_of_two_tensors(lib, mine, theirs):
    other = {**MUON, **{k: MUON[k] + 0x1000000 for k in ("param", "param_bf16", "grad", "momentum", "update")}}
    _muon(lib, [MUON, other], NO_DEVICE) if not torch.cuda.is_available() else None
    for pair in ([MUON, {**other, mine: MUON[theirs]}], [{**other, mine: MUON[theirs]}, MUON]):
        _muon(lib, pair, INVALID)
    # a gradient may be read for two tensors, and an empty tensor shares nothing
    if not torch.cuda.is_available():
        _muon(lib, [MUON, {**other, "grad": MUON["grad"]}], NO_DEVICE)
        _muon(lib, [MUON, {**other, mine: MUON[theirs], "rows": 0}], NO_DEVICE)


def test_muon_workspace(lib):
    arr = (B.MuonTensor * 1)(B.MuonTensor(**MUON))
    need = lib.noble_muon_workspace_bytes(arr, 1, 1)
    assert need > 0 and lib.noble_muon_workspace_bytes(arr, 1, 8) == 0 and lib.noble_muon_workspace_bytes(arr, -1, 0) == 0
    _muon(lib, [MUON], SMALL, room=need - 1)
    _muon(lib, [MUON], INVALID, ws=None)
    _muon(lib, [MUON], MISALIGNED, ws=FAKE + 8)
    # nothing to do: no device is asked for
    assert lib.noble_muon_step(None, 0, ctypes.byref(B.MuonHparams(**HP)), None, 0, None) == 0
    arr[0].rows = 0
    assert lib.noble_muon_step(arr, 1, ctypes.byref(B.MuonHparams(**HP)), None, 0, None) == 0


def test_torch_side_refuses(lib):
    from paper_2603_06492_gb300 import layers as L
    t = torch.zeros(4, 6)
    with pytest.raises(ValueError):
        B.muon_workspace([{"grad": t, "momentum": t}])  # not on a GPU
    with pytest.raises(ValueError):
        B.muon_workspace([{"grad": torch.zeros(4), "momentum": t}])
    b = L.NormBuffers(4, 8, "fp32", device="cpu", with_grads=False)
    x = torch.zeros(4, 8)
    for bad in (x, x.bfloat16(), x[:3], torch.zeros(4, 16)[:, :8], x.T.contiguous()):
        with pytest.raises(ValueError):
            L.norm_forward(b, bad)
    with pytest.raises(ValueError):
        L.norm_forward(b, x, gain=torch.ones(7))
    with pytest.raises(ValueError):
        L.norm_forward(b, x, res=x)
    with pytest.raises(ValueError):
        L.norm_backward(b, x, x)
    e = L.EmbedBuffers(4, 5, 8, "fp32", device="cpu", with_grads=False)
    with pytest.raises(ValueError):
        L.embed_forward(e, torch.zeros(4, dtype=torch.int64), torch.zeros(5, 8))
    with pytest.raises(ValueError):
        L.embed_forward(e, torch.zeros(4, dtype=torch.int32), torch.zeros(6, 8))
    with pytest.raises(ValueError):
        L.embed_backward(e, torch.zeros(4, dtype=torch.int32), x)


# kernels that start before the one before them has ended and then read what it wrote
@pytest.mark.parametrize("name", ["embed.cuh", "muon.cuh", "muon_gemm.cuh", "norm.cuh"])
def test_no_read_only_loads_in_programmatic_dependents(name):
    with open(os.path.join(CSRC, name)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    assert "griddep_wait" in text and re.findall(r"__ldg\w*|ld\.global\S*\.nc|__restrict__", text) == []


def _body(text, head):
    start = text.index("\n{", text.index(head))
    return text[start:text.index("\n}", start)]


# the shape decides how sums are cut, so that results and sizes are the same on every device
@pytest.mark.parametrize("head", ["int norm_rows_per_part(", "EmbedWork embed_work(", "bool embed_few(", "void muon_cut(", "MuonPlan muon_plan("])
def test_orders_of_sums_do_not_depend_on_the_device(head):
    with open(os.path.join(CSRC, "train_api.cu")) as f:
        text = f.read()
    body = _body(text, head) if not head.startswith("bool") else text[text.index(head):text.index("\n", text.index(head))]
    assert len(body) > 60 and "num_sms" not in body
