"""Refusals of the attention operators, on the host: a wrong argument gives its status
before any device is touched; a right call reaches the device check."""
import ctypes

import pytest
import torch

from paper_2603_06492_gb300 import binding as B
from paper_2603_06492_gb300.build import build

FAKE = 0x100000  # aligned, never dereferenced
INVALID, MISALIGNED, UNSUPPORTED, SMALL, NO_DEVICE = 1, 2, 3, 4, 7


@pytest.fixture(scope="module")
def lib():
    build()
    return B.load()


def _heads(n, d, **over):
    h = B.Heads(FAKE, n * d, d)
    for k, v in over.items():
        setattr(h, k, v)
    return ctypes.byref(h)


def _refused(fn, args, status):
    if status == NO_DEVICE and torch.cuda.is_available():
        pytest.skip("device present: an accepted call would read the fake pointers")
    with pytest.raises(B.NobleError) as e:
        B._check(fn(*args))
    assert e.value.status == status, str(e.value)


def _desc(cls, base, over):
    return cls(**{**base, **over})


ROPE = dict(T=10, n_q=4, n_kv=2, d=64, rot=64, positions=100, eps=1e-6, dtype=0, flags=2)
ATTN = dict(T=10, n_docs=1, n_q=4, n_kv=2, d=64, window=0, scale=0.125, softcap=0.0, dtype=0, flags=1)
PAGED = dict(n_seq=3, q_len=1, n_q=4, n_kv=2, d=64, max_pages=8, max_len=500, window=0, scale=0.125, softcap=0.0, dtype=0,
             flags=0)
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("over,status", [
    ({}, NO_DEVICE), (dict(T=-1), INVALID), (dict(positions=-1), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=NAN), INVALID),
    (dict(eps=INF), INVALID), (dict(n_q=0), INVALID), (dict(n_kv=-2), INVALID), (dict(n_q=5000), INVALID), (dict(d=12), UNSUPPORTED),
    (dict(d=0), UNSUPPORTED), (dict(d=264), UNSUPPORTED), (dict(rot=66), UNSUPPORTED), (dict(rot=3), UNSUPPORTED),
    (dict(rot=-2), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(flags=4), UNSUPPORTED), (dict(T=2 ** 31), UNSUPPORTED)])
def test_rope_descriptors(lib, over, status):
    d = ctypes.byref(_desc(B.RopeDesc, ROPE, over))
    q, k = _heads(4, 64), _heads(2, 64)
    _refused(lib.noble_rope_fwd, (d, q, k, FAKE, FAKE, FAKE, FAKE, q, k, None), status)
    _refused(lib.noble_rope_bwd, (d, q, k, q, k, FAKE, FAKE, FAKE, FAKE, q, k, FAKE, FAKE, FAKE, 1 << 40, None), status)
    cache = ctypes.byref(B.KvCache(FAKE, FAKE, 4, 16, 16 * 128, 128, 64))
    _refused(lib.noble_kv_append, (d, q, k, k, FAKE, FAKE, FAKE, FAKE, FAKE, q, cache, None), status)
    if status in (INVALID, UNSUPPORTED):
        assert lib.noble_rope_bwd_workspace_bytes(d) == 0


@pytest.mark.parametrize("over,status", [
    ({}, NO_DEVICE), (dict(T=-1), INVALID), (dict(n_docs=-1), INVALID), (dict(n_q=5), INVALID), (dict(n_kv=0), INVALID),
    (dict(d=136), UNSUPPORTED), (dict(d=4), UNSUPPORTED), (dict(window=-1), INVALID), (dict(scale=NAN), INVALID),
    (dict(scale=INF), INVALID), (dict(softcap=-1.0), INVALID), (dict(softcap=NAN), INVALID), (dict(dtype=7), UNSUPPORTED),
    (dict(flags=8), UNSUPPORTED), (dict(T=2 ** 24 + 1), UNSUPPORTED), (dict(n_docs=2 ** 24 + 1), UNSUPPORTED)])
def test_attn_descriptors(lib, over, status):
    d = ctypes.byref(_desc(B.AttnDesc, ATTN, over))
    q, k = _heads(4, 64), _heads(2, 64)
    _refused(lib.noble_attn_fwd, (d, q, k, k, FAKE, None, None, q, FAKE, None), status)
    _refused(lib.noble_attn_bwd, (d, q, q, k, k, FAKE, None, None, q, FAKE, q, k, k, FAKE, 1 << 40, None), status)
    if status in (INVALID, UNSUPPORTED):
        assert lib.noble_attn_bwd_workspace_bytes(d) == 0


@pytest.mark.parametrize("over,status", [
    ({}, NO_DEVICE), (dict(n_seq=-1), INVALID), (dict(q_len=0), INVALID), (dict(q_len=65), UNSUPPORTED), (dict(n_q=3), INVALID),
    (dict(d=20), UNSUPPORTED), (dict(max_pages=-1), INVALID), (dict(max_len=-1), INVALID), (dict(max_len=2 ** 31), UNSUPPORTED),
    (dict(n_seq=65536), UNSUPPORTED), (dict(window=-5), INVALID), (dict(scale=NAN), INVALID), (dict(flags=1), UNSUPPORTED)])
def test_paged_descriptors(lib, over, status):
    d = ctypes.byref(_desc(B.PagedDesc, PAGED, over))
    cache = ctypes.byref(B.KvCache(FAKE, FAKE, 4, 16, 16 * 128, 128, 64))
    q = _heads(4, 64)
    _refused(lib.noble_attn_paged, (d, q, cache, FAKE, FAKE, None, q, None, FAKE, 1 << 50, None), status)
    if status in (INVALID, UNSUPPORTED):
        assert lib.noble_attn_paged_workspace_bytes(d) == 0


@pytest.mark.parametrize("at,over,status", [
    (0, dict(p=None), INVALID), (1, dict(p=FAKE + 8), MISALIGNED), (2, dict(row=100), MISALIGNED), (0, dict(head=4), MISALIGNED),
    (2, dict(row=2 ** 50), UNSUPPORTED), (6, dict(p=None), INVALID), (6, dict(row=0), UNSUPPORTED), (6, dict(head=32), UNSUPPORTED),
    (6, dict(row=128), UNSUPPORTED), (0, dict(row=0), NO_DEVICE), (1, dict(row=-512), NO_DEVICE), (6, dict(row=64, head=640), NO_DEVICE)])
def test_attn_tensors(lib, at, over, status):
    d = ctypes.byref(_desc(B.AttnDesc, ATTN, {}))
    q, k = _heads(4, 64), _heads(2, 64)
    args = [q, k, k, FAKE, None, None, q, FAKE, None]
    args[at] = _heads(2 if at in (1, 2) else 4, 64, **over)
    _refused(lib.noble_attn_fwd, (d, *args), status)


@pytest.mark.parametrize("at,value,status", [
    (0, None, INVALID), (3, None, INVALID), (3, FAKE + 2, MISALIGNED), (4, FAKE + 2, MISALIGNED), (5, FAKE + 1, MISALIGNED),
    (6, None, INVALID), (7, None, INVALID), (7, FAKE + 4, MISALIGNED), (4, FAKE + 4, NO_DEVICE)])
def test_attn_pointers(lib, at, value, status):
    d = ctypes.byref(_desc(B.AttnDesc, ATTN, {}))
    q, k = _heads(4, 64), _heads(2, 64)
    args = [q, k, k, FAKE, None, None, q, FAKE, None]
    args[at] = value
    _refused(lib.noble_attn_fwd, (d, *args), status)


def test_null_descriptors_and_workspaces(lib):
    q, k = _heads(4, 64), _heads(2, 64)
    _refused(lib.noble_attn_fwd, (None, q, k, k, FAKE, None, None, q, FAKE, None), INVALID)
    d = ctypes.byref(_desc(B.AttnDesc, ATTN, {}))
    need = lib.noble_attn_bwd_workspace_bytes(d)
    args = (d, q, q, k, k, FAKE, None, None, q, FAKE, q, k, k)
    _refused(lib.noble_attn_bwd, (*args, FAKE, need - 1, None), SMALL)
    _refused(lib.noble_attn_bwd, (*args, None, need, None), INVALID)
    _refused(lib.noble_attn_bwd, (*args, FAKE, need, None), NO_DEVICE)
    r = ctypes.byref(_desc(B.RopeDesc, ROPE, {}))
    need = lib.noble_rope_bwd_workspace_bytes(r)
    args = (r, q, k, q, k, FAKE, FAKE, FAKE, FAKE, q, k)
    _refused(lib.noble_rope_bwd, (*args, FAKE, FAKE, FAKE, need - 1, None), SMALL)
    _refused(lib.noble_rope_bwd, (*args, FAKE, FAKE, None, need, None), INVALID)
    _refused(lib.noble_rope_bwd, (*args, None, None, None, 0, None), NO_DEVICE)  # no gain gradients, no workspace
    p = ctypes.byref(_desc(B.PagedDesc, PAGED, dict(max_len=100000)))
    need = lib.noble_attn_paged_workspace_bytes(p)
    cache = ctypes.byref(B.KvCache(FAKE, FAKE, 4, 16, 16 * 128, 128, 64))
    _refused(lib.noble_attn_paged, (p, q, cache, FAKE, FAKE, None, q, None, FAKE, need - 1, None), SMALL)
    _refused(lib.noble_attn_paged, (p, q, cache, FAKE, FAKE, None, q, None, None, need, None), INVALID)
    _refused(lib.noble_attn_paged, (p, q, None, FAKE, FAKE, None, q, None, FAKE, need, None), INVALID)


@pytest.mark.parametrize("over,status", [
    (dict(k=None), INVALID), (dict(v=FAKE + 8), MISALIGNED), (dict(page=2052), MISALIGNED), (dict(page=128), UNSUPPORTED),
    (dict(row=64), UNSUPPORTED), (dict(head=-64), UNSUPPORTED), (dict(page_size=0), INVALID), (dict(pages=-1), INVALID),
    (dict(page_size=2 ** 20 + 1), UNSUPPORTED), (dict(row=64, head=16 * 64), NO_DEVICE)])
def test_append_caches(lib, over, status):
    d = ctypes.byref(_desc(B.RopeDesc, ROPE, {}))
    q, k = _heads(4, 64), _heads(2, 64)
    cache = _desc(B.KvCache, dict(k=FAKE, v=FAKE, pages=4, page_size=16, page=16 * 128, row=128, head=64), over)
    _refused(lib.noble_kv_append, (d, q, k, k, FAKE, FAKE, FAKE, FAKE, FAKE, q, ctypes.byref(cache), None), status)


@pytest.mark.parametrize("args,status", [
    ((-1, 64, {}), INVALID), ((10, 63, {}), INVALID), ((10, 512, {}), INVALID), ((10, 64, dict(base=0.0)), INVALID),
    ((10, 64, dict(factor=-1.0)), INVALID), ((10, 64, dict(original=0.0)), INVALID), ((10, 64, dict(low_turns=2.0)), INVALID),
    ((10, 64, dict(low_turns=NAN)), INVALID), ((10, 64, dict(amplitude=INF)), INVALID), ((10, 64, {}), NO_DEVICE)])
def test_rope_table(lib, args, status):
    n, rot, over = args
    s = B.RopeScaling(**{**dict(base=1e4, factor=1.0, original=1.0, low_turns=0.0, high_turns=0.0, amplitude=1.0), **over})
    _refused(lib.noble_rope_table, (n, rot, ctypes.byref(s), FAKE, None), status)


def test_torch_side_refuses_other_tensors(lib):
    from paper_2603_06492_gb300 import attention as A
    x = torch.zeros(3, 2, 8)
    with pytest.raises(ValueError):
        A._Slots(1).put(0, x, (3, 2, 8), torch.float32)  # not on a GPU
    with pytest.raises(ValueError):
        A._flat(x, "x", torch.float32, (3, 2, 9))
