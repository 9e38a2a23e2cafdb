"""A stack's number of blocks and the table of rotations that they share, on the host; a stack without
blocks, which is its table and its last norm, on a GPU."""
import pytest
import torch

from paper_2603_06492_gb300.block import Stack

SIZES = (50, 64, 4, 2, 16, 8)  # vocab, d_model, heads, heads of keys, d, r


def _stack(blocks, **options):
    return Stack(SIZES[0], blocks, *SIZES[1:], dtype="fp32", **options)


@pytest.mark.parametrize("blocks", [0, 1, 2, 5])
def test_blocks_and_their_table(blocks):
    table = torch.zeros(128, 16)
    s = _stack(blocks, table=table, positions=128, window=7)
    assert len(s.blocks) == blocks and len({id(b) for b in s.blocks}) == blocks
    assert all(b.table is table and b.scores["window"] == 7 for b in s.blocks)


def test_less_than_none():
    with pytest.raises(ValueError):
        _stack(-1, table=torch.zeros(128, 16))


@pytest.mark.gpu
def test_no_blocks():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2603_06492_gb300.block import Update
    s, T, V, d = _stack(0, scale=2.0), 37, SIZES[0], SIZES[1]
    g = torch.Generator().manual_seed(0)
    rn = lambda *n: torch.randn(n, generator=g)  # noqa: E731
    params = {"table": rn(V, d).cuda(), "norms": [{"gain": (1 + 0.1 * rn(d)).cuda(), "bias": rn(d).cuda()}], "blocks": []}
    ids, dy = torch.randint(-1, V, (T,), generator=g).int().cuda(), rn(T, d).cuda()
    b = s.buffers(T)
    y = s.forward(b, ids, params, None, None)
    grads = s.backward(b, ids, dy, params, None, None)
    # the same in 64 bits
    leaves = [params["table"], params["norms"][0]["gain"], params["norms"][0]["bias"]]
    e, gain, bias = (p.double().requires_grad_() for p in leaves)
    live = (ids >= 0)[:, None]
    want = torch.nn.functional.layer_norm(2.0 * e[ids.long().clamp(min=0)] * live, (d,), gain, bias, 1e-5)
    want.backward(dy.double())
    got = (y, grads["table"], grads["norms"][0]["gain"], grads["norms"][0]["bias"])
    # three operators in fp32, sums of up to 64 terms: 100 roundings of the largest value; a row of padding has no variance,
    # and only the gain's and the bias' gradients see it
    for a, w in zip(got, (want, e.grad, gain.grad, bias.grad)):
        assert (a.double() - w).abs().max() <= 100 * 2.0 ** -24 * (1 + w.abs().max())
    u, old = Update(params, grads), [p.clone() for p in leaves]
    u.step(lr=1e-2, lr_matrices=0.1)
    torch.cuda.synchronize()
    assert not u.muon and all(p.isfinite().all() and not torch.equal(p, q) for p, q in zip(leaves, old))
    step = s.step_buffers(3, max_len=8)
    last = s.step(step, s.caches(4, 8), ids[:3].contiguous(), params, None, None, None, None)
    again = s.forward(b, ids, params, None, None)
    assert torch.equal(last, again[:3])
