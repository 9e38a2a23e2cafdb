"""Gradients of norm and rotation where eps is 0 and where a token has no position, against
their definitions in 64 bits.  Errors and tolerances as in test_rope_gpu.py."""
import pytest
import torch

from tests import attention_ref as ref
from tests.gpu_helpers import TOL, rel_err
from tests.test_rope_gpu import _case, _cuda

pytestmark = pytest.mark.gpu
both = pytest.mark.parametrize("dtype", ["bf16", "fp32"])


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2603_06492_gb300 import binding
    from paper_2603_06492_gb300.build import build
    build()
    binding.load()


@both
@pytest.mark.parametrize("T,nq,nkv,d,rot", [(5, 16, 4, 128, 128), (7, 3, 3, 80, 20), (40, 5, 1, 64, 64), (3, 1, 1, 256, 0)])
def test_gains_without_eps(T, nq, nkv, d, rot, dtype):
    # heads that do not fill a warp's batch: the places left over have no norm
    from paper_2603_06492_gb300 import attention as A
    qkv, pos, table, (gq, gk), dq, dk = _case(T, nq, nkv, d, rot, dtype)
    buf = A.RopeBuffers(T, nq, nkv, d, dtype, rot=rot, positions=50, eps=0.0)
    args = _cuda(qkv, pos, table, gq, gk)
    yq, yk = A.rope_forward(buf, *args)
    dxq, dxk = A.rope_backward(buf, *_cuda(dq, dk), *args)
    h = qkv.view(T, nq + 2 * nkv, d)
    for x, y, dx, dy, gain, dgain in ((h[:, :nq], yq, dxq, dq, gq, buf.dgain_q),
                                      (h[:, nq:nq + nkv], yk, dxk, dk, gk, buf.dgain_k)):
        wy, wdx, wdg = ref.rope(x, pos, table, rot, False, gain, 0.0, True, dy)
        assert rel_err(y.float().cpu(), wy) <= TOL[dtype] and rel_err(dx.float().cpu(), wdx) <= TOL[dtype]
        assert rel_err(dgain.cpu(), wdg) <= 1e-5


@both
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_of_a_token_without_a_position(bad, dtype):
    # its outputs are 0, so its inputs have no gradient and no part in the gains'
    from paper_2603_06492_gb300 import attention as A, binding
    T, nq, nkv, d = 6, 4, 2, 64
    qkv, pos, table, (gq, gk), dq, dk = _case(T, nq, nkv, d, d, dtype)
    keep = torch.arange(T) != 3
    h = qkv.view(T, -1, d)
    _, wdx, wdg = ref.rope(h[keep, :nq], pos[keep], table, d, False, gq, 1e-6, True, dq[keep])
    pos[3], qkv[3], dq[3], dk[3] = -1, bad, bad, bad
    buf = A.RopeBuffers(T, nq, nkv, d, dtype, positions=50)
    args = _cuda(qkv, pos, table, gq, gk)
    yq, _ = A.rope_forward(buf, *args)
    dxq, dxk = A.rope_backward(buf, *_cuda(dq, dk), *args)
    with pytest.raises(binding.NobleError):
        binding.noble_get_device_status(None)
    assert not yq[3].any() and not dxq[3].any() and not dxk[3].any()
    assert rel_err(dxq.float().cpu()[keep], wdx) <= TOL[dtype]
    assert rel_err(buf.dgain_q.cpu(), wdg) <= 1e-5 and torch.isfinite(buf.dgain_k).all()
