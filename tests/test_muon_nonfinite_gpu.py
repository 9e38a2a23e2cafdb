"""A matrix whose u is not finite gets NaN throughout, whatever the number of steps (0 among them: X is
then u over its norm), and no other matrix of the call changes by a bit."""
import pytest
import torch

from tests.test_muon_gpu import _inputs, _run, lib  # noqa: F401

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("steps", [0, 1, 5])
@pytest.mark.parametrize("value", [INF, -INF, NAN, 3.3e38])  # the last one overflows in the momentum
@pytest.mark.parametrize("shape", [(300, 310), (310, 301), (40, 70), (90, 33), (1, 9), (1, 1)])
def test_all_of_it_and_none_else(shape, value, steps):
    t = _inputs([(280, 300), shape, (64, 50)], 3)
    good = _run(t, lr=0.1, steps=steps)
    t[1]["grad"][-1, shape[1] // 2] = value
    t[1]["momentum"][-1, shape[1] // 2] = value
    dev = _run(t, lr=0.1, steps=steps)
    for k in ("update", "param", "param_bf16"):
        assert dev[1][k].isnan().all(), k
        assert all(torch.equal(dev[i][k], good[i][k]) for i in (0, 2)), k


@pytest.mark.parametrize("steps", [0, 5])
def test_largest_finite_elements(steps):
    # u up to 3e38 is finite, and so is its norm in 64 bits
    t = _inputs([(300, 310), (40, 70)], 4)
    for x in t:
        x["grad"], x["momentum"] = 1.5e38 * x["grad"].sign(), 0.0 * x["momentum"]
    for d in _run(t, lr=0.1, steps=steps):
        assert all(d[k].isfinite().all() for k in ("update", "param", "param_bf16")) and d["update"].any()
