"""The workspace that noble_muon_step takes for itself comes from the memory of the stream that the
step runs on: on the host with the device's part replaced, and on a GPU with the current stream
writing to all the memory it is given while the step runs on another one."""
import contextlib

import pytest
import torch

from paper_2603_06492_gb300 import binding as B


class _Stream:
    cuda_stream = 77


@pytest.mark.parametrize("stream", [None, _Stream()])
def test_taken_on_the_stream_of_the_step(monkeypatch, stream):
    events, current = [], [None]

    @contextlib.contextmanager
    def on(s):
        before, current[0] = current[0], s
        yield
        current[0] = before

    class Workspace:
        is_cuda, dtype, device = True, torch.uint8, torch.device("cuda", 0)

        def is_contiguous(self):
            return True

        def data_ptr(self):
            return 0x1000

        def numel(self):
            return 256

    class Library:
        def noble_muon_step(self, arr, n, hp, ws, size, handle):
            events.append(("step", handle))
            return 0

    def workspace(tensors, precise=False):
        events.append(("workspace", current[0]))
        return Workspace()

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(B, "load", Library)
    monkeypatch.setattr(B, "muon_workspace", workspace)
    monkeypatch.setattr(B, "_muon_array", lambda tensors: None)
    monkeypatch.setattr(B, "_stream_handle", lambda s: getattr(s, "cuda_stream", 11))
    B.noble_muon_step([], 0.1, stream=stream)
    assert events == [("workspace", stream), ("step", 77 if stream else 11)] and current == [None]


@pytest.mark.gpu
@pytest.mark.parametrize("shapes", [[(300, 900), (70, 40)], [(100, 2000), (64, 64)]])
def test_memory_of_the_current_stream_stays_apart(shapes):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    g = torch.Generator(device="cuda").manual_seed(1)
    first = [{k: torch.randn(s, generator=g, device="cuda") for k in ("grad", "momentum", "param")} for s in shapes]
    copies = lambda: [{k: v.clone() for k, v in t.items()} for t in first]  # noqa: E731
    want = copies()
    B.noble_muon_step(want, 0.1)
    size = B.muon_workspace(want).numel()
    side, busy = torch.cuda.Stream(), torch.randn((4096, 4096), device="cuda")
    for _ in range(5):
        got = copies()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(10):  # the step waits behind this
                busy @ busy
        B.noble_muon_step(got, 0.1, stream=side)
        kept = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        assert all(torch.equal(a[k], b[k]) for a, b in zip(got, want) for k in b)
        assert all(bool((k == 255).all()) for k in kept)
    B.noble_get_device_status(None)
