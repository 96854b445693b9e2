"""Whose memory the binding's scratch buffers are, without a GPU: the caching allocator's streams and captures are stand-ins."""
import types

import pytest
import torch

from paper_2304_13134_amd import binding as lb

HOST = torch.device("cpu")


@pytest.fixture
def cuda(monkeypatch):
    """Stream 7 of device 0, `state.capturing` to say whether it is; buffers are host memory."""
    state = types.SimpleNamespace(capturing=False)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state.capturing)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=7))
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: state.capturing, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 7, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(lb, "_workspaces", {})
    monkeypatch.setattr(lb, "_placement", {0: True})
    return state


def test_scratch_is_kept_and_grows(cuda):
    first = lb.workspace(1000, HOST)
    assert lb.workspace(500, HOST) is first
    second = lb.workspace(2000, HOST)
    assert second is not first and lb.workspace(2000, HOST) is second
    assert list(lb._workspaces.values()) == [second]


def test_a_capture_has_scratch_of_its_own(cuda):
    """A graph holds the addresses that it was captured with: they are the graph's own memory, not a buffer that a larger call
    outside of it replaces (and gives back to the allocator while replays go on writing there); and what came out of the
    graph's memory is not what calls outside of it are given."""
    kept = lb.workspace(1000, HOST)
    cuda.capturing = True
    inside = lb.workspace(500, HOST)
    assert inside is not kept
    larger = lb.workspace(4000, HOST)
    assert larger.numel() >= 4000 and list(lb._workspaces.values()) == [kept]
    cuda.capturing = False
    assert lb.workspace(1000, HOST) is kept
    assert lb.workspace(4000, HOST) is not larger


def test_layer_calls_under_capture(cuda, monkeypatch):
    """The same of the layer's calls, which try the buffer that is there first."""
    kept = lb.workspace(1000, HOST)
    used = []
    tensor = types.SimpleNamespace(get_device=lambda: 0, device=HOST)
    monkeypatch.setattr(lb, "load_library", lambda: types.SimpleNamespace(last_layer_workspace_bytes=lambda *a: 800))

    def call(ws, nbytes, stream):
        used.append((ws, nbytes))
        return 0
    lb._with_scratch(call, lb.OP_PRODUCT, None, 1, 1, None, None, tensor)
    assert used.pop() == (kept.data_ptr(), kept.numel())
    cuda.capturing = True
    lb._with_scratch(call, lb.OP_PRODUCT, None, 1, 1, None, None, tensor)
    ws, nbytes = used.pop()
    assert nbytes >= 800 and not kept.data_ptr() <= ws < kept.data_ptr() + kept.numel()
    assert list(lb._workspaces.values()) == [kept]
