"""Which device a layer's call runs on, without a GPU: operands are stand-ins that know a device index."""
import contextlib
import types

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2304_13134_amd import binding as lb


@pytest.fixture
def devices(monkeypatch):
    """Three devices, of which `state.current` is the current one; each one's current stream is the default one, whose handle is 0."""
    state = types.SimpleNamespace(current=0, launched=[])

    @contextlib.contextmanager
    def on(index):
        before, state.current = state.current, index
        yield
        state.current = before
    monkeypatch.setattr(torch.cuda, "device", on)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: state.current)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=0))
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: False, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: state.current, raising=False)
    monkeypatch.setattr(lb, "_workspaces", {(2, 0): torch.empty(4096, dtype=torch.uint8)})
    monkeypatch.setattr(torch.Tensor, "data_ptr", lambda t: 0x10000)

    def library():
        return types.SimpleNamespace(**{name: lambda *a, name=name: state.launched.append((name, state.current)) or 0
                                        for name in lb.EXPORTS if name != "last_status_string"})
    monkeypatch.setattr(lb, "load_library", library)
    return state


def calls(dev):
    """Every call of the layer, on operands of device `dev` but for one of them on `off`."""
    bf, kind = torch.bfloat16, {"device": "cuda:%d" % dev}
    x, w, dy = torch.empty(4, 6, 64, dtype=bf, **kind), torch.empty(40, 64, dtype=bf, **kind), torch.empty(4, 6, 40, dtype=bf, **kind)
    lengths, gain, inv, bias = (torch.empty(4, dtype=torch.int32, **kind), torch.empty(64, **kind), torch.empty(4, 6, **kind), torch.empty(40, **kind))
    kept = lb.Kept(torch.empty(4, 6, 64, dtype=torch.int8, **kind), torch.empty(4, 6, 2, dtype=torch.uint8, **kind))
    return {
        "last_residual_norm": (lb.last_residual_norm, dict(x=x, gain=gain, residual=x, lengths=lengths)),
        "last_residual_norm_grad": (lb.last_residual_norm_grad, dict(dy=x, s=kept, gain=gain, inv=inv, ds=x, lengths=lengths)),
        "last_product": (lb.last_product, dict(x=x, w=w, bias=bias, residual=dy, lengths=lengths)),
        "last_product_grad_input": (lb.last_product_grad_input, dict(dy=dy, w=w, kept=kept, activation="silu", lengths=lengths)),
        "last_product_grad_weight": (lb.last_product_grad_weight, dict(dy=dy, x=kept, activation="silu", lengths=lengths)),
        "last_keep": (lb.last_keep, dict(x=x, lengths=lengths)),
        "last_kept_values": (lb.last_kept_values, dict(kept=kept, lengths=lengths)),
        "last_kept_grad": (lb.last_kept_grad, dict(dy=x, kept=kept, activation="silu", lengths=lengths)),
    }


NAMES = ["last_residual_norm", "last_residual_norm_grad", "last_product", "last_product_grad_input", "last_product_grad_weight", "last_keep",
         "last_kept_values", "last_kept_grad"]


@pytest.mark.parametrize("name", NAMES)
def test_calls_run_on_their_tensors_device(devices, name):
    """Handle 0 is the default stream of the current device: the tensors' device has to be that."""
    with FakeTensorMode():
        call, arguments = calls(2)[name]
        call(**arguments)
    assert devices.launched == [(name, 2)] and devices.current == 0


@pytest.mark.parametrize("name", NAMES)
def test_operands_of_two_devices_are_refused(devices, name):
    with FakeTensorMode():
        call, arguments = calls(2)[name]
        others = calls(1)[name][1]
        for k, v in arguments.items():
            if isinstance(v, str) or len([a for a in arguments.values() if not isinstance(a, str)]) == 1:
                continue
            with pytest.raises(ValueError):
                call(**dict(arguments, **{k: others[k]}))
            if isinstance(v, lb.Kept):                              # codes and scales apart
                with pytest.raises(ValueError):
                    call(**dict(arguments, **{k: lb.Kept(v[0], others[k][1])}))
    assert not devices.launched
