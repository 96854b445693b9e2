"""Vectors of float32 that a gradient reads, without a GPU: where one is None the binding refuses the call.  (An address that stands for a tensor without
elements went to the kernel instead, which would have read there.)"""
import pytest
from torch._subclasses.fake_tensor import FakeTensorMode

import test_attention_host
import test_layer_devices_host
from test_layer_devices_host import devices  # noqa: F401  (a fixture)


@pytest.mark.parametrize("module,name,vector", [(test_attention_host, "last_attention_grad", "lse"), (test_layer_devices_host, "last_residual_norm_grad", "inv")])
def test_none_is_refused(devices, module, name, vector):  # noqa: F811
    with FakeTensorMode():
        f, arguments = module.calls(0)[name]
        f(**arguments)
        assert devices.launched.pop()[0] == name
        devices.launched.clear()
        with pytest.raises(TypeError, match=vector):
            f(**{**arguments, vector: None})
    assert not devices.launched
