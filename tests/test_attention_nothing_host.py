"""What the binding says to calls in which frames see each other that lack an operand: the errors of the other calls."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2304_13134_amd import binding as lb
from test_attention_host import NAMES, calls
from test_layer_devices_host import devices  # noqa: F401  (a fixture)

MAY_BE_NONE = {"last_head_norm": {"gain_q", "gain_k", "rotation", "lengths", "q", "k"}, "last_attention": {"lengths"},
               "last_head_norm_grad": {"gain_q", "gain_k", "rotation", "lengths", "dyq", "dyk"}, "last_attention_grad": {"lengths"},
               "last_cache_append": {"q", "gain_q", "gain_k", "frequencies", "lengths", "item_status"},
               "last_cached_attention": {"lengths", "item_status"}}


@pytest.mark.parametrize("name", NAMES)
def test_missing_operands(devices, name):  # noqa: F811
    with FakeTensorMode():
        f, arguments = calls(0)[name]
        for key in arguments:
            if key == "width" or key in MAY_BE_NONE[name]:
                continue
            for bad in (None, 3, "x"):
                with pytest.raises((TypeError, ValueError)):
                    f(**{**arguments, key: bad})
        for pair in (("q", "k"), ("dyq", "dyk")):
            if name.startswith("last_head_norm") and pair[0] in arguments and pair[0] in MAY_BE_NONE[name]:
                with pytest.raises((TypeError, ValueError)):
                    f(**{**arguments, pair[0]: None, pair[1]: None})
    assert not devices.launched


@pytest.mark.parametrize("name", ["last_cache_append", "last_cached_attention"])
def test_what_is_no_cache(devices, name):  # noqa: F811
    with FakeTensorMode():
        f, arguments = calls(0)[name]
        c = arguments["cache"]
        for bad in ((), c[:3], tuple(c) + (None,), (None, c.v, c.table, c.used), (c.k[0], c.v, c.table, c.used), (c.k, None, c.table, c.used),
                    (c.k, c.v, None, c.used), (c.k, c.v, c.table, None), (c.k[:, :0], c.v[:, :0], c.table, c.used), torch.empty(4, device="cuda:0")):
            with pytest.raises((TypeError, ValueError)):
                f(**{**arguments, "cache": bad})
        q = torch.empty((), dtype=torch.bfloat16, device="cuda:0")
        with pytest.raises((TypeError, ValueError)):
            f(**{**arguments, "q": q})
    assert not devices.launched
