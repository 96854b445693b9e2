"""What the binding does around a call with scratch memory, without a GPU: short calls are bound by it."""
import sys
import types

import pytest

from paper_2304_13134_amd import binding as lb
from test_scratch_host import HOST, cuda  # noqa: F401  (a fixture)


def functions_of_the_binding(f):
    """names of the binding's own functions that f() enters, in order"""
    seen = []

    def note(frame, event, _):
        if event == "call" and frame.f_code.co_filename == lb.__file__:
            seen.append(frame.f_code.co_name)
    sys.setprofile(note)
    try:
        f()
    finally:
        sys.setprofile(None)
    return seen


TENSOR = types.SimpleNamespace(get_device=lambda: 0, device=HOST)
CALLS = [(lb.OP_PRODUCT, ("frames", 3, 4, "a", "b")), (lb.OP_RESIDUAL_NORM_GRAD, ("frames", 1, 4, None, None)),
         (lb.OP_PRODUCT_GRAD_WEIGHT, ("frames", 3, 4, "a", "b")), (lb.OP_ATTENTION_GRAD, ("frames", "heads", "band", None)),
         (lb.OP_HEAD_NORM_GRAD, ("frames", "heads", None, None)), (lb.OP_CACHED_ATTENTION, ("frames", "heads", "band", "cache"))]


@pytest.mark.parametrize("op,sizes", CALLS)
def test_a_buffer_that_is_there(cuda, monkeypatch, op, sizes):  # noqa: F811
    """One function, no question for the size."""
    monkeypatch.setattr(lb, "load_library", lambda: pytest.fail("asked for the size"))
    kept = lb.workspace(1000, HOST)
    got = []

    def call(*arguments):
        got.append(arguments)
        return 0
    assert functions_of_the_binding(lambda: lb._with_scratch(call, op, *sizes, TENSOR)) == ["_with_scratch", "_check"]
    assert got == [(kept.data_ptr(), kept.numel(), 7)]


@pytest.mark.parametrize("op,sizes", CALLS)
def test_a_buffer_that_is_too_small(cuda, monkeypatch, op, sizes):  # noqa: F811
    """The call's own question for the size, with the call's arguments, and a second try with that much."""
    lb.workspace(300, HOST)
    asked, got = [], []
    monkeypatch.setattr(lb, "load_library", lambda: types.SimpleNamespace(
        last_layer_workspace_bytes=lambda *a: asked.append(("layer", *a)) or 5000,
        last_attention_workspace_bytes=lambda *a: asked.append(("attention", *a)) or 5000))

    def call(ws, nbytes, stream):
        got.append(nbytes)
        return 0 if nbytes >= 5000 else 5
    lb._with_scratch(call, op, *sizes, TENSOR)
    assert asked == [("attention" if op >= lb.OP_HEAD_NORM_GRAD else "layer", op, *sizes)]
    assert len(got) == 2 and got[0] < 5000 <= got[1]
