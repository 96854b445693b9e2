"""A batch without items, with lengths and without: nothing to write but the sums over frames, which are zeros."""
import pytest
import torch

from paper_2304_13134_amd import binding as lb
from gpu_util import announce

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ragged", [False, True])
def test_no_items(ragged):
    announce("no items", ragged)
    x, dy = torch.empty(0, 7, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 7, 40, dtype=torch.bfloat16, device="cuda")
    w, gain = torch.ones(40, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(64, device="cuda")
    lengths = torch.empty(0, dtype=torch.int32, device="cuda") if ragged else None
    fw = lb.last_residual_norm(x, gain, residual=x, lengths=lengths, keep=torch.int8, dtype=torch.bfloat16)
    assert fw.y.shape == x.shape and fw.inv.shape == (0, 7) and fw.kept[1].shape == (0, 7, 2)
    y, kept = lb.last_product(x, w, lengths=lengths, keep=torch.int8)
    assert y.shape == (0, 7, 40) and kept[0].shape == y.shape
    assert lb.last_product_grad_input(dy, w, lengths=lengths).shape == x.shape
    for given in (x, fw.kept):
        dw, db = lb.last_product_grad_weight(dy, given, lengths=lengths)
        assert dw.shape == w.shape and not dw.any() and not db.any()
    dx, dgain = lb.last_residual_norm_grad(x, x, gain, fw.inv, lengths=lengths)
    assert dx.shape == x.shape and not dgain.any()
    assert lb.last_kept_grad(x, lb.last_keep(x, lengths=lengths), "silu", lengths=lengths).shape == x.shape
    assert lb.last_kept_values(fw.kept, "silu", lengths=lengths).shape == x.shape
