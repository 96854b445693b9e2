"""Results of the layer at the last bit, and at the ends of what their types hold."""
import numpy as np
import pytest
import torch

from paper_2304_13134_amd import binding as lb
from layer_oracle import EIGHT, assert_within, decode, encode, f64
from gpu_util import announce

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("R,H", [(5, 31), (3, 512), (7, 2048), (2, 4100), (2, 9000)])
def test_float32_norm_beside_codes_is_rounded_to_nearest(R, H, kind):
    """A row beside its codes is formed in 64 bits: float32 results are within half a unit of the exact row, and 2^-16 of a unit for what
    64 bits and the order of the sum leave."""
    announce("float32 norm beside codes", R, H, kind)
    rng = np.random.default_rng(H)
    x, r, gain = (rng.standard_normal(n).astype(np.float32) for n in ((R, H), (R, H), (H,)))
    eps = float(np.float32(1e-5))
    s = x.astype(np.float64) + r
    want = s / np.sqrt((s * s).mean(-1, keepdims=True) + eps) * gain
    dev = [torch.from_numpy(v).cuda() for v in (x, gain, r)]
    got = lb.last_residual_norm(dev[0], dev[1], residual=dev[2], eps=eps, dtype=torch.float32, keep=EIGHT[kind])
    unit = np.exp2(np.frexp(np.abs(want))[1].astype(float) - 24)
    assert_within(got.y, want, unit * (0.5 + 2.0 ** -16), "y")


def test_float32_norm_beside_codes_overflows():
    """A result that passes the largest float32 is an infinity, with codes as without, and its block stands for NaN."""
    announce("norm that overflows")
    x = torch.ones(2, 64, device="cuda")
    x[0, 3], x[1, 40] = 7.0, -7.0
    gain = torch.ones(64, device="cuda")
    gain[3] = gain[40] = 2e38
    plain = lb.last_residual_norm(x, gain, eps=0.0).y.cpu()
    got = lb.last_residual_norm(x, gain, eps=0.0, dtype=torch.float32, keep=torch.int8)
    y = got.y.cpu()
    assert y[0, 3] == INF and y[1, 40] == -INF and torch.equal(torch.isinf(y), torch.isinf(plain))
    assert torch.allclose(y[torch.isfinite(y)], plain[torch.isfinite(plain)], rtol=1e-6)
    k = decode(got.kept)
    assert np.array_equal(np.isnan(k), np.repeat([[True, False], [False, True]], 32, -1))
    for t in (torch.bfloat16, torch.float16):
        assert torch.equal(torch.isinf(lb.last_residual_norm(x, gain, eps=0.0, dtype=t, keep=torch.int8).y),
                           torch.isinf(lb.last_residual_norm(x, gain, eps=0.0, dtype=t).y))


@pytest.mark.parametrize("type_", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("where", ["x", "residual", "sum"])
def test_infinite_sums_beside_codes(type_, where):
    """An infinity in x or in the residual, or a sum that passes the type's largest number in 32 bits: NaN in its own place and zeros
    in the rest of the row, whose inverse root mean square is 0, with codes as without; the codes' other blocks stand for zeros."""
    announce("infinite sums beside codes", type_, where)
    x, r = torch.ones(4, 96, device="cuda", dtype=type_), torch.full((4, 96), 0.5, device="cuda", dtype=type_)
    if where == "sum":
        if type_ == torch.float16:
            pytest.skip("sums of float16 stay below the largest float32")
        x[2, 40] = r[2, 40] = 3e38
    else:
        (x if where == "x" else r)[2, 40] = -INF
    gain = torch.full((96,), 2.0, device="cuda")
    plain = lb.last_residual_norm(x, gain, residual=r, dtype=torch.float32)
    got = lb.last_residual_norm(x, gain, residual=r, dtype=torch.float32, keep=torch.int8)
    assert float(got.inv[2]) == float(plain.inv[2]) == 0.0
    for y in (plain.y.cpu(), got.y.cpu()):
        assert torch.isnan(y[2, 40]) and int(torch.isnan(y).sum()) == 1
        assert not y[2, :40].any() and not y[2, 41:].any()
    assert torch.equal(got.s.isinf(), plain.s.isinf()) and bool(got.s[2, 40].isinf())
    k = decode(got.kept)
    assert np.isnan(k[2, 32:64]).all() and not k[2, :32].any() and not k[2, 64:].any() and np.isfinite(k[[0, 1, 3]]).all()
