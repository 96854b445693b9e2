"""Products of 8-bit operands with a result in 32 bits: their terms are added in 32 bits."""
import numpy as np
import pytest
import torch

from paper_2304_13134_amd import binding as lb
from layer_oracle import EIGHT, U32, act, assert_kept, assert_within, decode, exists, f64, rounding
from gpu_util import announce
from test_gpu_layer import dev_lengths, draw, lengths_of, spoil, zeros_where

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
# rows on both sides of what the kernels take, reductions that end inside a block, a step, or go in shares
SHAPES = [(1, 1, 1, 1), (1, 1, 7, 3), (2, 8, 17, 33), (1, 17, 257, 512), (3, 21, 65, 129), (1, 64, 48, 200), (1, 65, 33, 64), (3, 100, 257, 512),
          (1, 40, 64, 4100), (1, 130, 96, 5000), (16, 70, 300, 96), (4, 1025, 1030, 160), (1, 4, 16500, 64)]


@pytest.mark.parametrize("B,T,N,K", SHAPES)
@pytest.mark.parametrize("name,bias,res,keep,lens", [("none", False, False, None, "all"), ("silu", True, True, None, "some"), ("gelu", True, False, "i8", "some")])
def test_float32_results_of_eight_bit_operands(B, T, N, K, name, bias, res, keep, lens):
    """Products of codes are exact in float32 and their sums are within K 2^-24 of the terms' magnitudes, like those of 16-bit operands;
    the operands' blocks are of unlike scales, within and across, so that terms drop out of any narrower sum."""
    announce("float32 result of 8-bit operands", B, T, N, K, name, bias, res, keep, lens)
    rng = np.random.default_rng(B * T + N + K)
    spread = torch.from_numpy(np.exp2(rng.integers(-9, 1, K)).astype(np.float32)).cuda()
    x = lb.last_keep(draw(rng, (B, T, K), "f32") * spread, E4M3)
    w = lb.last_keep(draw(rng, (N, K), "f32", K ** -0.5) / spread, E4M3)
    n = lengths_of(lens, B, T, rng)
    there = exists(B, T, n)
    b, r = draw(rng, (N,), "f32", 0.3) if bias else None, draw(rng, (B, T, N), "f32") if res else None
    xv, wv = zeros_where(decode(x), there), decode(w)
    bv, rv = (f64(b) if bias else 0), (f64(r) if res else np.zeros((B, T, N)))
    h = zeros_where(xv @ wv.T + bv, there)
    e_h = (K + 4) * U32 * (np.abs(xv) @ np.abs(wv).T + np.abs(bv))
    y = zeros_where(act(h, name) + rv, there)
    e_y = 1.13 * e_h + 4e-6 * np.abs(act(h, name)) * (name != "none") + 2e-7 * (name != "none") + 2 * U32 * np.abs(y)
    spoil(x, there)
    if res:
        spoil(r, there)
    got, kept = lb.last_product(x, w, bias=b, activation=name, residual=r, lengths=dev_lengths(n), dtype=torch.float32, keep=EIGHT.get(keep))
    there = there[..., None]
    assert_within(got, y, np.where(there, e_y, 0) + rounding(y, "f32"), "y")
    if keep:
        assert_kept(kept, h, np.where(there, e_h, 0), keep, "kept")


def test_cancelling_terms_of_a_block():
    """Two large terms that cancel beside thirty small ones of the same block, 2^-14 of them and less: the small ones are the sum."""
    announce("cancelling terms of a block")
    for rows in (3, 100):
        x, w = torch.zeros(rows, 64, device="cuda"), torch.zeros(40, 64, device="cuda")
        x[:, 0], x[:, 1], x[:, 2:32] = 1.0, -1.0, 2.0 ** -9
        w[:, 0], w[:, 1], w[:, 2:32] = 1.0, 1.0, 2.0 ** -6
        y = lb.last_product(lb.last_keep(x, E4M3), lb.last_keep(w, E4M3), dtype=torch.float32)[0]
        assert torch.equal(y, torch.full((rows, 40), 30 * 2.0 ** -15, device="cuda"))


@pytest.mark.parametrize("rows", [5, 100, 2000])
def test_blocks_that_are_no_numbers(rows):
    rng = np.random.default_rng(8)
    announce("NaN blocks in wide products", rows)
    x = draw(rng, (rows, 160), "f32")
    w = lb.last_keep(draw(rng, (600, 160), "f32"), E4M3)
    good = lb.last_product(lb.last_keep(x, E4M3), w, dtype=torch.float32)[0]
    x[3, 70] = float("nan")
    bad = lb.last_product(lb.last_keep(x, E4M3), w, dtype=torch.float32)[0]
    keep = [r for r in range(rows) if r != 3]
    assert torch.isnan(bad[3]).all() and torch.equal(bad[keep], good[keep])


@pytest.mark.parametrize("rows", [5, 100])
@pytest.mark.parametrize("scale", [2.0 ** -100, 2.0 ** 100])
def test_small_and_large_scales(rows, scale):
    """Scales near the ends of what bfloat16 holds: the sums of the operands at scale 1, exactly, times the scale."""
    rng = np.random.default_rng(9)
    announce("scales of wide products", rows, scale)
    x, w = draw(rng, (rows, 96), "f32"), lb.last_keep(draw(rng, (50, 96), "f32"), E4M3)
    want = lb.last_product(lb.last_keep(x, E4M3), w, dtype=torch.float32)[0] * scale
    assert torch.equal(lb.last_product(lb.last_keep(x * scale, E4M3), w, dtype=torch.float32)[0], want)


def test_smallest_codes():
    """Values down to bfloat16's smallest subnormal number are multiplied as they are."""
    announce("smallest codes")
    for e in (-125, -127, -130, -133):
        for rows in (3, 100):
            x, w = torch.zeros(rows, 32, device="cuda"), torch.zeros(40, 32, device="cuda")
            x[:, 0], w[:, 0] = 2.0 ** e, 2.0 ** 100
            y = lb.last_product(lb.last_keep(x, E4M3), lb.last_keep(w, E4M3), dtype=torch.float32)[0]
            assert torch.equal(y, torch.full((rows, 40), 2.0 ** (e + 100), device="cuda")), e
