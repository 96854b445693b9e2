"""Frames that do not exist are zeros in every result of the heads' norms, whatever stands in their place and in the parameters."""
import numpy as np
import pytest
import torch

from paper_2304_13134_amd import binding as lb
from gpu_util import announce
from test_gpu_heads import dev, draw, spoil

pytestmark = pytest.mark.gpu
BAD = [float("nan"), float("inf"), float("-inf")]


def bad_parameters(rng, D, bad, which):
    """(gain, frequencies) of which one element of the named one is `bad`"""
    gain, f = dev(1 + 0.2 * rng.standard_normal(D), torch.float32), dev(0.9 ** np.arange(D // 2), torch.float32)
    (gain if which == "gain" else f)[3] = bad
    return gain, f


@pytest.mark.parametrize("which", ["gain", "frequency"])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("kind,T,D", [("f32", 9, 40), ("bf16", 70, 64), ("f16", 3, 128), ("bf16", 5000, 16)])
def test_norm_and_gradient(kind, T, D, bad, which):
    announce("absent frames", kind, T, D, bad, which)
    rng = np.random.default_rng(T + D)
    B, H, G = 3, 3, 1
    n = np.array([T, T // 2, 0])
    there = np.arange(T)[None] < n[:, None]
    q, k, dq, dk = (spoil(draw(rng, (B, T, c * D), kind), there) for c in (H, G, H, G))
    gain, f = bad_parameters(rng, D, bad, which)
    gone = torch.from_numpy(~there).cuda()
    for rotation in (f, lb.Rotation(f, dev([7, 0, 100000]))):
        for gains in ((gain, gain), (gain, None), (None, None)):
            args = (D, *gains, rotation, dev(n))
            for x in (*lb.last_head_norm(q, k, *args), *lb.last_head_norm_grad(dq, dk, q, k, *args)[:2]):
                assert not x[gone].any()


@pytest.mark.parametrize("which", ["gain", "frequency"])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("T", [4, 600])
def test_queries_beside_a_cache(T, bad, which):
    announce("absent queries", T, bad, which)
    rng = np.random.default_rng(T)
    B, H, G, D, page = 2, 4, 2, 64, 16
    n = np.array([T - 1, 0])
    there = np.arange(T)[None] < n[:, None]
    q, k, v = (spoil(draw(rng, (B, T, c * D), "bf16"), there) for c in (H, G, G))
    gain, f = bad_parameters(rng, D, bad, which)
    entries = -(-T // page)
    pages = [torch.zeros(B * entries, G, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = lb.Cache(*pages, dev(np.arange(B * entries).reshape(B, entries)), dev([0, 0]))
    yq = lb.last_cache_append(k, v, cache, q=q, gain_q=gain, gain_k=gain, frequencies=f, lengths=dev(n))
    lb.check_item_status()
    assert not yq[torch.from_numpy(~there).cuda()].any()
    assert not pages[0][entries:].any() and not pages[0][entries - 1, :, n[0] - (entries - 1) * page:].any()
