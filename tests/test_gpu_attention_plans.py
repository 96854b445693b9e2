"""How calls in which frames see each other are taken apart: heads that share keys in parts of unequal size, more workgroups than a launch takes."""
import numpy as np
import pytest
import torch

from paper_2304_13134_amd import binding as lb
from attention_oracle import rounded, whole_attention_grad
from layer_oracle import U32, assert_within, f64
from gpu_util import announce
from test_gpu_attention import inputs
from test_gpu_heads import dev, much_memory, spoil  # noqa: F401

pytestmark = pytest.mark.gpu

PARTS = [  # B, T, heads, kv_heads, width, left, right, sinks, kind, ragged, columns around; heads of a group and their parts
    (64, 200, 5, 1, 64, None, None, 0, "bf16", True, 0),       # 5 in 4
    (128, 200, 3, 1, 128, 20, 5, 7, "f16", True, 0),           # 3 in 2
    (45, 200, 7, 1, 24, 60, 0, 40, "bf16", False, 1),          # 7 in 5
    (22, 200, 14, 2, 64, 100, None, 3, "f16", True, 0),        # 7 in 5 of two groups
]


@pytest.mark.parametrize("case", PARTS, ids=str)
def test_parts_of_unequal_size(case):
    announce("unequal parts", case)
    q, k, v, dy, n, there, band = inputs(case)
    D, kind = case[4], case[8]
    y, lse = lb.last_attention(q, k, v, D, lengths=dev(n), **band)
    want = whole_attention_grad(*(f64(x) for x in (dy, q, k, v, y, lse)), D, n, *band.values(), D ** -0.5, kind)
    for x in (q, k, v, dy, y):
        spoil(x, there)
    got = lb.last_attention_grad(dy, q, k, v, y, lse, D, lengths=dev(n), **band)
    for x, (w, e), name in zip(got, want, ("dq", "dk", "dv")):
        assert_within(x, w, rounded(e, w, kind), name)


B, H, D = 130050, 65, 8                # 8453250 heads of frames, a workgroup each, of which a launch takes 2^23


def many(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(B, 1, H * D, generator=g, device="cuda").bfloat16() for _ in range(4)]


def heads(x):
    return x.double().view(B, 1, H, D)


def test_more_workgroups_than_a_launch_takes(much_memory):  # noqa: F811
    """Items of one frame, which sees itself alone: P = 1, so y = v and dv = dy to the bit (P's error of some 2^-20 is far below half a step), the
    logarithm is the score, and dq and dk are what is left of dP - delta, two sums of D products."""
    announce("many workgroups")
    q, k, v, dy = many(0)
    y, lse = lb.last_attention(q, k, v, D)
    assert torch.equal(y, v)
    score = (heads(q) * heads(k)).sum(-1) * D ** -0.5
    size = (heads(q) * heads(k)).abs().sum(-1) * D ** -0.5
    assert bool(((lse.double() - score).abs() <= 2 * (D + 2) * U32 * size + 4 * U32 * (score.abs() + 1) + 2.0 ** -21).all())
    dq, dk, dv = lb.last_attention_grad(dy, q, k, v, y, lse, D)
    assert torch.equal(dv, dy)
    dS = 2 * (D + 4) * U32 * (heads(dy) * heads(v)).abs().sum(-1, keepdim=True) * D ** -0.5 * (1 + 2.0 ** -8)
    for got, other in ((dq, k), (dk, q)):
        assert bool((heads(got).abs() <= dS * heads(other).abs() * (1 + 2.0 ** -7) + 1e-38).all())


def test_more_workgroups_of_a_cache_than_a_launch_takes(much_memory):  # noqa: F811
    """The same of streams of one frame."""
    announce("many workgroups of a cache")
    q, k, v, _ = many(1)
    pages = [torch.full((B, H, 1, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.randperm(B, device="cuda").to(torch.int32)[:, None].contiguous()
    cache = lb.Cache(*pages, table, torch.zeros(B, dtype=torch.int32, device="cuda"))
    lb.last_cache_append(k, v, cache)
    lb.check_item_status()
    for p, x in zip(pages, (k, v)):
        assert torch.equal(p[table[:, 0].long()].view(B, 1, H * D), x)
    y = lb.last_cached_attention(q, cache)
    lb.check_item_status()
    assert torch.equal(y, v)
