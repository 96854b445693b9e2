"""Attention over a band of frames and its gradient against plain float64 forms (attention_oracle.py, which derives the bounds)."""
import numpy as np
import pytest
import torch

from paper_2304_13134_amd import binding as lb
from attention_oracle import frames_there, rounded, whole_attention, whole_attention_grad
from layer_oracle import assert_within, f64
from gpu_util import announce
from test_gpu_heads import dev, draw, much_memory, some_lengths, spoil  # noqa: F401

pytestmark = pytest.mark.gpu

CASES = [  # B, T, heads, kv_heads, width, left, right, sinks, kind, ragged, columns around
    (1, 1, 1, 1, 8, None, 0, 0, "bf16", False, 0),
    (3, 2, 2, 1, 64, None, None, 0, "f16", True, 0),
    (2, 31, 2, 2, 40, None, 0, 0, "bf16", True, 0),
    (2, 33, 4, 2, 64, 0, 0, 0, "bf16", False, 0),
    (1, 64, 1, 1, 128, 5, 3, 2, "f16", False, 0),
    (2, 65, 3, 1, 72, 7, 0, 1, "bf16", True, 3),
    (1, 127, 2, 2, 32, None, None, 0, "f16", False, 1),
    (2, 129, 4, 1, 128, 20, 10, 33, "bf16", True, 8),
    (3, 200, 6, 2, 64, 64, 64, 64, "f16", True, 5),
    (1, 300, 2, 1, 96, 31, 0, 4, "bf16", False, 0),
    (2, 321, 8, 8, 16, 130, None, 3, "bf16", True, 0),
    (1, 640, 4, 2, 128, None, 0, 0, "f16", False, 0),
    (1, 700, 2, 1, 64, 40, 7, 17, "bf16", False, 0),
    (2, 1300, 2, 2, 24, 10, 1, 40, "f16", True, 0),
    (1, 2600, 2, 1, 64, 3, 0, 64, "bf16", False, 0),
    (1, 513, 2, 2, 128, 1000, 1000, 5, "bf16", False, 0),
]


def inputs(case, seed=0):
    B, T, H, G, D, left, right, sinks, kind, ragged, around = case
    rng = np.random.default_rng(T * 31 + D + seed)
    n = some_lengths(rng, B, T, ragged)
    _, there = frames_there(B, T, n)
    q, k, v, dy = (draw(rng, (B, T, c * D), kind, s, around, around) for c, s in ((H, 1.3), (G, 1.3), (G, 1.0), (H, 1.0)))
    return q, k, v, dy, n, there, {"left": left, "right": right, "sinks": sinks}


@pytest.mark.parametrize("case", CASES, ids=str)
def test_attention(case):
    announce("attention", case)
    q, k, v, _, n, there, band = inputs(case)
    D, kind = case[4], case[8]
    want, e, L, eL = whole_attention(f64(q), f64(k), f64(v), D, n, *band.values(), D ** -0.5, kind)
    for x in (q, k, v):
        spoil(x, there)
    y, lse = lb.last_attention(q, k, v, D, lengths=dev(n), **band)
    assert_within(lse, L, eL, "lse")
    assert_within(y, want, rounded(e, want, kind), "y")


@pytest.mark.parametrize("case", CASES, ids=str)
def test_attention_gradient(case):
    announce("attention gradient", case)
    q, k, v, dy, n, there, band = inputs(case)
    D, kind = case[4], case[8]
    y, lse = lb.last_attention(q, k, v, D, lengths=dev(n), **band)
    want = whole_attention_grad(*(f64(x) for x in (dy, q, k, v, y, lse)), D, n, *band.values(), D ** -0.5, kind)
    for x in (q, k, v, dy, y):
        spoil(x, there)
    got = lb.last_attention_grad(dy, q, k, v, y, lse, D, lengths=dev(n), **band)
    for x, (w, e), name in zip(got, want, ("dq", "dk", "dv")):
        assert_within(x, w, rounded(e, w, kind), name)
    out = tuple(torch.full_like(x, 3.0) for x in (q, k, v))
    assert all(torch.equal(a, b) for a, b in zip(lb.last_attention_grad(dy, q, k, v, y, lse, D, lengths=dev(n), out=out, **band), got))


@pytest.mark.parametrize("scale", [1e-3, 3.0])
def test_scales_and_large_scores(scale):
    """Scores of a few hundred, whose maximum grows from tile to tile, and nearly equal ones."""
    case = (1, 400, 2, 1, 64, None, None, 0, "bf16", False, 0)
    announce("large scores", scale)
    q, k, v, dy, n, there, band = inputs(case)
    k *= torch.linspace(0.1, 3.0, 400, device="cuda")[:, None].bfloat16()
    want, e, L, eL = whole_attention(f64(q), f64(k), f64(v), 64, n, *band.values(), scale, "bf16")
    y, lse = lb.last_attention(q, k, v, 64, scale=scale, **band)
    assert_within(lse, L, eL, "lse")
    assert_within(y, want, rounded(e, want, "bf16"), "y")
    want = whole_attention_grad(*(f64(x) for x in (dy, q, k, v, y, lse)), 64, n, *band.values(), scale, "bf16")
    got = lb.last_attention_grad(dy, q, k, v, y, lse, 64, scale=scale, **band)
    for x, (w, e), name in zip(got, want, ("dq", "dk", "dv")):
        assert_within(x, w, rounded(e, w, "bf16"), name)


MANY = [  # of more than 512 workgroups of 128 frames, which have one wavefront for 32 frames
    (44, 300, 4, 2, 64, None, None, 0, "f16", True, 0),
    (70, 260, 4, 1, 40, 100, 20, 5, "bf16", True, 1),
    (66, 520, 2, 1, 128, 300, 0, 3, "bf16", True, 0),
    (130, 400, 1, 1, 24, None, 0, 0, "f16", False, 0),
]


@pytest.mark.parametrize("grows", [0.0, 3.0])
@pytest.mark.parametrize("case", MANY, ids=str)
def test_many_workgroups(case, grows):
    """Also with scores that pass the ones before them by more than what sums are kept relative to, again and again."""
    announce(case, grows)
    q, k, v, dy, n, there, band = inputs(case)
    if grows:
        k *= torch.linspace(0.1, grows, case[1], device="cuda")[:, None].to(k.dtype)
    D, kind, scale = case[4], case[8], 2.0 if grows else case[4] ** -0.5
    want, e, L, eL = whole_attention(f64(q), f64(k), f64(v), D, n, *band.values(), scale, kind)
    for x in (q, k, v):
        spoil(x, there)
    y, lse = lb.last_attention(q, k, v, D, lengths=dev(n), scale=scale, **band)
    assert_within(lse, L, eL, "lse")
    assert_within(y, want, rounded(e, want, kind), "y")
    for x in (q, k, v):
        x[torch.from_numpy(~there).cuda()] = 0
    want = whole_attention_grad(*(f64(x) for x in (dy, q, k, v, y, lse)), D, n, *band.values(), scale, kind)
    for x in (q, k, v, dy, y):
        spoil(x, there)
    got = lb.last_attention_grad(dy, q, k, v, y, lse, D, lengths=dev(n), scale=scale, **band)
    for x, (w, e), name in zip(got, want, ("dq", "dk", "dv")):
        assert_within(x, w, rounded(e, w, kind), name)


@pytest.mark.parametrize("B", [2, 70])
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_a_bad_key_that_many_see(B, bad):
    """A frame of item 1 with a NaN or an infinity in its key, in a tile that others see whole: theirs are NaN, or what they are without it where the
    score is -inf; other items' results are what they are."""
    case = (B, 400, 2, 1, 64, 200, 50, 0, "bf16", False, 0)
    announce("bad key", B, bad)
    q, k, v, _, n, there, band = inputs(case)
    y0, l0 = lb.last_attention(q, k, v, 64, **band)
    k[1, 130, 7] = float(bad)
    y, lse = lb.last_attention(q, k, v, 64, **band)
    one = torch.ones(B, dtype=torch.bool, device="cuda")
    one[1] = False
    assert torch.equal(y[one], y0[one]) and torch.equal(lse[one], l0[one])
    t = torch.arange(400, device="cuda")
    sees = (130 <= t + 50) & (130 >= t - 200)
    assert torch.equal(lse[1, ~sees], l0[1, ~sees]) and torch.equal(y[1, ~sees], y0[1, ~sees])
    heads = torch.isnan(y[1].view(400, 2, 64)).any(-1)
    assert torch.equal(heads, torch.isnan(y[1].view(400, 2, 64)).all(-1)) and torch.equal(heads, torch.isnan(lse[1]))
    assert bool(heads[sees].all()) if bad == "nan" else bool((heads[sees] == (q[1, sees].view(-1, 2, 64)[:, :, 7] >= 0)).all())


@pytest.mark.parametrize("B", [1, 150])
def test_scores_of_minus_infinity_first(B):
    """Three tiles of keys whose scores are -inf, which have no part, before scores that are far below zero: the others' result, as when they are alone."""
    announce("-inf first", B)
    T, D, none = 400, 64, 192
    q, k, v, _, n, _, _ = inputs((B, T, 1, 1, D, None, None, 0, "bf16", False, 0))
    q[..., 7], q[..., 8], k[:, :none, 7], k[:, none:, 7], k[:, :, 8] = 1, 4, float("-inf"), 0, -100
    y, lse = lb.last_attention(q, k, v, D, right=None, scale=1.0)
    some = T - none
    want, e, L, eL = whole_attention(f64(q[:1, :some]), f64(k[:1, none:]), f64(v[:1, none:]), D, n, None, None, 0, 1.0, "bf16")
    assert_within(lse[:1, :some], L, eL, "lse")
    assert_within(y[:1, :some], want, rounded(e, want, "bf16"), "y")
    assert bool(torch.isfinite(y).all()) and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("bad", ["nan value", "nan key", "inf value", "inf key"])
@pytest.mark.parametrize("width", [40, 128])
def test_what_is_not_seen_has_no_part(bad, width):
    """A frame with infinities or NaN: the frames that do not see it have the results that they have without it, the others NaN (or,
    an infinite value seen with a positive probability, that infinity)."""
    B, T, H, G, D = 2, 300, 2, 1, width
    announce("not seen", bad, width)
    case = (B, T, H, G, D, 20, 4, 3, "bf16", False, 0)
    q, k, v, _, n, there, band = inputs(case)
    want, e, L, eL = whole_attention(f64(q), f64(k), f64(v), D, n, *band.values(), D ** -0.5, "bf16")
    t = k if "key" in bad else v
    at = [1, 150, 290]
    for s in at:
        t[0, s, 5] = float("nan") if "nan" in bad else float("inf")
    y, lse = lb.last_attention(q, k, v, D, **band)
    sees = np.zeros((B, T), bool)
    for s in at:
        i = np.arange(T)
        sees[0] |= (s <= i + 4) & ((s >= i - 20) | (s < 3))
    y, lse = f64(y), f64(lse)
    assert_within(y[~sees], want[~sees], rounded(e, want, "bf16")[~sees], "y")
    assert_within(lse[~sees], L[~sees], eL[~sees], "lse")
    if "key" in bad:
        heads = np.broadcast_to(np.isnan(lse)[..., None], (B, T, H, D)).reshape(B, T, -1)
        if bad == "nan key":
            assert np.isnan(y[sees]).all() and heads[sees].all()
        else:                                          # +inf: NaN; -inf: the frame has no part
            assert (np.isnan(y) == heads).all() and heads[sees].any()
    else:
        assert not np.isfinite(y.reshape(B, T, H, D)[sees][..., 5]).any()
        others = np.delete(y.reshape(B, T, H, D)[sees], 5, -1)
        assert np.isfinite(others).all()


def test_gradient_against_differences():
    """Of sum(c y) in float16: differences of results rounded by 2^-11 each, over steps of 2^-4, in 2000 directions at once."""
    announce("attention differences")
    case = (2, 70, 4, 2, 32, 15, 6, 4, "f16", True, 0)
    q, k, v, c, n, there, band = inputs(case)
    lengths, D = dev(n), 32
    c.mul_(torch.from_numpy(there).cuda()[..., None])

    def value(*x):
        y, _ = lb.last_attention(*x, D, lengths=lengths, **band)
        return float((y.double() * c.double()).sum())
    y, lse = lb.last_attention(q, k, v, D, lengths=lengths, **band)
    grads = lb.last_attention_grad(c, q, k, v, y, lse, D, lengths=lengths, **band)
    rng = np.random.default_rng(1)
    for i, g in enumerate(grads):
        x = (q, k, v)[i]
        d = draw(rng, tuple(x.shape), "f16", 1.0)
        up, down = ((x.double() + s * d.double() / 16).half() for s in (1, -1))
        step = (up.double() - down.double()) / 2                      # (as rounded)
        args = [q, k, v]
        got = (value(*args[:i], up, *args[i + 1:]) - value(*args[:i], down, *args[i + 1:])) / 2
        # results' roundings, independent: 2^-11 sqrt(sum c^2 y^2), four deviations of the difference of two; P's add as much; the
        # third derivative of softmax along a step of score size 1/16 leaves 2^-8 of the sum's terms; gradients' roundings 2^-11 of theirs
        noise = 4 * 2.0 ** -11 * 2 * float((c.double() * y.double()).square().sum().sqrt())
        size = float((g.double().abs() * step.abs()).sum())
        assert abs(got - float((g.double() * step).sum())) <= noise + 2.0 ** -8 * size, (i, got, float((g.double() * step).sum()), noise, size)


def test_columns_of_one_matrix():
    """Queries, keys and values as a product's columns, gradients to columns of one matrix; one item without lengths as [T, columns]."""
    announce("one matrix")
    rng = np.random.default_rng(8)
    T, H, G, D = 150, 4, 2, 64
    qkv = draw(rng, (T, (H + 2 * G) * D), "bf16")
    q, k, v = qkv.split([H * D, G * D, G * D], -1)
    y, lse = lb.last_attention(q, k, v, D, left=30)
    assert y.shape == (T, H * D) and lse.shape == (T, H)
    y3, lse3 = lb.last_attention(*(t.contiguous()[None] for t in (q, k, v)), D, left=30)
    assert torch.equal(y, y3[0]) and torch.equal(lse, lse3[0])
    dy = draw(rng, (T, H * D), "bf16")
    d = lb.last_attention_grad(dy, q, k, v, y, lse, D, left=30)
    whole = d[0]._base
    assert whole.shape == (T, (H + 2 * G) * D) and torch.equal(whole, torch.cat(d, -1))


def test_no_frames():
    announce("attention without frames")
    for B, T in ((0, 5), (3, 0)):
        q = torch.empty(B, T, 128, dtype=torch.bfloat16, device="cuda")
        n = torch.zeros(B, dtype=torch.int32, device="cuda")
        y, lse = lb.last_attention(q, q, q, 64, lengths=n)
        assert y.shape == q.shape and lse.shape == (B, T, 2)
        assert [g.shape for g in lb.last_attention_grad(q, q, q, q, y, lse, 64, lengths=n)] == [q.shape] * 3
        assert lb.last_head_norm(q, q, 64, lengths=n)[1].shape == q.shape
        g = torch.ones(64, device="cuda")
        assert float(lb.last_head_norm_grad(q, q, q, q, 64, g, g, lengths=n)[2].abs().sum()) == 0
    q = torch.randn(2, 9, 64, device="cuda").bfloat16()
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    y, lse = lb.last_attention(q, q, q, 64, lengths=n)
    assert not y.any() and not lse.any()
    assert not any(g.any() for g in lb.last_attention_grad(q, q, q, q, y, lse, 64, sinks=2, left=1, lengths=n))


def test_bits_streams_and_replays():
    announce("attention replays")
    case = (3, 700, 4, 2, 64, 50, 20, 10, "bf16", True, 0)
    q, k, v, dy, n, there, band = inputs(case)
    lengths = dev(n)

    def step():
        y, lse = lb.last_attention(q, k, v, 64, lengths=lengths, **band)
        return [y, lse, *lb.last_attention_grad(dy, q, k, v, y, lse, 64, lengths=lengths, **band)]
    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    here = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(other, want)) and all(torch.equal(a, b) for a, b in zip(here, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        for t in got:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        assert all(torch.equal(a, b) for a, b in zip(step(), want)), i


def test_far_rows(much_memory):  # noqa: F811
    """Rows whose offsets pass 2^32 bytes: pitches of 2 MiB."""
    announce("far rows")
    T, D = 2600, 64
    rng = np.random.default_rng(2)
    big = torch.empty(T, 1 << 20, dtype=torch.bfloat16, device="cuda")
    near = [draw(rng, (T, c * D), "bf16") for c in (2, 1, 1, 2)]
    far = []
    for i, t in enumerate(near):
        w = big[:, (i * 4) * D:(i * 4) * D + t.shape[1]]
        w.copy_(t)
        far.append(w)
    for a, b in zip(lb.last_head_norm(*near[:2], D), lb.last_head_norm(*far[:2], D)):
        assert torch.equal(a, b)
    got, want = lb.last_attention(*far[:3], D, left=100, sinks=3), lb.last_attention(*near[:3], D, left=100, sinks=3)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    g, w = (lb.last_attention_grad(x[3], *x[:3], *want, D, left=100, sinks=3) for x in (far, near))
    assert all(torch.equal(a, b) for a, b in zip(g, w))
