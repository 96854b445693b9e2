"""The calls in which frames see each other together: an attention block that is trained through the lattice and streamed."""
import numpy as np
import pytest
import torch

from paper_2304_13134_amd import binding as lb
from paper_2304_13134_amd import frame_attention as fa
from attention_oracle import frames_there, rotate, seen, split
from layer_oracle import f64
from gpu_util import announce
from test_gpu_heads import dev, draw

pytestmark = pytest.mark.gpu


def plain_block(block, p, lengths):
    """The block in float64; p: parameters and x by name."""
    x, D = p["x"], block.width
    B, T, _ = x.shape
    n, there = frames_there(B, T, lengths)
    norm = x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-5) * p["gain"]
    qkv = norm @ p["wqkv"].T + p["bqkv"]
    q, k, v = (split(t, D) for t in np.split(qkv, np.cumsum(block.split)[:2], -1))
    at = np.broadcast_to(np.arange(T), (B, T))
    f = f64(block.frequencies)

    def heads(t, gain):
        return rotate(t / np.sqrt((t * t).mean(-1, keepdims=True) + 1e-5) * gain, at, f)
    q, k = heads(q, p["gain_q"]), heads(k, p["gain_k"])
    a = np.zeros_like(q)
    for b in range(B):
        m = seen(np.arange(n[b]), n[b], n[b], *block.band.values())
        for h in range(block.heads):
            g = h * block.kv_heads // block.heads
            S = np.where(m, q[b, :n[b], h] @ k[b, :n[b], g].T * D ** -0.5, -np.inf)
            e = np.exp(S - S.max(-1, keepdims=True))
            a[b, :n[b], h] = e / e.sum(-1, keepdims=True) @ v[b, :n[b], g]
    return np.where(there[..., None], x + a.reshape(B, T, -1) @ p["wo"].T + p["bo"], 0.0)


def a_block(rng, **more):
    block = fa.FrameAttention(64, 4, 2, seed=5, **more)
    for t in (block.gain, block.gain_q, block.gain_k):
        t.copy_(1 + 0.2 * draw(rng, tuple(t.shape), "f32"))
    for t in (block.bqkv, block.bo):
        t.copy_(0.2 * draw(rng, tuple(t.shape), "f32"))
    return block


@pytest.mark.parametrize("band", [{}, {"left": 6, "right": 3, "sinks": 2}], ids=str)
def test_block_gradient_against_differences(band):
    """The block's gradients along random directions against differences of its float64 form.  The chain rounds the norm, the projection, queries and
    keys, probabilities, the attention's result and their gradients to bfloat16 (0.2 % of the rms each) and keeps one tensor in int8 (0.9 % at
    most): errors that are independent over 10^3 and more terms; 3 % of the norm of a gradient covers them, and a direction sees at most
    that."""
    announce("attention block gradient", band)
    rng = np.random.default_rng(21)
    block = a_block(rng, **band)
    B, T, H = 2, 40, 64
    x, c = draw(rng, (B, T, H), "bf16"), draw(rng, (B, T, H), "bf16")
    n = np.array([40, 23])
    _, there = frames_there(B, T, n)
    y, saved = block.forward(x, dev(n))
    dx, grads = block.backward(c, saved, dev(n))
    p = {k: f64(v) for k, v in block.parameters().items()}
    p["x"] = f64(x)
    want = plain_block(block, p, n)
    assert np.linalg.norm(f64(y) - want) < 0.01 * np.linalg.norm(want)

    def loss(p):
        return float((plain_block(block, p, n) * np.where(there[..., None], f64(c), 0)).sum())
    for k, g in dict(grads, x=dx).items():
        g = f64(g)
        for _ in range(2):
            d = rng.standard_normal(g.shape)
            d *= np.linalg.norm(g) / np.linalg.norm(d)
            d += g                                                  # half along the gradient, so that there is something to see
            e = 1e-5 / np.abs(d).max()
            num = (loss(dict(p, **{k: p[k] + e * d})) - loss(dict(p, **{k: p[k] - e * d}))) / (2 * e)
            assert abs(num - float((g * d).sum())) < 0.03 * np.linalg.norm(g) * np.linalg.norm(d), (k, num, float((g * d).sum()))


def test_streams_are_the_block():
    """Streams of unequal length, given chunks of unequal size and none at times, come out as the block on whole utterances."""
    announce("streaming a block")
    rng = np.random.default_rng(22)
    block = a_block(rng, left=9, sinks=3)
    B, T = 3, 50
    x = draw(rng, (B, T, 64), "bf16")
    want, _ = block.forward(x)
    page, entries = 7, 8
    table = rng.permutation(B * entries).reshape(B, entries)
    cache = lb.Cache(*block.pages(B * entries, page), dev(table), torch.zeros(B, dtype=torch.int32, device="cuda"))
    done = np.zeros(B, int)
    while (done < T).any():
        new = np.minimum(rng.integers(0, 9, B), T - done)
        size = max(1, new.max())
        chunk = torch.full((B, size, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
        for b in range(B):
            chunk[b, :new[b]] = x[b, done[b]:done[b] + new[b]]
        y = block.stream(chunk, cache, dev(new))
        lb.check_item_status()
        for b in range(B):
            # both round probabilities and results to bfloat16, in other orders: 2^-8 of the attention's part each, with the residual's rounding
            a, w = y[b, :new[b]].float(), want[b, done[b]:done[b] + new[b]].float()
            assert float((a - w).norm()) <= 0.01 * float(w.norm()) + 1e-6
            assert not y[b, new[b]:].any()
        cache.used.add_(dev(new))
        done += new


def test_encoder_trains_through_the_lattice():
    """A step's loss is finite and its gradients are, captured replays of it give the eager step's bits, and the model without attention is as it was."""
    announce("training an encoder through the lattice")
    model = fa.FrameEncoder()
    batch = fa.synthetic_batch()
    first = model.step(*batch)
    last = [model.step(*batch) for _ in range(3)][-1]
    assert np.isfinite(first) and np.isfinite(last)

    def grads():
        x, lengths = batch[:2]
        z, saved = model.attention.forward(x, lengths)
        dx, g = model.attention.backward(z, saved, lengths)
        return [z, dx, *g.values()]
    want = [t.clone() for t in grads()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = grads()
    for i in range(4):
        for t in got:
            t.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        assert all(torch.equal(a, b) for a, b in zip(grads(), want)), i
    plain = fa.FrameModel()
    loss, gradients = plain.loss_and_gradients(*batch)
    again = fa.FrameModel().loss_and_gradients(*batch)
    assert torch.equal(loss, again[0]) and len(gradients) == len(again[1])
