"""The gradients that an encoder with an attention block is trained with, through the lattice loss, against a float64 chain: the blocks by automatic
differentiation, the lattice by the oracle.

Bounds, relative to the norm of a gradient.  The blocks' chains round to bfloat16 and keep tensors in int8: 3 % each, as derived where each block is
tested alone.  f itself is off by some 0.6 % of its rms (its rounding and the chain's), so arc weights, sums of 128 products with columns of W of
norm 1, by 0.006; the log-odds of paths that differ in m <= 24 frames by 0.006 sqrt(2 m) <= 0.042, posteriors by as much of themselves at most: 4 %.
Together 10 %.  A gradient with the wrong sign, or without a term, is off by its own size."""
import numpy as np
import pytest
import torch

import oracle
from paper_2304_13134_amd import binding as lb
from paper_2304_13134_amd import frame_attention as fa
from paper_2304_13134_amd import frame_block as fb
from attention_oracle import seen
from gpu_util import announce
from test_gpu_heads import draw

pytestmark = pytest.mark.gpu

B, T, HIDDEN, V, U = 3, 24, 128, 5, 4
LENGTHS, REFS = np.array([24, 17, 20], np.int32), np.array([[1, 3, 2, 5], [4, 4, 1, 2], [2, 5, 3, 1]], np.int32)


def an_encoder(rng, **band):
    model = fa.FrameEncoder(HIDDEN, 160, V, heads=4, kv_heads=2, seed=7, **band)
    for t in (model.gain, model.block.gain, model.attention.gain, model.attention.gain_q, model.attention.gain_k):
        t.copy_(1 + 0.2 * draw(rng, tuple(t.shape), "f32"))
    for t in (model.block.b1, model.block.b2, model.attention.bqkv, model.attention.bo):
        t.copy_(0.2 * draw(rng, tuple(t.shape), "f32"))
    return model


def batch(rng):
    x = draw(rng, (B, T, HIDDEN), "bf16")
    return x, *(torch.from_numpy(a).cuda() for a in (LENGTHS, REFS, np.full(B, U, np.int32)))


def parameters(model):
    p = {"e": model.e, "W": model.W, "last gain": model.gain}
    p.update(("block " + k, v) for k, v in model.block.parameters().items())
    if isinstance(model, fa.FrameEncoder):
        p.update(("attention " + k, v) for k, v in model.attention.parameters().items())
    return p


def norm(x, gain):
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5) * gain


def attention(block, p, x):
    D, R = block.width, 2 * len(block.frequencies)
    q, k, v = (t.reshape(B, T, -1, D) for t in (norm(x, p["attention gain"]) @ p["attention wqkv"].T + p["attention bqkv"]).split(block.split, -1))
    a = torch.arange(T, dtype=torch.float64)[:, None, None] * block.frequencies.double().cpu()

    def turn(t):
        f, g = t[..., :R // 2], t[..., R // 2:R]
        return torch.cat([f * a.cos() - g * a.sin(), g * a.cos() + f * a.sin(), t[..., R:]], -1)
    q, k = turn(norm(q, p["attention gain_q"])), turn(norm(k, p["attention gain_k"]))
    k, v = (t.repeat_interleave(block.heads // block.kv_heads, 2) for t in (k, v))
    m = torch.from_numpy(np.stack([seen(np.arange(T), n, T, *block.band.values()) for n in LENGTHS]))[:, None]
    S = (q.transpose(1, 2) @ k.permute(0, 2, 3, 1) * D ** -0.5).masked_fill(~m, -1e300)
    y = (torch.softmax(S, -1) @ v.transpose(1, 2)).transpose(1, 2).reshape(B, T, -1)
    return x + y @ p["attention wo"].T + p["attention bo"]


def bits(t):
    return t.to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


def float64_chain(model, x):
    """(loss [B], gradients by name, that of x among them)"""
    p = {k: v.detach().double().cpu().requires_grad_() for k, v in parameters(model).items()}
    p["x"] = x.double().cpu().requires_grad_()
    z = attention(model.attention, p, p["x"]) if isinstance(model, fa.FrameEncoder) else p["x"]
    h = norm(z, p["block gain"]) @ p["block w1"].T + p["block b1"]
    y = z + torch.nn.functional.silu(h) @ p["block w2"].T + p["block b2"]
    f = norm(y, p["last gain"])
    args = bits(f.detach()), bits(p["e"].detach()), bits(p["W"].detach()), LENGTHS
    d = oracle.fused_forward_backward(*args, order=2)
    n = oracle.fused_numerator(*args, REFS, np.full(B, U, np.int32), order=2)
    f.backward(torch.from_numpy(d["df"] - n["df"]))
    grads = {k: v.grad for k, v in p.items() if v.grad is not None}
    grads["e"], grads["W"] = torch.from_numpy(d["de"] - n["de"]), torch.from_numpy(d["dW"] - n["dW"])
    return d["D"] - n["N"], grads


def compare(got, want, names):
    assert set(got) == set(names)
    for k in names:
        g, w = got[k].double().cpu(), want[k]
        assert g.shape == w.shape and bool(torch.isfinite(g).all()) and float(w.norm()) > 0, k
        off = float((g - w).norm() / w.norm())
        print("  %-18s %.4f" % (k, off), flush=True)
        assert off < 0.1, (k, off)


@pytest.mark.parametrize("band", [{"left": 6, "right": 2, "sinks": 2}, {"left": None, "right": None, "sinks": 0}], ids=str)
def test_encoder_gradients_through_the_lattice(band):
    announce("encoder gradients", band)
    rng = np.random.default_rng(31)
    model = an_encoder(rng, **band)
    arguments = batch(rng)
    loss, gradients = model.loss_and_gradients(*arguments)
    lb.check_item_status()
    want_loss, want = float64_chain(model, arguments[0])
    names = parameters(model)
    by_tensor = {id(v): k for k, v in names.items()}
    assert len(gradients) == len(names)
    compare({by_tensor[id(t)]: g for t, g in gradients}, want, names)
    # (sums of 24 weights that are off by 0.006 each, twice)
    assert np.abs(loss.double().cpu().numpy() - want_loss).max() < 2 * 24 * 0.006


def test_model_without_attention():
    """The same of the model that the encoder builds on, with the gradient of its frames; and its loss and gradients, to the bit, are those of the calls that it
    is made of."""
    announce("model gradients")
    rng = np.random.default_rng(32)
    model = an_encoder(rng)
    plain = fb.FrameModel(HIDDEN, 160, V)
    plain.block, plain.gain, plain.e, plain.W = model.block, model.gain, model.e, model.W
    x, lengths, refs, ref_lengths = batch(rng)
    loss, gradients, dx = plain.loss_of_frames(x, lengths, refs, ref_lengths)
    lb.check_item_status()
    _, want = float64_chain(plain, x)
    names = dict(parameters(plain), x=x)
    by_tensor = {id(v): k for k, v in names.items()}
    compare(dict({by_tensor[id(t)]: g for t, g in gradients}, x=dx), want, names)
    assert not dx[torch.arange(T, device="cuda") >= lengths[:, None]].any()
    y, saved = plain.block.forward(x, lengths)
    f = lb.last_residual_norm(y, plain.gain, lengths=lengths)
    dist, num, (df, de, dW) = lb.last_globally_normalized_loss(lb.SharedEmb(f.y, plain.e, plain.W), lengths, refs, ref_lengths, order=2)
    dy, dgain = lb.last_residual_norm_grad(df, y, plain.gain, f.inv, lengths=lengths)
    dz, grads = plain.block.backward(dy, saved, lengths)
    again = dict({"e": de, "W": dW, "last gain": dgain, "x": dz}, **{"block " + k: v for k, v in grads.items()})
    two = plain.loss_and_gradients(x, lengths, refs, ref_lengths)
    assert torch.equal(loss, dist - num) and torch.equal(two[0], loss) and len(two) == 2
    for t, g in list(gradients) + list(two[1]) + [(x, dx)]:
        assert torch.equal(again[by_tensor[id(t)]], g), by_tensor[id(t)]
